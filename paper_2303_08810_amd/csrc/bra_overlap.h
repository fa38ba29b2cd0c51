// Whether strided arrays share memory (host, internal).
#pragma once

#include <algorithm>
#include <cstdint>

namespace bra {

// Pieces of `bytes` bytes at p + sum of i_k stride[k] with 0 <= i_k < count[k]; none where a count is 0 or p is NULL.
struct Pieces {
    const char *p = nullptr;
    long bytes = 0;
    long count[3] = {1, 1, 1}, stride[3] = {0, 0, 0};
    bool any() const { return p && bytes > 0 && count[0] > 0 && count[1] > 0 && count[2] > 0; }
    long last() const { return stride[0] * (count[0] - 1) + stride[1] * (count[1] - 1) + stride[2] * (count[2] - 1); }
};

// Looks for numbers 0 <= x_k < n_k with |delta + sum of s_k x_k| < bytes, s_k > 0 from the largest to the smallest.  In layouts whose dimensions lie within each other a
// number has a few candidates; where dimensions run through each other they may be many, and after kSteps of them the answer is that there may be some.
class Meeting {
public:
    explicit Meeting(long bytes) : bytes_(bytes) {}
    void add(long stride, long n)
    {
        if (n <= 1 || stride == 0) return;
        for (int k = 0; k < count_; ++k)
            if (dims_[k].stride == stride) {        // the sum of both numbers
                dims_[k].n += n - 1;
                return;
            }
        dims_[count_++] = Dim{stride, n};
    }
    // `but`: whether x_k = (n_k - 1) / 2 for all k, with which an array meets itself, does not count
    bool find(long delta, bool but)
    {
        std::sort(dims_, dims_ + count_, [](const Dim &a, const Dim &b) { return a.stride > b.stride; });
        rest_[count_] = 0;
        for (int k = count_; k--;) rest_[k] = rest_[k + 1] + dims_[k].stride * (dims_[k].n - 1);
        return look(delta, 0, but);
    }

private:
    static constexpr int kSteps = 4096;
    struct Dim {
        long stride, n;
    };
    bool look(long delta, int k, bool but)
    {
        if (++steps_ > kSteps) return true;
        if (k == count_) return !but && delta > -bytes_ && delta < bytes_;
        const Dim &d = dims_[k];
        // delta + s x + (0 .. rest) comes within (-bytes, bytes)
        const long low = -bytes_ - delta - rest_[k + 1], high = bytes_ - delta;         // low < s x < high
        if (high <= 0) return false;
        const long first = low < 0 ? 0 : low / d.stride + 1, last = std::min((high - 1) / d.stride, d.n - 1);
        for (long x = first; x <= last; ++x)
            if (look(delta + d.stride * x, k + 1, but && 2 * x == d.n - 1)) return true;
        return false;
    }
    long bytes_, rest_[7] = {};
    Dim dims_[6];
    int count_ = 0, steps_ = 0;
};

// Whether two arrays of pieces of one size share a byte.
inline bool share_memory(const Pieces &a, const Pieces &b)
{
    if (!a.any() || !b.any()) return false;
    const uintptr_t at = (uintptr_t)a.p, bt = (uintptr_t)b.p;
    if (at + a.last() + a.bytes <= bt || bt + b.last() + b.bytes <= at) return false;
    // a's place less b's: b's numbers are counted from the other end.  (Sizes apart, pieces within (-b.bytes, a.bytes) of each other meet; moved to the middle.)
    long delta = (long)(at - bt) - b.last();
    const long bytes = a.bytes + b.bytes;
    Meeting m(bytes);
    for (int k = 0; k < 3; ++k) {
        m.add(2 * a.stride[k], a.count[k]);
        m.add(2 * b.stride[k], b.count[k]);
    }
    return m.find(2 * delta + (a.bytes - b.bytes), false);
}

// Whether two pieces of an array share a byte.
inline bool meets_itself(const Pieces &a)
{
    if (!a.any()) return false;
    long inner = a.bytes;           // what the dimensions so far take
    bool nested = true;
    for (int k = 3; k--;)
        if (a.count[k] > 1) {
            nested = nested && a.stride[k] >= inner;
            inner += a.stride[k] * (a.count[k] - 1);
        }
    if (nested) return false;
    Meeting m(a.bytes);
    for (int k = 0; k < 3; ++k) {
        if (a.count[k] <= 1) continue;
        if (a.stride[k] == 0) return true;
        for (int j = 0; j < k; ++j)
            if (a.count[j] > 1 && a.stride[j] == a.stride[k]) return true;
        m.add(a.stride[k], 2 * a.count[k] - 1);
    }
    return m.find(-a.last(), true);
}

// Whether they are the same pieces in the same order.
inline bool same_place(const Pieces &a, const Pieces &b)
{
    if (a.p != b.p || a.bytes != b.bytes) return false;
    for (int k = 0; k < 3; ++k)
        if (a.count[k] != b.count[k] || (a.count[k] > 1 && a.stride[k] != b.stride[k])) return false;
    return true;
}

}  // namespace bra
