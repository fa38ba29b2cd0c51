// bra_overlap.h against brute force: small layouts, nested and not, whose answers have to be the same; large ones of the kinds that programs have, whose answers are known.
#include <cstdio>
#include <random>
#include <vector>

#include "../../paper_2303_08810_amd/csrc/bra_overlap.h"

using namespace bra;

static char *const kBase = (char *)(1l << 40);

static void touch(const Pieces &a, std::vector<int> &seen, int &most)
{
    for (long i = 0; i < a.count[0]; ++i)
        for (long j = 0; j < a.count[1]; ++j)
            for (long k = 0; k < a.count[2]; ++k)
                for (long c = 0; c < a.bytes; ++c) most = std::max(most, ++seen[(a.p - kBase) + i * a.stride[0] + j * a.stride[1] + k * a.stride[2] + c]);
}

int main()
{
    int wrong = 0, hits = 0, selves = 0;
    std::mt19937 rng(5);
    auto pick = [&](int lo, int hi) { return (long)(lo + rng() % (hi - lo + 1)); };
    for (int n = 0; n < 8000; ++n) {
        auto make = [&] {
            Pieces a;
            a.p = kBase + 16 * pick(0, 60);
            a.bytes = 16 * pick(1, 4);
            const bool nested = pick(0, 2) > 0;
            long step = a.bytes;
            for (int k = 3; k--;) {
                a.count[k] = pick(1, 4);
                a.stride[k] = nested ? step + 16 * pick(0, 3) * pick(0, 1) : 16 * pick(0, 14);
                if (nested) step = a.stride[k] * (pick(0, 2) ? a.count[k] : pick(1, 5));
            }
            if (pick(0, 3) == 0) std::swap(a.stride[0], a.stride[2]);
            if (pick(0, 30) == 0) a.count[pick(0, 2)] = 0;
            return a;
        };
        const Pieces a = make(), b = make();
        std::vector<int> of_a(1 << 16), both;
        int self = 0, with = 0;
        if (a.any()) touch(a, of_a, self);
        both = of_a;
        for (int &v : both) v = v > 0;
        bool meet = false;
        if (a.any() && b.any()) {
            std::vector<int> of_b(1 << 16);
            touch(b, of_b, with);
            for (size_t i = 0; i < of_b.size(); ++i) meet = meet || (both[i] && of_b[i]);
        }
        if (share_memory(a, b) != meet || share_memory(b, a) != meet || meets_itself(a) != (self > 1)) ++wrong;
        hits += meet;
        selves += self > 1;
    }
    // parts of a packed buffer [B, N, heads, d], shifted by whole heads and by one piece of 16 bytes, and a cache with the heads outside
    const long B = 64, N = 8192, H = 48, row = 256, token = H * row;
    auto part = [&](long first, long heads, long shift = 0) { return Pieces{kBase + first * row + shift, row, {B, N, heads}, {N * token, token, row}}; };
    for (long h = 1; h < H; ++h) {
        wrong += share_memory(part(0, h), part(h, H - h)) != false;
        wrong += share_memory(part(0, h), part(h - 1, H - h)) != true;
        wrong += share_memory(part(0, h), part(h, H - h, -16)) != true;
        wrong += meets_itself(part(0, h)) != false;
    }
    const Pieces even{kBase, row, {B, N, H / 2}, {N * token, token, 2 * row}}, odd{kBase + row, row, {B, N, H / 2}, {N * token, token, 2 * row}};
    wrong += share_memory(even, odd) != false;
    wrong += share_memory(even, part(1, 2)) != true;
    const Pieces cache{kBase, row, {B, N, H}, {N * token, row, N * row}}, half{kBase + N / 2 * row, row, {B, N / 2, H}, {N * token, row, N * row}}, first{kBase, row, {B, N / 2, H}, {N * token, row, N * row}};
    wrong += share_memory(first, half) != false;
    wrong += share_memory(cache, half) != true;
    wrong += share_memory(cache, part(3, 5)) != true;
    wrong += meets_itself(Pieces{kBase, row, {B, N, H}, {N * token, token, row - 16}}) != true;
    wrong += meets_itself(Pieces{kBase, row, {B, N, H}, {(N - 1) * token, token, row}}) != true;
    wrong += meets_itself(cache) != false;
    std::printf("%d wrong, %d of 8000 share memory, %d with themselves\n", wrong, hits, selves);
    return wrong || hits < 800 || selves < 800;
}
