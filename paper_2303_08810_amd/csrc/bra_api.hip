// C-ABI entry points of libbra: argument checks and dispatch to a kernel family.
#include "bra_common.h"
#include "bra_adamw.h"
#include "bra_ffn.h"
#include "bra_norm.h"
#include "bra_attention.h"
#include "bra_overlap.h"
#include "bra_qk_norm.h"

#include <math.h>

#include <algorithm>
#include <cmath>
#include <initializer_list>
#include <mutex>
#include <utility>
#include <vector>

// Scratch memory of bra_forward_static: one copy per GPU, held by the code object until the
// process ends.  In host code the array's name is only a handle for hipGetSymbolAddress; the
// address that kernels, copies and fills take is the one that call returns for the current device.
static __device__ __align__(256) unsigned char scratch[BRA_STATIC_SCRATCH_BYTES];

namespace bra {

// Device address of `scratch` on the current device, looked up once per device.
static int static_scratch(void **out)
{
    constexpr int kMaxDevices = 64;
    static std::mutex mu;
    static void *ptrs[kMaxDevices] = {};
    int dev = -1;
    if (hipGetDevice(&dev) != hipSuccess || dev < 0 || dev >= kMaxDevices) return BRA_ERR_LAUNCH;
    std::lock_guard<std::mutex> lock(mu);
    if (!ptrs[dev]) {
        void *p = nullptr;
        if (hipGetSymbolAddress(&p, HIP_SYMBOL(scratch)) != hipSuccess || !p) return BRA_ERR_LAUNCH;
        if ((uintptr_t)p % 256 != 0) return BRA_ERR_LAUNCH;
        ptrs[dev] = p;
    }
    *out = ptrs[dev];
    return BRA_OK;
}

// Validates `s` and fills D.  Returns a BRA_* code.
static int make_dims(const bra_shape *s, Dims &D)
{
    if (!s) return BRA_ERR_NULL;
    if (s->B < 1 || s->H < 1 || s->W < 1 || s->C < 1 || s->heads < 1 || s->S < 1) return BRA_ERR_SHAPE;
    if (s->H % s->S || s->W % s->S || s->C % s->heads) return BRA_ERR_SHAPE;
    if ((long)s->S * s->S > (1L << 20)) return BRA_ERR_SHAPE;
    if (s->k < 1 || s->k > s->S * s->S) return BRA_ERR_K;
    if (s->dtype != BRA_F32 && s->dtype != BRA_BF16) return BRA_ERR_DTYPE;
    if (s->path != BRA_PATH_AUTO && s->path != BRA_PATH_GENERIC && s->path != BRA_PATH_MFMA)
        return BRA_ERR_DTYPE;
    // element counts must stay addressable with the 31-bit token indices the kernels use
    if ((long)s->H * s->W > (1L << 30) || (long)s->B * s->H * s->W > (1L << 30)) return BRA_ERR_SHAPE;
    D.B = s->B; D.H = s->H; D.W = s->W; D.C = s->C; D.heads = s->heads; D.S = s->S; D.k = s->k;
    D.dtype = s->dtype;
    D.rh = s->H / s->S; D.rw = s->W / s->S; D.n = D.rh * D.rw; D.R = s->S * s->S;
    D.N = s->H * s->W; D.d = s->C / s->heads; D.kn = D.k * D.n;
    D.scale = (s->scale > 0.f) ? s->scale : 1.0f / sqrtf((float)D.d);
    return BRA_OK;
}

// Picks the kernel family: returns BRA_PATH_GENERIC / BRA_PATH_MFMA or an error.
static int pick_path(const bra_shape *s, const Dims &D)
{
    const bool mfma_ok = mfma_supported(D);
    if (s->path == BRA_PATH_MFMA) return mfma_ok ? BRA_PATH_MFMA : BRA_ERR_UNSUPPORTED;
    if (s->path == BRA_PATH_AUTO && mfma_ok) return BRA_PATH_MFMA;
    return generic_supported(D) ? BRA_PATH_GENERIC : BRA_ERR_UNSUPPORTED;
}

// The shape with H and W rounded up to multiples of S (the map after zero padding).
static int make_padded_dims(const bra_shape *s, Dims &Dp)
{
    if (!s) return BRA_ERR_NULL;
    if (s->H < 1 || s->W < 1 || s->S < 1 || s->S > 1024) return BRA_ERR_SHAPE;
    if (s->H > (1 << 24) || s->W > (1 << 24)) return BRA_ERR_SHAPE;
    bra_shape p = *s;
    p.H = (s->H + s->S - 1) / s->S * s->S;
    p.W = (s->W + s->S - 1) / s->S * s->S;
    return make_dims(&p, Dp);
}

static int make_ffn_sizes(const bra_ffn_shape *s, ffn::Sizes &S)
{
    if (!s) return BRA_ERR_NULL;
    if (s->M < 0 || s->M > (1L << 30) || s->C < 1 || s->hidden < 1 || s->C > (1 << 20) || s->hidden > (1 << 20)) return BRA_ERR_SHAPE;
    if (s->dtype != BRA_F32 && s->dtype != BRA_BF16) return BRA_ERR_DTYPE;
    if (s->act != BRA_SILU && s->act != BRA_GELU) return BRA_ERR_DTYPE;
    S.M = s->M; S.C = s->C; S.h = s->hidden; S.act = s->act;
    S.f32 = s->dtype == BRA_F32;
    S.Cp = (S.C + 7) / 8 * 8; S.hp = (S.h + 7) / 8 * 8;
    return BRA_OK;
}

// Whether every pointer that is not NULL is a multiple of `bytes`.
static bool aligned(size_t bytes, std::initializer_list<const void *> pointers)
{
    for (const void *p : pointers)
        if ((uintptr_t)p % bytes != 0) return false;
    return true;
}

// Alignment of the block's matrices, rows of C or of hidden elements of `element` bytes: whole 16-byte pieces where the rows are.
static size_t row_alignment(int columns, size_t element) { return columns % 8 == 0 ? 16 : element; }

static int make_norm_sizes(const bra_norm_shape *s, bool post, NormSizes &S)
{
    if (!s) return BRA_ERR_NULL;
    if (s->rows < 0 || s->rows > (1L << 30) || s->C < 1 || s->groups < 1 || s->rows % s->groups || !(s->eps >= 0.f)) return BRA_ERR_SHAPE;
    if (s->dtype != BRA_F32 && s->dtype != BRA_BF16) return BRA_ERR_DTYPE;
    if (s->kind != BRA_LAYERNORM && s->kind != BRA_RMSNORM) return BRA_ERR_DTYPE;
    if (s->C > 8192) return BRA_ERR_UNSUPPORTED;
    S.rows = s->rows; S.groups = s->groups; S.per_group = s->rows / s->groups; S.C = s->C;
    S.f32 = s->dtype == BRA_F32; S.layer = s->kind == BRA_LAYERNORM; S.post = post; S.eps = s->eps;
    S.vec = S.C % 8 == 0;
    return BRA_OK;
}

static bool ws_ok(const void *ws, size_t have, size_t need)
{
    return ws && ((uintptr_t)ws % 256 == 0) && have >= need;
}

// Attention's sizes; what depends on the tensors comes later.
static int make_attention_sizes(const bra_attention_shape *s, att::Sizes &S)
{
    if (!s) return BRA_ERR_NULL;
    constexpr int kMost = 1 << 28;
    if (s->B < 0 || s->Nq < 0 || s->Nk < 0 || s->B > kMost || s->Nq > kMost || s->Nk > kMost || s->kv_heads < 1 || s->heads < s->kv_heads || s->heads % s->kv_heads || s->heads > 65536 ||
        s->d < 1 || !std::isfinite(s->scale) || s->scale > 1e38f)
        return BRA_ERR_SHAPE;
    if ((long)s->B * s->heads > (1L << 30) || (long)s->Nq * s->heads > (1L << 30)) return BRA_ERR_SHAPE;
    if ((long)s->B * s->heads > (1L << 40) / std::max({s->Nq, s->Nk, 1})) return BRA_ERR_SHAPE;
    if (s->dtype != BRA_F32 && s->dtype != BRA_BF16) return BRA_ERR_DTYPE;
    if (s->d % 8 || s->d > 128) return BRA_ERR_UNSUPPORTED;
    S = att::Sizes{s->B, s->Nq, s->Nk, s->heads, s->kv_heads, s->d, s->dtype == BRA_F32, s->causal != 0, s->scale > 0.f ? s->scale : 1.0f / sqrtf((float)s->d), nullptr, nullptr};
    return BRA_OK;
}

// A [B, N, heads, d] tensor's place, strides in bytes; a tensor without elements may have no memory.
static int make_rows(const bra_rows *r, long B, long N, long heads, size_t element, att::Rows &R)
{
    R = att::Rows{};
    if (B == 0 || N == 0 || heads == 0) return BRA_OK;
    if (!r || !r->data) return BRA_ERR_NULL;
    const long e = (long)element;
    // (what lies further away than 2^56 bytes is no tensor)
    constexpr long far = 1L << 56;
    if ((B > 1 && r->batch > far / e / (B - 1)) || (N > 1 && r->token > far / e / (N - 1)) || (heads > 1 && r->head > far / e / (heads - 1))) return BRA_ERR_SHAPE;
    if ((B > 1 && r->batch < 0) || (N > 1 && r->token < 0) || (heads > 1 && r->head < 0)) return BRA_ERR_SHAPE;
    R = att::Rows{(char *)r->data, B > 1 ? r->batch * e : 0, N > 1 ? r->token * e : 0, heads > 1 ? r->head * e : 0};
    if ((uintptr_t)R.p % 16 || R.batch % 16 || R.token % 16 || R.head % 16) return BRA_ERR_ALIGN;
    return BRA_OK;
}

// Where a call's tensors lie.  What is written may be what it is given as (`same`, at the same places), and meets nothing else of the call.
static Pieces pieces_of(const att::Rows &R, long B, long N, long heads, long bytes) { return Pieces{R.p, bytes, {B, N, heads}, {R.batch, R.token, R.head}}; }
static Pieces pieces_of(const void *p, size_t bytes) { return Pieces{(const char *)p, (long)bytes, {1, 1, 1}, {0, 0, 0}}; }
struct Written {
    Pieces at;
    const Pieces *same[2];
};
static bool meet(std::initializer_list<Written> written, std::initializer_list<const Pieces *> read)
{
    for (const Written &w : written) {
        if (!w.at.any()) continue;
        if (meets_itself(w.at)) return true;
        const uintptr_t from = (uintptr_t)w.at.p, to = from + w.at.last() + w.at.bytes;
        for (const Written *o = written.begin(); o != &w; ++o)
            if (share_memory(w.at, o->at)) return true;
        for (const Pieces *r : read) {
            if ((uintptr_t)r->p >= to || (uintptr_t)r->p + r->last() + r->bytes <= from) continue;      // (nearly always)
            const bool allowed = r == w.same[0] || r == w.same[1];
            if (!(allowed && same_place(w.at, *r)) && share_memory(w.at, *r)) return true;
        }
    }
    return false;
}

static int make_qk_norm_sizes(const bra_qk_norm_shape *s, QkNormSizes &S)
{
    if (!s) return BRA_ERR_NULL;
    if (s->B < 0 || s->N < 0 || s->heads < 1 || s->kv_heads < 0 || s->d < 1 || s->turned < 0 || s->turned > s->d || s->turned % 2 || !(s->eps >= 0.f)) return BRA_ERR_SHAPE;
    const long most = 1L << 30, tokens = (long)s->B * s->N, heads = (long)s->heads + s->kv_heads;
    if (tokens > most || heads > most || tokens * heads > most) return BRA_ERR_SHAPE;
    if (s->dtype != BRA_F32 && s->dtype != BRA_BF16) return BRA_ERR_DTYPE;
    if (s->pairs != BRA_PAIRS_HALVES && s->pairs != BRA_PAIRS_NEIGHBOURS) return BRA_ERR_DTYPE;
    if (s->d % 8 || s->d > 128) return BRA_ERR_UNSUPPORTED;
    S = QkNormSizes{tokens, s->N, s->heads, s->kv_heads, s->d, s->turned, s->table_rows, s->dtype == BRA_F32, s->pairs == BRA_PAIRS_HALVES, s->eps};
    return BRA_OK;
}

// The vectors of norms and rotation.
static int qk_norm_in(const bra_qk_norm_shape *s, const QkNormSizes &S, const bra_qk_norm_params *p, QkNormIn &I)
{
    if (!p) return BRA_ERR_NULL;
    if ((S.turned && (!p->cos || !p->sin)) || (p->k_gamma && !p->q_gamma) || (S.kv_heads && p->q_gamma && !p->k_gamma)) return BRA_ERR_NULL;
    if (S.turned && (s->table_rows < 1 || (!p->positions && s->table_rows < s->N))) return BRA_ERR_SHAPE;
    if (!aligned(4, {p->q_gamma, p->k_gamma, p->cos, p->sin, p->positions})) return BRA_ERR_ALIGN;
    I.q_gamma = p->q_gamma;
    I.k_gamma = p->k_gamma;
    I.cos = p->cos;
    I.sin = p->sin;
    I.positions = p->positions;
    return BRA_OK;
}

}  // namespace bra

using namespace bra;

extern "C" {

int bra_workspace_bytes(const bra_shape *shape, size_t *out_bytes)
{
    if (!out_bytes) return BRA_ERR_NULL;
    Dims D;
    int rc = make_dims(shape, D);
    if (rc != BRA_OK) return rc;
    int path = pick_path(shape, D);
    if (path < 0) return path;
    *out_bytes = (path == BRA_PATH_MFMA) ? mfma_workspace_bytes(D) : generic_workspace_bytes(D);
    return BRA_OK;
}

int bra_route(const bra_shape *shape, const void *X, const void *Wqkv, int32_t *Ir, float *Ar_opt,
              void *ws, size_t ws_bytes, void *hip_stream)
{
    Dims D;
    int rc = make_dims(shape, D);
    if (rc != BRA_OK) return rc;
    if (!X || !Wqkv || !Ir) return BRA_ERR_NULL;
    int path = pick_path(shape, D);
    if (path < 0) return path;
    size_t need = (path == BRA_PATH_MFMA) ? mfma_workspace_bytes(D) : generic_workspace_bytes(D);
    if (!ws_ok(ws, ws_bytes, need)) return BRA_ERR_WORKSPACE;
    hipStream_t st = (hipStream_t)hip_stream;
    if (path == BRA_PATH_MFMA) return mfma_route(D, X, Wqkv, Ir, Ar_opt, ws, st);
    return generic_route(D, X, Wqkv, Ir, Ar_opt, ws, st);
}

int bra_forward(const bra_shape *shape, const void *X, const void *Wqkv, const void *Wo,
                const void *Wlce, void *Y, int32_t *Ir_out_opt, const int32_t *Ir_in_opt, void *ws,
                size_t ws_bytes, void *hip_stream)
{
    Dims D;
    int rc = make_dims(shape, D);
    if (rc != BRA_OK) return rc;
    if (!X || !Wqkv || !Wo || !Wlce || !Y) return BRA_ERR_NULL;
    int path = pick_path(shape, D);
    if (path < 0) return path;
    size_t need = (path == BRA_PATH_MFMA) ? mfma_workspace_bytes(D) : generic_workspace_bytes(D);
    if (!ws_ok(ws, ws_bytes, need)) return BRA_ERR_WORKSPACE;
    hipStream_t st = (hipStream_t)hip_stream;
    if (path == BRA_PATH_MFMA)
        return mfma_forward(D, X, Wqkv, Wo, Wlce, Y, Ir_out_opt, Ir_in_opt, ws, st);
    return generic_forward(D, X, Wqkv, Wo, Wlce, Y, Ir_out_opt, Ir_in_opt, ws, st);
}

int bra_forward_static(const bra_shape *shape, const void *X, const void *Wqkv, const void *Wo,
                       const void *Wlce, void *Y, int32_t *Ir_out_opt, const int32_t *Ir_in_opt,
                       void *hip_stream)
{
    Dims D;
    int rc = make_dims(shape, D);
    if (rc != BRA_OK) return rc;
    if (!X || !Wqkv || !Wo || !Wlce || !Y) return BRA_ERR_NULL;
    int path = pick_path(shape, D);
    if (path < 0) return path;
    size_t need = (path == BRA_PATH_MFMA) ? mfma_forward_bytes(D, Ir_in_opt) : generic_workspace_bytes(D);
    const bool compact = path == BRA_PATH_MFMA && need > (size_t)BRA_STATIC_SCRATCH_BYTES;
    if (compact) need = mfma_compact_bytes(D, Ir_in_opt);
    if (need > (size_t)BRA_STATIC_SCRATCH_BYTES) return BRA_ERR_TOO_LARGE;
    void *ws = nullptr;
    rc = static_scratch(&ws);
    if (rc != BRA_OK) return rc;
    hipStream_t st = (hipStream_t)hip_stream;
    // no kernel of the forward pass expects zeroed scratch (no counters, no accumulation into it):
    // every buffer carved from it is written before it is read within the call
    if (path == BRA_PATH_MFMA)
        return mfma_forward(D, X, Wqkv, Wo, Wlce, Y, Ir_out_opt, Ir_in_opt, ws, st, compact);
    return generic_forward(D, X, Wqkv, Wo, Wlce, Y, Ir_out_opt, Ir_in_opt, ws, st);
}

int bra_padded_workspace_bytes(const bra_shape *shape, size_t *out_bytes)
{
    if (!out_bytes) return BRA_ERR_NULL;
    Dims Dp;
    int rc = make_padded_dims(shape, Dp);
    if (rc != BRA_OK) return rc;
    bra_shape ps = *shape;
    ps.H = Dp.H; ps.W = Dp.W;
    int path = pick_path(&ps, Dp);
    if (path < 0) return path;
    if (Dp.H == shape->H && Dp.W == shape->W) return bra_workspace_bytes(&ps, out_bytes);
    const size_t inner = (path == BRA_PATH_MFMA) ? mfma_padded_workspace_bytes(Dp) : generic_workspace_bytes(Dp);
    *out_bytes = padded_workspace_bytes(Dp, inner);
    return BRA_OK;
}

int bra_forward_padded(const bra_shape *shape, const void *X, const void *Wqkv, const void *Wo, const void *Wlce,
                       void *Y, int32_t *Ir_out_opt, const int32_t *Ir_in_opt, void *ws, size_t ws_bytes,
                       void *hip_stream)
{
    Dims Dp;
    int rc = make_padded_dims(shape, Dp);
    if (rc != BRA_OK) return rc;
    if (!X || !Wqkv || !Wo || !Wlce || !Y) return BRA_ERR_NULL;
    bra_shape ps = *shape;
    ps.H = Dp.H; ps.W = Dp.W;
    if (Dp.H == shape->H && Dp.W == shape->W)
        return bra_forward(&ps, X, Wqkv, Wo, Wlce, Y, Ir_out_opt, Ir_in_opt, ws, ws_bytes, hip_stream);
    int path = pick_path(&ps, Dp);
    if (path < 0) return path;
    const size_t inner = (path == BRA_PATH_MFMA) ? mfma_padded_workspace_bytes(Dp) : generic_workspace_bytes(Dp);
    if (!ws_ok(ws, ws_bytes, padded_workspace_bytes(Dp, inner))) return BRA_ERR_WORKSPACE;
    return padded_forward(Dp, shape->H, shape->W, X, Wqkv, Wo, Wlce, Y, Ir_out_opt, Ir_in_opt, ws, path,
                          (hipStream_t)hip_stream);
}

// Kernel family of the backward pass: the matrix-core kernels where they apply (bf16, heads of
// 32 or 64 channels, C a multiple of 64, at most 4096 routing entries per image), else the
// float32 kernels.
static int pick_backward_path(const bra_shape *s, const Dims &D)
{
    const bool mfma_ok = mfma_backward_supported(D);
    if (s->path == BRA_PATH_MFMA) return mfma_ok ? BRA_PATH_MFMA : BRA_ERR_UNSUPPORTED;
    if (s->path == BRA_PATH_AUTO && mfma_ok) return BRA_PATH_MFMA;
    return generic_backward_supported(D) ? BRA_PATH_GENERIC : BRA_ERR_UNSUPPORTED;
}

int bra_backward_workspace_bytes(const bra_shape *shape, size_t *out_bytes)
{
    if (!out_bytes) return BRA_ERR_NULL;
    Dims D;
    int rc = make_dims(shape, D);
    if (rc != BRA_OK) return rc;
    const int path = pick_backward_path(shape, D);
    if (path < 0) return path;
    *out_bytes = (path == BRA_PATH_MFMA) ? mfma_backward_workspace_bytes(D) : generic_backward_workspace_bytes(D);
    return BRA_OK;
}

int bra_backward(const bra_shape *shape, const void *X, const void *Wqkv, const void *Wo, const void *Wlce,
                 const int32_t *Ir, const void *dY, void *dX, float *dWqkv, float *dWo, float *dWlce, void *ws,
                 size_t ws_bytes, void *hip_stream)
{
    Dims D;
    int rc = make_dims(shape, D);
    if (rc != BRA_OK) return rc;
    if (!X || !Wqkv || !Wo || !Wlce || !Ir || !dY || !dX || !dWqkv || !dWo || !dWlce) return BRA_ERR_NULL;
    const int path = pick_backward_path(shape, D);
    if (path < 0) return path;
    if (path == BRA_PATH_MFMA) {
        if (!ws_ok(ws, ws_bytes, mfma_backward_workspace_bytes(D))) return BRA_ERR_WORKSPACE;
        return mfma_backward(D, X, Wqkv, Wo, Wlce, Ir, dY, dX, dWqkv, dWo, dWlce, ws, (hipStream_t)hip_stream);
    }
    if (!ws_ok(ws, ws_bytes, generic_backward_workspace_bytes(D))) return BRA_ERR_WORKSPACE;
    return generic_backward(D, X, Wqkv, Wo, Wlce, Ir, dY, dX, dWqkv, dWo, dWlce, ws, (hipStream_t)hip_stream);
}

int bra_block_workspace_bytes(const bra_shape *shape, int32_t hidden, size_t *out_bytes)
{
    if (!out_bytes) return BRA_ERR_NULL;
    Dims D;
    int rc = make_dims(shape, D);
    if (rc != BRA_OK) return rc;
    if (hidden < 1) return BRA_ERR_SHAPE;
    if (!block_supported(D, hidden)) return BRA_ERR_UNSUPPORTED;
    int path = pick_path(shape, D);
    if (path < 0) return path;
    const size_t inner = (path == BRA_PATH_MFMA) ? mfma_workspace_bytes(D) : generic_workspace_bytes(D);
    *out_bytes = block_workspace_bytes(D, hidden, inner);
    return BRA_OK;
}

int bra_block_forward(const bra_shape *shape, int32_t hidden, float eps, const void *X,
                      const bra_block_params *p, void *Xout, int32_t *Ir_out_opt, const int32_t *Ir_in_opt,
                      void *ws, size_t ws_bytes, void *hip_stream)
{
    Dims D;
    int rc = make_dims(shape, D);
    if (rc != BRA_OK) return rc;
    if (hidden < 1 || !(eps >= 0.f)) return BRA_ERR_SHAPE;
    if (!X || !p || !Xout) return BRA_ERR_NULL;
    if (!p->Wpos || !p->bpos || !p->ln1_gamma || !p->ln1_beta || !p->Wqkv || !p->Wo || !p->Wlce ||
        !p->ln2_gamma || !p->ln2_beta || !p->W1 || !p->b1 || !p->W2 || !p->b2)
        return BRA_ERR_NULL;
    if (!block_supported(D, hidden)) return BRA_ERR_UNSUPPORTED;
    int path = pick_path(shape, D);
    if (path < 0) return path;
    const size_t inner = (path == BRA_PATH_MFMA) ? mfma_workspace_bytes(D) : generic_workspace_bytes(D);
    if (!ws_ok(ws, ws_bytes, block_workspace_bytes(D, hidden, inner))) return BRA_ERR_WORKSPACE;
    return block_forward(D, hidden, eps, X, *p, Xout, Ir_out_opt, Ir_in_opt, ws, inner, path,
                         (hipStream_t)hip_stream);
}

int bra_ffn_workspace_bytes(const bra_ffn_shape *shape, size_t *out_bytes)
{
    if (!out_bytes) return BRA_ERR_NULL;
    ffn::Sizes S;
    const int rc = make_ffn_sizes(shape, S);
    if (rc != BRA_OK) return rc;
    *out_bytes = ffn_workspace_bytes(S);
    return BRA_OK;
}

int bra_ffn_forward(const bra_ffn_shape *shape, const void *X, const void *W1, const float *b1, const void *W2, const float *b2, void *Y, void *pre, void *ws,
                    size_t ws_bytes, void *hip_stream)
{
    ffn::Sizes S;
    const int rc = make_ffn_sizes(shape, S);
    if (rc != BRA_OK) return rc;
    if (S.M == 0) return BRA_OK;
    if (!X || !W1 || !W2 || !Y) return BRA_ERR_NULL;
    const size_t e = S.f32 ? 4 : 2;
    if (!aligned(row_alignment(S.C, e), {X, W2, Y}) || !aligned(row_alignment(S.h, e), {W1, pre}) || !aligned(4, {b1, b2})) return BRA_ERR_ALIGN;
    if (!ws_ok(ws, ws_bytes, ffn_workspace_bytes(S))) return BRA_ERR_WORKSPACE;
    return ffn_forward(S, X, W1, b1, W2, b2, Y, pre, ws, (hipStream_t)hip_stream);
}

int bra_ffn_backward_workspace_bytes(const bra_ffn_shape *shape, size_t *out_bytes)
{
    if (!out_bytes) return BRA_ERR_NULL;
    ffn::Sizes S;
    const int rc = make_ffn_sizes(shape, S);
    if (rc != BRA_OK) return rc;
    *out_bytes = ffn_backward_workspace_bytes(S);
    return BRA_OK;
}

int bra_ffn_backward(const bra_ffn_shape *shape, const void *X, const void *W1, const float *b1, const void *W2, const void *pre, const void *dY, void *dX, void *dW1,
                     void *dW2, void *db1, void *db2, int32_t grad_dtype, void *ws, size_t ws_bytes, void *hip_stream)
{
    ffn::Sizes S;
    const int rc = make_ffn_sizes(shape, S);
    if (rc != BRA_OK) return rc;
    if (S.M == 1L << 30) return BRA_ERR_SHAPE;          // (as the header has it)
    if (grad_dtype != BRA_F32 && grad_dtype != BRA_BF16) return BRA_ERR_DTYPE;
    if (!dW1 || !dW2 || (S.M > 0 && (!X || !W1 || !W2 || !dY || !dX))) return BRA_ERR_NULL;
    const size_t e = S.f32 ? 4 : 2, ge = grad_dtype == BRA_F32 ? 4 : 2;
    if (!aligned(row_alignment(S.C, e), {X, W2, dY, dX}) || !aligned(row_alignment(S.h, e), {W1, pre}) || !aligned(4, {b1})) return BRA_ERR_ALIGN;
    if (!aligned(row_alignment(S.h, ge), {dW1}) || !aligned(row_alignment(S.C, ge), {dW2}) || !aligned(ge, {db1, db2})) return BRA_ERR_ALIGN;
    if (!ws_ok(ws, ws_bytes, ffn_backward_workspace_bytes(S))) return BRA_ERR_WORKSPACE;
    return ffn_backward(S, X, W1, b1, W2, pre, dY, dX, dW1, dW2, db1, db2, grad_dtype == BRA_F32, ws, (hipStream_t)hip_stream);
}

int bra_norm_forward(const bra_norm_shape *shape, const void *X, const void *Y, const bra_norm_params *p, void *R, void *N, void *hip_stream)
{
    NormSizes S;
    const int rc = make_norm_sizes(shape, p && p->post_gamma, S);
    if (rc != BRA_OK) return rc;
    if (!p) return BRA_ERR_NULL;
    if (S.rows == 0) return BRA_OK;
    if (!X || !Y != !R || !p->gamma != !N || (!Y && !N)) return BRA_ERR_NULL;
    const size_t element = S.f32 ? 4 : 2;
    if (!aligned(element, {X, Y, R, N, p->gate}) || !aligned(4, {p->gamma, p->beta, p->post_gamma, p->post_beta, p->scale})) return BRA_ERR_ALIGN;
    S.vec = S.vec && aligned(16, {X, Y, R, N, p->gate});
    S.post = S.post && Y;
    const NormIn I{X, Y, Y ? p->gate : nullptr, p->gamma, p->beta, p->post_gamma, p->post_beta, p->scale};
    return norm_forward(S, I, R, N, (hipStream_t)hip_stream);
}

int bra_norm_backward_workspace_bytes(const bra_norm_shape *shape, int32_t post, size_t *out_bytes)
{
    if (!out_bytes) return BRA_ERR_NULL;
    NormSizes S;
    const int rc = make_norm_sizes(shape, post != 0, S);
    if (rc != BRA_OK) return rc;
    *out_bytes = norm_backward_workspace_bytes(S);
    S.vec = false;          // pointers that are not aligned share the rows out differently
    *out_bytes = std::max(*out_bytes, norm_backward_workspace_bytes(S));
    return BRA_OK;
}

int bra_norm_backward(const bra_norm_shape *shape, const void *R, const void *Y, const bra_norm_params *p, const void *dN, const void *dR, const bra_norm_grads *g,
                      void *ws, size_t ws_bytes, void *hip_stream)
{
    NormSizes S;
    const int rc = make_norm_sizes(shape, p && p->post_gamma && Y, S);
    if (rc != BRA_OK) return rc;
    if (!p || !g) return BRA_ERR_NULL;
    if (S.rows > 0 && (!R || !g->dX || (Y && !g->dY) || (!dN && !dR) || (dN && !p->gamma))) return BRA_ERR_NULL;
    const size_t element = S.f32 ? 4 : 2;
    if (!aligned(element, {R, Y, p->gate, dN, dR, g->dX, g->dY, g->dgate})) return BRA_ERR_ALIGN;
    if (!aligned(4, {p->gamma, p->beta, p->post_gamma, p->post_beta, p->scale, g->dgamma, g->dbeta, g->dpost_gamma, g->dpost_beta, g->dscale})) return BRA_ERR_ALIGN;
    S.vec = S.vec && aligned(16, {R, Y, p->gate, dN, dR, g->dX, g->dY, g->dgate});
    const size_t need = norm_backward_workspace_bytes(S);
    if (need && !ws_ok(ws, ws_bytes, need)) return BRA_ERR_WORKSPACE;
    const NormIn I{R, Y, Y ? p->gate : nullptr, p->gamma, p->beta, p->post_gamma, p->post_beta, p->scale};
    const NormGrads G{g->dX, g->dY, Y || S.rows == 0 ? g->dgate : nullptr, g->dgamma, g->dbeta, g->dpost_gamma, g->dpost_beta, g->dscale};
    return norm_backward(S, I, dN, dR, G, ws, (hipStream_t)hip_stream);
}

int bra_adamw_step(const bra_adamw_tensor *tensors, int32_t count, const bra_adamw_args *a, void *hip_stream)
{
    if (!a || (count > 0 && !tensors)) return BRA_ERR_NULL;
    auto fine = [](double v) { return v >= 0 && std::isfinite(v); };
    if (count < 0 || !fine(a->lr) || !fine(a->eps) || !(a->beta1 >= 0 && a->beta1 < 1) || !(a->beta2 >= 0 && a->beta2 < 1)) return BRA_ERR_SHAPE;
    if (!a->step_device && a->step < 1) return BRA_ERR_SHAPE;
    if (a->bits != 32 && a->bits != 8) return BRA_ERR_DTYPE;
    long total = 0;
    bool any = false;
    for (int i = 0; i < count; ++i) {
        const bra_adamw_tensor &t = tensors[i];
        if (t.n < 0 || t.n > (1L << 34) || !fine(t.weight_decay)) return BRA_ERR_SHAPE;
        if ((t.param_dtype != BRA_F32 && t.param_dtype != BRA_BF16) || (t.grad_dtype != BRA_F32 && t.grad_dtype != BRA_BF16)) return BRA_ERR_DTYPE;
        if (t.copy && t.param_dtype != BRA_F32) return BRA_ERR_DTYPE;
        total += (t.n + BRA_ADAMW_BLOCK - 1) / BRA_ADAMW_BLOCK;
        if (total > (1L << 31)) return BRA_ERR_SHAPE;
        if (!t.n || !t.grad) continue;
        any = true;
        if (!t.param) return BRA_ERR_NULL;
        if ((uintptr_t)t.param % (t.param_dtype == BRA_F32 ? 4 : 2) || (uintptr_t)t.grad % (t.grad_dtype == BRA_F32 ? 4 : 2) || (uintptr_t)t.copy % 2) return BRA_ERR_ALIGN;
    }
    if (!any) return BRA_OK;
    if (!a->exp_avg || !a->exp_avg_sq || (a->bits == 8 && (!a->exp_avg_scale || !a->exp_avg_sq_scale)) || (a->step_device && !a->scalars)) return BRA_ERR_NULL;
    if (!aligned(32, {a->exp_avg, a->exp_avg_sq}) || !aligned(4, {a->step_device, a->scalars, a->grad_scale})) return BRA_ERR_ALIGN;
    // what is written must be each tensor's own
    try {
        std::vector<std::pair<uintptr_t, uintptr_t>> spans;
        spans.reserve(2 * (size_t)count);
        for (int i = 0; i < count; ++i) {
            const bra_adamw_tensor &t = tensors[i];
            if (!t.n || !t.grad) continue;
            spans.emplace_back((uintptr_t)t.param, (uintptr_t)t.param + (size_t)t.n * (t.param_dtype == BRA_F32 ? 4 : 2));
            if (t.copy) spans.emplace_back((uintptr_t)t.copy, (uintptr_t)t.copy + (size_t)t.n * 2);
        }
        if (!std::is_sorted(spans.begin(), spans.end())) std::sort(spans.begin(), spans.end());
        for (size_t i = 1; i < spans.size(); ++i)
            if (spans[i].first < spans[i - 1].second) return BRA_ERR_OVERLAP;
    } catch (...) {
        return BRA_ERR_LAUNCH;
    }
    return adamw_step(tensors, count, *a, (hipStream_t)hip_stream);
}

// Where they lie.
struct QkNormVectors {
    Pieces at[5];
    QkNormVectors(const QkNormSizes &S, const QkNormIn &I)
    {
        const size_t gamma = 4 * (size_t)S.d, table = 4 * (size_t)S.table_rows * (S.turned / 2);
        at[0] = pieces_of(I.q_gamma, gamma);
        at[1] = pieces_of(I.k_gamma, gamma);
        at[2] = pieces_of(S.turned ? I.cos : nullptr, table);
        at[3] = pieces_of(S.turned ? I.sin : nullptr, table);
        at[4] = pieces_of(S.turned ? I.positions : nullptr, 4 * (size_t)S.tokens);
    }
};

int bra_attention_workspace_bytes(const bra_attention_shape *shape, size_t *out_bytes)
{
    if (!out_bytes) return BRA_ERR_NULL;
    att::Sizes S;
    const int rc = make_attention_sizes(shape, S);
    if (rc != BRA_OK) return rc;
    *out_bytes = attention_workspace_bytes(S);
    return BRA_OK;
}

int bra_attention_forward(const bra_attention_shape *shape, const bra_rows *Q, const bra_rows *K, const bra_rows *V, const int32_t *q_lens, const int32_t *k_lens, const bra_rows *O,
                          float *lse, void *ws, size_t ws_bytes, void *hip_stream)
{
    att::Sizes S;
    int rc = make_attention_sizes(shape, S);
    if (rc != BRA_OK) return rc;
    const size_t e = S.f32 ? 4 : 2;
    att::Rows q, k, v, o;
    if ((rc = make_rows(Q, S.B, S.Nq, S.H, e, q)) || (rc = make_rows(K, S.B, S.Nk, S.Hk, e, k)) || (rc = make_rows(V, S.B, S.Nk, S.Hk, e, v)) ||
        (rc = make_rows(O, S.B, S.Nq, S.H, e, o)))
        return rc;
    if (!aligned(4, {q_lens, k_lens, lse})) return BRA_ERR_ALIGN;
    if (S.B == 0 || S.Nq == 0) return BRA_OK;
    const size_t need = attention_workspace_bytes(S);
    if (need && !ws_ok(ws, ws_bytes, need)) return BRA_ERR_WORKSPACE;
    const long row = (long)e * S.d;
    const Pieces in[] = {pieces_of(q, S.B, S.Nq, S.H, row), pieces_of(k, S.B, S.Nk, S.Hk, row), pieces_of(v, S.B, S.Nk, S.Hk, row), pieces_of(q_lens, 4 * (size_t)S.B), pieces_of(k_lens, 4 * (size_t)S.B)};
    if (meet({{pieces_of(o, S.B, S.Nq, S.H, row), {}}, {pieces_of(lse, 4 * (size_t)S.B * S.H * S.Nq), {}}}, {&in[0], &in[1], &in[2], &in[3], &in[4]})) return BRA_ERR_OVERLAP;
    S.q_lens = q_lens;
    S.k_lens = k_lens;
    return attention_forward(S, q, k, v, o, lse, ws, (hipStream_t)hip_stream);
}

int bra_attention_backward_workspace_bytes(const bra_attention_shape *shape, size_t *out_bytes)
{
    if (!out_bytes) return BRA_ERR_NULL;
    att::Sizes S;
    const int rc = make_attention_sizes(shape, S);
    if (rc != BRA_OK) return rc;
    *out_bytes = attention_backward_workspace_bytes(S);
    return BRA_OK;
}

int bra_attention_backward(const bra_attention_shape *shape, const bra_rows *Q, const bra_rows *K, const bra_rows *V, const bra_rows *O, const float *lse, const bra_rows *dO,
                           const int32_t *q_lens, const int32_t *k_lens, const bra_rows *dQ, const bra_rows *dK, const bra_rows *dV, void *ws, size_t ws_bytes, void *hip_stream)
{
    att::Sizes S;
    int rc = make_attention_sizes(shape, S);
    if (rc != BRA_OK) return rc;
    const size_t e = S.f32 ? 4 : 2;
    att::Rows q, k, v, o, go, dq, dk, dv;
    if ((rc = make_rows(Q, S.B, S.Nq, S.H, e, q)) || (rc = make_rows(K, S.B, S.Nk, S.Hk, e, k)) || (rc = make_rows(V, S.B, S.Nk, S.Hk, e, v)) ||
        (rc = make_rows(O, S.B, S.Nq, S.H, e, o)) || (rc = make_rows(dO, S.B, S.Nq, S.H, e, go)) || (rc = make_rows(dQ, S.B, S.Nq, S.H, e, dq)) ||
        (rc = make_rows(dK, S.B, S.Nk, S.Hk, e, dk)) || (rc = make_rows(dV, S.B, S.Nk, S.Hk, e, dv)))
        return rc;
    if (S.B > 0 && S.Nq > 0 && !lse) return BRA_ERR_NULL;
    if (!aligned(4, {q_lens, k_lens, lse})) return BRA_ERR_ALIGN;
    if (S.B == 0 || (S.Nq == 0 && S.Nk == 0)) return BRA_OK;
    const size_t need = attention_backward_workspace_bytes(S);
    if (need && !ws_ok(ws, ws_bytes, need)) return BRA_ERR_WORKSPACE;
    const long row = (long)e * S.d;
    auto queries = [&](const att::Rows &R) { return pieces_of(R, S.B, S.Nq, S.H, row); };
    auto keys = [&](const att::Rows &R) { return pieces_of(R, S.B, S.Nk, S.Hk, row); };
    const Pieces in[] = {queries(q), keys(k), keys(v), queries(o), queries(go), pieces_of(lse, 4 * (size_t)S.B * S.H * S.Nq), pieces_of(q_lens, 4 * (size_t)S.B), pieces_of(k_lens, 4 * (size_t)S.B)};
    if (meet({{queries(dq), {}}, {keys(dk), {}}, {keys(dv), {}}}, {&in[0], &in[1], &in[2], &in[3], &in[4], &in[5], &in[6], &in[7]})) return BRA_ERR_OVERLAP;
    S.q_lens = q_lens;
    S.k_lens = k_lens;
    return attention_backward(S, q, k, v, o, lse, go, dq, dk, dv, ws, (hipStream_t)hip_stream);
}

int bra_qk_norm_forward(const bra_qk_norm_shape *shape, const bra_rows *Q, const bra_rows *K, const bra_qk_norm_params *params, const bra_rows *Qout, const bra_rows *Kout,
                        void *hip_stream)
{
    QkNormSizes S;
    int rc = make_qk_norm_sizes(shape, S);
    if (rc != BRA_OK) return rc;
    QkNormIn I{};
    if ((rc = qk_norm_in(shape, S, params, I)) != BRA_OK) return rc;
    const size_t e = S.f32 ? 4 : 2;
    att::Rows q, k;
    if ((rc = make_rows(Q, shape->B, S.N, S.heads, e, I.Q)) || (rc = make_rows(K, shape->B, S.N, S.kv_heads, e, I.K)) || (rc = make_rows(Qout, shape->B, S.N, S.heads, e, q)) ||
        (rc = make_rows(Kout, shape->B, S.N, S.kv_heads, e, k)))
        return rc;
    const long row = (long)e * S.d, B = shape->B;
    const QkNormVectors vectors(S, I);
    const Pieces in[] = {pieces_of(I.Q, B, S.N, S.heads, row), pieces_of(I.K, B, S.N, S.kv_heads, row)};
    if (meet({{pieces_of(q, B, S.N, S.heads, row), {&in[0]}}, {pieces_of(k, B, S.N, S.kv_heads, row), {&in[1]}}},
             {&in[0], &in[1], &vectors.at[0], &vectors.at[1], &vectors.at[2], &vectors.at[3], &vectors.at[4]}))
        return BRA_ERR_OVERLAP;
    return qk_norm_forward(S, I, q, k, (hipStream_t)hip_stream);
}

int bra_qk_norm_backward_workspace_bytes(const bra_qk_norm_shape *shape, size_t *out_bytes)
{
    if (!out_bytes) return BRA_ERR_NULL;
    QkNormSizes S;
    const int rc = make_qk_norm_sizes(shape, S);
    if (rc != BRA_OK) return rc;
    *out_bytes = qk_norm_backward_workspace_bytes(S);
    return BRA_OK;
}

int bra_qk_norm_backward(const bra_qk_norm_shape *shape, const bra_rows *Q, const bra_rows *K, const bra_qk_norm_params *params, const bra_rows *gQ, const bra_rows *gK,
                         const bra_rows *dQ, const bra_rows *dK, float *dq_gamma, float *dk_gamma, void *ws, size_t ws_bytes, void *hip_stream)
{
    QkNormSizes S;
    int rc = make_qk_norm_sizes(shape, S);
    if (rc != BRA_OK) return rc;
    QkNormIn I{};
    if ((rc = qk_norm_in(shape, S, params, I)) != BRA_OK) return rc;
    const size_t e = S.f32 ? 4 : 2;
    att::Rows gq, gk, dq, dk;
    if ((I.q_gamma && ((rc = make_rows(Q, shape->B, S.N, S.heads, e, I.Q)) || (rc = make_rows(K, shape->B, S.N, S.kv_heads, e, I.K)))) ||
        (rc = make_rows(gQ, shape->B, S.N, S.heads, e, gq)) || (rc = make_rows(gK, shape->B, S.N, S.kv_heads, e, gk)) ||
        (rc = make_rows(dQ, shape->B, S.N, S.heads, e, dq)) || (rc = make_rows(dK, shape->B, S.N, S.kv_heads, e, dk)))
        return rc;
    if (!aligned(4, {dq_gamma, dk_gamma})) return BRA_ERR_ALIGN;
    const size_t need = qk_norm_backward_workspace_bytes(S);
    if (I.q_gamma && need && !ws_ok(ws, ws_bytes, need)) return BRA_ERR_WORKSPACE;
    const long row = (long)e * S.d, B = shape->B;
    auto queries = [&](const att::Rows &R) { return pieces_of(R, B, S.N, S.heads, row); };
    auto keys = [&](const att::Rows &R) { return pieces_of(R, B, S.N, S.kv_heads, row); };
    const QkNormVectors vectors(S, I);
    const Pieces in[] = {queries(I.Q), keys(I.K), queries(gq), keys(gk)};
    const size_t sums = I.q_gamma ? 4 * (size_t)S.d : 0;
    if (meet({{queries(dq), {&in[0], &in[2]}}, {keys(dk), {&in[1], &in[3]}}, {pieces_of(dq_gamma, sums), {}}, {pieces_of(dk_gamma, sums), {}}},
             {&in[0], &in[1], &in[2], &in[3], &vectors.at[0], &vectors.at[1], &vectors.at[2], &vectors.at[3], &vectors.at[4]}))
        return BRA_ERR_OVERLAP;
    return qk_norm_backward(S, I, gq, gk, dq, dk, dq_gamma, dk_gamma, ws, (hipStream_t)hip_stream);
}

const char *bra_strerror(int code)
{
    switch (code) {
    case BRA_OK: return "ok";
    case BRA_ERR_NULL: return "a required pointer is NULL";
    case BRA_ERR_SHAPE: return "invalid shape (sizes must be positive, S must divide H and W, heads must divide C)";
    case BRA_ERR_K: return "k must satisfy 1 <= k <= S*S";
    case BRA_ERR_DTYPE: return "unknown dtype or path";
    case BRA_ERR_WORKSPACE: return "workspace is NULL, not 256-byte aligned, or too small";
    case BRA_ERR_UNSUPPORTED: return "shape not supported by the requested kernel family";
    case BRA_ERR_LAUNCH: return "HIP runtime error while enqueueing";
    case BRA_ERR_TOO_LARGE: return "shape needs more scratch memory than the library's built-in buffer holds";
    case BRA_ERR_OVERLAP: return "what is written shares memory with another part of itself or of the call";
    case BRA_ERR_ALIGN: return "a tensor is not aligned as its entry point asks";
    default: return "unknown error code";
    }
}

int bra_version(void) { return 100; }

}  // extern "C"
