// Entry points of the window attention: the descriptor's check, the choice of kernels.
#include <initializer_list>
#include "psf_window.h"

namespace psf {
namespace {

psf_status make_window(const psf_window_desc *desc, Window *out)
{
    if (!desc) return PSF_ERR_NULL;
    if (desc->batch <= 0 || desc->heads <= 0 || desc->kv_heads <= 0 || desc->n <= 0 || desc->d <= 0 || desc->window <= 0 ||
        desc->sinks < 0 || desc->heads % desc->kv_heads != 0)
        return PSF_ERR_SHAPE;
    if (desc->dtype != PSF_F32 && desc->dtype != PSF_BF16) return PSF_ERR_UNSUPPORTED;
    if (desc->layout != PSF_HEADS_FIRST && desc->layout != PSF_TOKENS_FIRST) return PSF_ERR_UNSUPPORTED;
    if (desc->d % 8 != 0 || desc->d > PSF_WINDOW_MAX_DIM) return PSF_ERR_UNSUPPORTED;
    // (batch, head) pairs index grid dimension y; positions plus a window stay inside 32 bits; a tile's rows
    // lie within 4 GB of each other
    if ((long long)desc->batch * desc->heads > 65535 || desc->n > (1 << 24) || (long long)desc->heads * desc->d > (1 << 20))
        return PSF_ERR_UNSUPPORTED;
    // a launch holds fewer than 2^32 work-items: 256 for 32 rows
    if ((long long)desc->batch * desc->heads * ((desc->n + 63) / 64) >= (1 << 23)) return PSF_ERR_UNSUPPORTED;
    Window w;
    w.batch = desc->batch; w.heads = desc->heads; w.kv_heads = desc->kv_heads; w.group = desc->heads / desc->kv_heads;
    w.n = desc->n; w.d = desc->d;
    w.window = desc->window < desc->n ? desc->window : desc->n;
    w.sinks = desc->sinks < desc->n ? desc->sinks : desc->n;
    w.bf16 = desc->dtype == PSF_BF16;
    if (!(fabsf(desc->scale) < INFINITY)) return PSF_ERR_UNSUPPORTED;
    w.scale = desc->scale;
    w.scale2 = desc->scale * kWindowLog2e;
    const int64_t n = w.n, d = w.d;
    const bool tokens = desc->layout == PSF_TOKENS_FIRST;
    w.batch_q = n * w.heads * d;    w.head_q = tokens ? d : n * d; w.row_q = tokens ? w.heads * d : d;
    w.batch_k = n * w.kv_heads * d; w.head_k = tokens ? d : n * d; w.row_k = tokens ? w.kv_heads * d : d;
    *out = w;
    return PSF_OK;
}

// Whether a call goes to the kernels that keep weights in three bf16 parts: fp32 storage, and calls of one tile, whose few
// weights' roundings to bf16 would not average out and where the products cost nothing (both directions, 16 x 32 heads, 32 tokens:
// 23 us against 27 at d = 64, 36 against 34 at d = 128; 64 tokens: 36 against 33, 56 against 46).
constexpr int kShort = 32;
bool in_parts(const Window &w) { return !w.bf16 || w.n <= kShort; }

size_t delta_bytes(const Window &w) { return align_up((size_t)w.batch * w.heads * w.n * sizeof(float), 256); }

bool aligned16(std::initializer_list<const void *> tensors)
{
    for (const void *p : tensors)
        if (((uintptr_t)p & 15u) != 0) return false;
    return true;
}

}  // namespace
}  // namespace psf

using namespace psf;

extern "C" {

psf_status psf_check_window_desc(const psf_window_desc *desc)
{
    Window w;
    return make_window(desc, &w);
}

psf_status psf_window_attn_fwd(const psf_window_desc *desc, const void *Q, const void *K, const void *V, const int32_t *lengths,
                               void *O, float *lse, void *hip_stream)
{
    Window w;
    const psf_status st = make_window(desc, &w);
    if (st != PSF_OK) return st;
    if (!Q || !K || !V || !O) return PSF_ERR_NULL;
    if (!aligned16({Q, K, V, O})) return PSF_ERR_ALIGNMENT;
    WindowPtrs p = {};
    p.Q = Q; p.K = K; p.V = V; p.lengths = lengths;
    return in_parts(w) ? window_parts_fwd(w, p, O, lse, (hipStream_t)hip_stream) : window_bf16_fwd(w, p, O, lse, (hipStream_t)hip_stream);
}

size_t psf_window_attn_bwd_workspace_bytes(const psf_window_desc *desc)
{
    Window w;
    if (make_window(desc, &w) != PSF_OK) return 0;
    return delta_bytes(w) + align_up(in_parts(w) ? window_parts_room(w) : window_bf16_room(w), 256);
}

psf_status psf_window_attn_bwd(const psf_window_desc *desc, const void *Q, const void *K, const void *V, const int32_t *lengths,
                               const void *O, const float *lse, const void *dO, void *dQ, void *dK, void *dV, void *workspace,
                               size_t workspace_bytes, void *hip_stream)
{
    Window w;
    psf_status st = make_window(desc, &w);
    if (st != PSF_OK) return st;
    if (!Q || !K || !V || !O || !lse || !dO || !dQ || !dK || !dV || !workspace) return PSF_ERR_NULL;
    if (workspace_bytes < psf_window_attn_bwd_workspace_bytes(desc)) return PSF_ERR_WORKSPACE;
    if (((uintptr_t)workspace & 255u) != 0) return PSF_ERR_WORKSPACE;
    if (!aligned16({Q, K, V, O, dO, dQ, dK, dV})) return PSF_ERR_ALIGNMENT;
    hipStream_t s = (hipStream_t)hip_stream;
    WindowPtrs p = {};
    p.Q = Q; p.K = K; p.V = V; p.O = O; p.dO = dO; p.lengths = lengths; p.lse = lse;
    p.dQ = dQ; p.dK = dK; p.dV = dV;
    p.delta = (float *)workspace;
    p.room = (float *)((char *)workspace + delta_bytes(w));
    return in_parts(w) ? window_parts_bwd(w, p, s) : window_bf16_bwd(w, p, s);
}

}  // extern "C"
