// Softmax attention with a sliding window and a few first tokens that stay visible: the shape as the
// kernels see it (psf_window.hip, psf_window_parts.hip, psf_window_bf16.hip).
//
//   row i < length:  p_ij = exp(scale <q_i, k_j> - L_i) over the visible j,  o_i = sum_j p_ij v_j,
//   visible: j <= i and (i - j < window or j < sinks);  L_i = log sum_j exp(scale <q_i, k_j>)
//   backward: D_i = <dO_i, o_i>,  dS_ij = p_ij (<dO_i, v_j> - D_i),
//     dQ_i = scale sum_j dS_ij k_j,  dK_j = scale sum_i dS_ij q_i,  dV_j = sum_i p_ij dO_i
//     (sums over i: over all query heads of the key head).
#ifndef PSF_WINDOW_H
#define PSF_WINDOW_H

#include "psf_internal.h"

namespace psf {

struct Window {
    int batch, heads, kv_heads, group, n, d, window, sinks;
    bool bf16;
    float scale, scale2;                   // of the scores, and with log2(e)
    // a row of Q (heads), of K and V (kv_heads): batch b, head h, token i at b * batch_* + h * head_* + i * row_*
    int64_t batch_q, head_q, row_q, batch_k, head_k, row_k;
};

struct WindowPtrs {
    const void *Q, *K, *V, *O, *dO;
    const int32_t *lengths;
    const float *lse;
    float *delta;                          // [batch, heads, n]
    void *dQ, *dK, *dV;
    float *room;                           // shares of gradients that several workgroups form
};

constexpr float kWindowLog2e = 1.4426950408889634f, kWindowLn2 = 0.6931471805599453f;

__device__ __forceinline__ int window_end(const int32_t *lengths, int b, int n)
{
    if (!lengths) return n;
    const int e = lengths[b];
    return e < 0 ? 0 : e < n ? e : n;
}
__device__ __forceinline__ bool window_sees(const Window &w, int i, int j)
{
    return j <= i && (i - j < w.window || j < w.sinks);
}

// The tiles of `size` keys that rows [first, last] see some of: those of the first tokens, then those of the window.
struct KeyTiles {
    int few, window_first, total;
    __device__ __forceinline__ KeyTiles(const Window &w, int first, int last, int size)
    {
        const int start = first >= w.window ? first - w.window + 1 : 0;
        const int shown = w.sinks < start ? w.sinks : start;
        few = (shown + size - 1) / size;
        window_first = start / size;
        if (window_first < few) window_first = few;
        total = few + (last / size + 1 - window_first);
    }
    __device__ __forceinline__ int at(int k) const { return k < few ? k : window_first + k - few; }
};

psf_status window_bf16_fwd(const Window &w, const WindowPtrs &p, void *O, float *lse, hipStream_t s);
psf_status window_bf16_bwd(const Window &w, const WindowPtrs &p, hipStream_t s);
size_t window_bf16_room(const Window &w);              // bytes of WindowPtrs::room
psf_status window_parts_fwd(const Window &w, const WindowPtrs &p, void *O, float *lse, hipStream_t s);
psf_status window_parts_bwd(const Window &w, const WindowPtrs &p, hipStream_t s);
size_t window_parts_room(const Window &w);

}  // namespace psf
#endif
