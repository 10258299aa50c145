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

__device__ __forceinline__ uint32_t bits_below(int n) { return n <= 0 ? 0u : n >= 32 ? 0xffffffffu : (1u << n) - 1u; }
// keys j0 .. j0 + 31 that row i sees, as bits
__device__ __forceinline__ uint32_t seen_keys(const Window &w, int i, int j0)
{
    return bits_below(i - j0 + 1) & (~bits_below(i - w.window + 1 - j0) | bits_below(w.sinks - j0));
}
// rows i0 .. i0 + 31 below `end` that see key j, as bits
__device__ __forceinline__ uint32_t seen_by(const Window &w, int j, int i0, int end)
{
    const int64_t reach = j < w.sinks ? (int64_t)end : (int64_t)j + w.window;
    return bits_below((reach < end ? (int)reach : end) - i0) & ~bits_below(j - i0);
}
// Whether rows [i0, i0 + rows - 1] see all / none of keys [j0, j0 + len - 1].
__device__ __forceinline__ bool all_seen(const Window &w, int i0, int rows, int j0, int len)
{
    return j0 + len - 1 <= i0 && (i0 + rows - 1 - j0 < w.window || j0 + len <= w.sinks);
}
__device__ __forceinline__ bool none_seen(const Window &w, int i0, int rows, int j0, int len)
{
    return j0 > i0 + rows - 1 || (i0 - (j0 + len - 1) >= w.window && j0 >= w.sinks);
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

// How the walks of the key side are shared out.  A workgroup of `own` keys walks the tiles of queries that see one of them, head
// after head of the group.  The first `few` workgroups of a unit hold the tokens that every later row sees; their
// walks are `parts` times as long as the others' and go to as many workgroups, whose shares a second kernel adds in order.
struct KeyWalks {
    int few, parts, groups;                // groups: workgroups of `own` keys of a unit
    __host__ __device__ int each() const { return groups - few + few * parts; }
};
// Workgroup `which` of a unit: its group of keys and its part of their walk.
struct KeyWalk {
    int group, part, parts;
    __device__ __forceinline__ KeyWalk(const KeyWalks &k, int which)
    {
        const int shared = k.few * k.parts;
        group = which < shared ? which / k.parts : which - shared + k.few;
        part = which < shared ? which % k.parts : 0;
        parts = which < shared ? k.parts : 1;
    }
};
// Queries that see one of the keys [first, first + own): tiles [tile0, tile0 + count) of `size` rows.
struct QueryTiles {
    int tile0, count;
    __device__ __forceinline__ QueryTiles(const Window &w, int first, int end, int own, int size)
    {
        const int64_t reach = first < w.sinks ? (int64_t)end - 1 : (int64_t)first + own - 1 + w.window - 1;
        const int last = reach < end ? (int)reach : end - 1;
        tile0 = first / size;
        count = last / size + 1 - tile0;
    }
};
// Long walks of the first tokens are cut to the length of the others', but into no more workgroups than a few for every
// CU in all (their shares lie in memory: 1 KB for a key at d = 128).
inline KeyWalks key_walks(const Window &w, int own, int size)
{
    KeyWalks k;
    k.groups = (w.n + own - 1) / own;
    k.few = 0;
    k.parts = 1;
    const int holding = (w.sinks + own - 1) / own;         // (sinks is at most n)
    if (holding == 0) return k;
    const int longest = (w.n + size - 1) / size, other = (w.window + own - 2) / size + 1;
    const int64_t most = 1024 / ((int64_t)holding * w.batch * w.kv_heads);
    int64_t parts = (longest + other - 1) / other;
    if (parts > most) parts = most;
    if (parts <= 1) return k;
    k.few = holding;
    k.parts = (int)parts;
    return k;
}
// Shares: [unit][group][part][dK, dV][own][d] floats.
inline size_t key_walks_room(const Window &w, const KeyWalks &k, int own)
{
    return k.parts == 1 ? 0 : (size_t)w.batch * w.kv_heads * k.few * k.parts * 2 * own * w.d * sizeof(float);
}

psf_status window_bf16_fwd(const Window &w, const WindowPtrs &p, void *O, float *lse, hipStream_t s);
psf_status window_bf16_bwd(const Window &w, const WindowPtrs &p, hipStream_t s);
size_t window_bf16_room(const Window &w);              // bytes of WindowPtrs::room
psf_status window_bf16_delta(const Window &w, const WindowPtrs &p, bool all, hipStream_t s);   // D of rows of few keys, or of all
psf_status window_parts_fwd(const Window &w, const WindowPtrs &p, void *O, float *lse, hipStream_t s);
psf_status window_parts_bwd(const Window &w, const WindowPtrs &p, hipStream_t s);
size_t window_parts_room(const Window &w);

}  // namespace psf
#endif
