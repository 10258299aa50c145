// Window attention on bf16 parts of its values and weights (psf_parts.h): fp32 storage in three parts, and short
// calls in bf16 storage, whose values are one part.  A wave owns 16 rows as the columns of its results; tiles of 32 rows of
// the other side go through LDS, where they are read along their rows for the scores and transposed for the
// sums.  In fp32 bound by the six products that stand for one fp32 product and by taking the tiles apart, which every
// workgroup does for itself.
#include "psf_parts.h"
#include "psf_window.h"

namespace psf {
namespace {

constexpr int kTile = 32;
constexpr int kRows = 64;                  // rows of a workgroup: four waves of 16

// A tile of 32 rows of both operands (keys and values, or queries and output gradients) on its way into LDS.
template <int NT, typename S>
struct TilePair {
    static constexpr int PITCH = row_pitch<NT>(), P = parts_of<S>(), PLANE = kTile * PITCH;
    PartTile<NT, kTile, PITCH, S> a, b;
    __device__ __forceinline__ void load(const S *x, const S *y, int ld, int valid, int width)
    {
        a.load(x, ld, valid, width);
        b.load(y, ld, valid, width);
    }
    // Returns bit 0 when the first operand, bit 1 when the second has shown an infinity or NaN to the workgroup so far
    // (`seen` in LDS, zero before the first tile).
    __device__ __forceinline__ int store(uint16_t *to_a, uint16_t *to_b, int valid, int width, int *seen) const
    {
        const bool odd_a = a.template store<true>(to_a, valid, width), odd_b = b.template store<true>(to_b, valid, width);
        if (odd_a || odd_b) atomicOr(seen, (odd_a ? 1 : 0) | (odd_b ? 2 : 0));
        __syncthreads();
        return *seen;
    }
};

__device__ __forceinline__ float max_over_groups(float x)
{
    const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
    const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}

// acc += tile^T w for this lane's eight places of the tile (tile order); seen: bit k for tile row k
template <int NT, int P>
__device__ __forceinline__ void add_tile(const uint16_t *tile, int plane, int pitch, const float (&w8)[8], f4 (&acc)[NT], int lane,
                                         bool odd, unsigned seen)
{
    if (odd) add_parts_odd<NT, P>(tile, plane, pitch, w8, acc, lane, seen);
    else {
        Parts<3> w;
        split8(w8, w);
        add_parts<NT, P>(tile, plane, pitch, w, acc, lane);
        settle_parts();
    }
}

// This lane's eight places of a tile (tile order), as bits of it
__device__ __forceinline__ constexpr int place(int e) { return 16 * (e / 4) + e % 4; }

template <int NT, typename S>
__global__ __launch_bounds__(256) void window_parts_fwd_kernel(const S *Q, const S *K, const S *V, const int32_t *lengths, S *O,
                                                               float *lse, Window w)
{
    constexpr int KS = NT / 2, P = parts_of<S>();
    using Tiles = TilePair<NT, S>;
    __shared__ uint16_t tk[P * Tiles::PLANE], tv[P * Tiles::PLANE];
    __shared__ int odd_seen;
    if (threadIdx.x == 0) odd_seen = 0;                    // (the loop's first barrier comes before its first use)
    const int lane = threadIdx.x & 63, li = lane & 15, g = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int b = blockIdx.y / w.heads, h = blockIdx.y % w.heads, d = w.d;
    const int end = window_end(lengths, b, w.n), first = blockIdx.x * kRows, i0 = first + 16 * wave, i = i0 + li;
    const int64_t at_q = b * w.batch_q + h * w.head_q, at_k = b * w.batch_k + h / w.group * w.head_k;
    f4 acc[NT];
    clear(acc);
    float top = -INFINITY, sum = 0.f;
    if (first < end) {                                     // (the same in the whole workgroup)
        Parts<P> own[KS];
        {
            OwnRow<KS, S> row;
            row.load(Q + at_q + (i < end ? i : end - 1) * w.row_q, d, 1, g);
            row.parts(own, d, g);
        }
        const int last = first + kRows < end ? first + kRows - 1 : end - 1;
        const KeyTiles tiles(w, first, last, kTile);
        Tiles next;
        auto load = [&](int k) {
            const int j0 = tiles.at(k) * kTile;
            next.load(K + at_k + j0 * w.row_k, V + at_k + j0 * w.row_k, (int)w.row_k, end - j0, d);
        };
        load(0);
        for (int k = 0; k < tiles.total; ++k) {
            const int j0 = tiles.at(k) * kTile;
            __syncthreads();
            const int odd = next.store(tk, tv, end - j0, d, &odd_seen);
            if (k + 1 < tiles.total) load(k + 1);
            f4 s[2];
            score_parts<2, KS, P, P>(tk, Tiles::PLANE, Tiles::PITCH, 0, own, lane, s);
            float w8[8], most = -INFINITY;
#pragma unroll
            for (int e = 0; e < 8; ++e) w8[e] = s[e / 4][e % 4] * w.scale2;
            uint32_t seen = 0xffffffffu;                   // the tile's rows, as this row sees them
            if (!all_seen(w, i0, 16, j0, kTile) || i0 + 15 >= end) {
                seen = i < end ? seen_keys(w, i, j0) : 0u;
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    if (!(seen >> 4 * g >> place(e) & 1u)) w8[e] = -INFINITY;
            }
#pragma unroll
            for (int e = 0; e < 8; ++e) most = fmaxf(most, w8[e]);
            most = fmaxf(top, max_over_groups(most));
            const float less = top == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(top - most), base = most == -INFINITY ? 0.f : most;
            top = most;
            sum *= less;
#pragma unroll
            for (int t = 0; t < NT; ++t) acc[t] *= less;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                w8[e] = __builtin_amdgcn_exp2f(w8[e] - base);
                sum += w8[e];
            }
            add_tile<NT, P>(tv, Tiles::PLANE, Tiles::PITCH, w8, acc, lane, odd & 2, seen);
        }
    }
    sum = over_groups(sum);
    if (i >= w.n) return;
    const float by = i < end ? 1.f / sum : 0.f;
#pragma unroll
    for (int t = 0; t < NT; ++t) store_piece(O + at_q + i * w.row_q, 16 * t + 4 * g, d, 1, acc[t] * by);
    if (lse && g == 0) lse[((size_t)b * w.heads + h) * w.n + i] = i < end ? (top + log2f(sum)) * kWindowLn2 : -INFINITY;
}

// dQ: as forward, a wave owns 16 queries; and D = <dO, o> of every row for the kernel below.
template <int NT, typename S>
__global__ __launch_bounds__(256, 2) void window_parts_dq_kernel(const S *Q, const S *K, const S *V, const S *O, const S *dO,
                                                              const int32_t *lengths, const float *lse, float *delta, S *dQ,
                                                              Window w)
{
    constexpr int KS = NT / 2, P = parts_of<S>();
    using Tiles = TilePair<NT, S>;
    __shared__ uint16_t tk[P * Tiles::PLANE], tv[P * Tiles::PLANE];
    __shared__ int odd_seen;
    if (threadIdx.x == 0) odd_seen = 0;                    // (the loop's first barrier comes before its first use)
    const int lane = threadIdx.x & 63, li = lane & 15, g = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int b = blockIdx.y / w.heads, h = blockIdx.y % w.heads, d = w.d;
    const int end = window_end(lengths, b, w.n), first = blockIdx.x * kRows, i0 = first + 16 * wave, i = i0 + li;
    const int64_t at_q = b * w.batch_q + h * w.head_q, at_k = b * w.batch_k + h / w.group * w.head_k;
    f4 acc[NT];
    clear(acc);
    if (first < end) {
        const int safe = i < end ? i : end - 1;
        Parts<P> own[KS], own_g[KS];
        float D = 0.f;
        {
            OwnRow<KS, S> row, row_g;
            row.load(Q + at_q + safe * w.row_q, d, 1, g);
            row_g.load(dO + at_q + safe * w.row_q, d, 1, g);
            if constexpr (P == 3) {
                OwnRow<KS, S> row_o;
                row_o.load(O + at_q + safe * w.row_q, d, 1, g);
#pragma unroll
                for (int e = 0; e < 2 * KS; ++e) {
                    const f4 x = row_g.at(e, d, g), y = row_o.at(e, d, g);
#pragma unroll
                    for (int k = 0; k < 4; ++k) D += x[k] * y[k];
                }
            }
            row.parts(own, d, g);
            row_g.parts(own_g, d, g);
        }
        const size_t row = ((size_t)b * w.heads + h) * w.n + safe;
        const float L = lse[row] * kWindowLog2e;
        if constexpr (P == 3) {
            D = over_groups(D);
            if (i < end && g == 0) delta[row] = D;
        } else {
            D = delta[row];                                // (formed from the weights before: o is rounded to bf16)
        }
        const int last = first + kRows < end ? first + kRows - 1 : end - 1;
        const KeyTiles tiles(w, first, last, kTile);
        Tiles next;
        auto load = [&](int k) {
            const int j0 = tiles.at(k) * kTile;
            next.load(K + at_k + j0 * w.row_k, V + at_k + j0 * w.row_k, (int)w.row_k, end - j0, d);
        };
        load(0);
        for (int k = 0; k < tiles.total; ++k) {
            const int j0 = tiles.at(k) * kTile;
            __syncthreads();
            const int odd = next.store(tk, tv, end - j0, d, &odd_seen);
            if (k + 1 < tiles.total) load(k + 1);
            f4 s[2], t[2];
            score_parts<2, KS, P, P>(tk, Tiles::PLANE, Tiles::PITCH, 0, own, lane, s);
            score_parts<2, KS, P, P>(tv, Tiles::PLANE, Tiles::PITCH, 0, own_g, lane, t);
            float w8[8];
#pragma unroll
            for (int e = 0; e < 8; ++e)
                w8[e] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[e / 4][e % 4], w.scale2, -L)) * (t[e / 4][e % 4] - D);
            uint32_t seen = 0xffffffffu;
            if (!all_seen(w, i0, 16, j0, kTile) || i0 + 15 >= end) {
                seen = i < end ? seen_keys(w, i, j0) : 0u;
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    if (!(seen >> 4 * g >> place(e) & 1u)) w8[e] = 0.f;
            }
            add_tile<NT, P>(tk, Tiles::PLANE, Tiles::PITCH, w8, acc, lane, odd & 1, seen);
        }
    }
    if (i >= w.n) return;
#pragma unroll
    for (int t = 0; t < NT; ++t) store_piece(dQ + at_q + i * w.row_q, 16 * t + 4 * g, d, 1, acc[t] * w.scale);
}

// dK, dV: a wave owns 16 keys, tiles of 32 queries pass, head after head of the group.  Two waves a SIMD where the sums of d = 64
// leave the room (2 x 12 x 1951, window 300, both kernels: 155 us instead of 168); at d = 128 they would not stay in registers
// (2 x 8 x 2000, window 500: 335 instead of 293).
template <int NT, typename S>
__global__ __launch_bounds__(256, NT == 4 ? 2 : 1) void window_parts_dkv_kernel(const S *Q, const S *K, const S *V, const S *dO,
                                                               const int32_t *lengths, const float *lse, const float *delta,
                                                               S *dK, S *dV, float *room, Window w, KeyWalks walks)
{
    constexpr int KS = NT / 2, P = parts_of<S>();
    using Tiles = TilePair<NT, S>;
    __shared__ uint16_t tq[P * Tiles::PLANE], tg[P * Tiles::PLANE];
    __shared__ float rows_l[kTile], rows_d[kTile];
    __shared__ int odd_seen;
    if (threadIdx.x == 0) odd_seen = 0;                    // (the loop's first barrier comes before its first use)
    const int lane = threadIdx.x & 63, li = lane & 15, g = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const KeyWalk walk(walks, blockIdx.x);
    const int b = blockIdx.y / w.kv_heads, kv = blockIdx.y % w.kv_heads, d = w.d;
    const int end = window_end(lengths, b, w.n), first = walk.group * kRows, own_at = 16 * wave + li, j0 = first + 16 * wave, j = j0 + li;
    const int64_t at_k = b * w.batch_k + kv * w.head_k;
    f4 acc_k[NT], acc_v[NT];
    clear(acc_k);
    clear(acc_v);
    if (first < end) {
        const int safe = j < end ? j : end - 1;
        Parts<P> own[KS], own_v[KS];
        {
            OwnRow<KS, S> row, row_v;
            row.load(K + at_k + safe * w.row_k, d, 1, g);
            row_v.load(V + at_k + safe * w.row_k, d, 1, g);
            row.parts(own, d, g);
            row_v.parts(own_v, d, g);
        }
        const QueryTiles tiles(w, first, end, kRows, kTile);
        const int tile0 = tiles.tile0, per = tiles.count, total = per * w.group;
        const int begin = (int)((int64_t)total * walk.part / walk.parts), stop = (int)((int64_t)total * (walk.part + 1) / walk.parts);
        Tiles next;
        float next_l = 0.f, next_d = 0.f;
        auto load = [&](int k) {
            const int h = kv * w.group + k / per, i0 = (tile0 + k % per) * kTile;
            const int64_t at = b * w.batch_q + h * w.head_q + i0 * w.row_q;
            next.load(Q + at, dO + at, (int)w.row_q, end - i0, d);
            if (threadIdx.x < kTile && i0 + (int)threadIdx.x < end) {
                const size_t row = ((size_t)b * w.heads + h) * w.n + i0 + threadIdx.x;
                next_l = lse[row];
                next_d = delta[row];
            }
        };
        if (begin < stop) load(begin);
        for (int k = begin; k < stop; ++k) {
            const int i0 = (tile0 + k % per) * kTile;
            __syncthreads();
            if (threadIdx.x < kTile) {
                rows_l[threadIdx.x] = next_l * kWindowLog2e;
                rows_d[threadIdx.x] = next_d;
            }
            const int odd = next.store(tq, tg, end - i0, d, &odd_seen);
            if (k + 1 < stop) load(k + 1);
            f4 s[2], t[2];
            score_parts<2, KS, P, P>(tq, Tiles::PLANE, Tiles::PITCH, 0, own, lane, s);
            score_parts<2, KS, P, P>(tg, Tiles::PLANE, Tiles::PITCH, 0, own_v, lane, t);
            float p8[8], w8[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const int r = place(e) + 4 * g;
                p8[e] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[e / 4][e % 4], w.scale2, -rows_l[r]));
                w8[e] = p8[e] * (t[e / 4][e % 4] - rows_d[r]);
            }
            uint32_t seen = 0xffffffffu;                   // the tile's rows that see this key
            if (i0 < j0 + 15 || (i0 + kTile - 1 - j0 >= w.window && j0 + 16 > w.sinks) || i0 + kTile > end || j0 + 15 >= end) {
                seen = j < end ? seen_by(w, j, i0, end) : 0u;
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    if (!(seen >> 4 * g >> place(e) & 1u)) p8[e] = w8[e] = 0.f;
            }
            add_tile<NT, P>(tg, Tiles::PLANE, Tiles::PITCH, p8, acc_v, lane, odd & 2, seen);
            add_tile<NT, P>(tq, Tiles::PLANE, Tiles::PITCH, w8, acc_k, lane, odd & 1, seen);
        }
    }
    if (j >= w.n) return;
    if (walk.parts > 1) {
        float *to = room + (((size_t)blockIdx.y * walks.few + walk.group) * walk.parts + walk.part) * 2 * kRows * d + (size_t)own_at * d;
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            store_piece(to, 16 * t + 4 * g, d, 1, acc_k[t]);
            store_piece(to + (size_t)kRows * d, 16 * t + 4 * g, d, 1, acc_v[t]);
        }
        return;
    }
#pragma unroll
    for (int t = 0; t < NT; ++t) {
        store_piece(dK + at_k + j * w.row_k, 16 * t + 4 * g, d, 1, acc_k[t] * w.scale);
        store_piece(dV + at_k + j * w.row_k, 16 * t + 4 * g, d, 1, acc_v[t]);
    }
}

// The shares of the first tokens' gradients added in order: a thread four columns of a row.
__global__ __launch_bounds__(256) void window_parts_share_kernel(float *dK, float *dV, const float *room, Window w, KeyWalks walks)
{
    const int pieces = w.d / 4, rows = walks.few * kRows;
    const int at = blockIdx.x * 256 + threadIdx.x, row = at / pieces, c = 4 * (at - row * pieces);
    const int b = blockIdx.y / w.kv_heads, kv = blockIdx.y % w.kv_heads;
    if (row >= rows || row >= w.n) return;
    const float *from = room + ((size_t)blockIdx.y * walks.few + row / kRows) * walks.parts * 2 * kRows * w.d + (size_t)(row % kRows) * w.d + c;
    f4 k = {0.f, 0.f, 0.f, 0.f}, v = k;
#pragma unroll 4
    for (int p = 0; p < walks.parts; ++p) {
        k += load4(from + (size_t)p * 2 * kRows * w.d);
        v += load4(from + ((size_t)p * 2 + 1) * kRows * w.d);
    }
    const int64_t to = b * w.batch_k + kv * w.head_k + row * w.row_k + c;
    store4(dK + to, k * w.scale);
    store4(dV + to, v);
}

// go(width, a value of the storage type)
template <class F>
psf_status with_kind(const Window &w, F &&go)
{
    if (w.bf16) return w.d <= 64 ? go(std::integral_constant<int, 4>{}, bf16_t{}) : go(std::integral_constant<int, 8>{}, bf16_t{});
    return w.d <= 64 ? go(std::integral_constant<int, 4>{}, 0.f) : go(std::integral_constant<int, 8>{}, 0.f);
}

}  // namespace

psf_status window_parts_fwd(const Window &w, const WindowPtrs &p, void *O, float *lse, hipStream_t s)
{
    return with_kind(w, [&](auto nt, auto value) -> psf_status {
        constexpr int NT = decltype(nt)::value;
        typedef decltype(value) S;
        hipLaunchKernelGGL((window_parts_fwd_kernel<NT, S>), dim3((w.n + kRows - 1) / kRows, w.batch * w.heads), dim3(256), 0, s,
                           (const S *)p.Q, (const S *)p.K, (const S *)p.V, p.lengths, (S *)O, lse, w);
        PSF_LAUNCH_CHECK();
        return PSF_OK;
    });
}

size_t window_parts_room(const Window &w) { return key_walks_room(w, key_walks(w, kRows, kTile), kRows); }

psf_status window_parts_bwd(const Window &w, const WindowPtrs &p, hipStream_t s)
{
    return with_kind(w, [&](auto nt, auto value) -> psf_status {
        constexpr int NT = decltype(nt)::value;
        typedef decltype(value) S;
        const unsigned tiles = (w.n + kRows - 1) / kRows;
        if (w.bf16)
            if (const psf_status st = window_bf16_delta(w, p, true, s); st != PSF_OK) return st;
        hipLaunchKernelGGL((window_parts_dq_kernel<NT, S>), dim3(tiles, w.batch * w.heads), dim3(256), 0, s, (const S *)p.Q,
                           (const S *)p.K, (const S *)p.V, (const S *)p.O, (const S *)p.dO, p.lengths, p.lse, p.delta, (S *)p.dQ, w);
        PSF_LAUNCH_CHECK();
        const KeyWalks walks = key_walks(w, kRows, kTile);
        const unsigned units = w.batch * w.kv_heads;
        hipLaunchKernelGGL((window_parts_dkv_kernel<NT, S>), dim3(walks.each(), units), dim3(256), 0, s, (const S *)p.Q,
                           (const S *)p.K, (const S *)p.V, (const S *)p.dO, p.lengths, p.lse, p.delta, (S *)p.dK, (S *)p.dV,
                           p.room, w, walks);
        PSF_LAUNCH_CHECK();
        if constexpr (std::is_same_v<S, float>) {          // (walks of short calls are whole)
            if (walks.parts == 1) return PSF_OK;
            hipLaunchKernelGGL(window_parts_share_kernel, dim3((walks.few * kRows * (w.d / 4) + 255) / 256, units), dim3(256), 0, s,
                               (S *)p.dK, (S *)p.dV, p.room, w, walks);
            PSF_LAUNCH_CHECK();
        }
        return PSF_OK;
    });
}

}  // namespace psf
