// Window attention in bf16 storage on the 32 x 32 x 16 products.
//
// A wave owns 32 rows as the columns of its results -- queries in the forward pass and for dQ, keys for dK and dV --, so
// that a row's scores, weights and sums stay in its two lanes and the weights of a tile, rounded to bf16, are
// the next product's operand as they stand.  Tiles of the other side (64 rows of both its tensors) are copied to
// LDS as they lie, two of them in turn, the next one on its way while this one is worked on; they are read along
// their rows for the scores and transposed for the sums (psf_lds.h).
#include "psf_lds.h"
#include "psf_window.h"

namespace psf {
namespace {

constexpr int kThreads = 256, kWaves = 4;
constexpr int kOwn = 32;                   // rows of a wave
constexpr int kOwnWg = kOwn * kWaves;      // of a workgroup
constexpr int kTile = 64;                  // rows of a tile
constexpr float kLazy = 8.0f;              // a maximum is left as it is until one above it by 2^8 comes

// A tile of rows of two tensors (keys and values, or queries and output gradients), copied by the workgroup.
template <int D, int TILE = kTile>
struct Staged {
    static constexpr int BYTES = TILE * D * 2, COPIES = BYTES / (kThreads * 16), ROWS = kThreads * 8 / D;   // rows a copy
    uint32_t wave_at, lane_row, lane_piece, step;          // LDS address of the wave's pieces; row, byte offset of the piece
    __device__ __forceinline__ Staged(const void *lds, int d)
    {
        wave_at = lds_address(lds) + (threadIdx.x >> 6) * 1024;
        lane_row = threadIdx.x / (D / 8);
        uint32_t piece = threadIdx.x % (D / 8) ^ row_swz<D>((int)lane_row);
        if (D != 64 || d != 64) piece = piece < (uint32_t)d / 8 ? piece : 0;   // (columns that are not there: any)
        lane_piece = piece * 16;
        step = 0;
    }
    // rows j0 .. of x and y (rows of `ld` values; those from `end` on: row end - 1 instead), to buffer `buf`
    __device__ __forceinline__ void copy(const bf16_t *x, const bf16_t *y, int64_t ld, int j0, int end, int buf) const
    {
        const bf16_t *at_x = x + j0 * ld, *at_y = y + j0 * ld;
        const uint32_t to = wave_at + (uint32_t)buf * 2 * BYTES, pitch = (uint32_t)ld * 2;
        const int left = end - j0 - 1;
#pragma unroll
        for (int q = 0; q < COPIES; ++q) {
            const int row = (int)lane_row + q * ROWS;
            const uint32_t off = (uint32_t)(row < left ? row : left) * pitch + lane_piece;
            dma16_sbase(at_x, off, to + q * (kThreads * 16));
            dma16_sbase(at_y, off, to + BYTES + q * (kThreads * 16));
        }
    }
};

// This lane's reads of a staged tile: operand A along the rows (row 32 t + lane % 32, piece 2 s + lane / 32), and
// transposed (columns 32 ct + lane % 32, rows 16 s + {4 h .. 4 h + 3, 8 + 4 h ..}, h = lane / 32).
template <int D>
struct Reads {
    uint32_t along[D / 16], turned[2][D / 32];
    __device__ __forceinline__ Reads(int lane)
    {
        const int x = lane & 31, h = lane >> 5;
#pragma unroll
        for (int s = 0; s < D / 16; ++s) along[s] = (uint32_t)((x * (D / 8) + ((2 * s + h) ^ row_swz<D>(x))) * 16);
#pragma unroll
        for (int e = 0; e < 2; ++e)
#pragma unroll
            for (int ct = 0; ct < D / 32; ++ct) turned[e][ct] = row_turned_offset<D>(lane, 8 * e + 4 * h, ct);
    }
    __device__ __forceinline__ bf16x8 row(const unsigned char *tile, int t, int s) const
    {
        return *(const bf16x8 *)(tile + along[s] + t * (32 * D * 2));
    }
    __device__ __forceinline__ bf16x8 column(const unsigned char *tile, int ct, int s) const
    {
        return read_turned(tile + turned[0][ct] + s * (16 * D * 2), tile + turned[1][ct] + s * (16 * D * 2));
    }
};

// A row as operand B: columns 16 s + 8 h .. of it (zero from d on), with the sign of `scale` (a query's scores are multiplied by
// |scale|, which leaves their order and a masked one's -inf as they are; scale 0: a row of zeros, by 1)
template <int D>
__device__ __forceinline__ void own_row(const bf16_t *row, int d, int h, float scale, bf16x8 (&f)[D / 16])
{
    typedef uint32_t u4 __attribute__((ext_vector_type(4)));
#pragma unroll
    for (int s = 0; s < D / 16; ++s) {
        u4 v = {0u, 0u, 0u, 0u};
        if (16 * s + 8 * h < d) v = *(const u4 *)(row + 16 * s + 8 * h);
        if (scale == 0.f) v = u4{0u, 0u, 0u, 0u};
        if (scale < 0.f) v ^= 0x80008000u;
        f[s] = __builtin_bit_cast(bf16x8, v);
    }
}

__device__ __forceinline__ float other_half(float x, bool take_max)
{
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    const float a = __uint_as_float(r[0]), b = __uint_as_float(r[1]);
    return take_max ? fmaxf(a, b) : a + b;
}

// scores of a tile's 32 rows (half t) with the wave's own rows
template <int D>
__device__ __forceinline__ f32x16 scores(const Reads<D> &at, const unsigned char *tile, int t, const bf16x8 (&own)[D / 16])
{
    f32x16 c = {0};
#pragma unroll
    for (int s = 0; s < D / 16; ++s) c = mfma32(at.row(tile, t, s), own[s], c);
    return c;
}
// acc += tile^T w: the tile's rows 32 t .. with weights w (as results hold them), columns of the tile as rows of acc
template <int D>
__device__ __forceinline__ void add_turned(const Reads<D> &at, const unsigned char *tile, int t, const f32x16 &w,
                                           f32x16 (&acc)[D / 32])
{
#pragma unroll
    for (int s = 0; s < 2; ++s) {
        const bf16x8 b = cvt8_from16(w, 8 * s);
#pragma unroll
        for (int ct = 0; ct < D / 32; ++ct) acc[ct] = mfma32(at.column(tile, ct, 2 * t + s), b, acc[ct]);
    }
}

// place in its 32 rows of element e of a result
__device__ __forceinline__ int place(int e, int h) { return 8 * (e / 4) + 4 * h + e % 4; }

// Whether rows [i0, i0 + 31] see all / none of keys [j0, j0 + len - 1].
__device__ __forceinline__ bool all_seen(const Window &w, int i0, int j0, int len)
{
    return j0 + len - 1 <= i0 && (i0 + kOwn - 1 - j0 < w.window || j0 + len <= w.sinks);
}
__device__ __forceinline__ bool none_seen(const Window &w, int i0, int j0, int len)
{
    return j0 > i0 + kOwn - 1 || (i0 - (j0 + len - 1) >= w.window && j0 >= w.sinks);
}

// Which workgroup of the call (unit by unit, neighbouring rows side by side) workgroup `id` of the launch is.  The launch
// deals its workgroups out to the 8 XCDs in turn; runs of 16 neighbours stay on one XCD, whose L2 serves the
// tiles that they share, and the runs go round the XCDs, one further every time round, so that neither sequences
// of unequal length nor the long and the short rows of all units meet on the same ones.
__device__ __forceinline__ uint32_t place_of(uint32_t id, uint32_t total)
{
    constexpr uint32_t RUN = 16;
    if (id >= total / (8 * RUN) * (8 * RUN)) return id;
    const uint32_t slot = id / 8, round = slot / RUN;
    return (round * 8 + (id + round) % 8) * RUN + slot % RUN;
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
// x where bit place(E, h) of the row's bits is set, `other` elsewhere; bits_h: those bits >> 4 h.  (The bit as a mask, by an
// instruction of its own: as a comparison and a select it takes five.)
template <int E>
__device__ __forceinline__ float pick(uint32_t bits_h, float x, uint32_t other)
{
    uint32_t mask;
    asm("v_bfe_i32 %0, %1, %2, 1" : "=v"(mask) : "v"(bits_h), "n"(8 * (E / 4) + E % 4));
    return __uint_as_float((__float_as_uint(x) & mask) | (other & ~mask));
}

// This lane's part of a result row (columns 32 ct + place(e, h)) times `by`, to `row` in storage type; zeros where the row lies
// behind its sequence.  Returns whether it holds an infinity or NaN.  (Columns from d on hold what the tile's
// columns there held, which are the row's first ones again: no others that are odd.)
template <int D>
__device__ __forceinline__ bool store_row(const f32x16 (&acc)[D / 32], float by, bool there, bf16_t *row, int d, int h)
{
    typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
    typedef float f32x4 __attribute__((ext_vector_type(4)));
    float probe = 0.f;
#pragma unroll
    for (int ct = 0; ct < D / 32; ++ct)
#pragma unroll
        for (int e = 0; e < 16; e += 4) {
            f32x4 v;
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                v[k] = there ? acc[ct][e + k] * by : 0.f;
                probe = __builtin_fmaf(v[k], 0.f, probe);
            }
            const int col = 32 * ct + 2 * e + 4 * h;
            if (col < d) *(bf16x4 *)(row + col) = __builtin_convertvector(v, bf16x4);
        }
    return probe != 0.f;
}

// Row i again, pair by pair in fp32 and without a masked pair: for rows whose result is not finite, so that an infinity
// or NaN of a token that the row does not see leaves nothing in it (0 * inf in a tile's product).
template <int D>
__device__ __forceinline__ void fwd_row_again(const Window &w, const bf16_t *q, const bf16_t *K, const bf16_t *V, bf16_t *o, int i)
{
    const int lane = threadIdx.x & 63;
    float top = -INFINITY, sum = 0.f, acc[D / 64];
#pragma unroll
    for (int k = 0; k < D / 64; ++k) acc[k] = 0.f;
    const KeyTiles tiles(w, i, i, 64);
    for (int k = 0; k < tiles.total; ++k) {
        const int j = tiles.at(k) * 64 + lane;
        const bool seen = window_sees(w, i, j);
        float s = 0.f;
        if (seen)
            for (int c = 0; c < w.d; ++c) s += bf16_to_f32(q[c]) * bf16_to_f32(K[j * w.row_k + c]);
        s = seen ? s * w.scale2 : -INFINITY;
        float most = s;
#pragma unroll
        for (int m = 1; m < 64; m <<= 1) most = fmaxf(most, __shfl_xor(most, m));
        most = fmaxf(most, top);
        const float less = top == -INFINITY ? 0.f : exp2f(top - most), p = seen ? exp2f(s - (most == -INFINITY ? 0.f : most)) : 0.f;
        top = most;
        float all = p;
#pragma unroll
        for (int m = 1; m < 64; m <<= 1) all += __shfl_xor(all, m);
        sum = sum * less + all;
#pragma unroll
        for (int c = 0; c < D / 64; ++c) acc[c] *= less;
        for (uint64_t bits = __ballot(seen); bits; bits &= bits - 1) {
            const int from = __ffsll((long long)bits) - 1;
            const float pj = __shfl(p, from);
            const bf16_t *row = V + (tiles.at(k) * 64 + from) * w.row_k;
#pragma unroll
            for (int c = 0; c < D / 64; ++c)
                if (64 * c + lane < w.d) acc[c] += pj * bf16_to_f32(row[64 * c + lane]);
        }
    }
#pragma unroll
    for (int c = 0; c < D / 64; ++c)
        if (64 * c + lane < w.d) o[64 * c + lane] = f32_to_bf16(acc[c] / sum);
}

template <int D>
__global__ __launch_bounds__(kThreads, 2) void window_fwd_kernel(const bf16_t *Q, const bf16_t *K, const bf16_t *V,
                                                                 const int32_t *lengths, bf16_t *O, float *lse, Window w,
                                                                 uint32_t groups)
{
    constexpr int KS = D / 16, CT = D / 32;
    using Tile = Staged<D>;
    __shared__ __align__(1024) unsigned char lds[2 * 2 * Tile::BYTES];
    const int lane = threadIdx.x & 63, x = lane & 31, h = lane >> 5, d = w.d;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);      // (in a scalar register: which tiles count is the wave's)
    const uint32_t at_grid = place_of(blockIdx.x, gridDim.x), unit = at_grid / groups;
    const int first = (int)(groups - 1 - (at_grid - unit * groups)) * kOwnWg;      // long rows first
    const int b = unit / w.heads, head = unit - b * w.heads;
    const int end = window_end(lengths, b, w.n), i0 = first + kOwn * wave, i = i0 + x;
    const bf16_t *q = Q + b * w.batch_q + head * w.head_q;
    const int64_t at_k = b * w.batch_k + head / w.group * w.head_k;
    const bf16_t *k_rows = K + at_k, *v_rows = V + at_k;
    f32x16 acc[CT];
#pragma unroll
    for (int ct = 0; ct < CT; ++ct) acc[ct] = f32x16{0};
    float top = -INFINITY, sum = 0.f;                      // top: in units of the scaled scores (exponents of 2)
    const float c = w.scale2 == 0.f ? 1.f : fabsf(w.scale2);
    if (first < end) {                                     // (the same in the whole workgroup)
        bf16x8 own[KS];
        own_row<D>(q + (i < end ? i : end - 1) * w.row_q, d, h, w.scale2, own);
        const int last = first + kOwnWg < end ? first + kOwnWg - 1 : end - 1;
        const KeyTiles tiles(w, first, last, kTile);
        const Tile stage(lds, d);
        const Reads<D> at(lane);
        stage.copy(k_rows, v_rows, w.row_k, tiles.at(0) * kTile, end, 0);
        for (int k = 0; k < tiles.total; ++k) {
            const int j0 = tiles.at(k) * kTile;
            wait_all_memory();                             // this wave's pieces of the tile, and its reads of the last one
            __builtin_amdgcn_s_barrier();
            asm volatile("" ::: "memory");
            if (k + 1 < tiles.total) stage.copy(k_rows, v_rows, w.row_k, tiles.at(k + 1) * kTile, end, (k + 1) & 1);
            if (none_seen(w, i0, j0, kTile)) continue;
            const unsigned char *tk = lds + (k & 1) * 2 * Tile::BYTES, *tv = tk + Tile::BYTES;
            f32x16 s[2];
#pragma unroll
            for (int t = 0; t < 2; ++t) s[t] = scores<D>(at, tk, t, own);
            if (!all_seen(w, i0, j0, kTile)) {
#pragma unroll
                for (int t = 0; t < 2; ++t) {
                    const uint32_t bits = seen_keys(w, i, j0 + 32 * t) >> (4 * h);
                    static_for<16>([&](auto e) { s[t][int(e)] = pick<e>(bits, s[t][int(e)], 0xff800000u); });   // -inf
                }
            }
            float most = s[0][0];
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int e = 0; e < 16; ++e) most = fmaxf(most, s[t][e]);
            most = other_half(most, true) * c;
            if (__any(most > top + kLazy)) {
                const float next = fmaxf(top, most), less = top == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(top - next);
                sum *= less;
#pragma unroll
                for (int ct = 0; ct < CT; ++ct) acc[ct] *= less;
                top = next;
            }
            const float base = top == -INFINITY ? 0.f : top;
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    s[t][e] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[t][e], c, -base));
                    sum += s[t][e];
                }
#pragma unroll
            for (int t = 0; t < 2; ++t) add_turned<D>(at, tv, t, s[t], acc);
            branch_wait();
        }
    }
    sum = other_half(sum, false);
    const bool there = i < end;
    bf16_t *o = O + b * w.batch_q + head * w.head_q;
    bool odd = false;
    if (i < w.n) {
        odd = store_row<D>(acc, 1.f / sum, there, o + i * w.row_q, d, h);
        if (lse && h == 0)
            lse[((size_t)b * w.heads + head) * w.n + i] = there ? (top + __builtin_log2f(sum)) * kWindowLn2 : -INFINITY;
    }
    const uint64_t which = __ballot(odd);
    for (uint32_t rows = (uint32_t)which | (uint32_t)(which >> 32); rows; rows &= rows - 1) {
        const int r = i0 + __ffs((int)rows) - 1;
        fwd_row_again<D>(w, q + r * w.row_q, k_rows, v_rows, o + r * w.row_q, r);
    }
}

// ---- backward ---------------------------------------------------------------------------------

// Row i of dQ again (see fwd_row_again).
template <int D>
__device__ __forceinline__ void dq_row_again(const Window &w, const bf16_t *q, const bf16_t *g, const bf16_t *K, const bf16_t *V,
                                             float L, float dot, bf16_t *dq, int i)
{
    const int lane = threadIdx.x & 63;
    float acc[D / 64];
#pragma unroll
    for (int k = 0; k < D / 64; ++k) acc[k] = 0.f;
    const KeyTiles tiles(w, i, i, 64);
    for (int k = 0; k < tiles.total; ++k) {
        const int j = tiles.at(k) * 64 + lane;
        const bool seen = window_sees(w, i, j);
        float s = 0.f, t = 0.f;
        if (seen)
            for (int c = 0; c < w.d; ++c) {
                s += bf16_to_f32(q[c]) * bf16_to_f32(K[j * w.row_k + c]);
                t += bf16_to_f32(g[c]) * bf16_to_f32(V[j * w.row_k + c]);
            }
        const float ds = exp2f(s * w.scale2 - L) * (t - dot);
        for (uint64_t bits = __ballot(seen); bits; bits &= bits - 1) {
            const int from = __ffsll((long long)bits) - 1;
            const float by = __shfl(ds, from);
            const bf16_t *row = K + (tiles.at(k) * 64 + from) * w.row_k;
#pragma unroll
            for (int c = 0; c < D / 64; ++c)
                if (64 * c + lane < w.d) acc[c] += by * bf16_to_f32(row[64 * c + lane]);
        }
    }
#pragma unroll
    for (int c = 0; c < D / 64; ++c)
        if (64 * c + lane < w.d) dq[64 * c + lane] = f32_to_bf16(acc[c] * w.scale);
}

// Row j of dK and dV again.  Q, dO, lse, delta: of the first query head of the key head in this batch.
template <int D>
__device__ __forceinline__ void dkv_row_again(const Window &w, const bf16_t *k, const bf16_t *v, const bf16_t *Q, const bf16_t *dO,
                                              const float *lse, const float *delta, int end, bf16_t *dk, bf16_t *dv, int j)
{
    const int lane = threadIdx.x & 63;
    float acc_k[D / 64], acc_v[D / 64];
#pragma unroll
    for (int c = 0; c < D / 64; ++c) acc_k[c] = acc_v[c] = 0.f;
    const int64_t reach = j < w.sinks ? (int64_t)end : (int64_t)j + w.window;
    const int stop = reach < end ? (int)reach : end;
    for (int head = 0; head < w.group; ++head)
        for (int at = j; at < stop; at += 64) {
            const int i = at + lane;
            const bool seen = i < stop;
            float s = 0.f, t = 0.f, p = 0.f, ds = 0.f;
            if (seen) {
                const int64_t row = head * w.head_q + i * w.row_q;
                for (int c = 0; c < w.d; ++c) {
                    s += bf16_to_f32(Q[row + c]) * bf16_to_f32(k[c]);
                    t += bf16_to_f32(dO[row + c]) * bf16_to_f32(v[c]);
                }
                p = exp2f(s * w.scale2 - lse[(size_t)head * w.n + i] * kWindowLog2e);
                ds = p * (t - delta[(size_t)head * w.n + i]);
            }
            for (uint64_t bits = __ballot(seen); bits; bits &= bits - 1) {
                const int from = __ffsll((long long)bits) - 1;
                const float by_k = __shfl(ds, from), by_v = __shfl(p, from);
                const int64_t row = head * w.head_q + (at + from) * w.row_q;
#pragma unroll
                for (int c = 0; c < D / 64; ++c)
                    if (64 * c + lane < w.d) {
                        acc_k[c] += by_k * bf16_to_f32(Q[row + 64 * c + lane]);
                        acc_v[c] += by_v * bf16_to_f32(dO[row + 64 * c + lane]);
                    }
            }
        }
#pragma unroll
    for (int c = 0; c < D / 64; ++c)
        if (64 * c + lane < w.d) {
            dk[64 * c + lane] = f32_to_bf16(acc_k[c] * w.scale);
            dv[64 * c + lane] = f32_to_bf16(acc_v[c]);
        }
}

// dQ, and D = <dO, o> of every row for the kernel below.
template <int D>
__global__ __launch_bounds__(kThreads, 2) void window_dq_kernel(const bf16_t *Q, const bf16_t *K, const bf16_t *V,
                                                                const int32_t *lengths, const bf16_t *O, const float *lse,
                                                                const bf16_t *dO, bf16_t *dQ, float *delta, Window w,
                                                                uint32_t groups)
{
    constexpr int KS = D / 16, CT = D / 32;
    using Tile = Staged<D>;
    __shared__ __align__(1024) unsigned char lds[2 * 2 * Tile::BYTES];
    const int lane = threadIdx.x & 63, x = lane & 31, h = lane >> 5, d = w.d;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);      // (in a scalar register: which tiles count is the wave's)
    const uint32_t at_grid = place_of(blockIdx.x, gridDim.x), unit = at_grid / groups;
    const int first = (int)(groups - 1 - (at_grid - unit * groups)) * kOwnWg;
    const int b = unit / w.heads, head = unit - b * w.heads;
    const int end = window_end(lengths, b, w.n), i0 = first + kOwn * wave, i = i0 + x;
    const int64_t at_q = b * w.batch_q + head * w.head_q, at_k = b * w.batch_k + head / w.group * w.head_k;
    const bf16_t *k_rows = K + at_k, *v_rows = V + at_k;
    f32x16 acc[CT];
#pragma unroll
    for (int ct = 0; ct < CT; ++ct) acc[ct] = f32x16{0};
    float L = 0.f, dot = 0.f;
    const float c = w.scale2 == 0.f ? 1.f : fabsf(w.scale2);
    if (first < end) {
        const int safe = i < end ? i : end - 1;
        const int last = first + kOwnWg < end ? first + kOwnWg - 1 : end - 1;
        const KeyTiles tiles(w, first, last, kTile);
        const Tile stage(lds, d);
        stage.copy(k_rows, v_rows, w.row_k, tiles.at(0) * kTile, end, 0);
        bf16x8 own[KS], own_g[KS];
        own_row<D>(Q + at_q + safe * w.row_q, d, h, w.scale2, own);
        own_row<D>(dO + at_q + safe * w.row_q, d, h, 1.f, own_g);
        {
            bf16x8 o[KS];
            own_row<D>(O + at_q + safe * w.row_q, d, h, 1.f, o);
#pragma unroll
            for (int s = 0; s < KS; ++s)
#pragma unroll
                for (int e = 0; e < 8; ++e) dot += (float)o[s][e] * (float)own_g[s][e];
        }
        dot = other_half(dot, false);
        const size_t row = ((size_t)b * w.heads + head) * w.n + safe;
        L = lse[row] * kWindowLog2e;
        if (i < end && h == 0) delta[row] = dot;
        const Reads<D> at(lane);
        for (int k = 0; k < tiles.total; ++k) {
            const int j0 = tiles.at(k) * kTile;
            wait_all_memory();
            __builtin_amdgcn_s_barrier();
            asm volatile("" ::: "memory");
            if (k + 1 < tiles.total) stage.copy(k_rows, v_rows, w.row_k, tiles.at(k + 1) * kTile, end, (k + 1) & 1);
            if (none_seen(w, i0, j0, kTile)) continue;
            const unsigned char *tk = lds + (k & 1) * 2 * Tile::BYTES, *tv = tk + Tile::BYTES;
            const bool all = all_seen(w, i0, j0, kTile);
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                f32x16 s = scores<D>(at, tk, t, own);
                const f32x16 u = scores<D>(at, tv, t, own_g);
#pragma unroll
                for (int e = 0; e < 16; ++e) s[e] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[e], c, -L)) * (u[e] - dot);
                if (!all) {
                    const uint32_t bits = seen_keys(w, i, j0 + 32 * t) >> (4 * h);
                    static_for<16>([&](auto e) { s[int(e)] = pick<e>(bits, s[int(e)], 0u); });
                }
                add_turned<D>(at, tk, t, s, acc);
            }
            branch_wait();
        }
    }
    bool odd = false;
    if (i < w.n) odd = store_row<D>(acc, w.scale, i < end, dQ + at_q + i * w.row_q, d, h);
    const uint64_t which = __ballot(odd);
    for (uint32_t rows = (uint32_t)which | (uint32_t)(which >> 32); rows; rows &= rows - 1) {
        const int at = __ffs((int)rows) - 1, r = i0 + at;
        const int64_t row = at_q + r * w.row_q;
        dq_row_again<D>(w, Q + row, dO + row, k_rows, v_rows, __shfl(L, at), __shfl(dot, at), dQ + row, r);
    }
}

template <int D>
__global__ __launch_bounds__(kThreads, 2) void window_dkv_kernel(
    const bf16_t *Q, const bf16_t *K, const bf16_t *V, const int32_t *lengths, const float *lse, const bf16_t *dO,
    const float *delta, bf16_t *dK, bf16_t *dV, float *room, Window w, KeyWalks walks)
{
    constexpr int KS = D / 16, CT = D / 32, TILE = D == 64 ? 64 : 32;
    constexpr bool V_IN_LDS = D == 128;
    using Tile = Staged<D, TILE>;
    __shared__ __align__(1024) unsigned char lds[2 * 2 * Tile::BYTES + (V_IN_LDS ? kOwnWg * D * 2 : 0)];
    __shared__ float2 row_data[2][TILE];                  // L (in exponents of 2) and D of the tile's rows
    const int lane = threadIdx.x & 63, x = lane & 31, h = lane >> 5, d = w.d;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);      // (in a scalar register: which tiles count is the wave's)
    const uint32_t at_grid = place_of(blockIdx.x, gridDim.x), each = walks.each(), unit = at_grid / each;
    const KeyWalk walk(walks, at_grid - unit * each);
    const int group = walk.group, part = walk.part, parts = walk.parts;
    const int first = group * kOwnWg;
    const int b = unit / w.kv_heads, kv = unit - b * w.kv_heads;
    const int end = window_end(lengths, b, w.n), j0 = first + kOwn * wave, j = j0 + x;
    const int64_t at_k = b * w.batch_k + kv * w.head_k, at_q = b * w.batch_q + (int64_t)kv * w.group * w.head_q;
    const size_t at_rows = ((size_t)b * w.heads + kv * w.group) * w.n;
    const float c = w.scale2 == 0.f ? 1.f : fabsf(w.scale2);
    f32x16 acc_k[CT], acc_v[CT];
#pragma unroll
    for (int ct = 0; ct < CT; ++ct) acc_k[ct] = acc_v[ct] = f32x16{0};
    if (first < end) {
        const QueryTiles tiles(w, first, end, kOwnWg, TILE);
        const int total = tiles.count * w.group, begin = (int)((int64_t)total * part / parts),
                  stop = (int)((int64_t)total * (part + 1) / parts);
        const Tile stage(lds, d);
        float2 next = make_float2(0.f, 0.f);
        int head = begin / tiles.count, tile = begin - head * tiles.count;     // of the next copy
        auto copy = [&](int buf) {
            const int i0 = (tiles.tile0 + tile) * TILE;
            stage.copy(Q + at_q + head * w.head_q, dO + at_q + head * w.head_q, w.row_q, i0, end, buf);
            if (threadIdx.x < TILE) {
                const size_t row = at_rows + (size_t)head * w.n + (i0 + (int)threadIdx.x < end ? i0 + (int)threadIdx.x : end - 1);
                next = make_float2(lse[row] * kWindowLog2e, delta[row]);
            }
            if (++tile == tiles.count) {
                tile = 0;
                ++head;
            }
        };
        int now = tile;
        if (begin < stop) copy(0);
        const Reads<D> at(lane);
        bf16x8 own[KS], own_v[V_IN_LDS ? 1 : KS];
        own_row<D>(K + at_k + (j < end ? j : end - 1) * w.row_k, d, h, w.scale2, own);
        unsigned char *wave_v = lds + 2 * 2 * Tile::BYTES + wave * (kOwn * D * 2);
        if constexpr (V_IN_LDS) {
            bf16x8 v[KS];
            own_row<D>(V + at_k + (j < end ? j : end - 1) * w.row_k, d, h, 1.f, v);
#pragma unroll
            for (int s = 0; s < KS; ++s) *(bf16x8 *)(wave_v + at.along[s]) = v[s];   // (read by this wave alone)
        } else own_row<D>(V + at_k + (j < end ? j : end - 1) * w.row_k, d, h, 1.f, own_v);
        for (int k = begin; k < stop; ++k) {
            const int buf = (k - begin) & 1, i0 = (tiles.tile0 + now) * TILE;
            now = tile;
            wait_all_memory();
            if (threadIdx.x < TILE) row_data[buf][threadIdx.x] = next;
            __syncthreads();
            if (k + 1 < stop) copy(buf ^ 1);
            // (rows behind the sequence are the last one again: masked)
            const bool none = i0 + TILE - 1 < j0 || (i0 - (j0 + kOwn - 1) >= w.window && j0 >= w.sinks);
            if (none) continue;
            const bool all = i0 >= j0 + kOwn - 1 && (i0 + TILE - 1 - j0 < w.window || j0 + kOwn <= w.sinks) && i0 + TILE <= end;
            const unsigned char *tq = lds + buf * 2 * Tile::BYTES, *tg = tq + Tile::BYTES;
#pragma unroll
            for (int t = 0; t < TILE / 32; ++t) {
                f32x16 s = scores<D>(at, tq, t, own);
                f32x16 u = {0};
#pragma unroll
                for (int q = 0; q < KS; ++q) {
                    if constexpr (V_IN_LDS) u = mfma32(at.row(tg, t, q), at.row(wave_v, 0, q), u);
                    else u = mfma32(at.row(tg, t, q), own_v[q], u);
                }
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    const float2 r = row_data[buf][32 * t + place(e, h)];
                    s[e] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[e], c, -r.x));
                    u[e] = s[e] * (u[e] - r.y);
                }
                if (!all) {
                    const uint32_t bits = seen_by(w, j, i0 + 32 * t, end) >> (4 * h);
                    static_for<16>([&](auto e) {
                        s[int(e)] = pick<e>(bits, s[int(e)], 0u);
                        u[int(e)] = pick<e>(bits, u[int(e)], 0u);
                    });
                }
                add_turned<D>(at, tg, t, s, acc_v);
                add_turned<D>(at, tq, t, u, acc_k);
            }
            branch_wait();
        }
    }
    if (parts > 1) {                                       // a share: [unit][group][part][dK, dV][128][d], added below
        if (j >= w.n) return;
        float *to = room + (((size_t)unit * walks.few + group) * parts + part) * 2 * kOwnWg * d + (size_t)(kOwn * wave + x) * d;
#pragma unroll
        for (int ct = 0; ct < CT; ++ct)
#pragma unroll
            for (int e = 0; e < 16; e += 4) {
                const int col = 32 * ct + place(e, h);
                if (col < d) {
                    *(float4 *)(to + col) = make_float4(acc_k[ct][e], acc_k[ct][e + 1], acc_k[ct][e + 2], acc_k[ct][e + 3]);
                    *(float4 *)(to + (size_t)kOwnWg * d + col) =
                        make_float4(acc_v[ct][e], acc_v[ct][e + 1], acc_v[ct][e + 2], acc_v[ct][e + 3]);
                }
            }
        return;
    }
    bool odd = false;
    if (j < w.n) {
        odd = store_row<D>(acc_k, w.scale, j < end, dK + at_k + j * w.row_k, d, h);
        odd |= store_row<D>(acc_v, 1.f, j < end, dV + at_k + j * w.row_k, d, h);
    }
    const uint64_t bad = __ballot(odd);
    for (uint32_t rows = (uint32_t)bad | (uint32_t)(bad >> 32); rows; rows &= rows - 1) {
        const int r = j0 + __ffs((int)rows) - 1;
        const int64_t row = at_k + r * w.row_k;
        dkv_row_again<D>(w, K + row, V + row, Q + at_q, dO + at_q, lse + at_rows, delta + at_rows, end, dK + row, dV + row, r);
    }
}

// The shares of the first tokens' gradients added in order: a wave a row of 128, lanes are columns.
template <int D>
__global__ __launch_bounds__(kThreads) void window_share_kernel(const bf16_t *Q, const bf16_t *K, const bf16_t *V,
                                                                const int32_t *lengths, const float *lse, const bf16_t *dO,
                                                                const float *delta, bf16_t *dK, bf16_t *dV, const float *room,
                                                                Window w, KeyWalks walks)
{
    const int lane = threadIdx.x & 63, d = w.d;
    const uint32_t row = blockIdx.x * kWaves + (threadIdx.x >> 6), block = row / kOwnWg;
    const int in_block = row % kOwnWg, unit = block / walks.few, group = block - unit * walks.few, j = group * kOwnWg + in_block;
    const int b = unit / w.kv_heads, kv = unit - b * w.kv_heads;
    if (j >= w.n) return;
    const int end = window_end(lengths, b, w.n);
    const int64_t at_k = b * w.batch_k + kv * w.head_k, at_q = b * w.batch_q + (int64_t)kv * w.group * w.head_q, to = at_k + j * w.row_k;
    const size_t at_rows = ((size_t)b * w.heads + kv * w.group) * w.n;
    const float *from = room + (size_t)block * walks.parts * 2 * kOwnWg * d + (size_t)in_block * d;
    bool odd = false;
#pragma unroll
    for (int c = 0; c < D / 64; ++c) {
        const int col = 64 * c + lane;
        float k = 0.f, v = 0.f;
        if (col < d && j < end) {
#pragma unroll 4
            for (int p = 0; p < walks.parts; ++p) {
                k += from[(size_t)p * 2 * kOwnWg * d + col];
                v += from[(size_t)p * 2 * kOwnWg * d + (size_t)kOwnWg * d + col];
            }
            k *= w.scale;
            odd |= !(fabsf(k) < INFINITY) || !(fabsf(v) < INFINITY);
        }
        if (col < d) {
            dK[to + col] = f32_to_bf16(k);
            dV[to + col] = f32_to_bf16(v);
        }
    }
    if (__any(odd)) dkv_row_again<D>(w, K + to, V + to, Q + at_q, dO + at_q, lse + at_rows, delta + at_rows, end, dK + to, dV + to, j);
}

KeyWalks walks_of(const Window &w) { return key_walks(w, kOwnWg, w.d <= 64 ? 64 : 32); }

}  // namespace

psf_status window_bf16_fwd(const Window &w, const WindowPtrs &p, void *O, float *lse, hipStream_t s)
{
    const uint32_t groups = (w.n + kOwnWg - 1) / kOwnWg, all = groups * w.batch * w.heads;
    auto go = [&](auto width) -> psf_status {
        constexpr int D = decltype(width)::value;
        hipLaunchKernelGGL((window_fwd_kernel<D>), dim3(all), dim3(kThreads), 0, s, (const bf16_t *)p.Q, (const bf16_t *)p.K,
                           (const bf16_t *)p.V, p.lengths, (bf16_t *)O, lse, w, groups);
        PSF_LAUNCH_CHECK();
        return PSF_OK;
    };
    return w.d <= 64 ? go(std::integral_constant<int, 64>{}) : go(std::integral_constant<int, 128>{});
}

size_t window_bf16_room(const Window &w)
{
    return key_walks_room(w, walks_of(w), kOwnWg);
}

psf_status window_bf16_bwd(const Window &w, const WindowPtrs &p, hipStream_t s)
{
    auto go = [&](auto width) -> psf_status {
        constexpr int D = decltype(width)::value;
        const bf16_t *Q = (const bf16_t *)p.Q, *K = (const bf16_t *)p.K, *V = (const bf16_t *)p.V, *O = (const bf16_t *)p.O,
                     *dO = (const bf16_t *)p.dO;
        bf16_t *dQ = (bf16_t *)p.dQ, *dK = (bf16_t *)p.dK, *dV = (bf16_t *)p.dV;
        const uint32_t groups = (w.n + kOwnWg - 1) / kOwnWg;
        hipLaunchKernelGGL((window_dq_kernel<D>), dim3(groups * w.batch * w.heads), dim3(kThreads), 0, s, Q, K, V, p.lengths, O, p.lse,
                           dO, dQ, p.delta, w, groups);
        PSF_LAUNCH_CHECK();
        const KeyWalks walks = walks_of(w);
        const uint32_t units = w.batch * w.kv_heads;
        hipLaunchKernelGGL((window_dkv_kernel<D>), dim3(units * walks.each()), dim3(kThreads), 0, s, Q, K, V, p.lengths, p.lse, dO,
                           p.delta, dK, dV, p.room, w, walks);
        PSF_LAUNCH_CHECK();
        if (walks.parts == 1) return PSF_OK;
        hipLaunchKernelGGL((window_share_kernel<D>), dim3(units * walks.few * kOwnWg / kWaves), dim3(kThreads), 0, s, Q, K, V,
                           p.lengths, p.lse, dO, p.delta, dK, dV, p.room, w, walks);
        PSF_LAUNCH_CHECK();
        return PSF_OK;
    };
    return w.d <= 64 ? go(std::integral_constant<int, 64>{}) : go(std::integral_constant<int, 128>{});
}

}  // namespace psf
