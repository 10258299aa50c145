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
    uint32_t wave_at, lane_row, lane_piece;                // LDS address of the wave's pieces; row, byte offset of the piece
    __device__ __forceinline__ Staged(const void *lds, int d)
    {
        wave_at = lds_address(lds) + (threadIdx.x >> 6) * 1024;
        lane_row = threadIdx.x / (D / 8);
        const uint32_t piece = threadIdx.x % (D / 8) ^ row_swz<D>((int)lane_row);
        lane_piece = (piece < (uint32_t)d / 8 ? piece : 0) * 16;               // (columns that are not there: any)
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
// transposed (columns 32 ct + lane % 32, rows 16 s + {4 h .. 4 h + 3, 8 + 4 h ..}, h = lane / 32).  A piece's place in
// its row is its number with bits of the row's flipped, so all places of a tile come from one address by flips of
// constant bits: two registers a tile instead of one for every place.
template <int D>
struct Reads {
    uint32_t along, turned;                                // LDS addresses (tiles start at multiples of 256 bytes)
    __device__ __forceinline__ Reads(int lane)
    {
        const int x = lane & 31, h = lane >> 5;
        along = (uint32_t)((x * (D / 8) + (h ^ row_swz<D>(x))) * 16);
        turned = row_turned_offset<D>(lane, 4 * h, 0);
    }
    __device__ __forceinline__ Reads(const Reads &in_tile, uint32_t tile) : along(in_tile.along + tile), turned(in_tile.turned + tile) {}
    __device__ __forceinline__ bf16x8 row(int t, int s) const
    {
        return *(__attribute__((address_space(3))) const bf16x8 *)(uintptr_t)((along ^ (32 * s)) + t * (32 * D * 2));
    }
    __device__ __forceinline__ bf16x8 column(int ct, int s) const
    {
        typedef short s16x4 __attribute__((ext_vector_type(4)));
        typedef short s16x8 __attribute__((ext_vector_type(8)));
        typedef __attribute__((address_space(3))) s16x4 *at;
        constexpr uint32_t EIGHT = (row_swz<D>(8) ^ row_swz<D>(0)) * 16;       // rows 8 further: their flips
        const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((at)(uintptr_t)((turned ^ (64 * ct)) + s * (16 * D * 2)));
        const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
            (at)(uintptr_t)((turned ^ (64 * ct) ^ EIGHT) + s * (16 * D * 2) + 8 * D * 2));
        return __builtin_bit_cast(bf16x8, (s16x8)__builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
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

// The order of a block's LDS reads and products, for a loop of PRODUCTS products that take READS reads each: AHEAD products'
// reads before the first one, then product and reads in turn.  Left alone the compiler puts a read right before
// its product and waits for it there, 100 cycles for a product of 32.
template <int PRODUCTS, int READS, int AHEAD>
__device__ __forceinline__ void read_ahead()
{
    constexpr int DS_READ = 0x100, MFMA = 0x8;
    __builtin_amdgcn_sched_group_barrier(DS_READ, READS * AHEAD, 0);
    static_for<PRODUCTS>([&](auto k) {
        __builtin_amdgcn_sched_group_barrier(MFMA, 1, 0);
        if constexpr (decltype(k)::value + AHEAD < PRODUCTS) __builtin_amdgcn_sched_group_barrier(DS_READ, READS, 0);
    });
}

// scores of a tile's 32 rows (half t) with the wave's own rows
template <int D>
__device__ __forceinline__ f32x16 scores(const Reads<D> &tile, int t, const bf16x8 (&own)[D / 16])
{
    f32x16 c = {0};
#pragma unroll
    for (int s = 0; s < D / 16; ++s) c = mfma32(tile.row(t, s), own[s], c);
    return c;
}
// acc += tile^T w: the tile's rows 32 t .. with weights w (as results hold them), columns of the tile as rows of acc
template <int D, int AHEAD = 3>
__device__ __forceinline__ void add_turned(const Reads<D> &tile, int t, const f32x16 &w, f32x16 (&acc)[D / 32])
{
#pragma unroll
    for (int s = 0; s < 2; ++s) {
        const bf16x8 b = cvt8_from16(w, 8 * s);
#pragma unroll
        for (int ct = 0; ct < D / 32; ++ct) acc[ct] = mfma32(tile.column(ct, 2 * t + s), b, acc[ct]);
    }
    read_ahead<2 * (D / 32), 2, AHEAD>();
}

// place in its 32 rows of element e of a result
__device__ __forceinline__ int place(int e, int h) { return 8 * (e / 4) + 4 * h + e % 4; }

// Which workgroup of the call (unit by unit, neighbouring rows side by side) workgroup `id` of the launch is.  The launch
// deals its workgroups out to the 8 XCDs in turn; runs of RUN neighbours stay on one XCD, whose L2 serves the
// tiles that they share, and the runs go round the XCDs, one further every time round, so that neither sequences
// of unequal length nor the long and the short rows of all units meet on the same ones.  16 for the query side (8 x 12 x
// 4096, window 1024, lengths from 0 to 4096: forward 86 us, with runs of 2 95), 2 for the key side, whose walks are longer and
// fewer at a time (172 us, with runs of 16 187).
template <uint32_t RUN>
__device__ __forceinline__ uint32_t place_of(uint32_t id, uint32_t total)
{
    if (id >= total / (8 * RUN) * (8 * RUN)) return id;
    const uint32_t slot = id / 8, round = slot / RUN;
    return (round * 8 + (id + round) % 8) * RUN + slot % RUN;
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

// The wave's 32 result rows times `by` to memory in storage type (rows that lie behind their sequence: zeros): through LDS,
// where every lane has 8-byte pieces of its own row (columns 32 ct + place(e, h)) and takes whole 16-byte pieces of 64 / (D / 8)
// rows at a time, so that lines are written whole.  at: LDS address of the wave's 64 D bytes; to: its first row;
// rows: how many of them exist.
template <int D>
__device__ __forceinline__ void store_rows(const f32x16 (&acc)[D / 32], float by, bool there, uint32_t at, bf16_t *to, int64_t ld, int rows,
                                           int d, int lane)
{
    typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
    typedef float f32x4 __attribute__((ext_vector_type(4)));
    typedef uint32_t u4 __attribute__((ext_vector_type(4)));
    const int x = lane & 31, h = lane >> 5;
#pragma unroll
    for (int ct = 0; ct < D / 32; ++ct)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            f32x4 v;
#pragma unroll
            for (int k = 0; k < 4; ++k) v[k] = there ? acc[ct][4 * e + k] * by : 0.f;
            *(__attribute__((address_space(3))) bf16x4 *)(uintptr_t)(at + x * (D * 2) + ((4 * ct + e) ^ row_swz<D>(x)) * 16 + 8 * h) =
                __builtin_convertvector(v, bf16x4);
        }
#pragma unroll
    for (int q = 0; q < D / 16; ++q) {
        const int slot = q * 64 + lane, row = slot / (D / 8), piece = slot % (D / 8);
        const u4 v = *(__attribute__((address_space(3))) const u4 *)(uintptr_t)(at + row * (D * 2) + (piece ^ row_swz<D>(row)) * 16);
        if (row < rows && 8 * piece < d) *(u4 *)(to + row * ld + 8 * piece) = v;
    }
}

// ---- walks without masked pairs ------------------------------------------------------------------
// Where a result holds an infinity or NaN its wave walks its tiles again, straight from memory, 32 rows at a time: scores from
// products as before, the sums pair by pair in fp32 over the pairs that see each other.  (In a tile's product a masked pair
// counts as 0 times the other row, and 0 * inf would carry a token's infinity to rows that do not see it.)

// acc += sum over the rows r of `rows` (32 of them) that this lane sees of w(r) times row r; w as results hold it
template <int D>
__device__ __forceinline__ void add_seen(const bf16_t *rows, int64_t ld, int d, const f32x16 &w, uint32_t seen, f32x16 (&acc)[D / 32])
{
    typedef uint32_t u2 __attribute__((ext_vector_type(2)));
    const int lane = threadIdx.x & 63, x = lane & 31, h = lane >> 5;
#pragma unroll 1
    for (int r = 0; r < 32; ++r) {
        const int from = 4 * (r >> 3) + (r & 3);           // element of the result that holds row r, in half (r >> 2) & 1
        float own = w[0];
#pragma unroll
        for (int e = 1; e < 16; ++e) own = from == e ? w[e] : own;
        const float by = __shfl(own, x + 32 * ((r >> 2) & 1));
        if ((seen >> r) & 1u)
#pragma unroll
            for (int ct = 0; ct < D / 32; ++ct)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int col = 32 * ct + 8 * e + 4 * h;
                    if (col >= d) continue;
                    const u2 v = *(const u2 *)(rows + r * ld + col);
                    acc[ct][4 * e] += by * __uint_as_float(v.x << 16);
                    acc[ct][4 * e + 1] += by * __uint_as_float(v.x & 0xffff0000u);
                    acc[ct][4 * e + 2] += by * __uint_as_float(v.y << 16);
                    acc[ct][4 * e + 3] += by * __uint_as_float(v.y & 0xffff0000u);
                }
    }
}
// scores of rows r0 .. r0 + 31 (row `last` for those behind it) with the wave's own row
template <int D>
__device__ __forceinline__ f32x16 far_scores(const bf16_t *rows, int64_t ld, int r0, int last, int d, const bf16x8 (&own)[D / 16])
{
    const int x = threadIdx.x & 31, h = (threadIdx.x & 63) >> 5;
    bf16x8 f[D / 16];
    own_row<D>(rows + (int64_t)(r0 + x < last ? r0 + x : last) * ld, d, h, 1.f, f);
    f32x16 c = {0};
#pragma unroll
    for (int s = 0; s < D / 16; ++s) c = mfma32(f[s], own[s], c);
    return c;
}
template <int CT>
__device__ __forceinline__ bool odd_values(const f32x16 (&acc)[CT])
{
    float probe = 0.f;
#pragma unroll
    for (int ct = 0; ct < CT; ++ct)
#pragma unroll
        for (int e = 0; e < 16; ++e) probe = __builtin_fmaf(acc[ct][e], 0.f, probe);
    return probe != 0.f;
}

template <int D>
__device__ __forceinline__ void fwd_again(const Window &w, const bf16_t *K, const bf16_t *V, const bf16x8 (&own)[D / 16], float c, int i0,
                                          int i, int end, f32x16 (&acc)[D / 32], float &top, float &sum)
{
    const int h = (threadIdx.x & 63) >> 5;
#pragma unroll
    for (int ct = 0; ct < D / 32; ++ct) acc[ct] = f32x16{0};
    top = -INFINITY;
    sum = 0.f;
    const KeyTiles tiles(w, i0, i0 + kOwn < end ? i0 + kOwn - 1 : end - 1, 32);
    for (int k = 0; k < tiles.total; ++k) {
        const int j0 = tiles.at(k) * 32;
        const uint32_t seen = i < end ? seen_keys(w, i, j0) : 0u;
        f32x16 s = far_scores<D>(K, w.row_k, j0, end - 1, w.d, own);
        branch_wait();
        float most = -INFINITY;
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            s[e] = (seen >> place(e, h)) & 1u ? s[e] * c : -INFINITY;
            most = fmaxf(most, s[e]);
        }
        most = fmaxf(other_half(most, true), top);
        const float less = top == -INFINITY ? 0.f : exp2f(top - most), base = most == -INFINITY ? 0.f : most;
        top = most;
        sum *= less;
#pragma unroll
        for (int ct = 0; ct < D / 32; ++ct) acc[ct] *= less;
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            s[e] = exp2f(s[e] - base);
            sum += s[e];
        }
        add_seen<D>(V + j0 * w.row_k, w.row_k, w.d, s, seen, acc);
    }
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
    const uint32_t at_grid = place_of<16>(blockIdx.x, gridDim.x), unit = at_grid / groups;
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
        const uint32_t lds_at = lds_address(lds);
        stage.copy(k_rows, v_rows, w.row_k, tiles.at(0) * kTile, end, 0);
        for (int k = 0; k < tiles.total; ++k) {
            const int j0 = tiles.at(k) * kTile;
            wait_all_memory();                             // this wave's pieces of the tile, and its reads of the last one
            __builtin_amdgcn_s_barrier();
            asm volatile("" ::: "memory");
            if (k + 1 < tiles.total) stage.copy(k_rows, v_rows, w.row_k, tiles.at(k + 1) * kTile, end, (k + 1) & 1);
            if (none_seen(w, i0, kOwn, j0, kTile)) continue;
            const uint32_t at_tile = lds_at + (k & 1) * 2 * Tile::BYTES;
            const Reads<D> tk(at, at_tile), tv(at, at_tile + Tile::BYTES);
            f32x16 s[2];
#pragma unroll
            for (int t = 0; t < 2; ++t) s[t] = scores<D>(tk, t, own);
            read_ahead<2 * KS, 1, 4>();
            if (!all_seen(w, i0, kOwn, j0, kTile)) {
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
            for (int t = 0; t < 2; ++t) add_turned<D>(tv, t, s[t], acc);
            branch_wait();
        }
        if (__any(i < end && odd_values(acc))) {
            own_row<D>(q + (i < end ? i : end - 1) * w.row_q, d, h, w.scale2, own);
            fwd_again<D>(w, k_rows, v_rows, own, c, i0, i, end, acc, top, sum);
        }
    }
    sum = other_half(sum, false);
    const bool there = i < end;
    __syncthreads();                                       // (the tiles have been read)
    store_rows<D>(acc, 1.f / sum, there, lds_address(lds) + wave * (64 * D), O + b * w.batch_q + head * w.head_q + i0 * w.row_q, w.row_q,
                  w.n - i0, d, lane);
    if (lse && h == 0 && i < w.n)
        lse[((size_t)b * w.heads + head) * w.n + i] = there ? (top + __builtin_log2f(sum)) * kWindowLn2 : -INFINITY;
}

// ---- backward ---------------------------------------------------------------------------------

template <int D>
__device__ __forceinline__ void dq_again(const Window &w, const bf16_t *K, const bf16_t *V, const bf16x8 (&own)[D / 16],
                                         const bf16x8 (&own_g)[D / 16], float c, float L, float dot, int i0, int i, int end,
                                         f32x16 (&acc)[D / 32])
{
    const int h = (threadIdx.x & 63) >> 5;
#pragma unroll
    for (int ct = 0; ct < D / 32; ++ct) acc[ct] = f32x16{0};
    const KeyTiles tiles(w, i0, i0 + kOwn < end ? i0 + kOwn - 1 : end - 1, 32);
    for (int k = 0; k < tiles.total; ++k) {
        const int j0 = tiles.at(k) * 32;
        f32x16 s = far_scores<D>(K, w.row_k, j0, end - 1, w.d, own);
        const f32x16 u = far_scores<D>(V, w.row_k, j0, end - 1, w.d, own_g);
        branch_wait();
#pragma unroll
        for (int e = 0; e < 16; ++e) s[e] = exp2f(__builtin_fmaf(s[e], c, -L)) * (u[e] - dot);
        add_seen<D>(K + j0 * w.row_k, w.row_k, w.d, s, i < end ? seen_keys(w, i, j0) : 0u, acc);
    }
}

// Tiles [begin, stop) of a walk of the key side (see QueryTiles; tiles of `size` rows).
template <int D>
__device__ __forceinline__ void dkv_again(const Window &w, const bf16_t *Q, const bf16_t *dO, const float *lse, const float *delta,
                                          const bf16x8 (&own)[D / 16], const bf16x8 (&own_v)[D / 16], float c, int j, int end,
                                          const QueryTiles &tiles, int size, int begin, int stop, f32x16 (&acc_k)[D / 32],
                                          f32x16 (&acc_v)[D / 32])
{
    const int h = (threadIdx.x & 63) >> 5;
#pragma unroll
    for (int ct = 0; ct < D / 32; ++ct) acc_k[ct] = acc_v[ct] = f32x16{0};
    for (int k = begin; k < stop; ++k) {
        const int head = k / tiles.count, first = (tiles.tile0 + k - head * tiles.count) * size;
        const bf16_t *q = Q + head * w.head_q, *g = dO + head * w.head_q;
        for (int i0 = first; i0 < first + size && i0 < end; i0 += 32) {
            f32x16 s = far_scores<D>(q, w.row_q, i0, end - 1, w.d, own);
            f32x16 u = far_scores<D>(g, w.row_q, i0, end - 1, w.d, own_v);
            branch_wait();
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                const int i = i0 + place(e, h) < end ? i0 + place(e, h) : end - 1;
                s[e] = exp2f(__builtin_fmaf(s[e], c, -lse[(size_t)head * w.n + i] * kWindowLog2e));
                u[e] = s[e] * (u[e] - delta[(size_t)head * w.n + i]);
            }
            const uint32_t seen = j < end ? seen_by(w, j, i0, end) : 0u;
            add_seen<D>(g + i0 * w.row_q, w.row_q, w.d, s, seen, acc_v);
            add_seen<D>(q + i0 * w.row_q, w.row_q, w.d, u, seen, acc_k);
        }
    }
}

// Whether the kernel below forms D of a wave's rows, from row i0 on.  In a row of few keys dS = p (<dO, v> - D) is a small difference:
// D from the stored o, rounded to bf16, leaves up to 2^-8 of <dO, v> where the formula has 0 (a row of one key).  The
// error of such an o falls with the root of its keys; from 64 on it is an eighth of dS's own rounding.
constexpr int kFew = 64;
__host__ __device__ inline bool few_keys(const Window &w, int i0)
{
    return i0 < kFew || (int64_t)w.window + w.sinks <= kFew;
}

// D_i = sum_j p_ij <dO_i, v_j> / sum_j p_ij of rows of few keys: a wave 32 rows, its tiles of keys (at most four) straight from
// memory.  Bound by the latency of those loads: 6 us for 96 heads' first rows.
template <int D>
__global__ __launch_bounds__(64) void window_delta_kernel(const bf16_t *Q, const bf16_t *K, const bf16_t *V, const int32_t *lengths,
                                                          const float *lse, const bf16_t *dO, float *delta, Window w, uint32_t groups)
{
    constexpr int KS = D / 16;
    const int x = threadIdx.x & 31, h = threadIdx.x >> 5;
    const uint32_t unit = blockIdx.x / groups;
    const int b = unit / w.heads, head = unit - b * w.heads;
    const int end = window_end(lengths, b, w.n), i0 = (int)(blockIdx.x - unit * groups) * kOwn, i = i0 + x;
    if (i0 >= end) return;
    const int safe = i < end ? i : end - 1;
    const int64_t at_q = b * w.batch_q + head * w.head_q + safe * w.row_q, at_k = b * w.batch_k + head / w.group * w.head_k;
    const float c = w.scale2 == 0.f ? 1.f : fabsf(w.scale2);
    bf16x8 own[KS], own_g[KS];
    own_row<D>(Q + at_q, w.d, h, w.scale2, own);
    own_row<D>(dO + at_q, w.d, h, 1.f, own_g);
    const size_t row = ((size_t)b * w.heads + head) * w.n + safe;
    const float L = lse[row] * kWindowLog2e;
    float dot = 0.f, sum = 0.f;
    const KeyTiles tiles(w, i0, i0 + kOwn < end ? i0 + kOwn - 1 : end - 1, 32);
    for (int k = 0; k < tiles.total; ++k) {
        const int j0 = tiles.at(k) * 32;
        const f32x16 s = far_scores<D>(K + at_k, w.row_k, j0, end - 1, w.d, own);
        const f32x16 u = far_scores<D>(V + at_k, w.row_k, j0, end - 1, w.d, own_g);
        branch_wait();
        const uint32_t bits = seen_keys(w, i, j0) >> (4 * h);
        static_for<16>([&](auto e) {
            const float p = __builtin_amdgcn_exp2f(__builtin_fmaf(s[int(e)], c, -L));
            sum += pick<e>(bits, p, 0u);
            dot += pick<e>(bits, p * u[int(e)], 0u);
        });
    }
    dot = other_half(dot, false) / other_half(sum, false);
    if (i < end && h == 0) delta[row] = dot;
}

// dQ, and D = <dO, o> of every other row for the kernel below.
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
    const uint32_t at_grid = place_of<16>(blockIdx.x, gridDim.x), unit = at_grid / groups;
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
        const size_t row = ((size_t)b * w.heads + head) * w.n + safe;
        if (few_keys(w, i0)) {
            dot = delta[row];
        } else {
            bf16x8 o[KS];
            own_row<D>(O + at_q + safe * w.row_q, d, h, 1.f, o);
#pragma unroll
            for (int s = 0; s < KS; ++s)
#pragma unroll
                for (int e = 0; e < 8; ++e) dot += (float)o[s][e] * (float)own_g[s][e];
            dot = other_half(dot, false);
            if (i < end && h == 0) delta[row] = dot;
        }
        L = lse[row] * kWindowLog2e;
        const Reads<D> at(lane);
        const uint32_t lds_at = lds_address(lds);
        for (int k = 0; k < tiles.total; ++k) {
            const int j0 = tiles.at(k) * kTile;
            wait_all_memory();
            __builtin_amdgcn_s_barrier();
            asm volatile("" ::: "memory");
            if (k + 1 < tiles.total) stage.copy(k_rows, v_rows, w.row_k, tiles.at(k + 1) * kTile, end, (k + 1) & 1);
            if (none_seen(w, i0, kOwn, j0, kTile)) continue;
            const uint32_t at_tile = lds_at + (k & 1) * 2 * Tile::BYTES;
            const Reads<D> tk(at, at_tile), tv(at, at_tile + Tile::BYTES);
            const bool all = all_seen(w, i0, kOwn, j0, kTile);
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                f32x16 s = scores<D>(tk, t, own);
                const f32x16 u = scores<D>(tv, t, own_g);
                read_ahead<2 * KS, 1, 4>();
#pragma unroll
                for (int e = 0; e < 16; ++e) s[e] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[e], c, -L)) * (u[e] - dot);
                if (!all) {
                    const uint32_t bits = seen_keys(w, i, j0 + 32 * t) >> (4 * h);
                    static_for<16>([&](auto e) { s[int(e)] = pick<e>(bits, s[int(e)], 0u); });
                }
                add_turned<D>(tk, t, s, acc);
            }
            branch_wait();
        }
        if (__any(i < end && odd_values(acc))) {
            own_row<D>(Q + at_q + safe * w.row_q, d, h, w.scale2, own);
            own_row<D>(dO + at_q + safe * w.row_q, d, h, 1.f, own_g);
            dq_again<D>(w, k_rows, v_rows, own, own_g, c, L, dot, i0, i, end, acc);
        }
    }
    __syncthreads();
    store_rows<D>(acc, w.scale, i < end, lds_address(lds) + wave * (64 * D), dQ + at_q + i0 * w.row_q, w.row_q, w.n - i0, d, lane);
}

// dK and dV.  The wave's values lie in LDS: with them in registers three waves a SIMD do not fit at d = 64 (161 us instead of 145,
// see place_of) and two do not at d = 128 (1850 us instead of 1100, 2 x 16 x 16384, window 4096, one sequence empty), where the
// tiles are of 32 queries, so that two workgroups share a CU.
template <int D>
__global__ __launch_bounds__(kThreads, D == 64 ? 3 : 2) void window_dkv_kernel(
    const bf16_t *Q, const bf16_t *K, const bf16_t *V, const int32_t *lengths, const float *lse, const bf16_t *dO,
    const float *delta, bf16_t *dK, bf16_t *dV, float *room, Window w, KeyWalks walks)
{
    constexpr int KS = D / 16, CT = D / 32, TILE = D == 64 ? 64 : 32;
    using Tile = Staged<D, TILE>;
    __shared__ __align__(1024) unsigned char lds[2 * 2 * Tile::BYTES + kOwnWg * D * 2];
    __shared__ float2 row_data[2][TILE];                  // L (in exponents of 2) and D of the tile's rows
    const int lane = threadIdx.x & 63, x = lane & 31, h = lane >> 5, d = w.d;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);      // (in a scalar register: which tiles count is the wave's)
    const uint32_t at_grid = place_of<2>(blockIdx.x, gridDim.x), each = walks.each(), unit = at_grid / each;
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
        const uint32_t lds_at = lds_address(lds);
        bf16x8 own[KS];
        own_row<D>(K + at_k + (j < end ? j : end - 1) * w.row_k, d, h, w.scale2, own);
        const Reads<D> mine(at, lds_at + 2 * 2 * Tile::BYTES + wave * (kOwn * D * 2));   // the wave's value rows
        {
            bf16x8 v[KS];
            own_row<D>(V + at_k + (j < end ? j : end - 1) * w.row_k, d, h, 1.f, v);
#pragma unroll
            for (int s = 0; s < KS; ++s)                   // (read by this wave alone)
                *(__attribute__((address_space(3))) bf16x8 *)(uintptr_t)(mine.along ^ (32 * s)) = v[s];
        }
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
            const uint32_t at_tile = lds_at + buf * 2 * Tile::BYTES;
            const Reads<D> tq(at, at_tile), tg(at, at_tile + Tile::BYTES);
#pragma unroll
            for (int t = 0; t < TILE / 32; ++t) {
                f32x16 s = scores<D>(tq, t, own);
                f32x16 u = {0};
#pragma unroll
                for (int q = 0; q < KS; ++q) u = mfma32(tg.row(t, q), mine.row(0, q), u);
                read_ahead<KS, 1, 4>();
                read_ahead<KS, 2, 2>();
                __builtin_amdgcn_sched_barrier(0);         // (else the reads of row_data get into the order above)
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
                add_turned<D>(tg, t, s, acc_v);
                add_turned<D>(tq, t, u, acc_k);
            }
            branch_wait();
        }
        if (__any(j < end && (odd_values(acc_k) || odd_values(acc_v)))) {
            bf16x8 v[KS];
            own_row<D>(K + at_k + (j < end ? j : end - 1) * w.row_k, d, h, w.scale2, own);
            own_row<D>(V + at_k + (j < end ? j : end - 1) * w.row_k, d, h, 1.f, v);
            dkv_again<D>(w, Q + at_q, dO + at_q, lse + at_rows, delta + at_rows, own, v, c, j, end, tiles, TILE, begin, stop, acc_k, acc_v);
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
    __syncthreads();
    const uint32_t rows_at = lds_address(lds) + wave * (64 * D);
    store_rows<D>(acc_k, w.scale, j < end, rows_at, dK + at_k + j0 * w.row_k, w.row_k, w.n - j0, d, lane);
    store_rows<D>(acc_v, 1.f, j < end, rows_at, dV + at_k + j0 * w.row_k, w.row_k, w.n - j0, d, lane);
}

// The shares of the first tokens' gradients added in order: a thread four columns of a row.
__global__ __launch_bounds__(kThreads) void window_share_kernel(bf16_t *dK, bf16_t *dV, const float *room, Window w, KeyWalks walks)
{
    typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
    typedef float f32x4 __attribute__((ext_vector_type(4)));
    const int pieces = w.d / 4, at = blockIdx.x * kThreads + threadIdx.x, row = at / pieces, c = 4 * (at - row * pieces);
    const int b = blockIdx.y / w.kv_heads, kv = blockIdx.y - b * w.kv_heads;
    if (row >= walks.few * kOwnWg || row >= w.n) return;
    const size_t share = 2 * (size_t)kOwnWg * w.d;
    const float *from = room + ((size_t)blockIdx.y * walks.few + row / kOwnWg) * walks.parts * share + (size_t)(row % kOwnWg) * w.d + c;
    f32x4 k = {0.f, 0.f, 0.f, 0.f}, v = k;
#pragma unroll 4
    for (int p = 0; p < walks.parts; ++p) {
        k += *(const f32x4 *)(from + p * share);
        v += *(const f32x4 *)(from + p * share + share / 2);
    }
    const int64_t to = b * w.batch_k + kv * w.head_k + row * w.row_k + c;
    *(bf16x4 *)(dK + to) = __builtin_convertvector(k * w.scale, bf16x4);
    *(bf16x4 *)(dV + to) = __builtin_convertvector(v, bf16x4);
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

psf_status window_bf16_delta(const Window &w, const WindowPtrs &p, bool all, hipStream_t s)
{
    const uint32_t groups = ((all || w.n < kFew ? w.n : kFew) + kOwn - 1) / kOwn;
    auto go = [&](auto width) -> psf_status {
        constexpr int D = decltype(width)::value;
        hipLaunchKernelGGL((window_delta_kernel<D>), dim3(groups * w.batch * w.heads), dim3(64), 0, s, (const bf16_t *)p.Q,
                           (const bf16_t *)p.K, (const bf16_t *)p.V, p.lengths, p.lse, (const bf16_t *)p.dO, p.delta, w, groups);
        PSF_LAUNCH_CHECK();
        return PSF_OK;
    };
    return w.d <= 64 ? go(std::integral_constant<int, 64>{}) : go(std::integral_constant<int, 128>{});
}

psf_status window_bf16_bwd(const Window &w, const WindowPtrs &p, hipStream_t s)
{
    auto go = [&](auto width) -> psf_status {
        constexpr int D = decltype(width)::value;
        const bf16_t *Q = (const bf16_t *)p.Q, *K = (const bf16_t *)p.K, *V = (const bf16_t *)p.V, *O = (const bf16_t *)p.O,
                     *dO = (const bf16_t *)p.dO;
        bf16_t *dQ = (bf16_t *)p.dQ, *dK = (bf16_t *)p.dK, *dV = (bf16_t *)p.dV;
        const uint32_t groups = (w.n + kOwnWg - 1) / kOwnWg;
        if (const psf_status st = window_bf16_delta(w, p, few_keys(w, kFew), s); st != PSF_OK) return st;
        hipLaunchKernelGGL((window_dq_kernel<D>), dim3(groups * w.batch * w.heads), dim3(kThreads), 0, s, Q, K, V, p.lengths, O, p.lse,
                           dO, dQ, p.delta, w, groups);
        PSF_LAUNCH_CHECK();
        const KeyWalks walks = walks_of(w);
        const uint32_t units = w.batch * w.kv_heads;
        hipLaunchKernelGGL((window_dkv_kernel<D>), dim3(units * walks.each()), dim3(kThreads), 0, s, Q, K, V, p.lengths, p.lse, dO,
                           p.delta, dK, dV, p.room, w, walks);
        PSF_LAUNCH_CHECK();
        if (walks.parts == 1) return PSF_OK;
        hipLaunchKernelGGL(window_share_kernel, dim3((walks.few * kOwnWg * (w.d / 4) + kThreads - 1) / kThreads, units), dim3(kThreads), 0,
                           s, dK, dV, p.room, w, walks);
        PSF_LAUNCH_CHECK();
        return PSF_OK;
    };
    return w.d <= 64 ? go(std::integral_constant<int, 64>{}) : go(std::integral_constant<int, 128>{});
}

}  // namespace psf
