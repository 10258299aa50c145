// Softmax attention of one new token a sequence over a paged key-value cache (psf_paged_attn).
//
// Bound by memory: every visible key and value is read once, by the one workgroup that holds all query heads of its
// key head (up to 16 a workgroup: the columns of a 16 x 16 product).  A wave takes 32 positions at a time, straight
// from the pool into the operands of the products -- no LDS, no barrier in the loop --, with the running maximum and
// sum of the softmax beside the sums of the values.  Results are formed transposed (columns: heads), so that
// a head's maximum, sum and values stay in its four lanes and the weights are the next product's operand as
// they stand.  The visible positions are shared out over `splits` workgroups of four waves; where there is
// more than one, a second kernel joins them in a fixed order.
#include <type_traits>
#include "psf_cache.h"
#include "psf_parts.h"

namespace psf {
namespace {

constexpr int kPagedStep = 32;             // positions a wave takes at a time
constexpr int kPagedWaves = 4, kPagedMany = 8;   // waves of a workgroup, and of one that has a short sequence to itself
constexpr float kLog2e = 1.4426950408889634f;

struct PagedShape {
    Cache c;
    int heads, group, head_tiles;          // query heads, those of a key head, tiles of 16 of them
    int window, sinks, splits;
    float scale;                           // of the scores, with log2(e)
    FastDiv page;
};

// eight columns of a row (operand A or B of the scores), and their product
template <typename T> struct Eight;
template <> struct Eight<bf16_t> {
    bf8 v;
    __device__ __forceinline__ void load(const bf16_t *at) { v = *(const bf8 *)at; }
    __device__ __forceinline__ void zero() { v = __builtin_bit_cast(bf8, u4v{0u, 0u, 0u, 0u}); }
    static __device__ __forceinline__ f4 product(const Eight &a, const Eight &b, f4 c) { return mm32(a.v, b.v, c); }
};
template <> struct Eight<float> {
    f4 v[2];
    __device__ __forceinline__ void load(const float *at) { v[0] = *(const f4 *)at; v[1] = *(const f4 *)(at + 4); }
    __device__ __forceinline__ void zero() { v[0] = v[1] = f4{0.f, 0.f, 0.f, 0.f}; }
    static __device__ __forceinline__ f4 product(const Eight &a, const Eight &b, f4 c)
    {
#pragma unroll
        for (int e = 0; e < 8; ++e) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a.v[e / 4][e % 4], b.v[e / 4][e % 4], c, 0, 0, 0);
        return c;
    }
};

// VW columns of a value row, and the sums of the values: column VW c + j of the output is row c of tile j
template <typename T, int VW> struct Values;
template <int VW> struct Values<bf16_t, VW> {
    typedef uint32_t words __attribute__((ext_vector_type(VW / 2)));
    words v;
    __device__ __forceinline__ void load(const bf16_t *at) { v = *(const words *)at; }
    __device__ __forceinline__ void zero()
    {
#pragma unroll
        for (int k = 0; k < VW / 2; ++k) v[k] = 0u;
    }
    // eight positions (tile order); weights rounded to bf16 for the product, their sum is formed before
    static __device__ __forceinline__ void add(const Values (&x)[8], const float (&w)[8], f4 (&acc)[VW])
    {
        u4v p;
#pragma unroll
        for (int k = 0; k < 4; ++k) p[k] = round_pair(w[2 * k], w[2 * k + 1]);
#pragma unroll
        for (int j = 0; j < VW; ++j) {
            u4v a;
#pragma unroll
            for (int k = 0; k < 4; ++k)
                a[k] = __builtin_amdgcn_perm(x[2 * k + 1].v[j / 2], x[2 * k].v[j / 2], j % 2 ? 0x07060302u : 0x05040100u);
            acc[j] = mm32(__builtin_bit_cast(bf8, a), __builtin_bit_cast(bf8, p), acc[j]);
        }
    }
};
template <int VW> struct Values<float, VW> {
    f4 v[VW / 4];
    __device__ __forceinline__ void load(const float *at)
    {
#pragma unroll
        for (int k = 0; k < VW / 4; ++k) v[k] = *(const f4 *)(at + 4 * k);
    }
    __device__ __forceinline__ void zero()
    {
#pragma unroll
        for (int k = 0; k < VW / 4; ++k) v[k] = f4{0.f, 0.f, 0.f, 0.f};
    }
    static __device__ __forceinline__ void add(const Values (&x)[8], const float (&w)[8], f4 (&acc)[VW])
    {
#pragma unroll
        for (int e = 0; e < 8; ++e)
#pragma unroll
            for (int j = 0; j < VW; ++j)
                acc[j] = __builtin_amdgcn_mfma_f32_16x16x4f32(x[e].v[j / 4][j % 4], w[e], acc[j], 0, 0, 0);
    }
};

__device__ __forceinline__ float max_over_groups(float x)   // over the four lanes of a column
{
    const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
    const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}

// The steps of 32 positions with visible ones: those of the first tokens, then those of the window.
struct Steps {
    int first_steps, window_first, total, window_start, length;
    __device__ __forceinline__ Steps(int len, const PagedShape &sh)
    {
        const long long most = (long long)sh.c.cols * sh.c.page;
        length = len <= 0 ? 0 : len < most ? len : (int)most;
        // (the window ends at the last token, which lies at len - 1 even where the table is too short for it)
        window_start = len > sh.window ? len - sh.window : 0;
        const int few = sh.sinks < window_start ? sh.sinks : window_start, shown = few < length ? few : length;
        first_steps = (shown + kPagedStep - 1) / kPagedStep;
        window_first = window_start / kPagedStep;
        if (window_first < first_steps) window_first = first_steps;
        const int last = (int)(((long long)length + kPagedStep - 1) / kPagedStep);
        total = first_steps + (last > window_first ? last - window_first : 0);
    }
    __device__ __forceinline__ int at(int k) const { return k < first_steps ? k : window_first + k - first_steps; }
};

// (At least two waves a SIMD: fp32 rows of 128 leave to itself at one, 90 us for 16 contexts of 5000 tokens and four key heads
// instead of 74; bf16 rows reach three.)
template <typename T, int DP, int WAVES>
__global__ __launch_bounds__(64 * WAVES, 2) void paged_attn_kernel(const T *q, const T *Kp, const T *Vp, const int32_t *table,
                                                                      const int32_t *lengths, T *o, float *sums, float *parts,
                                                                      PagedShape sh)
{
    constexpr int KS = DP / 32, VW = DP / 16;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, li = lane & 15, g = lane >> 4;
    const int split = blockIdx.x % sh.splits;
    uint32_t unit = blockIdx.x / sh.splits;
    const int tile = unit % sh.head_tiles;
    unit /= sh.head_tiles;
    const int kv = unit % sh.c.kv_heads, seq = unit / sh.c.kv_heads;
    const int d = sh.c.d;
    const Steps steps(lengths[seq], sh);
    const int begin = (int)((long long)steps.total * split / sh.splits), end = (int)((long long)steps.total * (split + 1) / sh.splits);
    const int32_t *row_table = table + (size_t)seq * sh.c.cols;

    const int head = 16 * tile + li;                       // of the group
    const bool there = head < sh.group;
    Eight<T> own[KS];
#pragma unroll
    for (int s = 0; s < KS; ++s) {
        own[s].zero();
        if (there && 32 * s + 8 * g < d) own[s].load(q + ((size_t)seq * sh.heads + kv * sh.group + head) * d + 32 * s + 8 * g);
    }
    f4 acc[VW];
    clear(acc);
    float top = -INFINITY, sum = 0.f;

    // row of the pool of position 32 step + (lane & 31); -1 where that one is not seen
    auto row_at = [&](int step) -> int {
        const long long pos = (long long)step * kPagedStep + (lane & 31);
        if (pos >= steps.length || (pos < steps.window_start && pos >= sh.sinks)) return -1;
        const uint32_t col = sh.page.div((uint32_t)pos), slot = (uint32_t)pos - col * sh.page.by;
        const int p = page_of(row_table, (int)col, sh.c.cols, sh.c.pages);
        return p < 0 ? -1 : (p * sh.c.kv_heads + kv) * sh.c.page + (int)slot;
    };
    int next = begin + wave < end ? row_at(steps.at(begin + wave)) : -1;
    for (int k = begin + wave; k < end; k += WAVES) {
        const int mine = next;
        Eight<T> key[2][KS];
        Values<T, VW> val[8];
        int rows[8];
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            const int row = __shfl(mine, 16 * t + li);
#pragma unroll
            for (int s = 0; s < KS; ++s) {
                key[t][s].zero();
                if (row >= 0 && 32 * s + 8 * g < d) key[t][s].load(Kp + (size_t)row * d + 32 * s + 8 * g);
            }
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            rows[e] = __shfl(mine, 16 * (e / 4) + 4 * g + e % 4);
            val[e].zero();
            if (rows[e] >= 0 && VW * li < d) val[e].load(Vp + (size_t)rows[e] * d + VW * li);
        }
        if (k + WAVES < end) next = row_at(steps.at(k + WAVES));
        float w[8];
        float most = -INFINITY;
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            f4 s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int c = 0; c < KS; ++c) s = Eight<T>::product(key[t][c], own[c], s);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                w[4 * t + e] = rows[4 * t + e] >= 0 ? s[e] * sh.scale : -INFINITY;
                most = fmaxf(most, w[4 * t + e]);
            }
        }
        most = fmaxf(top, max_over_groups(most));
        if (__any(most > top)) {
            const float less = top == -INFINITY ? 0.f : exp2f(top - most);
            sum *= less;
#pragma unroll
            for (int j = 0; j < VW; ++j) acc[j] *= less;
            top = most;
        }
        const float base = top == -INFINITY ? 0.f : top;   // (nothing seen yet: every weight is 0)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            w[e] = exp2f(w[e] - base);
            sum += w[e];
        }
        Values<T, VW>::add(val, w, acc);
        settle_parts();                                    // the sums are read at the next step's head
    }

    // the waves together
    __shared__ float tops[WAVES][16], totals[WAVES][16];
    __shared__ float lds[WAVES][16][DP + 4];
    sum = over_groups(sum);
    if (g == 0) {
        tops[wave][li] = top;
        totals[wave][li] = sum;
    }
    __syncthreads();
    auto highest = [&](int h) {
        float most = tops[0][h];
#pragma unroll
        for (int w = 1; w < WAVES; ++w) most = fmaxf(most, tops[w][h]);
        return most;
    };
    float all = highest(li);
    const float share = top == -INFINITY ? 0.f : exp2f(top - all);
#pragma unroll
    for (int j = 0; j < VW; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) lds[wave][li][VW * (4 * g + e) + j] = acc[j][e] * share;
    __syncthreads();
    const int h = threadIdx.x / 16, c = threadIdx.x % 16;  // 256 threads: 16 heads, VW columns each
    if (h >= 16 || 16 * tile + h >= sh.group || VW * c >= d) return;
    all = highest(h);
    float total = 0.f;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) total += tops[w][h] == -INFINITY ? 0.f : totals[w][h] * exp2f(tops[w][h] - all);
    const size_t row = (size_t)seq * sh.heads + kv * sh.group + 16 * tile + h;
    const float by = sh.splits > 1 ? 1.f : total > 0.f || total != total ? 1.f / total : 0.f;
    float out[VW];
#pragma unroll
    for (int j = 0; j < VW; ++j) {
        out[j] = lds[0][h][VW * c + j];
#pragma unroll
        for (int w = 1; w < WAVES; ++w) out[j] += lds[w][h][VW * c + j];
        out[j] *= by;
    }
    if (sh.splits == 1) {
#pragma unroll
        for (int j = 0; j < VW; j += 4) store4(o + row * d + VW * c + j, f4{out[j], out[j + 1], out[j + 2], out[j + 3]});
        return;
    }
    const size_t rows = (size_t)sh.c.seqs * sh.heads, at = (size_t)split * rows + row;
    if (c == 0) {
        sums[2 * at] = all;
        sums[2 * at + 1] = total;
    }
#pragma unroll
    for (int j = 0; j < VW; j += 4) store4(parts + at * d + VW * c + j, f4{out[j], out[j + 1], out[j + 2], out[j + 3]});
}

// One workgroup a row: the splits' sums, weighted by their maxima.  16 lanes hold 64 columns (four each), D / 64 times; the
// groups of lanes share the splits out, each adds its own in turn, then the groups are added in order.  (One wave a row that
// walked the splits one by one took 132 us for 171 of them, 48 rows, d = 128; this takes 6.)
constexpr int kJoinThreads = 256, kJoinMost = 256;         // splits at most
template <typename T, int D>
__global__ __launch_bounds__(kJoinThreads) void paged_join_kernel(const float *sums, const float *parts, T *o, int rows, int d,
                                                                  int splits)
{
    constexpr int LANES = D / 4, GROUPS = kJoinThreads / LANES;
    __shared__ float weight[kJoinMost], tops[4], totals[4];
    __shared__ f4 lds[GROUPS][LANES];
    const int tid = threadIdx.x, wave = tid >> 6;
    const size_t row = blockIdx.x;
    float top = -INFINITY, sum = 0.f;
    if (tid < splits) {
        const float2 v = *(const float2 *)(sums + 2 * ((size_t)tid * rows + row));
        top = v.x;
        sum = v.y;
    }
    float all = top;
#pragma unroll
    for (int k = 1; k < 64; k <<= 1) all = fmaxf(all, __shfl_xor(all, k));
    if ((tid & 63) == 0) tops[wave] = all;
    __syncthreads();
    all = fmaxf(fmaxf(tops[0], tops[1]), fmaxf(tops[2], tops[3]));
    const float by = top == -INFINITY ? 0.f : exp2f(top - all);
    weight[tid] = by;
    sum *= by;
#pragma unroll
    for (int k = 1; k < 64; k <<= 1) sum += __shfl_xor(sum, k);
    if ((tid & 63) == 0) totals[wave] = sum;
    __syncthreads();
    const float total = (totals[0] + totals[1]) + (totals[2] + totals[3]);
    const int c = 4 * (tid % LANES), group = tid / LANES;
    f4 acc = {0.f, 0.f, 0.f, 0.f};
    if (c < d)
#pragma unroll 8
        for (int s = group; s < splits; s += GROUPS) acc += *(const f4 *)(parts + ((size_t)s * rows + row) * d + c) * weight[s];
    lds[group][tid % LANES] = acc;
    __syncthreads();
    if (group == 0 && c < d) {
        for (int k = 1; k < GROUPS; ++k) acc += lds[k][tid % LANES];
        store4(o + row * d + c, acc * (total > 0.f || total != total ? 1.f / total : 0.f));
    }
}

long long paged_units(const Cache &c, int heads) { return (long long)c.seqs * c.kv_heads * ((heads / c.kv_heads + 15) / 16); }

// Where a table holds short sequences only, a workgroup of kPagedMany waves has one to itself, which saves the second launch:
// up to 4 steps a wave, one in fp32 (its products take four times as long), four times that where there are as
// many workgroups as CUs.  Without the split and with it, us: one sequence, 12 key heads of 64, bf16, 1000 tokens 11.3 and
// 13.6, 1500 14.7 and 13.4; 64 such sequences, 500 20.0 and 22.6, 4000 138 and 143; fp32, 4 key heads of 128, one sequence of
// 100 11.0 and 13.2, of 500 20 and 13.4; 64 of 500 27 and 32.
bool paged_short(const Cache &c, int heads)
{
    const int steps = (c.bf16 ? 4 : 1) * (paged_units(c, heads) >= 256 ? 4 : 1);
    return (long long)c.cols * c.page <= steps * kPagedMany * kPagedStep;
}

// Workgroups that share a sequence's positions: as many as make 1024 workgroups of the whole call (four a CU), but
// no fewer than 128 positions (a step for every wave) of the longest sequence the table can hold.  Measured with 512, 768,
// 1024 and 1536 (us): 64 contexts of 300 to 12000 tokens 179, 180, 166, 160; three of 100000 70, 67, 68, 74; 16 of 2500
// 32, 34, 33, 35; 64 behind a window of 1024 31, 32, 34, 34.
int paged_splits(const Cache &c, int heads)
{
    if (paged_short(c, heads)) return 1;
    const long long units = paged_units(c, heads);
    const long long steps = ((long long)c.cols * c.page + kPagedWaves * kPagedStep - 1) / (kPagedWaves * kPagedStep);
    long long splits = (1024 + units - 1) / units;
    if (splits > steps) splits = steps;
    return splits < 1 ? 1 : splits > kJoinMost ? kJoinMost : (int)splits;
}

psf_status check(const psf_cache_desc *desc, int heads, Cache *c)
{
    const psf_status st = make_cache(desc, c);
    if (st != PSF_OK) return st;
    if (heads <= 0 || heads % c->kv_heads != 0) return PSF_ERR_SHAPE;
    if ((long long)c->seqs * heads > 0x7fffff) return PSF_ERR_UNSUPPORTED;
    return PSF_OK;
}

template <typename T, int DP>
psf_status launch(const void *q, const void *Kp, const void *Vp, const int32_t *table, const int32_t *lengths, void *o,
                  void *ws, const PagedShape &sh, hipStream_t s)
{
    const size_t rows = (size_t)sh.c.seqs * sh.heads;
    float *sums = (float *)ws, *parts = sums ? sums + align_up(2 * rows * sh.splits, 64) : nullptr;
    const uint32_t groups = (uint32_t)sh.c.seqs * sh.c.kv_heads * sh.head_tiles * sh.splits;
    auto go = [&](auto waves) {
        constexpr int WAVES = decltype(waves)::value;
        hipLaunchKernelGGL((paged_attn_kernel<T, DP, WAVES>), dim3(groups), dim3(64 * WAVES), 0, s, (const T *)q, (const T *)Kp,
                           (const T *)Vp, table, lengths, (T *)o, sums, parts, sh);
    };
    if (paged_short(sh.c, sh.heads)) go(std::integral_constant<int, kPagedMany>{});
    else go(std::integral_constant<int, kPagedWaves>{});
    PSF_LAUNCH_CHECK();
    if (sh.splits == 1) return PSF_OK;
    hipLaunchKernelGGL((paged_join_kernel<T, DP>), dim3((uint32_t)rows), dim3(kJoinThreads), 0, s, sums, parts, (T *)o, (int)rows, sh.c.d,
                       sh.splits);
    PSF_LAUNCH_CHECK();
    return PSF_OK;
}

}  // namespace
}  // namespace psf

using namespace psf;

extern "C" {

size_t psf_paged_workspace_bytes(const psf_cache_desc *desc, int32_t heads)
{
    Cache c;
    if (check(desc, heads, &c) != PSF_OK) return 0;
    const size_t splits = paged_splits(c, heads), rows = (size_t)c.seqs * heads;
    if (splits == 1) return 0;
    return align_up((align_up(2 * rows * splits, 64) + rows * splits * c.d) * sizeof(float), 256);
}

psf_status psf_paged_attn(const psf_cache_desc *desc, int32_t heads, int32_t window, int32_t sinks, float scale, const void *q,
                          const void *Kp, const void *Vp, const int32_t *table, const int32_t *lengths, void *o,
                          void *workspace, size_t workspace_bytes, void *hip_stream)
{
    PagedShape sh;
    const psf_status st = check(desc, heads, &sh.c);
    if (st != PSF_OK) return st;
    if (window <= 0 || sinks < 0) return PSF_ERR_SHAPE;
    if (!(fabsf(scale) < INFINITY)) return PSF_ERR_UNSUPPORTED;
    if (!q || !Kp || !Vp || !table || !lengths || !o) return PSF_ERR_NULL;
    const size_t need = psf_paged_workspace_bytes(desc, heads);
    if (need > 0 && !workspace) return PSF_ERR_NULL;
    if (workspace_bytes < need) return PSF_ERR_WORKSPACE;
    if (((uintptr_t)workspace & 255u) != 0) return PSF_ERR_WORKSPACE;
    if ((((uintptr_t)q | (uintptr_t)Kp | (uintptr_t)Vp | (uintptr_t)o) & 15u) != 0) return PSF_ERR_ALIGNMENT;
    sh.heads = heads;
    sh.group = heads / sh.c.kv_heads;
    sh.head_tiles = (sh.group + 15) / 16;
    sh.window = window;
    sh.sinks = sinks;
    sh.splits = paged_splits(sh.c, heads);
    sh.scale = scale * kLog2e;
    sh.page = fast_div(sh.c.page);
    hipStream_t s = (hipStream_t)hip_stream;
    void *ws = need > 0 ? workspace : nullptr;
    if (sh.c.bf16)
        return sh.c.d <= 64 ? launch<bf16_t, 64>(q, Kp, Vp, table, lengths, o, ws, sh, s)
                            : launch<bf16_t, 128>(q, Kp, Vp, table, lengths, o, ws, sh, s);
    return sh.c.d <= 64 ? launch<float, 64>(q, Kp, Vp, table, lengths, o, ws, sh, s)
                        : launch<float, 128>(q, Kp, Vp, table, lengths, o, ws, sh, s);
}

}  // extern "C"
