// Upkeep of a paged key-value cache: new tokens into their pages, sequences forked, the pages in use
// brought to the front of the pool.  All of it moves bytes and is bound by memory (or, for one token a
// sequence, by the latency of a launch): 16 bytes a lane, a page's K and V in the same launch.
// Everything that selects a place -- lengths, counts, tables, lists of sequences -- is read on the device and
// checked there: what lies outside the table or the pool is left out.
#include <initializer_list>
#include "psf_cache.h"

namespace psf {

psf_status make_cache(const psf_cache_desc *desc, Cache *out)
{
    if (!desc) return PSF_ERR_NULL;
    if (desc->pages <= 0 || desc->page <= 0 || desc->kv_heads <= 0 || desc->d <= 0 || desc->seqs <= 0 || desc->cols <= 0)
        return PSF_ERR_SHAPE;
    if (desc->dtype != PSF_F32 && desc->dtype != PSF_BF16) return PSF_ERR_UNSUPPORTED;
    if (desc->d % 8 != 0 || desc->d > PSF_CACHE_MAX_DIM) return PSF_ERR_UNSUPPORTED;
    // a row of the pool has an index of 31 bits, and so has a place of the table and a position
    const long long rows = (long long)desc->pages * desc->page;
    if (desc->pages > PSF_CACHE_MAX_PAGES || rows > 0x7fffffffll || rows * desc->kv_heads > 0x7fffffffll ||
        (long long)desc->seqs * desc->cols > 0x7fffffffll || (long long)desc->cols * desc->page > 0x7fffffffll)
        return PSF_ERR_UNSUPPORTED;
    out->pages = desc->pages; out->page = desc->page; out->kv_heads = desc->kv_heads; out->d = desc->d;
    out->seqs = desc->seqs; out->cols = desc->cols; out->bf16 = desc->dtype == PSF_BF16;
    return PSF_OK;
}

namespace {

typedef uint32_t u4 __attribute__((ext_vector_type(4)));
constexpr int kCacheThreads = 256;

// New rows K, V [seqs][kv_heads][n][row] to the places behind the sequences' lengths.  blockIdx.x walks the 16-byte pieces of
// one (sequence, head), blockIdx.y those pairs; where one pair has few pieces `fold` pairs share a workgroup.
__global__ __launch_bounds__(kCacheThreads) void cache_append_kernel(const u4 *K, const u4 *V, u4 *Kp, u4 *Vp,
                                                                     const int32_t *table, const int32_t *lengths,
                                                                     const int32_t *counts, Cache c, int n, FastDiv pieces,
                                                                     FastDiv page, FastDiv heads, int fold)
{
    const uint32_t per = pieces.by * (uint32_t)n, lanes = kCacheThreads / fold;
    for (uint32_t first = blockIdx.y * fold; first < (uint32_t)c.seqs * c.kv_heads; first += gridDim.y * fold) {
        const uint32_t pair = first + threadIdx.x / lanes;
        if (pair >= (uint32_t)c.seqs * c.kv_heads) continue;
        const uint32_t seq = heads.div(pair), head = pair - seq * heads.by;
        const int have = lengths[seq], count = counts ? counts[seq] : n;
        const int use = count < n ? count : n;
        if (have < 0 || use <= 0) continue;
        const int32_t *row = table + (size_t)seq * c.cols;
        const uint32_t most = pieces.by * (uint32_t)use;
        for (uint32_t i = blockIdx.x * lanes + threadIdx.x % lanes; i < most; i += gridDim.x * lanes) {
            const uint32_t t = pieces.div(i), piece = i - t * pieces.by;
            const int64_t at = (int64_t)have + t;
            if (at >= (int64_t)c.cols * c.page) break;
            const uint32_t col = page.div((uint32_t)at), slot = (uint32_t)at - col * page.by;
            const int p = page_of(row, (int)col, c.cols, c.pages);
            if (p < 0) continue;
            const size_t to = (((size_t)p * c.kv_heads + head) * c.page + slot) * pieces.by + piece;
            const size_t from = (size_t)pair * per + i;
            const u4 a = K[from], b = V[from];
            Kp[to] = a;
            Vp[to] = b;
        }
    }
}

// 16-byte pieces of one page, both pools, shared out over gridDim.x workgroups.
__device__ __forceinline__ void copy_page(u4 *Kp, u4 *Vp, size_t pieces, int from, int to, uint32_t part, uint32_t parts)
{
    const size_t src = (size_t)from * pieces, dst = (size_t)to * pieces;
    size_t i = (size_t)part * kCacheThreads + threadIdx.x;
    const size_t step = (size_t)parts * kCacheThreads;
    for (; i + 3 * step < pieces; i += 4 * step) {
        u4 a[4], b[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            a[k] = Kp[src + i + k * step];
            b[k] = Vp[src + i + k * step];
        }
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            Kp[dst + i + k * step] = a[k];
            Vp[dst + i + k * step] = b[k];
        }
    }
    for (; i < pieces; i += step) {
        const u4 a = Kp[src + i], b = Vp[src + i];
        Kp[dst + i] = a;
        Vp[dst + i] = b;
    }
}

// Fork k: row children[k] of the table becomes row parents[k], with a copy of the last page of its own (fresh[k])
// where that page is not full.
__global__ __launch_bounds__(kCacheThreads) void cache_fork_kernel(u4 *Kp, u4 *Vp, int32_t *table, int32_t *lengths,
                                                                   const int32_t *parents, const int32_t *children,
                                                                   const int32_t *fresh, Cache c, size_t pieces)
{
    const int k = blockIdx.y, parent = parents[k], child = children[k];
    if ((unsigned)parent >= (unsigned)c.seqs || (unsigned)child >= (unsigned)c.seqs || parent == child) return;
    const int32_t *from = table + (size_t)parent * c.cols;
    int32_t *to = table + (size_t)child * c.cols;
    const int length = lengths[parent], last = length > 0 ? length / c.page : 0;
    const bool part = length > 0 && length % c.page != 0 && last < c.cols;
    const int own = (unsigned)fresh[k] < (unsigned)c.pages ? fresh[k] : -1;
    const int old = part ? page_of(from, last, c.cols, c.pages) : -1;      // (no page there: the child has none either)
    if (blockIdx.x == 0) {
        for (int i = threadIdx.x; i < c.cols; i += kCacheThreads) to[i] = old >= 0 && i == last ? own : from[i];
        if (threadIdx.x == 0) lengths[child] = length;
    }
    if (old >= 0 && own >= 0) copy_page(Kp, Vp, pieces, old, own, blockIdx.x, gridDim.x);
}

// Which pages move: one workgroup, a bit for every page in LDS.  `live` pages are in use; the k-th free page
// below that number, to[k], takes the k-th used page from it on, from[k]; place[from[k]] = k.  Bound by the latency of its steps
// (lengths, table, two scans), so the table's entries are loaded four a lane and row at a time.
constexpr int kPlanThreads = 1024, kPlanWaves = kPlanThreads / 64;
__global__ __launch_bounds__(kPlanThreads) void cache_plan_kernel(const int32_t *table, const int32_t *lengths, Cache c,
                                                                  int32_t *live, int32_t *n_moves, int32_t *from, int32_t *to,
                                                                  int32_t *place)
{
    constexpr int AHEAD = 4, ROWS = 1024;                  // ROWS: lengths held in LDS at a time
    __shared__ uint32_t used[PSF_CACHE_MAX_PAGES / 32];
    __shared__ int2 sums[kPlanWaves];
    __shared__ int needs[ROWS];
    const int words = (c.pages + 31) / 32, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    for (int i = tid; i < words; i += kPlanThreads) used[i] = 0u;
    for (int base = 0; base < c.seqs; base += ROWS) {
        __syncthreads();
        if (base + tid < c.seqs) {
            const int length = lengths[base + tid], need = length <= 0 ? 0 : (length - 1) / c.page + 1;
            needs[tid] = need < c.cols ? need : c.cols;
        }
        __syncthreads();
        const int rows = c.seqs - base < ROWS ? c.seqs - base : ROWS;
        for (int r = wave; r < rows; r += kPlanWaves) {
            const int32_t *row = table + (size_t)(base + r) * c.cols;
            const int need = needs[r];
            for (int i = lane; i < need; i += 64 * AHEAD) {
                int p[AHEAD];
#pragma unroll
                for (int k = 0; k < AHEAD; ++k) p[k] = i + 64 * k < need ? row[i + 64 * k] : -1;
#pragma unroll
                for (int k = 0; k < AHEAD; ++k)
                    if ((unsigned)p[k] < (unsigned)c.pages) atomicOr(&used[p[k] >> 5], 1u << (p[k] & 31));
            }
        }
    }
    __syncthreads();
    // words of a thread: [first, last); sums over the threads before it, and over all
    const int each = (words + kPlanThreads - 1) / kPlanThreads, first = tid * each < words ? tid * each : words,
              last = first + each < words ? first + each : words;
    auto before = [&](int2 mine, int2 &total) {
        int2 run = mine;
#pragma unroll
        for (int k = 1; k < 64; k <<= 1) {
            const int x = __shfl_up(run.x, k), y = __shfl_up(run.y, k);
            if (lane >= k) {
                run.x += x;
                run.y += y;
            }
        }
        __syncthreads();
        if (lane == 63) sums[wave] = run;
        __syncthreads();
        int2 base = make_int2(0, 0);
        total = make_int2(0, 0);
#pragma unroll
        for (int k = 0; k < kPlanWaves; ++k) {
            const int2 s = sums[k];
            if (k < wave) {
                base.x += s.x;
                base.y += s.y;
            }
            total.x += s.x;
            total.y += s.y;
        }
        return make_int2(base.x + run.x - mine.x, base.y + run.y - mine.y);
    };
    int2 mine = make_int2(0, 0), total, moving;
    for (int i = first; i < last; ++i) mine.x += __popc(used[i]);
    (void)before(mine, total);
    // bits of word i that stand for pages below `live`
    auto below = [&](int i) -> uint32_t {
        const int left = total.x - 32 * i;
        return left <= 0 ? 0u : left >= 32 ? 0xffffffffu : (1u << left) - 1u;
    };
    mine = make_int2(0, 0);
    for (int i = first; i < last; ++i) {
        mine.x += __popc(~used[i] & below(i));
        mine.y += __popc(used[i] & ~below(i));
    }
    int2 at = before(mine, moving);
    for (int i = first; i < last; ++i) {
        for (uint32_t bits = ~used[i] & below(i); bits; bits &= bits - 1) to[at.x++] = 32 * i + __ffs(bits) - 1;
        for (uint32_t bits = used[i] & ~below(i); bits; bits &= bits - 1) {
            const int p = 32 * i + __ffs(bits) - 1;
            place[p] = at.y;
            from[at.y++] = p;
        }
    }
    if (tid == 0) {
        *live = total.x;
        *n_moves = moving.y;
    }
}

// The moves of the plan (a workgroup takes whole parts of a page), and the table with the pages' new places.
__global__ __launch_bounds__(kCacheThreads) void cache_move_kernel(u4 *Kp, u4 *Vp, const int32_t *table, const int32_t *lengths,
                                                                   int32_t *new_table, Cache c, size_t pieces, uint32_t parts,
                                                                   const int32_t *live, const int32_t *n_moves,
                                                                   const int32_t *from, const int32_t *to,
                                                                   const int32_t *place, FastDiv cols, FastDiv page)
{
    const int most = *live;
    const uint32_t entries = (uint32_t)c.seqs * c.cols;
    for (uint32_t i = blockIdx.x * kCacheThreads + threadIdx.x; i < entries; i += gridDim.x * kCacheThreads) {
        const uint32_t seq = cols.div(i), col = i - seq * cols.by;
        const int length = lengths[seq];
        int now = -1;
        if (length > 0 && col <= page.div((uint32_t)length - 1)) {
            const int p = table[i];
            if ((unsigned)p < (unsigned)c.pages) now = p < most ? p : to[place[p]];
        }
        new_table[i] = now;
    }
    const uint64_t units = (uint64_t)*n_moves * parts;
    for (uint64_t u = blockIdx.x; u < units; u += gridDim.x) {
        const uint32_t k = (uint32_t)(u / parts), part = (uint32_t)(u - (uint64_t)k * parts);
        copy_page(Kp, Vp, pieces, from[k], to[k], part, parts);
    }
}

bool aligned16(std::initializer_list<const void *> tensors)
{
    for (const void *p : tensors)
        if (((uintptr_t)p & 15u) != 0) return false;
    return true;
}

// A workgroup's part of a page: 16 KB of either pool (four 16-byte pieces a lane).
uint32_t page_parts(size_t pieces)
{
    const size_t parts = (pieces + 4 * kCacheThreads - 1) / (4 * kCacheThreads);
    return (uint32_t)(parts < 4096 ? parts : 4096);
}

}  // namespace
}  // namespace psf

using namespace psf;

extern "C" {

psf_status psf_check_cache_desc(const psf_cache_desc *desc)
{
    Cache c;
    return make_cache(desc, &c);
}

psf_status psf_cache_append(const psf_cache_desc *desc, int32_t n, const void *K, const void *V, void *Kp, void *Vp,
                            const int32_t *table, const int32_t *lengths, const int32_t *counts, void *hip_stream)
{
    Cache c;
    const psf_status st = make_cache(desc, &c);
    if (st != PSF_OK) return st;
    if (n <= 0) return PSF_ERR_SHAPE;
    if (!K || !V || !Kp || !Vp || !table || !lengths) return PSF_ERR_NULL;
    const uint32_t pieces = (uint32_t)(c.row_bytes() / 16);
    if ((long long)n * pieces > 0x7fffffffll || (long long)c.seqs * c.kv_heads > 0x7fffffffll) return PSF_ERR_UNSUPPORTED;
    if (!aligned16({K, V, Kp, Vp})) return PSF_ERR_ALIGNMENT;
    const uint32_t per = pieces * (uint32_t)n, pairs = (uint32_t)c.seqs * c.kv_heads;
    int fold = 1;                                           // pairs a workgroup, a power of two
    while (fold < 32 && per * fold * 2 <= (uint32_t)kCacheThreads) fold *= 2;
    const uint32_t lanes = kCacheThreads / fold, groups = (per + lanes - 1) / lanes, ys = (pairs + fold - 1) / fold;
    hipLaunchKernelGGL(cache_append_kernel, dim3(groups < 65536 ? groups : 65536, ys < 65535 ? ys : 65535), dim3(kCacheThreads), 0,
                       (hipStream_t)hip_stream, (const u4 *)K, (const u4 *)V, (u4 *)Kp, (u4 *)Vp, table, lengths, counts, c, n,
                       fast_div(pieces), fast_div(c.page), fast_div(c.kv_heads), fold);
    PSF_LAUNCH_CHECK();
    return PSF_OK;
}

psf_status psf_cache_fork(const psf_cache_desc *desc, int32_t forks, void *Kp, void *Vp, int32_t *table, int32_t *lengths,
                          const int32_t *parents, const int32_t *children, const int32_t *fresh, void *hip_stream)
{
    Cache c;
    const psf_status st = make_cache(desc, &c);
    if (st != PSF_OK) return st;
    if (forks <= 0) return PSF_ERR_SHAPE;
    if (forks > 65535) return PSF_ERR_UNSUPPORTED;
    if (!Kp || !Vp || !table || !lengths || !parents || !children || !fresh) return PSF_ERR_NULL;
    if (!aligned16({Kp, Vp})) return PSF_ERR_ALIGNMENT;
    const size_t pieces = c.page_bytes() / 16;
    hipLaunchKernelGGL(cache_fork_kernel, dim3(page_parts(pieces), forks), dim3(kCacheThreads), 0, (hipStream_t)hip_stream,
                       (u4 *)Kp, (u4 *)Vp, table, lengths, parents, children, fresh, c, pieces);
    PSF_LAUNCH_CHECK();
    return PSF_OK;
}

size_t psf_cache_compact_workspace_bytes(const psf_cache_desc *desc)
{
    Cache c;
    if (make_cache(desc, &c) != PSF_OK) return 0;
    return align_up(64 + (size_t)c.pages * 3 * sizeof(int32_t), 256);
}

psf_status psf_cache_compact(const psf_cache_desc *desc, void *Kp, void *Vp, const int32_t *table, const int32_t *lengths,
                             int32_t *new_table, int32_t *live, void *workspace, size_t workspace_bytes, void *hip_stream)
{
    Cache c;
    const psf_status st = make_cache(desc, &c);
    if (st != PSF_OK) return st;
    if (!Kp || !Vp || !table || !lengths || !new_table || !live || !workspace) return PSF_ERR_NULL;
    if (workspace_bytes < psf_cache_compact_workspace_bytes(desc)) return PSF_ERR_WORKSPACE;
    if (((uintptr_t)workspace & 255u) != 0) return PSF_ERR_WORKSPACE;
    if (!aligned16({Kp, Vp})) return PSF_ERR_ALIGNMENT;
    int32_t *n_moves = (int32_t *)workspace;
    int32_t *from = n_moves + 16, *to = from + c.pages, *place = to + c.pages;
    hipStream_t s = (hipStream_t)hip_stream;
    hipLaunchKernelGGL(cache_plan_kernel, dim3(1), dim3(kPlanThreads), 0, s, table, lengths, c, live, n_moves, from, to, place);
    PSF_LAUNCH_CHECK();
    const size_t pieces = c.page_bytes() / 16;
    const uint32_t parts = page_parts(pieces);
    const uint64_t most = (uint64_t)c.pages * parts / 2 + 1;  // moves there can be: as many as free pages
    const uint64_t entries = ((uint64_t)c.seqs * c.cols + kCacheThreads - 1) / kCacheThreads;
    const uint64_t want = most > entries ? most : entries;
    hipLaunchKernelGGL(cache_move_kernel, dim3((uint32_t)(want < 2048 ? want : 2048)), dim3(kCacheThreads), 0, s, (u4 *)Kp,
                       (u4 *)Vp, table, lengths, new_table, c, pieces, parts, live, n_moves, from, to, place, fast_div(c.cols),
                       fast_div(c.page));
    PSF_LAUNCH_CHECK();
    return PSF_OK;
}

}  // extern "C"
