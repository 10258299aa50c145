// Layer normalisation of rows, forward and backward (the step the paper puts before the attention,
// Section 2.1): with mean m and deviation s = sqrt(var + eps) of a row x of w columns, u = (x - m) / s,
//   y = u weight + bias,   dx = (g - <g>/w - u <g u>/w) / s with g = dy weight,
//   dweight = sum over rows of dy u,   dbias = sum over rows of dy.
// Bound by memory: one read and one write of the rows forward, two reads and one write backward.  A row lives
// in the registers of G lanes (16-byte pieces, piece k of a row with lane k mod G), so it is read once and its
// statistics are formed from the values themselves (mean first, then the squares around it), all sums in fp32.
#include <initializer_list>
#include <type_traits>
#include "psf_internal.h"

namespace psf {
namespace {

constexpr int kNormThreads = 256;
constexpr int kNormWide = 256;             // lanes of a row that takes a whole workgroup

// 16 bytes of a row.  Rows need no alignment beyond their type's: global loads and stores of whole
// pieces may start at any address on this hardware.
template <typename T> struct Piece;
template <> struct Piece<float> {
    static constexpr int N = 4;
    typedef uint32_t raw __attribute__((ext_vector_type(4), aligned(4)));
    static __device__ __forceinline__ void get(raw v, float (&x)[4])
    {
#pragma unroll
        for (int e = 0; e < 4; ++e) x[e] = __uint_as_float(v[e]);
    }
    static __device__ __forceinline__ raw put(const float (&x)[4])
    {
        raw v;
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = __float_as_uint(x[e]);
        return v;
    }
};
template <> struct Piece<bf16_t> {
    static constexpr int N = 8;
    typedef uint32_t raw __attribute__((ext_vector_type(4), aligned(2)));
    typedef __bf16 two __attribute__((ext_vector_type(2)));
    typedef float ftwo __attribute__((ext_vector_type(2)));
    static __device__ __forceinline__ void get(raw v, float (&x)[8])
    {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            x[2 * e] = __uint_as_float(v[e] << 16);
            x[2 * e + 1] = __uint_as_float(v[e] & 0xffff0000u);
        }
    }
    static __device__ __forceinline__ raw put(const float (&x)[8])
    {
        raw v;
#pragma unroll
        for (int e = 0; e < 4; ++e)
            v[e] = __builtin_bit_cast(uint32_t, __builtin_convertvector(ftwo{x[2 * e], x[2 * e + 1]}, two));
        return v;
    }
};

// Columns c .. c + N - 1 of a row; those from `width` on are zero (only the last piece of a row has any).
template <typename T>
__device__ __forceinline__ typename Piece<T>::raw norm_load(const T *row, int c, int width)
{
    constexpr int N = Piece<T>::N;
    if (c + N <= width) return *(const typename Piece<T>::raw *)(row + c);
    T v[N];
#pragma unroll
    for (int e = 0; e < N; ++e) v[e] = c + e < width ? row[c + e] : (T)0;
    typename Piece<T>::raw r;
    __builtin_memcpy(&r, v, 16);
    return r;
}
template <typename T>
__device__ __forceinline__ void norm_store(T *row, int c, int width, const float (&x)[Piece<T>::N])
{
    constexpr int N = Piece<T>::N;
    if (c + N <= width) {
        *(typename Piece<T>::raw *)(row + c) = Piece<T>::put(x);
        return;
    }
#pragma unroll
    for (int e = 0; e < N; ++e)
        if (c + e < width) store_f(row, c + e, x[e]);
}

template <int CTRL>
__device__ __forceinline__ float dpp(float x)
{
    return __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(x), CTRL, 0xf, 0xf, true));
}
// Sum over aligned groups of G lanes, in all of them: neighbours, pairs, then mirrored halves of 8 and
// 16 lanes (where all lanes of a half agree already), then the rows of 16.
template <int G>
__device__ __forceinline__ float sum_lanes(float x)
{
    if constexpr (G >= 2) x += dpp<0xB1>(x);            // quad_perm 1,0,3,2
    if constexpr (G >= 4) x += dpp<0x4E>(x);            // quad_perm 2,3,0,1
    if constexpr (G >= 8) x += dpp<0x141>(x);           // row_half_mirror
    if constexpr (G >= 16) x += dpp<0x140>(x);          // row_mirror
    if constexpr (G >= 32) {
        const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
        x = __uint_as_float(a[0]) + __uint_as_float(a[1]);
    }
    if constexpr (G >= 64) {
        const auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
        x = __uint_as_float(a[0]) + __uint_as_float(a[1]);
    }
    return x;
}
// Sums over the G lanes of a row: K of them for each of R rows.  A row that takes the workgroup adds its four
// waves' sums in LDS; all threads of the workgroup call this, the same number of times.
template <int G, int K>
__device__ __forceinline__ void sum_row(float (&x)[K], float (*lds)[K])
{
#pragma unroll
    for (int k = 0; k < K; ++k) x[k] = sum_lanes<(G < 64 ? G : 64)>(x[k]);
    if constexpr (G == kNormWide) {
        __syncthreads();                                // the previous sums have been read
        if ((threadIdx.x & 63) == 0)
#pragma unroll
            for (int k = 0; k < K; ++k) lds[threadIdx.x >> 6][k] = x[k];
        __syncthreads();
#pragma unroll
        for (int k = 0; k < K; ++k) x[k] = (lds[0][k] + lds[1][k]) + (lds[2][k] + lds[3][k]);
    }
}

// R rows in flight for every G lanes.  PER pieces a lane: columns (k G + lane) N of piece k.
template <typename T, int G, int PER, int R>
__global__ __launch_bounds__(kNormThreads) void norm_fwd_kernel(const T *x, const T *weight, const T *bias, T *y,
                                                                float2 *stats, int64_t rows, int width, float eps)
{
    constexpr int N = Piece<T>::N, ROWS = kNormThreads / G;
    __shared__ float lds[4][R];
    const int lane = threadIdx.x % G;
    const float inv_w = 1.0f / (float)width;
    // (one pass but for calls of more rows than a launch has workgroups for)
    for (int64_t at = (int64_t)blockIdx.x * (ROWS * R); at < rows; at += (int64_t)gridDim.x * (ROWS * R)) {
        const int64_t first = at + threadIdx.x / G;
        typename Piece<T>::raw raw[R][PER];
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const int64_t row = first + r * ROWS;
            const T *src = x + (row < rows ? row : rows - 1) * width;      // (rows that are not there: the last one, unused)
#pragma unroll
            for (int k = 0; k < PER; ++k)
                if ((k * G + lane) * N < width) raw[r][k] = norm_load(src, (k * G + lane) * N, width);
        }
        float s[R];
#pragma unroll
        for (int r = 0; r < R; ++r) {
            s[r] = 0.f;
#pragma unroll
            for (int k = 0; k < PER; ++k)
                if ((k * G + lane) * N < width) {
                    float v[N];
                    Piece<T>::get(raw[r][k], v);
#pragma unroll
                    for (int e = 0; e < N; ++e) s[r] += v[e];              // (zeros behind the row)
                }
        }
        sum_row<G, R>(s, lds);
        float mean[R];
#pragma unroll
        for (int r = 0; r < R; ++r) {
            mean[r] = s[r] * inv_w;
            s[r] = 0.f;
#pragma unroll
            for (int k = 0; k < PER; ++k) {
                const int c = (k * G + lane) * N;
                if (c < width) {
                    float v[N];
                    Piece<T>::get(raw[r][k], v);
#pragma unroll
                    for (int e = 0; e < N; ++e) {
                        const float t = c + e < width ? v[e] - mean[r] : 0.f;
                        s[r] += t * t;
                    }
                }
            }
        }
        sum_row<G, R>(s, lds);
        float inv[R];
#pragma unroll
        for (int r = 0; r < R; ++r) {
            inv[r] = 1.0f / sqrtf(s[r] * inv_w + eps);
            const int64_t row = first + r * ROWS;
            if (stats && lane == 0 && row < rows) stats[row] = make_float2(mean[r], inv[r]);
        }
#pragma unroll
        for (int k = 0; k < PER; ++k) {
            const int c = (k * G + lane) * N;
            if (c >= width) continue;
            float w[N], b[N];
            Piece<T>::get(norm_load(weight, c, width), w);
            if (bias) Piece<T>::get(norm_load(bias, c, width), b);
            else
#pragma unroll
                for (int e = 0; e < N; ++e) b[e] = 0.f;
#pragma unroll
            for (int r = 0; r < R; ++r) {
                const int64_t row = first + r * ROWS;
                if (row >= rows) continue;
                float v[N];
                Piece<T>::get(raw[r][k], v);
#pragma unroll
                for (int e = 0; e < N; ++e) v[e] = (v[e] - mean[r]) * inv[r] * w[e] + b[e];
                norm_store(y + row * width, c, width, v);
            }
        }
    }
}

// Gradient of the rows, and this workgroup's share of the gradients of weight and bias: a lane keeps the sums of its
// columns over the rows it walks (steps of ROWS R rows, gridDim.x workgroups side by side), the workgroup adds
// its lanes at the end.  partial [workgroups][2][width]; the order of all sums is fixed.
template <typename T, int G, int PER, int R>
__global__ __launch_bounds__(kNormThreads) void norm_bwd_kernel(const T *x, const T *weight, const float2 *stats, const T *dy,
                                                                T *dx, float *partial, int64_t rows, int width)
{
    constexpr int N = Piece<T>::N, ROWS = kNormThreads / G;
    __shared__ float lds[4][2 * R];
    __shared__ float fold[G < kNormWide ? kNormThreads * (N + 1) : 1];
    const int lane = threadIdx.x % G;
    const float inv_w = 1.0f / (float)width;
    float dw[PER][N], db[PER][N];
#pragma unroll
    for (int k = 0; k < PER; ++k)
#pragma unroll
        for (int e = 0; e < N; ++e) dw[k][e] = db[k][e] = 0.f;
    const int64_t step = (int64_t)gridDim.x * (ROWS * R);
    for (int64_t at = (int64_t)blockIdx.x * (ROWS * R); at < rows; at += step) {
        typename Piece<T>::raw rx[R][PER], rg[R][PER];
        float2 st[R];
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const int64_t row = at + r * ROWS + threadIdx.x / G, safe = row < rows ? row : rows - 1;
            st[r] = stats[safe];
#pragma unroll
            for (int k = 0; k < PER; ++k) {
                const int c = (k * G + lane) * N;
                if (c < width) {
                    rx[r][k] = norm_load(x + safe * width, c, width);
                    rg[r][k] = norm_load(dy + safe * width, c, width);
                }
            }
        }
        float s[2 * R];
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const bool there = at + r * ROWS + threadIdx.x / G < rows;
            s[2 * r] = s[2 * r + 1] = 0.f;
#pragma unroll
            for (int k = 0; k < PER; ++k) {
                const int c = (k * G + lane) * N;
                if (c >= width) continue;
                float v[N], g[N], w[N];
                Piece<T>::get(rx[r][k], v);
                Piece<T>::get(rg[r][k], g);
                Piece<T>::get(norm_load(weight, c, width), w);
#pragma unroll
                for (int e = 0; e < N; ++e) {
                    const float u = (v[e] - st[r].x) * st[r].y;        // (times g = 0 behind the row)
                    if (there) {
                        dw[k][e] += g[e] * u;
                        db[k][e] += g[e];
                    }
                    s[2 * r] += g[e] * w[e];
                    s[2 * r + 1] += g[e] * w[e] * u;
                }
            }
        }
        sum_row<G, 2 * R>(s, lds);
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const int64_t row = at + r * ROWS + threadIdx.x / G;
            if (row >= rows) continue;
            const float c1 = s[2 * r] * inv_w, c2 = s[2 * r + 1] * inv_w;
#pragma unroll
            for (int k = 0; k < PER; ++k) {
                const int c = (k * G + lane) * N;
                if (c >= width) continue;
                float v[N], g[N], w[N];
                Piece<T>::get(rx[r][k], v);
                Piece<T>::get(rg[r][k], g);
                Piece<T>::get(norm_load(weight, c, width), w);
#pragma unroll
                for (int e = 0; e < N; ++e) {
                    const float u = (v[e] - st[r].x) * st[r].y;
                    v[e] = (g[e] * w[e] - c1 - u * c2) * st[r].y;
                }
                norm_store(dx + row * width, c, width, v);
            }
        }
    }
    float *out = partial + (size_t)blockIdx.x * 2 * width;
#pragma unroll
    for (int k = 0; k < PER; ++k)
#pragma unroll
        for (int what = 0; what < 2; ++what) {
            float v[N];
#pragma unroll
            for (int e = 0; e < N; ++e) v[e] = what == 0 ? dw[k][e] : db[k][e];
            if constexpr (G < kNormWide) {
                __syncthreads();
#pragma unroll
                for (int e = 0; e < N; ++e) fold[threadIdx.x * (N + 1) + e] = v[e];
                __syncthreads();
                if (threadIdx.x < G)
#pragma unroll 1
                    for (int r = 1; r < ROWS; ++r)
#pragma unroll
                        for (int e = 0; e < N; ++e) v[e] += fold[(threadIdx.x + r * G) * (N + 1) + e];
            }
            if (threadIdx.x < G)
#pragma unroll
                for (int e = 0; e < N; ++e) {
                    const int c = (k * G + lane) * N + e;
                    if (c < width) out[(size_t)what * width + c] = v[e];
                }
        }
}

// dweight, dbias: the workgroups' shares added, 16 columns a workgroup, 16 slices of the shares side by side.
template <typename T>
__global__ __launch_bounds__(kNormThreads) void norm_sum_kernel(const float *partial, int shares, int width, T *dweight,
                                                                T *dbias)
{
    __shared__ float lds[16][17];
    const int c = blockIdx.x * 16 + threadIdx.x % 16, slice = threadIdx.x / 16;
    const size_t cols = 2 * (size_t)width;
    float v = 0.f;
    if (c < (int)cols)
#pragma unroll 8
        for (int i = slice; i < shares; i += 16) v += partial[i * cols + c];
    lds[slice][threadIdx.x % 16] = v;
    __syncthreads();
    if (slice == 0 && c < (int)cols) {
        for (int i = 1; i < 16; ++i) v += lds[i][threadIdx.x];
        if (c < width) store_f(dweight, c, v);
        else if (dbias) store_f(dbias, c - width, v);
    }
}

// Lanes of a row and pieces a lane: as few lanes as hold the row with one piece each, up to a wave; then up to
// four pieces a lane, then the workgroup.  go(G, PER).
template <typename T, class F>
psf_status norm_shape(int width, F &&go)
{
    const int pieces = (width + Piece<T>::N - 1) / Piece<T>::N;
    auto with = [&](auto g, auto per) { return go(g, per); };
    if (pieces <= 8) return with(std::integral_constant<int, 8>{}, std::integral_constant<int, 1>{});
    if (pieces <= 16) return with(std::integral_constant<int, 16>{}, std::integral_constant<int, 1>{});
    if (pieces <= 32) return with(std::integral_constant<int, 32>{}, std::integral_constant<int, 1>{});
    if (pieces <= 64) return with(std::integral_constant<int, 64>{}, std::integral_constant<int, 1>{});
    if (pieces <= 128) return with(std::integral_constant<int, 64>{}, std::integral_constant<int, 2>{});
    if (pieces <= 192) return with(std::integral_constant<int, 64>{}, std::integral_constant<int, 3>{});
    if (pieces <= 256) return with(std::integral_constant<int, 64>{}, std::integral_constant<int, 4>{});
    if (pieces <= 512) return with(std::integral_constant<int, kNormWide>{}, std::integral_constant<int, 2>{});
    if (pieces <= 1024) return with(std::integral_constant<int, kNormWide>{}, std::integral_constant<int, 4>{});
    if constexpr (PSF_NORM_MAX_WIDTH / Piece<T>::N > 1024) return with(std::integral_constant<int, kNormWide>{}, std::integral_constant<int, 8>{});
    return PSF_ERR_UNSUPPORTED;                             // (not reached: check())
}

// Rows in flight for every group of lanes: enough bytes a lane to cover the memory's latency.
template <int PER> constexpr int rows_fwd() { return PER == 1 ? 4 : PER <= 2 ? 2 : 1; }
template <int PER> constexpr int rows_bwd() { return PER == 1 ? 2 : 1; }

template <typename T>
psf_status fwd_launch(int64_t rows, int width, float eps, const void *x, const void *weight, const void *bias, void *y,
                      float *stats, hipStream_t s)
{
    return norm_shape<T>(width, [&](auto g, auto per) -> psf_status {
        constexpr int G = decltype(g)::value, PER = decltype(per)::value, R = rows_fwd<PER>();
        const int64_t each = kNormThreads / G * R, need = (rows + each - 1) / each, most = 1 << 23;   // (work-items below 2^32)
        hipLaunchKernelGGL((norm_fwd_kernel<T, G, PER, R>), dim3((uint32_t)(need < most ? need : most)), dim3(kNormThreads), 0, s,
                           (const T *)x, (const T *)weight, (const T *)bias, (T *)y, (float2 *)stats, rows, width, eps);
        PSF_LAUNCH_CHECK();
        return PSF_OK;
    });
}

template <typename T>
int bwd_workgroups(int64_t rows, int width)
{
    int64_t each = 1;
    (void)norm_shape<T>(width, [&](auto g, auto per) {
        each = kNormThreads / decltype(g)::value * rows_bwd<decltype(per)::value>();
        return PSF_OK;
    });
    const int64_t need = (rows + each - 1) / each;
    return (int)(need < 1024 ? need : 1024);
}

template <typename T>
psf_status bwd_launch(int64_t rows, int width, const void *x, const void *weight, const float *stats, const void *dy,
                      void *dx, void *dweight, void *dbias, float *partial, hipStream_t s)
{
    const int groups = bwd_workgroups<T>(rows, width);
    const psf_status st = norm_shape<T>(width, [&](auto g, auto per) -> psf_status {
        constexpr int G = decltype(g)::value, PER = decltype(per)::value, R = rows_bwd<PER>();
        hipLaunchKernelGGL((norm_bwd_kernel<T, G, PER, R>), dim3(groups), dim3(kNormThreads), 0, s, (const T *)x,
                           (const T *)weight, (const float2 *)stats, (const T *)dy, (T *)dx, partial, rows, width);
        PSF_LAUNCH_CHECK();
        return PSF_OK;
    });
    if (st != PSF_OK) return st;
    hipLaunchKernelGGL((norm_sum_kernel<T>), dim3((2 * width + 15) / 16), dim3(kNormThreads), 0, s, partial, groups, width,
                       (T *)dweight, (T *)dbias);
    PSF_LAUNCH_CHECK();
    return PSF_OK;
}

psf_status check(int64_t rows, int32_t width, int32_t dtype)
{
    if (rows <= 0 || width <= 0) return PSF_ERR_SHAPE;
    if (dtype != PSF_F32 && dtype != PSF_BF16) return PSF_ERR_UNSUPPORTED;
    if (width > PSF_NORM_MAX_WIDTH || rows > 0x7fffffff) return PSF_ERR_UNSUPPORTED;
    return PSF_OK;
}

// rows start at multiples of their type's size
bool aligned_to(int32_t dtype, std::initializer_list<const void *> tensors)
{
    for (const void *p : tensors)
        if (((uintptr_t)p & (dtype == PSF_F32 ? 3u : 1u)) != 0) return false;
    return true;
}

}  // namespace
}  // namespace psf

using namespace psf;

extern "C" {

psf_status psf_layer_norm_fwd(int64_t rows, int32_t width, int32_t dtype, float eps, const void *x, const void *weight,
                              const void *bias, void *y, float *stats, void *hip_stream)
{
    const psf_status st = check(rows, width, dtype);
    if (st != PSF_OK) return st;
    if (!(eps > 0.0f)) return PSF_ERR_UNSUPPORTED;
    if (!x || !weight || !y) return PSF_ERR_NULL;
    if (!aligned_to(dtype, {x, weight, bias, y}) || ((uintptr_t)stats & 7u) != 0) return PSF_ERR_ALIGNMENT;
    return dtype == PSF_F32 ? fwd_launch<float>(rows, width, eps, x, weight, bias, y, stats, (hipStream_t)hip_stream)
                            : fwd_launch<bf16_t>(rows, width, eps, x, weight, bias, y, stats, (hipStream_t)hip_stream);
}

size_t psf_layer_norm_bwd_workspace_bytes(int64_t rows, int32_t width, int32_t dtype)
{
    if (check(rows, width, dtype) != PSF_OK) return 0;
    const int groups = dtype == PSF_F32 ? bwd_workgroups<float>(rows, width) : bwd_workgroups<bf16_t>(rows, width);
    return align_up((size_t)groups * 2 * width * sizeof(float), 256);
}

psf_status psf_layer_norm_bwd(int64_t rows, int32_t width, int32_t dtype, const void *x, const void *weight,
                              const float *stats, const void *dy, void *dx, void *dweight, void *dbias, void *workspace,
                              size_t workspace_bytes, void *hip_stream)
{
    const psf_status st = check(rows, width, dtype);
    if (st != PSF_OK) return st;
    if (!x || !weight || !stats || !dy || !dx || !dweight || !workspace) return PSF_ERR_NULL;
    if (workspace_bytes < psf_layer_norm_bwd_workspace_bytes(rows, width, dtype)) return PSF_ERR_WORKSPACE;
    if (((uintptr_t)workspace & 255u) != 0) return PSF_ERR_WORKSPACE;
    if (!aligned_to(dtype, {x, weight, dy, dx, dweight, dbias}) || ((uintptr_t)stats & 7u) != 0) return PSF_ERR_ALIGNMENT;
    float *partial = (float *)workspace;
    return dtype == PSF_F32
               ? bwd_launch<float>(rows, width, x, weight, stats, dy, dx, dweight, dbias, partial, (hipStream_t)hip_stream)
               : bwd_launch<bf16_t>(rows, width, x, weight, stats, dy, dx, dweight, dbias, partial, (hipStream_t)hip_stream);
}

}  // extern "C"
