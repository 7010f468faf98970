// pex_norm.hip -- layer norm: forward pass, backward pass with the per-example statistics of scale and offset.
//
// Forward, a row x of d values:  mu = mean(x), r = 1 / sqrt(mean((x - mu)^2) + eps), y = (x - mu) r gamma + beta.
// Backward, with xh = (x - mu) r and w = g gamma:  dx = r (w - mean(w) - xh mean(w xh));
//   scale:  v_b[j] = sum_t g[b,t,j] xh[b,t,j],  offset: v_b[j] = sum_t g[b,t,j],  s = sum_b phi(v_b)  (phi as in pex_vec_stat).
//
// Bound by HBM: two bytes of traffic per byte of X forward, three backward, a dozen operations per value.  So every value is read
// once: a row lives in the registers of the lanes that share it, both passes over it (mean, then the sum of squared
// differences: no cancellation where the mean is large) run there, in fp32, and one rounding to the storage type ends it.
// Measured (of 4.9 TB/s, the rate of a large copy): forward bf16 32768 x 4096 106 us = 5.1 TB/s, fp32 4000 x 1001 6.9 us = 4.6 TB/s (from
// the last cache); backward bf16 65536 x 768 69 us = 4.4 TB/s, 32768 x 2048 88 us = 4.6 TB/s, fp32 4000 x 1002 15.6 us, 5 of them the
// second launch, which adds up the columns.  One row of 768: 4 us, the launch.
//   * A row belongs to LANES lanes of a block of THREADS, N chunks of VEC values (16 bytes) each: one wave for short rows, so that
//     no barrier is needed, a block of up to 512 for long ones.  The next row of a lane is loaded before the sums of the present one.
//   * Backward, a block owns a range of rows of one example; every lane owns its columns, keeps their two sums in registers
//     over the whole range, and the block writes them once: B * ranges * d floats each, which the second pass of pex_vec_stat turns
//     into the statistics.  Fixed order of additions, no atomics.
//   * Rows whose width is no multiple of a chunk: chunks at any element's alignment (a dwordx4 access needs no more), and the last one
//     ends with the row.  What it shares with its neighbour counts once in the sums and is written twice, the same bits.
#include <type_traits>

#include "pex_internal.h"

namespace pex {
namespace {

typedef __attribute__((ext_vector_type(4))) unsigned int uint4_t;
typedef __attribute__((ext_vector_type(4))) float float4_t;
typedef __attribute__((ext_vector_type(2))) float float2_t;
typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2_t;
typedef uint4_t __attribute__((aligned(2))) uint4_at2;     // a chunk at any element's address
typedef uint4_t __attribute__((aligned(4))) uint4_at4;
typedef float4_t __attribute__((aligned(4))) float4_at4;

template <typename T> struct Chunk;
template <> struct Chunk<uint16_t> { static constexpr int N = 8; typedef uint4_at2 loose_t; };
template <> struct Chunk<float> { static constexpr int N = 4; typedef uint4_at4 loose_t; };

__device__ __forceinline__ uint16_t narrow(float f, uint16_t) { return __builtin_bit_cast(uint16_t, (__bf16)f); }
__device__ __forceinline__ float narrow(float f, float) { return f; }

// 16 bytes of a row as they are: values [j, j + VEC), zeros past the end of the row (of `d` values)
template <typename T>
__device__ __forceinline__ uint4_t load_chunk(const T* row, int64_t j, int64_t d)
{
    typedef typename Chunk<T>::loose_t loose_t;
    constexpr int V = Chunk<T>::N;
    uint4_t u = {0, 0, 0, 0};
    if (j + V <= d) u = *(const loose_t*)(row + j);
    else {
#pragma unroll
        for (int e = 0; e < V - 1; ++e)
            if (j + e < d) {
                if constexpr (sizeof(T) == 2) u[e / 2] |= (uint32_t)row[j + e] << (16 * (e & 1));
                else u[e] = __float_as_uint(row[j + e]);
            }
    }
    return u;
}

template <typename T>
__device__ __forceinline__ float value_of(const uint4_t& u, int e)
{
    if constexpr (sizeof(T) == 2) return __uint_as_float(e & 1 ? u[e / 2] & 0xffff0000u : u[e / 2] << 16);
    else return __uint_as_float(u[e]);
}

template <typename T>
__device__ __forceinline__ void store_chunk(T* row, int64_t j, int64_t d, const float (&v)[Chunk<T>::N])
{
    typedef typename Chunk<T>::loose_t loose_t;
    constexpr int V = Chunk<T>::N;
    if (j + V <= d) {
        uint4_t u;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            if constexpr (sizeof(T) == 2) u[e] = __builtin_bit_cast(uint32_t, __builtin_convertvector((float2_t{v[2 * e], v[2 * e + 1]}), bf16x2_t));
            else u[e] = __float_as_uint(v[e]);
        }
        *(loose_t*)(row + j) = u;
    } else {
#pragma unroll
        for (int e = 0; e < V - 1; ++e)
            if (j + e < d) row[j + e] = narrow(v[e], T{});
    }
}

// `n` floats of a parameter vector from column j; `other` where there is no vector or no column
template <int V>
__device__ __forceinline__ void load_param(const float* p, int64_t j, int64_t d, float other, float (&v)[V])
{
    if (p && j + V <= d) {
#pragma unroll
        for (int q = 0; q < V / 4; ++q) {
            const float4_t f = *(const float4_at4*)(p + j + 4 * q);
#pragma unroll
            for (int e = 0; e < 4; ++e) v[4 * q + e] = f[e];
        }
    } else {
#pragma unroll
        for (int e = 0; e < V; ++e) v[e] = p && j + e < d ? p[j + e] : other;
    }
}

// Sums of NV values over the LANES lanes of a row.  LANES > 64: through LDS, in the order of the waves; `slot` alternates, so that
// one barrier per call is enough (a wave writes a slot again only after a barrier that follows every read of it).
template <int LANES, int THREADS, int NV>
__device__ __forceinline__ void row_sum(float (&s)[NV], float (*red)[THREADS / 64][NV], int& slot)
{
#pragma unroll
    for (int k = 0; k < NV; ++k)
#pragma unroll
        for (int o = 32; o >= 1; o >>= 1) s[k] += __shfl_xor(s[k], o);
    if constexpr (LANES > 64) {
        static_assert(LANES == THREADS, "rows of several waves have the block to themselves");
        const int wave = threadIdx.x >> 6;
        if ((threadIdx.x & 63) == 0)
#pragma unroll
            for (int k = 0; k < NV; ++k) red[slot][wave][k] = s[k];
        __syncthreads();
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            s[k] = 0.f;
#pragma unroll
            for (int w = 0; w < THREADS / 64; ++w) s[k] += red[slot][w][k];
        }
        slot ^= 1;
    }
}

// Where the N chunks of a lane lie in a row of d >= V values, and how many values at the front of each are not its own: none but of the chunk
// that ends with the row, all of one past it (which reads the row's last chunk and writes nothing)
template <int V, int LANES, int N>
struct Columns {
    int at[N], skip[N];
    __device__ __forceinline__ Columns(int lane, int d)
    {
#pragma unroll
        for (int n = 0; n < N; ++n) {
            const int j = (n * LANES + lane) * V;
            at[n] = min(j, d - V);
            skip[n] = min(j - at[n], V);
        }
    }
    __device__ __forceinline__ bool has(int n) const { return skip[n] < V; }
    __device__ __forceinline__ bool own(int n, int e) const { return e >= skip[n]; }
};
template <typename T>
__device__ __forceinline__ uint4_t load_at(const T* row, int at) { return *(const typename Chunk<T>::loose_t*)(row + at); }
template <typename T>
__device__ __forceinline__ void store_at(T* row, int at, const float (&v)[Chunk<T>::N])
{
    uint4_t u;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        if constexpr (sizeof(T) == 2) u[e] = __builtin_bit_cast(uint32_t, __builtin_convertvector((float2_t{v[2 * e], v[2 * e + 1]}), bf16x2_t));
        else u[e] = __float_as_uint(v[e]);
    }
    *(typename Chunk<T>::loose_t*)(row + at) = u;
}

template <typename T, int LANES, int THREADS, int N>
__global__ __launch_bounds__(THREADS) void norm_kernel(const T* X, const float* __restrict__ gamma, const float* __restrict__ beta, int64_t rows, int d,
                                                       float eps, T* Y, float* __restrict__ mean_out, float* __restrict__ rstd_out)
{
    constexpr int V = Chunk<T>::N, GROUPS = THREADS / LANES;
    __shared__ float red[2][THREADS / 64][1];
    const int lane = threadIdx.x % LANES, group = __builtin_amdgcn_readfirstlane((int)threadIdx.x / LANES);
    const Columns<V, LANES, N> col(lane, d);
    const int64_t step = (int64_t)gridDim.x * GROUPS;
    int64_t row = (int64_t)blockIdx.x * GROUPS + group;
    int slot = 0;
    float ga[N][V], be[N][V];
#pragma unroll
    for (int n = 0; n < N; ++n) {
        load_param(gamma, col.at[n], d, 1.f, ga[n]);
        load_param(beta, col.at[n], d, 0.f, be[n]);
    }
    uint4_t raw[N];
    auto load = [&](int64_t r) {
#pragma unroll
        for (int n = 0; n < N; ++n) raw[n] = load_at(X + r * d, col.at[n]);
    };
    if (row < rows) load(row);
    const float inv = 1.f / (float)d;
    for (; row < rows; row += step) {      // rows of several waves: the same `row` in the whole block
        float x[N][V];
        float s[1] = {0.f};
#pragma unroll
        for (int n = 0; n < N; ++n)
#pragma unroll
            for (int e = 0; e < V; ++e) {
                x[n][e] = value_of<T>(raw[n], e);
                s[0] += col.own(n, e) ? x[n][e] : 0.f;
            }
        if (row + step < rows) load(row + step);
        row_sum<LANES, THREADS, 1>(s, red, slot);
        const float mu = s[0] * inv;
        s[0] = 0.f;
#pragma unroll
        for (int n = 0; n < N; ++n)
#pragma unroll
            for (int e = 0; e < V; ++e) {
                x[n][e] -= mu;
                const float t = col.own(n, e) ? x[n][e] : 0.f;
                s[0] = fmaf(t, t, s[0]);
            }
        row_sum<LANES, THREADS, 1>(s, red, slot);
        const float rstd = 1.f / sqrtf(s[0] * inv + eps);
#pragma unroll
        for (int n = 0; n < N; ++n) {
            float y[V];
#pragma unroll
            for (int e = 0; e < V; ++e) y[e] = fmaf(x[n][e] * rstd, ga[n][e], be[n][e]);
            if (col.has(n)) store_at(Y + row * d, col.at[n], y);
        }
        if (lane == 0) {
            if (mean_out) mean_out[row] = mu;
            if (rstd_out) rstd_out[row] = rstd;
        }
    }
}

// Rows too long for registers: a block takes a row at a time, which it reads three times (the second and third time from the caches)
template <typename T>
__global__ __launch_bounds__(1024) void norm_long_kernel(const T* X, const float* __restrict__ gamma, const float* __restrict__ beta, int64_t rows, int64_t d,
                                                         float eps, T* Y, float* __restrict__ mean_out, float* __restrict__ rstd_out)
{
    constexpr int V = Chunk<T>::N;
    __shared__ float red[2][16][1];
    int slot = 0;
    const float inv = 1.f / (float)d;
    for (int64_t row = blockIdx.x; row < rows; row += gridDim.x) {
        const T* x = X + row * d;
        float s[1] = {0.f};
        for (int64_t j = (int64_t)threadIdx.x * V; j < d; j += 1024 * V) {
            const uint4_t u = load_chunk(x, j, d);
#pragma unroll
            for (int e = 0; e < V; ++e) s[0] += value_of<T>(u, e);
        }
        row_sum<1024, 1024, 1>(s, red, slot);
        const float mu = s[0] * inv;
        s[0] = 0.f;
        for (int64_t j = (int64_t)threadIdx.x * V; j < d; j += 1024 * V) {
            const uint4_t u = load_chunk(x, j, d);
#pragma unroll
            for (int e = 0; e < V; ++e) {
                const float t = j + e < d ? value_of<T>(u, e) - mu : 0.f;
                s[0] = fmaf(t, t, s[0]);
            }
        }
        row_sum<1024, 1024, 1>(s, red, slot);
        const float rstd = 1.f / sqrtf(s[0] * inv + eps);
        for (int64_t j = (int64_t)threadIdx.x * V; j < d; j += 1024 * V) {
            const uint4_t u = load_chunk(x, j, d);
            float ga[V], be[V], y[V];
            load_param(gamma, j, d, 1.f, ga);
            load_param(beta, j, d, 0.f, be);
#pragma unroll
            for (int e = 0; e < V; ++e) y[e] = fmaf((value_of<T>(u, e) - mu) * rstd, ga[e], be[e]);
            store_chunk(Y + row * d, j, d, y);
        }
        if (threadIdx.x == 0) {
            if (mean_out) mean_out[row] = mu;
            if (rstd_out) rstd_out[row] = rstd;
        }
    }
}

// Block (range, example): rows [range * per_range, ..) of the example's T.  partial_s, partial_o: [B][ranges][d]
template <typename T, int LANES, int THREADS, int N, bool STATS>
__global__ __launch_bounds__(THREADS, LANES == 64 && N <= 2 ? 4 : 2) void norm_grad_kernel(
    const T* G, const T* X, const float* __restrict__ mean, const float* __restrict__ rstd, const float* __restrict__ gamma, int64_t rows_of_example, int d,
    int ranges, int64_t per_range, T* dX, float* __restrict__ partial_s, float* __restrict__ partial_o)
{
    constexpr int V = Chunk<T>::N, GROUPS = THREADS / LANES;
    __shared__ float red[2][THREADS / 64][2];
    const int lane = threadIdx.x % LANES, group = __builtin_amdgcn_readfirstlane((int)threadIdx.x / LANES);
    const Columns<V, LANES, N> col(lane, d);
    const int64_t example = blockIdx.x / ranges, range = blockIdx.x % ranges;
    const int64_t t0 = range * per_range, t1 = t0 + per_range < rows_of_example ? t0 + per_range : rows_of_example;
    const int64_t first = example * rows_of_example;
    int slot = 0;
    float ga[N][V], as[STATS ? N : 1][V], ao[STATS ? N : 1][V];
#pragma unroll
    for (int n = 0; n < N; ++n) load_param(gamma, col.at[n], d, 1.f, ga[n]);
#pragma unroll
    for (int n = 0; n < (STATS ? N : 1); ++n)
#pragma unroll
        for (int e = 0; e < V; ++e) as[n][e] = ao[n][e] = 0.f;
    uint4_t rg[N], rx[N];
    float mu = 0.f, rs = 0.f;
    auto load = [&](int64_t r) {
#pragma unroll
        for (int n = 0; n < N; ++n) {
            rg[n] = load_at(G + r * d, col.at[n]);
            rx[n] = load_at(X + r * d, col.at[n]);
        }
        mu = mean[r];
        rs = rstd[r];
    };
    const float inv = 1.f / (float)d;
    int64_t t = t0 + group;
    if (t < t1) load(first + t);
    for (; t < t1; t += GROUPS) {
        // the row in hand stays as it is: w and xh are formed twice, before and after their sums, which costs less than their registers
        uint4_t hg[N], hx[N];
        const float m = mu, r = rs;
#pragma unroll
        for (int n = 0; n < N; ++n) {
            hg[n] = rg[n];
            hx[n] = rx[n];
        }
        if (t + GROUPS < t1) load(first + t + GROUPS);
        float s[2] = {0.f, 0.f};
#pragma unroll
        for (int n = 0; n < N; ++n)
#pragma unroll
            for (int e = 0; e < V; ++e) {
                const float g = col.own(n, e) ? value_of<T>(hg[n], e) : 0.f, xh = (value_of<T>(hx[n], e) - m) * r, w = g * ga[n][e];
                if (STATS) {
                    as[n][e] = fmaf(g, xh, as[n][e]);
                    ao[n][e] += g;
                    asm volatile("" : "+v"(as[n][e]), "+v"(ao[n][e]));       // here, not after the sums, up to which g and xh would be kept
                }
                s[0] += w;
                s[1] = fmaf(w, xh, s[1]);
            }
        row_sum<LANES, THREADS, 2>(s, red, slot);
        const float c1 = s[0] * inv, c2 = s[1] * inv;
#pragma unroll
        for (int n = 0; n < N; ++n) {
            asm volatile("" : "+v"(hg[n]), "+v"(hx[n]));       // (the compiler would keep what it formed above)
            float y[V];
#pragma unroll
            for (int e = 0; e < V; ++e) {
                const float xh = (value_of<T>(hx[n], e) - m) * r, w = value_of<T>(hg[n], e) * ga[n][e];
                y[e] = r * (w - fmaf(xh, c2, c1));
            }
            if (col.has(n)) store_at(dX + (first + t) * d, col.at[n], y);
        }
    }
    if constexpr (STATS) {
        if constexpr (GROUPS > 1) {        // the groups' sums in their order, through LDS
            __shared__ float sums[GROUPS - 1][LANES * V];
#pragma unroll
            for (int which = 0; which < 2; ++which)
#pragma unroll
                for (int n = 0; n < N; ++n) {
                    float (&a)[V] = which ? ao[n] : as[n];
                    __syncthreads();
                    if (group > 0)
#pragma unroll
                        for (int e = 0; e < V; ++e) sums[group - 1][e * LANES + lane] = a[e];
                    __syncthreads();
                    if (group == 0)
#pragma unroll
                        for (int k = 0; k < GROUPS - 1; ++k)
#pragma unroll
                            for (int e = 0; e < V; ++e) a[e] += sums[k][e * LANES + lane];
                }
        }
        if (group == 0) {
            float* ps = partial_s + (int64_t)blockIdx.x * d;
            float* po = partial_o + (int64_t)blockIdx.x * d;
#pragma unroll
            for (int n = 0; n < N; ++n) {
                if (col.skip[n] == 0) {
#pragma unroll
                    for (int e = 0; e < V; e += 4) {
                        store_at<float>(ps, col.at[n] + e, {as[n][e], as[n][e + 1], as[n][e + 2], as[n][e + 3]});
                        store_at<float>(po, col.at[n] + e, {ao[n][e], ao[n][e + 1], ao[n][e + 2], ao[n][e + 3]});
                    }
                } else {
#pragma unroll
                    for (int e = 0; e < V; ++e)
                        if (e >= col.skip[n]) {
                            ps[col.at[n] + e] = as[n][e];
                            po[col.at[n] + e] = ao[n][e];
                        }
                }
            }
        }
    }
}

// Rows too long for registers: the input cotangents, a row of a block at a time
template <typename T>
__global__ __launch_bounds__(1024) void norm_grad_long_kernel(const T* G, const T* X, const float* __restrict__ mean, const float* __restrict__ rstd,
                                                              const float* __restrict__ gamma, int64_t rows, int64_t d, T* dX)
{
    constexpr int V = Chunk<T>::N;
    __shared__ float red[2][16][2];
    int slot = 0;
    for (int64_t row = blockIdx.x; row < rows; row += gridDim.x) {
        const T *g = G + row * d, *x = X + row * d;
        const float mu = mean[row], r = rstd[row];
        float s[2] = {0.f, 0.f};
        auto each = [&](int64_t j, auto f) {
            const uint4_t ug = load_chunk(g, j, d), ux = load_chunk(x, j, d);
            float ga[V];
            load_param(gamma, j, d, 1.f, ga);
#pragma unroll
            for (int e = 0; e < V; ++e) f(e, value_of<T>(ug, e) * ga[e], j + e < d ? (value_of<T>(ux, e) - mu) * r : 0.f);
        };
        for (int64_t j = (int64_t)threadIdx.x * V; j < d; j += 1024 * V)
            each(j, [&](int, float w, float xh) {
                s[0] += w;
                s[1] = fmaf(w, xh, s[1]);
            });
        row_sum<1024, 1024, 2>(s, red, slot);
        const float c1 = s[0] / (float)d, c2 = s[1] / (float)d;
        for (int64_t j = (int64_t)threadIdx.x * V; j < d; j += 1024 * V) {
            float y[V];
            each(j, [&](int e, float w, float xh) { y[e] = r * (w - fmaf(xh, c2, c1)); });
            store_chunk(dX + row * d, j, d, y);
        }
    }
}

// ... and the sums over a range of rows: a lane owns VEC columns.  Runs before the kernel above (dX may be G or X).
template <typename T>
__global__ __launch_bounds__(256) void norm_grad_columns_kernel(const T* G, const T* X, const float* __restrict__ mean, const float* __restrict__ rstd,
                                                                int64_t rows_of_example, int64_t d, int64_t parts, int ranges, int64_t per_range,
                                                                float* __restrict__ partial_s, float* __restrict__ partial_o)
{
    constexpr int V = Chunk<T>::N;
    const int64_t j = ((int64_t)blockIdx.x * 256 + threadIdx.x) * V;
    if (j >= d) return;
    for (int64_t part = blockIdx.y; part < parts; part += gridDim.y) {
        const int64_t example = part / ranges, t0 = part % ranges * per_range, t1 = t0 + per_range < rows_of_example ? t0 + per_range : rows_of_example;
        float as[V], ao[V];
#pragma unroll
        for (int e = 0; e < V; ++e) as[e] = ao[e] = 0.f;
        for (int64_t t = t0; t < t1; ++t) {
            const int64_t row = example * rows_of_example + t;
            const uint4_t ug = load_chunk(G + row * d, j, d), ux = load_chunk(X + row * d, j, d);
            const float mu = mean[row], r = rstd[row];
#pragma unroll
            for (int e = 0; e < V; ++e) {
                const float g = value_of<T>(ug, e);
                as[e] = fmaf(g, j + e < d ? (value_of<T>(ux, e) - mu) * r : 0.f, as[e]);
                ao[e] += g;
            }
        }
        float* ps = partial_s + part * d;
        float* po = partial_o + part * d;
#pragma unroll
        for (int e = 0; e < V; ++e)
            if (j + e < d) {
                ps[j + e] = as[e];
                po[j + e] = ao[e];
            }
    }
}

// How the lanes share a row of d values: calls go(lanes, threads, chunks of a lane), all integral constants; false where it is too long
template <typename T, bool GRAD, typename F>
bool with_shape(int64_t d, F&& go)
{
    if (d < Chunk<T>::N) return false;       // (the kernels of long rows take any width)
    const int64_t chunks = (d + Chunk<T>::N - 1) / Chunk<T>::N;
    using std::integral_constant;
    auto as = [&](auto lanes, auto threads, auto n) { go(lanes, threads, n); return true; };
#define PEX_NORM_SHAPE(LANES, THREADS, N) return as(integral_constant<int, LANES>{}, integral_constant<int, THREADS>{}, integral_constant<int, N>{})
    if (chunks <= 64) PEX_NORM_SHAPE(64, 256, 1);
    if (chunks <= 128) PEX_NORM_SHAPE(64, 256, 2);
    if (chunks <= 256) PEX_NORM_SHAPE(64, 256, 4);
    if (chunks <= 512) PEX_NORM_SHAPE(256, 256, 2);
    if (chunks <= 1024) PEX_NORM_SHAPE(512, 512, 2);
    // 256 registers hold 16 columns of a lane with their sums (32 spill), 32 without
    if constexpr (sizeof(T) == 4 || !GRAD)
        if (chunks <= 2048) PEX_NORM_SHAPE(512, 512, 4);
    if constexpr (sizeof(T) == 4 && !GRAD)
        if (chunks <= 4096) PEX_NORM_SHAPE(512, 512, 8);
#undef PEX_NORM_SHAPE
    return false;
}

constexpr int64_t NORM_BLOCKS = 2048;       // eight blocks of 256 per compute unit: what is resident at once
constexpr int64_t LONG_BLOCKS = (int64_t)1 << 20;       // of 1024: a launch holds fewer than 2^32 threads

template <typename T>
hipError_t norm_typed(const T* X, const float* gamma, const float* beta, int64_t rows, int64_t d, float eps, T* Y, float* mean, float* rstd, hipStream_t stream)
{
    const bool fits = with_shape<T, false>(d, [&](auto lanes, auto threads, auto n) {
        constexpr int L = decltype(lanes)::value, TH = decltype(threads)::value;
        const int64_t need = (rows + TH / L - 1) / (TH / L), most = NORM_BLOCKS * 256 / TH;
        norm_kernel<T, L, TH, decltype(n)::value><<<dim3((unsigned)(need < most ? need : most)), dim3(TH), 0, stream>>>(X, gamma, beta, rows, (int)d, eps, Y, mean, rstd);
    });
    if (!fits) norm_long_kernel<T><<<dim3((unsigned)(rows < LONG_BLOCKS ? rows : LONG_BLOCKS)), dim3(1024), 0, stream>>>(X, gamma, beta, rows, d, eps, Y, mean, rstd);
    return hipGetLastError();
}

template <typename T>
hipError_t norm_grad_typed(const T* G, const T* X, const float* mean, const float* rstd, const float* gamma, int64_t B, int64_t rows, int64_t d, const NormGradPlan& plan,
                           T* dX, float* partial_s, float* partial_o, hipStream_t stream)
{
    const bool fits = with_shape<T, true>(d, [&](auto lanes, auto threads, auto n) {
        constexpr int L = decltype(lanes)::value, TH = decltype(threads)::value, N = decltype(n)::value;
        auto go = [&](auto kern) {
            kern<<<dim3((unsigned)(B * plan.ranges)), dim3(TH), 0, stream>>>(G, X, mean, rstd, gamma, rows, (int)d, plan.ranges, plan.per_range, dX, partial_s, partial_o);
        };
        partial_s ? go(norm_grad_kernel<T, L, TH, N, true>) : go(norm_grad_kernel<T, L, TH, N, false>);
    });
    if (fits) return hipGetLastError();
    constexpr int64_t cols = 256 * Chunk<T>::N;
    if (partial_s) {
        const int64_t parts = B * plan.ranges;
        const dim3 grid((unsigned)((d + cols - 1) / cols), (unsigned)(parts < 65535 ? parts : 65535));
        norm_grad_columns_kernel<T><<<grid, dim3(256), 0, stream>>>(G, X, mean, rstd, rows, d, parts, plan.ranges, plan.per_range, partial_s, partial_o);
    }
    norm_grad_long_kernel<T><<<dim3((unsigned)(B * rows < LONG_BLOCKS ? B * rows : LONG_BLOCKS)), dim3(1024), 0, stream>>>(G, X, mean, rstd, gamma, B * rows, d, dX);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_layer_norm(const void* X, const float* gamma, const float* beta, int64_t rows, int64_t d, pex_dtype dt, float eps, void* Y, float* mean,
                             float* rstd, hipStream_t stream)
{
    return dt == PEX_F32 ? norm_typed((const float*)X, gamma, beta, rows, d, eps, (float*)Y, mean, rstd, stream)
                         : norm_typed((const uint16_t*)X, gamma, beta, rows, d, eps, (uint16_t*)Y, mean, rstd, stream);
}

NormGradPlan plan_layer_norm_grad(int64_t B, int64_t T, int64_t d, pex_dtype dt)
{
    // as many blocks as are resident at once (no second, mostly empty round of them); at least four rows per group of lanes, so that
    // the partial sums, eight bytes a column, stay a part of the traffic.  Waves of a SIMD by the registers of the kernels with sums.
    int groups = 1, threads = 1024, waves = 4;
    auto shape = [&](auto lanes, auto th, auto n) {
        constexpr int N = decltype(n)::value;
        threads = decltype(th)::value;
        groups = threads / decltype(lanes)::value;
        waves = dt == PEX_BF16 ? (N == 1 ? 7 : N == 2 ? 4 : 2) : (N == 1 ? 8 : N == 2 ? 4 : N == 4 && threads == 256 ? 3 : 2);
    };
    dt == PEX_F32 ? with_shape<float, true>(d, shape) : with_shape<uint16_t, true>(d, shape);
    int64_t ranges = 256 * (waves * 256 / threads) / B;
    const int64_t most = (T + 4 * groups - 1) / (4 * groups);
    if (ranges > most) ranges = most;
    if (ranges < 1) ranges = 1;
    NormGradPlan p{};
    p.per_range = (T + ranges - 1) / ranges;
    p.ranges = (int)((T + p.per_range - 1) / p.per_range);
    p.partial_bytes = ((size_t)B * (size_t)p.ranges * (size_t)d * sizeof(float) + 255) & ~(size_t)255;
    return p;
}

hipError_t launch_layer_norm_grad(const void* G, const void* X, const float* mean, const float* rstd, const float* gamma, int64_t B, int64_t T, int64_t d,
                                  pex_dtype dt, const NormGradPlan& plan, void* dX, const VecSums& scale, const VecSums& offset, void* workspace,
                                  hipStream_t stream)
{
    float* ps = (float*)workspace;
    float* po = (float*)((char*)workspace + plan.partial_bytes);
    if (!workspace) po = nullptr;
    const hipError_t e = dt == PEX_F32 ? norm_grad_typed((const float*)G, (const float*)X, mean, rstd, gamma, B, T, d, plan, (float*)dX, ps, po, stream)
                                       : norm_grad_typed((const uint16_t*)G, (const uint16_t*)X, mean, rstd, gamma, B, T, d, plan, (uint16_t*)dX, ps, po, stream);
    if (e != hipSuccess || !workspace) return e;
    return launch_vec_finalize_pair(B, d, plan.ranges, ps, po, scale, offset, stream);
}

}  // namespace pex
