// Layer norm over the rows of a matrix: forward, and backward with the gradients of weight and bias.  See include/qsr.h.
#include <cuda_runtime.h>

#include <algorithm>
#include <atomic>
#include <cmath>

#include "checks.h"
#include "rows.cuh"

namespace qsr {

namespace {

constexpr int kBlocks = 148;          // most partial sums of the weight's gradient: a block on each multiprocessor
constexpr int kResident = 592;        // blocks of the forward kernel whose warps stay: four on each
constexpr int kMaxHeld = 4;           // most granules of eight elements that a thread holds of a row
constexpr int kMaxThreads = 1024;

struct Params {
    const void *x, *dy;
    void *y, *dx;
    const void *w, *b;
    float *mean, *rstd;
    float *partial;                   // [blocks, 2, width]
    int64_t rows, x_stride, y_stride, dy_stride, dx_stride;
    int32_t width, granules, wtype;
    int32_t wvec;                     // weight and bias aligned to eight elements
    int32_t want_weight, want_bias;
    float eps, inverse;            // inverse: one over the width
    long long patience;               // clocks that a wait for a row's copy may take
};

// Weights and biases: read by every row, so through the cache.
template <bool VEC>
__device__ __forceinline__ void weights(float (&v)[8], const void *base, float otherwise, int lane, int lanes, int k, int width, int type, bool vec)
{
    const int c0 = column<VEC>(lane, lanes, k, 0);
    if (!base) {
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = otherwise;
    } else if (VEC && vec && c0 + 8 <= width) {
        Raw8 r;
        const uint4 *p = reinterpret_cast<const uint4 *>(static_cast<const char *>(base) + size_t(c0) * (type == QSR_F32 ? 4 : 2));
        const uint4 lo = __ldg(p), hi = type == QSR_F32 ? __ldg(p + 1) : make_uint4(0, 0, 0, 0);
        r.w[0] = lo.x; r.w[1] = lo.y; r.w[2] = lo.z; r.w[3] = lo.w;
        r.w[4] = hi.x; r.w[5] = hi.y; r.w[6] = hi.z; r.w[7] = hi.w;
        widen8(v, r, type);
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int c = column<VEC>(lane, lanes, k, j);
            v[j] = c < width ? widen1(load1(base, c, type), type) : otherwise;
        }
    }
}

// Eight elements of a row, zeros if there is no such row.
template <bool VEC, bool FULL>
__device__ __forceinline__ void fetch_row(Raw8 &r, const void *row, int lane, int lanes, int k, bool live, int width, int type)
{
    if (!FULL) fetch<VEC>(r, row, lane, lanes, k, live ? width : 0, type);
    else if (live) load8(r, row, column<true>(lane, lanes, k, 0), type);
    else
#pragma unroll
        for (int j = 0; j < 8; ++j) r.w[j] = 0u;
}
template <bool VEC, bool FULL>
__device__ __forceinline__ void put_row(void *row, const float (&v)[8], int lane, int lanes, int k, int width, int type)
{
    if (FULL) store8(row, column<true>(lane, lanes, k, 0), v, type);
    else put<VEC>(row, v, lane, lanes, k, width, type);
}

// Sum over the lanes that share a row: 2^n lanes of a warp, or all threads of the block (scratch: a float per warp).
__device__ __forceinline__ float row_sum(float v, int lanes, float *scratch)
{
    if (lanes >= 32) v = warp_sum(v);
    else
        for (int d = lanes >> 1; d; d >>= 1) v += __shfl_xor_sync(0xffffffffu, v, d);
    if (lanes <= 32) return v;
    __syncthreads();                              // the sums before this one have been read
    if ((threadIdx.x & 31) == 0) scratch[threadIdx.x >> 5] = v;
    __syncthreads();
    const int n = lanes >> 5;
    v = (threadIdx.x & 31) < n ? scratch[threadIdx.x & 31] : 0.0f;
    return warp_sum(v);
}

// 1 / sqrt(x) to about one unit in the last place: one step of Newton's method on the instruction's 22 bits.
__device__ __forceinline__ float inverse_root(float x)
{
    const float r = rsqrtf(x);
    return x > 1e-30f && x < 1e30f ? r * fmaf(-0.5f * x * r, r, 1.5f) : 1.0f / sqrtf(x);
}

// FULL kernels compare nothing with the width.  Forward: every thread has all its elements, the row is lanes * HELD whole granules.
// Backward: the row is whole granules, and a thread has one or none.

// A mean is off by some 2^-24 of the row's values, and with it every x - mean by the same, which the division by the spread makes large
// where the row is far from zero: 0.03 to 0.09 for rows of one value near 1000.  Rows whose mean is further from zero than so many
// standard deviations have the mean of what is left taken off too, and the variance taken anew.  For the others the error is within a few
// roundings: of fp32 from four on (some 2^-20), of fp16, whose roundings are 2^-11, from 64 on (2^-16).
template <typename T>
__device__ __forceinline__ bool far_from_zero(float mean, float rstd) { return fabsf(mean) * rstd > (sizeof(T) == 4 ? 4.0f : 64.0f); }

// That for rows in registers; x: what is left.  All lanes of a warp come here together, with rows of their own.
template <typename T, int HELD, bool VEC, bool FULL>
__device__ __forceinline__ void settle_row(float (&x)[HELD][8], float &mean, float &rstd, const Params &p, int lane, int lanes, float *scratch)
{
    const bool far = far_from_zero<T>(mean, rstd);
    if (!__any_sync(0xffffffffu, far)) return;                   // of rows that a block shares, the same for the block
    float s = 0.0f, q = 0.0f;
#pragma unroll
    for (int k = 0; k < HELD; ++k)
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (FULL || column<VEC>(lane, lanes, k, j) < p.width) s += x[k][j];
    const float left = row_sum(s, lanes, scratch) * p.inverse, rest = far ? left : 0.0f;
#pragma unroll
    for (int k = 0; k < HELD; ++k)
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            x[k][j] -= rest;
            if (FULL || column<VEC>(lane, lanes, k, j) < p.width) q = fmaf(x[k][j], x[k][j], q);
        }
    const float anew = inverse_root(fmaf(row_sum(q, lanes, scratch), p.inverse, p.eps));
    if (far) {
        mean += rest;
        rstd = anew;
    }
}

// Rows that fit in registers: HELD granules a thread, `lanes` threads a row (a power of two up to 32, or the whole block).  Mean and
// variance take two passes over the registers, and rows far from zero two more.
template <typename T, int HELD, bool VEC, bool FULL>
__global__ void __launch_bounds__(kMaxThreads) forward_kernel(const __grid_constant__ Params p, int lanes)
{
    __shared__ float scratch[32];
    constexpr int TYPE = Kind<T>::type;
    const int lane = int(threadIdx.x) & (lanes - 1);
    const int64_t row = int64_t(blockIdx.x) * (int(blockDim.x) / lanes) + int(threadIdx.x) / lanes;
    const bool live = row < p.rows;
    float x[HELD][8];
    float s = 0.0f;
    {
        Raw8 raw[HELD];
        const void *from = row_of<T>(p.x, live ? row : 0, p.x_stride);
#pragma unroll
        for (int k = 0; k < HELD; ++k) fetch_row<VEC, FULL>(raw[k], from, lane, lanes, k, live, p.width, TYPE);
#pragma unroll
        for (int k = 0; k < HELD; ++k) {
            widen8(x[k], raw[k], TYPE);
#pragma unroll
            for (int j = 0; j < 8; ++j) s += x[k][j];
        }
    }
    float mean = row_sum(s, lanes, scratch) * p.inverse;
    float q = 0.0f;
#pragma unroll
    for (int k = 0; k < HELD; ++k)
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            x[k][j] -= mean;
            if (FULL || column<VEC>(lane, lanes, k, j) < p.width) q = fmaf(x[k][j], x[k][j], q);
        }
    float rstd = inverse_root(fmaf(row_sum(q, lanes, scratch), p.inverse, p.eps));
    settle_row<T, HELD, VEC, FULL>(x, mean, rstd, p, lane, lanes, scratch);
    if (!live) return;
    if (lane == 0) {
        if (p.mean) p.mean[row] = mean;
        if (p.rstd) p.rstd[row] = rstd;
    }
    void *to = row_of<T>(p.y, row, p.y_stride);
#pragma unroll
    for (int k = 0; k < HELD; ++k) {
        if (!FULL && column<VEC>(lane, lanes, k, 0) >= p.width) break;
        float w[8], b[8];
        weights<VEC>(w, p.w, 1.0f, lane, lanes, k, p.width, p.wtype, p.wvec != 0);
        weights<VEC>(b, p.b, 0.0f, lane, lanes, k, p.width, p.wtype, p.wvec != 0);
#pragma unroll
        for (int j = 0; j < 8; ++j) w[j] = fmaf(x[k][j] * rstd, w[j], b[j]);
        put_row<VEC, FULL>(to, w, lane, lanes, k, p.width, TYPE);
    }
}

// The same for many rows of up to 1024 elements: warps that stay, with weight and bias in shared memory in fp32, each loading its next
// row while it works on one.  (A launch with a warp for every row waits for its weights as long as for its row.)
template <typename T, int HELD, bool VEC, bool FULL>
__global__ void __launch_bounds__(256, 4) forward_rows_kernel(const __grid_constant__ Params p, int lanes)
{
    // elements 8 g + 4 h .. + 3 of a granule g at [h][g]: neighbours' 16-byte accesses are adjacent
    __shared__ float4 ws[2][32 * HELD], bs[2][32 * HELD];
    constexpr int TYPE = Kind<T>::type;
    const auto slot = [](float4 (&a)[2][32 * HELD], int c) { return VEC ? reinterpret_cast<float *>(&a[(c >> 2) & 1][c >> 3]) + (c & 3) : reinterpret_cast<float *>(a) + c; };
    for (int c = threadIdx.x; c < p.width; c += 256) {
        *slot(ws, c) = p.w ? widen1(load1(p.w, c, p.wtype), p.wtype) : 1.0f;
        *slot(bs, c) = p.b ? widen1(load1(p.b, c, p.wtype), p.wtype) : 0.0f;
    }
    __syncthreads();
    const int lane = int(threadIdx.x) & (lanes - 1), groups = 256 / lanes;
    const int64_t step = int64_t(gridDim.x) * groups;
    Raw8 raw[HELD];
    const auto load = [&](int64_t row) {
        const bool live = row < p.rows;
        const void *from = row_of<T>(p.x, live ? row : 0, p.x_stride);
#pragma unroll
        for (int k = 0; k < HELD; ++k) fetch_row<VEC, FULL>(raw[k], from, lane, lanes, k, live, p.width, TYPE);
    };
    int64_t row = int64_t(blockIdx.x) * groups + int(threadIdx.x) / lanes;
    load(row);
    for (int64_t first = int64_t(blockIdx.x) * groups; first < p.rows; first += step, row += step) {        // `first`: the same for the block
        float x[HELD][8], s = 0.0f, q = 0.0f;
#pragma unroll
        for (int k = 0; k < HELD; ++k) {
            widen8(x[k], raw[k], TYPE);
#pragma unroll
            for (int j = 0; j < 8; ++j) s += x[k][j];
        }
        load(row + step);
        float mean = row_sum(s, lanes, nullptr) * p.inverse;
#pragma unroll
        for (int k = 0; k < HELD; ++k)
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                x[k][j] -= mean;
                if (FULL || column<VEC>(lane, lanes, k, j) < p.width) q = fmaf(x[k][j], x[k][j], q);
            }
        float rstd = inverse_root(fmaf(row_sum(q, lanes, nullptr), p.inverse, p.eps));
        settle_row<T, HELD, VEC, FULL>(x, mean, rstd, p, lane, lanes, nullptr);
        if (row >= p.rows) continue;
        if (lane == 0) {
            if (p.mean) p.mean[row] = mean;
            if (p.rstd) p.rstd[row] = rstd;
        }
        void *to = row_of<T>(p.y, row, p.y_stride);
#pragma unroll
        for (int k = 0; k < HELD; ++k) {
            if (!FULL && column<VEC>(lane, lanes, k, 0) >= p.width) break;
            float y[8];
            if (VEC) {
                const int g = lane + k * lanes;
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const float4 w = ws[h][g], b = bs[h][g];
                    y[4 * h] = fmaf(x[k][4 * h] * rstd, w.x, b.x);
                    y[4 * h + 1] = fmaf(x[k][4 * h + 1] * rstd, w.y, b.y);
                    y[4 * h + 2] = fmaf(x[k][4 * h + 2] * rstd, w.z, b.z);
                    y[4 * h + 3] = fmaf(x[k][4 * h + 3] * rstd, w.w, b.w);
                }
            } else {
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const int c = column<VEC>(lane, lanes, k, j);
                    y[j] = c < p.width ? fmaf(x[k][j] * rstd, *slot(ws, c), *slot(bs, c)) : 0.0f;
                }
            }
            put_row<VEC, FULL>(to, y, lane, lanes, k, p.width, TYPE);
        }
    }
}

// Rows of any length, read three times (from the caches after the first), five times if they are far from zero; one block a row.
template <typename T, bool VEC>
__global__ void __launch_bounds__(kMaxThreads) forward_long_kernel(const __grid_constant__ Params p)
{
    __shared__ float scratch[32];
    constexpr int TYPE = Kind<T>::type;
    const int lane = threadIdx.x, lanes = blockDim.x, steps = (p.granules + lanes - 1) / lanes;
    const void *from = row_of<T>(p.x, blockIdx.x, p.x_stride);
    float s = 0.0f, q = 0.0f, x[8];
    Raw8 r;
    for (int k = 0; k < steps; ++k) {
        fetch<VEC>(r, from, lane, lanes, k, p.width, TYPE);
        widen8(x, r, TYPE);
#pragma unroll
        for (int j = 0; j < 8; ++j) s += x[j];
    }
    const float mean = __fmul_rn(row_sum(s, lanes, scratch), p.inverse);          // one number in all that follows, not part of an fma
    float rest = 0.0f, rstd;                                     // rest: the mean of what is left
    const auto spread = [&] {
        q = 0.0f;
        for (int k = 0; k < steps; ++k) {
            fetch<VEC>(r, from, lane, lanes, k, p.width, TYPE);
            widen8(x, r, TYPE);
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (column<VEC>(lane, lanes, k, j) < p.width) q = fmaf(x[j] - mean - rest, x[j] - mean - rest, q);
        }
        rstd = inverse_root(fmaf(row_sum(q, lanes, scratch), p.inverse, p.eps));
    };
    spread();
    if (far_from_zero<T>(mean, rstd)) {                             // the same for the block
        s = 0.0f;
        for (int k = 0; k < steps; ++k) {
            fetch<VEC>(r, from, lane, lanes, k, p.width, TYPE);
            widen8(x, r, TYPE);
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (column<VEC>(lane, lanes, k, j) < p.width) s += x[j] - mean;
        }
        rest = __fmul_rn(row_sum(s, lanes, scratch), p.inverse);
        spread();
    }
    if (lane == 0) {
        if (p.mean) p.mean[blockIdx.x] = mean + rest;
        if (p.rstd) p.rstd[blockIdx.x] = rstd;
    }
    void *to = row_of<T>(p.y, blockIdx.x, p.y_stride);
    for (int k = 0; k < steps; ++k) {
        fetch<VEC>(r, from, lane, lanes, k, p.width, TYPE);
        widen8(x, r, TYPE);
        float w[8], b[8];
        weights<VEC>(w, p.w, 1.0f, lane, lanes, k, p.width, p.wtype, p.wvec != 0);
        weights<VEC>(b, p.b, 0.0f, lane, lanes, k, p.width, p.wtype, p.wvec != 0);
#pragma unroll
        for (int j = 0; j < 8; ++j) w[j] = fmaf((x[j] - mean - rest) * rstd, w[j], b[j]);
        put<VEC>(to, w, lane, lanes, k, p.width, TYPE);
    }
}

__device__ __forceinline__ void group_barrier(int group, int threads)
{
    asm volatile("bar.sync %0, %1;" ::"r"(group + 1), "r"(threads) : "memory");
}

// Two numbers to an instruction (sm_100).
__device__ __forceinline__ unsigned long long pair_of(float2 a) { return *reinterpret_cast<unsigned long long *>(&a); }
__device__ __forceinline__ float2 add2(float2 a, float2 b)
{
    float2 y;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(*reinterpret_cast<unsigned long long *>(&y)) : "l"(pair_of(a)), "l"(pair_of(b)));
    return y;
}
__device__ __forceinline__ float2 mul2(float2 a, float2 b)
{
    float2 y;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(*reinterpret_cast<unsigned long long *>(&y)) : "l"(pair_of(a)), "l"(pair_of(b)));
    return y;
}
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c)
{
    float2 y;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(*reinterpret_cast<unsigned long long *>(&y)) : "l"(pair_of(a)), "l"(pair_of(b)), "l"(pair_of(c)));
    return y;
}
struct Pairs { float2 v[4]; };
__device__ __forceinline__ void widen_pairs(Pairs &o, const Raw8 &r, int type)
{
#pragma unroll
    for (int j = 0; j < 4; ++j) o.v[j] = type == QSR_F32 ? make_float2(__uint_as_float(r.w[2 * j]), __uint_as_float(r.w[2 * j + 1])) : widen2(r.w[j], type);
}

// Sums of N values (2 or 4) over a warp: value i ends up in the lanes whose number has i in its upper bits.  N / 2 + N / 4 + ... exchanges
// instead of N for the first steps.
template <int N>
__device__ __forceinline__ float spread_sum(const float (&v)[N], int lane)
{
    float a[N];
#pragma unroll
    for (int i = 0; i < N; ++i) a[i] = v[i];
    int d = 16;
#pragma unroll
    for (int n = N; n > 1; n /= 2, d /= 2) {
        const bool upper = lane & d;
#pragma unroll
        for (int i = 0; i < n / 2; ++i) {
            const float mine = upper ? a[i + n / 2] : a[i], other = upper ? a[i] : a[i + n / 2];
            a[i] = mine + __shfl_xor_sync(0xffffffffu, other, d);
        }
    }
    for (; d; d /= 2) a[0] += __shfl_xor_sync(0xffffffffu, a[0], d);
    return a[0];
}

// A thread's eight columns in the backward pass: weights, and the column sums that stay in its registers.
struct Columns { float2 w[4], dw[4], db[4]; };
template <bool VEC>
__device__ __forceinline__ void start_columns(Columns &c, const Params &p, int lane, int lanes)
{
    float v[8];
    weights<VEC>(v, p.w, 1.0f, lane, lanes, 0, p.width, p.wtype, p.wvec != 0);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        c.w[j] = make_float2(v[2 * j], v[2 * j + 1]);
        c.dw[j] = c.db[j] = make_float2(0.0f, 0.0f);
    }
}
// a: x becomes x - mean; d: dy becomes dy w; sum, product: this thread's shares of the row's two sums.
template <bool VEC, bool FULL>
__device__ __forceinline__ void add_columns(Pairs &a, Pairs &d, Columns &c, float &sum, float &product, float mean, float rstd, int lane, int lanes, int width)
{
    const float2 minus = make_float2(-mean, -mean), times = make_float2(rstd, rstd);
    float2 s1 = make_float2(0.0f, 0.0f), s2 = s1;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        a.v[j] = add2(a.v[j], minus);
        float2 hat = mul2(a.v[j], times);
        if (!FULL) {       // beyond the row both are zero: a finite statistic gives no sum, one that is not finite is kept out
            if (column<VEC>(lane, lanes, 0, 2 * j) >= width) hat.x = 0.0f;
            if (column<VEC>(lane, lanes, 0, 2 * j + 1) >= width) hat.y = 0.0f;
        }
        c.dw[j] = fma2(d.v[j], hat, c.dw[j]);
        c.db[j] = add2(c.db[j], d.v[j]);
        d.v[j] = mul2(d.v[j], c.w[j]);
        s1 = add2(s1, d.v[j]);
        s2 = fma2(d.v[j], hat, s2);
    }
    sum = s1.x + s1.y;
    product = s2.x + s2.y;
}
// N sums over the `warps` warps of a group; at: [warps][N] of shared memory, which calls use two of in turn.
template <int N>
__device__ __forceinline__ void group_sums(float (&s)[N], float *at, int warps, int group, int lanes, int lane)
{
    constexpr int SHARE = 32 / N;                 // lanes that have the same value
    const float v = spread_sum(s, lane & 31);
    if ((lane & (SHARE - 1)) == 0) at[(lane >> 5) * N + (lane & 31) / SHARE] = v;
    group_barrier(group, lanes);
    if (warps <= 4) {
#pragma unroll
        for (int i = 0; i < N; ++i) s[i] = 0.0f;
        for (int u = 0; u < warps; ++u)
#pragma unroll
            for (int i = 0; i < N; ++i) s[i] += at[u * N + i];
    } else {
        const int u = lane & 31;
#pragma unroll
        for (int i = 0; i < N; ++i) s[i] = u < warps ? at[u * N + i] : 0.0f;
        const float all = spread_sum(s, u);
#pragma unroll
        for (int i = 0; i < N; ++i) s[i] = __shfl_sync(0xffffffffu, all, i * SHARE);
    }
}
__device__ __forceinline__ void row_gradient(float (&out)[8], const Pairs &a, const Pairs &d, float sum, float product, float inverse, float rstd)
{
    const float c1 = -sum * inverse, c2 = -product * inverse * rstd;
    const float2 along = make_float2(c2, c2), level = make_float2(c1, c1), times = make_float2(rstd, rstd);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const float2 v = mul2(fma2(a.v[j], along, add2(d.v[j], level)), times);
        out[2 * j] = v.x;
        out[2 * j + 1] = v.y;
    }
}
// The groups' column sums, joined in their order, to the block's partial sums.  shared: eight floats a thread.
template <bool VEC>
__device__ __forceinline__ void leave_columns(const Params &p, const Columns &c, float *shared, int groups, int group, int lane, int lanes)
{
    float *out = p.partial + int64_t(blockIdx.x) * 2 * p.width;
    for (int pass = 0; pass < 2; ++pass) {
        float v[8];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            v[2 * j] = pass ? c.db[j].x : c.dw[j].x;
            v[2 * j + 1] = pass ? c.db[j].y : c.dw[j].y;
        }
        if (groups > 1) {
            __syncthreads();
#pragma unroll
            for (int j = 0; j < 8; ++j) shared[j * blockDim.x + threadIdx.x] = v[j];
            __syncthreads();
            if (group == 0)
                for (int g = 1; g < groups; ++g)
#pragma unroll
                    for (int j = 0; j < 8; ++j) v[j] += shared[j * blockDim.x + g * lanes + lane];
        }
        if (group == 0)
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const int col = column<VEC>(lane, lanes, 0, j);
                if (col < p.width) out[int64_t(pass) * p.width + col] = v[j];
            }
    }
}

// Backward for rows of up to 8 x 1024 elements.  `lanes` threads (a power of two up to 32, or whole warps) take a row at a time, each thread
// the same eight columns of every row, so that the column sums stay in its registers; groups of lanes share a block, which leaves
// one partial sum for each column.  The next row is loaded while one is worked on.  12544 x 768 bf16: 15 us and 2 more for the sums of the blocks'
// sums (58 MB, 3.8 TB/s): bound by instructions (issue 65 %), and by its beginning and end, since a group has but eleven rows.
template <typename T, bool VEC, bool FULL, int THREADS>
__global__ void __launch_bounds__(THREADS) backward_kernel(const __grid_constant__ Params p, int lanes)
{
    extern __shared__ float shared[];             // a group's row sums: [groups][2][warps of a group][2]; then column sums
    constexpr int TYPE = Kind<T>::type;
    const int groups = int(blockDim.x) / lanes, group = int(threadIdx.x) / lanes, lane = int(threadIdx.x) - group * lanes;
    const int warps = lanes >> 5;
    const bool mine = column<VEC>(lane, lanes, 0, 0) < p.width;
    Columns c;
    start_columns<VEC>(c, p, lane, lanes);
    Raw8 x, dy;
    float next_mean, next_rstd;
    // rows below 2^31, and pointers that are moved on: the loop is short of instructions
    const unsigned rows = unsigned(p.rows), step = gridDim.x * unsigned(groups);
    unsigned row = blockIdx.x * unsigned(groups) + unsigned(group);
    const T *from_x = static_cast<const T *>(p.x) + int64_t(row) * p.x_stride, *from_dy = static_cast<const T *>(p.dy) + int64_t(row) * p.dy_stride;
    T *to = static_cast<T *>(p.dx) + int64_t(row) * p.dx_stride;
    const float *from_mean = p.mean + row, *from_rstd = p.rstd + row;
    const int64_t x_step = step * p.x_stride, dy_step = step * p.dy_stride, dx_step = step * p.dx_stride;
    const auto load = [&](unsigned at) {
        const bool live = at < rows && mine;
        fetch_row<VEC, FULL>(x, from_x, lane, lanes, 0, live, p.width, TYPE);
        fetch_row<VEC, FULL>(dy, from_dy, lane, lanes, 0, live, p.width, TYPE);
        next_mean = live ? *from_mean : 0.0f;
        next_rstd = live ? *from_rstd : 0.0f;
        from_x += x_step; from_dy += dy_step;
        from_mean += step; from_rstd += step;
    };
    int turn = 0;
    load(row);
    for (unsigned base = blockIdx.x * unsigned(groups); base < rows; base += step, row += step, to += dx_step) {       // `base`: the same for the block
        Pairs a, d;
        widen_pairs(a, x, TYPE);
        widen_pairs(d, dy, TYPE);
        const float mean = next_mean, rstd = next_rstd;
        load(row + step);
        float s[2];
        add_columns<VEC, FULL>(a, d, c, s[0], s[1], mean, rstd, lane, lanes, p.width);
        if (!p.dx) continue;
        if (lanes > 32) {
            group_sums(s, shared + (group * 2 + turn) * warps * 2, warps, group, lanes, lane);
            turn ^= 1;
        } else if (lanes == 32) {
            const float v = spread_sum(s, lane);
            s[0] = __shfl_sync(0xffffffffu, v, 0);
            s[1] = __shfl_sync(0xffffffffu, v, 16);
        } else {
#pragma unroll
            for (int k = 0; k < 2; ++k)
                for (int e = lanes >> 1; e; e >>= 1) s[k] += __shfl_xor_sync(0xffffffffu, s[k], e);
        }
        if (row >= rows || !mine) continue;
        float out[8];
        row_gradient(out, a, d, s[0], s[1], p.inverse, rstd);
        put_row<VEC, FULL>(to, out, lane, lanes, 0, p.width, TYPE);
    }
    if (p.partial) leave_columns<VEC>(p, c, shared, groups, group, lane, lanes);
}

// The same for aligned rows that a whole block takes: they come by bulk copies into a ring of shared memory, `stages` rows of x and dy
// ahead, issued by one thread, and are worked on ROWS at a time, whose sums cross the block together.  So many rows under way would not
// fit in registers beside the column sums.  Against the kernel above, which has one row ahead: 4099 x 5003 fp32 60 us instead of 66,
// 8192 x 4096 bf16 55 instead of 59, 4096 x 8192 bf16 56 instead of 76.  A multiprocessor's bulk copies follow one another at a few hundred
// clocks each, so that rows of which a block holds several at once gain nothing (12544 x 768 bf16: 21 to 24 us, when the kernel above took 18.4).  Bound
// by what a row costs its block in instructions and exchanges, beside the copies: 3.6 to 4.9 TB/s.
constexpr int kMaxStages = 8;
constexpr long long kPatience = 6000000000;       // clocks that a wait may take, some seconds
std::atomic<long long> g_patience{kPatience};     // of the launches to come; other than that only by the test hook

__device__ __forceinline__ bool copied(uint32_t bar, unsigned parity)
{
    uint32_t done;
    asm volatile("{.reg .pred p; mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2; selp.u32 %0, 1, 0, p;}" : "=r"(done) : "r"(bar), "r"(parity) : "memory");
    return done != 0;
}
// A limit of zero has run out at once, whether the copy is there or not.
__device__ __forceinline__ bool wait_for_copy(uint32_t bar, unsigned parity, long long patience)
{
    if (patience <= 0) return false;
    if (copied(bar, parity)) return true;
    for (const long long begin = clock64(); clock64() - begin < patience;)
        for (int i = 0; i < 64; ++i)
            if (copied(bar, parity)) return true;
    return false;
}
// Eight elements of a row in shared memory.  `left`: how many the row has from there on; behind it lies whatever follows it in memory.
template <typename T, bool FULL>
__device__ __forceinline__ void take_shared(Raw8 &r, uint32_t from, int left)
{
#pragma unroll
    for (int h = 0; h < int(sizeof(T)) / 2; ++h)
        asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(r.w[4 * h]), "=r"(r.w[4 * h + 1]), "=r"(r.w[4 * h + 2]), "=r"(r.w[4 * h + 3])
                     : "r"(from + h * 16) : "memory");
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        if (j < left || (FULL && left > 0)) continue;
        if (sizeof(T) == 4) r.w[j] = 0u;
        else r.w[j / 2] &= j & 1 ? 0xffffu : 0xffff0000u;
    }
}

template <typename T, bool FULL, int ROWS, int THREADS>
__global__ void __launch_bounds__(THREADS) backward_ring_kernel(const __grid_constant__ Params p, int stages)
{
    extern __shared__ __align__(128) char ring[];                // [stages][x, dy]
    __shared__ __align__(8) unsigned long long full[kMaxStages];
    __shared__ float sums[2][THREADS / 32][2 * ROWS];     // used in turn
    constexpr int TYPE = Kind<T>::type, BYTES = int(sizeof(T));
    const int lanes = int(blockDim.x), lane = int(threadIdx.x), left = p.width - lane * 8, slot = lanes * 8 * BYTES;
    const uint32_t bars = uint32_t(__cvta_generic_to_shared(full)), slots = uint32_t(__cvta_generic_to_shared(ring));
    // Copies are of 16 bytes and more: what follows a row up to there lies in the matrix, except behind the last row, whose end is
    // read as it is wanted.
    const auto issue = [&](int stage, int64_t row) {
        const unsigned n = unsigned(row + 1 < p.rows ? (p.width * BYTES + 15) & ~15 : p.width * BYTES & ~15);
        const uint32_t bar = bars + stage * 8, to = slots + stage * 2 * slot;
        asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(2 * n) : "memory");
        asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(to), "l"(row_of<T>(p.x, row, p.x_stride)), "r"(n),
                     "r"(bar) : "memory");
        asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(to + slot), "l"(row_of<T>(p.dy, row, p.dy_stride)),
                     "r"(n), "r"(bar) : "memory");
    };
    int under_way = 0;
    if (lane == 0) {
        for (int i = 0; i < stages; ++i) asm volatile("mbarrier.init.shared::cta.b64 [%0], 1;" ::"r"(bars + i * 8) : "memory");
        asm volatile("fence.mbarrier_init.release.cluster;\n\tfence.proxy.async.shared::cta;" ::: "memory");
        for (; under_way < stages && blockIdx.x + under_way * gridDim.x < p.rows; ++under_way) issue(under_way, blockIdx.x + under_way * gridDim.x);
    }
    Columns c;
    start_columns<true>(c, p, lane, lanes);
    float next_mean[ROWS], next_rstd[ROWS];
    const unsigned rows = unsigned(p.rows), step = gridDim.x;    // below 2^31, and pointers that are moved on: fewer instructions
    const float *from_mean = p.mean + blockIdx.x, *from_rstd = p.rstd + blockIdx.x;
    T *to = static_cast<T *>(p.dx) + int64_t(blockIdx.x) * p.dx_stride;
    const int64_t dx_step = step * p.dx_stride;
    const auto statistics = [&](unsigned row) {                  // zeros where there is no row, or no column
#pragma unroll
        for (int r = 0; r < ROWS; ++r) {
            const bool live = row + r * step < rows && left > 0;
            next_mean[r] = live ? *from_mean : 0.0f;
            next_rstd[r] = live ? *from_rstd : 0.0f;
            from_mean += step;
            from_rstd += step;
        }
    };
    statistics(blockIdx.x);
    __syncthreads();
    int turn = 0, stage = 0;
    unsigned phase = 0;
    bool all_came = true;
    for (unsigned row = blockIdx.x; row < rows; row += ROWS * step) {
        const int live = row + step < rows ? ROWS : 1;         // of ROWS, one or two
        float mean[ROWS], rstd[ROWS], s[2 * ROWS];
        Pairs a[ROWS], d[ROWS];
#pragma unroll
        for (int r = 0; r < ROWS; ++r) {
            mean[r] = next_mean[r];
            rstd[r] = next_rstd[r];
        }
        statistics(row + ROWS * step);
        int at = stage;
        unsigned parity = phase;
#pragma unroll
        for (int r = 0; r < ROWS; ++r) {
            Raw8 x, dy;
            if (r < live) {
                all_came = all_came && wait_for_copy(bars + at * 8, parity, p.patience);
                const uint32_t from = slots + at * 2 * slot + lane * 8 * BYTES;
                const unsigned here = row + r * step;
                if (!FULL && left < 8 && here + 1 == rows) {
                    fetch<true>(x, row_of<T>(p.x, here, p.x_stride), lane, lanes, 0, p.width, TYPE);
                    fetch<true>(dy, row_of<T>(p.dy, here, p.dy_stride), lane, lanes, 0, p.width, TYPE);
                } else {
                    take_shared<T, FULL>(x, from, left);
                    take_shared<T, FULL>(dy, from + slot, left);
                }
                if (++at == stages) { at = 0; parity ^= 1u; }
            } else
#pragma unroll
                for (int j = 0; j < 8; ++j) x.w[j] = dy.w[j] = 0u;
            widen_pairs(a[r], x, TYPE);
            widen_pairs(d[r], dy, TYPE);
            if (!all_came)                                       // a wait ran out: no number passes for a gradient, the columns' sums included
#pragma unroll
                for (int j = 0; j < 4; ++j) d[r].v[j] = make_float2(quiet_nan(), quiet_nan());
            add_columns<true, FULL>(a[r], d[r], c, s[2 * r], s[2 * r + 1], mean[r], rstd[r], lane, lanes, p.width);
        }
        if (p.dx) group_sums(s, sums[turn][0], lanes >> 5, 0, lanes, lane);
        else __syncthreads();
        turn ^= 1;
#pragma unroll
        for (int r = 0; r < ROWS; ++r) {                         // all threads have taken these rows
            if (r >= live || !all_came) break;
            under_way--;
            const unsigned next = row + unsigned(r + stages) * step;
            if (lane == 0 && next < rows) {
                issue(stage, next);
                under_way++;
            }
            if (++stage == stages) { stage = 0; phase ^= 1u; }
        }
        if (!p.dx || left <= 0) continue;
#pragma unroll
        for (int r = 0; r < ROWS; ++r, to += dx_step) {
            if (r >= live) break;
            float out[8];
            row_gradient(out, a[r], d[r], s[2 * r], s[2 * r + 1], p.inverse, rstd[r]);
            put_row<true, FULL>(to, out, lane, lanes, 0, p.width, TYPE);
        }
    }
    for (; lane == 0 && under_way > 0; --under_way) {            // a wait ran out: the copies under way are waited for, each with the limit once more
        wait_for_copy(bars + stage * 8, phase, kPatience);
        if (++stage == stages) { stage = 0; phase ^= 1u; }
    }
    if (p.partial) leave_columns<true>(p, c, nullptr, 1, 0, lane, lanes);
}

// Forward over many aligned rows, in the same way: blocks that stay, each thread with the weight and bias of its sixteen columns, so that a
// row's exchanges are few beside its elements.  Mean and variance take two passes over the registers.  8192 x 4096 bf16: 31 us (4.4 TB/s) instead of
// 37 with the first kernel above, 8192 x 5120 40 instead of 56, 4096 x 5120 fp32 31 instead of 35 (5.4 TB/s); eight columns a thread, two rows at a
// time: 37.  Bound by instructions (widening, exchanges, the loop) beside the copies.  (Backward, sixteen columns a thread leave
// too few warps: 64 us for 4099 x 5003 fp32 instead of 60, 73 for 8192 x 4096 bf16 instead of 56.)
//
// Rows far from zero are noted and come after up to 256 rows of the block, read once more: the registers for them here, where there is none to
// spare, would cost all rows (8192 x 5120 bf16 49 us instead of 40).  Nothing of such a row has been written, so that y may be x.  Where
// all rows are far, 8192 x 4096 bf16 takes 88 us.
constexpr int kFarRows = 256;
template <typename T, bool FULL, int THREADS>
__global__ void __launch_bounds__(THREADS, kMaxThreads / THREADS) forward_ring_kernel(const __grid_constant__ Params p, int stages)
{
    extern __shared__ __align__(128) char ring[];                // [stages] rows
    __shared__ __align__(8) unsigned long long full[kMaxStages];
    __shared__ float sums[2][THREADS / 32];                      // used in turn
    __shared__ unsigned far_rows[kFarRows], n_far;
    __shared__ float far_means[kFarRows];
    constexpr int TYPE = Kind<T>::type, BYTES = int(sizeof(T)), HELD = 2;
    const int lanes = int(blockDim.x), lane = int(threadIdx.x), warps = lanes >> 5, slot = HELD * lanes * 8 * BYTES;
    const uint32_t bars = uint32_t(__cvta_generic_to_shared(full)), slots = uint32_t(__cvta_generic_to_shared(ring));
    const unsigned rows = unsigned(p.rows), step = gridDim.x;    // below 2^31
    const auto issue = [&](int stage, unsigned row) {             // of the last row, whole 16 bytes, as above
        const unsigned n = unsigned(row + 1 < rows ? (p.width * BYTES + 15) & ~15 : p.width * BYTES & ~15);
        const uint32_t bar = bars + stage * 8;
        asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(n) : "memory");
        asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(slots + stage * slot),
                     "l"(row_of<T>(p.x, row, p.x_stride)), "r"(n), "r"(bar) : "memory");
    };
    int under_way = 0;
    if (lane == 0) {
        for (int i = 0; i < stages; ++i) asm volatile("mbarrier.init.shared::cta.b64 [%0], 1;" ::"r"(bars + i * 8) : "memory");
        asm volatile("fence.mbarrier_init.release.cluster;\n\tfence.proxy.async.shared::cta;" ::: "memory");
        for (; under_way < stages && blockIdx.x + under_way * step < rows; ++under_way) issue(under_way, blockIdx.x + under_way * step);
    }
    const auto left = [&](int k) { return p.width - (lane + k * lanes) * 8; };
    const auto block_sum = [&](float2 v, float *at) {
        const float mine = warp_sum(v.x + v.y);
        if ((lane & 31) == 0) at[lane >> 5] = mine;
        __syncthreads();
        return warp_sum((lane & 31) < warps ? at[lane & 31] : 0.0f);
    };
    if (lane == 0) n_far = 0;
    __syncthreads();
    int stage = 0;
    unsigned phase = 0;
    bool all_came = true;
    for (unsigned row = blockIdx.x; row < rows;) {
        const unsigned end = min(rows, row + kFarRows * step);
        Pairs w[HELD], b[HELD];
#pragma unroll
        for (int k = 0; k < HELD; ++k) {
            float v[8];
            weights<true>(v, p.w, 1.0f, lane, lanes, k, p.width, p.wtype, p.wvec != 0);
#pragma unroll
            for (int j = 0; j < 4; ++j) w[k].v[j] = make_float2(v[2 * j], v[2 * j + 1]);
            weights<true>(v, p.b, 0.0f, lane, lanes, k, p.width, p.wtype, p.wvec != 0);
#pragma unroll
            for (int j = 0; j < 4; ++j) b[k].v[j] = make_float2(v[2 * j], v[2 * j + 1]);
        }
        for (; row < end; row += step) {
            all_came = all_came && wait_for_copy(bars + stage * 8, phase, p.patience);
            Pairs x[HELD];
            float2 s = make_float2(0.0f, 0.0f), q = s;
#pragma unroll
            for (int k = 0; k < HELD; ++k) {
                Raw8 raw;
                if (!FULL && left(k) < 8 && row + 1 == rows) fetch<true>(raw, row_of<T>(p.x, row, p.x_stride), lane, lanes, k, p.width, TYPE);
                else take_shared<T, FULL>(raw, slots + stage * slot + (lane + k * lanes) * 8 * BYTES, left(k));
                widen_pairs(x[k], raw, TYPE);
                if (!all_came) x[k].v[0].x = quiet_nan();        // a wait ran out: no number passes for a result
#pragma unroll
                for (int j = 0; j < 4; ++j) s = add2(s, x[k].v[j]);
            }
            const float mean = block_sum(s, sums[0]) * p.inverse;
            if (all_came) {                                      // and all threads have taken this row
                under_way--;
                if (lane == 0 && row + stages * step < rows) {
                    issue(stage, row + stages * step);
                    under_way++;
                }
                if (++stage == stages) { stage = 0; phase ^= 1u; }
            }
#pragma unroll
            for (int k = 0; k < HELD; ++k) {
                if (FULL && left(k) <= 0) break;                 // nothing beyond the row
                const float2 minus = make_float2(-mean, -mean);
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    x[k].v[j] = add2(x[k].v[j], minus);
                    if (!FULL) {
                        if (2 * j >= left(k)) x[k].v[j].x = 0.0f;
                        if (2 * j + 1 >= left(k)) x[k].v[j].y = 0.0f;
                    }
                    q = fma2(x[k].v[j], x[k].v[j], q);
                }
            }
            const float rstd = inverse_root(fmaf(block_sum(q, sums[1]), p.inverse, p.eps));
            const bool far = far_from_zero<T>(mean, rstd);       // the same for the block
            if (lane == 0) {
                if (p.mean) p.mean[row] = mean;
                if (p.rstd) p.rstd[row] = rstd;
                if (far) {
                    far_rows[n_far] = row;
                    far_means[n_far++] = mean;
                }
            }
            void *to = row_of<T>(p.y, row, p.y_stride);
            const float2 times = make_float2(rstd, rstd);
#pragma unroll
            for (int k = 0; k < HELD; ++k) {
                if (left(k) <= 0 || far) break;
                float y[8];
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const float2 v = fma2(mul2(x[k].v[j], times), w[k].v[j], b[k].v[j]);
                    y[2 * j] = v.x;
                    y[2 * j + 1] = v.y;
                }
                put_row<true, FULL>(to, y, lane, lanes, k, p.width, TYPE);
            }
        }
        __syncthreads();                                         // what is noted is there, and all y before it is written
        const unsigned n = n_far;
#pragma unroll 1
        for (unsigned i = 0; i < n; ++i) {
            const unsigned row = far_rows[i];
            const float mean = far_means[i];
            float x[8], s = 0.0f, q = 0.0f;
            const auto take = [&](int k) {
                Raw8 raw;
                fetch<true>(raw, row_of<T>(p.x, row, p.x_stride), lane, lanes, k, p.width, TYPE);
                widen8(x, raw, TYPE);
            };
            const auto sum = [&](const auto &add) {
#pragma unroll 1
                for (int k = 0; k < HELD; ++k) {
                    take(k);
#pragma unroll
                    for (int j = 0; j < 8; ++j)
                        if (j < left(k)) add(x[j]);
                }
            };
            sum([&](float v) { s += v - mean; });
            const float rest = __fmul_rn(block_sum(make_float2(s, 0.0f), sums[0]), p.inverse);        // one number in all that follows, not part of an fma
            sum([&](float v) { q = fmaf(v - mean - rest, v - mean - rest, q); });
            const float rstd = inverse_root(fmaf(block_sum(make_float2(q, 0.0f), sums[1]), p.inverse, p.eps));
            if (lane == 0) {
                if (p.mean) p.mean[row] = mean + rest;
                if (p.rstd) p.rstd[row] = rstd;
            }
            void *to = row_of<T>(p.y, row, p.y_stride);
#pragma unroll 1
            for (int k = 0; k < HELD; ++k) {
                if (left(k) <= 0) break;
                float wk[8], bk[8];
                take(k);
                weights<true>(wk, p.w, 1.0f, lane, lanes, k, p.width, p.wtype, p.wvec != 0);
                weights<true>(bk, p.b, 0.0f, lane, lanes, k, p.width, p.wtype, p.wvec != 0);
#pragma unroll
                for (int j = 0; j < 8; ++j) x[j] = fmaf((x[j] - mean - rest) * rstd, wk[j], bk[j]);
                put<true>(to, x, lane, lanes, k, p.width, TYPE);
            }
        }
        if (lane == 0) n_far = 0;
    }
    for (; lane == 0 && under_way > 0; --under_way) {            // a wait ran out: the copies under way are waited for, each with the limit once more
        wait_for_copy(bars + stage * 8, phase, kPatience);
        if (++stage == stages) { stage = 0; phase ^= 1u; }
    }
}

// Longer rows: their gradient by a block a row, which reads the row twice ...
template <typename T, bool VEC>
__global__ void __launch_bounds__(kMaxThreads) backward_long_kernel(const __grid_constant__ Params p)
{
    __shared__ float scratch[32];
    constexpr int TYPE = Kind<T>::type;
    const int lane = threadIdx.x, lanes = blockDim.x, steps = (p.granules + lanes - 1) / lanes;
    const void *xr = row_of<T>(p.x, blockIdx.x, p.x_stride), *dr = row_of<T>(p.dy, blockIdx.x, p.dy_stride);
    void *to = row_of<T>(p.dx, blockIdx.x, p.dx_stride);
    const float mean = p.mean[blockIdx.x], rstd = p.rstd[blockIdx.x];
    float s1 = 0.0f, s2 = 0.0f, a[8], d[8], w[8];
    Raw8 rx, rd;
    for (int k = 0; k < steps; ++k) {
        fetch<VEC>(rx, xr, lane, lanes, k, p.width, TYPE);
        fetch<VEC>(rd, dr, lane, lanes, k, p.width, TYPE);
        widen8(a, rx, TYPE);
        widen8(d, rd, TYPE);
        weights<VEC>(w, p.w, 1.0f, lane, lanes, k, p.width, p.wtype, p.wvec != 0);
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (column<VEC>(lane, lanes, k, j) < p.width) {
                s1 = fmaf(d[j], w[j], s1);
                s2 = fmaf(d[j] * w[j], (a[j] - mean) * rstd, s2);
            }
    }
    const float c1 = row_sum(s1, lanes, scratch) * p.inverse, c2 = row_sum(s2, lanes, scratch) * p.inverse;
    for (int k = 0; k < steps; ++k) {
        fetch<VEC>(rx, xr, lane, lanes, k, p.width, TYPE);
        fetch<VEC>(rd, dr, lane, lanes, k, p.width, TYPE);
        widen8(a, rx, TYPE);
        widen8(d, rd, TYPE);
        weights<VEC>(w, p.w, 1.0f, lane, lanes, k, p.width, p.wtype, p.wvec != 0);
#pragma unroll
        for (int j = 0; j < 8; ++j) d[j] = (fmaf(d[j], w[j], -c1) - (a[j] - mean) * rstd * c2) * rstd;
        put<VEC>(to, d, lane, lanes, k, p.width, TYPE);
    }
}

// ... and the column sums by blocks of 256 granules over a part of the rows.  Runs first, since the gradient may be
// written over its operands.
template <typename T, bool VEC>
__global__ void __launch_bounds__(256) column_sums_kernel(const __grid_constant__ Params p)
{
    constexpr int TYPE = Kind<T>::type;
    const int lanes = int(gridDim.x) * 256, lane = int(blockIdx.x) * 256 + int(threadIdx.x);
    if (column<VEC>(lane, lanes, 0, 0) >= p.width) return;
    float dw[8], db[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) dw[j] = db[j] = 0.0f;
#pragma unroll 2
    for (int64_t row = blockIdx.y; row < p.rows; row += gridDim.y) {
        Raw8 rx, rd;
        float a[8], d[8];
        fetch<VEC>(rx, row_of<T>(p.x, row, p.x_stride), lane, lanes, 0, p.width, TYPE);
        fetch<VEC>(rd, row_of<T>(p.dy, row, p.dy_stride), lane, lanes, 0, p.width, TYPE);
        const float mean = p.mean[row], rstd = p.rstd[row];
        widen8(a, rx, TYPE);
        widen8(d, rd, TYPE);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            dw[j] = fmaf(d[j], (a[j] - mean) * rstd, dw[j]);
            db[j] += d[j];
        }
    }
    float *out = p.partial + int64_t(blockIdx.y) * 2 * p.width;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const int c = column<VEC>(lane, lanes, 0, j);
        if (c < p.width) {
            out[c] = dw[j];
            out[p.width + c] = db[j];
        }
    }
}

// Adds the blocks' partial sums, always in the same order: 32 columns a block, 16 threads a column.
constexpr int kFinish = 16;
__global__ void __launch_bounds__(32 * kFinish) finish_kernel(const float *partial, int blocks, int width, void *dw, void *db, int type)
{
    __shared__ float part[kFinish][33];
    asm volatile("griddepcontrol.wait;" ::: "memory");       // launched ahead of the end of the kernel that it follows
    const int64_t c = int64_t(blockIdx.x) * 32 + (threadIdx.x & 31), all = int64_t(2) * width;
    const int y = threadIdx.x >> 5;
    float s = 0.0f;
    if (c < all)
#pragma unroll 10
        for (int b = y; b < blocks; b += kFinish) s += partial[b * all + c];
    part[y][threadIdx.x & 31] = s;
    __syncthreads();
    if (y != 0 || c >= all) return;
#pragma unroll
    for (int i = 1; i < kFinish; ++i) s += part[i][threadIdx.x & 31];
    void *to = c < width ? dw : db;
    if (to) store1(to, c < width ? c : c - width, s, type);
}

template <typename T, int HELD, bool VEC, bool FULL>
int launch_held(const Params &p, int lanes, cudaStream_t st)
{
    // Warps that stay where each gets two rows and more: 12544 x 768 in bf16 takes 9.4 us, 14.4 with a warp for every row.
    if (lanes <= 32 && p.rows >= int64_t(2) * kResident * (256 / lanes)) {
        forward_rows_kernel<T, HELD, VEC, FULL><<<unsigned(kResident), 256, 0, st>>>(p, lanes);
        return int(cudaGetLastError());
    }
    const int threads = std::max(lanes, 128), rows = threads / lanes;
    forward_kernel<T, HELD, VEC, FULL><<<unsigned((p.rows + rows - 1) / rows), unsigned(threads), 0, st>>>(p, lanes);
    return int(cudaGetLastError());
}

template <typename T, bool VEC, bool FULL>
int launch_granules(const Params &p, int lanes, int held, cudaStream_t st)
{
    switch (held) {
    case 1: return launch_held<T, 1, VEC, FULL>(p, lanes, st);
    case 2: return launch_held<T, 2, VEC, FULL>(p, lanes, st);
    case 3: return launch_held<T, 3, VEC, FULL>(p, lanes, st);
    default: return launch_held<T, 4, VEC, FULL>(p, lanes, st);
    }
}

template <typename T, bool FULL, int THREADS>
int launch_forward_ring(const Params &p, int lanes, cudaStream_t st)
{
    constexpr int BLOCKS = kMaxThreads / THREADS, BYTES = 200 * 1024 / BLOCKS;         // on a multiprocessor; of each
    const int slot = lanes * 16 * int(sizeof(T)), stages = std::min(kMaxStages, BYTES / slot);
    const auto kernel = forward_ring_kernel<T, FULL, THREADS>;
    static std::atomic<uint64_t> raised{0};
    if (int err = allow_shared(reinterpret_cast<const void *>(kernel), BYTES, raised)) return err;
    kernel<<<unsigned(kBlocks * BLOCKS), unsigned(lanes), size_t(stages) * slot, st>>>(p, stages);
    return int(cudaGetLastError());
}
template <typename T, bool FULL>
int launch_forward_ring(const Params &p, int lanes, cudaStream_t st)
{
    return lanes > 512 ? launch_forward_ring<T, FULL, 1024>(p, lanes, st)
           : lanes > 256 ? launch_forward_ring<T, FULL, 512>(p, lanes, st)
           : lanes > 128 ? launch_forward_ring<T, FULL, 256>(p, lanes, st) : launch_forward_ring<T, FULL, 128>(p, lanes, st);
}

template <typename T, bool VEC>
int launch_forward(const Params &p, cudaStream_t st)
{
    if (VEC && p.granules > 32 * kMaxHeld && p.granules <= 2 * kMaxThreads) {
        const int lanes = (p.granules + 63) / 64 * 32, blocks = kBlocks * (kMaxThreads / std::max(128, power_of_two(lanes)));
        // two rows and more for each block: 1200 x 4096 bf16 6.9 us against 8.7 below, 2400 x 2048 6.7 against 7.4; 600 x 2048 4.0 against 3.8
        if (p.rows >= 2 * int64_t(blocks))
            return p.width % 8 == 0 ? launch_forward_ring<T, true>(p, lanes, st) : launch_forward_ring<T, false>(p, lanes, st);
    }
    // a warp a row up to 1024 elements, then the smallest block that holds a row in its registers
    int lanes = p.granules <= 32 ? power_of_two(p.granules) : 32;
    if (p.granules > 32 * kMaxHeld) lanes = 128;
    while (lanes >= 128 && p.granules > lanes * kMaxHeld) lanes *= 2;
    if (lanes > kMaxThreads) {
        forward_long_kernel<T, VEC><<<unsigned(p.rows), kMaxThreads, 0, st>>>(p);
        return int(cudaGetLastError());
    }
    const int held = (p.granules + lanes - 1) / lanes;
    if (VEC && p.width == lanes * held * 8) return launch_granules<T, true, true>(p, lanes, held, st);
    return launch_granules<T, VEC, false>(p, lanes, held, st);
}

constexpr int kRingBytes = 100 * 1024;            // 200 KB are one to three per cent slower
template <typename T, bool FULL, int ROWS, int THREADS>
int launch_ring(const Params &p, int lanes, int blocks, cudaStream_t st)
{
    const int row = lanes * 16 * int(sizeof(T)), stages = std::max(2 * ROWS, std::min(kMaxStages, kRingBytes / row));
    const auto kernel = backward_ring_kernel<T, FULL, ROWS, THREADS>;
    static std::atomic<uint64_t> raised{0};
    if (int err = allow_shared(reinterpret_cast<const void *>(kernel), std::max(kRingBytes, 2 * ROWS * THREADS * 16 * int(sizeof(T))), raised)) return err;
    kernel<<<unsigned(blocks), unsigned(lanes), size_t(stages) * row, st>>>(p, stages);
    return int(cudaGetLastError());
}
// Two rows at a time (8192 x 4096 bf16 55.3 us, 58.6 one by one; 4096 x 4096 fp32 41.4 and 44.6), one where a thread has 64 registers.
template <typename T, bool FULL>
int launch_ring(const Params &p, int lanes, int blocks, cudaStream_t st)
{
    return lanes > 768 ? launch_ring<T, FULL, 1, kMaxThreads>(p, lanes, blocks, st)
           : lanes > 640 ? launch_ring<T, FULL, 2, 768>(p, lanes, blocks, st) : launch_ring<T, FULL, 2, 640>(p, lanes, blocks, st);
}

template <typename T, bool VEC>
int launch_backward(const Params &p, void *dw, void *db, cudaStream_t st)
{
    int blocks = 0;
    if (p.granules <= kMaxThreads) {
        // as many groups as fit 768 threads, one block on a multiprocessor; rows that need more threads have fewer registers
        const int lanes = p.granules <= 32 ? power_of_two(p.granules) : (p.granules + 31) / 32 * 32;
        const int groups = std::max(1, lanes <= 32 ? 512 / lanes : std::min(768 / lanes, 15)), threads = groups * lanes;
        blocks = int(std::min<int64_t>((p.rows + groups - 1) / groups, kBlocks));
        const bool full = VEC && p.width % 8 == 0;
        const size_t sums = size_t(groups) * size_t(lanes / 32) * 16, columns = groups > 1 ? size_t(threads) * 8 * 4 : 0;
        if (VEC && lanes > 768 / 2) {
            const int err = full ? launch_ring<T, true>(p, lanes, blocks, st) : launch_ring<T, false>(p, lanes, blocks, st);
            if (err) return err;
        } else {
            const auto kernel = threads > 768 ? backward_kernel<T, false, false, kMaxThreads>
                                : threads > 640 ? (full ? backward_kernel<T, VEC, VEC, 768> : backward_kernel<T, VEC, false, 768>)
                                                : (full ? backward_kernel<T, VEC, VEC, 640> : backward_kernel<T, VEC, false, 640>);
            kernel<<<unsigned(blocks), unsigned(threads), std::max(sums, columns), st>>>(p, lanes);
        }
    } else {
        if (p.partial) {
            const int wide = (p.granules + 255) / 256;
            blocks = int(std::min<int64_t>(std::max(1, 2 * kBlocks / wide), std::min<int64_t>(p.rows, kBlocks)));
            column_sums_kernel<T, VEC><<<dim3(unsigned(wide), unsigned(blocks)), 256, 0, st>>>(p);
            if (cudaError_t err = cudaGetLastError()) return int(err);
        }
        if (p.dx) backward_long_kernel<T, VEC><<<unsigned(p.rows), kMaxThreads, 0, st>>>(p);
    }
    if (cudaError_t err = cudaGetLastError()) return int(err);
    if (!p.partial) return 0;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(unsigned((int64_t(2) * p.width + 31) / 32));
    cfg.blockDim = dim3(32 * kFinish);
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return int(cudaLaunchKernelEx(&cfg, finish_kernel, static_cast<const float *>(p.partial), blocks, int(p.width), dw, db, int(p.wtype)));
}

constexpr int64_t kMaxWidth = int64_t(1) << 24;      // up to which a width is a number in fp32

int shared_checks(const qsr_layer_norm_args &a)
{
    if (!type_bytes(a.type) || !type_bytes(a.weight_type)) return QSR_EINVAL;
    if (a.rows < 0 || a.rows > 0x7fffffff || a.width < 1 || a.width > kMaxWidth || a.x_stride < a.width) return QSR_ERANGE;
    const unsigned e = unsigned(type_bytes(a.type)), w = unsigned(type_bytes(a.weight_type));
    if (!aligned_to(a.x, e) || !aligned_to(a.weight, w) || !aligned_to(a.mean, 4) || !aligned_to(a.rstd, 4)) return QSR_EALIGN;
    return QSR_OK;
}

Params params_of(const qsr_layer_norm_args &a)
{
    Params p = {};
    p.x = a.x; p.x_stride = a.x_stride;
    p.w = a.weight; p.wtype = a.weight_type;
    p.mean = a.mean; p.rstd = a.rstd;
    p.rows = a.rows; p.width = int32_t(a.width);
    p.granules = int32_t((a.width + 7) / 8);
    p.inverse = 1.0f / float(a.width);
    p.patience = g_patience.load(std::memory_order_relaxed);
    return p;
}

}  // namespace

}  // namespace qsr

extern "C" {

int qsr_layer_norm(const qsr_layer_norm_args *a, void *cuda_stream)
{
    using namespace qsr;
    if (!a || !(a->eps >= 0.0) || !std::isfinite(float(a->eps))) return QSR_EINVAL;
    if (int rc = shared_checks(*a)) return rc;
    if (a->y_stride < a->width || (a->y == a->x && a->rows > 1 && a->y_stride != a->x_stride)) return QSR_ERANGE;
    if (a->rows == 0) return QSR_OK;
    if (!a->x || !a->y) return QSR_EINVAL;
    const int e = type_bytes(a->type), we = type_bytes(a->weight_type);
    if (!aligned_to(a->y, unsigned(e)) || !aligned_to(a->bias, unsigned(we))) return QSR_EALIGN;
    if (a->y != a->x && share_bytes(a->x, a->x_stride, a->width, e, a->rows, a->y, a->y_stride, a->width, e, a->rows)) return QSR_EINVAL;
    Params p = params_of(*a);
    p.y = a->y; p.y_stride = a->y_stride;
    p.b = a->bias;
    p.eps = float(a->eps);
    p.wvec = aligned_to(a->weight, 16) && aligned_to(a->bias, 16);
    const bool vec = rows_aligned(a->x, a->x_stride, a->rows, e) && rows_aligned(a->y, a->y_stride, a->rows, e);
    const cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    int err;
    if (a->type == QSR_F32) err = vec ? launch_forward<float, true>(p, st) : launch_forward<float, false>(p, st);
    else if (a->type == QSR_BF16) err = vec ? launch_forward<__nv_bfloat16, true>(p, st) : launch_forward<__nv_bfloat16, false>(p, st);
    else err = vec ? launch_forward<__half, true>(p, st) : launch_forward<__half, false>(p, st);
    return launch_status(err);
}

int64_t qsr_layer_norm_workspace_bytes(int64_t rows, int64_t width)
{
    if (rows < 0 || rows > 0x7fffffff || width < 1 || width > qsr::kMaxWidth) return QSR_ERANGE;
    return std::max<int64_t>(256, std::min<int64_t>(std::max<int64_t>(rows, 1), qsr::kBlocks) * 2 * width * 4);
}

int qsr_layer_norm_grad(const qsr_layer_norm_args *a, void *cuda_stream)
{
    using namespace qsr;
    if (!a) return QSR_EINVAL;
    if (int rc = shared_checks(*a)) return rc;
    if (a->d_y_stride < a->width || (a->d_x && a->d_x_stride < a->width)) return QSR_ERANGE;
    const int e = type_bytes(a->type), we = type_bytes(a->weight_type);
    const bool sums = a->d_weight || a->d_bias;
    if (!aligned_to(a->d_weight, unsigned(we)) || !aligned_to(a->d_bias, unsigned(we)) || !aligned_to(a->d_y, unsigned(e)) || !aligned_to(a->d_x, unsigned(e)))
        return QSR_EALIGN;
    if (sums) {
        if (!a->workspace) return QSR_EINVAL;
        if (!aligned_to(a->workspace, 256)) return QSR_EALIGN;
        if (a->workspace_bytes < qsr_layer_norm_workspace_bytes(a->rows, a->width)) return QSR_ERANGE;
    }
    const cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    if (a->rows == 0) {               // sums over nothing
        if (a->d_weight)
            if (cudaError_t err = cudaMemsetAsync(a->d_weight, 0, size_t(a->width) * size_t(we), st)) return launch_status(int(err));
        if (a->d_bias)
            if (cudaError_t err = cudaMemsetAsync(a->d_bias, 0, size_t(a->width) * size_t(we), st)) return launch_status(int(err));
        return QSR_OK;
    }
    if (!a->x || !a->d_y || !a->mean || !a->rstd) return QSR_EINVAL;
    if (!sums && !a->d_x) return QSR_OK;
    if (a->d_x) {
        const struct { const void *p; int64_t stride; } of[2] = {{a->x, a->x_stride}, {a->d_y, a->d_y_stride}};
        for (const auto &o : of) {
            if (o.p == a->d_x && (o.stride == a->d_x_stride || a->rows == 1)) continue;      // in place
            if (share_bytes(o.p, o.stride, a->width, e, a->rows, a->d_x, a->d_x_stride, a->width, e, a->rows)) return QSR_EINVAL;
        }
    }
    Params p = params_of(*a);
    p.dy = a->d_y; p.dy_stride = a->d_y_stride;
    p.dx = a->d_x; p.dx_stride = a->d_x_stride;
    p.partial = sums ? static_cast<float *>(a->workspace) : nullptr;
    p.wvec = aligned_to(a->weight, 16);
    const bool vec = rows_aligned(a->x, a->x_stride, a->rows, e) && rows_aligned(a->d_y, a->d_y_stride, a->rows, e) &&
                     (!a->d_x || rows_aligned(a->d_x, a->d_x_stride, a->rows, e));
    int err;
    if (a->type == QSR_F32) err = vec ? launch_backward<float, true>(p, a->d_weight, a->d_bias, st) : launch_backward<float, false>(p, a->d_weight, a->d_bias, st);
    else if (a->type == QSR_BF16) err = vec ? launch_backward<__nv_bfloat16, true>(p, a->d_weight, a->d_bias, st) : launch_backward<__nv_bfloat16, false>(p, a->d_weight, a->d_bias, st);
    else err = vec ? launch_backward<__half, true>(p, a->d_weight, a->d_bias, st) : launch_backward<__half, false>(p, a->d_weight, a->d_bias, st);
    return launch_status(err);
}

int qsr_debug_copy_patience(int64_t clocks)
{
    qsr::g_patience.store(clocks < 0 ? qsr::kPatience : clocks, std::memory_order_relaxed);
    return QSR_OK;
}

}  // extern "C"
