// Lists of tensors: the AdamW step (OPT of Eq. 1, arXiv 2310.14423) over many tensors in one launch, states in fp32 or in
// 8 bits, and the replica mean that ends a round (Algorithm 2).  Element-wise streams: no contraction, no tensor cores.
#include <cuda_runtime.h>

#include <cstdint>

#include "internal.h"
#include "wide.cuh"

namespace qsr {
namespace {

constexpr int kThreads = 256;
constexpr int kWarps = kThreads / 32;
constexpr float kCodeMax = 448.0f;               // largest E4M3 value
constexpr float kCodeMin = 0.001953125f;         // smallest positive one, 2^-9
constexpr float kAmaxMin = 0x1p-100f;            // blocks below this are stored as zeros

__device__ __forceinline__ bool aligned_to(const void *p, unsigned bytes) { return (reinterpret_cast<uintptr_t>(p) & (bytes - 1)) == 0; }
__device__ __forceinline__ unsigned bytes_of_8(int type) { return type == QSR_F32 ? 32u : 16u; }

// The 8-bit block format: scale and its reciprocal from the block's amax (see the public header).  Every operation here
// and around it (dequantization, moments, root) is one IEEE rounding, so that the codes are a function of the formulas alone
// and do not depend on which of them the compiler fused.
struct BlockScale { float scale, inv; };
__device__ __forceinline__ BlockScale block_scale(float amax)
{
    BlockScale b;
    b.scale = amax >= kAmaxMin ? __fmul_rn(amax, 1.0f / kCodeMax) : 0.0f;
    b.inv = b.scale > 0.0f ? __frcp_rn(b.scale) : 0.0f;
    return b;
}

// Largest finite magnitude of the warp's 256 values.  Infinities are rare: only a block that holds one pays for the test.
__device__ __forceinline__ float block_amax(const float (&x)[8])
{
    float a = 0.0f;
#pragma unroll
    for (int i = 0; i < 8; ++i) a = fmaxf(a, fabsf(x[i]));
    a = warp_max(a);
    if (a == infinity()) {
        a = 0.0f;
#pragma unroll
        for (int i = 0; i < 8; ++i) a = fmaxf(a, fabsf(x[i]) < infinity() ? fabsf(x[i]) : 0.0f);
        a = warp_max(a);
    }
    return a;
}

__device__ __forceinline__ float code_of(float x, float inv, bool positive)
{
    const float q = __fmul_rn(x, inv);
    return positive && q > 0.0f ? fmaxf(q, kCodeMin) : q;
}

// Eight codes of a lane: two words when the lane owns eight consecutive elements, single bytes otherwise.
template <bool VEC>
__device__ __forceinline__ void load_codes(float (&x)[8], const uint8_t *base, int64_t e0, int n, int lane)
{
    if (VEC) {
        const uint2 w = *reinterpret_cast<const uint2 *>(base + e0 + lane * 8);
        const uint32_t ws[2] = {w.x, w.y};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float2 f = from_e4m3x2((ws[i >> 1] >> (16 * (i & 1))) & 0xffffu);
            x[2 * i] = f.x; x[2 * i + 1] = f.y;
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = lane + 32 * i < n ? from_e4m3x2(base[e0 + lane + 32 * i]).x : 0.0f;
    }
}
template <bool VEC>
__device__ __forceinline__ void store_codes(uint8_t *base, int64_t e0, int n, int lane, const float (&x)[8], float inv, bool positive)
{
    if (VEC) {
        uint32_t h[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) h[i] = to_e4m3x2(code_of(x[2 * i], inv, positive), code_of(x[2 * i + 1], inv, positive));
        *reinterpret_cast<uint2 *>(base + e0 + lane * 8) = make_uint2(h[0] | h[1] << 16, h[2] | h[3] << 16);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (lane + 32 * i < n) base[e0 + lane + 32 * i] = uint8_t(to_e4m3x2(code_of(x[i], inv, positive), 0.0f));
    }
}

// A warp's 256 elements e0 .. e0 + 255 of one operand: with VEC eight consecutive elements per lane, otherwise (ragged or
// unaligned) lane, lane + 32, ..., which keeps single-element accesses of a warp next to each other.
template <bool VEC>
__device__ __forceinline__ void load_raw(Raw8 &r, const void *base, int64_t e0, int n, int lane, int type)
{
    if (VEC) load8(r, base, e0 + lane * 8, type);
    else {
#pragma unroll
        for (int i = 0; i < 8; ++i) r.w[i] = lane + 32 * i < n ? load1(base, e0 + lane + 32 * i, type) : 0u;
    }
}
template <bool VEC>
__device__ __forceinline__ void widen(float (&x)[8], const Raw8 &r, int type)
{
    if (VEC) widen8(x, r, type);
    else {
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = widen1(r.w[i], type);
    }
}
template <bool VEC>
__device__ __forceinline__ void store(void *base, int64_t e0, int n, int lane, const float (&x)[8], int type)
{
    if (VEC) store8(base, e0 + lane * 8, x, type);
    else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (lane + 32 * i < n) store1(base, e0 + lane + 32 * i, x[i], type);
    }
}

// ---------------------------------------------------------------------------------------------- AdamW step

// One warp, 256 elements of one tensor (n of them valid).
template <bool S8, bool VEC>
__device__ __forceinline__ void step_block(const ListStepParams &p, const ListTensor &t, const void *grad, int64_t e0, int n, int lane,
                                           float g_scale, float eta_wd)
{
    Raw8 rp, rg, rm, rv;
    float th[8], g[8], m[8], v[8];
    load_raw<VEC>(rp, t.param, e0, n, lane, t.param_type);
    load_raw<VEC>(rg, grad, e0, n, lane, t.grad_type);
    if (S8) {
        const int64_t b = e0 >> 8;
        const float ms = t.m_scale[b], vs = t.v_scale[b];
        load_codes<VEC>(m, static_cast<const uint8_t *>(t.m), e0, n, lane);
        load_codes<VEC>(v, static_cast<const uint8_t *>(t.v), e0, n, lane);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            m[i] = __fmul_rn(m[i], ms);
            v[i] = __fmul_rn(v[i], vs);
            v[i] = __fmul_rn(v[i], v[i]);
        }
    } else {
        load_raw<VEC>(rm, t.m, e0, n, lane, QSR_F32);
        load_raw<VEC>(rv, t.v, e0, n, lane, QSR_F32);
        widen<VEC>(m, rm, QSR_F32);
        widen<VEC>(v, rv, QSR_F32);
    }
    widen<VEC>(th, rp, t.param_type);
    widen<VEC>(g, rg, t.grad_type);
    float u[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float gi = __fmul_rn(g[i], g_scale);
        if (S8) {
            m[i] = __fadd_rn(m[i], __fmul_rn(p.omb1, __fsub_rn(gi, m[i])));
            v[i] = __fadd_rn(v[i], __fmul_rn(p.omb2, __fsub_rn(__fmul_rn(gi, gi), v[i])));
            u[i] = __fsqrt_rn(v[i]);
        } else {
            // moments in the interpolation form: a constant gradient is a fixed point exactly
            m[i] = fmaf(p.omb1, gi - m[i], m[i]);
            v[i] = fmaf(p.omb2, fmaf(gi, gi, -v[i]), v[i]);
            u[i] = sqrt_1(v[i]);
        }
        // the decay and the update are summed before they meet theta: see opt_update of the slab kernels
        th[i] -= fmaf(eta_wd, th[i], (p.step_size * m[i]) * rcp_1(fmaf(u[i], p.inv_sqrt_bc2, p.eps)));
    }
    store<VEC>(t.param, e0, n, lane, th, t.param_type);
    if (t.copy_type != QSR_NONE) store<VEC>(t.copy, e0, n, lane, th, t.copy_type);
    if (S8) {
        const int64_t b = e0 >> 8;
        const BlockScale bm = block_scale(block_amax(m)), bu = block_scale(block_amax(u));
        store_codes<VEC>(static_cast<uint8_t *>(t.m), e0, n, lane, m, bm.inv, false);
        store_codes<VEC>(static_cast<uint8_t *>(t.v), e0, n, lane, u, bu.inv, true);
        if (lane == 0) { t.m_scale[b] = bm.scale; t.v_scale[b] = bu.scale; }
    } else {
        store<VEC>(t.m, e0, n, lane, m, QSR_F32);
        store<VEC>(t.v, e0, n, lane, v, QSR_F32);
    }
}

template <bool S8>
__device__ __forceinline__ bool step_aligned(const ListTensor &t, const void *grad)
{
    return aligned_to(t.param, bytes_of_8(t.param_type)) && aligned_to(grad, bytes_of_8(t.grad_type)) &&
           aligned_to(t.m, S8 ? 8 : 32) && aligned_to(t.v, S8 ? 8 : 32) &&
           (t.copy_type == QSR_NONE || aligned_to(t.copy, bytes_of_8(t.copy_type)));
}

template <bool S8>
__global__ void __launch_bounds__(kThreads) list_step_kernel(const ListStepParams p)
{
    const ListChunk c = p.chunks[blockIdx.x];
    const ListTensor t = p.tensors[c.tensor];
    const void *grad = p.grads[c.tensor];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const float g_scale = p.clip ? p.grad_scale * p.clip[c.tensor / p.tensors_per_worker] : p.grad_scale;
    const float eta_wd = p.eta_wd * t.wd_scale;
    const bool vec = step_aligned<S8>(t, grad);
    for (int b = warp; b * 256 < c.n; b += kWarps) {
        const int64_t e0 = c.offset + b * 256;
        const int n = min(256, c.n - b * 256);
        if (vec && n == 256) step_block<S8, true>(p, t, grad, e0, n, lane, g_scale, eta_wd);
        else step_block<S8, false>(p, t, grad, e0, n, lane, g_scale, eta_wd);
    }
}

// ---------------------------------------------------------------------------------------------- clipping

__device__ __forceinline__ float block_sum(float x, float *smem)
{
    x = warp_sum(x);
    if ((threadIdx.x & 31) == 0) smem[threadIdx.x >> 5] = x;
    __syncthreads();
    float s = 0.0f;
#pragma unroll
    for (int i = 0; i < kWarps; ++i) s += smem[i];
    __syncthreads();
    return s;
}

// Sum of squares of each chunk's gradients; the last block of a worker to finish adds its chunks up -- in chunk order, so
// the result does not depend on which block that is -- and leaves the factor.
__global__ void __launch_bounds__(kThreads) list_norm_kernel(const ListNormParams p)
{
    __shared__ float part[kWarps];
    __shared__ double dpart[kThreads];
    __shared__ bool last;
    const ListChunk c = p.chunks[blockIdx.x];
    const int type = p.tensors[c.tensor].grad_type;
    const void *grad = p.grads[c.tensor];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const bool vec = aligned_to(grad, bytes_of_8(type));
    float s = 0.0f;
    for (int b = warp; b * 256 < c.n; b += kWarps) {
        const int64_t e0 = c.offset + b * 256;
        const int n = min(256, c.n - b * 256);
        Raw8 r;
        float g[8];
        if (vec && n == 256) {
            load_raw<true>(r, grad, e0, n, lane, type);
            widen<true>(g, r, type);
        } else {
            load_raw<false>(r, grad, e0, n, lane, type);
            widen<false>(g, r, type);
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float x = g[i] * p.grad_scale;
            s = fmaf(x, x, s);
        }
    }
    s = block_sum(s, part);
    const int worker = blockIdx.x / p.chunks_per_worker;
    if (threadIdx.x == 0) {
        p.partial[blockIdx.x] = s;
        __threadfence();
        last = atomicAdd(p.arrived + worker, 1u) == unsigned(p.chunks_per_worker) - 1;
    }
    __syncthreads();
    if (!last) return;
    __threadfence();
    const float *mine = p.partial + int64_t(worker) * p.chunks_per_worker;
    double d = 0.0;
    for (int i = threadIdx.x; i < p.chunks_per_worker; i += kThreads) d += double(__ldcg(mine + i));
    dpart[threadIdx.x] = d;
    __syncthreads();
    for (int k = kThreads / 2; k; k >>= 1) {
        if (threadIdx.x < k) dpart[threadIdx.x] += dpart[threadIdx.x + k];
        __syncthreads();
    }
    if (threadIdx.x == 0) {
        const float norm = float(sqrt(dpart[0]));
        const float f = p.max_norm / (norm + 1e-6f);
        p.clip[worker] = f > 1.0f ? 1.0f : f;          // NaN stays NaN
        if (p.grad_norm) p.grad_norm[worker] = norm;
        p.arrived[worker] = 0u;                          // ready for the next step
    }
}

// ---------------------------------------------------------------------------------------------- replica mean

// Address of operand A of worker k's tensor: 0 parameter, 1 m, 2 v.
template <int A>
__device__ __forceinline__ void *operand(const ListTensor &t) { return A == 0 ? t.param : A == 1 ? t.m : t.v; }

__device__ __forceinline__ void *shfl_ptr(const void *p, int lane)
{
    return reinterpret_cast<void *>(__shfl_sync(0xffffffffu, reinterpret_cast<unsigned long long>(p), lane));
}

// Mean over the workers of 256 elements in the caller's type, written back to every worker (and to the working copies).
template <int A, bool VEC>
__device__ __forceinline__ void mean_block(const ListSyncParams &p, int tensor, int type, int copy_type, int64_t e0, int n, int lane)
{
    float s[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) s[i] = 0.0f;
    for (int k0 = 0; k0 < p.workers; k0 += 32) {
        const int kl = k0 + lane < p.workers ? k0 + lane : k0;
        const void *mine = operand<A>(p.tensors[kl * p.tensors_per_worker + tensor]);
        const int here = min(32, p.workers - k0);
        int k = 0;
        for (; k + 4 <= here; k += 4) {
            Raw8 r[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) load_raw<VEC>(r[j], shfl_ptr(mine, k + j), e0, n, lane, type);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                float x[8];
                widen<VEC>(x, r[j], type);
#pragma unroll
                for (int i = 0; i < 8; ++i) s[i] += x[i];
            }
        }
        for (; k < here; ++k) {
            Raw8 r;
            float x[8];
            load_raw<VEC>(r, shfl_ptr(mine, k), e0, n, lane, type);
            widen<VEC>(x, r, type);
#pragma unroll
            for (int i = 0; i < 8; ++i) s[i] += x[i];
        }
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) s[i] = s[i] / p.divisor;
    for (int k0 = 0; k0 < p.workers; k0 += 32) {
        const int kl = k0 + lane < p.workers ? k0 + lane : k0;
        const ListTensor &t = p.tensors[kl * p.tensors_per_worker + tensor];
        void *mine = operand<A>(t), *copy = t.copy;
        const int here = min(32, p.workers - k0);
        for (int k = 0; k < here; ++k) {
            store<VEC>(shfl_ptr(mine, k), e0, n, lane, s, type);
            if (A == 0 && copy_type != QSR_NONE) store<VEC>(shfl_ptr(copy, k), e0, n, lane, s, copy_type);
        }
    }
}

// The same for a block of 8-bit states: the mean of the values they stand for (of the squares of v's codes), rounded to 8
// bits once.
template <int A, bool VEC>
__device__ __forceinline__ void mean_codes(const ListSyncParams &p, int tensor, int64_t e0, int n, int lane)
{
    float s[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) s[i] = 0.0f;
    const int64_t b = e0 >> 8;
    for (int k = 0; k < p.workers; ++k) {
        const ListTensor &t = p.tensors[k * p.tensors_per_worker + tensor];
        const float scale = (A == 1 ? t.m_scale : t.v_scale)[b];
        float x[8];
        load_codes<VEC>(x, static_cast<const uint8_t *>(operand<A>(t)), e0, n, lane);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            x[i] = __fmul_rn(x[i], scale);
            s[i] = __fadd_rn(s[i], A == 1 ? x[i] : __fmul_rn(x[i], x[i]));
        }
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        s[i] = s[i] / p.divisor;
        if (A == 2) s[i] = __fsqrt_rn(s[i]);
    }
    const BlockScale q = block_scale(block_amax(s));
    for (int k = 0; k < p.workers; ++k) {
        const ListTensor &t = p.tensors[k * p.tensors_per_worker + tensor];
        store_codes<VEC>(static_cast<uint8_t *>(operand<A>(t)), e0, n, lane, s, q.inv, A == 2);
        if (lane == 0) (A == 1 ? t.m_scale : t.v_scale)[b] = q.scale;
    }
}

// Whether every worker's operand may be accessed eight elements at a time.
template <int A>
__device__ __forceinline__ bool sync_aligned(const ListSyncParams &p, int tensor, int type, int copy_type, bool codes, int lane)
{
    bool ok = true;
    for (int k = lane; k < p.workers; k += 32) {
        const ListTensor &t = p.tensors[k * p.tensors_per_worker + tensor];
        ok = ok && aligned_to(operand<A>(t), codes ? 8u : bytes_of_8(type));
        if (A == 0 && copy_type != QSR_NONE) ok = ok && aligned_to(t.copy, bytes_of_8(copy_type));
    }
    return __all_sync(0xffffffffu, ok);
}

template <int A, bool CODES>
__device__ __forceinline__ void sync_chunk(const ListSyncParams &p)
{
    const ListChunk c = p.chunks[blockIdx.x];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int type = A == 0 ? p.tensors[c.tensor].param_type : QSR_F32;
    const int copy_type = p.tensors[c.tensor].copy_type;
    const bool vec = sync_aligned<A>(p, c.tensor, type, copy_type, CODES, lane);
    for (int b = warp; b * 256 < c.n; b += kWarps) {
        const int64_t e0 = c.offset + b * 256;
        const int n = min(256, c.n - b * 256);
        if (CODES) {
            if (vec && n == 256) mean_codes<A, true>(p, c.tensor, e0, n, lane);
            else mean_codes<A, false>(p, c.tensor, e0, n, lane);
        } else {
            if (vec && n == 256) mean_block<A, true>(p, c.tensor, type, copy_type, e0, n, lane);
            else mean_block<A, false>(p, c.tensor, type, copy_type, e0, n, lane);
        }
    }
}

// Grid: worker 0's chunks by 1 (parameters) or 3 (parameters, m, v).
template <bool S8>
__global__ void __launch_bounds__(kThreads) list_sync_kernel(const ListSyncParams p)
{
    if (blockIdx.y == 0) sync_chunk<0, false>(p);
    else if (blockIdx.y == 1) sync_chunk<1, S8>(p);
    else sync_chunk<2, S8>(p);
}

// Zeroes m and v (and their scales) of every worker.  Grid: all chunks.
template <bool S8>
__global__ void __launch_bounds__(kThreads) list_reset_kernel(const ListSyncParams p)
{
    const ListChunk c = p.chunks[blockIdx.x];
    const ListTensor t = p.tensors[c.tensor];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const bool vec = aligned_to(t.m, S8 ? 8 : 32) && aligned_to(t.v, S8 ? 8 : 32);
    const float zero[8] = {0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f};
    for (int b = warp; b * 256 < c.n; b += kWarps) {
        const int64_t e0 = c.offset + b * 256;
        const int n = min(256, c.n - b * 256);
#pragma unroll
        for (int a = 0; a < 2; ++a) {
            void *x = a ? t.v : t.m;
            if (S8) {
                if (vec && n == 256) store_codes<true>(static_cast<uint8_t *>(x), e0, n, lane, zero, 0.0f, false);
                else store_codes<false>(static_cast<uint8_t *>(x), e0, n, lane, zero, 0.0f, false);
                if (lane == 0) (a ? t.v_scale : t.m_scale)[e0 >> 8] = 0.0f;
            } else {
                if (vec && n == 256) store<true>(x, e0, n, lane, zero, QSR_F32);
                else store<false>(x, e0, n, lane, zero, QSR_F32);
            }
        }
    }
}

}  // namespace

int launch_list_step(const ListStepParams &p, bool states8, int64_t chunks, void *stream)
{
    const cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (states8) list_step_kernel<true><<<unsigned(chunks), kThreads, 0, st>>>(p);
    else list_step_kernel<false><<<unsigned(chunks), kThreads, 0, st>>>(p);
    return int(cudaGetLastError());
}

int launch_list_norm(const ListNormParams &p, int64_t chunks, void *stream)
{
    list_norm_kernel<<<unsigned(chunks), kThreads, 0, static_cast<cudaStream_t>(stream)>>>(p);
    return int(cudaGetLastError());
}

int launch_list_sync(const ListSyncParams &p, bool states8, bool average, int64_t chunks_per_worker, void *stream)
{
    const dim3 grid(unsigned(chunks_per_worker), average ? 3 : 1);
    const cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (states8) list_sync_kernel<true><<<grid, kThreads, 0, st>>>(p);
    else list_sync_kernel<false><<<grid, kThreads, 0, st>>>(p);
    return int(cudaGetLastError());
}

int launch_list_reset(const ListSyncParams &p, bool states8, int64_t chunks, void *stream)
{
    const cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (states8) list_reset_kernel<true><<<unsigned(chunks), kThreads, 0, st>>>(p);
    else list_reset_kernel<false><<<unsigned(chunks), kThreads, 0, st>>>(p);
    return int(cudaGetLastError());
}

}  // namespace qsr
