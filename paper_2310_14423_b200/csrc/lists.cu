// Lists of tensors: the AdamW step (OPT of Eq. 1, arXiv 2310.14423) over many tensors in one launch, states in fp32 or in
// 8 bits, and the replica mean that ends a round (Algorithm 2).  Element-wise streams: no contraction, no tensor cores.
#include <cuda_runtime.h>

#include <cstdint>

#include "internal.h"
#include "wide.cuh"

namespace qsr {
namespace {

constexpr int kWarps = kListWarps;
constexpr int kThreads = kWarps * 32;
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
    // 1 / scale rounded to nearest: one Newton step whose residual a fused multiply-add forms exactly (Markstein, IBM J. Res.
    // Dev. 34, 1990); scale is 0 or at least 2^-109, and its reciprocal a normal number
    const float y = rcp_1(b.scale);
    b.inv = b.scale > 0.0f ? fmaf(y, fmaf(-b.scale, y, 1.0f), y) : 0.0f;
    return b;
}

__device__ __forceinline__ float finite_or_0(float a) { return a < infinity() ? a : 0.0f; }

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
        for (int i = 0; i < 8; ++i) a = fmaxf(a, finite_or_0(fabsf(x[i])));
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

// theta after the step, from its new moments (m) and the root of the second one (u).  The decay and the update are summed
// before they meet theta: see opt_update of the slab kernels.
__device__ __forceinline__ float step_theta(const ListStepParams &p, float theta, float m, float u, float eta_wd)
{
    return theta - fmaf(eta_wd, theta, (p.step_size * m) * rcp_1(fmaf(u, p.inv_sqrt_bc2, p.eps)));
}

// One warp, 256 elements of one tensor (n of them valid), states in fp32.
template <bool VEC>
__device__ __forceinline__ void step_block_f32(const ListStepParams &p, const ListTensor &t, const void *grad, int64_t e0, int n, int lane,
                                               float g_scale, float eta_wd)
{
    Raw8 rp, rg, rm, rv;
    float th[8], g[8], m[8], v[8];
    load_raw<VEC>(rp, t.param, e0, n, lane, t.param_type);
    load_raw<VEC>(rg, grad, e0, n, lane, t.grad_type);
    load_raw<VEC>(rm, t.m, e0, n, lane, QSR_F32);
    load_raw<VEC>(rv, t.v, e0, n, lane, QSR_F32);
    widen<VEC>(m, rm, QSR_F32);
    widen<VEC>(v, rv, QSR_F32);
    widen<VEC>(th, rp, t.param_type);
    widen<VEC>(g, rg, t.grad_type);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float gi = g[i] * g_scale;
        // moments in the interpolation form: a constant gradient is a fixed point exactly
        m[i] = fmaf(p.omb1, gi - m[i], m[i]);
        v[i] = fmaf(p.omb2, fmaf(gi, gi, -v[i]), v[i]);
        th[i] = step_theta(p, th[i], m[i], sqrt_1(v[i]), eta_wd);
    }
    store<VEC>(t.param, e0, n, lane, th, t.param_type);
    if (t.copy_type != QSR_NONE) store<VEC>(t.copy, e0, n, lane, th, t.copy_type);
    store<VEC>(t.m, e0, n, lane, m, QSR_F32);
    store<VEC>(t.v, e0, n, lane, v, QSR_F32);
}

// The same with states in 8 bits, one element at a time: ragged blocks and unaligned tensors.
// Not inlined, so that the registers of this rare path do not count against the common one.
__device__ __noinline__ void step_block_codes_any(const ListStepParams &p, int tensor, int64_t e0, int n, int lane, float g_scale, float eta_wd)
{
    const ListTensor &t = p.tensors[tensor];
    const void *const grad = p.grads[tensor];
    const int64_t b = e0 >> 8;
    const float ms = t.m_scale[b], vs = t.v_scale[b];
    float m[8], u[8];
    load_codes<false>(m, static_cast<const uint8_t *>(t.m), e0, n, lane);
    load_codes<false>(u, static_cast<const uint8_t *>(t.v), e0, n, lane);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        if (lane + 32 * i >= n) { m[i] = u[i] = 0.0f; continue; }
        const int64_t e = e0 + lane + 32 * i;
        const float g = __fmul_rn(widen1(load1(grad, e, t.grad_type), t.grad_type), g_scale);
        const float m0 = __fmul_rn(m[i], ms), u0 = __fmul_rn(u[i], vs), v0 = __fmul_rn(u0, u0);
        m[i] = __fadd_rn(m0, __fmul_rn(p.omb1, __fsub_rn(g, m0)));
        u[i] = __fsqrt_rn(__fadd_rn(v0, __fmul_rn(p.omb2, __fsub_rn(__fmul_rn(g, g), v0))));
        const float th = step_theta(p, widen1(load1(t.param, e, t.param_type), t.param_type), m[i], u[i], eta_wd);
        store1(t.param, e, th, t.param_type);
        if (t.copy_type != QSR_NONE) store1(t.copy, e, th, t.copy_type);
    }
    const BlockScale bm = block_scale(block_amax(m)), bu = block_scale(block_amax(u));
    store_codes<false>(static_cast<uint8_t *>(t.m), e0, n, lane, m, bm.inv, false);
    store_codes<false>(static_cast<uint8_t *>(t.v), e0, n, lane, u, bu.inv, true);
    if (lane == 0) { t.m_scale[b] = bm.scale; t.v_scale[b] = bu.scale; }
}

// Two fp32 operations per instruction (sm_100), each rounded like its scalar form.  Sums are written as fused multiply-adds with
// a factor of one: nvcc 12.9 makes one fused operation of a packed product and the packed sum that takes it (also of
// mul.rn.f32x2 and add.rn.f32x2), and the codes would not be those of the formulas (the tests compare them bit for bit).
__device__ __forceinline__ float2 both(float x) { return make_float2(x, x); }
__device__ __forceinline__ float2 mul2(float2 a, float2 b) { return __fmul2_rn(a, b); }
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) { return __ffma2_rn(a, b, c); }
__device__ __forceinline__ float2 add2(float2 a, float2 b, float one) { return __ffma2_rn(b, both(one), a); }
__device__ __forceinline__ float2 sub2(float2 a, float2 b) { return __ffma2_rn(b, both(-1.0f), a); }

// sqrt(v) rounded to nearest for v >= 2^-100: one Newton step on s = v * rsqrt(v) with the residual v - s^2 formed by a fused
// multiply-add (Markstein, IBM J. Res. Dev. 34, 1990).  Half the instructions of the general root, which also has to deal
// with the operands excluded here.
__device__ __forceinline__ float2 root2(float2 v)
{
    float2 y;
    asm("rsqrt.approx.ftz.f32 %0, %1;" : "=f"(y.x) : "f"(v.x));
    asm("rsqrt.approx.ftz.f32 %0, %1;" : "=f"(y.y) : "f"(v.y));
    const float2 s = mul2(v, y), r = fma2(mul2(s, both(-1.0f)), s, v);
    return fma2(r, mul2(y, both(0.5f)), s);
}

template <int BYTES>
__device__ __forceinline__ void copy_async(unsigned smem, const void *gmem)
{
    if (BYTES == 16) asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(smem), "l"(gmem) : "memory");
    else asm volatile("cp.async.ca.shared.global [%0], [%1], 8;" ::"r"(smem), "l"(gmem) : "memory");
}
template <int N>
__device__ __forceinline__ void copy_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

// Where the 16-byte piece k of a block's fp32 operand lies in shared memory: pieces 8..15 of each 16 swap with their
// neighbours, so that a lane's two adjacent pieces can be read without bank conflicts.
__device__ __forceinline__ unsigned piece(unsigned k) { return k ^ ((k >> 3) & 1); }

__device__ __forceinline__ unsigned bytes_of(int type) { return type == QSR_F32 ? 4u : 2u; }

// Starts the copy of the 256 elements `at` .. of one operand of a chunk (in the end eight consecutive ones per lane): fp32 in
// two coalesced halves, 16-bit types as one piece per lane.
__device__ __forceinline__ void fetch_operand(unsigned smem, const char *chunk, unsigned at, unsigned lane, int type)
{
    if (type == QSR_F32) {
        copy_async<16>(smem + piece(lane) * 16, chunk + (at * 4 + lane * 16));
        copy_async<16>(smem + piece(32 + lane) * 16, chunk + (at * 4 + lane * 16 + 512));
    } else copy_async<16>(smem + lane * 16, chunk + (at * 2 + lane * 16));
}
__device__ __forceinline__ void read_operand(float (&x)[8], const char *smem, unsigned lane, int type)
{
    Raw8 r;
    if (type == QSR_F32) {
        const uint4 a = *reinterpret_cast<const uint4 *>(smem + piece(2 * lane) * 16), b = *reinterpret_cast<const uint4 *>(smem + piece(2 * lane + 1) * 16);
        r.w[0] = a.x; r.w[1] = a.y; r.w[2] = a.z; r.w[3] = a.w;
        r.w[4] = b.x; r.w[5] = b.y; r.w[6] = b.z; r.w[7] = b.w;
    } else {
        const uint4 a = *reinterpret_cast<const uint4 *>(smem + lane * 16);
        r.w[0] = a.x; r.w[1] = a.y; r.w[2] = a.z; r.w[3] = a.w;
    }
    widen8(x, r, type);
}

// The operands of a chunk: addresses of its first element (the same for the whole thread block) and types.  PT, GT: the types
// of parameters and gradients where the whole list has the same, known to the compiler then, or -1.
template <int PT, int GT>
struct Chunk {
    char *param, *copy, *m, *v;
    const char *grad;
    int param_type_, grad_type_, copy_type;
    __device__ __forceinline__ int param_type() const { return PT >= 0 ? PT : param_type_; }
    __device__ __forceinline__ int grad_type() const { return GT >= 0 ? GT : grad_type_; }
};

// A whole aligned block whose operands have arrived in shared memory (parameter, gradient, codes of m, codes of v): eight
// consecutive elements per lane, in pairs.  ms, vs: the block's scales before; returned: after.
template <int PT, int GT>
__device__ __forceinline__ float2 step_block_codes(const ListStepParams &p, const Chunk<PT, GT> &t, const char *stage, unsigned at, unsigned lane,
                                                   float ms, float vs, float g_scale, float eta_wd)
{
    float g[8];
    const char *const s_grad = stage + 256 * bytes_of(t.param_type()), *const s_codes = s_grad + 256 * bytes_of(t.grad_type());
    read_operand(g, s_grad, lane, t.grad_type());
    const uint2 mw = *reinterpret_cast<const uint2 *>(s_codes + lane * 8), vw = *reinterpret_cast<const uint2 *>(s_codes + 256 + lane * 8);
    float2 m[4], u[4];
    from_e4m3x4(m[0], m[1], mw.x);
    from_e4m3x4(m[2], m[3], mw.y);
    from_e4m3x4(u[0], u[1], vw.x);
    from_e4m3x4(u[2], u[3], vw.y);
    float least = infinity();
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        float2 gi = make_float2(g[2 * i], g[2 * i + 1]);
        if (g_scale != 1.0f) gi = mul2(gi, both(g_scale));
        const float2 m0 = mul2(m[i], both(ms)), u0 = mul2(u[i], both(vs)), v0 = mul2(u0, u0);
        m[i] = add2(m0, mul2(both(p.omb1), sub2(gi, m0)), p.one);
        u[i] = add2(v0, mul2(both(p.omb2), sub2(mul2(gi, gi), v0)), p.one);
        least = min3(least, u[i].x, u[i].y);
    }
    const bool tiny = least < 0x1p-100f;
    if (!tiny) {
#pragma unroll
        for (int i = 0; i < 4; ++i) u[i] = root2(u[i]);
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) u[i] = make_float2(__fsqrt_rn(u[i].x), __fsqrt_rn(u[i].y));
    }
    float th[8];
    read_operand(th, stage, lane, t.param_type());
    float am = 0.0f, au = 0.0f;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2 d = fma2(u[i], both(p.inv_sqrt_bc2), both(p.eps));
        const float2 step = mul2(mul2(both(p.step_size), m[i]), make_float2(rcp_1(d.x), rcp_1(d.y)));
        const float2 x = make_float2(th[2 * i], th[2 * i + 1]);
        const float2 y = sub2(x, fma2(both(eta_wd), x, step));
        th[2 * i] = y.x; th[2 * i + 1] = y.y;
        am = max3_abs(am, m[i].x, m[i].y);
        au = max3_abs(au, u[i].x, u[i].y);
    }
    const unsigned mine = at + lane * 8;
    store8(t.param + mine * bytes_of(t.param_type()), 0, th, t.param_type());
    if (t.copy_type != QSR_NONE) store8(t.copy + mine * bytes_of(t.copy_type), 0, th, t.copy_type);
    am = warp_max(am);
    au = warp_max(au);
    if (fmaxf(am, au) == infinity()) {                // only finite values make the scale
        am = au = 0.0f;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            am = fmaxf(am, fmaxf(finite_or_0(fabsf(m[i].x)), finite_or_0(fabsf(m[i].y))));
            au = fmaxf(au, fmaxf(finite_or_0(u[i].x), finite_or_0(u[i].y)));
        }
        am = warp_max(am);
        au = warp_max(au);
    }
    const BlockScale bm = block_scale(am), bu = block_scale(au);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        m[i] = mul2(m[i], both(bm.inv));
        u[i] = mul2(u[i], both(bu.inv));
        // what is positive stays positive; a lane without zeros need not ask which elements are
        if (!tiny) u[i] = make_float2(max_nan(u[i].x, kCodeMin), max_nan(u[i].y, kCodeMin));
        else u[i] = make_float2(u[i].x > 0.0f ? fmaxf(u[i].x, kCodeMin) : u[i].x, u[i].y > 0.0f ? fmaxf(u[i].y, kCodeMin) : u[i].y);
    }
    *reinterpret_cast<uint2 *>(t.m + mine) = make_uint2(to_e4m3x4(m[0], m[1]), to_e4m3x4(m[2], m[3]));
    *reinterpret_cast<uint2 *>(t.v + mine) = make_uint2(to_e4m3x4(u[0], u[1]), to_e4m3x4(u[2], u[3]));
    return make_float2(bm.scale, bu.scale);
}

template <bool S8>
__device__ __forceinline__ bool step_aligned(const ListTensor &t, const void *grad)
{
    return aligned_to(t.param, bytes_of_8(t.param_type)) && aligned_to(grad, bytes_of_8(t.grad_type)) &&
           aligned_to(t.m, S8 ? 8 : 32) && aligned_to(t.v, S8 ? 8 : 32) &&
           (t.copy_type == QSR_NONE || aligned_to(t.copy, bytes_of_8(t.copy_type)));
}

__global__ void __launch_bounds__(kThreads) list_step_kernel(const __grid_constant__ ListStepParams p)
{
    const ListChunk c = p.chunks[blockIdx.x];
    const ListTensor t = p.tensors[c.tensor];
    const void *grad = p.grads[c.tensor];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const float g_scale = p.clip ? p.grad_scale * p.clip[c.tensor / p.tensors_per_worker] : p.grad_scale;
    const float eta_wd = p.eta_wd * t.wd_scale;
    const bool vec = step_aligned<false>(t, grad);
    for (int b = warp; b * 256 < c.n; b += kWarps) {
        const int64_t e0 = c.offset + b * 256;
        const int n = min(256, c.n - b * 256);
        if (vec && n == 256) step_block_f32<true>(p, t, grad, e0, n, lane, g_scale, eta_wd);
        else step_block_f32<false>(p, t, grad, e0, n, lane, g_scale, eta_wd);
    }
}

// States in 8 bits.  A warp starts the copies of all its blocks (at most kListStages) into shared memory before it works on the
// first one: the work per byte is too much to leave the loads waiting in registers for it.
template <int PT, int GT>
__global__ void __launch_bounds__(kThreads, 4) list_step_codes_kernel(const __grid_constant__ ListStepParams p, const unsigned stage_bytes,
                                                                      const unsigned n_stages)
{
    extern __shared__ uint4 stages[];
    const ListChunk c = p.chunks[blockIdx.x];
    const ListTensor &tensor = p.tensors[c.tensor];
    const void *const grad = p.grads[c.tensor];
    const unsigned warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const bool vec = step_aligned<true>(tensor, grad);
    Chunk<PT, GT> t;
    t.param_type_ = tensor.param_type; t.grad_type_ = tensor.grad_type; t.copy_type = tensor.copy_type;
    t.param = static_cast<char *>(tensor.param) + c.offset * bytes_of(t.param_type());
    t.grad = static_cast<const char *>(grad) + c.offset * bytes_of(t.grad_type());
    t.copy = static_cast<char *>(tensor.copy) + c.offset * bytes_of(t.copy_type);
    t.m = static_cast<char *>(tensor.m) + c.offset;
    t.v = static_cast<char *>(tensor.v) + c.offset;
    const unsigned whole = vec ? c.n >> 8 : 0;            // whole blocks on the fast path: 0 .. whole - 1
    const unsigned mine = whole > warp ? (whole - warp + kWarps - 1) / kWarps : 0;
    const char *const my_stages = reinterpret_cast<const char *>(stages) + warp * n_stages * stage_bytes;
    const unsigned smem = unsigned(__cvta_generic_to_shared(my_stages));
    for (unsigned i = 0; i < mine; ++i) {
        const unsigned at = (warp + i * kWarps) * 256;
        const unsigned s_param = smem + i * stage_bytes, s_grad = s_param + 256 * bytes_of(t.param_type()), s_codes = s_grad + 256 * bytes_of(t.grad_type());
        fetch_operand(s_param, t.param, at, lane, t.param_type());
        fetch_operand(s_grad, t.grad, at, lane, t.grad_type());
        copy_async<8>(s_codes + lane * 8, t.m + (at + lane * 8));
        copy_async<8>(s_codes + 256 + lane * 8, t.v + (at + lane * 8));
        asm volatile("cp.async.commit_group;" ::: "memory");
    }
    // lane i holds the scales of the warp's i-th block
    float ms = 0.0f, vs = 0.0f;
    float *const m_scale = tensor.m_scale + (c.offset >> 8), *const v_scale = tensor.v_scale + (c.offset >> 8);
    if (lane < mine) { ms = m_scale[warp + lane * kWarps]; vs = v_scale[warp + lane * kWarps]; }
    const float g_scale = p.clip ? p.grad_scale * p.clip[c.tensor / p.tensors_per_worker] : p.grad_scale;
    const float eta_wd = p.eta_wd * tensor.wd_scale;
    for (unsigned i = 0; i < mine; ++i) {
        const unsigned later = mine - 1 - i;                  // groups that may still be on their way
        if (later >= 3) copy_wait<3>();
        else if (later == 2) copy_wait<2>();
        else if (later == 1) copy_wait<1>();
        else copy_wait<0>();
        __syncwarp();
        const float2 s = step_block_codes(p, t, my_stages + i * stage_bytes, (warp + i * kWarps) * 256, lane,
                                          __shfl_sync(0xffffffffu, ms, i), __shfl_sync(0xffffffffu, vs, i), g_scale, eta_wd);
        if (lane == i) { ms = s.x; vs = s.y; }
    }
    if (lane < mine) { m_scale[warp + lane * kWarps] = ms; v_scale[warp + lane * kWarps] = vs; }
    for (unsigned b = whole + warp; b * 256 < unsigned(c.n); b += kWarps)
        step_block_codes_any(p, c.tensor, c.offset + b * 256, min(256, c.n - int(b * 256)), lane, g_scale, eta_wd);
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

namespace {

template <int PT, int GT>
int launch_codes(const ListStepParams &p, const ListShape &s, cudaStream_t st)
{
    const int smem = kWarps * s.stages * s.stage_bytes;
    const auto kernel = list_step_codes_kernel<PT, GT>;
    static std::atomic<uint64_t> raised{0};
    if (smem > 48 * 1024)
        if (int err = allow_shared(reinterpret_cast<const void *>(kernel), 56 * 1024, raised)) return err;
    kernel<<<unsigned(s.chunks), kThreads, size_t(smem), st>>>(p, unsigned(s.stage_bytes), unsigned(s.stages));
    return int(cudaGetLastError());
}

template <int PT>
int launch_codes_grad(const ListStepParams &p, const ListShape &s, cudaStream_t st)
{
    if (s.grad_type == QSR_F32) return launch_codes<PT, QSR_F32>(p, s, st);
    if (s.grad_type == QSR_BF16) return launch_codes<PT, QSR_BF16>(p, s, st);
    return launch_codes<PT, QSR_F16>(p, s, st);
}

}  // namespace

int allow_shared(const void *kernel, int bytes, std::atomic<uint64_t> &raised)
{
    int dev = 0;
    if (cudaError_t err = cudaGetDevice(&dev)) return int(err);
    const uint64_t bit = dev < 64 ? uint64_t(1) << dev : 0;
    if (raised.load(std::memory_order_relaxed) & bit) return 0;
    if (cudaError_t err = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes)) return int(err);
    raised.fetch_or(bit, std::memory_order_relaxed);
    return 0;
}

int launch_list_step(const ListStepParams &p, const ListShape &s, void *stream)
{
    const cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (s.stage_bytes == 0) {
        list_step_kernel<<<unsigned(s.chunks), kThreads, 0, st>>>(p);
        return int(cudaGetLastError());
    }
    if (s.param_type == QSR_NONE) return launch_codes<QSR_NONE, QSR_NONE>(p, s, st);
    if (s.param_type == QSR_F32) return launch_codes_grad<QSR_F32>(p, s, st);
    if (s.param_type == QSR_BF16) return launch_codes_grad<QSR_BF16>(p, s, st);
    return launch_codes_grad<QSR_F16>(p, s, st);
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
