// Lists of tensors: the AdamW step (OPT of Eq. 1, arXiv 2310.14423) over many tensors in one launch, states in fp32 or in
// 8 bits, and the replica mean that ends a round (Algorithm 2).  Element-wise streams: no contraction, no tensor cores.
//
// A thread block works on one chunk of one tensor (the table says which), its eight warps on blocks of 256 consecutive elements,
// eight per lane.  The chunk's types, addresses and factors are the same for the whole block, so nothing diverges.
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

// The largest magnitude of a lane's N values; infinities (a sum or a square beyond fp32) do not count, and become the largest
// finite number, whose code is 448 as theirs, or 0 where the scale is 0 (infinity * 0 would be NaN).
template <int N>
__device__ __forceinline__ float amax_of_finite(float (&x)[N])
{
    float amax = 0.0f;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        if (fabsf(x[i]) == infinity()) x[i] = copysignf(3.402823466e38f, x[i]);
        else amax = fmaxf(amax, fabsf(x[i]));
    }
    return amax;
}

__device__ __forceinline__ float code_of(float x, float inv, bool positive)
{
    const float q = __fmul_rn(x, inv);
    return positive && q > 0.0f ? fmaxf(q, kCodeMin) : q;
}

// Eight codes of a lane: two words when the lane owns eight consecutive elements, otherwise single bytes packed the same way.
template <bool VEC>
__device__ __forceinline__ uint2 load_codes_raw(const uint8_t *base, int64_t e0, int n, int lane)
{
    if (VEC) return *reinterpret_cast<const uint2 *>(base + e0 + lane * 8);
    uint2 w = make_uint2(0u, 0u);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if (lane + 32 * i < n) w.x |= uint32_t(base[e0 + lane + 32 * i]) << (8 * i);
        if (lane + 32 * (i + 4) < n) w.y |= uint32_t(base[e0 + lane + 32 * (i + 4)]) << (8 * i);
    }
    return w;
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

// Two fp32 operations per instruction (sm_100), each rounded like its scalar form.  Sums are written as fused multiply-adds with
// a factor of one: nvcc 12.9 makes one fused operation of a packed product and the packed sum that takes it (also of
// mul.rn.f32x2 and add.rn.f32x2), and the codes would not be those of the formulas (the tests compare them bit for bit).
__device__ __forceinline__ float2 both(float x) { return make_float2(x, x); }
__device__ __forceinline__ float2 mul2(float2 a, float2 b) { return __fmul2_rn(a, b); }
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) { return __ffma2_rn(a, b, c); }
__device__ __forceinline__ float2 add2(float2 a, float2 b, float one) { return __ffma2_rn(b, both(one), a); }
__device__ __forceinline__ float2 sub2(float2 a, float2 b) { return __ffma2_rn(b, both(-1.0f), a); }

// sqrt(v) rounded to nearest for finite v >= 2^-100: one Newton step on s = v * rsqrt(v) with the residual v - s^2 formed by a fused
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

// The same element by element, zeros beyond n: ragged blocks and unaligned tensors.
__device__ __forceinline__ char *element_of(char *smem, unsigned e, int type)
{
    return type == QSR_F32 ? smem + piece(e >> 2) * 16 + (e & 3) * 4 : smem + e * 2;
}
__device__ __forceinline__ void fill_operand(char *smem, const char *chunk, unsigned at, int n, int lane, int type)
{
    Raw8 r;
    load_raw<false>(r, chunk, at, n, lane, type);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        char *const to = element_of(smem, lane + 32 * i, type);
        if (type == QSR_F32) *reinterpret_cast<uint32_t *>(to) = r.w[i];
        else *reinterpret_cast<uint16_t *>(to) = uint16_t(r.w[i]);
    }
}
__device__ __forceinline__ void fill_codes(char *smem, const char *chunk, unsigned at, int n, int lane)
{
    const uint2 w = load_codes_raw<false>(reinterpret_cast<const uint8_t *>(chunk), at, n, lane);
#pragma unroll
    for (int i = 0; i < 8; ++i) smem[lane + 32 * i] = char((i < 4 ? w.x : w.y) >> (8 * (i & 3)));
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

// A block whose operands have arrived in shared memory (parameter, gradient, codes of m, codes of v): eight consecutive
// elements per lane, in pairs.  ms, vs: the block's scales before; returned: after.  Without `vec` the results go through the
// same shared memory and are written element by element, the first n of them.
template <int PT, int GT>
__device__ __forceinline__ float2 step_block_codes(const ListStepParams &p, const Chunk<PT, GT> &t, char *stage, unsigned at, int n, bool vec,
                                                   unsigned lane, float ms, float vs, float g_scale, float eta_wd)
{
    float g[8];
    char *const s_grad = stage + 256 * bytes_of(t.param_type()), *const s_codes = s_grad + 256 * bytes_of(t.grad_type());
    read_operand(g, s_grad, lane, t.grad_type());
    const uint2 mw = *reinterpret_cast<const uint2 *>(s_codes + lane * 8), vw = *reinterpret_cast<const uint2 *>(s_codes + 256 + lane * 8);
    float2 m[4], u[4];
    from_e4m3x4(m[0], m[1], mw.x);
    from_e4m3x4(m[2], m[3], mw.y);
    from_e4m3x4(u[0], u[1], vw.x);
    from_e4m3x4(u[2], u[3], vw.y);
    float least = infinity(), most = 0.0f;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        float2 gi = make_float2(g[2 * i], g[2 * i + 1]);
        if (g_scale != 1.0f) gi = mul2(gi, both(g_scale));
        const float2 m0 = mul2(m[i], both(ms)), u0 = mul2(u[i], both(vs)), v0 = mul2(u0, u0);
        m[i] = add2(m0, mul2(both(p.omb1), sub2(gi, m0)), p.one);
        u[i] = add2(v0, mul2(both(p.omb2), sub2(mul2(gi, gi), v0)), p.one);
        least = min3(least, u[i].x, u[i].y);
        most = max3_abs(most, u[i].x, u[i].y);
    }
    const bool general = least < 0x1p-100f || most == infinity();       // g * g may overflow where g does not
    if (!general) {
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
    if (vec) {
        store8(t.param + mine * bytes_of(t.param_type()), 0, th, t.param_type());
        if (t.copy_type != QSR_NONE) store8(t.copy + mine * bytes_of(t.copy_type), 0, th, t.copy_type);
    } else {
        __syncwarp();                                 // parameter and gradient have been read: 1024 bytes at least
        *reinterpret_cast<float4 *>(stage + piece(2 * lane) * 16) = make_float4(th[0], th[1], th[2], th[3]);
        *reinterpret_cast<float4 *>(stage + piece(2 * lane + 1) * 16) = make_float4(th[4], th[5], th[6], th[7]);
    }
    if (fmaxf(am, au) == infinity()) {                // only finite values make the scale
        am = amax_of_finite(reinterpret_cast<float (&)[8]>(m));
        au = amax_of_finite(reinterpret_cast<float (&)[8]>(u));
    }
    const BlockScale bm = block_scale(warp_max(am)), bu = block_scale(warp_max(au));
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        m[i] = mul2(m[i], both(bm.inv));
        u[i] = mul2(u[i], both(bu.inv));
        // what is positive stays positive; a lane without zeros need not ask which elements are
        if (!general) u[i] = make_float2(max_nan(u[i].x, kCodeMin), max_nan(u[i].y, kCodeMin));
        else u[i] = make_float2(u[i].x > 0.0f ? fmaxf(u[i].x, kCodeMin) : u[i].x, u[i].y > 0.0f ? fmaxf(u[i].y, kCodeMin) : u[i].y);
    }
    const uint2 m_codes = make_uint2(to_e4m3x4(m[0], m[1]), to_e4m3x4(m[2], m[3])), v_codes = make_uint2(to_e4m3x4(u[0], u[1]), to_e4m3x4(u[2], u[3]));
    if (vec) {
        *reinterpret_cast<uint2 *>(t.m + mine) = m_codes;
        *reinterpret_cast<uint2 *>(t.v + mine) = v_codes;
    } else {
        *reinterpret_cast<uint2 *>(s_codes + lane * 8) = m_codes;
        *reinterpret_cast<uint2 *>(s_codes + 256 + lane * 8) = v_codes;
        __syncwarp();
#pragma unroll 1
        for (int e = lane; e < n; e += 32) {
            const float x = *reinterpret_cast<const float *>(element_of(stage, e, QSR_F32));
            store1(t.param, at + e, x, t.param_type());
            if (t.copy_type != QSR_NONE) store1(t.copy, at + e, x, t.copy_type);
            t.m[at + e] = s_codes[e];
            t.v[at + e] = s_codes[256 + e];
        }
    }
    return make_float2(bm.scale, bu.scale);
}

__device__ __forceinline__ bool step_aligned(const ListTensor &t, const void *grad)
{
    return aligned_to(t.param, bytes_of_8(t.param_type)) && aligned_to(grad, bytes_of_8(t.grad_type)) && aligned_to(t.m, 8) &&
           aligned_to(t.v, 8) && (t.copy_type == QSR_NONE || aligned_to(t.copy, bytes_of_8(t.copy_type)));
}

// How many elements a pointer lies past the last place where eight of them may be accessed at once.
__device__ __forceinline__ int phase_of(const void *p, int type)
{
    const unsigned a = unsigned(reinterpret_cast<uintptr_t>(p));
    return type == QSR_F32 ? (a & 31u) >> 2 : (a & 15u) >> 1;
}
// A chunk of a tensor whose operands all have the same phase moves up to the next place where that access is allowed (and
// over its end by as much, unless the tensor ends there); the tensor's first elements become a block of their own.
// Tensors cut out of one buffer at odd offsets then run at full width (2 x 61 of them, clipped: 69 -> 57 us).
struct Span { int64_t begin; int n, head; };
__device__ __forceinline__ Span span_of(const ListChunk &c, int64_t numel, int phase)
{
    Span s;
    s.head = (8 - phase) & 7;
    s.begin = c.offset + s.head;
    const int64_t end = c.offset + c.n == numel ? numel : c.offset + c.n + s.head;
    s.n = int(max(int64_t(0), min(end, numel) - s.begin));
    return s;
}

// States in fp32.  Bound by memory: 16 to 32 bytes per element against about 30 instructions.  Two blocks per multiprocessor
// with 128 bytes of loads per thread on their way (256-bit accesses) are enough; caps of 80 and 64 registers for more of them
// cost 2 % and 12 %.  ViT-B/16's 150 tensors, fp32 parameters, bf16 gradients and copies: 364 us for 2.42 GB, 6.65 TB/s.
__global__ void __launch_bounds__(kThreads) list_step_kernel(const __grid_constant__ ListStepParams p)
{
    const ListChunk c = p.chunks[blockIdx.x];
    const ListTensor t = p.tensors[c.tensor];
    const void *grad = p.grads[c.tensor];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const float g_scale = p.clip ? p.grad_scale * p.clip[c.tensor / p.tensors_per_worker] : p.grad_scale;
    const float eta_wd = p.eta_wd * t.wd_scale;
    const int phase = phase_of(t.param, t.param_type);
    const bool vec = phase_of(grad, t.grad_type) == phase && phase_of(t.m, QSR_F32) == phase && phase_of(t.v, QSR_F32) == phase &&
                     (t.copy_type == QSR_NONE || phase_of(t.copy, t.copy_type) == phase);
    const Span s = span_of(c, t.numel, vec ? phase : 0);
    for (int b = warp; b * 256 < s.n; b += kWarps) {
        const int64_t e0 = s.begin + b * 256;
        const int n = min(256, s.n - b * 256);
        if (vec && n == 256) step_block_f32<true>(p, t, grad, e0, n, lane, g_scale, eta_wd);
        else step_block_f32<false>(p, t, grad, e0, n, lane, g_scale, eta_wd);
    }
    if (c.offset == 0 && s.head > 0 && warp == kWarps - 1)
        step_block_f32<false>(p, t, grad, 0, int(min(int64_t(s.head), t.numel)), lane, g_scale, eta_wd);
}

// States in 8 bits.  A warp starts the copies of all its blocks (at most kListStages) into shared memory before it works on the
// first one: with the loads in registers instead (and as many warps as fit) the same work took 350 us where it now takes 229,
// waiting for memory half the time.  Now the instructions count: about 50 per element, so lists with 16 bytes per element run at
// memory speed (ViT-B/16, fp32 parameters, bf16 gradients and copies: 229 us for 1.39 GB, 6.05 TB/s) and lists with 10 are bound
// by issue (ResNet-152, all bf16: 123 us for 0.61 GB, 4.9 TB/s).  Four blocks per multiprocessor; three and five were 8 % slower.
template <int PT, int GT>
__global__ void __launch_bounds__(kThreads, 4) list_step_codes_kernel(const __grid_constant__ ListStepParams p, const unsigned stage_bytes,
                                                                      const unsigned n_stages)
{
    extern __shared__ uint4 stages[];
    const ListChunk c = p.chunks[blockIdx.x];
    const ListTensor &tensor = p.tensors[c.tensor];
    const void *const grad = p.grads[c.tensor];
    const unsigned warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const bool vec = step_aligned(tensor, grad);
    Chunk<PT, GT> t;
    t.param_type_ = tensor.param_type; t.grad_type_ = tensor.grad_type; t.copy_type = tensor.copy_type;
    t.param = static_cast<char *>(tensor.param) + c.offset * bytes_of(t.param_type());
    t.grad = static_cast<const char *>(grad) + c.offset * bytes_of(t.grad_type());
    t.copy = static_cast<char *>(tensor.copy) + c.offset * bytes_of(t.copy_type);
    t.m = static_cast<char *>(tensor.m) + c.offset;
    t.v = static_cast<char *>(tensor.v) + c.offset;
    const unsigned blocks = unsigned(c.n + 255) >> 8, mine = blocks > warp ? (blocks - warp + kWarps - 1) / kWarps : 0;
    char *const my_stages = reinterpret_cast<char *>(stages) + warp * n_stages * stage_bytes;
    for (unsigned i = 0; i < mine; ++i) {
        const unsigned at = (warp + i * kWarps) * 256;
        const int n = c.n - int(at);
        char *const s_param = my_stages + i * stage_bytes, *const s_grad = s_param + 256 * bytes_of(t.param_type()), *const s_codes = s_grad + 256 * bytes_of(t.grad_type());
        if (vec && n >= 256) {
            const unsigned to = unsigned(__cvta_generic_to_shared(s_param)), grad_at = unsigned(s_grad - s_param), codes_at = unsigned(s_codes - s_param);
            fetch_operand(to, t.param, at, lane, t.param_type());
            fetch_operand(to + grad_at, t.grad, at, lane, t.grad_type());
            copy_async<8>(to + codes_at + lane * 8, t.m + (at + lane * 8));
            copy_async<8>(to + codes_at + 256 + lane * 8, t.v + (at + lane * 8));
        } else {
            fill_operand(s_param, t.param, at, n, lane, t.param_type());
            fill_operand(s_grad, t.grad, at, n, lane, t.grad_type());
            fill_codes(s_codes, t.m, at, n, lane);
            fill_codes(s_codes + 256, t.v, at, n, lane);
        }
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
        const unsigned at = (warp + i * kWarps) * 256;
        const int n = c.n - int(at);
        const float2 s = step_block_codes(p, t, my_stages + i * stage_bytes, at, min(n, 256), vec && n >= 256, lane, __shfl_sync(0xffffffffu, ms, i),
                                          __shfl_sync(0xffffffffu, vs, i), g_scale, eta_wd);
        if (lane == i) { ms = s.x; vs = s.y; }
    }
    if (lane < mine) { m_scale[warp + lane * kWarps] = ms; v_scale[warp + lane * kWarps] = vs; }
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

// Clipping's norms (reads the gradients once more: bound by memory).  Sum of squares of each chunk's gradients; the last block of a worker to finish adds its chunks up -- in chunk order, so
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
    const Span span = span_of(c, p.tensors[c.tensor].numel, phase_of(grad, type));
    float s = 0.0f;
    auto add = [&](const Raw8 &r, bool vec) {
        float g[8];
        if (vec) widen<true>(g, r, type);
        else widen<false>(g, r, type);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float x = g[i] * p.grad_scale;
            s = fmaf(x, x, s);
        }
    };
    for (int b = warp; b * 256 < span.n; b += kWarps) {
        const int64_t e0 = span.begin + b * 256;
        const int n = min(256, span.n - b * 256);
        Raw8 r;
        if (n == 256) load_raw<true>(r, grad, e0, n, lane, type);
        else load_raw<false>(r, grad, e0, n, lane, type);
        add(r, n == 256);
    }
    if (c.offset == 0 && span.head > 0 && warp == kWarps - 1) {
        Raw8 r;
        load_raw<false>(r, grad, 0, int(min(int64_t(span.head), p.tensors[c.tensor].numel)), lane, type);
        add(r, false);
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

// What lane k knows of worker k0 + k's tensor: where operand A (0 parameter, 1 m, 2 v) lies, its working copy, its scales.
struct Place { char *data, *copy; float *scale; };
template <int A>
__device__ __forceinline__ Place place_of(const ListSyncParams &p, int tensor, int k)
{
    const ListTensor &t = p.tensors[min(k, p.workers - 1) * p.tensors_per_worker + tensor];
    return Place{static_cast<char *>(A == 0 ? t.param : A == 1 ? t.m : t.v), static_cast<char *>(t.copy), A == 1 ? t.m_scale : t.v_scale};
}
__device__ __forceinline__ char *of_lane(char *p, int lane)
{
    return reinterpret_cast<char *>(__shfl_sync(0xffffffffu, reinterpret_cast<unsigned long long>(p), lane));
}

// Four elements of a lane as they lie in memory: adjacent ones (VEC; 16 bytes of fp32, 8 of a 16-bit type), otherwise lane,
// lane + 32, ... of the warp's 128, n of which are valid.
template <bool F32, bool VEC>
__device__ __forceinline__ uint4 load_quad(const char *base, int64_t e0, int n, int lane)
{
    uint4 r = make_uint4(0u, 0u, 0u, 0u);
    if (VEC && F32) {
        asm volatile("ld.global.L1::no_allocate.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(r.x), "=r"(r.y), "=r"(r.z), "=r"(r.w) : "l"(base + (e0 + lane * 4) * 4) : "memory");
    } else if (VEC) {
        asm volatile("ld.global.L1::no_allocate.v2.b32 {%0, %1}, [%2];" : "=r"(r.x), "=r"(r.y) : "l"(base + (e0 + lane * 4) * 2) : "memory");
    } else {
        const int type = F32 ? QSR_F32 : QSR_BF16;            // the width is what counts here
        if (lane < n) r.x = load1(base, e0 + lane, type);
        if (lane + 32 < n) r.y = load1(base, e0 + lane + 32, type);
        if (lane + 64 < n) r.z = load1(base, e0 + lane + 64, type);
        if (lane + 96 < n) r.w = load1(base, e0 + lane + 96, type);
    }
    return r;
}
template <bool F32, bool VEC>
__device__ __forceinline__ void add_quad(float (&s)[4], uint4 r, int type)
{
    if (F32) {
        s[0] += __uint_as_float(r.x); s[1] += __uint_as_float(r.y); s[2] += __uint_as_float(r.z); s[3] += __uint_as_float(r.w);
    } else if (VEC) {
        const float2 a = widen2(r.x, type), b = widen2(r.y, type);
        s[0] += a.x; s[1] += a.y; s[2] += b.x; s[3] += b.y;
    } else {
        s[0] += widen1(r.x, type); s[1] += widen1(r.y, type); s[2] += widen1(r.z, type); s[3] += widen1(r.w, type);
    }
}
template <bool VEC>
__device__ __forceinline__ void store_quad(char *base, int64_t e0, int n, int lane, const float (&s)[4], int type)
{
    if (VEC && type == QSR_F32) *reinterpret_cast<float4 *>(base + (e0 + lane * 4) * 4) = make_float4(s[0], s[1], s[2], s[3]);
    else if (VEC) *reinterpret_cast<uint2 *>(base + (e0 + lane * 4) * 2) = make_uint2(narrow2(s[0], s[1], type), narrow2(s[2], s[3], type));
    else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (lane + 32 * i < n) store1(base, e0 + lane + 32 * i, s[i], type);
    }
}

// Adds N workers' elements, k ascending, all N loads started before the first is waited for.
template <bool F32, bool VEC, int N>
__device__ __forceinline__ void add_workers(float (&s)[4], char *data, int k, int64_t e0, int n, int lane, int type)
{
    uint4 r[N];
#pragma unroll
    for (int j = 0; j < N; ++j) r[j] = load_quad<F32, VEC>(of_lane(data, k + j), e0, n, lane);
#pragma unroll
    for (int j = 0; j < N; ++j) add_quad<F32, VEC>(s, r[j], type);
}

__device__ __forceinline__ float mean_of(float sum, const ListSyncParams &p) { return p.inverse > 0.0f ? sum * p.inverse : sum / p.divisor; }

// Mean over the workers of 128 elements in the caller's type, written back to every worker (parameters: to the working copies
// too).  `mine`: the first 32 workers' places, loaded anew where there are more.
template <int A, bool F32, bool VEC>
__device__ __forceinline__ void mean_block(const ListSyncParams &p, Place mine, int tensor, int type, int copy_type, int64_t e0, int n, int lane)
{
    float s[4] = {0.0f, 0.0f, 0.0f, 0.0f};
    for (int k0 = 0; k0 < p.workers; k0 += 32) {
        if (p.workers > 32) mine = place_of<A>(p, tensor, k0 + lane);
        const int here = min(32, p.workers - k0);
        int k = 0;
        for (; k + 4 <= here; k += 4) add_workers<F32, VEC, 4>(s, mine.data, k, e0, n, lane, type);
        if ((here & 3) == 3) add_workers<F32, VEC, 3>(s, mine.data, k, e0, n, lane, type);
        else if (here & 2) add_workers<F32, VEC, 2>(s, mine.data, k, e0, n, lane, type);
        else if (here & 1) add_workers<F32, VEC, 1>(s, mine.data, k, e0, n, lane, type);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) s[i] = mean_of(s[i], p);
    for (int k0 = 0; k0 < p.workers; k0 += 32) {
        if (p.workers > 32) mine = place_of<A>(p, tensor, k0 + lane);
        const int here = min(32, p.workers - k0);
        for (int k = 0; k < here; ++k) {
            store_quad<VEC>(of_lane(mine.data, k), e0, n, lane, s, F32 ? QSR_F32 : type);
            if (A == 0 && copy_type != QSR_NONE) store_quad<VEC>(of_lane(mine.copy, k), e0, n, lane, s, copy_type);
        }
    }
}

// Adds N workers' 8-bit states, 4 * WORDS codes of a lane: the values they stand for (of v: the squares of its codes).
template <int A, int WORDS>
__device__ __forceinline__ void add_codes(float (&s)[4 * WORDS], const uint32_t (&w)[WORDS], float scale)
{
#pragma unroll
    for (int i = 0; i < WORDS; ++i) {
        float2 f[2];
        from_e4m3x4(f[0], f[1], w[i]);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const float y = __fmul_rn(j & 1 ? f[j >> 1].y : f[j >> 1].x, scale);
            s[4 * i + j] = __fadd_rn(s[4 * i + j], A == 1 ? y : __fmul_rn(y, y));
        }
    }
}
template <int A, int N>
__device__ __forceinline__ float finish_states(float (&s)[N], const ListSyncParams &p)
{
    float amax = 0.0f;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        s[i] = mean_of(s[i], p);
        if (A == 2) s[i] = __fsqrt_rn(s[i]);
        amax = fmaxf(amax, fabsf(s[i]));
    }
    return amax == infinity() ? amax_of_finite(s) : amax;
}

// Mean of a block of 256 8-bit states, rounded to 8 bits once: ragged blocks and unaligned tensors, byte by byte.
template <int A>
__device__ __noinline__ void mean_codes_any(const ListSyncParams &p, int tensor, int64_t e0, int n, int lane)
{
    const int64_t b = e0 >> 8;
    float s[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) s[i] = 0.0f;
    for (int k0 = 0; k0 < p.workers; k0 += 32) {
        const Place mine = place_of<A>(p, tensor, k0 + lane);
        const int here = min(32, p.workers - k0);
        const float scale = mine.scale[b];
        for (int k = 0; k < here; k += 4) {
            uint2 r[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) r[j] = load_codes_raw<false>(reinterpret_cast<const uint8_t *>(of_lane(mine.data, min(k + j, here - 1))), e0, n, lane);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const uint32_t w[2] = {r[j].x, r[j].y};
                const float sc = __shfl_sync(0xffffffffu, scale, k + j);
                if (k + j < here) add_codes<A, 2>(s, w, sc);
            }
        }
    }
    const BlockScale q = block_scale(warp_max(finish_states<A, 8>(s, p)));
    for (int k0 = 0; k0 < p.workers; k0 += 32) {
        const Place mine = place_of<A>(p, tensor, k0 + lane);
        const int here = min(32, p.workers - k0);
        for (int k = 0; k < here; ++k) store_codes<false>(reinterpret_cast<uint8_t *>(of_lane(mine.data, k)), e0, n, lane, s, q.inv, A == 2);
        if (lane < here) mine.scale[b] = q.scale;
    }
}

// Two whole blocks of 256 at once: sixteen adjacent codes per lane, a block per half warp, so that a warp reads 512 bytes of each
// worker at a time and has eight workers' loads on their way.
template <int A, int N>
__device__ __forceinline__ void add_codes_of(float (&s)[16], char *data, float scale0, float scale1, int k, int64_t e0, int lane)
{
    uint4 r[N];
#pragma unroll
    for (int j = 0; j < N; ++j) r[j] = load_quad<true, true>(of_lane(data, k + j) + e0, 0, 128, lane);
#pragma unroll
    for (int j = 0; j < N; ++j) {
        const float a = __shfl_sync(0xffffffffu, scale0, k + j), b = __shfl_sync(0xffffffffu, scale1, k + j);
        const uint32_t w[4] = {r[j].x, r[j].y, r[j].z, r[j].w};
        add_codes<A, 4>(s, w, lane < 16 ? a : b);
    }
}
template <int A>
__device__ __forceinline__ void mean_codes(const ListSyncParams &p, Place mine, int tensor, int64_t e0, int lane)
{
    const int64_t b = e0 >> 8;
    float s[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) s[i] = 0.0f;
    for (int k0 = 0; k0 < p.workers; k0 += 32) {
        if (p.workers > 32) mine = place_of<A>(p, tensor, k0 + lane);
        const int here = min(32, p.workers - k0);
        const float scale0 = lane < here ? mine.scale[b] : 0.0f, scale1 = lane < here ? mine.scale[b + 1] : 0.0f;
        int k = 0;
        for (; k + 8 <= here; k += 8) add_codes_of<A, 8>(s, mine.data, scale0, scale1, k, e0, lane);
        if (here & 4) { add_codes_of<A, 4>(s, mine.data, scale0, scale1, k, e0, lane); k += 4; }
        for (; k < here; ++k) add_codes_of<A, 1>(s, mine.data, scale0, scale1, k, e0, lane);
    }
    float amax = finish_states<A, 16>(s, p);
#pragma unroll
    for (int d = 8; d; d >>= 1) amax = fmaxf(amax, __shfl_xor_sync(0xffffffffu, amax, d));
    const BlockScale q = block_scale(amax);
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i)
        w[i] = to_e4m3x4(make_float2(code_of(s[4 * i], q.inv, A == 2), code_of(s[4 * i + 1], q.inv, A == 2)),
                         make_float2(code_of(s[4 * i + 2], q.inv, A == 2), code_of(s[4 * i + 3], q.inv, A == 2)));
    const float scale0 = __shfl_sync(0xffffffffu, q.scale, 0), scale1 = __shfl_sync(0xffffffffu, q.scale, 16);
    for (int k0 = 0; k0 < p.workers; k0 += 32) {
        if (p.workers > 32) mine = place_of<A>(p, tensor, k0 + lane);
        const int here = min(32, p.workers - k0);
        for (int k = 0; k < here; ++k)
            *reinterpret_cast<uint4 *>(of_lane(mine.data, k) + e0 + lane * 16) = make_uint4(w[0], w[1], w[2], w[3]);
        if (lane < here) { mine.scale[b] = scale0; mine.scale[b + 1] = scale1; }
    }
}

// Whether every worker's operand may be accessed four (codes: sixteen) elements at a time.
template <int A>
__device__ __forceinline__ bool sync_aligned(const ListSyncParams &p, Place x, int tensor, int type, int copy_type, bool codes, int lane)
{
    bool ok = true;
    for (int k = lane; k < p.workers; k += 32) {
        if (k >= 32) x = place_of<A>(p, tensor, k);
        ok = ok && aligned_to(x.data, codes ? 16u : bytes_of_8(type) / 2);
        if (A == 0 && copy_type != QSR_NONE) ok = ok && aligned_to(x.copy, bytes_of_8(copy_type) / 2);
    }
    return __all_sync(0xffffffffu, ok);
}

template <int A, bool F32>
__device__ __forceinline__ void sync_blocks(const ListSyncParams &p, const ListChunk &c, int type, int copy_type)
{
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const Place mine = place_of<A>(p, c.tensor, lane);
    const bool vec = sync_aligned<A>(p, mine, c.tensor, type, copy_type, false, lane);
    for (int b = warp; b * 128 < c.n; b += kWarps) {
        const int64_t e0 = c.offset + b * 128;
        const int n = min(128, c.n - b * 128);
        if (vec && n == 128) mean_block<A, F32, true>(p, mine, c.tensor, type, copy_type, e0, n, lane);
        else mean_block<A, F32, false>(p, mine, c.tensor, type, copy_type, e0, n, lane);
    }
}
template <int A>
__device__ __forceinline__ void sync_codes(const ListSyncParams &p, const ListChunk &c)
{
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const Place mine = place_of<A>(p, c.tensor, lane);
    const int pairs = sync_aligned<A>(p, mine, c.tensor, QSR_F32, QSR_NONE, true, lane) ? c.n / 512 : 0;
    for (int b = warp; b < pairs; b += kWarps) mean_codes<A>(p, mine, c.tensor, c.offset + b * 512, lane);
    for (int b = 2 * pairs + warp; b * 256 < c.n; b += kWarps)
        mean_codes_any<A>(p, c.tensor, c.offset + b * 256, min(256, c.n - b * 256), lane);
}
template <int A, bool S8>
__device__ __forceinline__ void sync_states(const ListSyncParams &p, const ListChunk &c)
{
    if (S8) sync_codes<A>(p, c);
    else sync_blocks<A, true>(p, c, QSR_F32, QSR_NONE);
}

// The round end.  Grid: worker 0's chunks by 1 (parameters) or 3 (parameters, m, v).  Bound by memory: every value is read and
// written once, and what counts is that all workers' loads of a block are on their way together, in pieces of 512 bytes per
// worker (8-bit states in pieces of 256 bytes: 2.20 instead of 1.70 ms).  Eight ViT-B/16 replicas with copies: parameters alone
// 1.13 ms (6.1 TB/s), with 8-bit states averaged 1.70 ms (5.7 TB/s).  The number of blocks per multiprocessor: fp32 states five
// (three packed bf16 replicas, element by element: 76 us with 48 bytes of spills; with four blocks 84 and none), 8-bit states
// three (1.70 ms with 28 bytes of spills; with four 1.73 and 360 bytes).
template <bool S8>
__global__ void __launch_bounds__(kThreads, S8 ? 3 : 5) list_sync_kernel(const __grid_constant__ ListSyncParams p)
{
    const ListChunk c = p.chunks[blockIdx.x];
    const int type = p.tensors[c.tensor].param_type, copy_type = p.tensors[c.tensor].copy_type;
    if (blockIdx.y == 0) {
        if (type == QSR_F32) sync_blocks<0, true>(p, c, type, copy_type);
        else sync_blocks<0, false>(p, c, type, copy_type);
    } else if (blockIdx.y == 1) sync_states<1, S8>(p, c);
    else sync_states<2, S8>(p, c);
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
