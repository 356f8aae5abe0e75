// Orthogonalised momentum: the kernels.  See include/qsr.h for the formulas and muon_api.cu for the launches.
//
// The iterate X (rows x cols) and the symmetric m x m matrices A = X X^T (X^T X if there are more rows than columns; m is the shorter
// side) and C = a I + b A + c A^2 are held as fp16 blocks of 64 x 64 (8 KB), each exactly as a tensor-core operand wants it in
// shared memory (rows of 128 bytes, 16-byte pieces exchanged by the row number's low three bits).  A block is one copy of 8 KB in a row
// and serves as an operand with either side along the products' sum: columns along it as it is, rows along it if
// the instruction is told so ("outer").  So X X^T and C X, or X^T X and X C, read the same blocks of X, no matrix is ever transposed,
// and of A and C only the tiles on and above the diagonal are computed; what lies below is read from its mirror image.
// Blocks are padded with zeros, hence any sizes.  Products of C with A or with another C, for which the last iterations of long matrices are
// taken (muon_api.cu), are symmetric too, since all of them are polynomials of the same A.
//
// With three products per multiplication, X, A and C are sums of two fp16 numbers and hi hi + hi lo + lo hi are accumulated.
#include <cuda.h>
#include <cuda_runtime.h>

#include "wide.cuh"

namespace qsr {

namespace {

constexpr float kA = kMuonA, kB = kMuonB, kC = kMuonC, kGramScale = kMuonGramScale, kFactorScale = kMuonFactorScale;

// The launches of a step follow one another closely: each is started before the one before it has ended, and waits for that.
__device__ __forceinline__ void wait_for_launch_before() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
__device__ __forceinline__ void let_next_launch_start() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }

// ---- momentum and norms ----------------------------------------------------------------------------------

__device__ __forceinline__ bool address_aligned(const void *p, unsigned bytes) { return (reinterpret_cast<uintptr_t>(p) & (bytes - 1)) == 0; }

constexpr int kMomentumThreads = 256;

__device__ __forceinline__ float updated(const MuonParams &p, float m, float g) { return fmaf(p.one_minus_beta, g - m, m); }
// What is orthogonalised, from the new momentum.
__device__ __forceinline__ float direction(const MuonParams &p, float m, float g) { return p.nesterov ? fmaf(p.beta, m - g, g) : m; }

// scale / (norm + eps), whose product with the largest element is at most `scale`; nothing to scale where the norm is 0.  As two factors that
// are taken one after the other, the first a power of two: the norm of numbers that fp32 holds lies between 2^-149 and 2^146, and for
// the far ends the quotient, or its full precision, is beyond fp32.
struct Scaling { float lift, factor; };
__device__ __forceinline__ Scaling scaling_of(float scale, double squares, float eps)
{
    const double length = sqrt(squares) + double(eps);
    if (length == 0.0) return {1.0f, 0.0f};
    const float lift = length < 0x1p-60 ? 0x1p80f : length > 0x1p60 ? 0x1p-64f : 1.0f;
    return {lift, float(double(scale) / (length * double(lift)))};                          // NaN stays NaN, infinity gives 0
}

// m <- m + (1 - beta)(g - m) and the sum of squares of u, chunk by chunk; the matrix's last chunk adds them in their order.
// Squares and sums in binary64: the norm neither overflows nor loses small elements.  Bound by memory: 85 M elements with bf16 gradients (10 bytes
// each) 143 us, 5.9 TB/s.
__global__ void __launch_bounds__(kMomentumThreads) momentum_kernel(const __grid_constant__ MuonParams p)
{
    __shared__ double scratch[kMomentumThreads / 32];
    __shared__ bool last;
    let_next_launch_start();
    const MuonChunk c = p.chunks[blockIdx.x];
    const MuonMatrix &t = p.matrices[c.matrix];
    const void *grad = p.grads[c.matrix];
    const int gt = t.grad_type;
    float *momentum = t.momentum;
    const bool vec = address_aligned(grad, gt == QSR_F32 ? 32 : 16) && address_aligned(momentum, 32);
    double s = 0.0;
    if (vec) {
#pragma unroll 2
        for (int i = int(threadIdx.x) * 8; i + 8 <= c.n; i += kMomentumThreads * 8) {
            Raw8 rg, rm;
            load8(rg, grad, c.offset + i, gt);
            load32(rm, momentum + c.offset + i);
            float g[8], m[8];
            widen8(g, rg, gt);
            widen8(m, rm, QSR_F32);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float gs = g[j] * p.grad_scale;
                m[j] = updated(p, m[j], gs);
                const double u = double(direction(p, m[j], gs));
                s = fma(u, u, s);
            }
            store8(momentum, c.offset + i, m, QSR_F32);
        }
    }
    for (int i0 = (vec ? c.n & ~7 : 0) + int(threadIdx.x); i0 < c.n; i0 += 8 * kMomentumThreads) {
        uint32_t g[8];
        float m[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int i = i0 + j * kMomentumThreads;
            g[j] = i < c.n ? load1(grad, c.offset + i, gt) : 0u;
            m[j] = i < c.n ? momentum[c.offset + i] : 0.0f;
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int i = i0 + j * kMomentumThreads;
            const float gs = widen1(g[j], gt) * p.grad_scale, to = updated(p, m[j], gs);
            const double u = double(direction(p, to, gs));
            if (i < c.n) {
                s = fma(u, u, s);
                momentum[c.offset + i] = to;
            }
        }
    }
#pragma unroll
    for (int d = 16; d; d >>= 1) s += __shfl_xor_sync(0xffffffffu, s, d);
    if ((threadIdx.x & 31) == 0) scratch[threadIdx.x >> 5] = s;
    __syncthreads();
    if (threadIdx.x == 0) {
        s = scratch[0];
        for (int w = 1; w < kMomentumThreads / 32; ++w) s += scratch[w];
        p.partial[blockIdx.x] = s;
        __threadfence();
        last = atomicAdd(&p.arrived[c.matrix], 1u) + 1u == unsigned(t.chunks);
        __threadfence();
    }
    __syncthreads();
    if (!last) return;
    s = 0.0;
    for (int i = threadIdx.x; i < t.chunks; i += kMomentumThreads) s += __ldcg(&p.partial[t.first_chunk + i]);
#pragma unroll
    for (int d = 16; d; d >>= 1) s += __shfl_xor_sync(0xffffffffu, s, d);
    __syncthreads();
    if ((threadIdx.x & 31) == 0) scratch[threadIdx.x >> 5] = s;
    __syncthreads();
    if (threadIdx.x == 0) {
        s = scratch[0];
        for (int w = 1; w < kMomentumThreads / 32; ++w) s += scratch[w];
        const Scaling z = scaling_of(t.scale, s, p.eps);
        p.factor[2 * c.matrix] = z.lift;
        p.factor[2 * c.matrix + 1] = z.factor;
        p.arrived[c.matrix] = 0;
    }
}

__global__ void __launch_bounds__(kMomentumThreads) clear_kernel(const __grid_constant__ MuonParams p)
{
    const MuonChunk c = p.chunks[blockIdx.x];
    float *to = p.matrices[c.matrix].momentum + c.offset;
    for (int i = threadIdx.x; i < c.n; i += kMomentumThreads) to[i] = 0.0f;
}

// ---- blocks ----------------------------------------------------------------------------------------------

constexpr int kBlockElements = 64 * 64;

// Where a block of 64 x 64 holds its element (r, c).
__device__ __forceinline__ int place(int r, int c) { return r * 64 + ((c >> 3) ^ (r & 7)) * 8 + (c & 7); }

// A thread's elements of a block, sixteen in two halves of eight.  WIDE: eight adjacent ones of a row, eight threads to a row (the
// matrix's rows are aligned to eight elements); otherwise eight of a column, 64 threads side by side.
template <bool WIDE> __device__ __forceinline__ int row_in(int half) { return WIDE ? half * 32 + (int(threadIdx.x) >> 3) : (int(threadIdx.x) >> 6) * 16 + half * 8; }
template <bool WIDE> __device__ __forceinline__ int column_in() { return WIDE ? (int(threadIdx.x) & 7) * 8 : int(threadIdx.x) & 63; }

// A half: how many of its elements the matrix has, the first one's place, and the distance from one to the next.
struct Half { int64_t at, step; int n; };
template <bool WIDE>
__device__ __forceinline__ Half half_of(const MuonMatrix &t, const MuonBlock &b, int half)
{
    const int64_t r = int64_t(b.p) * 64 + row_in<WIDE>(half), c = int64_t(b.q) * 64 + column_in<WIDE>(), rows = t.rows, cols = t.cols;
    return Half{r * cols + c, WIDE ? 1 : cols, c >= cols || r >= rows ? 0 : WIDE ? 8 : int(min(rows - r, int64_t(8)))};
}
template <bool WIDE>
__device__ __forceinline__ void take(Raw8 &raw, const void *base, int type, const Half &o)
{
    if (WIDE && o.n) {
        load8(raw, base, o.at, type);
        return;
    }
#pragma unroll
    for (int k = 0; k < 8; ++k) raw.w[k] = !WIDE && k < o.n ? load1(base, o.at + k * o.step, type) : 0u;
}
template <bool WIDE>
__device__ __forceinline__ void widen(float (&x)[8], const Raw8 &raw, int type)
{
    if (WIDE) widen8(x, raw, type);
    else
#pragma unroll
        for (int k = 0; k < 8; ++k) x[k] = widen1(raw.w[k], type);
}
template <bool WIDE>
__device__ __forceinline__ void give(void *base, const float (&x)[8], int type, const Half &o)
{
    if (WIDE) {
        if (o.n) store8(base, o.at, x, type);
        return;
    }
#pragma unroll
    for (int k = 0; k < 8; ++k)
        if (k < o.n) store1(base, o.at + k * o.step, x[k], type);
}
__device__ __forceinline__ bool wide_rows(const MuonMatrix &t, const void *base, int type) { return t.cols % 8 == 0 && address_aligned(base, type == QSR_F32 ? 32 : 16); }

// One block of the first iterate: u from the new momentum, times scale / (norm + eps); zeros beyond the matrix.
template <bool WIDE>
__device__ __forceinline__ void pack_block(const MuonParams &p, const MuonMatrix &t, const MuonBlock &b, const void *grad)
{
    const bool both = p.products == 3;
    uint16_t *block = t.x + (int64_t(b.q) * t.rb + b.p) * kBlockElements;
    const int64_t lo = int64_t(t.rb) * t.cb * kBlockElements;
    const int grad_type = t.grad_type;
    const float *momentum = t.momentum;
    const float *by = p.factor + 2 * b.matrix;                   // read where they are wanted: held, they cost a block on a multiprocessor (152 us)
    Half o[2];
    Raw8 g[2], m[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        o[h] = half_of<WIDE>(t, b, h);
        take<WIDE>(g[h], grad, grad_type, o[h]);
        take<WIDE>(m[h], momentum, QSR_F32, o[h]);
    }
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        float gs[8], x[8];
        widen<WIDE>(gs, g[h], grad_type);
        widen<WIDE>(x, m[h], QSR_F32);
        Raw8 hi, rest;
#pragma unroll
        for (int k = 0; k < 8; ++k) x[k] = direction(p, x[k], gs[k] * p.grad_scale);
        if (!WIDE || by[0] != 1.0f)
#pragma unroll
            for (int k = 0; k < 8; ++k) x[k] *= by[0];
#pragma unroll
        for (int k = 0; k < 8; ++k) x[k] = k < o[h].n ? x[k] * by[1] : 0.0f;      // whatever the factor
#pragma unroll
        for (int k = 0; k < 8; k += 2) {
            const __half2 f = __floats2half2_rn(x[k], x[k + 1]);
            const float2 back = __half22float2(f);
            hi.w[k / 2] = *reinterpret_cast<const uint32_t *>(&f);
            rest.w[k / 2] = narrow2(x[k] - back.x, x[k + 1] - back.y, QSR_F16);
        }
        if (WIDE) {
            uint16_t *to = block + place(row_in<true>(h), column_in<true>());
            store16(to, hi);
            if (both) store16(to + lo, rest);
        } else {
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                uint16_t *to = block + place(row_in<false>(h) + k, column_in<false>());
                *to = uint16_t(hi.w[k / 2] >> (k % 2 * 16));
                if (both) to[lo] = uint16_t(rest.w[k / 2] >> (k % 2 * 16));
            }
        }
    }
}
// The blocks are taken from the last one on: the end of what the launch before has written is still in the second-level cache.  Bound by memory:
// 85 M elements 121 us with one product (8 bytes each), 139 us with three (10 bytes).
__global__ void __launch_bounds__(256) pack_kernel(const __grid_constant__ MuonParams p)
{
    let_next_launch_start();
    const MuonBlock b = p.blocks[gridDim.x - 1 - blockIdx.x];
    const MuonMatrix &t = p.matrices[b.matrix];
    const void *grad = p.grads[b.matrix];
    wait_for_launch_before();
    if (wide_rows(t, grad, t.grad_type) && wide_rows(t, t.momentum, QSR_F32)) pack_block<true>(p, t, b, grad);
    else pack_block<false>(p, t, b, grad);
}

// theta <- theta - (lr wd theta + lr update_scale X) for one block of the last iterate.  85 M elements: 103 us in bf16 (6 bytes each), 178 us in fp32
// with three products and bf16 copies (14 bytes, 6.7 TB/s).  The last product's threads doing this with the sums they have saves
// 1 % of the step with one product, and costs 3 % with three, whose sums leave no registers for the parameters.
template <bool WIDE>
__device__ __forceinline__ void apply_block(const MuonParams &p, const MuonMatrix &t, const MuonBlock &b)
{
    const bool both = p.products == 3;
    const float decay = p.lr_decay * t.wd_scale, step = p.lr * t.update_scale / t.scale;
    const uint16_t *block = t.x_last + (int64_t(b.q) * t.rb + b.p) * kBlockElements;
    const int64_t lo = int64_t(t.rb) * t.cb * kBlockElements;
    const int type = t.param_type, copy_type = t.copy_type;
    void *param = t.param, *copy = t.copy;
    Half o[2];
    Raw8 old[2], hi[2], rest[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        o[h] = half_of<WIDE>(t, b, h);
        take<WIDE>(old[h], param, type, o[h]);
        if (WIDE) {
            const uint16_t *x = block + place(row_in<true>(h), column_in<true>());
            load16(hi[h], x);
            if (both) load16(rest[h], x + lo);
        } else {
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const uint16_t *x = block + place(row_in<false>(h) + k, column_in<false>());
                hi[h].w[k] = *x;
                if (both) rest[h].w[k] = x[lo];
            }
        }
    }
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        float theta[8], x[8], more[8];
        widen<WIDE>(theta, old[h], type);
        widen<WIDE>(x, hi[h], QSR_F16);
        if (both) {
            widen<WIDE>(more, rest[h], QSR_F16);
#pragma unroll
            for (int k = 0; k < 8; ++k) x[k] += more[k];
        }
#pragma unroll
        for (int k = 0; k < 8; ++k) theta[k] -= fmaf(decay, theta[k], step * x[k]);
        give<WIDE>(param, theta, type, o[h]);
        if (copy_type != QSR_NONE) give<WIDE>(copy, theta, copy_type, o[h]);
    }
}
__global__ void __launch_bounds__(256) apply_kernel(const __grid_constant__ MuonParams p)
{
    const MuonBlock b = p.blocks[gridDim.x - 1 - blockIdx.x];
    const MuonMatrix &t = p.matrices[b.matrix];
    wait_for_launch_before();
    if (wide_rows(t, t.param, t.param_type) && (t.copy_type == QSR_NONE || wide_rows(t, t.copy, t.copy_type))) apply_block<true>(p, t, b);
    else apply_block<false>(p, t, b);
}

// ---- products --------------------------------------------------------------------------------------------

enum { GRAM = 0, FACTOR = 1, ITERATE = 2 };

struct Maps { CUtensorMap single, pair; };

constexpr int kResultWarps = 8;
constexpr int kProductThreads = 128 + kResultWarps * 32;      // warps: 0 and 3 copies, 1 products, 2 accumulators' allocation, then results
constexpr int kBlockBytes = kBlockElements * 2;
constexpr int kOperandBlocks = 4;            // of a stage in each block of a pair: two of its 128 rows, two of its 128 columns
constexpr int kStageBlocks = 24;             // shared memory for operands: 6 stages of one product, 3 of three
constexpr int kTurn = 2;                     // blocks along the sum that tensor memory adds up, with three products
constexpr unsigned kAccumulators = 512;      // columns of tensor memory: two tiles of 256
constexpr long long kPatience = 6000000000;  // clocks that a wait may take, some seconds

__device__ __forceinline__ uint32_t shared_address(const void *p) { return uint32_t(__cvta_generic_to_shared(p)); }

__device__ __forceinline__ void barrier_init(uint32_t bar, unsigned count)
{
    asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count) : "memory");
}
// The barrier at the same place in the shared memory of the pair's first block.
__device__ __forceinline__ void barrier_arrive_first(uint32_t bar)
{
    asm volatile("{.reg .b32 a; mapa.shared::cluster.u32 a, %0, 0; mbarrier.arrive.shared::cluster.b64 _, [a];}" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void pair_sync()
{
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ void barrier_expect(uint32_t bar, unsigned bytes)
{
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
__device__ __forceinline__ bool barrier_try(uint32_t bar, unsigned parity)
{
    uint32_t done;
    asm volatile("{.reg .pred p; mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2; selp.u32 %0, 1, 0, p;}"
                 : "=r"(done) : "r"(bar), "r"(parity) : "memory");
    return done != 0;
}
// False, with *stop set, if the phase does not end in time; false too where another role has given up, if `heed`.
__device__ __forceinline__ bool barrier_wait(uint32_t bar, unsigned parity, volatile unsigned *stop, bool heed = true)
{
    if (barrier_try(bar, parity)) return true;
    const long long begin = clock64();
    for (;;) {
        for (int i = 0; i < 64; ++i)
            if (barrier_try(bar, parity)) return true;
        if (heed && *stop) return false;
        if (clock64() - begin > kPatience) break;
    }
    *stop = 1;
    return false;
}
__device__ __forceinline__ bool elected()
{
    uint32_t e;
    asm volatile("{.reg .pred p; elect.sync _|p, 0xffffffff; selp.u32 %0, 1, 0, p;}" : "=r"(e));
    return e != 0;
}
// Blocks of 64 x 64 into this thread block's shared memory, one (`single`) or two neighbours (`pair`), reported to the barrier at that
// place in the pair's first thread block.  The maps see the workspace's blocks as rows of 128 bytes, and a copy is 64 or 128 whole
// rows: the tiled form is used because only that one may report to the other thread block's barrier.
__device__ __forceinline__ void copy_blocks(uint32_t to, const CUtensorMap *map, int row, uint32_t bar)
{
    asm volatile("cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];" ::"r"(to), "l"(map),
                 "r"(0), "r"(row), "r"(bar & 0xfeffffffu) : "memory");
}

// Operand descriptor: rows of 128 bytes with 128-byte swizzle, groups of eight rows 1024 bytes apart; with the sum along the
// columns of blocks ("outer"), the next 64 rows or columns of the operand are `next` bytes further (otherwise right behind).
__device__ __forceinline__ uint64_t operand(uint32_t address, uint32_t next = kBlockBytes)
{
    return uint64_t((address >> 4) & 0x3fff) | uint64_t(next >> 4) << 16 | uint64_t(1024 >> 4) << 32 | uint64_t(1) << 46 | uint64_t(2) << 61;
}
// Instruction descriptor: fp16 operands, fp32 accumulators, m x n; outer_a / outer_b: the operand's rows in memory run along the sum.
__device__ __forceinline__ uint32_t instruction(int m, int n, bool outer_a, bool outer_b)
{
    return 1u << 4 | uint32_t(outer_a) << 15 | uint32_t(outer_b) << 16 | uint32_t(n >> 3) << 17 | uint32_t(m >> 4) << 24;
}
__device__ __forceinline__ void multiply(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, bool add)
{
    asm volatile("{.reg .pred p; setp.ne.b32 p, %4, 0; tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;}" ::"r"(d), "l"(a), "l"(b),
                 "r"(idesc), "r"(uint32_t(add)) : "memory");
}
// Arrives at both blocks' barriers when the products issued so far are done.
__device__ __forceinline__ void commit(uint32_t bar)
{
    asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(bar), "h"(uint16_t(3)) : "memory");
}
__device__ __forceinline__ void load_accumulators(float (&v)[16], uint32_t address)
{
    uint32_t r[16];
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];\n\t"
                 "tcgen05.wait::ld.sync.aligned;"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]),
                   "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
                 : "r"(address) : "memory");
#pragma unroll
    for (int i = 0; i < 16; ++i) v[i] = __uint_as_float(r[i]);
}
__device__ __forceinline__ void load_accumulators(float (&v)[32], uint32_t address)
{
    uint32_t r[32];
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, %17, %18, %19, %20, "
                 "%21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];\n\t"
                 "tcgen05.wait::ld.sync.aligned;"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]),
                   "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]),
                   "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
                 : "r"(address) : "memory");
#pragma unroll
    for (int i = 0; i < 32; ++i) v[i] = __uint_as_float(r[i]);
}
__device__ __forceinline__ void fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }

// Whether an operand's blocks at step k of the sum lie with the sum along their rows ("outer").  Of a symmetric matrix the blocks in row
// tile P, column tile T (four blocks each) are held where P <= T; elsewhere their mirror images are read, the other way round.
__device__ __forceinline__ bool outer_left(const MuonTile &w, int k) { return w.flags & MUON_LEFT_ITERATE ? (w.flags & MUON_LEFT_OUTER) != 0 : w.i > (k >> 2); }
__device__ __forceinline__ bool outer_right(const MuonTile &w, int k) { return w.flags & MUON_RIGHT_ITERATE ? (w.flags & MUON_RIGHT_OUTER) != 0 : (w.q >> 2) > (k >> 2); }

// Half a row of a block, 32 elements: where 32-byte pair `pair` (0 or 1) of it lies, in elements.  A thread has a row in its registers and
// writes it 32 bytes at a time, a sector each.  (Passing the tile through shared memory, so that a warp's accesses are adjacent, was
// slower: the operands' copies and the products take most of what shared memory can do.)
__device__ __forceinline__ int pair_at(int row, int half, int pair) { return row * 64 + ((half * 2 + pair) ^ ((row & 7) >> 1)) * 16; }
// The words of 16 elements, in the order in which odd rows and even rows hold their two 16-byte pieces.
__device__ __forceinline__ void exchange(Raw8 &r, bool odd)
{
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const uint32_t a = r.w[k], b = r.w[k + 4];
        r.w[k] = odd ? b : a;
        r.w[k + 4] = odd ? a : b;
    }
}
// 32 elements in fp16, and what fp16 leaves of them `lo` elements further.
template <bool REST>
__device__ __forceinline__ void store_half(uint16_t *block, int64_t lo, int row, int half, const float (&v)[32])
{
#pragma unroll
    for (int pair = 0; pair < 2; ++pair) {
        uint16_t *to = block + pair_at(row, half, pair);
        Raw8 hi, rest;
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const float a = v[pair * 16 + 2 * k], b = v[pair * 16 + 2 * k + 1];
            hi.w[k] = narrow2(a, b, QSR_F16);
            if (REST) {
                const float2 f = widen2(hi.w[k], QSR_F16);
                rest.w[k] = narrow2(a - f.x, b - f.y, QSR_F16);
            }
        }
        exchange(hi, row & 1);
        store32(to, hi);
        if (REST) {
            exchange(rest, row & 1);
            store32(to + lo, rest);
        }
    }
}
__device__ __forceinline__ void load_half(Raw8 (&r)[2], const uint16_t *block, int row, int half)
{
#pragma unroll
    for (int pair = 0; pair < 2; ++pair) load32(r[pair], block + pair_at(row, half, pair));
}
__device__ __forceinline__ void add_half(float (&v)[32], Raw8 (&r)[2], int row, float factor)
{
#pragma unroll
    for (int pair = 0; pair < 2; ++pair) {
        exchange(r[pair], row & 1);
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const float2 f = widen2(r[pair].w[k], QSR_F16);
            v[pair * 16 + 2 * k] = fmaf(factor, f.x, v[pair * 16 + 2 * k]);
            v[pair * 16 + 2 * k + 1] = fmaf(factor, f.y, v[pair * 16 + 2 * k + 1]);
        }
    }
}

// From sums to what is held: all but the polynomial's middle term.
template <bool POLYNOMIAL>
__device__ __forceinline__ void finish_half(float (&x)[32], float factor, int diagonal)
{
#pragma unroll
    for (int k = 0; k < 32; ++k) x[k] = POLYNOMIAL ? x[k] * factor + (k == diagonal ? kA * kFactorScale : 0.0f) : x[k] * factor;
}
constexpr float kMiddle = kB * kFactorScale / kGramScale;

// Where a warp's part of a tile goes: 32 rows of blocks (bp, bq) and (bp, bq + 1), a row to a thread.
struct Target {
    int blocks;                        // of the two, how many the result has
    int row, diagonal;                 // in its block; where it meets the matrix's diagonal, in their columns
    uint16_t *to;
    const uint16_t *gram;              // polynomial: the same elements of A
    int64_t column, lo;                // from a block to the next, from fp16 to what it leaves
    float factor;
    __device__ __forceinline__ Target(const MuonTile &w, const MuonParams &p, int rank, int group, int part, int lane)
    {
        const int bp = w.i * 4 + rank * 2 + (group >> 1), bq = w.q + part * 2;
        blocks = bp < w.rows ? min(2, min(w.columns, w.q + w.width) - bq) : 0;
        row = (group & 1) * 32 + lane;
        diagonal = (bp - bq) * 64 + row;
        const int64_t at = int64_t(bq) * w.rows + bp;
        to = p.data + (w.to + at) * kBlockElements;
        gram = p.data + (w.gram + at) * kBlockElements;
        column = int64_t(w.rows) * kBlockElements;
        lo = int64_t(w.columns) * column;
        factor = w.factor;
    }
};

struct Shared {
    uint64_t full[6], empty[6], ready[2], drained[2];
    uint32_t tensor_memory;
    unsigned stop;
};

// A pair of blocks (one per multiprocessor) takes tiles of 256 x 256 elements (or 256 x 128), pair, + pairs, ...; each has 128 of the tile's rows and
// 128 of its columns in its shared memory, a stage at a time of 64 along the sum, and 128 x 256 sums in its tensor memory.  Two warps of
// each block copy; one thread of the first block issues the products of both; eight warps take the tile before out of the other half of tensor memory.  Compared with 128 x 256 tiles of
// single blocks, each multiprocessor copies and reads two thirds of the bytes for a product.  Bound by the tensor cores at the clock that the power limit
// leaves (1.5 to 1.6 GHz): C X for 85 M elements with m = 768 takes 96 us, 1.36 PFLOP/s, and 293 us with three products (1.34); symmetric
// m x m products, whose diagonal tiles are half wasted, 30 and 83 us for 48 matrices.  Staging results through shared memory and
// sixteen warps for them were slower.
template <bool POLYNOMIAL, int PRODUCTS>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kProductThreads, 1)
product_kernel(const __grid_constant__ MuonParams p, const __grid_constant__ Maps maps, const MuonTile *tiles, int n_tiles)
{
    extern __shared__ char raw[];
    __shared__ Shared sh;
    constexpr int PARTS = PRODUCTS == 3 ? 2 : 1, STAGES = kStageBlocks / (kOperandBlocks * PARTS);
    constexpr int STEPS = PRODUCTS == 3 ? kTurn : 1;
    const uint32_t stage0 = (shared_address(raw) + 1023u) & ~1023u;
    constexpr uint32_t kStage = kOperandBlocks * PARTS * kBlockBytes;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int rank = int(blockIdx.x & 1), pair = int(blockIdx.x >> 1), pairs = int(gridDim.x >> 1);
    volatile unsigned *stop = &sh.stop;
    let_next_launch_start();
    if (threadIdx.x == 0) {
        for (int i = 0; i < STAGES; ++i) {
            barrier_init(shared_address(&sh.full[i]), 1);
            barrier_init(shared_address(&sh.empty[i]), 1);
        }
        for (int i = 0; i < 2; ++i) {
            barrier_init(shared_address(&sh.ready[i]), 1);
            barrier_init(shared_address(&sh.drained[i]), 2 * kResultWarps);
        }
        sh.stop = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
    __syncthreads();
    if (warp == 2) {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(shared_address(&sh.tensor_memory)), "r"(kAccumulators) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    }
    fence_before();
    pair_sync();
    fence_after();
    const uint32_t accumulators = sh.tensor_memory;
    wait_for_launch_before();

    if (warp == 0 || warp == 3) {
        // Copies: warp 0 those of the left operand, warp 3 those of the right one.  Everything is the same for the whole warp and one elected
        // thread issues: copies issued by several threads of a warp go out one by one, at a hundred clocks and more each.
        const bool left = warp == 0, one = elected();
        int stage = 0, issued = 0;
        unsigned phase = 0;
        bool going = true;
        MuonTile ahead = tiles[min(pair, n_tiles - 1)];          // read while the tile before is copied
        for (int tile = pair; tile < n_tiles && going; tile += pairs) {
            const MuonTile w = ahead;
            const int columns = min(w.width, w.columns - w.q), sums = w.sums, wide = columns > 2;
            const int at = left ? w.i * 4 + rank * 2 : w.q + (wide ? rank * 2 : rank);           // first of up to two blocks
            const int here = max(0, left ? min(2, w.rows - at) : min(wide ? 2 : 1, w.q + columns - at));
            const int both = min(4, w.rows - w.i * 4) + columns;                // blocks that the pair copies
            const int base = left ? w.left : w.right, pitch = left ? w.left_pitch : w.right_pitch, lo = left ? w.left_lo : w.right_lo;
            ahead = tiles[min(tile + pairs, n_tiles - 1)];
            for (int k = 0; k < sums; ++k) {
                if (!barrier_wait(shared_address(&sh.empty[stage]), phase ^ 1u, stop)) { going = false; break; }
                const uint32_t bar = shared_address(&sh.full[stage]), to = stage0 + stage * kStage + (left ? 0 : 2) * kBlockBytes;
                // blocks (at, k), (at + 1, k), which are neighbours, or blocks (k, at), (k, at + 1): of a symmetric matrix, their mirror images
                const bool outer = left ? outer_left(w, k) : outer_right(w, k);
                const int first = base + (outer ? at * pitch + k : k * pitch + at);
                if (one) {
                    if (left && rank == 0) barrier_expect(bar, unsigned(both * PARTS * kBlockBytes));
#pragma unroll
                    for (int part = 0; part < PARTS; ++part) {
                        const uint32_t into = to + part * kOperandBlocks * kBlockBytes;
                        const int row = (first + part * lo) * 64;
                        if (here == 2 && !outer) copy_blocks(into, &maps.pair, row, bar);
                        else {
                            if (here > 0) copy_blocks(into, &maps.single, row, bar);
                            if (here > 1) copy_blocks(into + kBlockBytes, &maps.single, row + pitch * 64, bar);
                        }
                    }
                }
                __syncwarp();
                issued++;
                if (++stage == STAGES) { stage = 0; phase ^= 1u; }
            }
        }
        // when the block ends nothing may be copying into its shared memory, or reading it: wait for the last stages
        for (int s = 0; s < STAGES && s < issued; ++s) {
            const int last = issued - 1 - s;
            const unsigned parity = unsigned(last / STAGES) & 1u;
            barrier_wait(shared_address(&sh.empty[last % STAGES]), parity, stop);
            if (rank == 0) barrier_wait(shared_address(&sh.full[last % STAGES]), parity, stop, false);
        }
    } else if (warp == 1 && rank == 0) {
        // the whole warp runs through the loop, so that descriptors are computed once for it, and one elected thread issues
        int stage = 0, buffer = 0;
        unsigned phase = 0, buffer_phase = 0;
        const bool one = elected();
        bool going = true;
        MuonTile ahead = tiles[min(pair, n_tiles - 1)];
        for (int tile = pair; tile < n_tiles && going; tile += pairs) {
            const MuonTile w = ahead;
            ahead = tiles[min(tile + pairs, n_tiles - 1)];
            const int sums = w.sums, wide = min(w.width, w.columns - w.q) > 2;
            for (int k = 0; k < sums; k += STEPS) {
                // STEPS stages at a time (with three products one turn of what tensor memory adds up), the smaller products of all of
                // them first: the fewer sums are added to an accumulator that has grown, the less is cut off
                const int steps = min(STEPS, sums - k);
                const bool last = k + steps == sums, begins = PRODUCTS == 3 || k == 0;
                const uint32_t d = accumulators + unsigned(buffer) * 256u;
                if (begins && !barrier_wait(shared_address(&sh.drained[buffer]), buffer_phase ^ 1u, stop)) { going = false; break; }
                uint64_t a[STEPS], b[STEPS], a_step[STEPS], b_step[STEPS];
                uint32_t idesc[STEPS], empty[STEPS];
                constexpr uint64_t lo = (kOperandBlocks * kBlockBytes) >> 4;
#pragma unroll
                for (int i = 0; i < STEPS; ++i) {
                    if (i >= steps) break;
                    if (!barrier_wait(shared_address(&sh.full[stage]), phase, stop)) { going = false; break; }
                    fence_after();
                    const bool outer_a = outer_left(w, k + i), outer_b = outer_right(w, k + i);
                    const uint32_t a0 = stage0 + stage * kStage;
                    idesc[i] = instruction(256, wide ? 256 : 128, outer_a, outer_b);
                    a[i] = operand(a0);
                    b[i] = operand(a0 + 2 * kBlockBytes);
                    a_step[i] = outer_a ? 2048 >> 4 : 32 >> 4;
                    b_step[i] = outer_b ? 2048 >> 4 : 32 >> 4;
                    empty[i] = shared_address(&sh.empty[stage]);
                    if (PRODUCTS == 3 && one)
#pragma unroll
                        for (int q = 0; q < 2; ++q)              // hi lo, lo hi
#pragma unroll
                            for (int s = 0; s < 4; ++s)
                                multiply(d, a[i] + q * lo + s * a_step[i], b[i] + (1 - q) * lo + s * b_step[i], idesc[i], i + q + s > 0);
                    if (++stage == STAGES) { stage = 0; phase ^= 1u; }
                }
                if (!going) break;
                if (one) {
#pragma unroll
                    for (int i = 0; i < STEPS; ++i) {
                        if (i >= steps) break;
#pragma unroll
                        for (int s = 0; s < 4; ++s)
                            multiply(d, a[i] + s * a_step[i], b[i] + s * b_step[i], idesc[i], PRODUCTS == 3 || k + i + s > 0);
                        commit(empty[i]);
                    }
                    if (PRODUCTS == 3 || last) commit(shared_address(&sh.ready[buffer]));
                }
                __syncwarp();
                if (PRODUCTS == 3 || last) {
                    buffer ^= 1;
                    if (buffer == 0) buffer_phase ^= 1u;
                }
            }
        }
    } else if (warp >= 4) {
        const int group = warp & 3, part = (warp - 4) >> 2;      // lanes 32 group.. of tensor memory, columns 128 part..
        int buffer = 0;
        unsigned buffer_phase = 0;
        const auto next = [&] {
            fence_before();
            __syncwarp();
            if (lane == 0) barrier_arrive_first(shared_address(&sh.drained[buffer]));
            buffer ^= 1;
            if (buffer == 0) buffer_phase ^= 1u;
        };
        const uint32_t from_lane = accumulators + unsigned(part * 128) + (unsigned(group * 32) << 16);
        bool going = true;
        for (int tile = pair; tile < n_tiles && going; tile += pairs) {
            if (PRODUCTS == 1) {
                const Target o(tiles[tile], p, rank, group, part, lane);
                Raw8 gram[2];
                if (POLYNOMIAL && o.blocks > 0) load_half(gram, o.gram, o.row, 0);
                if (!barrier_wait(shared_address(&sh.ready[buffer]), buffer_phase, stop)) break;
                fence_after();
#pragma unroll 1
                for (int h = 0; h < 2 * o.blocks; ++h) {         // 32 columns each
                    float v[32];
                    load_accumulators(v, from_lane + unsigned(buffer * 256 + h * 32));
                    finish_half<POLYNOMIAL>(v, o.factor, o.diagonal - h * 32);
                    if (POLYNOMIAL) {
                        add_half(v, gram, o.row, kMiddle);
                        if (h + 1 < 2 * o.blocks) load_half(gram, o.gram + ((h + 1) >> 1) * o.column, o.row, (h + 1) & 1);
                    }
                    store_half<false>(o.to + (h >> 1) * o.column, 0, o.row, h & 1, v);
                }
                next();
            } else {
                float v[4][32];
#pragma unroll
                for (int h = 0; h < 4; ++h)
#pragma unroll
                    for (int k = 0; k < 32; ++k) v[h][k] = 0.0f;
                int turns = (tiles[tile].sums + STEPS - 1) / STEPS;
#pragma unroll 1
                for (; turns > 0; --turns) {
                    if (!barrier_wait(shared_address(&sh.ready[buffer]), buffer_phase, stop)) { going = false; break; }
                    fence_after();
#pragma unroll
                    for (int h = 0; h < 8; ++h) {
                        float add[16];
                        load_accumulators(add, from_lane + unsigned(buffer * 256 + h * 16));
#pragma unroll
                        for (int k = 0; k < 16; ++k) v[h / 2][h % 2 * 16 + k] += add[k];
                    }
                    next();
                }
                if (!going) break;
                const Target o(tiles[tile], p, rank, group, part, lane);
#pragma unroll
                for (int h = 0; h < 4; ++h) {                    // 32 columns each
                    if (h >= 2 * o.blocks) break;
                    finish_half<POLYNOMIAL>(v[h], o.factor, o.diagonal - h * 32);
                    if (POLYNOMIAL) {
                        Raw8 gram[2];
#pragma unroll
                        for (int s = 0; s < 2; ++s) {
                            load_half(gram, o.gram + (h >> 1) * o.column + s * o.lo, o.row, h & 1);
                            add_half(v[h], gram, o.row, kMiddle);
                        }
                    }
                    store_half<true>(o.to + (h >> 1) * o.column, o.lo, o.row, h & 1, v[h]);
                }
            }
        }
    }
    __syncwarp();
    fence_before();
    pair_sync();                         // the other block's products read this one's shared memory and write its tensor memory
    if (threadIdx.x == 0 && *stop) *p.late = 1u;          // behind the barrier: any warp may have been the last to give up
    if (warp == 2) {
        fence_after();
        asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(accumulators), "r"(kAccumulators) : "memory");
    }
}

// ---- small matrices --------------------------------------------------------------------------------------

// A whole step of one matrix by one block: its shorter side is at most 128, its longer one at most 512 (with three products 256, or 512 for a
// shorter side of 64), and X and A fit in shared memory, where they stay through all iterations (C takes the place of A, every product that of its operand, once all sums are in tensor
// memory).  The general way takes a launch for every product, whatever its size: 115 us for four of 128 x 128, 25 us this way, of which
// fifteen products take 1.3 us each: one after the other, copies in and out of tensor memory included, and far from its rate.
constexpr int kSmallThreads = 512;

template <int PRODUCTS>
struct Resident {
    static constexpr int PARTS = PRODUCTS == 3 ? 2 : 1;
    char *x, *a;                          // blocks of X (rb x cb), then of A (mb x mb), column of blocks by column; the second part behind the first
    int rb, cb, mb;
    __device__ __forceinline__ int x_part() const { return rb * cb * kBlockBytes; }
    __device__ __forceinline__ int a_part() const { return mb * mb * kBlockBytes; }
};

// Issues D = left right for all its rows, 128 at a time into `columns` columns of tensor memory each.  Operands: address of their first
// block, bytes from a part to the next, blocks in a column (pitch), and whether the sum runs along the blocks' rows.
struct Operand { uint32_t at; int part, pitch; bool outer; };
template <int PRODUCTS>
__device__ __forceinline__ void issue_all(bool one, uint32_t d, const Operand &l, const Operand &r, int row_blocks, int column_blocks, int sums)
{
    const uint64_t l_step = l.outer ? 2048 >> 4 : 32 >> 4, r_step = r.outer ? 2048 >> 4 : 32 >> 4;                       // 16 along the sum
    const uint64_t l_next = uint64_t(l.outer ? 1 : l.pitch) * (kBlockBytes >> 4), r_next = uint64_t(r.outer ? 1 : r.pitch) * (kBlockBytes >> 4);      // 64
    for (int i = 0; i < row_blocks; i += 2)
        for (int j = 0; j < column_blocks; j += 4) {
            const uint32_t idesc = instruction(128, min(4, column_blocks - j) * 64, l.outer, r.outer), to = d + unsigned(i / 2 * column_blocks * 64 + j * 64);
            // no second block of 64 rows: the first once more
            const uint64_t l0 = operand(l.at + (l.outer ? i * l.pitch : i) * kBlockBytes, i + 1 < row_blocks ? l.pitch * kBlockBytes : 0);
            const uint64_t r0 = operand(r.at + (r.outer ? j * r.pitch : j) * kBlockBytes, r.pitch * kBlockBytes);
            uint32_t add = 0;
#pragma unroll
            for (int q = PRODUCTS == 3 ? 2 : 0; q >= 0; --q) {         // the small products first, over the whole sum
                uint64_t a = l0 + (q == 1 ? uint64_t(l.part >> 4) : 0), b = r0 + (q == 2 ? uint64_t(r.part >> 4) : 0);
                for (int k = 0; k < sums; ++k) {
                    if (one)
#pragma unroll
                        for (int s = 0; s < 4; ++s) {
                            asm volatile("{.reg .pred p; setp.ne.b32 p, %4, 0; tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;}" ::"r"(to), "l"(a + s * l_step),
                                         "l"(b + s * r_step), "r"(idesc), "r"(add) : "memory");
                            add = 1;
                        }
                    a += l_next;
                    b += r_next;
                }
            }
            __syncwarp();
        }
}

// 32 numbers of a row, half a block's, into a block in shared memory: fp16, and what it leaves.
template <int PRODUCTS>
__device__ __forceinline__ void keep_half(char *block, int part, int row, int half, const float (&v)[32])
{
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        uint4 hi, rest;
        uint32_t *h = &hi.x, *l = &rest.x;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float a = v[k * 8 + 2 * i], b = v[k * 8 + 2 * i + 1];
            h[i] = narrow2(a, b, QSR_F16);
            if (PRODUCTS == 3) {
                const float2 f = widen2(h[i], QSR_F16);
                l[i] = narrow2(a - f.x, b - f.y, QSR_F16);
            }
        }
        char *to = block + row * 128 + ((half * 4 + k) ^ (row & 7)) * 16;
        *reinterpret_cast<uint4 *>(to) = hi;
        if (PRODUCTS == 3) *reinterpret_cast<uint4 *>(to + part) = rest;
    }
}
__device__ __forceinline__ void add_kept(float (&v)[32], const char *block, int row, int half, float factor)
{
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const uint4 w = *reinterpret_cast<const uint4 *>(block + row * 128 + ((half * 4 + k) ^ (row & 7)) * 16);
        const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float2 f = widen2(u[i], QSR_F16);
            v[k * 8 + 2 * i] = fmaf(factor, f.x, v[k * 8 + 2 * i]);
            v[k * 8 + 2 * i + 1] = fmaf(factor, f.y, v[k * 8 + 2 * i + 1]);
        }
    }
}

// A thread's eight elements of block (p, q): adjacent ones of a row, or of a column where rows are not aligned.
template <bool WIDE>
__device__ __forceinline__ Half eighth_of(const MuonMatrix &t, int p, int q, int &row, int &col)
{
    row = WIDE ? int(threadIdx.x) >> 3 : (int(threadIdx.x) >> 6) * 8;
    col = WIDE ? (int(threadIdx.x) & 7) * 8 : int(threadIdx.x) & 63;
    const int64_t r = p * 64 + row, c = q * 64 + col, rows = t.rows, cols = t.cols;
    return Half{r * cols + c, WIDE ? 1 : cols, c >= cols || r >= rows ? 0 : WIDE ? 8 : int(min(rows - r, int64_t(8)))};
}
// Momentum, and the sum of squares of what is orthogonalised, which is kept for the first kKept blocks.
constexpr int kKept = 4;
struct Kept { float u[kKept][8]; };
template <bool WIDE>
__device__ __forceinline__ double small_momentum(const MuonParams &p, const MuonMatrix &t, const void *grad, Kept &kept)
{
    double s = 0.0;
    const int blocks = t.rb * t.cb, rb = t.rb, gt = t.grad_type;
    float *momentum = t.momentum;
    {
        Half o[kKept];
        Raw8 g[kKept], m[kKept];
        int bp = 0, bq = 0;
#pragma unroll
        for (int b = 0; b < kKept; ++b) {
            int row, col;
            o[b] = eighth_of<WIDE>(t, bp, bq, row, col);
            if (b >= blocks) o[b].n = 0;
            take<WIDE>(g[b], grad, gt, o[b]);
            take<WIDE>(m[b], momentum, QSR_F32, o[b]);
            if (++bp == rb) { bp = 0; ++bq; }
        }
#pragma unroll
        for (int b = 0; b < kKept; ++b) {
            float gs[8], ms[8];
            widen<WIDE>(gs, g[b], gt);
            widen<WIDE>(ms, m[b], QSR_F32);
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const float x = gs[k] * p.grad_scale;
                ms[k] = updated(p, ms[k], x);
                kept.u[b][k] = k < o[b].n ? direction(p, ms[k], x) : 0.0f;
                s = fma(double(kept.u[b][k]), double(kept.u[b][k]), s);
            }
            give<WIDE>(momentum, ms, QSR_F32, o[b]);
        }
    }
#pragma unroll 2
    for (int b = kKept; b < blocks; ++b) {
        int row, col;
        const Half o = eighth_of<WIDE>(t, b % rb, b / rb, row, col);
        Raw8 g, m;
        take<WIDE>(g, grad, gt, o);
        take<WIDE>(m, momentum, QSR_F32, o);
        float gs[8], ms[8];
        widen<WIDE>(gs, g, gt);
        widen<WIDE>(ms, m, QSR_F32);
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const float x = gs[k] * p.grad_scale;
            ms[k] = updated(p, ms[k], x);
            const double u = double(direction(p, ms[k], x));
            if (k < o.n) s = fma(u, u, s);
        }
        give<WIDE>(momentum, ms, QSR_F32, o);
    }
    return s;
}
// The first iterate.
template <bool WIDE, int PRODUCTS>
__device__ __forceinline__ void pack_eighth(const Resident<PRODUCTS> &z, int b, int row, int col, const float (&x)[8])
{
    uint32_t hi[4], rest[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        hi[k] = narrow2(x[2 * k], x[2 * k + 1], QSR_F16);
        const float2 f = widen2(hi[k], QSR_F16);
        rest[k] = narrow2(x[2 * k] - f.x, x[2 * k + 1] - f.y, QSR_F16);
    }
    uint16_t *block = reinterpret_cast<uint16_t *>(z.x + b * kBlockBytes);
    const int lo = z.x_part() / 2;
    if (WIDE) {
        uint16_t *to = block + place(row, col);
        *reinterpret_cast<uint4 *>(to) = make_uint4(hi[0], hi[1], hi[2], hi[3]);
        if (PRODUCTS == 3) *reinterpret_cast<uint4 *>(to + lo) = make_uint4(rest[0], rest[1], rest[2], rest[3]);
    } else {
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            uint16_t *to = block + place(row + k, col);
            *to = uint16_t(hi[k / 2] >> (k % 2 * 16));
            if (PRODUCTS == 3) to[lo] = uint16_t(rest[k / 2] >> (k % 2 * 16));
        }
    }
}
template <bool WIDE, int PRODUCTS>
__device__ __forceinline__ void small_pack(const MuonParams &p, const MuonMatrix &t, const void *grad, const Resident<PRODUCTS> &z, Scaling by, const Kept &kept)
{
    const int blocks = t.rb * t.cb, rb = t.rb, gt = t.grad_type;
    int row, col;
    eighth_of<WIDE>(t, 0, 0, row, col);
#pragma unroll
    for (int b = 0; b < kKept; ++b) {
        if (b >= blocks) break;
        float x[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) x[k] = kept.u[b][k] == 0.0f ? 0.0f : kept.u[b][k] * by.lift * by.factor;        // padding stays zero, whatever the factor
        pack_eighth<WIDE, PRODUCTS>(z, b, row, col, x);
    }
#pragma unroll 2
    for (int b = kKept; b < blocks; ++b) {
        const Half o = eighth_of<WIDE>(t, b % rb, b / rb, row, col);
        Raw8 g, m;
        take<WIDE>(g, grad, gt, o);
        take<WIDE>(m, t.momentum, QSR_F32, o);
        float gs[8], x[8];
        widen<WIDE>(gs, g, gt);
        widen<WIDE>(x, m, QSR_F32);
#pragma unroll
        for (int k = 0; k < 8; ++k) x[k] = k < o.n ? direction(p, x[k], gs[k] * p.grad_scale) * by.lift * by.factor : 0.0f;
        pack_eighth<WIDE, PRODUCTS>(z, b, row, col, x);
    }
}
template <bool WIDE, int PRODUCTS>
__device__ __forceinline__ void small_apply(const MuonParams &p, const MuonMatrix &t, const Resident<PRODUCTS> &z)
{
    const float decay = p.lr_decay * t.wd_scale, step = p.lr * t.update_scale / t.scale;
    const int blocks = t.rb * t.cb, rb = t.rb, type = t.param_type, copy_type = t.copy_type;
    void *param = t.param, *copy = t.copy;
#pragma unroll 2
    for (int b = 0; b < blocks; ++b) {
        int row, col;
        const Half o = eighth_of<WIDE>(t, b % rb, b / rb, row, col);
        Raw8 old;
        take<WIDE>(old, param, type, o);
        const __half *block = reinterpret_cast<const __half *>(z.x + b * kBlockBytes);
        const int lo = z.x_part() / 2;
        float theta[8];
        widen<WIDE>(theta, old, type);
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const __half *x = block + place(WIDE ? row : row + k, WIDE ? col + k : col);
            const float v = __half2float(x[0]) + (PRODUCTS == 3 ? __half2float(x[lo]) : 0.0f);
            theta[k] -= fmaf(decay, theta[k], step * v);
        }
        give<WIDE>(param, theta, type, o);
        if (copy_type != QSR_NONE) give<WIDE>(copy, theta, copy_type, o);
    }
}

template <int PRODUCTS>
__global__ void __launch_bounds__(kSmallThreads, 1) small_kernel(const __grid_constant__ MuonParams p, const int32_t *which, unsigned columns)
{
    extern __shared__ char raw[];
    __shared__ double sums[kSmallThreads / 32];
    __shared__ Scaling factor;
    __shared__ uint64_t done;
    __shared__ uint32_t tensor_memory;
    __shared__ unsigned stop_flag;
    constexpr int PARTS = Resident<PRODUCTS>::PARTS;
    const int matrix = which[blockIdx.x], warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const MuonMatrix t = p.matrices[matrix];
    const void *grad = p.grads[matrix];
    Resident<PRODUCTS> z;
    z.rb = t.rb; z.cb = t.cb; z.mb = t.mb;
    z.x = raw + (((shared_address(raw) + 1023u) & ~1023u) - shared_address(raw));
    z.a = z.x + PARTS * z.x_part();
    if (threadIdx.x == 0) {
        barrier_init(shared_address(&done), 1);
        stop_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
    if (warp == 0) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(shared_address(&tensor_memory)), "r"(columns) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    const bool wide = wide_rows(t, grad, t.grad_type) && wide_rows(t, t.momentum, QSR_F32);
    Kept kept;
    double s = wide ? small_momentum<true>(p, t, grad, kept) : small_momentum<false>(p, t, grad, kept);
#pragma unroll
    for (int d = 16; d; d >>= 1) s += __shfl_xor_sync(0xffffffffu, s, d);
    if (lane == 0) sums[warp] = s;
    __syncthreads();
    if (threadIdx.x == 0) {
        s = sums[0];
        for (int w = 1; w < kSmallThreads / 32; ++w) s += sums[w];
        factor = scaling_of(t.scale, s, p.eps);
    }
    __syncthreads();
    if (wide) small_pack<true, PRODUCTS>(p, t, grad, z, factor, kept);
    else small_pack<false, PRODUCTS>(p, t, grad, z, factor, kept);

    const uint32_t accumulators = tensor_memory, x_at = shared_address(z.x), a_at = shared_address(z.a);
    const bool tall = t.tall;
    const int group = warp & 3, share = warp >> 2;          // lanes 32 group.., every fourth half of a block's columns
    const float gram_factor = kGramScale / (t.scale * t.scale);
    constexpr float factor_factor = kC * kFactorScale / (kGramScale * kGramScale);
    unsigned phase = 0;
    for (int product = 0; product < 3 * p.iterations; ++product) {
        const int kind = product % 3;
        const int rows = kind == ITERATE ? z.rb : z.mb, cols = kind == ITERATE ? z.cb : z.mb;
        // what has been written to shared memory is read by the tensor cores
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        fence_before();
        __syncthreads();
        if (warp == 0) {                                    // one elected thread issues, the whole warp computes with it
            fence_after();
            const bool one = elected();
            const Operand x{x_at, z.x_part(), z.rb, false}, x_outer{x_at, z.x_part(), z.rb, true}, a{a_at, z.a_part(), z.mb, false};
            if (kind == GRAM) issue_all<PRODUCTS>(one, accumulators, tall ? x_outer : x, tall ? x_outer : x, z.mb, z.mb, tall ? z.rb : z.cb);
            else if (kind == FACTOR) issue_all<PRODUCTS>(one, accumulators, a, a, z.mb, z.mb, z.mb);
            else issue_all<PRODUCTS>(one, accumulators, tall ? x : a, tall ? a : x_outer, z.rb, z.cb, z.mb);
            if (one) asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(shared_address(&done)) : "memory");
            __syncwarp();
        }
        barrier_wait(shared_address(&done), phase, &stop_flag);
        phase ^= 1u;
        fence_after();
        const int row = (group & 1) * 32 + lane;
        int first = 0, h = share;                           // 128 rows from block `first` on, x 32 columns each
        for (int u = share;; u += 4, h += 4) {
            for (; h >= cols * 2; h -= cols * 2) first += 2;
            if (first >= rows) break;
            const int i = first + (group >> 1), j = h >> 1, half = h & 1;
            float v[32];
            load_accumulators(v, accumulators + unsigned(u * 32) + (unsigned(group * 32) << 16));
            if (i >= rows) continue;
            char *block = (kind == ITERATE ? z.x : z.a) + (j * rows + i) * kBlockBytes;
            if (kind == GRAM) {
#pragma unroll
                for (int k = 0; k < 32; ++k) v[k] *= gram_factor;
                keep_half<PRODUCTS>(block, z.a_part(), row, half, v);
            } else if (kind == FACTOR) {
                finish_half<true>(v, factor_factor, (i - j) * 64 + row - half * 32);
                add_kept(v, block, row, half, kMiddle);
                if (PRODUCTS == 3) add_kept(v, block + z.a_part(), row, half, kMiddle);
                keep_half<PRODUCTS>(block, z.a_part(), row, half, v);
            } else {
#pragma unroll
                for (int k = 0; k < 32; ++k) v[k] *= 1.0f / kFactorScale;
                keep_half<PRODUCTS>(block, z.x_part(), row, half, v);
            }
        }
    }
    fence_before();
    __syncthreads();
    if (wide_rows(t, t.param, t.param_type) && (t.copy_type == QSR_NONE || wide_rows(t, t.copy, t.copy_type))) small_apply<true, PRODUCTS>(p, t, z);
    else small_apply<false, PRODUCTS>(p, t, z);
    if (threadIdx.x == 0 && stop_flag) *p.late = 1u;
    if (warp == 0) {
        fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(accumulators), "r"(columns) : "memory");
    }
}

template <int PRODUCTS>
int launch_small(const MuonParams &p, const int32_t *which, int n, int shared_blocks, unsigned columns, cudaStream_t st)
{
    const auto kernel = small_kernel<PRODUCTS>;
    static std::atomic<uint64_t> raised{0};
    // a block more than the matrix has: where an operand has an odd number of them, the products read one behind it (and nobody the result)
    if (int err = allow_shared(reinterpret_cast<const void *>(kernel), (kMuonSmallBlocks + 1) * kBlockBytes + 1024, raised)) return err;
    kernel<<<unsigned(n), kSmallThreads, size_t(shared_blocks + 1) * kBlockBytes + 1024, st>>>(p, which, columns);
    return int(cudaGetLastError());
}

template <typename... A>
int launch_close(void (*kernel)(A...), unsigned blocks, unsigned threads, size_t shared, cudaStream_t st, const A &...args)
{
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(blocks);
    cfg.blockDim = dim3(threads);
    cfg.dynamicSmemBytes = shared;
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return int(cudaLaunchKernelEx(&cfg, kernel, args...));
}

constexpr int kProductShared = kStageBlocks * kBlockBytes + 1024;

template <bool POLYNOMIAL, int PRODUCTS>
int launch_product(const MuonParams &p, const Maps &maps, const MuonTile *tiles, int n, int blocks, cudaStream_t st)
{
    const auto kernel = product_kernel<POLYNOMIAL, PRODUCTS>;
    static std::atomic<uint64_t> raised{0};
    if (int err = allow_shared(reinterpret_cast<const void *>(kernel), kProductShared, raised)) return err;
    return launch_close(kernel, unsigned(blocks), kProductThreads, kProductShared, st, p, maps, tiles, n);
}

}  // namespace

// The driver's function is looked up at run time: the library is not linked against the driver.
int encode_muon_maps(void *tensor_maps, const void *data, int64_t bytes)
{
    void *entry = nullptr;
    cudaDriverEntryPointQueryResult found;
    if (cudaError_t err = cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &entry, 12000, cudaEnableDefault, &found)) return int(err);
    if (found != cudaDriverEntryPointSuccess || !entry) return int(cudaErrorNotSupported);
    const cuuint64_t size[2] = {64, cuuint64_t(bytes / 128)}, pitch[1] = {128};
    const cuuint32_t step[2] = {1, 1};
    Maps &maps = *static_cast<Maps *>(tensor_maps);
    for (cuuint32_t blocks = 1; blocks <= 2; ++blocks) {
        const cuuint32_t box[2] = {64, 64 * blocks};
        const CUresult err = reinterpret_cast<decltype(&cuTensorMapEncodeTiled)>(entry)(
            blocks == 1 ? &maps.single : &maps.pair, CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 2, const_cast<void *>(data), size, pitch, box, step,
            CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_NONE, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
        if (err != CUDA_SUCCESS) return int(cudaErrorInvalidValue);
    }
    return 0;
}

int launch_muon_clear(const MuonParams &p, int64_t chunks, void *stream)
{
    clear_kernel<<<unsigned(chunks), kMomentumThreads, 0, static_cast<cudaStream_t>(stream)>>>(p);
    return int(cudaGetLastError());
}

int launch_muon_momentum(const MuonParams &p, int64_t chunks, void *stream)
{
    momentum_kernel<<<unsigned(chunks), kMomentumThreads, 0, static_cast<cudaStream_t>(stream)>>>(p);
    return int(cudaGetLastError());
}

int launch_muon_pack(const MuonParams &p, int64_t blocks, void *stream)
{
    return launch_close(pack_kernel, unsigned(blocks), 256, 0, static_cast<cudaStream_t>(stream), p);
}

int launch_muon_apply(const MuonParams &p, int64_t blocks, void *stream)
{
    return launch_close(apply_kernel, unsigned(blocks), 256, 0, static_cast<cudaStream_t>(stream), p);
}

int launch_muon_small(const MuonParams &p, const int32_t *which, int n, int shared_blocks, unsigned columns, void *stream)
{
    const cudaStream_t st = static_cast<cudaStream_t>(stream);
    return p.products == 3 ? launch_small<3>(p, which, n, shared_blocks, columns, st) : launch_small<1>(p, which, n, shared_blocks, columns, st);
}

int launch_muon_product(const MuonParams &p, const void *tensor_maps, bool polynomial, const MuonTile *tiles, int64_t n_tiles, int multiprocessors, void *stream)
{
    const Maps &maps = *static_cast<const Maps *>(tensor_maps);
    const cudaStream_t st = static_cast<cudaStream_t>(stream);
    const int n = int(n_tiles), blocks = 2 * (n < multiprocessors / 2 ? n : multiprocessors / 2);
    if (p.products == 3) return polynomial ? launch_product<true, 3>(p, maps, tiles, n, blocks, st) : launch_product<false, 3>(p, maps, tiles, n, blocks, st);
    return polynomial ? launch_product<true, 1>(p, maps, tiles, n, blocks, st) : launch_product<false, 1>(p, maps, tiles, n, blocks, st);
}

}  // namespace qsr
