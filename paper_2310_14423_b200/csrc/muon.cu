// Orthogonalised momentum: the kernels.  See include/qsr.h for the formulas and muon_api.cu for the launches.
//
// The iterate X (m x n, m <= n: the transpose of a tall matrix) and the symmetric m x m matrices A = X X^T and C = a I + b A + c A^2
// are held as fp16 blocks of 64 x 64 (8 KB), each exactly as a tensor-core operand wants it in shared memory (rows of 128 bytes,
// 16-byte pieces exchanged by the row number's low three bits).  A block is one untiled bulk copy, needs no tensor map, and serves as an
// operand with either side along the products' sum: rows along it if read as it is, columns along it if the instruction is told so
// ("major" bit).  So X X^T and C X read the same blocks of X, and of A and C only the tiles on and above the diagonal are
// computed; what lies below is read from its mirror image.  Blocks are padded with zeros, hence any m and n.
//
// With three products per multiplication, X, A and C are sums of two fp16 numbers and hi hi + hi lo + lo hi are accumulated.
#include <cuda_runtime.h>

#include "wide.cuh"

namespace qsr {

namespace {

constexpr float kA = 3.4445f, kB = -4.7750f, kC = 2.0315f;
// Powers of two that A and C are held at, for fp16's range: singular values of X stay below 1.2025 (the polynomial's
// maximum on [0, 1.2025]), so entries of A stay below 1.45 and those of C, whose eigenvalues lie in [0.63, 3.45], below 3.45.
constexpr float kGramScale = 16384.0f, kFactorScale = 16384.0f;

// ---- momentum and norms ----------------------------------------------------------------------------------

__device__ __forceinline__ bool address_aligned(const void *p, unsigned bytes) { return (reinterpret_cast<uintptr_t>(p) & (bytes - 1)) == 0; }

constexpr int kMomentumThreads = 256;

__device__ __forceinline__ float updated(const MuonParams &p, float m, float g) { return fmaf(p.one_minus_beta, g - m, m); }
// What is orthogonalised, from the new momentum.
__device__ __forceinline__ float direction(const MuonParams &p, float m, float g) { return p.nesterov ? fmaf(p.beta, m - g, g) : m; }

// m <- m + (1 - beta)(g - m) and the sum of squares of u, chunk by chunk; the matrix's last chunk adds them in their order.
// Squares and sums in binary64: the norm neither overflows nor loses small elements.
__global__ void __launch_bounds__(kMomentumThreads) momentum_kernel(const __grid_constant__ MuonParams p)
{
    __shared__ double scratch[kMomentumThreads / 32];
    __shared__ bool last;
    const MuonChunk c = p.chunks[blockIdx.x];
    const MuonMatrix &t = p.matrices[c.matrix];
    const void *grad = p.grads[c.matrix];
    const int gt = t.grad_type;
    const bool vec = address_aligned(grad, gt == QSR_F32 ? 32 : 16) && address_aligned(t.momentum, 32);
    double s = 0.0;
    if (vec) {
#pragma unroll 2
        for (int i = int(threadIdx.x) * 8; i + 8 <= c.n; i += kMomentumThreads * 8) {
            Raw8 rg, rm;
            load8(rg, grad, c.offset + i, gt);
            load32(rm, t.momentum + c.offset + i);
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
            store8(t.momentum, c.offset + i, m, QSR_F32);
        }
    }
    for (int i = (vec ? c.n & ~7 : 0) + int(threadIdx.x); i < c.n; i += kMomentumThreads) {
        const float gs = widen1(load1(grad, c.offset + i, gt), gt) * p.grad_scale, m = updated(p, t.momentum[c.offset + i], gs);
        const double u = double(direction(p, m, gs));
        s = fma(u, u, s);
        t.momentum[c.offset + i] = m;
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
        const double length = sqrt(s) + double(p.eps);            // 0: nothing to scale
        p.factor[c.matrix] = length == 0.0 ? 0.0f : float(isnan(length) ? length : fmin(double(t.scale) / length, 3.0e38));
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

// Two fp16 numbers whose sum is x to 22 bits (hi alone: 11).
__device__ __forceinline__ void split(float x, __half &hi, __half &lo)
{
    hi = __float2half_rn(x);
    lo = __float2half_rn(x - __half2float(hi));
}

// One block of the first iterate: u from the new momentum, times scale / (norm + eps).
__global__ void __launch_bounds__(256) pack_kernel(const __grid_constant__ MuonParams p)
{
    __shared__ __align__(16) __half hi[kBlockElements], lo[kBlockElements];
    const MuonBlock b = p.blocks[blockIdx.x];
    const MuonMatrix &t = p.matrices[b.matrix];
    const void *grad = p.grads[b.matrix];
    const float factor = p.factor[b.matrix];
    const int gt = t.grad_type;
    // the matrix's rows r0.. and columns c0.. in its own orientation
    const int64_t r0 = int64_t(t.tall ? b.q : b.p) * 64, c0 = int64_t(t.tall ? b.p : b.q) * 64;
    const bool vec = t.cols % 8 == 0 && address_aligned(grad, gt == QSR_F32 ? 32 : 16) && address_aligned(t.momentum, 32);
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const int r = h * 32 + int(threadIdx.x) / 8, c = (int(threadIdx.x) & 7) * 8;
        const int64_t at = (r0 + r) * t.cols + c0 + c;
        float g[8], m[8];
        if (vec && r0 + r < t.rows && c0 + c < t.cols) {
            Raw8 rg, rm;
            load8(rg, grad, at, gt);
            load32(rm, t.momentum + at);
            widen8(g, rg, gt);
            widen8(m, rm, QSR_F32);
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const bool in = r0 + r < t.rows && c0 + c + j < t.cols;
                g[j] = in ? widen1(load1(grad, at + j, gt), gt) : 0.0f;
                m[j] = in ? t.momentum[at + j] : 0.0f;
            }
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int row = t.tall ? c + j : r, col = t.tall ? r : c + j;      // in the block
            const bool in = r0 + r < t.rows && c0 + c + j < t.cols;            // padding stays zero, whatever the factor
            const int to = row * 64 + ((col / 8) ^ (row & 7)) * 8 + (col & 7);
            split(in ? direction(p, m[j], g[j] * p.grad_scale) * factor : 0.0f, hi[to], lo[to]);
        }
    }
    __syncthreads();
    uint4 *out = reinterpret_cast<uint4 *>(t.x[0] + (int64_t(b.q) * t.mb + b.p) * kBlockElements);
    uint4 *out_lo = out + int64_t(t.mb) * t.nb * (kBlockElements / 8);
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const int i = h * 256 + int(threadIdx.x);
        out[i] = reinterpret_cast<const uint4 *>(hi)[i];
        if (p.products == 3) out_lo[i] = reinterpret_cast<const uint4 *>(lo)[i];
    }
}

// ---- products --------------------------------------------------------------------------------------------

enum { GRAM = 0, FACTOR = 1, ITERATE = 2, UPDATE = 3 };

constexpr int kProductThreads = 384;         // warps: 0 copies, 1 products, 2 accumulators' allocation, 4 to 11 results
constexpr int kBlockBytes = kBlockElements * 2;
constexpr int kOperandBlocks = 4;            // of a stage in each block of a pair: two of its 128 rows, two of its 128 columns
constexpr int kStageBlocks = 24;             // shared memory for operands: 6 stages of one product, 3 of three
constexpr int kTurn = 1;                     // blocks along the sum that tensor memory adds up, with three products
constexpr unsigned kAccumulators = 512;      // columns of tensor memory: two tiles of 256
constexpr long long kPatience = 6000000000;  // clocks that a wait may take, some seconds

__device__ __forceinline__ uint32_t shared_address(const void *p) { return uint32_t(__cvta_generic_to_shared(p)); }

__device__ __forceinline__ void barrier_init(uint32_t bar, unsigned count)
{
    asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count) : "memory");
}
__device__ __forceinline__ void barrier_arrive(uint32_t bar) { asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory"); }
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
__device__ __forceinline__ void copy_block(uint32_t to, const void *from, uint32_t bar)
{
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(to), "l"(from), "r"(kBlockBytes), "r"(bar)
                 : "memory");
}

// Operand descriptor: rows of 128 bytes with 128-byte swizzle, groups of eight rows 1024 bytes apart; with the sum along the
// columns of blocks ("outer"), the next 64 rows or columns of the operand are a block further.
__device__ __forceinline__ uint64_t operand(uint32_t address)
{
    return uint64_t((address >> 4) & 0x3fff) | uint64_t(kBlockBytes >> 4) << 16 | uint64_t(1024 >> 4) << 32 | uint64_t(1) << 46 | uint64_t(2) << 61;
}
// Instruction descriptor: fp16 operands, fp32 accumulators, 256 x n over the pair; outer_a / outer_b: the operand's rows in memory run along the sum.
__device__ __forceinline__ uint32_t instruction(int n, bool outer_a, bool outer_b)
{
    return 1u << 4 | uint32_t(outer_a) << 15 | uint32_t(outer_b) << 16 | uint32_t(n >> 3) << 17 | uint32_t(256 >> 4) << 24;
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

// Whether the blocks in row tile P, column tile T (256 elements each) of a symmetric matrix are held; otherwise their mirror images are.
__device__ __forceinline__ bool held(int P, int T) { return P <= T; }

// Half a row of a block, 32 elements: where 16-byte pair `pair` (0 or 1) of it lies, in elements.
__device__ __forceinline__ int pair_at(int row, int half, int pair) { return row * 64 + ((half * 2 + pair) ^ ((row & 7) >> 1)) * 16; }

__device__ __forceinline__ void store_half(uint16_t *block, uint16_t *block_lo, int row, int half, const float (&v)[32], bool both)
{
#pragma unroll
    for (int pair = 0; pair < 2; ++pair) {
        Raw8 hi, lo;
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const float a = v[pair * 16 + 2 * k], b = v[pair * 16 + 2 * k + 1];
            const __half2 h = __floats2half2_rn(a, b);
            const float2 f = __half22float2(h);
            hi.w[k] = *reinterpret_cast<const uint32_t *>(&h);
            if (both) lo.w[k] = narrow2(a - f.x, b - f.y, QSR_F16);
        }
        if (row & 1) {                       // odd rows: the two pieces of a pair change places
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                uint32_t x = hi.w[k]; hi.w[k] = hi.w[k + 4]; hi.w[k + 4] = x;
                if (both) { x = lo.w[k]; lo.w[k] = lo.w[k + 4]; lo.w[k + 4] = x; }
            }
        }
        store32(block + pair_at(row, half, pair), hi);
        if (both) store32(block_lo + pair_at(row, half, pair), lo);
    }
}

__device__ __forceinline__ void add_half(float (&v)[32], const uint16_t *block, int row, int half, float factor)
{
#pragma unroll
    for (int pair = 0; pair < 2; ++pair) {
        Raw8 r;
        load32(r, block + pair_at(row, half, pair));
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const float2 f = widen2((row & 1) ? r.w[k ^ 4] : r.w[k], QSR_F16);
            v[pair * 16 + 2 * k] = fmaf(factor, f.x, v[pair * 16 + 2 * k]);
            v[pair * 16 + 2 * k + 1] = fmaf(factor, f.y, v[pair * 16 + 2 * k + 1]);
        }
    }
}

// Eight elements of the parameter that belong to columns col.. of a row of the iterate, as they lie in memory: adjacent (`vec`), or
// one to a word.
__device__ __forceinline__ void fetch_theta(Raw8 &r, const MuonMatrix &t, int row, int col, bool vec)
{
    const int type = t.param_type;
    if (row >= t.m || col >= t.n) return;
    if (vec) {
        load8(r, t.param, int64_t(row) * t.cols + col, type);
        return;
    }
    const int64_t step = t.tall ? t.cols : 1, at = t.tall ? col * t.cols + row : row * t.cols + col;
#pragma unroll
    for (int j = 0; j < 8; ++j) r.w[j] = col + j < t.n ? load1(t.param, at + j * step, type) : 0u;
}
// 32 rows (row: this lane's) and 128 columns of the iterate: the parameter's elements into the second-level cache.
__device__ __forceinline__ void prefetch_theta(const MuonMatrix &t, int row, int col)
{
    const int bytes = t.param_type == QSR_F32 ? 4 : 2, lane = threadIdx.x & 31;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        const int m = t.tall ? row - lane : row, n = col + q * 32 + (t.tall ? lane : 0);
        if (m >= t.m || n >= t.n) continue;
        const char *at = static_cast<const char *>(t.param) + (t.tall ? int64_t(n) * t.cols + m : int64_t(m) * t.cols + n) * bytes;
        asm volatile("prefetch.global.L2 [%0];" ::"l"(at));
    }
}
// theta <- theta - (decay theta + step X) for the eight elements.
__device__ __forceinline__ void update_theta(const Raw8 &r, const MuonMatrix &t, int row, int col, bool vec, float decay, float step, const float *x)
{
    const int type = t.param_type, copy = t.copy_type;
    if (row >= t.m || col >= t.n) return;
    float theta[8];
    if (vec) widen8(theta, r, type);
    else {
#pragma unroll
        for (int j = 0; j < 8; ++j) theta[j] = widen1(r.w[j], type);
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) theta[j] -= fmaf(decay, theta[j], step * x[j]);
    if (vec) {
        const int64_t at = int64_t(row) * t.cols + col;
        store8(t.param, at, theta, type);
        if (copy != QSR_NONE) store8(t.copy, at, theta, copy);
        return;
    }
    const int64_t pitch = t.tall ? t.cols : 1, at = t.tall ? col * t.cols + row : row * t.cols + col;
#pragma unroll
    for (int j = 0; j < 8; ++j)
        if (col + j < t.n) {
            store1(t.param, at + j * pitch, theta[j], type);
            if (copy != QSR_NONE) store1(t.copy, at + j * pitch, theta[j], copy);
        }
}

// What becomes of 32 sums of a tile: row `row` of block (bp, bq), its first or second half.
template <int KIND, int PRODUCTS>
__device__ __forceinline__ void result(const MuonParams &p, const MuonMatrix &t, int bp, int bq, int row, int half, int from, float (&v)[32])
{
    const int mb = t.mb;
    if (bp >= mb || bq >= (KIND >= ITERATE ? t.nb : mb)) return;
    const int64_t block = int64_t(bq) * mb + bp;
    if (KIND == GRAM) {
        const float f = kGramScale / (t.scale * t.scale);
#pragma unroll
        for (int k = 0; k < 32; ++k) v[k] *= f;
        store_half(t.gram + block * kBlockElements, t.gram + (int64_t(mb) * mb + block) * kBlockElements, row, half, v, PRODUCTS == 3);
    } else if (KIND == FACTOR) {
        const uint16_t *gram = t.gram + block * kBlockElements;
        constexpr float f = kC * kFactorScale / (kGramScale * kGramScale), g = kB * kFactorScale / kGramScale;
        const int diagonal = (bp - bq) * 64 + row - half * 32;      // which of them is on the diagonal
#pragma unroll
        for (int k = 0; k < 32; ++k) v[k] = v[k] * f + (k == diagonal ? kA * kFactorScale : 0.0f);
        add_half(v, gram, row, half, g);
        if (PRODUCTS == 3) add_half(v, gram + int64_t(mb) * mb * kBlockElements, row, half, g);
        store_half(t.factor + block * kBlockElements, t.factor + (int64_t(mb) * mb + block) * kBlockElements, row, half, v, PRODUCTS == 3);
    } else {
#pragma unroll
        for (int k = 0; k < 32; ++k) v[k] *= 1.0f / kFactorScale;
        store_half(t.x[from ^ 1] + block * kBlockElements, t.x[from ^ 1] + (int64_t(mb) * t.nb + block) * kBlockElements, row, half, v, PRODUCTS == 3);
    }
}

struct Shared {
    uint64_t full[6], other[6], empty[6], ready[2], drained[2];
    uint32_t tensor_memory;
    unsigned stop;
};

// A pair of blocks (one per multiprocessor) takes tiles of 256 x 256 elements, pair, + pairs, ...; each has 128 of the tile's rows and
// 128 of its columns in its shared memory, a stage at a time of 64 along the sum, and 128 x 256 sums in its tensor memory.  One warp of
// each block copies; one thread of the first block issues the products of both (in the second block that thread tells the first
// when a stage has arrived); eight warps take the tile before out of the other half of tensor memory.  Compared with 128 x 256 tiles of
// single blocks, each multiprocessor copies and reads two thirds of the bytes for a product.
template <int KIND, int PRODUCTS>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kProductThreads, 1)
product_kernel(const __grid_constant__ MuonParams p, const MuonTile *tiles, int n_tiles, int from)
{
    extern __shared__ char raw[];
    __shared__ Shared sh;
    constexpr int PARTS = PRODUCTS == 3 ? 2 : 1, STAGES = kStageBlocks / (kOperandBlocks * PARTS);
    constexpr int TURN = PRODUCTS == 3 ? kTurn : 1 << 30;
    const uint32_t stage0 = (shared_address(raw) + 1023u) & ~1023u;
    constexpr uint32_t kStage = kOperandBlocks * PARTS * kBlockBytes;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int rank = int(blockIdx.x & 1), pair = int(blockIdx.x >> 1), pairs = int(gridDim.x >> 1);
    volatile unsigned *stop = &sh.stop;
    if (threadIdx.x == 0) {
        for (int i = 0; i < STAGES; ++i) {
            barrier_init(shared_address(&sh.full[i]), 1);
            barrier_init(shared_address(&sh.other[i]), 1);
            barrier_init(shared_address(&sh.empty[i]), 1);
        }
        for (int i = 0; i < 2; ++i) {
            barrier_init(shared_address(&sh.ready[i]), 1);
            barrier_init(shared_address(&sh.drained[i]), 16);
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

    if (warp == 0) {
        int stage = 0, issued = 0;
        unsigned phase = 0;
        bool going = true;
        for (int tile = pair; tile < n_tiles && going; tile += pairs) {
            const MuonTile w = tiles[tile];
            const MuonMatrix &t = p.matrices[w.matrix];
            const int mb = t.mb, nb = t.nb, sums = KIND == GRAM ? nb : mb;
            const int columns = KIND >= ITERATE ? nb : mb, wide = columns - w.j * 4 > 2;
            const int p0 = w.i * 4 + rank * 2, q0 = w.j * 4 + (wide ? rank * 2 : rank);
            const int rows = max(0, min(2, mb - p0)), cols = max(0, min(wide ? 2 : 1, columns - q0));
            const uint16_t *left = KIND == GRAM ? t.x[from] : KIND == FACTOR ? t.gram : t.factor;
            const uint16_t *right = KIND == FACTOR ? t.gram : t.x[from];
            const int64_t left_lo = int64_t(mb) * (KIND == GRAM ? nb : mb), right_lo = int64_t(mb) * (KIND == FACTOR ? mb : nb);
            // this lane's block of each stage: part, then rows of the left or columns of the right operand
            const int part = lane / kOperandBlocks, slot = lane % kOperandBlocks;
            const bool is_left = slot < 2;
            const bool mine = part < PARTS && (is_left ? slot < rows : slot - 2 < cols);
            const int at = is_left ? p0 + slot : q0 + slot - 2;
            const uint16_t *base = is_left ? left + part * left_lo * kBlockElements : right + part * right_lo * kBlockElements;
            for (int k = 0; k < sums; ++k) {
                if (!barrier_wait(shared_address(&sh.empty[stage]), phase ^ 1u, stop)) { going = false; break; }
                const uint32_t bar = shared_address(&sh.full[stage]);
                if (lane == 0) barrier_expect(bar, unsigned((rows + cols) * PARTS * kBlockBytes));
                __syncwarp();
                if (mine) {
                    bool direct;               // block (at, k), or its mirror image (k, at)
                    if (is_left) direct = KIND == GRAM || held(w.i, k >> 2);
                    else direct = KIND == GRAM || (KIND == FACTOR && held(w.j, k >> 2));
                    const int64_t index = direct ? int64_t(k) * mb + at : int64_t(at) * mb + k;
                    copy_block(stage0 + stage * kStage + (part * kOperandBlocks + slot) * kBlockBytes, base + index * kBlockElements, bar);
                }
                issued++;
                if (++stage == STAGES) { stage = 0; phase ^= 1u; }
            }
        }
        // when the block ends nothing may be copying into its shared memory, or reading it: wait for the last stages
        for (int s = 0; s < STAGES && s < issued; ++s) {
            const int last = issued - 1 - s;
            const unsigned parity = unsigned(last / STAGES) & 1u;
            barrier_wait(shared_address(&sh.empty[last % STAGES]), parity, stop);
            barrier_wait(shared_address(&sh.full[last % STAGES]), parity, stop, false);
        }
    } else if (warp == 1) {
        // the whole warp runs through the loop, so that descriptors are computed once for it, and one elected thread issues
        int stage = 0, buffer = 0;
        unsigned phase = 0, buffer_phase = 0;
        const bool one = elected();
        bool going = true;
        for (int tile = pair; tile < n_tiles && going; tile += pairs) {
            const MuonTile w = tiles[tile];
            const MuonMatrix &t = p.matrices[w.matrix];
            const int sums = KIND == GRAM ? t.nb : t.mb, wide = (KIND >= ITERATE ? t.nb : t.mb) - w.j * 4 > 2;
            for (int k = 0; k < sums; ++k) {
                const uint32_t full = shared_address(&sh.full[stage]), other = shared_address(&sh.other[stage]);
                if (rank == 1) {
                    if (!barrier_wait(full, phase, stop)) { going = false; break; }
                    if (one) barrier_arrive_first(other);
                    if (++stage == STAGES) { stage = 0; phase ^= 1u; }
                    continue;
                }
                const int part = k % TURN;                     // of what is added up in tensor memory
                const uint32_t d = accumulators + unsigned(buffer) * 256u;
                if (part == 0 && !barrier_wait(shared_address(&sh.drained[buffer]), buffer_phase ^ 1u, stop)) { going = false; break; }
                if (!barrier_wait(full, phase, stop) || !barrier_wait(other, phase, stop)) { going = false; break; }
                fence_after();
                const bool outer_a = KIND != GRAM && !held(w.i, k >> 2);
                const bool outer_b = KIND >= ITERATE || (KIND == FACTOR && !held(w.j, k >> 2));
                const uint32_t idesc = instruction(wide ? 256 : 128, outer_a, outer_b);
                const uint32_t a0 = stage0 + stage * kStage, b0 = a0 + 2 * kBlockBytes;
                const uint64_t a = operand(a0), b = operand(b0);
                const uint64_t a_step = outer_a ? 2048 >> 4 : 32 >> 4, b_step = outer_b ? 2048 >> 4 : 32 >> 4;
                constexpr uint64_t lo = (kOperandBlocks * kBlockBytes) >> 4;
                if (one) {
#pragma unroll
                    for (int q = PRODUCTS - 1; q >= 0; --q)        // hi lo, lo hi, hi hi
#pragma unroll
                        for (int s = 0; s < 4; ++s)
                            multiply(d, a + (q == 1 ? lo : 0) + s * a_step, b + (q == 2 ? lo : 0) + s * b_step, idesc, part > 0 || q < PRODUCTS - 1 || s > 0);
                    commit(shared_address(&sh.empty[stage]));
                    if (part == TURN - 1 || k == sums - 1) commit(shared_address(&sh.ready[buffer]));
                }
                __syncwarp();
                if (++stage == STAGES) { stage = 0; phase ^= 1u; }
                if (part == TURN - 1 || k == sums - 1) {
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
        bool going = true;
        for (int tile = pair; tile < n_tiles && going; tile += pairs) {
            const MuonTile w = tiles[tile];
            const MuonMatrix &t = p.matrices[w.matrix];
            const int row = (group & 1) * 32 + lane, bp = w.i * 4 + rank * 2 + (group >> 1);      // in block row bp
            const int bq = w.j * 4 + part * 2;
            const uint32_t from_lane = accumulators + unsigned(part * 128) + (unsigned(group * 32) << 16);
            // the last product of a step: a pipeline over eight columns of the parameter at a time
            constexpr int DEPTH = PRODUCTS == 3 ? 2 : 4;
            Raw8 theta[KIND == UPDATE ? DEPTH : 1];
            const int r = bp * 64 + row, c = bq * 64;
            bool vec = false;
            float decay = 0.0f, step = 0.0f;
            if (KIND == UPDATE) {
                if (tile + pairs < n_tiles) {
                    const MuonTile ahead = tiles[tile + pairs];
                    prefetch_theta(p.matrices[ahead.matrix], (ahead.i * 4 + rank * 2 + (group >> 1)) * 64 + row, (ahead.j * 4 + part * 2) * 64);
                }
                const int type = t.param_type, copy = t.copy_type;
                vec = !t.tall && t.cols % 8 == 0 && address_aligned(t.param, type == QSR_F32 ? 32 : 16) &&
                      (copy == QSR_NONE || address_aligned(t.copy, copy == QSR_F32 ? 32 : 16));
                decay = p.lr_decay * t.wd_scale;
                step = p.lr * t.update_scale / (t.scale * kFactorScale);
                if (PRODUCTS == 1)
#pragma unroll
                    for (int g = 0; g < DEPTH; ++g) fetch_theta(theta[g], t, r, c + g * 8, vec);
            }
            if (PRODUCTS == 1) {
                if (!barrier_wait(shared_address(&sh.ready[buffer]), buffer_phase, stop)) break;
                fence_after();
#pragma unroll 1
                for (int h = 0; h < 4; ++h) {                    // 32 columns each
                    float v[32];
                    load_accumulators(v, from_lane + unsigned(buffer * 256 + h * 32));
                    if (KIND != UPDATE) result<KIND, PRODUCTS>(p, t, bp, bq + (h >> 1), row, h & 1, from, v);
                    else
#pragma unroll
                        for (int g = 0; g < 4; ++g) {
                            update_theta(theta[g % DEPTH], t, r, c + h * 32 + g * 8, vec, decay, step, v + g * 8);
                            if (h < 3) fetch_theta(theta[g % DEPTH], t, r, c + h * 32 + 32 + g * 8, vec);
                        }
                }
                next();
            } else {
                float v[4][32];
#pragma unroll
                for (int h = 0; h < 4; ++h)
#pragma unroll
                    for (int k = 0; k < 32; ++k) v[h][k] = 0.0f;
                const int turns = ((KIND == GRAM ? t.nb : t.mb) + TURN - 1) / TURN;
#pragma unroll 1
                for (int turn = 0; turn < turns; ++turn) {
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
                if (KIND != UPDATE) {
#pragma unroll
                    for (int h = 0; h < 4; ++h) result<KIND, PRODUCTS>(p, t, bp, bq + (h >> 1), row, h & 1, from, v[h]);
                } else {
#pragma unroll
                    for (int g = 0; g < DEPTH; ++g) fetch_theta(theta[g % DEPTH], t, r, c + g * 8, vec);
#pragma unroll
                    for (int g = 0; g < 16; ++g) {
                        update_theta(theta[g % DEPTH], t, r, c + g * 8, vec, decay, step, v[g / 4] + g % 4 * 8);
                        if (g + DEPTH < 16) fetch_theta(theta[g % DEPTH], t, r, c + (g + DEPTH) * 8, vec);
                    }
                }
            }
        }
    }
    __syncwarp();
    fence_before();
    if (threadIdx.x == 0 && sh.stop) *p.late = 1u;
    pair_sync();                         // the other block's products read this one's shared memory and write its tensor memory
    if (warp == 2) {
        fence_after();
        asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(accumulators), "r"(kAccumulators) : "memory");
    }
}

constexpr int kProductShared = kStageBlocks * kBlockBytes + 1024;

template <int KIND, int PRODUCTS>
int launch_product(const MuonParams &p, int from, const MuonTile *tiles, int n, int blocks, cudaStream_t st)
{
    const auto kernel = product_kernel<KIND, PRODUCTS>;
    static std::atomic<uint64_t> raised{0};
    if (int err = allow_shared(reinterpret_cast<const void *>(kernel), kProductShared, raised)) return err;
    kernel<<<unsigned(blocks), kProductThreads, kProductShared, st>>>(p, tiles, n, from);
    return int(cudaGetLastError());
}

}  // namespace

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
    pack_kernel<<<unsigned(blocks), 256, 0, static_cast<cudaStream_t>(stream)>>>(p);
    return int(cudaGetLastError());
}

int launch_muon_product(const MuonParams &p, int kind, int from, const MuonTile *tiles, int64_t n_tiles, int multiprocessors, void *stream)
{
    const cudaStream_t st = static_cast<cudaStream_t>(stream);
    const int n = int(n_tiles), blocks = 2 * (n < multiprocessors / 2 ? n : multiprocessors / 2);
    if (p.products == 3) {
        if (kind == GRAM) return launch_product<GRAM, 3>(p, from, tiles, n, blocks, st);
        if (kind == FACTOR) return launch_product<FACTOR, 3>(p, from, tiles, n, blocks, st);
        if (kind == ITERATE) return launch_product<ITERATE, 3>(p, from, tiles, n, blocks, st);
        return launch_product<UPDATE, 3>(p, from, tiles, n, blocks, st);
    }
    if (kind == GRAM) return launch_product<GRAM, 1>(p, from, tiles, n, blocks, st);
    if (kind == FACTOR) return launch_product<FACTOR, 1>(p, from, tiles, n, blocks, st);
    if (kind == ITERATE) return launch_product<ITERATE, 1>(p, from, tiles, n, blocks, st);
    return launch_product<UPDATE, 1>(p, from, tiles, n, blocks, st);
}

}  // namespace qsr
