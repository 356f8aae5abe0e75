// Log probabilities of given tokens with entropy, top alternatives and gradient (formulas in the public header).
//
// A row of logits is read once from global memory: a block (or, for long rows and few of them, a cluster of up to eight
// blocks that exchange their partial results through distributed shared memory) keeps its slice of the row in shared
// memory, so the maximum, the sums, the search for the alternatives and the gradient all work from there.  A slice is
// split into 16-byte granules; a thread loads, reduces and writes only its own granules, so nothing but the reductions
// needs a barrier.  Granules at a row's ends may be partial (rows of odd length start anywhere): those are loaded and
// written element by element.
//
// What bounds it.  A 16-bit logit costs two bytes forward and four with the gradient, against one and two exponentials and about
// 9 and 14 instructions: close to what a multiprocessor issues at memory speed, so the loops are kept lean (32-bit granule
// numbers, row ends outside the loops, one fused operation per exponent, two elements per arithmetic instruction) and several
// blocks share a multiprocessor, so that loads, sums and gradients of different rows overlap.  8192 x 32768 bf16 with gradient:
// 208 to 218 us for 1.07 GB (4.9 to 5.2 TB/s).  Without exponentials it took 191 us, with all traffic in L2 181: the rest
// is the chain of waits inside a block.  Measured and not kept: exponentials by polynomial for a quarter to a half of the
// elements (+0.5 to +8 %), blocks that stay and refill the stash during the gradient (+7 %), 512 threads for rows of 64 KB (+3
// to +13 %).  2048 x 50001 bf16, five alternatives, then the gradient call: 66 and 77 us.
#include <cooperative_groups.h>
#include <cuda_runtime.h>

#include <atomic>
#include <cmath>
#include <cstdint>

#include "internal.h"
#include "wide.cuh"

namespace qsr {
namespace {

namespace cg = cooperative_groups;

constexpr int kMaxWarps = 16;
constexpr int kMaxCluster = 8;
constexpr int kGroup = 4;                    // granules a thread loads and sums up at a time
constexpr int kGroups = 64;                  // groups of threads whose maxima bound the n-th largest logit from below
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
// The fast exponents c x - K take a rounded K = c m, so the largest term's own is up to ulp(K) / 2 instead of 0.
constexpr float kBaseMax = 0x1p31f;          // sums: at most 64, so terms stay within 2^64 of what they are relative to m
constexpr float kGradMax = 0x1p24f;          // gradient, whose constant holds log2 S too: at most 2, so nothing cancels in A and B
constexpr float kLowest2 = -200.0f;          // 2^-200 = 0 in fp32: log2-probabilities below are raised to it, so that 0 * (-inf) never forms

template <typename T> struct Num;            // how sixteen bytes of a type are taken apart
template <> struct Num<float> {
    static constexpr int kPer = 4;
    typedef float Max;                       // running maximum, NaN if a NaN was seen
    static __device__ __forceinline__ void widen(float (&x)[4], uint4 w)
    {
        x[0] = __uint_as_float(w.x); x[1] = __uint_as_float(w.y); x[2] = __uint_as_float(w.z); x[3] = __uint_as_float(w.w);
    }
    static __device__ __forceinline__ uint4 narrow(const float (&x)[4])
    {
        return make_uint4(__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3]));
    }
    static __device__ __forceinline__ float lowest() { return -infinity(); }
    static __device__ __forceinline__ float to_float(float x) { return x; }
    static __device__ __forceinline__ Max nothing() { return -infinity(); }
    static __device__ __forceinline__ Max max_of(Max m, uint4 w)
    {
        float x[4];
        widen(x, w);
        return max_nan(m, max_nan(max_nan(x[0], x[1]), max_nan(x[2], x[3])));
    }
    static __device__ __forceinline__ float value(Max m) { return m; }
};
// The two 16-bit types: elements two to a register, extrema of both at once.
template <typename T, typename T2, int TYPE> struct Num16 {
    static constexpr int kPer = 8;
    typedef T2 Max;
    static __device__ __forceinline__ T2 pair(uint32_t w) { return *reinterpret_cast<const T2 *>(&w); }
    static __device__ __forceinline__ void widen(float (&x)[8], uint4 w)
    {
        const uint32_t v[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) { const float2 f = widen2(v[i], TYPE); x[2 * i] = f.x; x[2 * i + 1] = f.y; }
    }
    static __device__ __forceinline__ uint4 narrow(const float (&x)[8])
    {
        return make_uint4(narrow2(x[0], x[1], TYPE), narrow2(x[2], x[3], TYPE), narrow2(x[4], x[5], TYPE), narrow2(x[6], x[7], TYPE));
    }
    static __device__ __forceinline__ Max nothing() { return pair(TYPE == QSR_BF16 ? 0xff80ff80u : 0xfc00fc00u); }
    static __device__ __forceinline__ Max max_of(Max m, uint4 w)
    {
        return __hmax2_nan(__hmax2_nan(__hmax2_nan(m, pair(w.x)), pair(w.y)), __hmax2_nan(pair(w.z), pair(w.w)));
    }
    static __device__ __forceinline__ float value(Max m) { return max_nan(__low2float(m), __high2float(m)); }
};
template <> struct Num<__nv_bfloat16> : Num16<__nv_bfloat16, __nv_bfloat162, QSR_BF16> {
    static __device__ __forceinline__ __nv_bfloat16 lowest() { return __ushort_as_bfloat16(0xff80); }
    static __device__ __forceinline__ float to_float(__nv_bfloat16 x) { return __bfloat162float(x); }
};
template <> struct Num<__half> : Num16<__half, __half2, QSR_F16> {
    static __device__ __forceinline__ __half lowest() { return __ushort_as_half(0xfc00); }
    static __device__ __forceinline__ float to_float(__half x) { return __half2float(x); }
};

// Orders floats as unsigned integers: -inf lowest, -0 = +0, NaN above everything.
__device__ __forceinline__ uint32_t sort_bits(float x)
{
    const uint32_t b = __float_as_uint(x + 0.0f);
    if ((b & 0x7fffffffu) > 0x7f800000u) return 0xffc00000u;
    return b ^ (b & 0x80000000u ? 0xffffffffu : 0x80000000u);
}
__device__ __forceinline__ float unsort_bits(uint32_t s)
{
    return __uint_as_float(s ^ (s & 0x80000000u ? 0x80000000u : 0xffffffffu));
}
// Value descending, then index ascending; 0 stands for "none" (no element maps to it: the lowest value's bits are not 0).
__device__ __forceinline__ unsigned long long key_of(float x, uint32_t index)
{
    return (static_cast<unsigned long long>(sort_bits(x)) << 32) | (0xffffffffu - index);
}

__device__ __forceinline__ void cp_async16(void *smem_dst, const void *gmem_src)
{
    const unsigned dst = static_cast<unsigned>(__cvta_generic_to_shared(smem_dst));
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(gmem_src) : "memory");
}

__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) { return __ffma2_rn(a, b, c); }
__device__ __forceinline__ float2 mul2(float2 a, float2 b) { return __fmul2_rn(a, b); }
__device__ __forceinline__ float2 add2(float2 a, float2 b) { return __fadd2_rn(a, b); }
__device__ __forceinline__ float2 both(float x) { return make_float2(x, x); }

// What a slice, and in the end the row, is reduced to: the largest logit, sum of e = 2^z and of e z with z = tau log2(e) (x - m).
struct Sums { float m, s, t; };

__device__ __forceinline__ Sums join(Sums a, Sums b, float c)
{
    if (a.s == 0.0f) return b;
    if (b.s == 0.0f) return a;
    Sums r;
    r.m = max_nan(a.m, b.m);
    const float da = (a.m - r.m) * c, db = (b.m - r.m) * c, fa = exp2_1(da), fb = exp2_1(db);
    r.s = fa * a.s + fb * b.s;
    // a slice that lies 2^200 below the other adds nothing: its factor is 0, and its offset must not meet that as -inf
    r.t = fa * fmaf(a.s, fmaxf(da, kLowest2), a.t) + fb * fmaf(b.s, fmaxf(db, kLowest2), b.t);
    return r;
}

// Reads a granule element by element, -inf outside the row; `first`: row index of its element 0.
template <typename T>
__device__ __noinline__ uint4 get_elements(const T *row, int64_t vocab, int64_t first)
{
    constexpr int kPer = Num<T>::kPer;
    union { uint4 w; T e[kPer]; } u;
#pragma unroll
    for (int i = 0; i < kPer; ++i) u.e[i] = first + i >= 0 && first + i < vocab ? row[first + i] : Num<T>::lowest();
    return u.w;
}

// One row's slice as a block sees it: n granules, of which those from `lo` to `hi` lie inside the row entirely.
template <typename T, bool STASH, int NT>
struct Slice {
    const T *row;             // the row's first element
    const char *src;          // the slice's granule 0
    uint4 *stash;
    int64_t vocab, first0;    // first0: row index of element 0 of granule 0 (negative where the row starts inside the granule)
    int n, lo, hi;

    static constexpr int kPer = Num<T>::kPer;

    __device__ __forceinline__ Slice(const T *r, int64_t v, int part, int log2_parts, uint4 *shared) : row(r), stash(shared), vocab(v)
    {
        const uintptr_t address = reinterpret_cast<uintptr_t>(r);
        const int head = int((address & 15u) / sizeof(T));              // elements of the row's granule 0 that lie before the row
        const int64_t granules = (head + v + kPer - 1) / kPer;
        const int64_t g0 = granules * part >> log2_parts, g1 = granules * (part + 1) >> log2_parts;
        src = reinterpret_cast<const char *>(address & ~uintptr_t(15)) + g0 * 16;
        first0 = g0 * kPer - head;
        n = int(g1 - g0);
        lo = first0 < 0 ? 1 : 0;
        hi = first0 + int64_t(n) * kPer > v ? n - 1 : n;
        if (hi < lo) hi = lo;                                           // one granule, partial at both ends
    }
    __device__ __forceinline__ int64_t first(int i) const { return first0 + int64_t(i) * kPer; }
    __device__ __forceinline__ bool whole(int i) const { return unsigned(i - lo) < unsigned(hi - lo); }
    __device__ __forceinline__ uint4 partial(int i) const { return get_elements<T>(row, vocab, first(i)); }
    __device__ __forceinline__ uint4 from_global(int i) const
    {
        return whole(i) ? *reinterpret_cast<const uint4 *>(src + int64_t(i) * 16) : partial(i);
    }
    // Starts the copies of the thread's granules, kGroup to a group; only the thread itself reads them back.
    __device__ __forceinline__ void fetch() const
    {
        if constexpr (STASH) {
            const char *from = src + threadIdx.x * 16;
            uint4 *to = stash + threadIdx.x;
            for (int i = threadIdx.x; i < n; i += kGroup * NT, from += kGroup * NT * 16, to += kGroup * NT) {
                if (i >= lo && i + (kGroup - 1) * NT < hi) {
#pragma unroll
                    for (int k = 0; k < kGroup; ++k) cp_async16(to + k * NT, from + k * NT * 16);
                } else {
                    for (int k = 0; k < kGroup; ++k) {
                        const int g = i + k * NT;
                        if (whole(g)) cp_async16(to + k * NT, from + k * NT * 16);
                        else if (g < n) to[k * NT] = partial(g);
                    }
                }
                asm volatile("cp.async.commit_group;" ::: "memory");
            }
        }
    }
    // Until all but the `later` youngest groups have arrived.
    __device__ __forceinline__ void wait(int later) const
    {
        if constexpr (STASH) {
            if (later >= 3) asm volatile("cp.async.wait_group 3;" ::: "memory");
            else if (later == 2) asm volatile("cp.async.wait_group 2;" ::: "memory");
            else if (later == 1) asm volatile("cp.async.wait_group 1;" ::: "memory");
            else asm volatile("cp.async.wait_group 0;" ::: "memory");
        }
    }
    __device__ __forceinline__ uint4 get(int i) const { return STASH ? stash[i] : from_global(i); }
};

struct Shared {
    float warp[3][kMaxWarps];                          // the warps' maxima and sums
    Sums part;                                         // this block's, read by the whole cluster
};
template <int NT>
struct TopShared {
    // one warp has short rows (and no cluster): with little shared memory more of them fit a multiprocessor
    static constexpr int kCandidates = NT == 32 ? 128 : 1024, kGathered = NT == 32 ? 1 : kMaxCluster * QSR_MAX_TOP;
    float group[kGroups];
    unsigned count;
    float threshold;
    unsigned long long best, warp_best[kMaxWarps];
    unsigned long long top[QSR_MAX_TOP];
    unsigned long long gathered[kGathered];
    unsigned long long cand[kCandidates];
};

// The k largest keys of the block's slice to sh.top (0 where the slice has fewer).  The k-th largest of the group maxima bounds
// the k-th largest element from below, and few elements reach it unless many are equal; those that do are ranked by
// counting.  If they do not fit (masked or constant rows), or a NaN is about, k rounds of "largest below the last one" follow.
template <typename T, bool STASH, int NT>
__device__ __forceinline__ void slice_top(const Slice<T, STASH, NT> &sl, TopShared<NT> &sh, int k, float thread_max, bool has_nan)
{
    constexpr int kPer = Num<T>::kPer;
    constexpr unsigned kCandidates = TopShared<NT>::kCandidates;
    const int tid = threadIdx.x, lane = tid & 31;
    constexpr int per_group = NT > kGroups ? NT / kGroups : 1, groups = NT / per_group;
    float gm = thread_max;
    for (int d = 1; d < per_group; d <<= 1) gm = fmaxf(gm, __shfl_xor_sync(0xffffffffu, gm, d));
    if (tid % per_group == 0) sh.group[tid / per_group] = gm;
    if (tid < k) sh.top[tid] = 0ull;
    if (tid == 0) { sh.count = 0u; sh.threshold = -infinity(); }
    __syncthreads();
    if (tid < groups && !has_nan) {
        const float mine = sh.group[tid];
        int rank = 0;
#pragma unroll 16
        for (int i = 0; i < groups; ++i) rank += sh.group[i] > mine || (sh.group[i] == mine && i < tid);
        if (rank == k - 1) sh.threshold = mine;
    }
    __syncthreads();
    const float thr = sh.threshold;
    if (!has_nan) {
        for (int g = tid; g < sl.n; g += NT) {
            const uint4 w = sl.get(g);
            if (Num<T>::value(Num<T>::max_of(Num<T>::nothing(), w)) < thr) continue;
            float x[kPer];
            Num<T>::widen(x, w);
            unsigned hits = 0u;
#pragma unroll
            for (int i = 0; i < kPer; ++i) {
                const int64_t j = sl.first(g) + i;
                if (x[i] >= thr && j >= 0 && j < sl.vocab) hits |= 1u << i;
            }
            if (hits == 0u) continue;
            unsigned at = atomicAdd(&sh.count, unsigned(__popc(hits)));      // one for all of the granule: it is the slow part
#pragma unroll
            for (int i = 0; i < kPer; ++i)
                if (hits >> i & 1u) {
                    if (at < kCandidates) sh.cand[at] = key_of(x[i], uint32_t(sl.first(g) + i));
                    ++at;
                }
        }
    }
    __syncthreads();
    const unsigned count = sh.count;
    if (!has_nan && count <= kCandidates) {
        for (unsigned i = tid; i < count; i += NT) {
            const unsigned long long mine = sh.cand[i];
            int rank = 0;
#pragma unroll 8
            for (unsigned j = 0; j < count; ++j) rank += sh.cand[j] > mine;
            if (rank < k) sh.top[rank] = mine;
        }
        __syncthreads();
        return;
    }
    unsigned long long last = ~0ull;
    for (int r = 0; r < k; ++r) {
        unsigned long long best = 0ull;
        for (int g = tid; g < sl.n; g += NT) {
            float x[kPer];
            Num<T>::widen(x, sl.get(g));
#pragma unroll
            for (int i = 0; i < kPer; ++i) {
                const int64_t j = sl.first(g) + i;
                if (j >= 0 && j < sl.vocab) {
                    const unsigned long long key = key_of(x[i], uint32_t(j));
                    if (key < last && key > best) best = key;
                }
            }
        }
#pragma unroll
        for (int d = 16; d; d >>= 1) {
            const unsigned long long other = __shfl_xor_sync(0xffffffffu, best, d);
            best = other > best ? other : best;
        }
        if (lane == 0) sh.warp_best[tid >> 5] = best;
        __syncthreads();
        if (tid == 0) {
            for (int i = 1; i < NT / 32; ++i) best = sh.warp_best[i] > best ? sh.warp_best[i] : best;
            sh.best = best;
            sh.top[r] = best;
        }
        __syncthreads();
        last = sh.best;
        if (last == 0ull) break;              // the slice has fewer than k elements
    }
    __syncthreads();
}

// Per-row scalars of the gradient: d = a [j = y] - p (A + B log2 p) with log2 p = c (x - m) - log2 S.
// fast: log2 p = l - delta with l = c x - L in one operation, L a rounded c m + log2 S and delta what it lacks; delta goes
// into A and B, so no accuracy is lost.
struct RowGrad {
    float m, log2_s, c, L, hot, A, B;
    int64_t y;
    bool fast;
};
__device__ __forceinline__ RowGrad row_grad(const LogprobParams &p, int64_t r, int64_t y, float m, float ln_s, float H, float nan_or_0)
{
    RowGrad q;
    const bool empty = m == -infinity();
    q.m = empty ? 0.0f : m;
    q.log2_s = empty ? 0.0f : ln_s * kLog2e;
    q.c = p.tau_log2e;
    q.y = y;
    const float a = p.d_logprob && y >= 0 && !empty ? p.tau * p.d_logprob[r] + nan_or_0 : 0.0f;
    const float b = p.d_entropy && !empty ? p.tau * p.d_entropy[r] : 0.0f;
    q.hot = a;
    q.A = fmaf(b, H, a);
    q.B = b * kLn2;
    const float K = q.c * q.m;
    q.L = K + q.log2_s;
    q.fast = fabsf(K) < kGradMax;
    if (q.fast) {
        // c m + log2 S - L, each step exact or as small as what it corrects
        const float delta = fmaf(q.c, q.m, -K) + ((K - q.L) + q.log2_s), f = exp2_1(-delta);
        q.A = f * fmaf(-q.B, delta, q.A);
        q.B *= f;
    }
    return q;
}

template <typename T, bool ENTROPY, bool FAST>
__device__ __forceinline__ void grad_terms(float (&x)[Num<T>::kPer], uint4 w, const RowGrad &q)
{
    Num<T>::widen(x, w);
#pragma unroll
    for (int i = 0; i < Num<T>::kPer; i += 2) {
        const float2 v = make_float2(x[i], x[i + 1]);
        const float2 l = FAST ? fma2(v, both(q.c), both(-q.L)) : fma2(add2(v, both(-q.m)), both(q.c), both(-q.log2_s));
        const float2 e = make_float2(exp2_1(l.x), exp2_1(l.y));
        float2 f = both(-q.A);
        if (ENTROPY) f = fma2(both(-q.B), make_float2(fmaxf(l.x, kLowest2), fmaxf(l.y, kLowest2)), f);
        const float2 o = mul2(e, f);
        x[i] = o.x; x[i + 1] = o.y;
    }
}
// The gradient of one granule, the token's own term aside.
template <typename T, bool ENTROPY, bool FAST>
__device__ __forceinline__ uint4 granule_grad(uint4 w, const RowGrad &q)
{
    constexpr int kPer = Num<T>::kPer;
    float x[kPer];
    grad_terms<T, ENTROPY, FAST>(x, w, q);
    return Num<T>::narrow(x);
}
// The gradient of the granule that holds the token, at `place`.
template <typename T>
__device__ __forceinline__ uint4 token_grad(uint4 w, const RowGrad &q, int place)
{
    constexpr int kPer = Num<T>::kPer;
    float x[kPer];
    if (q.fast) grad_terms<T, true, true>(x, w, q);
    else grad_terms<T, true, false>(x, w, q);
#pragma unroll
    for (int i = 0; i < kPer; ++i) x[i] += i == place ? q.hot : 0.0f;
    return Num<T>::narrow(x);
}

// Writes a granule element by element; `first`: row index of its element 0.
template <typename T>
__device__ __noinline__ void put_elements(T *out_row, int64_t vocab, int64_t first, uint4 w)
{
    constexpr int kPer = Num<T>::kPer;
    union { uint4 w; T e[kPer]; } u;
    u.w = w;
#pragma unroll
    for (int i = 0; i < kPer; ++i)
        if (first + i >= 0 && first + i < vocab) out_row[first + i] = u.e[i];
}

template <typename T>
__device__ __forceinline__ bool same_phase(const T *a, const T *b)
{
    return ((reinterpret_cast<uintptr_t>(a) ^ reinterpret_cast<uintptr_t>(b)) & 15u) == 0;
}

// Where the token lies in a slice: its granule (or -1) and its place there.
struct HotSpot { int granule, place; };
template <int PER>
__device__ __forceinline__ HotSpot hot_spot(const RowGrad &q, int64_t first0, int n)
{
    const int64_t at = q.y - first0;
    if (q.y < 0 || q.hot == 0.0f || at < 0 || at >= int64_t(n) * PER) return HotSpot{-1, -1};
    return HotSpot{int(at / PER), int(at % PER)};
}

// Gradient of a thread's granules of a slice.  The granule that holds the token is written twice, the second time with the
// token's term, so that the loop need not look for it.
template <typename T, bool STASH, int NT, bool ENTROPY, bool FAST>
__device__ __forceinline__ void write_grad(const Slice<T, STASH, NT> &sl, T *out, const RowGrad &q)
{
    const HotSpot hot = hot_spot<Num<T>::kPer>(q, sl.first0, sl.n);
    const int tid = threadIdx.x;
    const bool mine = hot.granule >= 0 && hot.granule % NT == tid;
    uint4 token_granule = make_uint4(0u, 0u, 0u, 0u);
    if (mine) token_granule = sl.get(hot.granule);            // before it is overwritten: out may be the logits
    // 16-byte stores where the output row lies like the input row modulo 16 bytes
    const bool vector = same_phase<T>(sl.row, out);
    if (vector) {
        int i = tid < sl.lo ? tid + NT : tid;
        char *dst = reinterpret_cast<char *>(out) + sl.first0 * int64_t(sizeof(T)) + int64_t(i) * 16;
#pragma unroll 4
        for (; i < sl.hi; i += NT, dst += NT * 16) *reinterpret_cast<uint4 *>(dst) = granule_grad<T, ENTROPY, FAST>(sl.get(i), q);
        if (tid < sl.lo) put_elements<T>(out, sl.vocab, sl.first(0), granule_grad<T, ENTROPY, FAST>(sl.get(0), q));
        if (sl.hi < sl.n && sl.hi % NT == tid)
            put_elements<T>(out, sl.vocab, sl.first(sl.hi), granule_grad<T, ENTROPY, FAST>(sl.get(sl.hi), q));
    } else {
        for (int i = tid; i < sl.n; i += NT) put_elements<T>(out, sl.vocab, sl.first(i), granule_grad<T, ENTROPY, FAST>(sl.get(i), q));
    }
    if (mine) put_elements<T>(out, sl.vocab, sl.first(hot.granule), token_grad<T>(token_granule, q, hot.place));
}

// A thread's running maximum and sums: e = 2^z and e z with z = c x - K, K a rounded c m.  One operation forms z and nothing is
// lost by it: the product is exact inside the fused multiply-add, and K is the same constant in every term; what K lacks of
// c m is put back at the end (relative_to).  That holds while |K| < kBaseMax.  A maximum below that range (a thread that
// has only seen a mask of -1e10, say) takes K = -kBaseMax: its sums are then 0 or something finite, and count for nothing next to
// a maximum inside the range.  `odd`: a NaN or a maximum above the range.
template <bool ENTROPY>
struct Running {
    float m = -infinity(), K = 0.0f;
    float2 s = make_float2(0.0f, 0.0f), t = make_float2(0.0f, 0.0f);
    bool odd = false;

    template <typename T, int N>
    __device__ __forceinline__ void add(const uint4 (&w)[N], float c)
    {
        constexpr int kPer = Num<T>::kPer;
        typename Num<T>::Max most = Num<T>::nothing();
#pragma unroll
        for (int k = 0; k < N; ++k) most = Num<T>::max_of(most, w[k]);
        const float x = Num<T>::value(most);
        if (!(x <= m)) {
            const float cx = x * c, K1 = fmaxf(cx, -kBaseMax);
            odd = odd || !(cx < kBaseMax);
            if (m > -infinity()) shift(K - K1);
            m = x;
            K = K1;
        }
#pragma unroll
        for (int k = 0; k < N; ++k) {
            float v[kPer];
            Num<T>::widen(v, w[k]);
#pragma unroll
            for (int i = 0; i < kPer; i += 2) {
                const float2 z = fma2(make_float2(v[i], v[i + 1]), both(c), both(-K));
                const float2 e = make_float2(exp2_1(z.x), exp2_1(z.y));
                s = add2(s, e);
                if (ENTROPY) t = fma2(e, make_float2(fmaxf(z.x, kLowest2), fmaxf(z.y, kLowest2)), t);
            }
        }
    }
    // Sums relative to a base d below the present one (d <= 0 where the base rises).
    __device__ __forceinline__ void shift(float d)
    {
        const float f = exp2_1(d);
        d = fmaxf(d, kLowest2);
        if (ENTROPY) t = mul2(both(f), fma2(both(d), s, t));
        s = mul2(both(f), s);
    }
    __device__ __forceinline__ Sums relative_to(float most, float c)
    {
        if (m > -infinity()) shift(fminf(fmaf(-c, most, K), 64.0f));      // 64 at most inside the range
        return Sums{most, s.x + s.y, t.x + t.y};
    }
};

// The slow way for slices whose maximum is a NaN or out of the fast exponents' range: the maximum first (NaN if there is one),
// then the terms with z = c (x - m).
template <typename T, bool STASH, int NT>
__device__ __forceinline__ Sums sums_of_odd(const Slice<T, STASH, NT> &sl, float c, Shared &sh)
{
    constexpr int kPer = Num<T>::kPer;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    typename Num<T>::Max running = Num<T>::nothing();
    for (int g = threadIdx.x; g < sl.n; g += NT) running = Num<T>::max_of(running, sl.get(g));
    float m = warp_max_nan(Num<T>::value(running));
    __syncthreads();
    if (lane == 0) sh.warp[0][warp] = m;
    __syncthreads();
    m = warp_max_nan(sh.warp[0][lane < NT / 32 ? lane : 0]);
    const float base = m == -infinity() ? 0.0f : m;
    float s = 0.0f, t = 0.0f;
    for (int g = threadIdx.x; g < sl.n; g += NT) {
        float x[kPer];
        Num<T>::widen(x, sl.get(g));
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            const float z = (x[i] - base) * c, e = exp2_1(z);
            s += e;
            t = fmaf(e, fmaxf(z, kLowest2), t);
        }
    }
    s = warp_sum(s);
    t = warp_sum(t);
    if (lane == 0) { sh.warp[1][warp] = s; sh.warp[2][warp] = t; }
    __syncthreads();
    s = warp_sum(lane < NT / 32 ? sh.warp[1][lane] : 0.0f);
    t = warp_sum(lane < NT / 32 ? sh.warp[2][lane] : 0.0f);
    Sums all{m, s, t};
    if (!(m < infinity())) all.m = all.s = quiet_nan();       // a NaN or +inf: the row is NaN
    return all;
}

// The slice's maximum and sums, the same in every thread of the block; thread_max: the thread's own maximum (NaNs aside).
template <typename T, bool STASH, int NT, bool ENTROPY>
__device__ __forceinline__ Sums sums_of(const Slice<T, STASH, NT> &sl, float c, Shared &sh, float &thread_max)
{
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    Running<ENTROPY> run;
    const int mine = sl.n > tid ? (sl.n - tid + NT - 1) / NT : 0;
    int i = tid, later = (mine + kGroup - 1) / kGroup;
    for (; i + (kGroup - 1) * NT < sl.n; i += kGroup * NT) {
        sl.wait(--later);
        uint4 w[kGroup];
#pragma unroll
        for (int k = 0; k < kGroup; ++k) w[k] = sl.get(i + k * NT);
        run.template add<T>(w, c);
    }
    sl.wait(0);
    for (; i < sl.n; i += NT) {
        const uint4 w[1] = {sl.get(i)};
        run.template add<T>(w, c);
    }
    thread_max = run.m;
    const float m = warp_max(run.m);
    Sums all = run.relative_to(m, c);
    all.s = warp_sum(all.s);
    if (ENTROPY) all.t = warp_sum(all.t);
    bool odd = run.odd;
    if (NT == 32) odd = __any_sync(0xffffffffu, odd);
    else {
        if (lane == 0) { sh.warp[0][warp] = all.m; sh.warp[1][warp] = all.s; sh.warp[2][warp] = all.t; }
        odd = __syncthreads_or(odd);
        all.m = -infinity();
        all.s = all.t = 0.0f;
        if (lane < NT / 32) all = Sums{sh.warp[0][lane], sh.warp[1][lane], sh.warp[2][lane]};
        const float most = warp_max(all.m);
        if (all.s > 0.0f) {
            const float d = (all.m - most) * c, f = exp2_1(d);
            all.t = f * fmaf(fmaxf(d, kLowest2), all.s, all.t);
            all.s *= f;
        }
        all.m = most;
        all.s = warp_sum(all.s);
        all.t = warp_sum(all.t);
    }
    // the slice's maximum itself below the range, or so near its end that threads below may count
    odd = odd || (all.m > -infinity() && !(all.m * c > 4096.0f - kBaseMax));
    return odd ? sums_of_odd<T, STASH, NT>(sl, c, sh) : all;
}

// One row per cluster.  TOP: alternatives are wanted; GRAD: d_logits is.
template <typename T, bool STASH, int NT, bool TOP, bool GRAD>
__global__ void __launch_bounds__(NT, 1024 / NT) logprob_kernel(const __grid_constant__ LogprobParams p, const int log2_cluster)
{
    extern __shared__ uint4 stash[];
    __shared__ Shared sh;
    __shared__ typename std::conditional<TOP, TopShared<NT>, int>::type top_sh;
    const int tid = threadIdx.x, cluster = 1 << log2_cluster;
    const int64_t r = blockIdx.x >> log2_cluster;
    const int rank = int(blockIdx.x) & (cluster - 1);

    const T *const row = static_cast<const T *>(p.logits) + r * p.stride;
    const Slice<T, STASH, NT> sl(row, p.vocab, rank, log2_cluster, stash);
    const int64_t y = p.tokens[r];
    float token_logit = 0.0f;
    if (tid == 0 && rank == 0 && y >= 0) token_logit = y < p.vocab ? Num<T>::to_float(row[y]) : quiet_nan();

    // a block's shared memory may only be written by another once both run: announced here, awaited before the first write
    if (TOP && cluster > 1) asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");
    sl.fetch();
    const float c = p.tau_log2e;
    float thread_max;
    Sums all = p.entropy || p.d_entropy ? sums_of<T, STASH, NT, true>(sl, c, sh, thread_max) : sums_of<T, STASH, NT, false>(sl, c, sh, thread_max);
    if (TOP) slice_top<T, STASH, NT>(sl, reinterpret_cast<TopShared<NT> &>(top_sh), p.n_top, thread_max, isnan(all.m));
    if (cluster > 1) {
        cg::cluster_group cl = cg::this_cluster();
        if (tid == 0) sh.part = all;
        if (TOP) {
            asm volatile("barrier.cluster.wait.aligned;" ::: "memory");
            TopShared<NT> &mine = reinterpret_cast<TopShared<NT> &>(top_sh);
            unsigned long long *gather = cl.map_shared_rank(mine.gathered, 0);
            if (tid < p.n_top) gather[rank * p.n_top + tid] = mine.top[tid];
        }
        cl.sync();
        all = *cl.map_shared_rank(&sh.part, 0);
        for (int i = 1; i < cluster; ++i) all = join(all, *cl.map_shared_rank(&sh.part, i), c);
        cl.sync();                                            // no block leaves (or reuses `part`) while another reads it
    }
    const bool empty = all.m == -infinity();
    const float ln_s = empty ? 0.0f : logf(all.s);
    const float H = empty ? 0.0f : fmaxf(ln_s - kLn2 * (all.t / all.s), 0.0f) + 0.0f * all.s;

    if (rank == 0) {
        if (tid == 0) {
            const float lp = empty ? -infinity() : fmaf(p.tau, token_logit - all.m, -ln_s);
            p.logprob[r] = y < 0 ? 0.0f : (y < p.vocab ? lp : quiet_nan());
            if (p.entropy) p.entropy[r] = H;
            if (p.stats) { p.stats[2 * r] = all.m; p.stats[2 * r + 1] = ln_s; }
        }
        if (TOP) {
            TopShared<NT> &mine = reinterpret_cast<TopShared<NT> &>(top_sh);
            if (cluster > 1) {
                const int n = cluster * p.n_top;
                for (int i = tid; i < n; i += NT) {
                    const unsigned long long key = mine.gathered[i];
                    int place = 0;
#pragma unroll 8
                    for (int j = 0; j < n; ++j) place += mine.gathered[j] > key;
                    if (key != 0ull && place < p.n_top) mine.top[place] = key;
                }
                __syncthreads();
            }
            if (tid < p.n_top) {
                const unsigned long long key = mine.top[tid];
                p.top_token[r * p.n_top + tid] = int64_t(0xffffffffu - uint32_t(key));
                p.top_logprob[r * p.n_top + tid] = empty ? -infinity() : fmaf(p.tau, unsort_bits(uint32_t(key >> 32)) - all.m, -ln_s);
            }
        }
    }
    if (GRAD) {
        __syncthreads();              // d_logits may be the logits: the token's logit has been read
        const RowGrad q = row_grad(p, r, y, all.m, ln_s, H, y < p.vocab ? 0.0f : quiet_nan());
        T *const out = static_cast<T *>(p.d_logits) + r * p.d_stride;
        if (!q.fast) write_grad<T, STASH, NT, true, false>(sl, out, q);
        else if (q.B == 0.0f) write_grad<T, STASH, NT, false, true>(sl, out, q);
        else write_grad<T, STASH, NT, true, true>(sl, out, q);
    }
}

constexpr int kGradPer = 4;                   // granules in flight per thread

// The gradient alone, from the statistics of an earlier call.  Grid: 2^log2_parts parts of a row by rows.  Six blocks of 256
// threads per multiprocessor (40 registers): with 43 and five blocks the two calls on 2048 x 50001 bf16 took 150 us instead of 146.
template <typename T, int NT>
__global__ void __launch_bounds__(NT, NT == 256 ? 6 : 1) logprob_grad_kernel(const __grid_constant__ LogprobParams p, const int log2_parts)
{
    const int64_t r = blockIdx.x >> log2_parts;
    const T *const row = static_cast<const T *>(p.logits) + r * p.stride;
    const Slice<T, false, NT> sl(row, p.vocab, int(blockIdx.x) & ((1 << log2_parts) - 1), log2_parts, nullptr);
    constexpr int step = NT;
    const int begin = threadIdx.x;
    uint4 w[kGradPer];
#pragma unroll
    for (int k = 0; k < kGradPer; ++k)
        if (begin + k * step < sl.n) w[k] = sl.from_global(begin + k * step);
    const int64_t y = p.tokens[r];
    const RowGrad q = row_grad(p, r, y, p.stats[2 * r], p.stats[2 * r + 1], p.d_entropy ? p.entropy[r] : 0.0f,
                               y < p.vocab ? 0.0f : quiet_nan());
    T *const out = static_cast<T *>(p.d_logits) + r * p.d_stride;
    const HotSpot hot = hot_spot<Num<T>::kPer>(q, sl.first0, sl.n);
    const bool vector = same_phase<T>(row, out);
    char *const dst = reinterpret_cast<char *>(out) + sl.first0 * int64_t(sizeof(T));
#pragma unroll
    for (int k = 0; k < kGradPer; ++k) {
        const int i = begin + k * step;
        if (i < sl.n) {
            uint4 d = !q.fast ? granule_grad<T, true, false>(w[k], q)
                      : q.B == 0.0f ? granule_grad<T, false, true>(w[k], q) : granule_grad<T, true, true>(w[k], q);
            if (i == hot.granule) d = token_grad<T>(w[k], q, hot.place);
            if (vector && sl.whole(i)) *reinterpret_cast<uint4 *>(dst + int64_t(i) * 16) = d;
            else put_elements<T>(out, p.vocab, sl.first(i), d);
        }
    }
}

// Two blocks of such a slice share a multiprocessor.  With alternatives, for which a block has 11 KB of its own, they do up to 102
// KB; slices between the two bounds run one block at a time there.
constexpr int64_t kSliceBytes = 110 * 1024;
constexpr int64_t kStashMax = 200 * 1024;
constexpr int kMultiprocessors = 148;

// How a row is shared out.
// Clusters: only where a row's slice would be longer than kSliceBytes (the exchange costs more than the second block of a
// multiprocessor gains: 2048 x 50001 bf16 in one block of 100 KB 169 us, in two of 50 KB 180), or where there are too few rows
// to fill the multiprocessors (8 x 131072 bf16: clusters of eight 5.1 us forward, of four 5.9).
// Threads: about sixteen granules each, since what a thread does once per row costs as much as two or three granules (8192 x
// 32768 bf16, 64 KB: 256 threads 215 us, 512 222 to 243), but enough warps for rows that leave room for two blocks only (100
// KB: 512 threads 158 us, 256 169); one warp for the shortest rows, which then need no barrier.
struct Shape { int log2_cluster, threads; int64_t smem; };

Shape shape_of(const LogprobParams &p, int element)
{
    const int64_t bytes = (p.vocab * element + 15 + 15) / 16 * 16;
    Shape s;
    s.log2_cluster = 0;
    while (1 << s.log2_cluster < kMaxCluster &&
           (bytes > kSliceBytes << s.log2_cluster || ((p.rows << s.log2_cluster) * 2 <= kMultiprocessors && bytes >= int64_t(8192) << s.log2_cluster)))
        s.log2_cluster++;
    const int64_t granules = ((bytes / 16 - 1) >> s.log2_cluster) + 2;
    s.threads = granules <= 256 && s.log2_cluster == 0 ? 32 : granules <= 1024 ? 128 : granules <= 4608 ? 256 : 512;
    s.smem = granules * 16;
    return s;
}

template <typename T, bool STASH, int NT, bool TOP, bool GRAD>
int launch_instance(const LogprobParams &p, const Shape &s, cudaStream_t st)
{
    const auto kernel = logprob_kernel<T, STASH, NT, TOP, GRAD>;
    const size_t smem = STASH ? size_t(s.smem) : 0;
    if (smem > 32 * 1024) {
        static std::atomic<uint64_t> raised{0};           // devices on which this instance may use kStashMax
        if (int err = allow_shared(reinterpret_cast<const void *>(kernel), int(kStashMax), raised)) return err;
    }
    if (s.log2_cluster == 0) {
        kernel<<<unsigned(p.rows), NT, smem, st>>>(p, 0);
        return int(cudaGetLastError());
    }
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(unsigned(p.rows << s.log2_cluster));
    cfg.blockDim = dim3(NT);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = 1u << s.log2_cluster;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return int(cudaLaunchKernelEx(&cfg, kernel, p, s.log2_cluster));
}

template <typename T, bool STASH, int NT>
int launch_outputs(const LogprobParams &p, const Shape &s, cudaStream_t st)
{
    if (p.n_top > 0) return p.d_logits ? launch_instance<T, STASH, NT, true, true>(p, s, st) : launch_instance<T, STASH, NT, true, false>(p, s, st);
    return p.d_logits ? launch_instance<T, STASH, NT, false, true>(p, s, st) : launch_instance<T, STASH, NT, false, false>(p, s, st);
}

template <typename T>
int launch_typed(const LogprobParams &p, cudaStream_t st)
{
    const Shape s = shape_of(p, int(sizeof(T)));
    if (s.smem > kStashMax) return launch_outputs<T, false, 512>(p, s, st);
    if (s.threads == 32) return launch_outputs<T, true, 32>(p, s, st);
    if (s.threads == 128) return launch_outputs<T, true, 128>(p, s, st);
    if (s.threads == 256) return launch_outputs<T, true, 256>(p, s, st);
    return launch_outputs<T, true, 512>(p, s, st);
}

template <typename T, int NT>
int launch_grad_instance(const LogprobParams &p, int64_t granules, cudaStream_t st)
{
    int log2_parts = 0;
    while ((granules >> log2_parts) + 1 > NT * kGradPer) log2_parts++;
    if (p.rows > (0x7fffffff >> log2_parts)) return int(cudaErrorInvalidConfiguration);
    logprob_grad_kernel<T, NT><<<unsigned(p.rows << log2_parts), NT, 0, st>>>(p, log2_parts);
    return int(cudaGetLastError());
}

template <typename T>
int launch_grad_typed(const LogprobParams &p, cudaStream_t st)
{
    const int64_t granules = (p.vocab * int64_t(sizeof(T)) + 15 + 15) / 16;
    return granules <= 32 * kGradPer ? launch_grad_instance<T, 32>(p, granules, st) : launch_grad_instance<T, 256>(p, granules, st);
}

}  // namespace

int launch_logprobs(const LogprobParams &p, void *stream)
{
    const cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (p.type == QSR_F32) return launch_typed<float>(p, st);
    if (p.type == QSR_BF16) return launch_typed<__nv_bfloat16>(p, st);
    return launch_typed<__half>(p, st);
}

int launch_logprobs_grad(const LogprobParams &p, void *stream)
{
    const cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (p.type == QSR_F32) return launch_grad_typed<float>(p, st);
    if (p.type == QSR_BF16) return launch_grad_typed<__nv_bfloat16>(p, st);
    return launch_grad_typed<__half>(p, st);
}

}  // namespace qsr

namespace {

bool element_aligned(const void *p, unsigned bytes) { return (reinterpret_cast<uintptr_t>(p) & (bytes - 1)) == 0; }

// Whether two matrices of rows x vocab elements of e bytes (strides in elements; not the same matrix) share one.  With equal
// strides, as columns of one buffer have them, rows meet exactly if the distance modulo the stride is less than a row from
// either side; otherwise matrices that lie in and out of one another count as sharing.
bool share_bytes(const void *a, int64_t a_stride, const void *b, int64_t b_stride, int64_t rows, int64_t vocab, int e)
{
    typedef __int128 wide;                          // strides have no upper limit
    const wide x = wide(reinterpret_cast<uintptr_t>(a)), y = wide(reinterpret_cast<uintptr_t>(b));
    const wide row = wide(vocab) * e, xs = wide(a_stride) * e, ys = wide(b_stride) * e;
    if (x + (rows - 1) * xs + row <= y || y + (rows - 1) * ys + row <= x) return false;
    if (xs != ys || rows == 1) return true;
    const wide d = (x > y ? x - y : y - x) % xs;
    return d < row || d > xs - row;
}

// Checks what both calls share and fills the kernel's arguments.
int logprob_params(const qsr_logprob_args *a, bool forward, qsr::LogprobParams &p)
{
    if (!a) return QSR_EINVAL;
    if (a->logits_type != QSR_F32 && a->logits_type != QSR_BF16 && a->logits_type != QSR_F16) return QSR_EINVAL;
    const float tau = float(a->inv_temperature), tau_log2e = float(a->inv_temperature * 1.4426950408889634);
    if (!(tau > 0.0f) || !std::isfinite(tau_log2e)) return QSR_EINVAL;
    if (a->rows < 0 || a->rows >= (int64_t(1) << 28) || a->vocab < 1 || a->vocab > 0x7fffffff || a->row_stride < a->vocab) return QSR_ERANGE;
    if (forward && (a->n_top < 0 || a->n_top > QSR_MAX_TOP || a->n_top > a->vocab)) return QSR_ERANGE;
    if (a->d_logits && (a->d_row_stride < a->vocab || (a->d_logits == a->logits && a->d_row_stride != a->row_stride))) return QSR_ERANGE;
    if (a->rows > 0) {
        if (!a->logits || !a->tokens) return QSR_EINVAL;
        if (forward && (!a->logprob || (a->n_top > 0 && (!a->top_logprob || !a->top_token)))) return QSR_EINVAL;
        if (!forward && (!a->d_logits || !a->row_stats || (a->d_entropy && !a->entropy))) return QSR_EINVAL;
    }
    const unsigned e = a->logits_type == QSR_F32 ? 4 : 2;
    if (!element_aligned(a->logits, e) || !element_aligned(a->d_logits, e) || !element_aligned(a->tokens, 8) ||
        !element_aligned(a->entropy, 4) || !element_aligned(a->row_stats, 8) || !element_aligned(a->d_logprob, 4) ||
        !element_aligned(a->d_entropy, 4))
        return QSR_EALIGN;
    if (forward && (!element_aligned(a->logprob, 4) || (a->n_top > 0 && (!element_aligned(a->top_logprob, 4) || !element_aligned(a->top_token, 8)))))
        return QSR_EALIGN;
    if (a->rows > 0 && a->d_logits && a->d_logits != a->logits &&
        share_bytes(a->logits, a->row_stride, a->d_logits, a->d_row_stride, a->rows, a->vocab, int(e)))
        return QSR_EINVAL;
    p.logits = a->logits; p.tokens = a->tokens;
    p.logprob = a->logprob; p.entropy = a->entropy; p.stats = a->row_stats;
    p.top_logprob = a->top_logprob; p.top_token = a->top_token;
    p.d_logprob = a->d_logprob; p.d_entropy = a->d_entropy; p.d_logits = a->d_logits;
    p.rows = a->rows; p.vocab = a->vocab; p.stride = a->row_stride; p.d_stride = a->d_row_stride;
    p.type = a->logits_type; p.n_top = a->n_top;
    p.tau = tau;
    p.tau_log2e = tau_log2e;
    return QSR_OK;
}

int launched(int err)
{
    if (err == 0) return QSR_OK;
    cudaGetLastError();
    return QSR_ECUDA;
}

}  // namespace

extern "C" {

int qsr_token_logprobs(const qsr_logprob_args *args, void *cuda_stream)
{
    qsr::LogprobParams p;
    if (int rc = logprob_params(args, true, p)) return rc;
    return p.rows == 0 ? QSR_OK : launched(qsr::launch_logprobs(p, cuda_stream));
}

int qsr_token_logprobs_grad(const qsr_logprob_args *args, void *cuda_stream)
{
    qsr::LogprobParams p;
    if (int rc = logprob_params(args, false, p)) return rc;
    return p.rows == 0 ? QSR_OK : launched(qsr::launch_logprobs_grad(p, cuda_stream));
}

}  // extern "C"
