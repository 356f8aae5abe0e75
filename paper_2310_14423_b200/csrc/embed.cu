// Embedding lookup with scaling, and its gradient by sorted tokens.  See include/qsr.h.
#include <cuda_runtime.h>

#include <algorithm>
#include <cmath>

#include "checks.h"
#include "rows.cuh"

namespace qsr {

namespace {

// ---- lookup ----------------------------------------------------------------------------------------------

struct LookupParams {
    const void *table;
    const int64_t *tokens;
    void *out;
    int64_t rows, vocab, table_stride, out_stride;
    int32_t width, out_type;
    int32_t lanes, parts;             // threads that share a part of a row (a power of two up to 32), parts of a row
    float scale;
};

constexpr int kHeld = 4;              // granules of eight elements a thread copies at a time

// A group of `lanes` threads copies a part of one row: all its loads first, then the stores.  Bound by memory: 65536 rows of 1024 out of an fp32 table
// into bf16, 38 us.
template <typename T, bool VEC>
__global__ void __launch_bounds__(256) lookup_kernel(const __grid_constant__ LookupParams p)
{
    const int lane = int(threadIdx.x) & (p.lanes - 1);
    const int64_t unit = int64_t(blockIdx.x) * (256 / p.lanes) + int(threadIdx.x) / p.lanes;
    const int64_t row = unit / p.parts;
    if (row >= p.rows) return;
    const int first = int(unit - row * p.parts) * p.lanes * kHeld * 8;       // first column of the part
    const int width = p.width - first;
    const int64_t token = p.tokens[row];
    const bool known = token >= 0 && token < p.vocab;
    const void *from = static_cast<const T *>(p.table) + (known ? token * p.table_stride : 0) + first;
    const int64_t to = row * p.out_stride + first;
    Raw8 raw[kHeld];
#pragma unroll
    for (int k = 0; k < kHeld; ++k) fetch<VEC>(raw[k], from, lane, p.lanes, k, known ? width : 0, Kind<T>::type);
    const float scale = token < p.vocab ? p.scale : quiet_nan();
    void *out = p.out_type == QSR_F32 ? static_cast<void *>(static_cast<float *>(p.out) + to) : static_cast<void *>(static_cast<uint16_t *>(p.out) + to);
#pragma unroll
    for (int k = 0; k < kHeld; ++k) {
        if (column<VEC>(lane, p.lanes, k, 0) >= width) break;
        float x[8];
        widen8(x, raw[k], Kind<T>::type);
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] *= scale;
        put<VEC>(out, x, lane, p.lanes, k, width, p.out_type);
    }
}

// ---- sorting the tokens ----------------------------------------------------------------------------------

// Many rows: a stable radix sort of (token, row), lowest digits first.  The blocks count their first digits, then there is one launch for
// each pass, in which every block finds its places from all blocks' counts and counts the next digits of what it places where they
// land.  Tokens that are not in the vocabulary sort behind it.  65536 rows, 50001 tokens: 3.5 us and twice 8.4, in part behind one another.
//
// The launches of a gradient follow one another closely: each is started before the one before it has ended and waits for that.
__device__ __forceinline__ void wait_for_launch_before() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
__device__ __forceinline__ void let_next_launch_start() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }

constexpr int kMaxDigit = 10;          // bits
constexpr int kSortThreads = 512, kSortWarps = kSortThreads / 32;
constexpr int kSortPer = 4;            // keys that a thread holds at a time
constexpr int kMaxSortBlocks = 128;

struct SortParams {
    const int64_t *tokens;             // first pass; otherwise keys and rows
    const uint32_t *keys, *rows;
    uint32_t *keys_out, *rows_out;
    uint32_t *counts, *next_counts;    // [blocks, 1 << bits]; the next pass's, or NULL
    int64_t n, per_warp;               // per_warp: a multiple of 32
    uint32_t vocab;
    int32_t shift, bits, passes;
};

__device__ __forceinline__ uint32_t key_of(int64_t token, uint32_t vocab) { return token >= 0 && token < int64_t(vocab) ? uint32_t(token) : vocab; }
__device__ __forceinline__ uint32_t key_at(const SortParams &p, int64_t i) { return p.tokens ? key_of(p.tokens[i], p.vocab) : p.keys[i]; }

__global__ void __launch_bounds__(kSortThreads) count_kernel(const __grid_constant__ SortParams p)
{
    __shared__ uint32_t count[1 << kMaxDigit];
    let_next_launch_start();
    const int digits = 1 << p.bits;
    for (int d = threadIdx.x; d < digits; d += kSortThreads) count[d] = 0;
    __syncthreads();
    const int64_t begin = int64_t(blockIdx.x) * p.per_warp * kSortWarps, end = min(p.n, begin + p.per_warp * kSortWarps);
    for (int64_t i0 = begin + threadIdx.x; i0 < end; i0 += kSortPer * kSortThreads) {
        uint32_t key[kSortPer];
#pragma unroll
        for (int k = 0; k < kSortPer; ++k) key[k] = i0 + k * kSortThreads < end ? key_at(p, i0 + k * kSortThreads) : 0u;
#pragma unroll
        for (int k = 0; k < kSortPer; ++k)
            if (i0 + k * kSortThreads < end) atomicAdd(&count[key[k] & uint32_t(digits - 1)], 1u);
    }
    __syncthreads();
    for (int d = threadIdx.x; d < digits; d += kSortThreads) {
        p.counts[int64_t(blockIdx.x) * digits + d] = count[d];
        for (int pass = 1; pass < p.passes; ++pass) p.next_counts[(int64_t(pass - 1) * gridDim.x + blockIdx.x) * digits + d] = 0;
    }
}

// Sum over the threads before this one.
template <int THREADS>
__device__ __forceinline__ uint32_t exclusive_scan(uint32_t v, uint32_t *scratch)
{
    uint32_t s = v;
#pragma unroll
    for (int d = 1; d < 32; d *= 2) {
        const uint32_t u = __shfl_up_sync(0xffffffffu, s, d);
        if (int(threadIdx.x & 31) >= d) s += u;
    }
    if ((threadIdx.x & 31) == 31) scratch[threadIdx.x >> 5] = s;
    __syncthreads();
    uint32_t w = (threadIdx.x & 31) < THREADS / 32 ? scratch[threadIdx.x & 31] : 0u;
    w = (threadIdx.x & 31) < (threadIdx.x >> 5) ? w : 0u;
    return __reduce_add_sync(0xffffffffu, w) + s - v;
}

// Places of a warp's keys: `place` holds the next place of each digit for this warp and is moved on.
__device__ __forceinline__ uint32_t take_place(uint32_t *place, uint32_t digit, bool live, int lane)
{
    const uint32_t same = __match_any_sync(0xffffffffu, live ? digit : 0xffffffffu);
    const int rank = __popc(same & ((1u << lane) - 1u));
    const uint32_t to = live ? place[digit] + uint32_t(rank) : 0u;
    __syncwarp();
    if (live && rank == 0) place[digit] += uint32_t(__popc(same));
    __syncwarp();
    return to;
}

__global__ void __launch_bounds__(kSortThreads) place_kernel(const __grid_constant__ SortParams p)
{
    extern __shared__ uint32_t places[];                        // [warps][digits]: next place of each digit, warp by warp
    __shared__ uint32_t scratch[kSortWarps];
    const int digits = 1 << p.bits, mask = digits - 1, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    uint32_t *place = places + warp * digits;
    for (int i = threadIdx.x; i < kSortWarps * digits; i += kSortThreads) places[i] = 0;
    __syncthreads();
    wait_for_launch_before();
    let_next_launch_start();
    const int64_t begin = (int64_t(blockIdx.x) * kSortWarps + warp) * p.per_warp, end = min(p.n, begin + p.per_warp);
    for (int64_t i0 = begin + lane; i0 < end; i0 += 32 * kSortPer) {
        uint32_t key[kSortPer];
#pragma unroll
        for (int k = 0; k < kSortPer; ++k) key[k] = i0 + k * 32 < end ? key_at(p, i0 + k * 32) : 0u;
#pragma unroll
        for (int k = 0; k < kSortPer; ++k)
            if (i0 + k * 32 < end) atomicAdd(&place[(key[k] >> p.shift) & mask], 1u);
    }
    // each digit's total and its share in the blocks before this one; consecutive digits to a thread, so that a scan over
    // threads is one over digits
    constexpr int kPer = (1 << kMaxDigit) / kSortThreads;
    const int per = max(1, digits / kSortThreads), d0 = int(threadIdx.x) * per;
    uint32_t total[kPer], earlier[kPer], all = 0;
#pragma unroll
    for (int k = 0; k < kPer; ++k) {
        uint32_t t = 0, e = 0;
        if (k < per && d0 + k < digits) {
#pragma unroll 16
            for (int b = 0; b < int(gridDim.x); ++b) {
                const uint32_t c = __ldcg(&p.counts[int64_t(b) * digits + d0 + k]);
                t += c;
                e += b < int(blockIdx.x) ? c : 0u;
            }
        }
        total[k] = t; earlier[k] = e;
        all += t;
    }
    uint32_t at = exclusive_scan<kSortThreads>(all, scratch);
    __syncthreads();                                            // all warps have counted
#pragma unroll
    for (int k = 0; k < kPer; ++k)
        if (k < per && d0 + k < digits) {
            uint32_t next = at + earlier[k];
#pragma unroll
            for (int w = 0; w < kSortWarps; ++w) {
                const uint32_t c = places[w * digits + d0 + k];
                places[w * digits + d0 + k] = next;
                next += c;
            }
            at += total[k];
        }
    __syncthreads();
    const uint32_t per_block = uint32_t(p.per_warp * kSortWarps);
    for (int64_t i0 = begin; i0 < end; i0 += 32 * kSortPer) {
        uint32_t key[kSortPer], row[kSortPer];
#pragma unroll
        for (int k = 0; k < kSortPer; ++k) {
            const int64_t i = i0 + k * 32 + lane;
            key[k] = i < end ? key_at(p, i) : 0u;
            row[k] = p.tokens ? uint32_t(i) : i < end ? p.rows[i] : 0u;
        }
#pragma unroll
        for (int k = 0; k < kSortPer; ++k) {
            const bool live = i0 + k * 32 + lane < end;
            const uint32_t to = take_place(place, (key[k] >> p.shift) & uint32_t(mask), live, lane);
            if (!live) continue;
            p.keys_out[to] = key[k];
            p.rows_out[to] = row[k];
            if (p.next_counts) atomicAdd(&p.next_counts[int64_t(to / per_block) * digits + ((key[k] >> (p.shift + p.bits)) & mask)], 1u);
        }
    }
}

// ---- adding the rows -------------------------------------------------------------------------------------

struct SumParams {
    const void *d_out;
    void *d_table;
    const uint32_t *keys, *rows;       // sorted; keys of `vocab` at the end stand for no token
    float *partial;                    // [chunks, 2, width]: sums of a chunk's first and last run where they go on outside
    int64_t n, vocab, d_out_stride, d_table_stride;
    int32_t width, table_type, accumulate;
    int32_t chunk, chunks;             // sorted positions that one group of threads adds up
    int32_t lanes, tiles;              // threads of a group, parts of a row
    int32_t join_lanes;                // the same where partial sums are joined
    int32_t sum_blocks;
    float scale;
};

constexpr int kSumThreads = 128;
constexpr int kRing = 8;               // rows that a thread has under way

template <bool VEC>
__device__ __forceinline__ void write_row(const SumParams &p, uint32_t token, const float (&s)[8], int lane, int lanes, int first)
{
    const int64_t at = int64_t(token) * p.d_table_stride + first;
    void *to = p.table_type == QSR_F32 ? static_cast<void *>(static_cast<float *>(p.d_table) + at) : static_cast<void *>(static_cast<uint16_t *>(p.d_table) + at);
    const int width = p.width - first;
    float v[8];
    if (p.accumulate) {
        Raw8 r;
        fetch<VEC>(r, to, lane, lanes, 0, width, p.table_type);
        widen8(v, r, p.table_type);
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = fmaf(s[j], p.scale, v[j]);
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = s[j] * p.scale;
    }
    put<VEC>(to, v, lane, lanes, 0, width, p.table_type);
}

// The gradient of tokens that do not occur: a warp looks up 32 of them in the sorted keys and zeroes what it does not find.
template <bool VEC>
__device__ void clear_rows(const SumParams &p, int64_t first)
{
    const int lane = threadIdx.x & 31;
    const int64_t token = first + lane;
    bool absent = false;
    if (token < p.vocab) {
        int64_t lo = 0, hi = p.n;
        while (lo < hi) {
            const int64_t mid = (lo + hi) >> 1;
            if (int64_t(p.keys[mid]) < token) lo = mid + 1;
            else hi = mid;
        }
        absent = lo == p.n || int64_t(p.keys[lo]) != token;
    }
    const float zero[8] = {0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f};
    for (uint32_t left = __ballot_sync(0xffffffffu, absent); left; left &= left - 1) {
        const int64_t at = (first + __ffs(int(left)) - 1) * p.d_table_stride;
        void *to = p.table_type == QSR_F32 ? static_cast<void *>(static_cast<float *>(p.d_table) + at) : static_cast<void *>(static_cast<uint16_t *>(p.d_table) + at);
        for (int k = 0; column<VEC>(lane, 32, k, 0) < p.width; ++k) put<VEC>(to, zero, lane, 32, k, p.width, p.table_type);
    }
}

__device__ __forceinline__ void copy_async(uint32_t to, const void *from, int bytes)       // of 16; the rest reads as zeros
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(to), "l"(from), "r"(bytes) : "memory");
}

// A thread's rows on their way: kRing of them by asynchronous copies into its own slots of shared memory (aligned rows), which needs
// no registers for them and no loop that is written out; otherwise one, in registers.
template <typename T, bool VEC>
struct Ring {
    static constexpr int BYTES = 8 * int(sizeof(T)), SHARED = VEC ? kRing * kSumThreads * BYTES : 16;
    uint32_t slots;
    int left;                                        // columns from this thread's first one on
    Raw8 next;
    __device__ __forceinline__ Ring(char *shared, int left_) : slots(uint32_t(__cvta_generic_to_shared(shared)) + threadIdx.x * 16), left(left_) {}
    // row: this thread's first column of it (VEC), or the group's first column; NULL: nothing
    __device__ __forceinline__ void issue(int slot, const T *row, int lane, int lanes)
    {
        if (VEC) {
            if (row && left > 0) {
                const uint32_t to = slots + slot * (kSumThreads * BYTES);
#pragma unroll
                for (int h = 0; h < BYTES / 16; ++h) {
                    const int n = max(0, min(16, (left - h * (16 / int(sizeof(T)))) * int(sizeof(T))));
                    copy_async(to + h * (kSumThreads * 16), row + (n > 0 ? h * (16 / int(sizeof(T))) : 0), n);
                }
            }
            asm volatile("cp.async.commit_group;" ::: "memory");
        } else fetch<false>(next, row, lane, lanes, 0, row ? left : 0, Kind<T>::type);
    }
    __device__ __forceinline__ void take(float (&x)[8], int slot)
    {
        if (!VEC) {
            widen8(x, next, Kind<T>::type);
            return;
        }
        asm volatile("cp.async.wait_group %0;" ::"n"(kRing - 1) : "memory");
        Raw8 r;
        const uint32_t from = slots + slot * (kSumThreads * BYTES);
#pragma unroll
        for (int h = 0; h < BYTES / 16; ++h)
            asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(r.w[4 * h]), "=r"(r.w[4 * h + 1]), "=r"(r.w[4 * h + 2]), "=r"(r.w[4 * h + 3])
                         : "r"(from + h * (kSumThreads * 16)) : "memory");
        widen8(x, r, Kind<T>::type);
    }
};

// A group of threads adds the rows of one chunk of sorted positions, run by run; the first blocks.  The others clear rows.  Bound by memory: 65536 x 1024
// bf16 into 50001 fp32 rows, 339 MB, 70 us (4.8 TB/s).
template <typename T, bool VEC>
__global__ void __launch_bounds__(kSumThreads) sum_kernel(const __grid_constant__ SumParams p)
{
    __shared__ __align__(16) char ring_memory[Ring<T, VEC>::SHARED];
    wait_for_launch_before();
    let_next_launch_start();
    if (int(blockIdx.x) >= p.sum_blocks) {
        const int64_t first = (int64_t(int(blockIdx.x) - p.sum_blocks) * (kSumThreads / 32) + (threadIdx.x >> 5)) * 32;
        if (first < p.vocab) clear_rows<VEC>(p, first);
        return;
    }
    const int lane = int(threadIdx.x) & (p.lanes - 1);
    const int64_t unit = int64_t(blockIdx.x) * (kSumThreads / p.lanes) + int(threadIdx.x) / p.lanes;
    const int64_t c = unit / p.tiles;
    if (c >= p.chunks) return;
    const int first = int(unit - c * p.tiles) * p.lanes * 8, width = p.width - first;
    const int64_t begin = c * p.chunk;
    const int count = int(min(p.n - begin, int64_t(p.chunk)));
    const uint32_t none = uint32_t(p.vocab), *keys = p.keys + begin, *rows = p.rows + begin;
    uint32_t token = keys[0];
    if (token == none) return;
    bool whole = begin == 0 || keys[-1] != token;               // the run begins in this chunk
    const int mine = VEC ? lane * 8 : 0;
    Ring<T, VEC> ring(ring_memory, width - mine);
    const T *base = static_cast<const T *>(p.d_out) + first + mine;
    const auto issue = [&](int i) { ring.issue(i & (kRing - 1), i < count ? base + int64_t(rows[i]) * p.d_out_stride : nullptr, lane, p.lanes); };
    constexpr int AHEAD = VEC ? kRing : 1;
    for (int i = 0; i < AHEAD; ++i) issue(i);
    float s[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) s[j] = 0.0f;
    float *part = p.partial + c * 2 * p.width + first;
    const auto leave = [&](int slot) {                          // -1: the run lies in this chunk alone
        if (slot < 0) {
            write_row<VEC>(p, token, s, lane, p.lanes, first);
            return;
        }
        float *to = part + int64_t(slot) * p.width;
        if (VEC && p.width % 8 == 0) {
            if (lane * 8 < width) store8(to, lane * 8, s, QSR_F32);
            return;
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int col = column<VEC>(lane, p.lanes, 0, j);
            if (col < width) to[col] = s[j];
        }
    };
    for (int i = 0; i < count; ++i) {
        const uint32_t key = keys[i];
        if (key != token) {
            leave(whole ? -1 : 0);
            token = key;
            whole = true;
            if (key == none) break;
#pragma unroll
            for (int j = 0; j < 8; ++j) s[j] = 0.0f;
        }
        float x[8];
        ring.take(x, i & (kRing - 1));
#pragma unroll
        for (int j = 0; j < 8; ++j) s[j] += x[j];
        issue(i + AHEAD);
    }
    asm volatile("cp.async.wait_all;" ::: "memory");
    if (token == none) return;
    const bool goes_on = begin + count < p.n && keys[count] == token;
    leave(!whole ? 0 : goes_on ? 1 : -1);
}

// Runs over several chunks: the block of the chunk that a run begins in adds up its partial sums, each of `ways` groups of threads those
// of every ways-th chunk behind it, and then the groups' sums in their order.  15 us in the same case, of which the search for what is to be
// joined runs beside the sums.
constexpr int kJoinThreads = 512;
template <bool VEC>
__global__ void __launch_bounds__(kJoinThreads) join_kernel(const __grid_constant__ SumParams p)
{
    __shared__ float shared[8][kJoinThreads];
    // The sorted keys are those of the launch before the one before, which had ended before that one let this one start: what there is
    // to join is found out while the sums are still being taken.  They are read from the second-level cache, where that launch left them.
    // The first block waits also where it has nothing to join: a launch none of whose blocks waits may end before the sums are written, and
    // whatever is ordered behind this launch alone (the next node of a graph, say) would not find them.  The others need not: they would
    // stand in the sums' way (131072 x 128 bf16 of 1000 tokens 48 us instead of 44).
    const int64_t c = int64_t(blockIdx.x), begin = c * p.chunk, end = begin + p.chunk;
    const uint32_t none = uint32_t(p.vocab), token = end < p.n ? __ldcg(p.keys + end - 1) : none;
    if (token == none || __ldcg(p.keys + end) != token || (begin > 0 && __ldcg(p.keys + begin) == token && __ldcg(p.keys + begin - 1) == token)) {
        if (blockIdx.x == 0) wait_for_launch_before();
        return;
    }
    const int lanes = p.join_lanes, ways = kJoinThreads / lanes, lane = int(threadIdx.x) & (lanes - 1), way = int(threadIdx.x) / lanes;
    const int first = int(blockIdx.y) * lanes * 8, width = p.width - first, col = column<VEC>(lane, lanes, 0, 0);
    int64_t lo = c;                              // the last chunk that begins with this token; they follow one another
    for (int same = 32; same == 32; lo += same) {
        const int64_t k = lo + 1 + (threadIdx.x & 31);
        same = __popc(__ballot_sync(0xffffffffu, k < p.chunks && __ldcg(p.keys + k * p.chunk) == token));
    }
    wait_for_launch_before();
    float s[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) s[j] = 0.0f;
    const bool aligned = VEC && p.width % 8 == 0;
    const auto load = [&](Raw8 &r, int64_t chunk, int slot) {
        const float *part = p.partial + (chunk * 2 + slot) * p.width + first;
        if (aligned && col < width) load32(r, part + col);
        else
#pragma unroll
            for (int j = 0; j < 8; ++j) r.w[j] = column<VEC>(lane, lanes, 0, j) < width ? __float_as_uint(part[column<VEC>(lane, lanes, 0, j)]) : 0u;
    };
    const auto add = [&](const Raw8 &r) {
#pragma unroll
        for (int j = 0; j < 8; ++j) s[j] += __uint_as_float(r.w[j]);
    };
    if (way == 0) {
        Raw8 r;
        load(r, c, 1);
        add(r);
    }
    for (int64_t k = c + 1 + way; k <= lo; k += 4 * ways) {
        Raw8 r[4];
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (k + i * ways <= lo) load(r[i], k + i * ways, 0);
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (k + i * ways <= lo) add(r[i]);
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) shared[j][threadIdx.x] = s[j];
    __syncthreads();
    if (way) return;
    for (int w = 1; w < ways; ++w)
#pragma unroll
        for (int j = 0; j < 8; ++j) s[j] += shared[j][w * lanes + lane];
    if (col < width) write_row<VEC>(p, token, s, lane, lanes, first);
}

// ---- few rows --------------------------------------------------------------------------------------------

// All in one launch, since launches and not bytes are what few rows cost.  A block has every 2^stride-th token (neighbours are often frequent
// together) and up to 64 columns: it picks the rows of its tokens out of all rows in their order, sorts them (stable, a digit at a time, in
// shared memory), and adds them.  A group of threads takes a token; the rows of one that occurs often are shared by all groups, whose
// sums are added in their order.  2048 rows of 128 bf16 numbers, 1000 tokens, a quarter of the rows with the five most frequent: 7.0 us in a graph, of
// which 2 are an empty launch's; what is left is the chain load, sort, load, add.
struct FewParams {
    SumParams sum;
    const int64_t *tokens;
    int32_t stride, passes, bits;      // stride: log2 of the blocks that share the tokens; of a token's number in its block, a pass's bits
};
constexpr int kFew = 16384, kFewThreads = 256, kFewWarps = kFewThreads / 32;
constexpr int kFewBlocks = 384;        // 768 were slower with few columns (9.5 us for 6.4) and with many (49 for 43)
constexpr int kFewLanes = 8;           // threads of a group, at most: 64 columns
constexpr int kFewRange = 8192;        // tokens of a block, at most
constexpr int kFewDigit = 7;           // bits
constexpr int kFewTokens = 8;          // of a thread at a time
constexpr int kOften = 16;             // rows from which on a token is everybody's: 32 take 8.0 us instead of 7.0 above, and 31 instead of
                                       // 36 for 4096 rows of 4096

// Adds rows list[first], list[first + step], ... of `count` to s.
template <typename T, bool VEC, int AHEAD>
__device__ __forceinline__ void add_rows(float (&s)[8], const SumParams &p, const T *base, const uint16_t *list, int first, int step, int count, int lane, int lanes, int width)
{
    for (int i = first; i < count; i += AHEAD * step) {
        Raw8 r[AHEAD];
#pragma unroll
        for (int k = 0; k < AHEAD; ++k)
            if (i + k * step < count) fetch<VEC>(r[k], base + int64_t(list[i + k * step]) * p.d_out_stride, lane, lanes, 0, width, Kind<T>::type);
#pragma unroll
        for (int k = 0; k < AHEAD; ++k) {
            if (i + k * step >= count) break;
            float x[8];
            widen8(x, r[k], Kind<T>::type);
#pragma unroll
            for (int j = 0; j < 8; ++j) s[j] += x[j];
        }
    }
}

// The first of positions [from, to) whose key is not `key`, or `to`; those with it come first.
__device__ __forceinline__ int end_of(const uint16_t *keys, uint32_t key, int from, int to)
{
    while (from < to) {
        const int mid = (from + to) >> 1;
        if (keys[mid] == key) from = mid + 1;
        else to = mid;
    }
    return from;
}

template <typename T, bool VEC>
__global__ void __launch_bounds__(kFewThreads) few_kernel(const __grid_constant__ FewParams f)
{
    extern __shared__ uint16_t memory[];                         // two sets of [n] keys and [n] rows, which are below 2^16
    __shared__ uint32_t scratch[kFewWarps], found[kFewWarps], often[kFew / kOften], n_often, n_runs;
    __shared__ uint32_t present[kFewRange / 32], places[kFewWarps << kFewDigit];
    __shared__ float shared[8][kFewWarps][kFewLanes];
    const SumParams &p = f.sum;
    const int n = int(p.n), warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t vocab = uint32_t(p.vocab), self = blockIdx.x, others = (1u << f.stride) - 1u;
    const int range = self < vocab ? int(((vocab - 1u - self) >> f.stride) + 1u) : 0;       // tokens self, self + 2^stride, ...
    uint16_t *keys = memory, *rows = keys + n, *keys_to = rows + n, *rows_to = keys_to + n;
    for (int i = threadIdx.x; i < (range + 31) / 32; i += kFewThreads) present[i] = 0;
    if (threadIdx.x == 0) n_often = n_runs = 0;
    __syncthreads();
    // a warp's share of the rows: those with the block's tokens to the front of its share, then all shares together
    const int per_warp = ((n + kFewThreads - 1) / kFewThreads) * 32, from = warp * per_warp, to = min(n, from + per_warp);
    int here = 0;
    for (int i0 = from; i0 < to; i0 += 32 * kFewTokens) {
        uint32_t token[kFewTokens];
#pragma unroll
        for (int k = 0; k < kFewTokens; ++k) {
            const int i = i0 + k * 32 + lane;
            token[k] = i < to ? key_of(f.tokens[i], vocab) : vocab;
        }
#pragma unroll
        for (int k = 0; k < kFewTokens; ++k) {
            const uint32_t t = token[k] >> f.stride;
            const bool mine = token[k] < vocab && (token[k] & others) == self;
            const uint32_t all = __ballot_sync(0xffffffffu, mine);
            if (mine) {
                const int at = from + here + __popc(all & ((1u << lane) - 1u));
                keys_to[at] = uint16_t(t);
                rows_to[at] = uint16_t(i0 + k * 32 + lane);
                if (!p.accumulate && !(present[t >> 5] >> (t & 31) & 1u)) atomicOr(&present[t >> 5], 1u << (t & 31));
            }
            here += __popc(all);
        }
    }
    if (lane == 0) found[warp] = uint32_t(here);
    __syncthreads();
    int before = 0, count = 0;
#pragma unroll
    for (int w = 0; w < kFewWarps; ++w) {
        before += w < warp ? int(found[w]) : 0;
        count += int(found[w]);
    }
    for (int i = lane; i < here; i += 32) {
        keys[before + i] = keys_to[from + i];
        rows[before + i] = rows_to[from + i];
    }
    __syncthreads();
    if (count > 1) {
        const int digits = 1 << f.bits, mask = digits - 1, share = ((count + kFewThreads - 1) / kFewThreads) * 32, b = warp * share, e = min(count, b + share);
        uint32_t *place = places + warp * digits;
        for (int pass = 0; pass < f.passes; ++pass) {
            const int shift = pass * f.bits;
            for (int i = threadIdx.x; i < kFewWarps * digits; i += kFewThreads) places[i] = 0;
            __syncthreads();
            for (int i0 = b; i0 < e; i0 += 32) {                 // one addition for equal digits: a frequent token may be all there is
                const int digit = i0 + lane < e ? int((keys[i0 + lane] >> shift) & uint32_t(mask)) : digits;
                const uint32_t same = __match_any_sync(0xffffffffu, digit);
                if (digit < digits && lane == __ffs(int(same)) - 1) place[digit] += uint32_t(__popc(same));
                __syncwarp();
            }
            __syncthreads();
            uint32_t total = 0;
            if (int(threadIdx.x) < digits)
#pragma unroll
                for (int w = 0; w < kFewWarps; ++w) total += places[w * digits + threadIdx.x];
            uint32_t at = exclusive_scan<kFewThreads>(total, scratch);
            if (int(threadIdx.x) < digits)
#pragma unroll
                for (int w = 0; w < kFewWarps; ++w) {
                    const uint32_t c = places[w * digits + threadIdx.x];
                    places[w * digits + threadIdx.x] = at;
                    at += c;
                }
            __syncthreads();
            for (int i0 = b; i0 < e; i0 += 32) {
                const bool live = i0 + lane < e;
                const uint32_t k = live ? keys[i0 + lane] : 0u, r = live ? rows[i0 + lane] : 0u, place_of = take_place(place, (k >> shift) & uint32_t(mask), live, lane);
                if (live) {
                    keys_to[place_of] = uint16_t(k);
                    rows_to[place_of] = uint16_t(r);
                }
            }
            __syncthreads();
            uint16_t *const k = keys, *const r = rows;
            keys = keys_to; rows = rows_to;
            keys_to = k; rows_to = r;
        }
    }
    const int lanes = p.lanes, groups = kFewThreads / lanes, group = int(threadIdx.x) / lanes, l = int(threadIdx.x) & (lanes - 1);
    const int first = int(blockIdx.y) * lanes * 8, width = p.width - first;
    const T *base = static_cast<const T *>(p.d_out) + first;
    uint16_t *runs = keys_to;                                    // where a token's rows begin, in any order
    for (int i = threadIdx.x; i < count; i += kFewThreads)
        if (i == 0 || keys[i - 1] != keys[i]) runs[atomicAdd(&n_runs, 1u)] = uint16_t(i);
    __syncthreads();
    for (int k = group; k < int(n_runs); k += groups) {
        const int i = int(runs[k]);
        const uint32_t key = keys[i];
        const int end = end_of(keys, key, i + 1, min(count, i + kOften));
        if (end == i + kOften) {                                 // kOften rows or more
            if (l == 0) often[atomicAdd(&n_often, 1u)] = uint32_t(i);
            continue;
        }
        float s[8] = {0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f};
        add_rows<T, VEC, 4>(s, p, base, rows + i, 0, 1, end - i, l, lanes, width);
        write_row<VEC>(p, (key << f.stride | self), s, l, lanes, first);
    }
    if (!p.accumulate) {
        const float zero[8] = {0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f};
        for (int t = group; t < range; t += groups)
            if (!(present[t >> 5] >> (t & 31) & 1u)) write_row<VEC>(p, uint32_t(t) << f.stride | self, zero, l, lanes, first);
    }
    __syncthreads();
    for (uint32_t o = 0; o < n_often; ++o) {
        const int i = int(often[o]);
        const uint32_t key = keys[i];
        float s[8] = {0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f};
        add_rows<T, VEC, 8>(s, p, base, rows + i, group, groups, end_of(keys, key, i + kOften, count) - i, l, lanes, width);
        for (int d = lanes; d < 32; d *= 2)
#pragma unroll
            for (int j = 0; j < 8; ++j) s[j] += __shfl_xor_sync(0xffffffffu, s[j], d);
        __syncthreads();
        if (lane < lanes)
#pragma unroll
            for (int j = 0; j < 8; ++j) shared[j][warp][l] = s[j];
        __syncthreads();
        if (group == 0) {
#pragma unroll
            for (int w = 1; w < kFewWarps; ++w)
#pragma unroll
                for (int j = 0; j < 8; ++j) s[j] += shared[j][w][l];
            write_row<VEC>(p, (key << f.stride | self), s, l, lanes, first);
        }
    }
}

// ---- host side -------------------------------------------------------------------------------------------

constexpr int64_t kMaxWidth = int64_t(1) << 20;

struct Layout { int64_t keys[2], rows[2], counts, partial, bytes; int32_t chunk, chunks, blocks, passes, bits; int64_t per_warp; };

// One launch for all, in which every block reads all tokens, instead of sorting them in launches of their own: 2048 x 128 (above) 7.0 us
// against 17.0, 64 rows 4.4 against 12.2, 4096 x 4096 of 1000 tokens 36 against 49.  Up to kFew rows where few parts of a row read them: 8192 x
// 128 14 against 20, 16384 x 15 of 57048 tokens 27 against 46; but 8192 x 1024 32 against 27, 16384 x 128 24 against 22.  The other way
// too where most of so many rows have one token, whose block then has most of the work: 8192 x 128 of one token 43 against 22.
bool is_few(int64_t rows, int64_t vocab, int64_t width)
{
    return (rows <= kFew / 4 || rows * ((width + 63) / 64) <= kFew) && vocab <= int64_t(1) << 21;
}

Layout layout_of(int64_t rows, int64_t vocab, int64_t width)
{
    Layout l = {};
    if (is_few(rows, vocab, width)) {
        l.bytes = 256;                                           // none is used
        return l;
    }
    // chunks: short enough that every multiprocessor has several, at most 32 (partial sums: two for a chunk's rows)
    l.chunk = 8;
    while (l.chunk < 32 && rows / l.chunk > 148 * 8) l.chunk *= 2;
    l.chunks = int32_t((rows + l.chunk - 1) / l.chunk);
    int bits = 1;
    while ((vocab >> bits) != 0) bits++;                        // of `vocab` itself, which stands for no token
    l.passes = (bits + kMaxDigit - 1) / kMaxDigit;
    l.bits = (bits + l.passes - 1) / l.passes;
    l.blocks = int32_t(std::min<int64_t>(std::max<int64_t>(1, (rows + 2047) / 2048), kMaxSortBlocks));
    l.per_warp = std::max<int64_t>(32, ((rows + l.blocks - 1) / l.blocks + kSortThreads - 1) / kSortThreads * 32);
    l.blocks = int32_t(std::max<int64_t>(1, (rows + l.per_warp * kSortWarps - 1) / (l.per_warp * kSortWarps)));
    int64_t at = 0;
    auto take = [&at](int64_t bytes) { const int64_t here = at; at += (bytes + 255) / 256 * 256; return here; };
    for (int i = 0; i < 2; ++i) {
        l.keys[i] = take(rows * 4);
        l.rows[i] = take(rows * 4);
    }
    l.counts = take(int64_t(l.passes) * l.blocks * (int64_t(4) << l.bits));
    l.partial = take(int64_t(l.chunks) * 2 * width * 4);
    l.bytes = std::max<int64_t>(at, 256);
    return l;
}

template <typename T, bool VEC>
int launch_lookup(const LookupParams &p, cudaStream_t st)
{
    const int64_t groups = 256 / p.lanes, blocks = (p.rows * p.parts + groups - 1) / groups;
    if (blocks > 0x7fffffff) return int(cudaErrorInvalidConfiguration);
    lookup_kernel<T, VEC><<<unsigned(blocks), 256, 0, st>>>(p);
    return int(cudaGetLastError());
}

// A launch that may start before the one before it on the stream has ended (its kernel waits for that).
template <typename P>
int launch_close(void (*kernel)(P), dim3 grid, unsigned threads, size_t shared, const P &p, cudaStream_t st)
{
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = dim3(threads);
    cfg.dynamicSmemBytes = shared;
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return int(cudaLaunchKernelEx(&cfg, kernel, p));
}

template <typename T>
int launch_sums(SumParams p, bool vec, int64_t sum_blocks, int64_t clear_blocks, cudaStream_t st)
{
    if (sum_blocks + clear_blocks > 0x7fffffff) return int(cudaErrorInvalidConfiguration);
    p.sum_blocks = int32_t(sum_blocks);
    return launch_close(vec ? sum_kernel<T, true> : sum_kernel<T, false>, dim3(unsigned(sum_blocks + clear_blocks)), kSumThreads, 0, p, st);
}

int launch_sort(SortParams &s, const Layout &l, uint32_t *const *keys, uint32_t *const *rows, cudaStream_t st)
{
    const int64_t counts = int64_t(l.blocks) << l.bits;
    uint32_t *const first = s.counts;
    s.next_counts = first + counts;
    count_kernel<<<unsigned(l.blocks), kSortThreads, 0, st>>>(s);
    if (cudaError_t err = cudaGetLastError()) return int(err);
    const size_t shared = size_t(kSortWarps) * (size_t(4) << l.bits);
    static std::atomic<uint64_t> raised{0};
    if (int err = allow_shared(reinterpret_cast<const void *>(place_kernel), kSortWarps * (4 << kMaxDigit), raised)) return err;
    for (int pass = 0; pass < l.passes; ++pass) {
        s.shift = pass * l.bits;
        s.counts = first + pass * counts;
        s.next_counts = pass + 1 < l.passes ? s.counts + counts : nullptr;
        s.keys_out = keys[pass & 1]; s.rows_out = rows[pass & 1];
        if (int err = launch_close(place_kernel, dim3(unsigned(l.blocks)), kSortThreads, shared, s, st)) return err;
        s.tokens = nullptr;
        s.keys = s.keys_out; s.rows = s.rows_out;
    }
    return 0;
}

template <typename T, bool VEC>
int launch_few(const FewParams &f, unsigned ranges, cudaStream_t st)
{
    const size_t shared = 4 * size_t(f.sum.n) * 2;
    static std::atomic<uint64_t> raised{0};
    if (int err = allow_shared(reinterpret_cast<const void *>(few_kernel<T, VEC>), 4 * kFew * 2, raised)) return err;
    few_kernel<T, VEC><<<dim3(ranges, unsigned(f.sum.tiles)), kFewThreads, shared, st>>>(f);
    return int(cudaGetLastError());
}

int launch_grad(const qsr_embed_args &a, bool vec, cudaStream_t st)
{
    SumParams p = {};
    p.d_out = a.out; p.d_table = a.table;
    p.n = a.rows; p.vocab = a.vocab; p.d_out_stride = a.out_stride; p.d_table_stride = a.table_stride;
    p.width = int32_t(a.width); p.table_type = a.table_type; p.accumulate = a.accumulate;
    p.scale = float(a.scale);
    const int granules = int((a.width + 7) / 8);
    if (is_few(a.rows, a.vocab, a.width)) {
        if (a.rows == 0 && a.accumulate) return 0;
        p.lanes = std::min(kFewLanes, power_of_two(granules));
        p.tiles = (granules + p.lanes - 1) / p.lanes;
        FewParams f = {p, a.tokens, 0, 0, 0};
        while ((int64_t(2) << f.stride) * p.tiles <= kFewBlocks && (int64_t(1) << f.stride) < a.vocab) f.stride++;
        while ((a.vocab - 1) >> f.stride >= kFewRange) f.stride++;
        int bits = 0;
        while (((a.vocab - 1) >> f.stride) >> bits) bits++;
        f.passes = (bits + kFewDigit - 1) / kFewDigit;
        f.bits = f.passes ? (bits + f.passes - 1) / f.passes : 0;
        const unsigned n = 1u << f.stride;
        if (a.out_type == QSR_F32) return vec ? launch_few<float, true>(f, n, st) : launch_few<float, false>(f, n, st);
        if (a.out_type == QSR_BF16) return vec ? launch_few<__nv_bfloat16, true>(f, n, st) : launch_few<__nv_bfloat16, false>(f, n, st);
        return vec ? launch_few<__half, true>(f, n, st) : launch_few<__half, false>(f, n, st);
    }
    const Layout l = layout_of(a.rows, a.vocab, a.width);
    char *ws = static_cast<char *>(a.workspace);
    uint32_t *keys[2], *rows[2];
    for (int i = 0; i < 2; ++i) {
        keys[i] = reinterpret_cast<uint32_t *>(ws + l.keys[i]);
        rows[i] = reinterpret_cast<uint32_t *>(ws + l.rows[i]);
    }
    SortParams s = {};
    s.tokens = a.tokens;
    s.counts = reinterpret_cast<uint32_t *>(ws + l.counts);
    s.n = a.rows; s.per_warp = l.per_warp; s.vocab = uint32_t(a.vocab); s.bits = l.bits; s.passes = l.passes;
    if (a.rows > 0)
        if (int err = launch_sort(s, l, keys, rows, st)) return err;
    p.keys = s.keys; p.rows = s.rows;
    p.partial = reinterpret_cast<float *>(ws + l.partial);
    p.chunk = l.chunk; p.chunks = l.chunks;
    p.lanes = std::min(kSumThreads, power_of_two(granules));
    p.tiles = (granules + p.lanes - 1) / p.lanes;
    const int64_t groups = kSumThreads / p.lanes, sum_blocks = (int64_t(l.chunks) * p.tiles + groups - 1) / groups;
    const int64_t clear_blocks = a.accumulate ? 0 : (a.vocab + kSumThreads - 1) / kSumThreads;
    if (sum_blocks + clear_blocks > 0) {
        const int err = a.out_type == QSR_F32 ? launch_sums<float>(p, vec, sum_blocks, clear_blocks, st)
                        : a.out_type == QSR_BF16 ? launch_sums<__nv_bfloat16>(p, vec, sum_blocks, clear_blocks, st)
                                                 : launch_sums<__half>(p, vec, sum_blocks, clear_blocks, st);
        if (err) return err;
    }
    if (l.chunks < 2) return 0;
    p.join_lanes = p.lanes;
    const dim3 grid(unsigned(l.chunks), unsigned((granules + p.join_lanes - 1) / p.join_lanes));
    return launch_close(vec ? join_kernel<true> : join_kernel<false>, grid, kJoinThreads, 0, p, st);
}

int shared_checks(const qsr_embed_args *a)
{
    if (!a) return QSR_EINVAL;
    const int te = type_bytes(a->table_type), oe = type_bytes(a->out_type);
    if (!te || !oe || !std::isfinite(float(a->scale)) || (a->accumulate != 0 && a->accumulate != 1) || a->reserved != 0) return QSR_EINVAL;
    if (a->rows < 0 || a->rows > 0x7fffffff || a->vocab < 1 || a->vocab > 0x7ffffffe || a->width < 1 || a->width > kMaxWidth ||
        a->table_stride < a->width || a->out_stride < a->width)
        return QSR_ERANGE;
    if (!aligned_to(a->table, unsigned(te)) || !aligned_to(a->out, unsigned(oe)) || !aligned_to(a->tokens, 8)) return QSR_EALIGN;
    if (!a->table || (a->rows > 0 && (!a->tokens || !a->out))) return QSR_EINVAL;
    if (a->rows > 0 && share_bytes(a->table, a->table_stride, a->width, te, a->vocab, a->out, a->out_stride, a->width, oe, a->rows)) return QSR_EINVAL;
    return QSR_OK;
}

bool vectors(const qsr_embed_args &a)
{
    return rows_aligned(a.table, a.table_stride, a.vocab, type_bytes(a.table_type)) && rows_aligned(a.out, a.out_stride, a.rows, type_bytes(a.out_type));
}

}  // namespace

}  // namespace qsr

extern "C" {

int qsr_embed(const qsr_embed_args *a, void *cuda_stream)
{
    using namespace qsr;
    if (int rc = shared_checks(a)) return rc;
    if (a->rows == 0) return QSR_OK;
    LookupParams p = {};
    p.table = a->table; p.tokens = a->tokens; p.out = a->out;
    p.rows = a->rows; p.vocab = a->vocab; p.table_stride = a->table_stride; p.out_stride = a->out_stride;
    p.width = int32_t(a->width); p.out_type = a->out_type;
    const int granules = int((a->width + 7) / 8);
    p.lanes = std::min(32, power_of_two((granules + kHeld - 1) / kHeld));
    p.parts = (granules + p.lanes * kHeld - 1) / (p.lanes * kHeld);
    p.scale = float(a->scale);
    const bool vec = vectors(*a);
    const cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    int err;
    if (a->table_type == QSR_F32) err = vec ? launch_lookup<float, true>(p, st) : launch_lookup<float, false>(p, st);
    else if (a->table_type == QSR_BF16) err = vec ? launch_lookup<__nv_bfloat16, true>(p, st) : launch_lookup<__nv_bfloat16, false>(p, st);
    else err = vec ? launch_lookup<__half, true>(p, st) : launch_lookup<__half, false>(p, st);
    return launch_status(err);
}

int64_t qsr_embed_workspace_bytes(int64_t rows, int64_t vocab, int64_t width)
{
    if (rows < 0 || rows > 0x7fffffff || vocab < 1 || vocab > 0x7ffffffe || width < 1 || width > qsr::kMaxWidth) return QSR_ERANGE;
    return qsr::layout_of(rows, vocab, width).bytes;
}

int qsr_embed_grad(const qsr_embed_args *a, void *cuda_stream)
{
    using namespace qsr;
    if (int rc = shared_checks(a)) return rc;
    if (!a->workspace) return QSR_EINVAL;
    if (!aligned_to(a->workspace, 256)) return QSR_EALIGN;
    if (a->workspace_bytes < qsr_embed_workspace_bytes(a->rows, a->vocab, a->width)) return QSR_ERANGE;
    return launch_status(launch_grad(*a, vectors(*a), static_cast<cudaStream_t>(cuda_stream)));
}

}  // extern "C"
