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

// A group of `lanes` threads copies a part of one row: all its loads first, then the stores.
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

// A stable radix sort of (token, row), lowest digits first.  Each pass takes two launches: the blocks count their digits, then every
// block finds its places from all blocks' counts.  Tokens that are not in the vocabulary sort behind it.
constexpr int kMaxDigit = 10;          // bits
constexpr int kSortThreads = 256, kSortWarps = kSortThreads / 32;
constexpr int kMaxSortBlocks = 256;

struct SortParams {
    const int64_t *tokens;             // first pass; otherwise keys and rows
    const uint32_t *keys, *rows;
    uint32_t *keys_out, *rows_out;
    uint32_t *counts;                  // [blocks, 1 << bits]
    int64_t n, per_warp;               // per_warp: a multiple of 32
    uint32_t vocab;
    int32_t shift, bits;
};

__device__ __forceinline__ uint32_t key_at(const SortParams &p, int64_t i)
{
    if (!p.tokens) return p.keys[i];
    const int64_t t = p.tokens[i];
    return t >= 0 && t < int64_t(p.vocab) ? uint32_t(t) : p.vocab;
}

__global__ void __launch_bounds__(kSortThreads) count_kernel(const __grid_constant__ SortParams p)
{
    __shared__ uint32_t count[1 << kMaxDigit];
    const int digits = 1 << p.bits;
    for (int d = threadIdx.x; d < digits; d += kSortThreads) count[d] = 0;
    __syncthreads();
    const int64_t begin = int64_t(blockIdx.x) * p.per_warp * kSortWarps, end = min(p.n, begin + p.per_warp * kSortWarps);
    for (int64_t i = begin + threadIdx.x; i < end; i += kSortThreads) atomicAdd(&count[(key_at(p, i) >> p.shift) & (digits - 1)], 1u);
    __syncthreads();
    for (int d = threadIdx.x; d < digits; d += kSortThreads) p.counts[int64_t(blockIdx.x) * digits + d] = count[d];
}

// Sum over the threads before this one, of a block of kSortThreads.
__device__ __forceinline__ uint32_t exclusive_scan(uint32_t v, uint32_t *scratch)
{
    uint32_t s = v;
    for (int d = 1; d < 32; d *= 2) {
        const uint32_t u = __shfl_up_sync(0xffffffffu, s, d);
        if (int(threadIdx.x & 31) >= d) s += u;
    }
    if ((threadIdx.x & 31) == 31) scratch[threadIdx.x >> 5] = s;
    __syncthreads();
    uint32_t before = 0;
    for (int w = 0; w < int(threadIdx.x >> 5); ++w) before += scratch[w];
    return before + s - v;
}

__global__ void __launch_bounds__(kSortThreads) place_kernel(const __grid_constant__ SortParams p)
{
    __shared__ uint32_t place[kSortWarps][1 << kMaxDigit];      // next place of each digit, warp by warp
    __shared__ uint32_t scratch[kSortWarps];
    const int digits = 1 << p.bits, mask = digits - 1, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    for (int i = threadIdx.x; i < kSortWarps << kMaxDigit; i += kSortThreads) (&place[0][0])[i] = 0;
    __syncthreads();
    const int64_t begin = (int64_t(blockIdx.x) * kSortWarps + warp) * p.per_warp, end = min(p.n, begin + p.per_warp);
    for (int64_t i = begin + lane; i < end; i += 32) atomicAdd(&place[warp][(key_at(p, i) >> p.shift) & mask], 1u);

    // this thread's digits: consecutive ones, so that a scan over threads is one over digits
    constexpr int kPer = (1 << kMaxDigit) / kSortThreads;
    const int per = max(1, digits / kSortThreads), d0 = int(threadIdx.x) * per;
    uint32_t total[kPer], earlier[kPer], all = 0;
    for (int k = 0; k < kPer; ++k) {
        total[k] = earlier[k] = 0;
        if (k < per && d0 + k < digits) {
            uint32_t t = 0, e = 0;
#pragma unroll 8
            for (int b = 0; b < int(gridDim.x); ++b) {
                const uint32_t c = p.counts[int64_t(b) * digits + d0 + k];
                t += c;
                e += b < int(blockIdx.x) ? c : 0u;
            }
            total[k] = t; earlier[k] = e;
        }
        all += total[k];
    }
    uint32_t at = exclusive_scan(all, scratch);
    __syncthreads();                                            // all warps have counted
    for (int k = 0; k < kPer; ++k)
        if (k < per && d0 + k < digits) {
            uint32_t next = at + earlier[k];
            for (int w = 0; w < kSortWarps; ++w) {
                const uint32_t c = place[w][d0 + k];
                place[w][d0 + k] = next;
                next += c;
            }
            at += total[k];
        }
    __syncthreads();
    for (int64_t i0 = begin; i0 < end; i0 += 32) {
        const int64_t i = i0 + lane;
        const bool live = i < end;
        const uint32_t key = live ? key_at(p, i) : 0u, row = p.tokens ? uint32_t(i) : live ? p.rows[i] : 0u;
        const uint32_t digit = live ? (key >> p.shift) & uint32_t(mask) : 0xffffffffu;
        const uint32_t same = __match_any_sync(0xffffffffu, digit);
        const int rank = __popc(same & ((1u << lane) - 1u));
        uint32_t to = 0;
        if (live) to = place[warp][digit] + uint32_t(rank);
        __syncwarp();
        if (live && rank == 0) place[warp][digit] += uint32_t(__popc(same));
        __syncwarp();
        if (live) {
            p.keys_out[to] = key;
            p.rows_out[to] = row;
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
    int32_t sum_blocks;
    float scale;
};

constexpr int kSumThreads = 128;
constexpr int kAhead = 8;              // rows whose loads are under way together

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

// A group of threads adds the rows of one chunk of sorted positions, run by run; the first blocks.  The others clear rows.
template <typename T, bool VEC>
__global__ void __launch_bounds__(kSumThreads) sum_kernel(const __grid_constant__ SumParams p)
{
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
    const int64_t begin = c * p.chunk, end = min(p.n, begin + p.chunk);
    const uint32_t none = uint32_t(p.vocab);
    uint32_t token = p.keys[begin];
    if (token == none) return;
    bool whole = begin == 0 || p.keys[begin - 1] != token;      // the run begins in this chunk
    float s[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) s[j] = 0.0f;
    float *part = p.partial + c * 2 * p.width + first;
    auto keep = [&](int slot) {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int col = column<VEC>(lane, p.lanes, 0, j);
            if (col < width) part[int64_t(slot) * p.width + col] = s[j];
        }
    };
    for (int64_t i0 = begin; i0 < end; i0 += kAhead) {
        uint32_t key[kAhead];
        Raw8 raw[kAhead];
#pragma unroll
        for (int a = 0; a < kAhead; ++a) {
            const bool live = i0 + a < end;
            key[a] = live ? p.keys[i0 + a] : none;
            const int64_t row = live ? int64_t(p.rows[i0 + a]) : 0;
            fetch<VEC>(raw[a], static_cast<const T *>(p.d_out) + row * p.d_out_stride + first, lane, p.lanes, 0, key[a] != none ? width : 0, Kind<T>::type);
        }
#pragma unroll
        for (int a = 0; a < kAhead; ++a) {
            if (key[a] != token) {
                if (token != none) {
                    if (whole) write_row<VEC>(p, token, s, lane, p.lanes, first);
                    else keep(0);
                }
                token = key[a];
                whole = true;
#pragma unroll
                for (int j = 0; j < 8; ++j) s[j] = 0.0f;
            }
            float x[8];
            widen8(x, raw[a], Kind<T>::type);
#pragma unroll
            for (int j = 0; j < 8; ++j) s[j] += x[j];
        }
    }
    // a chunk shorter than a multiple of kAhead has met `none` above and has nothing left
    if (token == none) return;
    const bool goes_on = end < p.n && p.keys[end] == token;
    if (!whole) keep(0);
    else if (goes_on) keep(1);
    else write_row<VEC>(p, token, s, lane, p.lanes, first);
}

// Runs over several chunks: the block of the chunk that a run begins in adds up the partial sums, warp w those of chunks w,
// w + 8, ... behind it, and the warps' sums in their order.
template <bool VEC>
__global__ void __launch_bounds__(256) join_kernel(const __grid_constant__ SumParams p)
{
    __shared__ float shared[8][8][32];
    const int64_t c = int64_t(blockIdx.x), begin = c * p.chunk, end = begin + p.chunk;
    if (end >= p.n) return;
    const uint32_t token = p.keys[end - 1];
    if (token == uint32_t(p.vocab) || p.keys[end] != token || (begin > 0 && p.keys[begin] == token && p.keys[begin - 1] == token)) return;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, first = int(blockIdx.y) * 256, width = p.width - first;
    float s[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) s[j] = 0.0f;
    auto add = [&](int64_t chunk, int slot) {
        const float *part = p.partial + (chunk * 2 + slot) * p.width + first;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int col = column<VEC>(lane, 32, 0, j);
            if (col < width) s[j] += part[col];
        }
    };
    if (warp == 0) add(c, 1);
    for (int64_t k = c + 1 + warp; k < p.chunks && p.keys[k * p.chunk] == token; k += 8) add(k, 0);
#pragma unroll
    for (int j = 0; j < 8; ++j) shared[warp][j][lane] = s[j];
    __syncthreads();
    if (warp) return;
    for (int w = 1; w < 8; ++w)
#pragma unroll
        for (int j = 0; j < 8; ++j) s[j] += shared[w][j][lane];
    if (column<VEC>(lane, 32, 0, 0) < width) write_row<VEC>(p, token, s, lane, 32, first);
}

// ---- host side -------------------------------------------------------------------------------------------

constexpr int64_t kMaxWidth = int64_t(1) << 20;

struct Layout { int64_t keys[2], rows[2], counts, partial, bytes; int32_t chunk, chunks, blocks, passes, bits; int64_t per_warp; };

Layout layout_of(int64_t rows, int64_t vocab, int64_t width)
{
    Layout l = {};
    // chunks: short enough that every multiprocessor has several, at most 64 (partial sums: 1/32 of a chunk's rows)
    l.chunk = 8;
    while (l.chunk < 64 && rows / l.chunk > 148 * 8) l.chunk *= 2;
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
    l.counts = take(int64_t(l.blocks) * (int64_t(4) << l.bits));
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

template <typename T>
int launch_sums(SumParams p, bool vec, int64_t sum_blocks, int64_t clear_blocks, cudaStream_t st)
{
    if (sum_blocks + clear_blocks > 0x7fffffff) return int(cudaErrorInvalidConfiguration);
    p.sum_blocks = int32_t(sum_blocks);
    const unsigned grid = unsigned(sum_blocks + clear_blocks);
    if (vec) sum_kernel<T, true><<<grid, kSumThreads, 0, st>>>(p);
    else sum_kernel<T, false><<<grid, kSumThreads, 0, st>>>(p);
    return int(cudaGetLastError());
}

int launch_grad(const qsr_embed_args &a, bool vec, cudaStream_t st)
{
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
    s.n = a.rows; s.per_warp = l.per_warp; s.vocab = uint32_t(a.vocab); s.bits = l.bits;
    int at = 0;
    for (int pass = 0; pass < l.passes && a.rows > 0; ++pass) {
        s.shift = pass * l.bits;
        s.keys_out = keys[at]; s.rows_out = rows[at];
        count_kernel<<<unsigned(l.blocks), kSortThreads, 0, st>>>(s);
        if (cudaError_t err = cudaGetLastError()) return int(err);
        place_kernel<<<unsigned(l.blocks), kSortThreads, 0, st>>>(s);
        if (cudaError_t err = cudaGetLastError()) return int(err);
        s.tokens = nullptr;
        s.keys = keys[at]; s.rows = rows[at];
        at ^= 1;
    }
    SumParams p = {};
    p.d_out = a.out; p.d_table = a.table;
    p.keys = s.keys; p.rows = s.rows;
    p.partial = reinterpret_cast<float *>(ws + l.partial);
    p.n = a.rows; p.vocab = a.vocab; p.d_out_stride = a.out_stride; p.d_table_stride = a.table_stride;
    p.width = int32_t(a.width); p.table_type = a.table_type; p.accumulate = a.accumulate;
    p.chunk = l.chunk; p.chunks = l.chunks;
    p.scale = float(a.scale);
    const int granules = int((a.width + 7) / 8);
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
    const dim3 grid(unsigned(l.chunks), unsigned((granules + 31) / 32));
    if (vec) join_kernel<true><<<grid, 256, 0, st>>>(p);
    else join_kernel<false><<<grid, 256, 0, st>>>(p);
    return int(cudaGetLastError());
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
