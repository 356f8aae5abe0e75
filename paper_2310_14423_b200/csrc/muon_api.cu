// C ABI of the matrices stepped by their orthogonalised momentum: checks, device tables, launches.  See include/qsr.h.
#include <cuda_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>
#include <cstring>
#include <vector>

#include "checks.h"
#include "internal.h"

struct MuonLaunch { int64_t first, n; bool polynomial; };          // which tiles

struct qsr_muon {
    qsr_muon_config cfg;
    cudaStream_t stream;
    int device, multiprocessors;
    qsr::MuonParams params;                     // tables; the step's numbers are filled in by each call
    const void **grads;
    const qsr::MuonTile *tiles;
    std::vector<MuonLaunch> products;               // of a step, in their order
    const int32_t *small;                       // matrices that one block each steps
    int32_t n_small, small_blocks;
    unsigned small_columns;
    const qsr::ListTensor *sync_tensors;
    const qsr::ListChunk *sync_chunks;
    int64_t chunks, large_chunks, blocks, param_sync_chunks, all_sync_chunks;
    std::vector<qsr_matrix> host;
    bool has_grads;
    int64_t launches;
    alignas(64) unsigned char maps[256];        // two CUtensorMaps
};

namespace {

using namespace qsr;

constexpr int64_t kChunk = 16384;                                  // elements that a block adds to the momentum
constexpr int64_t kSyncChunk = int64_t(kListWarps) * 256 * kListStages;
constexpr int64_t kMaxSide = int64_t(1) << 20, kMaxShortSide = 32768;
constexpr int64_t kBlockBytes = 64 * 64 * 2;

int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

struct Sides { int64_t m, n, mb, nb; };
Sides sides_of(int64_t rows, int64_t cols)
{
    const int64_t m = std::min(rows, cols), n = std::max(rows, cols);
    return Sides{m, n, ceil_div(m, 64), ceil_div(n, 64)};
}
// Tiles of 256 rows and `width` blocks of columns: those of an m x m matrix that reach the diagonal's 256 x 256 tiles or lie above,
// and those of an r x c matrix (blocks).
int64_t half_tiles(int64_t mb, int64_t width)
{
    int64_t count = 0;
    for (int64_t q = 0; q < mb; q += width) count += q / 4 + 1;
    return count;
}
int64_t whole_tiles(int64_t rb, int64_t cb, int64_t width) { return ceil_div(rb, 4) * ceil_div(cb, width); }

// Iterations at the end whose products of X and C are saved.  X_k = P_k X with symmetric m x m matrices that are all polynomials of A:
// C' = C_last C_(last-1), and A_last = C A C.  With the last two iterations on these alone, four m x m x m products (three of them with A
// and C) take the place of one A = X X^T and one C X.  No more than two, because A holds small singular values by their squares: of 300 x 577
// matrices of rank 20, 60 and 100 over noise of 0.01, the update by one product is 3.6e-2, 2.0e-2 and 1.4e-2 off (of its norm), as with all
// iterations on X, and 5.9e-2, 4.6e-2 and 3.4e-2 with the last three on A; by three products 2.8e-5, 1.6e-5 and 1.1e-5 (1 to 1.4 times what fp32
// products leave), and 7.0e-5, 4.6e-5 and 3.4e-5.  From n = 2 m on: six 1024 x 2048 take 333 us against 347 with all iterations on
// X, two 2048 x 8192 860 to 900 against 953 (three products: 2600 and 3000), ViT-B/16's list, whose three matrices in four have n = 3 m or 4 m,
// 1305 against 1395 to 1440 (3460 to 3530 and 3800).
int64_t short_iterations(const Sides &s, int32_t iterations) { return s.nb >= 2 * s.mb && iterations >= 4 ? 2 : 0; }
// Symmetric matrices that a matrix needs: A and C, or A, C, C A and the last C.
int64_t squares(int64_t r) { return r ? 4 : 2; }

// Columns of a tile, in blocks: two instead of four where that ends earlier on `pairs` pairs of multiprocessors.  A narrow tile takes
// about 0.65 of a wide one's time (its products take half, but it copies three quarters as much).  Two workers' ragged list, 1023 x 2047
// the largest, takes 446 us by this rule, 517 with wide tiles alone and 452 with narrow ones; ViT-B/16's bf16 list 1444, 1444 and 1804.
int32_t tile_width(int64_t wide, int64_t narrow, int64_t pairs) { return ceil_div(narrow, pairs) * 65 < ceil_div(wide, pairs) * 100 ? 2 : 4; }

// The products of a step.  Three slots an iteration -- A, C, and what takes C -- and one more for matrices whose last iterations are short.
struct Operand { int32_t at, pitch, lo; bool iterate, outer; };
struct Product { Operand left, right; int32_t to, gram, rows, columns, sums; bool symmetric; float factor; };
class Plan {
public:
    explicit Plan(int32_t iterations) : iterations_(iterations), slots_(size_t(3 * iterations + 1)) {}

    // All products of a matrix with the last r iterations short; x, square: its iterates' and symmetric matrices' places.  Returns which of the
    // two iterates is the last.
    int add(const MuonMatrix &y, const int32_t *x, const int32_t *square, int32_t r)
    {
        const int32_t mb = y.mb, lo = mb * mb, first_short = r ? iterations_ - r : iterations_;
        const auto whole = [&](int k, bool outer) { return Operand{x[k], y.rb, y.rb * y.cb, true, outer}; };
        const auto half = [&](int32_t at) { return Operand{at, mb, lo, false, false}; };
        const float to_gram = kMuonGramScale / (y.scale * y.scale), keep = 1.0f / kMuonFactorScale;
        const auto square_product = [&](int slot, int32_t a, int32_t b, int32_t to, float factor) {
            slots_[size_t(slot)].push_back(Product{half(a), half(b), to, to, mb, mb, mb, true, factor});
        };
        const auto iterate = [&](int slot, int from, int32_t c, float factor) {
            const Operand l = y.tall ? whole(from, false) : half(c), right = y.tall ? half(c) : whole(from, true);      // X C, or C X
            slots_[size_t(slot)].push_back(Product{l, right, x[from ^ 1], 0, y.rb, y.cb, mb, false, factor});
        };
        const int32_t a = square[0], c = square[1], ca = square[2], last = square[3];
        int now = 0;
        for (int32_t k = 0; k < iterations_; ++k) {
            const int slot = 3 * k;
            const int32_t factor = k > first_short ? last : c;
            if (k <= first_short) slots_[size_t(slot)].push_back(Product{whole(now, y.tall), whole(now, y.tall), a, 0, mb, mb, y.nb, true, to_gram});
            else square_product(slot, c, ca, a, keep);                                   // A <- C (C A)
            slots_[size_t(slot + 1)].push_back(Product{half(a), half(a), factor, a, mb, mb, mb, true, kMuonC * kMuonFactorScale / (kMuonGramScale * kMuonGramScale)});
            if (k < first_short) {
                iterate(slot + 2, now, c, keep);
                now ^= 1;
            } else if (k == first_short) square_product(slot + 2, c, a, ca, keep);        // C A
            else square_product(slot + 2, last, c, a, 0.25f * keep);                     // the last C times this one, up to 3.45^2, where A was
        }
        if (r) {
            iterate(3 * iterations_, now, a, 4.0f * keep);
            now ^= 1;
        }
        return now;
    }

    // The launches' tiles, one launch for each slot that has products; their places are numbers for now.
    void tiles(std::vector<MuonTile> &out, std::vector<MuonLaunch> &launches, int64_t pairs)
    {
        for (size_t slot = 0; slot < slots_.size(); ++slot) {
            std::vector<Product> &all = slots_[slot];
            if (all.empty()) continue;
            int64_t wide = 0, narrow = 0;
            for (const Product &p : all) {
                wide += p.symmetric ? half_tiles(p.rows, 4) : whole_tiles(p.rows, p.columns, 4);
                narrow += p.symmetric ? half_tiles(p.rows, 2) : whole_tiles(p.rows, p.columns, 2);
            }
            const int32_t width = tile_width(wide, narrow, pairs);
            // long products first, so that short ones fill the end
            std::stable_sort(all.begin(), all.end(), [](const Product &a, const Product &b) { return a.sums > b.sums; });
            const size_t begin = out.size();
            for (const Product &p : all) {
                const auto tile = [&](int32_t i, int32_t q) {
                    const int32_t flags = (p.left.iterate ? MUON_LEFT_ITERATE : 0) | (p.left.outer ? MUON_LEFT_OUTER : 0) |
                                          (p.right.iterate ? MUON_RIGHT_ITERATE : 0) | (p.right.outer ? MUON_RIGHT_OUTER : 0);
                    out.push_back(MuonTile{i, q, width, flags, p.rows, p.columns, p.sums, p.factor, p.left.at, p.left.pitch, p.left.lo, p.right.at,
                                           p.right.pitch, p.right.lo, p.to, p.gram});
                };
                // neighbours share what is longer: the iterate's tile, not the factor's
                if (p.rows > p.columns) {
                    for (int32_t i = 0; i * 4 < p.rows; ++i)
                        for (int32_t q = 0; q < p.columns; q += width) tile(i, q);
                } else {
                    for (int32_t q = 0; q < p.columns; q += width)
                        for (int32_t i = 0; i * 4 < p.rows && (!p.symmetric || i <= q / 4); ++i) tile(i, q);
                }
            }
            launches.push_back(MuonLaunch{int64_t(begin), int64_t(out.size() - begin), slot % 3 == 1});
        }
    }

private:
    int32_t iterations_;
    std::vector<std::vector<Product>> slots_;
};

// Blocks of shared memory and columns of tensor memory that a matrix stepped by one block needs; whether it is one.
bool is_small(int64_t rows, int64_t cols, int64_t parts, int64_t &blocks, int64_t &columns)
{
    const Sides s = sides_of(rows, cols);
    blocks = (s.mb * s.nb + s.mb * s.mb) * parts;
    columns = std::max(s.mb, rows > cols ? (s.nb + 1) / 2 * s.mb : s.nb) * 64;
    return s.mb <= 2 && s.nb <= 8 && blocks <= kMuonSmallBlocks;
}

struct Layout {
    int64_t small, n_small;
    int64_t matrices, grads, chunks, blocks, tiles, sync_tensors, sync_chunks, partial, factor, arrived, late, data, bytes;
    int64_t n_chunks, n_blocks, n_tiles, n_sync, n_param_sync;
    int status;
};

// Where everything lies in the workspace, from the matrices' sizes.
Layout layout_of(const int64_t *rows, const int64_t *cols, int32_t n, int32_t workers, int32_t products, int32_t iterations)
{
    Layout l;
    std::memset(&l, 0, sizeof l);
    int64_t data = 0;
    const int64_t parts = products == 3 ? 2 : 1;
    for (int32_t i = 0; i < n; ++i) {
        if (rows[i] < 0 || cols[i] < 0) { l.status = QSR_EINVAL; return l; }
        if (rows[i] > kMaxSide || cols[i] > kMaxSide || std::min(rows[i], cols[i]) > kMaxShortSide) { l.status = QSR_ERANGE; return l; }
        const int64_t size = rows[i] * cols[i];
        if (size == 0) continue;
        const Sides s = sides_of(rows[i], cols[i]);
        int64_t blocks, columns;
        l.n_chunks += ceil_div(size, kChunk);
        if (i < n / workers) l.n_param_sync += ceil_div(size, kSyncChunk);
        if (is_small(rows[i], cols[i], parts, blocks, columns)) {
            l.n_small++;
            continue;
        }
        const int64_t r = short_iterations(s, iterations), half = half_tiles(s.mb, 2), whole = std::max(whole_tiles(s.mb, s.nb, 2), whole_tiles(s.nb, s.mb, 2));
        l.n_blocks += s.mb * s.nb;
        l.n_tiles += iterations * (2 * half + whole) + (r ? 2 * half : 0);               // room for tiles of either width
        data += (2 * s.mb * s.nb + squares(r) * s.mb * s.mb) * parts * kBlockBytes;
    }
    l.n_sync = 2 * l.n_param_sync;
    if (l.n_chunks > 0x7fffffff || l.n_blocks > 0x7fffffff || l.n_tiles > 0x7fffffff || data / kBlockBytes > (int64_t(1) << 25)) { l.status = QSR_ERANGE; return l; }
    int64_t at = 0;
    auto take = [&at](int64_t bytes) { const int64_t here = at; at += (bytes + 255) / 256 * 256; return here; };
    l.matrices = take(int64_t(n) * int64_t(sizeof(MuonMatrix)));
    l.grads = take(int64_t(n) * int64_t(sizeof(void *)));
    l.chunks = take(l.n_chunks * int64_t(sizeof(MuonChunk)));
    l.blocks = take(l.n_blocks * int64_t(sizeof(MuonBlock)));
    l.tiles = take(l.n_tiles * int64_t(sizeof(MuonTile)));
    l.small = take(l.n_small * int64_t(sizeof(int32_t)));
    l.sync_tensors = take(2 * int64_t(n) * int64_t(sizeof(ListTensor)));
    l.sync_chunks = take(l.n_sync * int64_t(sizeof(ListChunk)));
    l.partial = take(l.n_chunks * int64_t(sizeof(double)));
    l.factor = take(2 * int64_t(n) * int64_t(sizeof(float)));
    l.arrived = take(int64_t(n) * int64_t(sizeof(unsigned)));
    l.late = take(int64_t(sizeof(unsigned)));
    l.data = take(data);
    l.bytes = std::max<int64_t>(at, 256);
    return l;
}

bool products_known(int32_t products) { return products == 1 || products == 3; }

int check_config(const qsr_muon_config &c)
{
    if (c.n_matrices < 1 || c.workers < 1 || c.n_matrices % c.workers != 0 || c.reserved != 0) return QSR_EINVAL;
    if (!products_known(c.products) || (c.nesterov != 0 && c.nesterov != 1)) return QSR_EINVAL;
    if (c.iterations < 1 || c.iterations > QSR_MUON_MAX_ITERATIONS) return QSR_ERANGE;
    if (!std::isfinite(c.beta) || c.beta < 0.0 || c.beta >= 1.0 || !std::isfinite(c.eps) || c.eps < 0.0 || !std::isfinite(c.weight_decay)) return QSR_EINVAL;
    return QSR_OK;
}

int check_matrices(const qsr_muon_config &c, const qsr_matrix *t)
{
    const int32_t per = c.n_matrices / c.workers;
    for (int32_t i = 0; i < c.n_matrices; ++i) {
        const qsr_matrix &x = t[i], &first = t[i % per];
        if (x.rows < 0 || x.cols < 0 || !type_bytes(x.param_type) || !type_bytes(x.grad_type) || (x.copy_type != QSR_NONE && !type_bytes(x.copy_type)) ||
            !std::isfinite(x.wd_scale) || !std::isfinite(x.update_scale) || x.reserved != 0)
            return QSR_EINVAL;
        if (x.rows != first.rows || x.cols != first.cols || x.param_type != first.param_type || x.copy_type != first.copy_type) return QSR_EINVAL;
        if (x.rows == 0 || x.cols == 0) continue;
        if (!x.param || !x.momentum || (x.copy_type != QSR_NONE && !x.copy)) return QSR_EINVAL;
        if (!aligned_to(x.param, unsigned(type_bytes(x.param_type))) || !aligned_to(x.momentum, 4) || !aligned_to(x.grad, unsigned(type_bytes(x.grad_type))) ||
            (x.copy_type != QSR_NONE && !aligned_to(x.copy, unsigned(type_bytes(x.copy_type)))))
            return QSR_EALIGN;
    }
    return QSR_OK;
}

int check_grads(const qsr_muon &x, const void *const *grads)
{
    for (size_t i = 0; i < x.host.size(); ++i) {
        if (x.host[i].rows == 0 || x.host[i].cols == 0) continue;
        if (!grads[i]) return QSR_EINVAL;
        if (!aligned_to(grads[i], unsigned(type_bytes(x.host[i].grad_type)))) return QSR_EALIGN;
    }
    return QSR_OK;
}

bool on_own_device(const qsr_muon &x)
{
    int dev = -1;
    return cudaGetDevice(&dev) == cudaSuccess && dev == x.device;
}

int create(qsr_muon **out, const qsr_muon_config &cfg, const qsr_matrix *t, void *workspace, int64_t workspace_bytes, void *cuda_stream)
{
    const int32_t n = cfg.n_matrices, per = n / cfg.workers;
    std::vector<int64_t> rows(static_cast<size_t>(n)), cols(static_cast<size_t>(n));
    for (int32_t i = 0; i < n; ++i) { rows[size_t(i)] = t[i].rows; cols[size_t(i)] = t[i].cols; }
    const Layout l = layout_of(rows.data(), cols.data(), n, cfg.workers, cfg.products, cfg.iterations);
    if (l.status) return l.status;
    if (!aligned_to(workspace, 256)) return QSR_EALIGN;
    if (workspace_bytes < l.bytes) return QSR_ERANGE;

    std::vector<Range> ranges;
    auto add = [&ranges](const void *p, int64_t bytes, bool written) {
        const uintptr_t b = reinterpret_cast<uintptr_t>(p);
        if (p && bytes > 0) ranges.push_back(Range{b, b + uintptr_t(bytes), written});
    };
    bool has_grads = true;
    for (int32_t i = 0; i < n; ++i) {
        const int64_t size = t[i].rows * t[i].cols;
        add(t[i].param, size * type_bytes(t[i].param_type), true);
        if (t[i].copy_type != QSR_NONE) add(t[i].copy, size * type_bytes(t[i].copy_type), true);
        add(t[i].momentum, size * 4, true);
        add(t[i].grad, size * type_bytes(t[i].grad_type), false);
        has_grads = has_grads && (t[i].grad || size == 0);
    }
    add(workspace, l.bytes, true);
    if (overlap(ranges)) return QSR_EINVAL;

    int dev = 0, multiprocessors = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || cudaDeviceGetAttribute(&multiprocessors, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess) {
        cudaGetLastError();
        return QSR_ECUDA;
    }

    char *ws = static_cast<char *>(workspace);
    std::vector<MuonMatrix> matrices(static_cast<size_t>(n));
    std::vector<const void *> grads(static_cast<size_t>(n));
    std::vector<MuonChunk> chunks, small_chunks;
    std::vector<int32_t> small;
    int64_t small_blocks = 0, small_columns = 32;
    std::vector<MuonBlock> blocks;
    std::vector<MuonTile> tiles;
    std::vector<MuonLaunch> launches;
    Plan plan(cfg.iterations);
    std::vector<ListTensor> sync_tensors(size_t(n) * 2);
    std::vector<ListChunk> sync_chunks;
    chunks.reserve(size_t(l.n_chunks));
    blocks.reserve(size_t(l.n_blocks));
    tiles.reserve(size_t(l.n_tiles));
    sync_chunks.reserve(size_t(l.n_sync));
    const int64_t parts = cfg.products == 3 ? 2 : 1;
    char *at = ws + l.data;
    auto take = [&at, parts](int64_t count) {
        uint16_t *here = reinterpret_cast<uint16_t *>(at);
        at += count * parts * kBlockBytes;
        return here;
    };
    for (int32_t i = 0; i < n; ++i) {
        const qsr_matrix &x = t[i];
        MuonMatrix &y = matrices[size_t(i)];
        std::memset(&y, 0, sizeof y);
        grads[size_t(i)] = x.grad;
        const int32_t k = i / per, j = i % per;          // worker by worker: its parameters, then its momenta
        sync_tensors[size_t(2 * k * per + j)] = ListTensor{x.param, x.copy, nullptr, nullptr, nullptr, nullptr, x.rows * x.cols, x.param_type, QSR_NONE, x.copy_type, 0.0f};
        sync_tensors[size_t((2 * k + 1) * per + j)] = ListTensor{x.momentum, nullptr, nullptr, nullptr, nullptr, nullptr, x.rows * x.cols, QSR_F32, QSR_NONE, QSR_NONE, 0.0f};
        if (x.rows == 0 || x.cols == 0) continue;
        const Sides s = sides_of(x.rows, x.cols);
        y.param = x.param; y.copy = x.copy; y.momentum = x.momentum;
        y.rows = x.rows; y.cols = x.cols;
        y.tall = x.rows > x.cols;
        y.mb = int32_t(s.mb); y.nb = int32_t(s.nb);
        y.rb = y.tall ? y.nb : y.mb; y.cb = y.tall ? y.mb : y.nb;
        y.param_type = x.param_type; y.copy_type = x.copy_type; y.grad_type = x.grad_type;
        y.wd_scale = x.wd_scale; y.update_scale = x.update_scale;
        // entries of the iterate have a root mean square of about one where it is sqrt(m n); fp16 holds up to 65504
        y.scale = float(std::ldexp(1.0, std::min(15, int(std::floor(0.5 * std::log2(double(s.m) * double(s.n)))))));
        int64_t need, columns;
        const bool alone = is_small(x.rows, x.cols, parts, need, columns);
        std::vector<MuonChunk> &to = alone ? small_chunks : chunks;
        y.first_chunk = int32_t(to.size());
        for (int64_t o = 0; o < x.rows * x.cols; o += kChunk) to.push_back(MuonChunk{i, int32_t(std::min(kChunk, x.rows * x.cols - o)), o});
        y.chunks = int32_t(to.size()) - y.first_chunk;
        if (alone) {
            small.push_back(i);
            small_blocks = std::max(small_blocks, need);
            while (small_columns < columns) small_columns *= 2;
            continue;
        }
        const int64_t r = short_iterations(s, cfg.iterations);
        int32_t whole[2], square[4] = {0, 0, 0, 0};
        uint16_t *iterate[2];
        for (int k = 0; k < 2; ++k) {
            whole[k] = int32_t((at - (ws + l.data)) / kBlockBytes);
            iterate[k] = take(s.mb * s.nb);
        }
        for (int64_t k = 0; k < squares(r); ++k) {
            square[k] = int32_t((at - (ws + l.data)) / kBlockBytes);
            take(s.mb * s.mb);
        }
        y.x = iterate[0];
        y.x_last = iterate[plan.add(y, whole, square, int32_t(r))];
        for (int32_t a = 0; a < y.rb; ++a)
            for (int32_t b = 0; b < y.cb; ++b) blocks.push_back(MuonBlock{i, a, b, 0});
    }
    for (int part = 0; part < 2; ++part)
        for (int32_t j = 0; j < per; ++j)
            for (int64_t o = 0; o < t[j].rows * t[j].cols; o += kSyncChunk)
                sync_chunks.push_back(ListChunk{part * per + j, int32_t(std::min(kSyncChunk, t[j].rows * t[j].cols - o)), o});
    const int64_t large_chunks = int64_t(chunks.size());
    chunks.insert(chunks.end(), small_chunks.begin(), small_chunks.end());       // momentum and norm of the others only; all are cleared
    plan.tiles(tiles, launches, std::max(1, multiprocessors / 2));
    if (int64_t(tiles.size()) > l.n_tiles || int64_t(chunks.size()) != l.n_chunks || int64_t(blocks.size()) != l.n_blocks ||
        int64_t(sync_chunks.size()) != l.n_sync || int64_t(small.size()) != l.n_small || at > ws + l.bytes)
        return QSR_EINVAL;                               // the tables do not fit what was reserved for them

    const cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    if (int rc = not_capturing(st)) return rc;
    qsr_muon *x = new qsr_muon;
    try {
        x->host.assign(t, t + n);
    } catch (...) {
        delete x;
        throw;
    }
    x->cfg = cfg;
    x->stream = st;
    x->device = dev;
    x->multiprocessors = multiprocessors;
    x->grads = reinterpret_cast<const void **>(ws + l.grads);
    x->tiles = reinterpret_cast<const MuonTile *>(ws + l.tiles);
    x->products = std::move(launches);
    x->sync_tensors = reinterpret_cast<const ListTensor *>(ws + l.sync_tensors);
    x->sync_chunks = reinterpret_cast<const ListChunk *>(ws + l.sync_chunks);
    x->small = reinterpret_cast<const int32_t *>(ws + l.small);
    x->n_small = int32_t(l.n_small); x->small_blocks = int32_t(small_blocks); x->small_columns = unsigned(small_columns);
    x->chunks = l.n_chunks; x->large_chunks = large_chunks; x->blocks = l.n_blocks;
    x->param_sync_chunks = l.n_param_sync; x->all_sync_chunks = l.n_sync;
    x->has_grads = has_grads;
    x->launches = 0;
    MuonParams &p = x->params;
    std::memset(&p, 0, sizeof p);
    p.matrices = reinterpret_cast<const MuonMatrix *>(ws + l.matrices);
    p.grads = x->grads;
    p.chunks = reinterpret_cast<const MuonChunk *>(ws + l.chunks);
    p.blocks = reinterpret_cast<const MuonBlock *>(ws + l.blocks);
    p.partial = reinterpret_cast<double *>(ws + l.partial);
    p.factor = reinterpret_cast<float *>(ws + l.factor);
    p.arrived = reinterpret_cast<unsigned *>(ws + l.arrived);
    p.late = reinterpret_cast<unsigned *>(ws + l.late);
    p.data = reinterpret_cast<uint16_t *>(ws + l.data);
    p.one_minus_beta = float(1.0 - cfg.beta);
    p.beta = float(cfg.beta);
    p.eps = float(cfg.eps);
    p.nesterov = cfg.nesterov; p.products = cfg.products; p.iterations = cfg.iterations;
    if (l.n_tiles > 0)
        if (int bad = encode_muon_maps(x->maps, p.data, l.bytes - l.data)) {
            delete x;
            return launch_status(bad);
        }
    cudaError_t err = upload(ws + l.matrices, matrices.data(), matrices.size() * sizeof(MuonMatrix), st);
    if (err == cudaSuccess) err = upload(ws + l.grads, grads.data(), grads.size() * sizeof(void *), st);
    if (err == cudaSuccess) err = upload(ws + l.chunks, chunks.data(), chunks.size() * sizeof(MuonChunk), st);
    if (err == cudaSuccess) err = upload(ws + l.blocks, blocks.data(), blocks.size() * sizeof(MuonBlock), st);
    if (err == cudaSuccess) err = upload(ws + l.tiles, tiles.data(), tiles.size() * sizeof(MuonTile), st);
    if (err == cudaSuccess) err = upload(ws + l.small, small.data(), small.size() * sizeof(int32_t), st);
    if (err == cudaSuccess) err = upload(ws + l.sync_tensors, sync_tensors.data(), sync_tensors.size() * sizeof(ListTensor), st);
    if (err == cudaSuccess) err = upload(ws + l.sync_chunks, sync_chunks.data(), sync_chunks.size() * sizeof(ListChunk), st);
    if (err == cudaSuccess) err = cudaMemsetAsync(p.arrived, 0, size_t(n) * sizeof(unsigned), st);
    if (err == cudaSuccess) err = cudaMemsetAsync(p.late, 0, sizeof(unsigned), st);
    if (err != cudaSuccess) {
        delete x;
        return launch_status(int(err));
    }
    *out = x;
    return QSR_OK;
}

}  // namespace

extern "C" {

int64_t qsr_muon_workspace_bytes(const int64_t *rows_host, const int64_t *cols_host, int32_t n_matrices, int32_t workers, int32_t products)
{
    if (!rows_host || !cols_host || n_matrices < 1 || workers < 1 || n_matrices % workers != 0 || !products_known(products)) return QSR_EINVAL;
    const Layout l = layout_of(rows_host, cols_host, n_matrices, workers, products, QSR_MUON_MAX_ITERATIONS);
    return l.status ? l.status : l.bytes;
}

int qsr_muon_create(qsr_muon **out, const qsr_muon_config *cfg, const qsr_matrix *matrices_host, void *workspace_dev, int64_t workspace_bytes,
                    void *cuda_stream)
{
    if (!out) return QSR_EINVAL;
    *out = nullptr;
    if (!cfg || !matrices_host || !workspace_dev) return QSR_EINVAL;
    if (int rc = check_config(*cfg)) return rc;
    if (int rc = check_matrices(*cfg, matrices_host)) return rc;
    try {
        return create(out, *cfg, matrices_host, workspace_dev, workspace_bytes, cuda_stream);
    } catch (...) {        // out of host memory
        return QSR_EINVAL;
    }
}

int qsr_muon_destroy(qsr_muon *muon)
{
    delete muon;
    return QSR_OK;
}

int qsr_muon_set_grads(qsr_muon *muon, const void *const *grads_host)
{
    if (!muon || !grads_host) return QSR_EINVAL;
    if (int rc = check_grads(*muon, grads_host)) return rc;
    if (!on_own_device(*muon)) return QSR_ESTATE;
    if (int rc = not_capturing(muon->stream)) return rc;
    try {              // a copy of the caller's array, which may be page-locked: see upload
        const std::vector<const void *> table(grads_host, grads_host + muon->cfg.n_matrices);
        const int rc = launch_status(int(upload(muon->grads, table.data(), table.size() * sizeof(void *), muon->stream)));
        muon->has_grads = rc == QSR_OK;
        return rc;
    } catch (...) {    // out of host memory
        return QSR_EINVAL;
    }
}

int qsr_muon_step(qsr_muon *muon, double lr, double grad_scale)
{
    if (!muon || !std::isfinite(float(lr)) || !std::isfinite(float(grad_scale)) || !std::isfinite(float(lr * muon->cfg.weight_decay))) return QSR_EINVAL;
    if (!muon->has_grads || !on_own_device(*muon)) return QSR_ESTATE;
    if (muon->chunks == 0) return QSR_OK;
    MuonParams p = muon->params;
    p.grad_scale = float(grad_scale);
    p.lr = float(lr);
    p.lr_decay = float(lr * muon->cfg.weight_decay);
    if (muon->n_small > 0) {
        muon->launches++;
        if (int err = launch_muon_small(p, muon->small, muon->n_small, muon->small_blocks, muon->small_columns, muon->stream)) return launch_status(err);
    }
    if (muon->large_chunks == 0) return QSR_OK;
    muon->launches++;
    if (int err = launch_muon_momentum(p, muon->large_chunks, muon->stream)) return launch_status(err);
    muon->launches++;
    if (int err = launch_muon_pack(p, muon->blocks, muon->stream)) return launch_status(err);
    for (const MuonLaunch &x : muon->products) {
        muon->launches++;
        if (int err = launch_muon_product(p, muon->maps, x.polynomial, muon->tiles + x.first, x.n, muon->multiprocessors, muon->stream)) return launch_status(err);
    }
    muon->launches++;
    return launch_status(launch_muon_apply(p, muon->blocks, muon->stream));
}

int qsr_muon_sync(qsr_muon *muon, int32_t state_sync)
{
    if (!muon || state_sync < QSR_STATE_KEEP || state_sync > QSR_STATE_RESET) return QSR_EINVAL;
    if (!on_own_device(*muon)) return QSR_ESTATE;
    if (muon->chunks == 0) return QSR_OK;
    const int32_t K = muon->cfg.workers;
    ListSyncParams p;
    p.tensors = muon->sync_tensors; p.chunks = muon->sync_chunks;
    p.workers = K; p.tensors_per_worker = 2 * (muon->cfg.n_matrices / K);
    p.divisor = float(K);
    p.inverse = (K & (K - 1)) == 0 ? 1.0f / float(K) : 0.0f;
    muon->launches++;
    const int64_t chunks = state_sync == QSR_STATE_AVERAGE ? muon->all_sync_chunks : muon->param_sync_chunks;
    if (int err = launch_list_sync(p, false, false, chunks, muon->stream)) return launch_status(err);
    if (state_sync != QSR_STATE_RESET) return QSR_OK;
    muon->launches++;
    return launch_status(launch_muon_clear(muon->params, muon->chunks, muon->stream));
}

int qsr_muon_check(qsr_muon *muon)
{
    if (!muon) return QSR_EINVAL;
    if (!on_own_device(*muon)) return QSR_ESTATE;
    if (int rc = not_capturing(muon->stream)) return rc;
    unsigned late = 0;
    cudaError_t err = cudaMemcpyAsync(&late, muon->params.late, sizeof late, cudaMemcpyDeviceToHost, muon->stream);
    if (err == cudaSuccess) err = cudaStreamSynchronize(muon->stream);
    if (err != cudaSuccess) return launch_status(int(err));
    return late ? QSR_ECUDA : QSR_OK;
}

int64_t qsr_muon_launch_count(const qsr_muon *muon) { return muon ? muon->launches : int64_t(QSR_EINVAL); }

}  // extern "C"
