// C ABI of the tensor lists: checks, the device tables, per-step scalars, launches.  See include/qsr.h.
#include <cuda_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>
#include <cstring>
#include <new>
#include <vector>

#include "checks.h"
#include "internal.h"

struct qsr_list {
    qsr_list_config cfg;
    cudaStream_t stream;
    int device;
    int64_t chunks, chunks_per_worker;
    qsr::ListTensor *tensors;       // device tables, in the caller's workspace
    const void **grads;
    qsr::ListChunk *chunk_table;
    float *partial, *clip;
    unsigned *arrived;
    std::vector<qsr_tensor> host;
    bool has_grads;
    qsr::ListShape shape;
    int64_t launches;
};

namespace {

using namespace qsr;

constexpr int64_t kBlock = 256;            // elements that share a scale in 8 bits: chunks are whole blocks

bool known(int type) { return type_bytes(type) != 0; }

constexpr int64_t kWarpBlocks = qsr::kListWarps * kBlock;      // elements of a thread block with one block per warp

// Elements per thread block where every multiprocessor has work many times over: as many blocks per warp as hide the latency of
// their loads.  fp32 states (operands in registers): four; ViT-B/16's list takes 364 us with four, 2 % more with three, 6 % with two.
// 8-bit states (operands in shared memory): as many as let four thread blocks share a multiprocessor, at most four; 229 us
// with three of fp32 parameters and bf16 gradients, 240 with four.
int stages_of(int stage_bytes)
{
    const int fit = stage_bytes == 0 ? qsr::kListStages : 56 * 1024 / (qsr::kListWarps * stage_bytes);
    return std::max(1, std::min(fit, qsr::kListStages));
}
// Small lists: one block per warp, so that more multiprocessors share the work, until they hold as many thread blocks as they
// can (8 M elements, clipped: 52.4 us with four blocks per warp, 57.5 with one; 1 M: the same).
bool is_small(int64_t total) { return total < int64_t(148) * 8 * kWarpBlocks; }

struct Layout { int64_t tensors, grads, chunks, partial, clip, arrived, bytes, n_chunks, chunk; };

// Where the tables lie in the workspace; n_chunks < 0 is a qsr_status.  stages = 0: as much as any types may need.
Layout layout_of(const int64_t *numel, int32_t n, int32_t workers, int stages)
{
    Layout l;
    std::memset(&l, 0, sizeof l);
    int64_t total = 0;
    for (int32_t i = 0; i < n; ++i) {
        if (numel[i] < 0 || numel[i] > (int64_t(1) << 44)) { l.n_chunks = QSR_EINVAL; return l; }
        total += numel[i];
        if (total > (int64_t(1) << 48)) { l.n_chunks = QSR_ERANGE; return l; }
    }
    l.chunk = kWarpBlocks * (is_small(total) ? 1 : stages > 0 ? stages : stages_of(int(kBlock) * 10));
    for (int32_t i = 0; i < n; ++i) l.n_chunks += (numel[i] + l.chunk - 1) / l.chunk;
    if (l.n_chunks > 0x7fffffff) { l.n_chunks = QSR_ERANGE; return l; }
    int64_t at = 0;
    auto take = [&at](int64_t bytes) { const int64_t here = at; at += (bytes + 255) / 256 * 256; return here; };
    l.tensors = take(int64_t(n) * int64_t(sizeof(qsr::ListTensor)));
    l.grads = take(int64_t(n) * int64_t(sizeof(void *)));
    l.chunks = take(l.n_chunks * int64_t(sizeof(qsr::ListChunk)));
    l.partial = take(l.n_chunks * int64_t(sizeof(float)));
    l.clip = take(int64_t(workers) * int64_t(sizeof(float)));
    l.arrived = take(int64_t(workers) * int64_t(sizeof(unsigned)));
    l.bytes = std::max<int64_t>(at, 256);
    return l;
}

int check_grads(const qsr_list_config &c, const qsr_tensor *t, const void *const *grads)
{
    for (int32_t i = 0; i < c.n_tensors; ++i) {
        if (t[i].numel == 0) continue;
        if (!grads[i]) return QSR_EINVAL;
        if (!aligned_to(grads[i], unsigned(type_bytes(t[i].grad_type)))) return QSR_EALIGN;
    }
    return QSR_OK;
}

bool unit_interval(double x) { return std::isfinite(x) && x >= 0.0 && x < 1.0; }

int check_list(const qsr_list_config &c, const qsr_tensor *t)
{
    if (c.n_tensors < 1 || c.workers < 1 || c.n_tensors % c.workers != 0 || c.reserved != 0) return QSR_EINVAL;
    if (c.states != QSR_STATES_F32 && c.states != QSR_STATES_E4M3) return QSR_EINVAL;
    if (!unit_interval(c.beta1) || !unit_interval(c.beta2) || !std::isfinite(c.eps) || c.eps < 0.0 || !std::isfinite(c.weight_decay))
        return QSR_EINVAL;
    if (!aligned_to(c.grad_norm, 4)) return QSR_EALIGN;
    const bool codes = c.states == QSR_STATES_E4M3;
    const int32_t per = c.n_tensors / c.workers;
    for (int32_t i = 0; i < c.n_tensors; ++i) {
        const qsr_tensor &x = t[i], &first = t[i % per];
        if (x.numel < 0 || !known(x.param_type) || !known(x.grad_type) || (x.copy_type != QSR_NONE && !known(x.copy_type)) ||
            !std::isfinite(x.wd_scale))
            return QSR_EINVAL;
        if (x.numel != first.numel || x.param_type != first.param_type || x.copy_type != first.copy_type) return QSR_EINVAL;
        if (x.numel == 0) continue;
        if (!x.param || !x.m || !x.v || (codes && (!x.m_scale || !x.v_scale)) || (x.copy_type != QSR_NONE && !x.copy)) return QSR_EINVAL;
        if (!aligned_to(x.param, unsigned(type_bytes(x.param_type))) || (!codes && (!aligned_to(x.m, 4) || !aligned_to(x.v, 4))) ||
            (codes && (!aligned_to(x.m_scale, 4) || !aligned_to(x.v_scale, 4))) ||
            (x.copy_type != QSR_NONE && !aligned_to(x.copy, unsigned(type_bytes(x.copy_type)))) ||
            !aligned_to(x.grad, unsigned(type_bytes(x.grad_type))))
            return QSR_EALIGN;
    }
    return QSR_OK;
}

bool on_own_device(const qsr_list &x)
{
    int dev = -1;
    return cudaGetDevice(&dev) == cudaSuccess && dev == x.device;
}

int create(qsr_list **out, const qsr_list_config &cfg, const qsr_tensor *t, void *workspace, int64_t workspace_bytes, void *cuda_stream)
{
    const int32_t n = cfg.n_tensors;
    std::vector<int64_t> numel(static_cast<size_t>(n));
    for (int32_t i = 0; i < n; ++i) numel[size_t(i)] = t[i].numel;
    const bool codes = cfg.states == QSR_STATES_E4M3;
    qsr::ListShape shape{0, 0, 0, t[0].param_type, t[0].grad_type};
    for (int32_t i = 0; i < n; ++i) {
        if (t[i].param_type != t[0].param_type || t[i].grad_type != t[0].grad_type) shape.param_type = shape.grad_type = QSR_NONE;
        if (codes) shape.stage_bytes = std::max(shape.stage_bytes, int(kBlock) * (type_bytes(t[i].param_type) + type_bytes(t[i].grad_type) + 2));
    }
    shape.stages = stages_of(shape.stage_bytes);
    const Layout l = layout_of(numel.data(), n, cfg.workers, shape.stages);
    if (l.n_chunks < 0) return int(l.n_chunks);
    if (!aligned_to(workspace, 256)) return QSR_EALIGN;
    if (workspace_bytes < l.bytes) return QSR_ERANGE;

    shape.chunks = l.n_chunks;
    shape.stages = int(l.chunk / kWarpBlocks);
    std::vector<Range> ranges;
    auto add = [&ranges](const void *p, int64_t bytes, bool written) {
        const uintptr_t b = reinterpret_cast<uintptr_t>(p);
        if (p && bytes > 0) ranges.push_back(Range{b, b + uintptr_t(bytes), written});
    };
    bool has_grads = true;
    for (int32_t i = 0; i < n; ++i) {
        const qsr_tensor &x = t[i];
        const int64_t scales = (x.numel + kBlock - 1) / kBlock * 4, state = x.numel * (codes ? 1 : 4);
        add(x.param, x.numel * type_bytes(x.param_type), true);
        if (x.copy_type != QSR_NONE) add(x.copy, x.numel * type_bytes(x.copy_type), true);
        add(x.m, state, true);
        add(x.v, state, true);
        if (codes) {
            add(x.m_scale, scales, true);
            add(x.v_scale, scales, true);
        }
        add(x.grad, x.numel * type_bytes(x.grad_type), false);
        has_grads = has_grads && (x.grad || x.numel == 0);
    }
    add(workspace, l.bytes, true);
    add(cfg.grad_norm, int64_t(cfg.workers) * 4, true);
    if (overlap(ranges)) return QSR_EINVAL;

    std::vector<qsr::ListTensor> table(static_cast<size_t>(n));
    std::vector<const void *> grads(static_cast<size_t>(n));
    std::vector<qsr::ListChunk> chunks;
    chunks.reserve(size_t(l.n_chunks));
    for (int32_t i = 0; i < n; ++i) {
        const qsr_tensor &x = t[i];
        table[size_t(i)] = qsr::ListTensor{x.param, x.copy, x.m, x.v, x.m_scale, x.v_scale, x.numel, x.param_type, x.grad_type, x.copy_type, x.wd_scale};
        grads[size_t(i)] = x.grad;
        for (int64_t o = 0; o < x.numel; o += l.chunk)
            chunks.push_back(qsr::ListChunk{i, int32_t(std::min(l.chunk, x.numel - o)), o});
    }

    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess) { cudaGetLastError(); return QSR_ECUDA; }
    if (int rc = not_capturing(static_cast<cudaStream_t>(cuda_stream))) return rc;
    qsr_list *x = new qsr_list;
    char *ws = static_cast<char *>(workspace);
    x->cfg = cfg;
    x->stream = static_cast<cudaStream_t>(cuda_stream);
    x->device = dev;
    x->chunks = l.n_chunks;
    x->chunks_per_worker = l.n_chunks / cfg.workers;
    x->tensors = reinterpret_cast<qsr::ListTensor *>(ws + l.tensors);
    x->grads = reinterpret_cast<const void **>(ws + l.grads);
    x->chunk_table = reinterpret_cast<qsr::ListChunk *>(ws + l.chunks);
    x->partial = reinterpret_cast<float *>(ws + l.partial);
    x->clip = reinterpret_cast<float *>(ws + l.clip);
    x->arrived = reinterpret_cast<unsigned *>(ws + l.arrived);
    x->has_grads = has_grads;
    x->launches = 0;
    x->shape = shape;
    cudaError_t err = cudaSuccess;
    try {
        x->host.assign(t, t + n);
    } catch (...) {
        delete x;
        throw;
    }
    if (err == cudaSuccess) err = upload(x->tensors, table.data(), table.size() * sizeof(qsr::ListTensor), x->stream);
    if (err == cudaSuccess) err = upload(x->grads, grads.data(), grads.size() * sizeof(void *), x->stream);
    if (err == cudaSuccess) err = upload(x->chunk_table, chunks.data(), chunks.size() * sizeof(qsr::ListChunk), x->stream);
    if (err == cudaSuccess) err = cudaMemsetAsync(x->arrived, 0, size_t(cfg.workers) * sizeof(unsigned), x->stream);
    if (err != cudaSuccess) {
        delete x;
        return launch_status(err);
    }
    *out = x;
    return QSR_OK;
}

}  // namespace

extern "C" {

int64_t qsr_list_workspace_bytes(const int64_t *numel_host, int32_t n_tensors, int32_t workers)
{
    if (!numel_host || n_tensors < 1 || workers < 1 || n_tensors % workers != 0) return QSR_EINVAL;
    const Layout l = layout_of(numel_host, n_tensors, workers, 0);
    return l.n_chunks < 0 ? l.n_chunks : l.bytes;
}

int qsr_list_create(qsr_list **out, const qsr_list_config *cfg, const qsr_tensor *tensors_host, void *workspace_dev,
                    int64_t workspace_bytes, void *cuda_stream)
{
    if (!out) return QSR_EINVAL;
    *out = nullptr;
    if (!cfg || !tensors_host || !workspace_dev) return QSR_EINVAL;
    if (int rc = check_list(*cfg, tensors_host)) return rc;
    try {
        return create(out, *cfg, tensors_host, workspace_dev, workspace_bytes, cuda_stream);
    } catch (...) {        // out of host memory
        return QSR_EINVAL;
    }
}

int qsr_list_destroy(qsr_list *list)
{
    delete list;
    return QSR_OK;
}

int qsr_list_set_grads(qsr_list *list, const void *const *grads_host)
{
    if (!list || !grads_host) return QSR_EINVAL;
    if (int rc = check_grads(list->cfg, list->host.data(), grads_host)) return rc;
    if (!on_own_device(*list)) return QSR_ESTATE;
    if (int rc = not_capturing(list->stream)) return rc;
    try {              // a copy of the caller's array, which may be page-locked: see upload
        const std::vector<const void *> table(grads_host, grads_host + list->cfg.n_tensors);
        const int rc = launch_status(upload(list->grads, table.data(), table.size() * sizeof(void *), list->stream));
        list->has_grads = rc == QSR_OK;
        return rc;
    } catch (...) {    // out of host memory
        return QSR_EINVAL;
    }
}

int qsr_list_step(qsr_list *list, int64_t n, double lr, double grad_scale)
{
    if (!list || !std::isfinite(lr) || !std::isfinite(grad_scale)) return QSR_EINVAL;
    if (n < 1) return QSR_ERANGE;
    if (!list->has_grads || !on_own_device(*list)) return QSR_ESTATE;
    if (list->chunks == 0) return QSR_OK;
    const qsr_list_config &c = list->cfg;
    // everything that depends on n is evaluated in binary64 and rounded to fp32 once
    const double bc1 = 1.0 - std::pow(c.beta1, double(n)), bc2 = 1.0 - std::pow(c.beta2, double(n));
    qsr::ListStepParams p;
    std::memset(&p, 0, sizeof p);
    p.tensors = list->tensors; p.grads = list->grads; p.chunks = list->chunk_table;
    p.tensors_per_worker = c.n_tensors / c.workers;
    p.omb1 = float(1.0 - c.beta1); p.omb2 = float(1.0 - c.beta2);
    p.eps = float(c.eps);
    p.eta_wd = float(lr * c.weight_decay);
    p.step_size = float(lr / bc1);
    p.inv_sqrt_bc2 = float(1.0 / std::sqrt(bc2));
    p.grad_scale = float(grad_scale);
    p.one = 1.0f;
    if (c.clip_norm > 0.0 && std::isfinite(c.clip_norm)) {
        qsr::ListNormParams q;
        std::memset(&q, 0, sizeof q);
        q.tensors = list->tensors; q.grads = list->grads; q.chunks = list->chunk_table;
        q.partial = list->partial; q.clip = list->clip; q.arrived = list->arrived;
        q.grad_norm = c.grad_norm;
        q.chunks_per_worker = int32_t(list->chunks_per_worker);
        q.max_norm = float(c.clip_norm); q.grad_scale = p.grad_scale;
        list->launches++;
        if (int err = qsr::launch_list_norm(q, list->chunks, list->stream)) return launch_status(err);
        p.clip = list->clip;
    }
    list->launches++;
    return launch_status(qsr::launch_list_step(p, list->shape, list->stream));
}

int qsr_list_sync(qsr_list *list, int32_t state_sync)
{
    if (!list || state_sync < QSR_STATE_KEEP || state_sync > QSR_STATE_RESET) return QSR_EINVAL;
    if (!on_own_device(*list)) return QSR_ESTATE;
    if (list->chunks == 0) return QSR_OK;
    const qsr_list_config &c = list->cfg;
    qsr::ListSyncParams p;
    p.tensors = list->tensors; p.chunks = list->chunk_table;
    p.workers = c.workers; p.tensors_per_worker = c.n_tensors / c.workers;
    p.divisor = float(c.workers);
    p.inverse = (c.workers & (c.workers - 1)) == 0 ? 1.0f / float(c.workers) : 0.0f;
    const bool codes = c.states == QSR_STATES_E4M3;
    list->launches++;
    if (int err = qsr::launch_list_sync(p, codes, state_sync == QSR_STATE_AVERAGE, list->chunks_per_worker, list->stream))
        return launch_status(err);
    if (state_sync != QSR_STATE_RESET) return QSR_OK;
    list->launches++;
    return launch_status(qsr::launch_list_reset(p, codes, list->chunks, list->stream));
}

int64_t qsr_list_launch_count(const qsr_list *list) { return list ? list->launches : int64_t(QSR_EINVAL); }

}  // extern "C"
