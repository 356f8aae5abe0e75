// Checks of arguments that several entry points share (host only).
#ifndef QSR_CHECKS_H_
#define QSR_CHECKS_H_

#include <cuda_runtime.h>

#include <algorithm>
#include <cstdint>
#include <vector>

#include "../../include/qsr.h"

namespace qsr {

// Bytes of an element of a qsr type, 0 for an unknown type.
inline int type_bytes(int type) { return type == QSR_F32 ? 4 : type == QSR_BF16 || type == QSR_F16 ? 2 : 0; }
inline bool aligned_to(const void *p, unsigned bytes) { return (reinterpret_cast<uintptr_t>(p) & (bytes - 1)) == 0; }

// Whether two matrices of rows x columns elements share a byte (strides and element sizes may differ; not the same matrix).
// With equal strides in bytes, as columns of one buffer have them, rows meet exactly if the distance modulo the stride is less
// than a row from either side; otherwise matrices that lie in and out of one another count as sharing.
inline bool share_bytes(const void *a, int64_t a_stride, int64_t a_columns, int a_bytes, int64_t a_rows, const void *b, int64_t b_stride,
                        int64_t b_columns, int b_bytes, int64_t b_rows)
{
    typedef __int128 wide;                          // strides have no upper limit
    const wide x = wide(reinterpret_cast<uintptr_t>(a)), y = wide(reinterpret_cast<uintptr_t>(b));
    const wide xr = wide(a_columns) * a_bytes, yr = wide(b_columns) * b_bytes, xs = wide(a_stride) * a_bytes, ys = wide(b_stride) * b_bytes;
    if (a_rows < 1 || b_rows < 1 || xr < 1 || yr < 1) return false;
    if (x + (a_rows - 1) * xs + xr <= y || y + (b_rows - 1) * ys + yr <= x) return false;
    if (xs != ys || a_rows == 1 || b_rows == 1) return true;
    const wide d = ((y - x) % xs + xs) % xs;         // where b's rows begin after the beginning of one of a's
    return d < xr || d > xs - yr;
}

// Whether every row of a matrix begins on a multiple of eight elements.
inline bool rows_aligned(const void *base, int64_t stride, int64_t rows, int bytes)
{
    return aligned_to(base, unsigned(8 * bytes)) && (rows <= 1 || stride % 8 == 0);
}

inline int power_of_two(int n)          // the smallest that is at least n
{
    int p = 1;
    while (p < n) p *= 2;
    return p;
}

inline int launch_status(int err)
{
    if (err == 0) return QSR_OK;
    cudaGetLastError();
    return QSR_ECUDA;
}

struct Range { uintptr_t begin, end; bool written; };

// Two ranges that share a byte, one of them written.
inline bool overlap(std::vector<Range> &r)
{
    std::sort(r.begin(), r.end(), [](const Range &a, const Range &b) { return a.begin < b.begin; });
    uintptr_t end_any = 0, end_written = 0;
    for (const Range &x : r) {
        if (x.begin < end_written || (x.written && x.begin < end_any)) return true;
        end_any = std::max(end_any, x.end);
        if (x.written) end_written = std::max(end_written, x.end);
    }
    return false;
}

// Enqueues a copy from pageable host memory: such a copy is staged before the call returns, so the source may be freed.  A copy from
// page-locked memory would read it whenever the stream gets there.
inline cudaError_t upload(void *dst, const void *src, size_t bytes, cudaStream_t st)
{
    return bytes ? cudaMemcpyAsync(dst, src, bytes, cudaMemcpyHostToDevice, st) : cudaSuccess;
}

// QSR_ESTATE during a capture: a captured copy from pageable memory would read it at every replay.  The legacy default stream
// takes no work while a blocking stream is being captured; the query says so with an error of its own, and an attempt would
// invalidate that capture.
inline int not_capturing(cudaStream_t st)
{
    cudaStreamCaptureStatus status = cudaStreamCaptureStatusNone;
    const cudaError_t err = cudaStreamIsCapturing(st, &status);
    if (err == cudaErrorStreamCaptureImplicit) {
        cudaGetLastError();
        return QSR_ESTATE;
    }
    if (err != cudaSuccess) return launch_status(int(err));
    return status == cudaStreamCaptureStatusNone ? QSR_OK : QSR_ESTATE;
}

}  // namespace qsr
#endif
