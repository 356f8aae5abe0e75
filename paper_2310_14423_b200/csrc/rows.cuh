// Rows of matrices in the caller's number types: which columns a thread has, loading and storing them eight at a time.
#ifndef QSR_ROWS_CUH_
#define QSR_ROWS_CUH_

#include "wide.cuh"

namespace qsr {

template <typename T> struct Kind;
template <> struct Kind<float> { static constexpr int type = QSR_F32; };
template <> struct Kind<__nv_bfloat16> { static constexpr int type = QSR_BF16; };
template <> struct Kind<__half> { static constexpr int type = QSR_F16; };

// Which columns a thread has.  VEC: granules of eight consecutive ones, `lanes` granules apart.  Otherwise (rows that are not all
// aligned to eight elements) single columns `lanes` apart, so that a warp's accesses are adjacent.
template <bool VEC>
__device__ __forceinline__ int column(int lane, int lanes, int k, int j)
{
    return VEC ? (lane + k * lanes) * 8 + j : lane + (k * 8 + j) * lanes;
}

// Eight elements of a row as they lie in memory (16-bit types: two to a word); what lies beyond the row reads as zero.
template <bool VEC>
__device__ __forceinline__ void fetch(Raw8 &r, const void *row, int lane, int lanes, int k, int width, int type)
{
    const int c0 = column<VEC>(lane, lanes, k, 0);
    if (VEC && c0 + 8 <= width) {
        load8(r, row, c0, type);
        return;
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const int c = column<VEC>(lane, lanes, k, j);
        const uint32_t w = c < width ? load1(row, c, type) : 0u;
        if (type == QSR_F32) r.w[j] = w;
        else if (j & 1) r.w[j / 2] |= w << 16;
        else r.w[j / 2] = w;
    }
}

template <bool VEC>
__device__ __forceinline__ void put(void *row, const float (&v)[8], int lane, int lanes, int k, int width, int type)
{
    const int c0 = column<VEC>(lane, lanes, k, 0);
    if (VEC && c0 + 8 <= width) {
        store8(row, c0, v, type);
        return;
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const int c = column<VEC>(lane, lanes, k, j);
        if (c < width) store1(row, c, v[j], type);
    }
}

template <typename T>
__device__ __forceinline__ const void *row_of(const void *base, int64_t row, int64_t stride) { return static_cast<const T *>(base) + row * stride; }
template <typename T>
__device__ __forceinline__ void *row_of(void *base, int64_t row, int64_t stride) { return static_cast<T *>(base) + row * stride; }

}  // namespace qsr
#endif
