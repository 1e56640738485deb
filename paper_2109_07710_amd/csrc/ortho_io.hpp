// What both forms of the orthogonalised update share: reading the matrices,
// their norms, and storing the update.
#pragma once

#include "common.hpp"
#include "block_kernels.hpp"

namespace cbw {

__device__ __forceinline__ float load_value(const void* p, int64_t i, bool f32)
{
    return f32 ? static_cast<const float*>(p)[i] : __uint_as_float((uint32_t) static_cast<const uint16_t*>(p)[i] << 16);
}
// Eight values from p's element i on, 16-byte aligned.
__device__ __forceinline__ void load_values(const void* p, int64_t i, bool f32, float (&v)[8])
{
    if (f32) {
        const float4 x = *reinterpret_cast<const float4*>(static_cast<const float*>(p) + i);
        const float4 y = *reinterpret_cast<const float4*>(static_cast<const float*>(p) + i + 4);
        v[0] = x.x, v[1] = x.y, v[2] = x.z, v[3] = x.w, v[4] = y.x, v[5] = y.y, v[6] = y.z, v[7] = y.w;
    } else {
        const uint4 x = *reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(p) + i);
        const uint32_t b[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] = __uint_as_float(k & 1 ? b[k / 2] & 0xffff0000u : b[k / 2] << 16);
    }
}

// 1 / (|M| + eps), from the sum of squares.  A norm that is no number, or
// infinite, leaves no number anywhere; nothing stays nothing.
__device__ __forceinline__ double inverse_of(double sum, double eps)
{
    const double norm = sqrt(sum), all = norm + eps;
    return all > 0.0 ? (norm < __builtin_inf() ? 1.0 / all : __builtin_nan("")) : all == 0.0 ? 0.0 : all;
}

// Eight values of a row of the output, from column `col` on.
__device__ __forceinline__ void store_out(const OrthoArgs& a, int mat, int row, int col, const float (&v)[8])
{
    if (row >= a.rows || col >= a.cols) return;
    const int64_t at = ((int64_t)mat * a.rows + row) * a.out_stride + col;
    const int n = min(8, a.cols - col);
    if (a.out_f32) {
        float* o = static_cast<float*>(a.o) + at;
        if (n == 8 && ((uintptr_t)o & 15) == 0) {
            *reinterpret_cast<float4*>(o) = make_float4(v[0], v[1], v[2], v[3]);
            *reinterpret_cast<float4*>(o + 4) = make_float4(v[4], v[5], v[6], v[7]);
        } else {
#pragma unroll
            for (int k = 0; k < 8; ++k)
                if (k < n) o[k] = v[k];
        }
    } else {
        uint16_t* o = static_cast<uint16_t*>(a.o) + at;
        const uint4 w = make_uint4(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7]));
        if (n == 8 && ((uintptr_t)o & 15) == 0) {
            *reinterpret_cast<uint4*>(o) = w;
        } else {
            const uint32_t b[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
            for (int k = 0; k < 8; ++k)
                if (k < n) o[k] = (uint16_t)(b[k / 2] >> 16 * (k & 1));
        }
    }
}

}  // namespace cbw
