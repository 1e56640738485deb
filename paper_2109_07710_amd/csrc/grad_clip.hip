// The norm of many gradients taken together, and their scaling to a limit.
//
//   norm = sqrt(sum over all tensors of g^2)   or   max |g|
//   c = min(1, max_norm / (norm + 1e-6)),  out = c g
//
// Bound by memory: every gradient is read once for the norm and once more to
// be scaled.  The tensors' addresses travel in the kernel arguments, 128 to a
// launch, so nothing is copied to the device and a captured call replays as
// it was.  Each workgroup sums a contiguous range of chunks in a fixed order
// and leaves one partial; the scaling kernel's workgroups each add all
// partials in the same order (8 KB from the L2) instead of waiting for a
// launch in between, so a call is two launches per 128 tensors.
#include "common.hpp"
#include "block_kernels.hpp"

namespace cbw {
namespace {

constexpr int GT = 256;   // threads per workgroup

// 16 bytes at any element alignment: gradients are often views into packed
// buffers (global memory takes unaligned vector accesses).
typedef u32x4 u32x4_any __attribute__((aligned(2)));

__device__ __forceinline__ float bf16_lo(uint32_t v) { return __uint_as_float(v << 16); }
__device__ __forceinline__ float bf16_hi(uint32_t v) { return __uint_as_float(v & 0xffff0000u); }

// The running value of a norm.  Squares are summed in 64 bits: the largest
// float32 squared still fits, so no scaling pass is needed, and the sum's
// rounding is nothing beside the result's.  The largest magnitude is kept as
// its bit pattern, which orders like the value and puts NaN above infinity.
struct SumSquares {
    double v = 0.0;
    __device__ void add(float g) { v = fma((double)g, (double)g, v); }
    __device__ void join(double o) { v += o; }
    __device__ double value() const { return v; }
    __device__ static double finish(double s) { return sqrt(s); }
};
struct MaxAbs {
    uint32_t v = 0;
    __device__ void add(float g)
    {
        const uint32_t b = __float_as_uint(g) & 0x7fffffffu;
        v = b > v ? b : v;
    }
    __device__ void join(double o) { add((float)o); }
    __device__ double value() const { return (double)__uint_as_float(v); }
    __device__ static double finish(double s) { return s; }
};

// All threads' values joined in a fixed order; every thread has the result.
template <typename R>
__device__ double join_workgroup(R r)
{
    __shared__ double wave_s[GT / 64];
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1) r.join(__shfl_xor(r.value(), o));
    if ((threadIdx.x & 63) == 0) wave_s[threadIdx.x >> 6] = r.value();
    __syncthreads();
    R all;
    for (int w = 0; w < GT / 64; ++w) all.join(wave_s[w]);
    return all.value();
}

// The tensor that chunk `c` belongs to: the last one that starts at or before
// it (tensors without elements start where the next one does).
__device__ __forceinline__ int tensor_of(const GradTable& t, int c)
{
    int lo = 0, hi = t.n;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (t.first[mid] <= c) lo = mid;
        else hi = mid;
    }
    return lo;
}

struct ChunkRange {
    int begin, end;
};
__device__ __forceinline__ ChunkRange my_chunks(int chunks)
{
    const int64_t g = gridDim.x, b = blockIdx.x;
    return {(int)(b * chunks / g), (int)((b + 1) * chunks / g)};
}

template <typename R>
__global__ __launch_bounds__(GT) void grad_norm_kernel(GradTable t, double* partial)
{
    R r;
    const ChunkRange range = my_chunks(t.chunks);
    for (int c = range.begin; c < range.end; ++c) {
        const int k = __builtin_amdgcn_readfirstlane(tensor_of(t, c));
        const int64_t count = t.count[k] & 0x7fffffffffffffffll;
        const int64_t e0 = (int64_t)(c - t.first[k]) * kGradChunk;
        const int n = (int)(count - e0 < kGradChunk ? count - e0 : kGradChunk);
        if (t.count[k] < 0) {
            const uint16_t* src = static_cast<const uint16_t*>(t.src[k]) + e0;
            constexpr int U = kGradChunk / (8 * GT);
            u32x4 v[U];
#pragma unroll
            for (int i = 0; i < U; ++i) {
                const int e = (i * GT + (int)threadIdx.x) * 8;
                v[i] = e + 8 <= n ? *reinterpret_cast<const u32x4_any*>(src + e) : u32x4{0, 0, 0, 0};
            }
#pragma unroll
            for (int i = 0; i < U; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    r.add(bf16_lo(v[i][j]));
                    r.add(bf16_hi(v[i][j]));
                }
            const int e = (n & ~7) + (int)threadIdx.x;
            if (e < n) r.add(bf16_lo(src[e]));
        } else {
            const float* src = static_cast<const float*>(t.src[k]) + e0;
            constexpr int U = kGradChunk / (4 * GT);
            u32x4 v[U];
#pragma unroll
            for (int i = 0; i < U; ++i) {
                const int e = (i * GT + (int)threadIdx.x) * 4;
                v[i] = e + 4 <= n ? *reinterpret_cast<const u32x4_any*>(src + e) : u32x4{0, 0, 0, 0};
            }
#pragma unroll
            for (int i = 0; i < U; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) r.add(__uint_as_float(v[i][j]));
            const int e = (n & ~3) + (int)threadIdx.x;
            if (e < n) r.add(src[e]);
        }
    }
    const double sum = join_workgroup(r);
    if (threadIdx.x == 0) partial[blockIdx.x] = sum;
}

template <typename R>
__device__ double norm_of(const double* partial, int npartial)
{
    R r;
    for (int i = threadIdx.x; i < npartial; i += GT) r.join(partial[i]);
    return R::finish(join_workgroup(r));
}

template <typename R>
__global__ __launch_bounds__(GT) void grad_finish_kernel(const double* partial, int npartial, float* norm)
{
    const double v = norm_of<R>(partial, npartial);
    if (threadIdx.x == 0) norm[0] = (float)v;
}

// The chunks go backwards: those that the norm pass read last are the ones
// that the 256 MB cache still holds.
template <typename R>
__global__ __launch_bounds__(GT) void grad_scale_kernel(GradTable t, const double* partial, int npartial, float max_norm,
                                                        float* norm)
{
    const double total = norm_of<R>(partial, npartial);
    const double q = (double)max_norm / (total + 1e-6);
    const float coef = q >= 1.0 ? 1.0f : (float)q;   // (a NaN stays one)
    if (norm && blockIdx.x == 0 && threadIdx.x == 0) {
        norm[0] = (float)total;
        norm[1] = coef;
    }
    const ChunkRange range = my_chunks(t.chunks);
    for (int c = range.end - 1; c >= range.begin; --c) {
        const int k = __builtin_amdgcn_readfirstlane(tensor_of(t, c));
        const int64_t count = t.count[k] & 0x7fffffffffffffffll;
        const int64_t e0 = (int64_t)(c - t.first[k]) * kGradChunk;
        const int n = (int)(count - e0 < kGradChunk ? count - e0 : kGradChunk);
        if (coef == 1.0f && t.src[k] == t.dst[k]) continue;   // in place and unclipped: every value stays
        if (t.count[k] < 0) {
            const uint16_t* src = static_cast<const uint16_t*>(t.src[k]) + e0;
            uint16_t* dst = static_cast<uint16_t*>(t.dst[k]) + e0;
            constexpr int U = kGradChunk / (8 * GT);
            u32x4 v[U];
#pragma unroll
            for (int i = 0; i < U; ++i) {
                const int e = (i * GT + (int)threadIdx.x) * 8;
                v[i] = e + 8 <= n ? *reinterpret_cast<const u32x4_any*>(src + e) : u32x4{0, 0, 0, 0};
            }
#pragma unroll
            for (int i = 0; i < U; ++i) {
                const int e = (i * GT + (int)threadIdx.x) * 8;
                u32x4 o;
#pragma unroll
                for (int j = 0; j < 4; ++j) o[j] = pack_bf16x2(bf16_lo(v[i][j]) * coef, bf16_hi(v[i][j]) * coef);
                if (e + 8 <= n) *reinterpret_cast<u32x4_any*>(dst + e) = o;
            }
            const int e = (n & ~7) + (int)threadIdx.x;
            if (e < n) dst[e] = (uint16_t)f32_to_bf16_rne(bf16_lo(src[e]) * coef);
        } else {
            const float* src = static_cast<const float*>(t.src[k]) + e0;
            float* dst = static_cast<float*>(t.dst[k]) + e0;
            constexpr int U = kGradChunk / (4 * GT);
            u32x4 v[U];
#pragma unroll
            for (int i = 0; i < U; ++i) {
                const int e = (i * GT + (int)threadIdx.x) * 4;
                v[i] = e + 4 <= n ? *reinterpret_cast<const u32x4_any*>(src + e) : u32x4{0, 0, 0, 0};
            }
#pragma unroll
            for (int i = 0; i < U; ++i) {
                const int e = (i * GT + (int)threadIdx.x) * 4;
                u32x4 o;
#pragma unroll
                for (int j = 0; j < 4; ++j) o[j] = __float_as_uint(__uint_as_float(v[i][j]) * coef);
                if (e + 4 <= n) *reinterpret_cast<u32x4_any*>(dst + e) = o;
            }
            const int e = (n & ~3) + (int)threadIdx.x;
            if (e < n) dst[e] = src[e] * coef;
        }
    }
}

}  // namespace

hipError_t launch_grad_norm(const GradTable& t, int kind, int grid, double* partial, hipStream_t s)
{
    if (kind == CBW_GRAD_NORM_2) grad_norm_kernel<SumSquares><<<grid, GT, 0, s>>>(t, partial);
    else grad_norm_kernel<MaxAbs><<<grid, GT, 0, s>>>(t, partial);
    return hipGetLastError();
}

hipError_t launch_grad_finish(int kind, const double* partial, int npartial, float* norm, hipStream_t s)
{
    if (kind == CBW_GRAD_NORM_2) grad_finish_kernel<SumSquares><<<1, GT, 0, s>>>(partial, npartial, norm);
    else grad_finish_kernel<MaxAbs><<<1, GT, 0, s>>>(partial, npartial, norm);
    return hipGetLastError();
}

hipError_t launch_grad_scale(const GradTable& t, int kind, int grid, const double* partial, int npartial, float max_norm,
                             float* norm, hipStream_t s)
{
    if (kind == CBW_GRAD_NORM_2)
        grad_scale_kernel<SumSquares><<<grid, GT, 0, s>>>(t, partial, npartial, max_norm, norm);
    else
        grad_scale_kernel<MaxAbs><<<grid, GT, 0, s>>>(t, partial, npartial, max_norm, norm);
    return hipGetLastError();
}

}  // namespace cbw
