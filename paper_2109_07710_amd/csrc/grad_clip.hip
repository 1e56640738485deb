// The norm of many gradients taken together, and their scaling to a limit.
//
//   norm = sqrt(sum over all tensors of g^2)   or   max |g|
//   c = min(1, max_norm / (norm + 1e-6)),  out = c g
//
// Bound by memory: every gradient is read once for the norm and once more to
// be scaled.  The tensors' addresses travel in the kernel arguments, 120 to a
// launch, so nothing is copied to the device and a captured call replays as
// it was; the norm's launches leave them in the workspace, where one scaling
// launch finds all of them.  Each workgroup sums a contiguous range of chunks
// in a fixed order and leaves one partial; the scaling kernel's workgroups
// each add all partials in the same order (8 KB from the L2, under their
// first chunk's loads) instead of waiting for a launch in between.  A call is
// two launches, one more for every 120 tensors past the first.  (13 tensors,
// 59 MB: 32 us; 300 packed ones, 90 MB: 67; 48 of 2.1 GB together: 1276, 5.05
// TB/s.)
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

// A workgroup's 16 KB of one tensor: four vectors a thread, and one of the up
// to seven elements that are left past a tensor's last whole vector.
struct Chunk {
    static constexpr int U = kGradChunk / (16 * GT);
    u32x4 v[U];
    uint32_t left;      // the element's bits (bf16: its 16)
    char* dst;
    int n;              // bytes
    bool bf16, has_left;

    __device__ __forceinline__ int at(int i) const { return (i * GT + (int)threadIdx.x) * 16; }
    __device__ __forceinline__ int left_at() const { return (n & ~15) + (int)threadIdx.x * (bf16 ? 2 : 4); }

    __device__ __forceinline__ void load(const GradEntry& e, int c)
    {
        const int64_t b0 = (int64_t)(c - e.first) * kGradChunk, all = e.bytes & INT64_MAX;
        const char* src = static_cast<const char*>(e.src) + b0;
        dst = static_cast<char*>(e.dst) + b0;
        n = (int)(all - b0 < kGradChunk ? all - b0 : kGradChunk);
        bf16 = e.bytes < 0;
#pragma unroll
        for (int i = 0; i < U; ++i)
            v[i] = at(i) + 16 <= n ? *reinterpret_cast<const u32x4_any*>(src + at(i)) : u32x4{0, 0, 0, 0};
        has_left = left_at() < n;
        left = 0;
        if (has_left)
            left = bf16 ? *reinterpret_cast<const uint16_t*>(src + left_at()) : *reinterpret_cast<const uint32_t*>(src + left_at());
    }
};

struct ChunkRange {
    int begin, end;
};
__device__ __forceinline__ ChunkRange my_chunks(int chunks)
{
    const int64_t g = gridDim.x, b = blockIdx.x;
    return {(int)(b * chunks / g), (int)((b + 1) * chunks / g)};
}

template <typename R>
__global__ __launch_bounds__(GT) void grad_norm_kernel(GradTable t, double* partial, GradEntry* table)
{
    // Kernel arguments lie far away (every first touch of a line takes a
    // microsecond or two): the table comes to the LDS at once, not entry by
    // entry.
    __shared__ GradEntry e_s[kGradTable];
    const int lane = threadIdx.x & 63;
    const ChunkRange range = my_chunks(t.chunks);
    static_assert(2 * kGradTable <= GT && sizeof(GradEntry) == 32 && alignof(GradEntry) == 16, "an aligned 16-byte half entry a thread");
    if ((int)threadIdx.x < 2 * kGradTable)
        reinterpret_cast<u32x4*>(e_s)[threadIdx.x] = reinterpret_cast<const u32x4*>(t.e)[threadIdx.x];
    __syncthreads();
    // the tensor of the first chunk: the last one that starts at or before it
    const int f0 = lane < t.n ? e_s[lane].first : INT32_MAX;
    const int f1 = lane + 64 < t.n ? e_s[lane + 64 < kGradTable ? lane + 64 : 0].first : INT32_MAX;
    int k = __popcll(__ballot(f0 <= range.begin)) + __popcll(__ballot(f1 <= range.begin)) - 1;
    if (table && blockIdx.x == 0 && (int)threadIdx.x < t.n) {
        GradEntry e = e_s[threadIdx.x];
        e.first += t.chunk0;
        table[t.entry0 + threadIdx.x] = e;
    }
    R r;
    Chunk next;
    next.load(e_s[k], range.begin);
    for (int c = range.begin; c < range.end; ++c) {
        const Chunk now = next;
        if (c + 1 < range.end) {
            if (k + 1 < t.n && e_s[k + 1].first <= c + 1) ++k;
            next.load(e_s[k], c + 1);
        }
        if (now.bf16) {
#pragma unroll
            for (int i = 0; i < Chunk::U; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    r.add(bf16_lo(now.v[i][j]));
                    r.add(bf16_hi(now.v[i][j]));
                }
            r.add(bf16_lo(now.left));
        } else {
#pragma unroll
            for (int i = 0; i < Chunk::U; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) r.add(__uint_as_float(now.v[i][j]));
            r.add(__uint_as_float(now.left));
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

// The tensor of chunk c in the table: a wave looks at 64 starts at a time.
__device__ __forceinline__ int tensor_of(const GradEntry* table, int n, int c)
{
    const int lane = threadIdx.x & 63;
    int lo = 0, hi = n;   // the tensor lies in [lo, hi)
    while (hi - lo > 1) {
        const int step = (hi - lo + 63) / 64, i = lo + lane * step;
        lo += (__popcll(__ballot(i < hi && table[i < hi ? i : lo].first <= c)) - 1) * step;
        hi = min(hi, lo + step);
    }
    return lo;
}

// The chunks go backwards: those that the norm pass read last are the ones
// that the 256 MB cache still holds.
template <typename R>
__global__ __launch_bounds__(GT) void grad_scale_kernel(const GradEntry* table, int n, int chunks, const double* partial,
                                                        int npartial, float max_norm, float* norm)
{
    const ChunkRange range = my_chunks(chunks);
    int k = 0;
    Chunk next;
    if (chunks > 0) {
        k = __builtin_amdgcn_readfirstlane(tensor_of(table, n, range.end - 1));
        next.load(table[k], range.end - 1);
    }
    const double total = norm_of<R>(partial, npartial);
    // A norm that is reported as infinity scales to zero, also where only
    // float32 cannot hold it and where the limit is infinite as well.
    const double q = isinf((float)total) ? 0.0 : (double)max_norm / (total + 1e-6);
    const float coef = q >= 1.0 ? 1.0f : (float)q;   // (a NaN stays one)
    if (blockIdx.x == 0 && threadIdx.x == 0) {
        norm[0] = (float)total;
        norm[1] = coef;
    }
    for (int c = range.end - 1; c >= range.begin; --c) {
        const Chunk now = next;
        // in place and unclipped every value stays
        const bool stays = coef == 1.0f && table[k].src == table[k].dst;
        if (c > range.begin) {
            if (table[k].first == c) --k;
            if (!(coef == 1.0f && table[k].src == table[k].dst)) next.load(table[k], c - 1);
        }
        if (stays) continue;
#pragma unroll
        for (int i = 0; i < Chunk::U; ++i) {
            u32x4 o;
#pragma unroll
            for (int j = 0; j < 4; ++j)
                o[j] = now.bf16 ? pack_bf16x2(bf16_lo(now.v[i][j]) * coef, bf16_hi(now.v[i][j]) * coef)
                                : __float_as_uint(__uint_as_float(now.v[i][j]) * coef);
            if (now.at(i) + 16 <= now.n) *reinterpret_cast<u32x4_any*>(now.dst + now.at(i)) = o;
        }
        if (now.has_left) {
            if (now.bf16) *reinterpret_cast<uint16_t*>(now.dst + now.left_at()) = (uint16_t)f32_to_bf16_rne(bf16_lo(now.left) * coef);
            else *reinterpret_cast<float*>(now.dst + now.left_at()) = __uint_as_float(now.left) * coef;
        }
    }
}

}  // namespace

hipError_t launch_grad_norm(const GradTable& t, int kind, int grid, double* partial, GradEntry* table, hipStream_t s)
{
    if (kind == CBW_GRAD_NORM_2) grad_norm_kernel<SumSquares><<<grid, GT, 0, s>>>(t, partial, table);
    else grad_norm_kernel<MaxAbs><<<grid, GT, 0, s>>>(t, partial, table);
    return hipGetLastError();
}

hipError_t launch_grad_finish(int kind, const double* partial, int npartial, float* norm, hipStream_t s)
{
    if (kind == CBW_GRAD_NORM_2) grad_finish_kernel<SumSquares><<<1, GT, 0, s>>>(partial, npartial, norm);
    else grad_finish_kernel<MaxAbs><<<1, GT, 0, s>>>(partial, npartial, norm);
    return hipGetLastError();
}

hipError_t launch_grad_scale(const GradEntry* table, int n, int chunks, int kind, int grid, const double* partial,
                             int npartial, float max_norm, float* norm, hipStream_t s)
{
    if (kind == CBW_GRAD_NORM_2)
        grad_scale_kernel<SumSquares><<<grid, GT, 0, s>>>(table, n, chunks, partial, npartial, max_norm, norm);
    else
        grad_scale_kernel<MaxAbs><<<grid, GT, 0, s>>>(table, n, chunks, partial, npartial, max_norm, norm);
    return hipGetLastError();
}

}  // namespace cbw
