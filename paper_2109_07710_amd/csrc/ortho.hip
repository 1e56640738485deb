// Orthogonalised updates: a few Newton-Schulz steps bring the singular values
// of a gradient's matrix near one.
//
//   X = M / (|M| + eps), n x m with n <= m (M transposed where it is tall);
//   each step:  A = X X^T,  B = b A + c A A,  X = a X + B X
//
// Three products a step, A and A A symmetric: their tiles on and below the
// diagonal are computed and stored at both places.  X is held in float32.  The
// products take its values, and A's and B's, as pairs of fp16 numbers, high
// and low part (hi = fp16(v), lo = fp16(v - hi): 22 bits of v), and sum hi hi +
// hi lo + lo hi in float32 on the matrix cores, 2^-22 from the full product: as
// near to 64 bits as the same steps in float32 (2.1e-6 against 2.1e-6 of the
// result's 2-norm, 256 x 2304 of full rank), at three instructions of the
// half-precision rate, which is a fifth of the float32 instructions' time.
// Where the update is stored in bf16, all steps but the last two take the high
// parts alone: what they leave off, 11 bits of the products but not of the a X
// beside them, is smaller than a bf16 value's rounding after the last two
// (7.7e-4 of the 2-norm against 1.7e-3; one such step at the end: 3e-3).
#include "common.hpp"
#include "block_kernels.hpp"
#include "expert_tiles.hpp"
#include "tiles.hpp"

#include <algorithm>

namespace cbw {
namespace {

typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef float floatx8 __attribute__((ext_vector_type(8)));

__device__ __forceinline__ floatx4 mfma_half(floatx4 acc, const uint4& a, const uint4& b)
{
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), acc, 0, 0, 0);
}

// What the planes hold: X 2^11, A 2^10, B 2^10.  Powers of two change no bit,
// and the low parts stay normal numbers for values of X down to 2^-13 (below
// that they lose no more than 2^-36 of the row's norm).  The descriptor's check
// keeps |X| <= 4, |A| <= 16 and |B| <= 32, so that nothing overflows.
constexpr float kX = 2048.f, kA = 1024.f, kB = 1024.f;

struct Pair {
    uint4 hi, lo;
};
__device__ __forceinline__ Pair split(const float (&v)[8])
{
    Pair p;
    uint32_t h[4], l[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const floatx2 x = {v[2 * k], v[2 * k + 1]};
        const f16x2 hi = __builtin_convertvector(x, f16x2);
        const floatx2 back = __builtin_convertvector(hi, floatx2);
        const floatx2 rest = {x.x - back.x, x.y - back.y};
        h[k] = __builtin_bit_cast(uint32_t, hi);
        l[k] = __builtin_bit_cast(uint32_t, __builtin_convertvector(rest, f16x2));
    }
    p.hi = make_uint4(h[0], h[1], h[2], h[3]);
    p.lo = make_uint4(l[0], l[1], l[2], l[3]);
    return p;
}
__device__ __forceinline__ void join(const Pair& p, float (&v)[8])
{
    const floatx8 h = __builtin_convertvector(__builtin_bit_cast(f16x8, p.hi), floatx8);
    const floatx8 l = __builtin_convertvector(__builtin_bit_cast(f16x8, p.lo), floatx8);
#pragma unroll
    for (int k = 0; k < 8; ++k) v[k] = h[k] + l[k];
}

// ------------------------------------------------------- norm and first X

__device__ __forceinline__ float load_value(const void* p, int64_t i, bool f32)
{
    return f32 ? static_cast<const float*>(p)[i] : __uint_as_float((uint32_t) static_cast<const uint16_t*>(p)[i] << 16);
}

// Sums of squares of a matrix, in 64 bits: part z of a.parts takes every
// a.parts-th chunk.  Contiguous matrices are one long row.
constexpr int kChunk = 4096;
__global__ __launch_bounds__(256) void ortho_norm_kernel(OrthoArgs a)
{
    const int z = blockIdx.x % a.parts, mat = blockIdx.x / a.parts;
    const bool flat = a.in_stride == a.cols;
    const int64_t rows = flat ? 1 : a.rows, cols = flat ? (int64_t)a.rows * a.cols : a.cols;
    const int64_t chunks = (cols + kChunk - 1) / kChunk;
    const int64_t base = (int64_t)mat * a.rows * a.in_stride;
    double s = 0.0;
    for (int64_t u = z; u < rows * chunks; u += a.parts) {
        const int64_t row = u / chunks, c0 = (u - row * chunks) * kChunk;
        const int64_t first = base + row * a.in_stride + c0;
        const int n = (int)min((int64_t)kChunk, cols - c0);
        for (int i = threadIdx.x; i < n; i += 256) {
            const double v = load_value(a.m, first + i, a.in_f32);
            s += v * v;
        }
    }
    __shared__ double sums[4];
    for (int k = 32; k >= 1; k >>= 1) s += __shfl_xor(s, k);
    if ((threadIdx.x & 63) == 0) sums[threadIdx.x >> 6] = s;
    __syncthreads();
    if (threadIdx.x == 0) a.partial[(int64_t)mat * a.parts + z] = sums[0] + sums[1] + sums[2] + sums[3];
}

// X and its planes, 64 x 64 values a workgroup, zeros past the matrix.
__global__ __launch_bounds__(256) void ortho_start_kernel(OrthoArgs a, bool pair)
{
    __shared__ float tile[64][65];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int bx = a.mp / 64, by = a.np / 64;
    const int mat = blockIdx.x / (bx * by), in = blockIdx.x - mat * (bx * by);
    const int i0 = in / bx * 64, j0 = in % bx * 64;   // of X

    double s = 0.0;
    for (int z = lane; z < a.parts; z += 64) s += a.partial[(int64_t)mat * a.parts + z];
    for (int k = 32; k >= 1; k >>= 1) s += __shfl_xor(s, k);
    // a norm that is no number, or infinite, leaves no number anywhere; nothing stays nothing
    const double norm = sqrt(s), by_norm = norm + a.eps;
    const double inv = by_norm > 0.0 ? (norm < __builtin_inf() ? 1.0 / by_norm : __builtin_nan("")) : by_norm == 0.0 ? 0.0 : by_norm;

    const int64_t base = (int64_t)mat * a.rows * a.in_stride;
    const int r0 = a.tall ? j0 : i0, c0 = a.tall ? i0 : j0;   // of M
    for (int r = wave; r < 64; r += 4) {
        const int row = r0 + r, col = c0 + lane;
        // (values past the matrix stay zero, also where the norm is no number)
        const float v = row < a.rows && col < a.cols ? (float)(load_value(a.m, base + row * a.in_stride + col, a.in_f32) * inv) : 0.f;
        if (a.tall) tile[lane][r] = v;
        else tile[r][lane] = v;
    }
    __syncthreads();
    const int64_t at0 = (int64_t)mat * a.np * a.mp;
    for (int t = threadIdx.x; t < 64 * 8; t += 256) {
        const int i = t / 8, j = t % 8 * 8;
        const int64_t at = at0 + (int64_t)(i0 + i) * a.mp + j0 + j;
        float v[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] = tile[i][j + k];
#pragma unroll
        for (int k = 0; k < 8; k += 4) *reinterpret_cast<float4*>(a.x + at + k) = make_float4(v[k], v[k + 1], v[k + 2], v[k + 3]);
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] *= kX;
        const Pair p = split(v);
        *reinterpret_cast<uint4*>(a.planes[0] + at) = p.hi;
        if (pair) *reinterpret_cast<uint4*>(a.planes[0] + a.x_plane + at) = p.lo;
    }
}

// ---------------------------------------------------------------- products

enum { GRAM = 0, SQUARE = 1, UPDATE = 2 };

// A tile's place: its matrix, rows i0 on, columns j0 on.
struct Spot {
    int mat, i0, j0;
};
template <int STAGE, int T>
__device__ __forceinline__ Spot spot_of(const OrthoArgs& a, int tile)
{
    Spot s;
    const int rows = a.np / T, cols = a.mp / T;
    const int per = STAGE == UPDATE ? rows * cols : rows * (rows + 1) / 2;
    s.mat = tile / per;
    const int in = tile - s.mat * per;
    if (STAGE == UPDATE) {
        s.i0 = in % rows * T;
        s.j0 = in / rows * T;
    } else {
        // row i has i + 1 tiles
        int i = (int)((sqrtf(8.f * (float)in + 1.f) - 1.f) * 0.5f);
        while (i * (i + 1) / 2 > in) --i;
        while ((i + 1) * (i + 2) / 2 <= in) ++i;
        s.i0 = i * T;
        s.j0 = (in - i * (i + 1) / 2) * T;
    }
    return s;
}

// A tile in LDS as [row][column], in float32.  A row's 16-byte chunks are moved
// so that both a row's vectors and a column's values are read without sharing
// banks.
template <int T>
struct Square {
    static constexpr int CHUNKS = T / 4;
    static __device__ __forceinline__ int swizzle(int q) { return (q ^ (q >> 3)) & (CHUNKS - 1); }
    static __device__ __forceinline__ float* chunk(float* t, int q, int c) { return t + q * T + ((c ^ swizzle(q)) << 2); }
    static __device__ __forceinline__ float* value(float* t, int q, int p) { return chunk(t, q, p >> 2) + (p & 3); }
};

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

// What becomes of a finished tile of sums, in LDS: A or B into their planes at
// both places, X and its planes, or the update.
template <int STAGE, int T, int THREADS>
__device__ __forceinline__ void finish(const OrthoArgs& a, const StepArgs& st, const Spot& s, float* tile)
{
    using Sq = Square<T>;
    const bool mirror = STAGE != UPDATE ? s.i0 != s.j0 : st.last && a.tall;
    const int64_t an = (int64_t)a.np * a.np, amat = s.mat * an, plane = an * a.batch;
    _Float16* out = STAGE == GRAM ? a.gram : a.poly;
#pragma unroll 2
    for (int t = threadIdx.x; t < T * T / 8; t += THREADS) {
        const int q = t / (T / 8), p = t % (T / 8) * 8;
        float v[8];
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            const floatx4 x = *reinterpret_cast<const floatx4*>(Sq::chunk(tile, q, p / 4 + k));
#pragma unroll
            for (int c = 0; c < 4; ++c) v[4 * k + c] = x[c];
        }
        if (STAGE == UPDATE) {
            const int64_t at = (int64_t)s.mat * a.np * a.mp + (int64_t)(s.i0 + q) * a.mp + s.j0 + p;
            const float4 x0 = *reinterpret_cast<const float4*>(a.x + at), x1 = *reinterpret_cast<const float4*>(a.x + at + 4);
            const float x[8] = {x0.x, x0.y, x0.z, x0.w, x1.x, x1.y, x1.z, x1.w};
#pragma unroll
            for (int k = 0; k < 8; ++k) v[k] = a.a * x[k] + v[k] * (1.f / (kB * kX));
            if (!st.last) {
                *reinterpret_cast<float4*>(a.x + at) = make_float4(v[0], v[1], v[2], v[3]);
                *reinterpret_cast<float4*>(a.x + at + 4) = make_float4(v[4], v[5], v[6], v[7]);
#pragma unroll
                for (int k = 0; k < 8; ++k) v[k] *= kX;
                const Pair w = split(v);
                _Float16* to = a.planes[st.from ^ 1] + at;
                *reinterpret_cast<uint4*>(to) = w.hi;
                if (st.next_pair) *reinterpret_cast<uint4*>(to + a.x_plane) = w.lo;
            } else if (!a.tall) {
                store_out(a, s.mat, s.i0 + q, s.j0 + p, v);
            }
        } else {
            const int64_t at = amat + (int64_t)(s.i0 + q) * a.np + s.j0 + p;
            if (STAGE == GRAM) {
#pragma unroll
                for (int k = 0; k < 8; ++k) v[k] *= kA / (kX * kX);
            } else {
                Pair g;
                g.hi = *reinterpret_cast<const uint4*>(a.gram + at);
                g.lo = *reinterpret_cast<const uint4*>(a.gram + plane + at);
                float x[8];
                join(g, x);
#pragma unroll
                for (int k = 0; k < 8; ++k) v[k] = (a.b * (kB / kA)) * x[k] + (a.c * (kB / (kA * kA))) * v[k];
            }
            const Pair w = split(v);
            *reinterpret_cast<uint4*>(out + at) = w.hi;
            if (STAGE == GRAM || st.pair) *reinterpret_cast<uint4*>(out + plane + at) = w.lo;
        }
        if (mirror) {
#pragma unroll
            for (int k = 0; k < 2; ++k)
                *reinterpret_cast<floatx4*>(Sq::chunk(tile, q, p / 4 + k)) = floatx4{v[4 * k], v[4 * k + 1], v[4 * k + 2], v[4 * k + 3]};
        }
    }
    if (!mirror) return;
    __syncthreads();
    for (int t = threadIdx.x; t < T * T / 8; t += THREADS) {
        const int p = t / (T / 8), q = t % (T / 8) * 8;
        float v[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] = *Sq::value(tile, q + k, p);
        if (STAGE == UPDATE) {
            store_out(a, s.mat, s.j0 + p, s.i0 + q, v);
        } else {
            const int64_t at = amat + (int64_t)(s.j0 + p) * a.np + s.i0 + q;
            const Pair w = split(v);
            *reinterpret_cast<uint4*>(out + at) = w.hi;
            if (STAGE == GRAM || st.pair) *reinterpret_cast<uint4*>(out + plane + at) = w.lo;
        }
    }
}

// T x T tile by NWP x NWQ waves, two buffers of 64 reduction indices of both
// operands, PAIR: of both planes.
template <int STAGE, bool PAIR, int T, int NWP, int NWQ>
struct Product {
    static constexpr int NW = NWP * NWQ, FM = T / NWP / 16, FN = T / NWQ / 16, PL = PAIR ? 2 : 1;
    using OP = Operand<uint16_t, T, STAGE == UPDATE, NW>;
    using OQ = Operand<uint16_t, T, false, NW>;
    static constexpr int COPIES = (OP::COPIES + OQ::COPIES) * PL, TILE = OP::BYTES, BUFFER = 2 * PL * TILE;
    static constexpr int LDS = 2 * BUFFER > T * T * 4 ? 2 * BUFFER : T * T * 4;
};

template <int T, int NWP, int NWQ, int FM, int FN>
__device__ __forceinline__ void to_lds(const floatx4 (&acc)[FM][FN], float* tile)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, wp = wave / NWQ, wq = wave % NWQ;
#pragma unroll
    for (int i = 0; i < FM; ++i)
#pragma unroll
        for (int j = 0; j < FN; ++j)
            *reinterpret_cast<floatx4*>(Square<T>::chunk(tile, wq * (T / NWQ) + j * 16 + (lane & 15),
                                                         (wp * (T / NWP) + i * 16) / 4 + (lane >> 4))) = acc[i][j];
}

template <int STAGE, bool PAIR, int T, int NWP, int NWQ>
__global__ __launch_bounds__(NWP* NWQ * 64) void ortho_product_kernel(OrthoArgs a, StepArgs st)
{
    using P = Product<STAGE, PAIR, T, NWP, NWQ>;
    using OP = typename P::OP;
    using OQ = typename P::OQ;
    constexpr int FM = P::FM, FN = P::FN, PL = P::PL, KB = 64;
    __shared__ __align__(1024) char lds[P::LDS];

    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wp = wave / NWQ, wq = wave % NWQ;
    const int unit = xcd_remap(blockIdx.x, gridDim.x);
    const int tile = unit / st.split, part = unit - tile * st.split;
    const Spot s = spot_of<STAGE, T>(a, tile);

    // rows i0 on of A's and B's left factors, and their columns: X, A or B
    const int64_t xmat = (int64_t)s.mat * a.np * a.mp, gmat = (int64_t)s.mat * a.np * a.np, gplane = (int64_t)a.np * a.np * a.batch;
    const _Float16* x = a.planes[st.from] + xmat;
    const _Float16 *pb, *qb;
    int64_t pplane, qplane, pstride, qstride;
    if (STAGE == GRAM) {
        pb = x + (int64_t)s.j0 * a.mp;
        qb = x + (int64_t)s.i0 * a.mp;
        pplane = qplane = a.x_plane;
        pstride = qstride = a.mp;
    } else if (STAGE == SQUARE) {
        pb = a.gram + gmat + (int64_t)s.j0 * a.np;
        qb = a.gram + gmat + (int64_t)s.i0 * a.np;
        pplane = qplane = gplane;
        pstride = qstride = a.np;
    } else {
        pb = x + s.j0;
        qb = a.poly + gmat + (int64_t)s.i0 * a.np;
        pplane = a.x_plane;
        qplane = gplane;
        pstride = a.mp;
        qstride = a.np;
    }
    const int len = STAGE == GRAM ? a.mp : a.np, all = len / KB;
    const int first = (int)((int64_t)part * all / st.split), steps = (int)((int64_t)(part + 1) * all / st.split) - first;

    OP op;
    OQ oq;
    op.init(wave, T, pstride);
    oq.init(wave, 0, qstride);
    auto copy = [&](int step, int buf) {
        const int64_t k = (int64_t)(first + step) * KB;
        char* to = lds + buf * P::BUFFER;
#pragma unroll
        for (int l = 0; l < PL; ++l) {
            // (across: KB rows of T columns; along: T rows of KB columns)
            const _Float16* p = pb + l * pplane + (STAGE == UPDATE ? k * pstride : k);
            const uint32_t n = (uint32_t)(((STAGE == UPDATE ? KB - 1 : T - 1) * pstride + (STAGE == UPDATE ? T : KB)) * 2);
            op.copy(wave, make_rsrc_words(p, n), 0, KB, to + l * P::TILE);
            oq.copy(wave, make_rsrc_words(qb + l * qplane + k, (uint32_t)(((T - 1) * qstride + KB) * 2)), 0, KB, to + (PL + l) * P::TILE);
        }
    };

    floatx4 acc[FM][FN];
#pragma unroll
    for (int i = 0; i < FM; ++i)
#pragma unroll
        for (int j = 0; j < FN; ++j) acc[i][j] = floatx4{0.f, 0.f, 0.f, 0.f};
    struct Fragments {
        uint4 p[PL][FM], q[PL][FN];
    };
    const int frag_p = OP::first(wp * (T / NWP)), frag_q = OQ::first(wq * (T / NWQ));
    auto read = [&](Fragments& f, int buf, int ks) {
        const char* at = lds + buf * P::BUFFER;
#pragma unroll
        for (int l = 0; l < PL; ++l) {
            OQ::fragments(at + (PL + l) * P::TILE, frag_q, ks, f.q[l]);
            OP::fragments(at + l * P::TILE, frag_p, ks, f.p[l]);
        }
    };
    auto multiply = [&](const Fragments& f) {
#pragma unroll
        for (int l = 0; l < (PAIR ? 3 : 1); ++l)
#pragma unroll
            for (int i = 0; i < FM; ++i)
#pragma unroll
                for (int j = 0; j < FN; ++j) acc[i][j] = mfma_half(acc[i][j], f.p[l == 2 ? PL - 1 : 0][i], f.q[l == 1 ? PL - 1 : 0][j]);
    };
    Fragments fa, fb;
    if (steps > 0) copy(0, 0);
    if (steps > 1) copy(1, 1);
    if (steps > 0) {
        if (steps > 1) wait_copies<P::COPIES>();
        else wait_copies<0>();
        barrier();
        read(fa, 0, 0);
        for (int k = 0; k < steps; ++k) {
            const int buf = k & 1;
            read(fb, buf, 1);
            multiply(fa);
            wait_copies<0>();
            wait_reads();
            barrier();
            if (k + 2 < steps) copy(k + 2, buf);
            if (k + 1 < steps) read(fa, buf ^ 1, 0);
            multiply(fb);
        }
    }
    if (st.split > 1) {
        // as the registers lie: the kernel that adds the parts up has the same threads
        floatx4* to = reinterpret_cast<floatx4*>(a.sums) + (int64_t)unit * (T * T / 4);
#pragma unroll
        for (int i = 0; i < FM; ++i)
#pragma unroll
            for (int j = 0; j < FN; ++j) to[(i * FN + j) * (P::NW * 64) + threadIdx.x] = acc[i][j];
        return;
    }
    __syncthreads();   // every wave is done with the operands
    float* out = reinterpret_cast<float*>(lds);
    to_lds<T, NWP, NWQ>(acc, out);
    __syncthreads();
    finish<STAGE, T, NWP * NWQ * 64>(a, st, s, out);
}

// The parts of a split tile, added in order, and what becomes of it.
template <int STAGE, int T, int NWP, int NWQ>
__global__ __launch_bounds__(NWP* NWQ * 64) void ortho_sum_kernel(OrthoArgs a, StepArgs st)
{
    constexpr int NW = NWP * NWQ, FM = T / NWP / 16, FN = T / NWQ / 16;
    __shared__ __align__(1024) float out[T * T];
    const int tile = blockIdx.x;
    const Spot s = spot_of<STAGE, T>(a, tile);
    const floatx4* from = reinterpret_cast<const floatx4*>(a.sums) + (int64_t)tile * st.split * (T * T / 4);
    floatx4 acc[FM][FN];
#pragma unroll
    for (int i = 0; i < FM; ++i)
#pragma unroll
        for (int j = 0; j < FN; ++j) acc[i][j] = floatx4{0.f, 0.f, 0.f, 0.f};
    for (int z = 0; z < st.split; ++z, from += T * T / 4)
#pragma unroll
        for (int i = 0; i < FM; ++i)
#pragma unroll
            for (int j = 0; j < FN; ++j) acc[i][j] += from[(i * FN + j) * (NW * 64) + threadIdx.x];
    to_lds<T, NWP, NWQ>(acc, out);
    __syncthreads();
    finish<STAGE, T, NW * 64>(a, st, s, out);
}

template <int STAGE, bool PAIR, int T, int NWP, int NWQ>
hipError_t launch_product(const OrthoArgs& a, StepArgs st, hipStream_t s)
{
    const int rows = a.np / T, tiles = a.batch * (STAGE == UPDATE ? rows * (a.mp / T) : rows * (rows + 1) / 2);
    st.split = STAGE == GRAM ? a.split_gram : STAGE == SQUARE ? a.split_square : a.split_update;
    ortho_product_kernel<STAGE, PAIR, T, NWP, NWQ><<<tiles * st.split, NWP * NWQ * 64, 0, s>>>(a, st);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || st.split == 1) return e;
    ortho_sum_kernel<STAGE, T, NWP, NWQ><<<tiles, NWP * NWQ * 64, 0, s>>>(a, st);
    return hipGetLastError();
}

template <bool PAIR, int T, int NWP, int NWQ>
hipError_t launch_step(const OrthoArgs& a, const StepArgs& st, hipStream_t s)
{
    hipError_t e = launch_product<GRAM, PAIR, T, NWP, NWQ>(a, st, s);
    if (e == hipSuccess) e = launch_product<SQUARE, PAIR, T, NWP, NWQ>(a, st, s);
    if (e == hipSuccess) e = launch_product<UPDATE, PAIR, T, NWP, NWQ>(a, st, s);
    return e;
}

int64_t round_up(int64_t v, int64_t by) { return (v + by - 1) / by * by; }
size_t region(size_t bytes) { return (bytes + 255) & ~(size_t)255; }

}  // namespace

OrthoPlan ortho_plan(const cbw_ortho_desc* d)
{
    OrthoPlan p{};
    const int64_t n = std::min(d->rows, d->cols), m = std::max(d->rows, d->cols);
    p.tile = n > 256 ? 128 : 64;
    p.np = (int)round_up(n, p.tile);
    p.mp = (int)round_up(m, p.tile);
    const int64_t elements = (int64_t)d->rows * d->cols;
    p.parts = (int)std::min<int64_t>(256, std::max<int64_t>(1, elements / 8192));
    const int64_t rows = p.np / p.tile, tri = d->batch * rows * (rows + 1) / 2, full = d->batch * rows * (p.mp / p.tile);
    auto split = [&](int64_t tiles, int64_t len) {
        return (int)std::max<int64_t>(1, std::min<int64_t>(CBW_NUM_CUS / std::max<int64_t>(tiles, 1), len / 64 / 2));
    };
    p.split_gram = split(tri, p.mp);
    p.split_square = split(tri, p.np);
    p.split_update = split(full, p.np);
    p.tiles = std::max(std::max(tri * p.split_gram, tri * p.split_square), full * p.split_update);
    size_t at = 0;
    auto take = [&](size_t bytes) {
        const size_t here = at;
        at += region(bytes);
        return here;
    };
    const size_t x = (size_t)d->batch * p.np * p.mp, g = (size_t)d->batch * p.np * p.np, t = (size_t)p.tile * p.tile * 4;
    p.partial = take((size_t)d->batch * p.parts * sizeof(double));
    p.x = take(x * 4);
    p.planes[0] = take(x * 4);
    p.planes[1] = take(x * 4);
    p.gram = take(g * 4);
    p.poly = take(g * 4);
    size_t sums = 0;
    if (p.split_gram > 1) sums = std::max(sums, (size_t)tri * p.split_gram * t);
    if (p.split_square > 1) sums = std::max(sums, (size_t)tri * p.split_square * t);
    if (p.split_update > 1) sums = std::max(sums, (size_t)full * p.split_update * t);
    p.sums = take(sums);
    p.ws_bytes = at;
    return p;
}

hipError_t launch_orthogonalize(const OrthoArgs& a, int tile, int steps, hipStream_t s)
{
    auto pair = [&](int k) { return a.out_f32 || k + 2 >= steps; };
    ortho_norm_kernel<<<a.batch * a.parts, 256, 0, s>>>(a);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    ortho_start_kernel<<<a.batch * (a.np / 64) * (a.mp / 64), 256, 0, s>>>(a, pair(0));
    if ((e = hipGetLastError()) != hipSuccess) return e;
    for (int k = 0; k < steps && e == hipSuccess; ++k) {
        StepArgs st{};
        st.from = k & 1;
        st.last = k + 1 == steps;
        st.pair = pair(k);
        st.next_pair = pair(k + 1);
        if (tile == 128) e = st.pair ? launch_step<true, 128, 2, 4>(a, st, s) : launch_step<false, 128, 2, 4>(a, st, s);
        else e = st.pair ? launch_step<true, 64, 2, 2>(a, st, s) : launch_step<false, 64, 2, 2>(a, st, s);
    }
    return e;
}

}  // namespace cbw
