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
// Every step takes both parts, whatever the type of the result.  High parts alone
// in the first steps would do for matrices whose singular values are alike, and
// for those only.  In an emulation of these roundings, four live rows of 1024 and
// three of five such steps leave an error of 5e-3 to 1e-2 of the 2-norm, where
// rounding the result to bf16 leaves 1.7e-3; one live row loses 1.5e-3 in its
// first step, so that no number of such steps follows from the sizes.  (2048 x
// 2048 to bf16: 505 us with three such steps, 676 without.)
#include "common.hpp"
#include "block_kernels.hpp"
#include "expert_tiles.hpp"
#include "ortho_io.hpp"
#include "tiles.hpp"

#include <algorithm>
#include <type_traits>

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

// Sums of squares of a matrix, in 64 bits: part z of a.parts takes every
// a.parts-th chunk.  Contiguous matrices are one long row.
constexpr int kChunk = 8192;
__global__ __launch_bounds__(256) void ortho_norm_kernel(OrthoArgs a)
{
    const int z = blockIdx.x % a.parts, mat = blockIdx.x / a.parts;
    const bool flat = a.in_stride == a.cols;
    const int64_t rows = flat ? 1 : a.rows, cols = flat ? (int64_t)a.rows * a.cols : a.cols;
    const int64_t chunks = (cols + kChunk - 1) / kChunk;
    const int64_t base = (int64_t)mat * a.rows * a.in_stride;
    const int size = a.in_f32 ? 4 : 2;
    double s = 0.0;
    for (int64_t u = z; u < rows * chunks; u += a.parts) {
        const int64_t row = u / chunks, c0 = (u - row * chunks) * kChunk;
        const int64_t first = base + row * a.in_stride + c0;
        const int n = (int)min((int64_t)kChunk, cols - c0);
        // up to the first 16-byte boundary, whole vectors, and the rest
        const int head = min(n, (int)((0 - ((uintptr_t)a.m + first * size)) % 16) / size), whole = (n - head) / 8;
        float v[4][8];   // four vectors' loads in flight
        for (int i = threadIdx.x; i < whole; i += 1024) {
#pragma unroll
            for (int k = 0; k < 4; ++k)
                load_values(a.m, first + head + (int64_t)min(i + k * 256, whole - 1) * 8, a.in_f32, v[k]);
#pragma unroll
            for (int k = 0; k < 4; ++k)
                if (i + k * 256 < whole)
#pragma unroll
                    for (int c = 0; c < 8; ++c) s += (double)v[k][c] * v[k][c];
        }
        // (fewer than eight on each side)
        const int i = (int)threadIdx.x < head ? (int)threadIdx.x : whole * 8 + (int)threadIdx.x;
        if ((int)threadIdx.x < n - whole * 8) {
            const double x = load_value(a.m, first + i, a.in_f32);
            s += x * x;
        }
    }
    __shared__ double sums[4];
    for (int k = 32; k >= 1; k >>= 1) s += __shfl_xor(s, k);
    if ((threadIdx.x & 63) == 0) sums[threadIdx.x >> 6] = s;
    __syncthreads();
    if (threadIdx.x == 0) a.partial[(int64_t)mat * a.parts + z] = sums[0] + sums[1] + sums[2] + sums[3];
}

// 1 / (|M| + eps) from the parts of the sum; called by whole waves.
__device__ __forceinline__ double inverse_norm(const OrthoArgs& a, int mat, bool& nothing)
{
    double s = 0.0;
    for (int z = threadIdx.x & 63; z < a.parts; z += 64) s += a.partial[(int64_t)mat * a.parts + z];
    for (int k = 32; k >= 1; k >>= 1) s += __shfl_xor(s, k);
    nothing = s == 0.0;
    return inverse_of(s, a.eps);
}

// Where a matrix's planes of `ld` columns hold the high part of (i, j); its low
// part lies kLow further.  32 high parts and the same columns' 32 low parts share
// 128 bytes, so that a step of a product's reduction is whole lines.
constexpr int kLow = 32;
struct Plane {
    int64_t mat;
    int ld;
    __device__ Plane(int which, int rows, int columns) : mat((int64_t)which * rows * columns * 2), ld(columns) {}
    __device__ __forceinline__ int64_t at(int i, int j) const { return mat + (int64_t)i * ld * 2 + (j >> 5) * 64 + (j & 31); }
};
__device__ __forceinline__ void put_pair(_Float16* at, const float (&v)[8])
{
    const Pair w = split(v);
    *reinterpret_cast<uint4*>(at) = w.hi;
    *reinterpret_cast<uint4*>(at + kLow) = w.lo;
}
__device__ __forceinline__ void put_x(const Plane& plane, _Float16* to, int i, int j, const float (&x)[8])
{
    float v[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) v[k] = x[k] * kX;
    put_pair(to + plane.at(i, j), v);
}

// X and its planes, 64 x 64 values a workgroup, zeros past the matrix.
__global__ __launch_bounds__(256) void ortho_start_kernel(OrthoArgs a)
{
    __shared__ float tile[64][65];
    const int bx = a.mp / 64, by = a.np / 64;
    const int mat = blockIdx.x / (bx * by), in = blockIdx.x - mat * (bx * by);
    const int i0 = in / bx * 64, j0 = in % bx * 64;   // of X

    const int64_t base = (int64_t)mat * a.rows * a.in_stride;
    const int size = a.in_f32 ? 4 : 2;
    const int r0 = a.tall ? j0 : i0, c0 = a.tall ? i0 : j0;   // of M
    float v[2][8];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const int t = threadIdx.x + h * 256, row = r0 + t / 8, col = c0 + t % 8 * 8;
        const int64_t at = base + row * a.in_stride + col;
        if (row < a.rows && col + 8 <= a.cols && ((uintptr_t)a.m + at * size) % 16 == 0) {
            load_values(a.m, at, a.in_f32, v[h]);
        } else {
#pragma unroll
            for (int k = 0; k < 8; ++k) v[h][k] = row < a.rows && col + k < a.cols ? load_value(a.m, at + k, a.in_f32) : 0.f;
        }
    }
    bool nothing;
    const double inv = inverse_norm(a, mat, nothing);
    if (in == 0 && threadIdx.x == 0) a.nothing[mat] = nothing;
    if (nothing) {
        // the products leave it out: its update is written here
        const float zeros[8] = {};
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int t = threadIdx.x + h * 256;
            store_out(a, mat, r0 + t / 8, c0 + t % 8 * 8, zeros);
        }
        return;
    }
    const Plane plane(mat, a.np, a.mp);
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const int t = threadIdx.x + h * 256, r = t / 8, c = t % 8 * 8;
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            // (values past the matrix stay zero, also where the norm is no number)
            v[h][k] = r0 + r < a.rows && c0 + c + k < a.cols ? (float)(v[h][k] * inv) : 0.f;
            if (a.tall) tile[c + k][r] = v[h][k];
        }
    }
    if (a.tall) __syncthreads();
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const int t = threadIdx.x + h * 256, i = t / 8, j = t % 8 * 8;
        if (a.tall)
#pragma unroll
            for (int k = 0; k < 8; ++k) v[h][k] = tile[i][j + k];
        float* x = a.x + (int64_t)mat * a.np * a.mp + (int64_t)(i0 + i) * a.mp + j0 + j;
        *reinterpret_cast<float4*>(x) = make_float4(v[h][0], v[h][1], v[h][2], v[h][3]);
        *reinterpret_cast<float4*>(x + 4) = make_float4(v[h][4], v[h][5], v[h][6], v[h][7]);
        put_x(plane, a.planes[0], i0 + i, j0 + j, v[h]);
    }
}

// ---------------------------------------------------------------- products

enum { GRAM = 0, SQUARE = 1, UPDATE = 2 };

// A tile's place: its matrix, rows i0 on, columns j0 on.
struct Spot {
    int mat, i0, j0;
};
// Matrices of zeros have no tiles, so that the others' are dealt out evenly
// over the chip: a lane looks at a matrix, up to 64 of them.
struct Tiles {
    uint64_t busy;
    int per, count;   // tiles of a matrix, and in all
    bool listed;
};
template <int STAGE, int T>
__device__ __forceinline__ Tiles tiles_of(const OrthoArgs& a)
{
    Tiles t;
    const int rows = (a.np + T - 1) / T, cols = (a.mp + T - 1) / T, lane = threadIdx.x & 63;
    t.per = STAGE == UPDATE ? rows * cols : rows * (rows + 1) / 2;
    // (one matrix is looked at only before its tiles are stored: that takes no time)
    t.listed = a.batch <= 64;
    t.busy = a.batch == 1 ? 1 : t.listed ? __ballot(lane < a.batch && a.nothing[lane < a.batch ? lane : 0] == 0) : 0;
    t.count = t.per * (t.listed ? __popcll(t.busy) : a.batch);
    return t;
}
template <int STAGE, int T>
__device__ __forceinline__ Spot spot_of(const OrthoArgs& a, const Tiles& tiles, int tile)
{
    Spot s;
    const int rows = (a.np + T - 1) / T;
    s.mat = tile / tiles.per;
    const int in = tile - s.mat * tiles.per;
    if (tiles.listed) {
        uint64_t m = tiles.busy;
        for (int k = 0; k < s.mat; ++k) m &= m - 1;
        s.mat = __builtin_ctzll(m);
    }
    // The tiles of one XCD, consecutive ones, lie in compact blocks, so that few
    // rows and columns of tiles pass its L2: what a product reads comes to every
    // XCD from the shared cache or memory.
    if (STAGE == UPDATE) {
        // panels of eight columns, row by row
        const int cols = (a.mp + T - 1) / T, panel = in / (8 * rows), w = min(8, cols - 8 * panel), at = in - panel * 8 * rows;
        s.i0 = at / w * T;
        s.j0 = (panel * 8 + at % w) * T;
    } else {
        // block rows of four tile rows, blocks of four columns from left to right,
        // the last one's part on and below the diagonal
        int b = 0, at = in, h = min(4, rows);
        for (int n = h * (h + 1) / 2; at >= n; n = 4 * b * h + h * (h + 1) / 2) {
            at -= n;
            ++b;
            h = min(4, rows - 4 * b);
        }
        int i = 0, j = 0;
        if (at < 4 * b * h) {
            const int block = at / (4 * h), left = at - block * 4 * h;
            i = left / 4;
            j = block * 4 + left % 4;
        } else {
            j = at - 4 * b * h;
            while (j > i) j -= ++i;   // row i of the corner has i + 1 tiles
            j += 4 * b;
        }
        s.i0 = (4 * b + i) * T;
        s.j0 = j * T;
    }
    // (the same in all lanes, which divisions hide)
    s.mat = __builtin_amdgcn_readfirstlane(s.mat);
    s.i0 = __builtin_amdgcn_readfirstlane(s.i0);
    s.j0 = __builtin_amdgcn_readfirstlane(s.j0);
    return s;
}

// How many of `count` tiles of 256 go as such, one to a CU at a time: whole
// turns of all CUs, and a last one that is nearly whole.  The rest go by
// quarters, two to a CU.
constexpr int kLeft = 199;   // (a turn of such tiles takes some 0.8 of a turn of as many quarters)
__device__ __forceinline__ int large_tiles(int count)
{
    const int rest = count % CBW_NUM_CUS;
    return rest > kLeft ? count : count - rest;
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

// The thread's number, which the compiler takes for a new one each time: it
// would keep all that follows from it in registers during the products.
__device__ __forceinline__ int my_thread()
{
    int t = threadIdx.x;
    asm volatile("" : "+v"(t));
    return t;
}

// What a finished T x T piece meets: X (B X) or A (A A), the thread's vectors of
// it, on their way while the sums are still being added up.
template <int STAGE, int T, int THREADS>
struct Meets {
    static constexpr int VECS = STAGE == GRAM ? 1 : T * T / 8 / THREADS;
    uint4 v[VECS][2];
    __device__ __forceinline__ void load(const OrthoArgs& a, const Spot& s)
    {
        if (STAGE == GRAM) return;
        const Plane square(s.mat, a.np, a.np);
        const int thread = my_thread();
#pragma unroll
        for (int k = 0; k < VECS; ++k) {
            const int t = thread + k * THREADS, q = t / (T / 8), p = t % (T / 8) * 8;
            if (STAGE == UPDATE) {
                const uint4* x = reinterpret_cast<const uint4*>(a.x + (int64_t)s.mat * a.np * a.mp + (int64_t)(s.i0 + q) * a.mp + s.j0 + p);
                v[k][0] = x[0];
                v[k][1] = x[1];
            } else {
                const _Float16* g = a.gram + square.at(s.i0 + q, s.j0 + p);
                v[k][0] = *reinterpret_cast<const uint4*>(g);
                v[k][1] = *reinterpret_cast<const uint4*>(g + kLow);
            }
        }
    }
};

// What becomes of a finished T x T piece of sums, in LDS: A or B into their
// planes, with `mirror` at the mirrored place too, X and its planes, or the update.
template <int STAGE, int T, int THREADS>
__device__ __forceinline__ void finish(const OrthoArgs& a, const StepArgs& st, const Spot& s, bool mirror,
                                       const Meets<STAGE, T, THREADS>& meets, float* tile)
{
    using Sq = Square<T>;
    const bool turned = STAGE == UPDATE && st.last && a.tall;
    _Float16* out = STAGE == GRAM ? a.gram : a.poly;
    const Plane square(s.mat, a.np, a.np), wide(s.mat, a.np, a.mp);
    auto put = [&](int i, int j, const float (&v)[8]) { put_pair(out + square.at(i, j), v); };
    const int thread = my_thread();
#pragma unroll
    for (int u = 0; u < T * T / 8 / THREADS; ++u) {
        const int t = thread + u * THREADS, q = t / (T / 8), p = t % (T / 8) * 8;
        float v[8];
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            const floatx4 x = *reinterpret_cast<const floatx4*>(Sq::chunk(tile, q, p / 4 + k));
#pragma unroll
            for (int c = 0; c < 4; ++c) v[4 * k + c] = x[c];
        }
        if (STAGE == UPDATE) {
            float* at = a.x + (int64_t)s.mat * a.np * a.mp + (int64_t)(s.i0 + q) * a.mp + s.j0 + p;
            const floatx4 x0 = __builtin_bit_cast(floatx4, meets.v[u][0]), x1 = __builtin_bit_cast(floatx4, meets.v[u][1]);
            const float x[8] = {x0[0], x0[1], x0[2], x0[3], x1[0], x1[1], x1[2], x1[3]};
#pragma unroll
            for (int k = 0; k < 8; ++k) v[k] = a.a * x[k] + v[k] * (1.f / (kB * kX));
            if (!st.last) {
                *reinterpret_cast<float4*>(at) = make_float4(v[0], v[1], v[2], v[3]);
                *reinterpret_cast<float4*>(at + 4) = make_float4(v[4], v[5], v[6], v[7]);
                put_x(wide, a.planes[st.from ^ 1], s.i0 + q, s.j0 + p, v);
            } else if (!a.tall) {
                store_out(a, s.mat, s.i0 + q, s.j0 + p, v);
            }
        } else {
            if (STAGE == GRAM) {
#pragma unroll
                for (int k = 0; k < 8; ++k) v[k] *= kA / (kX * kX);
            } else {
                float x[8];
                join(Pair{meets.v[u][0], meets.v[u][1]}, x);
#pragma unroll
                for (int k = 0; k < 8; ++k) v[k] = (a.b * (kB / kA)) * x[k] + (a.c * (kB / (kA * kA))) * v[k];
            }
            put(s.i0 + q, s.j0 + p, v);
        }
        if (mirror || turned) {
#pragma unroll
            for (int k = 0; k < 2; ++k)
                *reinterpret_cast<floatx4*>(Sq::chunk(tile, q, p / 4 + k)) = floatx4{v[4 * k], v[4 * k + 1], v[4 * k + 2], v[4 * k + 3]};
        }
    }
    if (!mirror && !turned) return;
    __syncthreads();
    for (int t = thread; t < T * T / 8; t += THREADS) {
        const int p = t / (T / 8), q = t % (T / 8) * 8;
        float v[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] = *Sq::value(tile, q + k, p);
        if (STAGE == UPDATE) store_out(a, s.mat, s.j0 + p, s.i0 + q, v);
        else put(s.j0 + p, s.i0 + q, v);
    }
}

// A finished tile, as the matrix instructions leave it.
template <int STAGE, int T, int NWP, int NWQ, int FM, int FN>
__device__ __forceinline__ void finish_tile(const OrthoArgs& a, const StepArgs& st, const Spot& s, const floatx4 (&acc)[FM][FN],
                                            const Meets<STAGE, T, NWP * NWQ * 64>& meets, float* lds)
{
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wp = wave / NWQ, wq = wave % NWQ, lane = my_thread() & 63;
    __syncthreads();   // every wave is done with the operands
#pragma unroll
    for (int i = 0; i < FM; ++i)
#pragma unroll
        for (int j = 0; j < FN; ++j)
            *reinterpret_cast<floatx4*>(Square<T>::chunk(lds, wq * (T / NWQ) + j * 16 + (lane & 15),
                                                         (wp * (T / NWP) + i * 16) / 4 + (lane >> 4))) = acc[i][j];
    __syncthreads();
    finish<STAGE, T, NWP * NWQ * 64>(a, st, s, STAGE != UPDATE && s.i0 != s.j0, meets, lds);
}

// 32 rows of the planes of pairs, T columns from the base on, as 64 LDS lines of
// T values: the rows' high parts, then their low ones.
template <int T, int NW>
struct PairsAcross {
    using O = Operand<uint16_t, T, true, NW>;
    static constexpr int COPIES = O::COPIES, CHUNKS = O::CHUNKS;
    uint32_t off[COPIES];
    __device__ __forceinline__ void init(int wave, int n, int64_t ld)
    {
#pragma unroll
        for (int j = 0; j < COPIES; ++j) {
            const int at = (wave + NW * j) * 64 + (threadIdx.x & 63), line = at / CHUNKS, lc = (at % CHUNKS) ^ O::swizzle(line);
            off[j] = lc * 8 >= n ? kOOB : (uint32_t)((line & 31) * ld * 2 + (line >> 5) * 32 + (lc >> 2) * 64 + (lc & 3) * 8) * 2u;
        }
    }
    __device__ __forceinline__ void copy(int wave, const u32x4_t& rsrc, char* lds) const
    {
#pragma unroll
        for (int j = 0; j < COPIES; ++j) buf_load16_lds(rsrc, off[j], lds_addr(lds + (wave + NW * j) * 1024));
    }
};

// A tile's operands, as they come into LDS: from step `first` on.  A step is 128
// bytes of both: 32 reduction indices.
constexpr int kStep = 32;
template <int STAGE, int T, int NW>
struct Feed {
    using Along = Operand<uint16_t, T, false, NW>;
    using OP = Operand<uint16_t, T, STAGE == UPDATE, NW>;   // (across: as its fragments are read)
    using OQ = Along;
    static constexpr int COPIES = OP::COPIES + OQ::COPIES, TILE = OP::BYTES, STEP = 2 * TILE;
    std::conditional_t<STAGE == UPDATE, PairsAcross<T, NW>, Along> op;
    OQ oq;
    const _Float16 *pb, *qb;
    int64_t pld, qld;
    int first, vp, vq;   // columns and rows there are

    __device__ __forceinline__ Feed(const OrthoArgs& a, const StepArgs& st, const Spot& s, int wave, int at) : first(at)
    {
        pld = (STAGE == SQUARE ? a.np : a.mp) * 2;
        qld = (STAGE == GRAM ? a.mp : a.np) * 2;
        vq = min(T, a.np - s.i0);
        vp = min(T, (STAGE == UPDATE ? a.mp : a.np) - s.j0);
        const Plane xs(s.mat, a.np, a.mp), gs(s.mat, a.np, a.np);
        const _Float16* x = a.planes[st.from];
        pb = STAGE == GRAM ? x + xs.at(s.j0, 0) : STAGE == SQUARE ? a.gram + gs.at(s.j0, 0) : x + xs.at(0, s.j0);
        qb = STAGE == GRAM ? x + xs.at(s.i0, 0) : STAGE == SQUARE ? a.gram + gs.at(s.i0, 0) : a.poly + gs.at(s.i0, 0);
        pb = uniform(pb);
        qb = uniform(qb);
        oq.init(wave, 0, qld);
        if constexpr (STAGE == UPDATE) op.init(wave, vp, a.mp);
        else op.init(wave, 0, pld);
    }
    static __device__ __forceinline__ const _Float16* uniform(const _Float16* p)
    {
        const uint64_t a = reinterpret_cast<uint64_t>(p);
        const uint32_t lo = __builtin_amdgcn_readfirstlane((int)a), hi = __builtin_amdgcn_readfirstlane((int)(a >> 32));
        return reinterpret_cast<const _Float16*>((uint64_t)hi << 32 | lo);
    }
    // The same, with offsets that the compiler takes for new ones: it would work
    // out those of all copies ahead and fill registers.
    __device__ __forceinline__ Feed here() const
    {
        Feed f = *this;
        auto hold = [](auto& o) {
#pragma unroll
            for (int j = 0; j < (int)(sizeof(o.off) / 4); ++j) asm volatile("" : "+v"(o.off[j]));
        };
        hold(f.op);
        hold(f.oq);
        return f;
    }
    __device__ __forceinline__ void copy(int wave, int step, char* to) const
    {
        const int64_t k = first + step;
        if constexpr (STAGE == UPDATE)
            op.copy(wave, make_rsrc_words(pb + k * kStep * pld, (uint32_t)(((kStep - 1) * pld + vp * 2) * 2)), to);
        else
            op.copy(wave, make_rsrc_words(pb + k * 64, (uint32_t)(((vp - 1) * pld + 64) * 2)), 0, 64, to);
        oq.copy(wave, make_rsrc_words(qb + k * 64, (uint32_t)(((vq - 1) * qld + 64) * 2)), 0, 64, to + TILE);
    }
};

// T x T tiles by NWP x NWQ waves.  SUB of them go from one barrier to
// the next, and as many again are on their way into LDS meanwhile.
//
// The steps of a tile are shared out to st.split workgroups, whose sums go to
// memory where there are several; a launch of their own adds them up.
//
// What bounds them: tiles of 128 run at 1030 to 1070 TFLOP/s of fp16 products
// where they fill the chip (7 matrices 4096 x 2048: A 358 us, A A 191, B X 675), a
// library product at 1200 to 1260.  One matrix of 2048 x 2048 has 136 tiles for
// 256 CUs (A 41 us).  Tiles of 64 wait: 0.5 us a step for 0.1 of matrix
// instructions, and 4 to 5 a launch.  (Counting them in and leaving that to the
// last workgroup of a tile took a fence for the whole device in each, and 98 us
// in place of 28 for A of 2048 x 2048 values, 136 tiles in 256 ranges.)
template <int STAGE, int T, int NWP, int NWQ, int SUB>
__global__ __launch_bounds__(NWP* NWQ * 64) void ortho_product_kernel(OrthoArgs a, StepArgs st)
{
    constexpr int NW = NWP * NWQ, FM = T / NWP / 16, FN = T / NWQ / 16;
    using Fd = Feed<STAGE, T, NW>;
    using OP = typename Fd::OP;
    using OQ = typename Fd::OQ;
    constexpr int COPIES = Fd::COPIES, TILE = Fd::TILE, STEP = Fd::STEP;
    constexpr int RING = 2 * SUB;
    __shared__ __align__(1024) char lds[RING * STEP > T * T * 4 ? RING * STEP : T * T * 4];

    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wp = wave / NWQ, wq = wave % NWQ;
    const int len = (STAGE == GRAM ? a.mp : a.np) / kStep;         // steps of a tile
    const bool quarters = STAGE != UPDATE && T == 128 && st.quarters;
    const Tiles tiles = quarters ? tiles_of<STAGE, 256>(a) : tiles_of<STAGE, T>(a);
    const int taken = quarters ? large_tiles(tiles.count) : 0;
    const int units = quarters ? (tiles.count - taken) * 4 : tiles.count * st.split;
    if ((int)blockIdx.x >= units) return;
    const int me = xcd_remap(blockIdx.x, units), tile = quarters ? taken + me / 4 : me / st.split;
    const int part = quarters ? 0 : me - tile * st.split;
    const int first = (int)((int64_t)part * len / st.split), steps = (int)((int64_t)(part + 1) * len / st.split) - first;
    Spot s = quarters ? spot_of<STAGE, 256>(a, tiles, tile) : spot_of<STAGE, T>(a, tiles, tile);
    if (quarters) {
        s.i0 += me % 4 / 2 * T;
        s.j0 += me % 2 * T;
        if (s.i0 >= a.np || s.j0 > s.i0) return;
    }
    if (!tiles.listed && a.nothing[s.mat] != 0) return;

    const int frag_p = OP::first(wp * (T / NWP)), frag_q = OQ::first(wq * (T / NWQ));

    const int nothing = a.nothing[0];
    Meets<STAGE, T, NW * 64> meets;
    if (T == 64 && st.split == 1) meets.load(a, s);
    const Fd feed(a, st, s, wave, first);
    auto copy = [&](int step) { feed.copy(wave, step, lds + step % RING * STEP); };

    floatx4 acc[FM][FN];
#pragma unroll
    for (int i = 0; i < FM; ++i)
#pragma unroll
        for (int j = 0; j < FN; ++j) acc[i][j] = floatx4{0.f, 0.f, 0.f, 0.f};
    auto multiply = [&](const uint4 (&p)[FM], const uint4 (&q)[FN]) {
#pragma unroll
        for (int i = 0; i < FM; ++i)
#pragma unroll
            for (int j = 0; j < FN; ++j) acc[i][j] = mfma_half(acc[i][j], p[i], q[j]);
    };
    // A step's fragments: its high and low parts.
    struct Fragments {
        uint4 p[2][FM], q[2][FN];
    };
    auto read = [&](Fragments& f, int step) {
        const char* at = lds + step % RING * STEP;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            OQ::fragments(at + TILE, frag_q, h, f.q[h]);
            OP::fragments(at, frag_p, h, f.p[h]);
        }
    };
    auto product = [&](const Fragments& f) {
        multiply(f.p[0], f.q[0]);
        multiply(f.p[0], f.q[1]);
        multiply(f.p[1], f.q[0]);
        // one or two reads between every few matrix instructions
        constexpr int READS = 2 * (FM * (STAGE == UPDATE ? 2 : 1) + FN), MUL = FM * FN * 3;
#pragma unroll
        for (int i = 0; i < READS; ++i) {
            __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);                    // an LDS read
            __builtin_amdgcn_sched_group_barrier(0x008, MUL / READS, 0);          // matrix instructions
        }
    };
    // from one barrier to the next: the following steps' copies have landed
    // everywhere, and the places of those from `k` on are free
    auto turn = [&](int k) {
        wait_copies<0>();
        wait_reads();
        barrier();
#pragma unroll
        for (int u = 0; u < SUB; ++u)
            if (k + RING + u < steps) copy(k + RING + u);
    };

#pragma unroll
    for (int k = 0; k < RING; ++k)
        if (k < steps) copy(k);
    if (RING <= steps) wait_copies<SUB * COPIES>();
    else wait_copies<0>();
    barrier();
    // While a step's matrix instructions run, the next one's fragments are read.
    Fragments f[2];
    read(f[0], 0);
    for (int k0 = 0; k0 < steps; k0 += 2) {
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const int k = k0 + u;
            if (u > 0 && k >= steps) break;
            if (SUB == 1 || u > 0) turn(k + 1 - SUB);
            read(f[u ^ 1], k + 1);   // (after the last step: what was there, unused)
            product(f[u]);
        }
    }

    if (st.split > 1) {
        // as the registers lie, a wave's together
        floatx4* mine = reinterpret_cast<floatx4*>(a.sums) + (int64_t)me * (T * T / 4) + wave * (FM * FN * 64) + (my_thread() & 63);
#pragma unroll
        for (int i = 0; i < FM; ++i)
#pragma unroll
            for (int j = 0; j < FN; ++j) mine[(i * FN + j) * 64] = acc[i][j];
    } else {
        if (a.batch == 1 && nothing) return;
        // (tiles of 64 have the registers to ask for it at the start)
        if (T > 64) meets.load(a, s);
        finish_tile<STAGE, T, NWP, NWQ>(a, st, s, acc, meets, reinterpret_cast<float*>(lds));
    }
}

// A and A A of large batches: 256 x 256 tiles by eight waves, two buffers of a
// step.  A wave's 64 x 128 sums leave registers for two sets of fragments,
// which take turns:
//
//   hi hi (meanwhile the low parts are read), lo hi, and behind the barrier hi lo
//   (and the next step's high parts, into the sets that are free: those of the
//   columns change places each step)
//
// (7 of 8 matrices 4096 x 2048, us, tiles of 128 and of 256: A 358 and 284, A A
// 191 and 160.  B X gained nothing, 686 and 682.)
template <int STAGE>
__global__ __launch_bounds__(512) void ortho_large_kernel(OrthoArgs a, StepArgs st)
{
    static_assert(STAGE != UPDATE, "see above");
    constexpr int T = 256, NWQ = 4, FM = 8, FN = 4;
    using Fd = Feed<STAGE, T, 8>;
    using OP = typename Fd::OP;
    using OQ = typename Fd::OQ;
    __shared__ __align__(1024) char lds[2 * Fd::STEP];
    static_assert(sizeof(lds) >= 128 * 128 * 4, "a quarter of a finished tile");

    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wp = wave / NWQ, wq = wave % NWQ;
    const int steps = (STAGE == GRAM ? a.mp : a.np) / kStep;   // an even number: sizes are multiples of 128
    const Tiles tiles = tiles_of<STAGE, T>(a);
    const int count = large_tiles(tiles.count);
    if ((int)blockIdx.x >= count) return;
    const Spot s = spot_of<STAGE, T>(a, tiles, xcd_remap(blockIdx.x, count));
    if ((a.batch == 1 || !tiles.listed) && a.nothing[s.mat] != 0) return;
    const int frag_p = OP::first(wp * (T / 2)), frag_q = OQ::first(wq * (T / NWQ));
    const Fd feed(a, st, s, wave, 0);
    auto copy = [&](const Fd& f, int step) { f.copy(wave, step, lds + (step & 1) * Fd::STEP); };

    floatx4 acc[FM][FN];
#pragma unroll
    for (int i = 0; i < FM; ++i)
#pragma unroll
        for (int j = 0; j < FN; ++j) acc[i][j] = floatx4{0.f, 0.f, 0.f, 0.f};
    uint4 p[2][FM], q[2][FN];
    auto read = [&](int buf, int half, int to_p, int to_q) {
        const char* at = lds + buf * Fd::STEP;
        OQ::fragments(at + Fd::TILE, frag_q, half, q[to_q]);
        OP::fragments(at, frag_p, half, p[to_p]);
    };
    auto multiply = [&](int of_p, int of_q) {
#pragma unroll
        for (int i = 0; i < FM; ++i)
#pragma unroll
            for (int j = 0; j < FN; ++j) acc[i][j] = mfma_half(acc[i][j], p[of_p][i], q[of_q][j]);
    };
    auto interleave = [&]() {
        constexpr int READS = FM + FN, MUL = FM * FN;
#pragma unroll
        for (int i = 0; i < READS; ++i) {
            __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);                    // an LDS read
            __builtin_amdgcn_sched_group_barrier(0x008, MUL / READS, 0);          // matrix instructions
        }
    };
    copy(feed.here(), 0);
    copy(feed.here(), 1);
    wait_copies<Fd::COPIES>();
    barrier();
    read(0, 0, 0, 0);
    for (int k0 = 0; k0 < steps; k0 += 2) {
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const int k = k0 + u, hi = u;
            read(u, 1, hi ^ 1, 1);
            multiply(hi, 0);
            interleave();
            multiply(hi ^ 1, 0);
            __builtin_amdgcn_sched_barrier(0);
            const Fd next = feed.here();
            wait_copies<0>();
            wait_reads();
            barrier();
            if (k + 2 < steps) copy(next, k + 2);
            read(u ^ 1, 0, hi ^ 1, 0);   // (after the last step: what was there, unused)
            multiply(hi, 1);
            interleave();
            __builtin_amdgcn_sched_barrier(0);   // (the next reads have no registers yet)
        }
    }
    wait_reads();
    float* tile = reinterpret_cast<float*>(lds);   // a quarter at a time
#pragma unroll
    for (int n = 0; n < 4; ++n) {
        const int hq = n >> 1, hp = n & 1;
        const Spot part{s.mat, s.i0 + hq * 128, s.j0 + hp * 128};
        if (part.i0 >= a.np || part.j0 > part.i0) continue;   // (past the matrix; the mirrored quarter's)
        Meets<STAGE, 128, 512> meets;
        meets.load(a, part);
        __syncthreads();   // every wave is done with the operands, or the quarter before
        if (wp == hp && wq >> 1 == hq) {
            const int lane = my_thread() & 63;
#pragma unroll
            for (int i = 0; i < FM; ++i)
#pragma unroll
                for (int j = 0; j < FN; ++j)
                    *reinterpret_cast<floatx4*>(Square<128>::chunk(tile, (wq & 1) * 64 + j * 16 + (lane & 15), i * 4 + (lane >> 4))) = acc[i][j];
        }
        __syncthreads();
        finish<STAGE, 128, 512>(a, st, part, part.i0 != part.j0, meets, tile);
    }
}

// The parts of split tiles of 64 x 64, added in order, and what becomes of them.
// A workgroup takes a quarter, what one wave left, so that the loads of most
// splits are in flight at once (256 x 2304, ten tiles in twelve parts, a whole
// call: 128.8 us for 139.3 with a workgroup a tile).
template <int STAGE>
__global__ __launch_bounds__(128) void ortho_sum_kernel(OrthoArgs a, StepArgs st)
{
    constexpr int T = 64, S = T / 2, THREADS = 128;
    __shared__ __align__(1024) float lds[S * S];
    const Tiles tiles = tiles_of<STAGE, T>(a);
    const int tile = blockIdx.x / 4, quarter = blockIdx.x % 4;
    if (tile >= tiles.count) return;
    const Spot s = spot_of<STAGE, T>(a, tiles, tile);
    if (!tiles.listed && a.nothing[s.mat] != 0) return;
    const Spot part{s.mat, s.i0 + quarter % 2 * S, s.j0 + quarter / 2 * S};
    const int nothing = a.nothing[0];
    Meets<STAGE, S, THREADS> meets;
    meets.load(a, part);
    const floatx4* sums = reinterpret_cast<const floatx4*>(a.sums) + (int64_t)tile * st.split * (T * T / 4) + quarter * (S * S / 4) + threadIdx.x;
    floatx4 acc[2] = {};
    constexpr int AHEAD = 12;   // parts whose loads are in flight
    for (int z = 0; z < st.split; z += AHEAD) {
        floatx4 v[AHEAD][2];
#pragma unroll
        for (int k = 0; k < AHEAD; ++k)
#pragma unroll
            for (int h = 0; h < 2; ++h) v[k][h] = sums[(int64_t)min(z + k, st.split - 1) * (T * T / 4) + h * THREADS];
#pragma unroll
        for (int k = 0; k < AHEAD; ++k)
            if (z + k < st.split)
#pragma unroll
                for (int h = 0; h < 2; ++h) acc[h] += v[k][h];
    }
    if (a.batch == 1 && nothing) return;
    // vector n is lane n % 64's of fragment (n / 128, n / 64 % 2)
#pragma unroll
    for (int h = 0; h < 2; ++h)
        *reinterpret_cast<floatx4*>(Square<S>::chunk(lds, (threadIdx.x >> 6) * 16 + (threadIdx.x & 15), h * 4 + (threadIdx.x >> 4 & 3))) = acc[h];
    __syncthreads();
    finish<STAGE, S, THREADS>(a, st, part, STAGE != UPDATE && s.i0 != s.j0, meets, lds);
}

template <int STAGE, int T, int NWP, int NWQ, int SUB>
hipError_t launch_tiles(const OrthoArgs& a, StepArgs st, const OrthoDeal& d, hipStream_t s)
{
    st.split = d.split;
    ortho_product_kernel<STAGE, T, NWP, NWQ, SUB><<<d.tiles * d.split, NWP * NWQ * 64, 0, s>>>(a, st);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || d.split == 1) return e;
    if constexpr (T == 64) ortho_sum_kernel<STAGE><<<4 * d.tiles, 128, 0, s>>>(a, st);
    return hipGetLastError();
}

template <int STAGE>
hipError_t launch_product(const OrthoArgs& a, const StepArgs& st, const OrthoDeal& d, hipStream_t s)
{
    switch (d.side) {
    case 256:
        if constexpr (STAGE != UPDATE) {
            // (how many there are without the matrices of zeros, the kernels find)
            ortho_large_kernel<STAGE><<<d.tiles, 512, 0, s>>>(a, st);
            const hipError_t e = hipGetLastError();
            if (e != hipSuccess) return e;
            StepArgs rest = st;
            rest.quarters = true;
            return launch_tiles<STAGE, 128, 2, 2, 1>(a, rest, {128, 4 * std::min(d.tiles, kLeft), 1}, s);
        }
    case 128:
        // two workgroups to a CU where there are as many, else twice the steps to a
        // barrier and twice the waves (2048 x 2048, A | A A | B X, us: 40 | 41 | 50 for
        // 52 | 53 | 60 with four waves and half the steps, and 44 | 45 | 52 with half
        // the steps)
        if (d.tiles > CBW_NUM_CUS) return launch_tiles<STAGE, 128, 2, 2, 1>(a, st, d, s);
        return launch_tiles<STAGE, 128, 2, 4, 2>(a, st, d, s);
    default:
        if (d.tiles * d.split > 2 * CBW_NUM_CUS) return launch_tiles<STAGE, 64, 2, 2, 1>(a, st, d, s);
        return launch_tiles<STAGE, 64, 2, 2, 2>(a, st, d, s);
    }
}

int64_t round_up(int64_t v, int64_t by) { return (v + by - 1) / by * by; }

// How a product of `tiles(side)` tiles of `len` reduction indices is dealt out.
// Tiles of 64 take some 0.5 us a step beside 4.4 for the start and the end; the
// parts of a split one and the launch that adds them up 7.5 beside their steps,
// and 0.25 a part.  (With 5.5 there more tiles were split, and calls took, us: 400 x
// 2000 198 for 164, 6 x 300 x 700 199 for 173, 3 x 333 x 1001 175 for 166; with
// 4.5, 256 x 2304 166 for 128; with 9.5 as with 7.5.)
template <typename F>
OrthoDeal deal(F tiles, int64_t len, bool by128, bool by256)
{
    OrthoDeal d{};
    // (those of 128 are finished whole: both sides are filled up to that)
    d.side = by256 && tiles(256) > kLeft ? 256 : by128 && tiles(128) >= 128 ? 128 : 64;
    d.tiles = (int)tiles(d.side);
    d.split = 1;
    const int64_t steps = len / kStep;
    double best = 4.4 + 0.5 * (double)steps - 1.0;   // (no split for less than 1 us)
    for (int s = 2; d.side == 64 && s <= steps && s <= 24 && (int64_t)d.tiles * s <= 2 * CBW_NUM_CUS; ++s) {
        const double us = 7.5 + 0.25 * s + 0.5 * (double)((steps + s - 1) / s);
        if (us < best) {
            best = us;
            d.split = s;
        }
    }
    return d;
}

}  // namespace

OrthoPlan ortho_plan(const cbw_ortho_desc* d)
{
    OrthoPlan p{};
    const int64_t n = std::min(d->rows, d->cols), m = std::max(d->rows, d->cols);
    if (ortho_narrow_plan(d, &p)) return p;
    p.np = (int)round_up(n, n > 256 ? 128 : 64);
    p.mp = (int)round_up(m, n > 256 ? 128 : 64);
    p.parts = (int)std::min<int64_t>(512, std::max<int64_t>(1, (int64_t)d->rows * d->cols / 8192));
    size_t sums = 0;
    for (int k = 0; k < 3; ++k) {
        auto tiles = [&](int side) {
            const int64_t rows = (p.np + side - 1) / side, cols = (p.mp + side - 1) / side;
            return d->batch * (k == UPDATE ? rows * cols : rows * (rows + 1) / 2);
        };
        OrthoDeal& e = p.deal[k];
        const bool by128 = p.np % 128 == 0 && p.mp % 128 == 0;
        e = deal(tiles, k == GRAM ? p.mp : p.np, by128, by128 && k != UPDATE);
        if (e.split > 1) sums = std::max(sums, (size_t)e.tiles * e.split * e.side * e.side * 4);
    }
    size_t at = 0;
    auto take = [&](size_t bytes) { return ortho_region(at, bytes); };
    const size_t x = (size_t)d->batch * p.np * p.mp, g = (size_t)d->batch * p.np * p.np;
    p.partial = take((size_t)d->batch * p.parts * sizeof(double));
    p.nothing = take((size_t)d->batch * 4);
    p.x = take(x * 4);
    p.planes[0] = take(x * 4);
    p.planes[1] = take(x * 4);
    p.gram = take(g * 4);
    p.poly = take(g * 4);
    p.sums = take(sums);
    p.ws_bytes = at;
    return p;
}

hipError_t launch_orthogonalize(const OrthoArgs& a, const OrthoPlan& p, int steps, hipStream_t s)
{
    if (p.rows) return launch_ortho_narrow(a, p, steps, s);
    ortho_norm_kernel<<<a.batch * a.parts, 256, 0, s>>>(a);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    ortho_start_kernel<<<a.batch * (a.np / 64) * (a.mp / 64), 256, 0, s>>>(a);
    if ((e = hipGetLastError()) != hipSuccess) return e;
    for (int k = 0; k < steps && e == hipSuccess; ++k) {
        StepArgs st{};
        st.from = k & 1;
        st.last = k + 1 == steps;
        e = launch_product<GRAM>(a, st, p.deal[GRAM], s);
        if (e == hipSuccess) e = launch_product<SQUARE>(a, st, p.deal[SQUARE], s);
        if (e == hipSuccess) e = launch_product<UPDATE>(a, st, p.deal[UPDATE], s);
    }
    return e;
}

}  // namespace cbw
