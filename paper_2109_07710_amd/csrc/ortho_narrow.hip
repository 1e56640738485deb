// Orthogonalised updates of matrices with at most 64 rows (or columns): the
// same steps in float32 throughout.
//
// A and B of such a matrix fit a workgroup's LDS, so a workgroup with a panel of
// X's columns has all a step needs but the other panels' part of A:
//
//   A = the panels' sums of x x^T,  B = b A + c A A,  x = a x + B x
//
// A launch a step: every workgroup adds up the panels' parts of A itself, in
// order, and leaves its own part of the next one.  The launch before them takes
// every panel by its own norm; the first step knows them all and sets the panels
// and their parts right.  Matrices of one panel take one launch in all, from the
// norm to the update.  What bounds it are launches
// and latency: the float32 matrix instructions take 16 times the half-precision
// ones' time, and still only 2 us a step for 64 rows by 64 columns, and they
// keep the full 24 bits where few rows average few roundings out.
#include "common.hpp"
#include "block_kernels.hpp"
#include "ortho_io.hpp"
#include "tiles.hpp"

#include <algorithm>
#include <type_traits>

namespace cbw {
namespace {

constexpr int kWaves = 8, kThreads = kWaves * 64;

// NB blocks of 16 rows, panels of up to W columns.  The waves stand side by side
// over COLS blocks of 16 columns; with four blocks of rows, two waves share a
// block of columns and take half of what is to be computed each.  Rows lie four values more
// than their length apart, so that neither 16 rows' vectors nor a column's
// values share banks.
template <int NB, int W>
struct Narrow {
    static constexpr int NP = 16 * NB, LD = W + 4, LDA = NP + 4, TRI = NB * (NB + 1) / 2;
    static constexpr int SHARE = NB == 4 ? 2 : 1, COLS = kWaves / SHARE;
    float x[NP * LD];
    float a[NP * LDA];
    union {
        float b[NP * LDA];
        floatx4 parts[COLS][TRI][64];   // the waves' parts of A's blocks on and below the diagonal, while there is no B
        double sums[kWaves];            // of the norm, before either
    };
};

// block row and column of the t-th block on or below the diagonal
__device__ __forceinline__ constexpr int row_block(int t) { return t >= 6 ? 3 : t >= 3 ? 2 : t >= 1 ? 1 : 0; }
__device__ __forceinline__ void block_of(int t, int& bi, int& bj)
{
    bi = row_block(t);
    bj = t - bi * (bi + 1) / 2;
}

__device__ __forceinline__ floatx4 vector_at(const float* p) { return *reinterpret_cast<const floatx4*>(p); }

// acc[i] += the four products of a[i]'s and b[i]'s elements.  An instruction
// waits for the one before it on the same sum, so the sums take turns.
template <int I, typename A, typename B>
__device__ __forceinline__ void multiply(floatx4 (&acc)[I], const A& a, const B& b)
{
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int i = 0; i < I; ++i) acc[i] = __builtin_amdgcn_mfma_f32_16x16x4f32(a(i)[j], b(i)[j], acc[i], 0, 0, 0);
}

// The panel's x x^T, of which the waves take 16 columns in turn, into l.parts.
template <int NB, int W>
__device__ __forceinline__ void panel_gram(Narrow<NB, W>& l, int width)
{
    using N = Narrow<NB, W>;
    constexpr int MINE = N::TRI / N::SHARE;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, col = wave % N::COLS, t0 = wave / N::COLS * MINE;
    floatx4 acc[MINE] = {};
    // (the blocks' numbers are known to the compiler: the two halves are two loops)
    auto run = [&](auto half) {
        for (int c = col * 16; c < width; c += N::COLS * 16) {
            floatx4 f[NB];
#pragma unroll
            for (int b = 0; b < NB; ++b) f[b] = vector_at(l.x + (b * 16 + (lane & 15)) * N::LD + c + 4 * (lane >> 4));
            auto row = [&](int t) { return row_block(t + half.value * MINE); };
            multiply(acc, [&](int t) { return f[row(t)]; }, [&](int t) { return f[t + half.value * MINE - row(t) * (row(t) + 1) / 2]; });
        }
    };
    if (N::SHARE == 1 || t0 == 0) run(std::integral_constant<int, 0>());
    else run(std::integral_constant<int, N::SHARE - 1>());
#pragma unroll
    for (int t = 0; t < MINE; ++t) l.parts[col][t0 + t][lane] = acc[t];
}
// The sum of the waves' parts of A's t-th vector.
template <int NB, int W>
__device__ __forceinline__ floatx4 sum_of_parts(const Narrow<NB, W>& l, int t)
{
    floatx4 s = l.parts[0][t / 64][t % 64];
#pragma unroll
    for (int k = 1; k < Narrow<NB, W>::COLS; ++k) s += l.parts[k][t / 64][t % 64];
    return s;
}

// Four rows r .. r + 3 of column c of a symmetric matrix's block (bi, bj), into both places.
template <int LDA>
__device__ __forceinline__ void put_block(float* m, int bi, int bj, int lane, const floatx4& v)
{
    const int r = bi * 16 + 4 * (lane >> 4), c = bj * 16 + (lane & 15);
#pragma unroll
    for (int k = 0; k < 4; ++k) m[(r + k) * LDA + c] = v[k];
    if (bi != bj) *reinterpret_cast<floatx4*>(m + c * LDA + r) = v;
}

// B from A, both in LDS.
template <int NB, int W>
__device__ __forceinline__ void polynomial(Narrow<NB, W>& l, float cb, float cc)
{
    using N = Narrow<NB, W>;
    const int lane = threadIdx.x & 63;
    // a wave's blocks, wave, wave + 8 (one too many is the last block again)
    constexpr int MINE = (N::TRI + kWaves - 1) / kWaves;
    const int wave = threadIdx.x >> 6, r = lane & 15, k4 = 4 * (lane >> 4);
    int bi[MINE], bj[MINE];
#pragma unroll
    for (int i = 0; i < MINE; ++i) block_of(min(wave + kWaves * i, N::TRI - 1), bi[i], bj[i]);
    floatx4 s[MINE] = {};
#pragma unroll
    for (int k = 0; k < NB; ++k)
        multiply(s, [&](int i) { return vector_at(l.a + (bi[i] * 16 + r) * N::LDA + k * 16 + k4); },
                 [&](int i) { return vector_at(l.a + (bj[i] * 16 + r) * N::LDA + k * 16 + k4); });
#pragma unroll
    for (int i = 0; i < MINE; ++i) {
        if (wave + kWaves * i >= N::TRI) break;
#pragma unroll
        for (int k = 0; k < 4; ++k) s[i][k] = cb * l.a[(bi[i] * 16 + k4 + k) * N::LDA + bj[i] * 16 + r] + cc * s[i][k];
        put_block<N::LDA>(l.b, bi[i], bj[i], lane, s[i]);
    }
}

// x = a x + B x, 16 columns a wave at a time.  A lane's values of a column are
// the second operand and, the same ones, the places of the result.
template <int NB, int W>
__device__ __forceinline__ void panel_update(Narrow<NB, W>& l, int width, float ca)
{
    using N = Narrow<NB, W>;
    constexpr int MINE = NB / N::SHARE;   // blocks of rows of the result
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, col = wave % N::COLS, b0 = wave / N::COLS * MINE;
    for (int c0 = 0; c0 < width; c0 += N::COLS * 16) {
        const int c = c0 + col * 16;
        float* at = l.x + 4 * (lane >> 4) * N::LD + c + (lane & 15);
        floatx4 x[NB], s[MINE] = {};
        if (c < width) {
#pragma unroll
            for (int b = 0; b < NB; ++b)
#pragma unroll
                for (int k = 0; k < 4; ++k) x[b][k] = at[(b * 16 + k) * N::LD];
#pragma unroll
            for (int k = 0; k < NB; ++k)
                multiply(s, [&](int i) { return vector_at(l.b + ((b0 + i) * 16 + (lane & 15)) * N::LDA + k * 16 + 4 * (lane >> 4)); },
                         [&](int) { return x[k]; });
        }
        if (N::SHARE > 1) __syncthreads();   // the other wave has read its columns as well
        if (c < width)
#pragma unroll
            for (int i = 0; i < MINE; ++i)
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const float old = N::SHARE == 1 || b0 == 0 ? x[i][k] : x[MINE * (N::SHARE - 1) + i][k];
                    at[((b0 + i) * 16 + k) * N::LD] = ca * old + s[i][k];
                }
    }
}

// The panel's values of M (columns p0 on of X), zeros past the matrix; the
// thread's share of their sum of squares.
template <int NB, int W>
__device__ __forceinline__ double load_panel(Narrow<NB, W>& l, const OrthoArgs& a, int mat, int p0, int width)
{
    using N = Narrow<NB, W>;
    // vectors along M's rows: `across` of them to a row of the panel, or (tall) to a row of M
    const int across = (a.tall ? N::NP : width) / 8, vectors = N::NP * width / 8;
    const int64_t base = (int64_t)mat * a.rows * a.in_stride;
    const int size = a.in_f32 ? 4 : 2;
    double s = 0.0;
    constexpr int AHEAD = 4;   // vectors whose loads are in flight
    for (int t0 = threadIdx.x; t0 < vectors; t0 += AHEAD * kThreads) {
        float v[AHEAD][8];
#pragma unroll
        for (int h = 0; h < AHEAD; ++h) {
            const int t = t0 + h * kThreads, row = t / across + (a.tall ? p0 : 0), col = t % across * 8 + (a.tall ? 0 : p0);
            const int64_t at = base + row * a.in_stride + col;
            const bool in = t < vectors && row < a.rows;
            if (in && col + 8 <= a.cols && ((uintptr_t)a.m + at * size) % 16 == 0) {
                load_values(a.m, at, a.in_f32, v[h]);
            } else {
#pragma unroll
                for (int k = 0; k < 8; ++k) v[h][k] = in && col + k < a.cols ? load_value(a.m, at + k, a.in_f32) : 0.f;
            }
        }
#pragma unroll
        for (int h = 0; h < AHEAD; ++h) {
            const int t = t0 + h * kThreads, r = t / across, c = t % across * 8;
            if (t >= vectors) break;
            float* to = a.tall ? l.x + c * N::LD + r : l.x + r * N::LD + c;
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                to[k * (a.tall ? N::LD : 1)] = v[h][k];
                s += (double)v[h][k] * v[h][k];
            }
        }
    }
    return s;
}

// The panel times `inv`.  (Values past the matrix stay zero, also
// where the norm is no number.)
template <int NB, int W>
__device__ __forceinline__ void scale_panel(Narrow<NB, W>& l, const OrthoArgs& a, int p0, int width, double inv)
{
    using N = Narrow<NB, W>;
    const int n = a.tall ? a.cols : a.rows, m = a.tall ? a.rows : a.cols;
    for (int i = threadIdx.x >> 6; i < n; i += kWaves)
        for (int c = threadIdx.x & 63; c < min(width, m - p0); c += 64) l.x[i * N::LD + c] = (float)(l.x[i * N::LD + c] * inv);
}

// The sum of the threads' `s`, by way of l.sums.
template <int NB, int W>
__device__ __forceinline__ double block_sum(Narrow<NB, W>& l, double s)
{
    for (int k = 32; k >= 1; k >>= 1) s += __shfl_xor(s, k);
    if ((threadIdx.x & 63) == 0) l.sums[threadIdx.x >> 6] = s;
    __syncthreads();
    s = 0.0;
    for (int k = 0; k < kWaves; ++k) s += l.sums[k];
    return s;
}

template <int NB, int W>
__device__ __forceinline__ void store_panel(const Narrow<NB, W>& l, const OrthoArgs& a, int mat, int p0, int width)
{
    using N = Narrow<NB, W>;
    float v[8];
    if (a.tall) {
        for (int t = threadIdx.x; t < width * (N::NP / 8); t += kThreads) {
            const int c = t / (N::NP / 8), i = t % (N::NP / 8) * 8;
#pragma unroll
            for (int k = 0; k < 8; ++k) v[k] = l.x[(i + k) * N::LD + c];
            store_out(a, mat, p0 + c, i, v);
        }
    } else {
        for (int t = threadIdx.x; t < N::NP * (width / 8); t += kThreads) {
            const int i = t / (width / 8), c = t % (width / 8) * 8;
#pragma unroll
            for (int k = 0; k < 8; ++k) v[k] = l.x[i * N::LD + c + k];
            store_out(a, mat, i, p0 + c, v);
        }
    }
}

// A, from the waves' parts of one panel.
template <int NB, int W>
__device__ __forceinline__ void whole_gram(Narrow<NB, W>& l)
{
    using N = Narrow<NB, W>;
    for (int t = threadIdx.x; t < N::TRI * 64; t += kThreads) {
        int bi, bj;
        block_of(t / 64, bi, bj);
        put_block<N::LDA>(l.a, bi, bj, t % 64, sum_of_parts(l, t));
    }
}

// A matrix of one panel: a workgroup from the norm to the update.
template <int NB, int W>
__global__ __launch_bounds__(kThreads) void ortho_whole_kernel(OrthoArgs a, int width, int steps)
{
    __shared__ __align__(16) Narrow<NB, W> l;
    const int mat = blockIdx.x;
    const double s = block_sum(l, load_panel(l, a, mat, 0, width));
    scale_panel(l, a, 0, width, inverse_of(s, a.eps));
    for (int k = 0; k < steps; ++k) {
        __syncthreads();
        panel_gram(l, width);
        __syncthreads();
        whole_gram(l);
        __syncthreads();
        polynomial(l, a.b, a.c);
        __syncthreads();
        panel_update(l, width, a.a);
    }
    __syncthreads();
    store_panel(l, a, mat, 0, width);
}

// The panel and its part of A into the workspace, for the next step.
template <int NB, int W>
__device__ __forceinline__ void leave_panel(Narrow<NB, W>& l, const OrthoArgs& a, const PanelArgs& p, int mat, int panel, int to)
{
    using N = Narrow<NB, W>;
    float* x = a.x + ((int64_t)mat * p.panels + panel) * N::NP * p.width;
    for (int t = threadIdx.x; t < N::NP * (p.width / 4); t += kThreads) {
        const int i = t / (p.width / 4), c = t % (p.width / 4) * 4;
        *reinterpret_cast<floatx4*>(x + i * p.width + c) = *reinterpret_cast<const floatx4*>(l.x + i * N::LD + c);
    }
    panel_gram(l, p.width);
    __syncthreads();
    floatx4* part = reinterpret_cast<floatx4*>(a.sums) + (((int64_t)to * a.batch + mat) * p.panels + panel) * N::TRI * 64;
    for (int t = threadIdx.x; t < N::TRI * 64; t += kThreads) part[t] = sum_of_parts(l, t);
}

template <int NB, int W>
__global__ __launch_bounds__(kThreads) void ortho_first_kernel(OrthoArgs a, PanelArgs p)
{
    __shared__ __align__(16) Narrow<NB, W> l;
    const int mat = blockIdx.x / p.panels, panel = blockIdx.x - mat * p.panels;
    const double s = block_sum(l, load_panel(l, a, mat, panel * p.width, p.width));
    if (threadIdx.x == 0) a.partial[(int64_t)mat * p.panels + panel] = s;
    scale_panel(l, a, panel * p.width, p.width, s > 0.0 ? 1.0 / sqrt(s) : 0.0);
    __syncthreads();
    leave_panel(l, a, p, mat, panel, 0);
}

template <int NB, int W>
__global__ __launch_bounds__(kThreads) void ortho_step_kernel(OrthoArgs a, PanelArgs p)
{
    using N = Narrow<NB, W>;
    __shared__ __align__(16) N l;
    const int mat = blockIdx.x / p.panels, panel = blockIdx.x - mat * p.panels;
    const float* x = a.x + ((int64_t)mat * p.panels + panel) * N::NP * p.width;
    const floatx4* x4 = reinterpret_cast<const floatx4*>(x);
    constexpr int XV = 4;
    const int vectors = N::NP * (p.width / 4);
    floatx4 ahead[XV];   // the panel's first values, on their way while A is added up
#pragma unroll
    for (int h = 0; h < XV; ++h) ahead[h] = x4[min((int)threadIdx.x + h * kThreads, vectors - 1)];
    const floatx4* parts = reinterpret_cast<const floatx4*>(a.sums) + ((int64_t)p.from * a.batch + mat) * p.panels * N::TRI * 64;
    // a thread's vectors of A's blocks; eight parts' loads of all of them in flight
    constexpr int MINE = (N::TRI * 64 + kThreads - 1) / kThreads, AHEAD = 8;
    floatx4 v[AHEAD][MINE], s[MINE] = {};
    auto fetch = [&](int z) {
#pragma unroll
        for (int k = 0; k < AHEAD; ++k)
#pragma unroll
            for (int i = 0; i < MINE; ++i)
                v[k][i] = parts[(int64_t)min(z + k, p.panels - 1) * N::TRI * 64 + min((int)threadIdx.x + i * kThreads, N::TRI * 64 - 1)];
    };
    fetch(0);
    // The panels' own norms beside the matrix's, a lane a panel: what X was left
    // divided by too much, and the square of that for the parts of A.
    float own = 1.f, square = 1.f;
    if (p.first) {
        const int z = threadIdx.x & 63;
        const double mine = z < p.panels ? a.partial[(int64_t)mat * p.panels + z] : 0.0;
        double all = mine;
        for (int k = 32; k >= 1; k >>= 1) all += __shfl_xor(all, k);
        const double f = sqrt(mine) * inverse_of(all, a.eps);
        own = (float)f;
        square = (float)(f * f);
    }
    auto of_panel = [](float v, int z) { return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), z)); };
    for (int z = 0;; z += AHEAD) {
#pragma unroll
        for (int k = 0; k < AHEAD; ++k)
            if (z + k < p.panels) {
                const float w = of_panel(square, p.first ? z + k : 0);
#pragma unroll
                for (int i = 0; i < MINE; ++i) s[i] += w * v[k][i];
            }
        if (z + AHEAD >= p.panels) break;
        fetch(z + AHEAD);
    }
#pragma unroll
    for (int i = 0; i < MINE; ++i) {
        const int t = threadIdx.x + i * kThreads;
        if (t >= N::TRI * 64) break;
        int bi, bj;
        block_of(t / 64, bi, bj);
        put_block<N::LDA>(l.a, bi, bj, t % 64, s[i]);
    }
    const float scale = of_panel(own, p.first ? panel : 0);
    for (int t0 = threadIdx.x; t0 < vectors; t0 += XV * kThreads) {
        if (t0 != (int)threadIdx.x)
#pragma unroll
            for (int h = 0; h < XV; ++h) ahead[h] = x4[min(t0 + h * kThreads, vectors - 1)];
#pragma unroll
        for (int h = 0; h < XV; ++h) {
            const int t = t0 + h * kThreads, i = t / (p.width / 4), c = t % (p.width / 4) * 4;
            if (t < vectors) *reinterpret_cast<floatx4*>(l.x + i * N::LD + c) = scale * ahead[h];
        }
    }
    __syncthreads();
    polynomial(l, a.b, a.c);
    __syncthreads();
    panel_update(l, p.width, a.a);
    __syncthreads();
    if (p.last) store_panel(l, a, mat, panel * p.width, p.width);
    else leave_panel(l, a, p, mat, panel, p.from ^ 1);
}

template <int NB, int W>
hipError_t launch(const OrthoArgs& a, const OrthoPlan& plan, int steps, hipStream_t s)
{
    if (plan.panels == 1) {
        ortho_whole_kernel<NB, W><<<a.batch, kThreads, 0, s>>>(a, plan.width, steps);
        return hipGetLastError();
    }
    PanelArgs p{plan.width, plan.panels, 0, false, false};
    ortho_first_kernel<NB, W><<<a.batch * plan.panels, kThreads, 0, s>>>(a, p);
    hipError_t e = hipGetLastError();
    for (int k = 0; k < steps && e == hipSuccess; ++k) {
        p.from = k & 1;
        p.first = k == 0;
        p.last = k + 1 == steps;
        ortho_step_kernel<NB, W><<<a.batch * plan.panels, kThreads, 0, s>>>(a, p);
        e = hipGetLastError();
    }
    return e;
}

// columns of a panel, at most, and those that one workgroup takes through all steps
constexpr int widest(int rows) { return rows == 16 ? 2048 : rows == 32 ? 512 : 256; }
constexpr int whole(int rows) { return rows == 16 ? 2048 : rows == 32 ? 512 : 128; }
constexpr int kPanels = 24;
static_assert(kPanels <= 64, "a lane for each");

}  // namespace

bool ortho_narrow_plan(const cbw_ortho_desc* d, OrthoPlan* p)
{
    const int n = std::min(d->rows, d->cols), m = std::max(d->rows, d->cols);
    if (n > 64) return false;
    const int rows = n <= 16 ? 16 : n <= 32 ? 32 : 64;
    auto width = [&](int panels) { return ((m + panels - 1) / panels + 63) / 64 * 64; };
    int w = width(1);
    if (w > whole(rows)) {
        if (width(kPanels) > widest(rows)) return false;
        w = std::max(width(kPanels), rows == 16 ? 256 : rows == 32 ? 128 : 64);
        // Narrow panels are quicker, while there is a CU for each (64 x 576, one matrix
        // and 16 of them, us: 48.5 and 58.7, by 128 columns 55.6 and 60.0); past that
        // fewer are (22 x 63 x 773: 90.6 and 73.2; 32 x 24 x 3000 by 128, 512: 79, 68).
        // Four of 16 rows find room on a CU (100 x 10 x 3000 by 256, 2048: 88, 95).
        while (rows > 16 && (int64_t)d->batch * ((m + w - 1) / w) > CBW_NUM_CUS && 2 * w <= widest(rows)) w *= 2;
    }
    p->rows = rows;
    p->width = w;
    p->panels = (m + w - 1) / w;
    if (p->panels == 1) return true;
    const size_t tri = (size_t)(rows / 16) * (rows / 16 + 1) / 2 * 1024;
    size_t at = 0;
    p->partial = ortho_region(at, (size_t)d->batch * p->panels * sizeof(double));
    p->x = ortho_region(at, (size_t)d->batch * p->panels * rows * w * 4);
    p->sums = ortho_region(at, (size_t)d->batch * p->panels * tri * 2);
    p->ws_bytes = at;
    return true;
}

hipError_t launch_ortho_narrow(const OrthoArgs& a, const OrthoPlan& p, int steps, hipStream_t s)
{
    switch (p.rows) {
    case 16: return p.width <= 256 ? launch<1, 256>(a, p, steps, s) : launch<1, 2048>(a, p, steps, s);
    case 32: return p.width <= 128 ? launch<2, 128>(a, p, steps, s) : launch<2, 512>(a, p, steps, s);
    default: return p.width <= 64 ? launch<4, 64>(a, p, steps, s) : launch<4, 256>(a, p, steps, s);
    }
}

}  // namespace cbw
