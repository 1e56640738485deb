// A gated layer's products grouped by expert on the gfx950 matrix cores, and
// their gradients behind the next filter.
//
//   forward    g[r,k] = sum_c X[r,c] Wg[e,k,c],  u[r,k] = sum_c X[r,c] Wu[e,k,c]
//              H[r,k] = act(g) u
//   backward   dH[r,k] = sum_c dY[r,c] W2[e,c,k]
//              dg = dH u act'(g),  du = dH act(g)
//
// Forward, the gate's and the up filter's features lie in a tile by turns of 16
// (the operand's pairs), so that the matrix instructions leave a feature's two
// sums in one lane: the activation and the product are taken in registers
// before the one rounding, and the two sums go to memory only where the
// backward pass will want them.  Backward, a tile of dH meets g and u on its
// way out and never goes to memory itself.
#include "common.hpp"
#include "block_kernels.hpp"
#include "expert_tiles.hpp"
#include "tiles.hpp"

#include <algorithm>
#include <type_traits>

namespace cbw {
namespace {

// act(g) and its derivative:
//
//   silu = g s(g),  silu' = s (1 + g (1 - s))
//   gelu = g s(z),  gelu' = s (1 + g (1 - s) z'),  z = 2 sqrt(2 / pi) (g + 0.044715 g^3),
//
// the form with tanh, as (1 + tanh(z / 2)) / 2 = s(z).  s = 1 / (1 + exp(-z)) has
// its relative accuracy at both ends; the error of 1 - s, 2^-24, is one beside 1
// / g.  The sigmoid's own derivative would lose its accuracy in s (1 - s) and
// comes from exp(-|g|).  Where g is past 110 in size, 1 - s and on the left s
// are zero in float32: from there on g stands still in the products with them,
// which would else be 0 times infinity.  (In bf16 exp is within |z| 2^-23 of
// itself, nothing beside the 2^-9 of what is stored.)
struct Act {
    float a, da;
};
template <typename T, int KIND>
__device__ __forceinline__ Act act_at(float g)
{
    constexpr bool EXACT = sizeof(T) == 4;
    auto exponential = [](float x) { return EXACT ? expf(x) : __expf(x); };
    auto reciprocal = [](float x) { return EXACT ? 1.f / x : __builtin_amdgcn_rcpf(x); };
    if (KIND == CBW_ACT_RELU) return {g > 0.f ? g : 0.f, g > 0.f ? 1.f : 0.f};
    if (KIND == CBW_ACT_SIGMOID) {
        const float e = exponential(-fabsf(g)), r = reciprocal(1.f + e), er = e * r;
        return {g < 0.f ? er : r, er * r};
    }
    constexpr float kGelu = 1.5957691216057308f;
    const float low = g < -110.f ? -110.f : g, mid = low > 110.f ? 110.f : low, square = mid * mid;
    const float z = KIND == CBW_ACT_GELU ? kGelu * mid * (1.f + 0.044715f * square) : mid;
    const float s = reciprocal(1.f + exponential(-z));
    const float slope = KIND == CBW_ACT_GELU ? mid * kGelu * (1.f + 0.134145f * square) : mid;
    return {low * s, s * (1.f + slope * (1.f - s))};
}

// f(kind) with the activation known to the compiler.
template <typename F>
__device__ __forceinline__ void with_act(int act, const F& f)
{
    if (act == CBW_ACT_SILU) f(std::integral_constant<int, CBW_ACT_SILU>());
    else if (act == CBW_ACT_GELU) f(std::integral_constant<int, CBW_ACT_GELU>());
    else if (act == CBW_ACT_SIGMOID) f(std::integral_constant<int, CBW_ACT_SIGMOID>());
    else f(std::integral_constant<int, CBW_ACT_RELU>());
}

// I blocks of 16 features by 16 rows, as the matrix instruction leaves them (a
// lane has four features of one row in each block), through a wave's piece of
// LDS: a lane gets whole vectors of consecutive features of one row, so that
// memory is touched by whole lines.  S: the type they pass in.
template <typename S, int I>
struct Passage {
    static constexpr int ROW = I * 16 * (int)sizeof(S), CHUNKS = ROW / 16;
    static constexpr int BYTES = 16 * ROW;
    static_assert(CHUNKS >= 4 && (CHUNKS & (CHUNKS - 1)) == 0 && 64 % CHUNKS == 0, "whole rows to an instruction");

    // (a row's chunks are moved by its number: the 16 rows' do not share banks)
    static __device__ __forceinline__ char* at(char* lds, int row, int chunk)
    {
        return lds + row * ROW + ((chunk ^ (row & (CHUNKS - 1))) << 4);
    }
    template <typename V>
    static __device__ __forceinline__ void put(char* lds, int lane, const V& v)
    {
        const int row = lane & 15;
        wave_fence();   // (what was there has been read)
#pragma unroll
        for (int i = 0; i < I; ++i) {
            const floatx4 x = v(i);
            if (sizeof(S) == 2)
                *reinterpret_cast<u32x2*>(at(lds, row, i * 2 + (lane >> 5)) + (lane >> 4 & 1) * 8) =
                    u32x2{pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3])};
            else
                *reinterpret_cast<u32x4*>(at(lds, row, i * 4 + (lane >> 4))) = __builtin_bit_cast(u32x4, x);
        }
        wave_fence();
    }
};

// the lane's number, which the compiler takes for a new one each time: it would
// keep all that follows from it in registers during the products
__device__ __forceinline__ int my_lane()
{
    int lane = threadIdx.x & 63;
    asm volatile("" : "+v"(lane));
    return lane;
}

// How a kernel's outputs go to memory: what the tiled ones write would push the
// operands out of the L2 and goes past it (16384 rows, 2048 -> 4096, us: forward
// 532 for 543 to 555, backward 365 for 368).  The streaming ones' few rows stay
// at hand.
enum { NEAR = 0, PAST = 2 };

// A tile's rows of H (or of nothing) and of the two sums or their gradients.
struct Tensor {
    __amdgpu_buffer_rsrc_t r;
    uint32_t stride;
    bool there;
};
template <typename T>
__device__ __forceinline__ Tensor rows_of(const void* p, int64_t row0, int rows, int64_t stride, int cols)
{
    const T* first = static_cast<const T*>(p) + (p ? row0 * stride : 0);
    return {make_rsrc(first, p ? (uint32_t)(((rows - 1) * stride + cols) * (int64_t)sizeof(T)) : 0u), (uint32_t)stride, p != nullptr};
}

// Forward: blocks 2 i and 2 i + 1 hold the gate's and the up filter's sums of
// the same 16 features; rows q0 .. q0 + 15 of the tile, features p0 on.
template <typename T, int I, int WAY>
struct ForwardOut {
    using Pass = Passage<T, I>;
    static constexpr int BYTES = Pass::BYTES;
    Tensor h, gu;
    int rows, K, act;

    __device__ ForwardOut(const GatedArgs& a, int64_t row0, int n) : rows(n), K(a.K), act(a.act)
    {
        h = rows_of<T>(a.h, row0, n, a.h_stride, a.K);
        gu = rows_of<T>(a.gu_out, row0, n, a.gu_stride, 2 * a.K);
    }
    __device__ __forceinline__ void store(const char* lds, int lane, const Tensor& t, int q0, int p0, int col0) const
    {
        constexpr int E = 16 / (int)sizeof(T), CHUNKS = Pass::CHUNKS;
#pragma unroll
        for (int v = 0; v < 16 * CHUNKS / 64; ++v) {
            const int rr = v * (64 / CHUNKS) + lane / CHUNKS, q = q0 + rr, p = p0 + lane % CHUNKS * E;
            const u32x4 w = *reinterpret_cast<const u32x4*>(Pass::at(const_cast<char*>(lds), rr, lane % CHUNKS));
            __builtin_amdgcn_raw_buffer_store_b128(
                w, t.r, q < rows && p < K ? ((uint32_t)q * t.stride + (uint32_t)(col0 + p)) * (uint32_t)sizeof(T) : kOOB, 0, WAY);
        }
    }
    // v(b): the lane's four sums of block b
    template <typename V>
    __device__ __forceinline__ void put(char* lds, int q0, int p0, const V& v) const
    {
        const int lane = my_lane();
        if (gu.there) {
            Pass::put(lds, lane, [&](int i) { return v(2 * i); });
            store(lds, lane, gu, q0, p0, 0);
            Pass::put(lds, lane, [&](int i) { return v(2 * i + 1); });
            store(lds, lane, gu, q0, p0, K);
        }
        with_act(act, [&](auto kind) {
            Pass::put(lds, lane, [&](int i) {
                const floatx4 g = v(2 * i), u = v(2 * i + 1);
                floatx4 x;
#pragma unroll
                for (int c = 0; c < 4; ++c) x[c] = act_at<T, decltype(kind)::value>(g[c]).a * u[c];
                return x;
            });
        });
        store(lds, lane, h, q0, p0, 0);
    }
};

// Backward: I blocks of dH (in float32 through the LDS, 16 rows) meet g and u,
// which are loaded ahead.  dg and du may lie where g and u did: a lane has read
// its own before it writes them.
template <typename T, int I, int WAY>
struct BackwardOut {
    using Pass = Passage<float, I>;
    static constexpr int BYTES = Pass::BYTES, E = 16 / (int)sizeof(T);
    static constexpr int LANES = I * 16 / E, VECS = 16 * LANES / 64;   // lanes to a row, vectors to a lane
    static_assert(VECS >= 1, "work for every lane");
    Tensor h, gu, dgu;
    int rows, K, act;

    __device__ BackwardOut(const GatedArgs& a, int64_t row0, int n) : rows(n), K(a.K), act(a.act)
    {
        h = rows_of<T>(a.h, row0, n, a.h_stride, a.K);
        gu = rows_of<T>(a.gu_in, row0, n, a.gu_stride, 2 * a.K);
        dgu = rows_of<T>(a.gu_out, row0, n, a.gu_stride, 2 * a.K);
    }
    struct Ahead {
        uint4 g[VECS], u[VECS];
    };
    __device__ __forceinline__ uint32_t place(uint32_t stride, int q, int p, int col0) const
    {
        return q < rows && p < K ? ((uint32_t)q * stride + (uint32_t)(col0 + p)) * (uint32_t)sizeof(T) : kOOB;
    }
    __device__ __forceinline__ void load(Ahead& x, int q0, int p0) const
    {
        const int lane = my_lane();
#pragma unroll
        for (int v = 0; v < VECS; ++v) {
            const int q = q0 + v * (64 / LANES) + lane / LANES, p = p0 + lane % LANES * E;
            x.g[v] = buf_load16(gu.r, place(gu.stride, q, p, 0));
            x.u[v] = buf_load16(gu.r, place(gu.stride, q, p, K));
        }
    }
    static __device__ __forceinline__ void expand(const uint4& w, float (&f)[E])
    {
        const uint32_t b[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
        for (int k = 0; k < E; ++k)
            f[k] = sizeof(T) == 4 ? __uint_as_float(b[k & 3]) : __uint_as_float(k & 1 ? b[k / 2] & 0xffff0000u : b[k / 2] << 16);
    }
    static __device__ __forceinline__ u32x4 narrow(const float (&f)[E])
    {
        u32x4 w;
#pragma unroll
        for (int k = 0; k < 4; ++k) w[k] = sizeof(T) == 4 ? __float_as_uint(f[k]) : pack_bf16x2(f[2 * k % E], f[(2 * k + 1) % E]);
        return w;
    }
    template <typename V>
    __device__ __forceinline__ void put(char* lds, int q0, int p0, const Ahead& x, const V& v) const
    {
        const int lane = my_lane();
        Pass::put(lds, lane, v);
        with_act(act, [&](auto kind) { meet<decltype(kind)::value>(lds, lane, q0, p0, x); });
    }
    template <int ACT>
    __device__ __forceinline__ void meet(char* lds, int lane, int q0, int p0, const Ahead& x) const
    {
#pragma unroll
        for (int t = 0; t < VECS; ++t) {
            const int rr = t * (64 / LANES) + lane / LANES, q = q0 + rr, p = p0 + lane % LANES * E;
            float d[E], g[E], u[E], dg[E], du[E], hh[E];
#pragma unroll
            for (int k = 0; k < E / 4; ++k) {
                const floatx4 part = *reinterpret_cast<const floatx4*>(Pass::at(lds, rr, lane % LANES * (E / 4) + k));
#pragma unroll
                for (int c = 0; c < 4; ++c) d[4 * k + c] = part[c];
            }
            expand(x.g[t], g);
            expand(x.u[t], u);
#pragma unroll
            for (int k = 0; k < E; ++k) {
                const Act f = act_at<T, ACT>(g[k]);
                dg[k] = d[k] * u[k] * f.da;
                du[k] = d[k] * f.a;
                hh[k] = f.a * u[k];
            }
            __builtin_amdgcn_raw_buffer_store_b128(narrow(dg), dgu.r, place(dgu.stride, q, p, 0), 0, WAY);
            __builtin_amdgcn_raw_buffer_store_b128(narrow(du), dgu.r, place(dgu.stride, q, p, K), 0, WAY);
            if (h.there) __builtin_amdgcn_raw_buffer_store_b128(narrow(hh), h.r, place(h.stride, q, p, 0), 0, WAY);
        }
    }
};

// A tile's operands: `tp` lines of the filters (forward: pairs), `rows` rows.
// Both products run over the C features of X or dY.
template <typename T, bool BACK, int TP, int TQ, int NW>
struct Tiles {
    static constexpr int FEATURES = BACK ? TP : TP / 2;   // of the layer, in a tile
    using OP = Operand<T, TP, BACK, NW, !BACK>;
    using OQ = Operand<T, TQ, false, NW>;
    static constexpr int KB = OP::KB, COPIES = OP::COPIES + OQ::COPIES;
    OP op;
    OQ oq;
    const char *base_p, *base_q;
    uint32_t bytes_p, bytes_q;
    const GatedArgs& a;
    int p0;

    __device__ Tiles(const GatedArgs& args) : a(args) {}
    __device__ __forceinline__ void aim(int wave, int e, int first_feature, int64_t row0, int qrows)
    {
        p0 = first_feature;
        const int64_t K = a.K, C = a.C;
        const T* w = static_cast<const T*>(a.p) + (int64_t)e * (BACK ? 1 : 2) * K * C;
        if (BACK) {
            base_p = reinterpret_cast<const char*>(w + p0);
            op.init(wave, K - p0, K);
        } else {
            base_p = reinterpret_cast<const char*>(w + p0 * C);
            bytes_p = (uint32_t)((K + min((int64_t)FEATURES, K - p0)) * C * (int64_t)sizeof(T));
            op.init(wave, 0, C, K * C);
        }
        base_q = reinterpret_cast<const char*>(static_cast<const T*>(a.q) + row0 * a.x_stride);
        bytes_q = (uint32_t)(((qrows - 1) * a.x_stride + C) * (int64_t)sizeof(T));
        oq.init(wave, 0, a.x_stride);
    }
    __device__ __forceinline__ void copy(int wave, int k, char* lds_p, char* lds_q) const
    {
        if (BACK) {
            const int64_t left = min(a.C - k, KB);
            const uint32_t n = (uint32_t)(((left - 1) * a.K + a.K - p0) * (int64_t)sizeof(T));
            op.copy(wave, make_rsrc_words(base_p + (int64_t)k * a.K * (int64_t)sizeof(T), n), 0, 0, lds_p);
        } else {
            op.copy(wave, make_rsrc_words(base_p, bytes_p), k, a.C, lds_p);
        }
        oq.copy(wave, make_rsrc_words(base_q, bytes_q), k, a.C, lds_q);
    }
};

// TP lines of the filters x TQ rows by NWP x NWQ waves, two buffers of a
// 128-byte step of both operands.  The steps go as the ungated products' do:
// fragments of a step's two halves in turn, the barrier between them.
//
// What bounds it: a step of a 256 x 256 tile takes 1.5 us, 1.07 of them matrix
// instructions at the clock that they leave, and a tile some 10 us beyond its
// steps; its results are ready at once in every CU (16384 rows, 2048 -> 4096, eight
// uneven experts: forward 524 us, 1050 TFLOP/s, nine turns of tiles for the work
// of 8.5; backward 366, 750 TFLOP/s and 870 MB in and out).  Four waves with 128
// x 128 sums each would halve the LDS reads but spill (920 us for 535); letting
// the stores run on into the next tile's steps cost registers too (568 for 554).
template <typename T, bool BACK, int TP, int TQ, int NWP, int NWQ>
__global__ __launch_bounds__(NWP* NWQ * 64) void gated_kernel(GatedArgs a)
{
    constexpr int NW = NWP * NWQ, FM = TP / NWP / 16, FN = TQ / NWQ / 16;
    using Tl = Tiles<T, BACK, TP, TQ, NW>;
    using OP = typename Tl::OP;
    using OQ = typename Tl::OQ;
    constexpr int KB = Tl::KB, COPIES = Tl::COPIES, FEATURES = Tl::FEATURES;
    constexpr int BI = FM < 4 ? FM : 4;   // blocks of dH that pass the LDS at a time
    using Forward = ForwardOut<T, BACK ? 4 : FM / 2, PAST>;
    using Backward = BackwardOut<T, BI, PAST>;
    __shared__ __align__(1024) char lds_p[2][OP::BYTES];
    __shared__ __align__(1024) char lds_q[2][OQ::BYTES];
    __shared__ __align__(1024) char lds_out[NW][BACK ? Backward::BYTES : Forward::BYTES];

    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    // A CU's four SIMDs take the waves in turn: each has rows of both halves, so
    // that a tile of half its rows, whose other waves have nothing to multiply,
    // takes half the time.
    const int wp = wave % NWP, wq = wave / NWP;
    struct Tile {
        int e, p0, qrows;
        int64_t row0;
    };
    const int ptiles = (a.K + FEATURES - 1) / FEATURES;
    auto all = number_units<false>(a, [&](const Group& g) { return (int)((g.count + TQ - 1) / TQ); });
    const int total = all.total * ptiles;
    // The workgroup's `turn`-th tile, in blocks of eight row tiles by all
    // feature tiles; an XCD's part of a turn is a contiguous range of them.
    auto tile_of = [&](int turn) {
        Tile t;
        t.e = -1;
        const int first = turn * (int)gridDim.x, n = min((int)gridDim.x, total - first);
        if ((int)blockIdx.x >= n) return t;
        constexpr int GR = 8;
        const int b = first + xcd_remap(blockIdx.x, n);
        const int blk = b / (GR * ptiles), in_blk = b - blk * GR * ptiles;
        const int h = min(GR, all.total - blk * GR);
        const int pt = in_blk / h;
        int within;
        t.e = __builtin_amdgcn_readfirstlane(all.find(blk * GR + in_blk - pt * h, within));
        within = __builtin_amdgcn_readfirstlane(within);
        if (t.e < 0) return t;
        const Group g = group_of(a, t.e);
        t.p0 = pt * FEATURES;
        t.row0 = g.first + (int64_t)within * TQ;
        const int64_t left = g.first + g.count - t.row0;
        if (within < 0 || left <= 0) t.e = -1;   // (offsets that decrease)
        t.qrows = (int)min((int64_t)TQ, left);
        return t;
    };

    Tile t = tile_of(0);
    if (t.e < 0) return;
    Tl tiles(a);
    auto copy = [&](int k, int buf) { tiles.copy(wave, k, lds_p[buf], lds_q[buf]); };
    auto start = [&](const Tile& t) {
        tiles.aim(wave, t.e, t.p0, t.row0, t.qrows);
        copy(0, 0);
        if (a.C > KB) copy(KB, 1);
    };

    floatx4 acc[FM][FN];
    struct Fragments {
        uint4 p[FM], q[FN];
    };
    const int frag_p = OP::first(wp * (TP / NWP)), frag_q = OQ::first(wq * (TQ / NWQ));
    auto read = [&](Fragments& f, int buf, int ks) {
        OQ::fragments(lds_q[buf], frag_q, ks, f.q);
        OP::fragments(lds_p[buf], frag_p, ks, f.p);
    };
    auto multiply = [&](const Fragments& f) {
#pragma unroll
        for (int i = 0; i < FM; ++i)
#pragma unroll
            for (int j = 0; j < FN; ++j) acc[i][j] = mfma_chunk(acc[i][j], f.p[i], f.q[j], T{});
    };
    auto interleave = [&]() {
        constexpr int READS = FM * (BACK ? 2 : 1) + FN, MUL = FM * FN;
        if (sizeof(T) != 2) return;
#pragma unroll
        for (int i = 0; i < READS; ++i) {
            __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);                    // an LDS read
            __builtin_amdgcn_sched_group_barrier(0x008, MUL / READS, 0);          // matrix instructions
        }
    };
    Fragments fa, fb;
    const int steps = (a.C + KB - 1) / KB;
    auto product = [&]() {
#pragma unroll
        for (int i = 0; i < FM; ++i)
#pragma unroll
            for (int j = 0; j < FN; ++j) acc[i][j] = floatx4{0.f, 0.f, 0.f, 0.f};
        if (steps > 1) wait_copies<COPIES>();
        else wait_copies<0>();
        barrier();
        if (wq * (TQ / NWQ) >= t.qrows) {
            // none of the wave's rows are there: it copies
            for (int s = 0; s < steps; ++s) {
                wait_copies<0>();
                barrier();
                if (s + 2 < steps) copy((s + 2) * KB, s & 1);
            }
            return;
        }
        read(fa, 0, 0);
        for (int s = 0; s < steps; ++s) {
            const int buf = s & 1;
            read(fb, buf, 1);
            multiply(fa);
            interleave();
            wait_copies<0>();
            wait_reads();
            barrier();
            if (s + 2 < steps) copy((s + 2) * KB, buf);
            read(fa, buf ^ 1, 0);   // (after the last step: what was there, unused)
            multiply(fb);
            interleave();
        }
    };

    start(t);
    for (int turn = 1;; ++turn) {
        const Tile next = tile_of(turn);
        product();
        if (next.e >= 0) {
            wait_reads();
            barrier();   // every wave is done with both buffers
            start(next);
        }
        const int q0 = wq * (TQ / NWQ), p0 = t.p0 + wp * (FEATURES / NWP);
        if (q0 >= t.qrows) {
            // (nothing to store)
        } else if constexpr (BACK) {
            const Backward out(a, t.row0, t.qrows);
            constexpr int H = FM / BI, N = FN * H;
            typename Backward::Ahead x[2];
            out.load(x[0], q0, p0);
#pragma unroll
            for (int n = 0; n < N; ++n) {
                const int j = n / H, h = n % H;
                if (n + 1 < N) out.load(x[(n + 1) & 1], q0 + (n + 1) / H * 16, p0 + (n + 1) % H * BI * 16);
                out.put(lds_out[wave], q0 + j * 16, p0 + h * BI * 16, x[n & 1], [&](int i) { return acc[h * BI + i][j]; });
            }
        } else {
            const Forward out(a, t.row0, t.qrows);
#pragma unroll
            for (int j = 0; j < FN; ++j) out.put(lds_out[wave], q0 + j * 16, p0, [&](int b) { return acc[b][j]; });
        }
        if (next.e < 0) return;
        t = next;
    }
}

// Few rows to an expert: bound by reading the filters.  As the ungated
// streaming kernel: the waves of a workgroup share out the reduction, each
// streaming its own steps through a ring of its own in LDS, and their sums are
// added in order.  (Two rows for two of eight experts, 2048 -> 4096: 63 MB of
// filters in 10.3 to 13.2 us, the rate of a copy.)
template <typename T, bool BACK, int TP, int FN, int NW, int RING>
__global__ __launch_bounds__(NW * 64) void gated_stream_kernel(GatedArgs a)
{
    constexpr int TQ = 16 * FN, FM = TP / 16;
    using Tl = Tiles<T, BACK, TP, TQ, 1>;
    using OP = typename Tl::OP;
    using OQ = typename Tl::OQ;
    constexpr int KB = Tl::KB, COPIES = Tl::COPIES, FEATURES = Tl::FEATURES, STAGE = OP::BYTES + OQ::BYTES;
    using Forward = ForwardOut<T, BACK ? 4 : FM / 2, NEAR>;
    using Backward = BackwardOut<T, BACK ? FM : 4, NEAR>;
    constexpr int SUMS = NW * FM * FN * 1024, OUT = BACK ? Backward::BYTES : Forward::BYTES;
    __shared__ __align__(1024) char lds[NW * RING * STAGE > SUMS + FN * OUT ? NW * RING * STAGE : SUMS + FN * OUT];

    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int ptiles = (a.K + FEATURES - 1) / FEATURES;
    auto all = number_units<false>(a, [&](const Group& g) { return (int)((g.count + TQ - 1) / TQ); });
    const int nunits = all.total, total = nunits * ptiles;
    const int64_t wg = (int64_t)blockIdx.y * gridDim.x + blockIdx.x;   // (launches of many have a second axis)
    if (wg >= total) return;
    constexpr int GR = 8;
    const int b = xcd_remap((int)wg, total);
    const int blk = b / (GR * ptiles), in_blk = b - blk * GR * ptiles;
    const int h = min(GR, nunits - blk * GR);
    const int pt = in_blk / h;
    int within;
    const int e = __builtin_amdgcn_readfirstlane(all.find(blk * GR + in_blk - pt * h, within));
    if (e < 0) return;
    const Group g = group_of(a, e);
    within = __builtin_amdgcn_readfirstlane(within);
    const int p0 = pt * FEATURES;
    const int64_t row0 = g.first + (int64_t)within * TQ;
    const int qrows = (int)min((int64_t)TQ, g.first + g.count - row0);
    if (within < 0 || qrows <= 0) return;   // (offsets that decrease)
    Tl tiles(a);
    tiles.aim(0, e, p0, row0, qrows);
    char* ring = lds + wave * RING * STAGE;
    const int frag_p = OP::first(0), frag_q = OQ::first(0);
    auto copy = [&](int step, int slot) { tiles.copy(0, step * KB, ring + slot * STAGE, ring + slot * STAGE + OP::BYTES); };

    floatx4 acc[FM][FN];
#pragma unroll
    for (int i = 0; i < FM; ++i)
#pragma unroll
        for (int j = 0; j < FN; ++j) acc[i][j] = floatx4{0.f, 0.f, 0.f, 0.f};

    // this wave's steps: wave, wave + NW, ...
    const int steps = ((a.C + KB - 1) / KB - wave + NW - 1) / NW;
#pragma unroll
    for (int t = 0; t < RING; ++t)
        if (t < steps) copy(wave + t * NW, t);
    int slot = 0;
    for (int t = 0; t < steps; ++t) {
        if (t + RING <= steps) wait_copies<(RING - 1) * COPIES>();
        else wait_copies<0>();
        const char *lp = ring + slot * STAGE, *lq = lp + OP::BYTES;
        uint4 fp[2][FM], fq[2][FN];
#pragma unroll
        for (int ks = 0; ks < 2; ++ks) {
            OQ::fragments(lq, frag_q, ks, fq[ks]);
            OP::fragments(lp, frag_p, ks, fp[ks]);
        }
        wait_reads();
        if (t + RING < steps) copy(wave + (t + RING) * NW, slot);
        slot = slot == RING - 1 ? 0 : slot + 1;
#pragma unroll
        for (int ks = 0; ks < 2; ++ks)
#pragma unroll
            for (int i = 0; i < FM; ++i)
#pragma unroll
                for (int j = 0; j < FN; ++j) acc[i][j] = mfma_chunk(acc[i][j], fp[ks][i], fq[ks][j], T{});
    }

    __syncthreads();   // every wave is done with its ring
    floatx4* sums = reinterpret_cast<floatx4*>(lds);
#pragma unroll
    for (int i = 0; i < FM; ++i)
#pragma unroll
        for (int j = 0; j < FN; ++j) sums[(wave * FM * FN + i * FN + j) * 64 + lane] = acc[i][j];
    __syncthreads();
    // a wave adds up 16 rows of all features at a time and stores them
    for (int j = wave; j < FN; j += NW) {
        floatx4 v[FM] = {};
#pragma unroll
        for (int z = 0; z < NW; ++z)
#pragma unroll
            for (int i = 0; i < FM; ++i) v[i] += sums[(z * FM * FN + i * FN + j) * 64 + lane];
        if constexpr (BACK) {
            const Backward out(a, row0, qrows);
            typename Backward::Ahead x;
            out.load(x, j * 16, p0);
            out.put(lds + SUMS + j * OUT, j * 16, p0, x, [&](int i) { return v[i]; });
        } else {
            const Forward out(a, row0, qrows);
            out.put(lds + SUMS + j * OUT, j * 16, p0, [&](int i) { return v[i]; });
        }
    }
}

// The most row tiles that any lengths can give.
int64_t most_units(int64_t rows, int E, int tile) { return rows / tile + std::min<int64_t>(E, rows); }

template <typename T, bool BACK, int TP, int TQ, int NWP, int NWQ>
hipError_t launch_tiles(const GatedArgs& a, hipStream_t s)
{
    constexpr int FEATURES = BACK ? TP : TP / 2, FM = TP / NWP / 16;
    const int64_t grid = most_units(a.rows, a.E, TQ) * ((a.K + FEATURES - 1) / FEATURES);
    if (grid == 0) return hipSuccess;
    if (grid > 0x7fffffff) return hipErrorInvalidValue;
    // as many workgroups as are resident (by their LDS), which stay for several tiles
    const int64_t out = BACK ? (FM < 4 ? FM : 4) * 1024 : FM / 2 * 256 * (int)sizeof(T);
    const int64_t resident = (int64_t)CBW_NUM_CUS * (163840 / ((TP + TQ) * 256 + NWP * NWQ * out));
    gated_kernel<T, BACK, TP, TQ, NWP, NWQ><<<(int)std::min(grid, resident), NWP * NWQ * 64, 0, s>>>(a);
    return hipGetLastError();
}

template <typename T, bool BACK, int TP, int FN, int NW, int RING>
hipError_t launch_stream(const GatedArgs& a, hipStream_t s)
{
    constexpr int FEATURES = BACK ? TP : TP / 2;
    const int64_t grid = most_units(a.rows, a.E, 16 * FN) * ((a.K + FEATURES - 1) / FEATURES);
    if (grid == 0) return hipSuccess;
    if (grid > 0x7fffffff) return hipErrorInvalidValue;
    // An axis of a launch takes 2^32 - 1 threads; more wrap without an error.
    const int64_t x = std::min<int64_t>(grid, 1 << 22);
    static_assert(NW * 64 <= 1 << 9, "threads along the first axis");
    gated_stream_kernel<T, BACK, TP, FN, NW, RING><<<dim3((unsigned)x, (unsigned)((grid + x - 1) / x)), NW * 64, 0, s>>>(a);
    return hipGetLastError();
}

// Tiles of `tile` rows by `width` features, the rows spread evenly over the
// experts (the host does not know the lengths).
int64_t likely_tiles(const GatedArgs& a, int tile, int width)
{
    const int64_t busy = std::max<int64_t>(1, std::min<int64_t>(a.E, a.rows)), mean = (a.rows + busy - 1) / busy;
    return busy * ((mean + tile - 1) / tile) * ((a.K + width - 1) / width);
}

// Which kernel: by the tiles that even lengths would give.
//
// Tiles pay where they fill most of the chip and the experts have rows for them
// (us, forward | backward, tiles against streaming: 1280 rows, 1024 -> 2560, 400
// | 200 tiles of 128: 25.8 | 21.2 against 45 | 30; 512 rows, 2048 -> 2048, 128 |
// 64 tiles: 28.9 | 31.8 against 22.1 | 13.4; 16 experts of 32 rows, 2048 -> 2048:
// 70.8 | 40.2 against 67.9 | 37.0, of 64 rows alike).  Which tiles, by turns: one
// of 256 x 256 counts 1, of 192 rows 0.8, of 128 x 128, two to a CU, 0.77, and
// 0.57 where it is half empty or more (3840 rows, 1024 -> 2560, forward, 300, 400
// or 1200 tiles: 61.4, 49.8, 59.1; backward, 150, 200 or 600: 37.3, 34.5, 43.9;
// 32 experts of 256 rows, 2048 -> 2048: 171, 216, 210 and 95, 120, 117).
//
// Streaming, 64 rows read the filters once where 16 read them several times, if
// that leaves a workgroup for each CU (4 experts of 48 rows, 2048 -> 1024: 12.0 |
// 12.7 with 64 rows, 12.7 | 9.4 with 16; 512 rows above: 22.1 | 13.4 and 34 | 21).
//
// float32, tiles of 64 and streaming: 32 experts of 50 rows, 512 -> 512, 512 | 256
// tiles, 25.2 | 17.8 and 36.6 | 21.6; 8 experts of 100 rows, 256 | 128 tiles, 16.4
// | 17.0 and 20.1 | 12.2; of 20 rows, 512 -> 1024, 15.3 | 16.3 and 12.3 | 9.4.
template <typename T, bool BACK>
hipError_t launch(const GatedArgs& a, hipStream_t s)
{
    constexpr bool BF16 = sizeof(T) == 2;
    constexpr int W = BACK ? 1 : 2;   // lines of the filters to a feature
    const int64_t mean = a.rows / std::max<int64_t>(1, std::min<int64_t>(a.E, a.rows));
    if constexpr (BF16) {
        const int64_t small = likely_tiles(a, 128, 128 / W);
        if (mean > 64 && small >= 200) {
            auto turns = [&](int rows) { return (likely_tiles(a, rows, 256 / W) + CBW_NUM_CUS - 1) / CBW_NUM_CUS; };
            const int64_t last = small % (2 * CBW_NUM_CUS);
            const double by256 = (double)turns(256), by192 = 0.8 * (double)turns(192);
            const double by128 = 0.77 * (double)(small / (2 * CBW_NUM_CUS)) + (last > CBW_NUM_CUS ? 0.77 : last > 0 ? 0.57 : 0.0);
            if (by128 < std::min(by256, by192)) return launch_tiles<T, BACK, 128, 128, 2, 2>(a, s);
            if (by192 < by256) return launch_tiles<T, BACK, 256, 192, 2, 4>(a, s);
            return launch_tiles<T, BACK, 256, 256, 2, 4>(a, s);
        }
        if (mean > 16 && likely_tiles(a, 64, 64 / W) >= CBW_NUM_CUS) return launch_stream<T, BACK, 64, 4, 4, 2>(a, s);
    } else {
        if (mean > 32 && likely_tiles(a, 64, 64 / W) >= CBW_NUM_CUS) return launch_tiles<T, BACK, 64, 64, 2, 2>(a, s);
    }
    return launch_stream<T, BACK, 64, 1, 4, 2>(a, s);
}

}  // namespace

hipError_t launch_gated_fwd(int dtype, const GatedArgs& a, hipStream_t s)
{
    return dtype == CBW_F32 ? launch<float, false>(a, s) : launch<uint16_t, false>(a, s);
}

hipError_t launch_gated_bwd(int dtype, const GatedArgs& a, hipStream_t s)
{
    return dtype == CBW_F32 ? launch<float, true>(a, s) : launch<uint16_t, true>(a, s);
}

}  // namespace cbw
