// Norms before and after a block, fused with its gate and residual scale.
//
//   z = N_post(u),  y = x + s act(g) z,  h = N_pre(y)
//   N(v) = (v - mu) r w + b,  r = 1 / sqrt(mean((v - mu)^2) + eps),  mu = 0 for the RMS form
//
// and the gradients of all inputs from those of y and h:
//
//   n = (y - mu) r,  d = dh w_pre,  gy = dy + r (d - mean(d) - n mean(d n))     (mean(d) in the layer form)
//   dx = gy,  ds = sum gy a z,  dg = gy s z act'(g),  dz = gy s a,  du likewise from dz
//   dw = sum (its output's gradient) n,  db = sum (its output's gradient)
//
// Bound by memory: a row is read once into registers, where its statistics,
// both norms and every gradient are computed, and written once (16384 rows of
// 4096, bf16, RMS norms, a gate of its own for each value: forward 129 us, 5.2
// TB/s, backward 237 us, 4.5 TB/s; with a float32 stream 173 and 313, float32
// throughout 246 and 473; 100352 rows of 256, layer norms, float32 stream, one
// gate row for 3136: backward 109 us, 4.25 TB/s).  One vector of 8 columns a
// thread: with two, half as many waves hid less of the loads' latency
// (backward 374 us).  Rows of more than 8192 columns have two, and their
// backward pass spills registers (4096 rows of 16384, bf16: forward 148 us, 4.5
// TB/s, backward 293, 3.7 TB/s, with biases and scale 816).  Statistics are
// two-pass (the mean, then the squares about it) in float32; y and h are
// rounded once each, h from the unrounded y.  The parameters' gradients are
// summed over a workgroup's rows in registers and over the workgroups by a
// second kernel, in a fixed order.
#include "common.hpp"
#include "block_kernels.hpp"

#include <algorithm>
#include <type_traits>

namespace cbw {
namespace {

struct V8 {
    float f[8];
};

// Eight consecutive elements as they lie in memory (16-byte aligned), kept
// packed until their row's turn.
template <typename T> struct Raw8;
template <> struct Raw8<uint16_t> {
    uint4 v;
    __device__ __forceinline__ void load(__amdgpu_buffer_rsrc_t r, uint32_t off) { v = buf_load16(r, off); }
    __device__ __forceinline__ V8 expand() const
    {
        V8 r;
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            r.f[2 * i] = __uint_as_float(w[i] << 16);
            r.f[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
        }
        return r;
    }
};
template <> struct Raw8<float> {
    uint4 a, b;
    __device__ __forceinline__ void load(__amdgpu_buffer_rsrc_t r, uint32_t off)
    {
        a = buf_load16(r, off);
        b = buf_load16(r, off + 16);
    }
    __device__ __forceinline__ V8 expand() const
    {
        return V8{{__uint_as_float(a.x), __uint_as_float(a.y), __uint_as_float(a.z), __uint_as_float(a.w),
                   __uint_as_float(b.x), __uint_as_float(b.y), __uint_as_float(b.z), __uint_as_float(b.w)}};
    }
};
__device__ __forceinline__ void store8(__amdgpu_buffer_rsrc_t r, uint32_t off, const V8& v, uint16_t)
{
    const u32x4 w = {pack_bf16x2(v.f[0], v.f[1]), pack_bf16x2(v.f[2], v.f[3]), pack_bf16x2(v.f[4], v.f[5]),
                     pack_bf16x2(v.f[6], v.f[7])};
    __builtin_amdgcn_raw_buffer_store_b128(w, r, off, 0, 0);
}
__device__ __forceinline__ void store8(__amdgpu_buffer_rsrc_t r, uint32_t off, const V8& v, float)
{
    const floatx4 a = {v.f[0], v.f[1], v.f[2], v.f[3]}, b = {v.f[4], v.f[5], v.f[6], v.f[7]};
    __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, a), r, off, 0, 0);
    __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, b), r, off + 16, 0, 0);
}
__device__ __forceinline__ V8 splat(float v) { return V8{{v, v, v, v, v, v, v, v}}; }
// A parameter's vector, or its neutral value where the caller has none.
__device__ __forceinline__ V8 param8(const float* p, int c, bool in, float neutral)
{
    if (!p || !in) return splat(neutral);
    const float4 a = reinterpret_cast<const float4*>(p + c)[0], b = reinterpret_cast<const float4*>(p + c)[1];
    return V8{{a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w}};
}

// Rows `row` and on of a tensor whose rows lie `stride` elements apart.  Lane
// offsets are relative to that row; kOOB (a column or a row that does not
// exist, or no tensor at all) reads zeros and writes nothing.
template <typename T>
__device__ __forceinline__ __amdgpu_buffer_rsrc_t rows_at(const void* p, int64_t row, int64_t stride)
{
    return make_rsrc(static_cast<const T*>(p) + row * stride, p ? 0x7fffffffu : 0u);
}

// Sum over the 2^k lanes of a team: within groups of 4, 8 and 16 lanes by
// register moves (the mirrors meet the other half), then by exchanging rows of
// 16 and halves of the wave.  Every lane has the same result, bit for bit.
__device__ __forceinline__ float lanes_sum(float v, int team)
{
    auto moved = [](float x, auto ctrl) {
        return __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(x), decltype(ctrl)::value, 0xf, 0xf, false));
    };
    v += moved(v, std::integral_constant<int, 0xb1>{});    // lane ^ 1
    v += moved(v, std::integral_constant<int, 0x4e>{});    // lane ^ 2
    v += moved(v, std::integral_constant<int, 0x141>{});   // mirrored in 8
    if (team >= 16) v += moved(v, std::integral_constant<int, 0x140>{});   // mirrored in 16
    if (team >= 32) {
        const auto s = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
        v = __uint_as_float(s[0]) + __uint_as_float(s[1]);
    }
    if (team >= 64) {
        const auto s = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
        v = __uint_as_float(s[0]) + __uint_as_float(s[1]);
    }
    return v;
}

// The threads that hold one row.  WIDE: a whole workgroup of `team` threads;
// otherwise `team` lanes of a wave, several rows side by side.
template <bool WIDE>
struct Team {
    int lane, slot, size;
    int turn = 0;   // which half of the exchange buffer the next sum takes

    __device__ Team(int team) : size(team)
    {
        lane = WIDE ? (int)threadIdx.x : (int)threadIdx.x & (team - 1);
        slot = WIDE ? 0 : (int)threadIdx.x / team;
    }

    // Sums of two values over the team; every thread has them.  The halves of
    // the buffer alternate, so that a wave that is ahead by one sum does not
    // overwrite what another still reads: one barrier a sum.
    __device__ void sum(float& a, float& b, float (*exch)[16][2])
    {
        a = lanes_sum(a, WIDE ? 64 : size);
        b = lanes_sum(b, WIDE ? 64 : size);
        if (!WIDE) return;
        const int wave = threadIdx.x >> 6;
        if ((threadIdx.x & 63) == 0) {
            exch[turn][wave][0] = a;
            exch[turn][wave][1] = b;
        }
        __syncthreads();
        a = b = 0.f;
        for (int w = 0; w < size / 64; ++w) {
            a += exch[turn][w][0];
            b += exch[turn][w][1];
        }
        turn ^= 1;
    }
    __device__ float sum(float a, float (*exch)[16][2])
    {
        float b = 0.f;
        sum(a, b, exch);
        return a;
    }
};

// The gate's activation a and its derivative da.  The sigmoid's from e =
// exp(-|g|), a = 1 / (1 + e) or e / (1 + e), da = e / (1 + e)^2: a (1 - a)
// would lose the derivative where a is near 1, exp(-g) the value past 88.  For
// bf16 gates the fast exponential and reciprocal (|g| 2^-23 and 2^-23 relative,
// nothing beside the outputs' 2^-9) with the fewer registers.
struct Gate {
    float a, da;
};
template <typename TB>
__device__ __forceinline__ Gate gate_at(float g, int act)
{
    if (act != CBW_GATE_SIGMOID) return {g, 1.f};
    const bool exact = sizeof(TB) == 4;
    const float e = exact ? expf(-fabsf(g)) : __expf(-fabsf(g));
    const float r = exact ? 1.f / (1.f + e) : __builtin_amdgcn_rcpf(1.f + e), er = e * r;
    return {g < 0.f ? er : r, er * r};
}

// Mean and reciprocal deviation of the row v (columns past C hold zeros).
template <bool WIDE, int VPT>
__device__ __forceinline__ void row_stats(Team<WIDE>& t, const V8 (&v)[VPT], const bool (&in)[VPT], int C, int kind, float eps,
                                          float& mu, float& r, float (*exch)[16][2])
{
    mu = 0.f;
    if (kind == CBW_NORM_LAYER) {
        float s = 0.f;
#pragma unroll
        for (int i = 0; i < VPT; ++i)
#pragma unroll
            for (int j = 0; j < 8; ++j) s += v[i].f[j];
        mu = t.sum(s, exch) / (float)C;
    }
    float q = 0.f;
#pragma unroll
    for (int i = 0; i < VPT; ++i)
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const float d = in[i] ? v[i].f[j] - mu : 0.f;
            q = fmaf(d, d, q);
        }
    r = 1.f / sqrtf(t.sum(q, exch) / (float)C + eps);
}

// WT: 0 where a workgroup of 256 threads holds several rows, else one row to a
// workgroup of up to WT threads (the bound lets the smaller ones keep more
// registers).  The next rows' loads go out before a row is worked on, except
// with more than 512 threads, whose registers cannot hold both.
template <typename TR, typename TB, int WT, int VPT>
__global__ __launch_bounds__(WT ? WT : 256) void norm_fwd_kernel(NormArgs a, int team)
{
    constexpr bool WIDE = WT != 0, AHEAD = WT != 1024;
    __shared__ float exch[2][16][2];
    Team<WIDE> t(team);
    const int slots = WIDE ? 1 : 256 / team;
    bool in[VPT];
    int col[VPT];
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
        col[i] = (i * team + t.lane) * 8;
        in[i] = col[i] < a.C;
    }
    struct Loaded {
        Raw8<TR> x[VPT];
        Raw8<TB> u[VPT], g[VPT];
    };
    auto load = [&](Loaded& l, int64_t base) {
        const bool live = base + t.slot < a.rows;
        const auto rx = rows_at<TR>(a.x, base, a.res_stride);
        const auto ru = rows_at<TB>(a.u, base, a.block_stride);
        // (a row past the last one is not read, but its gate row must be a number)
        const uint32_t g0 = fdiv((uint32_t)min(base, a.rows - 1), a.gate_div);
        const uint32_t dg = fdiv((uint32_t)min(base + t.slot, a.rows - 1), a.gate_div) - g0;
        const auto rg = rows_at<TB>(a.gate, g0, a.gate_stride);
#pragma unroll
        for (int i = 0; i < VPT; ++i) {
            const uint32_t dead = live && in[i] ? 0u : kOOB;
            l.x[i].load(rx, (uint32_t)(t.slot * a.res_stride + col[i]) * (uint32_t)sizeof(TR) | dead);
            l.u[i].load(ru, (uint32_t)(t.slot * a.block_stride + col[i]) * (uint32_t)sizeof(TB) | dead);
            l.g[i].load(rg, (uint32_t)(dg * a.gate_stride + col[i]) * (uint32_t)sizeof(TB) | dead);
        }
    };
    const int64_t step = (int64_t)gridDim.x * slots;
    Loaded next;
    if (AHEAD) load(next, (int64_t)blockIdx.x * slots);
    for (int64_t base = (int64_t)blockIdx.x * slots; base < a.rows; base += step) {
        if (!AHEAD) load(next, base);
        const bool live = base + t.slot < a.rows;
        V8 y[VPT], u[VPT], g[VPT];
#pragma unroll
        for (int i = 0; i < VPT; ++i) {
            y[i] = next.x[i].expand();
            u[i] = next.u[i].expand();
            g[i] = next.g[i].expand();
        }
        if (AHEAD && base + step < a.rows) load(next, base + step);
        float mu_u = 0.f, r_u = 0.f, mu_y = 0.f, r_y = 0.f;
        if (a.u) {
            if (a.post != CBW_NORM_NONE) row_stats<WIDE, VPT>(t, u, in, a.C, a.post, a.eps, mu_u, r_u, exch);
            const auto ry = rows_at<TR>(a.y, base, a.res_stride);
#pragma unroll
            for (int i = 0; i < VPT; ++i) {
                const V8 w = param8(a.w_post, col[i], in[i], 1.f), b = param8(a.b_post, col[i], in[i], 0.f),
                         s = param8(a.scale, col[i], in[i], 1.f);
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    // (columns past C stay zeros)
                    const float n = a.post == CBW_NORM_NONE ? u[i].f[j] : in[i] ? (u[i].f[j] - mu_u) * r_u : 0.f;
                    const float z = fmaf(n, w.f[j], b.f[j]) * s.f[j];
                    y[i].f[j] = fmaf(z, a.gate ? gate_at<TB>(g[i].f[j], a.act).a : 1.f, y[i].f[j]);
                }
                store8(ry, (uint32_t)(t.slot * a.res_stride + col[i]) * (uint32_t)sizeof(TR) | (live && in[i] ? 0u : kOOB), y[i],
                       TR{});
            }
        }
        if (a.h) {
            row_stats<WIDE, VPT>(t, y, in, a.C, a.pre, a.eps, mu_y, r_y, exch);
            const auto rh = rows_at<TB>(a.h, base, a.block_stride);
#pragma unroll
            for (int i = 0; i < VPT; ++i) {
                const V8 w = param8(a.w_pre, col[i], in[i], 1.f), b = param8(a.b_pre, col[i], in[i], 0.f);
                V8 h;
#pragma unroll
                for (int j = 0; j < 8; ++j) h.f[j] = fmaf((y[i].f[j] - mu_y) * r_y, w.f[j], b.f[j]);
                store8(rh, (uint32_t)(t.slot * a.block_stride + col[i]) * (uint32_t)sizeof(TB) | (live && in[i] ? 0u : kOOB), h,
                       TB{});
            }
        }
        if (a.stats && live && t.lane == 0)
            reinterpret_cast<float4*>(a.stats)[base + t.slot] = make_float4(mu_y, r_y, mu_u, r_u);
    }
}

// FULL: gradients of biases or the scale are asked for as well (their sums
// take registers that the usual call has no use for).  The bound on registers
// keeps four waves to a SIMD where they nearly fit (us, 16384 rows of 4096,
// with the bound | without: float32 stream 313 | 339, bf16 238 | 238; not kept
// for FULL, 337 | 302, with a float32 stream 496 | 360, nor for a float32 block,
// 462 | 473).
template <typename TR, typename TB, int WT, int VPT, bool FULL>
__global__ __launch_bounds__(WT ? WT : 256, WT == 512 && !FULL && sizeof(TB) == 2 ? 4 : 1) void norm_bwd_kernel(NormBackArgs a, int team)
{
    constexpr bool WIDE = WT != 0, AHEAD = WT != 1024;
    __shared__ float exch[2][16][2];
    __shared__ float comb_s[WIDE ? 1 : 256 * 8];
    Team<WIDE> t(team);
    const int slots = WIDE ? 1 : 256 / team;
    bool in[VPT];
    int col[VPT];
    uint32_t res_off[VPT], blk_off[VPT];   // byte offsets from a workgroup's first row, kOOB past the last column
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
        col[i] = (i * team + t.lane) * 8;
        in[i] = col[i] < a.C;
        const uint32_t dead = in[i] ? 0u : kOOB;
        res_off[i] = (uint32_t)(t.slot * a.res_stride + col[i]) * (uint32_t)sizeof(TR) | dead;
        blk_off[i] = (uint32_t)(t.slot * a.block_stride + col[i]) * (uint32_t)sizeof(TB) | dead;
    }
    V8 acc[NG_COUNT][VPT];   // (without FULL all but two stay zeros and take no registers)
#pragma unroll
    for (int k = 0; k < NG_COUNT; ++k)
#pragma unroll
        for (int i = 0; i < VPT; ++i) acc[k][i] = splat(0.f);
    const bool shared_gate = a.dgate && a.gate_rows > 1;
    const float inv_c = 1.f / (float)a.C;

    // the slots' sums of vector i, added in slot order; slot 0 has the result
    auto over_slots = [&](V8& v) {
        if (WIDE) return;
        __syncthreads();
#pragma unroll
        for (int j = 0; j < 8; ++j) comb_s[j * 256 + threadIdx.x] = v.f[j];
        __syncthreads();
        if (t.slot == 0)
            for (int s = 1; s < slots; ++s)
#pragma unroll
                for (int j = 0; j < 8; ++j) v.f[j] += comb_s[j * 256 + s * team + t.lane];
    };

    // Parameters: of narrow rows, which pass quickly, kept in registers; of
    // wide ones read at every row (they are in the L1 or L2, and the registers
    // hold another wave instead).
    struct Params {
        V8 w_pre, w_post, b_post, scale;
    };
    auto params_at = [&](int i) {
        return Params{param8(a.w_pre, col[i], in[i], 1.f), param8(a.w_post, col[i], in[i], 1.f),
                      param8(a.b_post, col[i], in[i], 0.f), param8(a.scale, col[i], in[i], 1.f)};
    };
    Params kept[WIDE ? 1 : VPT];
    if (!WIDE)
#pragma unroll
        for (int i = 0; i < (WIDE ? 1 : VPT); ++i) kept[i] = params_at(i);

    struct Loaded {
        Raw8<TR> y[VPT], dy[VPT];
        Raw8<TB> dh[VPT], u[VPT], g[VPT];
        uint4 st;
    };
    const int64_t i0 = blockIdx.x * a.split.items / gridDim.x, i1 = (blockIdx.x + 1) * a.split.items / gridDim.x;
    for (int64_t item = i0; item < i1; ++item) {
        const int64_t group = item / a.split.parts, part = item - group * a.split.parts;
        const int64_t g0 = group * a.split.group_rows, g1 = min(g0 + a.split.group_rows, a.rows);
        const int64_t r0 = min(g0 + part * a.split.item_rows, g1), r1 = min(r0 + a.split.item_rows, g1);
        auto load = [&](Loaded& l, int64_t base) {
            const auto ry = rows_at<TR>(a.dh ? a.y : nullptr, base, a.res_stride), rdy = rows_at<TR>(a.dy, base, a.res_stride);
            const auto rdh = rows_at<TB>(a.dh, base, a.block_stride), ru = rows_at<TB>(a.u, base, a.block_stride);
            const auto rg = rows_at<TB>(a.gate, a.gate_rows > 1 ? group : base, a.gate_stride);
            const uint32_t dead = base + t.slot < r1 ? 0u : kOOB;
            l.st = buf_load16(rows_at<float>(a.stats, base, 4), (uint32_t)t.slot * 16u | dead);
#pragma unroll
            for (int i = 0; i < VPT; ++i) {
                l.y[i].load(ry, res_off[i] | dead);
                l.dh[i].load(rdh, blk_off[i] | dead);
                l.dy[i].load(rdy, res_off[i] | dead);
                l.u[i].load(ru, blk_off[i] | dead);
                l.g[i].load(rg, (uint32_t)((a.gate_rows > 1 ? 0 : t.slot) * a.gate_stride + col[i]) * (uint32_t)sizeof(TB) |
                                    (in[i] ? dead : kOOB));
            }
        };
        V8 dgs[VPT];
#pragma unroll
        for (int i = 0; i < VPT; ++i) dgs[i] = splat(0.f);
        Loaded next;
        if (AHEAD && r0 < r1) load(next, r0);
        for (int64_t base = r0; base < r1; base += slots) {
            if (!AHEAD) load(next, base);
            const uint32_t dead = base + t.slot < r1 ? 0u : kOOB;
            V8 n[VPT], d[VPT], gy[VPT], u[VPT], g[VPT];
            const float4 st = make_float4(__uint_as_float(next.st.x), __uint_as_float(next.st.y), __uint_as_float(next.st.z),
                                          __uint_as_float(next.st.w));
#pragma unroll
            for (int i = 0; i < VPT; ++i) {
                n[i] = next.y[i].expand();
                d[i] = next.dh[i].expand();
                gy[i] = next.dy[i].expand();
                u[i] = next.u[i].expand();
                g[i] = next.g[i].expand();
            }
            if (AHEAD && base + slots < r1) load(next, base + slots);
            if (a.dh) {
                float sd = 0.f, sn = 0.f;
#pragma unroll
                for (int i = 0; i < VPT; ++i) {
                    const V8 w = WIDE ? param8(a.w_pre, col[i], in[i], 1.f) : kept[WIDE ? 0 : i].w_pre;
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        // (a row or column that does not exist: all loads and r are zero)
                        const float v = in[i] ? (n[i].f[j] - st.x) * st.y : 0.f;
                        acc[NG_W_PRE][i].f[j] = fmaf(d[i].f[j], v, acc[NG_W_PRE][i].f[j]);
                        if (FULL) acc[NG_B_PRE][i].f[j] += d[i].f[j];
                        const float e = d[i].f[j] * w.f[j];
                        n[i].f[j] = v;
                        d[i].f[j] = e;
                        sd += e;
                        sn = fmaf(e, v, sn);
                    }
                }
                t.sum(sd, sn, exch);
                const float md = a.pre == CBW_NORM_LAYER ? sd * inv_c : 0.f, mn = sn * inv_c;
#pragma unroll
                for (int i = 0; i < VPT; ++i)
#pragma unroll
                    for (int j = 0; j < 8; ++j)
                        gy[i].f[j] = in[i] ? fmaf(st.y, d[i].f[j] - md - n[i].f[j] * mn, gy[i].f[j]) : 0.f;
            }
            const auto rdx = rows_at<TR>(a.dx, base, a.res_stride);
#pragma unroll
            for (int i = 0; i < VPT; ++i) store8(rdx, res_off[i] | dead, gy[i], TR{});
            if (!a.u) continue;
            float sd = 0.f, sn = 0.f;
            const auto rdg = rows_at<TB>(shared_gate ? nullptr : a.dgate, base, a.gate_stride);
#pragma unroll
            for (int i = 0; i < VPT; ++i) {
                const Params pm = WIDE ? params_at(i) : kept[WIDE ? 0 : i];
                const V8 &w = pm.w_post, &b = pm.b_post, &s = pm.scale;
                V8 dg;
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const float v = a.post == CBW_NORM_NONE ? u[i].f[j] : in[i] ? (u[i].f[j] - st.z) * st.w : 0.f;
                    const float z = fmaf(v, w.f[j], b.f[j]);
                    const Gate gate = a.gate ? gate_at<TB>(g[i].f[j], a.act) : Gate{1.f, 1.f};
                    const float act = gate.a;
                    dg.f[j] = gy[i].f[j] * s.f[j] * z * gate.da;
                    if (FULL) acc[NG_SCALE][i].f[j] = fmaf(gy[i].f[j] * act, z, acc[NG_SCALE][i].f[j]);
                    const float dz = gy[i].f[j] * s.f[j] * act;
                    acc[NG_W_POST][i].f[j] = fmaf(dz, v, acc[NG_W_POST][i].f[j]);
                    if (FULL) acc[NG_B_POST][i].f[j] += dz;
                    const float e = dz * w.f[j];
                    u[i].f[j] = v;
                    g[i].f[j] = e;
                    sd += e;
                    sn = fmaf(e, v, sn);
                }
                if (shared_gate) {
#pragma unroll
                    for (int j = 0; j < 8; ++j) dgs[i].f[j] += dg.f[j];
                } else {
                    store8(rdg, (uint32_t)(t.slot * a.gate_stride + col[i]) * (uint32_t)sizeof(TB) | (in[i] ? dead : kOOB), dg, TB{});
                }
            }
            if (!a.du) continue;
            if (a.post != CBW_NORM_NONE) {
                t.sum(sd, sn, exch);
                const float md = a.post == CBW_NORM_LAYER ? sd * inv_c : 0.f, mn = sn * inv_c;
#pragma unroll
                for (int i = 0; i < VPT; ++i)
#pragma unroll
                    for (int j = 0; j < 8; ++j) g[i].f[j] = st.w * (g[i].f[j] - md - u[i].f[j] * mn);
            }
            const auto rdu = rows_at<TB>(a.du, base, a.block_stride);
#pragma unroll
            for (int i = 0; i < VPT; ++i) store8(rdu, blk_off[i] | dead, g[i], TB{});
        }
        if (shared_gate) {
#pragma unroll
            for (int i = 0; i < VPT; ++i) {
                over_slots(dgs[i]);
                const bool mine = t.slot == 0 && in[i];
                if (a.gate_partial)
                    store8(rows_at<float>(a.gate_partial, item, a.C), mine ? (uint32_t)col[i] * 4u : kOOB, dgs[i], 0.f);
                else
                    store8(rows_at<TB>(a.dgate, group, a.gate_stride), mine ? (uint32_t)col[i] * (uint32_t)sizeof(TB) : kOOB,
                           dgs[i], TB{});
            }
        }
    }

    int at = 0;
#pragma unroll
    for (int k = 0; k < NG_COUNT; ++k) {
        if (!a.grads[k]) continue;
#pragma unroll
        for (int i = 0; i < VPT; ++i) {
            over_slots(acc[k][i]);
            const float* to = a.partial ? a.partial + (int64_t)blockIdx.x * a.C * NG_COUNT + at * a.C : a.grads[k];
            store8(rows_at<float>(to, 0, 0), t.slot == 0 && in[i] ? (uint32_t)col[i] * 4u : kOOB, acc[k][i], 0.f);
        }
        ++at;
    }
}

// Sums of partials over workgroups (the parameters' gradients) and over the
// parts of a group (a shared gate's): a workgroup takes 64 columns, its 16
// waves every sixteenth partial, and adds the waves' sums in order.
struct SumArgs {
    const float* partial;
    float* out[NG_COUNT];
    int n, nvec;                 // partials, vectors asked for
    const float* gate_partial;
    void* dgate;
    int64_t groups, parts, gate_stride;
    int C, ctiles;
};

template <typename TB>
__device__ __forceinline__ void put(TB* p, float v);
template <>
__device__ __forceinline__ void put<float>(float* p, float v) { *p = v; }
template <>
__device__ __forceinline__ void put<uint16_t>(uint16_t* p, float v) { *p = (uint16_t)f32_to_bf16_rne(v); }

template <typename TB>
__global__ __launch_bounds__(1024) void norm_sum_kernel(SumArgs a)
{
    __shared__ float sum_s[16][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t job = blockIdx.x / a.ctiles;
    const int c = (int)(blockIdx.x % a.ctiles) * 64 + lane;
    const bool gate = job >= a.nvec;
    const int64_t group = job - a.nvec;
    const float* p = gate ? a.gate_partial + group * a.parts * a.C : a.partial + job * a.C;
    const int64_t step = gate ? a.C : (int64_t)NG_COUNT * a.C, n = gate ? a.parts : a.n;
    float s = 0.f;
    if (c < a.C) {
        // sixteen loads in flight, added in order
        for (int64_t i = wave; i < n; i += 256) {
            float v[16];
#pragma unroll
            for (int k = 0; k < 16; ++k) v[k] = i + 16 * k < n ? p[(i + 16 * k) * step + c] : 0.f;
#pragma unroll
            for (int k = 0; k < 16; ++k) s += v[k];
        }
    }
    sum_s[wave][lane] = s;
    __syncthreads();
    if (wave != 0 || c >= a.C) return;
    for (int w = 1; w < 16; ++w) s += sum_s[w][lane];
    if (gate) put(static_cast<TB*>(a.dgate) + group * a.gate_stride + c, s);
    else a.out[job][c] = s;
}

template <typename TR, typename TB>
hipError_t fwd_types(const NormArgs& a, hipStream_t s)
{
    const NormShape n = norm_shape(a.C);
    const int64_t want = (a.rows + n.slots - 1) / n.slots;
    // four workgroups of 256 threads a CU, each with rows enough to load ahead
    const int grid = (int)std::min<int64_t>(want, 256 * std::max(1, 1024 / n.threads));
    if (n.slots > 1) norm_fwd_kernel<TR, TB, 0, 1><<<grid, n.threads, 0, s>>>(a, n.team);
    else if (n.vpt == 2) norm_fwd_kernel<TR, TB, 1024, 2><<<grid, n.threads, 0, s>>>(a, n.team);
    else if (n.team <= 512) norm_fwd_kernel<TR, TB, 512, 1><<<grid, n.threads, 0, s>>>(a, n.team);
    else norm_fwd_kernel<TR, TB, 1024, 1><<<grid, n.threads, 0, s>>>(a, n.team);
    return hipGetLastError();
}

template <typename TR, typename TB, bool FULL>
void bwd_shapes(const NormBackArgs& a, hipStream_t s)
{
    const NormShape n = norm_shape(a.C);
    const int grid = a.split.grid;
    if (n.slots > 1) norm_bwd_kernel<TR, TB, 0, 1, FULL><<<grid, n.threads, 0, s>>>(a, n.team);
    else if (n.vpt == 2) norm_bwd_kernel<TR, TB, 1024, 2, FULL><<<grid, n.threads, 0, s>>>(a, n.team);
    else if (n.team <= 512) norm_bwd_kernel<TR, TB, 512, 1, FULL><<<grid, n.threads, 0, s>>>(a, n.team);
    else norm_bwd_kernel<TR, TB, 1024, 1, FULL><<<grid, n.threads, 0, s>>>(a, n.team);
}

template <typename TR, typename TB>
hipError_t bwd_types(const NormBackArgs& a, hipStream_t s)
{
    if (a.grads[NG_B_PRE] || a.grads[NG_B_POST] || a.grads[NG_SCALE]) bwd_shapes<TR, TB, true>(a, s);
    else bwd_shapes<TR, TB, false>(a, s);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || (!a.partial && !a.gate_partial)) return e;
    SumArgs r{};
    r.partial = a.partial;
    for (int k = 0; k < NG_COUNT; ++k)
        if (a.partial && a.grads[k]) r.out[r.nvec++] = a.grads[k];
    r.n = a.split.grid;
    r.gate_partial = a.gate_partial;
    r.dgate = a.dgate;
    r.groups = a.gate_partial ? a.split.groups : 0;
    r.parts = a.split.parts;
    r.gate_stride = a.gate_stride;
    r.C = a.C;
    r.ctiles = (a.C + 63) / 64;
    const int64_t jobs = (r.nvec + r.groups) * r.ctiles;
    if (jobs == 0) return hipSuccess;
    if (jobs > 0x7fffffff) return hipErrorInvalidValue;
    norm_sum_kernel<TB><<<(int)jobs, 1024, 0, s>>>(r);
    return hipGetLastError();
}

}  // namespace

// Workgroups enough to fill the chip, each with a contiguous range of rows.
// With a shared gate the rows of a gate row are split into equal parts when
// there are fewer gate rows than workgroups.
NormSplit norm_split(const cbw_norm_desc* d)
{
    const NormShape n = norm_shape(d->C);
    NormSplit s{};
    const int64_t steps = (d->rows + n.slots - 1) / n.slots;
    const int most = 256 * std::max(1, 1024 / n.threads);
    s.grid = (int)std::max<int64_t>(1, std::min<int64_t>(steps, most));
    if (d->gate_act != CBW_GATE_NONE && d->gate_rows > 1) {
        s.group_rows = std::min(d->gate_rows, d->rows);
        s.groups = d->rows > 0 ? (d->rows - 1) / d->gate_rows + 1 : 1;   // (gate_rows may be its type's largest value)
    } else {
        s.group_rows = d->rows;
        s.groups = 1;
    }
    int64_t parts = std::max<int64_t>(1, s.grid / s.groups);
    s.item_rows = std::max<int64_t>(1, (s.group_rows + parts - 1) / parts);
    s.item_rows = (s.item_rows + n.slots - 1) / n.slots * n.slots;
    s.parts = std::max<int64_t>(1, (s.group_rows + s.item_rows - 1) / s.item_rows);
    s.items = s.groups * s.parts;
    s.grid = (int)std::max<int64_t>(1, std::min<int64_t>(s.items, most));
    return s;
}

hipError_t launch_norm_fwd(int dtype, int res_dtype, const NormArgs& a, hipStream_t s)
{
    if (dtype == CBW_F32) return fwd_types<float, float>(a, s);
    if (res_dtype == CBW_F32) return fwd_types<float, uint16_t>(a, s);
    return fwd_types<uint16_t, uint16_t>(a, s);
}

hipError_t launch_norm_bwd(int dtype, int res_dtype, const NormBackArgs& a, hipStream_t s)
{
    if (dtype == CBW_F32) return bwd_types<float, float>(a, s);
    if (res_dtype == CBW_F32) return bwd_types<float, uint16_t>(a, s);
    return bwd_types<uint16_t, uint16_t>(a, s);
}

}  // namespace cbw
