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
// both norms and every gradient are computed, and written once.  Statistics
// are two-pass (the mean, then the squares about it) in float32; y and h are
// rounded once each, h from the unrounded y.  The parameters' gradients are
// summed over a workgroup's rows in registers and over the workgroups by a
// second kernel, in a fixed order.
#include "common.hpp"
#include "block_kernels.hpp"

#include <algorithm>

namespace cbw {
namespace {

struct V8 {
    float f[8];
};

__device__ __forceinline__ V8 unpack(const uint4& a)
{
    V8 r;
    const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        r.f[2 * i] = __uint_as_float(w[i] << 16);
        r.f[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
    return r;
}

// Eight consecutive elements (16-byte aligned) as float32.
__device__ __forceinline__ V8 load8(const uint16_t* p) { return unpack(*reinterpret_cast<const uint4*>(p)); }
__device__ __forceinline__ V8 load8(const float* p)
{
    const float4 a = reinterpret_cast<const float4*>(p)[0], b = reinterpret_cast<const float4*>(p)[1];
    return V8{{a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w}};
}
__device__ __forceinline__ void store8(uint16_t* p, const V8& v)
{
    *reinterpret_cast<uint4*>(p) = make_uint4(pack_bf16x2(v.f[0], v.f[1]), pack_bf16x2(v.f[2], v.f[3]),
                                              pack_bf16x2(v.f[4], v.f[5]), pack_bf16x2(v.f[6], v.f[7]));
}
__device__ __forceinline__ void store8(float* p, const V8& v)
{
    reinterpret_cast<float4*>(p)[0] = make_float4(v.f[0], v.f[1], v.f[2], v.f[3]);
    reinterpret_cast<float4*>(p)[1] = make_float4(v.f[4], v.f[5], v.f[6], v.f[7]);
}
__device__ __forceinline__ V8 splat(float v) { return V8{{v, v, v, v, v, v, v, v}}; }
// A parameter's vector, or its neutral value where the caller has none.
__device__ __forceinline__ V8 param8(const float* p, int c, float neutral) { return p ? load8(p + c) : splat(neutral); }

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
    __device__ void sum(float& a, float& b, float (*exch)[2][16])
    {
        const int span = WIDE ? 64 : size;
        for (int o = span / 2; o >= 1; o >>= 1) {
            a += __shfl_xor(a, o);
            b += __shfl_xor(b, o);
        }
        if (!WIDE) return;
        const int wave = threadIdx.x >> 6;
        if ((threadIdx.x & 63) == 0) {
            exch[turn][0][wave] = a;
            exch[turn][1][wave] = b;
        }
        __syncthreads();
        a = b = 0.f;
        for (int w = 0; w < size / 64; ++w) {
            a += exch[turn][0][w];
            b += exch[turn][1][w];
        }
        turn ^= 1;
    }
    __device__ float sum(float a, float (*exch)[2][16])
    {
        float b = 0.f;
        sum(a, b, exch);
        return a;
    }
};

// The gate's activation and its derivative.
__device__ __forceinline__ float gate_value(float g, int act)
{
    return act == CBW_GATE_SIGMOID ? 1.f / (1.f + __expf(-g)) : g;
}

// Mean and reciprocal deviation of the row v (columns past C hold zeros).
template <bool WIDE, int VPT>
__device__ __forceinline__ void row_stats(Team<WIDE>& t, const V8 (&v)[VPT], const bool (&in)[VPT], int C, int kind, float eps,
                                          float& mu, float& r, float (*exch)[2][16])
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
// registers).
template <typename TR, typename TB, int WT, int VPT>
__global__ __launch_bounds__(WT ? WT : 256) void norm_fwd_kernel(NormArgs a, int team)
{
    constexpr bool WIDE = WT != 0;
    __shared__ float exch[2][2][16];
    Team<WIDE> t(team);
    const int slots = WIDE ? 1 : 256 / team;
    bool in[VPT];
    int col[VPT];
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
        col[i] = (i * team + t.lane) * 8;
        in[i] = col[i] < a.C;
    }
    for (int64_t base = (int64_t)blockIdx.x * slots; base < a.rows; base += (int64_t)gridDim.x * slots) {
        const int64_t row = base + t.slot;
        const bool live = row < a.rows;
        V8 y[VPT], u[VPT], g[VPT];
#pragma unroll
        for (int i = 0; i < VPT; ++i) {
            const bool ok = live && in[i];
            y[i] = ok ? load8(static_cast<const TR*>(a.x) + row * a.res_stride + col[i]) : splat(0.f);
            u[i] = ok && a.u ? load8(static_cast<const TB*>(a.u) + row * a.block_stride + col[i]) : splat(0.f);
            g[i] = ok && a.gate ? load8(static_cast<const TB*>(a.gate) +
                                        (a.gate_rows > 1 ? row / a.gate_rows : row) * a.gate_stride + col[i])
                                : splat(0.f);
        }
        float mu_u = 0.f, r_u = 0.f, mu_y = 0.f, r_y = 0.f;
        if (a.u) {
            if (a.post != CBW_NORM_NONE) row_stats<WIDE, VPT>(t, u, in, a.C, a.post, a.eps, mu_u, r_u, exch);
#pragma unroll
            for (int i = 0; i < VPT; ++i) {
                if (!in[i]) continue;
                const V8 w = param8(a.w_post, col[i], 1.f), b = param8(a.b_post, col[i], 0.f),
                         s = param8(a.scale, col[i], 1.f);
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const float n = a.post == CBW_NORM_NONE ? u[i].f[j] : (u[i].f[j] - mu_u) * r_u;
                    const float z = fmaf(n, w.f[j], b.f[j]) * s.f[j];
                    y[i].f[j] = fmaf(z, a.gate ? gate_value(g[i].f[j], a.act) : 1.f, y[i].f[j]);
                }
                if (live) store8(static_cast<TR*>(a.y) + row * a.res_stride + col[i], y[i]);
            }
        }
        if (a.h) {
            row_stats<WIDE, VPT>(t, y, in, a.C, a.pre, a.eps, mu_y, r_y, exch);
#pragma unroll
            for (int i = 0; i < VPT; ++i) {
                if (!in[i]) continue;
                const V8 w = param8(a.w_pre, col[i], 1.f), b = param8(a.b_pre, col[i], 0.f);
                V8 h;
#pragma unroll
                for (int j = 0; j < 8; ++j) h.f[j] = fmaf((y[i].f[j] - mu_y) * r_y, w.f[j], b.f[j]);
                if (live) store8(static_cast<TB*>(a.h) + row * a.block_stride + col[i], h);
            }
        }
        if (a.stats && live && t.lane == 0)
            reinterpret_cast<float4*>(a.stats)[row] = make_float4(mu_y, r_y, mu_u, r_u);
    }
}

// FULL: gradients of biases or the scale are asked for as well (their sums
// take registers that the usual call has no use for).
template <typename TR, typename TB, int WT, int VPT, bool FULL>
__global__ __launch_bounds__(WT ? WT : 256) void norm_bwd_kernel(NormBackArgs a, int team)
{
    constexpr bool WIDE = WT != 0;
    __shared__ float exch[2][2][16];
    __shared__ float comb_s[WIDE ? 1 : 256 * 8];
    Team<WIDE> t(team);
    const int slots = WIDE ? 1 : 256 / team;
    bool in[VPT];
    int col[VPT];
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
        col[i] = (i * team + t.lane) * 8;
        in[i] = col[i] < a.C;
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

    const int64_t i0 = blockIdx.x * a.split.items / gridDim.x, i1 = (blockIdx.x + 1) * a.split.items / gridDim.x;
    for (int64_t item = i0; item < i1; ++item) {
        const int64_t group = item / a.split.parts, part = item - group * a.split.parts;
        const int64_t g0 = group * a.split.group_rows, g1 = min(g0 + a.split.group_rows, a.rows);
        const int64_t r0 = min(g0 + part * a.split.item_rows, g1), r1 = min(r0 + a.split.item_rows, g1);
        V8 dgs[VPT];
#pragma unroll
        for (int i = 0; i < VPT; ++i) dgs[i] = splat(0.f);
        for (int64_t base = r0; base < r1; base += slots) {
            const int64_t row = base + t.slot;
            const bool live = row < r1;
            V8 y[VPT], dh[VPT], dy[VPT], u[VPT], g[VPT];
            float4 st = make_float4(0.f, 0.f, 0.f, 0.f);
            if (live) st = reinterpret_cast<const float4*>(a.stats)[row];
#pragma unroll
            for (int i = 0; i < VPT; ++i) {
                const bool ok = live && in[i];
                dy[i] = ok && a.dy ? load8(static_cast<const TR*>(a.dy) + row * a.res_stride + col[i]) : splat(0.f);
                y[i] = ok && a.dh ? load8(static_cast<const TR*>(a.y) + row * a.res_stride + col[i]) : splat(0.f);
                dh[i] = ok && a.dh ? load8(static_cast<const TB*>(a.dh) + row * a.block_stride + col[i]) : splat(0.f);
                u[i] = ok && a.u ? load8(static_cast<const TB*>(a.u) + row * a.block_stride + col[i]) : splat(0.f);
                g[i] = ok && a.gate ? load8(static_cast<const TB*>(a.gate) +
                                            (a.gate_rows > 1 ? row / a.gate_rows : row) * a.gate_stride + col[i])
                                    : splat(0.f);
            }
            if (a.dh) {
                float sd = 0.f, sn = 0.f;
#pragma unroll
                for (int i = 0; i < VPT; ++i) {
                    if (!in[i]) continue;
                    const V8 w = param8(a.w_pre, col[i], 1.f);
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        const float n = live ? (y[i].f[j] - st.x) * st.y : 0.f;
                        acc[NG_W_PRE][i].f[j] = fmaf(dh[i].f[j], n, acc[NG_W_PRE][i].f[j]);
                        if (FULL) acc[NG_B_PRE][i].f[j] += dh[i].f[j];
                        const float d = dh[i].f[j] * w.f[j];
                        y[i].f[j] = n;
                        dh[i].f[j] = d;
                        sd += d;
                        sn = fmaf(d, n, sn);
                    }
                }
                t.sum(sd, sn, exch);
                const float md = a.pre == CBW_NORM_LAYER ? sd * inv_c : 0.f, mn = sn * inv_c;
#pragma unroll
                for (int i = 0; i < VPT; ++i)
#pragma unroll
                    for (int j = 0; j < 8; ++j)
                        dy[i].f[j] = fmaf(st.y, dh[i].f[j] - md - y[i].f[j] * mn, dy[i].f[j]);
            }
#pragma unroll
            for (int i = 0; i < VPT; ++i)
                if (live && in[i]) store8(static_cast<TR*>(a.dx) + row * a.res_stride + col[i], dy[i]);
            if (!a.u) continue;
            float sd = 0.f, sn = 0.f;
#pragma unroll
            for (int i = 0; i < VPT; ++i) {
                if (!in[i]) continue;
                const V8 w = param8(a.w_post, col[i], 1.f), b = param8(a.b_post, col[i], 0.f),
                         s = param8(a.scale, col[i], 1.f);
                V8 dg;
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const float gy = live ? dy[i].f[j] : 0.f;
                    const float n = a.post == CBW_NORM_NONE ? u[i].f[j] : live ? (u[i].f[j] - st.z) * st.w : 0.f;
                    const float z = fmaf(n, w.f[j], b.f[j]);
                    const float act = a.gate ? gate_value(g[i].f[j], a.act) : 1.f;
                    const float da = a.act == CBW_GATE_SIGMOID ? act * (1.f - act) : 1.f;
                    dg.f[j] = gy * s.f[j] * z * da;
                    if (FULL) acc[NG_SCALE][i].f[j] = fmaf(gy * act, z, acc[NG_SCALE][i].f[j]);
                    const float dz = gy * s.f[j] * act;
                    acc[NG_W_POST][i].f[j] = fmaf(dz, n, acc[NG_W_POST][i].f[j]);
                    if (FULL) acc[NG_B_POST][i].f[j] += dz;
                    const float d = dz * w.f[j];
                    u[i].f[j] = n;
                    g[i].f[j] = d;
                    sd += d;
                    sn = fmaf(d, n, sn);
                }
                if (a.dgate) {
                    if (shared_gate) {
#pragma unroll
                        for (int j = 0; j < 8; ++j) dgs[i].f[j] += dg.f[j];
                    } else if (live) {
                        store8(static_cast<TB*>(a.dgate) + row * a.gate_stride + col[i], dg);
                    }
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
#pragma unroll
            for (int i = 0; i < VPT; ++i)
                if (live && in[i]) store8(static_cast<TB*>(a.du) + row * a.block_stride + col[i], g[i]);
        }
        if (shared_gate) {
#pragma unroll
            for (int i = 0; i < VPT; ++i) {
                over_slots(dgs[i]);
                if (t.slot != 0 || !in[i]) continue;
                if (a.gate_partial) store8(a.gate_partial + item * a.C + col[i], dgs[i]);
                else store8(static_cast<TB*>(a.dgate) + group * a.gate_stride + col[i], dgs[i]);
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
            if (t.slot != 0 || !in[i]) continue;
            float* to = a.partial ? a.partial + (int64_t)blockIdx.x * a.C * NG_COUNT + at * a.C : a.grads[k];
            store8(to + col[i], acc[k][i]);
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
        int64_t i = wave;
        for (; i + 48 < n; i += 64) {
            const float v0 = p[i * step + c], v1 = p[(i + 16) * step + c], v2 = p[(i + 32) * step + c],
                        v3 = p[(i + 48) * step + c];
            s += v0;
            s += v1;
            s += v2;
            s += v3;
        }
        for (; i < n; i += 16) s += p[i * step + c];
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
    const int grid = (int)std::min<int64_t>(want, 1 << 20);
    if (n.slots == 1) {
        if (n.team <= 256) norm_fwd_kernel<TR, TB, 256, 2><<<grid, n.threads, 0, s>>>(a, n.team);
        else if (n.team <= 512) norm_fwd_kernel<TR, TB, 512, 2><<<grid, n.threads, 0, s>>>(a, n.team);
        else norm_fwd_kernel<TR, TB, 1024, 2><<<grid, n.threads, 0, s>>>(a, n.team);
    } else if (n.vpt == 1) {
        norm_fwd_kernel<TR, TB, 0, 1><<<grid, n.threads, 0, s>>>(a, n.team);
    } else {
        norm_fwd_kernel<TR, TB, 0, 2><<<grid, n.threads, 0, s>>>(a, n.team);
    }
    return hipGetLastError();
}

template <typename TR, typename TB, bool FULL>
void bwd_shapes(const NormBackArgs& a, hipStream_t s)
{
    const NormShape n = norm_shape(a.C);
    if (n.slots == 1) {
        if (n.team <= 256) norm_bwd_kernel<TR, TB, 256, 2, FULL><<<a.split.grid, n.threads, 0, s>>>(a, n.team);
        else if (n.team <= 512) norm_bwd_kernel<TR, TB, 512, 2, FULL><<<a.split.grid, n.threads, 0, s>>>(a, n.team);
        else norm_bwd_kernel<TR, TB, 1024, 2, FULL><<<a.split.grid, n.threads, 0, s>>>(a, n.team);
    } else if (n.vpt == 1) {
        norm_bwd_kernel<TR, TB, 0, 1, FULL><<<a.split.grid, n.threads, 0, s>>>(a, n.team);
    } else {
        norm_bwd_kernel<TR, TB, 0, 2, FULL><<<a.split.grid, n.threads, 0, s>>>(a, n.team);
    }
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
        s.groups = std::max<int64_t>(1, (d->rows + d->gate_rows - 1) / d->gate_rows);
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
