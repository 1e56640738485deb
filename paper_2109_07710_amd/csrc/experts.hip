// Products grouped by expert on the gfx950 matrix cores: the forward product
// of an expert layer and its two gradients, over groups of rows whose lengths
// only the device knows.
//
//   forward   Y[r,k]    = sum_c W[e,k,c] X[r,c]
//   data      dX[r,c]   = sum_k W[e,k,c] dY[r,k]
//   weight    dW[e,k,c] = sum_r X[r,c] dY[r,k]
//
// One tiled kernel serves all three.  Its P operand supplies the output's
// contiguous features (the rows of the matrix instruction's result, so a lane
// ends up with four consecutive ones), its Q operand the other dimension.  An
// operand whose reduction index is contiguous in memory ("along") is read
// from LDS 16 bytes a lane; one whose reduction index is its row ("across":
// the filter of the data gradient, both operands of the weight gradient) is
// copied as it lies and transposed on its way out of LDS (bf16) or read
// element by element (float32, whose matrix instruction takes one reduction
// index a lane).
//
// Every workgroup finds its expert and tile itself: a wave scans the group
// lengths (E + 1 offsets, in the cache) and looks its own number up.  The
// grid covers the most tiles any lengths can give; surplus workgroups leave.
#include "common.hpp"
#include "block_kernels.hpp"

#include <algorithm>
#include <type_traits>

namespace cbw {
namespace {

enum { FWD = 0, DATA = 1, WEIGHT = 2 };

// Rows of group e, whatever the offsets hold: inside [0, rows], at least 0.
struct Group {
    int64_t first, count;
};
__device__ __forceinline__ Group group_of(const ExpertArgs& a, int e)
{
    const int64_t lo = min(max((int64_t)a.offsets[e], (int64_t)0), a.rows);
    const int64_t hi = min(max((int64_t)a.offsets[e + 1], lo), a.rows);
    return {lo, hi - lo};
}

__device__ __forceinline__ int wave_inclusive_sum(int v)
{
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const int w = __shfl_up(v, o, 64);
        if (lane >= o) v += w;
    }
    return v;
}

// Units of work over the experts: units(e, group) each, numbered through.
// Called by whole waves; every result is the same in all lanes.
template <typename F>
__device__ __forceinline__ int count_units(const ExpertArgs& a, F units)
{
    int total = 0;
    for (int e0 = 0; e0 < a.E; e0 += 64) {
        const int e = e0 + (threadIdx.x & 63);
        int n = e < a.E ? units(group_of(a, e)) : 0;
        n = wave_inclusive_sum(n);
        total += __builtin_amdgcn_readlane(n, 63);
    }
    return total;
}

// The expert that unit `u` belongs to, and its number within the expert.
template <typename F>
__device__ __forceinline__ int find_unit(const ExpertArgs& a, int u, F units, int& within)
{
    int before = 0;
    for (int e0 = 0; e0 < a.E; e0 += 64) {
        const int e = e0 + (threadIdx.x & 63);
        const int n = e < a.E ? units(group_of(a, e)) : 0;
        const int incl = before + wave_inclusive_sum(n);
        const uint64_t m = __ballot(incl > u);
        if (m != 0) {
            const int at = __builtin_ctzll(m);
            within = u - __builtin_amdgcn_readlane(incl - n, at);
            return e0 + at;
        }
        before = __builtin_amdgcn_readlane(incl, 63);
    }
    within = 0;
    return -1;
}

// LDS placement of 16-byte chunks.  Along: rows of 128 bytes; a fragment read
// takes one chunk of 16 consecutive rows per cycle, and rows of equal parity
// share a half of the banks, so the chunk is moved by the row's bits 1 to 3.
__device__ __forceinline__ int along_swizzle(int row) { return (row >> 1) & 7; }
// Across, bf16: a transposing read takes 32 bytes of rows b .. b+3 and
// b+8 .. b+11 per cycle: eight chunk pairs that must not share banks.
__device__ __forceinline__ int across_swizzle(int row, uint16_t) { return 2 * ((row & 3) | (((row >> 3) & 1) << 2)); }
// (tiles of 64 columns: rows of 128 bytes, of which two share the banks)
__device__ __forceinline__ int across_swizzle_64(int row) { return 2 * (((row >> 1) & 1) | (((row >> 3) & 1) << 1)); }
// Across, float32: a read takes 64 bytes of rows 4 apart per cycle.
__device__ __forceinline__ int across_swizzle(int row, float) { return ((row >> 2) & 3) << 2; }

typedef short v4i16 __attribute__((ext_vector_type(4)));
__device__ __forceinline__ uint2 lds_read_transposed(const void* lds)
{
    const v4i16 v = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) v4i16*)lds);
    return __builtin_bit_cast(uint2, v);
}

// One operand tile in LDS: N columns (output features or rows) by KB
// reduction indices, 128 * N bytes either way.
template <typename T, int N, bool ACROSS, int NW>
struct Operand {
    static constexpr int ESZ = sizeof(T), E = 16 / ESZ, KB = 128 / ESZ;
    static constexpr int CHUNKS = ACROSS ? N / E : 8;            // per LDS row
    static constexpr int LINES = ACROSS ? KB : N;                // LDS rows
    static constexpr int COPIES = LINES * CHUNKS / 64 / NW;      // 1 KB copies per wave and step
    static constexpr int BYTES = N * 128;
    static_assert(COPIES >= 1 && LINES * CHUNKS % (64 * NW) == 0, "whole copies");

    static __device__ __forceinline__ int swizzle(int line)
    {
        if (!ACROSS) return along_swizzle(line);
        if (ESZ == 2 && N == 64) return across_swizzle_64(line);
        return across_swizzle(line, T{});
    }

    uint32_t off[COPIES];   // byte offset of the lane's 16 bytes at step 0, kOOB: never valid
    int k0;                 // along: the lane's first reduction index at step 0
    const char* base;       // (uniform) where offset 0 is
    uint32_t bytes;

    // along: `n` valid rows of `stride` elements from `p`, `len` reduction
    // indices.  across: `n` valid columns from `p`, rows of `stride` elements.
    __device__ void init(const void* p, int64_t n, int64_t stride)
    {
        const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
        base = static_cast<const char*>(p);
#pragma unroll
        for (int j = 0; j < COPIES; ++j) {
            const int at = (wave + NW * j) * 64 + lane;
            const int line = at / CHUNKS, lc = (at % CHUNKS) ^ swizzle(line);
            if (ACROSS) {
                off[j] = lc * E < n ? (uint32_t)(line * stride + lc * E) * ESZ : kOOB;
            } else {
                off[j] = (uint32_t)(line * stride + lc * E) * ESZ;
                k0 = lc * E;   // the same for every j: a wave's rows differ by multiples of 16
            }
        }
        static_assert(ACROSS || COPIES == 1 || NW % 2 == 0, "the lane's chunk is the same in every copy");
    }

    // Copy of a step's tile to LDS.  along: reduction indices from `k` on, of
    // `len`; across: the descriptor already starts at the step's first row.
    __device__ __forceinline__ void copy(const u32x4_t& rsrc, int k, int len, uint4* lds) const
    {
        const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        const uint32_t kill = ACROSS || k + k0 < len ? 0u : kOOB;
#pragma unroll
        for (int j = 0; j < COPIES; ++j)
            buf_load16_lds(rsrc, ACROSS ? off[j] : (off[j] + (uint32_t)k * ESZ) | kill, lds_addr(lds + (wave + NW * j) * 64));
    }
};

// The 16-wide fragment of columns cb .. cb+15 at the ks-th 64-byte part of a
// step (32 bf16 or 16 float32 reduction indices).
template <typename T, int N, bool ACROSS, int NW>
__device__ __forceinline__ uint4 fragment(const char* lds, int cb, int ks)
{
    using O = Operand<T, N, ACROSS, NW>;
    const int lane = threadIdx.x & 63;
    if (!ACROSS) {
        const int row = cb + (lane & 15);
        return *reinterpret_cast<const uint4*>(lds + row * 128 + (((ks * 4 + (lane >> 4)) ^ O::swizzle(row)) << 4));
    }
    if (sizeof(T) == 2) {
        const int line = ks * 32 + 8 * (lane >> 4) + ((lane >> 2) & 3), col = cb + 4 * (lane & 3);
        auto at = [&](int r) { return lds + r * (N * 2) + (((col >> 3) ^ O::swizzle(r)) << 4) + ((col & 7) << 1); };
        const uint2 lo = lds_read_transposed(at(line)), hi = lds_read_transposed(at(line + 4));
        return make_uint4(lo.x, lo.y, hi.x, hi.y);
    }
    const int line = ks * 16 + 4 * (lane >> 4), col = cb + (lane & 15);
    auto at = [&](int r) {
        return *reinterpret_cast<const uint32_t*>(lds + r * (N * 4) + (((col >> 2) ^ O::swizzle(r)) << 4) + ((col & 3) << 2));
    };
    return make_uint4(at(line), at(line + 1), at(line + 2), at(line + 3));
}

// Four consecutive output features of one row.
__device__ __forceinline__ void store_features(__amdgpu_buffer_rsrc_t r, uint32_t elem, bool ok, const floatx4& v, uint16_t)
{
    const u32x2 w = {pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3])};
    __builtin_amdgcn_raw_buffer_store_b64(w, r, ok ? elem * 2u : kOOB, 0, 0);
}
__device__ __forceinline__ void store_features(__amdgpu_buffer_rsrc_t r, uint32_t elem, bool ok, const floatx4& v, float)
{
    __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, v), r, ok ? elem * 4u : kOOB, 0, 0);
}

// Where a tile of rows lies: expert, first row, rows.
struct RowTile {
    int expert;
    int64_t row0;
    int rows;
};

// TP x TQ output tile by NWP x NWQ waves, two buffers of a 128-byte step of
// both operands, the next step's copies in flight during this one's products.
template <typename T, int KIND, int TP, int TQ, int NWP, int NWQ>
__global__ __launch_bounds__(NWP* NWQ * 64) void expert_kernel(ExpertArgs a)
{
    constexpr int NW = NWP * NWQ, FM = TP / NWP / 16, FN = TQ / NWQ / 16;
    using OP = Operand<T, TP, KIND != FWD, NW>;
    using OQ = Operand<T, TQ, KIND == WEIGHT, NW>;
    constexpr int KB = OP::KB;
    __shared__ uint4 lds_p[2][OP::BYTES / 16];
    __shared__ uint4 lds_q[2][OQ::BYTES / 16];

    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wp = wave / NWQ, wq = wave % NWQ;

    // the workgroup's tile
    const int P = KIND == FWD ? a.K : a.C;                     // features of the output
    const int ptiles = (P + TP - 1) / TP, qtiles = KIND == WEIGHT ? (a.K + TQ - 1) / TQ : 1;
    auto units = [&](const Group& g) -> int {
        if (KIND == WEIGHT) return (int)max((g.count + a.split_rows - 1) / a.split_rows, (int64_t)1);
        return (int)((g.count + TQ - 1) / TQ);
    };
    const int nunits = count_units(a, units);
    const int per = ptiles * qtiles, total = nunits * per;
    if ((int)blockIdx.x >= total) return;
    const int b = xcd_remap(blockIdx.x, total);
    int unit, pt, qt = 0;
    if (KIND == WEIGHT) {
        unit = b / per;
        const int t = b - unit * per;
        qt = t / ptiles;
        pt = t - qt * ptiles;
    } else {
        // blocks of a few row tiles by all feature tiles, so that the tiles
        // that run at one time share both operands in the cache
        constexpr int GR = 4;
        const int blk = b / (GR * ptiles), in_blk = b - blk * GR * ptiles;
        const int h = min(GR, nunits - blk * GR);
        pt = in_blk / h;
        unit = blk * GR + in_blk - pt * h;
    }
    int within;
    const int e = __builtin_amdgcn_readfirstlane(find_unit(a, unit, units, within));
    if (e < 0) return;
    const Group g = group_of(a, e);
    within = __builtin_amdgcn_readfirstlane(within);
    const int p0 = pt * TP, q0 = qt * TQ;

    OP op;
    OQ oq;
    int64_t row0 = 0;       // first row of the tile (weight: of the part)
    int64_t len;            // reduction indices
    int64_t qrows = 0;
    if (KIND == WEIGHT) {
        row0 = g.first + (int64_t)within * a.split_rows;
        len = min((int64_t)a.split_rows, g.first + g.count - row0);
        op.init(static_cast<const T*>(a.p) + row0 * a.x_stride + p0, a.C - p0, a.x_stride);
        oq.init(static_cast<const T*>(a.q) + row0 * a.y_stride + q0, a.K - q0, a.y_stride);
    } else {
        const int64_t qstride = KIND == FWD ? a.x_stride : a.y_stride;
        const T* w = static_cast<const T*>(a.p) + (int64_t)e * a.K * a.C;
        row0 = g.first + (int64_t)within * TQ;
        qrows = min((int64_t)TQ, g.first + g.count - row0);
        len = KIND == FWD ? a.C : a.K;
        if (KIND == FWD) op.init(w + (int64_t)p0 * a.C, min(TP, a.K - p0), a.C);
        else op.init(w + p0, a.C - p0, a.C);
        oq.init(static_cast<const T*>(a.q) + row0 * qstride, qrows, qstride);
    }

    auto copy = [&](int64_t k, int buf) {
        // P
        if (KIND == FWD) {
            const uint32_t n = (uint32_t)min(TP, a.K - p0) * (uint32_t)a.C * sizeof(T);
            op.copy(make_rsrc_words(op.base, n), (int)k, (int)len, lds_p[buf]);
        } else {
            const int64_t stride = KIND == WEIGHT ? a.x_stride : (int64_t)a.C;
            const int64_t left = min(len - k, (int64_t)KB);
            // the last row ends with its own columns
            const uint32_t n = (uint32_t)(((left - 1) * stride + a.C - p0) * (int64_t)sizeof(T));
            op.copy(make_rsrc_words(op.base + k * stride * (int64_t)sizeof(T), n), 0, 0, lds_p[buf]);
        }
        if (KIND == WEIGHT) {
            const int64_t left = min(len - k, (int64_t)KB);
            const uint32_t n = (uint32_t)(((left - 1) * a.y_stride + a.K - q0) * (int64_t)sizeof(T));
            oq.copy(make_rsrc_words(oq.base + k * a.y_stride * (int64_t)sizeof(T), n), 0, 0, lds_q[buf]);
        } else {
            const int64_t stride = KIND == FWD ? a.x_stride : a.y_stride;
            const uint32_t n = (uint32_t)(((qrows - 1) * stride + len) * (int64_t)sizeof(T));
            oq.copy(make_rsrc_words(oq.base, n), (int)k, (int)len, lds_q[buf]);
        }
    };

    floatx4 acc[FM][FN];
#pragma unroll
    for (int i = 0; i < FM; ++i)
#pragma unroll
        for (int j = 0; j < FN; ++j) acc[i][j] = floatx4{0.f, 0.f, 0.f, 0.f};

    const int64_t steps = (len + KB - 1) / KB;
    if (steps > 0) {
        copy(0, 0);
        wait_vmem();
        __syncthreads();
    }
    for (int64_t s = 0; s < steps; ++s) {
        const int buf = (int)(s & 1);
        if (s + 1 < steps) copy((s + 1) * KB, buf ^ 1);
        const char* lp = reinterpret_cast<const char*>(lds_p[buf]);
        const char* lq = reinterpret_cast<const char*>(lds_q[buf]);
#pragma unroll
        for (int ks = 0; ks < 2; ++ks) {
            uint4 fp[FM], fq[FN];
#pragma unroll
            for (int i = 0; i < FM; ++i) fp[i] = fragment<T, TP, KIND != FWD, NW>(lp, wp * (TP / NWP) + i * 16, ks);
#pragma unroll
            for (int j = 0; j < FN; ++j) fq[j] = fragment<T, TQ, KIND == WEIGHT, NW>(lq, wq * (TQ / NWQ) + j * 16, ks);
#pragma unroll
            for (int i = 0; i < FM; ++i)
#pragma unroll
                for (int j = 0; j < FN; ++j) acc[i][j] = mfma_chunk(acc[i][j], fp[i], fq[j], T{});
        }
        wait_vmem();
        __syncthreads();
    }

    const int pl = p0 + wp * (TP / NWP) + 4 * (lane >> 4), ql = wq * (TQ / NWQ) + (lane & 15);
    if (KIND == WEIGHT) {
        float* out = nullptr;
        auto slots = [&](const Group& gg) -> int {
            const int n = units(gg);
            return n > 1 ? n : 0;
        };
        if (units(g) > 1) {
            // the expert's slots follow those of the split experts before it
            int before = 0;
            for (int e0 = 0; e0 < e; e0 += 64) {
                const int x = e0 + lane;
                before += __builtin_amdgcn_readlane(wave_inclusive_sum(x < e ? slots(group_of(a, x)) : 0), 63);
            }
            if (before + within < a.slots) out = a.partial + (int64_t)(before + within) * a.K * a.C;   // (offsets that decrease)
        } else {
            out = static_cast<float*>(a.out) + (int64_t)e * a.K * a.C;
        }
        const __amdgpu_buffer_rsrc_t r = make_rsrc(out, out ? (uint32_t)a.K * (uint32_t)a.C * 4u : 0u);
#pragma unroll
        for (int j = 0; j < FN; ++j) {
            const int k = q0 + ql + j * 16;
#pragma unroll
            for (int i = 0; i < FM; ++i)
                store_features(r, (uint32_t)k * (uint32_t)a.C + pl + i * 16, k < a.K && pl + i * 16 < a.C, acc[i][j], 0.f);
        }
        return;
    }
    const int64_t ostride = KIND == FWD ? a.y_stride : a.x_stride;
    const __amdgpu_buffer_rsrc_t r = make_rsrc(static_cast<T*>(a.out) + row0 * ostride,
                                               (uint32_t)(((qrows - 1) * ostride + P) * (int64_t)sizeof(T)));
#pragma unroll
    for (int j = 0; j < FN; ++j) {
        const int q = ql + j * 16;
        const bool row_in = q < qrows;
        uint32_t bits16 = 0;
#pragma unroll
        for (int i = 0; i < FM; ++i) {
            const int p = pl + i * 16;
            floatx4 v = acc[i][j];
            if (KIND == FWD && a.relu)
#pragma unroll
                for (int c = 0; c < 4; ++c) v[c] = v[c] > 0.f ? v[c] : 0.f;
            if (KIND == DATA && a.mask && row_in && p < P) {
                const int64_t bit = (row0 + q) * (int64_t)P + p;
                const uint32_t m = reinterpret_cast<const uint8_t*>(a.mask)[bit >> 3] >> (bit & 7);
#pragma unroll
                for (int c = 0; c < 4; ++c) v[c] = (m >> c) & 1u ? v[c] : 0.f;
            }
            store_features(r, (uint32_t)(q * ostride + p), row_in && p < P, v, T{});
            if (KIND == FWD && a.out_mask) {
                // the footprint of what is stored (a sum below the smallest bf16 rounds to zero); the four lane groups' nibbles
                // make 16 bits, two blocks a word
                uint32_t nib = 0;
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    const float s = sizeof(T) == 2 ? __uint_as_float(f32_to_bf16_rne(v[c]) << 16) : v[c];
                    nib |= (s > 0.f ? 1u : 0u) << c;
                }
                nib <<= 4 * (lane >> 4);
                nib |= __shfl_xor(nib, 16);
                nib |= __shfl_xor(nib, 32);
                if (i & 1) {
                    const int pw = p0 + wp * (TP / NWP) + (i - 1) * 16;   // a multiple of 32
                    if (lane < 16 && row_in && pw < P)
                        a.out_mask[((row0 + q) * (int64_t)P + pw) >> 5] = bits16 | (nib << 16);
                } else {
                    bits16 = nib;
                }
            }
        }
    }
}

// Sums of the split experts' parts, in order.
__global__ __launch_bounds__(256) void expert_sum_kernel(ExpertArgs a)
{
    const int64_t vecs = (int64_t)a.K * a.C / 4;
    int64_t slot = 0;
    for (int e0 = 0; e0 < a.E; e0 += 64) {
        const int x = e0 + (threadIdx.x & 63);
        int n = 0;
        if (x < a.E) n = (int)((group_of(a, x).count + a.split_rows - 1) / a.split_rows);
        uint64_t todo = __ballot(n > 1);
        for (; todo != 0; todo &= todo - 1) {
            const int at = __builtin_ctzll(todo);
            const int parts = __builtin_amdgcn_readlane(n, at);
            if (slot + parts > a.slots) return;   // (offsets that decrease)
            const floatx4* src = reinterpret_cast<const floatx4*>(a.partial) + slot * vecs;
            floatx4* dst = reinterpret_cast<floatx4*>(static_cast<float*>(a.out)) + (int64_t)(e0 + at) * vecs;
            for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < vecs; i += (int64_t)gridDim.x * 256) {
                floatx4 s = src[i];
                for (int z = 1; z < parts; ++z) s += src[z * vecs + i];
                dst[i] = s;
            }
            slot += parts;
        }
    }
}

// The most row tiles that any lengths can give.
int64_t most_units(int64_t rows, int E, int tile) { return rows / tile + std::min<int64_t>(E, rows); }

template <typename T, int KIND, int TP, int TQ, int NWP, int NWQ>
hipError_t launch_tiles(const ExpertArgs& a, hipStream_t s)
{
    const int P = KIND == FWD ? a.K : a.C;
    const int64_t per = (int64_t)((P + TP - 1) / TP) * (KIND == WEIGHT ? (a.K + TQ - 1) / TQ : 1);
    const int64_t units = KIND == WEIGHT ? a.rows / a.split_rows + a.E : most_units(a.rows, a.E, TQ);
    if (units == 0) return hipSuccess;
    if (units * per > 0x7fffffff) return hipErrorInvalidValue;
    expert_kernel<T, KIND, TP, TQ, NWP, NWQ><<<(int)(units * per), NWP * NWQ * 64, 0, s>>>(a);
    return hipGetLastError();
}

}  // namespace

ExpertPlan expert_plan(const cbw_expert_desc* d)
{
    ExpertPlan p{};
    const int64_t tiles = (int64_t)((d->C + 255) / 256) * ((d->K + 255) / 256);
    int64_t len = d->rows * tiles / 1024;
    len = std::max<int64_t>(1024, (len + 63) / 64 * 64);
    p.split_rows = (int)std::min<int64_t>(len, 1 << 30);
    p.slots = d->rows > p.split_rows ? 2 * d->rows / p.split_rows : 0;
    p.ws_bytes = (size_t)p.slots * d->K * d->C * 4;
    return p;
}

hipError_t launch_expert_fwd(int dtype, const ExpertArgs& a, hipStream_t s)
{
    if (dtype == CBW_F32) return launch_tiles<float, FWD, 64, 64, 2, 2>(a, s);
    return launch_tiles<uint16_t, FWD, 256, 256, 2, 4>(a, s);
}

hipError_t launch_expert_bwd_data(int dtype, const ExpertArgs& a, hipStream_t s)
{
    if (dtype == CBW_F32) return launch_tiles<float, DATA, 64, 64, 2, 2>(a, s);
    return launch_tiles<uint16_t, DATA, 256, 256, 2, 4>(a, s);
}

hipError_t launch_expert_bwd_weight(int dtype, const ExpertArgs& a, hipStream_t s)
{
    hipError_t e = dtype == CBW_F32 ? launch_tiles<float, WEIGHT, 64, 64, 2, 2>(a, s)
                                    : launch_tiles<uint16_t, WEIGHT, 256, 256, 2, 4>(a, s);
    if (e != hipSuccess || a.rows <= a.split_rows) return e;
    expert_sum_kernel<<<2048, 256, 0, s>>>(a);
    return hipGetLastError();
}

}  // namespace cbw
