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
// Every workgroup finds its experts and tiles itself: a wave scans the group
// lengths (E + 1 offsets, in the cache) and looks its own number up.  The
// tiled kernel has as many workgroups as are resident, which go through the
// tiles in turn; the streaming kernel has one for every tile that any lengths
// could give, and the surplus ones leave.
//
// Bound by the matrix cores where an expert has some hundred rows (16384 rows
// over 8 experts, 2048 -> 8192 features, bf16: 502 us, 1095 TFLOP/s; with groups
// of whole tiles 475 us, 1155), by reading the filters where it has few (12
// rows over 32 experts, 2048 -> 1408: 14.6 to 15.1 us, 4.0 TB/s, filters read from
// memory; 10.5 to 13 where calls in turn leave part of them in the 256 MB
// cache).  The weight gradient of narrow experts takes its products and the
// writing of its results in turn (64 uneven experts, 32768 rows, 2048 -> 1408:
// 310 to 343 us, 3.1 to 2.8 TB/s beside 610 to 550 TFLOP/s).  float32: 8192
// rows over 8 experts, 1024 -> 2048, forward 292 us, data 303, weight 296,
// 118 to 113 TFLOP/s.
#include "common.hpp"
#include "block_kernels.hpp"
#include "tiles.hpp"

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

// Inclusive sum over the wave's lanes: shifts within rows of 16 lanes, then the
// rows' totals carried on (register moves, no trip through the LDS).
__device__ __forceinline__ int wave_inclusive_sum(int v)
{
    v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xf, 0xf, false);   // row_shr 1, 2, 4, 8
    v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xf, 0xf, false);
    v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xf, 0xf, false);
    v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xf, 0xf, false);
    v += __builtin_amdgcn_update_dpp(0, v, 0x142, 0xa, 0xf, false);   // lane 15 of a row to the next one
    v += __builtin_amdgcn_update_dpp(0, v, 0x143, 0xc, 0xf, false);   // lane 31 to the upper half
    return v;
}

// The work of all experts, numbered through: expert e has units(e's group) of
// it.  Up to 64 experts a lane keeps its expert's numbers; more are gone
// through 64 at a time, again for every question.  SORTED: up to 64 experts go
// by their rows, most first, more stay as they are.  Called by whole waves;
// every result is the same in all lanes.
template <bool SORTED, typename F>
struct Units {
    const ExpertArgs& a;
    F units;
    int e, n, incl, total;   // the lane's expert and its units; of all

    __device__ Units(const ExpertArgs& args, F f) : a(args), units(f)
    {
        total = 0;
        if (SORTED && a.E <= 64) {
            const int lane = threadIdx.x & 63;
            const int rows = lane < a.E ? (int)group_of(a, lane).count : -1;
            int rank = 0;
            for (int j = 0; j < a.E; ++j) {
                const int other = __builtin_amdgcn_readlane(rows, j);
                rank += other > rows || (other == rows && j < lane) ? 1 : 0;
            }
            // the expert of rank l to lane l (lanes past the last expert keep their place)
            e = __builtin_amdgcn_ds_permute((lane < a.E ? rank : lane) * 4, lane);
        } else {
            e = threadIdx.x & 63;
        }
        for (int e0 = 0; e0 < a.E; e0 += 64) {
            load(e0, total);
            total = __builtin_amdgcn_readlane(incl, 63);
        }
    }
    __device__ void load(int e0, int before)
    {
        n = e0 + e < a.E ? units(group_of(a, e0 + e)) : 0;
        incl = before + wave_inclusive_sum(n);
    }
    // The expert that unit u belongs to, and its number within the expert.
    __device__ int find(int u, int& within)
    {
        for (int e0 = 0, before = 0; e0 < a.E; e0 += 64) {
            if (a.E > 64) load(e0, before);
            const uint64_t m = __ballot(incl > u);
            if (m != 0) {
                const int at = __builtin_ctzll(m);
                within = u - __builtin_amdgcn_readlane(incl - n, at);
                return e0 + __builtin_amdgcn_readlane(e, at);
            }
            before = __builtin_amdgcn_readlane(incl, 63);
        }
        within = 0;
        return -1;
    }
};
template <bool SORTED, typename F>
__device__ __forceinline__ Units<SORTED, F> number_units(const ExpertArgs& a, F f) { return Units<SORTED, F>(a, f); }

// Waits until at most N of the wave's copies to LDS are in flight; the LDS reads
// that follow stay behind it.
template <int N>
__device__ __forceinline__ void wait_copies()
{
    static_assert(N <= 63, "the counter's range");
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}
// Until the wave's LDS reads have returned: what they read may be overwritten.
__device__ __forceinline__ void wait_reads() { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); }
__device__ __forceinline__ void barrier() { asm volatile("s_barrier" ::: "memory"); }
// Between LDS accesses by which the lanes of one wave exchange values: the
// LDS serves a wave's in their order, the compiler has to leave them in it.
__device__ __forceinline__ void wave_fence()
{
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

typedef short v4i16 __attribute__((ext_vector_type(4)));
__device__ __forceinline__ uint2 lds_read_transposed(const void* lds)
{
    const v4i16 v = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) v4i16*)lds);
    return __builtin_bit_cast(uint2, v);
}

// One operand tile in LDS: N columns (output features or rows) by 128 bytes of
// reduction indices, filled by NW waves.
template <typename T, int N, bool ACROSS, int NW>
struct Operand {
    static constexpr int ESZ = sizeof(T), E = 16 / ESZ, KB = 128 / ESZ;
    static constexpr int CHUNKS = ACROSS ? N / E : 8;            // per LDS row
    static constexpr int LINES = ACROSS ? KB : N;                // LDS rows
    static constexpr int COPIES = LINES * CHUNKS / 64 / NW;      // 1 KB copies per wave and step
    static constexpr int BYTES = N * 128;
    static_assert(COPIES >= 1 && LINES * CHUNKS % (64 * NW) == 0, "whole copies");

    // Placement of the 16-byte chunks of an LDS row.  The LDS serves 256 bytes
    // (all banks) a cycle.  Along: a fragment read takes one chunk of 16
    // consecutive rows per cycle; of its rows of 128 bytes two share the
    // banks, so the chunk is moved by the row's bits 1 to 3.  Across, bf16: a transposing read takes 32
    // bytes of rows b .. b+3 and b+8 .. b+11 per cycle: eight chunk pairs that
    // must not share banks (tiles of 64 columns: rows of 128 bytes, two of
    // them to the banks; of 32: four).  Across, float32: 64 bytes of rows 4 apart.
    static __device__ __forceinline__ int swizzle(int line)
    {
        if (!ACROSS) return (line >> 1) & 7;
        if (ESZ == 4) return N >= 64 ? ((line >> 2) & 3) << 2 : ((line >> 2) & 1) << 2;
        if (N >= 128) return 2 * ((line & 3) | (((line >> 3) & 1) << 2));
        if (N == 64) return 2 * (((line >> 1) & 1) | (((line >> 3) & 1) << 1));
        return 2 * ((line >> 3) & 1);
    }

    // Copies DIST apart lie a multiple of 16 LDS rows apart, which the swizzle
    // does not see: the same lane has the same chunk, so its byte offset grows
    // by a uniform amount.
    static constexpr int LINES_PER_COPY = NW * 64 / CHUNKS;
    static constexpr int DIST = LINES_PER_COPY % 16 == 0 ? 1 : 16 / LINES_PER_COPY;
    static_assert(COPIES < DIST || COPIES % DIST == 0, "every distinct copy as often");
    static constexpr int OWN = COPIES < DIST ? COPIES : DIST;

    uint32_t off[OWN];   // byte offset of the lane's 16 bytes at step 0, kOOB: never valid
    uint32_t apart;      // (uniform) bytes from a copy to the one DIST further

    // along: rows of `stride` elements; across: `n` valid columns
    __device__ __forceinline__ void init(int wave, int64_t n, int64_t stride)
    {
        const int lane = threadIdx.x & 63;
#pragma unroll
        for (int j = 0; j < OWN; ++j) {
            const int at = (wave + NW * j) * 64 + lane;
            const int line = at / CHUNKS, lc = (at % CHUNKS) ^ swizzle(line);
            off[j] = ACROSS && lc * E >= n ? kOOB : (uint32_t)(line * stride + lc * E) * ESZ;
        }
        apart = (uint32_t)(DIST * LINES_PER_COPY * stride) * ESZ;
    }

    // Copy of a step's tile to LDS.  along: reduction indices from `k` on, of
    // `len`; across: the descriptor already starts at the step's first row.
    __device__ __forceinline__ void copy(int wave, const u32x4_t& rsrc, int k, int len, char* lds) const
    {
        const int lane = threadIdx.x & 63;
#pragma unroll
        for (int j = 0; j < COPIES; ++j) {
            uint32_t o = off[j % OWN] + (uint32_t)(j / OWN) * apart;
            if (!ACROSS) {
                // (only a last, short step has indices to leave out)
                const int lc = (lane % CHUNKS) ^ swizzle(((wave + NW * (j % OWN)) * 64 + lane) / CHUNKS);
                o += (uint32_t)k * ESZ;
                if (k + KB > len && k + lc * E >= len) o = kOOB;
            }
            buf_load16_lds(rsrc, o, lds_addr(lds + (wave + NW * j) * 1024));
        }
    }

    // Fragments of the F blocks of 16 columns from cb on (a multiple of 16 F), at
    // the ks-th 64-byte part of a step (32 bf16 or 16 float32 reduction
    // indices).  Within a tile a fragment's place differs from the first one's
    // by bits that the swizzle leaves to a plain exclusive or, so that one
    // register serves all of them: kept apart they would fill the registers of
    // the 256 x 256 tile.
    static __device__ __forceinline__ int first(int cb)
    {
        const int lane = threadIdx.x & 63;
        if (!ACROSS) return (cb + (lane & 15)) * 128 + (((lane >> 4) ^ swizzle(lane & 15)) << 4);
        if (ESZ == 2) {
            const int line = 8 * (lane >> 4) + ((lane >> 2) & 3), col = cb + 4 * (lane & 3);
            return line * (N * 2) + (((col >> 3) ^ swizzle(line)) << 4) + ((col & 7) << 1);
        }
        const int line = 4 * (lane >> 4), col = cb + (lane & 15);
        return line * (N * 4) + (((col >> 2) ^ swizzle(line)) << 4) + ((col & 3) << 2);
    }
    template <int F>
    static __device__ __forceinline__ void fragments(const char* lds, int at, int ks, uint4 (&f)[F])
    {
        static_assert((F & (F - 1)) == 0, "a power of two");
        asm volatile("" : "+v"(at));   // (not to be worked out ahead for every block)
#pragma unroll
        for (int i = 0; i < F; ++i) {
            if (!ACROSS) {
                f[i] = *reinterpret_cast<const uint4*>(lds + (at ^ (ks * 64)) + i * 2048);
            } else if (ESZ == 2) {
                const char* p = lds + (at ^ (i * 32)) + ks * 64 * N;
                const uint2 lo = lds_read_transposed(p), hi = lds_read_transposed(p + 8 * N);
                f[i] = make_uint4(lo.x, lo.y, hi.x, hi.y);
            } else {
                const uint32_t* p = reinterpret_cast<const uint32_t*>(lds + (at ^ (i * 64)) + ks * 64 * N);
                f[i] = make_uint4(p[0], p[N], p[2 * N], p[3 * N]);
            }
        }
    }
};

// Output rows of P features, `stride` elements apart, a tile's first row at
// offset 0 (weight gradient: an output feature's row of input features).
//
// A wave has 16 rows by 16 I features at a time, a lane four features of each
// block of 16: stored so, an instruction would write 32 bytes to each of 16
// rows (bf16).  They pass through the wave's own piece of LDS instead, and a
// lane takes a vector of consecutive features of one row, with the footprint's
// bits for them next to each other: an instruction writes whole lines.  (16384
// rows, 2048 -> 8192: 550 us, 507 so.  Weight gradient of 64 experts, 32768
// rows, 2048 -> 1408, whose lines would be written by halves: 1.1 GB written
// for 0.74 GB of results and 402 us, 313 so.)
template <typename T, int KIND, int I>
struct Output {
    static constexpr int E = 16 / (int)sizeof(T);              // features of a vector
    static constexpr int ROW = I * 16 * (int)sizeof(T);        // bytes of a row in LDS
    static constexpr int CHUNKS = ROW / 16, VECS = I * (int)sizeof(T) / 4;
    static constexpr int BYTES = 16 * ROW;                     // LDS per wave
    static_assert(CHUNKS >= 4 && (CHUNKS & (CHUNKS - 1)) == 0 && 64 % CHUNKS == 0, "whole rows to an instruction");

    const ExpertArgs& a;
    __amdgpu_buffer_rsrc_t r;
    int64_t row0, stride;
    int rows, P;

    __device__ Output(const ExpertArgs& args, int64_t first, int n)
        : a(args), row0(first), stride(KIND == FWD ? args.y_stride : args.x_stride), rows(n), P(KIND == FWD ? args.K : args.C)
    {
        r = make_rsrc(static_cast<T*>(a.out) + row0 * stride, (uint32_t)(((rows - 1) * stride + P) * (int64_t)sizeof(T)));
    }
    // (weight gradient: n rows of `out`, null: nothing is written)
    __device__ Output(const ExpertArgs& args, float* out, int n) : a(args), row0(0), stride(args.C), rows(n), P(args.C)
    {
        r = make_rsrc(out, out ? (uint32_t)rows * (uint32_t)P * 4u : 0u);
    }

    // the row and the feature of the lane's t-th vector, from the block's first
    static __device__ __forceinline__ int row_of(int lane, int t) { return t * (64 / CHUNKS) + lane / CHUNKS; }
    static __device__ __forceinline__ int feature_of(int lane) { return (lane % CHUNKS) * E; }
    // the lane's number, which the compiler takes for a new one each time: it
    // would keep all that follows from it in registers during the products
    static __device__ __forceinline__ int my_lane()
    {
        int lane = threadIdx.x & 63;
        asm volatile("" : "+v"(lane));
        return lane;
    }
    __device__ __forceinline__ int64_t bit_of(int q, int p) const { return (row0 + q) * (int64_t)P + p; }

    // The footprint of rows q0 .. q0 + 15, features p0 on (data gradient): where
    // its rows are whole words, a word to a lane, row by row.
    __device__ __forceinline__ bool words() const { return (P & 31) == 0; }
    __device__ __forceinline__ uint32_t load_live(int q0, int p0) const
    {
        if (KIND != DATA || !a.mask || !words()) return 0;
        const int lane = my_lane(), q = q0 + lane / (I / 2), p = p0 + lane % (I / 2) * 32;
        return lane < 8 * I && q < rows && p < P ? a.mask[bit_of(q, p) >> 5] : 0u;
    }
    // the bits of the lane's vector of row rr
    __device__ __forceinline__ uint32_t live_bits(uint32_t word, int lane, int rr, int q, int p) const
    {
        if (!a.mask) return ~0u;
        if (words()) return __shfl(word, rr * (I / 2) + feature_of(lane) / 32) >> (feature_of(lane) % 32);
        return q < rows && p < P ? reinterpret_cast<const uint8_t*>(a.mask)[bit_of(q, p) >> 3] >> (bit_of(q, p) & 7) : 0u;
    }

    // v[i]: the lane's four features of block i of rows q0 .. q0 + 15.
    template <typename V>
    __device__ __forceinline__ void put(char* lds, int q0, int p0, const V& v, uint32_t live) const
    {
        const int lane = my_lane(), row = lane & 15;
        wave_fence();   // (the block before this one has been read)
        // (a row's chunks are moved by its number: the 16 rows' do not share banks)
        auto at = [&](int rr, int chunk) { return lds + rr * ROW + ((chunk ^ (rr & (CHUNKS - 1))) << 4); };
#pragma unroll
        for (int i = 0; i < I; ++i) {
            floatx4 x = v(i);
            if (KIND == FWD && a.relu)
#pragma unroll
                for (int c = 0; c < 4; ++c) x[c] = x[c] > 0.f ? x[c] : 0.f;
            if (sizeof(T) == 2)
                *reinterpret_cast<u32x2*>(at(row, i * 2 + (lane >> 5)) + (lane >> 4 & 1) * 8) =
                    u32x2{pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3])};
            else
                *reinterpret_cast<u32x4*>(at(row, i * 4 + (lane >> 4))) = __builtin_bit_cast(u32x4, x);
        }
        wave_fence();
#pragma unroll
        for (int t = 0; t < VECS; ++t) {
            const int rr = row_of(lane, t), q = q0 + rr, p = p0 + feature_of(lane);
            const bool ok = q < rows && p < P;
            u32x4 w = *reinterpret_cast<const u32x4*>(at(rr, lane % CHUNKS));
            if (KIND == DATA) {
                const uint32_t b = live_bits(live, lane, rr, q, p);
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    w[k] &= sizeof(T) == 2 ? ((b >> 2 * k) & 1u ? 0xffffu : 0u) | ((b >> (2 * k + 1)) & 1u ? 0xffff0000u : 0u)
                                           : ((b >> k) & 1u ? ~0u : 0u);
            }
            // Weight gradients are stored non-temporally: they are not read again
            // here, and as ordinary stores they push the operands out of the L2
            // (64 experts of 512 rows on average, 2048 -> 1408: 333 us, 313 so).
            __builtin_amdgcn_raw_buffer_store_b128(w, r, ok ? (uint32_t)(q * stride + p) * (uint32_t)sizeof(T) : kOOB, 0,
                                                   KIND == WEIGHT ? 2 : 0);
            if (KIND == FWD && a.out_mask) {
                // (after ReLU a stored value is positive unless its bits are zero)
                uint32_t b = 0;
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    b |= sizeof(T) == 2 ? (uint32_t)((w[k] & 0xffffu) != 0) << 2 * k | (uint32_t)((w[k] >> 16) != 0) << (2 * k + 1)
                                        : (uint32_t)(w[k] != 0) << k;
                if (sizeof(T) == 4) b |= __shfl_xor(b, 1) << 4;   // (the even lane's four features are the lower half)
                if (ok && (sizeof(T) == 2 || (lane & 1) == 0))
                    reinterpret_cast<uint8_t*>(a.out_mask)[bit_of(q, p) >> 3] = (uint8_t)b;
            }
        }
    }
};

// TP x TQ output tile by NWP x NWQ waves, two buffers of a 128-byte step of
// both operands.
template <typename T, int KIND, int TP, int TQ, int NWP, int NWQ>
__global__ __launch_bounds__(NWP* NWQ * 64) void expert_kernel(ExpertArgs a)
{
    constexpr int NW = NWP * NWQ, FM = TP / NWP / 16, FN = TQ / NWQ / 16;
    using OP = Operand<T, TP, KIND != FWD, NW>;
    using OQ = Operand<T, TQ, KIND == WEIGHT, NW>;
    constexpr int KB = OP::KB, COPIES = OP::COPIES + OQ::COPIES;
    __shared__ __align__(1024) char lds_p[2][OP::BYTES];
    __shared__ __align__(1024) char lds_q[2][OQ::BYTES];
    using Out = Output<T, KIND, FM>;
    constexpr int WI = FM < 4 ? FM : 4;   // blocks of the weight gradient to a row in LDS
    using OutW = Output<float, KIND, WI>;
    __shared__ __align__(1024) char lds_out[NW][KIND == WEIGHT ? OutW::BYTES : Out::BYTES];

    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wp = wave / NWQ, wq = wave % NWQ;

    // A tile's place: its expert, the first of its rows (weight: of the part's)
    // and how many, its first columns, its reduction indices.
    struct Tile {
        int e, within, p0, q0;
        int64_t row0, len;
        int qrows;
    };
    const int P = KIND == FWD ? a.K : a.C;                     // features of the output
    const int ptiles = (P + TP - 1) / TP, qtiles = KIND == WEIGHT ? (a.K + TQ - 1) / TQ : 1;
    // units of work: row tiles, or (weight) experts and parts of one
    auto all = number_units<KIND == WEIGHT>(a, [&](const Group& g) {
        return KIND == WEIGHT ? (int)max((g.count + a.split_rows - 1) / a.split_rows, (int64_t)1) : (int)((g.count + TQ - 1) / TQ);
    });
    const int per = ptiles * qtiles, total = all.total * per;
    auto place = [&](int unit, int pt, int qt) {
        Tile t;
        int within;
        t.e = __builtin_amdgcn_readfirstlane(all.find(unit, within));
        t.within = __builtin_amdgcn_readfirstlane(within);
        if (t.e < 0) return t;
        const Group g = group_of(a, t.e);
        t.p0 = pt * TP;
        t.q0 = qt * TQ;
        t.row0 = g.first + (int64_t)t.within * (KIND == WEIGHT ? a.split_rows : TQ);
        const int64_t left = g.first + g.count - t.row0;
        // (offsets that decrease can count up to anything: no tile outside its group)
        if (t.within < 0 || left < 0 || (left == 0 && (KIND != WEIGHT || t.within > 0))) t.e = -1;
        t.qrows = KIND == WEIGHT ? 0 : (int)min((int64_t)TQ, left);
        t.len = KIND == WEIGHT ? min((int64_t)a.split_rows, left) : KIND == FWD ? a.C : a.K;
        return t;
    };
    // The workgroup's `turn`-th tile; e < 0: there is none.  A turn is a
    // contiguous range of all tiles, and an XCD's part of it is one as well, so
    // that tiles that run at one time share operands in the cache.
    auto tile_of = [&](int turn) {
        Tile none;
        none.e = -1;
        const int first = turn * (int)gridDim.x, n = min((int)gridDim.x, total - first);
        if ((int)blockIdx.x >= n) return none;
        const int at = xcd_remap(blockIdx.x, n);
        if (KIND == WEIGHT) {
            // The units come longest first, and every other turn goes
            // backwards: who had one of a turn's longer ones has one of the next
            // turn's shorter ones.
            const int b = first + (turn & 1 ? n - 1 - at : at);
            const int unit = b / per, in_unit = b - unit * per;
            return place(unit, in_unit / qtiles, in_unit % qtiles);
        }
        // blocks of eight row tiles by all feature tiles (four: 2 to 10% slower
        // at 16384 rows, 2048 -> 8192 features, 8 experts)
        constexpr int GR = 8;
        const int b = first + at;
        const int blk = b / (GR * ptiles), in_blk = b - blk * GR * ptiles;
        const int h = min(GR, all.total - blk * GR);
        const int pt = in_blk / h;
        return place(blk * GR + in_blk - pt * h, pt, 0);
    };

    Tile t = tile_of(0);
    if (t.e < 0) return;

    OP op;
    OQ oq;
    const char *base_p, *base_q;
    auto aim = [&](const Tile& t) {
        if (KIND == WEIGHT) {
            base_p = reinterpret_cast<const char*>(static_cast<const T*>(a.p) + t.row0 * a.x_stride + t.p0);
            base_q = reinterpret_cast<const char*>(static_cast<const T*>(a.q) + t.row0 * a.y_stride + t.q0);
            op.init(wave, a.C - t.p0, a.x_stride);
            oq.init(wave, a.K - t.q0, a.y_stride);
        } else {
            const int64_t qstride = KIND == FWD ? a.x_stride : a.y_stride;
            const T* w = static_cast<const T*>(a.p) + (int64_t)t.e * a.K * a.C;
            base_p = reinterpret_cast<const char*>(w + (KIND == FWD ? (int64_t)t.p0 * a.C : (int64_t)t.p0));
            base_q = reinterpret_cast<const char*>(static_cast<const T*>(a.q) + t.row0 * qstride);
            op.init(wave, KIND == FWD ? 0 : a.C - t.p0, a.C);
            oq.init(wave, 0, qstride);
        }
    };
    auto copy = [&](const Tile& t, int64_t k, int buf) {
        const int64_t left = min(t.len - k, (int64_t)KB);
        // (an operand that goes across: the step's rows, the last of which ends with its own columns)
        if (KIND == FWD) {
            const uint32_t n = (uint32_t)min(TP, a.K - t.p0) * (uint32_t)a.C * sizeof(T);
            op.copy(wave, make_rsrc_words(base_p, n), (int)k, (int)t.len, lds_p[buf]);
        } else {
            const int64_t stride = KIND == WEIGHT ? a.x_stride : (int64_t)a.C;
            const uint32_t n = (uint32_t)(((left - 1) * stride + a.C - t.p0) * (int64_t)sizeof(T));
            op.copy(wave, make_rsrc_words(base_p + k * stride * (int64_t)sizeof(T), n), 0, 0, lds_p[buf]);
        }
        if (KIND == WEIGHT) {
            const uint32_t n = (uint32_t)(((left - 1) * a.y_stride + a.K - t.q0) * (int64_t)sizeof(T));
            oq.copy(wave, make_rsrc_words(base_q + k * a.y_stride * (int64_t)sizeof(T), n), 0, 0, lds_q[buf]);
        } else {
            const int64_t stride = KIND == FWD ? a.x_stride : a.y_stride;
            const uint32_t n = (uint32_t)(((t.qrows - 1) * stride + t.len) * (int64_t)sizeof(T));
            oq.copy(wave, make_rsrc_words(base_q, n), (int)k, (int)t.len, lds_q[buf]);
        }
    };
    // the first two steps' copies of a tile
    auto start = [&](const Tile& t) {
        aim(t);
        if (t.len > 0) copy(t, 0, 0);
        if (t.len > KB) copy(t, KB, 1);
    };

    floatx4 acc[FM][FN];
    // Fragments of a step's two halves in turn: while the matrix instructions of
    // one run, the reads of the next are under way, so that the LDS latency is
    // under them and not behind the barrier.  The barrier stands between the
    // halves: there every wave holds the step's second half in registers, the
    // buffer is free for the copies two steps ahead, and the next step's have
    // landed.
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
    // one or two reads between every few matrix instructions
    auto interleave = [&]() {
        constexpr int READS = (FM * (KIND != FWD ? 2 : 1) + FN * (KIND == WEIGHT ? 2 : 1)), MUL = FM * FN;
        if (sizeof(T) != 2) return;
#pragma unroll
        for (int i = 0; i < READS; ++i) {
            __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);                    // an LDS read
            __builtin_amdgcn_sched_group_barrier(0x008, MUL / READS, 0);          // matrix instructions
        }
    };
    Fragments fa, fb;
    auto product = [&](const Tile& t) {
#pragma unroll
        for (int i = 0; i < FM; ++i)
#pragma unroll
            for (int j = 0; j < FN; ++j) acc[i][j] = floatx4{0.f, 0.f, 0.f, 0.f};
        const int steps = (int)((t.len + KB - 1) / KB);
        if (steps == 0) return;
        if (steps > 1) wait_copies<COPIES>();
        else wait_copies<0>();
        barrier();
        read(fa, 0, 0);
        for (int s = 0; s < steps; ++s) {
            const int buf = s & 1;
            read(fb, buf, 1);
            multiply(fa);
            interleave();
            wait_copies<0>();
            wait_reads();
            barrier();
            if (s + 2 < steps) copy(t, (int64_t)(s + 2) * KB, buf);
            read(fa, buf ^ 1, 0);   // (after the last step: what was there, unused)
            multiply(fb);
            interleave();
        }
    };

    // A finished tile of the weight gradient, into the gradient or, of a part
    // of an expert, into its slot of partial sums.
    auto put_weight = [&](const Tile& t) {
        float* out = nullptr;
        if (group_of(a, t.e).count > a.split_rows) {
            // the expert's slots follow those of the split experts before it
            auto slots = [&](const Group& gg) {
                return gg.count > a.split_rows ? (int)((gg.count + a.split_rows - 1) / a.split_rows) : 0;
            };
            int before = 0;
            for (int e0 = 0; e0 < t.e; e0 += 64) {
                const int x = e0 + lane;
                before += __builtin_amdgcn_readlane(wave_inclusive_sum(x < t.e ? slots(group_of(a, x)) : 0), 63);
            }
            if (before + t.within < a.slots) out = a.partial + (int64_t)(before + t.within) * a.K * a.C;   // (offsets that decrease)
        } else {
            out = static_cast<float*>(a.out) + (int64_t)t.e * a.K * a.C;
        }
        const OutW rows(a, out ? out + (int64_t)t.q0 * a.C : nullptr, min(TQ, a.K - t.q0));
#pragma unroll
        for (int j = 0; j < FN; ++j)
#pragma unroll
            for (int h = 0; h < FM; h += WI)
                rows.put(lds_out[wave], wq * (TQ / NWQ) + j * 16, t.p0 + wp * (TP / NWP) + h * 16,
                         [&](int i) { return acc[h + i][j]; }, 0u);
    };

    // A workgroup stays for all its tiles: the next one's first copies are
    // under way while a finished one is stored.
    start(t);
    for (int turn = 1;; ++turn) {
        const Tile next = tile_of(turn);
        product(t);
        uint32_t live[FN];
        if (KIND == DATA) {
            const Out out(a, t.row0, t.qrows);
#pragma unroll
            for (int j = 0; j < FN; ++j) live[j] = out.load_live(wq * (TQ / NWQ) + j * 16, t.p0 + wp * (TP / NWP));
        }
        if (next.e >= 0) {
            wait_reads();
            barrier();   // every wave is done with both buffers
            start(next);
        }
        if (KIND == WEIGHT) {
            put_weight(t);
        } else {
            const Out out(a, t.row0, t.qrows);
#pragma unroll
            for (int j = 0; j < FN; ++j)
                out.put(lds_out[wave], wq * (TQ / NWQ) + j * 16, t.p0 + wp * (TP / NWP), [&](int i) { return acc[i][j]; },
                        KIND == DATA ? live[j] : 0u);
        }
        if (next.e < 0) return;
        t = next;
    }
}

// Few rows to an expert (serving, or many experts): bound by reading the
// filters.  A workgroup takes TP features by 16 FN rows and its waves share out
// the reduction, each streaming its own steps through a ring of its own in LDS
// without a barrier, so that a CU has all its waves' copies in flight; the
// waves' sums are added in order at the end.
template <typename T, int KIND, int TP, int FN, int NW, int RING>
__global__ __launch_bounds__(NW * 64) void expert_stream_kernel(ExpertArgs a)
{
    constexpr int TQ = 16 * FN, FM = TP / 16;
    using OP = Operand<T, TP, KIND != FWD, 1>;
    using OQ = Operand<T, TQ, false, 1>;
    constexpr int KB = OP::KB, COPIES = OP::COPIES + OQ::COPIES, STAGE = OP::BYTES + OQ::BYTES;
    constexpr int SUMS = NW * FM * FN * 1024, OUT = 16 * TP * (int)sizeof(T);
    __shared__ __align__(1024) char lds[NW * RING * STAGE > SUMS + FN * OUT ? NW * RING * STAGE : SUMS + FN * OUT];

    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int P = KIND == FWD ? a.K : a.C, ptiles = (P + TP - 1) / TP;
    auto all = number_units<false>(a, [&](const Group& g) { return (int)((g.count + TQ - 1) / TQ); });
    const int nunits = all.total, total = nunits * ptiles;
    const int64_t wg = (int64_t)blockIdx.y * gridDim.x + blockIdx.x;   // (launches of many have a second axis)
    if (wg >= total) return;
    // as in the tiled kernel: row tiles of one expert meet in one XCD
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
    const int p0 = pt * TP;
    const int64_t row0 = g.first + (int64_t)within * TQ;
    const int qrows = (int)min((int64_t)TQ, g.first + g.count - row0);
    if (within < 0 || qrows <= 0) return;   // (offsets that decrease)
    const int64_t qstride = KIND == FWD ? a.x_stride : a.y_stride;
    const int len = KIND == FWD ? a.C : a.K;
    const T* w = static_cast<const T*>(a.p) + (int64_t)e * a.K * a.C;
    const char* base_p = reinterpret_cast<const char*>(w + (KIND == FWD ? (int64_t)p0 * a.C : (int64_t)p0));
    const char* base_q = reinterpret_cast<const char*>(static_cast<const T*>(a.q) + row0 * qstride);
    const u32x4_t rq = make_rsrc_words(base_q, (uint32_t)(((qrows - 1) * qstride + len) * (int64_t)sizeof(T)));
    OP op;
    OQ oq;
    op.init(0, KIND == FWD ? 0 : a.C - p0, a.C);
    oq.init(0, 0, qstride);
    char* ring = lds + wave * RING * STAGE;
    const int frag_p = OP::first(0), frag_q = OQ::first(0);

    auto copy = [&](int step, int slot) {
        const int64_t k = (int64_t)step * KB;
        if (KIND == FWD) {
            const uint32_t n = (uint32_t)min(TP, a.K - p0) * (uint32_t)a.C * sizeof(T);
            op.copy(0, make_rsrc_words(base_p, n), (int)k, len, ring + slot * STAGE);
        } else {
            const int64_t left = min(len - k, (int64_t)KB);
            const uint32_t n = (uint32_t)(((left - 1) * a.C + a.C - p0) * (int64_t)sizeof(T));
            op.copy(0, make_rsrc_words(base_p + k * a.C * (int64_t)sizeof(T), n), 0, 0, ring + slot * STAGE);
        }
        oq.copy(0, rq, (int)k, len, ring + slot * STAGE + OP::BYTES);
    };

    floatx4 acc[FM][FN];
#pragma unroll
    for (int i = 0; i < FM; ++i)
#pragma unroll
        for (int j = 0; j < FN; ++j) acc[i][j] = floatx4{0.f, 0.f, 0.f, 0.f};

    // this wave's steps: wave, wave + NW, ...
    const int steps = ((len + KB - 1) / KB - wave + NW - 1) / NW;
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
    using Out = Output<T, KIND, FM>;
    const Out out(a, row0, qrows);
    static_assert(Out::BYTES <= OUT, "room for a wave's rows");
    for (int j = wave; j < FN; j += NW) {
        floatx4 v[FM] = {};
#pragma unroll
        for (int z = 0; z < NW; ++z)
#pragma unroll
            for (int i = 0; i < FM; ++i) v[i] += sums[(z * FM * FN + i * FN + j) * 64 + lane];
        out.put(lds + SUMS + j * OUT, j * 16, p0, [&](int i) { return v[i]; }, out.load_live(j * 16, p0));
    }
}

// Sums of the split experts' parts, in order.  Pieces of 256 vectors of all
// split experts are dealt out to the workgroups.
__global__ __launch_bounds__(256) void expert_sum_kernel(ExpertArgs a)
{
    const int64_t vecs = (int64_t)a.K * a.C / 4, pieces = (vecs + 255) / 256;
    int64_t slot0 = 0, piece = blockIdx.x;   // slots of the experts before; the next piece, from this group of experts on
    for (int e0 = 0; e0 < a.E; e0 += 64) {
        const int x = e0 + (threadIdx.x & 63);
        const int n = x < a.E ? (int)((group_of(a, x).count + a.split_rows - 1) / a.split_rows) : 0;
        const int parts = n > 1 ? n : 0, last = wave_inclusive_sum(parts);
        const uint64_t split = __ballot(parts > 0);
        const int before = __popcll(split & ((1ull << (threadIdx.x & 63)) - 1));   // split experts before the lane's
        const int64_t mine = __popcll(split) * pieces;
        for (; piece < mine; piece += gridDim.x) {
            const int64_t rank = piece / pieces;
            const int at = __builtin_ctzll(__ballot(parts > 0 && before == (int)rank));
            const int np = __builtin_amdgcn_readlane(parts, at);
            const int64_t slot = slot0 + __builtin_amdgcn_readlane(last, at) - np;
            const int64_t i = (piece - rank * pieces) * 256 + threadIdx.x;
            if (slot + np > a.slots) return;   // (offsets that decrease)
            if (i >= vecs) continue;
            const floatx4* src = reinterpret_cast<const floatx4*>(a.partial) + slot * vecs;
            // eight loads in flight, added in order
            floatx4 s = {};
            for (int z = 0; z < np; z += 8) {
                floatx4 v[8];
#pragma unroll
                for (int k = 0; k < 8; ++k) v[k] = src[(int64_t)min(z + k, np - 1) * vecs + i];
#pragma unroll
                for (int k = 0; k < 8; ++k)
                    if (z + k < np) s += v[k];
            }
            reinterpret_cast<floatx4*>(static_cast<float*>(a.out))[(e0 + at) * vecs + i] = s;
        }
        piece -= mine;
        slot0 += __builtin_amdgcn_readlane(last, 63);
    }
}

// The most row tiles that any lengths can give.
int64_t most_units(int64_t rows, int E, int tile) { return rows / tile + std::min<int64_t>(E, rows); }

template <typename T, int KIND, int TP, int TQ, int NWP, int NWQ>
hipError_t launch_tiles(const ExpertArgs& a, hipStream_t s)
{
    const int P = KIND == FWD ? a.K : a.C;
    const int64_t per = (int64_t)((P + TP - 1) / TP) * (KIND == WEIGHT ? (a.K + TQ - 1) / TQ : 1);
    const int64_t grid = (KIND == WEIGHT ? a.rows / a.split_rows + a.E : most_units(a.rows, a.E, TQ)) * per;
    if (grid == 0) return hipSuccess;
    if (grid > 0x7fffffff) return hipErrorInvalidValue;
    // as many workgroups as are resident (by their LDS), which stay for several tiles
    const int64_t lds = (TP + TQ) * 256 + (KIND == WEIGHT ? NWP * NWQ * std::min(64, TP / NWP) * 64 : NWQ * TP * 16 * (int)sizeof(T));
    const int64_t resident = (int64_t)CBW_NUM_CUS * (163840 / lds);
    expert_kernel<T, KIND, TP, TQ, NWP, NWQ><<<(int)std::min(grid, resident), NWP * NWQ * 64, 0, s>>>(a);
    return hipGetLastError();
}

template <typename T, int KIND, int TP, int FN, int NW, int RING>
hipError_t launch_stream(const ExpertArgs& a, hipStream_t s)
{
    const int P = KIND == FWD ? a.K : a.C;
    const int64_t grid = most_units(a.rows, a.E, 16 * FN) * ((P + TP - 1) / TP);
    if (grid == 0) return hipSuccess;
    if (grid > 0x7fffffff) return hipErrorInvalidValue;
    // An axis of a launch takes 2^32 - 1 threads; more wrap without an error.
    const int64_t x = std::min<int64_t>(grid, 1 << 22);
    static_assert(NW * 64 <= 1 << 9, "threads along the first axis");
    expert_stream_kernel<T, KIND, TP, FN, NW, RING><<<dim3((unsigned)x, (unsigned)((grid + x - 1) / x)), NW * 64, 0, s>>>(a);
    return hipGetLastError();
}

// Tiles of `tile` rows by `width` features, the rows spread evenly over the
// experts (the host does not know the lengths).
int64_t likely_tiles(const ExpertArgs& a, int tile, int P, int width)
{
    const int64_t busy = std::max<int64_t>(1, std::min<int64_t>(a.E, a.rows)), mean = (a.rows + busy - 1) / busy;
    return busy * ((mean + tile - 1) / tile) * ((P + width - 1) / width);
}

// Forward product and data gradient.  Large tiles need the fewest bytes from
// the caches but rows enough to fill them and tiles enough to fill the chip;
// where there are neither, the streaming kernel splits the reduction over its
// waves.  Measured (us, bf16, forward; 256 x 256 | 128 x 128 | stream, 16 rows |
// stream, 64 rows): 16384 rows, 8 experts, 2048 -> 8192: 511 | 653 | - | -;
// 6935 rows, 36 experts, 1736 -> 1312: 52 | 69 | 141 | 105; 3676, 3, 264 ->
// 1576: 14 | 12 | 37 | 26; 256, 8, 2048 -> 8192: 52 | 45 | 52 | 54; 755, 1, 2664
// -> 536: 57 | 38 | 14 | 13 (15.4 in a later run); 2108, 46, 848 -> 152: 22 | 14 | 7 | 7; 12, 32, 2048
// -> 1408: 43 | 26 | 12 | 13.  Few tiles of 64 features: 16 rows, 1 expert, 8192
// -> 512: 18, and 10 with 32 features and eight waves.  (The small ones' filters
// lay in the caches.  From memory, 64 features and four waves | 32 and eight:
// 12 rows, 32 experts, 2048 -> 1408: 15.7 | 16.9; 300, 64, 1024 -> 512: 15 | 22;
// 1, 1, 2048 -> 8192: 10.3 | 9.5.)
//
// float32, forward, from memory (us, 64 x 64 tiles | stream, 16 rows; in
// brackets the tiles of 64 x 64, of which the rule asks for 400): 640 rows, 16
// experts, 2048 -> 256 (64): 50 | 18; 1000, 32, 512 -> 512 (256): 16.7 | 17.2;
// 1024, 8, 1024 -> 1024 (256): 40 | 38; 300, 4, 4096 -> 4096 (512): 146 | 137;
// 1800, 8, 1024 -> 1024 (512): 41 | 56; 4096, 1, 512 -> 512 (512): 23 | 36;
// 2000, 64, 256 -> 1024 (1024): 25 | 31.  One wide group of few tiles goes the
// slower way: 2000, 1, 512 -> 512 (256): 14.8 | 18.3.
template <typename T, int KIND>
hipError_t launch_rows(const ExpertArgs& a, hipStream_t s)
{
    constexpr bool BF16 = sizeof(T) == 2;
    const int P = KIND == FWD ? a.K : a.C;
    const int64_t mean = a.rows / std::max<int64_t>(1, std::min<int64_t>(a.E, a.rows));
    if constexpr (BF16) {
        if (mean >= 160 && likely_tiles(a, 256, P, 256) >= 200) return launch_tiles<T, KIND, 256, 256, 2, 4>(a, s);
        if (mean > 16 && likely_tiles(a, 128, P, 128) >= 200) return launch_tiles<T, KIND, 128, 128, 2, 2>(a, s);
        if (mean > 64) return launch_stream<T, KIND, 64, 4, 4, 2>(a, s);   // (float32: the matrix unit would be the bound)
    } else {
        if (mean > 16 && likely_tiles(a, 64, P, 64) >= 400) return launch_tiles<T, KIND, 64, 64, 2, 2>(a, s);
    }
    if (likely_tiles(a, 16, P, 64) >= 192) return launch_stream<T, KIND, 64, 1, 4, 2>(a, s);
    return launch_stream<T, KIND, 32, 1, 8, 3>(a, s);
}

}  // namespace

// Weight gradient: tiles and parts.
//
// bf16, large tiles where an expert's rows make the product outweigh a tile's
// start and end and there is one for every CU (us, 256 x 256 | 128 x 128: 512
// rows for each of 64 experts, 2048 -> 1408: 242 | 308; 4 of 1024, 2048 ->
// 2048: 42 | 51; 25 of 92, 2048 -> 4096: 181 | 158; 8 of 2048, 1024 -> 1024: 51
// | 44).
//
// Splitting an expert's rows sends every part's sums through memory and back,
// the products' own time for parts of about 1000 rows (bf16).  So they are
// split where the experts' tiles leave half the chip idle or more, into three
// parts or more that fill it (16384 rows, 1 expert, 1024 -> 1024: 190 us whole,
// 52 by 2048 rows, 63 by 1024; 1531 rows, 792 -> 3432: 26 whole, 35 by 512);
// and otherwise only an expert that is three times the mean
// and would alone take half the call's time (64 uneven experts, 32768 rows,
// 2048 -> 1408, the longest 5591: 377 us whole, 332 in the parts of half a
// workgroup's share that follow; 8 even ones of 2048 rows, 1024 -> 1024: 44
// whole, 73 by 1024).  (The small ones' rows lay in the caches: the 17 and 26
// us calls take 20 and 30 from memory.)  The launch that adds parts up is
// made wherever the capacity exceeds a part's rows, also where no expert turns
// out to have as many.
ExpertPlan expert_plan(const cbw_expert_desc* d)
{
    ExpertPlan p{};
    const bool f32 = d->dtype == CBW_F32;
    const int64_t busy = std::max<int64_t>(1, std::min<int64_t>(d->E, d->rows)), mean = (d->rows + busy - 1) / busy;
    auto tiles = [&](int side) { return (int64_t)((d->C + side - 1) / side) * ((d->K + side - 1) / side); };
    p.large = !f32 && mean >= 256 && tiles(256) * busy >= CBW_NUM_CUS;
    const int64_t per = tiles(f32 ? 64 : p.large ? 256 : 128), resident = CBW_NUM_CUS * (f32 ? 4 : p.large ? 1 : 2);
    const int64_t share = d->rows * per / resident;   // rows of one tile that a workgroup takes on average
    // (1024 rows of one tile take some 10 us: no more than the launch that adds parts up costs)
    int64_t len = std::max<int64_t>(1024, std::max(3 * mean, share / 2));
    // (small filters' sums are soon moved: 26 experts of 1683 rows, 56 -> 248, 26 us whole, 17 by 512 rows, 22 by 1024)
    const int64_t filling = std::max<int64_t>((int64_t)d->K * d->C <= 1 << 18 ? 512 : 1024, share);
    if (2 * per * busy <= resident && mean >= 3 * filling) len = filling;
    p.split_rows = (int)std::min<int64_t>((len + 63) / 64 * 64, 1 << 30);
    p.slots = d->rows > p.split_rows ? 2 * d->rows / p.split_rows : 0;
    p.ws_bytes = (size_t)p.slots * d->K * d->C * 4;
    return p;
}

hipError_t launch_expert_fwd(int dtype, const ExpertArgs& a, hipStream_t s)
{
    return dtype == CBW_F32 ? launch_rows<float, FWD>(a, s) : launch_rows<uint16_t, FWD>(a, s);
}

hipError_t launch_expert_bwd_data(int dtype, const ExpertArgs& a, hipStream_t s)
{
    return dtype == CBW_F32 ? launch_rows<float, DATA>(a, s) : launch_rows<uint16_t, DATA>(a, s);
}

hipError_t launch_expert_bwd_weight(int dtype, const ExpertArgs& a, bool large, hipStream_t s)
{
    hipError_t e;
    if (dtype == CBW_F32) e = launch_tiles<float, WEIGHT, 64, 64, 2, 2>(a, s);
    else if (large) e = launch_tiles<uint16_t, WEIGHT, 256, 256, 2, 4>(a, s);
    else e = launch_tiles<uint16_t, WEIGHT, 128, 128, 2, 2>(a, s);
    if (e != hipSuccess || a.rows <= a.split_rows) return e;
    expert_sum_kernel<<<1024, 256, 0, s>>>(a);
    return hipGetLastError();
}

}  // namespace cbw
