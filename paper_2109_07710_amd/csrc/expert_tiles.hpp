// What the kernels of products grouped by expert share: the groups and how a
// workgroup finds its own, waits and fences, and an operand's tile in LDS.
#pragma once

#include "common.hpp"
#include "block_kernels.hpp"

namespace cbw {

// Rows of group e, whatever the offsets hold: inside [0, rows], at least 0.
struct Group {
    int64_t first, count;
};
template <typename A>
__device__ __forceinline__ Group group_of(const A& a, int e)
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
template <bool SORTED, typename A, typename F>
struct Units {
    const A& a;
    F units;
    int e, n, incl, total;   // the lane's expert and its units; of all

    __device__ Units(const A& args, F f) : a(args), units(f)
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
template <bool SORTED, typename A, typename F>
__device__ __forceinline__ Units<SORTED, A, F> number_units(const A& a, F f) { return Units<SORTED, A, F>(a, f); }

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
// reduction indices, filled by NW waves.  PAIRS (along): the columns are 16 of
// one filter and 16 of another in turn, both from the same feature on, so that
// a lane has a feature's two sums.
template <typename T, int N, bool ACROSS, int NW, bool PAIRS = false>
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

    // Copies DIST apart lie a multiple of 16 LDS rows (pairs: of 32) apart, which
    // the swizzle does not see: the same lane has the same chunk, so its byte offset grows
    // by a uniform amount.
    static constexpr int LINES_PER_COPY = NW * 64 / CHUNKS;
    static constexpr int TURN = PAIRS ? 32 : 16;
    static constexpr int DIST = LINES_PER_COPY % TURN == 0 ? 1 : TURN / LINES_PER_COPY;
    static_assert(!PAIRS || !ACROSS, "pairs go along");
    static_assert(COPIES < DIST || COPIES % DIST == 0, "every distinct copy as often");
    static constexpr int OWN = COPIES < DIST ? COPIES : DIST;

    uint32_t off[OWN];   // byte offset of the lane's 16 bytes at step 0, kOOB: never valid
    uint32_t apart;      // (uniform) bytes from a copy to the one DIST further

    // along: rows of `stride` elements, pairs: the other filter's `second`
    // elements further; across: `n` valid columns
    __device__ __forceinline__ void init(int wave, int64_t n, int64_t stride, int64_t second = 0)
    {
        const int lane = threadIdx.x & 63;
#pragma unroll
        for (int j = 0; j < OWN; ++j) {
            const int at = (wave + NW * j) * 64 + lane;
            const int line = at / CHUNKS, lc = (at % CHUNKS) ^ swizzle(line);
            const int64_t row = PAIRS ? (int64_t)((line >> 5) * 16 + (line & 15)) * stride + (line & 16 ? second : 0) : line * stride;
            off[j] = ACROSS && lc * E >= n ? kOOB : (uint32_t)(row + lc * E) * ESZ;
        }
        apart = (uint32_t)(DIST * LINES_PER_COPY / (PAIRS ? 2 : 1) * stride) * ESZ;
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
        static_assert(!ACROSS || (F & (F - 1)) == 0, "a power of two");
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

}  // namespace cbw
