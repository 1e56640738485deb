// Launch interfaces of the expert-block operators (grouped products, block
// norms, gradient clipping) between the C entry points and the kernels.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/convbwd.h"
#include "common.hpp"

namespace cbw {

// ------------------------------------------------------------ block norms

// One row is held by a team of threads, vectors of 8 columns each: up to 64
// lanes of a wave where the row fits one vector a lane (several rows to a
// workgroup then), else a whole workgroup of up to 16 waves, whose threads
// take two vectors past 8192 columns.
constexpr int kNormMaxC = 16384;

struct NormShape {
    int team;       // threads per row: a power of two up to 64, or a multiple of 64
    int vpt;        // vectors of 8 columns per thread, 1 or 2
    int threads;    // per workgroup
    int slots;      // rows a workgroup holds at a time
};

inline NormShape norm_shape(int C)
{
    NormShape s;
    const int vecs = (C + 7) / 8;
    if (vecs <= 64) {
        s.team = 8;
        while (s.team < vecs) s.team *= 2;
        s.vpt = 1;
        s.threads = 256;
        s.slots = s.threads / s.team;
    } else {
        s.vpt = vecs > 1024 ? 2 : 1;
        s.team = (vecs + 64 * s.vpt - 1) / (64 * s.vpt) * 64;
        s.threads = s.team;
        s.slots = 1;
    }
    return s;
}

// The backward pass's split of the rows: `items` ranges of rows, none across
// two gate rows where the gate is shared, dealt out to `grid` workgroups.
struct NormSplit {
    int grid;
    int64_t items, item_rows;   // an item's rows; the last of a group may be short
    int64_t groups, parts;      // groups of rows that share a gate row, items per group
    int64_t group_rows;
};
NormSplit norm_split(const cbw_norm_desc* d);

// Order of the parameters' gradients in the partial sums.
enum { NG_W_PRE = 0, NG_B_PRE, NG_W_POST, NG_B_POST, NG_SCALE, NG_COUNT };

struct NormArgs {
    const void *x, *u, *gate;
    const float *w_pre, *b_pre, *w_post, *b_post, *scale;
    void *y, *h;
    float* stats;
    int64_t rows, res_stride, block_stride, gate_stride, gate_rows;
    int C, pre, post, act;
    float eps;
    FastDiv gate_div;           // by gate_rows
};

struct NormBackArgs {
    const void *y, *u, *gate, *dy, *dh;
    const float *w_pre, *w_post, *b_post, *scale;
    const float* stats;
    void *dx, *du, *dgate;
    float* grads[NG_COUNT];     // where each gradient goes, null: not asked for
    float* partial;             // [grid][NG_COUNT][C], those asked for first; null where one workgroup writes them itself
    float* gate_partial;        // [items][C] where a gate row's rows are split, else null
    int64_t rows, res_stride, block_stride, gate_stride, gate_rows;
    int C, pre, post, act;
    NormSplit split;
};

hipError_t launch_norm_fwd(int dtype, int res_dtype, const NormArgs& a, hipStream_t s);
hipError_t launch_norm_bwd(int dtype, int res_dtype, const NormBackArgs& a, hipStream_t s);

// ------------------------------------------------------- grouped products

struct ExpertArgs {
    const void *p, *q;          // the operand whose columns are the output's features, the other one
    const int32_t* offsets;
    void* out;
    const uint32_t* mask;       // footprint read (data gradient)
    uint32_t* out_mask;         // footprint written (forward)
    float* partial;             // weight gradient: sums of split experts, [slots][K][C]
    int64_t rows, x_stride, y_stride;
    int E, C, K;
    int relu;
    int split_rows;             // weight gradient: rows per part
    int64_t slots;              // and slots of partial sums
};

// Weight gradient: an expert's rows are taken in parts of split_rows, each by
// workgroups of its own.  An expert with more than one part has a slot of
// partial sums for each: fewer than 2 rows / split_rows slots in all.
struct ExpertPlan {
    bool large;                 // tiles of 256 x 256
    int split_rows;
    int64_t slots;
    size_t ws_bytes;
};
ExpertPlan expert_plan(const cbw_expert_desc* d);

hipError_t launch_expert_fwd(int dtype, const ExpertArgs& a, hipStream_t s);
hipError_t launch_expert_bwd_data(int dtype, const ExpertArgs& a, hipStream_t s);
hipError_t launch_expert_bwd_weight(int dtype, const ExpertArgs& a, bool large, hipStream_t s);

// ------------------------------------------------------- gradient clipping

constexpr int kGradTable = 120;       // tensors per launch: the table travels in the kernel's arguments
constexpr int kGradChunk = 16384;     // bytes a workgroup takes at a time
// Workgroups of a pass, shared out over its launches, of which each has at
// least kGradMinWgs if it has the chunks.  (us a clipping call with 512 | 1024 |
// 2048 in all: 13 tensors, 59 MB: 38 | 37 | 37; 3 of 160 MB together: 104 |
// 101 | 103; 48 of 2.1 GB: 1245 | 1280 | 1308; 400 of 80 MB: 66 | 66 | 63.  With
// 128 | 256 | 512 at least: 300 packed tensors, 90 MB: 68.2 | 67.2 | 66.6; 400
// of 80 MB: 67 | 66 | 64.)
constexpr int kGradMaxWgs = 1024;
constexpr int kGradMinWgs = 256;

struct alignas(16) GradEntry {   // (copied by 16-byte vectors)
    const void* src;
    void* dst;
    int64_t bytes;              // bit 63: bf16
    int32_t first, pad;         // first chunk of the tensor
};
struct GradTable {
    GradEntry e[kGradTable];
    int32_t n, chunks;          // tensors and chunks of this launch
    int32_t entry0, chunk0;     // of the launches before it
};
static_assert(sizeof(GradTable) <= 3872, "the table fits the kernel arguments");

hipError_t launch_grad_norm(const GradTable& t, int kind, int grid, double* partial, GradEntry* table, hipStream_t s);
hipError_t launch_grad_finish(int kind, const double* partial, int npartial, float* norm, hipStream_t s);
hipError_t launch_grad_scale(const GradEntry* table, int n, int chunks, int kind, int grid, const double* partial,
                             int npartial, float max_norm, float* norm, hipStream_t s);

}  // namespace cbw
