// C-ABI entry points of the expert-block operators: validation, workspace
// carving and kernel launches on the caller's stream.  See
// include/convbwd.h for the contract.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "../../include/convbwd.h"
#include "block_kernels.hpp"

using namespace cbw;

namespace {

bool aligned(const void* p, uintptr_t n) { return ((uintptr_t)p & (n - 1)) == 0; }

int hip_status(hipError_t e)
{
    if (e == hipSuccess) return CBW_OK;
    (void)hipGetLastError();
    return CBW_ERR_HIP;
}

bool known_dtype(int t) { return t == CBW_F32 || t == CBW_BF16; }

int check_ws(const void* ws, size_t ws_bytes, size_t need)
{
    if (need > 0 && ws == nullptr) return CBW_ERR_WORKSPACE;
    if (ws_bytes < need) return CBW_ERR_WORKSPACE;
    if (!aligned(ws, 16)) return CBW_ERR_UNSUPPORTED;
    return CBW_OK;
}

size_t round256(size_t n) { return (n + 255) & ~(size_t)255; }

// ------------------------------------------------------------------ experts

int expert_check(const cbw_expert_desc* d, const void* a, const void* b, const int32_t* offsets, const void* out,
                 const void* ws, size_t ws_bytes, bool needs_ws, ExpertPlan* plan)
{
    int st = cbw_validate_expert_desc(d);
    if (st != CBW_OK) return st;
    if (!offsets) return CBW_ERR_INVALID_ARG;
    if (!aligned(offsets, 4)) return CBW_ERR_UNSUPPORTED;
    // (tensors without rows may have no address)
    if (d->rows > 0 && (!a || !b || !out)) return CBW_ERR_INVALID_ARG;
    if (!aligned(a, 16) || !aligned(b, 16) || !aligned(out, 16)) return CBW_ERR_UNSUPPORTED;
    *plan = expert_plan(d);
    return needs_ws ? check_ws(ws, ws_bytes, plan->ws_bytes) : CBW_OK;
}

ExpertArgs expert_args(const cbw_expert_desc* d, const void* p, const void* q, const int32_t* offsets, void* out)
{
    ExpertArgs a{};
    a.p = p;
    a.q = q;
    a.offsets = offsets;
    a.out = out;
    a.rows = d->rows;
    a.x_stride = d->x_stride;
    a.y_stride = d->y_stride;
    a.E = d->E;
    a.C = d->C;
    a.K = d->K;
    return a;
}

// -------------------------------------------------------------------- norms

// Pointers of a parameter set against the descriptor: INVALID_ARG for one of
// a norm that is left out (or of the block where there is none).
int check_params(const cbw_norm_desc* d, const cbw_norm_params* p, bool block)
{
    if (d->pre_norm == CBW_NORM_NONE && (p->w_pre || p->b_pre)) return CBW_ERR_INVALID_ARG;
    if ((d->post_norm == CBW_NORM_NONE || !block) && (p->w_post || p->b_post)) return CBW_ERR_INVALID_ARG;
    if (!block && p->scale) return CBW_ERR_INVALID_ARG;
    if (!aligned(p->w_pre, 16) || !aligned(p->b_pre, 16) || !aligned(p->w_post, 16) || !aligned(p->b_post, 16) ||
        !aligned(p->scale, 16))
        return CBW_ERR_UNSUPPORTED;
    return CBW_OK;
}

// The backward pass's workspace: partial sums of the parameters' gradients,
// then those of a shared gate whose rows are split.
struct NormRegions {
    size_t partial, gate_partial, total;
};
NormRegions norm_regions(const cbw_norm_desc* d, const NormSplit& s)
{
    NormRegions r{};
    r.partial = s.grid > 1 ? round256((size_t)s.grid * NG_COUNT * d->C * 4) : 0;
    r.gate_partial = s.parts > 1 && d->gate_act != CBW_GATE_NONE && d->gate_rows > 1 ? round256((size_t)s.items * d->C * 4) : 0;
    r.total = r.partial + r.gate_partial;
    return r;
}

// ---------------------------------------------------------------- gradients

int64_t grad_bytes(const cbw_grad& g) { return g.count * (g.dtype == CBW_F32 ? 4 : 2); }
int64_t grad_chunks(const cbw_grad& g) { return (grad_bytes(g) + kGradChunk - 1) / kGradChunk; }

// What a call has to do: tensors with elements, and their chunks.
struct GradWork {
    int64_t tensors, chunks;
    // the workspace: partial sums, then the table of all tensors
    size_t partial_bytes() const
    {
        return ((size_t)(kGradMaxWgs + (tensors + kGradTable - 1) / kGradTable * kGradMinWgs) * sizeof(double) + 255) & ~(size_t)255;
    }
    size_t ws_bytes() const { return partial_bytes() + (((size_t)tensors * sizeof(GradEntry) + 255) & ~(size_t)255); }
};

// Checks the list and sums up its work.
int check_grads(const cbw_grad* grads, int32_t n, bool with_out, GradWork* work)
{
    if (n < 0 || (n > 0 && !grads)) return CBW_ERR_INVALID_ARG;
    *work = {};
    for (int32_t i = 0; i < n; ++i) {
        const cbw_grad& g = grads[i];
        if (g.count < 0 || !known_dtype(g.dtype) || g.reserved != 0) return CBW_ERR_INVALID_ARG;
        if (g.count == 0) continue;
        if (!g.grad || (with_out && !g.out)) return CBW_ERR_INVALID_ARG;
        const uintptr_t size = g.dtype == CBW_F32 ? 4 : 2;
        if (!aligned(g.grad, size) || (with_out && !aligned(g.out, size))) return CBW_ERR_UNSUPPORTED;
        if (g.count > ((int64_t)1 << 40)) return CBW_ERR_UNSUPPORTED;
        work->chunks += grad_chunks(g);
        ++work->tensors;
        if (work->chunks > 0x3fffffff) return CBW_ERR_UNSUPPORTED;
    }
    return CBW_OK;
}

// The next table of at most kGradTable tensors from entry `i` on; i moves on.
bool next_table(const cbw_grad* grads, int32_t n, int32_t& i, GradTable& t)
{
    t.n = t.chunks = 0;
    for (; i < n && t.n < kGradTable; ++i) {
        const cbw_grad& g = grads[i];
        if (g.count == 0) continue;
        t.e[t.n] = {g.grad, g.out, grad_bytes(g) | (g.dtype == CBW_BF16 ? INT64_MIN : 0), t.chunks, 0};
        t.chunks += (int32_t)grad_chunks(g);
        ++t.n;
    }
    return t.n > 0;
}

// Workgroups of a launch: its share of kGradMaxWgs by chunks.
int grad_grid(int64_t chunks, int64_t all)
{
    return (int)std::min(chunks, std::max<int64_t>(kGradMinWgs, kGradMaxWgs * chunks / std::max<int64_t>(all, 1)));
}

// Partials of all tensors into the workspace, with `table` the tensors as well; the number of partials.
int norm_pass(const cbw_grad* grads, int32_t n, int32_t kind, const GradWork& work, double* partial, GradEntry* table,
              hipStream_t s, int* count)
{
    GradTable t;
    t.entry0 = t.chunk0 = 0;
    *count = 0;
    for (int32_t i = 0; next_table(grads, n, i, t);) {
        const int grid = grad_grid(t.chunks, work.chunks);
        const hipError_t e = launch_grad_norm(t, kind, grid, partial + *count, table, s);
        if (e != hipSuccess) return hip_status(e);
        *count += grid;
        t.entry0 += t.n;
        t.chunk0 += t.chunks;
    }
    return CBW_OK;
}

int check_norm_call(const cbw_grad* grads, int32_t n, int32_t kind, bool with_out, const float* norm, const void* ws,
                    size_t ws_bytes, GradWork* work)
{
    int st = check_grads(grads, n, with_out, work);
    if (st != CBW_OK) return st;
    if (kind != CBW_GRAD_NORM_2 && kind != CBW_GRAD_NORM_INF) return CBW_ERR_INVALID_ARG;
    if (!norm) return CBW_ERR_INVALID_ARG;
    if (!aligned(norm, 4)) return CBW_ERR_UNSUPPORTED;
    return check_ws(ws, ws_bytes, work->ws_bytes());
}

}  // namespace

extern "C" {

int cbw_validate_expert_desc(const cbw_expert_desc* d)
{
    if (!d) return CBW_ERR_INVALID_ARG;
    if (d->E <= 0 || d->C <= 0 || d->K <= 0 || d->rows < 0 || !known_dtype(d->dtype)) return CBW_ERR_INVALID_ARG;
    if (d->x_stride < d->C || d->y_stride < d->K) return CBW_ERR_INVALID_ARG;
    const int vec = d->dtype == CBW_F32 ? 4 : 8;
    if (d->C % vec || d->K % vec || d->x_stride % vec || d->y_stride % vec) return CBW_ERR_UNSUPPORTED;
    if (d->E > CBW_MAX_EXPERTS || d->rows > 0x7fffffff) return CBW_ERR_UNSUPPORTED;
    if (d->x_stride >= 1 << 20 || d->y_stride >= 1 << 20) return CBW_ERR_UNSUPPORTED;
    if ((int64_t)d->C * d->K * 4 >= (int64_t)1 << 31) return CBW_ERR_UNSUPPORTED;
    return CBW_OK;
}

int cbw_expert_workspace_size(const cbw_expert_desc* desc, size_t* bytes)
{
    if (!bytes) return CBW_ERR_INVALID_ARG;
    const int st = cbw_validate_expert_desc(desc);
    if (st != CBW_OK) return st;
    *bytes = expert_plan(desc).ws_bytes;
    return CBW_OK;
}

int expert_fwd(const cbw_expert_desc* desc, const void* X, const void* W, const int32_t* offsets, void* Y,
               uint32_t* y_mask, void* workspace, size_t workspace_bytes, uint32_t flags, void* stream)
{
    ExpertPlan plan;
    int st = expert_check(desc, X, W, offsets, Y, workspace, workspace_bytes, false, &plan);
    if (st != CBW_OK) return st;
    if (flags & ~CBW_FLAG_RELU) return CBW_ERR_INVALID_ARG;
    if (y_mask && (!(flags & CBW_FLAG_RELU) || desc->K % 32 != 0 || !aligned(y_mask, 4))) return CBW_ERR_UNSUPPORTED;
    if (desc->rows == 0) return CBW_OK;
    ExpertArgs a = expert_args(desc, W, X, offsets, Y);
    a.relu = flags & CBW_FLAG_RELU ? 1 : 0;
    a.out_mask = y_mask;
    return hip_status(launch_expert_fwd(desc->dtype, a, static_cast<hipStream_t>(stream)));
}

int expert_bwd_data(const cbw_expert_desc* desc, const void* dY, const void* W, const int32_t* offsets,
                    const uint32_t* x_mask, void* dX, void* workspace, size_t workspace_bytes, void* stream)
{
    ExpertPlan plan;
    int st = expert_check(desc, dY, W, offsets, dX, workspace, workspace_bytes, false, &plan);
    if (st != CBW_OK) return st;
    if (!aligned(x_mask, 4)) return CBW_ERR_UNSUPPORTED;
    if (desc->rows == 0) return CBW_OK;
    ExpertArgs a = expert_args(desc, W, dY, offsets, dX);
    a.mask = x_mask;
    return hip_status(launch_expert_bwd_data(desc->dtype, a, static_cast<hipStream_t>(stream)));
}

int expert_bwd_weight(const cbw_expert_desc* desc, const void* X, const void* dY, const int32_t* offsets, float* dW,
                      void* workspace, size_t workspace_bytes, void* stream)
{
    if (!dW && cbw_validate_expert_desc(desc) == CBW_OK) return CBW_ERR_INVALID_ARG;   // written without rows as well
    ExpertPlan plan;
    int st = expert_check(desc, X, dY, offsets, dW, workspace, workspace_bytes, true, &plan);
    if (st != CBW_OK) return st;
    ExpertArgs a = expert_args(desc, X, dY, offsets, dW);
    a.partial = static_cast<float*>(workspace);
    a.split_rows = plan.split_rows;
    a.slots = plan.slots;
    return hip_status(launch_expert_bwd_weight(desc->dtype, a, plan.large, static_cast<hipStream_t>(stream)));
}

int cbw_validate_norm_desc(const cbw_norm_desc* d)
{
    if (!d) return CBW_ERR_INVALID_ARG;
    if (d->rows < 0 || d->C <= 0 || d->gate_rows < 1 || !known_dtype(d->dtype) || !known_dtype(d->res_dtype))
        return CBW_ERR_INVALID_ARG;
    for (int k : {d->pre_norm, d->post_norm})
        if (k < CBW_NORM_NONE || k > CBW_NORM_LAYER) return CBW_ERR_INVALID_ARG;
    if (d->gate_act < CBW_GATE_NONE || d->gate_act > CBW_GATE_SIGMOID) return CBW_ERR_INVALID_ARG;
    if (!(d->eps >= 0.f) || std::isinf(d->eps)) return CBW_ERR_INVALID_ARG;
    if (d->res_stride < d->C || d->block_stride < d->C || d->gate_stride < d->C) return CBW_ERR_INVALID_ARG;
    if (d->C > kNormMaxC || d->C % 8 || d->res_stride % 8 || d->block_stride % 8 || d->gate_stride % 8)
        return CBW_ERR_UNSUPPORTED;
    if (d->dtype == CBW_F32 && d->res_dtype != CBW_F32) return CBW_ERR_UNSUPPORTED;
    if (d->rows > 0x7fffffff || d->res_stride > (int64_t)1 << 20 || d->block_stride > (int64_t)1 << 20 ||
        d->gate_stride > (int64_t)1 << 20)
        return CBW_ERR_UNSUPPORTED;
    return CBW_OK;
}

int cbw_norm_workspace_size(const cbw_norm_desc* desc, size_t* bytes)
{
    if (!bytes) return CBW_ERR_INVALID_ARG;
    const int st = cbw_validate_norm_desc(desc);
    if (st != CBW_OK) return st;
    *bytes = norm_regions(desc, norm_split(desc)).total;
    return CBW_OK;
}

int block_norm_fwd(const cbw_norm_desc* desc, const void* x, const void* u, const void* gate,
                   const cbw_norm_params* params, void* y, void* h, float* stats, void* stream)
{
    int st = cbw_validate_norm_desc(desc);
    if (st != CBW_OK) return st;
    static const cbw_norm_params none = {};
    if (!params) params = &none;
    if (desc->rows == 0) return CBW_OK;   // (tensors without rows may have no address)
    if (!x || (u != nullptr) != (y != nullptr)) return CBW_ERR_INVALID_ARG;
    if ((desc->pre_norm != CBW_NORM_NONE) != (h != nullptr) || (!u && !h)) return CBW_ERR_INVALID_ARG;
    if ((gate != nullptr) != (u && desc->gate_act != CBW_GATE_NONE)) return CBW_ERR_INVALID_ARG;
    if ((st = check_params(desc, params, u != nullptr)) != CBW_OK) return st;
    if (!aligned(x, 16) || !aligned(u, 16) || !aligned(gate, 16) || !aligned(y, 16) || !aligned(h, 16) || !aligned(stats, 16))
        return CBW_ERR_UNSUPPORTED;
    NormArgs a{};
    a.x = x;
    a.u = u;
    a.gate = gate;
    a.w_pre = params->w_pre;
    a.b_pre = params->b_pre;
    a.w_post = params->w_post;
    a.b_post = params->b_post;
    a.scale = params->scale;
    a.y = y;
    a.h = h;
    a.stats = stats;
    a.rows = desc->rows;
    a.res_stride = desc->res_stride;
    a.block_stride = desc->block_stride;
    a.gate_stride = desc->gate_stride;
    a.gate_rows = desc->gate_rows;
    a.C = desc->C;
    a.pre = desc->pre_norm;
    a.post = desc->post_norm;
    a.act = desc->gate_act;
    a.eps = desc->eps;
    a.gate_div = make_fastdiv((uint32_t)std::min(desc->gate_rows, desc->rows));
    return hip_status(launch_norm_fwd(desc->dtype, desc->res_dtype, a, static_cast<hipStream_t>(stream)));
}

int block_norm_bwd(const cbw_norm_desc* desc, const void* y, const void* u, const void* gate,
                   const cbw_norm_params* params, const float* stats, const void* dy, const void* dh, void* dx,
                   void* du, void* dgate, const cbw_norm_params* grads, void* workspace, size_t workspace_bytes,
                   void* stream)
{
    int st = cbw_validate_norm_desc(desc);
    if (st != CBW_OK) return st;
    static const cbw_norm_params none = {};
    if (!params) params = &none;
    if (!grads) grads = &none;
    const bool any = desc->rows > 0;   // (tensors without rows may have no address)
    if (any) {
        if (!y || !stats || !dx) return CBW_ERR_INVALID_ARG;
        if ((desc->pre_norm != CBW_NORM_NONE) != (dh != nullptr) || (!dy && !dh)) return CBW_ERR_INVALID_ARG;
        if ((gate != nullptr) != (u && desc->gate_act != CBW_GATE_NONE)) return CBW_ERR_INVALID_ARG;
        if ((du && !u) || (dgate && !gate)) return CBW_ERR_INVALID_ARG;
    }
    if ((st = check_params(desc, params, u || !any)) != CBW_OK) return st;
    if ((st = check_params(desc, grads, u || !any)) != CBW_OK) return st;
    for (const void* p : {y, u, gate, dy, dh, (const void*)dx, (const void*)du, (const void*)dgate, (const void*)stats})
        if (!aligned(p, 16)) return CBW_ERR_UNSUPPORTED;
    NormBackArgs a{};
    a.split = norm_split(desc);
    const NormRegions r = norm_regions(desc, a.split);
    if ((st = check_ws(workspace, workspace_bytes, r.total)) != CBW_OK) return st;
    a.y = y;
    a.u = u;
    a.gate = gate;
    a.dy = dy;
    a.dh = dh;
    a.w_pre = params->w_pre;
    a.w_post = params->w_post;
    a.b_post = params->b_post;
    a.scale = params->scale;
    a.stats = stats;
    a.dx = dx;
    a.du = du;
    a.dgate = desc->rows > 0 ? dgate : nullptr;   // (without rows it has none either)
    a.grads[NG_W_PRE] = grads->w_pre;
    a.grads[NG_B_PRE] = grads->b_pre;
    a.grads[NG_W_POST] = grads->w_post;
    a.grads[NG_B_POST] = grads->b_post;
    a.grads[NG_SCALE] = grads->scale;
    a.partial = r.partial ? static_cast<float*>(workspace) : nullptr;
    a.gate_partial = r.gate_partial && a.dgate ? reinterpret_cast<float*>(static_cast<char*>(workspace) + r.partial) : nullptr;
    a.rows = desc->rows;
    a.res_stride = desc->res_stride;
    a.block_stride = desc->block_stride;
    a.gate_stride = desc->gate_stride;
    a.gate_rows = desc->gate_rows;
    a.C = desc->C;
    a.pre = desc->pre_norm;
    a.post = desc->post_norm;
    a.act = desc->gate_act;
    return hip_status(launch_norm_bwd(desc->dtype, desc->res_dtype, a, static_cast<hipStream_t>(stream)));
}

int cbw_grad_workspace_size(const cbw_grad* grads, int32_t n, size_t* bytes)
{
    if (!bytes) return CBW_ERR_INVALID_ARG;
    GradWork work;
    const int st = check_grads(grads, n, false, &work);
    if (st != CBW_OK) return st;
    *bytes = work.ws_bytes();
    return CBW_OK;
}

int grad_norm(const cbw_grad* grads, int32_t n, int32_t kind, float* norm, void* workspace, size_t workspace_bytes,
              void* stream)
{
    GradWork work;
    int st = check_norm_call(grads, n, kind, false, norm, workspace, workspace_bytes, &work);
    if (st != CBW_OK) return st;
    hipStream_t s = static_cast<hipStream_t>(stream);
    double* partial = static_cast<double*>(workspace);
    int count;
    if ((st = norm_pass(grads, n, kind, work, partial, nullptr, s, &count)) != CBW_OK) return st;
    return hip_status(launch_grad_finish(kind, partial, count, norm, s));
}

int grad_clip(const cbw_grad* grads, int32_t n, int32_t kind, float max_norm, float* norm, void* workspace,
              size_t workspace_bytes, void* stream)
{
    GradWork work;
    int st = check_norm_call(grads, n, kind, true, norm, workspace, workspace_bytes, &work);
    if (st != CBW_OK) return st;
    if (!(max_norm >= 0.f)) return CBW_ERR_INVALID_ARG;
    hipStream_t s = static_cast<hipStream_t>(stream);
    double* partial = static_cast<double*>(workspace);
    GradEntry* table = reinterpret_cast<GradEntry*>(static_cast<char*>(workspace) + work.partial_bytes());
    int count;
    if ((st = norm_pass(grads, n, kind, work, partial, table, s, &count)) != CBW_OK) return st;
    // (without tensors one workgroup writes the norm, 0, and c)
    const int grid = work.chunks ? grad_grid(work.chunks, work.chunks) : 1;
    return hip_status(launch_grad_scale(table, (int)work.tensors, (int)work.chunks, kind, grid, partial, count, max_norm, norm, s));
}

}  // extern "C"
