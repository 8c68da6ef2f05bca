// C entries of the block norms: checks, how the rows are cut among workers, and the sum of the workgroups' parameter gradients.
#include <initializer_list>
#include "net_norm.hpp"

namespace kannet {
namespace {

constexpr int kColumns = 64, kSegments = 16;     // a workgroup of the reduction: columns, and threads that share one

struct NormReduce {
    const float *part, *gate_part;
    kan_block_norm_params p;
    kan_block_norm_grads g;
    int64_t B, gate_rows;
    int n, blocks, parts;
    bool grouped, pre, post;
};

__device__ __forceinline__ float column_sum(const float *from, int64_t stride, int count, int column, int n, float (*lds)[kColumns])
{
    const int s = threadIdx.x / kColumns, c = threadIdx.x % kColumns;
    float t = 0.0f;
    if (column < n)
        for (int i = s; i < count; i += kSegments) t += from[i * stride + column];
    __syncthreads();
    lds[s][c] = t;
    __syncthreads();
    float total = 0.0f;
    for (int i = 0; i < kSegments; ++i) total += lds[i][c];
    return total;
}

// blockIdx.y: 0 w_pre, 1 b_pre, 2 w_post (and the gate, where there is one), 3 b_post, 4 + group: a group's gate
__global__ __launch_bounds__(kColumns *kSegments) void norm_reduce_kernel(NormReduce a)
{
    __shared__ float lds[kSegments][kColumns];
    const int which = blockIdx.y, n = a.n, c = blockIdx.x * kColumns + threadIdx.x % kColumns;
    const bool mine = threadIdx.x < kColumns && c < n;
    if (which >= 4) {
        const int64_t group = which - 4;
        const float t = column_sum(a.gate_part + group * a.parts * n, n, a.parts, c, n, lds);
        if (mine) a.g.ggate[group * n + c] = t;
        return;
    }
    const bool there = which < 2 ? a.pre : a.post;
    const float t = there ? column_sum(a.part + (int64_t)which * n, 4ll * n, a.blocks, c, n, lds) : 0.0f;
    const float gate = mine && !a.grouped && a.post && a.p.gate ? a.p.gate[c] : 1.0f;
    if (which == 0 && mine && a.g.gw_pre) a.g.gw_pre[c] = t;
    if (which == 1 && mine && a.g.gb_pre) a.g.gb_pre[c] = t;
    if (which == 2 && mine && a.g.gw_post) a.g.gw_post[c] = t * gate;
    if (which == 3 && mine && a.g.gb_post) a.g.gb_post[c] = t * gate;
    if (which == 2 && a.g.ggate && !a.grouped) {
        const float t0 = there && a.p.b_post ? column_sum(a.part + 3ll * n, 4ll * n, a.blocks, c, n, lds) : 0.0f;
        if (mine) a.g.ggate[c] = t * (a.post && a.p.w_post ? a.p.w_post[c] : 1.0f) + (a.post && a.p.b_post ? t0 * a.p.b_post[c] : 0.0f);
    }
}

struct Cut {
    int64_t span;
    int parts, blocks;
    int64_t workers;
};

int workers_of_block(int n) { return lanes_of_row(n) > 64 ? 1 : 256 / lanes_of_row(n); }

// Rows of a worker in the backward pass: about two workgroups a CU (1024 threads: one), four rows at least, so that the partial sums of
// the parameters stay below what the rows themselves cost.
Cut cut_rows(const kan_block_norm_desc *d, int64_t B)
{
    const int per_block = workers_of_block(d->n);
    const int64_t most = (int64_t)per_block * (lanes_of_row(d->n) >= 1024 ? 256 : 512);
    Cut c;
    c.span = div_up(B, most);
    if (c.span < 4) c.span = 4;
    c.parts = 0;
    if (d->gate_rows > 0) {
        if (d->gate_rows >= c.span && d->gate_rows < B) {
            c.parts = (int)div_up(d->gate_rows, c.span);
            c.span = div_up(d->gate_rows, (int64_t)c.parts);
            c.workers = div_up(B, d->gate_rows) * c.parts;
            c.blocks = (int)div_up(c.workers, (int64_t)per_block);
            return c;
        }
        if (d->gate_rows < c.span) c.span = c.span / d->gate_rows * d->gate_rows;
    }
    c.workers = div_up(B, c.span);
    c.blocks = (int)div_up(c.workers, (int64_t)per_block);
    return c;
}

// one group holds all rows: the same as one gate for all
bool grouped(const kan_block_norm_desc *d, int64_t B) { return d->gate_rows > 0 && d->gate_rows < B; }

int check(const kan_block_norm_desc *d)
{
    if (!d || d->n <= 0 || !(d->eps > 0.0f) || d->gate_rows < 0) return KAN_ERR_INVALID_ARG;
    if (d->n > 16384 || (d->norm != KAN_NORM_RMS && d->norm != KAN_NORM_LAYER)) return KAN_ERR_UNSUPPORTED;
    if (!known_type(d->stream_type) || !known_type(d->branch_type)) return KAN_ERR_UNSUPPORTED;
    if (d->branch_type == KAN_BF16 && d->stream_type == KAN_F32) return KAN_ERR_UNSUPPORTED;
    return KAN_OK;
}

int check_pointers(const kan_block_norm_desc *d, std::initializer_list<const void *> stream, std::initializer_list<const void *> branch,
                   std::initializer_list<const void *> floats)
{
    for (const void *p : stream)
        if (misplaced(p, d->stream_type)) return KAN_ERR_INVALID_ARG;
    for (const void *p : branch)
        if (misplaced(p, d->branch_type)) return KAN_ERR_INVALID_ARG;
    for (const void *p : floats)
        if (misplaced(p, KAN_F32)) return KAN_ERR_INVALID_ARG;
    return KAN_OK;
}

hipError_t launch(const kan_block_norm_desc *d, const NormCall &a, bool backward, bool by_group, int blocks, hipStream_t st)
{
    const bool layer = d->norm == KAN_NORM_LAYER;
    return d->stream_type == KAN_F32 ? launch_norm_f32(a, layer, backward, by_group, blocks, st)
         : d->branch_type == KAN_F32 ? launch_norm_bf16_f32(a, layer, backward, by_group, blocks, st)
                                     : launch_norm_bf16(a, layer, backward, by_group, blocks, st);
}

NormCall call_of(const kan_block_norm_desc *d, int64_t B, const void *x, const void *f, const kan_block_norm_params *p)
{
    NormCall a = {};
    a.x = x;
    a.f = f;
    if (p) a.p = *p;
    a.B = B;
    a.gate_rows = grouped(d, B) ? d->gate_rows : 0;
    a.n = d->n;
    a.eps = d->eps;
    a.residual_scale = d->residual_scale;
    a.inv_n = 1.0f / (float)d->n;
    return a;
}

size_t part_bytes(const kan_block_norm_desc *d, const Cut &c) { return align_up((size_t)c.blocks * 4 * (size_t)d->n * sizeof(float)); }

}  // namespace
}  // namespace kannet

using namespace kannet;

extern "C" int kan_block_norm_forward(const kan_block_norm_desc *desc, int64_t B, const void *x, const void *f,
                                      const kan_block_norm_params *p, void *x_out, void *h, float *stats, void *stream)
{
    int rc = check(desc);
    if (rc != KAN_OK) return rc;
    if (B < 0) return KAN_ERR_INVALID_ARG;
    if (B == 0) return KAN_OK;
    if (!x || (f && !x_out) || (!f && !h)) return KAN_ERR_INVALID_ARG;
    const kan_block_norm_params none = {};
    const kan_block_norm_params *q = p ? p : &none;
    rc = check_pointers(desc, {x, f ? x_out : nullptr}, {f, h}, {q->w_post, q->b_post, q->gate, q->w_pre, q->b_pre, stats});
    if (rc != KAN_OK) return rc;
    NormCall a = call_of(desc, B, x, f, p);
    a.x_out = x_out;
    a.h = h;
    a.stats = stats;
    const int64_t blocks = div_up(B, (int64_t)workers_of_block(desc->n));
    const int64_t most = lanes_of_row(desc->n) >= 512 ? 1024 : 2048;
    return status_of(launch(desc, a, false, false, (int)(blocks < most ? blocks : most), (hipStream_t)stream));
}

extern "C" size_t kan_block_norm_workspace_bytes(const kan_block_norm_desc *desc, int64_t B)
{
    if (check(desc) != KAN_OK || B <= 0) return 0;
    const Cut c = cut_rows(desc, B);
    return part_bytes(desc, c) + (c.parts ? align_up((size_t)c.workers * (size_t)desc->n * sizeof(float)) : 0);
}

extern "C" int kan_block_norm_backward(const kan_block_norm_desc *desc, int64_t B, const void *x, const void *f,
                                       const kan_block_norm_params *p, const float *stats, const void *gx_out, const void *gh, void *gx,
                                       void *gf, const kan_block_norm_grads *g, void *ws, size_t ws_bytes, void *stream)
{
    int rc = check(desc);
    if (rc != KAN_OK) return rc;
    if (B < 0) return KAN_ERR_INVALID_ARG;
    const kan_block_norm_params no_params = {};
    const kan_block_norm_grads no_grads = {};
    const kan_block_norm_params *q = p ? p : &no_params;
    const kan_block_norm_grads *w = g ? g : &no_grads;
    if (B > 0 && (!x || !stats || (!gx_out && !gh) || (!f && (gf || w->gw_post || w->gb_post || w->ggate)))) return KAN_ERR_INVALID_ARG;
    rc = check_pointers(desc, {x, gx_out, gx}, {f, gh, gf},
                        {q->w_post, q->b_post, q->gate, q->w_pre, q->b_pre, stats, w->gw_post, w->gb_post, w->ggate, w->gw_pre, w->gb_pre});
    if (rc != KAN_OK) return rc;
    const bool params = w->gw_post || w->gb_post || w->ggate || w->gw_pre || w->gb_pre;
    hipStream_t st = (hipStream_t)stream;
    const Cut c = B > 0 ? cut_rows(desc, B) : Cut{0, 0, 0, 0};
    if (B > 0 && params && bad_workspace(ws, ws_bytes, kan_block_norm_workspace_bytes(desc, B))) return KAN_ERR_WORKSPACE;
    const bool by_group = grouped(desc, B > 0 ? B : 1);
    if (B > 0) {
        NormCall a = call_of(desc, B, x, f, p);
        a.stats = const_cast<float *>(stats);
        a.gx_out = gx_out;
        a.gh = gh;
        a.gx = gx;
        a.gf = gf;
        a.ggate = w->ggate;
        a.part = params ? (float *)ws : nullptr;
        a.gate_part = params ? (float *)((char *)ws + part_bytes(desc, c)) : nullptr;
        a.span = c.span;
        a.parts = c.parts;
        const hipError_t e = launch(desc, a, true, by_group, c.blocks, st);
        if (e != hipSuccess) return KAN_ERR_HIP;
    }
    if (!params) return KAN_OK;
    NormReduce r = {};
    r.part = (const float *)ws;
    r.gate_part = (const float *)((const char *)ws + (B > 0 ? part_bytes(desc, c) : 0));
    r.p = *q;
    r.g = *w;
    r.B = B;
    r.gate_rows = desc->gate_rows;
    r.n = desc->n;
    r.blocks = c.blocks;
    r.parts = c.parts;
    r.grouped = B > 0 ? by_group : desc->gate_rows > 0;
    r.pre = B > 0 && gh;
    r.post = B > 0 && f;
    const unsigned groups = c.parts && w->ggate && f ? (unsigned)div_up(B, desc->gate_rows) : 0;
    prof::Timed timed("block_norm_reduce", st);
    norm_reduce_kernel<<<dim3((unsigned)div_up(desc->n, kColumns), 4 + groups), kColumns * kSegments, 0, st>>>(r);
    return status_of(hipGetLastError());
}
