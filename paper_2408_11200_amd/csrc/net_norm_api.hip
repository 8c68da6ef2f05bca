// C entries of the block norms: checks, how the rows are cut among workers, and the sum of the workgroups' parameter gradients.
#include <initializer_list>
#include "net_norm.hpp"

namespace kannet {
namespace {

constexpr int kColumns = 32, kSegments = 32;     // a workgroup of the reduction: columns, and threads that share one
constexpr int kFewParts = 16;                    // of a group: summed by one thread a column

struct NormReduce {
    const float *part, *gate_part;
    kan_block_norm_params p;
    kan_block_norm_grads g;
    int64_t gates;          // groups * n
    int n, blocks, parts;
    bool by_group, bias, pre, post;
};

// sum over `count` rows of partial sums, in a fixed order: segments of rows a thread each, several loads in flight
__device__ __forceinline__ float column_sum(const float *from, int64_t stride, int count, int column, int n, float (*lds)[kColumns])
{
    const int s = threadIdx.x / kColumns, c = threadIdx.x % kColumns;
    float t[4] = {0.0f, 0.0f, 0.0f, 0.0f};
    if (column < n) {
        int i = s;
        for (; i + 3 * kSegments < count; i += 4 * kSegments)
#pragma unroll
            for (int k = 0; k < 4; ++k) t[k] += from[(i + k * kSegments) * stride + column];
        for (; i < count; i += kSegments) t[0] += from[i * stride + column];
    }
    __syncthreads();
    lds[s][c] = (t[0] + t[1]) + (t[2] + t[3]);
    __syncthreads();
    float total = 0.0f;
    if (s == 0)
        for (int i = 0; i < kSegments; ++i) total += lds[i][c];
    return total;
}

// blockIdx.y: 0 w_pre, 1 b_pre, 2 w_post, b_post and a gate that all rows share, 3 + group: a group's gate from its parts (few parts: 3 + ..., all
// groups' columns a thread each)
__global__ __launch_bounds__(kColumns *kSegments) void norm_reduce_kernel(NormReduce a)
{
    __shared__ float lds[kSegments][kColumns];
    const int which = blockIdx.y, n = a.n, c = blockIdx.x * kColumns + threadIdx.x % kColumns;
    const bool mine = threadIdx.x < kColumns && c < n;
    if (which >= 3 && a.parts <= kFewParts) {
        const int64_t i = ((int64_t)(which - 3) * gridDim.x + blockIdx.x) * blockDim.x + threadIdx.x;
        if (i >= a.gates) return;
        const int64_t group = i / n;
        const float *from = a.gate_part + group * a.parts * n + (i - group * n);
        float t = 0.0f;
        for (int k = 0; k < a.parts; ++k) t += from[(int64_t)k * n];
        a.g.ggate[i] = t;
        return;
    }
    if (which >= 3) {
        const int64_t group = which - 3;
        const float t = column_sum(a.gate_part + group * a.parts * n, n, a.parts, c, n, lds);
        if (mine) a.g.ggate[group * n + c] = t;
        return;
    }
    const bool there = which < 2 ? a.pre && (which == 0 || a.bias) : a.post;
    const float t = there ? column_sum(a.part + (int64_t)which * n, 4ll * n, a.blocks, c, n, lds) : 0.0f;
    if (which == 0 && mine && a.g.gw_pre) a.g.gw_pre[c] = t;
    if (which == 1 && mine && a.g.gb_pre) a.g.gb_pre[c] = t;
    if (which < 2) return;
    const float t0 = there && a.bias ? column_sum(a.part + 3ll * n, 4ll * n, a.blocks, c, n, lds) : 0.0f;
    if (!mine) return;
    const float gate = !a.by_group && there && a.p.gate ? a.p.gate[c] : 1.0f;
    if (a.g.gw_post) a.g.gw_post[c] = t * gate;
    if (a.g.gb_post) a.g.gb_post[c] = t0 * gate;
    if (a.g.ggate && !a.by_group) a.g.ggate[c] = t * (there && a.p.w_post ? a.p.w_post[c] : 1.0f) + (there && a.p.b_post ? t0 * a.p.b_post[c] : 0.0f);
}

struct Cut {
    int64_t span;
    int parts, blocks;
    int64_t workers;
};

int forward_workers(int n) { return lanes_of_row(n) > 64 ? 1 : 256 / lanes_of_row(n); }
int backward_workers(int n) { return lanes_of_row(n) > 512 ? 1 : 512 / lanes_of_row(n); }

// Rows of a worker in the backward pass: one workgroup a CU (its registers fill one), two rows at least, so that the partial sums of the
// parameters stay below what the rows themselves cost.  A worker has rows of one group of a gate, or whole groups; of both ways to cut, the one
// with the least rows behind each other on a CU, a workgroup's start and end taken as four rows more.  (22369 x 1500 fp32, a gate every
// 7 rows: 267 workgroups of 42 rows left most CUs idle while the last eleven ran, 310 us; 229 of 49 rows
// 208.  Every 40 rows: 280 of two whole groups 287 us, 560 of half a group 184.)
Cut cut_rows(const kan_block_norm_desc *d, int64_t B)
{
    const int per_block = backward_workers(d->n);
    const int64_t most = (int64_t)per_block * 256;
    Cut c;
    c.span = div_up(B, most);
    if (c.span < 2) c.span = 2;
    c.parts = 0;
    c.workers = div_up(B, c.span);
    if (d->gate_rows > 0 && d->gate_rows < B) {
        const int64_t groups = div_up(B, d->gate_rows), fair = c.span;
        int64_t least = INT64_MAX;
        const auto consider = [&](int64_t span, int64_t workers, int64_t parts) {
            const int64_t cost = div_up(workers, most) * (span + 4);
            if (cost >= least) return;
            least = cost;
            c.span = span;
            c.workers = workers;
            c.parts = (int)parts;
        };
        if (d->gate_rows < fair) {
            const int64_t some = fair / d->gate_rows;
            for (int64_t m = some; m <= some + 1; ++m) consider(m * d->gate_rows, div_up(groups, m), 0);
        }
        for (int64_t parts = 1; groups <= 4 * most && parts <= div_up(d->gate_rows, fair) + 3; ++parts) {
            const int64_t span = div_up(d->gate_rows, parts);
            if (span < 2) break;
            consider(span, groups * div_up(d->gate_rows, span), div_up(d->gate_rows, span));
        }
    }
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

hipError_t launch(const kan_block_norm_desc *d, const NormCall &a, const NormPick &p, hipStream_t st)
{
    return d->stream_type == KAN_F32 ? launch_norm_f32(a, p, st) : d->branch_type == KAN_F32 ? launch_norm_bf16_f32(a, p, st) : launch_norm_bf16(a, p, st);
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
    a.lanes = div_up(d->n, 512) * 64;
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
    const int64_t blocks = div_up(B, (int64_t)forward_workers(desc->n));
    const NormPick pick = {desc->norm == KAN_NORM_LAYER, false, false, false, (int)(blocks < 65536 ? blocks : 65536)};
    return status_of(launch(desc, a, pick, (hipStream_t)stream));
}

extern "C" size_t kan_block_norm_workspace_bytes(const kan_block_norm_desc *desc, int64_t B)
{
    if (check(desc) != KAN_OK || B <= 0) return 0;
    const Cut c = cut_rows(desc, B);
    return part_bytes(desc, c) + (c.parts > 1 ? align_up((size_t)c.workers * (size_t)desc->n * sizeof(float)) : 0);
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
    const bool by_group = B > 0 ? grouped(desc, B) : desc->gate_rows > 0;
    const bool bias = q->b_post || w->gb_post || w->gb_pre;
    if (B > 0) {
        NormCall a = call_of(desc, B, x, f, p);
        a.stats = const_cast<float *>(stats);
        a.gx_out = gx_out;
        a.gh = gh;
        a.gx = gx;
        a.gf = gf;
        a.ggate = w->ggate;
        a.part = params ? (float *)ws : nullptr;
        // a group in one part: its gate's gradient is whole
        a.gate_part = c.parts == 1 ? w->ggate : params ? (float *)((char *)ws + part_bytes(desc, c)) : nullptr;
        a.span = c.span;
        a.parts = c.parts;
        const NormPick pick = {desc->norm == KAN_NORM_LAYER, true, by_group && !c.parts, bias, c.blocks};
        const hipError_t e = launch(desc, a, pick, st);
        if (e != hipSuccess) return KAN_ERR_HIP;
    }
    if (!params) return KAN_OK;
    NormReduce r = {};
    r.part = (const float *)ws;
    r.gate_part = (const float *)((const char *)ws + (B > 0 ? part_bytes(desc, c) : 0));
    r.p = *q;
    r.g = *w;
    r.n = desc->n;
    r.blocks = c.blocks;
    r.parts = c.parts;
    r.by_group = by_group;
    r.bias = bias;
    r.pre = B > 0 && gh;
    r.post = B > 0 && f;
    const unsigned across = (unsigned)div_up(desc->n, kColumns);
    int64_t more = c.parts > 1 && w->ggate && f ? div_up(B, desc->gate_rows) : 0;
    r.gates = more * desc->n;
    if (c.parts <= kFewParts) more = div_up(r.gates, (int64_t)across * kColumns * kSegments);
    prof::Timed timed("block_norm_reduce", st);
    norm_reduce_kernel<<<dim3(across, 3 + (unsigned)more), kColumns * kSegments, 0, st>>>(r);
    return status_of(hipGetLastError());
}
