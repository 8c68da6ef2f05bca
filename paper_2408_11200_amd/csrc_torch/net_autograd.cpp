// Autograd nodes of the operators of kan_net.h, and those that have no gradient (the clipping of a list of gradients, the steps of a beam search): nothing is computed here.  Without gradients to
// record (a server's calls) the node is passed by and nothing is kept.  Forward-mode tangents, which none of the operators has, go to the node,
// which refuses them: outputs without one would stand for a derivative of zero.
#include "kan_torch.hpp"
#include "kan_net.h"
#include <c10/core/DeviceGuard.h>
#include <torch/csrc/autograd/forward_grad.h>

namespace {

// whether there can be tangents at all: asked once a call, a list of 180 tensors would ask for 3 us
bool forward_mode() { return torch::autograd::ForwardADLevel::try_get_by_idx(0) != nullptr; }

bool has_tangent(const Tensor &t) { return t.defined() && t._fw_grad(0).defined(); }

bool recorded(std::initializer_list<const Tensor *> tensors)
{
    if (forward_mode())
        for (const Tensor *t : tensors)
            if (has_tangent(*t)) return true;
    if (!at::GradMode::is_enabled()) return false;
    for (const Tensor *t : tensors)
        if (t->defined() && t->requires_grad()) return true;
    return false;
}

int32_t type_of(at::ScalarType t)
{
    if (t != at::kFloat && t != at::kBFloat16) refuse("float32 and bfloat16 tensors only");
    return t == at::kFloat ? KAN_F32 : KAN_BF16;
}

// pointer of a device-resident contiguous tensor of a type (null: no tensor)
void *data(const Tensor &t, at::ScalarType type)
{
    if (!t.defined()) return nullptr;
    if (t.scalar_type() != type || !t.is_cuda() || !t.is_contiguous()) refuse("device-resident contiguous tensors of the operator's type only");
    return t.data_ptr();
}

const int64_t *ids_of(const Tensor &t)
{
    if (!t.defined()) return nullptr;
    if (t.scalar_type() != at::kLong || !t.is_cuda() || !t.is_contiguous()) refuse("device-resident contiguous int64 ids only");
    return static_cast<const int64_t *>(t.data_ptr());
}

void same(bool ok, const char *what)
{
    if (!ok) refuse(what);
}

// every tensor of a call on the device of the first
void together(std::initializer_list<const Tensor *> tensors)
{
    const Tensor &first = **tensors.begin();
    if (!first.is_cuda()) refuse("device-resident tensors only");
    for (const Tensor *t : tensors)
        if (t->defined() && t->device() != first.device()) refuse("tensors on one device only");
}

// backward(create_graph=True) would take these gradients for constants
void first_derivatives_only(const char *what) { TORCH_CHECK(!at::GradMode::is_enabled(), what, ": gradients of gradients are not available"); }

// ---- block norm -----------------------------------------------------------------------------

struct NormCall {
    kan_block_norm_desc d;
    bool want_h;
};

struct NormRows {
    Tensor x_out, h, stats;
};

constexpr const char *kNames[5] = {"w_post", "b_post", "gate", "w_pre", "b_pre"};

kan_block_norm_params params_of(const Tensor (&p)[5]) { return {f32(p[0]), f32(p[1]), f32(p[2]), f32(p[3]), f32(p[4])}; }

NormRows norm_forward(const Tensor &x, const Tensor &f, const Tensor (&p)[5], const NormCall &c, bool keep_stats)
{
    const Tensor xc = whole(x), fc = whole(f);
    const int64_t B = xc.numel() / c.d.n;
    const at::ScalarType stream_type = c.d.stream_type == KAN_F32 ? at::kFloat : at::kBFloat16, branch_type = c.d.branch_type == KAN_F32 ? at::kFloat : at::kBFloat16;
    NormRows r;
    if (f.defined()) r.x_out = at::empty(x.sizes(), x.options());
    if (c.want_h) r.h = at::empty(x.sizes(), x.options().dtype(branch_type));
    if (keep_stats) r.stats = at::empty({B, 4}, x.options().dtype(at::kFloat));
    const Tensor whole_p[5] = {whole(p[0]), whole(p[1]), whole(p[2]), whole(p[3]), whole(p[4])};
    const kan_block_norm_params q = params_of(whole_p);
    check(kan_block_norm_forward(&c.d, B, data(xc, stream_type), data(fc, branch_type), &q, data(r.x_out, stream_type), data(r.h, branch_type),
                                 f32(r.stats), stream()),
          "kan_block_norm_forward");
    return r;
}

struct BlockNorm : torch::autograd::Function<BlockNorm> {
    static variable_list forward(AutogradContext *ctx, const Tensor &x, const std::optional<Tensor> &f, const std::optional<Tensor> &w_post,
                                 const std::optional<Tensor> &b_post, const std::optional<Tensor> &gate, const std::optional<Tensor> &w_pre,
                                 const std::optional<Tensor> &b_pre, NormCall c)
    {
        const Tensor branch = or_none(f);
        const Tensor p[5] = {or_none(w_post), or_none(b_post), or_none(gate), or_none(w_pre), or_none(b_pre)};
        const NormRows r = norm_forward(x, branch, p, c, true);
        ctx->set_materialize_grads(false);
        ctx->saved_data["call"] = pack(c);
        ctx->save_for_backward({x, branch, p[0], p[1], p[2], p[3], p[4], r.stats});
        variable_list out;
        if (branch.defined()) out.push_back(r.x_out);
        if (c.want_h) out.push_back(r.h);
        return out;
    }

    static variable_list backward(AutogradContext *ctx, variable_list grads)
    {
        first_derivatives_only("block_norm");
        const NormCall c = unpack<NormCall>(ctx->saved_data["call"]);
        const variable_list saved = ctx->get_saved_variables();
        const Tensor x = whole(saved[0]), f = whole(saved[1]);
        const Tensor p[5] = {whole(saved[2]), whole(saved[3]), whole(saved[4]), whole(saved[5]), whole(saved[6])};
        const int64_t B = x.numel() / c.d.n;
        const at::ScalarType stream_type = x.scalar_type(), branch_type = c.d.branch_type == KAN_F32 ? at::kFloat : at::kBFloat16;
        variable_list g(8);
        const Tensor gx_out = f.defined() ? whole(grads[0]) : Tensor(), gh = c.want_h ? whole(grads[f.defined() ? 1 : 0]) : Tensor();
        if (!gx_out.defined() && !gh.defined()) return g;
        bool any = false;
        size_t edge = 0;        // of the tensors that are there
        for (int i = 0; i < 7; ++i) {
            if (!saved[i].defined()) continue;
            if (ctx->needs_input_grad(edge++)) g[i] = at::empty(saved[i].sizes(), saved[i].options()), any = true;
        }
        if (!any) return g;
        const kan_block_norm_params q = params_of(p);
        const kan_block_norm_grads w = {f32(g[2]), f32(g[3]), f32(g[4]), f32(g[5]), f32(g[6])};
        const bool sums = w.gw_post || w.gb_post || w.ggate || w.gw_pre || w.gb_pre;
        const Tensor ws = sums ? bytes_like(x, kan_block_norm_workspace_bytes(&c.d, B)) : Tensor();
        check(kan_block_norm_backward(&c.d, B, data(x, stream_type), data(f, branch_type), &q, static_cast<const float *>(kept(saved[7])),
                                      data(gx_out, stream_type), data(gh, branch_type), data(g[0], stream_type), data(g[1], branch_type), &w,
                                      sums ? ws.data_ptr() : nullptr, sums ? (size_t)ws.numel() : 0, stream()),
              "kan_block_norm_backward");
        return g;
    }
};

using Maybe = std::optional<Tensor>;

variable_list block_norm(const Tensor &x, const Maybe &f, const Maybe &w_post, const Maybe &b_post, const Maybe &gate, const Maybe &w_pre,
                         const Maybe &b_pre, int64_t n, int64_t norm, double eps, double residual_scale, int64_t gate_rows, int64_t branch_type,
                         bool want_h)
{
    const Tensor branch = or_none(f);
    const Tensor p[5] = {or_none(w_post), or_none(b_post), or_none(gate), or_none(w_pre), or_none(b_pre)};
    same(n > 0 && x.dim() >= 1 && x.size(-1) == n, "x: rows of n channels");
    same(!branch.defined() || branch.sizes() == x.sizes(), "f: the shape of x");
    together({&x, &branch, &p[0], &p[1], &p[2], &p[3], &p[4]});
    const c10::DeviceGuard on(x.device());
    same(branch.defined() || want_h, "no branch and no norm behind it: nothing to compute");
    const int64_t B = x.numel() / n, groups = gate_rows > 0 ? (B + gate_rows - 1) / gate_rows : 1;
    for (int i = 0; i < 5; ++i) same(!p[i].defined() || p[i].numel() == (i == 2 ? groups * n : n), kNames[i]);
    const NormCall c = {{(int32_t)n, (int32_t)norm, (float)eps, (float)residual_scale, gate_rows, type_of(x.scalar_type()),
                         branch.defined() ? type_of(branch.scalar_type()) : (int32_t)branch_type}, want_h};
    if (recorded({&x, &branch, &p[0], &p[1], &p[2], &p[3], &p[4]})) return BlockNorm::apply(x, f, w_post, b_post, gate, w_pre, b_pre, c);
    const NormRows r = norm_forward(x, branch, p, c, false);
    variable_list out;
    if (branch.defined()) out.push_back(r.x_out);
    if (want_h) out.push_back(r.h);
    return out;
}

// ---- embedding ------------------------------------------------------------------------------

Tensor embedding_rows(const Tensor &ids, const Tensor &table, double scale, at::ScalarType out)
{
    const Tensor ic = whole(ids), tc = whole(table);
    std::vector<int64_t> shape = ids.sizes().vec();
    shape.push_back(table.size(1));
    const Tensor y = at::empty(shape, table.options().dtype(out));
    check(kan_embedding_forward(ic.numel(), tc.size(0), (int32_t)tc.size(1), ids_of(ic), data(tc, table.scalar_type()), type_of(table.scalar_type()),
                                (float)scale, data(y, out), type_of(out), stream()),
          "kan_embedding_forward");
    return y;
}

struct Embedding : torch::autograd::Function<Embedding> {
    static Tensor forward(AutogradContext *ctx, const Tensor &ids, const Tensor &table, double scale, at::ScalarType out)
    {
        ctx->saved_data["scale"] = scale;
        ctx->saved_data["rows"] = table.size(0);
        ctx->saved_data["n"] = table.size(1);
        ctx->saved_data["type"] = (int64_t)table.scalar_type();
        ctx->save_for_backward({ids});
        return embedding_rows(ids, table, scale, out);
    }

    static variable_list backward(AutogradContext *ctx, variable_list grads)
    {
        first_derivatives_only("embedding");
        variable_list g(4);
        if (!ctx->needs_input_grad(1)) return g;
        const Tensor ids = whole(ctx->get_saved_variables()[0]), gy = whole(grads[0]);
        const int64_t V = ctx->saved_data["rows"].toInt(), n = ctx->saved_data["n"].toInt();
        const at::ScalarType type = (at::ScalarType)ctx->saved_data["type"].toInt();
        g[1] = at::empty({V, n}, gy.options().dtype(type));
        const Tensor ws = bytes_like(gy, kan_embedding_workspace_bytes(ids.numel(), V, (int32_t)n));
        check(kan_embedding_backward(ids.numel(), V, (int32_t)n, ids_of(ids), data(gy, gy.scalar_type()), type_of(gy.scalar_type()),
                                     (float)ctx->saved_data["scale"].toDouble(), data(g[1], type), type_of(type), ws.data_ptr(),
                                     (size_t)ws.numel(), stream()),
              "kan_embedding_backward");
        return g;
    }
};

Tensor embedding(const Tensor &ids, const Tensor &table, double scale, at::ScalarType out)
{
    same(table.dim() == 2 && table.size(0) > 0 && table.size(1) > 0 && table.size(1) < (1ll << 31), "table: rows of n channels");
    together({&table, &ids});
    const c10::DeviceGuard on(table.device());
    return recorded({&table}) ? Embedding::apply(ids, table, scale, out) : embedding_rows(ids, table, scale, out);
}

// ---- log probabilities ----------------------------------------------------------------------

struct LogprobCall {
    double temperature;
    int64_t top;
};

// Rows of logits as the C entries take them: two dimensions, the second one dense.  A slice of a wider buffer stays where it is.
Tensor rows_of(const Tensor &logits)
{
    const int64_t V = logits.size(-1);
    if (logits.dim() == 2 && logits.stride(1) == 1 && (logits.size(0) <= 1 || logits.stride(0) >= V)) return logits;
    return logits.contiguous().view({V ? logits.numel() / V : 0, V});
}

int64_t row_stride(const Tensor &rows) { return rows.size(0) > 1 ? rows.stride(0) : rows.size(1); }

struct LogprobRows {
    Tensor logp, entropy, stats, top_ids, top_logp;
};

LogprobRows logprob_forward(const Tensor &logits, const Tensor &ids, const LogprobCall &c, bool keep_stats)
{
    const Tensor rows = rows_of(logits), ic = whole(ids);
    const int64_t R = rows.size(0), V = rows.size(1);
    const auto f = logits.options().dtype(at::kFloat);
    std::vector<int64_t> shape = logits.sizes().vec();
    shape.pop_back();
    LogprobRows r;
    r.logp = at::empty(shape, f);
    r.entropy = at::empty(shape, f);
    if (keep_stats) r.stats = at::empty({R, 2}, f);
    if (c.top > 0) {
        shape.push_back(c.top);
        r.top_ids = at::empty(shape, f.dtype(at::kLong));
        r.top_logp = at::empty(shape, f);
    }
    const size_t need = kan_token_logprob_workspace_bytes(R, V, (int32_t)c.top);
    const Tensor ws = need ? bytes_like(logits, need) : Tensor();
    check(kan_token_logprob_forward(R, V, rows.data_ptr(), type_of(rows.scalar_type()), row_stride(rows), ids_of(ic), (float)c.temperature, (int32_t)c.top,
                                    f32(r.logp), f32(r.entropy), f32(r.stats), const_cast<int64_t *>(ids_of(r.top_ids)), f32(r.top_logp),
                                    need ? ws.data_ptr() : nullptr, need ? (size_t)ws.numel() : 0, stream()),
          "kan_token_logprob_forward");
    return r;
}

struct TokenLogprob : torch::autograd::Function<TokenLogprob> {
    static variable_list forward(AutogradContext *ctx, const Tensor &logits, const Tensor &ids, LogprobCall c)
    {
        const LogprobRows r = logprob_forward(logits, ids, c, true);
        ctx->set_materialize_grads(false);
        ctx->saved_data["call"] = pack(c);
        ctx->save_for_backward({logits, ids, r.stats, r.entropy});
        variable_list out = {r.logp, r.entropy};
        if (c.top > 0) {
            ctx->mark_non_differentiable({r.top_ids, r.top_logp});
            out.push_back(r.top_ids);
            out.push_back(r.top_logp);
        }
        return out;
    }

    static variable_list backward(AutogradContext *ctx, variable_list grads)
    {
        first_derivatives_only("token_logprob");
        variable_list g(3);
        const Tensor g_logp = whole(grads[0]), g_entropy = whole(grads[1]);
        if (!ctx->needs_input_grad(0) || (!g_logp.defined() && !g_entropy.defined())) return g;
        const LogprobCall c = unpack<LogprobCall>(ctx->saved_data["call"]);
        const variable_list saved = ctx->get_saved_variables();
        const Tensor rows = rows_of(saved[0]), ids = whole(saved[1]), entropy = whole(saved[3]);
        g[0] = at::empty(saved[0].sizes(), saved[0].options());
        check(kan_token_logprob_backward(rows.size(0), rows.size(1), rows.data_ptr(), type_of(rows.scalar_type()), row_stride(rows), ids_of(ids),
                                         (float)c.temperature, static_cast<const float *>(kept(saved[2])), f32(entropy), f32(g_logp), f32(g_entropy),
                                         g[0].data_ptr(), stream()),
              "kan_token_logprob_backward");
        return g;
    }
};

variable_list token_logprob(const Tensor &logits, const Tensor &ids, double temperature, int64_t top)
{
    same(logits.dim() >= 1 && logits.size(-1) > 0, "logits: rows of V values");
    same(ids.sizes() == logits.sizes().slice(0, logits.dim() - 1), "ids: one for each row of logits");
    same(top >= 0 && top <= logits.size(-1) && top <= KAN_TOP_MAX, "top: at most 64 and at most the vocabulary");
    together({&logits, &ids});
    const c10::DeviceGuard on(logits.device());
    const LogprobCall c = {temperature, top};
    if (recorded({&logits})) return TokenLogprob::apply(logits, ids, c);
    const LogprobRows r = logprob_forward(logits, ids, c, false);
    variable_list out = {r.logp, r.entropy};
    if (top > 0) out.insert(out.end(), {r.top_ids, r.top_logp});
    return out;
}

// ---- gradients of a network -----------------------------------------------------------------

Tensor clip_gradients(const std::vector<Tensor> &grads, double max_norm, const std::optional<std::vector<Tensor>> &out)
{
    const auto &to = out ? *out : grads;
    same(!grads.empty() && to.size() == grads.size(), "a list of gradients, and as many outputs");
    std::vector<kan_tensor_ref> list(grads.size());
    const bool forward = forward_mode(), graph = at::GradMode::is_enabled();
    for (size_t i = 0; i < grads.size(); ++i) {
        const Tensor &g = grads[i], &o = to[i];
        TORCH_CHECK(!(forward && (has_tangent(g) || has_tangent(o))) && !(graph && (g.requires_grad() || o.requires_grad())),
                    "clip_gradients: not differentiable, its tensors must not require gradients (or call it under torch.no_grad())");
        // any order of the elements will do, where the output's is the same
        if (!g.is_cuda() || !g.is_non_overlapping_and_dense()) refuse("device-resident dense tensors only");
        same(g.is_same(o) || (o.device() == g.device() && o.scalar_type() == g.scalar_type() && o.sizes() == g.sizes() && o.strides() == g.strides()),
             "an output of a gradient's type, shape and strides");
        same(g.device() == grads[0].device(), "gradients on one device");
        list[i] = {g.data_ptr(), o.data_ptr(), g.numel(), type_of(g.scalar_type())};
    }
    const c10::DeviceGuard on(grads[0].device());
    const Tensor norm = at::empty({}, grads[0].options().dtype(at::kFloat));
    const Tensor ws = bytes_like(norm, kan_clip_workspace_bytes((int32_t)list.size()));
    check(kan_clip_gradients((int32_t)list.size(), list.data(), (float)max_norm, f32(norm), ws.data_ptr(), (size_t)ws.numel(), stream()),
          "kan_clip_gradients");
    for (const Tensor &o : to)
        if (!o.is_inference()) o.unsafeGetTensorImpl()->bump_version();
    return norm;
}

// ---- divergence from a teacher's likely tokens ----------------------------------------------

struct DistillCall {
    double temperature;
    int64_t teacher, K;
};

struct DistillRows {
    Tensor loss, stats;
};

DistillRows distill_forward(const Tensor &logits, const Tensor &ids, const Tensor &values, const DistillCall &c, bool keep_stats)
{
    const Tensor rows = rows_of(logits), ic = whole(ids), vc = whole(values);
    const int64_t R = rows.size(0), V = rows.size(1);
    const auto f = logits.options().dtype(at::kFloat);
    DistillRows r;
    r.loss = at::empty(logits.sizes().slice(0, logits.dim() - 1), f);
    if (keep_stats) r.stats = at::empty({R, c.K + 2}, f);
    const size_t need = kan_token_distill_workspace_bytes(R, V, (int32_t)c.K);
    const Tensor ws = need ? bytes_like(logits, need) : Tensor();
    check(kan_token_distill_forward(R, V, rows.data_ptr(), type_of(rows.scalar_type()), row_stride(rows), (int32_t)c.K, ids_of(ic), data(vc, vc.scalar_type()),
                                    type_of(vc.scalar_type()), (int32_t)c.teacher, (float)c.temperature, f32(r.loss), f32(r.stats),
                                    need ? ws.data_ptr() : nullptr, need ? (size_t)ws.numel() : 0, stream()),
          "kan_token_distill_forward");
    return r;
}

struct TokenDistill : torch::autograd::Function<TokenDistill> {
    static Tensor forward(AutogradContext *ctx, const Tensor &logits, const Tensor &ids, const Tensor &values, DistillCall c)
    {
        const DistillRows r = distill_forward(logits, ids, values, c, true);
        ctx->saved_data["call"] = pack(c);
        ctx->save_for_backward({logits, ids, r.stats});
        return r.loss;
    }

    static variable_list backward(AutogradContext *ctx, variable_list grads)
    {
        first_derivatives_only("token_distill");
        variable_list g(4);
        if (!ctx->needs_input_grad(0) || !grads[0].defined()) return g;
        const DistillCall c = unpack<DistillCall>(ctx->saved_data["call"]);
        const variable_list saved = ctx->get_saved_variables();
        const Tensor rows = rows_of(saved[0]), ids = whole(saved[1]), g_loss = whole(grads[0]);
        g[0] = at::empty(saved[0].sizes(), saved[0].options());
        check(kan_token_distill_backward(rows.size(0), rows.size(1), rows.data_ptr(), type_of(rows.scalar_type()), row_stride(rows), (int32_t)c.K, ids_of(ids),
                                         (float)c.temperature, static_cast<const float *>(kept(saved[2])), f32(g_loss), g[0].data_ptr(), stream()),
              "kan_token_distill_backward");
        return g;
    }
};

Tensor token_distill(const Tensor &logits, const Tensor &ids, const Tensor &values, double temperature, int64_t teacher)
{
    same(logits.dim() >= 1 && logits.size(-1) > 0, "logits: rows of V values");
    same(ids.dim() == logits.dim() && ids.sizes() == values.sizes() && ids.sizes().slice(0, ids.dim() - 1) == logits.sizes().slice(0, logits.dim() - 1),
         "teacher: a list of ids and one of values for each row of logits");
    same(ids.size(-1) > 0 && ids.size(-1) <= KAN_TEACHER_MAX, "teacher: 1 to 256 tokens a row");
    together({&logits, &ids, &values});
    const c10::DeviceGuard on(logits.device());
    TORCH_CHECK(!recorded({&values}), "token_distill: not differentiable in the teacher's values (detach them)");
    const DistillCall c = {temperature, teacher, ids.size(-1)};
    if (recorded({&logits})) return TokenDistill::apply(logits, ids, values, c);
    return distill_forward(logits, ids, values, c, false).loss;
}

// ---- beam search ----------------------------------------------------------------------------

uint8_t *flags(const Tensor &t)
{
    if (!t.defined()) return nullptr;
    if (t.scalar_type() != at::kBool && t.scalar_type() != at::kByte) refuse("flags of type bool or uint8");
    return static_cast<uint8_t *>(data(t, t.scalar_type()));
}

variable_list beam_select(const Tensor &logits, const Tensor &scores, int64_t top, const Maybe &ended_, int64_t end_id, const Maybe &rank_scale_, double temperature)
{
    const Tensor ended = whole(or_none(ended_)), rank_scale = whole(or_none(rank_scale_)), sc = whole(scores);
    same(scores.dim() == 2 && scores.size(1) > 0 && scores.size(1) <= KAN_BEAM_MAX, "scores: a row of 1 to 64 beams for each search");
    const int64_t N = scores.size(0), B = scores.size(1);
    same((logits.dim() == 2 || logits.dim() == 3) && logits.size(-1) > 0, "logits: rows of V values");
    same(logits.dim() == 2 ? logits.size(0) == N * B : logits.size(0) == N && logits.size(1) == B, "logits: a row for each beam");
    same((!ended.defined() || ended.sizes() == scores.sizes()) && (!rank_scale.defined() || rank_scale.sizes() == scores.sizes()), "a flag and a scale for each beam");
    same(top > 0 && top <= KAN_TOP_MAX, "top: 1 to 64");
    together({&logits, &scores, &ended, &rank_scale});
    const c10::DeviceGuard on(logits.device());
    TORCH_CHECK(!recorded({&logits, &scores, &rank_scale}), "beam_select: not differentiable (detach its inputs, or call it under torch.no_grad())");
    const Tensor rows = rows_of(logits);
    const int64_t V = rows.size(1);
    const auto f = logits.options().dtype(at::kFloat);
    const variable_list out = {at::empty({N, top}, f), at::empty({N, top}, f.dtype(at::kLong)), at::empty({N, top}, f.dtype(at::kLong)), at::empty({N, top}, f.dtype(at::kBool))};
    const Tensor ws = bytes_like(logits, kan_beam_select_workspace_bytes(N, (int32_t)B, V, (int32_t)top));
    check(kan_beam_select(N, (int32_t)B, V, rows.data_ptr(), type_of(rows.scalar_type()), row_stride(rows), f32(sc), flags(ended), f32(rank_scale), end_id,
                          (float)temperature, (int32_t)top, f32(out[0]), const_cast<int64_t *>(ids_of(out[1])), const_cast<int64_t *>(ids_of(out[2])), flags(out[3]),
                          ws.data_ptr(), (size_t)ws.numel(), stream()),
          "kan_beam_select");
    return out;
}

struct Dimension {
    int64_t count = 1, stride = 0, out_stride = 0;
    // one more dimension in front
    void put_before(int64_t n, int64_t s, int64_t o)
    {
        if (n == 1) return;
        same(count == 1 || (s == stride * count && o == out_stride * count), "states whose dimensions before the rows, and behind them, lie evenly");
        if (count == 1) stride = s, out_stride = o;
        count *= n;
    }
};

// rows in dimension `dim`, a contiguous end of a row as one run, what is before and between as one dimension each
kan_state_ref state_of(const Tensor &t, const Tensor &o, int64_t dim)
{
    const int64_t size = (int64_t)t.element_size();
    int64_t run = size, d = t.dim() - 1;
    for (; d > dim && (t.size(d) == 1 || (t.stride(d) * size == run && o.stride(d) * size == run)); --d) run *= t.size(d);
    Dimension inner, outer;
    for (; d > dim; --d) inner.put_before(t.size(d), t.stride(d) * size, o.stride(d) * size);
    for (--d; d >= 0; --d) outer.put_before(t.size(d), t.stride(d) * size, o.stride(d) * size);
    return {t.data_ptr(), o.data_ptr(), outer.count, inner.count, run, {outer.stride, t.stride(dim) * size, inner.stride},
            {outer.out_stride, o.stride(dim) * size, inner.out_stride}};
}

void beam_reorder(const Tensor &parents, const std::vector<Tensor> &tensors, int64_t beams, const std::vector<Tensor> &out, int64_t dim)
{
    const Tensor order = whole(parents);
    same(parents.dim() == 2 && parents.size(1) > 0 && parents.size(1) <= KAN_BEAM_MAX, "parents: a row of 1 to 64 for each search");
    same(beams > 0 && beams <= KAN_BEAM_MAX, "beams: 1 to 64");
    same(tensors.size() == out.size(), "an output for each tensor");
    together({&parents});
    const int64_t N = parents.size(0), top = parents.size(1);
    std::vector<kan_state_ref> list;
    list.reserve(tensors.size());
    const bool forward = forward_mode(), graph = at::GradMode::is_enabled();
    for (size_t i = 0; i < tensors.size(); ++i) {
        const Tensor &t = tensors[i], &o = out[i];
        const int64_t d = dim < 0 ? dim + t.dim() : dim;
        TORCH_CHECK(!(forward && (has_tangent(t) || has_tangent(o))) && !(graph && (t.requires_grad() || o.requires_grad())),
                    "beam_reorder: not differentiable, its tensors must not require gradients (or call it under torch.no_grad())");
        same(t.device() == parents.device() && o.device() == parents.device() && t.scalar_type() == o.scalar_type(), "states on the device of the parents, outputs of their type");
        same(d >= 0 && d < t.dim() && o.dim() == t.dim() && t.size(d) == N * beams && o.size(d) == N * top, "a row of a state for each beam");
        for (int64_t k = 0; k < t.dim(); ++k) same(k == d || t.size(k) == o.size(k), "an output of a state's shape");
        if (o.numel() && t.numel()) list.push_back(state_of(t, o, d));
    }
    const c10::DeviceGuard on(parents.device());
    check(kan_beam_reorder(N, (int32_t)beams, (int32_t)top, ids_of(order), (int32_t)list.size(), list.data(), stream()), "kan_beam_reorder");
    for (const Tensor &o : out)
        if (!o.is_inference()) o.unsafeGetTensorImpl()->bump_version();
}

constexpr const char *kDistillOp = "paper_2408_11200_amd::token_distill", *kSelectOp = "paper_2408_11200_amd::beam_select";
constexpr const char *kNormOp = "paper_2408_11200_amd::block_norm", *kEmbeddingOp = "paper_2408_11200_amd::embedding",
                     *kLogprobOp = "paper_2408_11200_amd::token_logprob";

Tensor embedding_op(const Tensor &ids, const Tensor &table, double scale, bool wide)
{
    return embedding(ids, table, scale, wide ? at::kFloat : at::kBFloat16);
}

}  // namespace

TORCH_LIBRARY_FRAGMENT(paper_2408_11200_amd, m)
{
    m.def("block_norm(Tensor x, Tensor? f, Tensor? w_post, Tensor? b_post, Tensor? gate, Tensor? w_pre, Tensor? b_pre, int n, int norm, float eps, "
          "float residual_scale, int gate_rows, int branch_type, bool want_h) -> Tensor[]", &block_norm);
    m.def("embedding(Tensor ids, Tensor table, float scale, bool wide) -> Tensor", &embedding_op);
    m.def("token_logprob(Tensor logits, Tensor ids, float temperature, int top) -> Tensor[]", &token_logprob);
    m.def("token_distill(Tensor logits, Tensor ids, Tensor values, float temperature, int teacher) -> Tensor", &token_distill);
    m.def("beam_select(Tensor logits, Tensor scores, int top, Tensor? ended, int end_id, Tensor? rank_scale, float temperature) -> Tensor[]", &beam_select);
}

void define_net(pybind11::module_ &m)
{
    m.def("block_norm", [](int64_t n, int64_t norm, double eps, double residual_scale, int64_t gate_rows, int64_t branch_type, bool want_h,
                           const Tensor &x, const Maybe &f, const Maybe &w_post, const Maybe &b_post, const Maybe &gate, const Maybe &w_pre,
                           const Maybe &b_pre) {
        return call(kNormOp, &block_norm, x, f, w_post, b_post, gate, w_pre, b_pre, n, norm, eps, residual_scale, gate_rows, branch_type, want_h);
    });
    m.def("embedding", [](const Tensor &ids, const Tensor &table, double scale, bool wide) {
        return call(kEmbeddingOp, &embedding_op, ids, table, scale, wide);
    });
    m.def("token_logprob", [](const Tensor &logits, const Tensor &ids, double temperature, int64_t top) {
        return call(kLogprobOp, &token_logprob, logits, ids, temperature, top);
    });
    m.def("token_distill", [](const Tensor &logits, const Tensor &ids, const Tensor &values, double temperature, int64_t teacher) {
        return call(kDistillOp, &token_distill, logits, ids, values, temperature, teacher);
    });
    m.def("beam_select", [](const Tensor &logits, const Tensor &scores, int64_t top, const Maybe &ended, int64_t end_id, const Maybe &rank_scale, double temperature) {
        return call(kSelectOp, &beam_select, logits, scores, top, ended, end_id, rank_scale, temperature);
    });
    m.def("beam_reorder", [](const Tensor &parents, const std::vector<Tensor> &tensors, int64_t beams, const std::vector<Tensor> &out, int64_t dim) {
        py::gil_scoped_release unlock;
        beam_reorder(parents, tensors, beams, out, dim);
    });
    m.def("clip_gradients", [](const std::vector<Tensor> &grads, double max_norm, const std::optional<std::vector<Tensor>> &out) {
        py::gil_scoped_release unlock;
        return clip_gradients(grads, max_norm, out);
    });
}
