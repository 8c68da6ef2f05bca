// Kernels of the norms at a block boundary (kan_net.h), one instance for each pair of types and kind of norm.
//
// Both passes are bound by HBM: a row is read into registers once (eight channels a lane and piece, TPR lanes a row), and everything that
// needs the whole row (mean, mean square, the two projections of the backward pass) is a sum over those lanes.  Workers are the groups of
// TPR lanes; rows of up to 512 channels lie within a wave, so that their sums are DPP moves and need no barrier.
#pragma once
#include "net_device.hpp"

namespace kannet {

struct NormCall {
    const void *x, *f;
    kan_block_norm_params p;
    void *x_out, *h;
    float *stats;
    const void *gx_out, *gh;
    void *gx, *gf;
    float *ggate;           // backward of grouped gates: rows of whole groups go straight there
    float *part;            // [workgroups][4][n]: sums for w_pre, b_pre, w_post, b_post
    float *gate_part;       // [workers][n]: a group's gate gradient in parts
    int64_t B, gate_rows;   // gate_rows = 0: one gate row
    int64_t span;           // rows of a worker (grouped: rows of a part of a group, or of whole groups)
    int parts;              // grouped: parts a group is cut into; 0: a worker has whole groups
    int n;
    float eps, residual_scale, inv_n;
};

template <int TPR>
constexpr int threads_of() { return TPR < 256 ? (TPR > 64 ? TPR : 256) : TPR; }

template <int P>
__device__ __forceinline__ void load_param(const float *w, int lane, int tpr, int n, float none, float (&v)[P][8])
{
#pragma unroll
    for (int q = 0; q < P; ++q) {
        const int c = (q * tpr + lane) * 8;
        if (w) {
            load_some(w + c, n - c, v[q]);
        } else {
#pragma unroll
            for (int k = 0; k < 8; ++k) v[q][k] = none;
        }
    }
}

template <int P, class T>
__device__ __forceinline__ void load_row(const void *base, int64_t row, int lane, int tpr, int n, float (&v)[P][8])
{
#pragma unroll
    for (int q = 0; q < P; ++q) {
        const int c = (q * tpr + lane) * 8;
        load_some((const T *)base + row * n + c, n - c, v[q]);
    }
}

template <int P, class T>
__device__ __forceinline__ void store_row(void *base, int64_t row, int lane, int tpr, int n, const float (&v)[P][8])
{
#pragma unroll
    for (int q = 0; q < P; ++q) {
        const int c = (q * tpr + lane) * 8;
        store_some((T *)base + row * n + c, n - c, v[q]);
    }
}

// v becomes norm(v) (0 in channels past the row's end); mean and 1/sigma.  The variance is that of the centred values: the mean of the
// squares less the squared mean would lose all digits where the mean is large.
template <int TPR, int P, bool LAYER>
__device__ __forceinline__ void normalise(float (&v)[P][8], int lane, int n, float inv_n, float eps, RowSum<TPR> &total, float &mean, float &r)
{
    mean = 0.0f;
    if constexpr (LAYER) {
        float s = 0.0f;
#pragma unroll
        for (int q = 0; q < P; ++q)
#pragma unroll
            for (int k = 0; k < 8; ++k) s += v[q][k];
        mean = total(s) * inv_n;
#pragma unroll
        for (int q = 0; q < P; ++q)
#pragma unroll
            for (int k = 0; k < 8; ++k) v[q][k] = (q * TPR + lane) * 8 + k < n ? v[q][k] - mean : 0.0f;
    }
    float s = 0.0f;
#pragma unroll
    for (int q = 0; q < P; ++q)
#pragma unroll
        for (int k = 0; k < 8; ++k) s += v[q][k] * v[q][k];
    r = 1.0f / sqrtf(total(s) * inv_n + eps);
#pragma unroll
    for (int q = 0; q < P; ++q)
#pragma unroll
        for (int k = 0; k < 8; ++k) v[q][k] *= r;
}

template <class X, class F, int TPR, int P, bool LAYER>
__global__ __launch_bounds__(threads_of<TPR>()) void norm_forward_kernel(NormCall a)
{
    constexpr int kWorkers = threads_of<TPR>() / TPR;
    __shared__ float slots[RowSum<TPR>::kSlots];
    RowSum<TPR> total{slots};
    const int lane = threadIdx.x % TPR, n = a.n;
    const int64_t step = (int64_t)gridDim.x * kWorkers;
    float w_post[P][8], b_post[P][8], gate[P][8], w_pre[P][8], b_pre[P][8];
    load_param<P>(a.p.w_pre, lane, TPR, n, 1.0f, w_pre);
    load_param<P>(a.p.b_pre, lane, TPR, n, 0.0f, b_pre);
    load_param<P>(a.f ? a.p.w_post : nullptr, lane, TPR, n, 1.0f, w_post);
    load_param<P>(a.f ? a.p.b_post : nullptr, lane, TPR, n, 0.0f, b_post);
    load_param<P>(a.f && !a.gate_rows ? a.p.gate : nullptr, lane, TPR, n, 1.0f, gate);
    for (int64_t row = (int64_t)blockIdx.x * kWorkers + threadIdx.x / TPR; row < a.B; row += step) {
        float v[P][8], st[4] = {0.0f, 0.0f, 0.0f, 0.0f};
        load_row<P, X>(a.x, row, lane, TPR, n, v);
        if (a.f) {
            float u[P][8];
            load_row<P, F>(a.f, row, lane, TPR, n, u);
            if (a.gate_rows && a.p.gate) load_param<P>(a.p.gate + row / a.gate_rows * n, lane, TPR, n, 1.0f, gate);
            normalise<TPR, P, LAYER>(u, lane, n, a.inv_n, a.eps, total, st[0], st[1]);
#pragma unroll
            for (int q = 0; q < P; ++q)
#pragma unroll
                for (int k = 0; k < 8; ++k) v[q][k] = a.residual_scale * v[q][k] + gate[q][k] * (u[q][k] * w_post[q][k] + b_post[q][k]);
            store_row<P, X>(a.x_out, row, lane, TPR, n, v);
        }
        if (a.h) {
            normalise<TPR, P, LAYER>(v, lane, n, a.inv_n, a.eps, total, st[2], st[3]);
#pragma unroll
            for (int q = 0; q < P; ++q)
#pragma unroll
                for (int k = 0; k < 8; ++k) v[q][k] = v[q][k] * w_pre[q][k] + b_pre[q][k];
            store_row<P, F>(a.h, row, lane, TPR, n, v);
        }
        if (a.stats && lane == 0) {
#pragma unroll
            for (int i = 0; i < 4; ++i) a.stats[row * 4 + i] = st[i];
        }
    }
}

// q, the gradient of norm(v), becomes that of v
template <int TPR, int P, bool LAYER>
__device__ __forceinline__ void norm_back(float (&q)[P][8], const float (&vhat)[P][8], float r, float inv_n, RowSum<TPR> &total)
{
    float s[2] = {0.0f, 0.0f};
#pragma unroll
    for (int p = 0; p < P; ++p)
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            s[0] += q[p][k] * vhat[p][k];
            if (LAYER) s[1] += q[p][k];
        }
    if constexpr (LAYER) {
        total.sum(s);
    } else {
        s[0] = total(s[0]);
    }
    const float c1 = s[0] * inv_n, c0 = s[1] * inv_n;
#pragma unroll
    for (int p = 0; p < P; ++p)
#pragma unroll
        for (int k = 0; k < 8; ++k) q[p][k] = (q[p][k] - vhat[p][k] * c1 - c0) * r;
}

// Gradients of the rows, and of the parameters summed over a worker's rows (consecutive ones).  With one gate for all rows the worker's
// sums of d and d * norm(f) are kept as they are: gate, w_post and b_post are common factors, put in when the workgroups' sums are added.
// Gates of groups: `parts` > 0, a worker has a part of one group, else whole groups.
template <class X, class F, int TPR, int P, bool LAYER, bool GROUPED>
__global__ __launch_bounds__(threads_of<TPR>()) void norm_backward_kernel(NormCall a)
{
    constexpr int NT = threads_of<TPR>(), kWorkers = NT / TPR;
    __shared__ float slots[RowSum<TPR>::kSlots];
    __shared__ float joined[kWorkers > 1 ? NT * 8 : 1];
    RowSum<TPR> total{slots};
    const int lane = threadIdx.x % TPR, n = a.n;
    const int64_t worker = (int64_t)blockIdx.x * kWorkers + threadIdx.x / TPR;
    int64_t row, end, group = 0;
    if (GROUPED && a.parts) {
        group = worker / a.parts;
        row = group * a.gate_rows + worker % a.parts * a.span;
        end = row + a.span < (group + 1) * a.gate_rows ? row + a.span : (group + 1) * a.gate_rows;
    } else {
        row = worker * a.span;
        end = row + a.span;
        if (GROUPED) group = row / a.gate_rows;
    }
    if (end > a.B) end = a.B;
    const bool any = row < end;

    float w_post[P][8], b_post[P][8], gate[P][8], w_pre[P][8];
    load_param<P>(a.p.w_pre, lane, TPR, n, 1.0f, w_pre);
    load_param<P>(a.f ? a.p.w_post : nullptr, lane, TPR, n, 1.0f, w_post);
    load_param<P>(a.f ? a.p.b_post : nullptr, lane, TPR, n, 0.0f, b_post);
    load_param<P>(a.f && !GROUPED ? a.p.gate : nullptr, lane, TPR, n, 1.0f, gate);
    float pre1[P][8] = {}, pre0[P][8] = {}, s1[P][8] = {}, s0[P][8] = {}, post1[P][8] = {}, post0[P][8] = {};
    bool fresh = true;          // the gate's row is still to be read
    for (; row < end; ++row) {
        if (GROUPED && fresh) {
            if (a.f && a.p.gate) load_param<P>(a.p.gate + group * n, lane, TPR, n, 1.0f, gate);
            fresh = false;
        }
        const float *st = a.stats + row * 4;
        const float mean_f = st[0], r_f = st[1], mean_x = st[2], r_x = st[3];
        float v[P][8], fhat[P][8], d[P][8];
        load_row<P, X>(a.x, row, lane, TPR, n, v);
        if (a.gx_out) {
            load_row<P, X>(a.gx_out, row, lane, TPR, n, d);
        } else {
#pragma unroll
            for (int q = 0; q < P; ++q)
#pragma unroll
                for (int k = 0; k < 8; ++k) d[q][k] = 0.0f;
        }
        if (a.f) {
            load_row<P, F>(a.f, row, lane, TPR, n, fhat);
#pragma unroll
            for (int q = 0; q < P; ++q)
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    const bool in = !LAYER || (q * TPR + lane) * 8 + k < n;
                    fhat[q][k] = in ? (fhat[q][k] - mean_f) * r_f : 0.0f;
                    v[q][k] = a.residual_scale * v[q][k] + gate[q][k] * (fhat[q][k] * w_post[q][k] + b_post[q][k]);
                }
        }
        if (a.gh) {
            float g[P][8];
            load_row<P, F>(a.gh, row, lane, TPR, n, g);
#pragma unroll
            for (int q = 0; q < P; ++q)
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    const bool in = !LAYER || (q * TPR + lane) * 8 + k < n;
                    v[q][k] = in ? (v[q][k] - mean_x) * r_x : 0.0f;
                    pre1[q][k] += g[q][k] * v[q][k];
                    pre0[q][k] += g[q][k];
                    g[q][k] *= w_pre[q][k];
                }
            norm_back<TPR, P, LAYER>(g, v, r_x, a.inv_n, total);
#pragma unroll
            for (int q = 0; q < P; ++q)
#pragma unroll
                for (int k = 0; k < 8; ++k) d[q][k] += g[q][k];
        }
        if (a.gx) {
            float g[P][8];
            const float scale = a.f ? a.residual_scale : 1.0f;
#pragma unroll
            for (int q = 0; q < P; ++q)
#pragma unroll
                for (int k = 0; k < 8; ++k) g[q][k] = scale * d[q][k];
            store_row<P, X>(a.gx, row, lane, TPR, n, g);
        }
        if (a.f) {
#pragma unroll
            for (int q = 0; q < P; ++q)
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    s1[q][k] += d[q][k] * fhat[q][k];
                    s0[q][k] += d[q][k];
                    d[q][k] = !LAYER || (q * TPR + lane) * 8 + k < n ? d[q][k] * gate[q][k] * w_post[q][k] : 0.0f;
                }
            if (a.gf) {
                norm_back<TPR, P, LAYER>(d, fhat, r_f, a.inv_n, total);
                store_row<P, F>(a.gf, row, lane, TPR, n, d);
            }
            if (GROUPED && (row + 1 == end || (!a.parts && (row + 1) % a.gate_rows == 0))) {
                float g[P][8];
#pragma unroll
                for (int q = 0; q < P; ++q)
#pragma unroll
                    for (int k = 0; k < 8; ++k) {
                        g[q][k] = s1[q][k] * w_post[q][k] + s0[q][k] * b_post[q][k];
                        post1[q][k] += gate[q][k] * s1[q][k];
                        post0[q][k] += gate[q][k] * s0[q][k];
                        s1[q][k] = s0[q][k] = 0.0f;
                    }
                if (a.ggate) store_row<P, float>(a.parts ? a.gate_part : a.ggate, a.parts ? worker : group, lane, TPR, n, g);
                ++group;
                fresh = true;
            }
        }
    }
    // a part without rows (the last group's, cut short by the end of the batch) still has its place among the parts
    if (GROUPED && a.parts && !any && a.ggate && a.f && group * a.gate_rows < a.B) {
        float g[P][8] = {};
        store_row<P, float>(a.gate_part, worker, lane, TPR, n, g);
    }
    if (!a.part) return;
    const auto leave = [&](float (&v)[P][8], int which) {
        float *to = a.part + ((int64_t)blockIdx.x * 4 + which) * n;
        if constexpr (kWorkers > 1) {
            static_assert(P == 1, "rows within a wave");
            __syncthreads();
#pragma unroll
            for (int k = 0; k < 8; ++k) joined[(threadIdx.x / TPR * 8 + k) * TPR + lane] = v[0][k];
            __syncthreads();
            if (threadIdx.x < TPR) {
                float t[8];
#pragma unroll
                for (int k = 0; k < 8; ++k) t[k] = 0.0f;
                for (int w = 0; w < kWorkers; ++w)
#pragma unroll
                    for (int k = 0; k < 8; ++k) t[k] += joined[(w * 8 + k) * TPR + lane];
                store_some(to + lane * 8, n - lane * 8, t);
            }
        } else {
            store_row<P, float>(to, 0, lane, TPR, n, v);
        }
    };
    if (a.gh) {
        leave(pre1, 0);
        leave(pre0, 1);
    }
    if (a.f) {
        leave(GROUPED ? post1 : s1, 2);
        leave(GROUPED ? post0 : s0, 3);
    }
}

template <class X, class F, bool LAYER, int TPR, int P>
hipError_t launch_norm(const NormCall &a, bool backward, bool grouped, int blocks, hipStream_t st)
{
    prof::Timed timed(backward ? "block_norm_backward" : "block_norm_forward", st);
    if (!backward) norm_forward_kernel<X, F, TPR, P, LAYER><<<blocks, threads_of<TPR>(), 0, st>>>(a);
    else if (grouped) norm_backward_kernel<X, F, TPR, P, LAYER, true><<<blocks, threads_of<TPR>(), 0, st>>>(a);
    else norm_backward_kernel<X, F, TPR, P, LAYER, false><<<blocks, threads_of<TPR>(), 0, st>>>(a);
    return hipGetLastError();
}

template <class X, class F, bool LAYER>
hipError_t launch_norm_types(const NormCall &a, bool backward, bool grouped, int blocks, hipStream_t st)
{
    switch (lanes_of_row(a.n)) {
    case 8: return launch_norm<X, F, LAYER, 8, 1>(a, backward, grouped, blocks, st);
    case 16: return launch_norm<X, F, LAYER, 16, 1>(a, backward, grouped, blocks, st);
    case 32: return launch_norm<X, F, LAYER, 32, 1>(a, backward, grouped, blocks, st);
    case 64: return launch_norm<X, F, LAYER, 64, 1>(a, backward, grouped, blocks, st);
    case 128: return launch_norm<X, F, LAYER, 128, 1>(a, backward, grouped, blocks, st);
    case 256: return launch_norm<X, F, LAYER, 256, 1>(a, backward, grouped, blocks, st);
    case 512: return launch_norm<X, F, LAYER, 512, 1>(a, backward, grouped, blocks, st);
    default: break;
    }
    return a.n <= 8192 ? launch_norm<X, F, LAYER, 1024, 1>(a, backward, grouped, blocks, st)
                       : launch_norm<X, F, LAYER, 1024, 2>(a, backward, grouped, blocks, st);
}

// one translation unit for each: the kernels of both passes for these types
hipError_t launch_norm_f32(const NormCall &a, bool layer, bool backward, bool grouped, int blocks, hipStream_t st);
hipError_t launch_norm_bf16_f32(const NormCall &a, bool layer, bool backward, bool grouped, int blocks, hipStream_t st);
hipError_t launch_norm_bf16(const NormCall &a, bool layer, bool backward, bool grouped, int blocks, hipStream_t st);

}  // namespace kannet
