// Kernels of the norms at a block boundary (kan_net.h), one instance for each pair of types and kind of norm.
//
// Both passes are bound by HBM: a row is read into registers once (eight channels a lane and piece, TPR lanes a row), and everything that
// needs the whole row (mean, mean square, the two projections of the backward pass) is a sum over those lanes.  Workers are the groups of
// TPR lanes; rows of up to 512 channels lie within a wave, so that their sums are DPP moves and need no barrier.  Forward and backward, us and
// TB/s of what a pass has to move: 16384 x 512 fp32 layer norm 23.0-25.7 (5.8-5.2) and 39.1 (5.1); 8190 x 771 bf16 stream and fp32 branch, a gate each
// 117 rows, 21.8 (3.5) and 32.4 (3.5); 16384 x 4096 bf16 RMS norm 100.5 (5.3) and 149 (5.4); 5461 x 6144 fp32 layer norm 116 (4.6) and 157 (5.1).
#pragma once
#include <atomic>
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
    int n, lanes;           // lanes of a row: those of its waves that reach it
    float eps, residual_scale, inv_n;
};

// threads of a workgroup: the forward pass has one worker where rows take several waves; the backward pass joins the parameters' sums of
// as many workers as 512 threads hold
template <int TPR>
constexpr int forward_threads() { return TPR > 64 ? TPR : 256; }
template <int TPR>
constexpr int backward_threads() { return TPR > 512 ? TPR : 512; }

// Waves wholly behind a row's end are not launched, where there can be any: bf16 forward, 27962 x 1200 layer norm 83 us with 256 lanes, 69-72 with 192, RMS norm
// 53 and 47; 13421 x 2500 90 with 512, 73 with 320, and 58 and 55; fp32 22369 x 1500 90.3 and 89.9.  The backward pass has one workgroup a CU whichever, and gains with
// 768 lanes (7456 x 4500 119 us, 101 with 576); 1024 have no register left for it.
template <int TPR>
constexpr bool kForwardTrims = TPR > 128 && TPR < 1024;
template <int TPR>
constexpr bool kBackwardTrims = TPR == 768;

// Parameters and their sums are fp32 whatever the rows are: where those have eight channels side by side a lane, two accesses
template <bool PAIR>
__device__ __forceinline__ void load_param_eight(const float *w, int base, int lane, int lanes, int n, float (&v)[8])
{
    if constexpr (PAIR) {
        load_eight<true>(w, base, lane, lanes, n, v);
    } else {
        const int c = base + 8 * lane;
        Raw<float, 4> a = raw_at<4>(w, c, n), b = raw_at<4>(w, c + 4, n);
        settle(a, c, n);
        settle(b, c + 4, n);
        unpack(a, v);
        unpack(b, v + 4);
    }
}

template <bool PAIR>
__device__ __forceinline__ void store_param_eight(float *w, int base, int lane, int lanes, int n, const float (&v)[8])
{
    if constexpr (PAIR) {
        store_eight<true>(w, base, lane, lanes, n, v);
    } else {
        store_at<4>(w, base + 8 * lane, n, v);
        store_at<4>(w, base + 8 * lane + 4, n, v + 4);
    }
}

template <int P, bool PAIR>
__device__ __forceinline__ void store_param(float *w, int lane, int tpr, int n, const float (&v)[P][8])
{
#pragma unroll
    for (int q = 0; q < P; ++q) store_param_eight<PAIR>(w, q * tpr * 8, lane, tpr, n, v[q]);
}

// `none` where there is no such parameter; 0 past the row's end in either case
template <int P, bool PAIR>
__device__ __forceinline__ void load_param(const float *w, int lane, int tpr, int n, float none, float (&v)[P][8])
{
#pragma unroll
    for (int q = 0; q < P; ++q) {
        if (w) {
            load_param_eight<PAIR>(w, q * tpr * 8, lane, tpr, n, v[q]);
        } else {
#pragma unroll
            for (int k = 0; k < 8; ++k) v[q][k] = channel_of<PAIR>(q * tpr * 8, lane, tpr, k) < n ? none : 0.0f;
        }
    }
}

// Past the caches where it is written once and read by other launches: of 16384 x 4096 bf16 the backward pass took 151 us with such stores and
// 171 without, of 16384 x 512 fp32 the forward pass 25 and 30.  (Such loads cost more than they gave: x and f are read by both passes.)
template <int P, bool PAIR, class T>
__device__ __forceinline__ void store_row(void *base, int64_t row, int lane, int tpr, int n, const float (&v)[P][8])
{
#pragma unroll
    for (int q = 0; q < P; ++q) store_eight<PAIR, true>((T *)base + row * n, q * tpr * 8, lane, tpr, n, v[q]);
}

// Rows of the largest and the smallest values keep their digits, and the others their instructions: a mean's sum is taken times 2^-20, the centred
// values by half (so neither overflows; powers of two change no digit), and a row whose sum of squares overflows, or whose variance with eps is below
// kLeast (where squares that count would lose digits), has its sums taken once more of values times 2^-80 or 2^80.
constexpr float kDown = 0x1p-80f, kUp = 0x1p80f, kLeast = 0x1p-90f;

// n as a value the compiler knows nothing of, for the layer norm of bf16 streams: the masks of a row's end are made for each row, where all of them, kept
// over the rows, do not fit the scalar registers and are fetched from lanes of vector registers (32768 x 200 bf16 forward 18.1 us, 14.1 so; 8190 x 771 in
// two types 20.0 and 18.9).  Others lose by it: bf16 rows of whole waves, 13421 x 2500 73 and 76, rows in two types within a wave, 280360 x 82 58 and 62.
__device__ __forceinline__ int afresh(int n)
{
    asm volatile("" : "+s"(n));
    return n;
}

// half of v - mean
__device__ __forceinline__ float half_centred(float v, float half_mean) { return __builtin_fmaf(v, 0.5f, -half_mean); }

// v becomes norm(v); mean and 1/sigma.  What it leaves in channels past the row's end counts nowhere: parameters are 0 there (load_param).  The variance is that of the centred values: the mean of the
// squares less the squared mean would lose all digits where the mean is large.  What the mean's own rounding left in the centred values
// is their mean, from the same sums as the variance.
template <int TPR, int P, bool PAIR, bool LAYER>
__device__ __forceinline__ void normalise(float (&v)[P][8], int lane, int lanes, int n, float inv_n, float eps, RowSum<TPR> &total, float &mean, float &r)
{
    float s[2] = {0.0f, 0.0f}, half_mean = 0.0f;
    if constexpr (LAYER) {
#pragma unroll
        for (int q = 0; q < P; ++q)
#pragma unroll
            for (int k = 0; k < 8; ++k) s[1] = __builtin_fmaf(v[q][k], 0x1p-20f, s[1]);
        half_mean = total(s[1]) * inv_n * 0x1p19f;
        s[1] = 0.0f;
    }
#pragma unroll
    for (int q = 0; q < P; ++q)
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            if (LAYER) {
                v[q][k] = channel_of<PAIR>(q * TPR * 8, lane, lanes, k) < n ? half_centred(v[q][k], half_mean) : 0.0f;
                s[1] += v[q][k];
            }
            s[0] += v[q][k] * v[q][k];
        }
    const auto join = [&] {
        if constexpr (LAYER) total.sum(s);
        else s[0] = total(s[0]);
    };
    // of what is in v: for a layer norm a quarter of the row's
    const auto variance = [&] { return LAYER ? fmaxf(s[0] * inv_n - s[1] * inv_n * (s[1] * inv_n), 0.0f) : s[0] * inv_n; };
    constexpr float kPart = LAYER ? 0.25f : 1.0f;
    join();
    const float square = variance() + kPart * eps;
    float rest = s[1] * inv_n, rs = 1.0f / sqrtf(square);
    // for a whole wave, and with it all waves of a row, whose sums have the same bits; the wave's other rows keep what they have
    if (__ballot(!(s[0] < INFINITY) || square < kLeast)) {
        const float scale = !(s[0] < INFINITY) ? kDown : square < kLeast ? kUp : 1.0f;
        s[0] = s[1] = 0.0f;
#pragma unroll
        for (int q = 0; q < P; ++q)
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                float c = v[q][k] * scale;
                if (P > 1) asm volatile("" : "+v"(c), "+v"(s[0]), "+v"(s[1]));        // one after the other: two pieces leave no registers for many at once
                if (LAYER) s[1] += c;
                s[0] += c * c;
            }
        join();
        total(0.0f);            // the sets of slots are taken in turn: an even number of sums here
        if (TPR >= 64 || scale != 1.0f) {
            rest = s[1] * inv_n / scale;
            rs = 1.0f / sqrtf(variance() + eps * scale * (kPart * scale)) * scale;
        }
    }
    r = LAYER ? 0.5f * rs : rs;
    mean = LAYER ? 2.0f * (half_mean + rest) : 0.0f;
#pragma unroll
    for (int q = 0; q < P; ++q)
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            v[q][k] = LAYER ? (v[q][k] - rest) * rs : v[q][k] * rs;
        }
}

// Waves a SIMD that the registers have to leave room for, of bf16 rows: their layer norm takes 10 to 30 % longer with four
template <class X, class F, int TPR>
constexpr int forward_waves() { return sizeof(X) == 2 && sizeof(F) == 2 && TPR < 1024 ? 5 : 1; }

template <class X, class F, int TPR, int P, bool LAYER>
__global__ __launch_bounds__(forward_threads<TPR>(), (forward_waves<X, F, TPR>())) void norm_forward_kernel(NormCall a)
{
    constexpr int kWorkers = forward_threads<TPR>() / TPR;
    constexpr bool PAIR = is_float<X> || is_float<F>;
    __shared__ float slots[RowSum<TPR>::kSlots];
    RowSum<TPR> total{slots};
    const int lanes = kForwardTrims<TPR> ? a.lanes : TPR, lane = threadIdx.x % TPR, n = a.n;
    total.clear(lane);
    const int64_t step = (int64_t)gridDim.x * kWorkers;
    float w_post[P][8], b_post[P][8], gate[P][8], w_pre[P][8], b_pre[P][8];
    load_param<P, PAIR>(a.p.w_pre, lane, lanes, n, 1.0f, w_pre);
    load_param<P, PAIR>(a.p.b_pre, lane, lanes, n, 0.0f, b_pre);
    load_param<P, PAIR>(a.f ? a.p.w_post : nullptr, lane, lanes, n, 1.0f, w_post);
    load_param<P, PAIR>(a.f ? a.p.b_post : nullptr, lane, lanes, n, 0.0f, b_post);
    load_param<P, PAIR>(a.f && !a.gate_rows ? a.p.gate : nullptr, lane, lanes, n, 1.0f, gate);
    // the wave's first row, in scalar registers, and which of its rows the lane has
    int64_t first = (int64_t)blockIdx.x * kWorkers + (TPR <= 64 ? __builtin_amdgcn_readfirstlane(threadIdx.x / 64) * (64 / (TPR < 64 ? TPR : 64)) : 0);
    const int sub = TPR < 64 ? threadIdx.x % 64 / TPR : 0;
    Eight<X, PAIR> next_x[P];
    Eight<F, PAIR> next_f[P];
    const auto read_ahead = [&](int64_t r) {
#pragma unroll
        for (int q = 0; q < P; ++q) {
            const int m = r < a.B ? n : 0;
            next_x[q] = eight_at<PAIR>((const X *)a.x + r * n, q * TPR * 8, lane, lanes, m);
            next_f[q] = eight_at<PAIR>((const F *)a.f + r * n, q * TPR * 8, lane, lanes, a.f ? m : 0);
        }
    };
    read_ahead(first + sub);
    for (; first + sub < a.B; first += step) {
        const int64_t row = first + sub;
        const int n = LAYER && sizeof(X) == 2 && (sizeof(F) == 2) == (TPR < 64) ? afresh(a.n) : a.n;
        float v[P][8], u[P][8], st[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int q = 0; q < P; ++q) {
            unpack_at<PAIR>(next_x[q], q * TPR * 8, lane, lanes, n, v[q]);
            unpack_at<PAIR>(next_f[q], q * TPR * 8, lane, lanes, n, u[q]);
        }
        read_ahead(row + step);
        if (a.f) {
            if (a.gate_rows && a.p.gate) load_param<P, PAIR>(a.p.gate + row / a.gate_rows * n, lane, lanes, n, 1.0f, gate);
            normalise<TPR, P, PAIR, LAYER>(u, lane, lanes, n, a.inv_n, a.eps, total, st[0], st[1]);
#pragma unroll
            for (int q = 0; q < P; ++q)
#pragma unroll
                for (int k = 0; k < 8; ++k) v[q][k] = a.residual_scale * v[q][k] + gate[q][k] * (u[q][k] * w_post[q][k] + b_post[q][k]);
            store_row<P, PAIR, X>(a.x_out, row, lane, lanes, n, v);
        }
        if (a.h) {
            normalise<TPR, P, PAIR, LAYER>(v, lane, lanes, n, a.inv_n, a.eps, total, st[2], st[3]);
#pragma unroll
            for (int q = 0; q < P; ++q)
#pragma unroll
                for (int k = 0; k < 8; ++k) v[q][k] = v[q][k] * w_pre[q][k] + b_pre[q][k];
            store_row<P, PAIR, F>(a.h, row, lane, lanes, n, v);
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

// A worker's rows of the backward pass as they lie in memory, read while the rows before are worked on
template <class X, class F, int P>
struct RowsAhead {
    static constexpr bool PAIR = is_float<X> || is_float<F>;
    Eight<X, PAIR> x[P], gx_out[P];
    Eight<F, PAIR> f[P], gh[P];
    float st[4];
};

template <class X, class F, int TPR, int P, bool LATE>
__device__ __forceinline__ void read_ahead(RowsAhead<X, F, P> &r, const NormCall &a, int64_t row, bool live, int lane, int lanes)
{
    constexpr bool PAIR = RowsAhead<X, F, P>::PAIR;
    const int n = live ? a.n : 0;
    const int64_t at = row * a.n;
#pragma unroll
    for (int q = 0; q < P; ++q) {
        const int base = q * TPR * 8;
        r.x[q] = eight_at<PAIR>((const X *)a.x + at, base, lane, lanes, n);
        r.f[q] = eight_at<PAIR>((const F *)a.f + at, base, lane, lanes, a.f ? n : 0);
        if (!LATE) r.gx_out[q] = eight_at<PAIR>((const X *)a.gx_out + at, base, lane, lanes, a.gx_out ? n : 0);
        r.gh[q] = eight_at<PAIR>((const F *)a.gh + at, base, lane, lanes, a.gh ? n : 0);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) r.st[i] = live ? a.stats[row * 4 + i] : 0.0f;
}

// Gradients of the rows, and of the parameters summed over a worker's rows (consecutive ones).
//
// WHOLE false: all rows of a worker share a gate row (the only one, or that of the group the worker has a part of).  Gate, w_post and b_post
// are then common factors of the sums of d and d * norm(f), put in at the end: here for a part of a group, when the workgroups' sums are
// added for a gate that all rows share.  WHOLE true: a worker has whole groups, and writes a group's gate gradient at its end.
// BIAS false: nobody asks for the gradient of a bias, and none is in the way of the gate's; their sums are left out.
template <class X, class F, int TPR, int P, bool LAYER, bool WHOLE, bool BIAS>
__global__ __launch_bounds__(backward_threads<TPR>()) void norm_backward_kernel(NormCall a)
{
    constexpr int NT = backward_threads<TPR>(), kWorkers = NT / TPR;
    constexpr bool PAIR = is_float<X> || is_float<F>;
    constexpr bool kTight = TPR == 768 && sizeof(F) == 4 && (WHOLE || BIAS), kLate = TPR == 1024 || kTight;
    __shared__ float slots[RowSum<TPR>::kSlots * (TPR > 64 ? kWorkers : 1)];
    constexpr int kJoin = TPR < 64 ? NT / 64 : kWorkers;       // workers of one wave are joined by shuffles first
    __shared__ float joined[kWorkers > 1 ? kJoin * TPR * 8 : 1];
    const int lanes = kBackwardTrims<TPR> ? a.lanes : TPR, here = threadIdx.x / lanes, lane = threadIdx.x - here * lanes, n = a.n;
    RowSum<TPR> total{slots + (TPR > 64 ? here * RowSum<TPR>::kSlots : 0)};
    total.clear(lane);
    const int64_t worker = (int64_t)blockIdx.x * kWorkers + here;
    int64_t row, end, group = 0;
    if (a.parts) {
        group = worker / a.parts;
        row = group * a.gate_rows + worker % a.parts * a.span;
        end = row + a.span < (group + 1) * a.gate_rows ? row + a.span : (group + 1) * a.gate_rows;
    } else {
        row = worker * a.span;
        end = row + a.span;
        if (WHOLE) group = row / a.gate_rows;
    }
    if (end > a.B) end = a.B;
    const bool there = row < a.B;
    const float *gate_row = a.f && a.p.gate && there ? a.p.gate + group * n : nullptr;

    // gate * w_post and gate * b_post; gate and the other two by themselves where the gate changes on the way
    float w_pre[P][8], w_post[P][8], b_post[P][8], gate[P][8];
    load_param<P, PAIR>(a.p.w_pre, lane, lanes, n, 1.0f, w_pre);
    load_param<P, PAIR>(a.f ? a.p.w_post : nullptr, lane, lanes, n, 1.0f, w_post);
    load_param<P, PAIR>(a.f && BIAS ? a.p.b_post : nullptr, lane, lanes, n, 0.0f, b_post);
    load_param<P, PAIR>(gate_row, lane, lanes, n, 1.0f, gate);
    if (!WHOLE)
#pragma unroll
        for (int q = 0; q < P; ++q)
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                w_post[q][k] *= gate[q][k];
                b_post[q][k] *= gate[q][k];
            }
    // 1024 threads have 128 registers each, 768 have 168: the parameters wait in LDS, each lane's own, until they are needed.  Layer norm with
    // biases in fp32, us with what does not fit in scratch and so: 4096 x 8192 234 and 174, 5461 x 6144 with a gate each row 405 and 233.  RMS norm
    // without biases 164 and 155, but of a bf16 stream 110 and 115: there they stay.
    constexpr bool kAside = P == 1 && ((TPR == 1024 && (LAYER || WHOLE || BIAS || sizeof(X) == 4)) || kTight);
    __shared__ f32x4 aside[kAside ? 6 : 1][kAside ? TPR : 1];
    const auto put_aside = [&](int which, const float (&v)[P][8]) {
        aside[2 * which][threadIdx.x] = f32x4{v[0][0], v[0][1], v[0][2], v[0][3]};
        aside[2 * which + 1][threadIdx.x] = f32x4{v[0][4], v[0][5], v[0][6], v[0][7]};
    };
    const auto fetch = [&](int which, float (&v)[P][8]) {
        if constexpr (kAside) {
            const f32x4 lo = aside[2 * which][threadIdx.x], hi = aside[2 * which + 1][threadIdx.x];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                v[0][k] = lo[k];
                v[0][4 + k] = hi[k];
            }
        }
    };
    if constexpr (kAside) {
        put_aside(0, w_pre);
        put_aside(1, w_post);
        if (BIAS) put_aside(2, b_post);
    }
    // of w_pre and b_pre; of w_post and b_post, without their common factors if not WHOLE; of the gate of a group if WHOLE
    float pre1[P][8] = {}, pre0[P][8] = {}, post1[P][8] = {}, post0[P][8] = {}, gates[P][8] = {};
    RowsAhead<X, F, P> next;
    read_ahead<X, F, TPR, P, kLate>(next, a, row, row < end, lane, lanes);
    // workers of several waves share their barriers: each goes through all rounds
    for (int64_t i = 0; i < a.span; ++i, ++row) {
        const bool live = row < end;
        if (TPR <= 64 && !live) break;
        // out of the registers the next row is read into
        const float half_mean_f = 0.5f * next.st[0], r_f = next.st[1], half_mean_x = 0.5f * next.st[2], r_x = next.st[3];
        float v[P][8], fhat[P][8], d[P][8], g[P][8];
        Eight<X, PAIR> gx_out[P];
#pragma unroll
        for (int q = 0; q < P; ++q) {
            unpack_at<PAIR>(next.x[q], q * TPR * 8, lane, lanes, n, v[q]);
            unpack_at<PAIR>(next.f[q], q * TPR * 8, lane, lanes, n, fhat[q]);
            unpack_at<PAIR>(next.gh[q], q * TPR * 8, lane, lanes, n, g[q]);
            // with few registers a lane it is read now; it is needed behind the first sum
            if (!kLate) gx_out[q] = next.gx_out[q];
            else gx_out[q] = eight_at<PAIR>((const X *)a.gx_out + row * n, q * TPR * 8, lane, lanes, a.gx_out && live ? n : 0);
        }
        read_ahead<X, F, TPR, P, kLate>(next, a, row + 1, row + 1 < end, lane, lanes);
        if (a.f) {
            fetch(1, w_post);
            if (BIAS) fetch(2, b_post);
#pragma unroll
            for (int q = 0; q < P; ++q)
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    const bool in = channel_of<PAIR>(q * TPR * 8, lane, lanes, k) < n;
                    fhat[q][k] = !LAYER ? fhat[q][k] * r_f : in ? half_centred(fhat[q][k], half_mean_f) * (2.0f * r_f) : 0.0f;
                    const float u = fhat[q][k] * w_post[q][k] + b_post[q][k];
                    v[q][k] = a.residual_scale * v[q][k] + (WHOLE ? gate[q][k] * u : u);
                }
        }
        if (a.gh) {
            fetch(0, w_pre);
#pragma unroll
            for (int q = 0; q < P; ++q)
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    const bool in = channel_of<PAIR>(q * TPR * 8, lane, lanes, k) < n;
                    v[q][k] = !LAYER ? v[q][k] * r_x : in ? half_centred(v[q][k], half_mean_x) * (2.0f * r_x) : 0.0f;
                    pre1[q][k] += g[q][k] * v[q][k];
                    if (BIAS) pre0[q][k] += g[q][k];
                    g[q][k] *= w_pre[q][k];
                }
            norm_back<TPR, P, LAYER>(g, v, r_x, a.inv_n, total);
        }
#pragma unroll
        for (int q = 0; q < P; ++q) {
            unpack_at<PAIR>(gx_out[q], q * TPR * 8, lane, lanes, n, d[q]);
#pragma unroll
            for (int k = 0; k < 8; ++k) d[q][k] += g[q][k];        // without gh: zeros
        }
        if (a.gx && live) {
            const float scale = a.f ? a.residual_scale : 1.0f;
#pragma unroll
            for (int q = 0; q < P; ++q)
#pragma unroll
                for (int k = 0; k < 8; ++k) g[q][k] = scale * d[q][k];
            store_row<P, PAIR, X>(a.gx, row, lane, lanes, n, g);
        }
        if (a.f) {
            fetch(1, w_post);
            if (WHOLE && BIAS) fetch(2, b_post);
#pragma unroll
            for (int q = 0; q < P; ++q)
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    const bool in = !LAYER || channel_of<PAIR>(q * TPR * 8, lane, lanes, k) < n;
                    float gu = d[q][k];
                    if (WHOLE) {
                        gates[q][k] += gu * (fhat[q][k] * w_post[q][k] + b_post[q][k]);
                        gu *= gate[q][k];
                    }
                    post1[q][k] += gu * fhat[q][k];
                    if (BIAS) post0[q][k] += gu;
                    d[q][k] = in ? gu * w_post[q][k] : 0.0f;
                }
            if (a.gf) {
                norm_back<TPR, P, LAYER>(d, fhat, r_f, a.inv_n, total);
                if (live) store_row<P, PAIR, F>(a.gf, row, lane, lanes, n, d);
            }
            if (WHOLE && live && (row + 1 == end || (row + 1) % a.gate_rows == 0)) {
                if (a.ggate) store_param<P, PAIR>(a.ggate + group * n, lane, lanes, n, gates);
                ++group;
#pragma unroll
                for (int q = 0; q < P; ++q)
#pragma unroll
                    for (int k = 0; k < 8; ++k) gates[q][k] = 0.0f;
                if (a.p.gate && row + 1 < end) load_param<P, PAIR>(a.p.gate + group * n, lane, lanes, n, 1.0f, gate);
            }
        }
    }
    if (!a.part) return;
    if (a.parts && a.f) {
        // a part of a group: its share of the gate's gradient, and the gate's factor of the others
        load_param<P, PAIR>(a.p.w_post, lane, lanes, n, 1.0f, w_post);
        load_param<P, PAIR>(BIAS ? a.p.b_post : nullptr, lane, lanes, n, 0.0f, b_post);
        load_param<P, PAIR>(gate_row, lane, lanes, n, 1.0f, gate);
#pragma unroll
        for (int q = 0; q < P; ++q)
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                gates[q][k] = post1[q][k] * w_post[q][k] + post0[q][k] * b_post[q][k];
                post1[q][k] *= gate[q][k];
                post0[q][k] *= gate[q][k];
            }
        if (a.ggate && group * a.gate_rows < a.B) store_param<P, PAIR>(a.gate_part + worker * n, lane, lanes, n, gates);
    }
    const auto leave = [&](float (&v)[P][8], int which) {
        float *to = a.part + ((int64_t)blockIdx.x * 4 + which) * n;
        if constexpr (kWorkers > 1) {
            static_assert(P == 1, "one piece a lane");
            for (int by = TPR; by < 64; by *= 2)
#pragma unroll
                for (int k = 0; k < 8; ++k) v[0][k] += __shfl_xor(v[0][k], by, 64);
            __syncthreads();
            const int part = TPR < 64 ? threadIdx.x / 64 : here;
            if (threadIdx.x % 64 < TPR)
#pragma unroll
                for (int k = 0; k < 8; ++k) joined[(part * 8 + k) * TPR + lane] = v[0][k];
            __syncthreads();
            if ((int)threadIdx.x < lanes) {
                float t[8];
#pragma unroll
                for (int k = 0; k < 8; ++k) t[k] = 0.0f;
                for (int w = 0; w < kJoin; ++w)
#pragma unroll
                    for (int k = 0; k < 8; ++k) t[k] += joined[(w * 8 + k) * TPR + lane];
                store_param_eight<PAIR>(to, 0, lane, lanes, n, t);
            }
        } else {
            store_param<P, PAIR>(to, lane, lanes, n, v);
        }
    };
    if (a.gh) {
        leave(pre1, 0);
        if (BIAS) leave(pre0, 1);
    }
    if (a.f) {
        leave(post1, 2);
        if (BIAS) leave(post0, 3);
    }
}

// Workgroups of a kernel that a CU holds at once, asked for once for each size: that many take the forward pass's rows in turn, so that all end
// together (1024 or 2048 of them, whatever fits: 22369 x 1500 bf16 RMS norm 61 us, 55 so).
template <void (*KERNEL)(NormCall)>
int resident_blocks(int threads)
{
    static std::atomic<int> known[17];
    std::atomic<int> &there = known[threads / 64];
    int blocks = there.load(std::memory_order_relaxed);
    if (blocks == 0) {
        if (hipOccupancyMaxActiveBlocksPerMultiprocessor(&blocks, (const void *)KERNEL, threads, 0) != hipSuccess || blocks < 1) blocks = 1;
        there.store(blocks, std::memory_order_relaxed);
    }
    return blocks;
}

// which kernel a call takes
struct NormPick {
    bool layer, backward, whole, bias;
    int blocks;
};

template <class X, class F, bool LAYER, int TPR, int P>
hipError_t launch_norm(const NormCall &a, const NormPick &p, hipStream_t st)
{
    prof::Timed timed(p.backward ? "block_norm_backward" : "block_norm_forward", st);
    const int NT = kBackwardTrims<TPR> ? a.lanes : backward_threads<TPR>();
    if (!p.backward) {
        const int threads = kForwardTrims<TPR> ? a.lanes : forward_threads<TPR>();
        const int64_t most = 256ll * resident_blocks<norm_forward_kernel<X, F, TPR, P, LAYER>>(threads), blocks = p.blocks < most ? p.blocks : most;
        norm_forward_kernel<X, F, TPR, P, LAYER><<<(unsigned)blocks, threads, 0, st>>>(a);
    }
    else if (p.whole && p.bias) norm_backward_kernel<X, F, TPR, P, LAYER, true, true><<<p.blocks, NT, 0, st>>>(a);
    else if (p.whole) norm_backward_kernel<X, F, TPR, P, LAYER, true, false><<<p.blocks, NT, 0, st>>>(a);
    else if (p.bias) norm_backward_kernel<X, F, TPR, P, LAYER, false, true><<<p.blocks, NT, 0, st>>>(a);
    else norm_backward_kernel<X, F, TPR, P, LAYER, false, false><<<p.blocks, NT, 0, st>>>(a);
    return hipGetLastError();
}

template <class X, class F, bool LAYER>
hipError_t launch_norm_types(const NormCall &a, const NormPick &p, hipStream_t st)
{
    switch (lanes_of_row(a.n)) {
    case 8: return launch_norm<X, F, LAYER, 8, 1>(a, p, st);
    case 16: return launch_norm<X, F, LAYER, 16, 1>(a, p, st);
    case 32: return launch_norm<X, F, LAYER, 32, 1>(a, p, st);
    case 64: return launch_norm<X, F, LAYER, 64, 1>(a, p, st);
    case 128: return launch_norm<X, F, LAYER, 128, 1>(a, p, st);
    case 256: return launch_norm<X, F, LAYER, 256, 1>(a, p, st);
    case 512: return launch_norm<X, F, LAYER, 512, 1>(a, p, st);
    case 768: return launch_norm<X, F, LAYER, 768, 1>(a, p, st);
    default: break;
    }
    return a.n <= 8192 ? launch_norm<X, F, LAYER, 1024, 1>(a, p, st) : launch_norm<X, F, LAYER, 1024, 2>(a, p, st);
}

// one translation unit for each: the kernels of both passes for these types
hipError_t launch_norm_f32(const NormCall &a, const NormPick &p, hipStream_t st);
hipError_t launch_norm_bf16_f32(const NormCall &a, const NormPick &p, hipStream_t st);
hipError_t launch_norm_bf16(const NormCall &a, const NormPick &p, hipStream_t st);

}  // namespace kannet
