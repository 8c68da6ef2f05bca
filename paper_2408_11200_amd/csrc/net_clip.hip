// The norm of all gradients of a network, and the gradients scaled to it (kan_net.h).
//
// Bound by HBM: the norm needs every element before the first one can be scaled, so the data are read twice and written once.  A launch takes
// up to kMost tensors from its arguments (no table is copied to the device) and goes through the list in chunks of 8192 elements, its
// workgroups side by side: squares are added in 64 bits (a float's square fits exactly, so neither range nor digits are lost), one sum a
// workgroup.  Every workgroup of the scaling launch adds all of these sums in the same order: no launch in between, and one factor for
// all.  It goes from the list's end to its start, where the first pass has been last: what the caches still hold is not read again, and
// what they cannot hold is read past them.  A network that fits eight chunks is one workgroup's work, in one launch.
// The gradients of sixteen layers of 1024 -> 1024 on 20 cells (1.68 GB, fp32): squares 246 us (6.8 TB/s, the rate of a plain read), scaling 620
// (5.4); those of 2 -> 5 -> 1 6.0 us in the one launch.
#include "net_device.hpp"

namespace kannet {
namespace {

constexpr int kMost = 96;                // tensors of a launch
constexpr int kThreads = 256;
constexpr int kChunk = 8192;             // elements of a chunk
constexpr int kSums = 1024;              // of all launches, but one for each launch at least
constexpr int kSmall = 8;                // chunks that one workgroup takes
constexpr double kCached = 192e6;        // bytes of the list's end that are read through the caches

struct ClipCall {
    const void *data[kMost];
    void *out[kMost];
    int64_t count[kMost];
    uint32_t first[kMost + 1];           // chunks of the tensors before
    uint8_t type[kMost];
    double *sums;
    float *norm;
    float max_norm;
    int n, sums_before, sums_all;
    uint32_t stream_until;               // chunks before this one are read past the caches
    bool writes_norm;
};
static_assert(sizeof(ClipCall) <= 4096, "kernel arguments");

// the tensor that has a chunk
__device__ __forceinline__ int tensor_of(const ClipCall &a, uint32_t chunk)
{
    int lo = 0, hi = a.n - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) / 2;
        if (a.first[mid] <= chunk) lo = mid;
        else hi = mid - 1;
    }
    return lo;
}

template <int NT>
__device__ __forceinline__ double block_sum(double v, double *lds)
{
#pragma unroll
    for (int d = 1; d < 64; d *= 2) v += __shfl_xor(v, d, 64);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
    __syncthreads();
    double t = lds[0];
    for (int w = 1; w < NT / 64; ++w) t += lds[w];
    return t;
}

// the elements of a chunk that a thread has, one of NT that share it: `f` gets N values and their place
template <int NT, bool STREAM, class T, class F>
__device__ __forceinline__ void each_piece(const T *p, int count, F f)
{
    constexpr int N = 16 / sizeof(T), AHEAD = kChunk / (N * NT) < 8 ? kChunk / (N * NT) : 8;
    for (int i = threadIdx.x % NT * N; i < count; i += NT * N * AHEAD) {
        Raw<T, N> r[AHEAD];
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) r[u] = raw_at<N, STREAM>(p, i + u * NT * N, count);
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) {
            float v[N];
            settle(r[u], i + u * NT * N, count);
            unpack(r[u], v);
            f(v, i + u * NT * N);
        }
    }
}

template <int NT, bool STREAM, class T>
__device__ __forceinline__ double chunk_squares(const T *p, int count)
{
    double t = 0.0;
    each_piece<NT, STREAM>(p, count, [&](const float(&v)[16 / sizeof(T)], int) {
#pragma unroll
        for (int k = 0; k < 16 / (int)sizeof(T); ++k) t += (double)v[k] * (double)v[k];
    });
    return t;
}

// max_norm / norm as a fraction near 1 and a power of two: the quotient can be below a float's range where the scaled values are not
struct Factor {
    float fraction;
    int exponent;
};

__device__ __forceinline__ float scaled(float v, Factor f) { return __builtin_ldexpf(v * f.fraction, f.exponent); }

template <int NT, class T>
__device__ __forceinline__ void scale_chunk(const T *p, T *to, int count, Factor factor)
{
    each_piece<NT, false>(p, count, [&](float(&v)[16 / sizeof(T)], int i) {
#pragma unroll
        for (int k = 0; k < 16 / (int)sizeof(T); ++k) v[k] = scaled(v[k], factor);
        store_at<16 / sizeof(T), true>(to, i, count, v);
    });
}

// chunk c of the list, or a quarter of it: its tensor, and where in it
struct Place {
    int i, count;
    int64_t at;
};

__device__ __forceinline__ Place place_of(const ClipCall &a, uint32_t c)
{
    Place p;
    p.i = tensor_of(a, c);
    p.at = (int64_t)(c - a.first[p.i]) * kChunk;
    const int64_t left = a.count[p.i] - p.at;
    p.count = left < kChunk ? (int)left : kChunk;
    return p;
}

__device__ __forceinline__ Place quarter_of(const ClipCall &a, uint32_t q)
{
    Place p = place_of(a, q / 4);
    const int from = (int)(q % 4) * (kChunk / 4);
    p.at += from;
    p.count = p.count - from < kChunk / 4 ? p.count - from : kChunk / 4;
    return p;
}

template <int NT, bool STREAM>
__device__ __forceinline__ double squares_at(const ClipCall &a, const Place &p)
{
    return a.type[p.i] == KAN_F32 ? chunk_squares<NT, STREAM>((const float *)a.data[p.i] + p.at, p.count)
                                  : chunk_squares<NT, STREAM>((const bf16 *)a.data[p.i] + p.at, p.count);
}

template <int NT>
__device__ __forceinline__ void scale_at(const ClipCall &a, const Place &p, Factor factor)
{
    if (factor.fraction == 1.0f && factor.exponent == 0 && a.out[p.i] == a.data[p.i]) return;        // in place, and nothing to change
    if (a.type[p.i] == KAN_F32) scale_chunk<NT>((const float *)a.data[p.i] + p.at, (float *)a.out[p.i] + p.at, p.count, factor);
    else scale_chunk<NT>((const bf16 *)a.data[p.i] + p.at, (bf16 *)a.out[p.i] + p.at, p.count, factor);
}

__device__ __forceinline__ Factor factor_of(float norm, float max_norm)
{
    if (!(norm < INFINITY && norm > max_norm)) return Factor{1.0f, 0};
    int most = 0, all = 0;
    const float f = frexpf(max_norm, &most) / frexpf(norm, &all);
    return Factor{f, most - all};
}

__global__ __launch_bounds__(kThreads) void clip_squares_kernel(ClipCall a)
{
    __shared__ double lds[kThreads / 64];
    double t = 0.0;
    for (uint32_t c = blockIdx.x; c < a.first[a.n]; c += gridDim.x) t += c < a.stream_until ? squares_at<kThreads, true>(a, place_of(a, c)) : squares_at<kThreads, false>(a, place_of(a, c));
    t = block_sum<kThreads>(t, lds);
    if (threadIdx.x == 0) a.sums[a.sums_before + blockIdx.x] = t;
}

// one order for every workgroup, so that all have the same bits
__device__ __forceinline__ float norm_of(const ClipCall &a, double *lds)
{
    double t = 0.0;
    for (int i = threadIdx.x; i < a.sums_all; i += kThreads) t += a.sums[i];
    return (float)sqrt(block_sum<kThreads>(t, lds));
}

__global__ __launch_bounds__(kThreads) void clip_scale_kernel(ClipCall a)
{
    __shared__ double lds[kThreads / 64];
    const float norm = norm_of(a, lds);
    if (a.writes_norm && blockIdx.x == 0 && threadIdx.x == 0) *a.norm = norm;
    const Factor factor = factor_of(norm, a.max_norm);
    const uint32_t all = a.first[a.n];
    for (uint32_t c = blockIdx.x; c < all; c += gridDim.x) scale_at<kThreads>(a, place_of(a, all - 1 - c), factor);
}

__global__ __launch_bounds__(kThreads) void clip_norm_kernel(ClipCall a)
{
    __shared__ double lds[kThreads / 64];
    const float norm = norm_of(a, lds);
    if (threadIdx.x == 0) *a.norm = norm;
}

// A wave for each quarter of a chunk, element by element: what counts here is the way to the first value and little code, not bandwidth.
template <class T, class F>
__device__ __forceinline__ void each_element(const T *p, int count, F f)
{
    for (int i = threadIdx.x & 63; i < count; i += 64 * 8) {
        float v[8];
#pragma unroll
        for (int u = 0; u < 8; ++u) v[u] = i + u * 64 < count ? widen(p[i + u * 64]) : 0.0f;
#pragma unroll
        for (int u = 0; u < 8; ++u)
            if (i + u * 64 < count) f(v[u], i + u * 64);
    }
}

__global__ __launch_bounds__(1024) void clip_small_kernel(ClipCall a, bool clip)
{
    __shared__ double lds[16];
    double t = 0.0;
    const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), quarters = 4 * a.first[a.n];
    for (uint32_t q = wave; q < quarters; q += 16) {
        const Place p = quarter_of(a, q);
        const auto square = [&](float v, int) { t += (double)v * (double)v; };
        if (a.type[p.i] == KAN_F32) each_element((const float *)a.data[p.i] + p.at, p.count, square);
        else each_element((const bf16 *)a.data[p.i] + p.at, p.count, square);
    }
    const float norm = (float)sqrt(block_sum<1024>(t, lds));
    if (threadIdx.x == 0) *a.norm = norm;
    if (!clip) return;
    const Factor factor = factor_of(norm, a.max_norm);
    for (uint32_t q = wave; q < quarters; q += 16) {
        const Place p = quarter_of(a, q);
        if (a.type[p.i] == KAN_F32) each_element((const float *)a.data[p.i] + p.at, p.count, [&](float v, int i) { put((float *)a.out[p.i] + p.at + i, scaled(v, factor)); });
        else each_element((const bf16 *)a.data[p.i] + p.at, p.count, [&](float v, int i) { put((bf16 *)a.out[p.i] + p.at + i, scaled(v, factor)); });
    }
}

int launches_of(int n) { return n > 0 ? div_up(n, kMost) : 1; }

int check(int32_t n, const kan_tensor_ref *list, bool outputs)
{
    if (n < 0 || (n > 0 && !list)) return KAN_ERR_INVALID_ARG;
    for (int i = 0; i < n; ++i) {
        const kan_tensor_ref &t = list[i];
        if (!known_type(t.type)) return KAN_ERR_UNSUPPORTED;
        if (t.count < 0) return KAN_ERR_INVALID_ARG;
        if (t.count == 0) continue;
        if (!t.data || misplaced(t.data, t.type) || (outputs && (!t.out || misplaced(t.out, t.type)))) return KAN_ERR_INVALID_ARG;
        if (t.count >= (int64_t)kChunk << 24) return KAN_ERR_UNSUPPORTED;
    }
    return KAN_OK;
}

int run(int32_t n, const kan_tensor_ref *list, float max_norm, bool clip, float *norm, void *ws, size_t ws_bytes, hipStream_t st)
{
    const int rc = check(n, list, clip);
    if (rc != KAN_OK) return rc;
    if (!norm || misplaced(norm, KAN_F32)) return KAN_ERR_INVALID_ARG;
    if (bad_workspace(ws, ws_bytes, kan_clip_workspace_bytes(n))) return KAN_ERR_WORKSPACE;
    const int launches = launches_of(n), most = kSums / launches > 1 ? kSums / launches : 1;
    double bytes = 0.0;
    for (int i = 0; i < n; ++i) bytes += (double)list[i].count * (double)size_of(list[i].type);
    int sums_all = 0;
    for (int phase = 0; phase < 2; ++phase) {
        int before = 0;
        double at = 0.0;
        // the second pass takes the launches from the last one on, too
        for (int k = 0; k < launches; ++k) {
            const int l = phase == 0 ? k : launches - 1 - k;
            ClipCall a = {};
            uint64_t chunks = 0, stream_until = 0;
            for (int i = l * kMost; i < n && i < (l + 1) * kMost; ++i) {
                if (list[i].count == 0) continue;
                a.data[a.n] = list[i].data;
                a.out[a.n] = list[i].out;
                a.count[a.n] = list[i].count;
                a.type[a.n] = (uint8_t)list[i].type;
                const uint64_t here = (uint64_t)div_up(list[i].count, (int64_t)kChunk);
                const double chunk_bytes = (double)kChunk * (double)size_of(list[i].type);
                // whole chunks of this tensor that end before the list's last kCached bytes
                const double before_cached = (bytes - kCached - at) / chunk_bytes;
                if (before_cached > 0.0) stream_until = chunks + (before_cached < (double)here ? (uint64_t)before_cached : here);
                at += (double)list[i].count * (double)size_of(list[i].type);
                chunks += here;
                if (chunks > 0xFFFFFFFFull) return KAN_ERR_UNSUPPORTED;
                a.first[++a.n] = (uint32_t)chunks;
            }
            a.stream_until = (uint32_t)stream_until;
            a.sums = (double *)ws;
            a.norm = norm;
            a.max_norm = max_norm;
            if (launches == 1 && chunks <= kSmall) {
                prof::Timed timed("gradient_clip", st);
                clip_small_kernel<<<1, 1024, 0, st>>>(a, clip);
                return status_of(hipGetLastError());
            }
            const int blocks = chunks < 1 ? 1 : chunks < (uint64_t)most ? (int)chunks : most;
            a.sums_before = before;
            a.sums_all = sums_all;
            a.writes_norm = l == 0;
            before += blocks;
            if (phase == 0) {
                prof::Timed timed("gradient_squares", st);
                clip_squares_kernel<<<blocks, kThreads, 0, st>>>(a);
            } else if (clip) {
                const int wide = chunks < 1 ? 1 : chunks < 2048 ? (int)chunks : 2048;
                prof::Timed timed("gradient_scale", st);
                clip_scale_kernel<<<wide, kThreads, 0, st>>>(a);
            } else if (l == 0) {
                prof::Timed timed("gradient_norm", st);
                clip_norm_kernel<<<1, kThreads, 0, st>>>(a);
            }
            if (hipGetLastError() != hipSuccess) return KAN_ERR_HIP;
        }
        sums_all = before;
    }
    return KAN_OK;
}

}  // namespace
}  // namespace kannet

using namespace kannet;

extern "C" size_t kan_clip_workspace_bytes(int32_t n)
{
    if (n < 0) return 0;
    const int launches = launches_of(n);
    return align_up((size_t)(launches > kSums ? launches : kSums) * sizeof(double));
}

extern "C" int kan_gradient_norm(int32_t n, const kan_tensor_ref *list, float *norm, void *ws, size_t ws_bytes, void *stream)
{
    return run(n, list, 0.0f, false, norm, ws, ws_bytes, (hipStream_t)stream);
}

extern "C" int kan_clip_gradients(int32_t n, const kan_tensor_ref *list, float max_norm, float *norm, void *ws, size_t ws_bytes, void *stream)
{
    if (!(max_norm >= 0.0f) || max_norm > 3.4028234663852886e38f) return KAN_ERR_INVALID_ARG;
    return run(n, list, max_norm, true, norm, ws, ws_bytes, (hipStream_t)stream);
}
