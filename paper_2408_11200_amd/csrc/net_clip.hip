// The norm of all gradients of a network, and the gradients scaled to it (kan_net.h).
//
// Bound by HBM: the norm needs every element before the first one can be scaled, so the data are read twice and written once.  A launch takes
// up to kMost tensors from its arguments (no table is copied to the device); its workgroups have consecutive chunks of the list, add squares
// in 64 bits (a float's square fits exactly, so neither range nor digits are lost) and leave one sum each.  Every workgroup of the
// scaling launch adds all of these sums in the same order: no launch in between, and one factor for all.
#include "net_device.hpp"

namespace kannet {
namespace {

constexpr int kMost = 96;                // tensors of a launch
constexpr int kThreads = 256;
constexpr int kChunk = 8192;             // elements of a chunk
constexpr int kSums = 1024;              // of all launches, but one for each launch at least

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
    bool writes_norm;
};
static_assert(sizeof(ClipCall) <= 4096, "kernel arguments");

// chunks of a workgroup
__device__ __forceinline__ void share(const ClipCall &a, uint32_t &chunk, uint32_t &end)
{
    const uint64_t all = a.first[a.n];
    chunk = (uint32_t)(all * blockIdx.x / gridDim.x);
    end = (uint32_t)(all * (blockIdx.x + 1) / gridDim.x);
}

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

template <class T>
__device__ __forceinline__ double chunk_squares(const T *p, int count)
{
    constexpr int N = 16 / sizeof(T);
    double t = 0.0;
    for (int i = threadIdx.x * N; i < count; i += kThreads * N) {
        float v[N];
        Raw<T, N> r = raw_at<N>(p, i, count);
        settle(r, i, count);
        unpack(r, v);
#pragma unroll
        for (int k = 0; k < N; ++k) t += (double)v[k] * (double)v[k];
    }
    return t;
}

__global__ __launch_bounds__(kThreads) void clip_squares_kernel(ClipCall a)
{
    __shared__ double lds[kThreads / 64];
    uint32_t chunk, end;
    share(a, chunk, end);
    double t = 0.0;
    int i = chunk < end ? tensor_of(a, chunk) : 0;
    for (; chunk < end; ++chunk) {
        while (chunk >= a.first[i + 1]) ++i;
        const int64_t at = (int64_t)(chunk - a.first[i]) * kChunk, left = a.count[i] - at;
        const int count = left < kChunk ? (int)left : kChunk;
        t += a.type[i] == KAN_F32 ? chunk_squares((const float *)a.data[i] + at, count) : chunk_squares((const bf16 *)a.data[i] + at, count);
    }
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

template <class T>
__device__ __forceinline__ void scale_chunk(const T *p, T *to, int count, float factor)
{
    constexpr int N = 16 / sizeof(T);
    for (int i = threadIdx.x * N; i < count; i += kThreads * N) {
        float v[N];
        Raw<T, N> r = raw_at<N>(p, i, count);
        settle(r, i, count);
        unpack(r, v);
#pragma unroll
        for (int k = 0; k < N; ++k) v[k] *= factor;
        store_at<N>(to, i, count, v);
    }
}

__global__ __launch_bounds__(kThreads) void clip_scale_kernel(ClipCall a)
{
    __shared__ double lds[kThreads / 64];
    const float norm = norm_of(a, lds);
    if (a.writes_norm && blockIdx.x == 0 && threadIdx.x == 0) *a.norm = norm;
    const bool finite = norm < INFINITY;
    const float factor = finite && norm > a.max_norm ? a.max_norm / norm : 1.0f;
    uint32_t chunk, end;
    share(a, chunk, end);
    int i = chunk < end ? tensor_of(a, chunk) : 0;
    for (; chunk < end; ++chunk) {
        while (chunk >= a.first[i + 1]) ++i;
        if (factor == 1.0f && a.out[i] == a.data[i]) continue;        // in place, and nothing to change
        const int64_t at = (int64_t)(chunk - a.first[i]) * kChunk, left = a.count[i] - at;
        const int count = left < kChunk ? (int)left : kChunk;
        if (a.type[i] == KAN_F32) scale_chunk((const float *)a.data[i] + at, (float *)a.out[i] + at, count, factor);
        else scale_chunk((const bf16 *)a.data[i] + at, (bf16 *)a.out[i] + at, count, factor);
    }
}

__global__ __launch_bounds__(kThreads) void clip_norm_kernel(ClipCall a)
{
    __shared__ double lds[kThreads / 64];
    const float norm = norm_of(a, lds);
    if (threadIdx.x == 0) *a.norm = norm;
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
    int sums_all = 0;
    for (int phase = 0; phase < 2; ++phase) {
        int before = 0;
        for (int l = 0; l < launches; ++l) {
            ClipCall a = {};
            uint64_t chunks = 0;
            for (int i = l * kMost; i < n && i < (l + 1) * kMost; ++i) {
                if (list[i].count == 0) continue;
                a.data[a.n] = list[i].data;
                a.out[a.n] = list[i].out;
                a.count[a.n] = list[i].count;
                a.type[a.n] = (uint8_t)list[i].type;
                chunks += (uint64_t)div_up(list[i].count, (int64_t)kChunk);
                a.first[++a.n] = (uint32_t)chunks;
            }
            const int blocks = chunks < 1 ? 1 : chunks < (uint64_t)most ? (int)chunks : most;
            a.sums = (double *)ws;
            a.norm = norm;
            a.max_norm = max_norm;
            a.sums_before = before;
            a.sums_all = sums_all;
            a.writes_norm = l == 0;
            before += blocks;
            if (phase == 0) {
                prof::Timed timed("gradient_squares", st);
                clip_squares_kernel<<<blocks, kThreads, 0, st>>>(a);
            } else if (clip) {
                const int wide = chunks < 1 ? 1 : chunks < 4096 ? (int)chunks : 4096;
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
