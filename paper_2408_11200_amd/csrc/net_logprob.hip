// Log probabilities of given tokens, entropy, most likely tokens, and the gradient of a loss on them (kan_net.h).
//
// Forward reads a row of logits once.  Every thread keeps, over its pieces of 16 bytes, the largest logit, the sum of the exponentials
// 2^y relative to it, y = (logit - largest) * log2(e) / temperature, and the sum of 2^y * y, rescaled when a larger one turns up; threads,
// then waves are joined the same way.  log sum = log of the first; entropy = log sum - (second / first), two terms of one sign.  The
// difference is taken before the scaling: logits of the type's lowest value stay finite, and a row with one likely token keeps the digits
// of what little the others add (one multiply-add with a rounded reference would be an instruction less, and lose them).
// Four pieces a thread are in flight while four are worked on: with one, 8192 x 131072 bf16 ran at 2.2 TB/s.
//
// The most likely tokens come out of the same read: a thread's largest logit with its place is the best of its pieces, so the top ones
// of the row all lie with the `top` threads whose bests are the largest.  Those threads' pieces are read again (from L2), and what is
// not below the last of these bests is sorted into a list that a wave holds one entry a lane.
#include "net_device.hpp"

namespace kannet {
namespace {

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr float kLowest = -3.4028234663852886e38f;
constexpr float kFar = -200.0f;          // 2^-200 is zero in 32 bits: what a term further down adds to the second sum

struct LogprobCall {
    const void *logits;
    int64_t row_stride, V, R;
    const int64_t *ids;
    float scale;            // log2(e) / temperature
    float inv_temperature;
    int top;
    float *logp, *entropy, *stats;
    int64_t *top_ids;
    float *top_logp;
    const float *g_logp, *g_entropy;
    void *glogits;
};

struct Sums {
    float m, s, t;          // largest logit (at least the lowest finite value), sum of 2^y, sum of 2^y y
};

__device__ __forceinline__ void rescale(Sums &a, float m, float scale)
{
    const float y = fmaxf((a.m - m) * scale, kFar), c = __builtin_amdgcn_exp2f(y);
    a.t = c * (a.t + y * a.s);
    a.s *= c;
    a.m = m;
}

__device__ __forceinline__ Sums join(Sums a, Sums b, float scale)
{
    const float m = fmaxf(a.m, b.m);
    rescale(a, m, scale);
    rescale(b, m, scale);
    return Sums{m, a.s + b.s, a.t + b.t};
}

// over a workgroup
template <int NT>
__device__ __forceinline__ Sums join_all(Sums s, float scale, Sums *lds)
{
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
        const Sums o = {__shfl_xor(s.m, d, 64), __shfl_xor(s.s, d, 64), __shfl_xor(s.t, d, 64)};
        s = join(s, o, scale);
    }
    if (NT == 64) return s;
    __syncthreads();
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = s;
    __syncthreads();
    s = lds[0];
    for (int w = 1; w < NT / 64; ++w) s = join(s, lds[w], scale);
    return s;
}

// Larger logits, and of equal ones the lower index, have the larger key; 0: none.  A NaN is above +infinity, both zeros are one value.
__device__ __forceinline__ uint64_t key_of(float v, uint32_t index)
{
    uint32_t b = __builtin_bit_cast(uint32_t, v);
    if (v != v) b = 0x7FC00000u;
    if (v == 0.0f) b = 0u;
    b = (b >> 31) ? ~b : b | 0x80000000u;
    return (uint64_t)b << 32 | (uint32_t)~index;
}

__device__ __forceinline__ float logit_of(uint64_t key)
{
    const uint32_t b = (uint32_t)(key >> 32);
    return __builtin_bit_cast(float, (b >> 31) ? b & 0x7FFFFFFFu : ~b);
}

__device__ __forceinline__ uint64_t shuffle(uint64_t v, int lane)
{
    return (uint64_t)(uint32_t)__shfl((int)(v >> 32), lane, 64) << 32 | (uint32_t)__shfl((int)(uint32_t)v, lane, 64);
}

// A wave's list of keys, best first, one a lane: puts in every lane's `key` (0: none) that is above entry `top` - 1
__device__ __forceinline__ void put_in(uint64_t &list, uint64_t key, int top, int lane)
{
    uint64_t last = shuffle(list, top - 1);
    uint64_t open = __ballot(key > last);
    while (open) {
        const int from = __ffsll((unsigned long long)open) - 1;
        const uint64_t k = shuffle(key, from);
        open &= open - 1;
        if (k <= last) continue;
        const int at = __popcll(__ballot(list > k));
        const uint64_t before = shuffle(list, lane > 0 ? lane - 1 : 0);
        list = lane < at ? list : lane == at ? k : before;
        last = shuffle(list, top - 1);
    }
}

constexpr int kAhead = 4;

// one piece: N logits
template <int N>
__device__ __forceinline__ void add_piece(const float (&v)[N], uint32_t at, float scale, Sums &s, float &most, uint32_t &most_at)
{
    float m = v[0];
#pragma unroll
    for (int k = 1; k < N; ++k) m = fmaxf(m, v[k]);
    if (m > most) {
        most = m;
        most_at = at;
        if (m > s.m) rescale(s, m, scale);
    }
#pragma unroll
    for (int k = 0; k < N; ++k) {
        const float y = (v[k] - s.m) * scale, e = __builtin_amdgcn_exp2f(y);
        s.s += e;
        s.t += e * fmaxf(y, kFar);
    }
}

template <class T, int NT>
__global__ __launch_bounds__(NT) void logprob_kernel(LogprobCall a)
{
    constexpr int kWaves = NT / 64, N = 16 / sizeof(T);
    __shared__ Sums wave_sums[kWaves];
    __shared__ uint64_t best[NT];                // top > 0: the threads' bests; then wave 0's
    const int64_t row = blockIdx.x;
    const T *z = (const T *)a.logits + row * a.row_stride;
    const uint32_t tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const uint32_t V = (uint32_t)a.V, whole = V / N, pieces = (V + N - 1) / N;
    const float scale = a.scale;

    Sums s = {kLowest, 0.0f, 0.0f};
    float most = -INFINITY;
    uint32_t most_at = tid, p = tid;
    {
        typedef typename Raw<T, N>::Wide Wide;
        const auto read = [&](Raw<T, N> (&r)[kAhead], uint32_t from) {
#pragma unroll
            for (int u = 0; u < kAhead; ++u) r[u].a = *(const Wide *)(z + (int64_t)(from + u * NT) * N);
        };
        const uint32_t reach = (kAhead - 1) * NT;
        Raw<T, N> next[kAhead];
        bool more = (uint64_t)p + reach < whole;
        if (more) read(next, p);
        while (more) {
            Raw<T, N> now[kAhead];
#pragma unroll
            for (int u = 0; u < kAhead; ++u) now[u] = next[u];
            const uint32_t at = p;
            p += kAhead * NT;
            more = (uint64_t)p + reach < whole;
            if (more) read(next, p);
#pragma unroll
            for (int u = 0; u < kAhead; ++u) {
                float v[N];
                unpack(now[u], v);
                add_piece<N>(v, at + u * NT, scale, s, most, most_at);
            }
        }
    }
    for (; p < pieces; p += NT) {
        float v[N];
        Raw<T, N> r = raw_at<N>(z, (int64_t)p * N, a.V);
        settle(r, (int64_t)p * N, a.V);
        unpack(r, v);
        if (p >= whole)
#pragma unroll
            for (int k = 0; k < N; ++k) v[k] = p * N + k < V ? v[k] : -INFINITY;
        add_piece<N>(v, p, scale, s, most, most_at);
    }
    if (a.top) best[tid] = tid < pieces ? key_of(most, most_at) : 0;     // of pieces, not of logits
    s = join_all<NT>(s, scale, wave_sums);
    if (wave != 0) return;
    const bool empty = s.s == 0.0f, wrong = s.s != s.s || s.m == INFINITY;
    const float log_sum = empty ? 0.0f : logf(s.s);
    const float entropy = empty ? 0.0f : wrong ? NAN : log_sum - kLn2 * (s.t / s.s);
    const auto logp_of = [&](float v) { return empty ? -INFINITY : wrong ? NAN : (v - s.m) * a.inv_temperature - log_sum; };
    if (lane == 0) {
        if (a.entropy) a.entropy[row] = entropy;
        if (a.stats) {
            a.stats[row * 2] = empty ? -INFINITY : wrong ? NAN : s.m;
            a.stats[row * 2 + 1] = empty ? 0.0f : s.s;
        }
        if (a.logp) {
            const int64_t id = a.ids[row];
            a.logp[row] = id >= 0 && id < a.V ? logp_of(widen(z[id])) : 0.0f;
        }
    }
    if (!a.top) return;

    // the last of the `top` best threads: below it nothing is looked at (a NaN has no place among the bests: then everything is)
    const bool all = s.s != s.s;
    uint64_t list = 0;
    for (int i = 0; i < kWaves; ++i) put_in(list, best[i * 64 + lane], a.top, lane);
    const uint64_t bound = all ? 0 : shuffle(list, a.top - 1);
    const uint32_t sources = all ? NT : a.top, each = (pieces + NT - 1) / NT, count = sources * each;
    uint64_t found = 0;
    if (lane < (uint32_t)a.top) best[lane] = list;
    __builtin_amdgcn_wave_barrier();
    for (uint32_t first = 0; first < count; first += 64) {
        // piece number i % each of source i / each: the thread that has the source's best
        const uint32_t i = first + lane, src = i / each;
        uint32_t at = pieces;
        if (src < sources) {
            const uint64_t k = all ? 1 : best[src];
            if (k) at = (all ? src : (uint32_t)~(uint32_t)k % NT) + i % each * NT;
        }
        float v[N];
        Raw<T, N> r = raw_at<N>(z, (int64_t)at * N, at < pieces ? a.V : 0);
        settle(r, (int64_t)at * N, at < pieces ? a.V : 0);
        unpack(r, v);
#pragma unroll
        for (int k = 0; k < N; ++k) {
            const uint32_t index = at * N + k;
            uint64_t key = at < pieces && index < V ? key_of(v[k], index) : 0;
            // a thread's best stands for its piece: compare by piece
            const uint64_t by_piece = key ? (key & 0xFFFFFFFF00000000ull) | (uint32_t)~at : 0;
            if (by_piece < bound) key = 0;
            put_in(found, key, a.top, lane);
        }
    }
    if (lane < (uint32_t)a.top) {
        const float v = logit_of(found);
        a.top_ids[row * a.top + lane] = (int64_t)(uint32_t)~(uint32_t)found;
        a.top_logp[row * a.top + lane] = logp_of(v);
    }
}

constexpr int kBackPieces = 4;      // of 16 bytes a thread

template <class T>
__global__ __launch_bounds__(256) void logprob_back_kernel(LogprobCall a)
{
    constexpr int N = 16 / sizeof(T);
    const int64_t row = blockIdx.y, V = a.V, first = ((int64_t)blockIdx.x * 256 * kBackPieces + threadIdx.x) * N;
    const T *z = (const T *)a.logits + row * a.row_stride;
    Raw<T, N> r[kBackPieces];
#pragma unroll
    for (int u = 0; u < kBackPieces; ++u) r[u] = raw_at<N>(z, first + u * 256 * N, V);
    const float m = a.stats[row * 2], sum = a.stats[row * 2 + 1];
    const int64_t id = a.g_logp ? a.ids[row] : -1;
    const bool given = id >= 0 && id < V;
    const float g = given ? a.g_logp[row] : 0.0f, ge = a.g_entropy ? a.g_entropy[row] : 0.0f;
    // -p (g + ge (log p + entropy)) / temperature = 2^y (c0 + c1 y)
    const float shift = a.g_entropy ? a.entropy[row] - logf(sum) : 0.0f, inv = -a.inv_temperature / sum;
    const float c0 = inv * (g + ge * shift), c1 = inv * ge * kLn2, hit = g * a.inv_temperature;
    const bool empty = m == -INFINITY;
#pragma unroll
    for (int u = 0; u < kBackPieces; ++u) {
        const int64_t c = first + u * 256 * N;
        float v[N];
        settle(r[u], c, V);
        unpack(r[u], v);
#pragma unroll
        for (int k = 0; k < N; ++k) {
            const float y = (v[k] - m) * a.scale;
            v[k] = empty ? 0.0f : __builtin_amdgcn_exp2f(y) * __builtin_fmaf(c1, fmaxf(y, kFar), c0);
        }
        if (given && !empty && id >= c && id < c + N)
#pragma unroll
            for (int k = 0; k < N; ++k) v[k] += c + k == id ? hit : 0.0f;
        store_at<N, true>((T *)a.glogits + row * V, c, V, v);
    }
}

int check(int64_t R, int64_t V, int32_t type, int64_t row_stride, float temperature)
{
    if (R < 0 || V <= 0 || row_stride < V || !(temperature >= 1e-30f && temperature <= 1e30f)) return KAN_ERR_INVALID_ARG;
    if (!known_type(type) || R >= (1ll << 31) || V >= (1ll << 31) - 1) return KAN_ERR_UNSUPPORTED;
    return KAN_OK;
}

template <class T>
hipError_t launch_forward(const LogprobCall &a, hipStream_t st)
{
    prof::Timed timed("token_logprob", st);
    const unsigned rows = (unsigned)a.R;
    if (a.V <= 4096) logprob_kernel<T, 64><<<rows, 64, 0, st>>>(a);
    else if (a.V <= 16384 || a.R >= 1024) logprob_kernel<T, 256><<<rows, 256, 0, st>>>(a);
    else logprob_kernel<T, 1024><<<rows, 1024, 0, st>>>(a);
    return hipGetLastError();
}

template <class T>
hipError_t launch_backward(const LogprobCall &all, hipStream_t st)
{
    prof::Timed timed("token_logprob_backward", st);
    for (int64_t first = 0; first < all.R; first += 65535) {
        LogprobCall a = all;
        const int64_t rows = all.R - first < 65535 ? all.R - first : 65535;
        a.logits = (const T *)all.logits + first * all.row_stride;
        a.glogits = (T *)all.glogits + first * all.V;
        a.stats = all.stats + first * 2;
        if (a.g_logp) {
            a.g_logp += first;
            a.ids += first;
        }
        if (a.g_entropy) {
            a.g_entropy += first;
            a.entropy += first;
        }
        logprob_back_kernel<T><<<dim3((unsigned)div_up(all.V, (int64_t)(256 * kBackPieces * 16 / sizeof(T))), (unsigned)rows), 256, 0, st>>>(a);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace
}  // namespace kannet

using namespace kannet;

extern "C" size_t kan_token_logprob_workspace_bytes(int64_t, int64_t, int32_t) { return 0; }

extern "C" int kan_token_logprob_forward(int64_t R, int64_t V, const void *logits, int32_t type, int64_t row_stride, const int64_t *ids,
                                         float temperature, int32_t top, float *logp, float *entropy, float *stats, int64_t *top_ids,
                                         float *top_logp, void *ws, size_t ws_bytes, void *stream)
{
    const int rc = check(R, V, type, row_stride, temperature);
    if (rc != KAN_OK) return rc;
    if (top < 0 || top > V) return KAN_ERR_INVALID_ARG;
    if (top > KAN_TOP_MAX) return KAN_ERR_UNSUPPORTED;
    if (R == 0) return KAN_OK;
    if (!logits || misplaced(logits, type) || (logp && !ids) || (top && (!top_ids || !top_logp))) return KAN_ERR_INVALID_ARG;
    if (misplaced8(ids) || misplaced8(top_ids) || misplaced(logp, KAN_F32) || misplaced(entropy, KAN_F32) || misplaced(stats, KAN_F32) ||
        misplaced(top_logp, KAN_F32))
        return KAN_ERR_INVALID_ARG;
    if (bad_workspace(ws, ws_bytes, kan_token_logprob_workspace_bytes(R, V, top))) return KAN_ERR_WORKSPACE;
    LogprobCall a = {};
    a.logits = logits;
    a.row_stride = row_stride;
    a.V = V;
    a.R = R;
    a.ids = ids;
    a.scale = kLog2e / temperature;
    a.inv_temperature = 1.0f / temperature;
    a.top = top;
    a.logp = logp;
    a.entropy = entropy;
    a.stats = stats;
    a.top_ids = top_ids;
    a.top_logp = top_logp;
    return status_of(type == KAN_F32 ? launch_forward<float>(a, (hipStream_t)stream) : launch_forward<bf16>(a, (hipStream_t)stream));
}

extern "C" int kan_token_logprob_backward(int64_t R, int64_t V, const void *logits, int32_t type, int64_t row_stride, const int64_t *ids,
                                          float temperature, const float *stats, const float *entropy, const float *g_logp,
                                          const float *g_entropy, void *glogits, void *stream)
{
    const int rc = check(R, V, type, row_stride, temperature);
    if (rc != KAN_OK) return rc;
    if (R == 0) return KAN_OK;
    if (!logits || !stats || !glogits || (!g_logp && !g_entropy) || (g_logp && !ids) || (g_entropy && !entropy)) return KAN_ERR_INVALID_ARG;
    if (misplaced(logits, type) || misplaced(glogits, type) || misplaced8(ids) || misplaced(stats, KAN_F32) || misplaced(entropy, KAN_F32) ||
        misplaced(g_logp, KAN_F32) || misplaced(g_entropy, KAN_F32))
        return KAN_ERR_INVALID_ARG;
    LogprobCall a = {};
    a.logits = logits;
    a.row_stride = row_stride;
    a.V = V;
    a.R = R;
    a.ids = ids;
    a.scale = kLog2e / temperature;
    a.inv_temperature = 1.0f / temperature;
    a.stats = const_cast<float *>(stats);
    a.entropy = const_cast<float *>(entropy);
    a.g_logp = g_logp;
    a.g_entropy = g_entropy;
    a.glogits = glogits;
    return status_of(type == KAN_F32 ? launch_backward<float>(a, (hipStream_t)stream) : launch_backward<bf16>(a, (hipStream_t)stream));
}
