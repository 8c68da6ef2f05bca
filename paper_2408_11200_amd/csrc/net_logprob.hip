// Log probabilities of given tokens, entropy, most likely tokens, and the gradient of a loss on them (kan_net.h).
//
// Forward reads a row of logits once.  Every thread keeps, over its pieces of 16 bytes, the largest logit, the sum of the exponentials
// 2^y relative to it, y = (logit - largest) * log2(e) / temperature, and the sum of 2^y * y, rescaled when a larger one turns up; threads,
// then waves are joined the same way.  log sum = log of the first; entropy = log sum - (second / first), two terms of one sign.  The
// difference is taken before the scaling: logits of the type's lowest value stay finite, and no digits go to a rounded reference.
//
// In a row with one likely token the largest logit's own 1 would round off what the others add, and with it the log probability and 1 - p of
// that token.  Such a row (a sum below 5/4) gets the sum without that 1 for a little more reading: only the thread that has the largest logit
// has added to it, so its pieces, one in 64 or 256, are summed once more without it and added to the other threads' sums.  From
// there on a row is known by that rest.
// Four pieces a thread are in flight while four are worked on: with one, 8192 x 131072 bf16 ran at 2.2 TB/s.  Measured: 4093 x 50001 fp32 135-141 us
// (819 MB, 5.9 TB/s), bound by HBM; 8192 x 131072 bf16 with eight top tokens 390-420 us (2.15 GB, 5.1-5.5 TB/s) and with none 383-390, bound by its vector
// instructions, and so by the clock: the first twenty launches behind a pause take up to 510.  Some twelve issue slots an element (widen, compare, subtract,
// scale, the exponential's four, two clamped sums) are 330 us by themselves.  Rows of one likely token cost 2 % more.
//
// The most likely tokens come out of the same read.  The `top`-th largest of the threads' largest logits is a bound that `top` logits reach: after
// the first round of pieces, still in registers, those that reach its bound are kept, and of every later piece those that reach it; behind
// the row the bound of all of it leaves hardly more than `top` of them, put in order by counting for each how many are above it.  (Reading
// the pieces of the threads that have the bound once more, at the end, cost a quarter of the row: they lie in as many lines.)  The first round's bound
// stays to the row's end: where it is low for the row, more logits reach it than there is room for, and a second search reads the row again.
#include "net_top.hpp"

namespace kannet {
namespace {

constexpr float kLn2 = 0.6931471805599453f;
constexpr float kFar = -200.0f;          // 2^-200 is zero in 32 bits: what a term further down adds to the second sum

struct Sums {
    float m, s, t;          // largest logit (at least the lowest finite value), sum of 2^y, sum of 2^y y
};

struct Part {
    float m, rest, t;       // the same, but the sum less 2^0 = 1 of the largest logit; -1: nothing but -infinity
};

// Sums below this: the rest is summed without the largest logit.  What is left above it is the difference to 1, off by five times the sum's error.
constexpr float kClear = 1.25f;

// log(1 + x), by W. Kahan's correction of log for the rounding of 1 + x
__device__ __forceinline__ float log_1p(float x)
{
    const float u = 1.0f + x;
    return u == 1.0f ? x : logf(u) * (x * __builtin_amdgcn_rcpf(u - 1.0f));
}

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
    int parts;              // of a row, in the forward pass
    uint32_t part_pieces;   // pieces of 16 bytes of a part
    Part *part_sums;        // [R][parts]
    uint64_t *part_keys;    // [R][parts][top]
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

// over a workgroup: everyone's sums brought to the largest logit first, then plain sums (joined two by two over the lanes, each time with two
// exponentials and three exchanges, 16384 rows of 256 took 13.2 us, 11.3 so)
template <int NT>
__device__ __forceinline__ Sums join_all(Sums s, float scale, Sums *lds)
{
    const float m = lane_max<64>(s.m);
    rescale(s, m, scale);
    s.s = lane_sum<64>(s.s);
    s.t = lane_sum<64>(s.t);
    if (NT == 64) {
        // the first lane's bits for all, which take one way behind them: the product in rescale and the first sum become one fused multiply-add, whose rounding is another one
        // in either lane of a pair
        s.s = __builtin_bit_cast(float, __builtin_amdgcn_readfirstlane(__builtin_bit_cast(int, s.s)));
        return s;
    }
    __syncthreads();
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = s;
    __syncthreads();
    s = lds[0];
    for (int w = 1; w < NT / 64; ++w) s = join(s, lds[w], scale);
    return s;
}

constexpr int kAhead = 4;

// one piece: N logits; the largest of them
template <int N>
__device__ __forceinline__ float add_piece(const float (&v)[N], float scale, Sums &s, float &most)
{
    float m = v[0];
#pragma unroll
    for (int k = 1; k < N; ++k) m = fmaxf(m, v[k]);
    if (m > most) {
        most = m;
        if (m > s.m) rescale(s, m, scale);
    }
#pragma unroll
    for (int k = 0; k < N; ++k) {
        const float y = (v[k] - s.m) * scale, e = __builtin_amdgcn_exp2f(y);
        s.s += e;
        s.t += e * fmaxf(y, kFar);
    }
    return m;
}

// What a row, or a part of one, leaves for the wave that writes the results: its sums, and the keys of its most likely tokens, one a lane.
__device__ __forceinline__ void finish(const LogprobCall &a, int64_t row, Part s, uint64_t found, int lane, float given, bool there)
{
    const bool empty = s.rest == -1.0f, wrong = s.rest != s.rest || s.m == INFINITY;
    const float log_sum = empty ? 0.0f : log_1p(s.rest);
    const auto logp_of = [&](float v) {
        const float down = v - s.m;         // past a float's range, it need not be after the temperature
        return empty ? -INFINITY : wrong ? NAN : (down == -INFINITY && v > -INFINITY ? v * a.inv_temperature - s.m * a.inv_temperature : down * a.inv_temperature) - log_sum;
    };
    if (lane == 0) {
        if (a.entropy) a.entropy[row] = empty ? 0.0f : wrong ? NAN : log_sum - kLn2 * (s.t / (1.0f + s.rest));
        if (a.stats) {
            a.stats[row * 2] = empty ? -INFINITY : wrong ? NAN : s.m;
            a.stats[row * 2 + 1] = empty ? 0.0f : s.rest;
        }
        if (a.logp) a.logp[row] = there ? logp_of(given) : 0.0f;
    }
    if (lane < a.top) {
        a.top_ids[row * a.top + lane] = (int64_t)(uint32_t)~(uint32_t)found;
        a.top_logp[row * a.top + lane] = logp_of(logit_of(found));
    }
}

// A row, or part blockIdx.x of it (a.parts > 1: few rows are cut, so that the chip is filled; logprob_join_kernel does the rest).
// STREAM: loads past the caches, for logits that do not stay there until the backward pass.
template <class T, int NT, bool STREAM>
__global__ __launch_bounds__(NT) void logprob_kernel(LogprobCall a)
{
    constexpr int kWaves = NT / 64, N = 16 / sizeof(T);
    __shared__ Sums wave_sums[kWaves];
    __shared__ float wave_rest[kWaves];
    __shared__ uint32_t holder;
    constexpr uint32_t kCandidates = 4 * NT;
    __shared__ uint64_t best[kCandidates], shortlist[NT], chosen[KAN_TOP_MAX];
    __shared__ uint32_t candidates, kept, sources;
    __shared__ uint16_t source[NT];
    __shared__ float thread_most[NT];
    const int64_t row = blockIdx.y * 65535ll + blockIdx.x / a.parts;
    if (row >= a.R) return;
    const uint32_t part = blockIdx.x % a.parts;
    const T *z = (const T *)a.logits + row * a.row_stride;
    const uint32_t tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const uint32_t V = (uint32_t)a.V, whole = V / N, pieces = (V + N - 1) / N;
    const uint32_t begin = part * a.part_pieces, end = pieces - begin < a.part_pieces ? pieces : begin + a.part_pieces;
    const float scale = a.scale;
    // the wave that writes the results has the given token's logit on the way from the start
    int64_t id = -1;
    if (wave == 0 && a.logp && a.parts == 1) id = a.ids[row];
    const bool there = id >= 0 && id < a.V;
    const float given = there ? widen(z[id]) : 0.0f;

    Sums s = {kLowest, 0.0f, 0.0f};
    float most = -INFINITY;
    Raw<T, N> next[kAhead];
    const auto read = [&](uint32_t from) {
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            const uint32_t p = from + u * NT;
            next[u] = raw_at<N, STREAM>(z, (int64_t)p * N, p < end ? a.V : 0);
        }
    };
    const auto logits_of = [&](Raw<T, N> r, uint32_t p, float (&v)[N]) {
        settle(r, (int64_t)p * N, a.V);
        unpack(r, v);
        if (p >= whole)
#pragma unroll
            for (int k = 0; k < N; ++k) v[k] = p * N + k < V ? v[k] : -INFINITY;
    };
    // the candidates: all logits that are not below the `top`-th largest of the threads' largest ones in the first round
    float bound = NAN;
    const auto collect = [&](const float (&v)[N], uint32_t p) {
#pragma unroll
        for (int k = 0; k < N; ++k)
            if (v[k] >= bound && p * N + k < V) {
                const uint32_t slot = atomicAdd(&candidates, 1u);
                if (slot < kCandidates) best[slot] = key_of(v[k], p * N + k);
            }
    };
    if (tid == 0) sources = candidates = kept = 0;
    if (tid < KAN_TOP_MAX) chosen[tid] = 0;
    read(begin + tid);
    __syncthreads();
    for (uint32_t first = begin; first < end; first += kAhead * NT) {
        const uint32_t at = first + tid;
        Raw<T, N> now[kAhead];
#pragma unroll
        for (int u = 0; u < kAhead; ++u) now[u] = next[u];
        read(at + kAhead * NT);
        // more than there is room for: the rest is not kept (bound is set anew behind the loop)
        if (__hip_atomic_load(&candidates, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP) > kCandidates) bound = NAN;
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            const uint32_t p = at + u * NT;
            if (p < end) {
                float v[N];
                logits_of(now[u], p, v);
                if (add_piece<N>(v, scale, s, most) >= bound) collect(v, p);
            }
        }
        if (a.top && first == begin) {
            bound = value_of_rank<NT>(most, a.top, lane, thread_most);
#pragma unroll
            for (int u = 0; u < kAhead; ++u) {
                const uint32_t p = at + u * NT;
                if (p < end) {
                    float v[N];
                    logits_of(now[u], p, v);
                    collect(v, p);
                }
            }
        }
    }
    const Sums mine = s;
    s = join_all<NT>(s, scale, wave_sums);
    float rest = s.s - 1.0f;
    if (s.s >= 1.0f && s.s < kClear) {              // the same in all threads; exactly one has the largest logit, and has it once
        if (most == s.m) holder = tid;
        __syncthreads();
        const uint32_t h = holder;
        rest = tid == h ? 0.0f : mine.s * __builtin_amdgcn_exp2f(fmaxf((mine.m - s.m) * scale, kFar));
        for (uint32_t p = begin + h + tid * NT; p < end; p += NT * NT) {
            float v[N];
            logits_of(raw_at<N>(z, (int64_t)p * N, a.V), p, v);
#pragma unroll
            for (int k = 0; k < N; ++k) rest += v[k] == s.m ? 0.0f : __builtin_amdgcn_exp2f((v[k] - s.m) * scale);
        }
        rest = lane_sum<64>(rest);
        if (NT > 64) {
            if (lane == 0) wave_rest[wave] = rest;
            __syncthreads();
            rest = wave_rest[0];
            for (int w = 1; w < kWaves; ++w) rest += wave_rest[w];
        }
    }

    uint64_t found = 0;
    if (a.top) {
        const bool all = s.s != s.s;                // a NaN hides in the maxima
        const bool rounds = end - begin > kAhead * NT;
        if (rounds && !all) bound = value_of_rank<NT>(most, a.top, lane, thread_most);
        __syncthreads();
        uint32_t n = candidates;
        if (!all && n <= kCandidates) {
            // of these, the ones that reach the bound of the whole row
            for (uint32_t i = tid; i < n; i += NT) {
                const uint64_t k = best[i];
                if (logit_of(k) >= bound) {
                    const uint32_t slot = atomicAdd(&kept, 1u);
                    if (slot < NT) shortlist[slot] = k;
                }
            }
            __syncthreads();
            const bool shorter = kept <= NT;
            const uint64_t *list = shorter ? shortlist : best;
            n = shorter ? kept : n;
            for (uint32_t i = tid; i < n; i += NT) {
                const uint64_t k = list[i];
                const int place = above(list, n, k);
                if (place < a.top) chosen[place] = k;
            }
            __syncthreads();
            if (wave == 0 && lane < (uint32_t)a.top) found = chosen[lane];
        } else {
            // A NaN in the row, or more candidates than there is room for (likely tokens behind the first round, rising logits, many equal ones; of 131072
            // random ones with 64 top tokens, some 1200 bf16 or 2300 fp32 reach the first round's bound): the pieces of the threads whose largest logit
            // reaches the bound are read again, by every wave into a sorted list of its own.  2048 x 32768 bf16, top 8: 159 us of equal logits
            // by one wave, 122 by all four; 52 us of random ones.
            if (begin + tid < end && (all || most >= bound)) source[atomicAdd(&sources, 1u)] = (uint16_t)tid;
            __syncthreads();
            const uint32_t each = (end - begin + NT - 1) / NT, count = sources * each;
            for (uint32_t first = 64 * wave; first < count; first += NT) {
                const uint32_t i = first + lane, p = i < count ? begin + source[i / each] + i % each * NT : end;
                float v[N];
                logits_of(raw_at<N>(z, (int64_t)p * N, p < end ? a.V : 0), p, v);
#pragma unroll
                for (int k = 0; k < N; ++k) put_in(found, p < end && p * N + k < V && (all || v[k] >= bound) ? key_of(v[k], p * N + k) : 0, a.top, lane);
            }
            if (NT > 64) {
                __syncthreads();                // the candidates' number has been read
                best[tid] = lane < (uint32_t)a.top ? found : 0;
                __syncthreads();
                if (wave == 0)
                    for (uint32_t w = 1; w < NT / 64; ++w) put_in(found, best[64 * w + lane], a.top, lane);
            }
        }
    }
    if (wave != 0) return;
    if (a.parts == 1) {
        finish(a, row, Part{s.m, rest, s.t}, found, lane, given, there);
        return;
    }
    const int64_t slot = row * a.parts + part;
    if (lane == 0) a.part_sums[slot] = Part{s.m, rest, s.t};
    if (lane < (uint32_t)a.top) a.part_keys[slot * a.top + lane] = found;
}

// A workgroup for each row that was cut, at most 64 parts: 3.5 us, one latency after another (16 x 32768, 8 parts, five tokens)
template <class T>
__global__ __launch_bounds__(256) void logprob_join_kernel(LogprobCall a)
{
    __shared__ uint64_t key[256], chosen[KAN_TOP_MAX];
    const int64_t row = blockIdx.x;
    const int tid = threadIdx.x, lane = tid & 63, keys = a.parts * a.top;
    uint64_t found = 0;
    if (keys > 0 && keys <= 256) {
        const uint64_t k = tid < keys ? a.part_keys[row * keys + tid] : 0;
        key[tid] = k;
        if (tid < KAN_TOP_MAX) chosen[tid] = 0;
        __syncthreads();
        const int at = above(key, keys, k);
        if (k && at < a.top) chosen[at] = k;
        __syncthreads();
        if (lane < a.top) found = chosen[lane];
    }
    if (tid >= 64) return;
    int64_t id = -1;
    if (a.logp) id = a.ids[row];
    const bool there = id >= 0 && id < a.V;
    const float given = there ? widen(((const T *)a.logits + row * a.row_stride)[id]) : 0.0f;
    // the parts' sums behind the row's largest logit; the first part that has it brings its rest
    Part s = {kLowest, -1.0f, 0.0f};
    if (lane < a.parts) s = a.part_sums[row * a.parts + lane];
    Sums all = {s.m, 1.0f + s.rest, s.t};
    s.m = lane_max<64>(all.m);
    const uint64_t holders = __ballot(all.m == s.m && s.rest != -1.0f);
    const bool holds = holders && lane == __ffsll((unsigned long long)holders) - 1;
    rescale(all, s.m, a.scale);
    s.rest = holders ? lane_sum<64>(holds ? s.rest : all.s) : -1.0f;
    s.t = lane_sum<64>(all.t);
    if (keys > 256)
        for (int i = 0; i < keys; i += 64) put_in(found, i + lane < keys ? a.part_keys[row * keys + i + lane] : 0, a.top, lane);
    finish(a, row, s, found, lane, given, there);
}

// The gradient's row, from the forward pass's largest logit and sum: no sum is left to take, so elements are independent and the pass is bound by HBM,
// a read and a write of the logits: 4093 x 50001 fp32 295 us (1.64 GB, 5.6 TB/s), 8192 x 131072 bf16 735 (4.3 GB, 5.8).
constexpr int kBackPieces = 4;      // of 16 bytes a thread, next to one another in a row or (ROWS) in four rows

template <class T, bool ROWS>
__global__ __launch_bounds__(256) void logprob_back_kernel(LogprobCall a)
{
    constexpr int N = 16 / sizeof(T);
    const int64_t V = a.V;
    int64_t row[kBackPieces], c[kBackPieces];
    Raw<T, N> r[kBackPieces];
#pragma unroll
    for (int u = 0; u < kBackPieces; ++u) {
        row[u] = ROWS ? (int64_t)blockIdx.y * kBackPieces + u : blockIdx.y;
        c[u] = ROWS ? ((int64_t)blockIdx.x * blockDim.x + threadIdx.x) * N : (((int64_t)blockIdx.x * kBackPieces + u) * blockDim.x + threadIdx.x) * N;
        if (ROWS && row[u] >= a.R) row[u] = a.R - 1, c[u] = V;
        r[u] = raw_at<N>((const T *)a.logits + row[u] * a.row_stride, c[u], V);
    }
    float m = 0.0f, c0 = 0.0f, c1 = 0.0f, hit = 0.0f, most = 0.0f;
    int64_t id = -1;
    bool empty = false;
#pragma unroll
    for (int u = 0; u < kBackPieces; ++u) {
        if (ROWS || u == 0) {
            // -p (g + ge (log p + entropy)) / temperature = 2^y (c0 + c1 y); `most`: the given token's where it is the largest logit,
            // of which 1 - p = rest / (1 + rest)
            const int64_t at = row[u];
            m = a.stats[at * 2];
            const float rest = a.stats[at * 2 + 1], sum = 1.0f + rest;
            id = a.g_logp ? a.ids[at] : -1;
            const bool given = id >= 0 && id < V;
            const float g = given ? a.g_logp[at] : 0.0f, ge = a.g_entropy ? a.g_entropy[at] : 0.0f;
            const float shift = a.g_entropy ? a.entropy[at] - log_1p(rest) : 0.0f, inv = -a.inv_temperature / sum;
            c0 = inv * (g + ge * shift);
            most = inv * (ge * shift - g * rest);
            c1 = inv * ge * kLn2;
            hit = g * a.inv_temperature;
            empty = m == -INFINITY;
            if (!given || empty) id = -1;
        }
        float v[N];
        settle(r[u], c[u], V);
        unpack(r[u], v);
#pragma unroll
        for (int k = 0; k < N; ++k) {
            const float y = (v[k] - m) * a.scale;
            v[k] = empty ? 0.0f : __builtin_amdgcn_exp2f(y) * __builtin_fmaf(c1, fmaxf(y, kFar), c0);
        }
        if (id >= c[u] && id < c[u] + N) {
            float logit[N];
            unpack(r[u], logit);
#pragma unroll
            for (int k = 0; k < N; ++k)
                if (c[u] + k == id) v[k] = logit[k] == m ? most : v[k] + hit;
        }
        store_at<N, true>((T *)a.glogits + row[u] * V, c[u], V, v);
    }
}

int check(int64_t R, int64_t V, int32_t type, int64_t row_stride, float temperature)
{
    if (R < 0 || V <= 0 || row_stride < V || !(temperature >= 1e-30f && temperature <= 1e30f)) return KAN_ERR_INVALID_ARG;
    if (!known_type(type) || R >= (1ll << 31) || V >= (1ll << 31) - 1) return KAN_ERR_UNSUPPORTED;
    return KAN_OK;
}

// How a row is cut: few rows of a large vocabulary are shared among workgroups, four a CU, of 4096 logits at least, and joined by a launch more.
// Whole and cut, us, bf16: 1 x 131072 with five alternatives 31.6 and 11.6, without 27.9 and 7.6; 64 x 131072 with twenty 34.8 and 21.6;
// 16 x 32768 with five 14.2 and 10.2, 128 x 32768 14.8 and 13.8, 1 x 16384 10.3 and 10.4; fp32: 64 x 50001 24.1 and 15.1, 400 x 100000 54.6 and 53.8.
// Where between 16384 and 32768 cutting begins to pay has not been measured.
int parts_of(int64_t R, int64_t V)
{
    if (R <= 0 || R > 512 || V < 32768) return 1;
    int64_t parts = 1024 / R;
    if (parts > V / 4096) parts = V / 4096;
    return (int)(parts > 64 ? 64 : parts);
}

template <class T>
hipError_t launch_forward(LogprobCall &a, hipStream_t st)
{
    constexpr uint32_t N = 16 / sizeof(T);
    const uint32_t pieces = (uint32_t)div_up(a.V, (int64_t)N);
    a.part_pieces = div_up(pieces, (uint32_t)a.parts);
    a.parts = (int)div_up(pieces, a.part_pieces);
    const dim3 grid((unsigned)(a.R < 65535 ? a.R : 65535) * a.parts, (unsigned)div_up(a.R, (int64_t)65535));
    {
        prof::Timed timed("token_logprob", st);
        // 4093 x 50001 fp32 (819 MB) 138 us with streaming loads, 151 without; where the caches hold the logits, the backward pass loses by them
        // more than that (400 x 100000, 160 MB: 58 us and 50)
        const bool stream = (double)a.R * (double)a.V * sizeof(T) >= 512e6;
        if (a.V <= 4096) logprob_kernel<T, 64, false><<<grid, 64, 0, st>>>(a);
        else if (stream) logprob_kernel<T, 256, true><<<grid, 256, 0, st>>>(a);
        else logprob_kernel<T, 256, false><<<grid, 256, 0, st>>>(a);
    }
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || a.parts == 1) return e;
    prof::Timed timed("token_logprob_join", st);
    logprob_join_kernel<T><<<(unsigned)a.R, 256, 0, st>>>(a);
    return hipGetLastError();
}

template <class T>
hipError_t launch_backward(const LogprobCall &all, hipStream_t st)
{
    constexpr int N = 16 / sizeof(T);
    prof::Timed timed("token_logprob_backward", st);
    // Rows of up to two workgroups' width: four rows a thread, a piece of each.
    const int64_t pieces = div_up(all.V, (int64_t)N);
    const bool by_rows = pieces <= 512;
    const int threads = pieces <= 64 ? 64 : pieces <= 128 ? 128 : 256;
    const int64_t most = by_rows ? 65535ll * kBackPieces : 65535;
    for (int64_t first = 0; first < all.R; first += most) {
        LogprobCall a = all;
        a.R = all.R - first < most ? all.R - first : most;
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
        if (by_rows)
            logprob_back_kernel<T, true><<<dim3((unsigned)div_up(pieces, (int64_t)threads), (unsigned)div_up(a.R, (int64_t)kBackPieces)), threads, 0, st>>>(a);
        else
            logprob_back_kernel<T, false><<<dim3((unsigned)div_up(pieces, (int64_t)(256 * kBackPieces)), (unsigned)a.R), 256, 0, st>>>(a);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace
}  // namespace kannet

using namespace kannet;

// nothing where rows are not cut
extern "C" size_t kan_token_logprob_workspace_bytes(int64_t R, int64_t V, int32_t top)
{
    if (V <= 0 || top < 0 || top > KAN_TOP_MAX) return 0;
    const int parts = parts_of(R, V);
    return parts > 1 ? align_up((size_t)R * parts * sizeof(Part)) + align_up((size_t)R * parts * top * sizeof(uint64_t)) : 0;
}

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
    a.parts = parts_of(R, V);
    a.part_sums = (Part *)ws;
    a.part_keys = (uint64_t *)((char *)ws + align_up((size_t)R * a.parts * sizeof(Part)));
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
