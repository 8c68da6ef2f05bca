// The divergence of a student's probabilities from a teacher's list of likely tokens, and its gradient (kan_net.h).
//
// A row's tokens are of two kinds: those of the teacher's list, at most 256, and the others.  One pass over the row sums the exponentials of the
// others alone: the listed ones are marked in a bit a token in LDS (V / 8 bytes), a piece of 16 bytes of logits asks for its bits with one read,
// and takes marked logits for -infinity.  The list's own logits are gathered beside it, and a wave adds what they do in 64 bits.  So neither
// kind is a difference of two larger sums: the probability of the others, a thousandth in a trained network, has all its digits, and
// so has the listed tokens' in a row where they have none.
//   total = sum_S exp(z - M) + rest exp(m - M),   rest and m: the sum and the largest logit of the others,   q_r = rest exp(m - M) / total
// The gradient of a token off the list is its exponential exp(z - m) times one factor of the row, g (q_r P - p_r) / (temperature rest), that of a
// listed one g (q P - p) / temperature: both differences are taken in 64 bits, where student and teacher nearly agree in all 32 kept ones.  The forward
// pass leaves them (K + 2 floats a row), the backward pass reads no teacher.
//
// Sixteen lanes a row where rows are short and many, a wave up to 8192 tokens (forward of 16384 x 8192 bf16 57 us, 86 with four), four up to 128 KB of logits, eight beyond (the step of
// 8192 x 131072 bf16 927 us with four, 898 so; 4096 x 50001 fp32 393 and 364; 8192 x 32768 bf16, below the line, 211 and 236).  Measured: 4093 x 50001
// fp32, an eighth of the rows without a teacher, forward 123 us (717 MB, 5.8 TB/s), backward 298 (1.54 GB, 5.1); 8192 x 131072 bf16 forward 328-378
// (2.15 GB, 5.7-6.5), backward 710 (4.3 GB, 6.05): HBM.  The step reads the logits twice as well, the second time from the row's end, where they have
// been read last: 860 us of 8192 x 131072 bf16, 3.8 GB read past the L2 caches (4.3 without what they still hold) and 2.2 written, 6.95 TB/s there.
// It has 96 registers, two workgroups a CU; a build for three spills and took 954 where this took 927.
#include "net_softmax.hpp"

namespace kannet {
namespace {

constexpr int kEntries = KAN_TEACHER_MAX / 64;          // of the list, a lane: E of them, one for up to 64 tokens
constexpr uint32_t kMarked = 1u << 18;                  // tokens that are marked at a time: 32 KB
constexpr double kNothing = 1e-300;

struct DistillCall {
    const void *logits;
    int64_t row_stride, V, R;
    const int64_t *ids;
    const void *teacher;
    int K, teacher_type, teacher_form;
    Temperature t;
    const float *g_loss;
    float *loss, *stats;
    void *glogits;
    int parts;              // of a row, in the forward pass
    uint32_t part_pieces;   // pieces of 16 bytes of a part
    Mass *part_sums;        // [R][parts]
    uint32_t chunks;        // workgroups of a row, in the backward pass
};

// The teacher's list of a row, over W lanes: entry e * W + lane.
template <int E>
struct List {
    int32_t id[E];                  // -1: nothing
    double p[E], log_p[E];
    float z[E];                     // the student's logit
    double p_sum, p_rest;
    bool some;
};

// whether it is so in any lane of a group of W
template <int W>
__device__ __forceinline__ bool any_of(bool v)
{
    if constexpr (W == 64) return __any(v);
    else return __ballot(v) >> (threadIdx.x & (64 - W)) & ((1ull << W % 64) - 1);
}

template <class T, int E, int W = 64>
__device__ __forceinline__ void read_list(const DistillCall &a, int64_t row, const T *z, int lane, List<E> &l)
{
    float value[E];
#pragma unroll
    for (int e = 0; e < E; ++e) {
        const int k = e * W + lane;
        l.id[e] = -1;
        l.z[e] = value[e] = -INFINITY;
        if (k < a.K) {
            const int64_t at = row * a.K + k, id = a.ids[at];
            if (id >= 0 && id < a.V) {
                l.id[e] = (int32_t)id;
                value[e] = a.teacher_type == KAN_F32 ? ((const float *)a.teacher)[at] : widen(((const bf16 *)a.teacher)[at]);
                l.z[e] = widen(z[id]);
            }
        }
    }
    double most = 0.0, log_sum = 0.0, sum = 0.0;
    if (a.teacher_form == KAN_TEACHER_LOGITS) {
        float m = -INFINITY;
#pragma unroll
        for (int e = 0; e < E; ++e) m = fmaxf(m, value[e]);
        most = (double)lane_max<W>(m);
        if (most == -(double)INFINITY) most = 0.0;
#pragma unroll
        for (int e = 0; e < E; ++e)
            if (e * W < a.K && l.id[e] >= 0) sum += exp_of(((double)value[e] - most) * a.t.inverse);
        log_sum = log_of(group_sum<W>(sum));
    }
    sum = 0.0;
    bool some = false;
#pragma unroll
    for (int e = 0; e < E; ++e) {
        l.p[e] = l.log_p[e] = 0.0;
        if (e * W < a.K && l.id[e] >= 0) {
            const bool logits = a.teacher_form == KAN_TEACHER_LOGITS && value[e] != -INFINITY;
            l.log_p[e] = logits ? ((double)value[e] - most) * a.t.inverse - log_sum : (double)value[e];
            l.p[e] = exp_of(l.log_p[e]);
            sum += l.p[e];
            some = some || l.p[e] != 0.0;
        }
    }
    l.p_sum = group_sum<W>(sum);
    l.p_rest = a.teacher_form == KAN_TEACHER_LOGP ? fmax(0.0, 1.0 - l.p_sum) : 0.0;
    l.some = any_of<W>(some);
}

// What a row's gradients are made of
template <int E>
struct RowGradient {
    float m, factor;            // of a token off the list: exp2((z - m) * scale) * factor
    float listed[E];            // of the list's
};

// Whether a token is in the list more than once, the same in all lanes
template <int E>
__device__ __forceinline__ bool repeats(const List<E> &l, int K, int lane)
{
    bool again = false;
#pragma unroll
    for (int of = 0; of < E; ++of)
        for (int k = 0; k < 64 && of * 64 + k < K; ++k) {
            const int32_t id = __builtin_amdgcn_readlane(l.id[of], k);
#pragma unroll
            for (int e = 0; e < E; ++e) again = again || (id >= 0 && l.id[e] == id && (e != of || lane != k));
        }
    return __any(again);
}

// A row's loss and gradients from its list and the sum over the other tokens, by W lanes.  `twice`: a token is in the list more than once.
template <int E, int W = 64>
__device__ __forceinline__ double finish_row(const DistillCall &a, const List<E> &l, Mass others, bool twice, int lane, RowGradient<E> &g)
{
    bool first[E];
    double p_all[E];                // of all entries of a token
#pragma unroll
    for (int e = 0; e < E; ++e) {
        first[e] = l.id[e] >= 0;
        p_all[e] = l.p[e];
    }
    if (twice) {
#pragma unroll
        for (int e = 0; e < E; ++e) p_all[e] = 0.0;
#pragma unroll
        for (int of = 0; of < E; ++of)
            for (int k = 0; k < W && of * W + k < a.K; ++k) {
                const int32_t id = of_group<W>(l.id[of], k);
                const uint64_t bits = __builtin_bit_cast(uint64_t, l.p[of]);
                const double p = __builtin_bit_cast(double, (uint64_t)(uint32_t)of_group<W>((int)(bits >> 32), k) << 32 | (uint32_t)of_group<W>((int)(uint32_t)bits, k));
#pragma unroll
                for (int e = 0; e < E; ++e)
                    if (l.id[e] == id) {
                        p_all[e] += p;
                        if (of * W + k < e * W + lane) first[e] = false;
                    }
            }
    }
    const bool rest = !(others.s == 0.0f);          // a NaN counts
    double rest_sum = (double)others.s;
    if (others.s > 1024.0f) {       // a reference far below the largest logit: one near it, which leaves the factor in a float's range
        const float from = others.m;
        others.m += __builtin_amdgcn_logf(others.s) / a.t.scale;
        rest_sum *= exp_of(((double)from - (double)others.m) * a.t.inverse);
    }
    float m = rest ? others.m : -INFINITY;
    bool nan = false;               // a NaN hides in the maximum
#pragma unroll
    for (int e = 0; e < E; ++e) {
        m = fmaxf(m, l.z[e]);
        nan = nan || l.z[e] != l.z[e];
    }
    const double M = (double)lane_max<W>(m);
    const bool empty = M == -(double)INFINITY && !rest && !any_of<W>(nan);
    double weight[E], sum = 0.0;
#pragma unroll
    for (int e = 0; e < E; ++e) {
        weight[e] = 0.0;
        if (e * W < a.K && l.id[e] >= 0) {
            weight[e] = exp_of(((double)l.z[e] - M) * a.t.inverse);
            if (first[e]) sum += weight[e];
        }
    }
    const double down = ((double)others.m - M) * a.t.inverse, off = rest ? rest_sum * exp_of(down) : 0.0;
    const double total = group_sum<W>(sum) + off, inverse = 1.0 / total, log_total = log_of(total), q_rest = off * inverse;
    const double p_rest = q_rest >= kNothing ? l.p_rest : 0.0, P = l.p_sum + p_rest;
    double loss = 0.0;
#pragma unroll
    for (int e = 0; e < E; ++e) {
        g.listed[e] = 0.0f;
        if (e * W < a.K && l.id[e] >= 0) {
            if (l.p[e] != 0.0) loss += l.p[e] * (l.log_p[e] - (((double)l.z[e] - M) * a.t.inverse - log_total));
            if (l.some && !empty) g.listed[e] = (float)((weight[e] * inverse * P - p_all[e]) * a.t.inverse);
        }
    }
    loss = group_sum<W>(loss);
    if (p_rest > 0.0) loss += p_rest * (log_of(p_rest) - (down + log_of(rest_sum) - log_total));
    // (without others no token asks for the factor but the masked ones of a row with a NaN among the listed)
    g.m = rest && l.some ? others.m : 0.0f;
    g.factor = !l.some || empty ? 0.0f : rest ? (float)((q_rest * P - p_rest) * a.t.inverse / rest_sum) : total == total ? 0.0f : NAN;
    return !l.some ? 0.0 : empty ? (double)INFINITY : loss;
}

template <int E, int W = 64>
__device__ __forceinline__ void write_row(const DistillCall &a, int64_t row, double loss, const RowGradient<E> &g, int lane)
{
    if (lane == 0 && a.loss) a.loss[row] = (float)loss;
    if (!a.stats) return;
    float *s = a.stats + row * (a.K + 2);
    if (lane == 0) {
        s[0] = g.m;
        s[1] = g.factor;
    }
#pragma unroll
    for (int e = 0; e < E; ++e)
        if (e * W + lane < a.K) s[2 + e * W + lane] = g.listed[e];
}

// What makes a row's gradients as if no token were listed: 2^(v * scale - reference) * factor, as in a tally, or where the reference is
// too large for that (a NaN) 2^((v - m) * scale) * factor; factor 0: zeros, whatever the logits are.
struct RowFactor {
    float m, reference, factor;
};

__device__ __forceinline__ float uniform(float v) { return __builtin_bit_cast(float, __builtin_amdgcn_readfirstlane(__builtin_bit_cast(int, v))); }

__device__ __forceinline__ RowFactor row_factor(float m, float factor, float scale)
{
    const float reference = m * scale;
    const bool near = fabsf(reference) <= kNear;
    return RowFactor{m, near ? reference : NAN, near ? factor * __builtin_amdgcn_exp2f(-__builtin_fmaf(m, scale, -reference)) : factor};
}

template <int N>
__device__ __forceinline__ void gradients(float (&v)[N], const RowFactor &g, float scale)
{
    if (g.factor == 0.0f) {
#pragma unroll
        for (int k = 0; k < N; ++k) v[k] = 0.0f;
    } else if (g.reference == g.reference) {
#pragma unroll
        for (int k = 0; k < N; ++k) v[k] = __builtin_amdgcn_exp2f(__builtin_fmaf(v[k], scale, -g.reference)) * g.factor;
    } else {
#pragma unroll
        for (int k = 0; k < N; ++k) v[k] = power(v[k], g.m, scale) * g.factor;
    }
}

template <class T, int NT>
__device__ __forceinline__ void write_round(const Round<T, NT> &r, T *to, uint32_t first, uint32_t V, const RowFactor &g, float scale)
{
    constexpr int N = 16 / (int)sizeof(T);
    const uint32_t tid = threadIdx.x, pieces = (V + N - 1) / N;
    if (first + kRound * NT <= V / N) {
        typedef typename Raw<T, N>::Wide *To;
#pragma unroll
        for (int u = 0; u < kRound; ++u) {
            float v[N];
            unpack(r.r[u], v);
            gradients(v, g, scale);
            __builtin_nontemporal_store(pack<N>(to, v).a, (To)(to + (int64_t)(first + u * NT) * N) + tid);
        }
    } else {
#pragma unroll 1
        for (int u = 0; u < kRound; ++u) {
            const uint32_t p = first + tid + u * NT;
            if (p >= pieces) continue;
            Raw<T, N> own = u == 0 ? r.r[0] : u == 1 ? r.r[1] : u == 2 ? r.r[2] : r.r[3];
            float v[N];
            settle(own, (int64_t)p * N, (int64_t)V);
            unpack(own, v);
            gradients(v, g, scale);
            store_at<N, true>(to, (int64_t)p * N, (int64_t)V, v);
        }
    }
}

// A row, or part blockIdx.x % a.parts of it (few rows are cut; distill_join_kernel does the rest).  STEP: and its gradients.
template <class T, int NT, int E, bool STREAM, bool STEP>
__global__ __launch_bounds__(NT) void distill_kernel(DistillCall a)
{
    constexpr int N = 16 / sizeof(T);
    extern __shared__ uint32_t marks[];
    __shared__ Mass wave_sums[NT / 64];
    __shared__ uint32_t twice, some;
    __shared__ float of_row[2];
    const uint32_t tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int64_t row = blockIdx.x / a.parts;
    const uint32_t part = blockIdx.x % a.parts, V = (uint32_t)a.V, pieces = (V + N - 1) / N;
    const uint32_t begin = part * a.part_pieces, end = pieces - begin < a.part_pieces ? pieces : begin + a.part_pieces;
    const T *z = (const T *)a.logits + row * a.row_stride;
    const float scale = a.t.scale;
    Round<T, NT> next;
    read_round<STREAM>(next, z, begin, end, V);
    if (tid == 0) twice = 0;
    List<E> list;
    if (wave == 0 && a.parts == 1) {
        read_list(a, row, z, lane, list);
        if (lane == 0) some = list.some;
    }
    Tally tally = no_tally();
    for (uint32_t base = begin; base < end; base += kMarked / N) {
        const uint32_t stop = end - base < kMarked / N ? end : base + kMarked / N;
        const uint32_t words = ((stop - base) * N + 31) / 32;
        if (base != begin) __syncthreads();
        for (uint32_t w = tid; w < words; w += NT) marks[w] = 0;
        __syncthreads();
        if (a.parts == 1 && !some) break;               // no teacher: the row is not read
        for (int k = tid; k < a.K; k += NT) {
            const int64_t id = a.ids[row * a.K + k];
            if (id < (int64_t)base * N || id >= (int64_t)stop * N || id >= a.V) continue;
            const uint32_t at = (uint32_t)(id - (int64_t)base * N);
            if (atomicOr(&marks[at / 32], 1u << at % 32) >> at % 32 & 1) twice = 1;
        }
        __syncthreads();
        for (uint32_t first = base; first < stop; first += kRound * NT) {
            const Round<T, NT> now = next;
            // behind the last round, what the next slice begins with
            read_round<STREAM>(next, z, first + kRound * NT < stop ? first + kRound * NT : stop, end, V);
            const auto unmarked = [&](float (&v)[N], uint32_t p) {
                const uint32_t bits = N == 8 ? ((const uint8_t *)marks)[p - base] : ((const uint8_t *)marks)[(p - base) / 2] >> ((p - base) % 2 * 4) & 15;
                if (bits)
#pragma unroll
                    for (int k = 0; k < N; ++k) v[k] = bits >> k & 1 ? -INFINITY : v[k];
            };
            const bool whole = first + kRound * NT <= (V / N < stop ? V / N : stop);
            if (!whole || tally.reference != tally.reference ||
                !add_whole_round(now, scale, tally, [&](float (&v)[N], int u) { unmarked(v, first + tid + u * NT); }))
                each_piece(now, first, stop, V, [&](float (&v)[N], uint32_t p, int) {
                    unmarked(v, p);
                    add_piece<N>(v, scale, tally);
                });
        }
    }
    const Mass sum = join_mass<NT>(mass_of(tally, scale), scale, wave_sums);
    if (a.parts > 1) {
        if (tid == 0) a.part_sums[row * a.parts + part] = sum;
        return;
    }
    RowGradient<E> g;
    float weight = 0.0f;
    if (wave == 0) {
        const double loss = finish_row(a, list, sum, twice != 0, lane, g);
        write_row(a, row, loss, g, lane);
        if constexpr (STEP) {
            weight = a.g_loss[row];
            if (lane == 0) {
                of_row[0] = g.m;
                of_row[1] = g.factor == 0.0f ? 0.0f : g.factor * weight;
            }
        }
    }
    if constexpr (STEP) {
        T *to = (T *)a.glogits + row * a.V;
        // the row once more, from its end, where it has been read last; rows without a teacher get zeros without a look at them
        const uint32_t rounds = (pieces + kRound * NT - 1) / (kRound * NT), n = some ? V : 0;
        Round<T, NT> r;
        read_round<true>(r, z, (rounds - 1) * (kRound * NT), pieces, n);
        __syncthreads();
        const RowFactor rest = row_factor(uniform(of_row[0]), uniform(of_row[1]), scale);
        for (uint32_t i = rounds; i-- > 0;) {
            const Round<T, NT> now = r;
            if (i) read_round<true>(r, z, (i - 1) * (kRound * NT), pieces, n);
            write_round(now, to, i * (kRound * NT), V, rest, scale);
        }
        __syncthreads();        // the listed tokens' gradients go on top
        if (wave == 0)
#pragma unroll
            for (int e = 0; e < E; ++e)
                if (list.id[e] >= 0) put(to + list.id[e], g.listed[e] == 0.0f ? 0.0f : g.listed[e] * weight);
    }
}

// A wave for each row that was cut, at most 64 parts
template <class T, int E>
__global__ __launch_bounds__(64) void distill_join_kernel(DistillCall a)
{
    const int64_t row = blockIdx.x;
    const int lane = threadIdx.x;
    Mass sum = {kLowest, 0.0f};
    if (lane < a.parts) sum = a.part_sums[row * a.parts + lane];
    List<E> list;
    read_list(a, row, (const T *)a.logits + row * a.row_stride, lane, list);
    sum = join_lanes<64>(sum, a.t.scale);
    RowGradient<E> g;
    const double loss = finish_row(a, list, sum, repeats(list, a.K, lane), lane, g);
    write_row(a, row, loss, g, lane);
}

// The gradient's row from what the forward pass has left: elements are independent, a read and a write of the logits.
template <class T, int NT, int E, bool STREAM>
__global__ __launch_bounds__(NT) void distill_back_kernel(DistillCall a)
{
    constexpr int N = 16 / sizeof(T);
    const int64_t row = blockIdx.x / a.chunks;
    const uint32_t V = (uint32_t)a.V, pieces = (V + N - 1) / N, first = blockIdx.x % a.chunks * (kRound * NT);
    const T *z = (const T *)a.logits + row * a.row_stride;
    T *to = (T *)a.glogits + row * a.V;
    const float *s = a.stats + row * (a.K + 2);
    const float g = a.g_loss[row];
    const RowFactor rest = row_factor(uniform(s[0]), uniform(s[1] == 0.0f ? 0.0f : s[1] * g), a.t.scale);
    Round<T, NT> r;
    read_round<STREAM>(r, z, first, pieces, rest.factor == 0.0f ? 0 : V);      // rows without a teacher are not read
    // the listed tokens that lie here, by every wave for itself: most workgroups have none, and nothing to wait for
    const int64_t from = (int64_t)first * N, until = from + kRound * NT * N < a.V ? from + kRound * NT * N : a.V;
    int64_t id[E];
#pragma unroll
    for (int e = 0; e < E; ++e) id[e] = (int)(e * 64 + (threadIdx.x & 63)) < a.K ? a.ids[row * a.K + e * 64 + (threadIdx.x & 63)] : -1;
    write_round(r, to, first, V, rest, a.t.scale);
    bool here = false;
#pragma unroll
    for (int e = 0; e < E; ++e) {
        if (id[e] < from || id[e] >= until) id[e] = -1;
        here = here || id[e] >= 0;
    }
    if (!__any(here)) return;
    __syncthreads();            // their gradients go on top
    if (threadIdx.x < 64)
#pragma unroll
        for (int e = 0; e < E; ++e)
            if (id[e] >= 0) {
                const float d = s[2 + e * 64 + threadIdx.x];
                put(to + id[e], d == 0.0f ? 0.0f : d * g);
            }
}

// Short rows: 16 lanes each, sixteen rows a workgroup, written through the caches (16384 x 501 fp32 backward 12.5 us, past them 18.2: rows begin and end within lines).  With a wave a
// row, half of the time is what a row costs in 64 bits, on no more lanes than the list has entries, and 65536 workgroups take 25 us before they do anything.
constexpr int kLanes = 16, kRowsOf = 256 / kLanes;

// whose row a thread works on; a workgroup's threads behind the last row go with it, and write nothing
struct ShortRow {
    int64_t row;
    uint32_t lane, group;
    bool there;
};

__device__ __forceinline__ ShortRow short_row(int64_t R)
{
    const uint32_t group = threadIdx.x / kLanes;
    const int64_t row = (int64_t)blockIdx.x * kRowsOf + group;
    return ShortRow{row < R ? row : R - 1, threadIdx.x % kLanes, group, row < R};
}

// f(logits, piece) for a lane's pieces of a row of n, four on their way while four are worked on
template <class T, class F>
__device__ __forceinline__ void each_of_short(const T *z, uint32_t lane, uint32_t pieces, uint32_t n, Raw<T, 16 / sizeof(T)> (&next)[kRound], F f)
{
    constexpr int N = 16 / (int)sizeof(T);
    for (uint32_t first = lane; first < pieces; first += kRound * kLanes) {
        Raw<T, N> now[kRound];
#pragma unroll
        for (int u = 0; u < kRound; ++u) now[u] = next[u];
        if (first + kRound * kLanes < pieces)
#pragma unroll
            for (int u = 0; u < kRound; ++u) next[u] = raw_at<N>(z, (int64_t)(first + (kRound + u) * kLanes) * N, (int64_t)n);
#pragma unroll
        for (int u = 0; u < kRound; ++u) {
            const uint32_t p = first + u * kLanes;
            if (p >= pieces) break;
            float v[N];
            piece_logits<N>(now[u], p, n, v);
            f(v, p);
        }
    }
}

template <class T>
__device__ __forceinline__ void first_of_short(const T *z, uint32_t lane, uint32_t n, Raw<T, 16 / sizeof(T)> (&next)[kRound])
{
    constexpr int N = 16 / (int)sizeof(T);
#pragma unroll
    for (int u = 0; u < kRound; ++u) next[u] = raw_at<N>(z, (int64_t)(lane + u * kLanes) * N, (int64_t)n);
}

template <class T, int E, bool STEP>
__global__ __launch_bounds__(256) void distill_short_kernel(DistillCall a)
{
    constexpr int N = 16 / (int)sizeof(T);
    extern __shared__ uint32_t all_marks[];
    __shared__ uint32_t twice[kRowsOf];
    const ShortRow of = short_row(a.R);
    const uint32_t V = (uint32_t)a.V, pieces = (V + N - 1) / N, words = (V + 31) / 32;
    const T *z = (const T *)a.logits + of.row * a.row_stride;
    const float scale = a.t.scale;
    uint32_t *marks = all_marks + of.group * words;
    Raw<T, N> next[kRound];
    first_of_short(z, of.lane, V, next);
    for (uint32_t w = of.lane; w < words; w += kLanes) marks[w] = 0;
    if (of.lane == 0) twice[of.group] = 0;
    List<E> list;
    read_list<T, E, kLanes>(a, of.row, z, of.lane, list);
    __syncthreads();
#pragma unroll
    for (int e = 0; e < E; ++e) {
        const int32_t id = list.id[e];
        if (id >= 0 && (atomicOr(&marks[id / 32], 1u << id % 32) >> id % 32 & 1)) twice[of.group] = 1;
    }
    __syncthreads();
    Tally tally = no_tally();
    each_of_short(z, of.lane, pieces, V, next, [&](float (&v)[N], uint32_t p) {
        const uint32_t bits = N == 8 ? ((const uint8_t *)marks)[p] : ((const uint8_t *)marks)[p / 2] >> (p % 2 * 4) & 15;
#pragma unroll
        for (int k = 0; k < N; ++k) v[k] = bits >> k & 1 ? -INFINITY : v[k];
        add_piece<N>(v, scale, tally);
    });
    const Mass sum = join_lanes<kLanes>(mass_of(tally, scale), scale);
    RowGradient<E> g;
    const double loss = finish_row<E, kLanes>(a, list, sum, twice[of.group] != 0, of.lane, g);
    if (of.there) write_row<E, kLanes>(a, of.row, loss, g, of.lane);
    if constexpr (STEP) {
        T *to = (T *)a.glogits + of.row * a.V;
        const float weight = a.g_loss[of.row];
        const RowFactor rest = row_factor(g.m, g.factor == 0.0f ? 0.0f : g.factor * weight, scale);
        const uint32_t n = of.there ? V : 0;
        first_of_short(z, of.lane, n, next);
        each_of_short(z, of.lane, of.there ? pieces : 0, n, next, [&](float (&v)[N], uint32_t p) {
            gradients(v, rest, scale);
            store_at<N>(to, (int64_t)p * N, (int64_t)V, v);
        });
        __syncthreads();        // the listed tokens' gradients go on top
        if (!of.there) return;
#pragma unroll
        for (int e = 0; e < E; ++e)
            if (list.id[e] >= 0) put(to + list.id[e], g.listed[e] == 0.0f ? 0.0f : g.listed[e] * weight);
    }
}

template <class T, int E>
__global__ __launch_bounds__(256) void distill_short_back_kernel(DistillCall a)
{
    constexpr int N = 16 / (int)sizeof(T);
    const ShortRow of = short_row(a.R);
    if (!of.there) return;      // no barrier that they would be missed at: rows lie within waves
    const uint32_t V = (uint32_t)a.V, pieces = (V + N - 1) / N;
    const T *z = (const T *)a.logits + of.row * a.row_stride;
    T *to = (T *)a.glogits + of.row * a.V;
    const float *s = a.stats + of.row * (a.K + 2);
    Raw<T, N> next[kRound];
    first_of_short(z, of.lane, V, next);
    const float g = a.g_loss[of.row], factor = s[1];
    const RowFactor rest = row_factor(s[0], factor == 0.0f ? 0.0f : factor * g, a.t.scale);
    int64_t id[E];
    float listed[E];
#pragma unroll
    for (int e = 0; e < E; ++e) {
        const int k = e * kLanes + of.lane;
        id[e] = k < a.K ? a.ids[of.row * a.K + k] : -1;
        listed[e] = k < a.K ? s[2 + k] : 0.0f;
    }
    each_of_short(z, of.lane, pieces, V, next, [&](float (&v)[N], uint32_t p) {
        gradients(v, rest, a.t.scale);
        store_at<N>(to, (int64_t)p * N, (int64_t)V, v);
    });
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");      // the listed tokens' gradients go on top
#pragma unroll
    for (int e = 0; e < E; ++e)
        if (id[e] >= 0 && id[e] < a.V) put(to + id[e], listed[e] == 0.0f ? 0.0f : listed[e] * g);
}

// The shortest ones always, longer ones where they are many: with few, a lane's longer way counts.  us, 16 lanes a row and a wave, forward, step, backward:
//   256 x 64 fp32, K = 8     4.8 5.6,   5.7 6.6,   3.4 3.4        16384 x 64      7.3 22.8,   9.1 27.2,  4.4 7.8
//   1024 x 256 fp32          5.7 5.9,   7.3 7.0,   4.1 3.6        65536 x 256 bf16 24 81,     33 100,    18 26
//   4096 x 512 fp32          7.5 9.3,  11.2 12.0,  6.1 5.3        16384 x 501    12.1 25.3,  20.3 33.2, 12.5 15.8
//   4096 x 1000 bf16, K = 20 8.9 9.5,  12.8 13.0,  6.8 6.3        65536 x 1000     50 93,     88 122,    59 58
//   8192 x 2000 bf16, K = 20 15.7 19.5, 26.5 29.5, 14.5 15.4      65536 x 2000     72 120,   174 177,   139 121
//   1024 x 1000 fp32, K = 8  10.2 7.1, 15.3 9.6,   7.6 4.9        65536 x 1000 fp32, K = 64  88 114, 217 168, 160 202
// The forward pass and the step go the same way, whose sums have to be the same bits: in the last line the step's 168 us decide, and the forward pass takes 114 where it could take 88.  The backward
// pass needs more rows (K = 20, rows twice and four times their bytes): 250 fp32 3.9 3.8 and 4.2 4.6, 501 5.9 5.6 and 7.8 8.4; bf16 500 4.3 4.0 and 4.6 5.0, 1002 6.6 6.1 and 8.4 9.0.
bool is_short(const DistillCall &a, size_t size, bool back)
{
    const double bytes = (double)a.V * (double)size;
    return a.K <= 64 && (bytes <= 512.0 || ((double)a.R >= (back ? 4.0 : 2.0) * bytes && (bytes <= 2048.0 || (bytes <= 4096.0 && a.K <= 32 && !back))));
}

// Few long rows are shared among workgroups, two a CU, and joined by a launch more.  Whole and cut, us, twenty tokens: 1 x 65536 bf16 8.2 and 7.6, 1 x 131072 11.3 and
// 7.7, 64 x 131072 12.0 and 9.9, 128 x 131072 16.0 and 18.1, 16 x 32768 7.7 and 9.2; fp32: 64 x 50001 9.6 and 10.0, 100 x 131072 18.9 and 16.8, 200 x 131072 20.4 and
// 22.8, 128 x 262144 32 and 27, 1 x 1000000 82 and 10.
int parts_of(int64_t R, int64_t V, size_t size)
{
    const double row = (double)V * (double)size / 262144.0;
    if (R <= 0 || R > 256 || row < 1.0 || (double)R > 96.0 * row) return 1;
    const int64_t parts = 512 / R < V / 8192 ? 512 / R : V / 8192;
    return (int)(parts > 64 ? 64 : parts);
}

constexpr int64_t kRows = 1 << 21, kShortRows = 1 << 27;        // of a launch: less than 2^32 threads

DistillCall rows_from(DistillCall a, int64_t first, int64_t most, size_t size)
{
    a.R = a.R - first < most ? a.R - first : most;
    a.logits = (const char *)a.logits + (size_t)(first * a.row_stride) * size;
    a.ids += first * a.K;
    if (a.teacher) a.teacher = (const char *)a.teacher + (size_t)(first * a.K) * size_of(a.teacher_type);
    if (a.g_loss) a.g_loss += first;
    if (a.loss) a.loss += first;
    if (a.stats) a.stats += first * (a.K + 2);
    if (a.glogits) a.glogits = (char *)a.glogits + (size_t)(first * a.V) * size;
    return a;
}

// whether the logits do not stay in the caches from one pass to the next (8192 x 131072 bf16 backward 708 us past them, 754 through them; 2000 x 33000, 132 MB, 57 and 52)
bool passes_by(const DistillCall &a, size_t size) { return (double)a.R * (double)a.V * (double)size >= kLastCache; }

template <class T, int E>
void launch_back(const DistillCall &a, int threads, bool stream, unsigned grid, hipStream_t st)
{
    if (threads == 64) distill_back_kernel<T, 64, E, false><<<grid, 64, 0, st>>>(a);
    else if (stream) distill_back_kernel<T, 256, E, true><<<grid, 256, 0, st>>>(a);
    else distill_back_kernel<T, 256, E, false><<<grid, 256, 0, st>>>(a);
}

template <class T>
hipError_t launch_backward(const DistillCall &all, hipStream_t st)
{
    constexpr int N = 16 / sizeof(T);
    prof::Timed timed("token_distill_backward", st);
    const int64_t pieces = div_up(all.V, (int64_t)N);
    const bool stream = passes_by(all, sizeof(T));
    const int threads = pieces <= 64 * kRound ? 64 : 256;
    const int64_t chunks = div_up(pieces, (int64_t)threads * kRound), most = (1ll << 23) / chunks > 1 ? (1ll << 23) / chunks : 1;
    if (is_short(all, sizeof(T), true)) {
        for (int64_t first = 0; first < all.R; first += kShortRows) {
            const DistillCall a = rows_from(all, first, kShortRows, sizeof(T));
            const unsigned grid = (unsigned)div_up(a.R, (int64_t)kRowsOf);
            if (a.K <= kLanes) distill_short_back_kernel<T, 1><<<grid, 256, 0, st>>>(a);
            else distill_short_back_kernel<T, 4><<<grid, 256, 0, st>>>(a);
            const hipError_t e = hipGetLastError();
            if (e != hipSuccess) return e;
        }
        return hipSuccess;
    }
    for (int64_t first = 0; first < all.R; first += most) {
        DistillCall a = rows_from(all, first, most, sizeof(T));
        a.chunks = (uint32_t)chunks;
        const unsigned grid = (unsigned)(a.R * chunks);
        if (a.K <= 64) launch_back<T, 1>(a, threads, stream, grid, st);
        else launch_back<T, kEntries>(a, threads, stream, grid, st);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

template <class T, int E, bool STEP>
void launch_kernel(const DistillCall &a, unsigned grid, unsigned lds, hipStream_t st)
{
    const bool stream = !STEP && passes_by(a, sizeof(T));
    const bool wide = (double)a.V * sizeof(T) >= 128e3 && a.parts == 1;
    if (a.V <= 8192) distill_kernel<T, 64, E, false, STEP><<<grid, 64, lds, st>>>(a);
    else if (wide && stream) distill_kernel<T, 512, E, !STEP, STEP><<<grid, 512, lds, st>>>(a);
    else if (wide) distill_kernel<T, 512, E, false, STEP><<<grid, 512, lds, st>>>(a);
    else if (stream) distill_kernel<T, 256, E, !STEP, STEP><<<grid, 256, lds, st>>>(a);
    else distill_kernel<T, 256, E, false, STEP><<<grid, 256, lds, st>>>(a);
}

template <class T, bool STEP>
hipError_t launch_rows(const DistillCall &all, hipStream_t st)
{
    prof::Timed timed(STEP ? "token_distill_step" : "token_distill", st);
    constexpr uint32_t N = 16 / sizeof(T);
    const uint32_t tokens = all.part_pieces * N < kMarked ? all.part_pieces * N : kMarked, lds = (tokens + 31) / 32 * 4;
    if (is_short(all, sizeof(T), false)) {
        const unsigned room = (unsigned)((all.V + 31) / 32 * 4) * kRowsOf;
        for (int64_t first = 0; first < all.R; first += kShortRows) {
            const DistillCall a = rows_from(all, first, kShortRows, sizeof(T));
            const unsigned rows = (unsigned)div_up(a.R, (int64_t)kRowsOf);
            if (a.K <= kLanes) distill_short_kernel<T, 1, STEP><<<rows, 256, room, st>>>(a);
            else distill_short_kernel<T, 4, STEP><<<rows, 256, room, st>>>(a);
            const hipError_t e = hipGetLastError();
            if (e != hipSuccess) return e;
        }
        return hipSuccess;
    }
    for (int64_t first = 0; first < all.R; first += kRows) {
        const DistillCall a = rows_from(all, first, kRows, sizeof(T));
        const unsigned grid = (unsigned)(a.R * a.parts);
        if (a.K <= 64) launch_kernel<T, 1, STEP>(a, grid, lds, st);
        else launch_kernel<T, kEntries, STEP>(a, grid, lds, st);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

template <class T>
hipError_t launch_forward(DistillCall &a, bool step, hipStream_t st)
{
    constexpr uint32_t N = 16 / sizeof(T);
    const uint32_t pieces = (uint32_t)div_up(a.V, (int64_t)N);
    a.part_pieces = div_up(pieces, (uint32_t)a.parts);
    a.parts = (int)div_up(pieces, a.part_pieces);
    if (a.parts == 1) return step ? launch_rows<T, true>(a, st) : launch_rows<T, false>(a, st);
    hipError_t e = launch_rows<T, false>(a, st);
    if (e != hipSuccess) return e;
    {
        prof::Timed timed("token_distill_join", st);
        if (a.K <= 64) distill_join_kernel<T, 1><<<(unsigned)a.R, 64, 0, st>>>(a);
        else distill_join_kernel<T, kEntries><<<(unsigned)a.R, 64, 0, st>>>(a);
        e = hipGetLastError();
    }
    return e != hipSuccess || !step ? e : launch_backward<T>(a, st);
}

int check(int64_t R, int64_t V, int32_t type, int64_t row_stride, int32_t K, float temperature)
{
    if (R < 0 || V <= 0 || row_stride < V || K < 1 || !(temperature >= 1e-30f && temperature <= 1e30f)) return KAN_ERR_INVALID_ARG;
    if (!known_type(type) || R >= (1ll << 31) || V >= (1ll << 31) - 1 || K > KAN_TEACHER_MAX) return KAN_ERR_UNSUPPORTED;
    return KAN_OK;
}

// whether gradients in place of the logits would lie elsewhere than their logits
bool shifts(int64_t R, int64_t V, const void *logits, int64_t row_stride, const void *glogits) { return glogits == logits && R > 1 && row_stride != V; }

// for the type whose rows are the longer ones
size_t sums_bytes(int64_t R, int64_t V)
{
    const int parts = parts_of(R, V, 4);
    return parts > 1 ? align_up((size_t)R * parts * sizeof(Mass)) : 0;
}

// the forward call, and the step where `glogits` is there
int run(int64_t R, int64_t V, const void *logits, int32_t type, int64_t row_stride, int32_t K, const int64_t *ids, const void *teacher,
        int32_t teacher_type, int32_t teacher_form, float temperature, bool step, const float *g_loss, float *loss, float *stats, void *glogits, void *ws,
        size_t ws_bytes, hipStream_t st)
{
    const int rc = check(R, V, type, row_stride, K, temperature);
    if (rc != KAN_OK) return rc;
    if (!known_type(teacher_type) || (teacher_form != KAN_TEACHER_LOGP && teacher_form != KAN_TEACHER_LOGITS)) return KAN_ERR_UNSUPPORTED;
    if (R == 0) return KAN_OK;
    if (!logits || !ids || !teacher || misplaced(logits, type) || misplaced8(ids) || misplaced(teacher, teacher_type) || misplaced(loss, KAN_F32) ||
        misplaced(stats, KAN_F32))
        return KAN_ERR_INVALID_ARG;
    if (step && (!g_loss || !glogits || misplaced(g_loss, KAN_F32) || misplaced(glogits, type) || shifts(R, V, logits, row_stride, glogits))) return KAN_ERR_INVALID_ARG;
    if (bad_workspace(ws, ws_bytes, kan_token_distill_workspace_bytes(R, V, K))) return KAN_ERR_WORKSPACE;
    DistillCall a = {};
    a.logits = logits;
    a.row_stride = row_stride;
    a.V = V;
    a.R = R;
    a.ids = ids;
    a.teacher = teacher;
    a.K = K;
    a.teacher_type = teacher_type;
    a.teacher_form = teacher_form;
    a.t = temperature_of(temperature);
    a.g_loss = g_loss;
    a.loss = loss;
    a.parts = parts_of(R, V, size_of(type));
    a.part_sums = (Mass *)ws;
    a.stats = step && a.parts > 1 ? (float *)((char *)ws + sums_bytes(R, V)) : stats;
    a.glogits = glogits;
    return status_of(type == KAN_F32 ? launch_forward<float>(a, step, st) : launch_forward<bf16>(a, step, st));
}

}  // namespace
}  // namespace kannet

using namespace kannet;

// nothing where rows are not cut; otherwise sums of the parts, and what the step keeps between its passes
extern "C" size_t kan_token_distill_workspace_bytes(int64_t R, int64_t V, int32_t K)
{
    if (V <= 0 || K < 1 || K > KAN_TEACHER_MAX) return 0;
    const size_t sums = sums_bytes(R, V);
    return sums ? sums + align_up((size_t)R * (K + 2) * sizeof(float)) : 0;
}

extern "C" int kan_token_distill_forward(int64_t R, int64_t V, const void *logits, int32_t type, int64_t row_stride, int32_t K,
                                         const int64_t *teacher_ids, const void *teacher, int32_t teacher_type, int32_t teacher_form, float temperature,
                                         float *loss, float *stats, void *ws, size_t ws_bytes, void *stream)
{
    return run(R, V, logits, type, row_stride, K, teacher_ids, teacher, teacher_type, teacher_form, temperature, false, nullptr, loss, stats, nullptr, ws, ws_bytes,
               (hipStream_t)stream);
}

extern "C" int kan_token_distill_step(int64_t R, int64_t V, const void *logits, int32_t type, int64_t row_stride, int32_t K, const int64_t *teacher_ids,
                                      const void *teacher, int32_t teacher_type, int32_t teacher_form, float temperature, const float *g_loss, float *loss,
                                      void *glogits, void *ws, size_t ws_bytes, void *stream)
{
    return run(R, V, logits, type, row_stride, K, teacher_ids, teacher, teacher_type, teacher_form, temperature, true, g_loss, loss, nullptr, glogits, ws, ws_bytes,
               (hipStream_t)stream);
}

extern "C" int kan_token_distill_backward(int64_t R, int64_t V, const void *logits, int32_t type, int64_t row_stride, int32_t K,
                                          const int64_t *teacher_ids, float temperature, const float *stats, const float *g_loss, void *glogits,
                                          void *stream)
{
    const int rc = check(R, V, type, row_stride, K, temperature);
    if (rc != KAN_OK) return rc;
    if (R == 0) return KAN_OK;
    if (!logits || !teacher_ids || !stats || !g_loss || !glogits || misplaced(logits, type) || misplaced(glogits, type) || misplaced8(teacher_ids) ||
        misplaced(stats, KAN_F32) || misplaced(g_loss, KAN_F32) || shifts(R, V, logits, row_stride, glogits))
        return KAN_ERR_INVALID_ARG;
    DistillCall a = {};
    a.logits = logits;
    a.row_stride = row_stride;
    a.V = V;
    a.R = R;
    a.ids = teacher_ids;
    a.K = K;
    a.t = temperature_of(temperature);
    a.stats = const_cast<float *>(stats);
    a.g_loss = g_loss;
    a.glogits = glogits;
    return status_of(type == KAN_F32 ? launch_backward<float>(a, (hipStream_t)stream) : launch_backward<bf16>(a, (hipStream_t)stream));
}
