// Sums of exponentials over a row of logits, in one pass: the largest logit so far and the sum relative to it, threads and waves joined the same
// way.  Shared by the operators that need no second sum (net_distill.hip, net_beam.hip).
#pragma once
#include "net_top.hpp"

namespace kannet {

// log2(e) / temperature in 32 bits, as the streaming sums take it; what the results are made of is divided by the temperature in 64
struct Temperature {
    float scale;
    double inverse;
};

inline Temperature temperature_of(float t) { return Temperature{(float)(1.4426950408889634 / (double)t), 1.0 / (double)t}; }

struct Mass {
    float m, s;         // a logit, the largest one or near it, and the sum of 2^((v - m) * scale); the lowest finite value and 0: nothing but -infinity
};

__device__ __forceinline__ float power(float v, float m, float scale) { return __builtin_amdgcn_exp2f((v - m) * scale); }

// Four pieces a thread are in flight while four are worked on: a round
constexpr int kRound = 4;

template <class T, int NT>
struct Round {
    static constexpr int N = 16 / (int)sizeof(T);
    Raw<T, N> r[kRound];
};

// A thread's sum while it goes over its pieces.  The exponents are v * scale - reference with one rounding, the reference being m * scale rounded to 32 bits:
// an exact number that all terms share, so what its rounding is off by is made up for once, in the end (a subtraction and a scaling take an instruction an
// element more).  Where m * scale is not small beside 2^24 that would be too much, or the product not finite: there `reference` is a NaN, and the difference is taken first, which
// keeps logits of the type's lowest value, and temperatures near 0, finite.
constexpr float kNear = 4194304.0f;     // 2^22

struct Tally {
    float m, s, reference;
};

__device__ __forceinline__ Tally no_tally() { return Tally{kLowest, 0.0f, NAN}; }

// what the terms of a tally are too large by, as an exponent
__device__ __forceinline__ float excess(const Tally &a, float scale) { return a.reference == a.reference ? __builtin_fmaf(a.m, scale, -a.reference) : 0.0f; }

__device__ __forceinline__ Mass mass_of(const Tally &a, float scale) { return Mass{a.m, a.s * __builtin_amdgcn_exp2f(-excess(a, scale))}; }

// one piece: N logits; the largest of them
template <int N>
__device__ __forceinline__ float add_piece(const float (&v)[N], float scale, Tally &a)
{
    float m = v[0];
#pragma unroll
    for (int k = 1; k < N; ++k) m = fmaxf(m, v[k]);
    if (m > a.m) {
        const Mass before = mass_of(a, scale);
        const float reference = m * scale;
        a.m = m;
        a.reference = fabsf(reference) <= kNear ? reference : NAN;
        a.s = before.s * power(before.m, m, scale) * __builtin_amdgcn_exp2f(excess(a, scale));
    }
    if (a.reference == a.reference) {
#pragma unroll
        for (int k = 0; k < N; ++k) a.s += __builtin_amdgcn_exp2f(__builtin_fmaf(v[k], scale, -a.reference));
    } else {
#pragma unroll
        for (int k = 0; k < N; ++k) a.s += power(v[k], a.m, scale);
    }
    return m;
}

// A round of whole pieces without a look for their largest logits: the reference is one of the row's logits, so the sum is 1 at least, and a sum past kHigh (or a
// NaN), which asks for a larger reference, is seen in the end.  An exponent y is off by up to 2^-24 y, and its term by as much of itself: 2^-20 for terms of up to 2^20 (2^-17 for
// terms of up to 2^96, which fit a float as well: a sum that is mostly one of them was off by 43 of its roundings).  masked(v, u) may take logits out of piece u.
constexpr float kHigh = 1048576.0f;     // 2^20

template <class T, int NT, class F>
__device__ __forceinline__ bool add_whole_round(const Round<T, NT> &of, float scale, Tally &a, F masked)
{
    constexpr int N = 16 / (int)sizeof(T);
    float t[kRound];
#pragma unroll
    for (int u = 0; u < kRound; ++u) {
        float v[N];
        unpack(of.r[u], v);
        masked(v, u);
        t[u] = 0.0f;
#pragma unroll
        for (int k = 0; k < N; ++k) t[u] += __builtin_amdgcn_exp2f(__builtin_fmaf(v[k], scale, -a.reference));
    }
    const float s = a.s + ((t[0] + t[1]) + (t[2] + t[3]));
    if (!(s < kHigh)) return false;
    a.s = s;
    return true;
}

// a value of lane k of each group of W, k the same in all of a group
template <int W>
__device__ __forceinline__ int of_group(int v, int k)
{
    if constexpr (W == 64) return __builtin_amdgcn_readlane(v, k);
    else return __shfl(v, k, W);
}

// over groups of W lanes: everyone's sum brought to the largest logit first.  All lanes get the first one's bits: the product and the first sum become one fused
// multiply-add, whose rounding is another one in either lane of a pair.
template <int W>
__device__ __forceinline__ Mass join_lanes(Mass a, float scale)
{
    const float m = lane_max<W>(a.m), s = lane_sum<W>(a.s * power(a.m, m, scale));
    return Mass{m, __builtin_bit_cast(float, of_group<W>(__builtin_bit_cast(int, s), 0))};
}

// over a workgroup, the same in all threads; the caller's LDS is free again behind the next barrier
template <int NT>
__device__ __forceinline__ Mass join_mass(Mass a, float scale, Mass *lds)
{
    a = join_lanes<64>(a, scale);
    if constexpr (NT > 64) {
        if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = a;
        __syncthreads();
        float m = lds[0].m;
#pragma unroll
        for (int w = 1; w < NT / 64; ++w) m = fmaxf(m, lds[w].m);
        float s = 0.0f;
#pragma unroll
        for (int w = 0; w < NT / 64; ++w) s += lds[w].s * power(lds[w].m, m, scale);
        a = Mass{m, s};
    }
    return a;
}

// the sum over groups of W lanes, 16 or 64, the same bits in all of a group (sums of two lanes each, whichever of them asks).  Between registers: through LDS six
// exchanges of two halves are a microsecond.
template <int W>
__device__ __forceinline__ double group_sum(double v)
{
    static_assert(W == 16 || W == 64, "lanes of a row");
    const int lane = threadIdx.x & 63;
    const auto with = [&](uint64_t partner) { v += __builtin_bit_cast(double, partner); };
    with(of_partner<1>(__builtin_bit_cast(uint64_t, v), lane));
    with(of_partner<2>(__builtin_bit_cast(uint64_t, v), lane));
    with(of_partner<7>(__builtin_bit_cast(uint64_t, v), lane));
    with(of_partner<15>(__builtin_bit_cast(uint64_t, v), lane));
    if constexpr (W == 64) {
        with(of_partner<16>(__builtin_bit_cast(uint64_t, v), lane));
        with(of_partner<32>(__builtin_bit_cast(uint64_t, v), lane));
    }
    return v;
}

// log x in 64 bits for x > 0: x = 2^e m, sqrt(1/2) <= m < sqrt(2), log m = 2 atanh((m - 1) / (m + 1)), |argument| <= 0.1716, whose series
// is below 2^-53 of it behind ten terms.  A NaN or an infinity gives a NaN.  (The library's functions are two and three times as long, and what runs once a row
// or a launch waits for its instructions.)
__device__ __forceinline__ double log_of(double x)
{
    double m = __builtin_amdgcn_frexp_mant(x);
    int e = __builtin_amdgcn_frexp_exp(x);
    if (m < 0.70710678118654752) m *= 2.0, e -= 1;
    const double s = (m - 1.0) / (m + 1.0), q = s * s;
    double t = 1.0 / 19;
    t = __builtin_fma(t, q, 1.0 / 17);
    t = __builtin_fma(t, q, 1.0 / 15);
    t = __builtin_fma(t, q, 1.0 / 13);
    t = __builtin_fma(t, q, 1.0 / 11);
    t = __builtin_fma(t, q, 1.0 / 9);
    t = __builtin_fma(t, q, 1.0 / 7);
    t = __builtin_fma(t, q, 1.0 / 5);
    t = __builtin_fma(t, q, 1.0 / 3);
    const double half = __builtin_fma(t * q, s, s);
    return __builtin_fma((double)e, 0.69314718055994531, half + half);
}

// e^x in 64 bits: x = n log 2 + r, |r| <= 0.3466, whose series is below 2^-51 of it behind thirteen terms; below e^-745 zero.  An infinity above gives a NaN.
__device__ __forceinline__ double exp_of(double x)
{
    const double n = __builtin_rint(x * 1.4426950408889634);
    double r = __builtin_fma(n, -0.69314718055994529, x);
    r = __builtin_fma(n, -2.3190468138462996e-17, r);
    double t = 1.0 / 479001600;
    t = __builtin_fma(t, r, 1.0 / 39916800);
    t = __builtin_fma(t, r, 1.0 / 3628800);
    t = __builtin_fma(t, r, 1.0 / 362880);
    t = __builtin_fma(t, r, 1.0 / 40320);
    t = __builtin_fma(t, r, 1.0 / 5040);
    t = __builtin_fma(t, r, 1.0 / 720);
    t = __builtin_fma(t, r, 1.0 / 120);
    t = __builtin_fma(t, r, 1.0 / 24);
    t = __builtin_fma(t, r, 1.0 / 6);
    t = __builtin_fma(t, r, 0.5);
    t = __builtin_fma(t * r, r, r) + 1.0;
    return x < -745.0 ? 0.0 : __builtin_ldexp(t, (int)n);
}

// The pieces first + tid + u * NT, u < kRound, of a row of n logits, where they lie before `end`.  A round all of whose pieces are whole ones needs no look at
// any of them, and a scalar address.
template <bool STREAM, class T, int NT>
__device__ __forceinline__ void read_round(Round<T, NT> &to, const T *row, uint32_t first, uint32_t end, uint32_t n)
{
    constexpr int N = 16 / (int)sizeof(T);
    const uint32_t tid = threadIdx.x, whole = n / N < end ? n / N : end;
    if (first + kRound * NT <= whole) {
        typedef const typename Raw<T, N>::Wide *From;
#pragma unroll
        for (int u = 0; u < kRound; ++u) {
            const From from = (From)(row + (int64_t)(first + u * NT) * N) + tid;
            if constexpr (STREAM) to.r[u].a = __builtin_nontemporal_load(from);
            else to.r[u].a = *from;
        }
    } else {
#pragma unroll
        for (int u = 0; u < kRound; ++u) {
            const uint32_t p = first + tid + u * NT;
            to.r[u] = raw_at<N, STREAM>(row, (int64_t)p * N, (int64_t)(p < end ? n : 0));
        }
    }
}

// What lies behind the row's end is -infinity.
template <int N, class T>
__device__ __forceinline__ void piece_logits(Raw<T, N> r, uint32_t p, uint32_t n, float (&v)[N])
{
    settle(r, (int64_t)p * N, (int64_t)n);
    unpack(r, v);
    if (p >= n / N)
#pragma unroll
        for (int k = 0; k < N; ++k) v[k] = (uint64_t)p * N + k < n ? v[k] : -INFINITY;
}

// f(logits, piece, its number in the round) for each piece of a round
template <class T, int NT, class F>
__device__ __forceinline__ void each_piece(const Round<T, NT> &of, uint32_t first, uint32_t end, uint32_t n, F f)
{
    constexpr int N = 16 / (int)sizeof(T);
    const uint32_t tid = threadIdx.x, whole = n / N < end ? n / N : end;
    if (first + kRound * NT <= whole) {
#pragma unroll
        for (int u = 0; u < kRound; ++u) {
            float v[N];
            unpack(of.r[u], v);
            f(v, first + tid + u * NT, u);
        }
    } else {
#pragma unroll 1
        for (int u = 0; u < kRound; ++u) {
            const uint32_t p = first + tid + u * NT;
            if (p >= end) continue;
            float v[N];
            piece_logits<N>(u == 0 ? of.r[0] : u == 1 ? of.r[1] : u == 2 ? of.r[2] : of.r[3], p, n, v);
            f(v, p, u);
        }
    }
}

}  // namespace kannet
