// Shared by the operators of kan_net.h: element types, rows in pieces of eight channels, sums over the lanes of a row.
#pragma once
#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>
#include "kan_net.h"
#include "kan_launch.hpp"

namespace kannet {

namespace prof = ::kanprof;

constexpr size_t kAlign = 256;
inline size_t align_up(size_t v) { return (v + kAlign - 1) / kAlign * kAlign; }
inline bool bad_workspace(const void *ws, size_t have, size_t need) { return need && (!ws || (uintptr_t)ws % kAlign != 0 || have < need); }
inline size_t size_of(int type) { return type == KAN_F32 ? 4 : 2; }
inline bool known_type(int type) { return type == KAN_F32 || type == KAN_BF16; }
inline bool misplaced(const void *p, int type) { return ((uintptr_t)p % size_of(type)) != 0; }
inline bool misplaced8(const void *p) { return ((uintptr_t)p % 8) != 0; }
inline int status_of(hipError_t e) { return e == hipSuccess ? KAN_OK : KAN_ERR_HIP; }
template <class I>
constexpr I div_up(I a, I b) { return (a + b - 1) / b; }

struct bf16 { uint16_t bits; };

template <class T>
inline constexpr bool is_float = false;
template <>
inline constexpr bool is_float<float> = true;

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef u32x2 u32x2_a2 __attribute__((aligned(2)));     // rows of odd length start at any element: the wide accesses of global memory need
typedef u32x4 u32x4_a2 __attribute__((aligned(2)));     // no more than the element's alignment
typedef u32x4 u32x4_a4 __attribute__((aligned(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

__device__ __forceinline__ float widen(float v) { return v; }
__device__ __forceinline__ float widen(bf16 v) { return __builtin_bit_cast(float, (uint32_t)v.bits << 16); }

__device__ __forceinline__ uint32_t two_bf16(float lo, float hi)       // rounded to nearest even
{
    return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{lo, hi}), bf16x2));
}

__device__ __forceinline__ void put(float *p, float v) { *p = v; }
__device__ __forceinline__ void put(bf16 *p, float v) { p->bits = (uint16_t)two_bf16(v, v); }

// N consecutive elements of a row as they lie in memory, what a lane reads or writes with one access: four of either type, or eight of bf16.
// A row's accesses have to lie side by side over the lanes: eight floats a lane in two accesses 32 bytes apart, each of which leaves every
// second half line, copied 500 MB at 3.7 TB/s with streaming stores and 5.8 side by side.
template <class T, int N>
struct Raw;
template <>
struct Raw<float, 4> {
    typedef u32x4_a4 Wide;
    u32x4 a;
};
template <>
struct Raw<bf16, 4> {
    typedef u32x2_a2 Wide;
    u32x2 a;
};
template <>
struct Raw<bf16, 8> {
    typedef u32x4_a2 Wide;
    u32x4 a;
};

template <class T, int N>
__device__ __forceinline__ Raw<T, N> no_raw()
{
    Raw<T, N> r;
    r.a = 0u;
    return r;
}

// fewer than N elements, one by one: only where a whole row is that short
template <int N>
__device__ __forceinline__ Raw<float, N> raw_few(const float *p, int count)
{
    Raw<float, N> r = no_raw<float, N>();
#pragma unroll
    for (int k = 0; k < N; ++k)
        if (k < count) r.a[k] = ((const uint32_t *)p)[k];
    return r;
}

template <int N>
__device__ __forceinline__ Raw<bf16, N> raw_few(const bf16 *p, int count)
{
    Raw<bf16, N> r = no_raw<bf16, N>();
#pragma unroll
    for (int k = 0; k < N / 2; ++k) {
        if (2 * k < count) r.a[k] = p[2 * k].bits;
        if (2 * k + 1 < count) r.a[k] |= (uint32_t)p[2 * k + 1].bits << 16;
    }
    return r;
}

// The elements c .. c + N - 1 of a row of n, c a multiple of N.  Where the row ends among them, its last N are read instead, with the same
// access as everywhere (element by element, a row's end costs as many waits as it has elements: 771 channels 60 us, 768 42 us), and settle()
// brings them to their places, zeros behind them: once they are needed, so that a read ahead is not waited for.
template <int N, bool NT = false, class T, class I>
__device__ __forceinline__ Raw<T, N> raw_at(const T *row, I c, I n)
{
    const I left = n - c;
    if (left <= 0) return no_raw<T, N>();
    if (left < N && c == 0) return raw_few<N>(row, (int)left);
    Raw<T, N> r;
    typedef const typename Raw<T, N>::Wide *From;       // (a template parameter of this type would lose its alignment)
    const T *p = row + (left < N ? n - N : c);
    if constexpr (NT) r.a = __builtin_nontemporal_load((From)p);
    else r.a = *(From)p;
    return r;
}

__device__ __forceinline__ void move_down(Raw<float, 4> &r, int by)
{
    if (by & 2) r.a = u32x4{r.a.z, r.a.w, 0u, 0u};
    if (by & 1) r.a = u32x4{r.a.y, r.a.z, r.a.w, 0u};
}

__device__ __forceinline__ void move_down(Raw<bf16, 4> &r, int by)
{
    if (by & 2) r.a = u32x2{r.a.y, 0u};
    if (by & 1) r.a = u32x2{r.a.x >> 16 | r.a.y << 16, r.a.y >> 16};
}

__device__ __forceinline__ void move_down(Raw<bf16, 8> &r, int by)
{
    if (by & 4) r.a = u32x4{r.a.z, r.a.w, 0u, 0u};
    if (by & 2) r.a = u32x4{r.a.y, r.a.z, r.a.w, 0u};
    if (by & 1)
        r.a = u32x4{r.a.x >> 16 | r.a.y << 16, r.a.y >> 16 | r.a.z << 16, r.a.z >> 16 | r.a.w << 16, r.a.w >> 16};
}

template <class T, int N, class I>
__device__ __forceinline__ void settle(Raw<T, N> &r, I c, I n)
{
    const I left = n - c;
    if (left < N && left > 0 && c > 0) move_down(r, N - (int)left);
}

template <int N>
__device__ __forceinline__ void unpack(const Raw<float, N> &r, float *v)
{
#pragma unroll
    for (int k = 0; k < N; ++k) {
        const uint32_t w = r.a[k];          // a bit cast of the vector's element itself takes element 0 (hipcc 7.2)
        v[k] = __builtin_bit_cast(float, w);
    }
}

template <int N>
__device__ __forceinline__ void unpack(const Raw<bf16, N> &r, float *v)
{
#pragma unroll
    for (int k = 0; k < N / 2; ++k) {
        const uint32_t w = r.a[k];
        v[2 * k] = __builtin_bit_cast(float, w << 16);
        v[2 * k + 1] = __builtin_bit_cast(float, w & 0xFFFF0000u);
    }
}

template <int N>
__device__ __forceinline__ Raw<float, N> pack(const float *, const float *v)
{
    Raw<float, N> r;
#pragma unroll
    for (int k = 0; k < N; ++k) r.a[k] = __builtin_bit_cast(uint32_t, v[k]);
    return r;
}

template <int N>
__device__ __forceinline__ Raw<bf16, N> pack(const bf16 *, const float *v)
{
    Raw<bf16, N> r;
#pragma unroll
    for (int k = 0; k < N / 2; ++k) r.a[k] = two_bf16(v[2 * k], v[2 * k + 1]);
    return r;
}

template <int N, bool NT = false, class T, class I>
__device__ __forceinline__ void store_at(T *row, I c, I n, const float *v)
{
    const I left = n - c;
    if (left >= N) {
        typedef typename Raw<T, N>::Wide *To;
        const auto w = pack<N>(row, v).a;
        if constexpr (NT) __builtin_nontemporal_store(w, (To)(row + c));
        else *(To)(row + c) = w;
    } else {
#pragma unroll
        for (int k = 0; k < N; ++k)
            if (k < left) put(row + c + k, v[k]);
    }
}

// Eight channels a lane of a row of n, those of all lanes a block of 8 * lanes that starts at `base`.  PAIR false (bf16 throughout): eight
// side by side, one access.  PAIR true (an fp32 array takes part): four from either half of the block, so that the accesses of both types lie side
// by side over the lanes.
template <bool PAIR>
__device__ __forceinline__ int channel_of(int base, int lane, int lanes, int k)
{
    return PAIR ? base + (k < 4 ? 0 : 4 * lanes - 4) + 4 * lane + k : base + 8 * lane + k;
}

template <class T, bool PAIR>
struct Eight {
    Raw<T, PAIR ? 4 : 8> a;
    Raw<T, PAIR ? 4 : 8> b;         // PAIR only
};

template <bool PAIR, bool NT = false, class T>
__device__ __forceinline__ Eight<T, PAIR> eight_at(const T *row, int base, int lane, int lanes, int n)
{
    Eight<T, PAIR> e;
    if constexpr (PAIR) {
        e.a = raw_at<4, NT>(row, base + 4 * lane, n);
        e.b = raw_at<4, NT>(row, base + 4 * lanes + 4 * lane, n);
    } else {
        e.a = raw_at<8, NT>(row, base + 8 * lane, n);
    }
    return e;
}

template <bool PAIR, class T>
__device__ __forceinline__ void unpack_at(Eight<T, PAIR> e, int base, int lane, int lanes, int n, float (&v)[8])
{
    if constexpr (PAIR) {
        settle(e.a, base + 4 * lane, n);
        settle(e.b, base + 4 * lanes + 4 * lane, n);
        unpack(e.a, v);
        unpack(e.b, v + 4);
    } else {
        settle(e.a, base + 8 * lane, n);
        unpack(e.a, v);
    }
}

template <bool PAIR, class T>
__device__ __forceinline__ void load_eight(const T *row, int base, int lane, int lanes, int n, float (&v)[8])
{
    unpack_at<PAIR>(eight_at<PAIR>(row, base, lane, lanes, n), base, lane, lanes, n, v);
}

template <bool PAIR, bool NT = false, class T>
__device__ __forceinline__ void store_eight(T *row, int base, int lane, int lanes, int n, const float (&v)[8])
{
    if constexpr (PAIR) {
        store_at<4, NT>(row, base + 4 * lane, n, v);
        store_at<4, NT>(row, base + 4 * lanes + 4 * lane, n, v + 4);
    } else {
        store_at<8, NT>(row, base + 8 * lane, n, v);
    }
}

// Both values of a pair of lanes that lie in different halves of W lanes: the lane's own and its partner's, in either order.
template <int W>
__device__ __forceinline__ f32x2 both_halves(float v)
{
    const int i = __builtin_bit_cast(int, v);
    if constexpr (W >= 32) {
        const auto t = W == 32 ? __builtin_amdgcn_permlane16_swap(i, i, false, false) : __builtin_amdgcn_permlane32_swap(i, i, false, false);
        return f32x2{__builtin_bit_cast(float, (int)t[0]), __builtin_bit_cast(float, (int)t[1])};
    }
    const int o = W == 2 ? __builtin_amdgcn_update_dpp(0, i, 0xB1, 0xF, 0xF, true)
                : W == 4 ? __builtin_amdgcn_update_dpp(0, i, 0x4E, 0xF, 0xF, true)
                : W == 8 ? __builtin_amdgcn_update_dpp(0, i, 0x141, 0xF, 0xF, true)
                         : __builtin_amdgcn_update_dpp(0, i, 0x140, 0xF, 0xF, true);
    return f32x2{v, __builtin_bit_cast(float, o)};
}

// the sum over each group of W lanes, the same bits in all of them
template <int W>
__device__ __forceinline__ float lane_sum(float v)
{
    if constexpr (W > 2) v = lane_sum<W / 2>(v);
    const f32x2 t = both_halves<W>(v);
    return t.x + t.y;
}

// the largest of each group of W lanes
template <int W>
__device__ __forceinline__ float lane_max(float v)
{
    if constexpr (W > 2) v = lane_max<W / 2>(v);
    const f32x2 t = both_halves<W>(v);
    return fmaxf(t.x, t.y);
}

// Sums of N values over the lanes that share a row, TPR at most: within a wave, or over the waves through LDS, with one barrier a call (two
// sets of slots taken in turn: a wave that writes a set again has passed the barrier of the call in between, and with it every wave's
// reads of that set).  Slots of waves that are not there hold zeros from clear() on.
template <int TPR>
struct RowSum {
    static constexpr int kWaves = TPR > 512 ? 16 : TPR > 64 ? TPR / 64 : 1, kMost = 2;
    static constexpr int kSlots = TPR > 64 ? 2 * kMost * kWaves : 1;
    float *slots;       // [2][kWaves][kMost]
    int turn = 0, wave = 0;
    __device__ __forceinline__ void clear(int lane)
    {
        if constexpr (TPR > 64) {
            wave = lane >> 6;
            if (lane < kSlots) slots[lane] = 0.0f;
            __syncthreads();
        }
    }
    template <int N>
    __device__ __forceinline__ void sum(float (&v)[N])
    {
        static_assert(N <= kMost, "slots");
        if constexpr (TPR <= 64) {
#pragma unroll
            for (int i = 0; i < N; ++i) v[i] = lane_sum<TPR>(v[i]);
        } else {
            float *s = slots + turn * kWaves * kMost;
            turn ^= 1;
#pragma unroll
            for (int i = 0; i < N; ++i) {
                v[i] = lane_sum<64>(v[i]);
                if ((threadIdx.x & 63) == 0) s[wave * kMost + i] = v[i];
            }
            __syncthreads();
#pragma unroll
            for (int i = 0; i < N; ++i) v[i] = lane_sum<kWaves>(s[(threadIdx.x & (kWaves - 1)) * kMost + i]);
        }
    }
    __device__ __forceinline__ float operator()(float v)
    {
        float a[1] = {v};
        sum(a);
        return a[0];
    }
};

// Lanes a row of n channels gets, at eight channels a lane: a power of two from 8 on, 2 * 1024 * 8 channels at most (two pieces a lane).  And
// 768 for up to 6144 channels: the block norm's backward pass has 168 registers a lane there (8192 x 6000 in two types 324 us with 1024 lanes, 190 so).
inline int lanes_of_row(int n)
{
    int t = 8;
    while (t < 1024 && t * 8 < n) t *= 2;
    return t == 1024 && n <= 768 * 8 ? 768 : t;
}

}  // namespace kannet
