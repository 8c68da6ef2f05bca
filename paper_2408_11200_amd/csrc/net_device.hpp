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

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef u32x4 u32x4_a2 __attribute__((aligned(2)));     // rows of odd length start at any element: the wide accesses of global memory need
typedef u32x4 u32x4_a4 __attribute__((aligned(4)));     // no more than the element's alignment
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

// Eight consecutive elements as they lie in memory: what a thread holds of a row it will need later.
template <class T>
struct Raw;
template <>
struct Raw<float> { u32x4 a, b; };
template <>
struct Raw<bf16> { u32x4 a; };

template <bool NT = false>
__device__ __forceinline__ Raw<float> raw8(const float *p)
{
    const u32x4_a4 *q = (const u32x4_a4 *)p;
    if constexpr (NT) return Raw<float>{__builtin_nontemporal_load(q), __builtin_nontemporal_load(q + 1)};
    else return Raw<float>{q[0], q[1]};
}

template <bool NT = false>
__device__ __forceinline__ Raw<bf16> raw8(const bf16 *p)
{
    const u32x4_a2 *q = (const u32x4_a2 *)p;
    if constexpr (NT) return Raw<bf16>{__builtin_nontemporal_load(q)};
    else return Raw<bf16>{q[0]};
}

__device__ __forceinline__ Raw<float> no_raw(const float *) { return Raw<float>{u32x4{0u, 0u, 0u, 0u}, u32x4{0u, 0u, 0u, 0u}}; }
__device__ __forceinline__ Raw<bf16> no_raw(const bf16 *) { return Raw<bf16>{u32x4{0u, 0u, 0u, 0u}}; }

// fewer than eight, one by one: only where a whole row is that short
__device__ __forceinline__ Raw<float> raw_few(const float *p, int count)
{
    Raw<float> r = no_raw(p);
    const uint32_t *q = (const uint32_t *)p;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        if (k < count) r.a[k] = q[k];
        if (4 + k < count) r.b[k] = q[4 + k];
    }
    return r;
}

__device__ __forceinline__ Raw<bf16> raw_few(const bf16 *p, int count)
{
    Raw<bf16> r = no_raw(p);
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        if (2 * k < count) r.a[k] = p[2 * k].bits;
        if (2 * k + 1 < count) r.a[k] |= (uint32_t)p[2 * k + 1].bits << 16;
    }
    return r;
}

// The elements c .. c + 7 of a row of n, c a multiple of 8.  Where the row ends among them, its last eight are read instead, with the same
// access as everywhere (element by element, a row's end costs as many waits as it has elements: 771 channels 60 us, 768 42 us), and settle()
// brings them to their places, zeros behind them: once they are needed, so that a read ahead is not waited for.
template <bool NT = false, class T, class I>
__device__ __forceinline__ Raw<T> raw_at(const T *row, I c, I n)
{
    const I left = n - c;
    if (left <= 0) return no_raw(row);
    if (left < 8 && c == 0) return raw_few(row, (int)left);
    return raw8<NT>(row + (left < 8 ? n - 8 : c));
}

__device__ __forceinline__ void move_down(Raw<float> &r, int by)
{
    if (by & 4) {
        r.a = r.b;
        r.b = u32x4{0u, 0u, 0u, 0u};
    }
    if (by & 2) {
        r.a = u32x4{r.a.z, r.a.w, r.b.x, r.b.y};
        r.b = u32x4{r.b.z, r.b.w, 0u, 0u};
    }
    if (by & 1) {
        r.a = u32x4{r.a.y, r.a.z, r.a.w, r.b.x};
        r.b = u32x4{r.b.y, r.b.z, r.b.w, 0u};
    }
}

__device__ __forceinline__ void move_down(Raw<bf16> &r, int by)
{
    if (by & 4) r.a = u32x4{r.a.z, r.a.w, 0u, 0u};
    if (by & 2) r.a = u32x4{r.a.y, r.a.z, r.a.w, 0u};
    if (by & 1)
        r.a = u32x4{r.a.x >> 16 | r.a.y << 16, r.a.y >> 16 | r.a.z << 16, r.a.z >> 16 | r.a.w << 16, r.a.w >> 16};
}

template <class T, class I>
__device__ __forceinline__ void settle(Raw<T> &r, I c, I n)
{
    const I left = n - c;
    if (left < 8 && left > 0 && c > 0) move_down(r, 8 - (int)left);
}

__device__ __forceinline__ void unpack(const Raw<float> &r, float (&v)[8])
{
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const uint32_t lo = r.a[k], hi = r.b[k];      // a bit cast of the vector's element itself takes element 0 (hipcc 7.2)
        v[k] = __builtin_bit_cast(float, lo);
        v[4 + k] = __builtin_bit_cast(float, hi);
    }
}

__device__ __forceinline__ void unpack(const Raw<bf16> &r, float (&v)[8])
{
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const uint32_t w = r.a[k];
        v[2 * k] = __builtin_bit_cast(float, w << 16);
        v[2 * k + 1] = __builtin_bit_cast(float, w & 0xFFFF0000u);
    }
}

template <bool NT = false, class T>
__device__ __forceinline__ void load8(const T *p, float (&v)[8])
{
    unpack(raw8<NT>(p), v);
}

template <bool NT = false>
__device__ __forceinline__ void store8(float *p, const float (&v)[8])
{
    u32x4 a, b;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        a[k] = __builtin_bit_cast(uint32_t, v[k]);
        b[k] = __builtin_bit_cast(uint32_t, v[4 + k]);
    }
    u32x4_a4 *q = (u32x4_a4 *)p;
    if (NT) {
        __builtin_nontemporal_store(a, q);
        __builtin_nontemporal_store(b, q + 1);
    } else {
        q[0] = a;
        q[1] = b;
    }
}

template <bool NT = false>
__device__ __forceinline__ void store8(bf16 *p, const float (&v)[8])
{
    u32x4 a;
#pragma unroll
    for (int k = 0; k < 4; ++k) a[k] = two_bf16(v[2 * k], v[2 * k + 1]);
    u32x4_a2 *q = (u32x4_a2 *)p;
    if (NT) __builtin_nontemporal_store(a, q);
    else *q = a;
}

template <bool NT = false, class T, class I>
__device__ __forceinline__ void load_at(const T *row, I c, I n, float (&v)[8])
{
    Raw<T> r = raw_at<NT>(row, c, n);
    settle(r, c, n);
    unpack(r, v);
}

template <bool NT = false, class T, class I>
__device__ __forceinline__ void store_at(T *row, I c, I n, const float (&v)[8])
{
    const I left = n - c;
    T *p = row + c;
    if (left >= 8) {
        store8<NT>(p, v);
    } else {
#pragma unroll
        for (int k = 0; k < 8; ++k)
            if (k < left) put(p + k, v[k]);
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

// the sum, or the largest value, over each group of W lanes, the same bits in all of them
template <int W>
__device__ __forceinline__ float lane_sum(float v)
{
    if constexpr (W > 2) v = lane_sum<W / 2>(v);
    const f32x2 t = both_halves<W>(v);
    return t.x + t.y;
}

template <int W>
__device__ __forceinline__ float lane_max(float v)
{
    if constexpr (W > 2) v = lane_max<W / 2>(v);
    const f32x2 t = both_halves<W>(v);
    return fmaxf(t.x, t.y);
}

// Sums of N values over the TPR lanes that share a row: within a wave, or over the TPR / 64 waves of the workgroup through LDS, with one
// barrier a call (two sets of slots taken in turn: a wave that writes a set again has passed the barrier of the call in between, and
// with it every wave's reads of that set).
template <int TPR>
struct RowSum {
    static constexpr int kWaves = TPR / 64, kMost = 2;
    static constexpr int kSlots = TPR > 64 ? 2 * kMost * kWaves : 1;
    float *slots;       // [2][kWaves][kMost]
    int turn = 0;
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
                if ((threadIdx.x & 63) == 0) s[(threadIdx.x % TPR >> 6) * kMost + i] = v[i];
            }
            __syncthreads();
#pragma unroll
            for (int i = 0; i < N; ++i) {
                v[i] = s[i];
#pragma unroll
                for (int w = 1; w < kWaves; ++w) v[i] += s[w * kMost + i];
            }
        }
    }
    __device__ __forceinline__ float operator()(float v)
    {
        float a[1] = {v};
        sum(a);
        return a[0];
    }
};

// Lanes a row of n channels gets, at eight channels a lane: a power of two from 8 on, 2 * 1024 * 8 channels at most (two pieces a lane)
inline int lanes_of_row(int n)
{
    int t = 8;
    while (t < 1024 && t * 8 < n) t *= 2;
    return t;
}

}  // namespace kannet
