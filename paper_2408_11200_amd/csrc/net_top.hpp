// The largest of many logits: keys that order them, a wave's sorted lists, values by rank over a workgroup.  Shared by the operators that look
// for likely tokens (net_logprob.hip, net_beam.hip).
#pragma once
#include "net_device.hpp"

namespace kannet {

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLowest = -3.4028234663852886e38f;

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

// of a lane that is the same for the whole wave
__device__ __forceinline__ uint64_t of_lane(uint64_t v, int lane)
{
    return (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(v >> 32), lane) << 32 | (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)v, lane);
}

// of the lane before (lane 0 keeps its own)
__device__ __forceinline__ uint64_t of_lane_before(uint64_t v)
{
    const int hi = (int)(v >> 32), lo = (int)(uint32_t)v;
    return (uint64_t)(uint32_t)__builtin_amdgcn_update_dpp(hi, hi, 0x138, 0xF, 0xF, false) << 32 |
           (uint32_t)__builtin_amdgcn_update_dpp(lo, lo, 0x138, 0xF, 0xF, false);
}

// A wave's list of keys, best first, one a lane: puts in every lane's `key` (0: none) that is above entry `top` - 1
__device__ __forceinline__ void put_in(uint64_t &list, uint64_t key, int top, int lane)
{
    uint64_t last = of_lane(list, top - 1);
    uint64_t open = __ballot(key > last);
    while (open) {
        const uint64_t k = of_lane(key, __ffsll((unsigned long long)open) - 1);
        open &= open - 1;
        if (k <= last) continue;
        const int at = __popcll(__ballot(list > k));
        const uint64_t before = of_lane_before(list);
        list = lane < at ? list : lane == at ? k : before;
        last = of_lane(list, top - 1);
    }
}

template <int CTRL>
__device__ __forceinline__ float dpp(float v)
{
    const int i = __builtin_bit_cast(int, v);
    return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, i, CTRL, 0xF, 0xF, true));
}

template <int D>
__device__ __forceinline__ float swapped(float v, int lane)
{
    const f32x2 t = both_halves<2 * D>(v);
    return (lane & D) ? t.x : t.y;
}

// of lane ^ X, X = 2^k or 2^k - 1
template <int X>
__device__ __forceinline__ float of_partner(float v, int lane)
{
    if constexpr (X == 1) return dpp<0xB1>(v);
    else if constexpr (X == 2) return dpp<0x4E>(v);
    else if constexpr (X == 3) return dpp<0x1B>(v);
    else if constexpr (X == 4) return dpp<0x1B>(dpp<0x141>(v));
    else if constexpr (X == 7) return dpp<0x141>(v);
    else if constexpr (X == 8) return dpp<0x128>(v);
    else if constexpr (X == 15) return dpp<0x140>(v);
    else if constexpr (X == 16) return swapped<16>(v, lane);
    else if constexpr (X == 31) return dpp<0x140>(swapped<16>(v, lane));
    else if constexpr (X == 32) return swapped<32>(v, lane);
    else return dpp<0x140>(swapped<16>(swapped<32>(v, lane), lane));
}

// the larger value to the lane of the pair whose bit D is clear
template <int X, int D>
__device__ __forceinline__ float ordered(float v, int lane)
{
    const float o = of_partner<X>(v, lane), hi = fmaxf(v, o), lo = fminf(v, o);
    return (lane & D) ? lo : hi;
}

// a wave's values that rise and then fall (or the other way round) in falling order
template <int D>
__device__ __forceinline__ float merged(float v, int lane)
{
    v = ordered<D, D>(v, lane);
    if constexpr (D > 1) v = merged<D / 2>(v, lane);
    return v;
}

// a wave's values in falling order: sorted halves, the second one mirrored
template <int S = 64>
__device__ __forceinline__ float sorted(float v, int lane)
{
    if constexpr (S > 2) v = sorted<S / 2>(v, lane);
    v = ordered<S - 1, S / 2>(v, lane);
    if constexpr (S > 2) v = merged<S / 4>(v, lane);
    return v;
}

// the `top`-th largest of the threads' values, the same in all threads
template <int NT>
__device__ __forceinline__ float value_of_rank(float v, int top, int lane, float *lds)
{
    v = sorted(v, lane);
    if constexpr (NT > 64) {
        lds[threadIdx.x] = v;
        __syncthreads();
        v = lds[lane];
        // of two sorted lists, the larger ones of the first against the other one backwards are the first 64 of both
        for (int w = 1; w < NT / 64; ++w) v = merged<32>(fmaxf(v, lds[w * 64 + 63 - lane]), lane);
    }
    return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), top - 1));
}

// the same networks on keys, and on what else has of_partner and above
template <int X>
__device__ __forceinline__ uint64_t of_partner(uint64_t v, int lane)
{
    const float lo = of_partner<X>(__builtin_bit_cast(float, (uint32_t)v), lane), hi = of_partner<X>(__builtin_bit_cast(float, (uint32_t)(v >> 32)), lane);
    return (uint64_t)__builtin_bit_cast(uint32_t, hi) << 32 | __builtin_bit_cast(uint32_t, lo);
}

__device__ __forceinline__ bool above(uint64_t a, uint64_t b) { return a > b; }

// Two numbers, the second one where the first ones are equal
struct Ranked {
    uint64_t rank, tie;
};

template <int X>
__device__ __forceinline__ Ranked of_partner(Ranked v, int lane) { return Ranked{of_partner<X>(v.rank, lane), of_partner<X>(v.tie, lane)}; }

__device__ __forceinline__ bool above(Ranked a, Ranked b) { return (a.rank > b.rank) | ((a.rank == b.rank) & (a.tie > b.tie)); }

__device__ __forceinline__ Ranked of_lane(Ranked v, int lane) { return Ranked{of_lane(v.rank, lane), of_lane(v.tie, lane)}; }

template <int X, int D, class K>
__device__ __forceinline__ K ordered(K v, int lane)
{
    const K o = of_partner<X>(v, lane);
    return (above(v, o) != ((lane & D) != 0)) ? v : o;
}

template <int D, class K>
__device__ __forceinline__ K merged(K v, int lane)
{
    v = ordered<D, D>(v, lane);
    if constexpr (D > 1) v = merged<D / 2>(v, lane);
    return v;
}

template <int S = 64, class K>
__device__ __forceinline__ K sorted(K v, int lane)
{
    if constexpr (S > 2) v = sorted<S / 2>(v, lane);
    v = ordered<S - 1, S / 2>(v, lane);
    if constexpr (S > 2) v = merged<S / 4>(v, lane);
    return v;
}

// of a wave's falling list and another one, backwards (entry 63 - lane), the first 64, falling
template <class K>
__device__ __forceinline__ K best_of(K list, K backwards, int lane) { return merged<32>(above(list, backwards) ? list : backwards, lane); }

// how many of `count` keys in LDS are above k
__device__ __forceinline__ int above(const uint64_t *keys, uint32_t count, uint64_t k)
{
    int n = 0;
#pragma unroll 8
    for (uint32_t i = 0; i < count; ++i) n += keys[i] > k ? 1 : 0;
    return n;
}

}  // namespace kannet
