// Order statistics inside a wave, shared by the kernels that pick the largest or smallest of many numbers (sk_logprobs.hip, sk_evict.hip).
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace sk_order {

// Orders floats as unsigned numbers: -0 is +0; a NaN has no place of its own.
__device__ __forceinline__ uint32_t rank_of(const float x)
{
    const uint32_t u = __float_as_uint(x + 0.0f);
    return u ^ (uint32_t)((int32_t)u >> 31 | INT32_MIN);
}
__device__ __forceinline__ float value_of(const uint32_t r) { return __uint_as_float(r & 0x80000000u ? r ^ 0x80000000u : ~r); }
constexpr uint32_t kRankNone = 0x007fffffu;       // of -inf

__device__ __forceinline__ int lanes(const bool b) { return __popcll(__ballot(b)); }
__device__ __forceinline__ int lanes_before(const uint64_t m)
{
    return __builtin_amdgcn_mbcnt_hi((uint32_t)(m >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)m, 0));
}
// Says where the LDS writes of a wave's lanes end that other lanes of it read (no instruction: a wave's LDS accesses stay in order).
__device__ __forceinline__ void wave_order() { __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront"); __builtin_amdgcn_wave_barrier(); }

// Maximum over the 64 lanes, in every lane, by lane exchanges within the vector unit.
template <int CTRL> __device__ __forceinline__ uint32_t dpp(const uint32_t x) { return __builtin_amdgcn_update_dpp(0u, x, CTRL, 0xf, 0xf, true); }
__device__ __forceinline__ uint32_t wave_max(uint32_t x)
{
    x = max(x, dpp<0xB1>(x)); x = max(x, dpp<0x4E>(x)); x = max(x, dpp<0x141>(x)); x = max(x, dpp<0x140>(x));
    { const auto r = __builtin_amdgcn_permlane16_swap(x, x, false, false); x = max((uint32_t)r[0], (uint32_t)r[1]); }
    { const auto r = __builtin_amdgcn_permlane32_swap(x, x, false, false); return max((uint32_t)r[0], (uint32_t)r[1]); }
}

__device__ __forceinline__ int wave_sum(int x)
{
    x += (int)dpp<0xB1>((uint32_t)x); x += (int)dpp<0x4E>((uint32_t)x); x += (int)dpp<0x141>((uint32_t)x); x += (int)dpp<0x140>((uint32_t)x);
    { const auto r = __builtin_amdgcn_permlane16_swap((uint32_t)x, (uint32_t)x, false, false); x = (int)r[0] + (int)r[1]; }
    { const auto r = __builtin_amdgcn_permlane32_swap((uint32_t)x, (uint32_t)x, false, false); return (int)r[0] + (int)r[1]; }
}

// Sum over the lanes up to and with this one: within a row of 16 lanes by shifts of it, then the last lane of a row added to the
// rows behind it.
__device__ __forceinline__ int wave_running_sum(int x)
{
    x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, true); x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, true);
    x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, true); x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, true);
    x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false); x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false);
    return x;
}

// A bound that at least k of the wave's numbers reach (N of them in a lane; 0: none), as high as it can be, or one that exactly k reach;
// `hits` receives how many do.  At least k are above 0.  Found by counting lanes, from the highest bit in which the numbers differ down.
template <int N>
__device__ __forceinline__ uint32_t bound_of(const uint32_t (&r)[N], const int k, int& hits)
{
    uint32_t hi = 0, lo = 0;
    hits = 0;
#pragma unroll
    for (int j = 0; j < N; ++j) {
        hi = max(hi, r[j]);
        lo = max(lo, r[j] ? ~r[j] : 0u);                  // (of the complement: the smallest)
        hits += lanes(r[j] != 0);
    }
    hi = __builtin_amdgcn_readfirstlane(wave_max(hi));
    lo = ~__builtin_amdgcn_readfirstlane(wave_max(lo));
    if (hits == k || hi == lo) return lo;
    // Two bits at a time: three candidates counted side by side take little longer than one, a dependent chain of a compare, a
    // count of lanes and a branch.
    int b = 31 - __builtin_clz(hi ^ lo);
    uint32_t t = hi & ~((2u << b) - 1);                   // what all have in common
    for (b &= ~1; b >= 0; b -= 2) {
        const uint32_t c1 = t | 1u << b, c2 = t | 2u << b, c3 = t | 3u << b;
        int n1 = 0, n2 = 0, n3 = 0;
#pragma unroll
        for (int j = 0; j < N; ++j) { n1 += lanes(r[j] >= c1); n2 += lanes(r[j] >= c2); n3 += lanes(r[j] >= c3); }
        if (n3 >= k) { t = c3; hits = n3; }
        else if (n2 >= k) { t = c2; hits = n2; }
        else if (n1 >= k) { t = c1; hits = n1; }
        if (hits == k) break;
    }
    return t;
}

}  // namespace sk_order
