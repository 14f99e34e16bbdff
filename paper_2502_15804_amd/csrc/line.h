// The line of all pairs: workgroups find their share of it by themselves, from numbers that only the GPU knows.
#pragma once
#include <hip/hip_runtime.h>

#include <cstdint>
#include <type_traits>

namespace fairkv {

// x plus those of the lanes below, by steps of the wave's own data paths; 32 or 64 bits.
template <class T>
__device__ __forceinline__ T wave_upto(T x)
{
    auto step = [&](auto ctrl, auto rows, auto banks) __attribute__((always_inline)) {
        const uint32_t lo = __builtin_amdgcn_update_dpp(0, static_cast<int>(x), ctrl(), rows(), banks(), false);
        if constexpr (sizeof(T) == 8) {
            const uint32_t hi = __builtin_amdgcn_update_dpp(0, static_cast<int>(x >> 32), ctrl(), rows(), banks(), false);
            x += static_cast<int64_t>((static_cast<uint64_t>(hi) << 32) | lo);
        } else {
            x += static_cast<T>(lo);
        }
    };
#define FAIRKV_N(n) std::integral_constant<int, n>{}
    step(FAIRKV_N(0x111), FAIRKV_N(0xf), FAIRKV_N(0xf));      // from 1, 2, 4, 8 lanes below in the row of 16
    step(FAIRKV_N(0x112), FAIRKV_N(0xf), FAIRKV_N(0xf));
    step(FAIRKV_N(0x114), FAIRKV_N(0xf), FAIRKV_N(0xf));
    step(FAIRKV_N(0x118), FAIRKV_N(0xf), FAIRKV_N(0xf));
    step(FAIRKV_N(0x142), FAIRKV_N(0xa), FAIRKV_N(0xf));      // from the end of the row below, of both rows below
    step(FAIRKV_N(0x143), FAIRKV_N(0xc), FAIRKV_N(0xf));
#undef FAIRKV_N
    return x;
}

// A share of the line of pairs 0 .. n_pairs - 1, each `units(pair)` >= 0 long: units begin .. begin + left - 1 of pair `pair` and of
// those behind it.  left is 0 where the line has ended.  Called by all NT threads of a workgroup; the same for all of them.
struct LineShare {
    int pair;
    int64_t begin, left;
    int64_t at, total;                // the share's place in the line, and the whole line's length
};
template <int NT, class Units>
__device__ __forceinline__ LineShare line_share(int n_pairs, int n_slots, int slot, Units units)
{
    constexpr int NW = NT / 64;
    __shared__ int64_t totals[NW];
    __shared__ LineShare found;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int run = (n_pairs + NT - 1) / NT, p0 = min(static_cast<int>(threadIdx.x) * run, n_pairs), p1 = min(p0 + run, n_pairs);
    int64_t mine = 0;
    for (int p = p0; p < p1; ++p) mine += units(p);
    const int64_t upto = wave_upto(mine);
    if (lane == 63) totals[wave] = upto;
    if (threadIdx.x == 0) found = LineShare{n_pairs, 0, 0, 0, 0};
    __syncthreads();
    int64_t before = upto - mine, total = 0;
#pragma unroll
    for (int w = 0; w < NW; ++w) {
        if (w < wave) before += totals[w];
        total += totals[w];
    }
    // total / n_slots units each, the first of them one more: no share is more than one unit longer than another
    const int64_t each = total / n_slots, more = total - each * n_slots;
    const int64_t begin = each * slot + min(static_cast<int64_t>(slot), more), left = each + (slot < more ? 1 : 0);
    if (left > 0 && before <= begin && begin < before + mine) {
        int p = p0;
        for (; p < p1 - 1; ++p) {
            const int64_t u = units(p);
            if (begin < before + u) break;
            before += u;
        }
        found = LineShare{p, begin - before, left, begin, total};
    }
    __syncthreads();
    auto uniform = [](int64_t x) __attribute__((always_inline)) {      // the same for all lanes: in scalar registers
        const uint32_t lo = __builtin_amdgcn_readfirstlane(static_cast<int>(x)), hi = __builtin_amdgcn_readfirstlane(static_cast<int>(x >> 32));
        return static_cast<int64_t>((static_cast<uint64_t>(hi) << 32) | lo);
    };
    return LineShare{__builtin_amdgcn_readfirstlane(found.pair), uniform(found.begin), uniform(found.left), uniform(found.at), uniform(total)};
}

// The first pair behind `pair` that has units, n_pairs if none has: 64 are looked at at once.
template <class Units>
__device__ __forceinline__ int next_pair(int pair, int n_pairs, Units units)
{
    const int lane = threadIdx.x & 63;
    for (int p = pair + 1; p < n_pairs; p += 64) {
        const uint64_t some = __builtin_amdgcn_ballot_w64(p + lane < n_pairs && units(min(p + lane, n_pairs - 1)) > 0);
        if (some) return p + __builtin_ctzll(some);
    }
    return n_pairs;
}

}  // namespace fairkv
