// Which rows of a growing cache stay: the protected ones, and the heaviest of the others up to a budget.
//
// Of a pair's len rows the first `sink` and the last `recent` are protected.  Every other one, a candidate, has the value
//     x[t] = max w[u] over the candidates u with |u - t| <= pool / 2,
// and of all candidates of a group (a pair, or the pairs of a sequence) those with the largest values stay, as many as the budget leaves room
// for behind the protected rows; of equal values the one of the lower head, then of the lower token.
//
// Values are compared as 32-bit whole numbers in the order of the floats.  The least one that stays is found digit by digit from the top, by
// counting how many candidates have which digit among those that share the digits found so far; then the rows are listed in their order.
#pragma once
#include "cache_rows.h"

namespace fairkv {

struct SelectArgs {
    RowMap rows;
    const float *weights;                 // [n_rows]
    const int32_t *len, *budget;          // [B * Hkv]; [groups]
    int32_t *keep, *n_keep, *bad;         // [B * Hkv][max_keep], [B * Hkv], [1] or null
    int32_t B, Hkv, max_len, max_keep, half, sink, recent, per_group;      // per_group: pairs of a group, 1 or Hkv
};

constexpr int kSelectThreads = 1024;

// The float's place in the order of floats.  -0 is +0, and a NaN is below all numbers (fmaxf has left it out).
__device__ __forceinline__ uint32_t order_of(float x)
{
    const uint32_t u = __float_as_uint(x + 0.f);
    return u ^ (u & 0x80000000u ? 0xffffffffu : 0x80000000u);
}

struct Candidates {                       // of a pair: its length, and the candidates' first token and the one behind the last
    int32_t len, first, end;
    __device__ __forceinline__ Candidates(const SelectArgs &a, int pair)
    {
        len = min(max(a.len[pair], 0), a.max_len);
        first = min(a.sink, len);
        end = max(first, len - min(a.recent, len));
    }
};

__device__ __forceinline__ uint32_t value_of(const SelectArgs &a, int pair, const Candidates &c, int32_t t)
{
    float x = -INFINITY;
    for (int32_t u = max(c.first, t - a.half); u <= min(c.end - 1, t + a.half); ++u) {
        const int64_t row = a.rows.row(pair, u);
        if (row >= 0) x = fmaxf(x, a.weights[row]);
    }
    return order_of(x);
}

// Sum over the workgroup of what the threads before this one have, and of all.
struct Before {
    int32_t before, total;
};
template <int NT>
__device__ __forceinline__ Before count_before(bool x, int32_t *of_waves /* LDS [NT / 64] */)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const uint64_t here = __builtin_amdgcn_ballot_w64(x);
    __syncthreads();
    if (lane == 0) of_waves[wave] = __builtin_popcountll(here);
    __syncthreads();
    Before r{__builtin_popcountll(here & ((1ull << lane) - 1)), 0};
    for (int w = 0; w < NT / 64; ++w) {
        if (w < wave) r.before += of_waves[w];
        r.total += of_waves[w];
    }
    return r;
}

// One workgroup per group.
__global__ __launch_bounds__(kSelectThreads) void fairkv_select_kernel(SelectArgs a)
{
    constexpr int NT = kSelectThreads;
    __shared__ int32_t bins[256], of_waves[NT / 64], of_waves2[NT / 64];
    __shared__ int64_t room_left;
    __shared__ uint32_t digit_found;
    const int group = blockIdx.x, first_pair = group * a.per_group;
    auto has_row = [&](int pair, int32_t t) { return a.rows.row(pair, t) >= 0; };

    // ---- how many candidates stay: what the budget leaves behind the protected rows ----
    int64_t room = 0, candidates = 0;
    {
        int32_t mine = 0, also = 0;
        for (int p = first_pair; p < first_pair + a.per_group; ++p) {
            const Candidates c(a, p);
            for (int32_t t = threadIdx.x; t < c.len; t += NT)
                if (has_row(p, t)) {
                    if (t < c.first || t >= c.end)
                        ++mine;
                    else
                        ++also;
                }
        }
        __shared__ unsigned long long total[2];
        if (threadIdx.x < 2) total[threadIdx.x] = 0;
        __syncthreads();
        atomicAdd(&total[0], static_cast<unsigned long long>(mine));
        atomicAdd(&total[1], static_cast<unsigned long long>(also));
        __syncthreads();
        room = max(static_cast<int64_t>(a.budget[group]) - static_cast<int64_t>(total[0]), static_cast<int64_t>(0));
        candidates = static_cast<int64_t>(total[1]);
    }
    uint32_t least = 0;                   // the least value that stays, and how many of those that have it
    int64_t ties = 0;
    if (room > 0 && room < candidates) {
        int64_t left = room;
        for (int shift = 24; shift >= 0; shift -= 8) {
            for (int i = threadIdx.x; i < 256; i += NT) bins[i] = 0;
            __syncthreads();
            for (int p = first_pair; p < first_pair + a.per_group; ++p) {
                const Candidates c(a, p);
                for (int32_t t = c.first + threadIdx.x; t < c.end; t += NT) {
                    if (!has_row(p, t)) continue;
                    const uint32_t x = value_of(a, p, c, t);
                    if (shift == 24 || x >> (shift + 8) == least >> (shift + 8)) atomicAdd(&bins[x >> shift & 255], 1);
                }
            }
            __syncthreads();
            if (threadIdx.x == 0) {
                int d = 255;
                int64_t n = left;
                for (; d > 0 && n > bins[d]; --d) n -= bins[d];
                room_left = n, digit_found = static_cast<uint32_t>(d);
            }
            __syncthreads();
            left = room_left, least |= digit_found << shift;
        }
        ties = left;
    } else if (room == 0) {
        least = 0xffffffffu;              // no value is as large: a float's order is at most that of a NaN, and those are none
    } else {
        ties = INT64_MAX;
    }

    // ---- the lists, in the order of the tokens ----
    int64_t ties_before = 0;
    for (int p = first_pair; p < first_pair + a.per_group; ++p) {
        const Candidates c(a, p);
        int32_t kept = 0;
        int32_t *to = a.keep + static_cast<int64_t>(p) * a.max_keep;
        for (int32_t t0 = 0; t0 < c.len; t0 += NT) {
            const int32_t t = t0 + threadIdx.x;
            bool stays = false, tie = false;
            if (t < c.len && has_row(p, t)) {
                if (t < c.first || t >= c.end) {
                    stays = true;
                } else {
                    const uint32_t x = value_of(a, p, c, t);
                    stays = x > least, tie = x == least;
                }
            }
            const Before equal = count_before<NT>(tie, of_waves2);
            if (tie && ties_before + equal.before < ties) stays = true;
            ties_before += equal.total;
            const Before n = count_before<NT>(stays, of_waves);
            if (stays && kept + n.before < a.max_keep) to[kept + n.before] = t;
            kept += n.total;
        }
        if (threadIdx.x == 0) {
            a.n_keep[p] = kept <= a.max_keep ? kept : -1;
            if (kept > a.max_keep && a.bad) atomicAdd(a.bad, 1);
        }
    }
}

}  // namespace fairkv
