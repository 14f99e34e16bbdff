// The rows of a growing cache that stay move to the front of their pair, or into another cache; the others are dropped.
//
// Row keep[i] of a pair becomes its row i, K and V as they are stored and the row's weight.  Only memory bounds it: what stays is read and
// written once.  Into another cache rows may move in any order.  In place keep ascends, so row i comes from i or behind it: a workgroup that has
// read the rows of a run of i may write them, for every later run reads behind its own i, which are behind what is written.
#pragma once
#include "cache_rows.h"
#include "common.h"
#include "line.h"

namespace fairkv {

struct EvictArgs {
    const char *k, *v;
    char *k_to, *v_to;
    const float *w;                       // weights or null
    float *w_to;
    RowMap from, to;
    const int32_t *cap_to;                // of another cache, null in place
    const int32_t *keep, *n_keep, *len;   // [pairs][max_keep], [pairs], [pairs]
    int32_t *len_out, *bad;               // len_out null: not written by this kernel
    int32_t n_pairs, max_keep;
};

typedef __attribute__((ext_vector_type(4))) uint32_t u32x4_row_t;

// Whether list entry i is what it has to be: a row of the pair that is in the cache, and a place for it; in place also behind the entry before.
__device__ __forceinline__ bool entry_ok(const EvictArgs &a, int pair, int32_t len, const int32_t *keep, int32_t i)
{
    const int32_t t = keep[i];
    if (t < 0 || t >= len || a.from.row(pair, t) < 0 || a.to.row(pair, i) < 0) return false;
    return a.cap_to || i == 0 || t > keep[i - 1];
}
// Whether a pair's list can be one, before its entries are looked at.
__device__ __forceinline__ bool list_ok(const EvictArgs &a, int pair, int32_t len, int32_t n)
{
    return len >= 0 && n >= 0 && n <= a.max_keep && (!a.cap_to || n <= a.cap_to[pair]) && (a.cap_to || n <= len);
}

// Lengths of all pairs, by whole lists: a pair whose list is not right keeps its length (into another cache: has none there) and is counted.
template <int NT>
__device__ __forceinline__ bool whole_list_ok(const EvictArgs &a, int pair, int32_t len, int32_t n, int32_t *flag /* LDS */)
{
    if (threadIdx.x == 0) *flag = list_ok(a, pair, len, n);
    __syncthreads();
    if (*flag) {
        const int32_t *keep = a.keep + static_cast<int64_t>(pair) * a.max_keep;
        bool ok = true;
        for (int32_t i = threadIdx.x; i < n; i += NT) ok = ok && entry_ok(a, pair, len, keep, i);
        if (!ok) *flag = 0;
    }
    __syncthreads();
    return *flag != 0;
}
__global__ __launch_bounds__(256) void fairkv_evict_lengths_kernel(EvictArgs a)
{
    __shared__ int32_t flag;
    const int pair = blockIdx.x;
    const int32_t len = a.len[pair], n = a.n_keep[pair];
    const bool ok = whole_list_ok<256>(a, pair, len, n, &flag);
    if (threadIdx.x == 0) {
        a.len_out[pair] = ok ? n : a.cap_to ? 0 : len;
        if (!ok && a.bad) atomicAdd(a.bad, 1);
    }
}

// Into another cache: the line of all lists, in blocks of so many entries.
template <int ROWB>
__global__ __launch_bounds__(256) void fairkv_evict_into_kernel(EvictArgs a)
{
    constexpr int PPR = ROWB / 16, kSlots = 256 / PPR, kBlock = 64;
    const int piece = threadIdx.x % PPR, slot = threadIdx.x / PPR;
    auto count = [&](int p) __attribute__((always_inline)) {
        const int32_t n = a.n_keep[p];
        return list_ok(a, p, a.len[p], n) ? n : 0;
    };
    auto blocks_of = [](int32_t n) __attribute__((always_inline)) { return (static_cast<int64_t>(n) + kBlock - 1) / kBlock; };
    const LineShare share = line_share<256>(a.n_pairs, gridDim.x, blockIdx.x, [&](int p) { return blocks_of(count(p)); });
    int pair = share.pair;
    int64_t block = share.begin;
    int32_t n = share.left > 0 ? count(pair) : 0;
    for (int64_t left = share.left; left > 0; --left, ++block) {
        if (block >= blocks_of(n)) {
            pair = next_pair(pair, a.n_pairs, count), block = 0;
            n = count(pair);
        }
        const int32_t len = a.len[pair], i0 = static_cast<int32_t>(block) * kBlock;
        const int32_t *keep = a.keep + static_cast<int64_t>(pair) * a.max_keep;
        for (int32_t i = i0 + slot; i < min(n, i0 + kBlock); i += kSlots) {
            if (!entry_ok(a, pair, len, keep, i)) continue;
            const int64_t from = a.from.row(pair, keep[i]), to = a.to.row(pair, i);
            const auto kk = *reinterpret_cast<const u32x4_row_t *>(a.k + from * ROWB + piece * 16), vv = *reinterpret_cast<const u32x4_row_t *>(a.v + from * ROWB + piece * 16);
            *reinterpret_cast<u32x4_row_t *>(a.k_to + to * ROWB + piece * 16) = kk;
            *reinterpret_cast<u32x4_row_t *>(a.v_to + to * ROWB + piece * 16) = vv;
            if (a.w && piece == 0) a.w_to[to] = a.w[from];
        }
    }
}

// In place: a workgroup per pair.
template <int ROWB>
__global__ __launch_bounds__(1024) void fairkv_evict_kernel(EvictArgs a)
{
    constexpr int PPR = ROWB / 16, kSlots = 1024 / PPR;
    __shared__ int32_t flag;
    const int pair = blockIdx.x, piece = threadIdx.x % PPR, slot = threadIdx.x / PPR;
    const int32_t len = a.len[pair], n = a.n_keep[pair];
    if (!whole_list_ok<1024>(a, pair, len, n, &flag)) return;
    const int32_t *keep = a.keep + static_cast<int64_t>(pair) * a.max_keep;
    for (int32_t i0 = 0; i0 < n; i0 += kSlots) {
        const int32_t i = i0 + slot;
        const int32_t t = i < n ? keep[i] : i;
        u32x4_row_t kk, vv;
        float w = 0.f;
        if (t != i) {
            const int64_t from = a.from.row(pair, t);
            kk = *reinterpret_cast<const u32x4_row_t *>(a.k + from * ROWB + piece * 16);
            vv = *reinterpret_cast<const u32x4_row_t *>(a.v + from * ROWB + piece * 16);
            if (a.w && piece == 0) w = a.w[from];
        }
        drain_vmem();                     // what another wave is about to write has been read
        __syncthreads();
        if (t != i) {
            const int64_t to = a.to.row(pair, i);
            *reinterpret_cast<u32x4_row_t *>(a.k_to + to * ROWB + piece * 16) = kk;
            *reinterpret_cast<u32x4_row_t *>(a.v_to + to * ROWB + piece * 16) = vv;
            if (a.w && piece == 0) a.w_to[to] = w;
        }
    }
}

}  // namespace fairkv
