// The rows of a growing cache that stay move to the front of their pair, or into another cache; the others are dropped.
//
// Row keep[i] of a pair becomes its row i, K and V as they are stored and the row's weight.  Only memory bounds it: what stays is read and
// written once.  Into another cache rows may move in any order.  In place keep ascends, so row i comes from i or behind it: a workgroup that has
// read the rows of a run of i may write them, for every later run reads behind its own i, which are behind what is written.
//
// Measured (MI355X): into another cache 128 x 8 pairs of 4096 8-bit rows halved, 1.02 GB read and written, 241 us (4.25 TB/s; a plain copy has 4.9); 16 x 8 pairs of
// 16000 bf16 rows to a sixteenth 28 us (4.4 TB/s); 8 pairs of 1024 halved 5.4 us, most of it the way from lists over pages to rows.  In place the order holds it
// back: the same 300, 35 and 9 us, 8 pairs of 131072 rows to a third 238 us (1.3 TB/s, 128 workgroups; 312 with 64 of 64 bytes each that went round the XCDs, 955 with 4
// waves each and nothing asked for ahead).
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
    int32_t n_pairs, max_keep, movers;    // movers: workgroups that move, of a launch into another cache
};

typedef __attribute__((ext_vector_type(4))) uint32_t u32x4_row_t;

// Whether the pair's token t >= 0 has a row in the cache, asked for without a branch.
__device__ __forceinline__ bool has_row(const RowMap &m, int pair, int32_t t)
{
    if (!m.pages) return m.row(pair, t) >= 0;
    const int32_t page = t >> m.page_shift;
    const bool in_pool = m.row_of_page(m.pages[static_cast<int64_t>(pair) * m.max_pages + min(page, m.max_pages - 1)], t) >= 0;
    return in_pool && page < m.max_pages;
}
// Whether a pair's list can be one, before its entries are looked at.
__device__ __forceinline__ bool list_ok(const EvictArgs &a, int pair, int32_t len, int32_t n)
{
    return len >= 0 && n >= 0 && n <= a.max_keep && (!a.cap_to || n <= a.cap_to[pair]) && (a.cap_to || n <= len);
}

// Whether a pair's whole list is right, and its first entry that moves.  Called by all NT threads.
struct ListFound {
    int32_t ok, first;
};
template <int NT>
__device__ __forceinline__ ListFound whole_list(const EvictArgs &a, int pair, int32_t len, int32_t n, ListFound *found /* LDS */)
{
    if (threadIdx.x == 0) *found = ListFound{list_ok(a, pair, len, n), n};
    __syncthreads();
    if (found->ok) {
        const int32_t *keep = a.keep + static_cast<int64_t>(pair) * a.max_keep;
        bool ok = true;
        int32_t first = n;
        // An entry is a row of the pair that is in the cache, with a place for it, and in place it is behind the entry before.  Four at once: past the last
        // one that one again.
        for (int32_t i0 = threadIdx.x; i0 < n; i0 += 4 * NT) {
            int32_t t[4], before[4];
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const int32_t i = min(i0 + u * NT, n - 1);
                t[u] = keep[i], before[u] = a.cap_to || i == 0 ? -1 : keep[i - 1];
            }
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const int32_t i = min(i0 + u * NT, n - 1);
                const bool there = has_row(a.from, pair, max(t[u], 0)), place = has_row(a.to, pair, i);
                ok = ok && (t[u] > before[u] || a.cap_to) && t[u] >= 0 && t[u] < len && there && place;
                if (t[u] != i) first = min(first, i);
            }
        }
        if (!ok) found->ok = 0;
        if (first < n) atomicMin(&found->first, first);
    }
    __syncthreads();
    return *found;
}
// The lengths: a pair whose list is not right keeps its own (into another cache: has none there) and is counted.
template <int NT>
__device__ __forceinline__ void set_length(const EvictArgs &a, int pair, ListFound *found /* LDS */)
{
    const int32_t len = a.len[pair], n = a.n_keep[pair];
    const bool ok = whole_list<NT>(a, pair, len, n, found).ok != 0;
    if (threadIdx.x == 0) {
        a.len_out[pair] = ok ? n : a.cap_to ? 0 : len;
        if (!ok && a.bad) atomicAdd(a.bad, 1);
    }
}
__global__ __launch_bounds__(256) void fairkv_evict_lengths_kernel(EvictArgs a)
{
    __shared__ ListFound found;
    set_length<256>(a, blockIdx.x, &found);
}

// Into another cache: the line of all lists, in blocks of ENTRIES, one to a lane of a wave; behind the workgroups that move are those that set a pair's
// length, where lengths are not written over those that are read.
template <int ROWB, int ENTRIES>
__global__ __launch_bounds__(256) void fairkv_evict_into_kernel(EvictArgs a)
{
    constexpr int PPR = ROWB / 16, RPW = 64 / PPR, PASSES = ENTRIES / RPW > 0 ? ENTRIES / RPW : 1, U = PASSES < 4 ? PASSES : 4;      // pieces of a row, rows of a wave-wide move, moves of a block, at once
    __shared__ ListFound found;
    if (static_cast<int>(blockIdx.x) >= a.movers) return set_length<256>(a, blockIdx.x - a.movers, &found);
    const int lane = threadIdx.x & 63, piece = lane % PPR, slot = lane / PPR;
    auto count = [&](int p) __attribute__((always_inline)) {
        const int32_t n = a.n_keep[p];
        return list_ok(a, p, a.len[p], n) ? n : 0;
    };
    auto blocks_of = [](int32_t n) __attribute__((always_inline)) { return (static_cast<int64_t>(n) + ENTRIES - 1) / ENTRIES; };
    const LineShare share = line_share<256>(a.n_pairs, a.movers, blockIdx.x, [&](int p) { return blocks_of(count(p)); });
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    int pair = share.pair;
    int64_t first = share.begin, left = share.left;
    int32_t n = left > 0 ? count(pair) : 0;
    while (left > 0) {
        if (first >= blocks_of(n)) {
            pair = next_pair(pair, a.n_pairs, count), first = 0;
            n = count(pair);
        }
        const int64_t end = min(first + left, blocks_of(n));
        const int32_t len = a.len[pair];
        for (int64_t block = first + wave; block < end; block += 4) {
            // the lane's entry: a row that is none stays where it is
            const int32_t i = static_cast<int32_t>(block) * ENTRIES + lane;
            const int32_t t = lane < ENTRIES && i < n ? a.keep[static_cast<int64_t>(pair) * a.max_keep + i] : -1;
            int64_t from = t >= 0 && t < len ? a.from.row(pair, t) : -1;
            const int64_t to = from >= 0 ? a.to.row(pair, i) : -1;
            if (to < 0) from = -1;
            if (a.w && from >= 0) a.w_to[to] = a.w[from];
#pragma unroll 1
            for (int p0 = 0; p0 < PASSES; p0 += U) {
                if (static_cast<int32_t>(block) * ENTRIES + p0 * RPW >= n) break;
                int64_t at[U], out[U];
                u32x4_row_t kk[U], vv[U];
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    at[u] = __shfl(from, (p0 + u) * RPW + slot), out[u] = __shfl(to, (p0 + u) * RPW + slot);
                    const int64_t byte = max(at[u], static_cast<int64_t>(0)) * ROWB + piece * 16;
                    if (at[u] >= 0) {
                        kk[u] = __builtin_nontemporal_load(reinterpret_cast<const u32x4_row_t *>(a.k + byte));
                        vv[u] = __builtin_nontemporal_load(reinterpret_cast<const u32x4_row_t *>(a.v + byte));
                    }
                }
#pragma unroll
                for (int u = 0; u < U; ++u)
                    if (at[u] >= 0) {
                        const int64_t byte = out[u] * ROWB + piece * 16;
                        *reinterpret_cast<u32x4_row_t *>(a.k_to + byte) = kk[u];
                        *reinterpret_cast<u32x4_row_t *>(a.v_to + byte) = vv[u];
                    }
            }
        }
        left -= end - first, first = end;
    }
}

// In place.  A workgroup has so many bytes, WIDTH, of a pair's rows of K or of V: those of different workgroups have nothing to do with one another.  Rows are
// moved in runs; a run's are in registers before one is written, and by then the next run's are on their way, the page numbers of the one behind it, and the
// entries of the one behind that.
// Workgroups go round the eight XCDs: eight pairs, one slice after the other, so that a pair's slices, which share lines of memory, are in one L2 at once.
__host__ __device__ constexpr int evict_blocks(int n_pairs, int slices) { return (n_pairs + 7) / 8 * 8 * slices; }
template <int ROWB, int WIDTH, int NT>
__global__ __launch_bounds__(NT) void fairkv_evict_kernel(EvictArgs a)
{
    constexpr int PPR = WIDTH / 16, SLICES = 2 * (ROWB / WIDTH), ROWS = NT / PPR, U = 4, RUN = ROWS * U;
    __shared__ ListFound found;
    const int movers = evict_blocks(a.n_pairs, SLICES);
    if (static_cast<int>(blockIdx.x) >= movers) return set_length<NT>(a, blockIdx.x - movers, &found);
    const int pair = blockIdx.x / (8 * SLICES) * 8 + blockIdx.x % 8, slice = blockIdx.x / 8 % SLICES, piece = threadIdx.x % PPR, slot = threadIdx.x / PPR;
    if (pair >= a.n_pairs) return;
    const int32_t len = a.len[pair], n = a.n_keep[pair];
    const ListFound list = whole_list<NT>(a, pair, len, n, &found);
    if (!list.ok || list.first >= n) return;
    const int32_t *keep = a.keep + static_cast<int64_t>(pair) * a.max_keep;
    const char *const from = (slice & 1 ? a.v : a.k) + slice / 2 * WIDTH + piece * 16;
    char *const to = (slice & 1 ? a.v_to : a.k_to) + slice / 2 * WIDTH + piece * 16;
    const bool weights = a.w && slice == 0 && piece == 0, paged = a.from.pages != nullptr;
    const int64_t off = paged ? 0 : a.from.off[pair];
    const int32_t *pages = paged ? a.from.pages + static_cast<int64_t>(pair) * a.from.max_pages : nullptr;
    const int shift = a.from.page_shift;
    auto entry = [&](int32_t i0, int u) __attribute__((always_inline)) { return min(i0 + u * ROWS + slot, n - 1); };      // past the last one: that one again
    auto row = [&](int32_t id, int32_t t) __attribute__((always_inline)) { return paged ? (static_cast<int64_t>(id) << shift) + (t & ((1 << shift) - 1)) : off + t; };      // (the list is right)

    struct Run {
        int32_t t[U], page[U], page_to[U];    // entries, and the pages of their rows and of the rows that they become
    };
    auto ask_entries = [&](Run &r, int32_t i0) __attribute__((always_inline)) {
#pragma unroll
        for (int u = 0; u < U; ++u) r.t[u] = keep[entry(i0, u)];
    };
    auto ask_pages = [&](Run &r, int32_t i0) __attribute__((always_inline)) {
#pragma unroll
        for (int u = 0; u < U; ++u) r.page[u] = paged ? pages[r.t[u] >> shift] : 0, r.page_to[u] = paged ? pages[entry(i0, u) >> shift] : 0;
    };
    u32x4_row_t x[U], x_ahead[U];
    float w[U], w_ahead[U];
    int64_t row_to[U], row_to_ahead[U];       // -1: the row stays where it is
    auto ask_rows = [&](const Run &r, int32_t i0) __attribute__((always_inline)) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int64_t at = row(r.page[u], r.t[u]);
            row_to_ahead[u] = i0 + u * ROWS + slot >= n || r.t[u] == entry(i0, u) ? -1 : row(r.page_to[u], entry(i0, u));
            x_ahead[u] = *reinterpret_cast<const u32x4_row_t *>(from + at * ROWB);
            w_ahead[u] = weights ? a.w[at] : 0.f;
        }
    };
    int32_t i0 = list.first / RUN * RUN;
    Run next, behind;
    ask_entries(next, i0);
    ask_entries(behind, i0 + RUN);
    ask_pages(next, i0);
    ask_rows(next, i0);
    next = behind;
    ask_pages(next, i0 + RUN);
    ask_entries(behind, i0 + 2 * RUN);
    for (; i0 < n; i0 += RUN) {
#pragma unroll
        for (int u = 0; u < U; ++u) x[u] = x_ahead[u], w[u] = w_ahead[u], row_to[u] = row_to_ahead[u];
#pragma unroll
        for (int u = 0; u < U; ++u) asm volatile("" : "+v"(x[u]), "+v"(w[u]));      // have come
        __syncthreads();                      // ... to all waves: what another one is about to write has been read
        if (i0 + RUN < n) {
            ask_rows(next, i0 + RUN);
            next = behind;
            ask_pages(next, i0 + 2 * RUN);
            ask_entries(behind, i0 + 3 * RUN);
        }
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (row_to[u] >= 0) {
                *reinterpret_cast<u32x4_row_t *>(to + row_to[u] * ROWB) = x[u];
                if (weights) a.w_to[row_to[u]] = w[u];
            }
    }
}

}  // namespace fairkv
