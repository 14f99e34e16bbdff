// Which rows of a growing cache stay: the protected ones, and the heaviest of the others up to a budget.
//
// Of a pair's len rows the first `sink` and the last `recent` are protected.  Every other one, a candidate, has the value
//     x[t] = max w[u] over the candidates u with |u - t| <= pool / 2,
// and of all candidates of a group (a pair, or the pairs of a sequence) those with the largest values stay, as many as the budget leaves room
// for behind the protected rows; of equal values the one of the lower head, then of the lower token.
//
// Values are compared as 32-bit whole numbers in the order of the floats.  The least one that stays is found digit by digit from the top, by
// counting how many candidates have which digit among those that share the digits found so far: 11, 11 and 10 bits.  Where all candidates that
// share some digits stay, the others need not be looked at.
//
// A group of up to `cap` units of 64 rows is one workgroup's, which reads its weights once and has its keys in LDS.  Rows of larger groups are dealt to
// the whole GPU in blocks of 4096: a kernel makes keys of them, in order, and counts the first digit, two count the others, the second of them block by
// block, and one lists what stays.  A group that is longer than the cache has rows, because tokens of it have none, is gone through by one workgroup, slowly.  Every list ascends and no sum depends on who comes first: counts are whole numbers.
//
// What bounds it (MI355X; times of a call in a row of them): not its bytes (a million weights are 4 MB, 1 us) but one thing after the other.  A workgroup's
// group: 9 us from lengths over pages, weights, three digits and ties to the list, 16 us with four of them on a compute unit, whose waves wait in 64 % of their cycles (128 x 8 pairs of
// 1024 rows; 8 pairs of 1024 rows in one group 9.4).  A large one: four kernels of 4 to 8 us each, of which the first one takes 12, for it finds the groups'
// blocks and reads the weights (one group of 8 pairs of 131072 rows 27 us; 16 groups of 8 pairs of 16000 rows 32, 34 where a fifth kernel counted what stays of
// every block, 48 where every kernel read the weights).
#pragma once
#include "cache_rows.h"
#include "line.h"

namespace fairkv {

constexpr int kDigits = 3;
constexpr int kDigitShift[kDigits] = {21, 10, 0}, kBins = 2048, kLastBins = 1024;      // bins of a digit, and of the last one
constexpr int kBlockRows = 4096;          // of a large group
constexpr int kMaxPairs = 64;             // of a group that one workgroup has
constexpr int kMostHalf = 31;             // of the window

// What the kernels of a large group hand on.  Slots are of groups: a group has at least min_blocks blocks, so the place of its first block in the
// line, divided by min_blocks, is no other's.  A step's workgroups read what the step before left.
struct SelectFound {
    int64_t need;                         // how many stay of the candidates that share the digits found so far
    uint32_t least;                       // these digits, the rest 0; with `done`: what is larger stays
    int32_t done;                         // no more digits need be looked at
};
struct SelectStart {                      // of the first step, which finds it 0: the third step leaves it so
    int32_t bins[kBins];
    unsigned long long protected_rows;    // with a row in the cache
};
struct SelectSlot {
    int32_t bins[kDigits - 1][kBins];     // of the other digits: the first step clears them
    SelectFound found[kDigits - 1];
};
struct SelectShare {                      // of a workgroup: its blocks in the line, and the place of the first block of the group that the first of them is in
    int64_t left, block, at, group_at;    // left: how many, -1: the line is longer than the workspace has room for; block: the first one's number in its pair
    int32_t pair, len;                    // of the first one
};
struct SelectArgs {
    RowMap rows;
    const float *weights;                 // [n_rows]
    const int32_t *len, *budget;          // [B * Hkv]; [groups]
    int32_t *keep, *n_keep, *bad;         // [B * Hkv][max_keep], [B * Hkv], [1] or null
    SelectStart *starts;
    SelectSlot *slots;
    uint32_t *keys;                       // [max_blocks][kBlockRows]: what the first step makes of the rows
    int32_t *above;                       // [max_blocks]: rows of a block that stay whatever the last digit is
    uint32_t *upto;                       // [max_blocks][kLastBins], 16 bits each: candidates with the digits found before whose last digit is this one or more
    SelectShare *shares;                  // of the large groups' workgroups
    int64_t max_blocks;
    int32_t n_pairs, n_groups, max_len, max_keep, half, sink, recent, per_group, cap, min_blocks;      // per_group: pairs of a group
};

// Not a candidate and does not stay; protected.  All candidates lie in between, from that of -inf to that of +inf.
constexpr uint32_t kNone = 0, kProtected = 0xffffffffu;

// The float's place in the order of floats.  -0 is +0; no float's is kNone or kProtected, NaN aside.
__device__ __forceinline__ uint32_t order_of(float x)
{
    const uint32_t u = __float_as_uint(x + 0.f);
    return u ^ (u & 0x80000000u ? 0xffffffffu : 0x80000000u);
}

__device__ __forceinline__ int32_t select_len(const SelectArgs &a, int pair) { return min(max(a.len[pair], 0), a.max_len); }
struct Candidates {                       // of a pair: the first token that is one, and the one behind the last
    int32_t first, end;
    __device__ __forceinline__ Candidates(const SelectArgs &a, int32_t len) : first(min(a.sink, len)), end(max(first, len - min(a.recent, len))) {}
    __device__ __forceinline__ bool has(int32_t t) const { return t >= first && t < end; }
};

// The bin, from the top, in which the need-th candidate lies (need >= 1 and at most the sum of all bins), how many are needed of that bin, and how
// many it has.  Called by all NT threads, the bins complete; ends with a barrier behind the last look at them.
template <class T>                        // that holds the sum
struct BinFound {
    int32_t bin, in_bin;
    T need;
};
template <int NT, class T, class At>
__device__ __forceinline__ BinFound<T> find_bin(T need, At bin_at)
{
    constexpr int PER = kBins / NT, NW = NT / 64;
    static_assert(kBins % NT == 0, "bins of a thread");
    __shared__ T totals[NW];
    __shared__ BinFound<T> found;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, top = kBins - 1 - static_cast<int>(threadIdx.x) * PER;
    int32_t n[PER];
    int64_t mine = 0;
#pragma unroll
    for (int i = 0; i < PER; ++i) n[i] = bin_at(top - i), mine += n[i];
    const T upto = wave_upto(mine);
    if (lane == 63) totals[wave] = upto;
    if (threadIdx.x == 0) found = BinFound<T>{0, 0, 0};
    __syncthreads();
    T before = upto - mine;
#pragma unroll
    for (int w = 0; w < NW; ++w) before += w < wave ? totals[w] : 0;
    if (before < need && need <= before + mine) {
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            if (before < need && need <= before + n[i]) found = BinFound<T>{top - i, n[i], need - before};
            before += n[i];
        }
    }
    __syncthreads();
    return found;
}

// Adds one to the bin of every lane whose `counts` is set.  Bins lie in LDS.
__device__ __forceinline__ void count_digit(int32_t *bins, uint32_t key, int digit, uint32_t least, bool counts)
{
    const int shift = kDigitShift[digit];
    // all digits in front are the ones found
    if (counts && (digit == 0 || (key ^ least) >> kDigitShift[digit > 0 ? digit - 1 : 0] == 0)) atomicAdd(&bins[key >> shift & (digit == kDigits - 1 ? kLastBins - 1 : kBins - 1)], 1);
}

// Weights of a thread's KPT rows, all on their way at once: first the pages' numbers, then the weights, with addresses that are always some of the
// array's.  state: kNone where the cache has no such row (or `place` says so), 1 for a candidate, kProtected.
template <int KPT, class Place>
__device__ __forceinline__ void load_values(const SelectArgs &a, int pair, uint32_t (&state)[KPT], float (&value)[KPT], Place place)
{
    int32_t t[KPT];
    int64_t row[KPT];
#pragma unroll
    for (int i = 0; i < KPT; ++i) state[i] = place(i, t[i]);
    if (a.rows.pages) {
        int32_t id[KPT];
#pragma unroll
        for (int i = 0; i < KPT; ++i) id[i] = a.rows.pages[static_cast<int64_t>(pair) * a.rows.max_pages + min(t[i] >> a.rows.page_shift, a.rows.max_pages - 1)];
#pragma unroll
        for (int i = 0; i < KPT; ++i) row[i] = a.rows.row_of_page(id[i], t[i]);
    } else {
        const int64_t first = a.rows.off[pair];
#pragma unroll
        for (int i = 0; i < KPT; ++i) row[i] = first >= 0 && static_cast<uint64_t>(first) + static_cast<uint32_t>(t[i]) < static_cast<uint64_t>(a.rows.n_rows) ? first + t[i] : -1;
    }
#pragma unroll
    for (int i = 0; i < KPT; ++i) value[i] = a.weights[max(row[i], static_cast<int64_t>(0))];
#pragma unroll
    for (int i = 0; i < KPT; ++i) {
        if (row[i] < 0) state[i] = kNone;
        value[i] = state[i] == 1 ? fmaxf(value[i], -INFINITY) : -INFINITY;      // a NaN is as low
    }
}
// Rows i NT + threadIdx.x, i < KPT, of which bit i of a thread's x says whether it is one of some: how many of them are in front of a row.
// count_rows is called by all threads and ends with a barrier; another one stands between the last rows_before and the next count_rows.
template <int NT, int KPT>
__device__ __forceinline__ void count_rows(int32_t (&counts)[KPT][NT / 64], uint32_t x, int32_t *total /* LDS */)
{
    constexpr int NW = NT / 64, PER = KPT * NW / 64;
    static_assert(KPT * NW % 64 == 0, "sums of a lane");
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
    for (int i = 0; i < KPT; ++i) {
        const int32_t n = __builtin_popcountll(__builtin_amdgcn_ballot_w64((x >> i & 1) != 0));
        if (lane == 0) counts[i][wave] = n;
    }
    __syncthreads();
    if (wave == 0) {
        int32_t n[PER], all = 0;
#pragma unroll
        for (int j = 0; j < PER; ++j) n[j] = (&counts[0][0])[lane * PER + j], all += n[j];
        int32_t before = wave_upto(all) - all;
        if (lane == 63) *total = before + all;
#pragma unroll
        for (int j = 0; j < PER; ++j) {
            (&counts[0][0])[lane * PER + j] = before;
            before += n[j];
        }
    }
    __syncthreads();
}
template <int NT, int KPT>
__device__ __forceinline__ int32_t rows_before(const int32_t (&counts)[KPT][NT / 64], uint32_t x, int i)
{
    return counts[i][threadIdx.x >> 6] + __builtin_popcountll(__builtin_amdgcn_ballot_w64((x >> i & 1) != 0) & ((1ull << (threadIdx.x & 63)) - 1));
}

// The kernel's arguments (these are all that its kernels have), read again: for what is hardly ever done, so that nothing of it is kept in scalar registers by
// those that do not come there (one sequence of 8 pairs of 1024 rows 9.6 us instead of 9.4).
__device__ __forceinline__ SelectArgs select_args_again()
{
    typedef __attribute__((address_space(4))) const uint64_t *words_t;
    struct Words {
        uint64_t x[sizeof(SelectArgs) / sizeof(uint64_t)];
    } words;
    static_assert(sizeof(Words) == sizeof(SelectArgs), "whole words");
    uint64_t at = reinterpret_cast<uint64_t>(__builtin_amdgcn_kernarg_segment_ptr());
    asm volatile("" : "+s"(at));
#pragma unroll
    for (size_t i = 0; i < sizeof(SelectArgs) / sizeof(uint64_t); ++i) words.x[i] = reinterpret_cast<words_t>(at)[i];
    return __builtin_bit_cast(SelectArgs, words);
}

// ---- a group that is longer than the host has counted on ----
// The host counts on no more rows than the cache has, but tokens count whether they have one or not.  Here a workgroup goes through a group's tokens once for
// every digit and once for the lists, and makes a token's key anew each time: what this takes from the kernels around it is kept small, not its time (8 pairs of
// 131072 tokens of which the last 1024 have rows: 1.7 ms in one group, 0.2 in 8).  A group that has more rows than the cache is refused: its pairs' rows overlap.
template <int NT>
__device__ __forceinline__ void select_slowly(const SelectArgs &a, int group, int32_t *bins, int32_t *counts /* both in LDS, kBins and NT / 64 */)
{
    __shared__ unsigned long long rows, protected_rows;
    const int p0 = group * a.per_group, p1 = p0 + a.per_group, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    auto key_of = [&](int pair, const Candidates &c, int32_t t) __attribute__((always_inline)) {
        const int64_t row = a.rows.row(pair, t);
        if (row < 0) return kNone;
        if (!c.has(t)) return kProtected;
        float x = fmaxf(a.weights[row], -INFINITY);
#pragma unroll 1
        for (int32_t u = a.half > 0 ? max(t - a.half, c.first) : c.end; u < min(t + a.half + 1, c.end); ++u) {
            const int64_t beside = a.rows.row(pair, u);
            if (beside >= 0) x = fmaxf(x, a.weights[beside]);
        }
        return order_of(x);
    };
    auto clear_bins = [&]() __attribute__((always_inline)) {
#pragma unroll 1
        for (int i = threadIdx.x; i < kBins; i += NT) bins[i] = 0;
    };
    __syncthreads();                      // the group before
    clear_bins();
    if (threadIdx.x == 0) rows = protected_rows = 0;
    __syncthreads();
    uint32_t least = 0;                   // what is larger stays
    int32_t need = 0;                     // how many of those that are equal to it
#pragma unroll 1
    for (int digit = 0; digit < kDigits; ++digit) {
        int32_t n = 0, n_protected = 0;   // of a thread
#pragma unroll 1
        for (int p = p0; p < p1; ++p) {
            const int32_t len = select_len(a, p);
            const Candidates c(a, len);
#pragma unroll 1
            for (int32_t t = threadIdx.x; t < len; t += NT) {
                const uint32_t key = key_of(p, c, t);
                n += key != kNone, n_protected += key == kProtected;
                count_digit(bins, key, digit, least, key != kNone && key != kProtected);
            }
        }
        if (digit == 0) atomicAdd(&rows, static_cast<unsigned long long>(n)), atomicAdd(&protected_rows, static_cast<unsigned long long>(n_protected));
        __syncthreads();
        if (digit == 0) {
            if (rows > static_cast<unsigned long long>(a.rows.n_rows)) {
                for (int p = p0 + threadIdx.x; p < p1; p += NT) {
                    a.n_keep[p] = -1;
                    if (a.bad) atomicAdd(a.bad, 1);
                }
                return;
            }
            need = static_cast<int32_t>(max(static_cast<int64_t>(a.budget[group]) - static_cast<int64_t>(protected_rows), static_cast<int64_t>(0)));
            if (need == 0) {
                least = kProtected - 1;
                break;
            }
        }
        const BinFound<int32_t> b = find_bin<NT>(need, [&](int x) { return bins[x]; });
        need = b.need;
        if (need == 0) break;             // there are no so many candidates: all of them stay
        least |= static_cast<uint32_t>(b.bin) << kDigitShift[digit];
        if (need == b.in_bin) {           // all that share these digits stay
            least -= 1, need = 0;
            break;
        }
        clear_bins();
        __syncthreads();
    }
    // NT tokens of a pair at a time: how many of those that `is` says are in front of the thread's, and all of them
    auto place = [&](bool is, int32_t &all) __attribute__((always_inline)) {
        const uint64_t here = __builtin_amdgcn_ballot_w64(is);
        __syncthreads();                  // the counts before have been read
        if (lane == 0) counts[wave] = __builtin_popcountll(here);
        __syncthreads();
        int32_t before = __builtin_popcountll(here & ((1ull << lane) - 1));
        all = 0;
#pragma unroll 1
        for (int w = 0; w < NT / 64; ++w) {
            if (w < wave) before += counts[w];
            all += counts[w];
        }
        return before;
    };
    int32_t ties = 0;                     // of the group, so far: no more than are needed count
#pragma unroll 1
    for (int p = p0; p < p1; ++p) {
        const int32_t len = select_len(a, p);
        const Candidates c(a, len);
        int32_t kept = 0, all;
#pragma unroll 1
        for (int32_t t0 = 0; t0 < len; t0 += NT) {
            const int32_t t = t0 + static_cast<int32_t>(threadIdx.x);
            const uint32_t key = t < len ? key_of(p, c, t) : kNone;
            bool stays = key > least;
            if (ties < need) {
                const bool equal = key == least;
                const int32_t before = place(equal, all);
                stays = stays || (equal && before < need - ties);
                ties += min(all, need - ties);
            }
            const int32_t n = kept + place(stays, all);
            if (stays && n < a.max_keep) a.keep[static_cast<int64_t>(p) * a.max_keep + n] = t;
            kept += all;
        }
        if (threadIdx.x == 0) {
            a.n_keep[p] = kept <= a.max_keep ? kept : -1;
            if (kept > a.max_keep && a.bad) atomicAdd(a.bad, 1);
        }
    }
}

// ---- a group that one workgroup has ----
// Its rows in units of 64, a pair's last one not full, so that all lanes of a wave are in one pair; wave w has units w, w + NW, ...  What a pair's
// rows need to know is held in lanes: lane p has pair p.  Keys lie in LDS.  With a window they are first the floats' bits, NaN for rows that are no
// candidates, which a maximum passes over; what becomes of them waits in registers until all windows have been looked at.  (A second array in LDS
// leaves a compute unit half its workgroups: 128 x 8 pairs of 1000 rows, window 7, 24 us instead of 20; one group of 8000 rows 17 instead of 18.)
constexpr uint32_t kRawNone = 0x7fc00001u, kRawProtected = 0x7fc00002u;
template <int UNITS>
struct GroupSpace {
    uint32_t keys[UNITS * 64];
    int32_t bins[kBins];
    int32_t counts[UNITS];
    int32_t total, protected_rows, candidate_rows;
};
template <int NT, int UNITS, bool POOL, bool ALONE>      // ALONE: no other kernel has larger groups
__device__ __forceinline__ void select_group(const SelectArgs &a, int group, GroupSpace<UNITS> &m)
{
    constexpr int NW = NT / 64, PER = (UNITS + 63) / 64;
    auto &keys = m.keys;
    auto &bins = m.bins;
    auto &counts = m.counts;
    int32_t &total = m.total, &protected_rows = m.protected_rows, &candidate_rows = m.candidate_rows;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), p0 = group * a.per_group;
    const int n_pairs = a.per_group;
    const uint64_t below = (1ull << lane) - 1;
    // ---- where the pairs begin, in units ----
    const bool one = lane < n_pairs;
    const int32_t budget = a.budget[group];
    const int32_t len = one ? select_len(a, p0 + lane) : 0;
    const int64_t off = one && !a.rows.pages ? a.rows.off[p0 + lane] : 0;
    const int64_t upto = wave_upto((static_cast<int64_t>(len) + 63) / 64), units64 = __shfl(upto, 63);
    if (n_pairs > kMaxPairs || units64 > a.cap) {     // a.cap is UNITS or less
        if constexpr (ALONE) select_slowly<NT>(select_args_again(), group, bins, counts);
        return;
    }
    const int32_t units = __builtin_amdgcn_readfirstlane(static_cast<int>(units64));
    const int32_t ends = static_cast<int32_t>(upto), begins = ends - (len + 63) / 64;      // of the lane's pair
    auto pair_of = [&](int32_t unit) __attribute__((always_inline)) { return __builtin_popcountll(__builtin_amdgcn_ballot_w64(one && ends <= unit)); };
    for (int i = threadIdx.x; i < kBins; i += NT) bins[i] = 0;
    if (threadIdx.x == 0) protected_rows = candidate_rows = 0;
    __syncthreads();

    // ---- values, from addresses that are always some of the arrays'.  (Two, three and four units of a wave on their way at once were 1.5, 4 and 5 % slower
    //      on 128 x 8 pairs of 1024 rows: the other waves are enough, and short pairs have no more units.) ----
    int32_t is_protected = 0, is_candidate = 0;
    for (int32_t unit = wave; unit < units; unit += NW) {
        const int p = pair_of(unit);
        const int32_t t = (unit - __builtin_amdgcn_readlane(begins, p)) * 64 + lane, n = __builtin_amdgcn_readlane(len, p);
        int64_t row;
        if (a.rows.pages) {
            row = a.rows.row_of_page(a.rows.pages[static_cast<int64_t>(p0 + p) * a.rows.max_pages + min(min(t, n - 1) >> a.rows.page_shift, a.rows.max_pages - 1)], t);
        } else {
            const int64_t first = static_cast<int64_t>((static_cast<uint64_t>(static_cast<uint32_t>(__builtin_amdgcn_readlane(static_cast<int>(off >> 32), p))) << 32) |
                                                       static_cast<uint32_t>(__builtin_amdgcn_readlane(static_cast<int>(off), p)));
            row = first >= 0 && static_cast<uint64_t>(first) + static_cast<uint32_t>(t) < static_cast<uint64_t>(a.rows.n_rows) ? first + t : -1;
        }
        float value = a.weights[max(row, static_cast<int64_t>(0))];
        const bool candidate = Candidates(a, n).has(t) && row >= 0, stays = t < n && row >= 0 && !candidate;
        value = fmaxf(candidate ? value : -INFINITY, -INFINITY);      // a NaN is as low
        is_candidate += __builtin_popcountll(__builtin_amdgcn_ballot_w64(candidate));
        is_protected += __builtin_popcountll(__builtin_amdgcn_ballot_w64(stays));
        if constexpr (POOL) {
            keys[unit * 64 + lane] = stays ? kRawProtected : candidate ? __float_as_uint(value) : kRawNone;
        } else {
            keys[unit * 64 + lane] = stays ? kProtected : candidate ? order_of(value) : kNone;
            if (candidate) atomicAdd(&bins[order_of(value) >> kDigitShift[0]], 1);
        }
    }
    if (lane == 0) atomicAdd(&candidate_rows, is_candidate), atomicAdd(&protected_rows, is_protected);
    __syncthreads();
    if constexpr (POOL) {                             // the window ends where the pair does
        constexpr int EACH = (UNITS + NW - 1) / NW;
        uint32_t key[EACH];
#pragma unroll
        for (int i = 0; i < EACH; ++i) {
            const int32_t unit = wave + i * NW;
            if (unit >= units) break;
            const int p = pair_of(unit);
            const int32_t at = unit * 64 + lane, lo = __builtin_amdgcn_readlane(begins, p) * 64, hi = __builtin_amdgcn_readlane(ends, p) * 64 - 1;
            const uint32_t own = keys[at];
            float x = __uint_as_float(own);
            for (int32_t d0 = 1; d0 <= a.half; d0 += 4) {      // eight reads at once: past the window's end those of its end again
                float y[8];
#pragma unroll
                for (int u = 0; u < 4; ++u) {
                    const int32_t d = min(d0 + u, a.half);
                    y[2 * u] = __uint_as_float(keys[max(lo, at - d)]), y[2 * u + 1] = __uint_as_float(keys[min(hi, at + d)]);
                }
#pragma unroll
                for (int u = 0; u < 8; ++u) x = fmaxf(x, y[u]);
            }
            key[i] = own == kRawProtected ? kProtected : own == kRawNone ? kNone : order_of(x);
            if (key[i] != kNone && key[i] != kProtected) atomicAdd(&bins[key[i] >> kDigitShift[0]], 1);
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < EACH; ++i) {
            const int32_t unit = wave + i * NW;
            if (unit >= units) break;
            keys[unit * 64 + lane] = key[i];
        }
        __syncthreads();
    }

    // ---- the least that stays, and how many of those that are equal to it ----
    const int64_t room = max(static_cast<int64_t>(budget) - protected_rows, static_cast<int64_t>(0));
    uint32_t least = 0;                               // what is larger stays
    int32_t ties = 0;
    if (room == 0) {
        least = kProtected - 1;
    } else if (room < candidate_rows) {
        ties = static_cast<int32_t>(room);
        for (int digit = 0; digit < kDigits; ++digit) {
            if (digit > 0) {
                for (int i = threadIdx.x; i < kBins; i += NT) bins[i] = 0;
                __syncthreads();
                for (int32_t unit = wave; unit < units; unit += NW) {
                    const uint32_t key = keys[unit * 64 + lane];
                    count_digit(bins, key, digit, least, key != kNone && key != kProtected);
                }
                __syncthreads();
            }
            const BinFound<int32_t> b = find_bin<NT>(ties, [&](int x) { return bins[x]; });
            ties = b.need;
            least |= static_cast<uint32_t>(b.bin) << kDigitShift[digit];
            if (ties == b.in_bin) {                   // all of them stay, whatever their other digits are
                least -= 1;
                ties = 0;
                break;
            }
        }
    }

    // ---- the lists: counts in front of every unit, in the order of the rows, of the ties and then of what stays ----
    auto count = [&](auto is) __attribute__((always_inline)) {
        for (int32_t unit = wave; unit < units; unit += NW) {
            const int32_t n = __builtin_popcountll(__builtin_amdgcn_ballot_w64(is(unit)));
            if (lane == 0) counts[unit] = n;
        }
        __syncthreads();
        if (wave == 0) {
            int32_t n[PER], all = 0;
#pragma unroll
            for (int i = 0; i < PER; ++i) n[i] = lane * PER + i < units ? counts[lane * PER + i] : 0, all += n[i];
            int32_t before = wave_upto(all) - all;
            if (lane == 63) total = before + all;
#pragma unroll
            for (int i = 0; i < PER; ++i) {
                if (lane * PER + i < units) counts[lane * PER + i] = before;
                before += n[i];
            }
        }
        __syncthreads();
    };
    if (ties > 0) {
        auto equal = [&](int32_t unit) { return keys[unit * 64 + lane] == least; };
        count(equal);
        for (int32_t unit = wave; unit < units; unit += NW) {
            const uint64_t here = __builtin_amdgcn_ballot_w64(equal(unit));
            if (equal(unit) && counts[unit] + __builtin_popcountll(here & below) < ties) keys[unit * 64 + lane] = kProtected;
        }
        __syncthreads();
    }
    auto stays = [&](int32_t unit) { return keys[unit * 64 + lane] > least; };
    count(stays);
    const int32_t from = begins < units ? counts[begins] : total, to = ends < units ? counts[ends] : total;      // of the lane's pair: how many stay in front of it, and up to its end
    for (int32_t unit = wave; unit < units; unit += NW) {
        const int p = pair_of(unit);
        const bool here = stays(unit);
        const int32_t n = counts[unit] + __builtin_popcountll(__builtin_amdgcn_ballot_w64(here) & below) - __builtin_amdgcn_readlane(from, p);
        if (here && n < a.max_keep) a.keep[static_cast<int64_t>(p0 + p) * a.max_keep + n] = (unit - __builtin_amdgcn_readlane(begins, p)) * 64 + lane;
    }
    if (wave == 0 && one) {
        a.n_keep[p0 + lane] = to - from <= a.max_keep ? to - from : -1;
        if (to - from > a.max_keep && a.bad) atomicAdd(a.bad, 1);
    }
}

template <int NT, int UNITS, bool POOL>
__global__ __launch_bounds__(NT, 8) void fairkv_select_kernel(SelectArgs a)
{
    __shared__ GroupSpace<UNITS> m;
    select_group<NT, UNITS, POOL, true>(a, blockIdx.x, m);
}

// ---- large groups: the line of their blocks ----
struct LargeGroups {
    const SelectArgs &a;
    int known = -1;                       // the group that was looked at last, and whether it is a large one
    bool large = false;
    __device__ __forceinline__ explicit LargeGroups(const SelectArgs &args) : a(args) {}
    __device__ __forceinline__ int64_t operator()(int pair)
    {
        const int group = pair / a.per_group;
        if (group != known) {
            known = group;
            large = a.per_group > kMaxPairs;
            if (!large) {
                int64_t units = 0;
#pragma unroll 8
                for (int p = group * a.per_group; p < (group + 1) * a.per_group; ++p) units += (select_len(a, p) + 63) / 64;
                large = units > a.cap;
            }
        }
        return large ? max(1, (select_len(a, pair) + kBlockRows - 1) / kBlockRows) : 0;      // one of an empty pair too: its list is one
    }
    // Where the group of a share's pair begins.
    __device__ __forceinline__ void group_of(SelectShare &s)
    {
        s.group_at = s.at - s.block;
#pragma unroll 8
        for (int p = s.pair / a.per_group * a.per_group; p < s.pair; ++p) s.group_at -= max(1, (select_len(a, p) + kBlockRows - 1) / kBlockRows);
    }
};

template <int STEP>
struct LargeSpace {
    float raw[STEP == 0 ? kBlockRows + 2 * kMostHalf : 1];
    int32_t bins[kBins];
    int32_t counts[kBlockRows / 64];
    unsigned long long sums[5];
    int32_t total, equals[8], aboves[8];
};
constexpr int kLargeThreads = 512;

constexpr int kLists = kDigits;           // the last step

// Workgroup `slot_index` of n: STEP 0 .. 2: a digit is counted, the last one in every block; 3: the lists.  The first step finds the workgroup's share of
// the line, the others have it from there.
template <int STEP>
__device__ __forceinline__ void select_large(const SelectArgs &a, int slot_index, int n_slots, LargeSpace<STEP> &m)
{
    constexpr int NT = kLargeThreads, KPT = kBlockRows / NT;
    constexpr bool kCounts = STEP < kDigits - 1, kBlocks = STEP == kDigits - 1;      // a digit of the workgroup's blocks of a group, of every block
    auto &raw = m.raw;
    auto &bins = m.bins;
    auto &counts = reinterpret_cast<int32_t (&)[KPT][NT / 64]>(m.counts);
    auto &sums = m.sums;
    int32_t &total = m.total;
    [[maybe_unused]] const int lane = threadIdx.x & 63;
    LargeGroups blocks_of(a);
    SelectShare share;
    if constexpr (STEP == 0) {
        const LineShare l = line_share<NT>(a.n_pairs, n_slots, slot_index, [&](int p) { return blocks_of(p); });
        share = {l.total > a.max_blocks ? -1 : l.left, l.begin, l.at, 0, l.pair, 0};      // tokens without rows: more blocks than the workspace has
        if (share.left > 0)
            share.len = select_len(a, share.pair);      // (its group is looked at when the first rows are on their way)
        else if (threadIdx.x == 0)
            a.shares[slot_index] = share;
    } else {
        share = a.shares[slot_index];
    }
    if constexpr (STEP == kLists)
        if (share.left < 0) {
            const SelectArgs again = select_args_again();
            LargeGroups blocks(again);
#pragma unroll 1
            for (int g = slot_index; g < again.n_groups; g += n_slots)
                if (blocks(g * again.per_group) > 0) select_slowly<NT>(again, g, bins, m.counts);
            return;
        }
    if (share.left <= 0) return;
    int pair = share.pair, group = -1;
    int64_t block = share.block, at = share.at, group_at = share.group_at;      // group_at: the place of the group's first block
    SelectStart *start = nullptr;
    SelectSlot *slot = nullptr;
    SelectFound f{0, 0, 0};
    int32_t protected_rows = 0, last = -1, last_ties = -1;      // the last digit of what stays, and that of ties: -1 where there is none

    auto end_group = [&]() __attribute__((always_inline)) {
        if constexpr (kCounts) {
            __syncthreads();
            for (int i = threadIdx.x; i < kBins; i += NT)
                if (bins[i]) atomicAdd(STEP == 0 ? &start->bins[i] : &slot->bins[0][i], bins[i]);
            if constexpr (STEP == 0) {
                const int64_t n = wave_upto(static_cast<int64_t>(protected_rows));
                if (lane == 63 && n) atomicAdd(&start->protected_rows, static_cast<unsigned long long>(n));
            }
            __syncthreads();
        }
    };
    auto begin_group = [&]() __attribute__((always_inline)) {
        if (STEP == 0 || group >= 0) {
            const bool first = group < 0;
            share.at = at, share.block = block, share.pair = pair;
            blocks_of.group_of(share);
            if (first && threadIdx.x == 0) a.shares[slot_index] = share;
            group_at = share.group_at;
        }
        group = pair / a.per_group;
        start = a.starts + group_at / a.min_blocks, slot = a.slots + group_at / a.min_blocks;
        if constexpr (STEP == 1) {
            f = {max(static_cast<int64_t>(a.budget[group]) - static_cast<int64_t>(start->protected_rows), static_cast<int64_t>(0)), 0, 0};
            if (f.need == 0) f = {0, kProtected - 1, 1};
        }
        if constexpr (STEP > 1) f = slot->found[STEP - 2];
        if constexpr (STEP >= 1) {
            last = last_ties = -1;
            if (!f.done) {
                const BinFound<int64_t> b = find_bin<NT>(f.need, [&](int x) { return STEP == 1 ? start->bins[x] : STEP == kLists && x >= kLastBins ? 0 : slot->bins[STEP > 1 ? STEP - 2 : 0][x]; });
                if (b.need == 0) {        // there are no so many candidates: all of them stay
                    f = {0, 0, 1};
                } else {
                    f.need = b.need, f.least |= static_cast<uint32_t>(b.bin) << kDigitShift[STEP - 1];
                    last = b.bin + 1, last_ties = b.bin;
                    if (f.need == b.in_bin) f = {0, f.least - 1, 1}, last = b.bin, last_ties = -1;      // all that share these digits stay
                }
            }
        }
        if (at == group_at) {             // this workgroup has the group's first block
            if constexpr (STEP >= 1 && STEP < kDigits)
                if (threadIdx.x == 0) slot->found[STEP - 1] = f;
            if constexpr (STEP == 0)
                for (int i = threadIdx.x; i < (kDigits - 1) * kBins; i += NT) (&slot->bins[0][0])[i] = 0;
            if constexpr (STEP == 2) {
                for (int i = threadIdx.x; i < kBins; i += NT) start->bins[i] = 0;
                if (threadIdx.x == 0) start->protected_rows = 0;
            }
        }
        if constexpr (kCounts || kBlocks) {
            for (int i = threadIdx.x; i < kBins; i += NT) bins[i] = 0;
            protected_rows = 0;
            __syncthreads();
        }
    };

    // Of a block: rows that stay without being ties, and ties.
    auto counts_of = [&](int64_t x) __attribute__((always_inline)) {
        const uint16_t *upto = reinterpret_cast<const uint16_t *>(a.upto + x * (kLastBins / 2));
        const int32_t more = last >= 0 && last < kLastBins ? upto[last] : 0;
        return make_int2(a.above[x] + more, last_ties >= 0 ? upto[last_ties] - more : 0);
    };
    auto blocks_of_large = [&](int32_t len) __attribute__((always_inline)) { return max(1, (len + kBlockRows - 1) / kBlockRows); };
    int32_t len = share.len;
    for (int64_t left = share.left; left > 0; --left, ++block, ++at) {
        if (block >= blocks_of_large(len)) {
            pair = next_pair(pair, a.n_pairs, [&](int p) { return blocks_of(p); }), block = 0;
            len = select_len(a, pair);
        }
        // ---- keys, on their way while the group's state is found: from the weights, or as the first step left them ----
        const int32_t t0 = static_cast<int32_t>(block) * kBlockRows;
        const int e = static_cast<int>(threadIdx.x);
        uint32_t *const keys = a.keys + at * kBlockRows + e;
        uint32_t key[KPT];
        float value[KPT], edge[1];        // edge: rows beside the block that its windows reach
        if constexpr (STEP > 0) {
#pragma unroll
            for (int i = 0; i < KPT; ++i) key[i] = keys[i * NT];
        } else if (len == 0) {            // of a cache without rows, maybe: nothing is read
#pragma unroll
            for (int i = 0; i < KPT; ++i) key[i] = kNone, value[i] = -INFINITY;
            edge[0] = -INFINITY;
        } else {
            const Candidates c(a, len);
            uint32_t edge_state[1];
            load_values<KPT>(a, pair, key, value, [&](int i, int32_t &t) {
                t = min(t0 + i * NT + e, max(len - 1, 0));
                return t0 + i * NT + e >= len ? kNone : c.has(t) ? 1u : kProtected;
            });
            if (a.half > 0)
                load_values<1>(a, pair, edge_state, edge, [&](int, int32_t &t) {
                    const int32_t at_edge = e < a.half ? t0 - a.half + e : t0 + kBlockRows + e - a.half;
                    t = min(max(at_edge, 0), max(len - 1, 0));
                    return e < 2 * a.half && c.has(at_edge) ? 1u : kNone;
                });
        }
        if (pair / a.per_group != group) {
            if (group >= 0) end_group();
            begin_group();
        }
        if (STEP == 1 && f.done) continue;
        // what stays of other blocks: in front of this one, and behind it where it is the pair's first (the first of them ahead of their use)
        const int64_t pair_at = at - block, pair_end = pair_at + blocks_of_large(len);
        const int64_t look_from = f.need > 0 ? group_at : pair_at, look_to = block == 0 ? pair_end : at;
        int2 look = make_int2(0, 0);
        if (STEP == kLists && look_from + static_cast<int64_t>(threadIdx.x) < look_to) look = counts_of(look_from + threadIdx.x);
        if constexpr (STEP == 0) {
            if (a.half > 0) {
                __syncthreads();              // the windows of the block before have been looked at
#pragma unroll
                for (int i = 0; i < KPT; ++i) raw[a.half + i * NT + e] = value[i];
                if (e < 2 * a.half) raw[e < a.half ? e : kBlockRows + e] = edge[0];
                __syncthreads();
                for (int d = 0; d <= 2 * a.half; ++d) {
#pragma unroll
                    for (int i = 0; i < KPT; ++i) value[i] = fmaxf(value[i], raw[i * NT + e + d]);
                }
            }
#pragma unroll
            for (int i = 0; i < KPT; ++i) {
                if (key[i] == kProtected) ++protected_rows;
                if (key[i] == 1) key[i] = order_of(value[i]);
            }
#pragma unroll
            for (int i = 0; i < KPT; ++i) keys[i * NT] = key[i];
        }
        // ---- counts ----
        if constexpr (kCounts) {
#pragma unroll
            for (int i = 0; i < KPT; ++i) count_digit(bins, key[i], STEP, f.least, key[i] != kNone && key[i] != kProtected);
            continue;
        }
        if constexpr (kBlocks) {
            const uint32_t most = f.done ? f.least : f.least | (kLastBins - 1);      // what is larger stays
            int32_t above = 0;
#pragma unroll
            for (int i = 0; i < KPT; ++i) {
                above += __builtin_popcountll(__builtin_amdgcn_ballot_w64(key[i] > most));
                count_digit(bins, key[i], STEP, f.least, !f.done && key[i] != kNone && key[i] != kProtected);
            }
            __syncthreads();
            // two bins of a thread, from the top; they are 0 again for the next block
            const int wave = threadIdx.x >> 6, bin = kLastBins - 2 - 2 * static_cast<int>(threadIdx.x);
            const int32_t high = bins[bin + 1], low = bins[bin], sum = wave_upto(high + low);
            bins[bin + 1] = bins[bin] = 0;
            if (lane == 63) m.equals[wave] = sum, m.aboves[wave] = above;
            __syncthreads();
            int32_t before = sum - high - low, all_above = 0;
#pragma unroll
            for (int w = 0; w < NT / 64; ++w) before += w < wave ? m.equals[w] : 0, all_above += m.aboves[w];
            if (!f.done) {
                a.upto[at * (kLastBins / 2) + bin / 2] = static_cast<uint32_t>(before + high + low) | static_cast<uint32_t>(before + high) << 16;
                if (high) atomicAdd(&slot->bins[1][bin + 1], high);
                if (low) atomicAdd(&slot->bins[1][bin], low);
            }
            if (threadIdx.x == 0) a.above[at] = all_above;
            continue;
        }
        uint32_t stays = 0, equal = 0;
#pragma unroll
        for (int i = 0; i < KPT; ++i) {
            stays |= (key[i] > f.least ? 1u : 0u) << i;
            equal |= (f.need > 0 && key[i] == f.least ? 1u : 0u) << i;
        }
        // ties in front of the pair, and of the block; rows in front of the block that stay anyhow; both of the whole pair
        __syncthreads();
        if (threadIdx.x < 5) sums[threadIdx.x] = 0;
        __syncthreads();
        unsigned long long s[5] = {0, 0, 0, 0, 0};
        for (int64_t x = look_from + threadIdx.x; x < look_to; x += NT) {
            const int2 n = x < look_from + NT ? look : counts_of(x);
            if (x < pair_at) s[0] += n.y;
            if (x < at) s[1] += n.y;
            if (x >= pair_at && x < at) s[2] += n.x;
            if (x >= pair_at) s[3] += n.y, s[4] += n.x;
        }
#pragma unroll
        for (int i = 0; i < 5; ++i) {
            const int64_t n = wave_upto(static_cast<int64_t>(s[i]));
            if (lane == 63 && n) atomicAdd(&sums[i], static_cast<unsigned long long>(n));
        }
        __syncthreads();
        const int64_t ties_pair = sums[0], ties_block = sums[1];
        const int64_t from = static_cast<int64_t>(sums[2]) + min(f.need, ties_block) - min(f.need, ties_pair);
        if (block == 0 && threadIdx.x == 0) {
            const int64_t n = static_cast<int64_t>(sums[4]) + min(f.need, ties_pair + static_cast<int64_t>(sums[3])) - min(f.need, ties_pair);
            a.n_keep[pair] = n <= a.max_keep ? static_cast<int32_t>(n) : -1;
            if (n > a.max_keep && a.bad) atomicAdd(a.bad, 1);
        }
        if (f.need > 0) {
            count_rows<NT, KPT>(counts, equal, &total);
#pragma unroll
            for (int i = 0; i < KPT; ++i) {
                const int32_t n = rows_before<NT, KPT>(counts, equal, i);
                if ((equal >> i & 1) && ties_block + n < f.need) stays |= 1u << i;
            }
            __syncthreads();
        }
        count_rows<NT, KPT>(counts, stays, &total);
#pragma unroll
        for (int i = 0; i < KPT; ++i) {
            const int64_t n = from + rows_before<NT, KPT>(counts, stays, i);
            if ((stays >> i & 1) && n < a.max_keep) a.keep[static_cast<int64_t>(pair) * a.max_keep + n] = t0 + i * NT + static_cast<int32_t>(threadIdx.x);
        }
    }
    end_group();
}

// The first step of the large groups, and beside it the groups that one workgroup has.
template <int UNITS, bool POOL>
__global__ __launch_bounds__(kLargeThreads, 6) void fairkv_select_first_kernel(SelectArgs a)
{
    __shared__ union Space {
        GroupSpace<UNITS> group;
        LargeSpace<0> large;
        __device__ Space() {}
    } m;
    if (static_cast<int>(blockIdx.x) < a.n_groups)
        select_group<kLargeThreads, UNITS, POOL, false>(a, blockIdx.x, m.group);
    else
        select_large<0>(a, blockIdx.x - a.n_groups, gridDim.x - a.n_groups, m.large);
}
template <int STEP>
__global__ __launch_bounds__(kLargeThreads) void fairkv_select_large_kernel(SelectArgs a)
{
    __shared__ LargeSpace<STEP> m;
    select_large<STEP>(a, blockIdx.x, gridDim.x, m);
}

}  // namespace fairkv
