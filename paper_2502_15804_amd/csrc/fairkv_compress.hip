// C ABI of the compression of a growing cache: argument checks, kernel selection and launches.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>
#include <initializer_list>

#include "attn_weights.h"
#include "cache_check.h"
#include "evict.h"
#include "fairkv.h"
#include "select.h"
#include "zero_words.h"

namespace {

using namespace fairkv;

constexpr int32_t kMovers = 8;            // workgroups of a compute unit that move rows into another cache
constexpr int64_t kMaxGroupsOfCall = 1 << 21;      // of a selection: a grid's threads are counted in 32 bits
constexpr int64_t kMaxPairsOfCall = 1 << 20;       // of an eviction: the same
constexpr int32_t kMaxSlots = 65536;      // most compute units that a caller may name
// Units of a group whose keys lie in a workgroup's LDS: four such workgroups of 512 threads share a CU's 160 KB, and two of 1024.  Beside the larger groups' first
// step three of 512: up to 10240 rows a workgroup is faster than the whole GPU in four steps (8 x 8 pairs of 1024 rows, shared, 23 us instead of 30; with 256
// units the step's own workgroups have too little room: 16 x 8 pairs of 10000 rows 37 instead of 31).
constexpr int32_t kSmallCap = 120, kLargeCap = 256, kMixedCap = 160;

// Tokens that a length or a list can count: 2^31 - 2^16, so that what is added to a token's number does not wrap around.
constexpr int32_t kMostTokens = INT32_MAX - 65535;
int32_t max_len(const fairkv_cache *c)
{
    const int64_t rows = c->n_rows < 1 ? 0 : c->pages ? static_cast<int64_t>(c->max_pages) * c->page_rows : c->n_rows;
    return static_cast<int32_t>(std::min<int64_t>(rows, kMostTokens));
}
// Whether two runs of bytes share one.
bool meet(const void *x, size_t nx, const void *y, size_t ny)
{
    const auto a = reinterpret_cast<uintptr_t>(x), b = reinterpret_cast<uintptr_t>(y);
    return a < static_cast<unsigned __int128>(b) + ny && b < static_cast<unsigned __int128>(a) + nx;
}
struct Bytes {
    const void *at;
    size_t n;
};
// Whether something that a call writes shares a byte with what it reads or with something else that it writes.  Those that are null are not there.
bool written_over(std::initializer_list<Bytes> written, std::initializer_list<Bytes> read)
{
    for (auto w = written.begin(); w != written.end(); ++w) {
        auto meets = [&](const Bytes &x) { return w->at && x.at && meet(w->at, w->n, x.at, x.n); };
        if (std::any_of(read.begin(), read.end(), meets) || std::any_of(w + 1, written.end(), meets)) return true;
    }
    return false;
}

// 16 waves of a compute unit (20 with heads of 64 and few columns: 64 x 8 pairs of 4096 8-bit rows 43 us instead of 48), in as many workgroups as its LDS
// has room for all columns of: a workgroup's waves wait for one another only where a pair begins.  64 queries x 8 heads over 64 x 8 pairs of 4096 rows, on one card: 316 us
// with 16 waves and 512 columns in LDS, 355 with 12; with two tiles of 32 tokens a wave 349 (12 waves), 365 (8) and 444 (16); with 128 columns in
// LDS at a time 859.  32 x 8 columns over 8 x 8 pairs of 16000 rows: 99 us in two workgroups of 8 waves or one of 16, 110 with 12 waves.
template <int D, bool KV8, int NW, int CC>
void launch_weights_kernel(const WeightsArgs &a, int32_t n_slots, hipStream_t st)
{
    hipLaunchKernelGGL((fairkv_attn_weights_kernel<D, KV8, NW, CC>), dim3(static_cast<unsigned>(n_slots) * (4 * kWeightWaves<D, NW> / NW)), dim3(NW * 64), 0, st, a);
}
template <int D, bool KV8>
void launch_weights(const WeightsArgs &a, int32_t n_slots, hipStream_t st)
{
    const int cols = a.G * a.q_len;
    if (cols <= 64)
        launch_weights_kernel<D, KV8, 4, 64>(a, n_slots, st);
    else if (cols <= 128)
        launch_weights_kernel<D, KV8, 4, 128>(a, n_slots, st);
    else if (cols <= 256)
        launch_weights_kernel<D, KV8, 8, 256>(a, n_slots, st);
    else
        launch_weights_kernel<D, KV8, 16, D == 128 ? 512 : 1024>(a, n_slots, st);
}

}  // namespace

extern "C" int fairkv_attn_weights(const fairkv_cache *c, const void *q, const uint64_t *tree, const int32_t *n_new, const int32_t *len,
                                   const float *lse, const float *weights, float *weights_out, float decay, int32_t n_slots, int32_t q_len,
                                   int32_t Hq, float scale, void *hip_stream)
{
    if (const int rc = check_cache(c)) return rc;
    if (!q || !len || !lse || !weights || !weights_out || Hq < 1 || q_len < 1 || n_slots < 1 || Hq % c->Hkv != 0) return FAIRKV_EINVAL;
    if (c->dtype == FAIRKV_F32 || q_len > FAIRKV_MAX_DRAFT || Hq / c->Hkv > 16 || n_slots > kMaxSlots) return FAIRKV_EUNSUPPORTED;
    if (!std::isfinite(scale) || !std::isfinite(decay)) return FAIRKV_EINVAL;
    if (!aligned(q, 16) || !aligned(lse, 4) || !aligned(weights, 4) || !aligned(weights_out, 4) || (tree && !aligned(tree, 8))) return FAIRKV_EINVAL;
    if (static_cast<int64_t>(c->B) * q_len * Hq * c->D > INT32_MAX) return FAIRKV_EINVAL;
    if (weights_out != weights && meet(weights, sizeof(float) * c->n_rows, weights_out, sizeof(float) * c->n_rows)) return FAIRKV_EINVAL;
    for (int32_t h = 0; h < std::max(c->n_scales, 1); ++h)
        if (!std::isfinite(scale * kLog2e * (c->n_scales > 0 ? c->k_scale[h] : 1.f))) return FAIRKV_EINVAL;
    WeightsArgs a{};
    a.q = static_cast<const char *>(q), a.k = static_cast<const char *>(c->k);
    a.rows = row_map(c);
    a.len = len, a.n_new = n_new, a.tree = reinterpret_cast<const int64_t *>(tree), a.lse = lse;
    a.weights = weights, a.out = weights_out;
    a.B = c->B, a.Hq = Hq, a.Hkv = c->Hkv, a.G = Hq / c->Hkv, a.q_len = q_len, a.max_len = max_len(c), a.n_scales = c->n_scales;
    a.scale_log2 = scale * kLog2e, a.decay = decay;
    for (int h = 0; h < kCacheScales; ++h) a.k_scale[h] = h < c->n_scales ? c->k_scale[h] : 1.f;
    hipStream_t st = static_cast<hipStream_t>(hip_stream);
    if (c->dtype == FAIRKV_E4M3)
        c->D == 128 ? launch_weights<128, true>(a, n_slots, st) : launch_weights<64, true>(a, n_slots, st);
    else
        c->D == 128 ? launch_weights<128, false>(a, n_slots, st) : launch_weights<64, false>(a, n_slots, st);
    return launched();
}

// ---- selection: which kernels a call takes --------------------------------------------------------
namespace {

struct SelectShape {
    int32_t cap, min_blocks;      // units of 64 rows of a group that one workgroup has; blocks that a larger one has at least
    int64_t max_blocks;           // of all larger groups, 0: there can be none
    int64_t slots, shares;        // of the large groups' kernels: groups, workgroups
};
SelectShape select_shape(const fairkv_cache *c, int32_t shared, int32_t n_slots)
{
    const int64_t pairs = static_cast<int64_t>(c->B) * c->Hkv, per_group = shared ? c->Hkv : 1;
    const int64_t each = max_len(c), most = std::min(std::max<int64_t>(c->n_rows, 0), each * pairs), group_most = std::min(most, each * per_group);
    SelectShape s{};
    auto fits = [&](int32_t cap) { return per_group <= kMaxPairs && (group_most + 63 * per_group) / 64 <= cap; };      // pairs' last units are not full
    s.cap = fits(kSmallCap) ? kSmallCap : kLargeCap;
    if (fits(s.cap)) return s;
    s.cap = kMixedCap;
    // A block of a pair has at most 64 units, so a large group has more than cap / 64 blocks; its rows are more than 64 cap - 63 per_group.
    s.min_blocks = per_group > kMaxPairs ? kMaxPairs : s.cap / (kBlockRows / 64) + 1;
    const int64_t least_rows = std::max<int64_t>(1, 64 * static_cast<int64_t>(s.cap) - 63 * per_group);
    const int64_t large_pairs = per_group > kMaxPairs ? pairs : std::min(pairs, most / least_rows * per_group);      // each has a block that is not full
    s.max_blocks = most / kBlockRows + large_pairs;
    s.slots = s.max_blocks / s.min_blocks + 1;
    s.shares = std::min<int64_t>(s.max_blocks, 4 * static_cast<int64_t>(n_slots));
    return s;
}
// What has to be zero when a call begins lies in the first third of a workspace, whatever the call's shape, and the rest in the others.
size_t start_bytes(const SelectShape &s) { return sizeof(SelectStart) * s.slots; }
size_t other_bytes(const SelectShape &s) { return sizeof(SelectSlot) * s.slots + sizeof(SelectShare) * s.shares + (sizeof(int32_t) + kLastBins * sizeof(uint16_t) + kBlockRows * sizeof(uint32_t)) * s.max_blocks; }
size_t third_of(size_t workspace_bytes) { return workspace_bytes / 3 / 256 * 256; }
size_t select_bytes(const SelectShape &s) { return 3 * ((std::max(start_bytes(s), (other_bytes(s) + 1) / 2) + 256) / 256 * 256); }

template <int NT, int UNITS>
void launch_select(const SelectArgs &a, unsigned groups, hipStream_t st)
{
    if (a.half > 0)
        hipLaunchKernelGGL((fairkv_select_kernel<NT, UNITS, true>), dim3(groups), dim3(NT), 0, st, a);
    else
        hipLaunchKernelGGL((fairkv_select_kernel<NT, UNITS, false>), dim3(groups), dim3(NT), 0, st, a);
}

}  // namespace

extern "C" size_t fairkv_select_workspace_bytes(const fairkv_cache *c, int32_t shared, int32_t n_slots)
{
    if (check_cache(c) != FAIRKV_OK || n_slots < 1 || n_slots > kMaxSlots || shared < 0 || shared > 1) return 0;
    return select_bytes(select_shape(c, shared, n_slots));
}

extern "C" int fairkv_select_workspace_reset(void *workspace, size_t workspace_bytes, void *hip_stream)
{
    if (!workspace || !aligned(workspace, 16)) return FAIRKV_EINVAL;
    if (workspace_bytes < select_bytes(SelectShape{})) return FAIRKV_EWORKSPACE;
    zero_words(workspace, workspace_bytes / 3 / sizeof(uint32_t), static_cast<hipStream_t>(hip_stream));
    return launched();
}

extern "C" int fairkv_select(const fairkv_cache *c, const fairkv_selection *s, const float *weights, const int32_t *len, int32_t *keep,
                             int32_t max_keep, int32_t *n_keep, int32_t *bad, void *workspace, size_t workspace_bytes, int32_t n_slots,
                             void *hip_stream)
{
    if (const int rc = check_cache(c)) return rc;
    if (!s || !s->budget || !weights || !len || !keep || !n_keep || max_keep < 1 || n_slots < 1) return FAIRKV_EINVAL;
    if (s->shared < 0 || s->shared > 1 || s->sink < 0 || s->recent < 0 || s->pool < 1 || s->pool % 2 == 0) return FAIRKV_EINVAL;
    if (s->pool > 2 * kMostHalf + 1 || n_slots > kMaxSlots) return FAIRKV_EUNSUPPORTED;
    if (!aligned(weights, 4) || !aligned(workspace, 16)) return FAIRKV_EINVAL;
    const int64_t pairs = static_cast<int64_t>(c->B) * c->Hkv, groups = s->shared ? c->B : pairs;
    if (groups > kMaxGroupsOfCall) return FAIRKV_EINVAL;
    const SelectShape shape = select_shape(c, s->shared, n_slots);
    if (!workspace || workspace_bytes < select_bytes(shape)) return FAIRKV_EWORKSPACE;
    // Workgroups read lengths, weights and tables while others write their lists.
    constexpr size_t word = sizeof(int32_t);
    if (written_over({{keep, word * pairs * max_keep}, {n_keep, word * pairs}, {bad, word}, {workspace, workspace_bytes}},
                     {{weights, sizeof(float) * c->n_rows}, {len, word * pairs}, {s->budget, word * groups}, {c->off, sizeof(int64_t) * pairs}, {c->pages, word * pairs * c->max_pages}}))
        return FAIRKV_EINVAL;
    SelectArgs a{};
    a.rows = row_map(c);
    a.weights = weights, a.len = len, a.budget = s->budget, a.keep = keep, a.n_keep = n_keep, a.bad = bad;
    a.n_pairs = static_cast<int32_t>(pairs), a.n_groups = static_cast<int32_t>(groups), a.max_len = max_len(c), a.max_keep = max_keep;
    a.half = s->pool / 2, a.sink = s->sink, a.recent = s->recent, a.per_group = s->shared ? c->Hkv : 1;
    a.cap = shape.cap, a.min_blocks = shape.min_blocks, a.max_blocks = shape.max_blocks;
    hipStream_t st = static_cast<hipStream_t>(hip_stream);
    if (shape.max_blocks == 0) {
        // Of few groups the wider workgroups are faster (8 pairs of 1024 rows in one group 10.3 us, 12.5 with 512 threads), of many the narrower ones, four of
        // which a compute unit has at once (128 x 8 groups of 1024 rows 18 us, 25 with 1024 threads, 23 with 256).
        if (shape.cap == kLargeCap)
            launch_select<1024, kLargeCap>(a, static_cast<unsigned>(groups), st);
        else if (groups <= n_slots)
            launch_select<1024, kSmallCap>(a, static_cast<unsigned>(groups), st);
        else
            launch_select<512, kSmallCap>(a, static_cast<unsigned>(groups), st);
        return launched();
    }
    char *others = static_cast<char *>(workspace) + third_of(workspace_bytes);
    a.starts = static_cast<SelectStart *>(workspace);
    a.slots = reinterpret_cast<SelectSlot *>(others);
    a.shares = reinterpret_cast<SelectShare *>(others + sizeof(SelectSlot) * shape.slots);
    a.above = reinterpret_cast<int32_t *>(others + sizeof(SelectSlot) * shape.slots + sizeof(SelectShare) * shape.shares);
    a.upto = reinterpret_cast<uint32_t *>(a.above + shape.max_blocks);
    a.keys = a.upto + shape.max_blocks * (kLastBins / 2);
    const dim3 grid(static_cast<unsigned>(shape.shares)), first(static_cast<unsigned>(groups + shape.shares)), threads(kLargeThreads);
    if (a.half > 0)
        hipLaunchKernelGGL((fairkv_select_first_kernel<kMixedCap, true>), first, threads, 0, st, a);
    else
        hipLaunchKernelGGL((fairkv_select_first_kernel<kMixedCap, false>), first, threads, 0, st, a);
    hipLaunchKernelGGL(fairkv_select_large_kernel<1>, grid, threads, 0, st, a);
    hipLaunchKernelGGL(fairkv_select_large_kernel<2>, grid, threads, 0, st, a);
    hipLaunchKernelGGL(fairkv_select_large_kernel<3>, grid, threads, 0, st, a);
    return launched();
}

// In place.  Whole rows (of fp32, halves) by a workgroup where there are pairs enough, or else 64 bytes of them, or 32 where that leaves half of the compute units
// without work.  128 x 8 pairs of 1024 bf16 rows halved 119 us with whole rows and 169 with 64 bytes, 8 x 8 pairs 32 and 16, 8 pairs of 131072 cut to a third 292 with 64
// bytes and 236 with 32.  256 threads a workgroup have shorter runs, 128 x 8 pairs of 4096 8-bit rows 372 us instead of 302 with 512, but wait less for one
// another where a list is short: of 200 rows (bf16) 27 us instead of 37.
namespace {
template <int ROWB, int WIDTH, int NT>
void launch_in_place(const EvictArgs &a, unsigned setters, hipStream_t st)
{
    hipLaunchKernelGGL((fairkv_evict_kernel<ROWB, WIDTH, NT>), dim3(evict_blocks(a.n_pairs, 2 * (ROWB / WIDTH)) + setters), dim3(NT), 0, st, a);
}
template <int ROWB>
void move_in_place(const EvictArgs &a, int32_t n_slots, unsigned setters, hipStream_t st)
{
    constexpr int WIDE = ROWB > 256 ? 256 : ROWB;
    if (a.n_pairs >= 2 * static_cast<int64_t>(n_slots))
        a.max_keep <= 1024 ? launch_in_place<ROWB, WIDE, 256>(a, setters, st) : launch_in_place<ROWB, WIDE, 512>(a, setters, st);
    else if (static_cast<int64_t>(a.n_pairs) * 2 * (ROWB / 64) * 2 > n_slots)
        launch_in_place<ROWB, 64, 512>(a, setters, st);
    else
        launch_in_place<ROWB, 32, 512>(a, setters, st);
}
}  // namespace

extern "C" int fairkv_evict(const fairkv_cache *c, const fairkv_cache *into, const int32_t *keep, int32_t max_keep, const int32_t *n_keep,
                            const int32_t *len, int32_t *len_out, const float *weights, float *weights_out, int32_t *bad, int32_t n_slots,
                            void *hip_stream)
{
    if (const int rc = check_cache(c)) return rc;
    const size_t row_bytes = static_cast<size_t>(c->D) * (c->dtype == FAIRKV_E4M3 ? 1 : c->dtype == FAIRKV_BF16 ? 2 : 4);
    if (into) {
        if (const int rc = check_cache(into)) return rc;
        if (into->B != c->B || into->Hkv != c->Hkv || into->D != c->D || into->dtype != c->dtype || into->n_scales != c->n_scales) return FAIRKV_EINVAL;
        for (int32_t h = 0; h < c->n_scales; ++h)      // bytes move as they are
            if (into->k_scale[h] != c->k_scale[h] || into->v_scale[h] != c->v_scale[h]) return FAIRKV_EINVAL;
        // Rows are written while others are read: the caches are one pool, or apart, and where they are one their pairs' rows are not the same.
        const bool pool = into->k == c->k && into->v == c->v && into->n_rows == c->n_rows;
        auto apart = [&](const void *x, const void *y) { return !meet(x, row_bytes * c->n_rows, y, row_bytes * into->n_rows); };
        const bool all_apart = apart(c->k, into->k) && apart(c->k, into->v) && apart(c->v, into->k) && apart(c->v, into->v);
        if (pool ? into->off == c->off && into->pages == c->pages : !all_apart) return FAIRKV_EINVAL;
        if (weights && !(pool && weights == weights_out) && meet(weights, sizeof(float) * c->n_rows, weights_out, sizeof(float) * into->n_rows)) return FAIRKV_EINVAL;
    }
    if (!keep || !n_keep || !len || !len_out || max_keep < 1 || n_slots < 1 || (weights == nullptr) != (weights_out == nullptr)) return FAIRKV_EINVAL;
    if (n_slots > kMaxSlots) return FAIRKV_EUNSUPPORTED;
    if (max_keep > kMostTokens) return FAIRKV_EINVAL;
    if (!aligned(weights, 4) || !aligned(weights_out, 4) || (!into && weights_out != weights)) return FAIRKV_EINVAL;
    const int64_t pairs = static_cast<int64_t>(c->B) * c->Hkv;
    if (pairs > kMaxPairsOfCall) return FAIRKV_EINVAL;
    const fairkv_cache *to = into ? into : c;
    const size_t words = sizeof(int32_t) * pairs;
    if (len_out != len && meet(len_out, words, len, words)) return FAIRKV_EINVAL;
    // Entries are read again once a list has been found right, while other workgroups write lengths, counts and weights.
    if (written_over({{len_out, words}, {bad, sizeof(int32_t)}, {weights_out, sizeof(float) * to->n_rows}},
                     {{keep, words * max_keep}, {n_keep, words}, {c->off, 2 * words}, {c->pages, words * c->max_pages}, {to->off, 2 * words}, {to->pages, words * to->max_pages},
                      {into ? into->cap : nullptr, words}}))
        return FAIRKV_EINVAL;
    // Rows of K and of V are moved by workgroups that do not wait for one another.
    if (meet(to->k, row_bytes * to->n_rows, to->v, row_bytes * to->n_rows)) return FAIRKV_EINVAL;
    EvictArgs a{};
    a.k = static_cast<const char *>(c->k), a.v = static_cast<const char *>(c->v);
    a.k_to = static_cast<char *>(to->k), a.v_to = static_cast<char *>(to->v);
    a.w = weights, a.w_to = weights_out;
    a.from = row_map(c), a.to = row_map(to);
    a.cap_to = into ? into->cap : nullptr;
    a.keep = keep, a.n_keep = n_keep, a.len = len, a.len_out = len_out, a.bad = bad;
    a.n_pairs = static_cast<int32_t>(pairs), a.max_keep = max_keep;
    hipStream_t st = static_cast<hipStream_t>(hip_stream);
    // Lengths that are written over those that the move reads are set behind it, by a kernel of their own.
    const bool over = len_out == len;
    const unsigned setters = over ? 0 : static_cast<unsigned>(pairs);
    // Blocks of 64 entries, or of 16 where lists as long as they can be do not give every wave one of those (8 pairs of 1024 rows halved: 5.4 us, 7.1 with 64).
    const int64_t most = n_slots * kMovers, few = pairs * ((static_cast<int64_t>(max_keep) + 63) / 64);
    const bool small = few <= 4 * most;
    a.movers = static_cast<int32_t>(std::min(most, small ? pairs * ((static_cast<int64_t>(max_keep) + 15) / 16) : few));
    auto move = [&](auto row_bytes) {
        constexpr int ROWB = decltype(row_bytes)::value;
        if (into && small)
            hipLaunchKernelGGL((fairkv_evict_into_kernel<ROWB, 16>), dim3(static_cast<unsigned>(a.movers) + setters), dim3(256), 0, st, a);
        else if (into)
            hipLaunchKernelGGL((fairkv_evict_into_kernel<ROWB, 64>), dim3(static_cast<unsigned>(a.movers) + setters), dim3(256), 0, st, a);
        else
            move_in_place<ROWB>(a, n_slots, setters, st);
    };
    if (row_bytes == 64)
        move(std::integral_constant<int, 64>{});
    else if (row_bytes == 128)
        move(std::integral_constant<int, 128>{});
    else if (row_bytes == 256)
        move(std::integral_constant<int, 256>{});
    else
        move(std::integral_constant<int, 512>{});
    if (const int rc = launched(); rc != FAIRKV_OK || !over) return rc;
    hipLaunchKernelGGL(fairkv_evict_lengths_kernel, dim3(static_cast<unsigned>(pairs)), dim3(256), 0, st, a);
    return launched();
}
