// C ABI of a step over a growing cache: argument checks, kernel selection and launches.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>

#include "append_rotated.h"
#include "cache_check.h"
#include "decode_tree.h"
#include "fairkv.h"
#include "zero_words.h"

namespace {

using namespace fairkv;

size_t align256(size_t x) { return (x + 255) / 256 * 256; }

template <typename T, typename C>
void launch_rotated(int D, unsigned grid, hipStream_t st, const RotateArgs &a)
{
    if (D == 64)
        hipLaunchKernelGGL((fairkv_append_rotated_kernel<T, C, 64>), dim3(grid), dim3(256), 0, st, a);
    else
        hipLaunchKernelGGL((fairkv_append_rotated_kernel<T, C, 128>), dim3(grid), dim3(256), 0, st, a);
}

}  // namespace

extern "C" int fairkv_append_rotated(const fairkv_cache *c, const fairkv_rotation *r, const void *q, int64_t q_stride, const void *k_new,
                                     int64_t k_stride, const void *v_new, int64_t v_stride, void *q_out, int32_t q_len, int32_t Hq,
                                     int32_t dtype, const int32_t *n_new, const int32_t *len, int32_t *len_out, int32_t *bad, void *hip_stream)
{
    if (const int rc = check_cache(c)) return rc;
    if (!r || !q || !k_new || !v_new || !q_out || !len || !len_out || q_len < 1 || Hq < 1) return FAIRKV_EINVAL;
    if (dtype != FAIRKV_BF16 && dtype != FAIRKV_F32) return FAIRKV_EUNSUPPORTED;
    if ((dtype == FAIRKV_F32) != (c->dtype == FAIRKV_F32) || q_len > FAIRKV_MAX_DRAFT) return FAIRKV_EUNSUPPORTED;
    const int64_t elem = dtype == FAIRKV_BF16 ? 2 : 4, tokens = static_cast<int64_t>(c->B) * q_len;
    if (q_stride < static_cast<int64_t>(Hq) * c->D || k_stride < static_cast<int64_t>(c->Hkv) * c->D || v_stride < static_cast<int64_t>(c->Hkv) * c->D)
        return FAIRKV_EINVAL;
    if (q_stride % (16 / elem) != 0 || k_stride % (16 / elem) != 0 || v_stride % (16 / elem) != 0) return FAIRKV_EINVAL;
    if (!aligned(q, 16) || !aligned(k_new, 16) || !aligned(v_new, 16) || !aligned(q_out, 16)) return FAIRKV_EINVAL;
    if ((r->q_norm || r->k_norm) && !(r->eps >= 0.f && std::isfinite(r->eps))) return FAIRKV_EINVAL;
    if (r->table && (!r->pos || r->n_pos < 1 || r->rot < 16 || r->rot % 16 != 0 || r->rot > c->D || !aligned(r->table, 16))) return FAIRKV_EINVAL;
    if (tokens > INT32_MAX - 256) return FAIRKV_EINVAL;
    // Queries are written while others are read: q_out is q itself, token by token, or apart from all that is read.
    const int64_t q_row = static_cast<int64_t>(Hq) * c->D, kv_row = static_cast<int64_t>(c->Hkv) * c->D;
    auto meets = [&](const void *from, int64_t stride, int64_t row) {
        const auto read = reinterpret_cast<uintptr_t>(from), written = reinterpret_cast<uintptr_t>(q_out);
        const auto end = static_cast<unsigned __int128>(read) + (static_cast<unsigned __int128>(tokens - 1) * stride + row) * elem;
        return written < end && read < static_cast<unsigned __int128>(written) + static_cast<unsigned __int128>(tokens) * q_row * elem;
    };
    if (meets(k_new, k_stride, kv_row) || meets(v_new, v_stride, kv_row)) return FAIRKV_EINVAL;
    if (!(q_out == q && q_stride == q_row) && meets(q, q_stride, q_row)) return FAIRKV_EINVAL;

    RotateArgs a{};
    a.q = static_cast<const char *>(q), a.k_new = static_cast<const char *>(k_new), a.v_new = static_cast<const char *>(v_new);
    a.q_out = static_cast<char *>(q_out), a.k = static_cast<char *>(c->k), a.v = static_cast<char *>(c->v);
    a.q_norm = r->q_norm, a.k_norm = r->k_norm, a.table = r->table, a.pos = r->pos;
    a.n_new = n_new, a.len = len, a.cap = c->cap, a.len_out = len_out, a.bad = bad;
    a.rows = row_map(c);
    a.q_stride = q_stride, a.k_stride = k_stride, a.v_stride = v_stride;
    a.B = c->B, a.Hq = Hq, a.Hkv = c->Hkv, a.q_len = q_len, a.n_pos = r->n_pos, a.rot = r->table ? r->rot : 0, a.pairs = r->pairs;
    a.eps = r->eps;
    a.n_scales = c->n_scales;
    for (int32_t h = 0; h < c->n_scales; ++h) a.k_scale[h] = c->k_scale[h], a.v_scale[h] = c->v_scale[h];
    const int slots = 256 / (c->D / kRow8);
    a.head_slots = 1;
    while (a.head_slots * 2 <= std::min(Hq, slots)) a.head_slots *= 2;
    // As many passes as leave a thousand workgroups, what the card has at a time, and at most the 64 tokens that a wave's lanes look after.
    // 128 sequences x 64 tokens, 64 + 16 heads: 66 us, 68 and 72 with two and four thousand workgroups, 81 with one of every token;
    // 256 x 64 of which half are none: 95, 99, 104 and 126 with a workgroup's tokens one behind the other, 78 as they lie.
    const int64_t groups = (tokens + slots / a.head_slots - 1) / (slots / a.head_slots);
    a.passes = static_cast<int32_t>(std::clamp<int64_t>(groups / 1024, 1, 64 / (slots / a.head_slots)));
    const int64_t tokens_each = slots / a.head_slots * a.passes, pairs_each = std::max(1, slots / q_len);
    a.q_groups = static_cast<int32_t>((tokens + tokens_each - 1) / tokens_each);
    a.apart = static_cast<int32_t>(std::max<int64_t>(1, q_len / tokens_each));      // the passes of a workgroup go once through a sequence
    const int64_t grid = a.q_groups + (static_cast<int64_t>(c->B) * c->Hkv + pairs_each - 1) / pairs_each;
    if (grid > kMaxGroups) return FAIRKV_EINVAL;
    hipStream_t st = static_cast<hipStream_t>(hip_stream);
    if (dtype == FAIRKV_F32)
        launch_rotated<float, float>(c->D, static_cast<unsigned>(grid), st, a);
    else if (c->dtype == FAIRKV_BF16)
        launch_rotated<uint16_t, uint16_t>(c->D, static_cast<unsigned>(grid), st, a);
    else
        launch_rotated<uint16_t, uint8_t>(c->D, static_cast<unsigned>(grid), st, a);
    return launched();
}

extern "C" int fairkv_accept_weights(const fairkv_cache *c, float *weights, const int32_t *path, const int32_t *n_path, const int32_t *n_new,
                                     const int32_t *len, int32_t *len_out, int32_t q_len, int32_t *bad, void *hip_stream)
{
    if (const int rc = check_cache(c)) return rc;
    if (!path || !n_path || !len || !len_out || q_len < 1) return FAIRKV_EINVAL;
    if (q_len > FAIRKV_MAX_DRAFT) return FAIRKV_EUNSUPPORTED;
    if (!aligned(weights, 4)) return FAIRKV_EINVAL;
    const AcceptArgs a{static_cast<char *>(c->k), static_cast<char *>(c->v), path, n_path, n_new, len, len_out, bad, row_map(c), c->B, c->Hkv, q_len, weights};
    const int rb = c->D * (c->dtype == FAIRKV_E4M3 ? 1 : c->dtype == FAIRKV_BF16 ? 2 : 4), slots = 256 / (rb / 16), each = std::max(1, slots / q_len);
    const int64_t groups = (static_cast<int64_t>(c->B) * c->Hkv + each - 1) / each;
    if (groups > kMaxGroups) return FAIRKV_EINVAL;
    const dim3 grid(static_cast<unsigned>(groups));
    hipStream_t st = static_cast<hipStream_t>(hip_stream);
    if (rb == 64)
        hipLaunchKernelGGL(fairkv_accept_kernel<64>, grid, dim3(256), 0, st, a);
    else if (rb == 128)
        hipLaunchKernelGGL(fairkv_accept_kernel<128>, grid, dim3(256), 0, st, a);
    else if (rb == 256)
        hipLaunchKernelGGL(fairkv_accept_kernel<256>, grid, dim3(256), 0, st, a);
    else
        hipLaunchKernelGGL(fairkv_accept_kernel<512>, grid, dim3(256), 0, st, a);
    return launched();
}

extern "C" int fairkv_accept(const fairkv_cache *c, const int32_t *path, const int32_t *n_path, const int32_t *n_new, const int32_t *len,
                             int32_t *len_out, int32_t q_len, int32_t *bad, void *hip_stream)
{
    return fairkv_accept_weights(c, nullptr, path, n_path, n_new, len, len_out, q_len, bad, hip_stream);
}

// ---- attention of a draft tree --------------------------------------------------------------------
namespace {

// How the columns of a pair are dealt: `waves` waves side by side (32 columns each), `blocks` workgroups, and the slots of each of those.
struct TreeShape {
    int32_t waves, blocks, slots;
};
// Rows that the pairs of a cache are expected to have in all, or can have; what they do have is known on the device alone.
int64_t cache_rows(const fairkv_cache *c)
{
    const int64_t rows = std::min<int64_t>(c->n_rows, int64_t(1) << 48), pairs = static_cast<int64_t>(c->B) * c->Hkv;      // no product below leaves 64 bits
    const int64_t each = c->pages ? static_cast<int64_t>(c->max_pages) * c->page_rows : rows;
    const int64_t most = each > rows / pairs ? rows : each * pairs;
    return c->expected_rows > 0 ? std::min(c->expected_rows, most) : most;
}
// Waves side by side read a tile of K and V from LDS that came once for all of them; waves that take the tiles in turn cut a pair into fewer
// pieces, and have fewer columns to hand over at the end of each.  So it is the work of a workgroup that decides, in tiles of 32 columns by 32
// tokens, counted with the expected rows or full caches, a pair's own costs as 20.  Measured (bf16 outputs, D 128, 256 slots; us with 1, 2, 4, 8 waves
// side by side; * what the rule takes):
//     192 columns, 1 x 8 pairs of 4000 rows, work 27           21*  27   33   44
//     64 columns, 4 x 8 pairs of 8000 rows, 69                 37*  42   55   79
//     128 columns, 2 x 8 pairs of 8000 rows, 68                31*  36   42   55
//     64 columns, 8 x 8 pairs of 4000 rows, 73                 40*  39   45   67
//     128 columns, 16 x 8 pairs of 512 rows, 76                22*  18   27   32
//     192 columns, 1 x 8 pairs of 16000 rows, 98               39   41*  54   67
//     192 columns, 4 x 8 pairs of 4000 rows, 110               40   38*  47   61
//     128 columns, 16 x 8 pairs of 2000 rows, 169              57   45*  49   66   (8-bit: 43   37   47   68)
//     64 columns, 32 x 8 pairs of 2000 rows, 169               64   59*  67  103
//     512 columns, 4 x 8 pairs of 4000 rows, 294               76   64   69*  78
//     128 columns, 16 x 8 pairs of 4000 rows, 294              98   76   77* 115   (rows of all lengths around that: 101   84   74  113)
//     512 columns, 8 x 8 pairs of 4000 rows, 588              153  126  114* 120
//     128 columns, 32 x 8 pairs of 4000 rows, 588             202  151  131* 202
//     512 columns, 10 x 8 pairs of 4000 rows, 735             189  160  145  141*
//     512 columns, 16 x 8 pairs of 4000 rows, 1176            293  246  222  210*
// Next to a border the other side is as good or up to a fifth better: one number for columns, pairs and rows does not order all of them.
// More waves than columns need gain nothing at any size.  Slots come in eights where there are as many, so that the workgroups with the same
// rows and other columns, n_slots further on, share an XCD and its cache (192 columns, 1 x 8 pairs of 16000 rows: 39 us, against 60 with 42 slots).
TreeShape tree_shape(const fairkv_cache *c, int32_t Hq, int32_t q_len, int32_t n_slots)
{
    const int32_t cols = Hq / c->Hkv * q_len, blocks32 = (cols + 31) / 32;
    const int64_t work = (cache_rows(c) / 32 + 20 * static_cast<int64_t>(c->B) * c->Hkv) * blocks32 / n_slots;
    TreeShape s{};
    s.waves = std::min(work < 80 ? 1 : work < 200 ? 2 : work < 640 ? 4 : 8, blocks32 <= 2 ? blocks32 : blocks32 <= 4 ? 4 : 8);
    s.blocks = (cols + 32 * s.waves - 1) / (32 * s.waves);
    s.slots = std::max(1, n_slots / s.blocks);
    if (s.slots > 8) s.slots &= ~7;
    return s;
}

constexpr int32_t kTreeBlocks = 32;      // of 32 columns: 16 heads of 64 nodes

// The counters come first and take what n_slots alone says, so that calls of different shapes may share a workspace.  The partials take what the
// widest workgroups that a shape up to this one could have would leave in all slots, so that a workspace for the longest draft is one for every
// shorter one: waves do not fall with the columns, and blocks * waves, the columns' blocks rounded up, does not either.
struct TreeSpace {
    size_t counters, ml, o;
};
size_t tree_counters(int32_t n_slots) { return align256((static_cast<size_t>(n_slots) + kTreeBlocks) * 2 * kLevels * sizeof(int32_t)); }
TreeSpace tree_space(const TreeShape &s, int32_t D, int32_t n_slots)
{
    const size_t groups = static_cast<size_t>(std::max(n_slots, s.blocks)), cols = 32 * static_cast<size_t>(s.waves);      // at least blocks * slots
    return {tree_counters(n_slots), align256(groups * 2 * cols * 2 * sizeof(float)), align256(groups * 2 * cols * D * sizeof(float))};
}

int check_tree(const fairkv_cache *c, int32_t Hq, int32_t q_len, int32_t n_slots)
{
    if (const int rc = check_cache(c)) return rc;
    if (Hq < 1 || q_len < 1 || n_slots < 1 || Hq % c->Hkv != 0) return FAIRKV_EINVAL;
    if (c->dtype == FAIRKV_F32 || q_len > FAIRKV_MAX_DRAFT || Hq / c->Hkv > 16 || n_slots > kTreeSlots) return FAIRKV_EUNSUPPORTED;
    return FAIRKV_OK;
}

template <int D, bool KV8, int WC, int WT, int STAGES, int PARTS>
void launch_tree_kernel(const TreeArgs &a, int32_t blocks, hipStream_t st)
{
    hipLaunchKernelGGL((fairkv_decode_tree_kernel<D, KV8, WC, WT, STAGES, PARTS>), dim3(static_cast<unsigned>(a.n_slots), static_cast<unsigned>(blocks)),
                       dim3(WC * WT * 64), 0, st, a);
}

template <int D, bool KV8>
void launch_tree(int waves, bool fine, const TreeArgs &a, int32_t blocks, hipStream_t st)
{
    // What a weight is rounded to goes by the output's type alone: the width is a matter of speed, which hints and the size of a pool decide.
    switch (waves) {
    case 1: return fine ? launch_tree_kernel<D, KV8, 1, 4, 2, 3>(a, blocks, st) : launch_tree_kernel<D, KV8, 1, 4, 2, 2>(a, blocks, st);
    case 2: return fine ? launch_tree_kernel<D, KV8, 2, 4, 2, 3>(a, blocks, st) : launch_tree_kernel<D, KV8, 2, 4, 2, 2>(a, blocks, st);
    case 4: return fine ? launch_tree_kernel<D, KV8, 4, 2, 3, 3>(a, blocks, st) : launch_tree_kernel<D, KV8, 4, 2, 3, 2>(a, blocks, st);
    default: return fine ? launch_tree_kernel<D, KV8, 8, 1, 4, 3>(a, blocks, st) : launch_tree_kernel<D, KV8, 8, 1, 4, 2>(a, blocks, st);
    }
}

}  // namespace

extern "C" size_t fairkv_tree_workspace_bytes(const fairkv_cache *c, int32_t Hq, int32_t q_len, int32_t n_slots)
{
    if (check_tree(c, Hq, q_len, n_slots) != FAIRKV_OK) return 0;
    const TreeSpace s = tree_space(tree_shape(c, Hq, q_len, n_slots), c->D, n_slots);
    return s.counters + s.ml + s.o;
}

extern "C" size_t fairkv_tree_counter_bytes(int32_t n_slots) { return n_slots < 1 || n_slots > kTreeSlots ? 0 : tree_counters(n_slots); }

extern "C" int fairkv_tree_workspace_reset(void *workspace, size_t workspace_bytes, int32_t n_slots, void *hip_stream)
{
    const size_t need = fairkv_tree_counter_bytes(n_slots);
    if (!workspace || need == 0 || !aligned(workspace, 16)) return FAIRKV_EINVAL;
    if (workspace_bytes < need) return FAIRKV_EWORKSPACE;
    zero_words(workspace, need / sizeof(uint32_t), static_cast<hipStream_t>(hip_stream));
    return launched();
}

extern "C" int fairkv_decode_attn_tree(const fairkv_cache *c, const void *q, const uint64_t *tree, const int32_t *n_new, const int32_t *len,
                                       void *workspace, size_t workspace_bytes, int32_t n_slots, void *out, float *lse, int32_t q_len, int32_t Hq,
                                       int32_t out_dtype, float scale, void *hip_stream)
{
    if (const int rc = check_tree(c, Hq, q_len, n_slots)) return rc;
    if (!q || !len || !out || !std::isfinite(scale)) return FAIRKV_EINVAL;
    if (out_dtype != FAIRKV_BF16 && out_dtype != FAIRKV_F32) return FAIRKV_EUNSUPPORTED;
    if (!aligned(q, 16) || !aligned(out, 16) || !aligned(workspace, 16) || (tree && !aligned(tree, 8))) return FAIRKV_EINVAL;
    if (static_cast<int64_t>(c->B) * q_len * Hq * c->D > INT32_MAX) return FAIRKV_EINVAL;
    for (int32_t h = 0; h < std::max(c->n_scales, 1); ++h)      // a score's factor that is no number would make scores of 0 NaN
        if (!std::isfinite(scale * kLog2e * (c->n_scales > 0 ? c->k_scale[h] : 1.f))) return FAIRKV_EINVAL;
    const TreeShape shape = tree_shape(c, Hq, q_len, n_slots);
    const TreeSpace space = tree_space(shape, c->D, n_slots);
    if (!workspace || workspace_bytes < space.counters + space.ml + space.o) return FAIRKV_EWORKSPACE;

    TreeArgs a{};
    a.q = q, a.k = c->k, a.v = c->v;
    a.rows = row_map(c);
    a.len = len, a.n_new = n_new, a.tree = reinterpret_cast<const int64_t *>(tree);
    a.out = out, a.lse = lse;
    char *ws = static_cast<char *>(workspace);
    a.arrivals = reinterpret_cast<int32_t *>(ws);
    a.part_ml = reinterpret_cast<float *>(ws + space.counters);
    a.part_o = reinterpret_cast<float *>(ws + space.counters + space.ml);
    a.B = c->B, a.Hq = Hq, a.Hkv = c->Hkv, a.G = Hq / c->Hkv, a.q_len = q_len, a.cols = a.G * q_len;
    a.n_slots = shape.slots;
    // 2^31 - 2^16 tokens: what is added to a token's number inside a tile or a batch of pages does not wrap around
    const int64_t rows = c->n_rows < 1 ? 0 : c->pages ? static_cast<int64_t>(c->max_pages) * c->page_rows : c->n_rows;
    a.max_len = static_cast<int32_t>(std::min<int64_t>(rows, INT32_MAX - 65535));
    a.out_dtype = out_dtype;
    a.n_scales = c->n_scales;
    a.scale_log2 = scale * kLog2e;
    for (int h = 0; h < kCacheScales; ++h) {
        a.k_scale[h] = h < c->n_scales ? c->k_scale[h] : 1.f;
        a.v_scale[h] = h < c->n_scales ? c->v_scale[h] : 1.f;
    }
    hipStream_t st = static_cast<hipStream_t>(hip_stream);
    const bool fine = out_dtype == FAIRKV_F32;
    if (c->dtype == FAIRKV_E4M3)
        c->D == 128 ? launch_tree<128, true>(shape.waves, fine, a, shape.blocks, st) : launch_tree<64, true>(shape.waves, fine, a, shape.blocks, st);
    else
        c->D == 128 ? launch_tree<128, false>(shape.waves, fine, a, shape.blocks, st) : launch_tree<64, false>(shape.waves, fine, a, shape.blocks, st);
    return launched();
}
