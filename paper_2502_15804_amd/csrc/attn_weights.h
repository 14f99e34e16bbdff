// The attention weight that the last tokens' queries give every row of a growing cache, added up.
//
// Mathematics.  A pair (b, h) has len rows, the last n = n_new[b] of them the queries' own.  With s = scale q . k and the log-sum-exp that the
// attention of the same queries left,
//     w[t] = decay w_old[t] [t < len - n] + sum over columns c = (node i < n, head g of the group) that see t of exp(s_ct - lse_c),
// the sums in fp32.  No maximum runs along: lse is at least every score that it is of.
//
// Tiles.  A wave has 32 tokens, whose rows of K it holds in registers as an operand of 32x32x16 matrix instructions, and goes through the
// columns 32 at a time:
//     S[column][token] = q K^T         D / 16 instructions a tile of 32
// A lane has one token (lane % 32) and 16 of the 32 columns, so a weight is added where it was computed; two lanes share a token.  Queries lie
// in LDS, for all waves of the workgroup, CC columns at a time.  Where fewer tiles are left than waves, several waves have one, other columns each, and one
// of them adds up: 256 columns over 8 pairs of 1000 rows 12 us instead of 18, 1024 over 8 pairs of 2000 rows 38 instead of 72.  Columns are added 32 by 32 in one
// order, so a weight is the same whichever waves have them.
//
// What bounds it (MI355X; times of a launch in a row of them).  Few columns: memory, 32 x 8 pairs of 4096 rows (bf16, heads of 128) 280 MB in 62 us
// (4.5 TB/s), and 4 to 5 us until the first rows are there, which is all that one sequence of 8 pairs of 1024 rows costs (4.6 us).  Many columns: power.
// 64 x 8 pairs of 4096 rows and 512 columns 316 to 336 us by card (830 to 880 TFLOP/s; a library's matrix product of 8192 rows has 1167) are 620 thousand
// cycles at 1.95 GHz, 266 thousand of matrix instructions beside 360 thousand of others, with 12 KB from LDS a wave for every 32 columns; the same instructions over numbers that are
// all alike take 530 thousand at 2.4 GHz.  In between, both: 256 columns over 8 x 8 pairs of 16000 rows 97 us (2.8 TB/s, 690 TFLOP/s), 67 without the columns'
// work, 90 without the rows' way from memory; matrix and other vector instructions are 158 of its 207 thousand cycles.  In short pairs waves wait (two thirds of
// their cycles: 32 trees of up to 8 nodes, heads of 64, 18 us): the line is dealt in tiles, but four waves take a turn together, and the longest workgroup has 4
// turns where 2 would do.  More columns than LDS holds wait half of the time (1024 over 8 x 8 pairs of 4096 rows, heads of 128, 131 us): one workgroup on a compute
// unit, which brings in 128 KB of queries and reads K in each of two passes.  Tried and slower: the next tile's rows in registers (spills at four waves of
// a SIMD, fewer waves without) or in LDS (fewer waves), two tiles a wave, scores of the next columns beside the weights of these, wave priorities.
#pragma once
#include "cache_rows.h"
#include "decode_mfma.h"
#include "line.h"

namespace fairkv {

typedef __attribute__((ext_vector_type(16))) float f32x16_t;

struct WeightsArgs {
    const char *q, *k;
    RowMap rows;
    const int32_t *len;               // [B * Hkv]
    const int32_t *n_new;             // [B] or null
    const int64_t *tree;              // [B][q_len] or null: node i sees nodes 0 .. i
    const float *lse;                 // [B][q_len][Hq]
    const float *weights;             // [n_rows], not read where decay is 0
    float *out;                       // [n_rows]
    int32_t B, Hq, Hkv, G, q_len, max_len, n_scales;
    float scale_log2, decay;
    float k_scale[kCacheScales];
};

// Waves of a SIMD that a launch counts on: what the registers allow.
template <int D, int NW>
constexpr int kWeightWaves = D == 64 && NW == 4 ? 5 : 4;

// NW waves, CC columns in LDS.
template <int D, bool KV8, int NW, int CC>
__global__ __launch_bounds__(NW * 64, (kWeightWaves<D, NW>)) void fairkv_attn_weights_kernel(WeightsArgs a)
{
    constexpr int NT = NW * 64, TOK = 32;
    constexpr int ROWB = KV8 ? D : 2 * D, QROWB = 2 * D;      // bytes of a row of K, of a query
    constexpr int NP = ROWB / 32, NSL = D / 16, PPQ = QROWB / 16;
    constexpr bool kMany = NW == 16 && CC < FAIRKV_MAX_DRAFT * 16;      // a pair may have more columns; the others' launches have no more
    // Tiles that several waves may have, each other columns: with up to 64 columns there are none, with all that LDS holds few.
    constexpr bool kSplit = CC > 64;
    constexpr int kShared = CC <= 256 ? NW / 2 : 2048 / CC;
    constexpr int AHEAD = CC > 64 ? 4 : 1;                            // pieces of queries that a thread asks for at once
    typedef __attribute__((ext_vector_type(4))) uint32_t u4;
    __shared__ __attribute__((aligned(1024))) char qs[CC * QROWB];
    __shared__ __attribute__((aligned(16))) float minus_lse[CC];      // in log2 units
    __shared__ uint64_t sees[CC];                                     // of every column: the nodes that it sees
    __shared__ float joins[kSplit ? kShared : 1][kSplit ? CC / 32 : 1][64];      // of tiles that several waves have, for every 32 columns

    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), l32 = lane & 31, hi = lane >> 5;
    const int n_pairs = a.B * a.Hkv;
    // Tokens of a pair that lie in the cache: none of a packed one whose run sticks out of it.
    auto len_of = [&](int p) __attribute__((always_inline)) {
        const int32_t len = min(max(a.len[p], 0), a.max_len);
        if (a.rows.pages) return len;
        const int64_t off = a.rows.off[p];
        return off >= 0 && static_cast<uint64_t>(off) + static_cast<uint32_t>(len) <= static_cast<uint64_t>(a.rows.n_rows) ? len : 0;
    };
    auto tiles_of = [](int32_t len) __attribute__((always_inline)) { return (static_cast<int64_t>(len) + TOK - 1) / TOK; };
    // Piece p of column c lies at piece p ^ swizzle(c): a row per lane, 16 of them take all banks.
    auto swizzle = [](int c) __attribute__((always_inline)) { return c / (256 / QROWB) % PPQ; };

    const LineShare share = line_share<NT>(n_pairs, gridDim.x, blockIdx.x, [&](int p) { return tiles_of(len_of(p)); });
    int pair = share.pair;
    int64_t first = share.begin, left = share.left;
    int32_t len = left > 0 ? __builtin_amdgcn_readfirstlane(len_of(pair)) : 0;      // (the compiler does not know that it is the same for all lanes)
    while (left > 0) {
        // ---- a run of tiles of one pair ----
        if (first >= tiles_of(len)) {
            pair = next_pair(pair, n_pairs, [&](int p) { return tiles_of(len_of(p)); }), first = 0;
            len = __builtin_amdgcn_readfirstlane(len_of(pair));
        }
        const int n_tiles = static_cast<int>(min(left, tiles_of(len) - first)), tile0 = static_cast<int>(first);
        const int b = pair / a.Hkv, h = pair - b * a.Hkv;
        const int32_t nn = a.n_new ? __builtin_amdgcn_readfirstlane(min(max(a.n_new[b], 0), a.q_len)) : a.q_len, base = len - nn;      // base: rows in front of the new ones
        const int cols = nn * a.G;
        const float s_mul = KV8 ? a.scale_log2 * a.k_scale[a.n_scales > 1 ? h : 0] : a.scale_log2;

        // More columns than LDS holds: the run's tiles are gone through once for each CC of them, what the others gave is added to.  (With all chunks of
        // columns in every turn: 64 queries x 16 heads over 8 x 8 pairs of 4096 rows 160 us.)
        for (int c_from = 0; c_from == 0 || (kMany && c_from < cols); c_from += CC) {
            const int chunk = kMany ? c_from / CC : 0;
            for (int turn = 0; turn * NW < n_tiles; ++turn) {
                // What comes of the number of columns is computed in every turn: held over the loop, it would take registers that a tile wants, and they
                // would be spilled (step over 64 x 8 pairs of 1024 rows 22 us instead of 20).
                int some_columns = kMany ? min(CC, cols - c_from) : cols;
                asm volatile("" : "+v"(some_columns));
                const int n = __builtin_amdgcn_readfirstlane(some_columns);
                // Where few tiles are left, 1 << shift waves have one, each every so many-th 32 of the columns.  The shift is that of the first columns in every pass, so
                // that a row's weight is read by the wave that wrote it.
                const int tiles = min(NW, n_tiles - turn * NW), n_shift = kMany ? min(CC, cols) : n;
                int shift = 0;
                while (kSplit && tiles <= kShared && tiles << (shift + 1) <= NW && 32 << shift < n_shift) ++shift;
                const int of_turn = wave >> shift, tile = tile0 + turn * NW + of_turn, part = wave & ((1 << shift) - 1);
                const bool mine = of_turn < tiles;
                const int32_t t0 = tile * TOK;
                // ---- rows of K, requested before the queries; where there is none the cache's first row stands in: what comes of it is not stored ----
                const int32_t t = t0 + l32;
                const int64_t row = mine && t < len ? a.rows.row(pair, t) : -1;
                const char *from = a.k + max(row, static_cast<int64_t>(0)) * ROWB + hi * 16;
                u4 raw[NP];
#pragma unroll
                for (int p = 0; p < NP; ++p) raw[p] = *reinterpret_cast<const u4 *>(from + p * 32);
                float old = 0.f;
                if (kMany && chunk > 0)
                    old = row >= 0 ? a.out[row] : 0.f;
                else
                    old = a.decay != 0.f && row >= 0 && t < base ? a.weights[row] * a.decay : 0.f;
                if (turn == 0) {
                    __syncthreads();
                    for (int x0 = threadIdx.x; x0 < n * PPQ; x0 += AHEAD * NT) {      // past the last piece: that one again
                        u4 piece[AHEAD];
#pragma unroll
                        for (int u = 0; u < AHEAD; ++u) {
                            const int x = min(x0 + u * NT, n * PPQ - 1), c = x / PPQ, p = x % PPQ, node = (chunk * CC + c) / a.G, g = chunk * CC + c - node * a.G;
                            piece[u] = *reinterpret_cast<const u4 *>(a.q + ((static_cast<size_t>(b) * a.q_len + node) * a.Hq + h * a.G + g) * QROWB + p * 16);
                        }
#pragma unroll
                        for (int u = 0; u < AHEAD; ++u) {
                            const int x = min(x0 + u * NT, n * PPQ - 1), c = x / PPQ, p = x % PPQ;
                            *reinterpret_cast<u4 *>(qs + c * QROWB + ((p ^ swizzle(c)) * 16)) = piece[u];
                        }
                    }
                    for (int c = threadIdx.x; c < n; c += NT) {
                        const int node = (chunk * CC + c) / a.G, g = chunk * CC + c - node * a.G;
                        const float lse = a.lse[(static_cast<size_t>(b) * a.q_len + node) * a.Hq + h * a.G + g];
                        minus_lse[c] = lse == -INFINITY ? -INFINITY : -lse * kLog2e;      // a node that sees nothing gives 0, or NaN to a row that is no number
                        sees[c] = a.tree ? static_cast<uint64_t>(a.tree[static_cast<size_t>(b) * a.q_len + node]) : ~0ull >> (63 - node);
                    }
                    __syncthreads();
                }
                if (!mine && shift == 0) continue;
                bf16x8_t k[NSL];
#pragma unroll
                for (int p = 0; p < NP; ++p) {
                    if constexpr (KV8) {
                        k[2 * p] = widen8(i32x2_t{static_cast<int>(raw[p][0]), static_cast<int>(raw[p][1])});
                        k[2 * p + 1] = widen8(i32x2_t{static_cast<int>(raw[p][2]), static_cast<int>(raw[p][3])});
                    } else {
                        k[p] = __builtin_bit_cast(bf16x8_t, raw[p]);
                    }
                }
                // 32 columns from c0.  some: not all of them are there; draft: some of the tile's tokens are the queries' own, and not seen by all; again: for a
                // tile of which a weight was NaN, without the nodes that see nothing
                float w = 0.f;
                auto columns = [&](int c0, auto some, auto draft, auto again, auto joined) __attribute__((always_inline)) {
                    constexpr bool kSome = decltype(some)::value, kDraft = decltype(draft)::value, kAgain = decltype(again)::value;
                    int at = l32, half = hi;
                    if constexpr (kAgain) asm volatile("" : "+v"(at), "+v"(half));      // or what comes of them would be kept in registers by tiles that never come here
                    const int c = kSome ? min(c0 + at, n - 1) : c0 + at;      // past the last one: that one again, and it does not count
                    bf16x8_t q[NSL];
#pragma unroll
                    for (int s = 0; s < NSL; ++s) {
                        const int p = KV8 ? (s & ~1) * 2 + 2 * half + (s & 1) : 2 * s + half;      // the order in which the lanes hold K
                        q[s] = *reinterpret_cast<const bf16x8_t *>(qs + c * QROWB + ((p ^ swizzle(kSome ? c : at)) * 16));
                    }
                    f32x16_t z;
#pragma unroll
                    for (int r = 0; r < 16; ++r) z[r] = 0.f;
#pragma unroll
                    for (int s = 0; s < NSL; ++s) z = __builtin_amdgcn_mfma_f32_32x32x16_bf16(q[s], k[s], z, 0, 0, 0);
                    const int32_t j = t0 + at - base;                          // of the queries' own tokens, below 0 in front of them
                    const uint32_t *words = reinterpret_cast<const uint32_t *>(sees) + (j >= 32 ? 1 : 0);
                    float s4[4] = {0.f, 0.f, 0.f, 0.f};
                    uint32_t sighted = 0;                                       // of the columns those whose node sees something
                    if constexpr (kAgain) {
                        const int node = (chunk * CC + c) / a.G, g = chunk * CC + c - node * a.G;
                        sighted = static_cast<uint32_t>(__builtin_amdgcn_ballot_w64(a.lse[(static_cast<size_t>(b) * a.q_len + node) * a.Hq + h * a.G + g] != -INFINITY));
                    }
#pragma unroll
                    for (int r4 = 0; r4 < 4; ++r4) {
                        if (kSome && c0 + 8 * r4 >= n) break;
                        const float4 ml4 = *reinterpret_cast<const float4 *>(minus_lse + c0 + 8 * r4 + 4 * half);
                        const float ml[4] = {ml4.x, ml4.y, ml4.z, ml4.w};
#pragma unroll
                        for (int x = 0; x < 4; ++x) {
                            const int cr = c0 + 8 * r4 + 4 * half + x;
                            float e = __builtin_amdgcn_exp2f(fmaf(z[4 * r4 + x], s_mul, ml[x]));
                            bool counts = true;
                            if constexpr (kSome) counts = cr < n;
                            if constexpr (kDraft) counts = counts && (j < 0 || (words[2 * min(cr, n - 1)] >> (j & 31) & 1) != 0);
                            if constexpr (kAgain) counts = counts && (sighted >> (8 * r4 + 4 * half + x) & 1) != 0;
                            s4[x] = r4 == 0 ? (counts ? e : 0.f) : s4[x] + (counts ? e : 0.f);
                        }
                    }
                    const float of_32 = (s4[0] + s4[1]) + (s4[2] + s4[3]);
                    if constexpr (decltype(joined)::value)
                        joins[of_turn][c0 / 32][lane] = of_32;
                    else
                        w += of_32;
                };
                auto all_columns = [&](int c0, int step, auto joined) __attribute__((always_inline)) {
                    constexpr std::true_type yes;
                    constexpr std::false_type no;
                    if (t0 + TOK > base) {
                        for (; c0 < n; c0 += step) columns(c0, yes, yes, no, joined);
                    } else {
                        for (; c0 + 32 <= n; c0 += step) columns(c0, no, no, no, joined);
                        if (c0 < n) columns(c0, yes, no, no, joined);
                    }
                };
                if (!kSplit || shift == 0)
                    all_columns(0, 32, std::false_type{});
                else if (mine)
                    all_columns(part * 32, 32 << shift, std::integral_constant<bool, kSplit>{});
                if (kSplit && shift > 0) {            // the same for all waves
                    __syncthreads();
                    if (!mine || part > 0) continue;
                    for (int x = 0; x * 32 < n; ++x) w += joins[of_turn][x][lane];      // in the order in which one wave adds
                }
                float both = w + __shfl_xor(w, 32);
                if (__builtin_amdgcn_ballot_w64(row >= 0 && both != both) != 0) {
                    w = 0.f;
#pragma unroll 1
                    for (int c0 = 0; c0 < n; c0 += 32) columns(c0, std::true_type{}, std::true_type{}, std::true_type{}, std::false_type{});
                    both = w + __shfl_xor(w, 32);
                }
                if (hi == 0 && row >= 0) a.out[row] = old + both;
            }
        }
        left -= n_tiles, first += n_tiles;
    }
}

}  // namespace fairkv
