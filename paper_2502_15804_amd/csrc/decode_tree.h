// Attention of a draft tree over a growing per-head cache.
//
// Mathematics.  A pair (b, h) has len rows, the last n = n_new[b] of them the draft's own.  Column c = (node i, head g of the group)
// sees every row in front of the draft and draft row j iff bit j of tree[b][i] is set:
//     out = sum_t 2^(s_t - m) v_t / sum_t 2^(s_t - m),   s_t = scale log2(e) q . k_t over the rows that are seen,
// in one pass over the rows with a running maximum m and sum, in fp32.
//
// Tiles.  A wave has 32 columns and works on 32 tokens at a time, with 32x32x16 matrix instructions:
//     S^T[token][column] = K q^T         D / 16 instructions
//     O^T[d][column]    += V^T P         D / 32 x 2 instructions
// A lane has one column (lane % 32) in scores, weights and outputs alike, and 16 of the 32 tokens (two lanes share a column).  The
// contraction index of the second product is taken in the order in which the first one leaves the tokens in a lane, so weights go from one
// to the other without leaving the lane, and V^T comes out of the LDS by the transposing read.
//
// WC waves side by side have 32 WC columns and share their tiles of K and V in LDS; WT such groups take the tiles of a run of tokens in turn
// and are added up at its end.  K and V go from HBM to LDS directly.
//
// Schedule.  Lengths change from step to step and stay on the GPU, so that a captured launch may be replayed while the cache grows: every
// workgroup adds up the lengths by itself and finds its share of the line of all pairs, each as long as its tiles and what a
// piece costs besides.  The pieces of a pair that is cut leave partial results in the workspace, and the workgroup that comes last adds them up,
// in the order of the pieces.
//
// What bounds it (MI355X, D 128, 8 KV heads, G 8; times of a launch in a row of them).  Long pairs with few columns: memory, 32 x 8 heavy-tailed
// pairs of 32 columns 166 MB in 39 us (4.3 TB/s).  Many columns: power, 64 x 8 pairs of 4096 rows and 512 columns 852 us (655 TFLOP/s, 980 with the
// weights' second halves; matrix cores busy in 46 % of the cycles while the clock falls from 2.3 to 1.6 GHz, so cycles that overlapping saves come
// back as a lower clock).  In between, the fixed parts: 5 us until the first tile is there (lengths, shares, first rows), 5 to 8 for a piece's
// queries, fold and join.  16 x 8 pairs of 1024 rows, 128 columns: 35 us, 32 from an 8-bit cache; one sequence with 24 nodes: 15 us.
#pragma once
#include "cache_rows.h"
#include "decode_mfma.h"

#include <type_traits>

namespace fairkv {

typedef __attribute__((ext_vector_type(16))) float f32x16_t;
typedef __attribute__((ext_vector_type(4))) uint32_t u32x4_t;

constexpr int kTreeTok = 32;          // tokens of a tile
constexpr int kTreeCols = 32;         // columns of a wave
constexpr int kJoin = 8;              // pieces of a pair that are added up at once
constexpr int kLevels = 6;            // of such sums, for pairs in up to 8^6 pieces
// What a piece costs besides its tiles, in tiles: queries, fold, outputs; a short pair that one wave has alone has no fold.  Measured with 6, 9
// and 13 a piece: 128 columns, 16 x 8 pairs of 2000 rows in fp32 63, 59 and 56 us (one wave side by side), 56, 52 and 53 us (four).  Short pairs
// of up to 4 or 8 tiles at 2 or 4: 32 x 8 heavy-tailed pairs of 32 columns 40.2 and 39.0, 43.6 and 41.8 us; 128 x 8 of 8 columns 34.4 and 33.2,
// 31.4 and 31.6 us.
constexpr int kPieceCost = 10, kSoloCost = 4;
constexpr int kTreeSlots = 65536;     // most workgroups of a block of columns
static_assert(kTreeSlots <= 1 << 3 * kLevels && kJoin == 8, "levels");

struct TreeArgs {
    const void *q, *k, *v;
    RowMap rows;
    const int32_t *len;               // [B * Hkv]
    const int32_t *n_new;             // [B] or null
    const int64_t *tree;              // [B][q_len] or null: node i sees nodes 0 .. i
    void *out;
    float *lse;
    float *part_o;                    // [column blocks][n_slots][2][D / 4][columns of a workgroup][4]
    float *part_ml;                   // [column blocks][n_slots][2][columns of a workgroup][2]
    int32_t *arrivals;                // [column blocks][kLevels][n_slots][2], 0 between calls
    int32_t B, Hq, Hkv, G, q_len, cols, n_slots, max_len, out_dtype, n_scales;
    float scale_log2;
    float k_scale[kCacheScales], v_scale[kCacheScales];
};

// Where a tile's rows lie in LDS.  A wave-wide load brings a chunk of 1 KB, kRows whole rows, and may put its 64 pieces of 16 bytes in any
// order: groups of `group` pieces, in a group the rows, in a row's place the group's pieces in turn.  So the pieces that a lane reads of its row
// are constants apart, which the instructions' immediate offsets hold.  K is read a row per lane: 16 rows (8-bit: twice as many, half a piece
// of each) take all 64 banks when a row is 16 `group` bytes behind the last and the chunks 16 bytes further apart.  V is read by the
// transposing instruction, 64 bytes of 4 rows or 32 bytes of 8 (8-bit; 0 .. 3 and 8 .. 11), which lie in one run of 256 bytes or two halves of it.
template <int ROWB, bool KV8>
struct TreeTile {
    static constexpr int kRows = 1024 / ROWB, kChunks = kTreeTok / kRows;
    static constexpr int kGroupK = ROWB == 256 ? 4 : ROWB == 128 ? 2 : 1, kGroupV = KV8 ? 2 : 4;
    static constexpr int kPitchK = ROWB == 64 ? 1024 : 1040, kPitchV = ROWB == 128 && KV8 ? 1152 : 1024;      // bytes from chunk to chunk
    static constexpr int kBytesK = kChunks * kPitchK, kStage = (kBytesK + kChunks * kPitchV + 255) / 256 * 256;
    // place of V's row r in its chunk and the row of a place: 64-byte rows with 4 .. 7 and 8 .. 11 swapped
    static __device__ __forceinline__ constexpr int place_v(int r) { return ROWB == 64 ? (r & 3) | (r >> 3 & 1) << 2 | (r >> 2 & 1) << 3 : r; }
    static __device__ __forceinline__ constexpr int piece(int group, int p) { return (p / group * kRows * group + p % group) * 16; }      // byte of piece p of row 0
};

// N wave-wide loads of 1 KB that lie 1 KB apart in memory, PITCH bytes apart in LDS: the instruction's immediate offset moves both addresses,
// so M0 is written once.  off[i] + PITCH i is the byte offset of load i from base.
template <int N, int PITCH>
__device__ __forceinline__ void load_chunks_to_lds(const void *base, const uint32_t (&off)[N], uint32_t lds_base)
{
    static_assert(N == 2 || N == 4, "loads of a run");
    uint64_t from;
    if constexpr (N == 2)
        asm volatile("s_mov_b32 m0, %4\n\ts_mov_b64 %0, %3\n\tglobal_load_lds_dwordx4 %1, %0 nt\n\t"
                     "global_load_lds_dwordx4 %2, %0 offset:%5 nt"
                     : "=&s"(from) : "v"(off[0]), "v"(off[1]), "s"(base), "s"(lds_base), "n"(PITCH) : "memory", "m0");
    else
        asm volatile("s_mov_b32 m0, %6\n\ts_mov_b64 %0, %5\n\tglobal_load_lds_dwordx4 %1, %0 nt\n\t"
                     "global_load_lds_dwordx4 %2, %0 offset:%7 nt\n\t"
                     "global_load_lds_dwordx4 %3, %0 offset:%8 nt\n\t"
                     "global_load_lds_dwordx4 %4, %0 offset:%9 nt"
                     : "=&s"(from) : "v"(off[0]), "v"(off[1]), "v"(off[2]), "v"(off[3]), "s"(base), "s"(lds_base), "n"(PITCH), "n"(2 * PITCH), "n"(3 * PITCH)
                     : "memory", "m0");
}

// Piece c of row r of the queries lies at piece c ^ query_swizzle(r): rows that fill the 256 bytes of all banks take different ones.
template <int ROWB>
__device__ __forceinline__ constexpr int query_swizzle(int r)
{
    return r / (256 / ROWB) % (ROWB / 16);
}

__device__ __forceinline__ float halves_max(float x)
{
    const uint32_t u = __float_as_uint(x);
    const auto a = __builtin_amdgcn_permlane32_swap(u, u, false, false);
    return fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
}
__device__ __forceinline__ float halves_sum(float x)
{
    const uint32_t u = __float_as_uint(x);
    const auto a = __builtin_amdgcn_permlane32_swap(u, u, false, false);
    return __uint_as_float(a[0]) + __uint_as_float(a[1]);
}

// Four consecutive outputs of a column that starts at element row_at of out; l, m as left by the softmax.
template <int D>
__device__ __forceinline__ void write_tree_out(const TreeArgs &a, uint32_t row, int d, float4 o, float m, float l, float v_mul)
{
    const float inv = l == 0.f ? 0.f : v_mul / l;
    const uint32_t at = row * D + d;
    if (a.out_dtype == FAIRKV_F32)
        *reinterpret_cast<float4 *>(static_cast<float *>(a.out) + at) = make_float4(o.x * inv, o.y * inv, o.z * inv, o.w * inv);
    else
        *reinterpret_cast<uint2 *>(static_cast<uint16_t *>(a.out) + at) = make_uint2(pack_bf16(o.x * inv, o.y * inv), pack_bf16(o.z * inv, o.w * inv));
    if (d == 0 && a.lse) a.lse[row] = l == 0.f ? -INFINITY : (m + __builtin_amdgcn_logf(l)) * kLn2;
}

// A column of the draft of a pair: its node and head, and the row of q and out.
struct Column {
    int node, head;
    __device__ __forceinline__ Column(const TreeArgs &a, int c) : node(c / a.G), head(c - node * a.G) {}
    __device__ __forceinline__ uint32_t row(const TreeArgs &a, int b, int h) const
    {
        return static_cast<uint32_t>((b * a.q_len + node) * a.Hq + h * a.G + head);
    }
};

__device__ __forceinline__ int32_t tree_new(const TreeArgs &a, int b)
{
    return a.n_new ? min(max(a.n_new[b], 0), a.q_len) : a.q_len;
}
// Tokens of a pair as far as a length can be one, and its place in the line.
__device__ __forceinline__ int32_t tree_len(const TreeArgs &a, int pair) { return min(max(a.len[pair], 0), a.max_len); }
__device__ __forceinline__ int32_t tiles_of(int32_t len) { return (len + kTreeTok - 1) / kTreeTok; }

// x plus those of the lanes below, by steps of the wave's own data paths.
__device__ __forceinline__ int64_t wave_upto(int64_t x)
{
    auto step = [&](auto ctrl, auto rows, auto banks) __attribute__((always_inline)) {
        const uint32_t lo = __builtin_amdgcn_update_dpp(0, static_cast<int>(x), ctrl(), rows(), banks(), false);
        const uint32_t hi = __builtin_amdgcn_update_dpp(0, static_cast<int>(x >> 32), ctrl(), rows(), banks(), false);
        x += static_cast<int64_t>((static_cast<uint64_t>(hi) << 32) | lo);
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

// A run of tiles of one pair.
struct TreePiece {
    int pair, b, h;
    int32_t len, nn, tiles, tile0, tile1;
    int from, apart;                  // this wave's tiles are tile0 + from, + apart, ...: its group's, or all of them
    bool solo;                        // a short pair that one wave has alone
    int64_t off;                      // first row of a packed pair, -1 if its run does not fit the cache
    int64_t first;                    // place of the pair's first tile in the line
};

// PARTS: a weight enters the second product as so many bf16 numbers, in as many times the instructions.  Three are all 24 bits of it and keep an
// fp32 output's accuracy; two are off by 2^-16 of a weight, which a bf16 output's own rounding, 2^-8, hides.  (One would be off by 2^-8 and make
// a bf16 output's error 1.4 times as large: 64 x 8 pairs of 4096 rows and 512 columns 670 us instead of 852.)
template <int D, bool KV8, int WC, int WT, int STAGES, int PARTS>
__global__ __launch_bounds__(WC *WT * 64, 1) void fairkv_decode_tree_kernel(TreeArgs a)
{
    constexpr int NW = WC * WT, NT = NW * 64, CB = WC * kTreeCols;
    constexpr int ROWB = KV8 ? D : 2 * D;             // bytes of a row of K or V
    using Tile = TreeTile<ROWB, KV8>;
    constexpr int RPI = Tile::kRows, LPT = Tile::kChunks;      // rows of a wave-wide load, loads of a tile of K
    constexpr int STAGEB = Tile::kStage;
    constexpr int LOADS = 2 * LPT >= WC ? 2 * LPT / WC : 1;     // a wave's share of the loads of a stage
    constexpr int NSL = D / 16, NDB = D / 32;
    constexpr int kAhead = WC == 1 ? STAGES : STAGES - 1;       // tiles on their way while one is waited for
    constexpr int RING = WT * STAGES * STAGEB;
    constexpr int kBlock = kTreeCols * 32 * 4;        // bytes of 32 coordinates of a wave's columns
    // A whole pair of at most so many tiles goes to one wave: no fold, four pairs side by side; of at most twice as many if the share has three of
    // those.  (128 x 8 pairs of 130 rows: 17.8 us, 31 without the longer ones, with rows of all lengths around that 31 and 36; 256 x 4 in 32
    // columns 48 and 60.  Always: 32 x 8 heavy-tailed pairs 42 us instead of 39, the other waves wait for the one.)
    constexpr int kSolo = WC == 1 && WT == 4 ? 4 : 0, kSoloMany = 2 * kSolo;
    auto overhead = [&](int tiles) __attribute__((always_inline)) { return tiles <= kSolo ? kSoloCost : kPieceCost; };
    constexpr int kRound = WT == 1 ? 0 : WC == 1 ? NDB : NDB / 2;      // such blocks of a group that are folded at once
    constexpr int FOLD = (WT - 1) * WC * kRound * kBlock;
    // The fold has memory of its own where that fits beside the ring, else the ring's last stage, which is empty then.
    constexpr bool kFoldInRing = RING + FOLD > 158 * 1024;
    constexpr int kFoldAt = kFoldInRing ? RING - WT * STAGEB : RING;
    static_assert(!kFoldInRing || FOLD <= WT * STAGEB, "a stage of all groups");
    // The queries of a piece come through LDS, whole rows at a time (straight into the registers a load would touch 32 rows): a wave's own 32 columns
    // into its ring's last stage, which is empty then; with waves side by side, the workgroup's into memory of their own, or the fold's.
    constexpr int QROWB = 2 * D, QBYTES = CB * QROWB;
    constexpr bool kOwnQueries = WC == 1;
    constexpr int kOwnMemory = RING + (kFoldInRing ? 0 : FOLD);
    constexpr bool kQueriesInFold = !kOwnQueries && kOwnMemory + QBYTES > 156 * 1024;
    static_assert(!kOwnQueries || QBYTES <= STAGEB, "a group's stage");
    static_assert(!kQueriesInFold || (!kFoldInRing && FOLD >= QBYTES), "the fold's memory");
    constexpr int kTail = (kFoldInRing ? 0 : FOLD) + (kOwnQueries || kQueriesInFold ? 0 : QBYTES);
    constexpr int kQueriesAt = kOwnQueries ? RING - WT * STAGEB : kQueriesInFold ? kFoldAt : kOwnMemory;
    static_assert(LOADS * kAhead < 64, "vmcnt is a 6-bit counter");
    static_assert(WT == 1 || NDB % kRound == 0, "rounds");

    constexpr int kTable = NT * 16;                   // what a pair's piece needs to know, of up to NT pairs; before the first fold
    __shared__ __attribute__((aligned(1024))) char lds[RING + (kTail > kTable ? kTail : kTable)];
    __shared__ uint32_t q_byte[CB];                   // of every column: its query behind those of the pair's first column
    __shared__ float2 st_ml[WT][CB];
    __shared__ int64_t scan[NW + 2];                  // totals of the waves; the pair the workgroup starts with and where it ends
    __shared__ int32_t counted;

    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wc = wave % WC, wt = wave / WC;
    const int l32 = lane & 31, hi = lane >> 5;
    const int n_pairs = a.B * a.Hkv, c0 = blockIdx.y * CB;
    const int my_slot = blockIdx.x;

    // ---- this workgroup's share of the line, which it walks from its end to its beginning: the piece at its end, whose pair goes on in the
    //      next workgroup, is done first, so that it is there when that one, having done the pair's other piece last, adds the two up ----
    for (int c = threadIdx.x; c < CB; c += NT) {
        const Column x(a, min(c0 + c, a.cols - 1));
        q_byte[c] = static_cast<uint32_t>(x.node * a.Hq + x.head) * QROWB;
    }
    int4 *const table = reinterpret_cast<int4 *>(lds + RING);
    const bool in_table = n_pairs <= NT;
    auto pair_entry = [&](int p) __attribute__((always_inline)) {      // length, new tokens, first row (-1: a run that does not fit the cache)
        const int32_t len = tree_len(a, p);
        int64_t off = a.rows.pages ? 0 : a.rows.off[p];
        if (off < 0 || (!a.rows.pages && static_cast<uint64_t>(off) + static_cast<uint32_t>(len) > static_cast<uint64_t>(a.rows.n_rows))) off = -1;
        return int4{len, tree_new(a, p / a.Hkv), static_cast<int32_t>(off), static_cast<int32_t>(off >> 32)};
    };
    int64_t begin, end, share, at;                    // at: where the pair ends
    int pair;
    bool small;                                       // places of the line fit 31 bits
    {
        const int run = (n_pairs + NT - 1) / NT, p0 = min(static_cast<int>(threadIdx.x) * run, n_pairs), p1 = min(p0 + run, n_pairs);
        int64_t mine = 0;
        if (in_table) {
            if (p0 < p1) {
                const int4 e = pair_entry(p0);
                table[p0] = e;
                mine = tiles_of(e.x) + overhead(tiles_of(e.x));
            }
        } else {
            for (int p = p0; p < p1; ++p) mine += tiles_of(tree_len(a, p)) + overhead(tiles_of(tree_len(a, p)));
        }
        const int64_t upto = wave_upto(mine);
        if (lane == 63) scan[wave] = upto;
        if (threadIdx.x == 0) scan[NW] = -1;
        __syncthreads();
        int64_t before = 0, total = 0;
#pragma unroll
        for (int w = 0; w < NW; ++w) {
            if (w < wave) before += scan[w];
            total += scan[w];
        }
        total = uniform64(total);
        small = total < (1ll << 30);
        share = small ? static_cast<uint32_t>(static_cast<uint32_t>(total) + a.n_slots - 1) / static_cast<uint32_t>(a.n_slots) : (total + a.n_slots - 1) / a.n_slots;
        share = uniform64(share);
        begin = share * my_slot;
        end = begin + share;
        before += upto - mine;
        const int64_t target = min(end, total) - 1;
        if (begin < total && before <= target && target < before + mine) {
            int p = p0;
            if (!in_table)
                for (; p < p1; ++p) {
                    const int cost = tiles_of(tree_len(a, p)) + overhead(tiles_of(tree_len(a, p)));
                    if (target < before + cost) break;
                    before += cost;
                }
            scan[NW] = p;
            scan[NW + 1] = before + (in_table ? mine : tiles_of(tree_len(a, p)) + overhead(tiles_of(tree_len(a, p))));
        }
        __syncthreads();
        pair = __builtin_amdgcn_readfirstlane(static_cast<int>(scan[NW]));
        at = uniform64(scan[NW + 1]);
    }
    if (pair < 0) return;                             // nothing is left of the line

    // ---- what depends on the lane alone ----
    const int col = c0 + wc * kTreeCols + l32;
    const Column column(a, min(col, a.cols - 1));
    const uint32_t ring = static_cast<uint32_t>(reinterpret_cast<uintptr_t>(FAIRKV_LDS_PTR(lds))) + wt * STAGEB;      // the group's stage 0
    constexpr uint32_t kStage = WT * STAGEB;          // from one stage of a group to the next
    // Where the lane reads in stage 0: its row of K, and its share of the transposing reads of V.
    const int x16 = lane & 15, dq = lane >> 4 & 1;
    const int v_row = KV8 ? (x16 < 8 ? x16 >> 1 : (x16 >> 1) + 4) + 4 * hi : 4 * hi + (x16 >> 2);
    const uint32_t k_rd = ring + l32 / RPI * Tile::kPitchK + l32 % RPI * Tile::kGroupK * 16 + (KV8 ? hi * 8 : hi * 16);
    const uint32_t v_rd = ring + Tile::kBytesK + v_row / RPI * Tile::kPitchV + Tile::place_v(v_row % RPI) * Tile::kGroupV * 16 +
                          (KV8 ? dq : 2 * dq + ((x16 & 3) >> 1)) * 16 + (x16 & 1) * 8;
    const char *const k_base = static_cast<const char *>(a.k), *const v_base = static_cast<const char *>(a.v);

    // ---- the pieces of the share: what 64 pairs' pieces need to know is held in lanes ----
    int held = pair;                                  // the pair of lane 0; lane i has the i-th before it
    int4 entry;
    entry = in_table ? table[max(pair - lane, 0)] : pair_entry(max(pair - lane, 0));
    if constexpr (!kOwnQueries) __syncthreads();      // the table's memory is the queries'
    int solo_most = kSolo;                            // tiles of a pair that one wave has alone
    if constexpr (kSolo > 0) {
        const int tiles = tiles_of(entry.x);
        const int64_t first = at - wave_upto(tiles + overhead(tiles)) + overhead(tiles);      // place of the lane's pair
        const bool fits = lane <= pair && tiles <= kSoloMany && first - overhead(tiles) >= begin && first + tiles <= end;
        if (__builtin_popcountll(__builtin_amdgcn_ballot_w64(fits)) >= 3) solo_most = kSoloMany;
    }
    auto next_piece = [&](TreePiece &pc) __attribute__((always_inline)) {      // false: the share has no more
        while (pair >= 0) {
            if (held - pair >= 64) {
                held = pair;
                entry = pair_entry(max(pair - lane, 0));
            }
            const int i = held - pair;
            pc.pair = pair;
            pc.b = pair / a.Hkv, pc.h = pair - pc.b * a.Hkv;
            pc.len = __builtin_amdgcn_readlane(entry.x, i), pc.nn = __builtin_amdgcn_readlane(entry.y, i);
            pc.off = static_cast<int64_t>((static_cast<uint64_t>(static_cast<uint32_t>(__builtin_amdgcn_readlane(entry.w, i))) << 32) |
                                          static_cast<uint32_t>(__builtin_amdgcn_readlane(entry.z, i)));
            pc.tiles = tiles_of(pc.len);
            pc.first = at - pc.tiles;
            at = pc.first - overhead(pc.tiles);
            pair = at <= begin ? -1 : pair - 1;
            pc.tile0 = static_cast<int32_t>(max(begin - pc.first, static_cast<int64_t>(0)));
            pc.tile1 = static_cast<int32_t>(min(end - pc.first, static_cast<int64_t>(pc.tiles)));
            const bool empty = pc.tiles == 0 && begin < pc.first && pc.first <= end;      // a pair without rows belongs to one workgroup too
            if ((pc.tile1 <= pc.tile0 && !empty) || c0 >= pc.nn * a.G) continue;
            pc.from = wt, pc.apart = WT, pc.solo = false;
            if constexpr (kSolo > 0) {
                pc.solo = pc.tile0 == 0 && pc.tile1 == pc.tiles && pc.tiles <= solo_most;
                if (pc.solo) {
                    pc.from = 0, pc.apart = 1;
                    if ((pc.pair & 3) != wave) continue;      // another wave's
                }
            }
            return true;
        }
        return false;
    };

    // The group's tiles of a piece: tile0 + wt, + WT, ...  Lane i holds the first cache rows of tile i's two halves of 16 tokens, for 64 tiles at
    // a time: -1 where the cache has none.  A half lies in one page.
    struct Rows {
        uint32_t lo[2], hi[2];
        __device__ __forceinline__ int64_t get(int half, int i) const
        {
            return static_cast<int64_t>((static_cast<uint64_t>(__builtin_amdgcn_readlane(hi[half], i)) << 32) | static_cast<uint32_t>(__builtin_amdgcn_readlane(lo[half], i)));
        }
    };
    auto fetch_pages = [&](const TreePiece &pc, int step) __attribute__((always_inline)) {      // page numbers of steps step .. step + 63, not waited for
        int2 ids = {0, 0};
        if (a.rows.pages && pc.len > 0) {
            const int t = min((pc.tile0 + pc.from + (step + lane) * pc.apart) * kTreeTok, pc.len - 1);
            const int32_t *of_pair = a.rows.pages + static_cast<int64_t>(pc.pair) * a.rows.max_pages;
            ids = {of_pair[t >> a.rows.page_shift], of_pair[min(t + 16, pc.len - 1) >> a.rows.page_shift]};
        }
        return ids;
    };
    auto rows_of = [&](const TreePiece &pc, int step, int2 ids) __attribute__((always_inline)) {
        Rows x;
        const int t = min((pc.tile0 + pc.from + (step + lane) * pc.apart) * kTreeTok, max(pc.len - 1, 0) & ~15);
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            const int th = half ? min(t + 16, max(pc.len - 1, 0) & ~15) : t;
            const int64_t row = a.rows.pages ? a.rows.row_of_page(half ? ids.y : ids.x, th) : pc.off < 0 ? -1 : pc.off + th;
            x.lo[half] = static_cast<uint32_t>(row), x.hi[half] = static_cast<uint32_t>(row >> 32);
            asm volatile("" : "+v"(x.lo[half]), "+v"(x.hi[half]));      // page numbers are waited for here and not where the lanes are read
        }
        return x;
    };
    // This wave's share of a stage: with more than one wave side by side all of it K or all of it V.  Loads of whole rows go in runs that neither
    // leave a half nor a wave's share.  Rows past the end of the pair are its last row again, rows that the cache does not have the cache's
    // first one: their weights are 0.  `missing` says of every stage which of its two halves the cache does not have.
    static_assert(WC == 1 || LPT % LOADS == 0, "a wave loads K or V");
    constexpr int kHalf = LPT / 2, kRun = kHalf < LOADS ? kHalf : LOADS;      // loads of a half, of a run
    const int load0 = wc * LOADS;                     // the wave's first load of a stage
    const bool loads = 2 * LPT >= WC || load0 < 2 * LPT;
    auto is_v = [&](int x) __attribute__((always_inline)) { return WC == 1 ? x >= LPT : load0 >= LPT; };
    auto nth = [&](int x) __attribute__((always_inline)) { return WC == 1 ? x % LPT : load0 % LPT + x; };      // load of the tile of K or V
    // The row of its chunk that the lane fetches of K and of V, and the byte of that row.
    constexpr int kKinds = WC == 1 ? 2 : 1;           // of a wave's loads
    int ld_row[kKinds];
    uint32_t ld_byte[kKinds], run_offset[kKinds][kRun];
    constexpr int kBehind = 512;                      // runs start so many bytes early: from load to load more is added to both addresses than to the global one
#pragma unroll
    for (int kind = 0; kind < kKinds; ++kind) {
        const bool v = is_v(kind * LPT);
        const int group = v ? Tile::kGroupV : Tile::kGroupK, at_row = lane / group % RPI;
        ld_row[kind] = v ? Tile::place_v(at_row) : at_row;
        ld_byte[kind] = (lane / (RPI * group) * group + lane % group) * 16;
#pragma unroll
        for (int x = 0; x < kRun; ++x) {
            run_offset[kind][x] = kBehind + ld_row[kind] * ROWB + ld_byte[kind] - x * ((v ? Tile::kPitchV : Tile::kPitchK) - 1024);
            asm volatile("" : "+v"(run_offset[kind][x]));
        }
    }
    static_assert((kRun - 1) * (Tile::kPitchV - 1024) <= kBehind && (kRun - 1) * (Tile::kPitchK - 1024) <= kBehind, "offsets are not negative");
    uint32_t missing = 0;
    auto place_of = [&](uint32_t stage, int x) __attribute__((always_inline)) { return stage + (is_v(x) ? Tile::kBytesK + nth(x) * Tile::kPitchV : nth(x) * Tile::kPitchK); };
    auto fetch = [&](const TreePiece &pc, const Rows &rows, int step, int at_stage) __attribute__((always_inline)) {
        const int last = pc.len - 1 - (pc.tile0 + pc.from + step * pc.apart) * kTreeTok;
        const uint32_t stage = ring + at_stage * kStage;
        const int64_t row0 = rows.get(0, step & 63), row1 = rows.get(1, step & 63);
        const bool full = last >= kTreeTok - 1 && (row0 | row1) >= 0;
        missing &= ~(3u << 2 * at_stage);
        if (!full) missing |= ((row0 < 0 ? 1u : 0u) | (row1 < 0 ? 2u : 0u)) << 2 * at_stage;      // a wave that loads nothing masks too
        if (!loads) return;
        if (full) {
#pragma unroll
            for (int x = 0; x < LOADS; x += kRun) {
                const char *from = (is_v(x) ? v_base : k_base) + ((nth(x) >= kHalf ? row1 : row0) + nth(x) % kHalf * RPI) * ROWB - kBehind;
                const uint32_t (&offsets)[kRun] = run_offset[WC == 1 && x >= LPT ? 1 : 0];
                if constexpr (kRun == 1)
                    load16_to_lds(from, offsets[0], place_of(stage, x));
                else if (is_v(x))
                    load_chunks_to_lds<kRun, Tile::kPitchV>(from, offsets, place_of(stage, x));
                else
                    load_chunks_to_lds<kRun, Tile::kPitchK>(from, offsets, place_of(stage, x));
            }
        } else {
#pragma unroll
            for (int x = 0; x < LOADS; ++x) {
                const int kind = WC == 1 && x >= LPT ? 1 : 0;
                const bool upper = nth(x) >= kHalf;
                const int64_t row = upper ? row1 : row0;
                const int behind = row < 0 ? 0 : min(nth(x) * RPI + ld_row[kind], last) - (upper && last >= 16 ? 16 : 0);
                load16_to_lds((is_v(x) ? v_base : k_base) + max(row, static_cast<int64_t>(0)) * ROWB, behind * ROWB + ld_byte[kind], place_of(stage, x));
            }
        }
    };
    auto mine_of = [&](const TreePiece &pc) __attribute__((always_inline)) { return WT == 1 ? pc.tile1 - pc.tile0 : pc.solo ? pc.tiles : max(0, (pc.tile1 - pc.tile0 - wt + WT - 1) / WT); };
    // A piece's first tile is requested with its queries, the others when both are there: all at once, and with them every workgroup's, the memory
    // would answer in no fair order.
    auto begin_ring = [&](const TreePiece &pc, const Rows &rows) __attribute__((always_inline)) {
        if (mine_of(pc) > 0) fetch(pc, rows, 0, 0);
    };
    auto wait_stage = [&](int later) __attribute__((always_inline)) {      // all but the loads of `later` stages have landed
        if (later <= 0)
            wait_vmcnt<0>();
        else if (later == 1)
            wait_vmcnt<LOADS>();
        else if (later == 2)
            wait_vmcnt<2 * LOADS>();
        else
            wait_vmcnt<3 * LOADS>();
    };
    static_assert(kAhead <= 4, "stages waited for");
    // The lane's column of the queries, and what it sees of the draft: requested, and read when they have come.
    bf16x8_t qb[NSL];
    uint64_t tree_word = 0;
    auto request_queries = [&](const TreePiece &pc) __attribute__((always_inline)) {
        constexpr int PPQ = QROWB / 16, RPQ = 64 / PPQ, QL = QBYTES / 1024, SHARE = kOwnQueries ? QL : (QL + NW - 1) / NW;      // loads, a wave's of them
        const char *from = static_cast<const char *>(a.q) + (static_cast<size_t>(pc.b) * a.q_len * a.Hq + static_cast<size_t>(pc.h) * a.G) * QROWB;
        const uint32_t to = static_cast<uint32_t>(reinterpret_cast<uintptr_t>(FAIRKV_LDS_PTR(lds))) + kQueriesAt + (kOwnQueries ? wt * STAGEB : 0);
#pragma unroll
        for (int x = 0; x < SHARE; ++x) {
            const int load = kOwnQueries ? x : wave * SHARE + x, r = load * RPQ + lane / PPQ;
            if (QL % SHARE != 0 || QL < NW) {
                if (load >= QL) break;
            }
            load16_to_lds_keep(from, q_byte[r] + ((lane % PPQ) ^ query_swizzle<QROWB>(r)) * 16, to + load * 1024);
        }
        tree_word = a.tree ? static_cast<uint64_t>(a.tree[pc.b * a.q_len + column.node]) : ~0ull >> (63 - column.node);
    };
    auto take_queries = [&]() __attribute__((always_inline)) {
        asm volatile("" : "+v"(tree_word));           // waited for here: in the loop, every turn would wait for all tiles
        drain_vmem();
        if constexpr (!kOwnQueries) __syncthreads();
        const uint32_t at_q = static_cast<uint32_t>(reinterpret_cast<uintptr_t>(FAIRKV_LDS_PTR(lds))) + kQueriesAt + (kOwnQueries ? wt * STAGEB : wc * kTreeCols * QROWB) +
                              l32 * QROWB + ((query_swizzle<QROWB>(l32) ^ hi) * 16);
#pragma unroll
        for (int s = 0; s < NSL; ++s) qb[s] = *lds_at<bf16x8_t>(at_q ^ (32 * s));
#pragma unroll
        for (int s = 0; s < NSL; ++s) asm volatile("" : "+v"(qb[s]));      // (and have left the LDS)
        if constexpr (!kOwnQueries) __syncthreads();
    };

    TreePiece pc;
    if (!next_piece(pc)) return;
    Rows rows = rows_of(pc, 0, fetch_pages(pc, 0));
    begin_ring(pc, rows);
    request_queries(pc);

    for (;;) {
        TreePiece ahead;
        const bool more = next_piece(ahead);
        int2 pages_ahead = {0, 0};
        if (more) pages_ahead = fetch_pages(ahead, 0);

        const int32_t base = pc.len - pc.nn;          // rows in front of the draft
        const int sc = a.n_scales > 1 ? pc.h : 0;
        // Scores to log2 units by a factor above 0 (a mask's -inf stays one; a factor of 0 is one under which every score is): the sign goes into q.
        const float s_mul = KV8 ? a.scale_log2 * a.k_scale[sc] : a.scale_log2, s_abs = fmaxf(fabsf(s_mul), 1e-37f);
        const int n_mine = mine_of(pc), n_steps = (pc.tile1 - pc.tile0 + WT - 1) / WT;
        f32x16_t o[NDB];
        float m_run = -INFINITY, l_run = 0.f;
#pragma unroll
        for (int nb = 0; nb < NDB; ++nb)
#pragma unroll
            for (int i = 0; i < 16; ++i) o[nb][i] = 0.f;

        auto more_rows = [&](int step) __attribute__((always_inline)) {
            rows = rows_of(pc, step, fetch_pages(pc, step));
            __builtin_amdgcn_s_waitcnt(0x0F70);       // said to the compiler, which would wait in every turn of the loop
        };
        take_queries();
        const uint64_t sees = tree_word & (pc.nn >= 64 ? ~0ull : (1ull << pc.nn) - 1);
        if (s_mul < 0.f) {
#pragma unroll
            for (int s = 0; s < NSL; ++s) qb[s] = __builtin_bit_cast(bf16x8_t, __builtin_bit_cast(u32x4_t, qb[s]) ^ 0x80008000u);
        }

#pragma clang loop unroll(disable)
        for (int s = 1; s < min(n_mine, kAhead); ++s) fetch(pc, rows, s, s);
        int c_stage = 0, free_stage = WC == 1 ? 0 : STAGES - 1;      // the stage of this step, and the one that is filled in it
        auto turn = [&]() __attribute__((always_inline)) {
            c_stage = c_stage == STAGES - 1 ? 0 : c_stage + 1;
            free_stage = free_stage == STAGES - 1 ? 0 : free_stage + 1;
        };
        for (int step = 0; step < (WC == 1 ? n_mine : n_steps); ++step, turn()) {
            wait_stage(min(n_mine - 1 - step, kAhead - 1));
            if constexpr (WC > 1) {
                // every wave's loads of this stage have landed, and every wave is through with the stage before, which the next loads fill
                asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
                const int next = step + kAhead;
                if (next < n_mine) {
                    if ((next & 63) == 0) more_rows(next);
                    fetch(pc, rows, next, free_stage);
                }
                if (step >= n_mine) continue;
            }
            const uint32_t stage = c_stage * kStage;
            const int32_t t0 = (pc.tile0 + pc.from + step * pc.apart) * kTreeTok;
            // ---- every LDS read of the tile, issued together: the scores wait for those of K, those of V come meanwhile ----
            bf16x8_t kw[NSL], va[2][NDB];
            i32x2_t kw8[NSL], va8[2][NDB];
#pragma unroll
            for (int s = 0; s < NSL; ++s) {
                if constexpr (KV8)
                    kw8[s] = *lds_at<i32x2_t>(k_rd + stage + Tile::piece(Tile::kGroupK, s));
                else
                    kw[s] = *lds_at<bf16x8_t>(k_rd + stage + Tile::piece(Tile::kGroupK, 2 * s));
            }
#pragma unroll
            for (int j = 0; j < 2; ++j)
#pragma unroll
                for (int nb = 0; nb < NDB; ++nb) {
                    if constexpr (KV8) {
                        const uint32_t at_v = v_rd + stage + Tile::piece(Tile::kGroupV, 2 * nb) + j * (16 / RPI) * Tile::kPitchV;
                        va8[j][nb] = __builtin_amdgcn_ds_read_tr8_b64_v2i32(lds_at<i32x2_t>(at_v));
                    } else {
                        const uint32_t at_v = v_rd + stage + Tile::piece(Tile::kGroupV, 4 * nb) + j * (16 / RPI) * Tile::kPitchV;
                        const uint2 x = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16(lds_at<i16x4_t>(at_v)));
                        const uint2 y = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16(lds_at<i16x4_t>(at_v + 8 / RPI * Tile::kPitchV)));
                        va[j][nb] = __builtin_bit_cast(bf16x8_t, u32x4_t{x.x, x.y, y.x, y.y});
                    }
                }
            __builtin_amdgcn_sched_barrier(0);

            // ---- scores; element r of a lane: token t0 + 8 (r / 4) + 4 hi + r % 4 ----
            f32x16_t sacc;
#pragma unroll
            for (int i = 0; i < 16; ++i) sacc[i] = 0.f;
#pragma unroll
            for (int s = 0; s < NSL; ++s) {
                if constexpr (KV8) kw[s] = widen8(kw8[s]);
                sacc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kw[s], qb[s], sacc, 0, 0, 0);
            }
            if constexpr (KV8) {
#pragma unroll
                for (int j = 0; j < 2; ++j)
#pragma unroll
                    for (int nb = 0; nb < NDB; ++nb) va[j][nb] = widen8(va8[j][nb]);
            }

            // ---- what is not seen: rows of the draft, rows past the end, rows that the cache does not have ----
            const uint32_t lacks = missing >> 2 * c_stage & 3;
            const bool masked = t0 + kTreeTok > base || lacks != 0;
            uint32_t seen = ~0u;                      // bit 8 (r / 4) + r % 4
            if (masked) {
                const int shift = t0 + 4 * hi - base;
                if (shift >= 0)
                    seen = shift < 64 ? static_cast<uint32_t>(sees >> shift) : 0u;
                else if (shift > -32)
                    seen = static_cast<uint32_t>(sees << -shift) | ((1u << -shift) - 1);
                if (lacks & 1) seen &= 0xffff0000u;
                if (lacks & 2) seen &= 0x0000ffffu;
#pragma unroll
                for (int r = 0; r < 16; ++r)
                    if (!(seen >> (8 * (r / 4) + r % 4) & 1)) sacc[r] = -INFINITY;
            }

            // ---- a reference maximum, in log2 units, that is raised when some score is far above it ----
            float mx = sacc[0];
#pragma unroll
            for (int r = 1; r < 16; ++r) mx = fmaxf(mx, sacc[r]);
            mx *= s_abs;
            if (__builtin_amdgcn_ballot_w64(mx > m_run + kBump) != 0) {
                const float m_new = fmaxf(m_run, halves_max(mx));
                const float alpha = m_new == m_run ? 1.f : __builtin_amdgcn_exp2f(m_run - m_new);
                l_run *= alpha;
#pragma unroll
                for (int nb = 0; nb < NDB; ++nb)
#pragma unroll
                    for (int i = 0; i < 16; ++i) o[nb][i] *= alpha;
                m_run = m_new;
            }
            const float m_ref = m_run == -INFINITY ? 0.f : m_run;      // nothing seen yet: weights of 0

            // ---- weights, as PARTS bf16 numbers that add up to them: the upper half, that of what it leaves, and the last rounded.  All of them
            //      are positive if the weight is, so an infinite V stays one: of a part that would be 0 the smallest number of bf16, 2^-133, is
            //      left (0 for a weight of 0).  The largest weight is at least 1, and one below 2^-126 is 0, as fp32 has it.  8-bit rows have no infinity. ----
            uint32_t pw[PARTS][8], ones = 0x00010001u;
            asm("" : "+s"(ones));                     // a minimum with a known 1 becomes two compares and two selects
#pragma unroll
            for (int r = 0; r < 16; r += 2) {
                float p0 = __builtin_amdgcn_exp2f(fmaf(sacc[r], s_abs, -m_ref)), p1 = __builtin_amdgcn_exp2f(fmaf(sacc[r + 1], s_abs, -m_ref));
                l_run += p0 + p1;
                u16x2_t least{};
#pragma unroll
                for (int part = 0; part < PARTS; ++part) {
                    uint32_t w = part == PARTS - 1 ? pack_bf16(p0, p1) : __builtin_amdgcn_perm(__float_as_uint(p1), __float_as_uint(p0), 0x07060302u);
                    p0 -= bf16_hi(__float_as_uint(p0)), p1 -= bf16_hi(__float_as_uint(p1));      // exact
                    if (!KV8 && part == 0) least = __builtin_elementwise_min(__builtin_bit_cast(u16x2_t, w), __builtin_bit_cast(u16x2_t, ones));
                    if (!KV8 && part > 0) w = __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2_t, w), least));
                    pw[part][r / 2] = w;
                }
            }

            if (masked) {
                // A weight of 0 times an infinite or NaN V is NaN: such elements go past the product, to the columns that see them only.
                uint32_t large = 0;
#pragma unroll
                for (int j = 0; j < 2; ++j)
#pragma unroll
                    for (int nb = 0; nb < NDB; ++nb) {
                        const u32x4_t w = __builtin_bit_cast(u32x4_t, va[j][nb]);
#pragma unroll
                        for (int i = 0; i < 4; ++i)
                            large = __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2_t, large), __builtin_bit_cast(u16x2_t, w[i] & 0x7fff7fffu)));
                    }
                const bool any = (large & 0xffffu) >= 0x7f80u || (large >> 16) >= 0x7f80u;
                if (__builtin_amdgcn_ballot_w64(any) != 0) {
                    bf16x8_t sees_row[2];             // 1 where the column sees the row
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        u32x4_t w;
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const int r = 8 * j + 2 * i, at_bit = 8 * (r / 4) + r % 4;
                            w[i] = (seen >> at_bit & 1 ? 0x3f80u : 0u) | (seen >> (at_bit + 1) & 1 ? 0x3f800000u : 0u);
                        }
                        sees_row[j] = __builtin_bit_cast(bf16x8_t, w);
                    }
#pragma unroll
                    for (int nb = 0; nb < NDB; ++nb) {
#pragma unroll
                        for (int kind = 0; kind < 3; ++kind) {          // +inf, -inf, NaN: how many of them a column sees
                            f32x16_t count;
#pragma unroll
                            for (int i = 0; i < 16; ++i) count[i] = 0.f;
#pragma unroll
                            for (int j = 0; j < 2; ++j) {
                                const u32x4_t w = __builtin_bit_cast(u32x4_t, va[j][nb]);
                                u32x4_t is;
#pragma unroll
                                for (int i = 0; i < 4; ++i) {
                                    auto one = [&](uint32_t x) { return kind == 0 ? x == 0x7f80u : kind == 1 ? x == 0xff80u : (x & 0x7fffu) > 0x7f80u; };
                                    is[i] = (one(w[i] & 0xffffu) ? 0x3f80u : 0u) | (one(w[i] >> 16) ? 0x3f800000u : 0u);
                                }
                                count = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, is), sees_row[j], count, 0, 0, 0);
                            }
                            const float add = kind == 0 ? INFINITY : kind == 1 ? -INFINITY : NAN;
#pragma unroll
                            for (int i = 0; i < 16; ++i) o[nb][i] += count[i] > 0.f ? add : 0.f;
                        }
#pragma unroll
                        for (int j = 0; j < 2; ++j) {
                            u32x4_t w = __builtin_bit_cast(u32x4_t, va[j][nb]);
#pragma unroll
                            for (int i = 0; i < 4; ++i) {
                                if ((w[i] & 0x7f80u) == 0x7f80u) w[i] &= 0xffff0000u;
                                if ((w[i] & 0x7f800000u) == 0x7f800000u) w[i] &= 0x0000ffffu;
                            }
                            va[j][nb] = __builtin_bit_cast(bf16x8_t, w);
                        }
                    }
                }
            }

            // ---- O^T += V^T P ----
#pragma unroll
            for (int part = 0; part < PARTS; ++part)
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    const bf16x8_t pb = __builtin_bit_cast(bf16x8_t, u32x4_t{pw[part][4 * j], pw[part][4 * j + 1], pw[part][4 * j + 2], pw[part][4 * j + 3]});
#pragma unroll
                    for (int nb = 0; nb < NDB; ++nb) o[nb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(va[j][nb], pb, o[nb], 0, 0, 0);
                }
            if constexpr (WC == 1) {
                const int next = step + kAhead;
                if (next < n_mine) {
                    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
                    if ((next & 63) == 0) more_rows(next);
                    fetch(pc, rows, next, free_stage);
                }
            }
        }

        // ---- the end of the piece: the next one's first tiles and queries are requested, and come while this one's results are folded ----
        l_run = halves_sum(l_run);
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        if constexpr (WC > 1) __syncthreads();        // nobody reads the ring any more
        const bool whole = pc.tile0 == 0 && pc.tile1 == pc.tiles, active = col < pc.nn * a.G;
        if (more) {
            rows = rows_of(ahead, 0, pages_ahead);
            begin_ring(ahead, rows);
            if (kSolo > 0 && pc.solo) request_queries(ahead);      // else behind the fold, whose memory it may be
        }

        const uint32_t out_row = column.row(a, pc.b, pc.h);
        const int c = wc * kTreeCols + l32;
        const float v_mul = KV8 ? a.v_scale[sc] : 1.f;
        float m_star = m_run, l_star = l_run;
        if (kSolo > 0 && pc.solo) {                   // this wave has seen all of the pair
            if (active) {
#pragma unroll
                for (int nb = 0; nb < NDB; ++nb)
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        write_tree_out<D>(a, out_row, 32 * nb + 8 * i + 4 * hi, make_float4(o[nb][4 * i], o[nb][4 * i + 1], o[nb][4 * i + 2], o[nb][4 * i + 3]), m_run,
                                          l_run, v_mul);
            }
            if (!more) break;
            pc = ahead;
            continue;
        }
        // What the workgroup's groups have found is added up through LDS: coordinates 32 nb .. + 31 by group nb % WT, as its block nb / WT.
        constexpr int kOwn = NDB < WT ? 1 : NDB / WT;
        const bool owns = wt < NDB;
        f32x16_t res[kOwn];
        if constexpr (WT > 1) {
            if (hi == 0) st_ml[wt][c] = make_float2(m_run, l_run);
            __syncthreads();
            float2 ml[WT];
#pragma unroll
            for (int w = 0; w < WT; ++w) ml[w] = st_ml[w][c], m_star = fmaxf(m_star, ml[w].x);
            l_star = 0.f;
#pragma unroll
            for (int w = 0; w < WT; ++w) l_star = fmaf(ml[w].y, ml[w].x == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(ml[w].x - m_star), l_star);
            const float f = m_run == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m_run - m_star);
#pragma unroll
            for (int nb = 0; nb < NDB; ++nb)
#pragma unroll
                for (int i = 0; i < 16; ++i) o[nb][i] *= f;
            // block j of a round, of the group u = 1 .. WT - 1 places behind the one that adds it up
            auto place = [&](int j, int u) __attribute__((always_inline)) {
                return reinterpret_cast<float4 *>(lds + kFoldAt + ((j * (WT - 1) + u - 1) * WC + wc) * kBlock) + hi * kTreeCols + l32;
            };
#pragma unroll
            for (int r = 0; r < NDB; r += kRound) {
                if (r > 0) __syncthreads();           // the round before has been read
#pragma unroll
                for (int j = 0; j < kRound; ++j) {
                    const int nb = r + j, u = (wt + WT - nb % WT) % WT;
                    if (u == 0) continue;
                    float4 *to = place(j, u);
#pragma unroll
                    for (int i = 0; i < 4; ++i) to[2 * i * kTreeCols] = make_float4(o[nb][4 * i], o[nb][4 * i + 1], o[nb][4 * i + 2], o[nb][4 * i + 3]);
                }
                __syncthreads();
#pragma unroll
                for (int j = 0; j < kRound; ++j) {
                    const int nb = r + j;
                    if (nb % WT != wt) continue;
#pragma unroll
                    for (int u = 1; u < WT; ++u) {
                        const float4 *from = place(j, u);
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const float4 x = from[2 * i * kTreeCols];
                            o[nb][4 * i] += x.x, o[nb][4 * i + 1] += x.y, o[nb][4 * i + 2] += x.z, o[nb][4 * i + 3] += x.w;
                        }
                    }
                    res[nb / WT] = o[nb];
                }
            }
        } else {
#pragma unroll
            for (int nb = 0; nb < NDB; ++nb) res[nb] = o[nb];
        }
        if constexpr (WT > 1 && (kFoldInRing || kQueriesInFold)) __syncthreads();      // the fold's memory is the ring's, or the queries', again
        if (more) request_queries(ahead);
        auto four = [&](int q, int i) __attribute__((always_inline)) { return make_float4(res[q][4 * i], res[q][4 * i + 1], res[q][4 * i + 2], res[q][4 * i + 3]); };
        auto first_of = [&](int q, int i) __attribute__((always_inline)) { return 32 * (q * WT + wt) + 8 * i + 4 * hi; };      // coordinate of four(q, i)
        bool finished = whole;
        if (!whole) {
            // ---- a piece of a pair that was cut: the last workgroup to come adds the pieces up, in their order, whichever it is ----
            auto slot_of = [&](int64_t place) __attribute__((always_inline)) {
                return static_cast<int>(small ? static_cast<uint32_t>(place) / static_cast<uint32_t>(share) : place / share);
            };
            const int from_slot = slot_of(pc.first), pieces = slot_of(pc.first + pc.tiles - 1) - from_slot + 1, me = my_slot - from_slot;
            const size_t block = static_cast<size_t>(blockIdx.y) * a.n_slots;
            auto part = [&](int piece) __attribute__((always_inline)) {      // where a piece's result is: the pair's first piece ends its workgroup's share
                return (block + from_slot + piece) * 2 + (piece == 0 ? 1 : 0);
            };
            // Pieces first, first + apart, ... (n of them, this workgroup's the mine_th) into this workgroup's registers, if it is the last of them to come.
            auto join = [&](int32_t *counter, int first, int apart, int n, int mine_th) __attribute__((always_inline)) {
                __syncthreads();                      // `counted` has been read
                // Where the others are there already, which the last piece's often are, nothing need be written.  (They counted in behind their
                // results' arrival.)
                bool last = false;
                if (mine_th == n - 1) {
                    if (threadIdx.x == 0) counted = __hip_atomic_load(counter, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
                    __syncthreads();
                    last = __builtin_amdgcn_readfirstlane(counted) == n - 1;
                    __syncthreads();
                }
                if (!last) {
                    const size_t to = part(first + mine_th * apart);
                    if (active && owns) {
#pragma unroll
                        for (int q = 0; q < kOwn; ++q)
#pragma unroll
                            for (int i = 0; i < 4; ++i) publish_f32x4(a.part_o + to * (D * CB), (first_of(q, i) / 4 * CB + c) * 16, four(q, i));
                        if (wt == 0 && hi == 0) publish_f32x2(a.part_ml + to * (CB * 2), c * 8, m_star, l_star);
                    }
                    drain_vmem();
                    __syncthreads();
                    if (threadIdx.x == 0) counted = __hip_atomic_fetch_add(counter, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
                    __syncthreads();
                    last = __builtin_amdgcn_readfirstlane(counted) == n - 1;
                }
                if (!last) return false;
                if (threadIdx.x == 0) __hip_atomic_store(counter, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
                f2_t ml[kJoin];
#pragma unroll
                for (int i = 0; i < kJoin; ++i) {
                    ml[i] = f2_t{-INFINITY, 0.f};
                    if (i < n && i != mine_th)
                        ml[i] = __builtin_bit_cast(f2_t, __builtin_amdgcn_raw_buffer_load_b64(parts_rsrc(a.part_ml + part(first + i * apart) * (CB * 2), CB * 8), c * 8, 0, kAgent));
                }
                float top = m_star, sum = 0.f;
#pragma unroll
                for (int i = 0; i < kJoin; ++i) {
                    if (i == mine_th) ml[i] = f2_t{m_star, l_star};
                    top = fmaxf(top, ml[i][0]);
                }
#pragma unroll
                for (int i = 0; i < kJoin; ++i) {
                    ml[i][0] = ml[i][0] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(ml[i][0] - top);
                    sum = fmaf(ml[i][1], ml[i][0], sum);
                }
                auto weight = [&](int i) __attribute__((always_inline)) {
                    float f = ml[0][0];
#pragma unroll
                    for (int j = 1; j < kJoin; ++j) f = i == j ? ml[j][0] : f;
                    return f;
                };
                constexpr int kAtOnce = kOwn > 2 ? 1 : kOwn;      // of a wave's blocks of coordinates
#pragma unroll
                for (int q0 = 0; q0 < kOwn; q0 += kAtOnce) {
                    float acc[kAtOnce][16] = {};
#pragma clang loop unroll(disable)
                    for (int i = 0; i < n; ++i) {
                        const float f = weight(i);
                        if (i == mine_th) {
#pragma unroll
                            for (int u = 0; u < kAtOnce; ++u)
#pragma unroll
                                for (int e = 0; e < 16; ++e) acc[u][e] = fmaf(res[q0 + u][e], f, acc[u][e]);
                            continue;
                        }
                        const __amdgpu_buffer_rsrc_t from = parts_rsrc(a.part_o + part(first + i * apart) * (D * CB), D * CB * 4);
                        f4_t x[kAtOnce][4];
#pragma unroll
                        for (int u = 0; u < kAtOnce; ++u)
#pragma unroll
                            for (int e = 0; e < 4; ++e)      // (where a group owns no block: past the end, and not used)
                                x[u][e] = __builtin_bit_cast(f4_t, __builtin_amdgcn_raw_buffer_load_b128(from, (first_of(q0 + u, e) / 4 * CB + c) * 16, 0, kAgent));
#pragma unroll
                        for (int u = 0; u < kAtOnce; ++u)
#pragma unroll
                            for (int e = 0; e < 16; ++e) acc[u][e] = fmaf(x[u][e / 4][e % 4], f, acc[u][e]);
                    }
#pragma unroll
                    for (int u = 0; u < kAtOnce; ++u)
#pragma unroll
                        for (int e = 0; e < 16; ++e) res[q0 + u][e] = acc[u][e];
                }
                m_star = top, l_star = sum;
                return true;
            };
            // Up to kJoin pieces at once; more in groups of as many, whose sums are joined in groups in turn.  A group's counter lies by its level
            // and the place of its first piece.
            finished = true;
            int unit = 1, at_level = me;
            int32_t *level = a.arrivals + block * (2 * kLevels);
#pragma clang loop unroll(disable)
            for (int left = pieces; finished && left > 1; left = (left + kJoin - 1) / kJoin) {
                const int group = at_level / kJoin, n = min(kJoin, left - group * kJoin), first = group * kJoin * unit;
                if (n > 1) finished = join(level + (from_slot + first) * 2 + (first == 0 ? 1 : 0), first, unit, n, at_level % kJoin);
                at_level = group, unit *= kJoin, level += 2 * a.n_slots;
            }
        }
        if (finished && active && owns) {
#pragma unroll
            for (int q = 0; q < kOwn; ++q)
#pragma unroll
                for (int i = 0; i < 4; ++i) write_tree_out<D>(a, out_row, first_of(q, i), four(q, i), m_star, l_star, v_mul);
        }
        if (!more) break;
        pc = ahead;
    }
}

}  // namespace fairkv
