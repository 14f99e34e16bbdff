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
// workgroup adds up the lengths by itself and finds its share of the line of all pairs, each as long as its tiles and kTreeOverhead more.
// The pieces of a pair that is cut leave partial results in the workspace, which a second small kernel adds up in the order of the pieces.
#pragma once
#include "cache_rows.h"
#include "decode_mfma.h"

namespace fairkv {

typedef __attribute__((ext_vector_type(16))) float f32x16_t;
typedef __attribute__((ext_vector_type(4))) uint32_t u32x4_t;

constexpr int kTreeTok = 32;          // tokens of a tile
constexpr int kTreeCols = 32;         // columns of a wave
constexpr int kTreeOverhead = 3;      // what a pair costs a workgroup beside its tiles, in tiles

struct TreeArgs {
    const void *q, *k, *v;
    RowMap rows;
    const int32_t *len;               // [B * Hkv]
    const int32_t *n_new;             // [B] or null
    const int64_t *tree;              // [B][q_len] or null: node i sees nodes 0 .. i
    void *out;
    float *lse;
    float *part_o;                    // [slots][D / 4][columns of a workgroup][4]
    float *part_ml;                   // [slots][columns of a workgroup][2]
    int32_t *cut;                     // [column blocks][n_slots][2]: the pair whose first piece a workgroup had, and its pieces (0: none was cut)
    int32_t B, Hq, Hkv, G, q_len, cols, n_slots, max_len, out_dtype, n_scales;
    float scale_log2;
    float k_scale[kCacheScales], v_scale[kCacheScales];
};

// log2 of how rows are swizzled: 16-byte piece c of row r lies at piece c ^ swz(r).  K is read a row per lane: consecutive rows that fill
// the 256 bytes of all banks take different pieces.  V is read by the transposing instruction, 64 (8-bit: 32) bytes of each of 4 (8) rows.
template <int ROWB>
__device__ __forceinline__ constexpr int k_swizzle(int r)
{
    return r / (256 / ROWB) % (ROWB / 16);
}
template <int ROWB, bool KV8>
__device__ __forceinline__ constexpr int v_swizzle(int r)
{
    if (!KV8) return ROWB == 256 ? 4 * (r & 3) : 4 * (r >> 1 & 1);
    return ROWB == 128 ? 2 * ((r >> 1 & 1) | (r >> 3 & 1) << 1) : 2 * (r >> 3 & 1);
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

// FINE: a weight enters the second product as two bf16 numbers (its rounding and what that leaves), in twice the instructions: an output in
// fp32 keeps fp32's accuracy.  Without, its error is that of weights rounded to 8 bits, about as large as a bf16 output's own rounding.
template <int D, bool KV8, int WC, int WT, int STAGES, bool FINE>
__global__ __launch_bounds__(WC *WT * 64, 1) void fairkv_decode_tree_kernel(TreeArgs a)
{
    constexpr int NW = WC * WT, NT = NW * 64, CB = WC * kTreeCols;
    constexpr int ROWB = KV8 ? D : 2 * D;             // bytes of a row of K or V
    constexpr int PPR = ROWB / 16, RPI = 64 / PPR;    // 16-byte pieces of a row, rows of a wave-wide load
    constexpr int LPT = kTreeTok / RPI;               // wave-wide loads of a tile of K
    constexpr int TILEB = kTreeTok * ROWB, STAGEB = 2 * TILEB;
    constexpr int LOADS = 2 * LPT >= WC ? 2 * LPT / WC : 1;     // a wave's share of the loads of a stage
    constexpr int NSL = D / 16, NDB = D / 32;
    constexpr int kAhead = WC == 1 ? STAGES : STAGES - 1;       // tiles on their way while one is waited for
    constexpr int RING = WT * STAGES * STAGEB;
    constexpr int FOLDROW = D + 4;
    constexpr int FOLD = (WT - 1) * CB * (FOLDROW + 2) * 4;
    static_assert(LOADS * kAhead < 64, "vmcnt is a 6-bit counter");

    __shared__ __attribute__((aligned(1024))) char lds[RING > FOLD ? RING : FOLD];
    __shared__ int64_t scan[NW + 3];                  // totals of the waves; the pair the workgroup starts in and where it begins

    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wc = wave % WC, wt = wave / WC;
    const int l32 = lane & 31, hi = lane >> 5;
    const int n_pairs = a.B * a.Hkv, c0 = blockIdx.y * CB;
    const int my_slot = blockIdx.x;
    int32_t *cut = a.cut + (static_cast<size_t>(blockIdx.y) * a.n_slots + my_slot) * 2;
    if (threadIdx.x == 0) cut[1] = 0;

    // ---- this workgroup's share of the line ----
    int64_t begin, end, share, at;
    int pair;
    {
        const int run = (n_pairs + NT - 1) / NT, p0 = min(static_cast<int>(threadIdx.x) * run, n_pairs), p1 = min(p0 + run, n_pairs);
        int64_t mine = 0;
        for (int p = p0; p < p1; ++p) mine += kTreeOverhead + tiles_of(tree_len(a, p));
        int64_t upto = mine;
#pragma unroll
        for (int o = 1; o < 64; o *= 2) {
            const int64_t x = __shfl_up(upto, o, 64);
            if (lane >= o) upto += x;
        }
        if (lane == 63) scan[wave] = upto;
        if (threadIdx.x == 0) scan[NW] = -1;
        __syncthreads();
        int64_t before = 0, total = 0;
#pragma unroll
        for (int w = 0; w < NW; ++w) {
            if (w < wave) before += scan[w];
            total += scan[w];
        }
        share = (total + a.n_slots - 1) / a.n_slots;
        begin = share * my_slot;
        end = begin + share;
        before += upto - mine;
        if (before <= begin && begin < before + mine) {
            int p = p0;
            for (; p < p1; ++p) {
                const int cost = kTreeOverhead + tiles_of(tree_len(a, p));
                if (begin < before + cost) break;
                before += cost;
            }
            scan[NW] = p;
            scan[NW + 1] = before;
        }
        __syncthreads();
        pair = __builtin_amdgcn_readfirstlane(static_cast<int>(scan[NW]));
        at = uniform64(scan[NW + 1]);
        begin = uniform64(begin), end = uniform64(end), share = uniform64(share);
    }
    if (pair < 0) return;                             // nothing is left of the line

    // ---- what depends on the lane alone ----
    const int col = c0 + wc * kTreeCols + l32;
    const Column column(a, min(col, a.cols - 1));
    const uint32_t ring = static_cast<uint32_t>(reinterpret_cast<uintptr_t>(FAIRKV_LDS_PTR(lds))) + wt * (STAGES * STAGEB);
    const int ld_row = lane / PPR, ld_col = lane % PPR;
    uint32_t k_rd[NSL], v_rd[NDB][2];                 // where the lane reads in stage 0: its row of K; of V for the first 16 tokens
#pragma unroll
    for (int s = 0; s < NSL; ++s)
        k_rd[s] = ring + l32 * ROWB + (KV8 ? (s ^ k_swizzle<ROWB>(l32)) * 16 + hi * 8 : ((2 * s + hi) ^ k_swizzle<ROWB>(l32)) * 16);
    const int x16 = lane & 15, dq = lane >> 4 & 1;
#pragma unroll
    for (int nb = 0; nb < NDB; ++nb) {
        if constexpr (KV8) {
            const int e = x16 >> 1, r = (e < 4 ? e : e + 4) + 4 * hi;
            v_rd[nb][0] = ring + TILEB + r * ROWB + ((2 * nb + dq) ^ v_swizzle<ROWB, true>(r)) * 16 + (x16 & 1) * 8;
            v_rd[nb][1] = 0;
        } else {
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                const int r = 8 * u + 4 * hi + (x16 >> 2);
                v_rd[nb][u] = ring + TILEB + r * ROWB + ((4 * nb + 2 * dq + ((x16 & 3) >> 1)) ^ v_swizzle<ROWB, false>(r)) * 16 + (x16 & 1) * 8;
            }
        }
    }
    const char *const k_base = static_cast<const char *>(a.k), *const v_base = static_cast<const char *>(a.v);

    for (; pair < n_pairs && at < end; ++pair) {
        const int b = pair / a.Hkv, h = pair - b * a.Hkv;
        const int32_t len = __builtin_amdgcn_readfirstlane(tree_len(a, pair)), tiles = tiles_of(len), nn = __builtin_amdgcn_readfirstlane(tree_new(a, b));
        const int64_t first = at + kTreeOverhead;     // place of the pair's first tile
        at = first + tiles;
        const int32_t tile0 = static_cast<int32_t>(max(begin - first, static_cast<int64_t>(0)));
        const int32_t tile1 = static_cast<int32_t>(min(end - first, static_cast<int64_t>(tiles)));
        const bool empty = tiles == 0 && begin < first && first <= end;      // a pair without rows belongs to one workgroup too
        if ((tile1 <= tile0 && !empty) || c0 >= nn * a.G) continue;
        const bool whole = tile0 == 0 && tile1 == tiles;
        const int32_t base = len - nn;                // rows in front of the draft
        const bool active = col < nn * a.G;

        // ---- queries, and what the column sees of the draft ----
        const uint32_t q_row = column.row(a, b, h);
        bf16x8_t qb[NSL];
#pragma unroll
        for (int s = 0; s < NSL; ++s)
            qb[s] = __builtin_bit_cast(bf16x8_t, *reinterpret_cast<const u32x4_t *>(static_cast<const char *>(a.q) + (static_cast<size_t>(q_row) * D + 16 * s + 8 * hi) * 2));
        uint64_t sees = a.tree ? static_cast<uint64_t>(a.tree[b * a.q_len + column.node]) : ~0ull >> (63 - column.node);
        sees &= nn >= 64 ? ~0ull : (1ull << nn) - 1;
        const int sc = a.n_scales > 1 ? h : 0;
        const float s_mul = KV8 ? a.scale_log2 * a.k_scale[sc] : a.scale_log2;
        const int64_t off = a.rows.pages ? 0 : uniform64(a.rows.off[pair]);
        const bool run_ok = a.rows.pages || (off >= 0 && static_cast<uint64_t>(off) + static_cast<uint32_t>(len) <= static_cast<uint64_t>(a.rows.n_rows));

        f32x16_t o[NDB];
        float m_run = -INFINITY, l_run = 0.f;
#pragma unroll
        for (int nb = 0; nb < NDB; ++nb)
#pragma unroll
            for (int i = 0; i < 16; ++i) o[nb][i] = 0.f;

        // The group's tiles: tile0 + wt, + WT, ...  Pages of 64 of them are held in lanes, those of the first and of the second 16 tokens.
        const int n_steps = (tile1 - tile0 + WT - 1) / WT;
        const int n_mine = max(0, (tile1 - tile0 - wt + WT - 1) / WT);
        int32_t page_lo = 0, page_hi = 0;
        auto fetch_pages = [&](int step) __attribute__((always_inline)) {      // of steps step .. step + 63
            const int t = min((tile0 + wt + (step + lane) * WT) * kTreeTok, len - 1);
            const int32_t *ids = a.rows.pages + static_cast<int64_t>(pair) * a.rows.max_pages;
            page_lo = ids[t >> a.rows.page_shift];
            page_hi = ids[min(t + 16, len - 1) >> a.rows.page_shift];
            drain_vmem();
        };
        // First row of 16 tokens from token t on, -1 if the cache has none there.
        auto row_of = [&](int step, int half, int32_t t) __attribute__((always_inline)) -> int64_t {
            if (!a.rows.pages) return run_ok ? off + t : -1;
            return a.rows.row_of_page(__builtin_amdgcn_readlane(half ? page_hi : page_lo, step & 63), t);
        };
        // This wave's share of a stage.  Rows past the end of the pair are its last row again, rows that the cache does not have the cache's first
        // one: their weights are 0.  `missing` says of every stage which of its two halves the cache does not have.
        uint32_t missing = 0;
        auto fetch = [&](int step) __attribute__((always_inline)) {
            const int32_t t0 = (tile0 + wt + step * WT) * kTreeTok;
            const int last = len - 1 - t0, at_stage = step % STAGES;
            const uint32_t stage = ring + at_stage * STAGEB;
            const int64_t row0 = row_of(step, 0, t0), row1 = last >= 16 ? row_of(step, 1, t0 + 16) : row0;
            missing = (missing & ~(3u << 2 * at_stage)) | ((row0 < 0 ? 1u : 0u) | (row1 < 0 ? 2u : 0u)) << 2 * at_stage;
#pragma unroll
            for (int x = 0; x < LOADS; ++x) {
                const int load = wc * LOADS + x;
                if (2 * LPT < WC && load >= 2 * LPT) break;
                const bool is_v = load >= LPT;
                const int i = is_v ? load - LPT : load;
                const bool upper = i * RPI >= 16;
                const int64_t row = upper ? row1 : row0;
                const int r = i * RPI + ld_row, behind = row < 0 ? 0 : min(r, last) - (upper && last >= 16 ? 16 : 0);      // rows behind `row`
                const int swizzled = ld_col ^ (is_v ? v_swizzle<ROWB, KV8>(r) : k_swizzle<ROWB>(r));
                load16_to_lds((is_v ? v_base : k_base) + max(row, static_cast<int64_t>(0)) * ROWB, behind * ROWB + swizzled * 16,
                              stage + (is_v ? TILEB : 0) + i * 1024);
            }
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

        __builtin_amdgcn_s_waitcnt(0x0F70);           // the queries are here: the ring's loads are counted from now on
        if (a.rows.pages && n_mine > 0) fetch_pages(0);
#pragma unroll
        for (int s = 0; s < kAhead; ++s)
            if (s < n_mine) fetch(s);

        for (int step = 0; step < (WC == 1 ? n_mine : n_steps); ++step) {
            wait_stage(min(n_mine - 1 - step, kAhead - 1));
            if constexpr (WC > 1) {
                // every wave's loads of this stage have landed, and every wave is through with the stage before, which the next loads fill
                asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
                const int next = step + kAhead;
                if (next < n_mine) {
                    if (a.rows.pages && (next & 63) == 0) fetch_pages(next);
                    fetch(next);
                }
                if (step >= n_mine) continue;
            }
            const uint32_t stage = (step % STAGES) * STAGEB;
            const int32_t t0 = (tile0 + wt + step * WT) * kTreeTok;

            // ---- scores ----
            f32x16_t sacc;
#pragma unroll
            for (int i = 0; i < 16; ++i) sacc[i] = 0.f;
            if constexpr (KV8) {
                i32x2_t kw[NSL];
#pragma unroll
                for (int s = 0; s < NSL; ++s) kw[s] = *lds_at<i32x2_t>(k_rd[s] + stage);
#pragma unroll
                for (int s = 0; s < NSL; ++s) sacc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(widen8(kw[s]), qb[s], sacc, 0, 0, 0);
            } else {
                bf16x8_t kw[NSL];
#pragma unroll
                for (int s = 0; s < NSL; ++s) kw[s] = *lds_at<bf16x8_t>(k_rd[s] + stage);
#pragma unroll
                for (int s = 0; s < NSL; ++s) sacc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kw[s], qb[s], sacc, 0, 0, 0);
            }
            bf16x8_t va[2][NDB];
#pragma unroll
            for (int j = 0; j < 2; ++j)
#pragma unroll
                for (int nb = 0; nb < NDB; ++nb) {
                    if constexpr (KV8) {
                        va[j][nb] = widen8(__builtin_amdgcn_ds_read_tr8_b64_v2i32(lds_at<i32x2_t>(v_rd[nb][0] + stage + j * 16 * ROWB)));
                    } else {
                        const uint2 x = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16(lds_at<i16x4_t>(v_rd[nb][0] + stage + j * 16 * ROWB)));
                        const uint2 y = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16(lds_at<i16x4_t>(v_rd[nb][1] + stage + j * 16 * ROWB)));
                        va[j][nb] = __builtin_bit_cast(bf16x8_t, u32x4_t{x.x, x.y, y.x, y.y});
                    }
                }
            // Element r of a lane: token t0 + 8 (r / 4) + 4 hi + r % 4.
            float sv[16];
#pragma unroll
            for (int r = 0; r < 16; ++r) sv[r] = sacc[r] * s_mul;

            // ---- what is not seen: rows of the draft, rows past the end, rows that the cache does not have ----
            const uint32_t lacks = missing >> 2 * (step % STAGES) & 3;
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
                    if (!(seen >> (8 * (r / 4) + r % 4) & 1)) sv[r] = -INFINITY;
            }

            // ---- a reference maximum that is raised when some score is far above it ----
            float mx = sv[0];
#pragma unroll
            for (int r = 1; r < 16; ++r) mx = fmaxf(mx, sv[r]);
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

            // ---- weights ----
            uint32_t pw[8], rest[8];
#pragma unroll
            for (int r = 0; r < 16; r += 2) {
                const float p0 = __builtin_amdgcn_exp2f(sv[r] - m_ref), p1 = __builtin_amdgcn_exp2f(sv[r + 1] - m_ref);
                l_run += p0 + p1;
                pw[r / 2] = pack_bf16(p0, p1);
                if constexpr (FINE) rest[r / 2] = pack_bf16(p0 - bf16_lo(pw[r / 2]), p1 - bf16_hi(pw[r / 2]));
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
            for (int j = 0; j < 2; ++j) {
                const bf16x8_t pb = __builtin_bit_cast(bf16x8_t, u32x4_t{pw[4 * j], pw[4 * j + 1], pw[4 * j + 2], pw[4 * j + 3]});
#pragma unroll
                for (int nb = 0; nb < NDB; ++nb) o[nb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(va[j][nb], pb, o[nb], 0, 0, 0);
                if constexpr (FINE) {
                    const bf16x8_t pr = __builtin_bit_cast(bf16x8_t, u32x4_t{rest[4 * j], rest[4 * j + 1], rest[4 * j + 2], rest[4 * j + 3]});
#pragma unroll
                    for (int nb = 0; nb < NDB; ++nb) o[nb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(va[j][nb], pr, o[nb], 0, 0, 0);
                }
            }
            if constexpr (WC == 1) {
                const int next = step + kAhead;
                if (next < n_mine) {
                    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
                    if (a.rows.pages && (next & 63) == 0) fetch_pages(next);
                    fetch(next);
                }
            }
        }

        // ---- the end of the piece ----
        l_run = halves_sum(l_run);
        if constexpr (WT > 1) {                       // the other groups' results to the first one, through the ring's memory
            float *fold = reinterpret_cast<float *>(lds);
            __syncthreads();
            if (wt > 0) {
                float *mine = fold + ((wt - 1) * CB + wc * kTreeCols + l32) * (FOLDROW + 2);
#pragma unroll
                for (int nb = 0; nb < NDB; ++nb)
#pragma unroll
                    for (int i = 0; i < 4; ++i)
#pragma unroll
                        for (int e = 0; e < 4; ++e) mine[32 * nb + 8 * i + 4 * hi + e] = o[nb][4 * i + e];
                if (hi == 0) mine[D] = m_run, mine[D + 1] = l_run;
            }
            __syncthreads();
            if (wt == 0) {
                float f[WT], m_star = m_run;
#pragma unroll
                for (int w = 1; w < WT; ++w) m_star = fmaxf(m_star, fold[((w - 1) * CB + wc * kTreeCols + l32) * (FOLDROW + 2) + D]);
                f[0] = m_run == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m_run - m_star);
                float l_star = l_run * f[0];
#pragma unroll
                for (int nb = 0; nb < NDB; ++nb)
#pragma unroll
                    for (int i = 0; i < 16; ++i) o[nb][i] *= f[0];
#pragma unroll
                for (int w = 1; w < WT; ++w) {
                    const float *theirs = fold + ((w - 1) * CB + wc * kTreeCols + l32) * (FOLDROW + 2);
                    f[w] = theirs[D] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(theirs[D] - m_star);
                    l_star = fmaf(theirs[D + 1], f[w], l_star);
#pragma unroll
                    for (int nb = 0; nb < NDB; ++nb)
#pragma unroll
                        for (int i = 0; i < 16; ++i) o[nb][i] = fmaf(theirs[32 * nb + 8 * (i / 4) + 4 * hi + i % 4], f[w], o[nb][i]);
                }
                m_run = m_star, l_run = l_star;
            }
            __syncthreads();                          // before the ring is filled again
        } else if constexpr (WC > 1) {
            __syncthreads();
        }
        if (wt == 0) {
            if (whole) {
                if (active) {
                    const float v_mul = KV8 ? a.v_scale[sc] : 1.f;
#pragma unroll
                    for (int nb = 0; nb < NDB; ++nb)
#pragma unroll
                        for (int i = 0; i < 4; ++i)
                            write_tree_out<D>(a, q_row, 32 * nb + 8 * i + 4 * hi, make_float4(o[nb][4 * i], o[nb][4 * i + 1], o[nb][4 * i + 2], o[nb][4 * i + 3]), m_run,
                                              l_run, v_mul);
                }
            } else {
                const size_t slot = (static_cast<size_t>(blockIdx.y) * a.n_slots + my_slot) * 2 + (tile0 == 0 ? 1 : 0);
                const int c = wc * kTreeCols + l32;
#pragma unroll
                for (int nb = 0; nb < NDB; ++nb)
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        *reinterpret_cast<float4 *>(a.part_o + ((slot * (D / 4) + 8 * nb + 2 * i + hi) * CB + c) * 4) =
                            make_float4(o[nb][4 * i], o[nb][4 * i + 1], o[nb][4 * i + 2], o[nb][4 * i + 3]);
                if (hi == 0) *reinterpret_cast<float2 *>(a.part_ml + (slot * CB + c) * 2) = make_float2(m_run, l_run);
                if (tile0 == 0 && threadIdx.x == 0) {
                    cut[0] = pair;
                    cut[1] = static_cast<int32_t>((first + tiles - 1) / share - first / share + 1);
                }
            }
        }
    }
}

// Adds up the pieces of the pair whose first piece workgroup x of column block y had: the first is in the slot of the end of that
// workgroup's share, the others in those of the beginnings of the next workgroups' shares.
template <int D, int CB>
__global__ __launch_bounds__(256) void fairkv_tree_merge_kernel(TreeArgs a)
{
    const size_t group = static_cast<size_t>(blockIdx.y) * a.n_slots + blockIdx.x;
    const int pieces = a.cut[group * 2 + 1];
    if (pieces == 0) return;
    const int pair = a.cut[group * 2], b = pair / a.Hkv, h = pair - b * a.Hkv, live = tree_new(a, b) * a.G;
    for (int idx = blockIdx.z * 256 + threadIdx.x; idx < CB * (D / 4); idx += gridDim.z * 256) {
        const int c = idx % CB, d4 = idx / CB, col = blockIdx.y * CB + c;
        if (col >= live) continue;
        float m_star = -INFINITY, l_star = 0.f;
        float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
        for (int i = 0; i < pieces; ++i) {
            const size_t slot = (group + i) * 2 + (i == 0 ? 1 : 0);
            const float2 ml = *reinterpret_cast<const float2 *>(a.part_ml + (slot * CB + c) * 2);
            const float4 o = *reinterpret_cast<const float4 *>(a.part_o + ((slot * (D / 4) + d4) * CB + c) * 4);
            const float m_new = fmaxf(m_star, ml.x);
            const float keep = m_star == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m_star - m_new), f = ml.x == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(ml.x - m_new);
            l_star = l_star * keep + ml.y * f;
            acc.x = acc.x * keep + o.x * f, acc.y = acc.y * keep + o.y * f, acc.z = acc.z * keep + o.z * f, acc.w = acc.w * keep + o.w * f;
            m_star = m_new;
        }
        const Column column(a, col);
        write_tree_out<D>(a, column.row(a, b, h), d4 * 4, acc, m_star, l_star, a.v_scale[a.n_scales > 1 ? h : 0]);
    }
}

}  // namespace fairkv
