// The attention weight that the last tokens' queries give every row of a growing cache, added up.
//
// Mathematics.  A pair (b, h) has len rows, the last n = n_new[b] of them the queries' own.  With s = scale q . k and the log-sum-exp that the
// attention of the same queries left,
//     w[t] = decay w_old[t] [t < len - n] + sum over columns c = (node i < n, head g of the group) that see t of exp(s_ct - lse_c),
// the sums in fp32.  No maximum runs along: lse is at least every score that it is of.
//
// Tiles.  A wave has T x 32 tokens, whose rows of K it holds in registers as an operand of 32x32x16 matrix instructions, and goes through the
// columns 32 at a time:
//     S[column][token] = q K^T         D / 16 instructions a tile
// A lane has one token (lane % 32) and 16 of the 32 columns, so a weight is added where it was computed; two lanes share a token.  Queries lie
// in LDS, for all waves of the workgroup, 128 columns at a time.
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

constexpr int kWeightWaves = 4;
constexpr int kWeightCols = 128;      // columns in LDS at a time

template <int D, bool KV8, int T>
__global__ __launch_bounds__(kWeightWaves * 64) void fairkv_attn_weights_kernel(WeightsArgs a)
{
    constexpr int NT = kWeightWaves * 64, BLOCK = kWeightWaves * T * 32, CC = kWeightCols;
    constexpr int ROWB = KV8 ? D : 2 * D, QROWB = 2 * D;      // bytes of a row of K, of a query
    constexpr int NP = ROWB / 32, NSL = D / 16, PPQ = QROWB / 16;
    typedef __attribute__((ext_vector_type(4))) uint32_t u4;
    __shared__ __attribute__((aligned(16))) char qs[CC * QROWB];
    __shared__ __attribute__((aligned(16))) float minus_lse[CC];      // in log2 units
    __shared__ uint64_t sees[CC];                                     // of every column: the nodes that it sees

    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), l32 = lane & 31, hi = lane >> 5;
    const int n_pairs = a.B * a.Hkv;
    // Tokens of a pair that lie in the cache: none of a packed one whose run sticks out of it.
    auto len_of = [&](int p) __attribute__((always_inline)) {
        const int32_t len = min(max(a.len[p], 0), a.max_len);
        if (a.rows.pages) return len;
        const int64_t off = a.rows.off[p];
        return off >= 0 && static_cast<uint64_t>(off) + static_cast<uint32_t>(len) <= static_cast<uint64_t>(a.rows.n_rows) ? len : 0;
    };
    auto blocks_of = [](int32_t len) __attribute__((always_inline)) { return (static_cast<int64_t>(len) + BLOCK - 1) / BLOCK; };
    // Piece p of column c lies at piece p ^ swizzle(c): a row per lane, 16 of them take all banks.
    auto swizzle = [](int c) __attribute__((always_inline)) { return c / (256 / QROWB) % PPQ; };

    const LineShare share = line_share<NT>(n_pairs, gridDim.x, blockIdx.x, [&](int p) { return blocks_of(len_of(p)); });
    int pair = share.pair, in_lds = -1, chunk_in_lds = 0;
    int64_t block = share.begin;
    int32_t len = share.left > 0 ? len_of(pair) : 0;
    for (int64_t left = share.left; left > 0; --left, ++block) {
        if (block >= blocks_of(len)) {
            pair = next_pair(pair, n_pairs, [&](int p) { return blocks_of(len_of(p)); }), block = 0;
            len = len_of(pair);
        }
        const int b = pair / a.Hkv, h = pair - b * a.Hkv;
        const int32_t nn = a.n_new ? min(max(a.n_new[b], 0), a.q_len) : a.q_len, base = len - nn;      // base: rows in front of the new ones
        const int cols = nn * a.G;
        const int32_t t0 = static_cast<int32_t>(block) * BLOCK + wave * T * 32;
        const float s_mul = KV8 ? a.scale_log2 * a.k_scale[a.n_scales > 1 ? h : 0] : a.scale_log2;

        // ---- rows of K ----
        int64_t row[T];
        bf16x8_t k[T][NSL];
        float old[T], sum[T][4];
#pragma unroll
        for (int i = 0; i < T; ++i) {
            const int32_t t = t0 + i * 32 + l32;
            row[i] = t < len ? a.rows.row(pair, t) : -1;
            // where there is none the cache's first row stands in: what comes of it is not stored
            const char *from = a.k + max(row[i], static_cast<int64_t>(0)) * ROWB + hi * 16;
            u4 raw[NP];
#pragma unroll
            for (int p = 0; p < NP; ++p) raw[p] = *reinterpret_cast<const u4 *>(from + p * 32);
            old[i] = a.decay != 0.f && row[i] >= 0 && t < base ? a.weights[row[i]] * a.decay : 0.f;
#pragma unroll
            for (int p = 0; p < NP; ++p) {
                if constexpr (KV8) {
                    k[i][2 * p] = widen8(i32x2_t{static_cast<int>(raw[p][0]), static_cast<int>(raw[p][1])});
                    k[i][2 * p + 1] = widen8(i32x2_t{static_cast<int>(raw[p][2]), static_cast<int>(raw[p][3])});
                } else {
                    k[i][p] = __builtin_bit_cast(bf16x8_t, raw[p]);
                }
            }
#pragma unroll
            for (int x = 0; x < 4; ++x) sum[i][x] = 0.f;
        }

        for (int chunk = 0; chunk * CC < cols; ++chunk) {
            const int n = min(CC, cols - chunk * CC);
            if (in_lds != pair || chunk_in_lds != chunk) {
                __syncthreads();
                for (int x = threadIdx.x; x < n * PPQ; x += NT) {
                    const int c = x / PPQ, p = x % PPQ, node = (chunk * CC + c) / a.G, g = chunk * CC + c - node * a.G;
                    const size_t at = ((static_cast<size_t>(b) * a.q_len + node) * a.Hq + h * a.G + g) * QROWB;
                    *reinterpret_cast<u4 *>(qs + c * QROWB + ((p ^ swizzle(c)) * 16)) = *reinterpret_cast<const u4 *>(a.q + at + p * 16);
                }
                for (int c = threadIdx.x; c < n; c += NT) {
                    const int node = (chunk * CC + c) / a.G, g = chunk * CC + c - node * a.G;
                    const float lse = a.lse[(static_cast<size_t>(b) * a.q_len + node) * a.Hq + h * a.G + g];
                    minus_lse[c] = lse == -INFINITY ? -INFINITY : -lse * kLog2e;      // a node that sees nothing gives no weight
                    sees[c] = a.tree ? static_cast<uint64_t>(a.tree[static_cast<size_t>(b) * a.q_len + node]) : ~0ull >> (63 - node);
                }
                in_lds = pair, chunk_in_lds = chunk;
                __syncthreads();
            }
            if (t0 >= len) continue;
            for (int c0 = 0; c0 < n; c0 += 32) {
                bf16x8_t q[NSL];
                const int c = min(c0 + l32, n - 1);      // columns past the last one are that one again, and do not count
#pragma unroll
                for (int s = 0; s < NSL; ++s) {
                    const int p = KV8 ? (s & ~1) * 2 + 2 * hi + (s & 1) : 2 * s + hi;      // the order in which the lanes hold K
                    q[s] = *reinterpret_cast<const bf16x8_t *>(qs + c * QROWB + ((p ^ swizzle(c)) * 16));
                }
                f32x16_t z[T];
#pragma unroll
                for (int i = 0; i < T; ++i) {
#pragma unroll
                    for (int r = 0; r < 16; ++r) z[i][r] = 0.f;
#pragma unroll
                    for (int s = 0; s < NSL; ++s) z[i] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(q[s], k[i][s], z[i], 0, 0, 0);
                }
                const bool masked = c0 + 32 > n || t0 + T * 32 > base;
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    const int cr = c0 + 8 * (r / 4) + 4 * hi + r % 4;
                    const float ml = minus_lse[min(cr, n - 1)];
#pragma unroll
                    for (int i = 0; i < T; ++i) {
                        float e = __builtin_amdgcn_exp2f(fmaf(z[i][r], s_mul, ml));
                        if (masked) {
                            const int32_t j = t0 + i * 32 + l32 - base;
                            if (cr >= n || (j >= 0 && !(sees[min(cr, n - 1)] >> min(j, 63) & 1))) e = 0.f;
                        }
                        sum[i][r % 4] += e;
                    }
                }
            }
        }
#pragma unroll
        for (int i = 0; i < T; ++i) {
            const float mine = (sum[i][0] + sum[i][1]) + (sum[i][2] + sum[i][3]), w = mine + __shfl_xor(mine, 32);
            if (hi == 0 && row[i] >= 0) a.out[row[i]] = old[i] + w;
        }
    }
}

}  // namespace fairkv
