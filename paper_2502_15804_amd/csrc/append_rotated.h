// The two ends of a step over a growing cache: the new tokens' heads are normalised, rotated and appended, and of a draft's rows
// those of the accepted path are kept.
#pragma once
#include <hip/hip_runtime.h>

#include <cstdint>

#include "cache_rows.h"
#include "common.h"
#include "fairkv.h"

namespace fairkv {

struct RotateArgs {
    const char *q, *k_new, *v_new;        // token (b, i) at element (b * q_len + i) * stride, its heads one behind the other
    char *q_out;                          // [B][q_len][Hq][D]
    char *k, *v;                          // the cache
    const float *q_norm, *k_norm;         // [D] or null
    const float *table;                   // [n_pos][rot]: cosines of the rot / 2 angles of a position, then their sines; or null
    const int32_t *pos;                   // [B][q_len]
    const int32_t *n_new;                 // [B] or null
    const int32_t *len, *cap;             // [B * Hkv]
    int32_t *len_out, *bad;
    RowMap rows;
    int64_t q_stride, k_stride, v_stride;
    int32_t B, Hq, Hkv, q_len, n_pos, rot, pairs;
    int32_t q_groups, head_slots, passes; // workgroups for the queries; rows of one token that a pass of a workgroup covers; its passes
    int32_t apart;                        // how many passes' tokens further on, but for the workgroups' number of them, its next pass's lie
    int32_t n_scales;
    float eps;
    float k_scale[kCacheScales], v_scale[kCacheScales];
};

constexpr int kRow8 = 8;                  // elements of a row that a lane has

// Eight elements as floats.
template <typename T>
struct Eight;
template <>
struct Eight<uint16_t> {                  // bf16
    typedef __attribute__((ext_vector_type(4))) uint32_t raw_t;
    static __device__ __forceinline__ raw_t load(const char *p) { return __builtin_nontemporal_load(reinterpret_cast<const raw_t *>(p)); }
    static __device__ __forceinline__ void floats(raw_t w, float (&x)[kRow8])
    {
#pragma unroll
        for (int i = 0; i < 4; ++i) x[2 * i] = bf16_lo(w[i]), x[2 * i + 1] = bf16_hi(w[i]);
    }
    static __device__ __forceinline__ void store(char *p, const float (&x)[kRow8])
    {
        *reinterpret_cast<raw_t *>(p) = raw_t{pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]), pack_bf16(x[4], x[5]), pack_bf16(x[6], x[7])};
    }
};
template <>
struct Eight<float> {
    typedef __attribute__((ext_vector_type(4))) float f4;
    struct raw_t {
        f4 lo, hi;
    };
    static __device__ __forceinline__ raw_t load(const char *p)
    {
        const f4 *w = reinterpret_cast<const f4 *>(p);
        return {__builtin_nontemporal_load(w), __builtin_nontemporal_load(w + 1)};
    }
    static __device__ __forceinline__ void floats(const raw_t &w, float (&x)[kRow8])
    {
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = w.lo[i], x[4 + i] = w.hi[i];
    }
    static __device__ __forceinline__ void store(char *p, const float (&x)[kRow8])
    {
        reinterpret_cast<f4 *>(p)[0] = f4{x[0], x[1], x[2], x[3]};
        reinterpret_cast<f4 *>(p)[1] = f4{x[4], x[5], x[6], x[7]};
    }
};
template <>
struct Eight<uint8_t> {                   // E4M3: what is larger than the format's largest number becomes that one, NaN stays NaN
    static __device__ __forceinline__ void store(char *p, const float (&x)[kRow8])
    {
        float c[kRow8];
#pragma unroll
        for (int i = 0; i < kRow8; ++i) c[i] = x[i] != x[i] ? x[i] : __builtin_amdgcn_fmed3f(x[i], -448.f, 448.f);
        typedef __attribute__((ext_vector_type(2))) int i2;
        i2 w = {0, 0};
        w[0] = __builtin_amdgcn_cvt_pk_fp8_f32(c[0], c[1], w[0], false);
        w[0] = __builtin_amdgcn_cvt_pk_fp8_f32(c[2], c[3], w[0], true);
        w[1] = __builtin_amdgcn_cvt_pk_fp8_f32(c[4], c[5], w[1], false);
        w[1] = __builtin_amdgcn_cvt_pk_fp8_f32(c[6], c[7], w[1], true);
        *reinterpret_cast<i2 *>(p) = w;
    }
};

// A lane's cosines and sines for its eight elements, as out = x * c + partner * s: of a pair (a, b) the first becomes a cos - b sin,
// the second b cos + a sin, so the first element's s is -sin.  Not used for elements behind `rot`.
struct Turn {
    float c[kRow8], s[kRow8];
};
__device__ __forceinline__ Turn turn_of(const RotateArgs &a, int32_t pos, int piece)
{
    Turn t{};
    const int d = piece * kRow8;
    if (!a.table || d >= a.rot) return t;
    const float *row = a.table + static_cast<int64_t>(pos) * a.rot;
    const int half = a.rot / 2;
    if (a.pairs) {                         // elements 2 i and 2 i + 1
#pragma unroll
        for (int i = 0; i < kRow8; i += 2) {
            const float c = row[(d + i) / 2], s = row[half + (d + i) / 2];
            t.c[i] = t.c[i + 1] = c, t.s[i] = -s, t.s[i + 1] = s;
        }
    } else {                               // elements i and i + rot / 2; rot / 2 is a multiple of 8
        const bool first = d < half;
        const float *c = row + (first ? d : d - half);
#pragma unroll
        for (int i = 0; i < kRow8; ++i) {
            t.c[i] = c[i];
            t.s[i] = first ? -c[half + i] : c[half + i];
        }
    }
    return t;
}

// x of another lane of the same 16, by the wave's own data paths.
template <int kCtrl>
__device__ __forceinline__ float from_lane(float x)
{
    return __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(x), kCtrl, 0xf, 0xf, false));
}
constexpr int kXor1 = 0xb1, kXor2 = 0x4e, kQuadMirror = 0x1b, kHalfMirror = 0x141, kMirror = 0x140, kRotate8 = 0x128;

// The sum over a row's L lanes, in each of them.
template <int L>
__device__ __forceinline__ float row_sum(float x)
{
    static_assert(L == 8 || L == 16, "lanes of a row");
    x += from_lane<kXor1>(x);
    x += from_lane<kXor2>(x);
    x += from_lane<kHalfMirror>(x);        // quads are uniform by now, and so are halves
    return L == 16 ? x + from_lane<kMirror>(x) : x;
}

// Norm and rotation of a row whose D / 8 lanes sit side by side in a wave; all of them are here.
template <int D>
__device__ __forceinline__ void norm_and_turn(const RotateArgs &a, float (&x)[kRow8], bool norm, const float (&weight)[kRow8], const Turn &t, int piece)
{
    if (norm) {
        float sum = 0.f;
#pragma unroll
        for (int i = 0; i < kRow8; ++i) sum = fmaf(x[i], x[i], sum);
        const float inv = rsqrtf(row_sum<D / kRow8>(sum) * (1.f / D) + a.eps);
#pragma unroll
        for (int i = 0; i < kRow8; ++i) x[i] = x[i] * inv * weight[i];
    }
    if (!a.table) return;
    float y[kRow8];
    if (a.pairs) {
#pragma unroll
        for (int i = 0; i < kRow8; ++i) y[i] = x[i ^ 1];
    } else if (a.rot == D) {               // half the row's lanes away
#pragma unroll
        for (int i = 0; i < kRow8; ++i) y[i] = D == 128 ? from_lane<kRotate8>(x[i]) : from_lane<kQuadMirror>(from_lane<kHalfMirror>(x[i]));
    } else {
        const int apart = a.rot / (2 * kRow8), lane = threadIdx.x & 63;
        const int from = piece < apart ? lane + apart : piece < 2 * apart ? lane - apart : lane;
#pragma unroll
        for (int i = 0; i < kRow8; ++i) y[i] = __shfl(x[i], from, 64);
    }
    if (piece * kRow8 >= a.rot) return;    // as it is, also an infinite one
#pragma unroll
    for (int i = 0; i < kRow8; ++i) x[i] = fmaf(x[i], t.c[i], y[i] * t.s[i]);
}

__device__ __forceinline__ int32_t new_tokens(const int32_t *n_new, int b, int q_len)
{
    return n_new ? min(max(n_new[b], 0), q_len) : q_len;
}
__device__ __forceinline__ bool in_table(const RotateArgs &a, int32_t pos) { return !a.table || (pos >= 0 && pos < a.n_pos); }

// T: element type of q, k_new and v_new; C: of the cache.  Workgroups 0 .. q_groups - 1 turn queries: a pass of one has 256 / (D / 8) rows in hand,
// head_slots heads of each of several tokens, so that a lane's cosines and sines serve all the heads it meets; it makes `passes` of them, and
// the next rows are requested before the ones in hand are turned.  The others have whole pairs: all the new rows of a pair are one
// workgroup's, which has read the pair's length before it writes it.
// Bound by memory, at 5.1 TB/s with all tokens there (128 x 64 tokens, 64 + 16 heads of 128, 336 MB in 66 us; without norms and rotation
// 5.8 TB/s: the arithmetic shows through); a step of one sequence is 4 us, three dependent reads after a launch.
template <typename T, typename C, int D>
__global__ __launch_bounds__(256) void fairkv_append_rotated_kernel(RotateArgs a)
{
    constexpr int L = D / kRow8, kSlots = 256 / L;          // lanes of a row, rows in hand
    constexpr int kPasses = FAIRKV_MAX_DRAFT / kSlots;      // of the rows of a pair
    constexpr int EB = sizeof(T), CB = sizeof(C);
    const int piece = threadIdx.x % L, slot = threadIdx.x / L;
    float weight[kRow8];
    const float *norm = static_cast<int>(blockIdx.x) < a.q_groups ? a.q_norm : a.k_norm;
#pragma unroll
    for (int i = 0; i < kRow8; ++i) weight[i] = norm ? norm[piece * kRow8 + i] : 1.f;

    if (static_cast<int>(blockIdx.x) < a.q_groups) {
        // Lane j of every wave looks after token j of the workgroup's: whether there is anything to do, and at which position.  A pass's tokens follow
        // one another; from pass to pass they lie all over the batch, and further on in their sequences, so that ragged drafts, whose last tokens
        // are none, leave every workgroup about as much to do (256 drafts of up to 64 tokens: 78 us instead of 95).
        const int each = kSlots / a.head_slots, n_tokens = a.B * a.q_len, lane = threadIdx.x & 63;
        const int of_lane = min(lane / each, a.passes - 1);
        const int token = (of_lane * a.q_groups + (static_cast<int>(blockIdx.x) + of_lane * a.apart) % a.q_groups) * each + lane % each;      // (fits 31 bits, and 256 more)
        const int looked = min(token, n_tokens - 1), of_b = looked / a.q_len;
        const bool live = lane < each * a.passes && token < n_tokens && looked - of_b * a.q_len < new_tokens(a.n_new, of_b, a.q_len);
        const int32_t held_pos = a.table ? a.pos[looked] : 0;
        const bool ok = live && in_table(a, held_pos);
        if (live && !ok && threadIdx.x < 64 && a.bad) atomicAdd(a.bad, 1);
        const uint64_t todo = __builtin_amdgcn_ballot_w64(ok);
        if (todo == 0) return;
        const int of_pass = slot / a.head_slots, h_slot = slot % a.head_slots;
        constexpr int kAhead = 4;
        struct Rows {
            typename Eight<T>::raw_t raw[kAhead];
            Turn t;
            int32_t token, h0;             // token < 0: nothing
        };
        int pass = 0, h_next = 0;          // of the rows to be requested next
        auto request = [&](Rows &x) __attribute__((always_inline)) {      // false: no more
            while (pass < a.passes && (todo >> (pass * each) & (~0ull >> (64 - each))) == 0) ++pass;
            if (pass >= a.passes) return false;
            const int j = pass * each + of_pass;
            const int32_t pos = __shfl(held_pos, j, 64), at = __shfl(token, j, 64);
            x.token = todo >> j & 1 ? at : -1, x.h0 = h_next + h_slot;
            if (x.token >= 0) {
                const char *src = a.q + (x.token * a.q_stride + piece * kRow8) * EB;
#pragma unroll
                for (int u = 0; u < kAhead; ++u) x.raw[u] = Eight<T>::load(src + static_cast<int64_t>(min(x.h0 + u * a.head_slots, a.Hq - 1)) * D * EB);
                x.t = turn_of(a, pos, piece);
            }
            h_next += kAhead * a.head_slots;
            if (h_next >= a.Hq) h_next = 0, ++pass;
            return true;
        };
        auto turn = [&](const Rows &x) __attribute__((always_inline)) {
            if (x.token < 0) return;       // whole rows: the lanes of the others stay
            char *dst = a.q_out + (static_cast<int64_t>(x.token) * a.Hq * D + piece * kRow8) * EB;
#pragma unroll
            for (int u = 0; u < kAhead; ++u) {
                const int h = x.h0 + u * a.head_slots;
                if (h >= a.Hq) break;
                float y[kRow8];
                Eight<T>::floats(x.raw[u], y);
                norm_and_turn<D>(a, y, norm != nullptr, weight, x.t, piece);
                Eight<T>::store(dst + static_cast<int64_t>(h) * D * EB, y);
            }
        };
        Rows one, other;
        bool more = request(one);
        while (more) {
            more = request(other);
            turn(one);
            if (!more) break;
            more = request(one);
            turn(other);
        }
        return;
    }

    __shared__ int32_t refused[kSlots];                     // per pair of the workgroup
    const int n_pairs = a.B * a.Hkv, per_group = max(1, kSlots / a.q_len);
    const int first = (static_cast<int>(blockIdx.x) - a.q_groups) * per_group;
    if (threadIdx.x < kSlots) refused[threadIdx.x] = 0;
    __syncthreads();
    typename Eight<T>::raw_t k_raw[kPasses], v_raw[kPasses];
    int64_t row[kPasses];
    int32_t pos[kPasses];
#pragma unroll
    for (int u = 0; u < kPasses; ++u) {
        const int r = slot + u * kSlots, own = r / a.q_len, pair = first + own, i = r % a.q_len;
        row[u] = -1;
        if (own >= per_group || pair >= n_pairs) continue;
        const int b = pair / a.Hkv, h = pair % a.Hkv;
        const int32_t nn = new_tokens(a.n_new, b, a.q_len);
        if (i >= nn) continue;
        const int64_t token = static_cast<int64_t>(b) * a.q_len + i;
        k_raw[u] = Eight<T>::load(a.k_new + (token * a.k_stride + h * D + piece * kRow8) * EB);
        v_raw[u] = Eight<T>::load(a.v_new + (token * a.v_stride + h * D + piece * kRow8) * EB);
        pos[u] = a.table ? a.pos[token] : 0;
        const int32_t l = a.len[pair], cap = a.cap[pair];
        // behind a length that leaves no room for all the new rows there is no row to look up
        if (l >= 0 && static_cast<int64_t>(l) + nn <= cap && in_table(a, pos[u])) row[u] = a.rows.row(pair, l + i);
        if (row[u] < 0 && piece == 0) refused[own] = 1;
    }
    int32_t l_new = 0;
    const bool counts = threadIdx.x < static_cast<unsigned>(per_group) && first + static_cast<int>(threadIdx.x) < n_pairs;
    if (counts) {
        const int pair = first + threadIdx.x;
        l_new = a.len[pair];
    }
    __syncthreads();
#pragma unroll
    for (int u = 0; u < kPasses; ++u) {
        const int r = slot + u * kSlots, own = r / a.q_len;
        if (row[u] < 0 || refused[own]) continue;
        const int h = (first + own) % a.Hkv;
        float x[kRow8], y[kRow8];
        Eight<T>::floats(k_raw[u], x);
        Eight<T>::floats(v_raw[u], y);
        norm_and_turn<D>(a, x, norm != nullptr, weight, turn_of(a, pos[u], piece), piece);
        if constexpr (CB == 1) {
            const int sc = a.n_scales > 1 ? h : 0;        // a rounded reciprocal would put one value in a thousand into the next step of the format
#pragma unroll
            for (int i = 0; i < kRow8; ++i) x[i] /= a.k_scale[sc], y[i] /= a.v_scale[sc];
        }
        Eight<C>::store(a.k + (row[u] * D + piece * kRow8) * CB, x);
        Eight<C>::store(a.v + (row[u] * D + piece * kRow8) * CB, y);
    }
    if (counts) {
        const int pair = first + threadIdx.x;
        const bool left_alone = refused[threadIdx.x] != 0;
        a.len_out[pair] = l_new + (left_alone ? 0 : new_tokens(a.n_new, pair / a.Hkv, a.q_len));
        if (left_alone && a.bad) atomicAdd(a.bad, 1);
    }
}

struct AcceptArgs {
    char *k, *v;
    const int32_t *path, *n_path;         // [B][q_len], [B]
    const int32_t *n_new;                 // [B] or null
    const int32_t *len;                   // [B * Hkv]
    int32_t *len_out, *bad;
    RowMap rows;
    int32_t B, Hkv, q_len;
};

// Row base + path[i] of a pair to row base + i, base being the length without the draft.  A workgroup has whole pairs and all
// the rows of a pair in registers before it writes one, so a path may be in any order.
template <int ROWB>
__global__ __launch_bounds__(256) void fairkv_accept_kernel(AcceptArgs a)
{
    constexpr int PPR = ROWB / 16, kSlots = 256 / PPR, kPasses = FAIRKV_MAX_DRAFT > kSlots ? FAIRKV_MAX_DRAFT / kSlots : 1;
    typedef __attribute__((ext_vector_type(4))) uint32_t u4;
    __shared__ int32_t refused[kSlots];
    const int piece = threadIdx.x % PPR, slot = threadIdx.x / PPR;
    const int n_pairs = a.B * a.Hkv, per_group = max(1, kSlots / a.q_len), first = blockIdx.x * per_group;
    for (int i = threadIdx.x; i < kSlots; i += 256) refused[i] = 0;
    __syncthreads();
    u4 kk[kPasses], vv[kPasses];
    int64_t to[kPasses];
#pragma unroll
    for (int u = 0; u < kPasses; ++u) {
        const int r = slot + u * kSlots, own = r / a.q_len, pair = first + own, i = r % a.q_len;
        to[u] = -1;
        if (own >= per_group || pair >= n_pairs) continue;
        const int b = pair / a.Hkv;
        const int32_t nn = new_tokens(a.n_new, b, a.q_len), kept = a.n_path[b], length = a.len[pair], base = max(length, nn) - nn;
        bool ok = kept >= 0 && kept <= nn && length >= nn;
        if (ok && i < kept) {
            const int32_t from = a.path[static_cast<int64_t>(b) * a.q_len + i];
            ok = from >= 0 && from < nn;
            const int64_t source = ok ? a.rows.row(pair, base + from) : -1;
            to[u] = source < 0 ? -1 : a.rows.row(pair, base + i);
            ok = to[u] >= 0;
            if (ok && from != i) {
                kk[u] = *reinterpret_cast<const u4 *>(a.k + source * ROWB + piece * 16);
                vv[u] = *reinterpret_cast<const u4 *>(a.v + source * ROWB + piece * 16);
            } else {
                to[u] = -1;                // in its place already, or refused
            }
        }
        if (!ok && piece == 0) refused[own] = 1;
    }
    int32_t l = 0;
    const bool counts = threadIdx.x < static_cast<unsigned>(per_group) && first + static_cast<int>(threadIdx.x) < n_pairs;
    if (counts) l = a.len[first + threadIdx.x];
    drain_vmem();                          // what another wave is about to write has been read
    __syncthreads();
#pragma unroll
    for (int u = 0; u < kPasses; ++u) {
        const int own = (slot + u * kSlots) / a.q_len;
        if (to[u] < 0 || refused[own]) continue;
        *reinterpret_cast<u4 *>(a.k + to[u] * ROWB + piece * 16) = kk[u];
        *reinterpret_cast<u4 *>(a.v + to[u] * ROWB + piece * 16) = vv[u];
    }
    if (counts) {
        const int pair = first + threadIdx.x, b = pair / a.Hkv;
        const bool left_alone = refused[threadIdx.x] != 0;
        a.len_out[pair] = left_alone ? l : l - new_tokens(a.n_new, b, a.q_len) + a.n_path[b];
        if (left_alone && a.bad) atomicAdd(a.bad, 1);
    }
}

}  // namespace fairkv
