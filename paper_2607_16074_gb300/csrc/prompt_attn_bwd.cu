// Gradients of the attention of packed prompts.
//
// With P = 2^(s c - lse) recomputed from the forward's log2-sum-exp, c = log2(e) /
// sqrt(hd), and D = rowsum(dO * O):  dV = P^T dO,  dS = P (dO V^T - D) / sqrt(hd),
// dQ = dS K,  dK = dS^T Q; a key head's gradients add over its group's query heads.
//
// Two passes of one launch, each summing in TMEM and writing its rows once, so no sum's
// order depends on anything but the sequence:
//   keys     a 128-key tile of a key head against the 128-row tiles (tokens x the
//            group's heads, as the forward's) that see it:
//            S^T = K Q^T, dP^T = V dO^T, dV += P^T dO, dK += dS^T Q
//   queries  a row tile against the 128-key tiles it sees:
//            S = Q K^T, dP = dO V^T, dQ += dS K
// Seven products for the gradients' five.  (Keeping dS for the second pass instead would move
// two bytes a score and head twice, 0.59 ps at 6.79 TB/s; the two products are 0.27 ps at the
// burst rate and 0.64 at the one reached.  Not built, not measured.)
//
// TMEM at head dim 128 holds S, dP and two accumulators of 128 columns each, so neither
// is double-buffered; instead the products and the elementwise warps take the halves of a
// tile in turn: P^T (over S) feeds dV, and S of the next tile follows dV while dS is
// formed; dS (over dP) feeds dK, and the next dP follows dK while P is formed.
// (In the queries' pass, whose one accumulator leaves room, a second dP was slower: 564 ->
// 598 us.)
//
// Six documents of up to 2,600 tokens, 32 heads of 128 (424 GFLOP with the forward): 428 us
// the passes and 34 the rows' values, 579 with the forward's 121 (588 in longer runs).
// The tensor core is busy for 42 % of it: the elementwise warps' P and dS and the products
// wait for each other, as there is no TMEM to double-buffer either.
//
// Warps (one CTA an SM, items claimed from one queue, the longest of each pass first):
//   0     claims items and hands them out; TMA: the item's outer tiles (K and V, or Q
//         and dO), inner tiles through two rings of two or three
//   1     MMA issuer
//   2     the rows' lse and D of each inner row tile (keys pass)
//   4-11  elementwise: warps 4-7 a tile's first 64 columns, 8-11 the others; then the
//         accumulators out
// Inner rows past a sequence's end belong to others and may be NaN: they are zeroed in
// shared memory, and their lse is +inf, which makes their probabilities zero.
#include <algorithm>
#include <type_traits>

#include "jnx_dev.cuh"
#include "jnx_kernels.h"
#include "jnx_text.h"
#include "jnx_trace.h"

namespace jnx {

jnx_status prompt_ok(const jnx_prompt* p, const char* what, int& rows, int& keys);
jnx_status prompt_launchable(const jnx_prompt* p, const char* what, bool gradients, int& rows,
                             int& keys);
PromptCounts prompt_counts(const jnx_prompt* p, int H, int Hkv, int hd, bool gradients);

namespace pbwd {
constexpr int BM = 128;
enum { KEYS = 0, QUERIES = 1 };
// barriers of a pass
enum { O_FULL = 0, O_EMPTY = 1, B1_FULL = 2, B1_EMPTY = 5, B2_FULL = 8, B2_EMPTY = 11, S_FULL = 14,
       DP_FULL = 15, P_FULL = 16, DS_FULL = 17, ACC_FULL = 18, ACC_FREE = 19, DRAIN = 20,
       ST_FULL = 21, ST_EMPTY = 25, W_FULL = 29, W_EMPTY = 32, N_BARS = 35 };
constexpr int ITEMS = 3;  // items handed out at a time
constexpr int ST = 4;  // slots of row values
constexpr int THREADS = 384, EW = 8;
constexpr int READERS = 2 + EW;  // warps that an item is handed to: MMA, row values, elementwise
}  // namespace pbwd

template <int HD>
struct PromptBwdCfg {
    static_assert(HD == 64 || HD == 128, "head dim");
    static constexpr int TILE = pbwd::BM * HD * 2;
    static constexpr int SLOTS = HD == 64 ? 3 : 2;  // of each ring
    static constexpr int OFF_B1 = 2 * TILE, OFF_B2 = OFF_B1 + SLOTS * TILE;
    static constexpr int OFF_STG = OFF_B2 + SLOTS * TILE;  // 2 KB an elementwise warp
    static constexpr int OFF_ST = OFF_STG + pbwd::EW * 2048;  // [ST][-lse, -D][128]
    static constexpr int OFF_BAR = OFF_ST + pbwd::ST * 2 * pbwd::BM * 4;
    static constexpr int SMEM = OFF_BAR + 2 * pbwd::N_BARS * 8 + 16 + pbwd::ITEMS * 36 + 1024;
    static_assert(SMEM <= 227 * 1024, "shared memory per CTA");
    static constexpr uint32_t S_COL = 0, DP_COL = 128, ACC_COL = 256;
};

struct PromptBwdArgs {
    const int *cu_q, *cu_kv, *prefix;
    const int2* items;  // of the keys pass, then of the queries pass
    int n_keys, n_queries, H, Hkv, group;
    int* claimed;       // items taken beyond the grid's first: 0 at launch
    float scale_log2, scale;
    const float2* row;  // [Hkv][rows][group]: lse (+inf where a row sees no key), D
    const float* few;   // alike: D of rows of few keys, in place of the other
    int n_seqs, rows, keys;  // what the items may name
    jnx_head_rows dq, dk, dv;
    // the sums of tiles taken in parts, [item of the keys' pass][Hkv][dk, dv][128][hd], for the
    // items up to the last one of such a tile
    float* part;
    int n_slabs;
    int* status;
};

// What the warps of a CTA are told of an item.
struct PromptBwdItem {
    int at, kvh, q0, Lq, k0, Lk, pre;  // at: first key or row; Lq < 0: no more in this pass
    int part, unit;                    // keys pass; number among the items' key heads

    // keys pass: parts of the tile, and this part's inner tiles [j0, j1) of T tokens from the
    // first row that sees the tile's first key
    __device__ __forceinline__ int parts(int group, int Hkv) const {
        return key_parts(at, Lq, Lk, pre, group, Hkv);
    }
    __device__ __forceinline__ void range(int group, int Hkv, int T, int& i0, int& n) const {
        const int first = first_row(at, Lq, Lk, pre), np = parts(group, Hkv);
        const int all = (Lq - first + T - 1) / T;
        const int j0 = (int)((long long)all * part / np), j1 = (int)((long long)all * (part + 1) / np);
        i0 = first + j0 * T;
        n = j1 - j0;
    }
};

// A claimed item's list entry: false, and reported, where it names no row, or no key and part,
// of the prompt.
template <bool KP>
__device__ __forceinline__ bool bwd_item(const PromptBwdArgs& p, int2 e, int unit, PromptBwdItem& x) {
    const int item = unit / p.Hkv;
    PromptSeq s;
    bool ok = prompt_seq(p.cu_q, p.cu_kv, p.prefix, p.n_seqs, p.rows, p.keys, e.x, s);
    x = PromptBwdItem{KP ? e.y & ~127 : e.y, unit - item * p.Hkv, s.q0, s.Lq, s.k0, s.Lk, s.pre,
                      KP ? e.y & 127 : 0, unit};
    ok = ok && (unsigned)x.at < (unsigned)(KP ? x.Lk : x.Lq);
    if (KP && ok && (x.part > 0 || item >= p.n_slabs)) {
        const int np = x.parts(p.group, p.Hkv);
        ok = x.part < np && (np == 1 || item < p.n_slabs);
    }
    if (!ok && (threadIdx.x & 31) == 0) report(p.status, JNX_ERR_DEVICE_BOUNDS);
    return ok;
}

constexpr int kFewKeys = 64, kFewTiles = 2;  // keys of a row at most; tiles of 16 rows a CTA

// lse and D of row i of an item's sequence and head hg of its group.
__device__ __forceinline__ float2 row_values(const PromptBwdArgs& p, const PromptBwdItem& x, int i, int hg) {
    const size_t at = ((size_t)x.kvh * p.rows + x.q0 + i) * p.group + hg;
    const int seen = keys_seen(i, x.Lq, x.Lk, x.pre);
    const float* d = 0 < seen && seen <= kFewKeys ? p.few + at : &p.row[at].y;  // (one load, no branch)
    return make_float2(p.row[at].x, *d);
}

__device__ __forceinline__ float dot8(const uint4& a, const uint4& b) {
    const uint32_t x[4] = {a.x, a.y, a.z, a.w}, y[4] = {b.x, b.y, b.z, b.w};
    float d = 0.f;
#pragma unroll
    for (int e = 0; e < 4; ++e)
        d += __uint_as_float(x[e] << 16) * __uint_as_float(y[e] << 16) +
             __uint_as_float(x[e] & 0xffff0000u) * __uint_as_float(y[e] & 0xffff0000u);
    return d;
}
__device__ __forceinline__ uint4 head_unit(const jnx_head_rows& r, long long at, int head, int c) {
    return *reinterpret_cast<const uint4*>(r.ptr + at * r.row_stride + head * r.head_stride + c);
}
template <int LANES>
__device__ __forceinline__ float lanes_sum(float d) {
#pragma unroll
    for (int o = LANES / 2; o; o >>= 1) d += __shfl_xor_sync(0xffffffffu, d, o);
    return d;
}

// Rows that see few keys: their D over again.  dS = P (dP - D) adds up to zero over a row's keys
// only as far as D is what the kernel's own P and dP add up to.  rowsum(dO * O) is off by the
// roundings of O and of the forward's P, which shows where few terms nearly cancel: dQ of
// sequences of two tokens was off by 0.0050 of its norm, of 12 to 64 tokens by 0.0026, against
// the 0.0024 that its own two roundings make.  Up to kFewKeys keys D is the sum of P dP in fp32;
// beyond, the rounding of O is one of several alike (400 tokens: 0.0025).
// Four warps 16 rows (token, head of the group) of a sequence and key head, 16 of the keys each,
// by mma.sync: 32 columns of the contraction at a time, of which a lane holds eight neighbours of
// each operand, so that both are loaded by 16 bytes and agree on which columns a product takes.
// Bound by the loads' latency, a step after another, while the other rows' loads keep HBM busy:
// 26 us in all of 26 samples of up to 840 tokens, 8 heads on one of 256.  (By a launch of its
// own, 24 and 9 us, or 26 with a warp for all 64 keys whose loads waited for one another.)
// A lane's two rows of such a tile.
struct FewRows {
    int at[2], head[2], seen[2];
    float l[2];
};
// What 16 keys from k0 on make up of D of a tile's rows; the loads of four steps are under way
// at once.
template <int HD>
__device__ __forceinline__ void few_rows(const jnx_head_rows& dout, const jnx_head_rows& q,
                                         const jnx_head_rows& k, const jnx_head_rows& v, const PromptSeq& s,
                                         int kvh, int k0, float scale_log2, const FewRows& r,
                                         float (&d)[2]) {
    const int lane = threadIdx.x & 31, g = lane >> 2, c = (lane & 3) * 8;
    constexpr int NT = 2;  // of eight keys
    float sc[NT][4] = {}, dp[NT][4] = {};
#pragma unroll 4
    for (int x = c; x < HD; x += 32) {
        uint4 qa[2], ga[2], kk[NT], vv[NT];
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            qa[e] = head_unit(q, r.at[e], r.head[e], x);
            ga[e] = head_unit(dout, r.at[e], r.head[e], x);
        }
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            const long long key = s.k0 + min(k0 + t * 8 + g, s.Lk - 1);
            kk[t] = head_unit(k, key, kvh, x);
            vv[t] = head_unit(v, key, kvh, x);
        }
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            mma_bf16(sc[t], qa[0].x, qa[1].x, qa[0].y, qa[1].y, kk[t].x, kk[t].y);
            mma_bf16(sc[t], qa[0].z, qa[1].z, qa[0].w, qa[1].w, kk[t].z, kk[t].w);
            mma_bf16(dp[t], ga[0].x, ga[1].x, ga[0].y, ga[1].y, vv[t].x, vv[t].y);
            mma_bf16(dp[t], ga[0].z, ga[1].z, ga[0].w, ga[1].w, vv[t].z, vv[t].w);
        }
    }
    d[0] = d[1] = 0.f;
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int e = i >> 1;
            if (k0 + t * 8 + (lane & 3) * 2 + (i & 1) < r.seen[e])
                d[e] += ex2_approx(fmaf(sc[t][i], scale_log2, -r.l[e])) * dp[t][i];
        }
#pragma unroll
    for (int e = 0; e < 2; ++e) {
        d[e] += __shfl_xor_sync(0xffffffffu, d[e], 1);
        d[e] += __shfl_xor_sync(0xffffffffu, d[e], 2);
    }
}

// A CTA's share, `of` CTAs a sequence and key head.
template <int HD>
__device__ __forceinline__ void few_tiles(const jnx_head_rows& dout, const jnx_head_rows& q,
                                          const jnx_head_rows& k, const jnx_head_rows& v, const float* lse,
                                          const PromptBwdArgs& p, float* few, int cta, int of) {
    __shared__ float part[kFewTiles][4][16];
    const int sq = cta / of / p.Hkv, kvh = cta / of % p.Hkv;
    PromptSeq s;
    if (!prompt_seq(p.cu_q, p.cu_kv, p.prefix, p.n_seqs, p.rows, p.keys, sq, s)) {
        if (threadIdx.x == 0) report(p.status, JNX_ERR_DEVICE_BOUNDS);
        return;
    }
    // rows [a, b): the first that sees a key, the first that sees too many
    const int a = first_row(0, s.Lq, s.Lk, s.pre);
    const int b = s.Lk > kFewKeys ? first_row(kFewKeys, s.Lq, s.Lk, s.pre) : s.Lq;
    const int n = s.Lk > 0 ? (b - a) * p.group : 0;
    const int lane = threadIdx.x & 31, g = lane >> 2;
    const int tile = threadIdx.x >> 7, quarter = warp_uniform(threadIdx.x >> 5) & 3;
    for (int c0 = cta % of * kFewTiles * 16; c0 < n; c0 += of * kFewTiles * 16) {
        const int t0 = c0 + tile * 16;
        FewRows r;  // one beyond the last goes along with it
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const int w = min(t0 + g + 8 * e, n - 1), i = a + w / p.group;
            r.at[e] = s.q0 + i;
            r.head[e] = kvh * p.group + w % p.group;
            r.seen[e] = keys_seen(i, s.Lq, s.Lk, s.pre);
            r.l[e] = lse[(long long)r.at[e] * p.H + r.head[e]];
        }
        // a warp's quarter of the keys, as far as the tile's last row sees them
        const int most = keys_seen(a + min(t0 + 15, n - 1) / p.group, s.Lq, s.Lk, s.pre);
        float d[2] = {0.f, 0.f};
        if (t0 < n && most > 16 * quarter)
            few_rows<HD>(dout, q, k, v, s, kvh, 16 * quarter, p.scale_log2, r, d);
        float(&sums)[4][16] = part[tile];
        if ((lane & 3) == 0) sums[quarter][g] = d[0], sums[quarter][g + 8] = d[1];
        __syncthreads();
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const int u = g + 8 * e;
            if (quarter == 0 && (lane & 3) == 0 && t0 + u < n)
                few[((long long)kvh * p.rows + r.at[e]) * p.group + r.head[e] - kvh * p.group] =
                    (sums[0][u] + sums[1][u]) + (sums[2][u] + sums[3][u]);
        }
        __syncthreads();
    }
}

// The rows' (lse, D = rowsum(dO * O)), D of rows of few keys beside it, and the claim counter to
// zero.  HD / 8 lanes a row, four rows of neighbouring heads a lane, whose loads are under way at
// once: bound by HBM.  (By tiles of a sequence and key head, 256 bytes a row, they were half as
// slow again.)  The first n_few CTAs take the rows of few keys meanwhile, whose place in a
// sequence the others do not know.
template <int HD>
__global__ void __launch_bounds__(256, 3)
    k_prompt_bwd_rows(jnx_head_rows out, jnx_head_rows dout, jnx_head_rows q, jnx_head_rows k,
                      jnx_head_rows v, const float* lse, const __grid_constant__ PromptBwdArgs p,
                      float2* row, float* few, int n_few, int of) {
    constexpr int LANES = HD / 8, PER = 256 / LANES;
    pdl_entry();
    if (blockIdx.x == 0 && threadIdx.x == 0) *p.claimed = 0;
    if ((int)blockIdx.x < n_few) {
        few_tiles<HD>(dout, q, k, v, lse, p, few, blockIdx.x, of);
        return;
    }
    const long long all = (long long)p.rows * p.H;
    const long long w0 = (long long)(blockIdx.x - n_few) * PER * 4 + threadIdx.x / LANES;
    const int c = threadIdx.x % LANES * 8;
    uint4 g[4], o[4];
    float l[4];
#pragma unroll
    for (int b = 0; b < 4; ++b) {
        const long long w = w0 + b * PER;
        g[b] = o[b] = make_uint4(0, 0, 0, 0);
        l[b] = 0.f;
        if (w < all) {
            const long long r = w / p.H;
            const int h = (int)(w - r * p.H);
            g[b] = head_unit(dout, r, h, c);
            o[b] = head_unit(out, r, h, c);
            l[b] = lse[w];
        }
    }
#pragma unroll
    for (int b = 0; b < 4; ++b) {
        const float d = lanes_sum<LANES>(dot8(o[b], g[b]));
        const long long w = w0 + b * PER;
        if (w < all && c == 0) {
            const long long r = w / p.H;
            const int h = (int)(w - r * p.H);
            row[((long long)(h / p.group) * p.rows + r) * p.group + h % p.group] =
                l[b] == -INFINITY ? make_float2(INFINITY, 0.f) : make_float2(l[b], d);
        }
    }
}

// 32 fp32 columns of a warp's 32 rows (a lane a row), scaled, out as bf16 through 2 KB of
// staging: lane l writes unit l % 4 of rows l / 4 + 8 u to base + at[u] (-1: no row).
__device__ __forceinline__ void bwd_rows_out(uint8_t* stg, int lane, const uint32_t (&v)[32], float f,
                                             uint16_t* base, const long long (&at)[4]) {
#pragma unroll
    for (int e = 0; e < 4; ++e)
        *reinterpret_cast<uint4*>(stg + lane * 64 + ((e ^ ((lane >> 1) & 3)) << 4)) = make_uint4(
            cvt_bf2(f * __uint_as_float(v[8 * e]), f * __uint_as_float(v[8 * e + 1])),
            cvt_bf2(f * __uint_as_float(v[8 * e + 2]), f * __uint_as_float(v[8 * e + 3])),
            cvt_bf2(f * __uint_as_float(v[8 * e + 4]), f * __uint_as_float(v[8 * e + 5])),
            cvt_bf2(f * __uint_as_float(v[8 * e + 6]), f * __uint_as_float(v[8 * e + 7])));
    __syncwarp();
#pragma unroll
    for (int u = 0; u < 4; ++u) {
        const int r = 8 * u + (lane >> 2), un = lane & 3;
        const uint4 q = *reinterpret_cast<const uint4*>(stg + r * 64 + ((un ^ ((r >> 1) & 3)) << 4));
        if (at[u] >= 0) *reinterpret_cast<uint4*>(base + at[u] + un * 8) = q;
    }
    __syncwarp();
}

// The same in fp32, unscaled, 16 columns at a time.
__device__ __forceinline__ void bwd_rows_part(uint8_t* stg, int lane, const uint32_t (&v)[32], float* base,
                                              const long long (&at)[4]) {
#pragma unroll
    for (int c = 0; c < 2; ++c) {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            *reinterpret_cast<uint4*>(stg + lane * 64 + ((e ^ ((lane >> 1) & 3)) << 4)) =
                make_uint4(v[16 * c + 4 * e], v[16 * c + 4 * e + 1], v[16 * c + 4 * e + 2],
                           v[16 * c + 4 * e + 3]);
        __syncwarp();
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const int r = 8 * u + (lane >> 2), un = lane & 3;
            const uint4 q = *reinterpret_cast<const uint4*>(stg + r * 64 + ((un ^ ((r >> 1) & 3)) << 4));
            if (at[u] >= 0) *reinterpret_cast<uint4*>(base + at[u] + c * 16 + un * 4) = q;
        }
        __syncwarp();
    }
}

// dk and dv of the tiles taken in parts: their sums in the parts' order, whose items follow one
// another in the list.  A CTA 8 keys of a tile and key head, of either gradient.  (Bound by
// reading the sums: CTAs of 16 keys, or a share of the keys to each part's item so that none is
// without work, took the same time: 12 us of 26 samples of up to 840 tokens, 8 heads on one
// of 256.)
__global__ void __launch_bounds__(256) k_prompt_bwd_join(const __grid_constant__ PromptBwdArgs p, int hd) {
    pdl_entry();
    const int2 e = p.items[blockIdx.x / p.Hkv];
    PromptSeq s;  // (an item that names no tile has been reported)
    if ((e.y & 127) || e.y < 0 ||
        !prompt_seq(p.cu_q, p.cu_kv, p.prefix, p.n_seqs, p.rows, p.keys, e.x, s) || e.y >= s.Lk)
        return;
    const int kvh = blockIdx.x % p.Hkv, k0 = s.k0, Lk = s.Lk;
    const int np = key_parts(e.y, s.Lq, Lk, s.pre, p.group, p.Hkv);
    if (np == 1 || blockIdx.x / p.Hkv + np > p.n_slabs) return;
    const int cols = hd / 4, which = blockIdx.z;
    for (int i = threadIdx.x; i < 8 * cols; i += 256) {
        const int r = blockIdx.y * 8 + i / cols, c = i % cols * 4;
        if (e.y + r >= Lk) return;
        const long long key = k0 + e.y + r;
        const float* from = p.part + ((long long)blockIdx.x * 2 + which) * 128 * hd + r * hd + c;
        const long long step = (long long)p.Hkv * 2 * 128 * hd;
        float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
        for (int k = 0; k < np; ++k) {
            const float4 v = *reinterpret_cast<const float4*>(from + k * step);
            s = make_float4(s.x + v.x, s.y + v.y, s.z + v.z, s.w + v.w);
        }
        const float f = which ? 1.f : p.scale;
        const jnx_head_rows& to = which ? p.dv : p.dk;
        *reinterpret_cast<uint2*>(to.ptr + key * to.row_stride + kvh * to.head_stride + c) =
            make_uint2(cvt_bf2(s.x * f, s.y * f), cvt_bf2(s.z * f, s.w * f));
    }
}

template <int HD, int PASS>
__device__ __forceinline__ int prompt_bwd_pass(const CUtensorMap& tq, const CUtensorMap& tk,
                                               const CUtensorMap& tv, const CUtensorMap& tdo,
                                               const PromptBwdArgs& p, uint8_t* sm, uint64_t* bar,
                                               volatile int* fail_flag, uint32_t tbase, int q_first,
                                               int claim) {
    using C = PromptBwdCfg<HD>;
    using namespace pbwd;
    constexpr bool KP = PASS == KEYS;
    constexpr int NCH = HD / 64, SLOTS = C::SLOTS;
    const int T = tile_tokens(p.group), row_bytes = p.group * T * HD * 2;
    const int warp = warp_uniform(threadIdx.x >> 5), lane = threadIdx.x & 31;
    uint8_t* b1 = sm + C::OFF_B1;
    uint8_t* b2 = sm + C::OFF_B2;
    float* st = reinterpret_cast<float*>(sm + C::OFF_ST);
    volatile int* slot = fail_flag + 1;  // [ITEMS][9]: items handed out
    const int2* items = p.items + (KP ? 0 : p.n_keys);
    const int n_work = (KP ? p.n_keys : p.n_queries) * p.Hkv;

    // the next item as warp 0 hands it out; item_done() gives its slot back
    int seen = 0;
    auto get_item = [&](int b) -> PromptBwdItem {
        const volatile int* s = slot + 9 * b;
        return PromptBwdItem{warp_uniform(s[0]), warp_uniform(s[1]), warp_uniform(s[2]), warp_uniform(s[3]),
                             warp_uniform(s[4]), warp_uniform(s[5]), warp_uniform(s[6]), warp_uniform(s[7]),
                             warp_uniform(s[8])};
    };
    auto item_done = [&]() {
        __syncwarp();
        if (elect_one()) mbar_arrive(&bar[W_EMPTY + seen % ITEMS]);
        __syncwarp();
        ++seen;
    };
    auto next_item = [&](bool& ok) -> PromptBwdItem {
        const int b = seen % ITEMS;
        if (!(ok = mbar_wait_warp(&bar[W_FULL + b], (seen / ITEMS) & 1)))
            return PromptBwdItem{0, 0, 0, -1, 0, 0, 0, 0, 0};
        return get_item(b);
    };
    // an item's inner tiles, and the keys pass's first inner row
    auto inner = [&](const PromptBwdItem& x, int& i0, int& n) {
        if (KP) {
            x.range(p.group, p.Hkv, T, i0, n);
        } else {
            i0 = x.at;
            n = (keys_seen(min(x.at + T, x.Lq) - 1, x.Lq, x.Lk, x.pre) + BM - 1) / BM;
        }
    };

    if (warp == 0) {
        // ---------------- claims and TMA ----------------
        bool ok = true;
        int told = 0;
        auto tell = [&](const PromptBwdItem& x) {
            const int b = told % ITEMS;
            if (!mbar_wait_warp(&bar[W_EMPTY + b], ((told / ITEMS) & 1) ^ 1)) return false;
            if (elect_one()) {
                slot[9 * b] = x.at;
                slot[9 * b + 1] = x.kvh;
                slot[9 * b + 2] = x.q0;
                slot[9 * b + 3] = x.Lq;
                slot[9 * b + 4] = x.k0;
                slot[9 * b + 5] = x.Lk;
                slot[9 * b + 6] = x.pre;
                slot[9 * b + 7] = x.part;
                slot[9 * b + 8] = x.unit;
                mbar_arrive(&bar[W_FULL + b]);
            }
            __syncwarp();
            ++told;
            return true;
        };
        int no = 0;       // outer pairs loaded
        uint32_t g = 0;   // inner pairs loaded
        auto load = [&](const CUtensorMap* m, uint8_t* dst, int head, int row, uint64_t* full) {
#pragma unroll
            for (int c = 0; c < NCH; ++c) tma_load_3d(dst + c * BM * 128, m, c * 64, head, row, full);
        };
        // the next item that names a tile
        PromptBwdItem nx{0, 0, 0, 0, 0, 0, 0, 0, 0};
        auto fetch = [&]() {
            for (;;) {
                claim = __shfl_sync(0xffffffffu, claim, 0);
                const int w = claim - q_first;
                if (w >= n_work || bwd_item<KP>(p, items[w / p.Hkv], w, nx)) return;
                if (lane == 0) claim = (int)gridDim.x + atomicAdd(p.claimed, 1);
            }
        };
        fetch();
        while (claim - q_first < n_work) {
            if (__any_sync(0xffffffffu, *fail_flag)) {
                ok = false;
                break;
            }
            PromptBwdItem x;
            x.at = warp_uniform(nx.at);
            x.kvh = warp_uniform(nx.kvh);
            x.q0 = warp_uniform(nx.q0);
            x.Lq = warp_uniform(nx.Lq);
            x.k0 = warp_uniform(nx.k0);
            x.Lk = warp_uniform(nx.Lk);
            x.pre = warp_uniform(nx.pre);
            x.part = warp_uniform(nx.part);
            x.unit = warp_uniform(nx.unit);
            if (lane == 0) claim = (int)gridDim.x + atomicAdd(p.claimed, 1);
            __syncwarp();
            if (!(ok = tell(x))) break;
            int i0, n;
            inner(x, i0, n);
            if (n > 0) {
                if (no > 0 && !(ok = mbar_wait_warp(&bar[O_EMPTY], (no - 1) & 1))) break;
                if (elect_one()) {
                    mbar_arrive_expect_tx(&bar[O_FULL], KP ? 2 * C::TILE : 2 * row_bytes);
                    if (KP) {
                        load(&tk, sm, x.kvh, x.k0 + x.at, &bar[O_FULL]);
                        load(&tv, sm + C::TILE, x.kvh, x.k0 + x.at, &bar[O_FULL]);
                    } else {
                        load(&tq, sm, x.kvh * p.group, x.q0 + x.at, &bar[O_FULL]);
                        load(&tdo, sm + C::TILE, x.kvh * p.group, x.q0 + x.at, &bar[O_FULL]);
                    }
                }
                __syncwarp();
                ++no;
            }
            for (int j = 0; j < n && ok; ++j, ++g) {
                const int s = g % SLOTS;
                const uint32_t ph = ((g / SLOTS) & 1) ^ 1;
                if (!(ok = mbar_wait_warp(&bar[B1_EMPTY + s], ph))) break;
                if (elect_one()) {
                    mbar_arrive_expect_tx(&bar[B1_FULL + s], KP ? row_bytes : C::TILE);
                    if (KP) load(&tq, b1 + s * C::TILE, x.kvh * p.group, x.q0 + i0 + j * T, &bar[B1_FULL + s]);
                    else load(&tk, b1 + s * C::TILE, x.kvh, x.k0 + j * BM, &bar[B1_FULL + s]);
                }
                __syncwarp();
                if (!(ok = mbar_wait_warp(&bar[B2_EMPTY + s], ph))) break;
                if (elect_one()) {
                    mbar_arrive_expect_tx(&bar[B2_FULL + s], KP ? row_bytes : C::TILE);
                    if (KP) load(&tdo, b2 + s * C::TILE, x.kvh * p.group, x.q0 + i0 + j * T, &bar[B2_FULL + s]);
                    else load(&tv, b2 + s * C::TILE, x.kvh, x.k0 + j * BM, &bar[B2_FULL + s]);
                }
                __syncwarp();
            }
            if (!ok) break;
            fetch();
        }
        ok = ok && tell(PromptBwdItem{0, 0, 0, -1, 0, 0, 0, 0, 0});
        if (!ok) *fail_flag = 1;
        // every copy has landed before the pass ends (at once in a normal run)
        if (no > 0) mbar_wait_warp(&bar[O_FULL], (no - 1) & 1, 100000000LL);
        for (uint32_t i = g > SLOTS ? g - SLOTS : 0; i < g; ++i) {
            mbar_wait_warp(&bar[B1_FULL + i % SLOTS], (i / SLOTS) & 1, 100000000LL);
            mbar_wait_warp(&bar[B2_FULL + i % SLOTS], (i / SLOTS) & 1, 100000000LL);
        }
    } else if (warp == 1) {
        // ---------------- MMA issuer ----------------
        constexpr uint32_t IDESC_S = idesc_bf16_f32(BM, BM);
        constexpr uint32_t IDESC_ACC = idesc_bf16_f32(BM, HD) | (1u << 16);  // B MN-major
        bool ok = true, issued = false;
        int no = 0, done = 0;  // outer pairs taken, items finished
        uint32_t g1 = 0, g2 = 0, gp = 0;  // inner tiles taken by S and by dP; P / dS tiles taken
        auto commit = [&](uint64_t* b) {
            if (elect_one()) tc_commit(b);
            __syncwarp();
        };
        auto score = [&](uint32_t d, uint32_t outer, uint8_t* inner) {
            const uint32_t a_lo = sw128_desc_lo(outer), b_lo = sw128_desc_lo(smem_u32(inner));
            if (elect_one()) {
#pragma unroll
                for (int ks = 0; ks < HD / 16; ++ks) {
                    const uint32_t off = (ks >> 2) * BM * 8 + (ks & 3) * 2;
                    tc_mma_f16(d, desc_of(a_lo + off, kSw128DescHi), desc_of(b_lo + off, kSw128DescHi),
                               IDESC_S, ks > 0);
                }
            }
            __syncwarp();
            issued = true;
        };
        // acc += X B, X bf16 in TMEM: 64 inner rows at column x, 64 at x + 64
        auto gather = [&](uint32_t acc, uint32_t x, uint8_t* inner, bool accumulate) {
            const uint32_t b_lo = sw128_desc_mn_lo(smem_u32(inner), BM * 128);
            if (elect_one()) {
#pragma unroll
                for (int ks = 0; ks < BM / 16; ++ks)
                    tc_mma_f16_ts(acc, x + (ks >> 2) * 64 + (ks & 3) * 8,
                                  desc_of(b_lo + ks * 128, kSw128DescHi), IDESC_ACC,
                                  accumulate || ks > 0);
            }
            __syncwarp();
        };
        auto zero_tail = [&](uint8_t* tile, int valid, int end) {
            for (int i = lane; i < (end - valid) * (HD / 8); i += 32) {
                const int r = valid + i / (HD / 8), u = i % (HD / 8);
                *reinterpret_cast<uint4*>(tile + (u >> 3) * BM * 128 + r * 128 + (u & 7) * 16) =
                    make_uint4(0, 0, 0, 0);
            }
            fence_proxy_async();
            __syncwarp();
        };
        while (ok) {
            const PromptBwdItem x = next_item(ok);
            if (!ok || x.Lq < 0 || __any_sync(0xffffffffu, *fail_flag)) break;
            item_done();
            int i0, n;
            inner(x, i0, n);
            if (n == 0) continue;
            if (!(ok = mbar_wait_warp(&bar[O_FULL], no & 1))) break;
            ++no;
            tc_fence_after();
            const uint32_t o1 = smem_u32(sm), o2 = o1 + C::TILE;
            // inner rows of tile j that are the sequence's, of those a box loads
            const int box = KP ? p.group * T : BM;
            auto valid = [&](int j) {
                return KP ? min(T, x.Lq - i0 - j * T) * p.group : min(BM, x.Lk - j * BM);
            };
            // a tile is waited for before the P or dS that its product follows in the queue:
            // it is mostly there, and those are what the tensor core then waits for
            auto wait_b1 = [&](int j) -> bool {
                const int s = g1 % SLOTS;
                if (!mbar_wait_warp(&bar[B1_FULL + s], (g1 / SLOTS) & 1)) return false;
                if (valid(j) < box) zero_tail(b1 + s * C::TILE, valid(j), box);
                return true;
            };
            auto wait_b2 = [&](int j) -> bool {
                const int s = g2 % SLOTS;
                if (!mbar_wait_warp(&bar[B2_FULL + s], (g2 / SLOTS) & 1)) return false;
                if (KP && valid(j) < box) zero_tail(b2 + s * C::TILE, valid(j), box);
                return true;
            };
            auto next_s = [&]() {
                const int s = g1 % SLOTS;
                tc_fence_after();
                score(tbase + C::S_COL, o1, b1 + s * C::TILE);
                commit(&bar[S_FULL]);
                ++g1;
            };
            auto next_dp = [&]() {
                const int s = g2 % SLOTS;
                tc_fence_after();
                score(tbase + C::DP_COL, o2, b2 + s * C::TILE);
                commit(&bar[DP_FULL]);
                if (!KP) commit(&bar[B2_EMPTY + s]);  // V is done with
                ++g2;
            };
            if (!(ok = wait_b1(0))) break;
            next_s();
            if (!(ok = wait_b2(0))) break;
            next_dp();
            if (n == 1) commit(&bar[O_EMPTY]);
            for (int j = 0; j < n && ok; ++j, ++gp) {
                const int s = gp % SLOTS;
                if (j + 1 < n && !(ok = wait_b1(j + 1))) break;
                // P^T over S (keys pass), or S read (queries pass)
                if (!(ok = mbar_wait_warp(&bar[P_FULL], gp & 1))) break;
                // the item's first sums overwrite the accumulators: the last epilogue has read them
                if (j == 0 && done > 0 && !(ok = mbar_wait_warp(&bar[ACC_FREE], (done - 1) & 1))) break;
                tc_fence_after();
                if (KP) {
                    gather(tbase + C::ACC_COL + HD, tbase + C::S_COL, b2 + s * C::TILE, j > 0);
                    commit(&bar[B2_EMPTY + s]);
                }
                if (j + 1 < n) {
                    next_s();
                    if (!(ok = wait_b2(j + 1))) break;
                }
                if (!(ok = mbar_wait_warp(&bar[DS_FULL], gp & 1))) break;
                tc_fence_after();
                gather(tbase + C::ACC_COL, tbase + C::DP_COL, b1 + s * C::TILE, j > 0);
                commit(&bar[B1_EMPTY + s]);
                if (j + 1 < n) {
                    next_dp();
                    if (j + 2 == n) commit(&bar[O_EMPTY]);
                }
            }
            if (!ok) break;
            commit(&bar[ACC_FULL]);
            ++done;
        }
        if (!ok) *fail_flag = 1;
        if (issued) {
            commit(&bar[DRAIN]);
            mbar_wait_warp(&bar[DRAIN], 0, 100000000LL);
        }
    } else if (warp == 2) {
        // ---------------- values of the inner rows (keys pass) ----------------
        bool ok = true;
        uint32_t g = 0;
        while (ok) {
            const PromptBwdItem x = next_item(ok);
            if (!ok || x.Lq < 0 || __any_sync(0xffffffffu, *fail_flag)) break;
            item_done();
            if (!KP) continue;
            int i0, n;
            inner(x, i0, n);
            for (int j = 0; j < n; ++j, ++g) {
                const int b = g % ST;
                float2 v[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int r = e * 32 + lane, t = r / p.group, i = i0 + j * T + t;
                    const bool live = t < T && i < x.Lq;
                    v[e] = live ? row_values(p, x, i, r - t * p.group) : make_float2(INFINITY, 0.f);
                }
                if (!(ok = mbar_wait_warp(&bar[ST_EMPTY + b], ((g / ST) & 1) ^ 1))) break;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int r = e * 32 + lane;
                    st[b * 256 + r] = -v[e].x;
                    st[b * 256 + 128 + r] = -v[e].y;
                }
                mbar_arrive(&bar[ST_FULL + b]);
            }
        }
        if (!ok) *fail_flag = 1;
    } else if (warp >= 4) {
        // ---------------- elementwise + epilogue ----------------
        const int quarter = warp & 3, half = (warp - 4) >> 2;
        const uint32_t lane_base = (uint32_t)(quarter * 32) << 16;
        const uint32_t tS = tbase + lane_base + C::S_COL + half * 64;
        const uint32_t tP = tbase + lane_base + C::DP_COL + half * 64;
        const int r = quarter * 32 + lane;
        uint8_t* stg = sm + C::OFF_STG + (warp - 4) * 2048;
        uint32_t g = 0;
        int done = 0;
        bool ok = true;
        while (ok) {
            // of the item, what the tiles need; the epilogue looks again
            int n, lim = 0x7fffffff, from = 0, whole_j = 0, two = 0;
            float nlse = -INFINITY, nD = 0.f;
            {
                const PromptBwdItem x = next_item(ok);
                if (!ok || x.Lq < 0 || __any_sync(0xffffffffu, *fail_flag)) break;
                int i0;
                inner(x, i0, n);
                if (KP) {
                    // columns that count of this thread's key: rows from `from` on (in tile 0);
                    // tiles from whole_j on count whole; rows before `two` see one key at
                    // most, and their dS is zero
                    from = (first_row(x.at + r, x.Lq, x.Lk, x.pre) - i0) * p.group;
                    whole_j = (first_row(min(x.at + BM, x.Lk) - 1, x.Lq, x.Lk, x.pre) - i0 + T - 1) / T;
                    two = ((x.Lk > 1 ? first_row(1, x.Lq, x.Lk, x.pre) : x.Lq) - i0) * p.group;
                } else if (r < T * p.group && x.at + r / p.group < x.Lq) {
                    // keys that this thread's row sees; a softmax over one does not move
                    const int i = x.at + r / p.group;
                    const float2 v = row_values(p, x, i, r % p.group);
                    nlse = -v.x;
                    nD = -v.y;
                    lim = keys_seen(i, x.Lq, x.Lk, x.pre);
                    if (lim == 1) lim = 0;
                }
            }
            const int box = T * p.group;
            for (int j = 0; j < n; ++j, ++g) {
                const float* sv = st + g % ST * 256 + half * 64;
                bool whole;  // every score of the tile counts
                if (KP) {
                    whole = j >= whole_j;
                    if (!(ok = __all_sync(0xffffffffu, mbar_wait(&bar[ST_FULL + g % ST], (g / ST) & 1))))
                        break;
                } else {
                    whole = __all_sync(0xffffffffu, lim >= (j + 1) * BM);
                }
                if (!(ok = __all_sync(0xffffffffu, mbar_wait(&bar[S_FULL], g & 1)))) break;
                tc_fence_after();
                uint64_t pr[32];  // P, pairs of columns
                {
                    uint32_t s[2][32];
                    tmem_ld32(tS, s[0]);
                    tmem_ld32(tS + 32, s[1]);
                    tmem_ld_wait_regs(s[0]);
                    tmem_ld_wait_regs(s[1]);
                    const uint64_t c2 = f2_pack(p.scale_log2, p.scale_log2);
#pragma unroll
                    for (int c = 0; c < 2; ++c)
#pragma unroll
                        for (int e = 0; e < 32; e += 4) {
                            float4 l4 = make_float4(nlse, nlse, nlse, nlse);
                            if (KP) l4 = *reinterpret_cast<const float4*>(sv + c * 32 + e);
                            const uint64_t l2[2] = {f2_pack(l4.x, l4.y), f2_pack(l4.z, l4.w)};
#pragma unroll
                            for (int u = 0; u < 2; ++u) {
                                float x0, x1;
                                f2_unpack(f2_fma(f2_pack(__uint_as_float(s[c][e + 2 * u]),
                                                         __uint_as_float(s[c][e + 2 * u + 1])),
                                                 c2, l2[u]),
                                          x0, x1);
                                pr[c * 16 + e / 2 + u] = f2_pack(ex2_approx(x0), ex2_approx(x1));
                            }
                        }
                }
                if (!whole) {
                    // columns that count: [0, hi) of a query, [lo, 64) of a key
                    const int lo = from - j * box - half * 64, hi = lim - j * BM - half * 64;
#pragma unroll
                    for (int e = 0; e < 32; ++e) {
                        float a, b;
                        f2_unpack(pr[e], a, b);
                        if (KP ? 2 * e < lo : 2 * e >= hi) a = 0.f;
                        if (KP ? 2 * e + 1 < lo : 2 * e + 1 >= hi) b = 0.f;
                        pr[e] = f2_pack(a, b);
                    }
                }
                if (KP) {
                    uint32_t pk[32];
#pragma unroll
                    for (int e = 0; e < 32; ++e) {
                        float a, b;
                        f2_unpack(pr[e], a, b);
                        pk[e] = cvt_bf2(a, b);
                    }
                    tmem_st32(tS, pk);
                    tmem_st_wait();
                }
                tc_fence_before();
                __syncwarp();
                if (elect_one()) mbar_arrive(&bar[P_FULL]);
                __syncwarp();
                if (!(ok = __all_sync(0xffffffffu, mbar_wait(&bar[DP_FULL], g & 1)))) break;
                tc_fence_after();
                if (KP && j * box < two) {  // P has gone to dV
                    const int ones = two - j * box - half * 64;
#pragma unroll
                    for (int e = 0; e < 32; ++e) {
                        float a, b;
                        f2_unpack(pr[e], a, b);
                        if (2 * e < ones) a = 0.f;
                        if (2 * e + 1 < ones) b = 0.f;
                        pr[e] = f2_pack(a, b);
                    }
                }
                uint32_t dk[32];
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                    uint32_t d[32];
                    tmem_ld32(tP + c * 32, d);
                    tmem_ld_wait_regs(d);
#pragma unroll
                    for (int e = 0; e < 32; e += 4) {
                        float4 d4 = make_float4(nD, nD, nD, nD);
                        if (KP) d4 = *reinterpret_cast<const float4*>(sv + 128 + c * 32 + e);
                        const uint64_t d2[2] = {f2_pack(d4.x, d4.y), f2_pack(d4.z, d4.w)};
#pragma unroll
                        for (int u = 0; u < 2; ++u) {
                            const uint64_t pp = pr[c * 16 + e / 2 + u];
                            float a, b;
                            f2_unpack(f2_mul(pp, f2_add(f2_pack(__uint_as_float(d[e + 2 * u]),
                                                                __uint_as_float(d[e + 2 * u + 1])),
                                                        d2[u])),
                                      a, b);
                            if (!KP && !whole) {  // V beyond the sequence's keys may be NaN
                                float p0, p1;
                                f2_unpack(pp, p0, p1);
                                if (p0 == 0.f) a = 0.f;
                                if (p1 == 0.f) b = 0.f;
                            }
                            dk[c * 16 + e / 2 + u] = cvt_bf2(a, b);
                        }
                    }
                }
                tmem_st32(tP, dk);
                tmem_st_wait();
                tc_fence_before();
                __syncwarp();
                if (elect_one()) {
                    mbar_arrive(&bar[DS_FULL]);
                    if (KP) mbar_arrive(&bar[ST_EMPTY + g % ST]);
                }
                __syncwarp();
            }
            if (!ok) break;
            // ---- the accumulators out: this warp's half of the columns ----
            if (n > 0) {
                if (!(ok = __all_sync(0xffffffffu, mbar_wait(&bar[ACC_FULL], done & 1)))) break;
                tc_fence_after();
                ++done;
            }
            const PromptBwdItem x = get_item(seen % ITEMS);
            item_done();
            const int tok = r / p.group, hg = r % p.group, key = x.at + r, i = x.at + tok;
            const bool live = KP ? key < x.Lk : tok < T && i < x.Lq;
            const bool in_parts = KP && x.parts(p.group, p.Hkv) > 1;
            float* part = p.part + (long long)x.unit * 2 * BM * HD;
            for (int acc = 0; acc < (KP ? 2 : 1); ++acc) {
                const float f = acc ? 1.f : p.scale;
                const jnx_head_rows& to = !KP ? p.dq : acc ? p.dv : p.dk;
                const long long o = !live ? -1
                                    : KP  ? (x.k0 + key) * to.row_stride + x.kvh * to.head_stride
                                          : (x.q0 + i) * to.row_stride + (x.kvh * p.group + hg) * to.head_stride;
                // (a tile taken in parts: its sums' rows)
                const long long po = live ? r * HD : -1;
                // this lane's row's four units into the warp's staging, out unit lane % 4 of
                // rows lane / 4 + 8 u
                long long at[4], pat[4];
#pragma unroll
                for (int u = 0; u < 4; ++u) {
                    at[u] = __shfl_sync(0xffffffffu, o, 8 * u + (lane >> 2));
                    if (KP) pat[u] = __shfl_sync(0xffffffffu, po, 8 * u + (lane >> 2));
                }
#pragma unroll 1
                for (int c = 0; c < HD / 64; ++c) {
                    const int col = half * (HD / 2) + c * 32;
                    uint32_t v[32];
                    if (n > 0) {
                        tmem_ld32(tbase + lane_base + C::ACC_COL + acc * HD + col, v);
                        tmem_ld_wait_regs(v);
                    } else {
#pragma unroll
                        for (int e = 0; e < 32; ++e) v[e] = 0;
                    }
                    if (in_parts)
                        bwd_rows_part(stg, lane, v, part + acc * BM * HD + col, pat);
                    else
                        bwd_rows_out(stg, lane, v, f, to.ptr + col, at);
                }
            }
            if (n > 0) {
                tc_fence_before();
                __syncwarp();
                if (elect_one()) mbar_arrive(&bar[ACC_FREE]);
                __syncwarp();
            }
        }
        if (!ok) *fail_flag = 1;
    }
    return claim;
}

template <int HD>
__global__ void __launch_bounds__(pbwd::THREADS, 1)
    k_prompt_attn_bwd(const __grid_constant__ CUtensorMap tq, const __grid_constant__ CUtensorMap tk,
                      const __grid_constant__ CUtensorMap tv, const __grid_constant__ CUtensorMap tdo,
                      const __grid_constant__ PromptBwdArgs p) {
    using C = PromptBwdCfg<HD>;
    using namespace pbwd;
    extern __shared__ uint8_t smem_raw[];
    uint8_t* sm = reinterpret_cast<uint8_t*>(
        (reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
    uint64_t* bar = reinterpret_cast<uint64_t*>(sm + C::OFF_BAR);
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(bar + 2 * N_BARS);
    volatile int* fail_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
    const int warp = warp_uniform(threadIdx.x >> 5);
    if (threadIdx.x == 0) {
        for (int k = 0; k < 2 * N_BARS; ++k) {
            const int i = k % N_BARS;
            mbar_init(&bar[k], i == P_FULL || i == DS_FULL || i == ACC_FREE ? EW
                               : i >= ST_EMPTY && i < W_FULL                ? EW
                               : i >= ST_FULL && i < ST_EMPTY               ? 32
                               : i >= W_EMPTY                               ? READERS
                                                                            : 1);
        }
        *fail_flag = 0;
        fence_barrier_init();
    }
    // rows that no box reaches (128 no multiple of the group) are zero for good
    const int box = p.group * tile_tokens(p.group);
    for (int i = threadIdx.x; i < 2 * C::SLOTS * (HD / 64) * (BM - box) * 8; i += THREADS) {
        const int u = i & 7, r = box + (i >> 3) % (BM - box), t = (i >> 3) / (BM - box);
        *reinterpret_cast<uint4*>(sm + C::OFF_B1 + t * BM * 128 + r * 128 + u * 16) =
            make_uint4(0, 0, 0, 0);
    }
    fence_proxy_async();
    pdl_entry();  // TMEM is taken once the grid ahead has given its own back
    if (warp == 1) {
        tmem_alloc(tmem_slot, 512);
        tmem_relinquish();
    }
    if (threadIdx.x == 0) {
        tma_prefetch_desc(&tq);
        tma_prefetch_desc(&tk);
        tma_prefetch_desc(&tv);
        tma_prefetch_desc(&tdo);
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tbase = warp_uniform(*tmem_slot);
    // a pass leaves no copy, MMA or TMEM read of its own behind; its barriers are its own
    int claim = prompt_bwd_pass<HD, KEYS>(tq, tk, tv, tdo, p, sm, bar, fail_flag, tbase, 0, blockIdx.x);
    __syncwarp();
    tc_fence_before();
    bool failed = __syncthreads_or(*fail_flag);
    tc_fence_after();
    if (!failed) {
        prompt_bwd_pass<HD, QUERIES>(tq, tk, tv, tdo, p, sm, bar + N_BARS, fail_flag, tbase,
                                     p.n_keys * p.Hkv, claim);
        __syncwarp();
        tc_fence_before();
        failed = __syncthreads_or(*fail_flag);
        tc_fence_after();
    }
    if (failed && threadIdx.x == 0) report(p.status, JNX_ERR_TIMEOUT);
    if (warp == 1) tmem_dealloc(tbase, 512);
}

template <int HD>
static jnx_status launch_prompt_bwd(const PromptBwdArgs& a, const jnx_head_rows& q,
                                    const jnx_head_rows& k, const jnx_head_rows& v,
                                    const jnx_head_rows& dout, int rows, int keys, cudaStream_t s) {
    using C = PromptBwdCfg<HD>;
    const char* what = "prompt attention backward";
    static std::atomic<uint64_t> attr{0};
    if (set_smem_limit(reinterpret_cast<const void*>(k_prompt_attn_bwd<HD>), C::SMEM, attr) != cudaSuccess)
        return fail(JNX_ERR_CUDA, "%s: smem attribute", what);
    CUtensorMap tq, tk, tv, tdo;
    const int T = tile_tokens(a.group);
    if (!make_tmap_heads(&tq, q, rows, a.H, HD, a.group, T) ||
        !make_tmap_heads(&tdo, dout, rows, a.H, HD, a.group, T) ||
        !make_tmap_heads(&tk, k, keys, a.Hkv, HD, 1, pbwd::BM) ||
        !make_tmap_heads(&tv, v, keys, a.Hkv, HD, 1, pbwd::BM))
        return fail(JNX_ERR_CUDA, "%s: tensor map encode failed", what);
    const int grid = (int)std::min<long long>((long long)(a.n_keys + a.n_queries) * a.Hkv, num_sms());
    pdl(k_prompt_attn_bwd<HD>, grid, pbwd::THREADS, C::SMEM, s)(tq, tk, tv, tdo, a);
    return launched(what);
}

// ---------------------------------------------------------------------------
// Head dim 256.  An accumulator is 256 columns, so the keys' pass is two, dK then dV, and
// the outer tiles take 64 KB of shared memory each.  The inner operand that a score and a
// sum both read, or the sum alone, has one 64 KB slot, released in halves as the sum's two
// products of 128 columns are through with them; the other streams through 16 KB units,
// 64 columns of a tile.
//   DK   S^T = K Q^T, dP^T = V dO^T, dK += dS^T Q       slot Q, units of dO
//   DV   S^T = K Q^T, dV += P^T dO                      slot dO, units of Q
//   DQ   S = Q K^T, dP = dO V^T, dQ += dS K             slot K, units of V
// DK and DQ: S, dP and the accumulator fill TMEM; dP is read first, and the next one runs
// while dS is formed, over S; then the sum and the next S.  DV: two S, issued two tiles
// ahead.  (Tiles of 64 inner rows, double-buffered, left the tensor core at half:
// a product of 128 x 64 x 16 from shared memory takes 48 clocks and one of 128 x 128 x 16
// takes 64, 128 bytes a clock of operands either way.)
// 26 samples of up to 840 tokens, 8 heads on one of 256 (108 GFLOP with the forward): 160 us
// the passes and 12 the parts' sums, 241 with the forward's 46 and the rows' values.  Eight
// products for the gradients' five, and the tensor core busy for 37 %: an item is a few tiles,
// and its first loads, its last products and its sums out are nobody's company, there being
// neither TMEM nor shared memory for a second item.
// ---------------------------------------------------------------------------
namespace pwide {
constexpr int BM = 128, HD = 256, NCH = 4;
enum { DK = 0, DV = 1, DQ = 2 };
constexpr int TILE = BM * HD * 2, UNIT = BM * 128;
// shared memory: DK, DQ: two outer tiles, the slot, 2 units; DV: one, 6 units, the slot
constexpr int OFF_ST = 3 * TILE + 2 * UNIT;  // -lse, -D [2][128]; DV: two slots of -lse
constexpr int OFF_BAR = OFF_ST + 2 * BM * 4;
// barriers of a pass
enum { O_FULL = 0, O_EMPTY = 1, H_FULL = 2, H_EMPTY = 4, U_FULL = 6, U_EMPTY = 12, S_FULL = 18,
       P_FULL = 20, ACC_FULL = 22, ACC_FREE = 23, DRAIN = 24, ST_FULL = 25, ST_EMPTY = 27, W_FULL = 29,
       W_EMPTY = 31, DP_READ = 33, N_BARS = 34 };
constexpr int SMEM = OFF_BAR + N_BARS * 8 + 80 + 1024;
static_assert(SMEM <= 227 * 1024, "shared memory per CTA");
constexpr int THREADS = 384, EW = 8, READERS = 2 + EW;
constexpr uint32_t S_COL = 0, DP_COL = 128, ACC_COL = 256;
}  // namespace pwide

// Four 16-byte units of each lane's row, turned over among lanes 4 k .. 4 k + 3: unit j of
// lane l becomes unit l % 4 of row 4 (l / 4) + j, so that a store of unit j covers 64 bytes of
// each of eight rows (16 bytes of 32 rows took a cycle a row: 8,400 clocks an item).
__device__ __forceinline__ void turn_units(uint4 (&u)[4], int lane) {
#pragma unroll
    for (int b = 1; b < 4; b <<= 1)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (i & b) continue;
            const bool up = lane & b;
            uint4 t = up ? u[i] : u[i | b];
            t.x = __shfl_xor_sync(0xffffffffu, t.x, b);
            t.y = __shfl_xor_sync(0xffffffffu, t.y, b);
            t.z = __shfl_xor_sync(0xffffffffu, t.z, b);
            t.w = __shfl_xor_sync(0xffffffffu, t.w, b);
            if (up) u[i] = t;
            else u[i | b] = t;
        }
}

template <int PASS>
__device__ __forceinline__ int prompt_bwd_wide_pass(const CUtensorMap& tq, const CUtensorMap& tk,
                                                    const CUtensorMap& tv, const CUtensorMap& tdo,
                                                    const PromptBwdArgs& p, uint8_t* sm, uint64_t* bar,
                                                    volatile int* fail_flag, uint32_t tbase,
                                                    int q_first, int claim) {
    using namespace pwide;
    constexpr bool KP = PASS != DQ, NEED_DP = PASS != DV;
    constexpr int NUNIT = NEED_DP ? 2 : 6, NST = NEED_DP ? 1 : 2;
    const int T = tile_tokens(p.group);
    const int warp = warp_uniform(threadIdx.x >> 5), lane = threadIdx.x & 31;
    uint8_t* sl = sm + (NEED_DP ? 2 * TILE : TILE + 6 * UNIT);
    uint8_t* un = sm + (NEED_DP ? 3 * TILE : TILE);
    float* st = reinterpret_cast<float*>(sm + OFF_ST);
    volatile int* slot = fail_flag + 1;  // [2][9]: items handed out
    const int2* items = p.items + (KP ? 0 : p.n_keys);
    const int n_work = (KP ? p.n_keys : p.n_queries) * p.Hkv;

    int seen = 0;
    auto next_item = [&](bool& ok) -> PromptBwdItem {
        const int b = seen & 1;
        PromptBwdItem x{0, 0, 0, -1, 0, 0, 0, 0, 0};
        if (!(ok = mbar_wait_warp(&bar[W_FULL + b], (seen >> 1) & 1))) return x;
        x.at = warp_uniform(slot[9 * b]);
        x.kvh = warp_uniform(slot[9 * b + 1]);
        x.q0 = warp_uniform(slot[9 * b + 2]);
        x.Lq = warp_uniform(slot[9 * b + 3]);
        x.k0 = warp_uniform(slot[9 * b + 4]);
        x.Lk = warp_uniform(slot[9 * b + 5]);
        x.pre = warp_uniform(slot[9 * b + 6]);
        x.part = warp_uniform(slot[9 * b + 7]);
        x.unit = warp_uniform(slot[9 * b + 8]);
        if (elect_one()) mbar_arrive(&bar[W_EMPTY + b]);
        __syncwarp();
        ++seen;
        return x;
    };
    // an item's inner tiles, and the keys' passes' first inner row
    auto inner = [&](const PromptBwdItem& x, int& i0, int& n) {
        if (KP) {
            x.range(p.group, p.Hkv, T, i0, n);
        } else {
            i0 = x.at;
            n = (keys_seen(min(x.at + T, x.Lq) - 1, x.Lq, x.Lk, x.pre) + BM - 1) / BM;
        }
    };

    if (warp == 0) {
        // ---------------- claims and TMA ----------------
        bool ok = true;
        int told = 0;
        auto tell = [&](const PromptBwdItem& x) {
            const int b = told & 1;
            if (!mbar_wait_warp(&bar[W_EMPTY + b], ((told >> 1) & 1) ^ 1)) return false;
            if (elect_one()) {
                slot[9 * b] = x.at;
                slot[9 * b + 1] = x.kvh;
                slot[9 * b + 2] = x.q0;
                slot[9 * b + 3] = x.Lq;
                slot[9 * b + 4] = x.k0;
                slot[9 * b + 5] = x.Lk;
                slot[9 * b + 6] = x.pre;
                slot[9 * b + 7] = x.part;
                slot[9 * b + 8] = x.unit;
                mbar_arrive(&bar[W_FULL + b]);
            }
            __syncwarp();
            ++told;
            return true;
        };
        int no = 0;             // outer tiles loaded
        uint32_t g = 0, u = 0;  // slot tiles, units loaded
        PromptBwdItem nx{0, 0, 0, 0, 0, 0, 0, 0, 0};
        auto fetch = [&]() {
            for (;;) {
                claim = __shfl_sync(0xffffffffu, claim, 0);
                const int w = claim - q_first;
                if (w >= n_work || bwd_item<KP>(p, items[w / p.Hkv], w, nx)) return;
                if (lane == 0) claim = (int)gridDim.x + atomicAdd(p.claimed, 1);
            }
        };
        const uint32_t row_bytes = p.group * T * 128;  // of 64 columns of a row tile
        fetch();
        while (claim - q_first < n_work) {
            if (__any_sync(0xffffffffu, *fail_flag)) {
                ok = false;
                break;
            }
            PromptBwdItem x;
            x.at = warp_uniform(nx.at);
            x.kvh = warp_uniform(nx.kvh);
            x.q0 = warp_uniform(nx.q0);
            x.Lq = warp_uniform(nx.Lq);
            x.k0 = warp_uniform(nx.k0);
            x.Lk = warp_uniform(nx.Lk);
            x.pre = warp_uniform(nx.pre);
            x.part = warp_uniform(nx.part);
            x.unit = warp_uniform(nx.unit);
            if (lane == 0) claim = (int)gridDim.x + atomicAdd(p.claimed, 1);
            __syncwarp();
            if (!(ok = tell(x))) break;
            int i0, n;
            inner(x, i0, n);
            const int qh = x.kvh * p.group;
            // columns [64 c, 64 c + 64) of inner tile j: of rows (m = Q or dO) or keys (K or V)
            auto rows_in = [&](const CUtensorMap* m, uint8_t* dst, int c, int j, uint64_t* full) {
                tma_load_3d(dst, m, c * 64, qh, x.q0 + i0 + j * T, full);
            };
            auto keys_in = [&](const CUtensorMap* m, uint8_t* dst, int c, int j, uint64_t* full) {
                tma_load_3d(dst, m, c * 64, x.kvh, x.k0 + j * BM, full);
            };
            auto load_slot = [&](int j) -> bool {
                for (int h = 0; h < 2; ++h) {
                    if (!mbar_wait_warp(&bar[H_EMPTY + h], (g & 1) ^ 1)) return false;
                    if (elect_one()) {
                        uint64_t* full = &bar[H_FULL + h];
                        mbar_arrive_expect_tx(full, KP ? 2 * row_bytes : 2 * UNIT);
#pragma unroll
                        for (int k = 0; k < 2; ++k) {
                            const int c = 2 * h + k;
                            if (PASS == DQ) keys_in(&tk, sl + c * UNIT, c, j, full);
                            else rows_in(PASS == DK ? &tq : &tdo, sl + c * UNIT, c, j, full);
                        }
                    }
                    __syncwarp();
                }
                ++g;
                return true;
            };
            auto load_units = [&](int j, int c0, int c1) -> bool {
                for (int c = c0; c < c1; ++c, ++u) {
                    const int b = u % NUNIT;
                    if (!mbar_wait_warp(&bar[U_EMPTY + b], ((u / NUNIT) & 1) ^ 1)) return false;
                    if (elect_one()) {
                        mbar_arrive_expect_tx(&bar[U_FULL + b], KP ? row_bytes : UNIT);
                        if (PASS == DQ) keys_in(&tv, un + b * UNIT, c, j, &bar[U_FULL + b]);
                        else rows_in(PASS == DK ? &tdo : &tq, un + b * UNIT, c, j, &bar[U_FULL + b]);
                    }
                    __syncwarp();
                }
                return true;
            };
            if (n > 0) {
                if (no > 0 && !(ok = mbar_wait_warp(&bar[O_EMPTY], (no - 1) & 1))) break;
                if (elect_one()) {
                    mbar_arrive_expect_tx(&bar[O_FULL], PASS == DK   ? 2 * TILE
                                                        : PASS == DV ? TILE
                                                                     : 8 * row_bytes);
#pragma unroll
                    for (int c = 0; c < NCH; ++c) {
                        if (KP) {
                            tma_load_3d(sm + c * UNIT, &tk, c * 64, x.kvh, x.k0 + x.at, &bar[O_FULL]);
                            if (NEED_DP)
                                tma_load_3d(sm + TILE + c * UNIT, &tv, c * 64, x.kvh, x.k0 + x.at,
                                            &bar[O_FULL]);
                        } else {
                            tma_load_3d(sm + c * UNIT, &tq, c * 64, qh, x.q0 + x.at, &bar[O_FULL]);
                            tma_load_3d(sm + TILE + c * UNIT, &tdo, c * 64, qh, x.q0 + x.at, &bar[O_FULL]);
                        }
                    }
                }
                __syncwarp();
                ++no;
            }
            // in the order the MMAs take them: DV's scores run two tiles ahead
            if (PASS == DV) {
                for (int j = 0; j < 2 && j < n && ok; ++j) ok = load_units(j, 0, NCH);
                for (int j = 0; j < n && ok; ++j) {
                    ok = load_slot(j);
                    if (ok && j + 2 < n) ok = load_units(j + 2, 0, NCH);
                }
            } else {
                ok = n == 0 || (load_units(0, 0, NUNIT) && load_slot(0) && load_units(0, NUNIT, NCH));
                for (int j = 1; j < n && ok; ++j) ok = load_units(j, 0, NCH) && load_slot(j);
            }
            if (!ok) break;
            fetch();
        }
        ok = ok && tell(PromptBwdItem{0, 0, 0, -1, 0, 0, 0, 0, 0});
        if (!ok) *fail_flag = 1;
        // every copy has landed, and every release has arrived, before the barriers are made anew
        if (no > 0) {
            mbar_wait_warp(&bar[O_FULL], (no - 1) & 1, 100000000LL);
            mbar_wait_warp(&bar[O_EMPTY], (no - 1) & 1, 100000000LL);
        }
        for (int h = 0; h < 2 && g > 0; ++h) {
            mbar_wait_warp(&bar[H_FULL + h], (g - 1) & 1, 100000000LL);
            mbar_wait_warp(&bar[H_EMPTY + h], (g - 1) & 1, 100000000LL);
        }
        for (uint32_t i = u > NUNIT ? u - NUNIT : 0; i < u; ++i) {
            mbar_wait_warp(&bar[U_FULL + i % NUNIT], (i / NUNIT) & 1, 100000000LL);
            mbar_wait_warp(&bar[U_EMPTY + i % NUNIT], (i / NUNIT) & 1, 100000000LL);
        }
    } else if (warp == 1) {
        // ---------------- MMA issuer ----------------
        constexpr uint32_t IDESC_S = idesc_bf16_f32(BM, BM);
        constexpr uint32_t IDESC_ACC = idesc_bf16_f32(BM, 128) | (1u << 16);  // B MN-major
        bool ok = true, issued = false;
        int no = 0, done = 0;
        uint32_t g = 0, u = 0, gs = 0, gp = 0;  // slot tiles, units, scores, P / dS taken
        const uint32_t o1 = smem_u32(sm), o2 = o1 + TILE;
        auto commit = [&](uint64_t* b) {
            if (elect_one()) tc_commit(b);
            __syncwarp();
        };
        // 64 columns of the contraction: chunk c of the outer tile at o with the inner's at b
        auto score = [&](uint32_t d, uint32_t o, int c, uint8_t* b) {
            const uint32_t a_lo = sw128_desc_lo(o + c * UNIT), b_lo = sw128_desc_lo(smem_u32(b));
            if (elect_one()) {
#pragma unroll
                for (int ks = 0; ks < 4; ++ks)
                    tc_mma_f16(d, desc_of(a_lo + 2 * ks, kSw128DescHi), desc_of(b_lo + 2 * ks, kSw128DescHi),
                               IDESC_S, (c | ks) != 0);
            }
            __syncwarp();
            issued = true;
        };
        auto zero_tail = [&](uint8_t* chunk, int valid, int end) {
            for (int i = lane; i < (end - valid) * 8; i += 32)
                *reinterpret_cast<uint4*>(chunk + (valid + (i >> 3)) * 128 + (i & 7) * 16) =
                    make_uint4(0, 0, 0, 0);
            fence_proxy_async();
            __syncwarp();
        };
        while (ok) {
            const PromptBwdItem x = next_item(ok);
            if (!ok || x.Lq < 0 || __any_sync(0xffffffffu, *fail_flag)) break;
            int i0, n;
            inner(x, i0, n);
            if (n == 0) continue;
            if (!(ok = mbar_wait_warp(&bar[O_FULL], no & 1))) break;
            ++no;
            const int box = KP ? p.group * T : BM;
            auto valid = [&](int j) {
                return KP ? min(T, x.Lq - i0 - j * T) * p.group : min(BM, x.Lk - j * BM);
            };
            // the slot's half h of tile j is there
            auto wait_half = [&](int h, int j) -> bool {
                if (!mbar_wait_warp(&bar[H_FULL + h], g & 1)) return false;
                if (valid(j) < box)
                    for (int k = 0; k < 2; ++k) zero_tail(sl + (2 * h + k) * UNIT, valid(j), box);
                tc_fence_after();
                return true;
            };
            auto from_units = [&](uint32_t d, uint32_t o, int j) -> bool {
                for (int c = 0; c < NCH; ++c, ++u) {
                    const int b = u % NUNIT;
                    if (!mbar_wait_warp(&bar[U_FULL + b], (u / NUNIT) & 1)) return false;
                    if (KP && valid(j) < box) zero_tail(un + b * UNIT, valid(j), box);
                    tc_fence_after();
                    score(d, o, c, un + b * UNIT);
                    commit(&bar[U_EMPTY + b]);
                }
                return true;
            };
            auto next_scores = [&](int j) -> bool {
                if constexpr (NEED_DP) {
                    for (int h = 0; h < 2; ++h) {
                        if (!wait_half(h, j)) return false;
                        for (int k = 0; k < 2; ++k)
                            score(tbase + S_COL, o1, 2 * h + k, sl + (2 * h + k) * UNIT);
                    }
                    commit(&bar[S_FULL]);
                } else {
                    if (!from_units(tbase + S_COL + (gs & 1) * BM, o1, j)) return false;
                    commit(&bar[S_FULL + (gs & 1)]);
                }
                ++gs;
                if (j + 1 == n) commit(&bar[O_EMPTY]);
                return true;
            };
            // acc += X B over the slot's 128 rows, X bf16 in TMEM: 64 rows at column xc, 64 at
            // xc + 64
            auto gather = [&](int h, uint32_t xc, bool accumulate) {
                const uint32_t b_lo = sw128_desc_mn_lo(smem_u32(sl + 2 * h * UNIT), UNIT);
                if (elect_one()) {
#pragma unroll
                    for (int ks = 0; ks < BM / 16; ++ks)
                        tc_mma_f16_ts(tbase + ACC_COL + h * 128, xc + (ks >> 2) * 64 + (ks & 3) * 8,
                                      desc_of(b_lo + ks * 128, kSw128DescHi), IDESC_ACC,
                                      accumulate || ks > 0);
                    tc_commit(&bar[H_EMPTY + h]);
                }
                __syncwarp();
            };
            if (NEED_DP && !(ok = from_units(tbase + DP_COL, o2, 0))) break;
            ok = next_scores(0) && (NEED_DP || n < 2 || next_scores(1));
            for (int j = 0; j < n && ok; ++j, ++gp, ++g) {
                const uint32_t b = NEED_DP ? 0 : gp & 1, ph = NEED_DP ? gp & 1 : (gp >> 1) & 1;
                if (PASS == DV && !(ok = wait_half(0, j) && wait_half(1, j))) break;
                // the next dP, while dS is formed of this one, which has been read
                if (NEED_DP && j + 1 < n &&
                    !(ok = mbar_wait_warp(&bar[DP_READ], gp & 1) && from_units(tbase + DP_COL, o2, j + 1)))
                    break;
                if (!(ok = mbar_wait_warp(&bar[P_FULL + b], ph))) break;
                // the item's first product overwrites the sums: the last epilogue has read them
                if (j == 0 && done > 0 && !(ok = mbar_wait_warp(&bar[ACC_FREE], (done - 1) & 1))) break;
                tc_fence_after();
                for (int h = 0; h < 2; ++h) gather(h, tbase + S_COL + b * BM, j > 0);
                if (NEED_DP) {
                    if (j + 1 < n) {
                        ++g;
                        ok = next_scores(j + 1);
                        --g;
                    }
                } else if (j + 2 < n) {
                    ok = next_scores(j + 2);
                }
            }
            if (!ok) break;
            commit(&bar[ACC_FULL]);
            ++done;
        }
        if (!ok) *fail_flag = 1;
        if (issued) {
            commit(&bar[DRAIN]);
            mbar_wait_warp(&bar[DRAIN], 0, 100000000LL);
        }
    } else if (warp == 2) {
        // ---------------- values of the inner rows (keys' passes) ----------------
        bool ok = true;
        uint32_t g = 0;
        while (ok) {
            const PromptBwdItem x = next_item(ok);
            if (!ok || x.Lq < 0 || __any_sync(0xffffffffu, *fail_flag)) break;
            if (!KP) continue;
            int i0, n;
            inner(x, i0, n);
            for (int j = 0; j < n; ++j, ++g) {
                const int b = g % NST;
                float2 v[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int r = e * 32 + lane, t = r / p.group, i = i0 + j * T + t;
                    const bool live = t < T && i < x.Lq;
                    v[e] = live ? row_values(p, x, i, r - t * p.group) : make_float2(INFINITY, 0.f);
                }
                if (!(ok = mbar_wait_warp(&bar[ST_EMPTY + b], ((g / NST) & 1) ^ 1))) break;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    st[b * 128 + e * 32 + lane] = -v[e].x;
                    if (NEED_DP) st[128 + e * 32 + lane] = -v[e].y;
                }
                mbar_arrive(&bar[ST_FULL + b]);
            }
        }
        if (!ok) *fail_flag = 1;
    } else if (warp >= 4) {
        // ---------------- elementwise + epilogue ----------------
        const int quarter = warp & 3, half = (warp - 4) >> 2;
        const uint32_t lane_base = (uint32_t)(quarter * 32) << 16;
        const int r = quarter * 32 + lane;
        uint32_t g = 0;
        int done = 0;
        bool ok = true;
        while (ok) {
            const PromptBwdItem x = next_item(ok);
            if (!ok || x.Lq < 0 || __any_sync(0xffffffffu, *fail_flag)) break;
            int i0, n;
            inner(x, i0, n);
            const int tok = r / p.group, hg = r % p.group;
            const int key = x.at + r, i = x.at + tok;
            const bool live = KP ? key < x.Lk : tok < T && i < x.Lq;
            float nlse = -INFINITY, nD = 0.f;
            // what counts of an outer row: a query's keys below lim, a key's rows from `from` on
            int lim = 0x7fffffff;
            // (DK: rows that see one key at most have no dS)
            const int two = PASS == DK ? (x.Lk > 1 ? first_row(1, x.Lq, x.Lk, x.pre) : x.Lq) : 0;
            const int from = KP ? (max(first_row(key, x.Lq, x.Lk, x.pre), two) - i0) * p.group : 0;
            if (!KP && live) {
                const float2 v = row_values(p, x, i, hg);
                nlse = -v.x;
                nD = -v.y;
                lim = keys_seen(i, x.Lq, x.Lk, x.pre);
                if (lim == 1) lim = 0;  // a softmax over one key does not move
            }
            for (int j = 0; j < n; ++j, ++g) {
                const uint32_t b = NEED_DP ? 0 : g & 1, ph = NEED_DP ? g & 1 : (g >> 1) & 1;
                const float* sv = st + (NEED_DP ? 0 : b * 128) + half * 64;
                const uint32_t tS = tbase + lane_base + S_COL + b * BM + half * 64;
                const uint32_t tP = tbase + lane_base + DP_COL + half * 64;
                bool whole;
                if (KP) {
                    whole = i0 + j * T >= two && keys_seen(min(i0 + j * T, x.Lq - 1), x.Lq, x.Lk, x.pre) >=
                                                     min(x.at + BM, x.Lk);
                    if (!(ok = __all_sync(0xffffffffu, mbar_wait(&bar[ST_FULL + b], ph)))) break;
                } else {
                    whole = __all_sync(0xffffffffu, lim >= (j + 1) * BM);
                }
                if (!(ok = __all_sync(0xffffffffu, mbar_wait(&bar[S_FULL + b], ph)))) break;
                tc_fence_after();
                const uint64_t c2 = f2_pack(p.scale_log2, p.scale_log2);
                uint32_t pk[32], dp[2][32];
                if (NEED_DP) {
                    tmem_ld32(tP, dp[0]);
                    tmem_ld32(tP + 32, dp[1]);
                    tmem_ld_wait_regs(dp[0]);
                    tmem_ld_wait_regs(dp[1]);
                    tc_fence_before();
                    __syncwarp();
                    if (elect_one()) mbar_arrive(&bar[DP_READ]);
                    __syncwarp();
                }
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                    uint32_t s[32];
                    uint32_t(&d)[32] = dp[c];
                    tmem_ld32(tS + c * 32, s);
                    tmem_ld_wait_regs(s);
                    // columns that count: [0, hi) of a query, [lo, 32) of a key
                    const int lo = from - j * T * p.group - half * 64 - c * 32;
                    const int hi = lim - j * BM - half * 64 - c * 32;
#pragma unroll
                    for (int e = 0; e < 32; e += 4) {
                        float4 l4 = make_float4(nlse, nlse, nlse, nlse), d4 = make_float4(nD, nD, nD, nD);
                        if (KP) {
                            l4 = *reinterpret_cast<const float4*>(sv + c * 32 + e);
                            if (NEED_DP) d4 = *reinterpret_cast<const float4*>(sv + 128 + c * 32 + e);
                        }
                        const uint64_t l2[2] = {f2_pack(l4.x, l4.y), f2_pack(l4.z, l4.w)};
                        const uint64_t d2[2] = {f2_pack(d4.x, d4.y), f2_pack(d4.z, d4.w)};
#pragma unroll
                        for (int w = 0; w < 2; ++w) {
                            const int k = e + 2 * w;
                            float a0, a1;
                            f2_unpack(f2_fma(f2_pack(__uint_as_float(s[k]), __uint_as_float(s[k + 1])), c2,
                                             l2[w]),
                                      a0, a1);
                            a0 = ex2_approx(a0);
                            a1 = ex2_approx(a1);
                            if (NEED_DP)
                                f2_unpack(f2_mul(f2_pack(a0, a1),
                                                 f2_add(f2_pack(__uint_as_float(d[k]),
                                                                __uint_as_float(d[k + 1])),
                                                        d2[w])),
                                          a0, a1);
                            if (!whole) {
                                if (KP ? k < lo : k >= hi) a0 = 0.f;
                                if (KP ? k + 1 < lo : k + 1 >= hi) a1 = 0.f;
                            }
                            pk[c * 16 + k / 2] = cvt_bf2(a0, a1);
                        }
                    }
                }
                tmem_st32(tS, pk);
                tmem_st_wait();
                tc_fence_before();
                __syncwarp();
                if (elect_one()) {
                    mbar_arrive(&bar[P_FULL + b]);
                    if (KP) mbar_arrive(&bar[ST_EMPTY + b]);
                }
                __syncwarp();
            }
            if (!ok) break;
            if (n > 0) {
                if (!(ok = __all_sync(0xffffffffu, mbar_wait(&bar[ACC_FULL], done & 1)))) break;
                tc_fence_after();
                ++done;
            }
            const float f = PASS == DV ? 1.f : p.scale;
            const jnx_head_rows& to = PASS == DQ ? p.dq : PASS == DV ? p.dv : p.dk;
            // a tile taken in parts: its sums' row
            const bool in_parts = KP && x.parts(p.group, p.Hkv) > 1;
            float* part = p.part + ((long long)x.unit * 2 + (PASS == DV)) * BM * HD;
            const long long row = !live      ? -1
                                  : in_parts ? r * HD
                                  : KP       ? (x.k0 + key) * to.row_stride + x.kvh * to.head_stride
                                             : (x.q0 + i) * to.row_stride +
                                                   (x.kvh * p.group + hg) * to.head_stride;
            long long at[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) at[k] = __shfl_sync(0xffffffffu, row, (lane & ~3) + k);
#pragma unroll 1
            for (int c = 0; c < HD / 64; ++c) {
                const int col = half * (HD / 2) + c * 32;
                uint32_t v[32];
                if (n > 0) {
                    tmem_ld32(tbase + lane_base + ACC_COL + col, v);
                    tmem_ld_wait_regs(v);
                } else {
#pragma unroll
                    for (int e = 0; e < 32; ++e) v[e] = 0;
                }
                uint4 u[4];
                if (in_parts) {
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            u[e] = make_uint4(v[16 * h + 4 * e], v[16 * h + 4 * e + 1],
                                              v[16 * h + 4 * e + 2], v[16 * h + 4 * e + 3]);
                        turn_units(u, lane);
#pragma unroll
                        for (int k = 0; k < 4; ++k)
                            if (at[k] >= 0)
                                *reinterpret_cast<uint4*>(part + at[k] + col + 16 * h + (lane & 3) * 4) = u[k];
                    }
                } else {
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        u[e] = make_uint4(
                            cvt_bf2(f * __uint_as_float(v[8 * e]), f * __uint_as_float(v[8 * e + 1])),
                            cvt_bf2(f * __uint_as_float(v[8 * e + 2]), f * __uint_as_float(v[8 * e + 3])),
                            cvt_bf2(f * __uint_as_float(v[8 * e + 4]), f * __uint_as_float(v[8 * e + 5])),
                            cvt_bf2(f * __uint_as_float(v[8 * e + 6]), f * __uint_as_float(v[8 * e + 7])));
                    turn_units(u, lane);
#pragma unroll
                    for (int k = 0; k < 4; ++k)
                        if (at[k] >= 0)
                            *reinterpret_cast<uint4*>(to.ptr + at[k] + col + (lane & 3) * 8) = u[k];
                }
            }
            if (n > 0) {
                tc_fence_before();
                __syncwarp();
                if (elect_one()) mbar_arrive(&bar[ACC_FREE]);
                __syncwarp();
            }
        }
        if (!ok) *fail_flag = 1;
    }
    return claim;
}

__global__ void __launch_bounds__(pwide::THREADS, 1)
    k_prompt_attn_bwd_wide(const __grid_constant__ CUtensorMap tq, const __grid_constant__ CUtensorMap tk,
                           const __grid_constant__ CUtensorMap tv, const __grid_constant__ CUtensorMap tdo,
                           const __grid_constant__ PromptBwdArgs p) {
    using namespace pwide;
    extern __shared__ uint8_t smem_raw[];
    uint8_t* sm = reinterpret_cast<uint8_t*>(
        (reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
    uint64_t* bar = reinterpret_cast<uint64_t*>(sm + OFF_BAR);
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(bar + N_BARS);
    volatile int* fail_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
    const int warp = warp_uniform(threadIdx.x >> 5);
    auto init_bars = [&](bool again) {
        if (threadIdx.x == 0) {
            for (int i = 0; i < N_BARS; ++i) {
                if (again) mbar_inval(&bar[i]);
                mbar_init(&bar[i], i == P_FULL || i == P_FULL + 1 || i == ACC_FREE ? EW
                                   : i >= ST_EMPTY && i < W_FULL                   ? EW
                                   : i >= ST_FULL && i < ST_EMPTY                  ? 32
                                   : i >= W_EMPTY && i < DP_READ                   ? READERS
                                   : i == DP_READ                                  ? EW
                                                                                   : 1);
            }
            fence_barrier_init();
        }
    };
    // inner rows that no box reaches (128 no multiple of the group) are zero in the keys'
    // passes
    const int box = p.group * tile_tokens(p.group);
    auto zero_rows = [&](uint8_t* at, int chunks) {
        for (int i = threadIdx.x; i < chunks * (BM - box) * 8; i += THREADS) {
            const int u = i & 7, r = box + (i >> 3) % (BM - box), t = (i >> 3) / (BM - box);
            *reinterpret_cast<uint4*>(at + t * UNIT + r * 128 + u * 16) = make_uint4(0, 0, 0, 0);
        }
        fence_proxy_async();
    };
    init_bars(false);
    if (threadIdx.x == 0) *fail_flag = 0;
    zero_rows(sm + 2 * TILE, NCH + 2);
    pdl_entry();  // TMEM is taken once the grid ahead has given its own back
    if (warp == 1) {
        tmem_alloc(tmem_slot, 512);
        tmem_relinquish();
    }
    if (threadIdx.x == 0) {
        tma_prefetch_desc(&tq);
        tma_prefetch_desc(&tk);
        tma_prefetch_desc(&tv);
        tma_prefetch_desc(&tdo);
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tbase = warp_uniform(*tmem_slot);
    // a pass leaves no copy, MMA or TMEM read of its own behind
    bool failed;
    auto end_pass = [&]() {
        __syncwarp();
        tc_fence_before();
        failed = __syncthreads_or(*fail_flag);
        init_bars(true);
        tc_fence_after();
    };
    const int nk = p.n_keys * p.Hkv;
    int claim = prompt_bwd_wide_pass<DK>(tq, tk, tv, tdo, p, sm, bar, fail_flag, tbase, 0, blockIdx.x);
    end_pass();
    zero_rows(sm + TILE, NCH);  // DV's units lie where V was
    __syncthreads();
    if (!failed) {
        claim = prompt_bwd_wide_pass<DV>(tq, tk, tv, tdo, p, sm, bar, fail_flag, tbase, nk, claim);
        end_pass();
        __syncthreads();
    }
    if (!failed) {
        prompt_bwd_wide_pass<DQ>(tq, tk, tv, tdo, p, sm, bar, fail_flag, tbase, 2 * nk, claim);
        __syncwarp();
        tc_fence_before();
        failed = __syncthreads_or(*fail_flag);
        tc_fence_after();
    }
    if (failed && threadIdx.x == 0) report(p.status, JNX_ERR_TIMEOUT);
    if (warp == 1) tmem_dealloc(tbase, 512);
}

static jnx_status launch_prompt_bwd_wide(const PromptBwdArgs& a, const jnx_head_rows& q,
                                         const jnx_head_rows& k, const jnx_head_rows& v,
                                         const jnx_head_rows& dout, int rows, int keys, cudaStream_t s) {
    using namespace pwide;
    const char* what = "prompt attention backward";
    static std::atomic<uint64_t> attr{0};
    if (set_smem_limit(reinterpret_cast<const void*>(k_prompt_attn_bwd_wide), SMEM, attr) != cudaSuccess)
        return fail(JNX_ERR_CUDA, "%s: smem attribute", what);
    const int T = tile_tokens(a.group);
    CUtensorMap tq, tk, tv, tdo;
    if (!make_tmap_heads(&tq, q, rows, a.H, HD, a.group, T) ||
        !make_tmap_heads(&tdo, dout, rows, a.H, HD, a.group, T) ||
        !make_tmap_heads(&tk, k, keys, a.Hkv, HD, 1, BM) ||
        !make_tmap_heads(&tv, v, keys, a.Hkv, HD, 1, BM))
        return fail(JNX_ERR_CUDA, "%s: tensor map encode failed", what);
    const int grid = (int)std::min<long long>(((long long)2 * a.n_keys + a.n_queries) * a.Hkv, num_sms());
    pdl(k_prompt_attn_bwd_wide, grid, THREADS, SMEM, s)(tq, tk, tv, tdo, a);
    return launched(what);
}

}  // namespace jnx

using namespace jnx;

// The claims; each row's lse and D, and the other D; the parts' sums, dk's and dv's.  (Room for every key as
// often as the longest sequence has parts, which this is in place of, was 5.0 GB of one
// sequence of 12,000 tokens beside 48 of 840, 8 heads on one of 256; 0.8 GB.)
static size_t bwd_row_bytes(int rows, int n_heads) {
    return 256 + (((size_t)rows * n_heads * (sizeof(float2) + sizeof(float)) + 255) & ~(size_t)255);
}
static size_t bwd_bytes(int rows, const PromptCounts& list, int n_heads, int n_kv_heads, int head_dim) {
    return bwd_row_bytes(rows, n_heads) +
           (size_t)list.slabs * n_kv_heads * 2 * 128 * head_dim * sizeof(float);
}

extern "C" size_t jnx_op_prompt_attention_backward_workspace_bytes(const jnx_prompt* p,
                                                                   int32_t n_heads,
                                                                   int32_t n_kv_heads,
                                                                   int32_t head_dim) {
    clear_error();
    int rows, keys;
    if (heads_ok(n_heads, n_kv_heads, head_dim, "prompt attention backward") ||
        prompt_ok(p, "prompt attention backward", rows, keys))
        return 0;
    return bwd_bytes(rows, prompt_counts(p, n_heads, n_kv_heads, head_dim, true), n_heads, n_kv_heads,
                     head_dim);
}

extern "C" jnx_status jnx_op_prompt_attention_backward(
    const jnx_prompt* p, int32_t n_heads, int32_t n_kv_heads, int32_t head_dim,
    const jnx_head_rows* q, const jnx_head_rows* k, const jnx_head_rows* v,
    const jnx_head_rows* out, const jnx_head_rows* /* rest */, const float* lse,
    const jnx_head_rows* dout, const jnx_head_rows* dq, const jnx_head_rows* dk,
    const jnx_head_rows* dv, void* workspace, size_t ws_bytes, int32_t* status, void* stream) {
    clear_error();
    const char* what = "prompt attention backward";
    int rows, keys;
    if (jnx_status st = heads_ok(n_heads, n_kv_heads, head_dim, what)) return st;
    if (jnx_status st = prompt_launchable(p, what, true, rows, keys)) return st;
    if (rows == 0 && keys == 0) return JNX_OK;
    if ((rows > 0 && (!rows_ok(q) || !rows_ok(out) || !rows_ok(dout) || !rows_ok(dq) || !lse)) ||
        (keys > 0 && (!rows_ok(k) || !rows_ok(v) || !rows_ok(dk) || !rows_ok(dv))))
        return fail(JNX_ERR_INVALID_ARG, "%s: null or misaligned rows", what);
    const PromptCounts list = prompt_counts(p, n_heads, n_kv_heads, head_dim, true);
    if (!workspace || !aligned16(workspace) ||
        ws_bytes < bwd_bytes(rows, list, n_heads, n_kv_heads, head_dim))
        return fail(JNX_ERR_WORKSPACE, "%s: workspace too small or misaligned", what);
    if (p->n_forward != list.forward || p->n_keys != list.keys || p->n_queries != list.queries ||
        p->n_parts != list.parts)
        return fail(JNX_ERR_INVALID_ARG, "%s: a work list of other heads or lengths", what);
    const long long n_work = ((long long)2 * p->n_keys + p->n_queries) * n_kv_heads;
    // (claims run past the last item by one for each CTA and pass)
    if (n_work > 0x7FFFFFFFLL - 4 * num_sms() || (long long)rows * n_heads > 0x7FFFFFF00LL ||
        (long long)p->n_seqs * n_kv_heads > 0x3FFFFFFFLL)
        return fail(JNX_ERR_UNSUPPORTED, "%s: too many work items", what);
    const jnx_head_rows none{nullptr, 0, 0};
    auto or_none = [&](const jnx_head_rows* r, int n) { return n ? *r : none; };
    int* claimed = static_cast<int*>(workspace);
    float2* row = reinterpret_cast<float2*>(static_cast<uint8_t*>(workspace) + 256);
    float* few = reinterpret_cast<float*>(row + (size_t)rows * n_heads);
    PromptBwdArgs a{p->cu_q, p->cu_kv, p->prefix,
                    reinterpret_cast<const int2*>(p->items) + p->n_forward, p->n_keys, p->n_queries,
                    n_heads, n_kv_heads, n_heads / n_kv_heads, claimed,
                    (float)(1.4426950408889634 / sqrt((double)head_dim)),
                    (float)(1.0 / sqrt((double)head_dim)), row, few, p->n_seqs, rows, keys, or_none(dq, rows),
                    or_none(dk, keys), or_none(dv, keys),
                    reinterpret_cast<float*>(static_cast<uint8_t*>(workspace) + bwd_row_bytes(rows, n_heads)),
                    (int)list.slabs, status};
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    TraceScope ts(JNX_K_PROMPT_ATTN_BWD, 0.0, s);
    auto prologue = [&](auto width) {
        constexpr int HD = decltype(width)::value, PER = 4 * 256 / (HD / 8);
        const long long all = (long long)rows * n_heads, heads = (long long)p->n_seqs * n_kv_heads;
        // a sequence's rows of few keys are 2 group tiles' pairs at most: a CTA each, or fewer
        // where there are sequences enough
        const int of = (int)std::min<long long>(kFewKeys * a.group / (16 * kFewTiles),
                                                std::max<long long>(1, 4 * 152 / heads));
        const long long n_few = rows && keys ? heads * of : 0;
        pdl(k_prompt_bwd_rows<HD>, (int)(n_few + std::max(1LL, (all + PER - 1) / PER)), 256, 0, s)(
            or_none(out, rows), or_none(dout, rows), or_none(q, rows), or_none(k, keys),
            or_none(v, keys), lse, a, row, few, (int)n_few, of);
    };
    if (head_dim == 64) prologue(std::integral_constant<int, 64>{});
    else if (head_dim == 128) prologue(std::integral_constant<int, 128>{});
    else prologue(std::integral_constant<int, 256>{});
    // where there are no rows or keys nothing is loaded, but the maps want an address
    const jnx_head_rows& any = rows ? *q : *k;
    const jnx_head_rows qq = rows ? *q : any, dd = rows ? *dout : any, kk = keys ? *k : any,
                        vv = keys ? *v : any;
    const int nr = std::max(rows, 1), nk = std::max(keys, 1);
    const jnx_status st = head_dim == 64    ? launch_prompt_bwd<64>(a, qq, kk, vv, dd, nr, nk, s)
                          : head_dim == 128 ? launch_prompt_bwd<128>(a, qq, kk, vv, dd, nr, nk, s)
                                            : launch_prompt_bwd_wide(a, qq, kk, vv, dd, nr, nk, s);
    if (st || list.slabs == 0) return st;
    pdl(k_prompt_bwd_join, dim3((int)list.slabs * n_kv_heads, 16, 2), 256, 0, s)(a, head_dim);
    return launched(what);
}
