// Norms of query and key heads with the position rotation, in one pass over the rows
// of the fused projection, and its gradients.
//
// A head row x [hd] becomes y = R(pos) (x r gamma), r = rsqrt(mean(x^2) + eps), where R
// turns each pair (i, i + hd / 2) by pos[axis(i)] theta^(-2 i / hd).  R is orthogonal, so
// with dn = R^T dy the gradients are dgamma = sum dn x r over all rows and
// dx = r (gamma dn) - x r^3 mean(gamma dn x).
//
// Bound by HBM: 4 bytes an element forward (6 backward).  A lane holds E elements of
// either half of a row, so a pair meets in one lane and the norm's sum is a few shuffles;
// the rows of the next pass are under way while one is worked on.  The angles of a CTA's
// tokens are computed once into shared memory and serve all of a token's heads, laid out
// so that a row's lanes read neighbours (they were 4 to 8 ways in conflict as they come).
// 9,001 tokens, 32 and 8 heads of 128: 33.6 us, 5.5 TB/s.  30,011 tokens, 16 and 16 of 64:
// 45 us forward (5.4 TB/s) and 86 its gradients (4.3); 8 and 1 of 256, where a token's 128
// angles weigh as much as its rows, 53 and 154.  One token each of 16 sequences, 8
// heads and 1 of 256 into a cache: 2.5 us, a launch's latency.  (Rows through bulk copies
// in shared memory were slower: 126 for 99 us forward at head dim 128, 356 for 212 back.)
//
// An angle is taken modulo whole turns before it is rounded: the frequency is a 64-bit
// fraction of a turn, so position times frequency in wrapping 64-bit integers is the
// turn's exact fraction (2^-33 of a turn kept), where a 32-bit float product is off by
// 6e-8 of the angle itself, 1e-3 rad at position 16,000.  What is left is the frequency's own
// rounding as a double, 2^-50 of the angle: 2e-6 rad at position 2^31.
#include <algorithm>
#include <climits>
#include <cmath>

#include "jnx_dev.cuh"
#include "jnx_kernels.h"
#include "jnx_text.h"
#include "jnx_trace.h"

namespace jnx {

namespace rope {
constexpr int THREADS = 256;
constexpr int MAX_HALF = 128;  // frequencies of the largest head

struct Args {
    const uint16_t* qkv;
    long long ldqkv;
    const int* pos;
    int n_tokens, H, Hkv, tok;  // tok: tokens of a block
    float eps;
    const uint16_t *gq, *gk;
    // forward: where rows go; backward: where the gradients of those rows come from
    uint16_t *q, *k;
    long long q_row, q_head, k_row, k_head;
    // append: the cache
    uint16_t* v;
    long long slot_stride;
    const int *slot, *at;  // paged: slot is the sequence
    int n_slots, room;
    Pages pages;
    int* status;
    // backward
    uint16_t* dqkv;
    int q_ctas;      // CTAs on query rows; the others take key rows
    float* partial;  // [hd][grid]
    // frequency i as a 64-bit fraction of a turn, and its axis
    unsigned long long turn[MAX_HALF];
    unsigned char axis[MAX_HALF];
};

// One frequency, whose turn and positions a thread looks up once for all of its tokens: lanes ask
// for different entries of the arguments, which are served one after another.  (Looked up for
// every token: 30,000 tokens of 9 heads of 256 64 us, so 53.)
struct Frequency {
    unsigned long long turn;
    const int* pos;
    __device__ __forceinline__ Frequency(const Args& a, int i)
        : turn(a.turn[i]), pos(a.pos + (size_t)a.axis[i] * a.n_tokens) {}
    // cos and sin for token t
    __device__ __forceinline__ float2 angle(int t) const {
        float2 cs = make_float2(1.f, 0.f);
        if (turn) {
            const int frac = (int)((unsigned long long)(long long)pos[t] * turn >> 32);  // 2^-32 turns, wrapped
            sincospif((float)frac * 4.656612873077393e-10f, &cs.y, &cs.x);  // 2^-31 half turns
        }
        return cs;
    }
};

// N bf16 elements (a multiple of 4) as loaded, and as floats.
template <int N>
struct Pack {
    uint32_t w[N / 2];
    __device__ __forceinline__ void load(const uint16_t* p) {
        if constexpr (N == 8) {
            const uint4 v = *reinterpret_cast<const uint4*>(p);
            w[0] = v.x, w[1] = v.y, w[2] = v.z, w[3] = v.w;
        } else {
            const uint2 v = *reinterpret_cast<const uint2*>(p);
            w[0] = v.x, w[1] = v.y;
        }
    }
    __device__ __forceinline__ void store(uint16_t* p) const {
        if constexpr (N == 8)
            *reinterpret_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
        else
            *reinterpret_cast<uint2*>(p) = make_uint2(w[0], w[1]);
    }
    // elements 2 i and 2 i + 1 as an fp32 pair
    __device__ __forceinline__ uint64_t pair(int i) const {
        return f2_pack(__uint_as_float(w[i] << 16), __uint_as_float(w[i] & 0xffff0000u));
    }
    __device__ __forceinline__ void set(int i, uint64_t f) {
        float a, b;
        f2_unpack(f, a, b);
        w[i] = cvt_bf2(a, b);
    }
    __device__ __forceinline__ void clear() {
#pragma unroll
        for (int i = 0; i < N / 2; ++i) w[i] = 0;
    }
};

// Sum over the LPR lanes of a row.
template <int LPR>
__device__ __forceinline__ float row_sum(float v) {
#pragma unroll
    for (int o = LPR / 2; o; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}

// E: elements of either half a lane holds; TOK: tokens of a block, at most.
template <int HD, int E_, int TOK_>
struct Cfg {
    static constexpr int E = E_, TOK = TOK_;
    static constexpr int LPR = HD / 2 / E;        // lanes a row
    static constexpr int RPP = THREADS / LPR;     // rows a pass
    // angles of TOK tokens from t0 on: [t][e][l] holds cos, cos, sin, sin of lane l's
    // elements 2 e and 2 e + 1
    static_assert(THREADS % (HD / 2) == 0, "a thread has one frequency");
    static __device__ __forceinline__ void angles(const Args& a, int t0, int nt, float4* cs) {
        const int i = threadIdx.x % (HD / 2);
        if ((int)threadIdx.x / (HD / 2) >= nt) return;
        const Frequency f(a, i);
        float* at = reinterpret_cast<float*>(cs) + (i % E / 2 * LPR + i / E) * 4 + (i & 1);
        for (int t = threadIdx.x / (HD / 2); t < nt; t += THREADS / (HD / 2)) {
            const float2 v = f.angle(t0 + t);
            at[t * (E / 2) * LPR * 4] = v.x;
            at[t * (E / 2) * LPR * 4 + 2] = v.y;
        }
    }
    static __device__ __forceinline__ void read(const float4* cs, int t, int e, int l, uint64_t& c,
                                                uint64_t& s) {
        const float4 v = cs[(t * (E / 2) + e) * LPR + l];
        c = f2_pack(v.x, v.y);
        s = f2_pack(v.z, v.w);
    }
};
template <int HD>
using Forward = Cfg<HD, 8, HD == 64 ? 16 : 8>;
template <int HD>
using Backward = Cfg<HD, 4, HD == 128 ? 8 : 16>;

// Where keys go: rows of a tensor, rows of cache slots, or rows of the pages of sequences.
enum { ROWS = 0, SLOTS = 1, PAGES = 2 };
constexpr long long NOWHERE = LLONG_MIN;  // (any other place may be one: strides may be negative)
}  // namespace rope

template <int HD, int TO>
__global__ void __launch_bounds__(rope::THREADS)
    k_qk_norm_rope(const __grid_constant__ rope::Args a) {
    constexpr bool APPEND = TO != rope::ROWS;
    using C = rope::Forward<HD>;
    constexpr int E = C::E;
    __shared__ float4 cs[C::TOK * HD / 4];
    __shared__ long long place[APPEND ? C::TOK : 1];  // where a token's keys go
    pdl_entry();
    const int t0 = blockIdx.x * a.tok, nt = min(a.tok, a.n_tokens - t0);
    if (APPEND && (int)threadIdx.x < nt) {  // (looked up at every row: 39.3 us of 9,000 tokens for 38.3)
        const int tok = t0 + threadIdx.x;
        int slot = a.slot[tok], at = a.at[tok];
        const bool there = TO == rope::PAGES ? a.pages.find(slot, at, slot, at)
                                             : slot >= 0 && slot < a.n_slots && at >= 0 && at < a.room;
        place[threadIdx.x] = there ? slot * a.slot_stride + at * a.k_row : rope::NOWHERE;
        if (!there) report(a.status, JNX_ERR_DEVICE_BOUNDS);
    }
    // rows of the CTA's tokens, token-major; an append's value heads come after the keys'
    const int heads = a.H + (APPEND ? 2 : 1) * a.Hkv;
    const int l = threadIdx.x % C::LPR, part = l * E;  // this lane's elements of each half
    // (token, head) of this lane's row in a pass
    int t = (threadIdx.x / C::LPR) / heads, head = (threadIdx.x / C::LPR) % heads;
    rope::Pack<E> lo, hi, g[2][2];
    auto load = [&]() {
        lo.clear();
        hi.clear();
        if (t >= nt) return;
        const uint16_t* x = a.qkv + (size_t)(t0 + t) * a.ldqkv + (size_t)head * HD + part;
        lo.load(x);
        hi.load(x + HD / 2);
    };
    load();
#pragma unroll
    for (int w = 0; w < 2; ++w)
        if (const uint16_t* gamma = w ? a.gk : a.gq) {
            g[w][0].load(gamma + part);
            g[w][1].load(gamma + HD / 2 + part);
        }
    C::angles(a, t0, nt, cs);
    __syncthreads();
    for (int r0 = 0; r0 < nt * heads; r0 += C::RPP) {
        const int tw = t, hw = head;
        uint64_t x[E / 2], y[E / 2], ss2 = f2_pack(0.f, 0.f);
#pragma unroll
        for (int e = 0; e < E / 2; ++e) {
            x[e] = lo.pair(e);
            y[e] = hi.pair(e);
            ss2 = f2_fma(x[e], x[e], ss2);
            ss2 = f2_fma(y[e], y[e], ss2);
        }
        float s0, s1;
        f2_unpack(ss2, s0, s1);
        const rope::Pack<E> raw[2] = {lo, hi};
        for (head += C::RPP; head >= heads; head -= heads) ++t;
        load();  // the next pass's row
        const float ss = rope::row_sum<C::LPR>(s0 + s1);
        if (tw >= nt) continue;
        const size_t tok = t0 + tw;
        const bool is_q = hw < a.H, is_v = APPEND && hw >= a.H + a.Hkv;
        rope::Pack<E> olo = raw[0], ohi = raw[1];
        if (!is_v) {
            if (is_q ? a.gq : a.gk) {
                const float s = rsqrtf(ss * (1.f / HD) + a.eps);
                const uint64_t sp = f2_pack(s, s);
#pragma unroll
                for (int e = 0; e < E / 2; ++e) {
                    x[e] = f2_mul(f2_mul(x[e], sp), (is_q ? g[0][0] : g[1][0]).pair(e));
                    y[e] = f2_mul(f2_mul(y[e], sp), (is_q ? g[0][1] : g[1][1]).pair(e));
                }
            }
#pragma unroll
            for (int e = 0; e < E / 2; ++e) {
                uint64_t c, s;
                C::read(cs, tw, e, l, c, s);
                const uint64_t ns = s ^ 0x8000000080000000ull;
                olo.set(e, f2_fma(x[e], c, f2_mul(y[e], ns)));
                ohi.set(e, f2_fma(y[e], c, f2_mul(x[e], s)));
            }
        }
        uint16_t* o;
        if (is_q) {
            o = a.q + tok * a.q_row + hw * a.q_head;
        } else if (APPEND) {
            if (place[tw] == rope::NOWHERE) continue;
            o = (is_v ? a.v : a.k) + place[tw] + (hw - a.H - (is_v ? a.Hkv : 0)) * a.k_head;
        } else {
            o = a.k + tok * a.k_row + (hw - a.H) * a.k_head;
        }
        olo.store(o + part);
        ohi.store(o + HD / 2 + part);
    }
}

// Gradients.  A CTA takes query rows or key rows of its share of the tokens, blocks of TOK in
// turn; their gains' gradients stay in its lanes' registers and are added over its rows in a
// fixed order at the end.  (Both kinds of rows in one CTA, so that no angle is needed twice, and
// two passes' loads under way each spill: 236 and 203 us for 188 at 30,000 tokens of 32 and 8
// heads of 128.)
template <int HD>
__global__ void __launch_bounds__(rope::THREADS, 4)
    k_qk_norm_rope_bwd(const __grid_constant__ rope::Args a) {
    using C = rope::Backward<HD>;
    constexpr int E = C::E;
    __shared__ float4 cs[C::TOK * HD / 4];
    __shared__ float sums[C::RPP][HD];
    pdl_entry();
    const bool is_q = (int)blockIdx.x < a.q_ctas;
    const int heads = is_q ? a.H : a.Hkv, first = is_q ? 0 : a.H;
    const int part_cta = is_q ? blockIdx.x : blockIdx.x - a.q_ctas;
    const int ctas = is_q ? a.q_ctas : gridDim.x - a.q_ctas;
    const uint16_t* dy = is_q ? a.q : a.k;
    const long long dy_row = is_q ? a.q_row : a.k_row, dy_head = is_q ? a.q_head : a.k_head;
    const uint16_t* gamma = is_q ? a.gq : a.gk;
    const int l = threadIdx.x % C::LPR, part = l * E, lane_row = threadIdx.x / C::LPR;
    uint64_t gain[E] = {}, gacc[E] = {};
    if (gamma) {
        rope::Pack<E> gl, gh;
        gl.load(gamma + part);
        gh.load(gamma + HD / 2 + part);
#pragma unroll
        for (int e = 0; e < E / 2; ++e) {
            gain[e] = gl.pair(e);
            gain[E / 2 + e] = gh.pair(e);
        }
    }
    const int end = (int)((long long)a.n_tokens * (part_cta + 1) / ctas);
    for (int t0 = (int)((long long)a.n_tokens * part_cta / ctas); heads > 0 && t0 < end; t0 += C::TOK) {
        const int nt = min(C::TOK, end - t0);
        int t = lane_row / heads, head = lane_row % heads;
        rope::Pack<E> xl, xh, yl, yh;
        auto load = [&]() {
            xl.clear(), xh.clear(), yl.clear(), yh.clear();
            if (t >= nt) return;
            const uint16_t* x = a.qkv + (size_t)(t0 + t) * a.ldqkv + (size_t)(first + head) * HD + part;
            const uint16_t* y = dy + (t0 + t) * dy_row + head * dy_head + part;
            xl.load(x);
            xh.load(x + HD / 2);
            yl.load(y);
            yh.load(y + HD / 2);
        };
        load();
        __syncthreads();  // the last block's angles have been read
        C::angles(a, t0, nt, cs);
        __syncthreads();
        for (int r0 = 0; r0 < nt * heads; r0 += C::RPP) {
            const int tw = t, hw = head;
            uint64_t x[E], d[E];  // pairs of the lower half, then of the upper
#pragma unroll
            for (int e = 0; e < E / 2; ++e) {
                uint64_t c, s;
                C::read(cs, min(tw, nt - 1), e, l, c, s);
                const uint64_t ns = s ^ 0x8000000080000000ull, u = yl.pair(e), v = yh.pair(e);
                x[e] = xl.pair(e);
                x[E / 2 + e] = xh.pair(e);
                d[e] = f2_fma(u, c, f2_mul(v, s));  // back by the same angle
                d[E / 2 + e] = f2_fma(v, c, f2_mul(u, ns));
            }
            for (head += C::RPP; head >= heads; head -= heads) ++t;
            load();  // the next pass's row
            uint16_t* o = a.dqkv + (size_t)(t0 + tw) * a.ldqkv + (size_t)(first + hw) * HD + part;
            if (gamma) {
                uint64_t ss2 = f2_pack(0.f, 0.f), dot2 = ss2, dx[E];
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    dx[e] = f2_mul(d[e], x[e]);
                    ss2 = f2_fma(x[e], x[e], ss2);
                    dot2 = f2_fma(gain[e], dx[e], dot2);
                }
                float s0, s1, d0, d1;
                f2_unpack(ss2, s0, s1);
                f2_unpack(dot2, d0, d1);
                const float ss = rope::row_sum<C::LPR>(s0 + s1), dot = rope::row_sum<C::LPR>(d0 + d1);
                const float s = tw < nt ? rsqrtf(ss * (1.f / HD) + a.eps) : 0.f;
                const float m = -dot * (1.f / HD) * s * s * s;
                const uint64_t sp = f2_pack(s, s), mp = f2_pack(m, m);
#pragma unroll
                for (int e = 0; e < E; ++e) {  // a lane without a row adds zeros
                    gacc[e] = f2_fma(dx[e], sp, gacc[e]);
                    d[e] = f2_fma(f2_mul(gain[e], sp), d[e], f2_mul(x[e], mp));
                }
            }
            if (tw < nt) {
                rope::Pack<E> ol, oh;
#pragma unroll
                for (int e = 0; e < E / 2; ++e) {
                    ol.set(e, d[e]);
                    oh.set(e, d[E / 2 + e]);
                }
                ol.store(o);
                oh.store(o + HD / 2);
            }
        }
    }
    if (!a.partial) return;
#pragma unroll
    for (int e = 0; e < E / 2; ++e) {
        float* to = &sums[lane_row][part + 2 * e];
        f2_unpack(gacc[e], to[0], to[1]);
        f2_unpack(gacc[E / 2 + e], to[HD / 2], to[HD / 2 + 1]);
    }
    __syncthreads();
    for (int c = threadIdx.x; c < HD; c += rope::THREADS) {
        float s = 0.f;
        for (int r = 0; r < C::RPP; ++r) s += sums[r][c];
        a.partial[(size_t)c * gridDim.x + blockIdx.x] = s;
    }
}

// dgamma = sum of the CTAs' parts, each column's in a fixed order: 32 lanes take the
// parts in turn, then add up.  A warp a column of the queries' or the keys' gains.
__global__ void __launch_bounds__(256)
    k_qk_gain_sum(const float* partial, int q_ctas, int ctas, int hd, float* dgq, float* dgk) {
    pdl_entry();
    const int w = blockIdx.x * 8 + (threadIdx.x >> 5), lane = threadIdx.x & 31;
    if (w >= 2 * hd) return;
    const int c = w < hd ? w : w - hd, from = w < hd ? 0 : q_ctas, to = w < hd ? q_ctas : ctas;
    float s = 0.f;
#pragma unroll 4
    for (int i = from + lane; i < to; i += 32) s += partial[(size_t)c * ctas + i];
#pragma unroll
    for (int o = 16; o; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
    float* out = w < hd ? dgq : dgk;
    if (lane == 0 && out) out[c] = s;
}

static jnx_status rope_args(const jnx_qk_rope* p, const uint16_t* qkv, int64_t ldqkv,
                            const int32_t* pos, int32_t n_tokens, const char* what,
                            rope::Args& a) {
    if (!p) return fail(JNX_ERR_INVALID_ARG, "%s: null description", what);
    if (p->head_dim != 64 && p->head_dim != 128 && p->head_dim != 256)
        return fail(JNX_ERR_UNSUPPORTED, "%s: head_dim %d not in {64,128,256}", what, p->head_dim);
    if (p->n_heads < 0 || p->n_kv_heads < 0 || n_tokens < 0 || p->n_axes < 0 || p->n_axes > 4)
        return fail(JNX_ERR_INVALID_ARG, "%s: bad sizes", what);
    const int heads = p->n_heads + 2 * p->n_kv_heads;
    if (ldqkv < (int64_t)heads * p->head_dim || ldqkv % 8)
        return fail(JNX_ERR_INVALID_ARG, "%s: row stride %lld", what, (long long)ldqkv);
    if (!(p->theta > 0.f) || !(p->eps >= 0.f))
        return fail(JNX_ERR_INVALID_ARG, "%s: theta %g, eps %g", what, p->theta, p->eps);
    int turned = 0;
    for (int x = 0; x < p->n_axes; ++x) {
        if (p->sections[x] < 0 || p->sections[x] > p->head_dim / 2 - turned)
            return fail(JNX_ERR_INVALID_ARG, "%s: sections exceed head_dim / 2", what);
        turned += p->sections[x];
    }
    if (n_tokens > 0 && (!qkv || (turned && !pos)))
        return fail(JNX_ERR_INVALID_ARG, "%s: null argument", what);
    if (!aligned16(qkv) || !aligned16(p->gamma_q) || !aligned16(p->gamma_k))
        return fail(JNX_ERR_INVALID_ARG, "%s: qkv and gains must be 16-byte aligned", what);
    a.qkv = qkv;
    a.ldqkv = ldqkv;
    a.pos = pos;
    a.n_tokens = n_tokens;
    a.H = p->n_heads;
    a.Hkv = p->n_kv_heads;
    a.eps = p->eps;
    a.gq = p->gamma_q;
    a.gk = p->gamma_k;
    // frequency i is theta^(-2 i / hd): every eighth by pow, the next seven by the ratio, which
    // leaves a double's rounding eight times over, 2^-50 (128 pows were a fifth of a call)
    const double ratio = std::pow((double)p->theta, -2.0 / p->head_dim);
    double power = 0.0;
    for (int i = 0, axis = 0, end = p->n_axes ? p->sections[0] : 0; i < turned; ++i) {
        while (i >= end) end += p->sections[++axis];
        power = i % 8 ? power * ratio : std::pow((double)p->theta, -2.0 * i / p->head_dim);
        // / (2 pi), modulo whole turns, in units of 2^-64
        double f = power / 6.283185307179586476925;
        f -= std::floor(f);
        const double hi = std::floor(f * 4294967296.0);
        const double lo = std::floor((f * 4294967296.0 - hi) * 4294967296.0);
        a.turn[i] = ((unsigned long long)hi << 32) | (unsigned long long)lo;
        a.axis[i] = (unsigned char)axis;
    }
    return JNX_OK;
}

// Tokens of a CTA: rows for four passes, fewer where that would leave SMs without a CTA.
// (30,000 tokens of 9 heads of 256: 88 us with two tokens a CTA, a pass and an eighth, 63
// with eight.)
template <int HD, int TO>
static void launch_rope_hd(rope::Args a, cudaStream_t s) {
    using C = rope::Forward<HD>;
    const int heads = a.H + (TO != rope::ROWS ? 2 : 1) * a.Hkv;
    a.tok = std::max(1, std::min({C::TOK, (4 * C::RPP + heads - 1) / heads, a.n_tokens / (152 * 6)}));
    pdl(k_qk_norm_rope<HD, TO>, (a.n_tokens + a.tok - 1) / a.tok, rope::THREADS, 0, s)(a);
}

template <int TO>
static jnx_status launch_rope(const rope::Args& a, int hd, const char* what, cudaStream_t s) {
    if (!a.H && !a.Hkv) return JNX_OK;
    TraceScope ts(JNX_K_QK_ROPE, 0.0, s);
    if (hd == 64) launch_rope_hd<64, TO>(a, s);
    else if (hd == 128) launch_rope_hd<128, TO>(a, s);
    else launch_rope_hd<256, TO>(a, s);
    return launched(what);
}

// Query rows and the cache that an append writes.
static jnx_status rope_cache(rope::Args& a, const jnx_head_rows* q, const jnx_kv_cache* cache,
                             const int32_t* slot, const int32_t* at, int32_t* status, const char* what) {
    if ((a.H && !rows_ok(q)) || !cache_ok(cache) || !slot || !at)
        return fail(JNX_ERR_INVALID_ARG, "%s: null or misaligned argument", what);
    if (a.H) a.q = q->ptr, a.q_row = q->row_stride, a.q_head = q->head_stride;
    a.k = cache->k;
    a.v = cache->v;
    a.k_row = cache->row_stride;
    a.k_head = cache->head_stride;
    a.slot_stride = cache->slot_stride;
    a.n_slots = cache->n_slots;
    a.room = cache->room;
    a.slot = slot;
    a.at = at;
    a.status = status;
    return JNX_OK;
}

// CTAs of the gradient kernel, at most what 152 SMs hold at once, shared out between query
// and key rows by what a token of either takes: its rows' passes, its angles, and a share of a
// block's waits (by rows alone the key rows of 8 heads on one, 256 wide, were the last by far:
// 30,000 tokens 275 us, so 154; 32 heads on 8 of 128 212 and 187 us); each kind has one at
// least, and a CTA tokens enough for a pass or two.
static int rope_bwd_grid(const jnx_qk_rope* p, int n_tokens, int& q_ctas) {
    const int hd = p->head_dim, tok = hd == 128 ? 8 : 16, least = hd == 64 ? 16 : 8;
    const int blocks = std::max(1, (int)(((long long)n_tokens + least - 1) / least)), most = 152 * 4;
    auto cost = [&](int heads) { return heads * hd / 2048.0 + 1.25 * hd / 512.0 + 1.0 / tok; };
    const double q = cost(p->n_heads), k = cost(p->n_kv_heads);
    q_ctas = std::min(blocks, std::max(1, (int)(most * q / (q + k))));
    return q_ctas + std::min(blocks, std::max(1, most - q_ctas));
}

}  // namespace jnx

using namespace jnx;

extern "C" jnx_status jnx_op_qk_norm_rope(const jnx_qk_rope* p, const uint16_t* qkv, int64_t ldqkv,
                                          const int32_t* pos, int32_t n_tokens,
                                          const jnx_head_rows* q, const jnx_head_rows* k,
                                          void* stream) {
    clear_error();
    rope::Args a{};
    if (jnx_status st = rope_args(p, qkv, ldqkv, pos, n_tokens, "qk norm rope", a)) return st;
    if (n_tokens == 0) return JNX_OK;
    if ((a.H && !rows_ok(q)) || (a.Hkv && !rows_ok(k)))
        return fail(JNX_ERR_INVALID_ARG, "qk norm rope: null or misaligned output rows");
    if (a.H) a.q = q->ptr, a.q_row = q->row_stride, a.q_head = q->head_stride;
    if (a.Hkv) a.k = k->ptr, a.k_row = k->row_stride, a.k_head = k->head_stride;
    return launch_rope<rope::ROWS>(a, p->head_dim, "qk norm rope", static_cast<cudaStream_t>(stream));
}

extern "C" jnx_status jnx_op_qk_norm_rope_append(const jnx_qk_rope* p, const uint16_t* qkv,
                                                 int64_t ldqkv, const int32_t* pos,
                                                 int32_t n_tokens, const jnx_head_rows* q,
                                                 const jnx_kv_cache* cache, const int32_t* slot,
                                                 const int32_t* at, int32_t* status,
                                                 void* stream) {
    clear_error();
    rope::Args a{};
    if (jnx_status st = rope_args(p, qkv, ldqkv, pos, n_tokens, "qk norm rope append", a)) return st;
    if (n_tokens == 0) return JNX_OK;
    if (jnx_status st = rope_cache(a, q, cache, slot, at, status, "qk norm rope append")) return st;
    return launch_rope<rope::SLOTS>(a, p->head_dim, "qk norm rope append",
                                    static_cast<cudaStream_t>(stream));
}

extern "C" jnx_status jnx_op_qk_norm_rope_append_paged(
    const jnx_qk_rope* p, const uint16_t* qkv, int64_t ldqkv, const int32_t* pos, int32_t n_tokens,
    const jnx_head_rows* q, const jnx_kv_cache* cache, const jnx_pages* pages, const int32_t* seq,
    const int32_t* at, int32_t* status, void* stream) {
    clear_error();
    const char* what = "qk norm rope append paged";
    rope::Args a{};
    if (jnx_status st = rope_args(p, qkv, ldqkv, pos, n_tokens, what, a)) return st;
    if (n_tokens == 0) return JNX_OK;
    if (jnx_status st = rope_cache(a, q, cache, seq, at, status, what)) return st;
    if (!pages_ok(pages)) return fail(JNX_ERR_INVALID_ARG, "%s: bad pages", what);
    a.pages = Pages(*pages, *cache);
    return launch_rope<rope::PAGES>(a, p->head_dim, what, static_cast<cudaStream_t>(stream));
}

extern "C" size_t jnx_op_qk_norm_rope_backward_workspace_bytes(const jnx_qk_rope* p,
                                                               int32_t n_tokens) {
    if (!p || n_tokens < 0 || p->head_dim <= 0 || p->n_heads < 0 || p->n_kv_heads < 0) return 0;
    int q_ctas;
    return (size_t)rope_bwd_grid(p, n_tokens, q_ctas) * p->head_dim * sizeof(float);
}

extern "C" jnx_status jnx_op_qk_norm_rope_backward(const jnx_qk_rope* p, const uint16_t* qkv,
                                                   int64_t ldqkv, const int32_t* pos,
                                                   int32_t n_tokens, const jnx_head_rows* dq,
                                                   const jnx_head_rows* dk, uint16_t* dqkv,
                                                   float* dgamma_q, float* dgamma_k,
                                                   void* workspace, size_t ws_bytes,
                                                   void* stream) {
    clear_error();
    rope::Args a{};
    if (jnx_status st = rope_args(p, qkv, ldqkv, pos, n_tokens, "qk norm rope backward", a))
        return st;
    if ((a.gq && !dgamma_q) || (a.gk && !dgamma_k))
        return fail(JNX_ERR_INVALID_ARG, "qk norm rope backward: null gain gradient");
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    const int hd = p->head_dim;
    const bool gains = a.gq || a.gk;
    if (n_tokens == 0) {
        if ((a.gq && cudaMemsetAsync(dgamma_q, 0, hd * sizeof(float), s) != cudaSuccess) ||
            (a.gk && cudaMemsetAsync(dgamma_k, 0, hd * sizeof(float), s) != cudaSuccess))
            return launched("qk norm rope backward");
        return JNX_OK;
    }
    if ((a.H && !rows_ok(dq)) || (a.Hkv && !rows_ok(dk)) || !dqkv || !aligned16(dqkv))
        return fail(JNX_ERR_INVALID_ARG, "qk norm rope backward: null or misaligned rows");
    if (gains && (!workspace || ws_bytes < jnx_op_qk_norm_rope_backward_workspace_bytes(p, n_tokens)))
        return fail(JNX_ERR_WORKSPACE, "qk norm rope backward: workspace too small");
    if (a.H) a.q = dq->ptr, a.q_row = dq->row_stride, a.q_head = dq->head_stride;
    if (a.Hkv) a.k = dk->ptr, a.k_row = dk->row_stride, a.k_head = dk->head_stride;
    a.dqkv = dqkv;
    a.partial = gains ? static_cast<float*>(workspace) : nullptr;
    const int grid = rope_bwd_grid(p, n_tokens, a.q_ctas);
    TraceScope ts(JNX_K_QK_ROPE, 0.0, s);
    if (hd == 64) pdl(k_qk_norm_rope_bwd<64>, grid, rope::THREADS, 0, s)(a);
    else if (hd == 128) pdl(k_qk_norm_rope_bwd<128>, grid, rope::THREADS, 0, s)(a);
    else pdl(k_qk_norm_rope_bwd<256>, grid, rope::THREADS, 0, s)(a);
    if (gains)
        pdl(k_qk_gain_sum, (2 * hd + 7) / 8, 256, 0, s)(a.partial, a.q_ctas, grid, hd,
                                                       a.gq ? dgamma_q : nullptr,
                                                       a.gk ? dgamma_k : nullptr);
    return launched("qk norm rope backward");
}
