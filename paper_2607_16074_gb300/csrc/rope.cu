// Norms of query and key heads with the position rotation, in one pass over the rows
// of the fused projection, and its gradients.
//
// A head row x [hd] becomes y = R(pos) (x r gamma), r = rsqrt(mean(x^2) + eps), where R
// turns each pair (i, i + hd / 2) by pos[axis(i)] theta^(-2 i / hd).  R is orthogonal, so
// with dn = R^T dy the gradients are dgamma = sum dn x r over all rows and
// dx = r (gamma dn) - x r^3 mean(gamma dn x).
//
// Bound by HBM: 4 bytes an element forward (6 backward).  hd / 16 lanes hold a row, each
// 8 elements of either half (two 16-byte loads), so a pair meets in one lane and the
// norm's sum is log2(hd / 16) shuffles.  The angles of a CTA's tokens are computed once
// into shared memory and serve all of a token's heads.
//
// An angle is taken modulo whole turns before it is rounded: the frequency is a 64-bit
// fraction of a turn, so position times frequency in wrapping 64-bit integers is the
// turn's exact fraction (2^-33 of a turn kept), where a 32-bit float product is off by
// 6e-8 of the angle itself, 1e-3 rad at position 16,000.
#include <algorithm>
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
    int n_tokens, H, Hkv, half;
    float eps;
    const uint16_t *gq, *gk;
    // forward: where rows go; backward: where the gradients of those rows come from
    uint16_t *q, *k;
    long long q_row, q_head, k_row, k_head;
    // append: the cache
    uint16_t* v;
    long long slot_stride;
    const int *slot, *at;
    int n_slots, room;
    int* status;
    // backward
    uint16_t* dqkv;
    float* partial;  // [grid][2][hd]
    // frequency i as a 64-bit fraction of a turn, and its axis
    unsigned long long turn[MAX_HALF];
    unsigned char axis[MAX_HALF];
};

// cos and sin of frequency i for token t.
__device__ __forceinline__ float2 angle(const Args& a, int t, int i) {
    const unsigned long long f = a.turn[i];
    float2 cs = make_float2(1.f, 0.f);
    if (f) {
        const long long p = a.pos[(size_t)a.axis[i] * a.n_tokens + t];
        const int frac = (int)((unsigned long long)p * f >> 32);  // 2^-32 turns, wrapped
        sincospif((float)frac * 4.656612873077393e-10f, &cs.y, &cs.x);  // 2^-31 half turns
    }
    return cs;
}

__device__ __forceinline__ void unpack8(const uint4& u, float (&f)[8]) {
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        f[2 * i] = __uint_as_float(w[i] << 16);
        f[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
}

__device__ __forceinline__ uint4 pack8(const float (&f)[8]) {
    return make_uint4(pack_bf2(f[0], f[1]), pack_bf2(f[2], f[3]), pack_bf2(f[4], f[5]),
                      pack_bf2(f[6], f[7]));
}

// Sum over the hd / 16 lanes of a row.
template <int HD>
__device__ __forceinline__ float row_sum(float v) {
#pragma unroll
    for (int o = HD / 32; o; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}
}  // namespace rope

// Tokens a CTA takes: their angles are two a thread (one at hd = 64).
template <int HD>
struct RopeCfg {
    static constexpr int TOK = HD == 64 ? 8 : HD == 128 ? 4 : 2;
    static constexpr int LPR = HD / 16;                   // lanes a row
    static constexpr int RPP = rope::THREADS / LPR;       // rows a pass
};

template <int HD, bool APPEND>
__global__ void __launch_bounds__(rope::THREADS)
    k_qk_norm_rope(const __grid_constant__ rope::Args a) {
    using C = RopeCfg<HD>;
    __shared__ float2 cs[C::TOK][HD / 2];
    pdl_entry();
    const int t0 = blockIdx.x * C::TOK, nt = min(C::TOK, a.n_tokens - t0);
    for (int i = threadIdx.x; i < nt * (HD / 2); i += rope::THREADS)
        cs[i / (HD / 2)][i % (HD / 2)] = rope::angle(a, t0 + i / (HD / 2), i % (HD / 2));
    __syncthreads();
    // rows of the CTA's tokens, token-major; an append's value heads come after the keys'
    const int heads = a.H + (APPEND ? 2 : 1) * a.Hkv;
    const int part = threadIdx.x % C::LPR * 8;  // this lane's elements of each half
    for (int r0 = 0; r0 < nt * heads; r0 += C::RPP) {
        const int r = r0 + threadIdx.x / C::LPR;
        const bool live = r < nt * heads;
        const int t = live ? r / heads : 0, head = live ? r % heads : 0;
        const size_t tok = t0 + t;
        float lo[8] = {}, hi[8] = {};
        uint4 ulo = make_uint4(0, 0, 0, 0), uhi = ulo;
        if (live) {
            const uint16_t* x = a.qkv + tok * a.ldqkv + (size_t)head * HD + part;
            ulo = *reinterpret_cast<const uint4*>(x);
            uhi = *reinterpret_cast<const uint4*>(x + HD / 2);
        }
        rope::unpack8(ulo, lo);
        rope::unpack8(uhi, hi);
        const bool is_q = head < a.H, is_v = head >= a.H + a.Hkv;
        const uint16_t* gamma = is_q ? a.gq : a.gk;
        float ss = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) ss += lo[e] * lo[e] + hi[e] * hi[e];
        ss = rope::row_sum<HD>(ss);
        if (!live) continue;
        if (!is_v) {
            if (gamma) {
                const float s = rsqrtf(ss * (1.f / HD) + a.eps);
                float gl[8], gh[8];
                rope::unpack8(*reinterpret_cast<const uint4*>(gamma + part), gl);
                rope::unpack8(*reinterpret_cast<const uint4*>(gamma + HD / 2 + part), gh);
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    lo[e] *= s * gl[e];
                    hi[e] *= s * gh[e];
                }
            }
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float2 c = cs[t][part + e];
                const float x = lo[e], y = hi[e];
                lo[e] = x * c.x - y * c.y;
                hi[e] = y * c.x + x * c.y;
            }
            ulo = rope::pack8(lo);
            uhi = rope::pack8(hi);
        }
        uint16_t* o;
        if (is_q) {
            o = a.q + tok * a.q_row + head * a.q_head;
        } else if (APPEND) {
            const int slot = a.slot[tok], at = a.at[tok];
            if (slot < 0 || slot >= a.n_slots || at < 0 || at >= a.room) {
                report(a.status, JNX_ERR_DEVICE_BOUNDS);
                continue;
            }
            o = (is_v ? a.v : a.k) + slot * a.slot_stride + at * a.k_row +
                (head - a.H - (is_v ? a.Hkv : 0)) * a.k_head;
        } else {
            o = a.k + tok * a.k_row + (head - a.H) * a.k_head;
        }
        *reinterpret_cast<uint4*>(o + part) = ulo;
        *reinterpret_cast<uint4*>(o + HD / 2 + part) = uhi;
    }
}

// Gradients.  A CTA walks blocks of TOK tokens; the gains' gradients stay in its lanes'
// registers, query heads' and key heads' rows apart, and are added over the CTA's rows
// in a fixed order at the end.
template <int HD>
__global__ void __launch_bounds__(rope::THREADS)
    k_qk_norm_rope_bwd(const __grid_constant__ rope::Args a) {
    using C = RopeCfg<HD>;
    __shared__ float2 cs[C::TOK][HD / 2];
    __shared__ float sums[C::RPP][HD];
    pdl_entry();
    const int heads = a.H + a.Hkv;
    const int part = threadIdx.x % C::LPR * 8, lane_row = threadIdx.x / C::LPR;
    float gacc[2][16] = {};
    for (int t0 = blockIdx.x * C::TOK; t0 < a.n_tokens; t0 += gridDim.x * C::TOK) {
        const int nt = min(C::TOK, a.n_tokens - t0);
        __syncthreads();
        for (int i = threadIdx.x; i < nt * (HD / 2); i += rope::THREADS)
            cs[i / (HD / 2)][i % (HD / 2)] = rope::angle(a, t0 + i / (HD / 2), i % (HD / 2));
        __syncthreads();
        for (int r0 = 0; r0 < nt * heads; r0 += C::RPP) {
            const int r = r0 + lane_row;
            const bool live = r < nt * heads;
            const int t = live ? r / heads : 0, head = live ? r % heads : 0;
            const size_t tok = t0 + t;
            const bool is_q = head < a.H;
            uint4 xl = make_uint4(0, 0, 0, 0), xh = xl, yl = xl, yh = xl;
            if (live) {
                const uint16_t* x = a.qkv + tok * a.ldqkv + (size_t)head * HD + part;
                const uint16_t* dy = is_q ? a.q + tok * a.q_row + head * a.q_head
                                          : a.k + tok * a.k_row + (head - a.H) * a.k_head;
                xl = *reinterpret_cast<const uint4*>(x);
                xh = *reinterpret_cast<const uint4*>(x + HD / 2);
                yl = *reinterpret_cast<const uint4*>(dy + part);
                yh = *reinterpret_cast<const uint4*>(dy + HD / 2 + part);
            }
            float lo[8], hi[8], dl[8], dh[8];
            rope::unpack8(xl, lo);
            rope::unpack8(xh, hi);
            rope::unpack8(yl, dl);
            rope::unpack8(yh, dh);
#pragma unroll
            for (int e = 0; e < 8; ++e) {  // back by the same angle
                const float2 c = cs[t][part + e];
                const float x = dl[e], y = dh[e];
                dl[e] = x * c.x + y * c.y;
                dh[e] = y * c.x - x * c.y;
            }
            const uint16_t* gamma = is_q ? a.gq : a.gk;
            float ss = 0.f, dot = 0.f, gl[8] = {}, gh[8] = {};
            if (gamma) {
                rope::unpack8(*reinterpret_cast<const uint4*>(gamma + part), gl);
                rope::unpack8(*reinterpret_cast<const uint4*>(gamma + HD / 2 + part), gh);
            }
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                ss += lo[e] * lo[e] + hi[e] * hi[e];
                dot += gl[e] * dl[e] * lo[e] + gh[e] * dh[e] * hi[e];
            }
            ss = rope::row_sum<HD>(ss);
            dot = rope::row_sum<HD>(dot);
            if (!live) continue;
            if (gamma) {
                const float s = rsqrtf(ss * (1.f / HD) + a.eps);
                const float m = dot * (1.f / HD) * s * s * s;
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float vl = dl[e] * lo[e] * s, vh = dh[e] * hi[e] * s;
                    if (is_q) {
                        gacc[0][e] += vl;
                        gacc[0][8 + e] += vh;
                    } else {
                        gacc[1][e] += vl;
                        gacc[1][8 + e] += vh;
                    }
                    dl[e] = s * gl[e] * dl[e] - lo[e] * m;
                    dh[e] = s * gh[e] * dh[e] - hi[e] * m;
                }
            }
            uint16_t* o = a.dqkv + tok * a.ldqkv + (size_t)head * HD + part;
            *reinterpret_cast<uint4*>(o) = rope::pack8(dl);
            *reinterpret_cast<uint4*>(o + HD / 2) = rope::pack8(dh);
        }
    }
    if (!a.partial) return;
    for (int w = 0; w < 2; ++w) {
        __syncthreads();
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            sums[lane_row][part + e] = gacc[w][e];
            sums[lane_row][HD / 2 + part + e] = gacc[w][8 + e];
        }
        __syncthreads();
        for (int c = threadIdx.x; c < HD; c += rope::THREADS) {
            float s = 0.f;
            for (int r = 0; r < C::RPP; ++r) s += sums[r][c];
            a.partial[((size_t)blockIdx.x * 2 + w) * HD + c] = s;
        }
    }
}

// dgamma = sum of the CTAs' parts, each column's in a fixed order: 32 lanes take the
// parts in turn, then add up.  One warp a column.
__global__ void __launch_bounds__(256)
    k_qk_gain_sum(const float* partial, int parts, int hd, float* dgq, float* dgk) {
    pdl_entry();
    const int c = blockIdx.x * 8 + (threadIdx.x >> 5), lane = threadIdx.x & 31;
    if (c >= 2 * hd) return;
    float s = 0.f;
    for (int i = lane; i < parts; i += 32) s += partial[(size_t)i * 2 * hd + c];
#pragma unroll
    for (int o = 16; o; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
    if (lane == 0) {
        if (c < hd && dgq) dgq[c] = s;
        if (c >= hd && dgk) dgk[c - hd] = s;
    }
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
    a.half = p->head_dim / 2;
    a.eps = p->eps;
    a.gq = p->gamma_q;
    a.gk = p->gamma_k;
    for (int i = 0, axis = 0, end = p->n_axes ? p->sections[0] : 0; i < turned; ++i) {
        while (i >= end) end += p->sections[++axis];
        // theta^(-2 i / hd) / (2 pi), modulo whole turns, in units of 2^-64
        double f = std::pow((double)p->theta, -2.0 * i / p->head_dim) / 6.283185307179586476925;
        f -= std::floor(f);
        const double hi = std::floor(f * 4294967296.0);
        const double lo = std::floor((f * 4294967296.0 - hi) * 4294967296.0);
        a.turn[i] = ((unsigned long long)hi << 32) | (unsigned long long)lo;
        a.axis[i] = (unsigned char)axis;
    }
    return JNX_OK;
}

template <bool APPEND>
static jnx_status launch_rope(const rope::Args& a, int hd, const char* what, cudaStream_t s) {
    const int tok = hd == 64 ? RopeCfg<64>::TOK : hd == 128 ? RopeCfg<128>::TOK : RopeCfg<256>::TOK;
    const int grid = (a.n_tokens + tok - 1) / tok;
    TraceScope ts(JNX_K_QK_ROPE, 0.0, s);
    if (hd == 64)
        pdl(k_qk_norm_rope<64, APPEND>, grid, rope::THREADS, 0, s)(a);
    else if (hd == 128)
        pdl(k_qk_norm_rope<128, APPEND>, grid, rope::THREADS, 0, s)(a);
    else
        pdl(k_qk_norm_rope<256, APPEND>, grid, rope::THREADS, 0, s)(a);
    return launched(what);
}

// CTAs of the gradient kernel: what the SMs hold at once, or one a block of tokens.
static int rope_bwd_grid(int hd, int n_tokens) {
    const int tok = hd == 64 ? RopeCfg<64>::TOK : hd == 128 ? RopeCfg<128>::TOK : RopeCfg<256>::TOK;
    return std::max(1, std::min((n_tokens + tok - 1) / tok, 152 * 3));
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
    return launch_rope<false>(a, p->head_dim, "qk norm rope", static_cast<cudaStream_t>(stream));
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
    if ((a.H && !rows_ok(q)) || !cache_ok(cache) || !slot || !at)
        return fail(JNX_ERR_INVALID_ARG, "qk norm rope append: null or misaligned argument");
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
    return launch_rope<true>(a, p->head_dim, "qk norm rope append",
                             static_cast<cudaStream_t>(stream));
}

extern "C" size_t jnx_op_qk_norm_rope_backward_workspace_bytes(const jnx_qk_rope* p,
                                                               int32_t n_tokens) {
    if (!p || n_tokens < 0 || p->head_dim <= 0) return 0;
    return (size_t)rope_bwd_grid(p->head_dim, n_tokens) * 2 * p->head_dim * sizeof(float);
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
    const int grid = rope_bwd_grid(hd, n_tokens);
    TraceScope ts(JNX_K_QK_ROPE, 0.0, s);
    if (hd == 64)
        pdl(k_qk_norm_rope_bwd<64>, grid, rope::THREADS, 0, s)(a);
    else if (hd == 128)
        pdl(k_qk_norm_rope_bwd<128>, grid, rope::THREADS, 0, s)(a);
    else
        pdl(k_qk_norm_rope_bwd<256>, grid, rope::THREADS, 0, s)(a);
    if (gains)
        pdl(k_qk_gain_sum, (2 * hd + 7) / 8, 256, 0, s)(a.partial, grid, hd, a.gq ? dgamma_q : nullptr,
                                                       a.gk ? dgamma_k : nullptr);
    return launched("qk norm rope backward");
}
