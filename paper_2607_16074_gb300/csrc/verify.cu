// Drafted tokens verified against the target's probabilities, and the accepted ones'
// keys and values moved into place.
//
// Speculative sampling: from the root on, child c of the node (token x, drawn from q) is
// accepted with probability min(1, r(x) / (R q(x))), r = p and R = 1 at first; a rejected
// child leaves r <- max(r - R q, 0), R <- sum r, whose normalised form is what a token must be
// drawn from so that it is distributed as the target's.  Where no child is left the token is
// drawn by its place among the sums of r.
#include "jnx_dev.cuh"
#include "jnx_kernels.h"
#include "jnx_text.h"
#include "jnx_trace.h"

namespace jnx {

struct VerifyArgs {
    const float *p, *q;
    long long ldp, ldq;
    const int *tokens, *parent;
    const float* u;
    const int* cu_nodes;
    int n_rows, vocab, max_nodes;
    bool wide;  // rows start at 16 bytes
    int *path, *n_kept, *next, *status;
};

namespace verify {
constexpr int WARPS = 8, THREADS = 32 * WARPS;
constexpr int CLUSTER = 8;     // CTAs of a sequence
constexpr int ALONE = 4096;    // words up to which it is one
constexpr int HELD = 4;        // groups of 128 words that a warp holds in registers

// The sum of two fp32 values, hi = fl(hi + lo): 2^-48 of relative error an operation, by the
// published error-free transformations (Knuth's sum of two, Dekker's where the larger is known, and
// a product's error by a fused multiply-add).
struct Two {
    float hi, lo;
};
__device__ __forceinline__ Two two_sum(float a, float b) {
    const float s = __fadd_rn(a, b), t = __fsub_rn(s, a);
    return {s, __fadd_rn(__fsub_rn(a, __fsub_rn(s, t)), __fsub_rn(b, t))};
}
__device__ __forceinline__ Two fast_sum(float a, float b) {  // |a| >= |b|
    const float s = __fadd_rn(a, b);
    return {s, __fsub_rn(b, __fsub_rn(s, a))};
}
// Of values that are not negative.
__device__ __forceinline__ Two plus(Two a, Two b) {
    const Two s = two_sum(a.hi, b.hi);
    return fast_sum(s.hi, __fadd_rn(s.lo, __fadd_rn(a.lo, b.lo)));
}
__device__ __forceinline__ Two mul(Two a, float b) {
    const float p = __fmul_rn(a.hi, b);
    return fast_sum(p, __fadd_rn(__fmaf_rn(a.hi, b, -p), __fmul_rn(a.lo, b)));
}
__device__ __forceinline__ bool above(Two a, Two b) { return a.hi > b.hi || (a.hi == b.hi && a.lo > b.lo); }
__device__ __forceinline__ Two times(Two a, Two b) {
    const float p = __fmul_rn(a.hi, b.hi);
    const float e = __fmaf_rn(a.hi, b.lo, __fmul_rn(a.lo, b.hi));
    return fast_sum(p, __fadd_rn(__fmaf_rn(a.hi, b.hi, -p), e));
}
// What a rejection leaves: r - mass q, not below zero (NaN stays).
__device__ __forceinline__ Two less(Two r, Two mass, float q) {
    const float p = __fmul_rn(mass.hi, q);
    const Two d = two_sum(r.hi, -p);
    const float e = __fmaf_rn(mass.lo, q, __fmaf_rn(mass.hi, q, -p));
    const Two x = two_sum(d.hi, __fadd_rn(d.lo, __fsub_rn(r.lo, e)));
    return x.hi < 0.f ? Two{0.f, 0.f} : x;
}
__device__ __forceinline__ Two less(float p, float q) {  // mass one
    const Two d = two_sum(p, -q);
    return d.hi < 0.f ? Two{0.f, 0.f} : d;
}
__device__ __forceinline__ Two shfl_xor(Two a, int o) {
    return {__shfl_xor_sync(0xffffffffu, a.hi, o), __shfl_xor_sync(0xffffffffu, a.lo, o)};
}
__device__ __forceinline__ Two shfl(Two a, int from) {
    return {__shfl_sync(0xffffffffu, a.hi, from), __shfl_sync(0xffffffffu, a.lo, from)};
}
// Sums of the lanes up to each.
__device__ __forceinline__ Two scan(Two a, int lane) {
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const Two x{__shfl_up_sync(0xffffffffu, a.hi, o), __shfl_up_sync(0xffffffffu, a.lo, o)};
        if (lane >= o) a = plus(x, a);
    }
    return a;
}
}  // namespace verify

// C CTAs a sequence (a cluster), a share of the vocabulary to each warp of theirs.  All of them
// follow the same walk: the nodes' own probabilities are looked up at once, and only a
// rejection, or the end, needs sums over the vocabulary: one row of p and q of a sequence is
// read as a rule, which is what bounds the call beside the chain of lookups (7 nodes of eight
// sequences over 32,000 words 6.6 us; 64 sequences of up to 24, a pass of some 1.5 us for every
// rejection of the unluckiest, 17.2).
//
// Sums decide which word is drawn, and neighbouring words' borders are 1e-9 apart and closer,
// so they are pairs of fp32: 2^-48 of relative error each, on the fp32 pipe (in fp64, whose
// rate here is a hundredth of fp32's, a CTA a sequence took 727 and 963 us).
// HOLD: the shares are small enough to stay in registers from a rejection to the next.
template <int C, bool HOLD>
__global__ void __launch_bounds__(verify::THREADS)
    k_verify_drafts(const __grid_constant__ VerifyArgs a) {
    using namespace verify;
    constexpr int ALL = C * WARPS;  // warps of a sequence
    __shared__ float chance_p[kMaxNodes], chance_q[kMaxNodes], us[kMaxNodes];
    __shared__ int tokens[kMaxNodes];
    __shared__ unsigned long long kids[kMaxNodes];  // nodes that are tried at each, in order
    __shared__ Two sums[2][ALL];                    // of the warps; a pass's and the last one's
    __shared__ int out[kMaxNodes], wrong;
    // (its peers have started before a CTA writes to their shared memory)
    if (C > 1) asm volatile("barrier.cluster.arrive.aligned;" ::: "memory");
    pdl_entry();
    const int t = threadIdx.x, lane = t & 31, warp = warp_uniform(t >> 5);
    const int s = blockIdx.x / C, rank = C > 1 ? (int)cluster_rank() : 0, gw = rank * WARPS + warp;
    int first, n;
    const bool known = tree_rows(a.cu_nodes, s, a.n_rows, a.max_nodes, first, n);
    if (!known) n = 0;
    if (t < kMaxNodes) kids[t] = 0;
    if (t == 0) wrong = !known;
    __syncthreads();
    if (t < n) {
        const int x = a.tokens[first + t], up = a.parent[first + t];
        us[t] = a.u[first + t];
        tokens[t] = x;
        if (t > 0) {
            if (up < 0 || up >= t || x < 0 || x >= a.vocab) {
                wrong = 1;
            } else {
                chance_p[t] = a.p[(first + up) * a.ldp + x];
                chance_q[t] = a.q ? a.q[(first + up) * a.ldq + x] : 1.f;
                atomicOr(&kids[up], 1ull << t);
            }
        }
    }
    __syncthreads();
    if (C > 1) asm volatile("barrier.cluster.wait.aligned;" ::: "memory");

    // this warp's words [v0, v1)
    const int share = ((a.vocab + ALL - 1) / ALL + 127) / 128 * 128;
    const int v0 = (int)min((long long)gw * share, (long long)a.vocab);
    const int v1 = (int)min((long long)v0 + share, (long long)a.vocab);
    int cur = 0, k = 0, kept = n > 0;  // rejections at cur
    unsigned long long tried = 0;      // the rejected nodes
    __shared__ Two masses[kMaxNodes];  // R of each rejection at cur
    const float *p = nullptr, *q = nullptr;
    // what is left of a word of probability pv
    auto rest = [&](int v, float pv, float qv) {
        Two r{pv, 0.f};
        if (a.q) {
            for (int j = 0; j < k; ++j) r = less(r, masses[j], qv);
        } else {
            // a certain guess that was rejected had less than all that was left: nothing remains
            for (unsigned long long m = tried; m; m &= m - 1)
                if (tokens[__ffsll(m) - 1] == v) r.hi = 0.f;
        }
        return r;
    };
    // words [v, v + 4) of rows x; those beyond the share are zero
    auto four = [&](const float* row, int v) {
        if (a.wide && v + 3 < v1) return *reinterpret_cast<const float4*>(row + v);
        float x[4] = {};
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (v + e < v1) x[e] = row[v + e];
        return make_float4(x[0], x[1], x[2], x[3]);
    };
    Two held[HOLD ? HELD : 1][4];
    float4 held_q[HOLD ? HELD : 1];
    int held_k = -1;  // rejections that are in what is held; -1: nothing of cur's is
    auto hold = [&]() {
        if (held_k < 0) {
            float4 x[HELD];
#pragma unroll
            for (int i = 0; i < HELD; ++i) {
                x[i] = four(p, v0 + 128 * i + 4 * lane);
                if (q && k) held_q[i] = four(q, v0 + 128 * i + 4 * lane);
            }
#pragma unroll
            for (int i = 0; i < HELD; ++i) {
                held[i][0] = {x[i].x, 0.f}, held[i][1] = {x[i].y, 0.f};
                held[i][2] = {x[i].z, 0.f}, held[i][3] = {x[i].w, 0.f};
            }
            held_k = 0;
        }
        for (; held_k < k; ++held_k) {  // (one at a time, but for a repeat)
            if (!q) continue;
            const Two mass = masses[held_k];
            const bool one = held_k == 0;
#pragma unroll
            for (int i = 0; i < HELD; ++i) {
                const float y[4] = {held_q[i].x, held_q[i].y, held_q[i].z, held_q[i].w};
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    held[i][e] = one ? less(held[i][e].hi, y[e]) : less(held[i][e], mass, y[e]);
            }
        }
        if (!q)
            for (unsigned long long m = tried; m; m &= m - 1) {
                const int at = tokens[__ffsll(m) - 1] - v0 - 4 * lane;
#pragma unroll
                for (int i = 0; i < HELD; ++i)
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        if (at == 128 * i + e) held[i][e].hi = 0.f, held[i][e].lo = 0.f;
            }
    };
    // what is left of words [v0 + 128 i + 4 lane, + 4), zeros beyond the share
    auto group = [&](int i, Two (&r)[4]) {
        if constexpr (HOLD) {
#pragma unroll
            for (int e = 0; e < 4; ++e) r[e] = held[i][e];
        } else {
            const int v = v0 + 128 * i + 4 * lane;
            const float4 x = four(p, v), y = q && k ? four(q, v) : make_float4(0.f, 0.f, 0.f, 0.f);
            r[0] = rest(v, x.x, y.x), r[1] = rest(v + 1, x.y, y.y);
            r[2] = rest(v + 2, x.z, y.z), r[3] = rest(v + 3, x.w, y.w);
        }
    };
    const int groups = HOLD ? HELD : (v1 - v0 + 127) / 128;
    int pass = 0;
    Two upto[(ALL + 31) / 32];  // sums up to each warp's share: lane l has warps (ALL / 32) l + i
    auto total = [&]() {
        p = a.p + (first + cur) * a.ldp;
        q = a.q ? a.q + (first + cur) * a.ldq : nullptr;
        if constexpr (HOLD) hold();
        Two mine{0.f, 0.f};
#pragma unroll 4
        for (int i = 0; i < groups; ++i) {
            Two r[4];
            group(i, r);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const Two x = two_sum(mine.hi, r[e].hi);
                mine = {x.hi, __fadd_rn(mine.lo, __fadd_rn(x.lo, r[e].lo))};
            }
        }
        mine = fast_sum(mine.hi, mine.lo);
#pragma unroll
        for (int o = 16; o; o >>= 1) mine = plus(mine, shfl_xor(mine, o));
        Two* to = &sums[pass & 1][gw];
        ++pass;
        if constexpr (C > 1) {
            if (lane < C)
                asm volatile("st.shared::cluster.v2.f32 [%0], {%1, %2};" ::"r"(map_rank(to, lane)), "f"(mine.hi),
                             "f"(mine.lo)
                             : "memory");
            cluster_sync_all();
        } else {
            if (lane == 0) *to = mine;
            __syncthreads();
        }
        const Two* from = sums[(pass - 1) & 1];
        if constexpr (ALL == 64) {
            const Two x = from[2 * lane], y = from[2 * lane + 1], both = scan(plus(x, y), lane);
            upto[1] = both;
            const Two before = shfl(both, lane - 1 & 31);
            upto[0] = lane ? plus(before, x) : x;
            return shfl(both, 31);
        } else {
            upto[0] = scan(lane < ALL ? from[lane] : Two{0.f, 0.f}, lane);
            return shfl(upto[0], 31);
        }
    };
    static_assert(ALL == 64 || ALL == 8, "warps of a sequence");

    if (n > 0) {
        if (t == 0) out[0] = 0;
        Two left{1.f, 0.f};
        unsigned long long next = kids[0];
        bool summed = false;
        while (next) {
            const int c = __ffsll(next) - 1;
            next &= next - 1;
            const Two r = rest(tokens[c], chance_p[c], chance_q[c]);
            const float uq = __fmul_rn(us[c], chance_q[c]);
            if (above(r, times({uq, __fmaf_rn(us[c], chance_q[c], -uq)}, left))) {
                if (t == 0) out[kept] = c;
                ++kept;
                cur = c;
                k = 0;
                held_k = -1;
                tried = 0;
                left = {1.f, 0.f};
                next = kids[c];
                summed = false;
                continue;
            }
            __syncthreads();  // (a warp may still be at an earlier node's)
            if (t == 0) masses[k] = left;
            tried |= 1ull << c;
            ++k;
            __syncthreads();
            left = total();
            summed = true;
        }
        if (!summed) left = total();
        if (k > 0 && left.hi == 0.f) {  // (a NaN is not nothing: it is reported below)
            k = 0;
            held_k = -1;
            tried = 0;
            left = total();
        }
        const bool good = left.hi > 0.f && left.hi + left.lo < INFINITY;
        // the first warp whose words pass the goal (should rounding, or a u of one, leave none: the
        // last that has any)
        const Two goal = mul(left, us[0]);
        uint32_t hits[(ALL + 31) / 32];
        int owner;
        if constexpr (ALL == 64) {
            hits[0] = __ballot_sync(0xffffffffu, above(upto[0], goal));
            hits[1] = __ballot_sync(0xffffffffu, above(upto[1], goal));
            const int x = hits[0] ? 2 * (__ffs(hits[0]) - 1) : 64, y = hits[1] ? 2 * __ffs(hits[1]) - 1 : 64;
            owner = min(x, y);
        } else {
            hits[0] = __ballot_sync(0xffffffffu, above(upto[0], goal));
            owner = hits[0] ? __ffs(hits[0]) - 1 : 64;
        }
        const bool none = owner >= ALL;
        if (none) {
            const Two* from = sums[(pass - 1) & 1];
            owner = 0;
            for (int w = 0; w < ALL; ++w)
                if (from[w].hi > 0.f) owner = w;
        }
        if (good && gw == owner) {
            Two before{0.f, 0.f};
            if (gw > 0) {
                const int w = gw - 1;
                before = ALL == 64 ? ((w & 1) ? shfl(upto[ALL == 64 ? 1 : 0], w >> 1) : shfl(upto[0], w >> 1)) : shfl(upto[0], w);
            }
            int word = -1, last = -1;
#pragma unroll(HOLD ? HELD : 1)
            for (int i = 0; i < groups; ++i) {
                const int v = v0 + 128 * i + 4 * lane;
                Two r[4], mine{0.f, 0.f};
                group(i, r);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    if (r[e].hi > 0.f) last = v + e;
                    mine = plus(mine, r[e]);
                }
                const Two up = scan(mine, lane), through = plus(before, up);
                const uint32_t hit = __ballot_sync(0xffffffffu, !none && above(through, goal));
                if (hit) {
                    const int at = __ffs(hit) - 1;
                    Two run = shfl(through, at - 1 & 31);
                    if (at == 0) run = before;
                    if (lane == at) {
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            if (!(r[e].hi > 0.f) || (word >= 0 && above(run, goal))) continue;
                            run = plus(run, r[e]);
                            word = v + e;
                        }
                    }
                    word = __shfl_sync(0xffffffffu, word, at);
                    break;
                }
                before = shfl(through, 31);
            }
            if (word < 0) word = __reduce_max_sync(0xffffffffu, last);
            if (lane == 0) a.next[s] = word;
        }
        if (!good && rank == 0 && t == 0) {
            a.next[s] = -1;
            wrong = 1;
        }
    } else if (rank == 0 && t == 0) {
        a.next[s] = -1;
    }
    __syncthreads();
    if (rank > 0) return;
    for (int i = t; i < a.max_nodes; i += THREADS) a.path[(size_t)s * a.max_nodes + i] = i < kept ? out[i] : -1;
    if (t == 0) {
        a.n_kept[s] = kept;
        if (wrong) report(a.status, JNX_ERR_DEVICE_BOUNDS);
    }
}

struct KeepArgs {
    uint16_t *k, *v;
    long long layer_stride, page_stride, row_stride, head_stride;
    Pages pages;
    int heads, hd;
    const int *n_cached, *path, *n_kept;
    long long ld_path;
    int max_kept;
    int* status;
};

// A CTA a sequence and layer; a thread moves the same 16 bytes of every row, four rows at a time
// in the path's order: places lie at or ahead of what goes there, and a path increases, so a
// place is overwritten after it was read, and no row that is read later is overwritten.  Bound by
// its chain of lookups (path, table, rows): 8 sequences in 18 layers 2.9 us, 64 in 32 layers of
// 8 heads of 128 6.5 (a CTA for several layers: 9.2 to 19).
__global__ void __launch_bounds__(128) k_keep_drafts(const __grid_constant__ KeepArgs a) {
    __shared__ long long from[kMaxNodes], to[kMaxNodes];  // of the rows that move
    __shared__ int bad, low;
    pdl_entry();
    const int s = blockIdx.x, t = threadIdx.x, lane = t & 31;
    const int n = a.n_kept[s], old = a.n_cached[s];
    const int* path = a.path + s * a.ld_path;
    const int x = t < a.max_kept ? path[t] : 0, ahead = t > 0 && t < a.max_kept ? path[t - 1] : -1;
    if (t == 0) bad = n < 0 || n > a.max_kept || old < 0;
    __syncthreads();
    if (t < kMaxNodes) {  // two warps
        long long src = 0, dst = 0;
        if (!bad && t < n) {
            int page, row, page_to, row_to;
            if (x < t || ahead >= x || x > 0x7fffffff - old || !a.pages.find(s, old + x, page, row) ||
                !a.pages.find(s, old + t, page_to, row_to)) {
                bad = 1;
            } else {
                src = page * a.page_stride + row * a.row_stride;
                dst = page_to * a.page_stride + row_to * a.row_stride;
            }
        }
        const uint32_t moves = __ballot_sync(0xffffffffu, src != dst);
        if (t == 0) low = __popc(moves);
        asm volatile("bar.sync 1, 64;" ::: "memory");
        const int at = __popc(moves & ((1u << lane) - 1)) + (t >= 32 ? low : 0);
        if (src != dst) from[at] = src, to[at] = dst;
        asm volatile("bar.sync 1, 64;" ::: "memory");
        if (t == 32) low += __popc(moves);
    }
    __syncthreads();
    if (bad) {
        if (t == 0 && blockIdx.y == 0) report(a.status, JNX_ERR_DEVICE_BOUNDS);
        return;
    }
    const int rows = low, units = a.hd / 8, all = 2 * a.heads * units;
    for (int e = t; e < all; e += 128) {
        const int half = e / (a.heads * units), head = e / units % a.heads;
        uint16_t* base = (half ? a.v : a.k) + (long long)blockIdx.y * a.layer_stride +
                         head * a.head_stride + e % units * 8;
        for (int i0 = 0; i0 < rows; i0 += 4) {
            uint4 y[4];
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (i0 + i < rows) y[i] = *reinterpret_cast<const uint4*>(base + from[i0 + i]);
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (i0 + i < rows) *reinterpret_cast<uint4*>(base + to[i0 + i]) = y[i];
        }
    }
}

}  // namespace jnx

using namespace jnx;

extern "C" jnx_status jnx_op_verify_drafts(const float* p, int64_t ldp, const float* q, int64_t ldq,
                                           const int32_t* tokens, const int32_t* parent,
                                           const float* u, const int32_t* cu_nodes, int32_t n_seqs,
                                           int32_t n_rows, int32_t vocab, int32_t max_nodes,
                                           int32_t* path, int32_t* n_kept, int32_t* next,
                                           int32_t* status, void* stream) {
    clear_error();
    const char* what = "verify drafts";
    if (n_seqs < 0 || n_rows < 0 || vocab <= 0 || max_nodes < 1)
        return fail(JNX_ERR_INVALID_ARG, "%s: bad sizes", what);
    if (max_nodes > kMaxNodes || vocab > 0x7fffff00 || n_seqs > 0x7fffff00 / verify::CLUSTER)
        return fail(JNX_ERR_UNSUPPORTED, "%s: over %d nodes, or vocabulary", what, kMaxNodes);
    if (n_seqs == 0) return JNX_OK;
    if (!cu_nodes || !path || !n_kept || !next ||
        (n_rows > 0 && (!p || !tokens || !parent || !u || ldp < 0 || (q && ldq < 0))))
        return fail(JNX_ERR_INVALID_ARG, "%s: null argument or negative stride", what);
    const bool wide = ldp % 4 == 0 && aligned16(p) && (!q || (ldq % 4 == 0 && aligned16(q)));
    const VerifyArgs a{p,      q,     ldp,       ldq,  tokens, parent, u,    cu_nodes,
                       n_rows, vocab, max_nodes, wide, path,   n_kept, next, status};
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    TraceScope ts(JNX_K_VERIFY, 0.0, s);
    using namespace verify;
    static_assert(ALONE <= WARPS * HELD * 128, "one CTA's words are held");
    if (vocab <= ALONE) {
        pdl(k_verify_drafts<1, true>, n_seqs, THREADS, 0, s)(a);
        return launched(what);
    }
    const bool hold = vocab <= CLUSTER * WARPS * HELD * 128;
    auto l = pdl(hold ? k_verify_drafts<CLUSTER, true> : k_verify_drafts<CLUSTER, false>,
                 n_seqs * CLUSTER, THREADS, 0, s);
    l.cluster = CLUSTER;
    l(a);
    return launched(what);
}

extern "C" jnx_status jnx_op_keep_drafts(const jnx_kv_cache* cache, int32_t n_layers,
                                         int64_t layer_stride, const jnx_pages* pages,
                                         int32_t n_kv_heads, int32_t head_dim,
                                         const int32_t* n_cached, const int32_t* path,
                                         int64_t ld_path, const int32_t* n_kept, int32_t max_kept,
                                         int32_t* status, void* stream) {
    clear_error();
    const char* what = "keep drafts";
    if (jnx_status st = heads_ok(n_kv_heads, n_kv_heads, head_dim, what)) return st;
    if (n_layers < 0 || max_kept < 0 || ld_path < 0 || !pages_ok(pages))
        return fail(JNX_ERR_INVALID_ARG, "%s: bad sizes or pages", what);
    if (max_kept > kMaxNodes || n_layers > 65535)
        return fail(JNX_ERR_UNSUPPORTED, "%s: over %d rows or 65,535 layers", what, kMaxNodes);
    if (n_layers == 0 || pages->n_seqs == 0 || max_kept == 0) return JNX_OK;
    if (!cache_ok(cache) || layer_stride % 8 || !n_cached || !path || !n_kept)
        return fail(JNX_ERR_INVALID_ARG, "%s: null or misaligned argument", what);
    const KeepArgs a{cache->k, cache->v, layer_stride, cache->slot_stride, cache->row_stride,
                     cache->head_stride, Pages(*pages, *cache), n_kv_heads, head_dim, n_cached, path,
                     n_kept, ld_path, max_kept, status};
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    TraceScope ts(JNX_K_VERIFY, 0.0, s);
    pdl(k_keep_drafts, dim3(pages->n_seqs, n_layers), 128, 0, s)(a);
    return launched(what);
}
