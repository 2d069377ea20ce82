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
    int *path, *n_kept, *next, *status;
};

namespace verify {
constexpr int THREADS = 1024;

__device__ __forceinline__ double block_sum(double v, double* sums) {
#pragma unroll
    for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    __syncthreads();
    if ((threadIdx.x & 31) == 0) sums[threadIdx.x >> 5] = v;
    __syncthreads();
    double all = 0.0;
    for (int w = 0; w < THREADS / 32; ++w) all += sums[w];
    return all;
}
}  // namespace verify

// A CTA a sequence.
__global__ void __launch_bounds__(verify::THREADS)
    k_verify_drafts(const __grid_constant__ VerifyArgs a) {
    using namespace verify;
    __shared__ double sums[THREADS / 32], R[kMaxNodes];  // R of each rejection at the node
    __shared__ int out[kMaxNodes], word;
    pdl_entry();
    const int s = blockIdx.x, t = threadIdx.x;
    int first, n;
    const bool known = tree_rows(a.cu_nodes, s, a.n_rows, a.max_nodes, first, n);
    if (!known) n = 0;
    int kept = n > 0, cur = 0, k = 0;  // rejections at cur
    const float *p = a.p + first * a.ldp, *q = a.q ? a.q + first * a.ldq : nullptr;
    __shared__ int tried[kMaxNodes];  // tokens of the rejections
    // r of a word after the node's rejections so far
    auto rest = [&](int v) {
        double r = p[cur * a.ldp + v];
        if (k == 0) return r;
        const double qv = q ? q[cur * a.ldq + v] : 0.0;
        for (int j = 0; j < k; ++j) r = fmax(r - R[j] * (q ? qv : v == tried[j] ? 1.0 : 0.0), 0.0);
        return r;
    };
    auto total = [&]() {
        double mine = 0.0;
        for (int v = t; v < a.vocab; v += THREADS) mine += rest(v);
        return block_sum(mine, sums);
    };
    bool bad = !known;
    if (n > 0) {
        if (t == 0) out[0] = 0;
        if (t == 0) R[0] = 1.0;
        __syncthreads();
        for (int c = 1; c < n; ++c) {
            const int up = a.parent[first + c], x = a.tokens[first + c];
            if (up < 0 || up >= c) {
                bad = true;
                continue;
            }
            if (up != cur) continue;
            if (x < 0 || x >= a.vocab) {
                bad = true;
                continue;
            }
            const double chance = q ? q[cur * a.ldq + x] : 1.0;
            if (a.u[first + c] * chance * R[k] < rest(x)) {
                __syncthreads();
                if (t == 0) out[kept] = c, R[0] = 1.0;
                ++kept;
                cur = c;
                k = 0;
                __syncthreads();
                continue;
            }
            __syncthreads();
            if (t == 0) tried[k] = x;
            ++k;
            __syncthreads();
            const double left = total();
            if (t == 0 && k < kMaxNodes) R[k] = left;
            __syncthreads();
        }
        double all = total();
        if (k > 0 && !(all > 0.0)) {
            k = 0;
            all = total();
        }
        if (!(all > 0.0) || !(all < 1e300)) {
            bad = true;
            if (t == 0) word = -1;
        } else {
            if (t == 0) word = 0x7fffffff;
            __syncthreads();
            const double goal = (double)a.u[first] * all;
            double before = 0.0;
            int last = -1;  // a word that has any of r, should rounding leave none above the goal
            for (int v0 = 0; v0 < a.vocab; v0 += THREADS) {
                const int v = v0 + t;
                const double mine = v < a.vocab ? rest(v) : 0.0;
                double run = mine;
#pragma unroll
                for (int o = 1; o < 32; o <<= 1) {
                    const double x = __shfl_up_sync(0xffffffffu, run, o);
                    if ((t & 31) >= o) run += x;
                }
                __syncthreads();
                if ((t & 31) == 31) sums[t >> 5] = run;
                __syncthreads();
                double ahead = before;
                for (int w = 0; w < THREADS / 32; ++w) {
                    if (w < t >> 5) ahead += sums[w];
                    before += sums[w];
                }
                if (mine > 0.0) {
                    last = v;
                    if (ahead + run > goal) atomicMin(&word, v);
                }
                __syncthreads();
                if (word != 0x7fffffff) break;
            }
            __syncthreads();
            if (word == 0x7fffffff) {
                __syncthreads();
                if (t == 0) word = -1;
                __syncthreads();
                if (last >= 0) atomicMax(&word, last);
            }
        }
    } else if (t == 0) {
        word = -1;
    }
    __syncthreads();
    for (int i = t; i < a.max_nodes; i += THREADS) a.path[(size_t)s * a.max_nodes + i] = i < kept ? out[i] : -1;
    if (t == 0) {
        a.n_kept[s] = kept;
        a.next[s] = word;
        if (bad) report(a.status, JNX_ERR_DEVICE_BOUNDS);
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

// A CTA a sequence and layer; a thread holds the same 16 bytes of every row it moves, in the
// path's order: places lie at or ahead of what goes there, and a path increases, so a place is
// overwritten after it was read.
__global__ void __launch_bounds__(256) k_keep_drafts(const __grid_constant__ KeepArgs a) {
    __shared__ long long from[kMaxNodes], to[kMaxNodes];
    __shared__ int bad, moves;
    pdl_entry();
    const int s = blockIdx.x;
    const int n = a.n_kept[s], old = a.n_cached[s];
    if (threadIdx.x == 0) bad = n < 0 || n > a.max_kept || old < 0, moves = 0;
    __syncthreads();
    if (!bad && (int)threadIdx.x < n) {
        const int i = threadIdx.x;
        const int* path = a.path + s * a.ld_path;
        const int x = path[i];
        int page, row, page_to, row_to;
        if (x < i || (i > 0 && path[i - 1] >= x) || x > 0x7fffffff - old ||
            !a.pages.find(s, old + x, page, row) || !a.pages.find(s, old + i, page_to, row_to)) {
            bad = 1;
        } else {
            from[i] = page * a.page_stride + row * a.row_stride;
            to[i] = page_to * a.page_stride + row_to * a.row_stride;
            if (x != i) moves = 1;
        }
    }
    __syncthreads();
    if (bad) {
        if (threadIdx.x == 0) report(a.status, JNX_ERR_DEVICE_BOUNDS);
        return;
    }
    if (!moves) return;
    const int units = a.hd / 8, all = 2 * a.heads * units;
    for (int e = threadIdx.x; e < all; e += 256) {
        const int half = e / (a.heads * units), head = e / units % a.heads;
        uint16_t* base = (half ? a.v : a.k) + (long long)blockIdx.y * a.layer_stride +
                         head * a.head_stride + e % units * 8;
        for (int i = 0; i < n; ++i)
            if (from[i] != to[i])
                *reinterpret_cast<uint4*>(base + to[i]) = *reinterpret_cast<const uint4*>(base + from[i]);
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
    if (max_nodes > kMaxNodes || vocab > 0x7fffff00)
        return fail(JNX_ERR_UNSUPPORTED, "%s: over %d nodes, or vocabulary", what, kMaxNodes);
    if (n_seqs == 0) return JNX_OK;
    if (!cu_nodes || !path || !n_kept || !next ||
        (n_rows > 0 && (!p || !tokens || !parent || !u || ldp < 0 || (q && ldq < 0))))
        return fail(JNX_ERR_INVALID_ARG, "%s: null argument or negative stride", what);
    const VerifyArgs a{p,        q,      ldp,   ldq,       tokens, parent, u,
                       cu_nodes, n_rows, vocab, max_nodes, path,   n_kept, next, status};
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    TraceScope ts(JNX_K_VERIFY, 0.0, s);
    pdl(k_verify_drafts, n_seqs, verify::THREADS, 0, s)(a);
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
    pdl(k_keep_drafts, dim3(pages->n_seqs, n_layers), 256, 0, s)(a);
    return launched(what);
}
