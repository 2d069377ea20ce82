// Attention of trees of drafted tokens against a paged cache.
//
// Node i of a sequence sees the cached tokens and the nodes that its bits name, whose keys
// and values lie behind the cached ones: O = softmax(Q K^T / sqrt(hd)) V over them, in one
// pass with a running maximum and sum.
#include "jnx_dev.cuh"
#include "jnx_kernels.h"
#include "jnx_text.h"
#include "jnx_trace.h"

namespace jnx {

struct TreeArgs {
    const uint16_t *k, *v;
    long long page_stride, kv_row, kv_head;
    Pages pages;
    int H, Hkv, group, n_rows;
    float scale_log2;
    const uint16_t* q;
    long long q_row, q_head;
    uint16_t* out;
    long long o_row, o_head;
    const int *cu_nodes, *n_cached;
    const unsigned long long* sees;
    int* status;
};

// A warp a node and head, a token at a time.
template <int HD>
__global__ void __launch_bounds__(128) k_tree_attn(const __grid_constant__ TreeArgs a) {
    constexpr int E = HD / 32;
    pdl_entry();
    const int s = blockIdx.x, lane = threadIdx.x & 31;
    int first, n;
    if (!tree_rows(a.cu_nodes, s, a.n_rows, kMaxNodes, first, n)) {
        if (threadIdx.x == 0 && blockIdx.y == 0) report(a.status, JNX_ERR_DEVICE_BOUNDS);
        return;
    }
    int old = a.n_cached[s], all = old + n;
    if (old < 0 || (long long)old + n > (long long)a.pages.max_pages * a.pages.room) {
        if (threadIdx.x == 0 && blockIdx.y == 0) report(a.status, JNX_ERR_DEVICE_BOUNDS);
        old = all = 0;
    }
    for (int w = blockIdx.y * 4 + (threadIdx.x >> 5); w < n * a.H; w += gridDim.y * 4) {
        const int i = w / a.H, h = w % a.H, g = h / a.group;
        const unsigned long long see = a.sees[first + i];
        float q[E], o[E] = {}, m = -INFINITY, l = 0.f;
#pragma unroll
        for (int e = 0; e < E; ++e)
            q[e] = bf2f(a.q[(first + i) * a.q_row + h * a.q_head + e * 32 + lane]);
        for (int j = 0; j < all; ++j) {
            if (j >= old && !(see >> (j - old) & 1)) continue;
            int page, row;
            const bool there = a.pages.find(s, j, page, row);
            if (!there && lane == 0) report(a.status, JNX_ERR_DEVICE_BOUNDS);
            const long long at = there ? page * a.page_stride + row * a.kv_row + g * a.kv_head : 0;
            float x = 0.f;
#pragma unroll
            for (int e = 0; e < E; ++e)
                if (there) x = fmaf(q[e], bf2f(a.k[at + e * 32 + lane]), x);
#pragma unroll
            for (int d = 16; d; d >>= 1) x += __shfl_xor_sync(0xffffffffu, x, d);
            x *= a.scale_log2;
            const float top = fmaxf(m, x), alpha = ex2_approx(m - top), p = ex2_approx(x - top);
            m = top;
            l = l * alpha + p;
#pragma unroll
            for (int e = 0; e < E; ++e)
                o[e] = o[e] * alpha + (there ? p * bf2f(a.v[at + e * 32 + lane]) : 0.f);
        }
        const float inv = l > 0.f ? 1.f / l : 0.f;
#pragma unroll
        for (int e = 0; e < E; ++e)
            a.out[(first + i) * a.o_row + h * a.o_head + e * 32 + lane] = f2bf(o[e] * inv);
    }
}

}  // namespace jnx

using namespace jnx;

extern "C" size_t jnx_op_tree_attention_workspace_bytes(int32_t n_seqs, int32_t n_rows,
                                                        int32_t n_heads, int32_t head_dim,
                                                        int64_t max_tokens) {
    (void)n_seqs, (void)n_rows, (void)n_heads, (void)head_dim, (void)max_tokens;
    return 0;
}

extern "C" jnx_status jnx_op_tree_attention(const jnx_kv_cache* cache, const jnx_pages* pages,
                                            int32_t n_heads, int32_t n_kv_heads, int32_t head_dim,
                                            int32_t n_rows, const jnx_head_rows* q,
                                            const int32_t* cu_nodes, const int32_t* n_cached,
                                            const uint64_t* sees, const jnx_head_rows* out,
                                            void* workspace, size_t ws_bytes, int32_t* status,
                                            void* stream) {
    clear_error();
    const char* what = "tree attention";
    (void)workspace, (void)ws_bytes;
    if (jnx_status st = heads_ok(n_heads, n_kv_heads, head_dim, what)) return st;
    if (n_rows < 0 || !pages_ok(pages)) return fail(JNX_ERR_INVALID_ARG, "%s: bad sizes or pages", what);
    if (n_rows == 0 || pages->n_seqs == 0) return JNX_OK;
    if (!cache_ok(cache) || !rows_ok(q) || !rows_ok(out) || !cu_nodes || !n_cached || !sees)
        return fail(JNX_ERR_INVALID_ARG, "%s: null or misaligned argument", what);
    if (pages->max_pages > 1 && cache->room % 16)
        return fail(JNX_ERR_UNSUPPORTED, "%s: pages of %d tokens, no multiple of 16", what, cache->room);
    if ((int64_t)pages->max_pages * cache->room > 0x7fffff00)
        return fail(JNX_ERR_UNSUPPORTED, "%s: sequences of over 2^31 tokens", what);
    const TreeArgs a{cache->k, cache->v, cache->slot_stride, cache->row_stride, cache->head_stride,
                     Pages(*pages, *cache), n_heads, n_kv_heads, n_heads / n_kv_heads, n_rows,
                     (float)(1.4426950408889634 / sqrt((double)head_dim)), q->ptr, q->row_stride,
                     q->head_stride, out->ptr, out->row_stride, out->head_stride, cu_nodes, n_cached,
                     reinterpret_cast<const unsigned long long*>(sees), status};
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    TraceScope ts(JNX_K_TREE_ATTN, 0.0, s);
    const dim3 grid(pages->n_seqs, 64);
    if (head_dim == 64) pdl(k_tree_attn<64>, grid, 128, 0, s)(a);
    else if (head_dim == 128) pdl(k_tree_attn<128>, grid, 128, 0, s)(a);
    else pdl(k_tree_attn<256>, grid, 128, 0, s)(a);
    return launched(what);
}
