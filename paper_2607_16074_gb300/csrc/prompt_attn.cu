// Attention of packed prompts: causal behind a prefix that every row sees, query rows
// the last of a sequence's positions, grouped heads.
#include <algorithm>
#include <vector>

#include "jnx_dev.cuh"
#include "jnx_kernels.h"
#include "jnx_text.h"
#include "jnx_trace.h"

namespace jnx {

struct PromptArgs {
    const int *cu_q, *cu_kv, *prefix;
    const int2* items;
    int H, Hkv, group;
    float scale_log2;
    jnx_head_rows q, k, v, out;
    float* lse;
};

// One warp a row (token, head), one key at a time.
template <int HD>
__global__ void __launch_bounds__(256) k_prompt_attn(const __grid_constant__ PromptArgs a) {
    constexpr int E = HD / 32;
    pdl_entry();
    const int2 it = a.items[blockIdx.x / a.Hkv];
    const int kvh = blockIdx.x % a.Hkv, s = it.x;
    const int q0 = a.cu_q[s], Lq = a.cu_q[s + 1] - q0, k0 = a.cu_kv[s], Lk = a.cu_kv[s + 1] - k0;
    const int pre = a.prefix ? a.prefix[s] : 0, lane = threadIdx.x & 31;
    const int rows = min(tile_tokens(a.group) * item_tiles(HD), Lq - it.y) * a.group;
    for (int r = threadIdx.x >> 5; r < rows; r += 8) {
        const int i = it.y + r / a.group, h = kvh * a.group + r % a.group;
        const int n = keys_seen(i, Lq, Lk, pre);
        float q[E], o[E] = {}, m = -INFINITY, l = 0.f;
        for (int e = 0; e < E; ++e)
            q[e] = bf2f(a.q.ptr[(q0 + i) * a.q.row_stride + h * a.q.head_stride + e * 32 + lane]);
        for (int j = 0; j < n; ++j) {
            const size_t ko = (k0 + j) * a.k.row_stride + kvh * a.k.head_stride + lane;
            const size_t vo = (k0 + j) * a.v.row_stride + kvh * a.v.head_stride + lane;
            float d = 0.f;
            for (int e = 0; e < E; ++e) d += q[e] * bf2f(a.k.ptr[ko + e * 32]);
            for (int x = 16; x; x >>= 1) d += __shfl_xor_sync(0xffffffffu, d, x);
            d *= a.scale_log2;
            const float mn = fmaxf(m, d), c = exp2f(m - mn), p = exp2f(d - mn);
            for (int e = 0; e < E; ++e) o[e] = o[e] * c + p * bf2f(a.v.ptr[vo + e * 32]);
            l = l * c + p;
            m = mn;
        }
        for (int e = 0; e < E; ++e)
            a.out.ptr[(q0 + i) * a.out.row_stride + h * a.out.head_stride + e * 32 + lane] =
                f2bf(n ? o[e] / l : 0.f);
        if (a.lse && lane == 0) a.lse[(size_t)(q0 + i) * a.H + h] = n ? m + log2f(l) : -INFINITY;
    }
}

jnx_status heads_ok(int H, int Hkv, int hd, const char* what) {
    if (hd != 64 && hd != 128 && hd != 256)
        return fail(JNX_ERR_UNSUPPORTED, "%s: head_dim %d not in {64,128,256}", what, hd);
    if (H <= 0 || Hkv <= 0 || H % Hkv)
        return fail(JNX_ERR_INVALID_ARG, "%s: %d query heads over %d key heads", what, H, Hkv);
    if (H / Hkv > kMaxGroup)
        return fail(JNX_ERR_UNSUPPORTED, "%s: groups of over %d query heads", what, kMaxGroup);
    return JNX_OK;
}

// The prompt's host arrays; rows and keys get its totals.
jnx_status prompt_ok(const jnx_prompt* p, const char* what, int& rows, int& keys) {
    if (!p || p->n_seqs < 0) return fail(JNX_ERR_INVALID_ARG, "%s: bad prompt", what);
    rows = keys = 0;
    if (p->n_seqs == 0) return JNX_OK;
    if (!p->h_cu_q || !p->h_cu_kv) return fail(JNX_ERR_INVALID_ARG, "%s: null host arrays", what);
    if (p->h_cu_q[0] < 0 || p->h_cu_kv[0] < 0)
        return fail(JNX_ERR_INVALID_ARG, "%s: negative row", what);
    for (int s = 0; s < p->n_seqs; ++s)
        if (p->h_cu_q[s + 1] < p->h_cu_q[s] || p->h_cu_kv[s + 1] < p->h_cu_kv[s] ||
            (p->h_prefix && p->h_prefix[s] < 0))
            return fail(JNX_ERR_INVALID_ARG, "%s: bad sequence %d", what, s);
    rows = p->h_cu_q[p->n_seqs];
    keys = p->h_cu_kv[p->n_seqs];
    return JNX_OK;
}

// ... and its device arrays, for a launch.
jnx_status prompt_launchable(const jnx_prompt* p, const char* what, int& rows, int& keys) {
    if (jnx_status st = prompt_ok(p, what, rows, keys)) return st;
    if (rows > 0 && (!p->cu_q || !p->cu_kv || !p->items || (p->h_prefix && !p->prefix)))
        return fail(JNX_ERR_INVALID_ARG, "%s: null device arrays", what);
    if (p->n_forward < 0 || p->n_keys < 0 || p->n_queries < 0)
        return fail(JNX_ERR_INVALID_ARG, "%s: bad work list", what);
    return JNX_OK;
}

}  // namespace jnx

using namespace jnx;

extern "C" int32_t jnx_prompt_items(jnx_prompt* p, int32_t n_heads, int32_t n_kv_heads,
                                    int32_t head_dim, int32_t* out, int32_t cap) {
    clear_error();
    int rows, keys;
    if (jnx_status st = heads_ok(n_heads, n_kv_heads, head_dim, "prompt items")) return st;
    if (jnx_status st = prompt_ok(p, "prompt items", rows, keys)) return st;
    struct Item {
        int seq, at;
        long long cost;
    };
    try {
        std::vector<Item> all;
        const int T = tile_tokens(n_heads / n_kv_heads);
        const int step[3] = {T * item_tiles(head_dim), 128, T};
        int count[3];
        for (int pass = 0; pass < 3; ++pass) {
            const size_t first = all.size();
            for (int s = 0; s < p->n_seqs; ++s) {
                const int Lq = p->h_cu_q[s + 1] - p->h_cu_q[s];
                const int Lk = p->h_cu_kv[s + 1] - p->h_cu_kv[s];
                const int pre = p->h_prefix ? p->h_prefix[s] : 0;
                const int end = pass == 1 ? Lk : Lq;
                for (long long at = 0; at < end; at += step[pass]) {
                    const int last = (int)std::min<long long>(at + step[pass], end) - 1;
                    const long long cost = pass == 1 ? Lq - first_row((int)at, Lq, Lk, pre)
                                                     : keys_seen(last, Lq, Lk, pre);
                    all.push_back({s, (int)at, cost});
                }
            }
            std::stable_sort(all.begin() + first, all.end(),
                             [](const Item& x, const Item& y) { return x.cost > y.cost; });
            count[pass] = (int)(all.size() - first);
        }
        if (all.size() > 0x3fffffff) return fail(JNX_ERR_UNSUPPORTED, "prompt items: too many");
        p->n_forward = count[0];
        p->n_keys = count[1];
        p->n_queries = count[2];
        if (out && cap >= (int)all.size())
            for (size_t i = 0; i < all.size(); ++i) {
                out[2 * i] = all[i].seq;
                out[2 * i + 1] = all[i].at;
            }
        return (int32_t)all.size();
    } catch (const std::bad_alloc&) {
        return fail(JNX_ERR_OVERFLOW, "prompt items: out of host memory");
    }
}

extern "C" jnx_status jnx_op_prompt_attention(const jnx_prompt* p, int32_t n_heads,
                                              int32_t n_kv_heads, int32_t head_dim,
                                              const jnx_head_rows* q, const jnx_head_rows* k,
                                              const jnx_head_rows* v, const jnx_head_rows* out,
                                              float* lse, int32_t* status, void* stream) {
    clear_error();
    int rows, keys;
    if (jnx_status st = heads_ok(n_heads, n_kv_heads, head_dim, "prompt attention")) return st;
    if (jnx_status st = prompt_launchable(p, "prompt attention", rows, keys)) return st;
    if (rows == 0) return JNX_OK;
    if (!rows_ok(q) || !rows_ok(out) || (keys > 0 && (!rows_ok(k) || !rows_ok(v))))
        return fail(JNX_ERR_INVALID_ARG, "prompt attention: null or misaligned rows");
    const jnx_head_rows none{nullptr, 0, 0};
    PromptArgs a{p->cu_q, p->cu_kv, p->prefix, reinterpret_cast<const int2*>(p->items),
                 n_heads, n_kv_heads, n_heads / n_kv_heads,
                 (float)(1.4426950408889634 / sqrt((double)head_dim)), *q, keys ? *k : none,
                 keys ? *v : none, *out, lse};
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    TraceScope ts(JNX_K_PROMPT_ATTN, 0.0, s);
    const int grid = p->n_forward * n_kv_heads;
    if (head_dim == 64)
        pdl(k_prompt_attn<64>, grid, 256, 0, s)(a);
    else if (head_dim == 128)
        pdl(k_prompt_attn<128>, grid, 256, 0, s)(a);
    else
        pdl(k_prompt_attn<256>, grid, 256, 0, s)(a);
    return launched("prompt attention");
}
