// Gradients of the attention of packed prompts.
//
// With P = 2^(s c - lse) recomputed from the forward's log2-sum-exp, c = log2(e) /
// sqrt(hd), and D = rowsum(dO * O):  dV = P^T dO,  dS = P (dO V^T - D) / sqrt(hd),
// dQ = dS K,  dK = dS^T Q; a key head's gradients add over its group's query heads.
#include <algorithm>

#include "jnx_dev.cuh"
#include "jnx_kernels.h"
#include "jnx_text.h"
#include "jnx_trace.h"

namespace jnx {

jnx_status prompt_launchable(const jnx_prompt* p, const char* what, int& rows, int& keys);

struct PromptBwdArgs {
    const int *cu_q, *cu_kv, *prefix;
    const int2* items;
    int H, Hkv, group;
    float scale_log2, scale;
    jnx_head_rows q, k, v, out, dout, dq, dk, dv;
    const float* lse;
    float* D;
};

template <int E>
__device__ __forceinline__ void row_load(float (&f)[E], const jnx_head_rows& r, long long row,
                                         int head, int lane) {
    for (int e = 0; e < E; ++e)
        f[e] = bf2f(r.ptr[row * r.row_stride + head * r.head_stride + e * 32 + lane]);
}

template <int E>
__device__ __forceinline__ float row_dot(const float (&x)[E], const float (&y)[E]) {
    float d = 0.f;
    for (int e = 0; e < E; ++e) d += x[e] * y[e];
    for (int o = 16; o; o >>= 1) d += __shfl_xor_sync(0xffffffffu, d, o);
    return d;
}

// Query rows, one warp each: D and dQ.
template <int HD>
__global__ void __launch_bounds__(256) k_prompt_attn_dq(const __grid_constant__ PromptBwdArgs a) {
    constexpr int E = HD / 32;
    pdl_entry();
    const int2 it = a.items[blockIdx.x / a.Hkv];
    const int kvh = blockIdx.x % a.Hkv, s = it.x;
    const int q0 = a.cu_q[s], Lq = a.cu_q[s + 1] - q0, k0 = a.cu_kv[s], Lk = a.cu_kv[s + 1] - k0;
    const int pre = a.prefix ? a.prefix[s] : 0, lane = threadIdx.x & 31;
    const int rows = min(tile_tokens(a.group), Lq - it.y) * a.group;
    for (int r = threadIdx.x >> 5; r < rows; r += 8) {
        const int i = it.y + r / a.group, h = kvh * a.group + r % a.group;
        const int n = keys_seen(i, Lq, Lk, pre);
        float q[E], o[E], go[E], dq[E] = {};
        row_load(q, a.q, q0 + i, h, lane);
        row_load(o, a.out, q0 + i, h, lane);
        row_load(go, a.dout, q0 + i, h, lane);
        const float D = row_dot(o, go), lse = a.lse[(size_t)(q0 + i) * a.H + h];
        if (lane == 0) a.D[(size_t)(q0 + i) * a.H + h] = D;
        for (int j = 0; j < n; ++j) {
            float k[E], v[E];
            row_load(k, a.k, k0 + j, kvh, lane);
            row_load(v, a.v, k0 + j, kvh, lane);
            const float p = exp2f(row_dot(q, k) * a.scale_log2 - lse);
            const float ds = p * (row_dot(go, v) - D) * a.scale;
            for (int e = 0; e < E; ++e) dq[e] += ds * k[e];
        }
        for (int e = 0; e < E; ++e)
            a.dq.ptr[(q0 + i) * a.dq.row_stride + h * a.dq.head_stride + e * 32 + lane] = f2bf(dq[e]);
    }
}

// Keys, one warp each.
template <int HD>
__global__ void __launch_bounds__(256) k_prompt_attn_dkv(const __grid_constant__ PromptBwdArgs a) {
    constexpr int E = HD / 32;
    pdl_entry();
    const int2 it = a.items[blockIdx.x / a.Hkv];
    const int kvh = blockIdx.x % a.Hkv, s = it.x;
    const int q0 = a.cu_q[s], Lq = a.cu_q[s + 1] - q0, k0 = a.cu_kv[s], Lk = a.cu_kv[s + 1] - k0;
    const int pre = a.prefix ? a.prefix[s] : 0, lane = threadIdx.x & 31;
    for (int j = it.y + (threadIdx.x >> 5); j < min(it.y + 128, Lk); j += 8) {
        float k[E], v[E], dk[E] = {}, dv[E] = {};
        row_load(k, a.k, k0 + j, kvh, lane);
        row_load(v, a.v, k0 + j, kvh, lane);
        for (int i = first_row(j, Lq, Lk, pre); i < Lq; ++i)
            for (int h = kvh * a.group; h < (kvh + 1) * a.group; ++h) {
                float q[E], go[E];
                row_load(q, a.q, q0 + i, h, lane);
                row_load(go, a.dout, q0 + i, h, lane);
                const size_t at = (size_t)(q0 + i) * a.H + h;
                const float p = exp2f(row_dot(q, k) * a.scale_log2 - a.lse[at]);
                const float ds = p * (row_dot(go, v) - a.D[at]) * a.scale;
                for (int e = 0; e < E; ++e) {
                    dk[e] += ds * q[e];
                    dv[e] += p * go[e];
                }
            }
        for (int e = 0; e < E; ++e) {
            a.dk.ptr[(k0 + j) * a.dk.row_stride + kvh * a.dk.head_stride + e * 32 + lane] = f2bf(dk[e]);
            a.dv.ptr[(k0 + j) * a.dv.row_stride + kvh * a.dv.head_stride + e * 32 + lane] = f2bf(dv[e]);
        }
    }
}

}  // namespace jnx

using namespace jnx;

extern "C" size_t jnx_op_prompt_attention_backward_workspace_bytes(int32_t n_q, int32_t n_heads) {
    if (n_q < 0 || n_heads <= 0) return 0;
    return (size_t)n_q * n_heads * sizeof(float);
}

extern "C" jnx_status jnx_op_prompt_attention_backward(
    const jnx_prompt* p, int32_t n_heads, int32_t n_kv_heads, int32_t head_dim,
    const jnx_head_rows* q, const jnx_head_rows* k, const jnx_head_rows* v,
    const jnx_head_rows* out, const float* lse, const jnx_head_rows* dout,
    const jnx_head_rows* dq, const jnx_head_rows* dk, const jnx_head_rows* dv, void* workspace,
    size_t ws_bytes, int32_t* status, void* stream) {
    clear_error();
    const char* what = "prompt attention backward";
    int rows, keys;
    if (jnx_status st = heads_ok(n_heads, n_kv_heads, head_dim, what)) return st;
    if (jnx_status st = prompt_launchable(p, what, rows, keys)) return st;
    if (rows == 0 && keys == 0) return JNX_OK;
    if ((rows > 0 && (!rows_ok(q) || !rows_ok(out) || !rows_ok(dout) || !rows_ok(dq) || !lse)) ||
        (keys > 0 && (!rows_ok(k) || !rows_ok(v) || !rows_ok(dk) || !rows_ok(dv))))
        return fail(JNX_ERR_INVALID_ARG, "%s: null or misaligned rows", what);
    if (rows > 0 && (!workspace || ws_bytes < jnx_op_prompt_attention_backward_workspace_bytes(
                                                  rows, n_heads)))
        return fail(JNX_ERR_WORKSPACE, "%s: workspace too small", what);
    const jnx_head_rows none{nullptr, 0, 0};
    auto or_none = [&](const jnx_head_rows* r, int n) { return n ? *r : none; };
    PromptBwdArgs a{p->cu_q, p->cu_kv, p->prefix,
                    reinterpret_cast<const int2*>(p->items) + p->n_forward + p->n_keys, n_heads,
                    n_kv_heads, n_heads / n_kv_heads,
                    (float)(1.4426950408889634 / sqrt((double)head_dim)),
                    (float)(1.0 / sqrt((double)head_dim)), or_none(q, rows), or_none(k, keys),
                    or_none(v, keys), or_none(out, rows), or_none(dout, rows), or_none(dq, rows),
                    or_none(dk, keys), or_none(dv, keys), lse, static_cast<float*>(workspace)};
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    TraceScope ts(JNX_K_PROMPT_ATTN_BWD, 0.0, s);
    auto go = [&](auto dq_kernel, auto dkv_kernel) {
        if (p->n_queries) pdl(dq_kernel, p->n_queries * n_kv_heads, 256, 0, s)(a);
        a.items -= p->n_keys;
        if (p->n_keys) pdl(dkv_kernel, p->n_keys * n_kv_heads, 256, 0, s)(a);
    };
    if (head_dim == 64)
        go(k_prompt_attn_dq<64>, k_prompt_attn_dkv<64>);
    else if (head_dim == 128)
        go(k_prompt_attn_dq<128>, k_prompt_attn_dkv<128>);
    else
        go(k_prompt_attn_dq<256>, k_prompt_attn_dkv<256>);
    return launched(what);
}
