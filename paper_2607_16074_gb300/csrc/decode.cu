// Attention of one new token of each live sequence against its cache.
#include <algorithm>

#include "jnx_dev.cuh"
#include "jnx_kernels.h"
#include "jnx_text.h"
#include "jnx_trace.h"

namespace jnx {

struct DecodeArgs {
    jnx_kv_cache c;
    int batch, H, Hkv;
    float scale_log2;
    jnx_head_rows q, out;
    const int *slot, *n;
    int* status;
};

// One warp a (sequence, query head).
template <int HD>
__global__ void __launch_bounds__(128) k_decode_attn(const __grid_constant__ DecodeArgs a) {
    constexpr int E = HD / 32;
    pdl_entry();
    const int w = blockIdx.x * 4 + (threadIdx.x >> 5), lane = threadIdx.x & 31;
    if (w >= a.batch * a.H) return;
    const int b = w / a.H, h = w % a.H, g = h / (a.H / a.Hkv);
    int slot = a.slot[b], n = a.n[b];
    if (n < 0 || n > a.c.room || (n > 0 && (slot < 0 || slot >= a.c.n_slots))) {
        report(a.status, JNX_ERR_DEVICE_BOUNDS);
        n = 0;
    }
    if (n == 0) slot = 0;
    const size_t base = slot * a.c.slot_stride + g * a.c.head_stride + lane;
    float q[E], o[E] = {}, m = -INFINITY, l = 0.f;
    for (int e = 0; e < E; ++e)
        q[e] = bf2f(a.q.ptr[b * a.q.row_stride + h * a.q.head_stride + e * 32 + lane]);
    for (int j = 0; j < n; ++j) {
        const size_t at = base + j * a.c.row_stride;
        float d = 0.f;
        for (int e = 0; e < E; ++e) d += q[e] * bf2f(a.c.k[at + e * 32]);
        for (int x = 16; x; x >>= 1) d += __shfl_xor_sync(0xffffffffu, d, x);
        d *= a.scale_log2;
        const float mn = fmaxf(m, d), c = exp2f(m - mn), p = exp2f(d - mn);
        for (int e = 0; e < E; ++e) o[e] = o[e] * c + p * bf2f(a.c.v[at + e * 32]);
        l = l * c + p;
        m = mn;
    }
    for (int e = 0; e < E; ++e)
        a.out.ptr[b * a.out.row_stride + h * a.out.head_stride + e * 32 + lane] =
            f2bf(n ? o[e] / l : 0.f);
}

}  // namespace jnx

using namespace jnx;

extern "C" size_t jnx_op_decode_attention_workspace_bytes(int32_t batch, int32_t n_heads,
                                                          int32_t head_dim) {
    return 0;
}

extern "C" jnx_status jnx_op_decode_attention(const jnx_kv_cache* cache, int32_t batch,
                                              int32_t n_heads, int32_t n_kv_heads,
                                              int32_t head_dim, const jnx_head_rows* q,
                                              const int32_t* slot, const int32_t* n_cached,
                                              const jnx_head_rows* out, void* workspace,
                                              size_t ws_bytes, int32_t* status, void* stream) {
    clear_error();
    if (jnx_status st = heads_ok(n_heads, n_kv_heads, head_dim, "decode attention")) return st;
    if (batch < 0) return fail(JNX_ERR_INVALID_ARG, "decode attention: negative batch");
    if (batch == 0) return JNX_OK;
    if (!cache_ok(cache) || !rows_ok(q) || !rows_ok(out) || !slot || !n_cached)
        return fail(JNX_ERR_INVALID_ARG, "decode attention: null or misaligned argument");
    if ((int64_t)batch * n_heads > 0x7fffff00)
        return fail(JNX_ERR_UNSUPPORTED, "decode attention: batch too large");
    DecodeArgs a{*cache, batch, n_heads, n_kv_heads,
                 (float)(1.4426950408889634 / sqrt((double)head_dim)), *q, *out, slot, n_cached,
                 status};
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    TraceScope ts(JNX_K_DECODE_ATTN, 0.0, s);
    const int grid = (batch * n_heads + 3) / 4;
    if (head_dim == 64)
        pdl(k_decode_attn<64>, grid, 128, 0, s)(a);
    else if (head_dim == 128)
        pdl(k_decode_attn<128>, grid, 128, 0, s)(a);
    else
        pdl(k_decode_attn<256>, grid, 128, 0, s)(a);
    return launched("decode attention");
}
