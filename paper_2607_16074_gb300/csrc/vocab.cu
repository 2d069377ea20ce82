// Next-token losses over the vocabulary and their gradients: logits x = h w^T,
// loss = logsumexp(x) - x_target, G = row_weight (softmax(x) - onehot),
// dh = G w, dw = G^T h.
#include <algorithm>

#include "jnx_dev.cuh"
#include "jnx_kernels.h"
#include "jnx_text.h"
#include "jnx_trace.h"

namespace jnx {

struct VocabArgs {
    const uint16_t *h, *w;
    long long ldh, ldw, lddh, lddw;
    const int* targets;
    const float* weight;
    int rows, vocab, d;
    float* loss;
    uint16_t *dh, *dw, *G;
    float* acc;  // fp32 sums of dw over the pieces
    int* status;
};

__device__ __forceinline__ float vocab_dot(const VocabArgs& a, int r, int v, int lane) {
    float s = 0.f;
    for (int c = lane; c < a.d; c += 32) s += bf2f(a.h[r * a.ldh + c]) * bf2f(a.w[v * a.ldw + c]);
    for (int o = 16; o; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
    return s;
}

// A CTA a row: its logits twice, first for their sum, then for G.
__global__ void __launch_bounds__(1024) k_vocab_rows(const __grid_constant__ VocabArgs a) {
    __shared__ float sm[32], sl[32], st, slse;
    pdl_entry();
    const int r = blockIdx.x, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    int t = a.targets[r];
    if (t >= a.vocab) {
        report(a.status, JNX_ERR_DEVICE_BOUNDS);
        t = -1;
    }
    float m = -INFINITY, l = 0.f;
    for (int v = warp; v < a.vocab; v += 32) {
        const float x = vocab_dot(a, r, v, lane), mn = fmaxf(m, x);
        l = l * expf(m - mn) + expf(x - mn);
        m = mn;
        if (v == t && lane == 0) st = x;
    }
    if (lane == 0) sm[warp] = m, sl[warp] = l;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int i = 1; i < 32; ++i) m = fmaxf(m, sm[i]);
        l = 0.f;
        for (int i = 0; i < 32; ++i) l += sl[i] > 0.f ? sl[i] * expf(sm[i] - m) : 0.f;
        slse = m + logf(l);
        a.loss[r] = t >= 0 ? slse - st : 0.f;
    }
    __syncthreads();
    if (!a.G) return;
    const float w = t >= 0 ? a.weight[r] : 0.f;
    for (int v = warp; v < a.vocab; v += 32) {
        const float p = w == 0.f ? 0.f : expf(vocab_dot(a, r, v, lane) - slse) - (v == t ? 1.f : 0.f);
        if (lane == 0) a.G[(size_t)r * a.vocab + v] = f2bf(w * p);
    }
}

__global__ void __launch_bounds__(256) k_vocab_dh(const __grid_constant__ VocabArgs a) {
    pdl_entry();
    const int r = blockIdx.x, c = blockIdx.y * 256 + threadIdx.x;
    if (c >= a.d) return;
    float s = 0.f;
    for (int v = 0; v < a.vocab; ++v) s += bf2f(a.G[(size_t)r * a.vocab + v]) * bf2f(a.w[v * a.ldw + c]);
    a.dh[r * a.lddh + c] = f2bf(s);
}

__global__ void __launch_bounds__(256)
    k_vocab_dw(const __grid_constant__ VocabArgs a, int first, int last) {
    pdl_entry();
    const int v = blockIdx.x, c = blockIdx.y * 256 + threadIdx.x;
    if (c >= a.d) return;
    float s = first ? 0.f : a.acc[(size_t)v * a.d + c];
    for (int r = 0; r < a.rows; ++r)  // an ignored row's h may hold anything
        if (a.targets[r] >= 0) s += bf2f(a.G[(size_t)r * a.vocab + v]) * bf2f(a.h[r * a.ldh + c]);
    if (last)
        a.dw[v * a.lddw + c] = f2bf(s);
    else
        a.acc[(size_t)v * a.d + c] = s;
}

static jnx_status vocab_check(const void* h, int64_t ldh, const void* w, int64_t ldw,
                              const void* targets, int n_rows, int vocab, int d, const void* loss,
                              const char* what) {
    if (n_rows < 0 || vocab <= 0 || d <= 0)
        return fail(JNX_ERR_INVALID_ARG, "%s: bad sizes", what);
    if (d % 8 || ldh % 8 || ldw % 8 || ldh < d || ldw < d)
        return fail(JNX_ERR_INVALID_ARG, "%s: d and strides must be multiples of 8", what);
    if (n_rows > 0 && (!h || !w || !targets || !loss || !aligned16(h) || !aligned16(w)))
        return fail(JNX_ERR_INVALID_ARG, "%s: null or misaligned argument", what);
    return JNX_OK;
}

static int vocab_piece(int n_rows, int piece_rows) {
    return std::max(1, std::min(n_rows, piece_rows > 0 ? piece_rows : 8192));
}

}  // namespace jnx

using namespace jnx;

extern "C" size_t jnx_op_vocab_loss_workspace_bytes(int32_t n_rows, int32_t vocab, int32_t d) {
    return 0;
}

extern "C" jnx_status jnx_op_vocab_loss(const uint16_t* h, int64_t ldh, const uint16_t* w,
                                        int64_t ldw, const int32_t* targets, int32_t n_rows,
                                        int32_t vocab, int32_t d, float* loss, void* workspace,
                                        size_t ws_bytes, int32_t* status, void* stream) {
    clear_error();
    if (jnx_status st = vocab_check(h, ldh, w, ldw, targets, n_rows, vocab, d, loss, "vocab loss"))
        return st;
    if (n_rows == 0) return JNX_OK;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    VocabArgs a{h, w, ldh, ldw, 0, 0, targets, nullptr, n_rows, vocab, d, loss};
    a.status = status;
    TraceScope ts(JNX_K_VOCAB, 0.0, s);
    pdl(k_vocab_rows, n_rows, 1024, 0, s)(a);
    return launched("vocab loss");
}

extern "C" size_t jnx_op_vocab_loss_train_workspace_bytes(int32_t n_rows, int32_t vocab, int32_t d,
                                                          int32_t piece_rows) {
    if (n_rows < 0 || vocab <= 0 || d <= 0) return 0;
    return (((size_t)vocab_piece(n_rows, piece_rows) * vocab * 2 + 15) & ~(size_t)15) +
           (size_t)vocab * d * 4;
}

extern "C" jnx_status jnx_op_vocab_loss_train(const uint16_t* h, int64_t ldh, const uint16_t* w,
                                              int64_t ldw, const int32_t* targets,
                                              const float* row_weight, int32_t n_rows,
                                              int32_t vocab, int32_t d, int32_t piece_rows,
                                              float* loss, uint16_t* dh, int64_t lddh,
                                              uint16_t* dw, int64_t lddw, void* workspace,
                                              size_t ws_bytes, int32_t* status, void* stream) {
    clear_error();
    const char* what = "vocab loss train";
    if (jnx_status st = vocab_check(h, ldh, w, ldw, targets, n_rows, vocab, d, loss, what)) return st;
    if (n_rows > 0 && (!row_weight || !dh || !aligned16(dh) || lddh % 8 || lddh < d))
        return fail(JNX_ERR_INVALID_ARG, "%s: null or misaligned gradients", what);
    if (dw && (!aligned16(dw) || lddw % 8 || lddw < d))
        return fail(JNX_ERR_INVALID_ARG, "%s: misaligned weight gradient", what);
    if (n_rows > 0 && (!workspace || ws_bytes < jnx_op_vocab_loss_train_workspace_bytes(
                                                    n_rows, vocab, d, piece_rows)))
        return fail(JNX_ERR_WORKSPACE, "%s: workspace too small", what);
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    if (n_rows == 0) {
        if (dw && cudaMemset2DAsync(dw, lddw * 2, 0, (size_t)d * 2, vocab, s) != cudaSuccess)
            return launched(what);
        return JNX_OK;
    }
    const int piece = vocab_piece(n_rows, piece_rows);
    TraceScope ts(JNX_K_VOCAB, 0.0, s);
    for (int r0 = 0; r0 < n_rows; r0 += piece) {
        const int rows = std::min(piece, n_rows - r0);
        VocabArgs a{h + r0 * ldh, w, ldh, ldw, lddh, lddw, targets + r0, row_weight + r0, rows,
                    vocab, d, loss + r0, dh + r0 * lddh, dw, static_cast<uint16_t*>(workspace)};
        a.acc = reinterpret_cast<float*>(static_cast<uint8_t*>(workspace) +
                                         (((size_t)piece * vocab * 2 + 15) & ~(size_t)15));
        a.status = status;
        pdl(k_vocab_rows, rows, 1024, 0, s)(a);
        pdl(k_vocab_dh, dim3(rows, (d + 255) / 256), 256, 0, s)(a);
        if (dw)
            pdl(k_vocab_dw, dim3(vocab, (d + 255) / 256), 256, 0, s)(a, r0 == 0 ? 1 : 0,
                                                                    r0 + rows == n_rows ? 1 : 0);
    }
    return launched(what);
}
