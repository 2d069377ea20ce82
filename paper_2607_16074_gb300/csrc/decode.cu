// Attention of one new token of each live sequence against its cache.
//
// Bound by reading the cache once (4 bytes x hd a token and key head).  A unit is a run of
// one sequence's tokens for one key head and up to 16 of its query heads; a warp takes
// units in turn and streams each one's keys and values through a ring of its own in
// shared memory, filled by TMA tiles ahead across the units' borders, so a warp waits for
// memory only when its SM's share of it is used up.  The products run on mma.sync, query
// heads as the 16 rows: a quarter of its rate suffices for the cache's bandwidth, and
// tcgen05's 128 rows would hold 16 in use.
//
// The run's length depends on the sequence's length alone, so a sequence's bits do not
// depend on the others; its runs' sums are joined in their order by a second kernel.
// (CTAs that share a unit and a join by the last CTA to finish took half as long again:
// 307 us where the warps' own units and the second kernel take 206.)
//
// 64 sequences of up to 8,100 tokens, 32 heads on 8 of 128 (1.17 GB): 203 us, 5.75 TB/s.
// 8 of up to 700, 8 heads on one of 256: 9.2 us, where memory is not what counts: the
// lengths, a unit's tiles, its sums and the join follow one another, 1-2 us each.
#include <algorithm>

#include "jnx_dev.cuh"
#include "jnx_kernels.h"
#include "jnx_text.h"
#include "jnx_trace.h"

namespace jnx {

namespace decode {
constexpr int WARPS = 4;
constexpr int STAGES = 3;
constexpr int ROWS = 16;       // query heads of a unit
constexpr int BATCH = 1024;    // sequences of one launch
constexpr int MAX_RUNS = 128;  // runs of a sequence

// Tokens of a sequence's runs: short ones for short sequences, so that a few sequences
// reach many SMs; long enough beyond that a run's sums (hd + 2 floats a head) are a few
// percent of what it reads.  (Runs half as long from 1,024 tokens on: 64 sequences of up to
// 4,000 tokens, 8 heads on one of 256, 38.6 us for 33.3; runs of 32 below, 128 of up to 700
// 23.8 for 18.9.)
__host__ __device__ inline int run_tokens(int n) {
    int r = n <= 1024 ? 64 : n <= 4096 ? 128 : 256;
    const int most = (n + MAX_RUNS - 1) / MAX_RUNS;
    return r >= most ? r : (most + 63) / 64 * 64;
}
__host__ __device__ inline int runs(int n) {
    return n <= 0 ? 1 : (n + run_tokens(n) - 1) / run_tokens(n);
}
}  // namespace decode

struct DecodeArgs {
    int batch, H, Hkv, group, blocks;  // blocks of up to 16 query heads of a group
    int n_slots, room;
    float scale_log2;
    const uint16_t* q;
    long long q_row, q_head;
    uint16_t* out;
    long long o_row, o_head;
    const int *slot, *n;
    int* first;   // [batch + 1]: a sequence's first run among all
    float2* ml;   // [run][H]: maxima and sums of exponentials
    float* part;  // [run][H][hd]: sums
    int* status;
};

// A sequence's cached tokens; one outside the cache counts as empty.
__device__ __forceinline__ int decode_length(const DecodeArgs& a, int b, bool tell) {
    const int n = a.n[b], s = a.slot[b];
    if (n == 0) return 0;
    if (n < 0 || n > a.room || s < 0 || s >= a.n_slots) {
        if (tell) report(a.status, JNX_ERR_DEVICE_BOUNDS);
        return 0;
    }
    return n;
}

template <int HD>
struct DecodeCfg {
    static constexpr int TILE = HD == 256 ? 16 : 32;  // tokens of a ring stage
    static constexpr int NCH = HD / 64;
    static constexpr int KV = TILE * HD * 2;  // bytes of its keys (and of its values)
    static constexpr int RING = decode::STAGES * 2 * KV;
    static constexpr int OFF_BAR = decode::WARPS * RING;
    static constexpr int OFF_FIRST = OFF_BAR + decode::WARPS * decode::STAGES * 8;
    static constexpr int SMEM = OFF_FIRST + (3 * decode::BATCH + 1) * 4 + 1024;
    static_assert(SMEM <= 227 * 1024, "shared memory per CTA");
};

// Where a warp is in the units: unit u, tokens [at, end) of sequence b still to take.
struct DecodeAt {
    int u, b, run, kvh, block, at, end, n;
};

template <int HD>
__global__ void __launch_bounds__(32 * decode::WARPS, 1)
    k_decode_attn(const __grid_constant__ CUtensorMap tk, const __grid_constant__ CUtensorMap tv,
                  const __grid_constant__ DecodeArgs a) {
    using C = DecodeCfg<HD>;
    using namespace decode;
    constexpr int TILE = C::TILE, NCH = C::NCH;
    extern __shared__ uint8_t smem_raw[];
    uint8_t* sm = reinterpret_cast<uint8_t*>(
        (reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
    int* first = reinterpret_cast<int*>(sm + C::OFF_FIRST);  // [batch + 1] first run of each
    int* length = first + BATCH + 1;                         // [batch]
    int* slots = length + BATCH;                             // [batch]
    const int warp = warp_uniform(threadIdx.x >> 5), lane = threadIdx.x & 31;
    uint8_t* ring = sm + warp * C::RING;
    uint64_t* full = reinterpret_cast<uint64_t*>(sm + C::OFF_BAR) + warp * STAGES;
    if (lane == 0) {
        for (int s = 0; s < STAGES; ++s) mbar_init(&full[s], 1);
        fence_barrier_init();
        fence_proxy_async();
    }
    pdl_entry();
    if (threadIdx.x == 0) {
        tma_prefetch_desc(&tk);
        tma_prefetch_desc(&tv);
    }
    // first runs: a warp scans the lengths
    for (int b = threadIdx.x; b < a.batch; b += 32 * WARPS)
        slots[b] = a.slot[b], length[b] = decode_length(a, b, blockIdx.x == 0);
    __syncthreads();
    if (warp == 0) {
        int total = 0;
        for (int base = 0; base < a.batch; base += 32) {
            const int b = base + lane;
            const int mine = b < a.batch ? runs(length[b]) : 0;
            int run = mine;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const int x = __shfl_up_sync(0xffffffffu, run, o);
                if (lane >= o) run += x;
            }
            if (b < a.batch) {
                first[b] = total + run - mine;
                if (blockIdx.x == 0) a.first[b] = total + run - mine;
            }
            total += __shfl_sync(0xffffffffu, run, 31);
        }
        if (lane == 0) {
            first[a.batch] = total;
            if (blockIdx.x == 0) a.first[a.batch] = total;
        }
    }
    __syncthreads();
    const int per_run = a.Hkv * a.blocks;  // units of a run: its heads, which lie together
    const int n_units = first[a.batch] * per_run;
    const int step = gridDim.x * WARPS, u0 = blockIdx.x + gridDim.x * warp;  // over the SMs first

    auto open = [&](int u) {
        DecodeAt x{u, 0, 0, 0, 0, 0, 0, 0};
        if (u >= n_units) return x;
        const int run = u / per_run, head = u - run * per_run;
        int lo = 0, hi = a.batch - 1;  // the last b with first[b] <= run
        while (lo < hi) {
            const int mid = (lo + hi + 1) >> 1;
            if (first[mid] <= run) lo = mid;
            else hi = mid - 1;
        }
        x.b = lo;
        x.run = run - first[lo];
        x.kvh = head / a.blocks;
        x.block = head % a.blocks;
        x.n = length[lo];
        x.at = x.run * run_tokens(x.n);
        x.end = min(x.n, x.at + run_tokens(x.n));
        return x;
    };
    // tiles are asked for by `ask`, STAGES ahead of the ones taken
    DecodeAt ask = open(u0);
    uint32_t asked = 0, taken = 0;
    auto ask_one = [&]() {
        while (ask.u < n_units && ask.at >= ask.end) ask = open(ask.u + step);
        if (ask.u >= n_units) return;
        const int s = asked % STAGES, slot = slots[ask.b];
        if (elect_one()) {
            mbar_arrive_expect_tx(&full[s], 2 * C::KV);
            uint8_t* dst = ring + s * 2 * C::KV;
#pragma unroll
            for (int c = 0; c < NCH; ++c) {
                tma_load_4d(dst + c * TILE * 128, &tk, c * 64, ask.kvh, ask.at, slot, &full[s]);
                tma_load_4d(dst + C::KV + c * TILE * 128, &tv, c * 64, ask.kvh, ask.at, slot, &full[s]);
            }
        }
        __syncwarp();
        ++asked;
        ask.at += TILE;
    };
    for (int i = 0; i < STAGES; ++i) ask_one();

    bool ok = true;
    for (DecodeAt x = open(u0); ok && x.u < n_units; x = open(x.u + step)) {
        const int h0 = x.kvh * a.group + x.block * ROWS;             // first query head
        const int heads = min(ROWS, a.group - x.block * ROWS);
        const int r0 = lane >> 2, cq = (lane & 3) * 2;               // fragment row and column
        uint32_t qf[HD / 16][4];
        const uint16_t* q0 = a.q + x.b * a.q_row + (h0 + r0) * a.q_head + cq;
#pragma unroll
        for (int k = 0; k < HD / 16; ++k)
#pragma unroll
            for (int i = 0; i < 4; ++i)
                qf[k][i] = r0 + (i & 1) * 8 < heads
                               ? *reinterpret_cast<const uint32_t*>(q0 + (i & 1) * 8 * a.q_head +
                                                                    k * 16 + (i >> 1) * 8)
                               : 0u;
        float o[HD / 8][4] = {}, m[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f};
        for (; x.at < x.end; x.at += TILE) {
            const int s = taken % STAGES;
            if (!(ok = mbar_wait_warp(&full[s], (taken / STAGES) & 1))) break;
            const uint32_t ks = smem_u32(ring + s * 2 * C::KV), vs = ks + C::KV;
            const int valid = x.end - x.at;  // tokens of the tile that are the run's
            if (valid < TILE) {
                // what lies behind may be NaN, which a probability of zero would not hide
                for (int i = lane; i < (TILE - valid) * (HD / 8); i += 32) {
                    const int r = valid + i / (HD / 8), u = i % (HD / 8);
                    *reinterpret_cast<uint4*>(ring + s * 2 * C::KV + C::KV + (u >> 3) * TILE * 128 +
                                              r * 128 + (u & 7) * 16) = make_uint4(0, 0, 0, 0);
                }
                fence_proxy_async();
                __syncwarp();
            }
            // S: 8 tokens a column tile
            float sc[TILE / 8][4] = {};
#pragma unroll
            for (int k = 0; k < HD / 16; ++k)
#pragma unroll
                for (int t = 0; t < TILE / 16; ++t) {
                    const int r = t * 16 + (lane & 7) + ((lane >> 4) << 3);
                    const int u = (k & 3) * 2 + ((lane >> 3) & 1);
                    uint32_t b0, b1, b2, b3;
                    ldsm_x4(ks + (k >> 2) * TILE * 128 + r * 128 + ((u ^ (r & 7)) << 4), b0, b1, b2, b3);
                    mma_bf16(sc[2 * t], qf[k][0], qf[k][1], qf[k][2], qf[k][3], b0, b1);
                    mma_bf16(sc[2 * t + 1], qf[k][0], qf[k][1], qf[k][2], qf[k][3], b2, b3);
                }
            float top[2] = {-INFINITY, -INFINITY};
#pragma unroll
            for (int t = 0; t < TILE / 8; ++t)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    if (t * 8 + cq + (i & 1) >= valid) sc[t][i] = -INFINITY;
                    top[i >> 1] = fmaxf(top[i >> 1], sc[t][i]);
                }
            float alpha[2], sum[2] = {0.f, 0.f};
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                top[i] = fmaxf(top[i], __shfl_xor_sync(0xffffffffu, top[i], 1));
                top[i] = fmaxf(top[i], __shfl_xor_sync(0xffffffffu, top[i], 2));
                const float mn = fmaxf(m[i], top[i] * a.scale_log2);  // finite: a tile has a token
                alpha[i] = ex2_approx(m[i] - mn);
                m[i] = mn;
            }
#pragma unroll
            for (int t = 0; t < TILE / 8; ++t)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    sc[t][i] = ex2_approx(fmaf(sc[t][i], a.scale_log2, -m[i >> 1]));
                    sum[i >> 1] += sc[t][i];
                }
            l[0] = l[0] * alpha[0] + sum[0];
            l[1] = l[1] * alpha[1] + sum[1];
            if (__any_sync(0xffffffffu, alpha[0] != 1.f || alpha[1] != 1.f)) {
#pragma unroll
                for (int c = 0; c < HD / 8; ++c) {
                    o[c][0] *= alpha[0];
                    o[c][1] *= alpha[0];
                    o[c][2] *= alpha[1];
                    o[c][3] *= alpha[1];
                }
            }
#pragma unroll
            for (int t = 0; t < TILE / 16; ++t) {
                const uint32_t p0 = cvt_bf2(sc[2 * t][0], sc[2 * t][1]);
                const uint32_t p1 = cvt_bf2(sc[2 * t][2], sc[2 * t][3]);
                const uint32_t p2 = cvt_bf2(sc[2 * t + 1][0], sc[2 * t + 1][1]);
                const uint32_t p3 = cvt_bf2(sc[2 * t + 1][2], sc[2 * t + 1][3]);
#pragma unroll
                for (int c = 0; c < HD / 16; ++c) {
                    const int r = t * 16 + (lane & 15);
                    const int u = (c & 3) * 2 + (lane >> 4);
                    uint32_t b0, b1, b2, b3;
                    ldsm_x4_t(vs + (c >> 2) * TILE * 128 + r * 128 + ((u ^ (r & 7)) << 4), b0, b1, b2, b3);
                    mma_bf16(o[2 * c], p0, p1, p2, p3, b0, b1);
                    mma_bf16(o[2 * c + 1], p0, p1, p2, p3, b2, b3);
                }
            }
            ++taken;
            __syncwarp();  // every lane has read the stage
            ask_one();
        }
        if (!ok) break;
        const bool alone = runs(x.n) == 1;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            l[i] += __shfl_xor_sync(0xffffffffu, l[i], 1);
            l[i] += __shfl_xor_sync(0xffffffffu, l[i], 2);
            const int r = r0 + 8 * i, h = h0 + r;
            if (r >= heads) continue;
            if (alone) {  // nothing to join
                const float inv = l[i] > 0.f ? 1.f / l[i] : 0.f;
                uint16_t* dst = a.out + x.b * a.o_row + h * a.o_head + cq;
#pragma unroll
                for (int c = 0; c < HD / 8; ++c)
                    *reinterpret_cast<uint32_t*>(dst + c * 8) =
                        cvt_bf2(o[c][2 * i] * inv, o[c][2 * i + 1] * inv);
            } else {
                const size_t at = (size_t)(first[x.b] + x.run) * a.H + h;
                float* dst = a.part + at * HD;
#pragma unroll
                for (int c = 0; c < HD / 8; ++c)
                    *reinterpret_cast<float2*>(dst + c * 8 + cq) =
                        make_float2(o[c][2 * i], o[c][2 * i + 1]);
                if ((lane & 3) == 0) a.ml[at] = make_float2(m[i], l[i]);
            }
        }
    }
    if (!ok) report(a.status, JNX_ERR_TIMEOUT);
    // every copy has landed before the CTA exits (all are taken in a normal run)
    for (; taken < asked; ++taken) mbar_wait_warp(&full[taken % STAGES], (taken / STAGES) & 1, 100000000LL);
}

// A sequence's runs joined: the runs' sums in G turns, each turn's in order, then the turns'
// in theirs.  WIDE: a CTA a query head and a group of threads a turn, so that all loads are
// under way at once; else a group takes a head's turns by itself, for more heads than the SMs
// hold CTAs of.  (8 sequences of up to 4,000 tokens, 8 heads on one of 256: 13.2 us wide, 16.8
// a warp a head.)
template <int HD, bool WIDE>
__global__ void __launch_bounds__(256) k_decode_join(const __grid_constant__ DecodeArgs a) {
    using namespace decode;
    constexpr int LANES = HD == 256 ? 64 : 32, E = HD / LANES, G = 256 / LANES;
    constexpr int HEADS = WIDE ? 1 : G;  // of a CTA
    __shared__ float sums[WIDE ? 256 * E : 1];
    pdl_entry();
    const int t = threadIdx.x, lane = t & 31, g = t / LANES, c = t % LANES;
    const int w = WIDE ? blockIdx.x : blockIdx.x * HEADS + g;
    if (w >= a.batch * a.H) return;
    const int b = w / a.H, h = w % a.H;
    const int r0 = a.first[b], nr = a.first[b + 1] - r0;
    if (nr == 1) return;
    const float2* ml = a.ml + (size_t)r0 * a.H + h;
    const float* src = a.part + ((size_t)r0 * a.H + h) * HD + c * E;
    const size_t step = (size_t)a.H * HD;
    float m[MAX_RUNS / 32], l[MAX_RUNS / 32], top = -INFINITY, sum = 0.f;
#pragma unroll
    for (int i = 0; i < MAX_RUNS / 32; ++i) {
        const int r = i * 32 + lane;
        const float2 x = r < nr ? ml[(size_t)r * a.H] : make_float2(-INFINITY, 0.f);
        m[i] = x.x;
        l[i] = x.y;
        top = fmaxf(top, m[i]);
    }
    constexpr int R = 8;  // runs of a thread under way
    float v[R][E];
    auto load = [&](int i, int r) {
        if (r >= nr) return;
        if constexpr (E == 4) {
            const float4 x = *reinterpret_cast<const float4*>(src + r * step);
            v[i][0] = x.x, v[i][1] = x.y, v[i][2] = x.z, v[i][3] = x.w;
        } else {
            const float2 x = *reinterpret_cast<const float2*>(src + r * step);
            v[i][0] = x.x, v[i][1] = x.y;
        }
    };
    constexpr int STEP = WIDE ? G : 1;
#pragma unroll
    for (int i = 0; i < R; ++i) load(i, (WIDE ? g : 0) + i * STEP);
#pragma unroll
    for (int o = 16; o; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
#pragma unroll
    for (int i = 0; i < MAX_RUNS / 32; ++i) {
        m[i] = ex2_approx(m[i] - top);
        sum += l[i] * m[i];
    }
#pragma unroll
    for (int o = 16; o; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    const float inv = 1.f / sum;
    auto factor = [&](int r) {
        const int i = r >> 5;
        const float x = i == 0 ? m[0] : i == 1 ? m[1] : i == 2 ? m[2] : m[3];
        return __shfl_sync(0xffffffffu, x, r & 31);
    };
    static_assert(MAX_RUNS == 128, "factors of four registers");
    float acc[HEADS][E] = {};  // WIDE: this group's turn, else every turn
    for (int r = WIDE ? g : 0; r < nr; r += R * STEP) {
        if (r >= R * STEP) {
#pragma unroll
            for (int i = 0; i < R; ++i) load(i, r + i * STEP);
        }
#pragma unroll
        for (int i = 0; i < R; ++i) {
            if (r + i * STEP >= nr) continue;
            const float f = factor(r + i * STEP);
#pragma unroll
            for (int e = 0; e < E; ++e) {
                float& to = acc[WIDE ? 0 : i % G][e];  // (R is a multiple of G)
                to = fmaf(f, v[i][e], to);
            }
        }
    }
    static_assert(R % G == 0, "turns of a batch");
    float all[E];
    if constexpr (WIDE) {
#pragma unroll
        for (int e = 0; e < E; ++e) sums[e * 256 + t] = acc[0][e];
        __syncthreads();
        if (g > 0) return;
#pragma unroll
        for (int e = 0; e < E; ++e) {
            all[e] = acc[0][e];
#pragma unroll
            for (int i = 1; i < G; ++i) all[e] += sums[e * 256 + i * LANES + c];
        }
    } else {
#pragma unroll
        for (int e = 0; e < E; ++e) {
            all[e] = acc[0][e];
#pragma unroll
            for (int i = 1; i < G; ++i) all[e] += acc[i][e];
        }
    }
    uint16_t* o = a.out + b * a.o_row + h * a.o_head + c * E;
#pragma unroll
    for (int e = 0; e < E; e += 2)
        *reinterpret_cast<uint32_t*>(o + e) = cvt_bf2(all[e] * inv, all[e + 1] * inv);
}

// The workspace: the first runs of a launch's sequences, then its runs' sums.
static size_t decode_sums_at(int batch) {
    return ((size_t)std::min(batch, decode::BATCH) + 1 + 3) / 4 * 16;
}
static size_t decode_runs(int batch) {
    return (size_t)std::min(batch, decode::BATCH) * decode::MAX_RUNS;
}

template <int HD>
static jnx_status launch_decode(const jnx_kv_cache& c, DecodeArgs a, cudaStream_t s) {
    using namespace decode;
    using C = DecodeCfg<HD>;
    static std::atomic<uint64_t> attr{0};
    if (set_smem_limit(reinterpret_cast<const void*>(k_decode_attn<HD>), C::SMEM, attr) != cudaSuccess)
        return fail(JNX_ERR_CUDA, "decode attention: smem attribute");
    CUtensorMap tk, tv;
    if (!make_tmap_cache(&tk, c.k, c, a.Hkv, HD, C::TILE) || !make_tmap_cache(&tv, c.v, c, a.Hkv, HD, C::TILE))
        return fail(JNX_ERR_CUDA, "decode attention: tensor map encode failed");
    const int batch = a.batch;
    for (int b0 = 0; b0 < batch; b0 += BATCH) {
        a.batch = std::min(BATCH, batch - b0);
        // a CTA an SM, or for each unit that the cache could hold (a sequence has most runs at
        // the end of a range: 16 of 64 tokens at 1,024, 9 of 128 at 1,025)
        long long most = 1;
        for (int n : {1024, 4096, 32768, c.room}) most = std::max<long long>(most, runs(std::min(n, c.room)));
        const long long units = (long long)a.batch * most * a.Hkv * a.blocks;
        const int grid = (int)std::min<long long>(units, num_sms());
        pdl(k_decode_attn<HD>, grid, 32 * WARPS, C::SMEM, s)(tk, tv, a);
        const int heads = a.batch * a.H, of_cta = HD == 256 ? 4 : 8;
        if (most > 1 && heads <= num_sms() * 8) pdl(k_decode_join<HD, true>, heads, 256, 0, s)(a);
        else if (most > 1) pdl(k_decode_join<HD, false>, (heads + of_cta - 1) / of_cta, 256, 0, s)(a);
        a.q += a.batch * a.q_row;
        a.out += a.batch * a.o_row;
        a.slot += a.batch;
        a.n += a.batch;
    }
    return launched("decode attention");
}

}  // namespace jnx

using namespace jnx;

extern "C" size_t jnx_op_decode_attention_workspace_bytes(int32_t batch, int32_t n_heads,
                                                          int32_t head_dim) {
    if (batch < 0 || n_heads <= 0 || head_dim <= 0) return 0;
    return decode_sums_at(batch) + decode_runs(batch) * n_heads * (head_dim + 2) * sizeof(float);
}

extern "C" jnx_status jnx_op_decode_attention(const jnx_kv_cache* cache, int32_t batch,
                                              int32_t n_heads, int32_t n_kv_heads,
                                              int32_t head_dim, const jnx_head_rows* q,
                                              const int32_t* slot, const int32_t* n_cached,
                                              const jnx_head_rows* out, void* workspace,
                                              size_t ws_bytes, int32_t* status, void* stream) {
    clear_error();
    const char* what = "decode attention";
    if (jnx_status st = heads_ok(n_heads, n_kv_heads, head_dim, what)) return st;
    if (batch < 0) return fail(JNX_ERR_INVALID_ARG, "%s: negative batch", what);
    if (batch == 0) return JNX_OK;
    if (!cache_ok(cache) || !rows_ok(q) || !rows_ok(out) || !slot || !n_cached)
        return fail(JNX_ERR_INVALID_ARG, "%s: null or misaligned argument", what);
    if ((int64_t)batch * n_heads > 0x7fffff00 ||
        (int64_t)decode::BATCH * decode::MAX_RUNS * n_heads > 0x7fff0000)
        return fail(JNX_ERR_UNSUPPORTED, "%s: sizes", what);
    if (!workspace || !aligned16(workspace) ||
        ws_bytes < jnx_op_decode_attention_workspace_bytes(batch, n_heads, head_dim))
        return fail(JNX_ERR_WORKSPACE, "%s: workspace too small or misaligned", what);
    const int group = n_heads / n_kv_heads;
    DecodeArgs a{batch, n_heads, n_kv_heads, group, (group + decode::ROWS - 1) / decode::ROWS,
                 cache->n_slots, cache->room, (float)(1.4426950408889634 / sqrt((double)head_dim)),
                 q->ptr, q->row_stride, q->head_stride, out->ptr, out->row_stride,
                 out->head_stride, slot, n_cached, static_cast<int*>(workspace), nullptr, nullptr,
                 status};
    // one launch's runs at a time: a launch starts when the one ahead is through
    uint8_t* ws = static_cast<uint8_t*>(workspace) + decode_sums_at(batch);
    a.part = reinterpret_cast<float*>(ws);
    a.ml = reinterpret_cast<float2*>(a.part + decode_runs(batch) * n_heads * head_dim);
    // an empty cache has no tiles, but the maps want extents
    jnx_kv_cache c = *cache;
    c.n_slots = std::max(c.n_slots, 1);
    c.room = std::max(c.room, 1);
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    TraceScope ts(JNX_K_DECODE_ATTN, 0.0, s);
    if (head_dim == 64) return launch_decode<64>(c, a, s);
    if (head_dim == 128) return launch_decode<128>(c, a, s);
    return launch_decode<256>(c, a, s);
}
