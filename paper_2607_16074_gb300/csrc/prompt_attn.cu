// Attention of packed prompts: causal behind a prefix that every row sees, query rows
// the last of a sequence's positions, grouped heads.
//
// O = softmax(Q K^T / sqrt(hd)) V in one pass over the keys with a running maximum m and
// sum l: P = 2^(S c - m), O <- O 2^(m_old - m) + P V, l likewise; O / l does not depend
// on m, so m (and O) only move when a tile's maximum is over 2^8 times the old one.
//
// A 128-row tile holds (token, query head of one group) pairs: 128 / group tokens times
// the group's heads, so the heads that share a key head share its tiles, and a causal
// edge wastes 128 / group tokens of a tile and not 128.  An item is two such tiles in a
// row (one at head dim 256, whose O leaves no TMEM for a second) of one key head and
// walks the 128-key tiles that its last row sees.
//
// One CTA per SM, persistent, over the items from the longest to the shortest, forwards
// and backwards in turn so that the rounds' inequalities cancel.  Roles:
//   warp 0       TMA: the item's Q tiles (3-D boxes: 64 columns x heads x tokens), then
//                K and V through one ring of whole tiles, or of 16 KB quarters at head
//                dim 256 (K: 128 keys x 64 columns, V: 32 keys x 256 columns), in the
//                order the MMAs take them
//   warp 1       MMA issuer.  Two tiles: S of a tile overwrites its P once PV is issued
//                and the other tile's products run while this one's softmax does.  One
//                tile (head dim 256): two score buffers, S two key tiles ahead of PV.
//   warp 3       hands out the items, looked up ahead and checked
//   warps 4-     softmax and epilogue, a warpgroup a tile, a thread a row: the row's 128
//                scores are in registers, so no row quantity is exchanged
// P (bf16) overwrites the first 64 columns of its scores and is the TMEM A operand of
// the PV product; V is the MN-major B operand as it lies.
//
// Rows beyond a sequence's keys in its last V tile are zeroed in shared memory: they
// belong to another sequence and may be NaN, and 0 * NaN would reach O.
//
// Bound by the softmax that feeds the tensor cores: one prompt of 12,289 tokens, 32 heads
// on 8 of 128, takes 751 us, 1,650 TFLOP/s of the pairs that count (floor 653); 24 of up to
// 2,900 tokens, 461 us (floor 305), the diagonal's tiles and an item's first and last steps
// weighing more; in longer runs, at the clock that the power cap leaves, 778 and 496.  Three
// stubs of up to 300 tokens, 8 heads on one of 256: 12.1 us, one item's loads, products and
// softmax after one another.
#include <algorithm>
#include <type_traits>
#include <vector>

#include "jnx_dev.cuh"
#include "jnx_kernels.h"
#include "jnx_text.h"
#include "jnx_trace.h"

namespace jnx {

namespace pattn {
constexpr int BM = 128, BN = 128;
constexpr int STAGE = 2048;  // epilogue staging of a softmax warp: 32 rows x 32 columns
constexpr float kLazy = 8.0f;  // log2 growth of the maximum that moves it
// barriers: ring full / empty, then
enum { Q_FULL = 0, Q_EMPTY = 2, S_FULL = 4, P_HALF = 6, P_FULL = 8, O_FREE = 10, PV_DONE = 12,
       O_FULL = 14, DRAIN = 16, W_FULL = 17, W_EMPTY = 20, N_BARS = 23 };
constexpr int ITEMS = 3;  // items handed out at a time
}  // namespace pattn

template <int HD>
struct PromptCfg {
    static constexpr int NST = HD == 256 ? 1 : 2;  // row tiles of an item
    static constexpr int NCH = HD / 64;            // 64-column chunks of a row
    // ring units: whole K and V tiles, or at head dim 256, where two tiles would fill the
    // ring, quarters
    static constexpr int NU = HD == 256 ? 4 : 1;   // units of a K or V tile
    static constexpr int UNIT = pattn::BN * HD * 2 / NU;
    static constexpr int RING = HD == 256 ? 9 : HD == 128 ? 4 : 8;
    static constexpr int KCH = NCH / NU;           // chunks of a K unit
    static constexpr int VKEYS = pattn::BN / NU;   // keys of a V unit
    static constexpr int QB = pattn::BM * HD * 2;
    static constexpr int OFF_RING = NST * QB;
    static constexpr int OFF_STG = OFF_RING + RING * UNIT;
    static constexpr int OFF_BAR = OFF_STG + 4 * NST * pattn::STAGE;
    static constexpr int SMEM = OFF_BAR + (2 * RING + pattn::N_BARS) * 8 + 16 + pattn::ITEMS * 32 + 1024;
    static_assert(SMEM <= 227 * 1024, "shared memory per CTA");
    static constexpr int THREADS = 128 + 128 * NST;
    static constexpr uint32_t O_COL = 256;
};

struct PromptArgs {
    const int *cu_q, *cu_kv, *prefix;
    const int2* items;
    int n_seqs, rows, keys;  // what the items may name
    int n_work, H, Hkv, group;
    float scale_log2;
    uint16_t* out;
    long long o_row, o_head;
    float* lse;
    int* status;
};

// One item: rows from token i0 of a sequence (global row q0 + i0) over its keys.
struct PromptWork {
    int q0, i0, Lq, k0, Lk, pre, kvh;  // i0 < 0: no more

    // key tiles that row tile t (T tokens) visits
    __device__ __forceinline__ int key_tiles(int t, int T) const {
        const int a = i0 + t * T;
        if (a >= Lq) return 0;
        return (keys_seen(min(a + T, Lq) - 1, Lq, Lk, pre) + pattn::BN - 1) / pattn::BN;
    }
};

// 32 fp32 columns of a warp's rows (a lane a row) as bf16 to base + to[j], rows lane / 4 + 8 j
// (-1: none), unit lane % 4, through 2 KB of staging.
__device__ __forceinline__ void stage_rows(uint8_t* stg, int lane, const uint32_t (&w)[32], uint16_t* base,
                                           const long long (&to)[4]) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        uint32_t q[4];
#pragma unroll
        for (int e = 0; e < 4; ++e)
            q[e] = cvt_bf2(__uint_as_float(w[8 * j + 2 * e]), __uint_as_float(w[8 * j + 2 * e + 1]));
        *reinterpret_cast<uint4*>(stg + lane * 64 + ((j ^ ((lane >> 1) & 3)) << 4)) =
            make_uint4(q[0], q[1], q[2], q[3]);
    }
    __syncwarp();
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const int rr = 8 * j + (lane >> 2), un = lane & 3;
        const uint4 q = *reinterpret_cast<const uint4*>(stg + rr * 64 + ((un ^ ((rr >> 1) & 3)) << 4));
        if (to[j] >= 0) *reinterpret_cast<uint4*>(base + to[j] + un * 8) = q;
    }
    __syncwarp();
}

template <int HD>
__global__ void __launch_bounds__(PromptCfg<HD>::THREADS, 1)
    k_prompt_attn(const __grid_constant__ CUtensorMap tq, const __grid_constant__ CUtensorMap tk,
                  const __grid_constant__ CUtensorMap tv, const __grid_constant__ PromptArgs a) {
    using C = PromptCfg<HD>;
    using namespace pattn;
    constexpr int NST = C::NST, NU = C::NU, UNIT = C::UNIT, RING = C::RING, NCH = C::NCH;
    extern __shared__ uint8_t smem_raw[];
    uint8_t* sm = reinterpret_cast<uint8_t*>(
        (reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
    uint8_t* ring = sm + C::OFF_RING;
    uint64_t* full = reinterpret_cast<uint64_t*>(sm + C::OFF_BAR);
    uint64_t* empty = full + RING;
    uint64_t* bar = empty + RING;
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(bar + N_BARS);
    volatile int* fail_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
    const int warp = warp_uniform(threadIdx.x >> 5), lane = threadIdx.x & 31;
    const int T = tile_tokens(a.group);

    if (threadIdx.x == 0) {
        for (int i = 0; i < 2 * RING; ++i) mbar_init(&full[i], 1);
        for (int i = 0; i < N_BARS; ++i)
            mbar_init(&bar[i], i >= P_HALF && i < PV_DONE ? BM : i >= W_EMPTY ? 2 + 4 * NST : 1);
        *fail_flag = 0;
        fence_barrier_init();
        fence_proxy_async();
    }
    pdl_entry();  // TMEM is taken once the grid ahead has given its own back
    if (warp == 1) {
        tmem_alloc(tmem_slot, 512);
        tmem_relinquish();
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tbase = warp_uniform(*tmem_slot);
    volatile int* slots = fail_flag + 1;  // [ITEMS][8]
    // the next item as warp 3 hands it out; done() gives its slot back
    int seen = 0;
    auto next_item = [&](bool& ok) -> PromptWork {
        const int b = seen % ITEMS;
        if (!(ok = mbar_wait_warp(&bar[W_FULL + b], (seen / ITEMS) & 1)))
            return PromptWork{0, -1, 0, 0, 0, 0, 0};
        const volatile int* s = slots + 8 * b;
        return PromptWork{warp_uniform(s[0]), warp_uniform(s[1]), warp_uniform(s[2]), warp_uniform(s[3]),
                          warp_uniform(s[4]), warp_uniform(s[5]), warp_uniform(s[6])};
    };
    auto item_done = [&]() {
        __syncwarp();
        if (elect_one()) mbar_arrive(&bar[W_EMPTY + seen % ITEMS]);
        __syncwarp();
        ++seen;
    };

    if (warp == 0) {
        // ---------------- TMA producer ----------------
        if (elect_one()) {
            tma_prefetch_desc(&tq);
            tma_prefetch_desc(&tk);
            tma_prefetch_desc(&tv);
        }
        bool ok = true;
        uint32_t u = 0;               // units loaded
        uint32_t nq[2] = {0, 0};      // Q tiles loaded
        const int qbytes = a.group * T * HD * 2;
        auto load_tile = [&](bool is_v, const PromptWork& x, int kt) -> bool {
            for (int c = 0; c < NU; ++c, ++u) {
                const int s = u % RING;
                if (!mbar_wait_warp(&empty[s], ((u / RING) & 1) ^ 1)) return false;
                if (elect_one()) {
                    mbar_arrive_expect_tx(&full[s], UNIT);
                    uint8_t* dst = ring + s * UNIT;
                    const int row = x.k0 + kt * BN;
                    if (!is_v) {
#pragma unroll
                        for (int j = 0; j < C::KCH; ++j)
                            tma_load_3d(dst + j * BN * 128, &tk, (c * C::KCH + j) * 64, x.kvh, row,
                                        &full[s]);
                    } else {
#pragma unroll
                        for (int j = 0; j < NCH; ++j)
                            tma_load_3d(dst + j * C::VKEYS * 128, &tv, j * 64, x.kvh,
                                        row + c * C::VKEYS, &full[s]);
                    }
                }
                __syncwarp();
            }
            return true;
        };
        while (ok) {
            const PromptWork x = next_item(ok);
            if (!ok || x.i0 < 0 || __any_sync(0xffffffffu, *fail_flag)) break;
            item_done();
            const int n = max(x.key_tiles(0, T), NST == 2 ? x.key_tiles(1, T) : 0);
            // the first keys do not wait for the last item's Q tiles to be free
            if (n > 0) ok = load_tile(false, x, 0);
            for (int t = 0; t < NST && ok; ++t) {
                if (x.key_tiles(t, T) == 0) continue;
                if (nq[t] > 0 && !(ok = mbar_wait_warp(&bar[Q_EMPTY + t], (nq[t] - 1) & 1))) break;
                if (elect_one()) {
                    mbar_arrive_expect_tx(&bar[Q_FULL + t], qbytes);
#pragma unroll
                    for (int c = 0; c < NCH; ++c)
                        tma_load_3d(sm + t * C::QB + c * BM * 128, &tq, c * 64, x.kvh * a.group,
                                    x.q0 + x.i0 + t * T, &bar[Q_FULL + t]);
                }
                __syncwarp();
                ++nq[t];
            }
            // K runs ahead of V by as many tiles as S runs ahead of PV
            constexpr int AHEAD = NST == 1 ? 2 : 1;
            for (int kt = 1; kt < AHEAD && kt < n && ok; ++kt) ok = load_tile(false, x, kt);
            for (int kt = 0; kt < n && ok; ++kt) {
                ok = load_tile(true, x, kt);
                if (ok && kt + AHEAD < n) ok = load_tile(false, x, kt + AHEAD);
            }
        }
        if (!ok) *fail_flag = 1;
        // every copy has landed before the CTA may exit (at once in a normal run)
        for (int t = 0; t < NST; ++t)
            if (nq[t] > 0) mbar_wait_warp(&bar[Q_FULL + t], (nq[t] - 1) & 1, 100000000LL);
        for (uint32_t i = u > RING ? u - RING : 0; i < u; ++i)
            mbar_wait_warp(&full[i % RING], (i / RING) & 1, 100000000LL);
    } else if (warp == 1) {
        // ---------------- MMA issuer ----------------
        constexpr uint32_t IDESC_S = idesc_bf16_f32(BM, BN);
        constexpr uint32_t IDESC_PV = idesc_bf16_f32(BM, HD) | (1u << 16);  // B MN-major
        bool ok = true, issued = false;
        uint32_t u = 0;                           // units taken
        uint32_t nq[2] = {0, 0}, gp[2] = {0, 0};  // Q tiles, P tiles taken (by P barrier)
        uint32_t no[2] = {0, 0};                  // items begun (per O accumulator)
        uint32_t gs = 0;                          // score tiles issued (NST == 1)
        const uint32_t q_lo = sw128_desc_lo(smem_u32(sm)), r_lo = sw128_desc_lo(smem_u32(ring));
        auto commit = [&](uint64_t* b) {
            if (elect_one()) tc_commit(b);
            __syncwarp();
        };
        auto wait_units = [&](uint32_t first) -> bool {
            for (uint32_t i = first; i < first + NU; ++i)
                if (!mbar_wait_warp(&full[i % RING], (i / RING) & 1)) return false;
            tc_fence_after();
            return true;
        };
        auto free_units = [&](uint32_t first) {
            if (elect_one())
                for (uint32_t i = first; i < first + NU; ++i) tc_commit(&empty[i % RING]);
            __syncwarp();
        };
        // S (columns d) of row tile t against the K tile in units [first, first + NU)
        auto issue_s = [&](int t, uint32_t first, uint32_t d, uint64_t* done) {
            const uint32_t a_lo = q_lo + t * (C::QB >> 4);
            uint32_t k_lo[NU];
#pragma unroll
            for (int c = 0; c < NU; ++c) k_lo[c] = r_lo + ((first + c) % RING) * (UNIT >> 4);
            if (elect_one()) {
#pragma unroll
                for (int c = 0; c < NCH; ++c)
#pragma unroll
                    for (int ks = 0; ks < 4; ++ks)
                        tc_mma_f16(d, desc_of(a_lo + c * (BM * 128 >> 4) + ks * 2, kSw128DescHi),
                                   desc_of(k_lo[c / C::KCH] + c % C::KCH * (BN * 128 >> 4) + ks * 2,
                                           kSw128DescHi),
                                   IDESC_S, (c | ks) != 0);
                tc_commit(done);
            }
            __syncwarp();
            issued = true;
        };
        // O (columns d) += P (columns p) times half h of the V tile in units [first, first + NU)
        const uint32_t v_lo = sw128_desc_mn_lo(smem_u32(ring), C::VKEYS * 128);
        auto issue_pv = [&](auto half, uint32_t p, uint32_t first, uint32_t d, bool accumulate) {
            constexpr int h = decltype(half)::value, UH = NU == 1 ? 1 : NU / 2;  // units of a half
            uint32_t lo[UH];
#pragma unroll
            for (int c = 0; c < UH; ++c)
                lo[c] = v_lo + ((first + (NU == 1 ? 0 : h * UH + c)) % RING) * (UNIT >> 4);
            if (elect_one()) {
#pragma unroll
                for (int k = 0; k < BN / 32; ++k) {
                    const int ks = h * (BN / 32) + k;
                    tc_mma_f16_ts(d, p + ks * 8,
                                  desc_of(lo[NU == 1 ? 0 : k * 16 / C::VKEYS] +
                                              ks * 16 % C::VKEYS * (128 >> 4),
                                          kSw128DescHi),
                                  IDESC_PV, accumulate || k > 0);
                }
            }
            __syncwarp();
        };
        // rows of the V tile from `valid` on are not the sequence's: zero them
        auto zero_tail = [&](uint32_t first, int valid) {
            for (int r = valid; r < BN; ++r) {
                uint8_t* row = ring + ((first + r / C::VKEYS) % RING) * UNIT + r % C::VKEYS * 128;
                for (int i = lane; i < HD / 8; i += 32)
                    *reinterpret_cast<uint4*>(row + (i >> 3) * C::VKEYS * 128 + (i & 7) * 16) =
                        make_uint4(0, 0, 0, 0);
            }
            fence_proxy_async();
            __syncwarp();
        };
        while (ok) {
            const PromptWork x = next_item(ok);
            if (!ok || x.i0 < 0 || __any_sync(0xffffffffu, *fail_flag)) break;
            item_done();
            int nt[2] = {x.key_tiles(0, T), NST == 2 ? x.key_tiles(1, T) : 0};
            const int n = max(nt[0], nt[1]);
            if (n == 0) continue;
            for (int t = 0; t < NST && ok; ++t)
                if (nt[t] > 0) {
                    ok = mbar_wait_warp(&bar[Q_FULL + t], nq[t] & 1);
                    ++nq[t];
                }
            tc_fence_after();
            if constexpr (NST == 2) {
                if (!ok || !(ok = wait_units(u))) break;
                for (int t = 0; t < 2; ++t)
                    if (nt[t] > 0) {
                        issue_s(t, u, tbase + t * BN, &bar[S_FULL + t]);
                        if (nt[t] == 1) commit(&bar[Q_EMPTY + t]);
                    }
                free_units(u);
                u += NU;
                for (int kt = 0; kt < n && ok; ++kt) {
                    const uint32_t uv = u, uk = u + NU;  // V(kt), K(kt + 1)
                    // the tiles that the products below take, waited for before P: they are
                    // mostly there, and P is what the tensor core then waits for
                    if (!(ok = wait_units(uv))) break;
                    if (x.Lk - kt * BN < BN) zero_tail(uv, x.Lk - kt * BN);
                    if (kt + 1 < n && !(ok = wait_units(uk))) break;
                    for (int t = 0; t < 2; ++t) {
                        if (kt >= nt[t]) continue;
                        if (!(ok = mbar_wait_warp(&bar[P_HALF + t], gp[t] & 1))) break;
                        // the item's first product overwrites O: the last epilogue has read it
                        if (kt == 0) {
                            if (no[t] > 0 && !(ok = mbar_wait_warp(&bar[O_FREE + t], (no[t] - 1) & 1)))
                                break;
                            ++no[t];
                        }
                        tc_fence_after();
                        issue_pv(std::integral_constant<int, 0>{}, tbase + t * BN, uv, tbase + C::O_COL + t * HD, kt > 0);
                        if (!(ok = mbar_wait_warp(&bar[P_FULL + t], gp[t] & 1))) break;
                        ++gp[t];
                        tc_fence_after();
                        issue_pv(std::integral_constant<int, 1>{}, tbase + t * BN, uv, tbase + C::O_COL + t * HD, true);
                        if (kt + 1 < nt[t]) {
                            issue_s(t, uk, tbase + t * BN, &bar[S_FULL + t]);
                            if (kt + 2 == nt[t]) commit(&bar[Q_EMPTY + t]);
                        } else {
                            commit(&bar[O_FULL + t]);
                        }
                    }
                    if (!ok) break;
                    free_units(uv);
                    u = uk;
                    if (kt + 1 < n) {
                        free_units(uk);
                        u += NU;
                    }
                }
            } else {
                // score tile i goes to buffer gs % 2
                auto next_s = [&](int kt) -> bool {
                    if (!wait_units(u)) return false;
                    issue_s(0, u, tbase + (gs & 1) * BN, &bar[S_FULL + (gs & 1)]);
                    free_units(u);
                    u += NU;
                    ++gs;
                    if (kt + 1 == n) commit(&bar[Q_EMPTY]);
                    return true;
                };
                ok = ok && next_s(0) && (n < 2 || next_s(1));
                for (int kt = 0; kt < n && ok; ++kt) {
                    const uint32_t b = gp[0] & 1;
                    if (!(ok = wait_units(u))) break;
                    if (x.Lk - kt * BN < BN) zero_tail(u, x.Lk - kt * BN);
                    if (!(ok = mbar_wait_warp(&bar[P_HALF + b], (gp[0] >> 1) & 1))) break;
                    if (kt == 0) {
                        if (no[0] > 0 && !(ok = mbar_wait_warp(&bar[O_FREE], (no[0] - 1) & 1))) break;
                        ++no[0];
                    }
                    tc_fence_after();
                    issue_pv(std::integral_constant<int, 0>{}, tbase + b * BN, u, tbase + C::O_COL, kt > 0);
                    if (!(ok = mbar_wait_warp(&bar[P_FULL + b], (gp[0] >> 1) & 1))) break;
                    ++gp[0];
                    tc_fence_after();
                    issue_pv(std::integral_constant<int, 1>{}, tbase + b * BN, u, tbase + C::O_COL, true);
                    commit(&bar[PV_DONE + b]);
                    free_units(u);
                    u += NU;
                    if (kt + 2 < n) ok = next_s(kt + 2);
                }
                if (ok) commit(&bar[O_FULL]);
            }
        }
        if (!ok) *fail_flag = 1;
        if (issued) {
            commit(&bar[DRAIN]);
            mbar_wait_warp(&bar[DRAIN], 0, 100000000LL);
        }
    } else if (warp == 3) {
        // ---------------- items ----------------
        // the longest first, forwards and backwards in turn over the CTAs
        bool ok = true;
        auto work = [&](int r) {
            const int G = gridDim.x, b = blockIdx.x;
            return r * G + ((r & 1) ? G - 1 - b : b);
        };
        auto entry = [&](int w) { return w < a.n_work ? a.items[w / a.Hkv] : make_int2(0, 0); };
        const int rounds = (a.n_work + gridDim.x - 1) / gridDim.x;
        int2 e = entry(work(0));
        int told = 0;
        auto room = [&]() {
            return mbar_wait_warp(&bar[W_EMPTY + told % ITEMS], ((told / ITEMS) & 1) ^ 1);
        };
        auto tell = [&](const PromptWork& x) {
            const int b = told % ITEMS;
            if (elect_one()) {
                volatile int* s = slots + 8 * b;
                s[0] = x.q0;
                s[1] = x.i0;
                s[2] = x.Lq;
                s[3] = x.k0;
                s[4] = x.Lk;
                s[5] = x.pre;
                s[6] = x.kvh;
                mbar_arrive(&bar[W_FULL + b]);
            }
            __syncwarp();
            ++told;
        };
        for (int r = 0; r < rounds && ok && !__any_sync(0xffffffffu, *fail_flag); ++r) {
            const int2 c = e;
            const int w = work(r);
            e = entry(work(r + 1));
            if (w >= a.n_work) continue;
            PromptSeq x;
            const bool known = prompt_seq(a.cu_q, a.cu_kv, a.prefix, a.n_seqs, a.rows, a.keys, c.x, x);
            if (!(ok = room())) break;
            if (known && (unsigned)c.y < (unsigned)x.Lq)
                tell(PromptWork{x.q0, c.y, x.Lq, x.k0, x.Lk, x.pre, w % a.Hkv});
            else if (lane == 0)
                report(a.status, JNX_ERR_DEVICE_BOUNDS);
        }
        ok = ok && room();
        if (ok) tell(PromptWork{0, -1, 0, 0, 0, 0, 0});
        else *fail_flag = 1;
    } else if (warp >= 4) {
        // ---------------- softmax + epilogue of row tile t ----------------
        const int t = (warp - 4) >> 2;
        const int row = (warp & 3) * 32 + lane;
        const uint32_t lane_base = (uint32_t)((warp & 3) * 32) << 16;
        const uint32_t tO = tbase + lane_base + C::O_COL + t * HD;
        uint32_t g = 0, items_done = 0;  // score tiles, items with keys
        bool ok = true;
        const int tok = row / a.group, hg = row % a.group;
        uint8_t* stg = sm + C::OFF_STG + (warp - 4) * STAGE;
        while (ok) {
            int n, lim;
            {
                const PromptWork x = next_item(ok);
                if (!ok || x.i0 < 0 || __any_sync(0xffffffffu, *fail_flag)) break;
                n = x.key_tiles(t, T);
                const int i = x.i0 + t * T + tok;
                // keys of this row; a row that is none of the tile's has no say in the masks
                lim = tok < T && i < x.Lq ? keys_seen(i, x.Lq, x.Lk, x.pre) : 0x7fffffff;
            }
            float m = -INFINITY, l = 0.f;
            for (int kt = 0; kt < n; ++kt) {
                const uint32_t b = NST == 1 ? g & 1 : t;
                const uint32_t ph = NST == 1 ? (g >> 1) & 1 : g & 1;
                const uint32_t tS = tbase + lane_base + b * BN;
                if (!(ok = __all_sync(0xffffffffu, mbar_wait(&bar[S_FULL + b], ph)))) break;
                tc_fence_after();
                uint32_t v[4][32];
#pragma unroll
                for (int c = 0; c < 4; ++c) tmem_ld32(tS + c * 32, v[c]);
#pragma unroll
                for (int c = 0; c < 4; ++c) tmem_ld_wait_regs(v[c]);
                const bool whole = __all_sync(0xffffffffu, lim >= (kt + 1) * BN);
                if (!whole) {
#pragma unroll
                    for (int c = 0; c < 4; ++c)
#pragma unroll
                        for (int e = 0; e < 32; ++e)
                            if (kt * BN + c * 32 + e >= lim) v[c][e] = 0xff800000u;  // -inf
                }
                float mx[4];
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    mx[c] = __uint_as_float(v[c][0]);
#pragma unroll
                    for (int e = 1; e < 31; e += 2)
                        mx[c] = fmax3(mx[c], __uint_as_float(v[c][e]), __uint_as_float(v[c][e + 1]));
                    mx[c] = fmaxf(mx[c], __uint_as_float(v[c][31]));
                }
                const float top = fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3])) * a.scale_log2;
                float alpha = 1.f;
                if (kt == 0) {
                    m = top;
                } else if (top > m + kLazy) {
                    alpha = ex2_approx(m - top);
                    m = top;
                }
                if (kt > 0 && __any_sync(0xffffffffu, alpha < 1.f)) {
                    // every earlier PV of the item is done: with one score buffer S was
                    // issued behind it, with two it is waited for
                    if (NST == 1) {
                        const uint32_t pb = (g - 1) & 1;
                        if (!(ok = __all_sync(0xffffffffu, mbar_wait(&bar[PV_DONE + pb],
                                                                     ((g - 1) >> 1) & 1))))
                            break;
                        tc_fence_after();
                    }
#pragma unroll 1
                    for (int c = 0; c < HD / 16; ++c) {
                        uint32_t o16[16];
                        tmem_ld16(tO + c * 16, o16);
                        tmem_ld_wait_regs16(o16);
#pragma unroll
                        for (int e = 0; e < 16; ++e)
                            o16[e] = __float_as_uint(__uint_as_float(o16[e]) * alpha);
                        tmem_st16(tO + c * 16, o16);
                    }
                    tmem_st_wait();
                }
                // a row that has seen no key yet subtracts nothing
                const float sub = m == -INFINITY ? 0.f : m;
                const uint64_t sc2 = f2_pack(a.scale_log2, a.scale_log2), nm2 = f2_pack(-sub, -sub);
                uint64_t rs[2] = {f2_pack(0.f, 0.f), f2_pack(0.f, 0.f)};
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    uint32_t pk[32];
#pragma unroll
                    for (int c = 0; c < 2; ++c)
#pragma unroll
                        for (int e = 0; e < 32; e += 2) {
                            float x0, x1, p0, p1;
                            f2_unpack(f2_fma(f2_pack(__uint_as_float(v[2 * h + c][e]),
                                                     __uint_as_float(v[2 * h + c][e + 1])),
                                             sc2, nm2),
                                      x0, x1);
                            p0 = ex2_approx(x0);
                            p1 = ex2_approx(x1);
                            rs[(e >> 1) & 1] = f2_add(rs[(e >> 1) & 1], f2_pack(p0, p1));
                            pk[c * 16 + e / 2] = cvt_bf2(p0, p1);
                        }
                    tmem_st32(tS + h * 32, pk);
                    // the first 64 keys' product starts while the others' P is formed
                    tmem_st_wait();
                    tc_fence_before();
                    if (h == 0) mbar_arrive(&bar[P_HALF + b]);
                }
                float r0, r1, r2, r3;
                f2_unpack(rs[0], r0, r1);
                f2_unpack(rs[1], r2, r3);
                l = l * alpha + ((r0 + r1) + (r2 + r3));
                mbar_arrive(&bar[P_FULL + b]);
                ++g;
            }
            if (!ok) break;
            if (n > 0) {
                if (!(ok = __all_sync(0xffffffffu, mbar_wait(&bar[O_FULL + t], items_done & 1)))) break;
                tc_fence_after();
                ++items_done;
            }
            const volatile int* s = slots + 8 * (seen % ITEMS);
            const int i = s[1] + t * T + tok, row0 = s[0], h = s[6] * a.group + hg;
            const bool live = tok < T && i < s[2];
            item_done();
            if (live && a.lse) a.lse[(size_t)(row0 + i) * a.H + h] = m + log2f(l);
            const float inv = l > 0.f ? 1.f / l : 0.f;
            // out through the warp's staging, 32 columns at a time: this lane writes its
            // row's four units and stores unit lane % 4 of rows lane / 4 + 8 j
            const long long o = live ? (long long)(row0 + i) * a.o_row + h * a.o_head : -1;
            long long to[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) to[j] = __shfl_sync(0xffffffffu, o, 8 * j + (lane >> 2));
#pragma unroll 1
            for (int c = 0; c < HD / 32; ++c) {
                uint32_t w[32];
                if (n > 0) {
                    tmem_ld32(tO + c * 32, w);
                    tmem_ld_wait_regs(w);
                    if (c + 1 == HD / 32) {
                        tc_fence_before();
                        mbar_arrive(&bar[O_FREE + t]);
                    }
                } else {
#pragma unroll
                    for (int e = 0; e < 32; ++e) w[e] = 0;
                }
                // a row without keys: O holds products of zeros
#pragma unroll
                for (int e = 0; e < 32; ++e)
                    w[e] = l > 0.f ? __float_as_uint(__uint_as_float(w[e]) * inv) : 0u;
                stage_rows(stg, lane, w, a.out + c * 32, to);
            }
        }
        if (!ok) *fail_flag = 1;
    }
    __syncwarp();
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    if (*fail_flag && threadIdx.x == 0) report(a.status, JNX_ERR_TIMEOUT);
    if (warp == 1) tmem_dealloc(tbase, 512);
}

template <int HD>
static jnx_status launch_prompt(const PromptArgs& a, const jnx_head_rows& q, const jnx_head_rows& k,
                                const jnx_head_rows& v, int rows, int keys, cudaStream_t s) {
    using C = PromptCfg<HD>;
    static std::atomic<uint64_t> attr{0};
    if (set_smem_limit(reinterpret_cast<const void*>(k_prompt_attn<HD>), C::SMEM, attr) != cudaSuccess)
        return fail(JNX_ERR_CUDA, "prompt attention: smem attribute");
    CUtensorMap tq, tk, tv;
    if (!make_tmap_heads(&tq, q, rows, a.H, HD, a.group, tile_tokens(a.group)) ||
        !make_tmap_heads(&tk, k, keys, a.Hkv, HD, 1, pattn::BN) ||
        !make_tmap_heads(&tv, v, keys, a.Hkv, HD, 1, C::VKEYS))
        return fail(JNX_ERR_CUDA, "prompt attention: tensor map encode failed");
    const int grid = std::min(a.n_work, num_sms());
    pdl(k_prompt_attn<HD>, grid, C::THREADS, C::SMEM, s)(tq, tk, tv, a);
    return launched("prompt attention");
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

// ... and its device arrays, for a launch over its rows (gradients: over its keys too).
jnx_status prompt_launchable(const jnx_prompt* p, const char* what, bool gradients, int& rows,
                             int& keys) {
    if (jnx_status st = prompt_ok(p, what, rows, keys)) return st;
    if ((rows > 0 || (gradients && keys > 0)) &&
        (!p->cu_q || !p->cu_kv || !p->items || (p->h_prefix && !p->prefix)))
        return fail(JNX_ERR_INVALID_ARG, "%s: null device arrays", what);
    // the parts of a key tile's rows, and with them the workspace, follow from the prefix
    if (gradients && p->prefix && !p->h_prefix)
        return fail(JNX_ERR_INVALID_ARG, "%s: prefix on the device alone", what);
    if (p->n_forward < 0 || p->n_keys < 0 || p->n_queries < 0 || p->n_parts < 0 ||
        p->n_parts > kMaxParts)
        return fail(JNX_ERR_INVALID_ARG, "%s: bad work list", what);
    return JNX_OK;
}

PromptCounts prompt_counts(const jnx_prompt* p, int H, int Hkv, int hd, bool gradients) {
    const int group = H / Hkv, T = tile_tokens(group), step = T * item_tiles(hd);
    PromptCounts n;
    int least = 0x7fffffff;  // rows of an item of a tile in parts
    for (int s = 0; s < p->n_seqs; ++s) {
        const int Lq = p->h_cu_q[s + 1] - p->h_cu_q[s], Lk = p->h_cu_kv[s + 1] - p->h_cu_kv[s];
        const int pre = p->h_prefix ? p->h_prefix[s] : 0;
        n.forward += ((long long)Lq + step - 1) / step;
        if (!gradients) continue;
        n.queries += ((long long)Lq + T - 1) / T;
        for (long long at = 0; at < Lk; at += 128) {
            const int np = key_parts((int)at, Lq, Lk, pre, group, Hkv);
            n.keys += np;
            n.parts = std::max(n.parts, np);
            if (np > 1) least = std::min(least, part_rows((int)at, Lq, Lk, pre, np));
        }
    }
    // the list has the items of most rows first
    for (int s = 0; s < p->n_seqs && n.parts > 1; ++s) {
        const int Lq = p->h_cu_q[s + 1] - p->h_cu_q[s], Lk = p->h_cu_kv[s + 1] - p->h_cu_kv[s];
        const int pre = p->h_prefix ? p->h_prefix[s] : 0;
        for (long long at = 0; at < Lk; at += 128) {
            const int np = key_parts((int)at, Lq, Lk, pre, group, Hkv);
            if (part_rows((int)at, Lq, Lk, pre, np) >= least) n.slabs += np;
        }
    }
    return n;
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
        int count[3], parts = 1;
        for (int pass = 0; pass < 3; ++pass) {
            const size_t first = all.size();
            for (int s = 0; s < p->n_seqs; ++s) {
                const int Lq = p->h_cu_q[s + 1] - p->h_cu_q[s];
                const int Lk = p->h_cu_kv[s + 1] - p->h_cu_kv[s];
                const int pre = p->h_prefix ? p->h_prefix[s] : 0;
                const int end = pass == 1 ? Lk : Lq;
                for (long long at = 0; at < end; at += step[pass]) {
                    const int last = (int)std::min<long long>(at + step[pass], end) - 1;
                    const int np = pass == 1 ? key_parts((int)at, Lq, Lk, pre, n_heads / n_kv_heads,
                                                         n_kv_heads)
                                             : 1;
                    const long long cost = pass == 1 ? part_rows((int)at, Lq, Lk, pre, np)
                                                     : keys_seen(last, Lq, Lk, pre);
                    parts = std::max(parts, np);
                    for (int k = 0; k < np; ++k) all.push_back({s, (int)at + k, cost});
                }
            }
            // (stable: a tile's parts stay together and in order)
            std::stable_sort(all.begin() + first, all.end(),
                             [](const Item& x, const Item& y) { return x.cost > y.cost; });
            count[pass] = (int)(all.size() - first);
        }
        if (all.size() > 0x3fffffff) return fail(JNX_ERR_UNSUPPORTED, "prompt items: too many");
        p->n_forward = count[0];
        p->n_keys = count[1];
        p->n_queries = count[2];
        p->n_parts = parts;
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
                                              const jnx_head_rows* /* rest */, float* lse,
                                              int32_t* status, void* stream) {
    clear_error();
    int rows, keys;
    if (jnx_status st = heads_ok(n_heads, n_kv_heads, head_dim, "prompt attention")) return st;
    if (jnx_status st = prompt_launchable(p, "prompt attention", false, rows, keys)) return st;
    if (rows == 0) return JNX_OK;
    if (!rows_ok(q) || !rows_ok(out) || (keys > 0 && (!rows_ok(k) || !rows_ok(v))))
        return fail(JNX_ERR_INVALID_ARG, "prompt attention: null or misaligned rows");
    const long long n_work = (long long)p->n_forward * n_kv_heads;
    if (n_work > 0x7FFFFFFFLL - 2 * num_sms())
        return fail(JNX_ERR_UNSUPPORTED, "prompt attention: too many work items");
    if (p->n_forward != prompt_counts(p, n_heads, n_kv_heads, head_dim, false).forward)
        return fail(JNX_ERR_INVALID_ARG, "prompt attention: a work list of other heads or lengths");
    // without any key no tile is loaded, but the maps want an address
    const jnx_head_rows kk = keys ? *k : *q, vv = keys ? *v : *q;
    PromptArgs a{p->cu_q, p->cu_kv, p->prefix, reinterpret_cast<const int2*>(p->items), p->n_seqs, rows,
                 keys, (int)n_work, n_heads, n_kv_heads, n_heads / n_kv_heads,
                 (float)(1.4426950408889634 / sqrt((double)head_dim)), out->ptr, out->row_stride,
                 out->head_stride, lse, status};
    if (!keys) keys = 1;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    TraceScope ts(JNX_K_PROMPT_ATTN, 0.0, s);
    if (head_dim == 64) return launch_prompt<64>(a, *q, kk, vv, rows, keys, s);
    if (head_dim == 128) return launch_prompt<128>(a, *q, kk, vv, rows, keys, s);
    return launch_prompt<256>(a, *q, kk, vv, rows, keys, s);
}
