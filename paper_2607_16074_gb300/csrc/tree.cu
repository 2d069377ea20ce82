// Attention of trees of drafted tokens against a paged cache.
//
// Node i of a sequence sees the cached tokens and the nodes that its bits name, whose keys
// and values lie behind the cached ones: O = softmax(Q K^T / sqrt(hd)) V over them, in one
// pass with a running maximum m and sum l.  P = 2^(S c - m), O <- O 2^(m_old - m) + P V; m
// moves only when a tile's maximum is over 2^8 times the old one, which O / l does not show.
//
// Bound by reading the cache once.  A 128-row tile holds (node, query head of one group)
// pairs, up to 128 / group nodes, so a key head's tokens are read once for all of them, and
// at 48 rows or 128 the products are past what mma.sync could do at the cache's rate.  A unit
// is such a tile over a run of its sequence's tokens.  Persistent CTAs take units in turn,
// two to an SM (one at head dim 256, whose O leaves no TMEM for a second): while one's
// softmax works, the other's keys come in.  Roles of a CTA:
//   warp 0      TMA: Q, then K and V tiles of 64 tokens, 16 to 64 to a box by what divides a
//               page, into a ring each; the table's entries are looked up ahead
//   warp 1      MMA issuer: S two key tiles ahead of P V
//   warps 2-5   softmax and epilogue, a thread a row
// P overwrites its scores and is the TMEM A operand of the P V product.  It is bf16, as V is (a
// product's operands are of one type); l sums what was not rounded.  Against 64 bits the outputs
// are off by 0.0017 to 0.0023 in norm, of which their own rounding is 0.0014 to 0.0017.
//
// The run's length depends on the sequence alone, so a sequence's bits do not depend on the
// others; its runs' sums are joined in their order by a second kernel.
//
// 64 trees of up to 12 nodes over up to 8,100 tokens, 32 heads on 8 of 128: 189 us, 5.7 TB/s
// (floor 158; the attention 185, the join's last CTAs 4).  One of 16 nodes over 60,001 tokens
// 51.3 (floor 36.5; start, last unit and join 8 or so of it), 8 of up to 6 over up to 700, 8
// heads on one of 256, 13: latency, two launches' chains of lookups, loads, three or four tiles
// and sums.  24 of up to 64 nodes over up to 3,500: 29.5, the tensor cores' and softmax's, tiles
// of 64 tokens for 128 rows, and 148 units of which the longest has 15 tiles, the mean 9.7 (floor
// 6.7).
//
// Not kept: the products the other way round, tokens as the rows and the pairs as 64 columns, so
// that few pairs cost no more than they are (a unit's sums and epilogue took 12,000 clocks: 260 us
// for 192 of the 64 trees' attention); tiles of 128 tokens at head dim 64 (64 of up to 20,000
// tokens, 14 heads on 2: 104 us for 90); S of the next unit ahead of this one's last products, or
// sequences in the order of their runs' lengths (no change, or 200 us for 195).
#include <algorithm>

#include "jnx_dev.cuh"
#include "jnx_kernels.h"
#include "jnx_text.h"
#include "jnx_trace.h"

namespace jnx {

namespace tree {
constexpr int KT = 64;         // tokens of a tile
constexpr int RINGS = 5;       // tiles of either ring, at most
constexpr int BATCH = 256;     // sequences of one launch
constexpr int MAX_RUNS = 64;   // of a sequence
constexpr int THREADS = 192;
constexpr float kLazy = 8.0f;  // log2 growth of the maximum that moves it
enum { K_FULL = 0, K_EMPTY = K_FULL + RINGS, V_FULL = K_EMPTY + RINGS, V_EMPTY = V_FULL + RINGS,
       Q_FULL = V_EMPTY + RINGS, Q_EMPTY = Q_FULL + 2, S_FULL = Q_EMPTY + 2, P_FULL = S_FULL + 2, PV_DONE = P_FULL + 2,
       O_FULL = PV_DONE + 2, O_FREE, DRAIN, N_BARS };

__host__ __device__ inline int round_up(int n, int to) { return (n + to - 1) / to * to; }

// Tokens of a run of L, for `rows` rows of a tile and `units` units of a run.  A run's sums are
// rows / tokens of what it reads, and its epilogue costs what two or three tiles do, hence long
// runs of long sequences (64 trees over up to 8,100 tokens 188 us; 197 with 32 times the rows, 184
// with 1,024 tokens of any, which takes a lone sequence of 4,000 18 us for 13.6), and as many of
// short ones as reach more SMs (8 over up to 700 tokens 13 us, 20 with 32 times the rows).  At
// head dim 256, where a tile's products are longer than its way from memory, a sequence of few
// heads has runs for a fifth of the card (8 nodes over 8,000 tokens, one key head: 13.4 us, 22.6
// without).  One that fills the card by itself has whole rounds of units.
__host__ __device__ inline int run_tokens(int L, int rows, int units, int slots, bool wide) {
    int least = L <= 2048 ? 4 * rows : L <= 4096 ? (8 * rows < 512 ? 512 : 8 * rows) : 1024;
    if (wide && L > 2048) {
        const int share = (int)((long long)L * units / 32 < 1024 ? (long long)L * units / 32 : 1024);
        const int sums = (units > 1 || rows > 64 ? 8 : 4) * rows;
        least = share > sums ? share : sums;
    }
    least = round_up(least < 256 ? 256 : least, KT);
    int n = (L + least - 1) / least;
    if (n > MAX_RUNS) n = MAX_RUNS;
    if ((long long)n * units > slots) n = (int)((long long)n * units / slots * slots / units);
    if (n < 1) n = 1;
    return round_up((L + n - 1) / n, KT);
}
// No sequence of up to max_tokens has more runs: at head dims 64 and 128 up to 8 of 256 tokens or
// of 512, then of 1,024; at 256, where a unit's share counts, up to 33 of 256 to 1,024.
inline long long most_runs(long long max_tokens, bool wide) {
    const long long shorts = std::min(wide ? 33ll : 8ll, (max_tokens + 255) / 256);
    return std::max({1ll, shorts, std::min<long long>(MAX_RUNS, (max_tokens + 1023) / 1024)});
}
}  // namespace tree

template <int HD>
struct TreeCfg {
    static constexpr int NCH = HD / 64;                  // 64-column chunks of a row
    static constexpr int CTAS = HD == 256 ? 1 : 2;       // of an SM
    static constexpr int SLOTS = 152 * CTAS;
    static constexpr int TILE = tree::KT * HD * 2;
    static constexpr int RING = HD == 64 ? 5 : 2;  // tiles of either ring
    static constexpr int QB = 128 * HD * 2;
    static constexpr int OFF_K = QB, OFF_V = OFF_K + RING * TILE;
    static constexpr int OFF_SEQ = OFF_V + RING * TILE;
    static constexpr int OFF_BAR = OFF_SEQ + (6 * tree::BATCH + 4) * 4 + tree::BATCH * 4;
    static constexpr int SMEM = OFF_BAR + tree::N_BARS * 8 + 16 + 1024;
    static_assert(SMEM <= (CTAS == 2 ? 113 : 226) * 1024, "shared memory per CTA");
    static constexpr uint32_t COLS = HD == 256 ? 512 : 256, O_COL = HD == 256 ? 256 : 128;
};

struct TreeArgs {
    Pages pages;
    int no_page;     // outside of the maps: read as zeros
    int n_seqs, s0;  // sequences of the launch, the first of them
    int H, Hkv, group, n_rows, box;
    float scale_log2;
    uint16_t* out;
    long long o_row, o_head;
    const int *cu_nodes, *n_cached;
    const unsigned long long* sees;
    int4* where;  // [n_rows]: a row's first place among the sums, its sequence's nodes, runs, number
    int2* spans;  // [n_seqs]: first row and nodes of the launch's sequences, as they count
    int* taken;   // [2]: where the last row so far ends, behind launches of even and of odd number
    float* part;  // [run, node][H][hd]: sums
    float2* ml;   // [run, node][H]: maxima and sums of exponentials
    int places;   // of a run and node
    int* status;
};

// A sequence's nodes, cached tokens and runs.
struct TreeSeq {
    int row0, n, old, L, run, runs, tiles;
};
template <int HD>
__device__ __forceinline__ TreeSeq tree_seq(const TreeArgs& a, int row0, int n, int old) {
    TreeSeq x{row0, n, old, 0, tree::KT, 1, 0};
    const int T = tile_tokens(a.group);
    x.tiles = (n + T - 1) / T;
    if (n > 0 && old >= 0) {  // else no token is seen
        x.L = old + n;
        x.run = tree::run_tokens(x.L, min(n, T) * a.group, a.Hkv * x.tiles, TreeCfg<HD>::SLOTS, HD == 256);
        x.runs = (x.L + x.run - 1) / x.run;
    }
    return x;
}

// Rows [i0, ...) of a sequence for one key head, over its tokens [at, end).
struct TreeUnit {
    int s, i0, kvh, run, at, end;
    bool half;  // up to 64 rows: Q takes half of its place, and the next unit's the other half
    TreeSeq q;
    __device__ __forceinline__ int tiles() const { return (end - at + tree::KT - 1) / tree::KT; }
};

// A sequence's nodes and cached tokens as they count: false is reported; old < 0: none is seen.
__device__ __forceinline__ bool tree_lengths(const TreeArgs& a, int s, int& row0, int& n, int& old) {
    old = -1;
    if (!tree_rows(a.cu_nodes, a.s0 + s, a.n_rows, kMaxNodes, row0, n)) {
        n = 0;
        return false;
    }
    if (n == 0) return true;
    const int c = a.n_cached[a.s0 + s];
    if (c < 0 || (long long)c + n > (long long)a.pages.max_pages * a.pages.room) return false;
    old = c;
    return true;
}

// 32 bytes, a sector, from registers.
__device__ __forceinline__ void store8(float* p, const uint32_t (&w)[32], int i) {
    asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p), "r"(w[i]),
                 "r"(w[i + 1]), "r"(w[i + 2]), "r"(w[i + 3]), "r"(w[i + 4]), "r"(w[i + 5]), "r"(w[i + 6]),
                 "r"(w[i + 7])
                 : "memory");
}

template <int HD>
__global__ void __launch_bounds__(tree::THREADS, TreeCfg<HD>::CTAS)
    k_tree_attn(const __grid_constant__ CUtensorMap tq, const __grid_constant__ CUtensorMap tq64,
                const __grid_constant__ CUtensorMap tk, const __grid_constant__ CUtensorMap tv,
                const __grid_constant__ TreeArgs a) {
    using C = TreeCfg<HD>;
    using namespace tree;
    constexpr int NCH = C::NCH, RING = C::RING;
    extern __shared__ uint8_t smem_raw[];
    uint8_t* sm = reinterpret_cast<uint8_t*>(
        (reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
    int* first = reinterpret_cast<int*>(sm + C::OFF_SEQ);  // [n_seqs + 1]: first unit of each
    int *rows0 = first + BATCH + 1, *nodes = rows0 + BATCH, *olds = nodes + BATCH, *base = olds + BATCH;
    int* run_of = base + BATCH;
    uint16_t *runs_of = reinterpret_cast<uint16_t*>(run_of + BATCH), *tiles_of = runs_of + BATCH;
    uint64_t* bar = reinterpret_cast<uint64_t*>(sm + C::OFF_BAR);
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(bar + N_BARS);
    volatile int* fail_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
    const int warp = warp_uniform(threadIdx.x >> 5), lane = threadIdx.x & 31;
    const int T = tile_tokens(a.group);

    if (threadIdx.x == 0) {
        for (int i = 0; i < N_BARS; ++i)
            mbar_init(&bar[i], (i >= P_FULL && i < PV_DONE) || i == O_FREE ? 128 : 1);
        *fail_flag = 0;
        fence_barrier_init();
        fence_proxy_async();
    }
    pdl_entry();  // TMEM is taken once the grid ahead has given its own back
    if (warp == 1) {
        tmem_alloc(tmem_slot, C::COLS);
        tmem_relinquish();
    }
    for (int s = threadIdx.x; s < a.n_seqs; s += THREADS) {
        int row0, n, old;
        if (!tree_lengths(a, s, row0, n, old) && blockIdx.x == 0) report(a.status, JNX_ERR_DEVICE_BOUNDS);
        rows0[s] = row0, nodes[s] = n, olds[s] = old;
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    if (warp == 0) {  // units and sums ahead of each sequence
        int units = 0, sums = 0;
        // Rows are one sequence's: one that starts ahead of an earlier one's end is left out, or its
        // sums would be more than the workspace has places for.
        const int launch = a.s0 / BATCH;
        int taken = launch > 0 ? a.taken[(launch - 1) & 1] : 0;
        for (int b = 0; b < a.n_seqs; b += 32) {
            const int s = b + lane;
            int u = 0, v = 0;
            int end = s < a.n_seqs && nodes[s] > 0 ? rows0[s] + nodes[s] : 0;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const int y = __shfl_up_sync(0xffffffffu, end, o);
                if (lane >= o) end = max(end, y);
            }
            const int ahead = __shfl_up_sync(0xffffffffu, end, 1);
            if (s < a.n_seqs && nodes[s] > 0 && rows0[s] < max(taken, lane ? ahead : 0)) {
                nodes[s] = 0, olds[s] = -1;
                if (blockIdx.x == 0) report(a.status, JNX_ERR_DEVICE_BOUNDS);
            }
            taken = max(taken, __shfl_sync(0xffffffffu, end, 31));
            TreeSeq x{};
            if (s < a.n_seqs) {
                x = tree_seq<HD>(a, rows0[s], nodes[s], olds[s]);
                u = x.runs * a.Hkv * x.tiles;
                v = x.runs > 1 ? x.runs * x.n : 0;
            }
            int ru = u, rv = v;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const int y = __shfl_up_sync(0xffffffffu, ru, o), z = __shfl_up_sync(0xffffffffu, rv, o);
                if (lane >= o) ru += y, rv += z;
            }
            if (s < a.n_seqs) {
                first[s] = units + ru - u;
                base[s] = sums + rv - v;
                run_of[s] = x.run, runs_of[s] = (uint16_t)x.runs, tiles_of[s] = (uint16_t)x.tiles;
            }
            units += __shfl_sync(0xffffffffu, ru, 31);
            sums += __shfl_sync(0xffffffffu, rv, 31);
        }
        if (lane == 0) {
            first[a.n_seqs] = units;
            if (blockIdx.x == 0) a.taken[launch & 1] = taken;
        }
    }
    __syncthreads();
    const uint32_t tbase = warp_uniform(*tmem_slot);
    const int n_units = warp_uniform(first[a.n_seqs]);
    // what the join needs of each row
    for (int s = blockIdx.x; s < a.n_seqs; s += gridDim.x) {
        const int i = threadIdx.x;
        if (i == 0) a.spans[s] = make_int2(rows0[s], nodes[s]);
        if (i >= nodes[s]) continue;
        a.where[rows0[s] + i] = make_int4(base[s] + i, nodes[s], runs_of[s], a.s0 + s);
    }

    auto open = [&](int u) {
        TreeUnit x{};
        if (u >= n_units) return x;
        int lo = -1;  // the last s with first[s] <= u, by all lanes
        for (int b = 0; b < a.n_seqs; b += 32) {
            const uint32_t ahead = __ballot_sync(0xffffffffu, b + lane < a.n_seqs && first[b + lane] <= u);
            if (ahead) lo = b + 31 - __clz(ahead);
            if (ahead != 0xffffffffu) break;
        }
        x.s = lo;
        const int old = olds[lo], nn = nodes[lo];
        x.q = TreeSeq{rows0[lo], nn, old, old < 0 ? 0 : old + nn, run_of[lo], runs_of[lo], tiles_of[lo]};
        int rest = u - first[lo];  // a run's tiles lie together, then its heads
        if (x.q.tiles > 1) {
            x.i0 = rest % x.q.tiles * T;
            rest /= x.q.tiles;
        }
        x.half = min(x.q.n - x.i0, T) * a.group <= 64;
        x.kvh = rest % a.Hkv;
        x.run = rest / a.Hkv;
        x.at = x.run * x.q.run;
        x.end = min(x.q.L, x.at + x.q.run);
        return x;
    };

    if (warp == 0) {
        // ---------------- TMA producer ----------------
        if (elect_one()) {
            tma_prefetch_desc(&tq);
            tma_prefetch_desc(&tq64);
            tma_prefetch_desc(&tk);
            tma_prefetch_desc(&tv);
        }
        bool ok = true;
        uint32_t nk = 0, nv = 0;  // K and V tiles loaded
        uint32_t qn = 0, qodd = 0, qany = 0;  // the next half; whether odd, or any, Q tiles went to each
        const int qrow = a.group * HD * 2, boxes = KT / a.box;
        // pages of the boxes [32 c, 32 c + 32) of a unit, one a lane
        auto look = [&](const TreeUnit& x, int c) {
            int page = a.no_page, row = 0;
            const long long token = x.at + (long long)(c * 32 + lane) * a.box;
            if (token < x.end && !a.pages.find(a.s0 + x.s, (int)token, page, row)) {
                page = a.no_page;
                report(a.status, JNX_ERR_DEVICE_BOUNDS);
            }
            __syncwarp();
            return page;
        };
        // tile t of a unit's tokens [at, end), whose first box's page is in lane `first` of pages
        struct Tile {
            int kvh, token, end, pages, first;
        };
        auto load = [&](bool v, const Tile& x) -> bool {
            uint32_t& n = v ? nv : nk;
            const int s = n % RING;
            uint64_t* full = &bar[(v ? V_FULL : K_FULL) + s];
            if (!mbar_wait_warp(&bar[(v ? V_EMPTY : K_EMPTY) + s], ((n / RING) & 1) ^ 1)) return false;
            ++n;
            uint8_t* dst = sm + (v ? C::OFF_V : C::OFF_K) + s * C::TILE;
            const CUtensorMap* map = v ? &tv : &tk;
            const int nb = min(boxes, (x.end - x.token + a.box - 1) / a.box);
            if (elect_one()) mbar_arrive_expect_tx(full, nb * a.box * HD * 2);
            __syncwarp();
            int r = x.token % a.pages.room;  // a box lies in one page
            for (int i = 0; i < nb; ++i) {
                const int page = __shfl_sync(0xffffffffu, x.pages, x.first + i);
                if (elect_one()) {
#pragma unroll
                    for (int c = 0; c < NCH; ++c)
                        tma_load_4d(dst + c * KT * 128 + i * a.box * 128, map, c * 64, x.kvh, r, page, full);
                }
                __syncwarp();
                r += a.box;
                if (r >= a.pages.room) r -= a.pages.room;
            }
            return true;
        };
        auto q_free = [&](int h) {
            return !(qany >> h & 1) || mbar_wait_warp(&bar[Q_EMPTY + h], (qodd >> h & 1) ^ 1);
        };
        // V one tile behind K, as S is taken ahead of P V: so K is asked for two tiles ahead
        Tile late{0, 0, 0, 0, -1};
        TreeUnit x = open(blockIdx.x);
        int pages = look(x, 0);
        for (int u = blockIdx.x; ok && u < n_units && !__any_sync(0xffffffffu, *fail_flag); u += gridDim.x) {
            const int n = warp_uniform(x.tiles()), at = warp_uniform(x.at), end = warp_uniform(x.end);
            const int kvh = warp_uniform(x.kvh);
            const TreeUnit next = open(u + gridDim.x);
            const int next_pages = look(next, 0);
            int more = look(x, 1);
            if (n > 0) {
                const bool half = warp_uniform(x.half);
                const int h = half ? qn : 0;
                if (!(ok = q_free(h) && (half || q_free(1)))) break;
                if (elect_one()) {
                    mbar_arrive_expect_tx(&bar[Q_FULL + h], (half ? 64 / a.group : T) * qrow);
                    if (!half) mbar_arrive(&bar[Q_FULL + 1]);
#pragma unroll
                    for (int c = 0; c < NCH; ++c)
                        tma_load_3d(sm + h * (C::QB / 2) + c * (half ? 64 : 128) * 128, half ? &tq64 : &tq,
                                    c * 64, kvh * a.group, x.q.row0 + x.i0, &bar[Q_FULL + h]);
                }
                __syncwarp();
                const uint32_t both = half ? 1u << h : 3u;
                qodd ^= both;
                qany |= both;
                qn = half ? qn ^ 1 : 0;
            }
            for (int t = 0; t < n && ok; ++t) {
                const int b0 = t * boxes;  // first box of the tile
                if (t > 0 && b0 % 32 == 0) {
                    pages = more;
                    more = look(x, b0 / 32 + 1);
                }
                const Tile tile{kvh, at + t * KT, end, pages, b0 & 31};
                ok = load(false, tile) && (late.first < 0 || load(true, late));
                late = tile;
            }
            x = next;
            pages = next_pages;
        }
        ok = ok && (late.first < 0 || load(true, late));
        if (!ok) *fail_flag = 1;
        // every copy has landed before the CTA may exit (at once in a normal run)
        for (int h = 0; h < 2; ++h)
            if (qany >> h & 1) mbar_wait_warp(&bar[Q_FULL + h], (qodd >> h & 1) ^ 1, 100000000LL);
        for (uint32_t i = nk > RING ? nk - RING : 0; i < nk; ++i)
            mbar_wait_warp(&bar[K_FULL + i % RING], (i / RING) & 1, 100000000LL);
        for (uint32_t i = nv > RING ? nv - RING : 0; i < nv; ++i)
            mbar_wait_warp(&bar[V_FULL + i % RING], (i / RING) & 1, 100000000LL);
    } else if (warp == 1) {
        // ---------------- MMA issuer ----------------
        constexpr uint32_t IDESC_S = idesc_bf16_f32(128, KT);
        constexpr uint32_t IDESC_PV = idesc_bf16_f32(128, HD) | (1u << 16);  // B MN-major
        bool ok = true, issued = false;
        uint32_t ks = 0, kv = 0, nu = 0;  // K tiles and V tiles taken, units with tokens
        const uint32_t q_lo = sw128_desc_lo(smem_u32(sm)), k_lo = sw128_desc_lo(smem_u32(sm + C::OFF_K));
        const uint32_t v_lo = sw128_desc_mn_lo(smem_u32(sm + C::OFF_V), KT * 128);
        auto commit = [&](uint64_t* b) {
            if (elect_one()) tc_commit(b);
            __syncwarp();
        };
        // score tile ks goes to buffer ks % 2, whose P the product two tiles back has read
        uint32_t qn = 0, qodd = 0;
        // the 64 rows behind a half are whatever lies there, landed or not: rows of the tile that
        // nobody reads
        auto next_s = [&](int h, bool half, bool last) -> bool {
            const int s = ks % RING;
            if (!mbar_wait_warp(&bar[K_FULL + s], (ks / RING) & 1)) return false;
            tc_fence_after();
            const uint32_t lo = k_lo + s * (C::TILE >> 4), d = tbase + (ks & 1) * KT;
            const uint32_t qa = q_lo + h * (C::QB / 2 >> 4), chunk = (half ? 64 : 128) * 128 >> 4;
            if (elect_one()) {
#pragma unroll
                for (int c = 0; c < NCH; ++c)
#pragma unroll
                    for (int k = 0; k < 4; ++k)
                        tc_mma_f16(d, desc_of(qa + c * chunk + k * 2, kSw128DescHi),
                                   desc_of(lo + c * (KT * 128 >> 4) + k * 2, kSw128DescHi), IDESC_S,
                                   (c | k) != 0);
                tc_commit(&bar[S_FULL + (ks & 1)]);
                tc_commit(&bar[K_EMPTY + s]);
                if (last) {
                    tc_commit(&bar[Q_EMPTY + h]);
                    if (!half) tc_commit(&bar[Q_EMPTY + 1]);
                }
            }
            __syncwarp();
            issued = true;
            ++ks;
            return true;
        };
        TreeUnit next = open(blockIdx.x);
        for (int u = blockIdx.x; ok && u < n_units && !__any_sync(0xffffffffu, *fail_flag); u += gridDim.x) {
            const TreeUnit x = next;
            next = open(u + gridDim.x);
            const int n = warp_uniform(x.tiles());
            if (n == 0) continue;
            const bool half = warp_uniform(x.half);
            const int h = half ? qn : 0;
            ok = mbar_wait_warp(&bar[Q_FULL + h], qodd >> h & 1) &&
                 (half || mbar_wait_warp(&bar[Q_FULL + 1], qodd >> 1 & 1));
            if (!ok) break;
            qodd ^= half ? 1u << h : 3u;
            qn = half ? qn ^ 1 : 0;
            tc_fence_after();
            ok = next_s(h, half, n == 1) && (n < 2 || next_s(h, half, n == 2));
            for (int t = 0; t < n && ok; ++t, ++kv) {
                const int s = kv % RING;
                const uint32_t b = kv & 1, p = tbase + b * KT;
                if (!(ok = mbar_wait_warp(&bar[V_FULL + s], (kv / RING) & 1))) break;
                const int valid = warp_uniform(x.end - x.at) - t * KT;
                if (valid < KT) {
                    // rows behind the run's last token may hold NaN: 0 * NaN would reach O
                    uint8_t* tile = sm + C::OFF_V + s * C::TILE;
                    for (int i = lane; i < (KT - valid) * (HD / 8); i += 32) {
                        const int r = valid + i / (HD / 8), w = i % (HD / 8);
                        *reinterpret_cast<uint4*>(tile + (w >> 3) * KT * 128 + r * 128 + (w & 7) * 16) =
                            make_uint4(0, 0, 0, 0);
                    }
                    fence_proxy_async();
                    __syncwarp();
                }
                if (!(ok = mbar_wait_warp(&bar[P_FULL + b], (kv >> 1) & 1))) break;
                // the unit's first product overwrites O: the last epilogue has read it
                if (t == 0 && nu > 0 && !(ok = mbar_wait_warp(&bar[O_FREE], (nu - 1) & 1))) break;
                tc_fence_after();
                const uint32_t lo = v_lo + s * (C::TILE >> 4);
                if (elect_one()) {
#pragma unroll
                    for (int k = 0; k < KT / 16; ++k)
                        tc_mma_f16_ts(tbase + C::O_COL, p + k * 8, desc_of(lo + k * 128, kSw128DescHi),
                                      IDESC_PV, t > 0 || k > 0);
                    tc_commit(&bar[PV_DONE + b]);
                    tc_commit(&bar[V_EMPTY + s]);
                    if (t + 1 == n) tc_commit(&bar[O_FULL]);
                }
                __syncwarp();
                if (t + 2 < n) ok = next_s(h, half, t + 3 == n);
            }
            ++nu;
        }
        if (!ok) *fail_flag = 1;
        if (issued) {
            commit(&bar[DRAIN]);
            mbar_wait_warp(&bar[DRAIN], 0, 100000000LL);
        }
    } else {
        // ---------------- softmax + epilogue ----------------
        const int row = (warp & 3) * 32 + lane;
        const uint32_t lane_base = (uint32_t)((warp & 3) * 32) << 16;
        const uint32_t tO = tbase + lane_base + C::O_COL;
        uint32_t g = 0, nu = 0;  // score tiles, units with tokens
        bool ok = true;
        const int tok = row / a.group, hg = row % a.group;
        // the bits of what this row sees, asked for ahead of the epilogue; a row that is none of the
        // tile's has no say in the masks
        auto sight = [&](const TreeUnit& x) {
            const int i = x.i0 + tok;
            return tok < T && i < x.q.n ? a.sees[x.q.row0 + i] : ~0ull;
        };
        TreeUnit next = open(blockIdx.x);
        unsigned long long next_see = sight(next);
        for (int u = blockIdx.x; ok && u < n_units && !__any_sync(0xffffffffu, *fail_flag); u += gridDim.x) {
            const TreeUnit x = next;
            const int n = warp_uniform(x.tiles()), i = x.i0 + tok;
            const bool live = tok < T && i < x.q.n;
            const unsigned long long see = next_see & (x.q.n >= 64 ? ~0ull : (1ull << x.q.n) - 1);
            const bool work = __any_sync(0xffffffffu, live);  // else nobody reads the warp's rows
            float m = -INFINITY, l = 0.f;
            for (int t = 0; t < n; ++t, ++g) {
                const uint32_t b = g & 1, tS = tbase + lane_base + b * KT;
                if (!(ok = __all_sync(0xffffffffu, mbar_wait(&bar[S_FULL + b], (g >> 1) & 1)))) break;
                if (!work) {
                    mbar_arrive(&bar[P_FULL + b]);
                    continue;
                }
                tc_fence_after();
                uint32_t v[2][32];
                tmem_ld32(tS, v[0]);
                tmem_ld32(tS + 32, v[1]);
                tmem_ld_wait_regs(v[0]);
                tmem_ld_wait_regs(v[1]);
                // tokens of the tile ahead of the nodes, then those of the nodes that are seen
                const int ahead = x.q.old - (x.at + t * KT);
                if (ahead < KT || x.end - (x.at + t * KT) < KT) {
                    unsigned long long word = ahead >= 64 ? ~0ull
                                              : ahead > 0 ? ((1ull << ahead) - 1) | (see << ahead)
                                                          : see >> -ahead;
                    const int valid = x.end - (x.at + t * KT);
                    if (valid < KT) word &= (1ull << valid) - 1;
#pragma unroll
                    for (int c = 0; c < 2; ++c)
#pragma unroll
                        for (int e = 0; e < 32; ++e)
                            if (!(word >> (c * 32 + e) & 1)) v[c][e] = 0xff800000u;  // -inf
                }
                float mx[2];
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                    mx[c] = __uint_as_float(v[c][0]);
#pragma unroll
                    for (int e = 1; e < 31; e += 2)
                        mx[c] = fmax3(mx[c], __uint_as_float(v[c][e]), __uint_as_float(v[c][e + 1]));
                    mx[c] = fmaxf(mx[c], __uint_as_float(v[c][31]));
                }
                const float top = fmaxf(mx[0], mx[1]) * a.scale_log2;
                float alpha = 1.f;
                if (t == 0) {
                    m = top;
                } else if (top > m + kLazy) {
                    alpha = ex2_approx(m - top);
                    m = top;
                }
                if (t > 0 && __any_sync(0xffffffffu, alpha < 1.f)) {
                    // every earlier P V of the unit is done
                    if (!(ok = __all_sync(0xffffffffu,
                                          mbar_wait(&bar[PV_DONE + (b ^ 1)], ((g - 1) >> 1) & 1))))
                        break;
                    tc_fence_after();
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
                // a row that has seen no token yet subtracts nothing
                const float sub = m == -INFINITY ? 0.f : m;
                const uint64_t sc2 = f2_pack(a.scale_log2, a.scale_log2), nm2 = f2_pack(-sub, -sub);
                uint64_t rs[2] = {f2_pack(0.f, 0.f), f2_pack(0.f, 0.f)};
                uint32_t pk[32];
#pragma unroll
                for (int c = 0; c < 2; ++c)
#pragma unroll
                    for (int e = 0; e < 32; e += 2) {
                        float x0, x1;
                        f2_unpack(f2_fma(f2_pack(__uint_as_float(v[c][e]), __uint_as_float(v[c][e + 1])),
                                         sc2, nm2),
                                  x0, x1);
                        const float p0 = ex2_approx(x0), p1 = ex2_approx(x1);
                        rs[(e >> 1) & 1] = f2_add(rs[(e >> 1) & 1], f2_pack(p0, p1));
                        pk[c * 16 + e / 2] = cvt_bf2(p0, p1);
                    }
                tmem_st32(tS, pk);
                tmem_st_wait();
                tc_fence_before();
                mbar_arrive(&bar[P_FULL + b]);
                float r0, r1, r2, r3;
                f2_unpack(rs[0], r0, r1);
                f2_unpack(rs[1], r2, r3);
                l = l * alpha + ((r0 + r1) + (r2 + r3));
            }
            if (!ok) break;
            next = open(u + gridDim.x);
            next_see = sight(next);
            if (n > 0) {
                if (!(ok = __all_sync(0xffffffffu, mbar_wait(&bar[O_FULL], nu & 1)))) break;
                tc_fence_after();
                ++nu;
            }
            const int h = x.kvh * a.group + hg;
            const bool joined = x.q.runs > 1;
            const long long slot =
                live ? ((long long)base[x.s] + (long long)x.run * x.q.n + i) * a.H + h : -1;
            if (joined && live) a.ml[slot] = make_float2(m, l);
            const float inv = joined ? 1.f : l > 0.f ? 1.f / l : 0.f;
            const long long o = !live ? -1
                                : joined ? slot * HD
                                         : (x.q.row0 + i) * a.o_row + h * a.o_head;
            // straight from the registers, a lane its row: 32 columns a time, the next ones' under way
            // (through staging, so that lanes write side by side: 1,000 cycles for every 32 columns)
            uint32_t w[2][32];
            __syncwarp();
            if (n > 0) tmem_ld32(tO, w[0]);
#pragma unroll
            for (int c = 0; c < HD / 32; ++c) {
                uint32_t(&y)[32] = w[c & 1];
                if (n > 0) {
                    tmem_ld_wait_regs(y);
                    if (c + 1 < HD / 32) {
                        tmem_ld32(tO + (c + 1) * 32, w[(c + 1) & 1]);
                    } else {
                        tc_fence_before();
                        mbar_arrive(&bar[O_FREE]);
                    }
                }
                // a row that saw nothing: O holds products of zeros
                const float f = n > 0 && l > 0.f ? inv : 0.f;
#pragma unroll
                for (int e = 0; e < 32; ++e) y[e] = f == 0.f ? 0u : __float_as_uint(__uint_as_float(y[e]) * f);
                if (live && joined) {
#pragma unroll
                    for (int j = 0; j < 4; ++j) store8(a.part + o + c * 32 + j * 8, y, j * 8);
                } else if (live) {
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        uint32_t z[4];
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            z[e] = cvt_bf2(__uint_as_float(y[8 * j + 2 * e]), __uint_as_float(y[8 * j + 2 * e + 1]));
                        *reinterpret_cast<uint4*>(a.out + o + c * 32 + j * 8) = make_uint4(z[0], z[1], z[2], z[3]);
                    }
                }
                __syncwarp();  // the next columns are taken by all lanes
            }
        }
        if (!ok) *fail_flag = 1;
    }
    __syncwarp();
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    if (*fail_flag && threadIdx.x == 0) report(a.status, JNX_ERR_TIMEOUT);
    if (warp == 1) tmem_dealloc(tbase, C::COLS);
}

// A sequence's runs joined: a warp a node and head and quarter of the runs, a fourth of them in
// turn, then the quarters in their order.  Four warps to a CTA, of one node and head where the
// card has room for as many, else of four (WIDE: no).
template <int HD, bool WIDE>
__global__ void __launch_bounds__(128) k_tree_join(const __grid_constant__ TreeArgs a) {
    using namespace tree;
    constexpr int E = HD / 32, R = 8;  // runs of a warp under way
    __shared__ float sums[WIDE ? 4 : 1][HD];
    pdl_entry();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int w = WIDE ? blockIdx.x : blockIdx.x * 4 + warp;
    const int row = w / a.H, h = w % a.H;
    if (row >= a.n_rows) return;
    // a row of no sequence of the launch has no record but what lay there: nothing is read beyond
    // the workspace for it, and nothing written
    const int4 x = a.where[row];
    const int runs = x.z;
    if (runs <= 1 || runs > MAX_RUNS || x.x < 0 || x.y < 1 || x.y > kMaxNodes ||
        (long long)x.x + (runs - 1) * x.y >= a.places || x.w < a.s0 || x.w >= a.s0 + a.n_seqs)
        return;
    const long long at = (long long)x.x * a.H + h, step = (long long)x.y * a.H;
    float v[R][E], m[2], l[2], top = -INFINITY, sum = 0.f;
    // runs first, first + by, ...: a warp of four has every fourth
    constexpr int BY = WIDE ? 4 : 1;
    const int mine = WIDE ? warp : 0;
    auto load = [&](int first) {
#pragma unroll
        for (int k = 0; k < R; ++k) {
            const int r = first + BY * k;
            if (r >= runs) continue;
            const float* src = a.part + (at + r * step) * HD + lane * E;
#pragma unroll
            for (int e = 0; e < E; e += 2) {
                const float2 y = *reinterpret_cast<const float2*>(src + e);
                v[k][e] = y.x, v[k][e + 1] = y.y;
            }
        }
    };
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        const int r = k * 32 + lane;
        const float2 y = r < runs ? a.ml[at + r * step] : make_float2(-INFINITY, 0.f);
        m[k] = y.x, l[k] = y.y;
        top = fmaxf(top, m[k]);
    }
    load(mine);
    const int2 span = a.spans[x.w - a.s0];
#pragma unroll
    for (int o = 16; o; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
    if (top == -INFINITY) top = 0.f;  // no run's token was seen
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        m[k] = ex2_approx(m[k] - top);
        sum += l[k] * m[k];
    }
#pragma unroll
    for (int o = 16; o; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    const float inv = sum > 0.f ? 1.f / sum : 0.f;
    float acc[WIDE ? 1 : 4][E] = {}, all[E];  // the quarters' sums
    for (int first = mine; first < runs; first += BY * R) {
        if (first > mine) load(first);
#pragma unroll
        for (int k = 0; k < R; ++k) {
            const int r = first + BY * k;
            if (r >= runs) continue;
            const float f = __shfl_sync(0xffffffffu, r >> 5 ? m[1] : m[0], r & 31);
#pragma unroll
            for (int e = 0; e < E; ++e) {
                float& to = acc[WIDE ? 0 : k & 3][e];  // (R is a multiple of four)
                to = fmaf(f, v[k][e], to);
            }
        }
    }
    static_assert(MAX_RUNS == 64, "factors of two registers");
    if constexpr (WIDE) {
#pragma unroll
        for (int e = 0; e < E; ++e) sums[warp][e * 32 + lane] = acc[0][e];
        __syncthreads();
        if (warp > 0) return;
#pragma unroll
        for (int e = 0; e < E; ++e)
            all[e] = (sums[0][e * 32 + lane] + sums[1][e * 32 + lane]) + (sums[2][e * 32 + lane] + sums[3][e * 32 + lane]);
    } else {
#pragma unroll
        for (int e = 0; e < E; ++e) all[e] = (acc[0][e] + acc[1][e]) + (acc[2][e] + acc[3][e]);
    }
    if (row < span.x || row >= span.x + span.y) return;
    uint16_t* o = a.out + row * a.o_row + h * a.o_head + lane * E;
#pragma unroll
    for (int e = 0; e < E; e += 2) *reinterpret_cast<uint32_t*>(o + e) = cvt_bf2(all[e] * inv, all[e + 1] * inv);
}

// The workspace: the rows' records, a launch's sequences, then (at 256 bytes) the sums.
static size_t tree_sums_at(int n_rows) {
    return ((size_t)n_rows * sizeof(int4) + tree::BATCH * sizeof(int2) + 2 * sizeof(int) + 255) & ~(size_t)255;
}

template <int HD>
static jnx_status launch_tree(const jnx_kv_cache& c, const jnx_pages& p, const jnx_head_rows& q, TreeArgs a,
                              long long runs, cudaStream_t s) {
    using namespace tree;
    using C = TreeCfg<HD>;
    static std::atomic<uint64_t> attr{0};
    if (set_smem_limit(reinterpret_cast<const void*>(k_tree_attn<HD>), C::SMEM, attr) != cudaSuccess)
        return fail(JNX_ERR_CUDA, "tree attention: smem attribute");
    CUtensorMap tq, tq64, tk, tv;
    if (!make_tmap_heads(&tq, q, a.n_rows, a.H, HD, a.group, tile_tokens(a.group)) ||
        !make_tmap_heads(&tq64, q, a.n_rows, a.H, HD, a.group, 64 / a.group) ||
        !make_tmap_cache(&tk, c.k, c, a.Hkv, HD, a.box) || !make_tmap_cache(&tv, c.v, c, a.Hkv, HD, a.box))
        return fail(JNX_ERR_CUDA, "tree attention: tensor map encode failed");
    const int most = std::min(kMaxNodes, a.n_rows), T = tile_tokens(a.group);
    for (int s0 = 0; s0 < p.n_seqs; s0 += BATCH) {
        a.s0 = s0;
        a.n_seqs = std::min(BATCH, p.n_seqs - s0);
        const long long units = a.n_seqs * runs * a.Hkv * ((most + T - 1) / T);
        const int grid = (int)std::min<long long>(units, (long long)num_sms() * C::CTAS);
        pdl(k_tree_attn<HD>, grid, THREADS, C::SMEM, s)(tq, tq64, tk, tv, a);
        const int heads = a.n_rows * a.H;
        if (runs > 1 && heads <= num_sms() * 8) pdl(k_tree_join<HD, true>, heads, 128, 0, s)(a);
        else if (runs > 1) pdl(k_tree_join<HD, false>, (heads + 3) / 4, 128, 0, s)(a);
    }
    return launched("tree attention");
}

}  // namespace jnx

using namespace jnx;

extern "C" size_t jnx_op_tree_attention_workspace_bytes(int32_t n_seqs, int32_t n_rows,
                                                        int32_t n_heads, int32_t head_dim,
                                                        int64_t max_tokens) {
    if (n_seqs < 0 || n_rows < 0 || n_heads <= 0 || head_dim <= 0 || max_tokens < 0) return 0;
    return tree_sums_at(n_rows) + 256 +
           (size_t)n_rows * tree::most_runs(max_tokens, head_dim == 256) * n_heads * (head_dim + 2) * sizeof(float);
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
    if (jnx_status st = heads_ok(n_heads, n_kv_heads, head_dim, what)) return st;
    if (n_rows < 0 || !pages_ok(pages)) return fail(JNX_ERR_INVALID_ARG, "%s: bad sizes or pages", what);
    if (n_rows == 0 || pages->n_seqs == 0) return JNX_OK;
    if (!cache_ok(cache) || !rows_ok(q) || !rows_ok(out) || !cu_nodes || !n_cached || !sees)
        return fail(JNX_ERR_INVALID_ARG, "%s: null or misaligned argument", what);
    if (pages->max_pages > 1 && cache->room % 16)
        return fail(JNX_ERR_UNSUPPORTED, "%s: pages of %d tokens, no multiple of 16", what, cache->room);
    const long long tokens = (long long)pages->max_pages * cache->room, runs = tree::most_runs(tokens, head_dim == 256);
    if (tokens > 0x7fffff00 || (long long)n_rows * n_heads > 0x7fffff00 ||
        (long long)n_rows * runs > 0x7fffff00 ||
        tree::BATCH * runs * n_kv_heads * kMaxNodes > 0x7fffff00)
        return fail(JNX_ERR_UNSUPPORTED, "%s: sizes", what);
    if (!workspace || !aligned16(workspace) ||
        ws_bytes < jnx_op_tree_attention_workspace_bytes(pages->n_seqs, n_rows, n_heads, head_dim, tokens))
        return fail(JNX_ERR_WORKSPACE, "%s: workspace too small or misaligned", what);
    // boxes of as many tokens as a tile and a page share
    int box = tree::KT;
    while (pages->max_pages > 1 && cache->room % box) box /= 2;
    // the maps want extents: an empty cache's have a page that no sequence's tokens are looked for in
    jnx_kv_cache c = *cache;
    c.n_slots = std::max(c.n_slots, 1);
    c.room = std::max(c.room, 1);
    TreeArgs a{Pages(*pages, *cache), c.n_slots, 0, 0, n_heads, n_kv_heads, n_heads / n_kv_heads, n_rows, box,
               (float)(1.4426950408889634 / sqrt((double)head_dim)), out->ptr, out->row_stride,
               out->head_stride, cu_nodes, n_cached, reinterpret_cast<const unsigned long long*>(sees),
               static_cast<int4*>(workspace), nullptr, nullptr, nullptr, nullptr, (int)(n_rows * runs), status};
    a.spans = reinterpret_cast<int2*>(a.where + n_rows);
    a.taken = reinterpret_cast<int*>(a.spans + tree::BATCH);
    const uintptr_t sums = reinterpret_cast<uintptr_t>(workspace) + tree_sums_at(n_rows) + 255;
    a.part = reinterpret_cast<float*>(sums & ~(uintptr_t)255);
    a.ml = reinterpret_cast<float2*>(a.part + (size_t)n_rows * runs * n_heads * head_dim);
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    TraceScope ts(JNX_K_TREE_ATTN, 0.0, s);
    if (head_dim == 64) return launch_tree<64>(c, *pages, *q, a, runs, s);
    if (head_dim == 128) return launch_tree<128>(c, *pages, *q, a, runs, s);
    return launch_tree<256>(c, *pages, *q, a, runs, s);
}
