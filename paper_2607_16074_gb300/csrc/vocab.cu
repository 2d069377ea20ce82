// Next-token losses over the vocabulary and their gradients: logits x = h w^T,
// loss = logsumexp(x) - x_target, G = row_weight (softmax(x) - onehot),
// dh = G w, dw = G^T h.  And losses against a teacher's top logits: T over a row's entries in
// place of the one-hot row, P = softmax(x / tau), G = row_weight / tau (P - T).
//
// The rows that count (target >= 0) are packed first: most rows of an observation are
// image rows without a next token, and an ignored row's h may hold anything, which must
// not meet G^T.  Then, for each piece of packed rows:
//   logits   a 256 x 256 tile on a CTA pair, d deep; the epilogue leaves of each row's
//            128 columns the maximum m and the sum s of e^(x - m) without the target's, the
//            target's logit, and, for gradients, e^(x - m) in bf16 (no logit is stored)
//   rows     each row's m and s into its loss, and the row of probabilities scaled to G in
//            place.  With o the others' sum and e the target's term, both against the row's
//            maximum, loss = log1p(o / e) and the target's entry is -row_weight o / (o + e):
//            where the target's probability is near one, o keeps its digits, which a sum
//            with e in it, or a log-sum-exp at the size of the logits, would round away
//            (1e-6 of other mass at a logit of 20 or 100 gave a loss of 0)
//   dh       G w, the vocabulary deep: w is the MN-major B operand as it lies
//   dw       G^T h, the rows deep: both operands MN-major as they lie
// which is three products of 2 rows vocab d operations for the minimum's three; forming
// the logits again instead of keeping the piece's probabilities would be a fourth.
//
// Bound by the tensor cores and the power cap: 8,191 rows of 4,096 on 32,000 columns with
// gradients take 3,590 us, 1,795 TFLOP/s over all (floor 3,400), 3,650 to 3,760 in longer runs:
// the products 1,040, 1,175 and 1,070 each by itself, the rows 150.  333 rows of 2,048 without
// gradients: 48 us, of which the logits 46 by themselves, two row blocks of 256 for 1.3 and four
// rounds of tiles for 3.3.
// Against a teacher's 32 entries a row, 8,191 rows of 2,048: 1,980 us (floor 1,671), the products
// 544, 569 and 534, the rows 187; 333 rows of 1,024 without gradients 31, the logits 20.5.
//
// G is bf16, as its products' other operands are, and rounded twice: when it is formed, whose
// row's maximum is not known yet (in 32 bits it would be twice the bytes of the rows' kernel), and
// when it is scaled.
#include <algorithm>

#include "jnx_dev.cuh"
#include "jnx_kernels.h"
#include "jnx_text.h"
#include "jnx_trace.h"

namespace jnx {

namespace vocab {
constexpr int BM = 256, BN = 256, BK = 64, STAGES = 6;
constexpr int A_BYTES = 128 * BK * 2, STAGE_BYTES = 2 * A_BYTES;  // one CTA's half of a stage
constexpr int EW = 8, SLOT = 4096;  // epilogue warps and their staging bytes
constexpr int SMEM = STAGES * STAGE_BYTES + EW * SLOT + 1024 + 256;
static_assert(SMEM <= 227 * 1024, "shared memory per CTA");
constexpr int BLK = 128;       // columns of one (m, s) pair
constexpr int PAD = 256;       // zero rows behind the packed ones
enum { LOGITS = 0, DH = 1, DW = 2 };

inline int blocks(int v) { return (v + BLK - 1) / BLK; }
inline int ld_g(int v) { return (v + 63) / 64 * 64; }
inline int pad_rows(int n) { return (n + BM - 1) / BM * BM; }

constexpr int TOP = 128;  // entries of a row's teacher, at most (places fit a byte)

// The tensor cores' sums are cut off below their last place, so that a logit falls short of its
// value by a part that grows with its terms: some 2^-30 of it a term where they are centred, up to
// three times that where all are positive, nothing where the sums are exact.  Of rows of 2,048 that
// is more than a teacher's losses are off by otherwise, so the logits against a teacher are sums
// of up to 768 terms on the tensor cores, added up in fp32 with rounding: losses of 512 rows of
// 2,048 on 32,000 words at a temperature of a half are off by 5.2e-7 in norm, 1.6e-6 as one sum,
// at 1 to 2 % of the time (8,191 rows).  The first sum is the longest: the epilogue of the tile
// before works under it.
constexpr int FIRST_K = 12, MORE_K = 10;  // K steps of the first such sum and of those behind it
// A warpgroup for the copies and the products, and two for the epilogue, whose 128 logits a
// thread stay in registers: each has its share of what the launch has, 168 for each of 384 threads
// (2,047 rows of 1,024 on 32,000 words without gradients: 99 us; 123 with 168 for all, which
// spills; 148 with the sum written back to its accumulator, which the next products wait for).
constexpr int TEACHER_THREADS = 128 + 32 * EW, FEW_REGS = 56, MANY_REGS = 224;
static_assert(128 * FEW_REGS + 32 * EW * MANY_REGS <= 168 * TEACHER_THREADS, "registers of the launch");
__host__ __device__ constexpr int threads(bool teacher) { return teacher ? TEACHER_THREADS : 64 + 32 * EW; }
}  // namespace vocab

struct VocabGemm {
    int rows_max;      // rows of the piece, at most
    const int* count;  // packed rows of the call (null: rows_max is exact)
    int r0;            // first packed row of the piece
    int vocab, d;
    int split;         // DH: parts of the vocabulary
    // LOGITS
    const int* targets;  // of the packed rows
    uint16_t* G;         // null: losses only
    float2* stats;       // [rows][blocks]: maximum, and sum without the target's term
    float* at_target;    // [rows]; of a teacher's entries [rows][top]
    // a teacher: by row of the call, its entries' words in order, and where each block's start
    const int* words;          // [n][top]
    const uint8_t* starts;     // [n][blocks + 1]
    int top;
    float log2e, scale;        // logits over the temperature: to base 2, and to base e
    // DH, DW
    const int* index;  // packed row -> row (null: the same)
    uint16_t* out;
    long long ldo;
    float* acc;        // DH: [split][rows_max][d] partial sums; DW: [vocab][d] sums so far
    int first, last;   // DW: the first / last piece
    int* status;
};

__device__ __forceinline__ int vocab_rows(const VocabGemm& p) {
    const int n = p.count ? *p.count - p.r0 : p.rows_max;
    return n < 0 ? 0 : min(n, p.rows_max);
}

// A tile's place; row blocks in groups of 8, whose operand rows stay in L2 while the
// group sweeps the columns.
struct VocabTile {
    int mb, nb, part;
};
__device__ __forceinline__ VocabTile vocab_tile(int tile, int num_m, int num_n) {
    constexpr int GM = 8;
    VocabTile t;
    t.part = tile / (num_m * num_n);
    tile -= t.part * num_m * num_n;
    const int g = tile / (GM * num_n), in = tile - g * GM * num_n, gm = min(GM, num_m - g * GM);
    t.mb = g * GM + in % gm;
    t.nb = in / gm;
    return t;
}

// 64 columns (32 bf16 pairs a lane: its row) through the warp's slot, out as 128-byte
// row pieces: row(r) is the address of row r's first column, null: not written; units
// of 8 columns from `units` on are not written.
template <class F>
__device__ __forceinline__ void vocab_store64(uint8_t* slot, int lane, const uint32_t (&pk)[32],
                                              int units, F row) {
    uint8_t* mine = slot + lane * 128;
#pragma unroll
    for (int u = 0; u < 8; ++u)
        *reinterpret_cast<uint4*>(mine + ((u ^ (lane & 7)) << 4)) =
            make_uint4(pk[4 * u], pk[4 * u + 1], pk[4 * u + 2], pk[4 * u + 3]);
    __syncwarp();
    const int u = lane & 7;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int r = 4 * i + (lane >> 3);
        const uint4 v = *reinterpret_cast<const uint4*>(slot + r * 128 + ((u ^ (r & 7)) << 4));
        uint16_t* o = row(r);
        if (o && u < units) *reinterpret_cast<uint4*>(o + u * 8) = v;
    }
    __syncwarp();
}

// 32 fp32 columns, alike: f(address, values) of each 16-byte unit.
template <class R, class F>
__device__ __forceinline__ void vocab_each32(uint8_t* slot, int lane, const uint32_t (&w)[32],
                                             int units, R row, F f) {
    uint8_t* mine = slot + lane * 128;
#pragma unroll
    for (int u = 0; u < 8; ++u)
        *reinterpret_cast<uint4*>(mine + ((u ^ (lane & 7)) << 4)) =
            make_uint4(w[4 * u], w[4 * u + 1], w[4 * u + 2], w[4 * u + 3]);
    __syncwarp();
    const int u = lane & 7;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int r = 4 * i + (lane >> 3);
        const float4 v = *reinterpret_cast<const float4*>(slot + r * 128 + ((u ^ (r & 7)) << 4));
        const long long o = row(r);
        if (o >= 0 && u < units) f(o + u * 4, v);
    }
    __syncwarp();
}

// TEACHER: LOGITS with a teacher's entries as the targets.  PAIR: a 256 x 256 tile on a CTA
// pair; else one of 128 x 256 on one CTA.
template <int MODE, bool TEACHER, bool PAIR>
__device__ __forceinline__ void vocab_tiles(const CUtensorMap& ta, const CUtensorMap& tb, const VocabGemm& p) {
    using namespace vocab;
    constexpr bool AMN = MODE == DW, BMN = MODE != LOGITS;
    static_assert(PAIR || (!AMN && !BMN), "a lone CTA's operands are K-major");
    constexpr int BM = PAIR ? vocab::BM : vocab::BM / 2;
    constexpr int STAGES = PAIR ? vocab::STAGES : 4;
    constexpr int STAGE_BYTES = A_BYTES + (PAIR ? A_BYTES : 2 * A_BYTES);  // one CTA's of a stage
    static_assert(STAGES * STAGE_BYTES == vocab::STAGES * vocab::STAGE_BYTES, "one shared memory size");
    constexpr uint32_t IDESC =
        idesc_bf16_f32(BM, BN) | (AMN ? 1u << 15 : 0u) | (BMN ? 1u << 16 : 0u);
    extern __shared__ uint8_t smem_raw[];
    uint8_t* smem = reinterpret_cast<uint8_t*>(
        (reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
    uint8_t* slots = smem + STAGES * STAGE_BYTES;
    uint64_t* full = reinterpret_cast<uint64_t*>(slots + EW * SLOT);
    uint64_t* empty = full + STAGES;
    uint64_t* tfull = empty + STAGES;
    uint64_t* tempty = tfull + 2;
    uint64_t* drain = tempty + 2;
    uint64_t* never = drain + 1;  // nothing arrives on it: a bounded pause when giving up
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(never + 1);
    volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
    const int warp = warp_uniform(threadIdx.x >> 5), lane = threadIdx.x & 31;
    const uint32_t rank = PAIR ? cluster_rank() : 0;

    if (threadIdx.x == 0) {
        for (int s = 0; s < STAGES; ++s) {
            mbar_init(&full[s], 1);
            mbar_init(&empty[s], 1);
        }
        for (int a = 0; a < 2; ++a) {
            mbar_init(&tfull[a], 1);
            mbar_init(&tempty[a], (PAIR ? 2 : 1) * EW);
        }
        mbar_init(drain, 1);
        mbar_init(never, 1);
        *abort_flag = 0;
        fence_barrier_init();
        fence_proxy_async();
    }
    pdl_entry();  // TMEM is taken once the grid ahead has given its own back
    if (warp == 1) {
        if constexpr (PAIR) {
            tmem_alloc_pair(tmem_slot, 2 * BN);
            tmem_relinquish_pair();
        } else {
            tmem_alloc(tmem_slot, 2 * BN);
            tmem_relinquish();
        }
    }
    if (warp == 0 && lane == 0) {
        tma_prefetch_desc(&ta);
        tma_prefetch_desc(&tb);
    }
    tc_fence_before();
    if constexpr (PAIR) cluster_sync_all();
    else __syncthreads();
    tc_fence_after();
    const uint32_t tmem_base = warp_uniform(*tmem_slot);

    const int rows = warp_uniform(vocab_rows(p));
    const int M = MODE == DW ? p.vocab : rows, N = MODE == LOGITS ? p.vocab : p.d;
    const int K = MODE == LOGITS ? p.d : MODE == DH ? p.vocab : rows;
    const int num_m = (M + BM - 1) / BM, num_n = (N + BN - 1) / BN;
    const int all_k = (K + BK - 1) / BK;
    const int parts = MODE == DH ? p.split : 1;
    const int num_tiles = num_m * num_n * parts;
    const int first = blockIdx.x >> (PAIR ? 1 : 0), step = gridDim.x >> (PAIR ? 1 : 0);
    // K steps [k0, k1) of a part
    auto k_begin = [&](int part) { return (int)((long long)all_k * part / parts); };
    // sums of a tile, each in an accumulator of its own
    const int pieces = !TEACHER || all_k <= FIRST_K ? 1 : 1 + (all_k - FIRST_K + MORE_K - 1) / MORE_K;
    constexpr int EW0 = TEACHER ? 4 : 2;  // the first epilogue warp

    if (warp < EW0) {
        if constexpr (TEACHER) reg_dealloc<FEW_REGS>();
        if (warp == 0) {
            int stage = 0;
            uint32_t phase = 0;
            bool ok = true;
            for (int tile = first; ok && tile < num_tiles && !__any_sync(0xffffffffu, *abort_flag);
                 tile += step) {
                const VocabTile t = vocab_tile(tile, num_m, num_n);
                const int arow = t.mb * BM + (int)rank * 128, brow = t.nb * BN + rank * 128;
                for (int kb = k_begin(t.part); kb < k_begin(t.part + 1); ++kb) {
                    if (!mbar_wait_warp(&empty[stage], phase ^ 1)) {
                        ok = false;
                        break;
                    }
                    if (elect_one()) {
                        uint8_t* sa = smem + stage * STAGE_BYTES;
                        uint8_t* sb = sa + A_BYTES;
                        if constexpr (!PAIR) {
                            mbar_arrive_expect_tx(&full[stage], STAGE_BYTES);
                            tma_load_2d(sa, &ta, kb * BK, arow, &full[stage]);
                            tma_load_2d(sb, &tb, kb * BK, brow, &full[stage]);
                            tma_load_2d(sb + A_BYTES, &tb, kb * BK, brow + 128, &full[stage]);
                        } else {
                            const uint32_t bar = map_rank(&full[stage], 0);
                            if (rank == 0) mbar_arrive_expect_tx(&full[stage], 2 * STAGE_BYTES);
                            if constexpr (AMN) {
                                tma_load_2d_pair(sa, &ta, arow, kb * BK, bar);
                                tma_load_2d_pair(sa + A_BYTES / 2, &ta, arow + 64, kb * BK, bar);
                            } else {
                                tma_load_2d_pair(sa, &ta, kb * BK, arow, bar);
                            }
                            if constexpr (BMN) {
                                tma_load_2d_pair(sb, &tb, brow, kb * BK, bar);
                                tma_load_2d_pair(sb + A_BYTES / 2, &tb, brow + 64, kb * BK, bar);
                            } else {
                                tma_load_2d_pair(sb, &tb, kb * BK, brow, bar);
                            }
                        }
                    }
                    __syncwarp();
                    if (++stage == STAGES) {
                        stage = 0;
                        phase ^= 1;
                    }
                }
            }
            if (!ok) {
                *abort_flag = 1;
                report(p.status, JNX_ERR_TIMEOUT);
            }
        } else if (warp == 1 && rank == 0) {
            auto commit = [](uint64_t* b) {
                if constexpr (PAIR) tc_commit_pair(b);
                else tc_commit(b);
            };
            int stage = 0, local = 0;
            uint32_t phase = 0;
            bool ok = true;
            const uint32_t a0 = smem_u32(smem), b0 = a0 + A_BYTES;
            const uint32_t a_lo = AMN ? sw128_desc_mn_lo(a0, A_BYTES / 2) : sw128_desc_lo(a0);
            const uint32_t b_lo = BMN ? sw128_desc_mn_lo(b0, A_BYTES / 2) : sw128_desc_lo(b0);
            for (int tile = first, piece = 0;
                 ok && tile < num_tiles && !__any_sync(0xffffffffu, *abort_flag); ++local) {
                const VocabTile t = vocab_tile(tile, num_m, num_n);
                const int k0 = !TEACHER ? k_begin(t.part) : piece ? FIRST_K + (piece - 1) * MORE_K : 0;
                const int k1 = TEACHER ? min(all_k, FIRST_K + piece * MORE_K) : k_begin(t.part + 1);
                const int acc = local & 1;
                if (++piece == pieces) piece = 0, tile += step;
                if (!mbar_wait_cluster_warp(&tempty[acc], ((local >> 1) & 1) ^ 1)) {
                    ok = false;
                    break;
                }
                tc_fence_after();
                const uint32_t dcol = tmem_base + acc * BN;
                for (int kb = k0; kb < k1; ++kb) {
                    if (!mbar_wait_cluster_warp(&full[stage], phase)) {
                        ok = false;
                        break;
                    }
                    tc_fence_after();
                    const uint32_t off = (uint32_t)(stage * STAGE_BYTES) >> 4;
                    if (elect_one()) {
#pragma unroll
                        for (int kk = 0; kk < BK / 16; ++kk)
                            // (16 K rows of an MN-major operand are two 8-row atoms)
                            if constexpr (PAIR)
                                tc_mma_f16_pair(dcol, desc_of(a_lo + off + kk * (AMN ? 128 : 2), kSw128DescHi),
                                                desc_of(b_lo + off + kk * (BMN ? 128 : 2), kSw128DescHi), IDESC,
                                                (kb - k0) | kk);
                            else
                                tc_mma_f16(dcol, desc_of(a_lo + off + kk * 2, kSw128DescHi),
                                           desc_of(b_lo + off + kk * 2, kSw128DescHi), IDESC, (kb - k0) | kk);
                        commit(&empty[stage]);
                    }
                    __syncwarp();
                    if (++stage == STAGES) {
                        stage = 0;
                        phase ^= 1;
                    }
                }
                if (!ok) break;
                if (elect_one()) commit(&tfull[acc]);
                __syncwarp();
            }
            if (!ok) {
                *abort_flag = 1;
                report(p.status, JNX_ERR_TIMEOUT);
            }
            // no MMA still reads or writes either CTA after this
            if (elect_one()) commit(drain);
            __syncwarp();
            mbar_wait(drain, 0);
        } else if (warp == 1) {
            mbar_wait(drain, 0);  // the leader's last commit has reached this CTA
        }
    } else {
        if constexpr (TEACHER) reg_alloc<MANY_REGS>();
        const int q = warp & 3;             // TMEM lane quarter this warp may access
        const int half = (warp - EW0) >> 2; // its 128 of the tile's columns
        uint8_t* slot = slots + (warp - EW0) * SLOT;
        int local = 0;
        // A teacher's entries of a row of a tile: their number and the first two's columns, 8 bits
        // each, the first one's place among the row's, and the 32-column chunks that hold any.
        // They are looked up a tile ahead, a step of the chain between parts of this tile's work
        // (2,047 rows of 1,024 on 32,000 words: 102 us with lookups behind the product, 92 so)
        constexpr int AHEAD = 2;
        int tg = 0, te = 0, src = -1, next_col0 = 0;
        uint32_t seen = 0, mine = 0;
        auto look_row = [&](int tile) {
            src = -1;
            if (tile >= num_tiles) return;
            const VocabTile t = vocab_tile(tile, num_m, num_n);
            const int row = t.mb * BM + (int)rank * 128 + q * 32 + lane;
            next_col0 = t.nb * BN + half * 128;
            if (row < M && next_col0 < N) src = p.index[p.r0 + row];
        };
        auto look_places = [&]() {
            tg = te = 0;
            if (src < 0) return;
            const uint8_t* st = p.starts + (size_t)src * ((N + BLK - 1) / BLK + 1) + next_col0 / BLK;
            tg = st[0], te = st[1];
        };
        auto look_words = [&]() {
            seen = te - tg, mine = 0;
            const int* words = p.words + (size_t)src * p.top + tg;
            for (int k = 0; tg + k < te; ++k) {
                const int col = words[k] - next_col0;
                mine |= 1u << (col >> 5);
                if (k < AHEAD) seen |= col << (8 + 8 * k);
            }
        };
        if constexpr (TEACHER) {
            look_row(first);
            look_places();
            look_words();
        }
        for (int tile = first; tile < num_tiles; tile += step) {
            const VocabTile t = vocab_tile(tile, num_m, num_n);
            const int row0 = t.mb * BM + rank * 128 + q * 32, row = row0 + lane;
            const int col0 = t.nb * BN + half * 128;
            const bool summed = k_begin(t.part + 1) > k_begin(t.part);  // else nothing was
            const auto full = [&]() {
                if (mbar_wait(&tfull[local & 1], (local >> 1) & 1) && !*abort_flag) {
                    tc_fence_after();
                    return true;
                }
                *abort_flag = 1;
                report(p.status, JNX_ERR_TIMEOUT);
                return false;
            };
            const auto empty_again = [&]() {
                __syncwarp();
                if (elect_one()) {
                    if constexpr (PAIR) mbar_arrive_cluster(map_rank(&tempty[local & 1], 0));
                    else mbar_arrive(&tempty[local & 1]);
                }
                __syncwarp();
            };
            const auto columns = [&]() {
                return tmem_base + (local & 1) * BN + half * 128 + ((uint32_t)(q * 32) << 16);
            };
            const uint32_t tc = columns();
            if constexpr (TEACHER) {
                // the logits gather in registers, and an accumulator is free again as soon as its
                // part is added
                uint32_t x[4][32];
                bool ok = true;
                for (int i = 0; i < pieces && (ok = __all_sync(0xffffffffu, full())); ++i) {
                    const uint32_t from = columns();
                    if (i == 0) {
#pragma unroll
                        for (int c = 0; c < 4; ++c) tmem_ld32(from + c * 32, x[c]);
#pragma unroll
                        for (int c = 0; c < 4; ++c) tmem_ld_wait_regs(x[c]);
                    } else {
#pragma unroll
                        for (int c = 0; c < 8; ++c) {
                            uint32_t v[16];
                            tmem_ld16(from + c * 16, v);
                            tmem_ld_wait_regs16(v);
#pragma unroll
                            for (int e = 0; e < 16; e += 2) {
                                uint32_t* to = &x[c >> 1][(c & 1) * 16 + e];
                                float x0, x1;
                                f2_unpack(f2_add(f2_pack(__uint_as_float(to[0]), __uint_as_float(to[1])),
                                                 f2_pack(__uint_as_float(v[e]), __uint_as_float(v[e + 1]))),
                                          x0, x1);
                                to[0] = __float_as_uint(x0), to[1] = __float_as_uint(x1);
                            }
                        }
                    }
                    tc_fence_before();
                    empty_again();
                    ++local;
                }
                if (!ok) break;
                const int cols = min(BLK, N - col0);  // may be negative: nothing here
                const int here = seen & 255, first_place = tg;
                int taken = 0;  // of the entries here
                // the 32-column chunks that hold an entry of the warp's rows
                const uint32_t hit = __reduce_or_sync(0xffffffffu, mine);
                look_row(tile + step);
                float m = -INFINITY;
                if (cols < BLK) {  // no columns: -inf is no maximum and no term
#pragma unroll
                    for (int e = 0; e < BLK; ++e)
                        if (e >= cols) x[e / 32][e % 32] = 0xff800000u;
                }
#pragma unroll
                for (int c = 0; c < 4; ++c) {
#pragma unroll
                    for (int e = 0; e < 32; e += 2)
                        m = fmax3(m, __uint_as_float(x[c][e]), __uint_as_float(x[c][e + 1]));
                    // an entry's logit is taken out: -inf is no term of the sum
                    if (hit >> c & 1) {
                        while (taken < here) {
                            const size_t place = (size_t)row * p.top + first_place + taken;
                            const int col =
                                taken < AHEAD
                                    ? seen >> (8 + 8 * taken) & 255
                                    : p.words[(size_t)p.index[p.r0 + row] * p.top + first_place + taken] - col0;
                            if (col >> 5 != c) break;
                            float at = 0.f;
#pragma unroll
                            for (int e = 0; e < 32; ++e)
                                if (col == c * 32 + e) {
                                    at = __uint_as_float(x[c][e]);
                                    x[c][e] = 0xff800000u;
                                }
                            p.at_target[place] = at;
                            ++taken;
                        }
                        __syncwarp();
                    }
                }
                look_places();
                // (a loss is of all digits near zero: the difference to the maximum first)
                const float sub = m == -INFINITY ? 0.f : m;
                const uint64_t nm2 = f2_pack(-sub, -sub), to2 = f2_pack(p.log2e, p.log2e);
                uint64_t sums = f2_pack(0.f, 0.f);
                uint16_t* g0 = p.G ? p.G + (size_t)row0 * ((N + 63) / 64 * 64) + col0 : nullptr;
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                    if (c * 64 >= cols) break;
                    uint32_t pk[32];
#pragma unroll
                    for (int e = 0; e < 64; e += 2) {
                        const uint32_t* y = &x[2 * c + e / 32][e % 32];
                        float x0, x1;
                        f2_unpack(f2_mul(f2_add(f2_pack(__uint_as_float(y[0]), __uint_as_float(y[1])), nm2), to2),
                                  x0, x1);
                        x0 = ex2_approx(x0), x1 = ex2_approx(x1);
                        sums = f2_add(sums, f2_pack(x0, x1));
                        pk[e / 2] = cvt_bf2(x0, x1);
                    }
                    if (p.G)
                        vocab_store64(slot, lane, pk, 8, [&](int r) {
                            return g0 + (size_t)r * ((N + 63) / 64 * 64) + c * 64;
                        });
                }
                float s0, s1;
                f2_unpack(sums, s0, s1);
                if (row < M && cols > 0)
                    p.stats[(size_t)row * ((N + BLK - 1) / BLK) + col0 / BLK] = make_float2(m, s0 + s1);
                look_words();
                __syncwarp();
                continue;
            }
            if (!full()) break;
            if constexpr (MODE == LOGITS) {
                const int cols = min(BLK, N - col0);  // may be negative: nothing here
                const int tg = row < M ? p.targets[p.r0 + row] - col0 : -1;
                // the 32-column chunks that hold a target of the warp's rows
                const uint32_t hit = __reduce_or_sync(
                    0xffffffffu, (unsigned)tg < (unsigned)BLK ? 1u << (tg >> 5) : 0u);
                float m = -INFINITY, s = 0.f, at = 0.f;
#pragma unroll 1
                for (int c = 0; c < 4; ++c) {
                    uint32_t v[32];
                    tmem_ld32(tc + c * 32, v);
                    tmem_ld_wait_regs(v);
                    if (cols - c * 32 >= 32) {
#pragma unroll
                        for (int e = 0; e < 32; e += 2)
                            m = fmax3(m, __uint_as_float(v[e]), __uint_as_float(v[e + 1]));
                    } else {
#pragma unroll
                        for (int e = 0; e < 32; ++e)
                            if (c * 32 + e < cols) m = fmaxf(m, __uint_as_float(v[e]));
                    }
                    // a target's logit is taken out of the accumulator: -inf is no term of the
                    // sum (7,000 rows of 256 on 32,000 words 150 us; with a test for it in the
                    // loop below 208, with the sum over all terms 189: the logit was picked
                    // out by way of local memory)
                    if (hit >> c & 1) {
#pragma unroll
                        for (int e = 0; e < 32; ++e)
                            if (tg == c * 32 + e) {
                                at = __uint_as_float(v[e]);
                                v[e] = 0xff800000u;
                            }
                        tmem_st32(tc + c * 32, v);
                        tmem_st_wait();
                    }
                }
                constexpr float LOG2E = 1.4426950408889634f;
                const float sub = m == -INFINITY ? 0.f : m * LOG2E;
                uint16_t* g0 = p.G ? p.G + (size_t)row0 * ((N + 63) / 64 * 64) + col0 : nullptr;
#pragma unroll 1
                for (int c = 0; c < 2; ++c) {
                    if (c * 64 >= cols) break;
                    uint32_t pk[32];
#pragma unroll
                    for (int d = 0; d < 2; ++d) {
                        uint32_t v[32];
                        tmem_ld32(tc + c * 64 + d * 32, v);
                        tmem_ld_wait_regs(v);
#pragma unroll
                        for (int e = 0; e < 32; e += 2) {
                            const int at_col = c * 64 + d * 32 + e;
                            float x0 = ex2_approx(fmaf(__uint_as_float(v[e]), LOG2E, -sub));
                            float x1 = ex2_approx(fmaf(__uint_as_float(v[e + 1]), LOG2E, -sub));
                            if (at_col >= cols) x0 = 0.f;
                            if (at_col + 1 >= cols) x1 = 0.f;
                            s += x0 + x1;
                            pk[d * 16 + e / 2] = cvt_bf2(x0, x1);
                        }
                    }
                    if (p.G)
                        vocab_store64(slot, lane, pk, 8, [&](int r) {
                            return g0 + (size_t)r * ((N + 63) / 64 * 64) + c * 64;
                        });
                }
                tc_fence_before();
                if (row < M && cols > 0) {
                    p.stats[(size_t)row * ((N + BLK - 1) / BLK) + col0 / BLK] = make_float2(m, s);
                    if (tg >= 0 && tg < cols) p.at_target[row] = at;
                }
            } else if (MODE == DH && parts > 1) {
#pragma unroll 1
                for (int c = 0; c < 4; ++c) {
                    uint32_t v[32];
                    tmem_ld32(tc + c * 32, v);
                    tmem_ld_wait_regs(v);
                    const int col = col0 + c * 32;
                    vocab_each32(
                        slot, lane, v, (N - col + 3) / 4,
                        [&](int r) -> long long {
                            return row0 + r < M ? ((long long)t.part * p.rows_max + row0 + r) * N + col
                                                : -1;
                        },
                        [&](long long o, float4 w) { *reinterpret_cast<float4*>(p.acc + o) = w; });
                }
                tc_fence_before();
            } else if (MODE == DW && !(p.first && p.last)) {
#pragma unroll 1
                for (int c = 0; c < 4; ++c) {
                    uint32_t v[32];
                    tmem_ld32(tc + c * 32, v);
                    tmem_ld_wait_regs(v);
                    if (!summed)
#pragma unroll
                        for (int e = 0; e < 32; ++e) v[e] = 0;
                    const int col = col0 + c * 32;
                    vocab_each32(
                        slot, lane, v, (N - col + 3) / 4,
                        [&](int r) -> long long {
                            return row0 + r < M ? (long long)(row0 + r) * N + col : -1;
                        },
                        [&](long long o, float4 w) {
                            float4* at = reinterpret_cast<float4*>(p.acc + o);
                            if (!p.first) {
                                const float4 b = *at;
                                w = make_float4(w.x + b.x, w.y + b.y, w.z + b.z, w.w + b.w);
                            }
                            if (p.last)
                                *reinterpret_cast<uint2*>(p.out + o / N * p.ldo + o % N) =
                                    make_uint2(cvt_bf2(w.x, w.y), cvt_bf2(w.z, w.w));
                            else
                                *at = w;
                        });
                }
                tc_fence_before();
            } else {
#pragma unroll 1
                for (int c = 0; c < 2; ++c) {
                    uint32_t pk[32];
#pragma unroll
                    for (int d = 0; d < 2; ++d) {
                        uint32_t v[32];
                        tmem_ld32(tc + c * 64 + d * 32, v);
                        tmem_ld_wait_regs(v);
#pragma unroll
                        for (int e = 0; e < 32; e += 2)
                            pk[d * 16 + e / 2] =
                                summed ? cvt_bf2(__uint_as_float(v[e]), __uint_as_float(v[e + 1]))
                                       : 0u;
                    }
                    const int col = col0 + c * 64;
                    vocab_store64(slot, lane, pk, (N - col) / 8, [&](int r) -> uint16_t* {
                        if (row0 + r >= M) return nullptr;
                        const long long to =
                            MODE == DH && p.index ? p.index[p.r0 + row0 + r] : row0 + r;
                        return p.out + to * p.ldo + col;
                    });
                }
                tc_fence_before();
            }
            empty_again();
            ++local;
        }
    }

    __syncwarp();
    tc_fence_before();
    __syncthreads();
    // giving up: time for copies in flight to land before any CTA leaves
    if (*abort_flag && warp == 0) mbar_wait(never, 0, 100000000LL);
    __syncthreads();
    if constexpr (PAIR) cluster_sync_all();
    tc_fence_after();
    if (warp == 1) {
        if constexpr (PAIR) tmem_dealloc_pair(tmem_base, 2 * BN);
        else tmem_dealloc(tmem_base, 2 * BN);
    }
}

template <int MODE, bool TEACHER = false>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(vocab::threads(TEACHER), 1)
    k_vocab_gemm(const __grid_constant__ CUtensorMap ta, const __grid_constant__ CUtensorMap tb,
                 const __grid_constant__ VocabGemm p) {
    vocab_tiles<MODE, TEACHER, true>(ta, tb, p);
}

// The logits of few rows against a teacher: blocks of 128 rows on single CTAs.
__global__ void __launch_bounds__(vocab::TEACHER_THREADS, 1)
    k_vocab_teacher_gemm(const __grid_constant__ CUtensorMap ta, const __grid_constant__ CUtensorMap tb,
                         const __grid_constant__ VocabGemm p) {
    vocab_tiles<vocab::LOGITS, true, false>(ta, tb, p);
}

constexpr int kCountRows = 8192;

struct VocabRows {
    const int* targets;
    int n, vocab, d;
    int *count, *index, *packed, *place, *status;
};

// Which rows count, in order: index[j] and the targets of packed row j, place[i] of row i
// (-1: ignored) and their number.  One CTA, 8 rows a thread at a time.  For calls of more than
// kCountRows rows; up to there k_vocab_gather's CTAs count what is ahead of their rows.
__global__ void __launch_bounds__(1024)
    k_vocab_pack(const __grid_constant__ VocabRows p) {
    __shared__ int sums[32];
    __shared__ int total;
    pdl_entry();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    if (threadIdx.x == 0) total = 0;
    for (int base = 0; base < p.n; base += 8192) {
        const int i0 = base + threadIdx.x * 8;
        int t[8], mine = 0;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            t[e] = i0 + e < p.n ? p.targets[i0 + e] : -1;
            if (t[e] >= p.vocab) {
                report(p.status, JNX_ERR_DEVICE_BOUNDS);
                t[e] = -1;
            }
            mine += t[e] >= 0;
        }
        int run = mine;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int x = __shfl_up_sync(0xffffffffu, run, o);
            if (lane >= o) run += x;
        }
        __syncthreads();  // the last round's sums and total have been read
        if (lane == 31) sums[warp] = run;
        __syncthreads();
        int at = total + run - mine;
        for (int w = 0; w < warp; ++w) at += sums[w];
        __syncthreads();
        if (threadIdx.x == 1023) total = at + mine;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            if (i0 + e >= p.n) break;
            if (t[e] >= 0) {
                p.index[at] = i0 + e;
                p.packed[at] = t[e];
            }
            p.place[i0 + e] = t[e] >= 0 ? at++ : -1;
        }
    }
    __syncthreads();
    if (threadIdx.x == 0) *p.count = total;
}

// h's rows to their packed places and zero rows behind them; ignored rows get loss 0 and
// gradient 0.  A CTA a row.  COUNT: it counts the rows ahead itself, a launch less: 2 of some 50
// us of 333 rows of 2,048 on 32,000 words, and training on 8,192 rows of 1,024 on 8,000 188 us for
// 200; the reads grow with the square of the rows, hence the limit.
template <bool COUNT>
__global__ void __launch_bounds__(256)
    k_vocab_gather(const uint16_t* h, long long ldh, const __grid_constant__ VocabRows p,
                   uint16_t* packed_h, float* loss, uint16_t* dh, long long lddh) {
    __shared__ int sums[8];
    pdl_entry();
    const int i = blockIdx.x;
    const uint4 zero = make_uint4(0, 0, 0, 0);
    int to;
    if constexpr (COUNT) {
        auto counts = [&](int t) { return t >= 0 && t < p.vocab; };
        const int mine = i < p.n ? p.targets[i] : 0;
        int ahead = 0;
#pragma unroll 4
        for (int j = threadIdx.x; j < min(i, p.n); j += 256) ahead += counts(p.targets[j]);
        ahead = __reduce_add_sync(0xffffffffu, ahead);
        if ((threadIdx.x & 31) == 0) sums[threadIdx.x >> 5] = ahead;
        __syncthreads();
        ahead = 0;
#pragma unroll
        for (int w = 0; w < 8; ++w) ahead += sums[w];
        to = i >= p.n ? ahead + (i - p.n) : counts(mine) ? ahead : -1;
        if (threadIdx.x == 0) {
            if (i == p.n) *p.count = ahead;
            if (i < p.n && to >= 0) {
                p.index[to] = i;
                p.packed[to] = mine;
            }
            if (mine >= p.vocab) report(p.status, JNX_ERR_DEVICE_BOUNDS);
        }
    } else {
        to = i < p.n ? p.place[i] : *p.count + (i - p.n);
    }
    const uint16_t* from = i < p.n ? h + i * ldh : nullptr;
    uint16_t* dst = to >= 0 ? packed_h + (size_t)to * p.d : dh ? dh + i * lddh : nullptr;
    if (to < 0) {
        from = nullptr;
        if (threadIdx.x == 0) loss[i] = 0.f;
    }
    if (dst)
        for (int c = threadIdx.x * 8; c < p.d; c += 2048)
            *reinterpret_cast<uint4*>(dst + c) = from ? *reinterpret_cast<const uint4*>(from + c) : zero;
}

// A row's loss from its blocks' (m, s) and its target's logit, and its probabilities scaled
// to G.  A CTA a row.
__global__ void __launch_bounds__(256)
    k_vocab_rows(const float2* stats, const float* at_target, const __grid_constant__ VocabGemm p,
                 const float* weight, float* loss) {
    __shared__ float red[16];
    pdl_entry();
    const int r = blockIdx.x, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    if (r >= vocab_rows(p)) return;
    const int nb = (p.vocab + vocab::BLK - 1) / vocab::BLK;
    const float2* st = stats + (size_t)r * nb;
    float m = -INFINITY, s = 0.f;
    for (int b = threadIdx.x; b < nb; b += 256) m = fmaxf(m, st[b].x);
#pragma unroll
    for (int o = 16; o; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
    if (lane == 0) red[warp] = m;
    __syncthreads();
    for (int w = 0; w < 8; ++w) m = fmaxf(m, red[w]);
    for (int b = threadIdx.x; b < nb; b += 256) s += st[b].y * expf(st[b].x - m);
#pragma unroll
    for (int o = 16; o; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
    if (lane == 0) red[8 + warp] = s;
    __syncthreads();
    s = 0.f;
    for (int w = 0; w < 8; ++w) s += red[8 + w];
    const int t = p.targets[p.r0 + r], row = p.index[p.r0 + r];  // (a packed row's target counts)
    if (!p.G && threadIdx.x > 0) return;
    const float below = m - at_target[r], e = expf(-below), z = s + e;
    // s / e may be large or overflow where the target is far below the maximum
    if (threadIdx.x == 0) loss[row] = s <= e ? log1pf(s / e) : below + logf(z);
    if (!p.G) return;
    const float w = weight[row], scale = w / z, at_t = -w * (s / z);
    uint16_t* g = p.G + (size_t)r * ((p.vocab + 63) / 64 * 64);
    for (int c = threadIdx.x * 8; c < p.vocab; c += 2048) {
        const float f = scale * expf(st[c / vocab::BLK].x - m);
        const uint4 u = *reinterpret_cast<const uint4*>(g + c);
        uint32_t v[4] = {u.x, u.y, u.z, u.w};
        const bool hit = (t & ~7) == c;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            float a = f * __uint_as_float(v[i] << 16), b = f * __uint_as_float(v[i] & 0xffff0000u);
            if (hit && (t & 7) == 2 * i) a = at_t;
            if (hit && (t & 7) == 2 * i + 1) b = at_t;
            v[i] = cvt_bf2(a, b);
        }
        *reinterpret_cast<uint4*>(g + c) = make_uint4(v[0], v[1], v[2], v[3]);
    }
}

// A row's teacher: the words of its entries in order, their probabilities and the logarithms of
// these, and where each block's words start.  A warp a row; every entry counts those ahead of
// it, 2 top^2 comparisons in all.
struct VocabTeacher {
    const int* ids;
    const float* logits;
    int n, vocab, top;
    float inv_tau;
    int *words, *flag, *count;  // flag: 0 for a row that has entries, else -1
    float *prob, *log_prob;
    uint8_t* starts;
    int* status;
};
__global__ void __launch_bounds__(128) k_vocab_teacher(const __grid_constant__ VocabTeacher a) {
    using vocab::TOP;
    constexpr int NONE = 0x7fffffff;
    __shared__ int4 id_s[4][TOP / 4], key_s[4][TOP / 4];
    __shared__ int word_s[4][TOP];
    __shared__ float x_s[4][TOP], p_s[4][TOP], lp_s[4][TOP];
    pdl_entry();
    const int w = threadIdx.x >> 5, lane = threadIdx.x & 31, row = blockIdx.x * 4 + w;
    if (row >= a.n) return;
    int *id = reinterpret_cast<int*>(id_s[w]), *key = reinterpret_cast<int*>(key_s[w]);
    float* x = x_s[w];
    const size_t at = (size_t)row * a.top;
    const int quads = (a.top + 3) / 4;
    float top = -INFINITY;
    for (int k = lane; k < 4 * quads; k += 32) {
        int v = k < a.top ? a.ids[at + k] : NONE;
        const float l = (k < a.top ? a.logits[at + k] : -INFINITY) * a.inv_tau;
        if (k < a.top && v >= a.vocab) report(a.status, JNX_ERR_DEVICE_BOUNDS);
        if (v < 0 || v >= a.vocab || !(l > -INFINITY)) v = NONE;
        id[k] = key[k] = v;
        x[k] = l;
        if (v != NONE) top = fmaxf(top, l);
    }
#pragma unroll
    for (int o = 16; o; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
    float z = 0.f;
    __syncwarp();
    for (int k = lane; k < a.top; k += 32)
        if (id[k] != NONE) z += expf(x[k] - top);
#pragma unroll
    for (int o = 16; o; o >>= 1) z += __shfl_xor_sync(0xffffffffu, z, o);
    const float log_z = logf(z);
    bool twice = false;
    for (int k = lane; k < a.top; k += 32) {
        const int v = id[k];
        lp_s[w][k] = x[k] - top - log_z;
        p_s[w][k] = expf(x[k] - top - log_z);
        int same = 0;
        for (int j = 0; j < quads; ++j) {
            const int4 u = id_s[w][j];
            same += (u.x == v) + (u.y == v) + (u.z == v) + (u.w == v);
        }
        twice |= v != NONE && same > 1;
    }
    // an entry whose word was given before adds to that one, and is none by itself.  The
    // logarithm is of what the word's entries are to the largest of them: their probabilities
    // may all be zero in 32 bits, as a row's that is filled up with a word
    if (__any_sync(0xffffffffu, twice)) {
        for (int k = lane; k < a.top; k += 32) {
            if (id[k] == NONE) continue;
            float sum = p_s[w][k], high = x[k];
            int same = 0;
            bool again = false;
            for (int j = 0; j < a.top; ++j) {
                if (id[j] != id[k] || j == k) continue;
                if (j < k) again = true;
                else sum += expf(x[j] - top - log_z), high = fmaxf(high, x[j]), ++same;
            }
            if (again) key[k] = NONE;
            if (again || !same) continue;
            float parts = 0.f;
            for (int j = k; j < a.top; ++j)
                if (id[j] == id[k]) parts += expf(x[j] - high);
            p_s[w][k] = sum, lp_s[w][k] = high - top - log_z + logf(parts);
        }
        __syncwarp();
    }
    int count = 0;
    for (int k = lane; k < a.top; k += 32) {
        const int v = key[k];
        if (v == NONE) continue;
        int rank = 0;
        for (int j = 0; j < quads; ++j) {
            const int4 u = key_s[w][j];
            rank += (u.x < v) + (u.y < v) + (u.z < v) + (u.w < v);
        }
        ++count;
        word_s[w][rank] = v;
        a.words[at + rank] = v;
        a.prob[at + rank] = p_s[w][k];
        a.log_prob[at + rank] = lp_s[w][k];
    }
    count = __reduce_add_sync(0xffffffffu, count);
    __syncwarp();
    const int nb = (a.vocab + vocab::BLK - 1) / vocab::BLK;
    for (int b = lane; b <= nb; b += 32) {
        int lo = 0, hi = count;
        while (lo < hi) {
            const int mid = (lo + hi) >> 1;
            if (word_s[w][mid] < b * vocab::BLK) lo = mid + 1;
            else hi = mid;
        }
        a.starts[(size_t)row * (nb + 1) + b] = (uint8_t)lo;
    }
    if (lane == 0) {
        a.count[row] = count;
        a.flag[row] = count > 0 ? 0 : -1;
    }
}

// T (e^d - 1 - d), `grad` being T (e^d - 1).  Near d = 0 by the series d^2 (1/2! + d/3! + ...),
// whose terms up to d^10 / 10! leave under 2^-33 of it at a half: the difference would keep 2^-24
// of d only, and might be below zero.
__device__ __forceinline__ float vocab_term(float T, float d, float grad) {
    if (fabsf(d) < 0.5f) {
        float s = 1.f / 3628800;
        s = fmaf(s, d, 1.f / 362880);
        s = fmaf(s, d, 1.f / 40320);
        s = fmaf(s, d, 1.f / 5040);
        s = fmaf(s, d, 1.f / 720);
        s = fmaf(s, d, 1.f / 120);
        s = fmaf(s, d, 1.f / 24);
        s = fmaf(s, d, 1.f / 6);
        s = fmaf(s, d, 0.5f);
        return T * (d * d) * s;
    }
    return grad - (T > 0.f ? T * d : 0.f);  // (where T is zero d may be beyond range)
}

// k_vocab_rows with a teacher.  With d = log P - log T at an entry, the loss is the sum of
// T (e^d - 1 - d) over the entries and of P over all other words: no term is negative, so that
// near the teacher a loss is off by what d is off by, times its gradient, and no more.  (As
// sum T (log T - log P), each rounded, a loss under 1e-6 was lost.)  A CTA a row; thread k has
// entry k.  Bound by the probabilities' way through memory: 8,191 rows of 32,000, nine tenths of
// them with entries, 187 us (the next-token losses' 171; with four loads ahead of the sums 211:
// fewer CTAs an SM).
__global__ void __launch_bounds__(256)
    k_vocab_rows_teacher(const float2* stats, const __grid_constant__ VocabGemm p,
                         const int* count, const float* prob, const float* log_prob,
                         const float* weight, float inv_tau, float* loss) {
    __shared__ float red[4][8];
    pdl_entry();
    const int r = blockIdx.x, t = threadIdx.x, lane = t & 31, warp = t >> 5;
    if (r >= vocab_rows(p)) return;
    const int row = p.index[p.r0 + r], n = count[row];
    const int nb = (p.vocab + vocab::BLK - 1) / vocab::BLK;
    const float2* st = stats + (size_t)r * nb;
    uint16_t* out = p.G ? p.G + (size_t)r * ((p.vocab + 63) / 64 * 64) : nullptr;
    const size_t at = (size_t)row * p.top + t;
    const float x = t < n ? p.at_target[(size_t)r * p.top + t] : 0.f;
    float m = -INFINITY;
    for (int b = t; b < nb; b += 256) m = fmaxf(m, st[b].x);
#pragma unroll
    for (int i = 16; i; i >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, i));
    if (lane == 0) red[0][warp] = m;
    __syncthreads();
    for (int w = 0; w < 8; ++w) m = fmaxf(m, red[0][w]);
    // the other words' sum, the entries' below the maximum, and how many have the maximum: their
    // terms are one, and one of them is left out of what is added to it, so that it keeps its digits
    float other = 0.f, mine = 0.f;
    for (int b = t; b < nb; b += 256) other += st[b].y * expf((st[b].x - m) * p.scale);
    const float below = t < n ? (m - x) * p.scale : 0.f, e = t < n ? expf(-below) : 0.f;
    if (below > 0.f) mine = e;
    const int at_top = __popc(__ballot_sync(0xffffffffu, t < n && !(below > 0.f)));
#pragma unroll
    for (int i = 16; i; i >>= 1) {
        other += __shfl_xor_sync(0xffffffffu, other, i);
        mine += __shfl_xor_sync(0xffffffffu, mine, i);
    }
    if (lane == 0) red[1][warp] = other, red[2][warp] = mine, red[3][warp] = (float)at_top;
    __syncthreads();
    other = mine = 0.f;
    float tops = 0.f;
    for (int w = 0; w < 8; ++w) other += red[1][w], mine += red[2][w], tops += red[3][w];
    const bool sure = tops > 0.f;
    const float rest = other + mine + (sure ? tops - 1.f : 0.f);
    const float z = sure ? 1.f + rest : rest, log_z = sure ? log1pf(rest) : logf(rest);
    float g = 0.f, grad = 0.f;  // by the warps that have entries
    if (t < n) {
        const float T = prob[at], d = -below - log_z - log_prob[at];
        grad = d < 1.f ? T * expm1f(d) : e / z - T;
        g = vocab_term(T, d, grad);
    }
#pragma unroll
    for (int i = 16; i; i >>= 1) g += __shfl_xor_sync(0xffffffffu, g, i);
    if (lane == 0) red[0][warp] = g;  // (all have read the maxima: a barrier ago)
    if (!out) {
        __syncthreads();
        if (t == 0) loss[row] = ((red[0][0] + red[0][1]) + (red[0][2] + red[0][3])) + other / z;
        return;
    }
    const float w = weight[row] * inv_tau, scale = w / z;
    for (int c = t * 8; c < p.vocab; c += 2048) {
        const float f = scale * expf((st[c / vocab::BLK].x - m) * p.scale);
        const uint4 y = *reinterpret_cast<const uint4*>(out + c);
        uint32_t v[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
        for (int i = 0; i < 4; ++i)
            v[i] = cvt_bf2(f * __uint_as_float(v[i] << 16), f * __uint_as_float(v[i] & 0xffff0000u));
        *reinterpret_cast<uint4*>(out + c) = make_uint4(v[0], v[1], v[2], v[3]);
    }
    __syncthreads();
    if (t == 0) loss[row] = ((red[0][0] + red[0][1]) + (red[0][2] + red[0][3])) + other / z;
    if (t < n) out[p.words[at]] = f2bf(w * grad);
}

// dh's rows from the parts' sums, in the parts' order.  A CTA a row.
__global__ void __launch_bounds__(256)
    k_vocab_dh_sum(const __grid_constant__ VocabGemm p) {
    pdl_entry();
    const int r = blockIdx.x;
    if (r >= vocab_rows(p)) return;
    uint16_t* o = p.out + (long long)(p.index ? p.index[p.r0 + r] : r) * p.ldo;
    for (int c = threadIdx.x * 4; c < p.d; c += 1024) {
        float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
        for (int k = 0; k < p.split; ++k) {
            const float4 v = *reinterpret_cast<const float4*>(
                p.acc + ((size_t)k * p.rows_max + r) * p.d + c);
            s = make_float4(s.x + v.x, s.y + v.y, s.z + v.z, s.w + v.w);
        }
        *reinterpret_cast<uint2*>(o + c) = make_uint2(cvt_bf2(s.x, s.y), cvt_bf2(s.z, s.w));
    }
}

// ---------------------------------------------------------------------------
// host side
// ---------------------------------------------------------------------------

// Whether a teacher's kernel was compiled with the registers that its warpgroups share out: with
// fewer, those that take some would wait for ever.
static bool vocab_registers(const void* kernel, std::atomic<int>& known) {
    if (known.load() == 0) {
        cudaFuncAttributes at{};
        if (cudaFuncGetAttributes(&at, kernel) != cudaSuccess) return false;
        using namespace vocab;
        known = at.numRegs * TEACHER_THREADS >= 128 * FEW_REGS + 32 * EW * MANY_REGS ? 1 : -1;
    }
    return known.load() > 0;
}

template <int MODE, bool TEACHER = false>
static jnx_status vocab_gemm(const CUtensorMap& ta, const CUtensorMap& tb, const VocabGemm& p,
                             const char* what, cudaStream_t s) {
    using namespace vocab;
    static std::atomic<uint64_t> attr{0};
    if (set_smem_limit(reinterpret_cast<const void*>(k_vocab_gemm<MODE, TEACHER>), SMEM, attr) != cudaSuccess)
        return fail(JNX_ERR_CUDA, "%s: smem attribute", what);
    if constexpr (TEACHER) {
        static std::atomic<int> known{0};
        if (!vocab_registers(reinterpret_cast<const void*>(k_vocab_gemm<MODE, TEACHER>), known))
            return fail(JNX_ERR_CUDA, "%s: the kernel's registers are not those that it shares out", what);
    }
    const long long m = MODE == DW ? p.vocab : p.rows_max, n = MODE == LOGITS ? p.vocab : p.d;
    const long long tiles =
        (m + BM - 1) / BM * ((n + BN - 1) / BN) * (MODE == DH ? p.split : 1);
    if (tiles > 0x7fff0000) return fail(JNX_ERR_UNSUPPORTED, "%s: too many tiles", what);
    const int grid = 2 * (int)std::min<long long>(tiles, num_sms() / 2);
    pdl(k_vocab_gemm<MODE, TEACHER>, grid, threads(TEACHER), SMEM, s)(ta, tb, p);
    return launched(what);
}

// Against a teacher, tiles of 128 rows on lone CTAs where they take fewer rounds of the card than
// pairs' of 256, each as long: 333 rows of 1,024 on 32,000 words three for four (20.5 us for 27.1),
// up to 128 one for two (11.2 for 16.6).  Equal rounds go to the pairs, which read the words half as often.
static jnx_status vocab_logits(const CUtensorMap& th, const CUtensorMap& tw, const VocabGemm& p,
                               const char* what, cudaStream_t s) {
    using namespace vocab;
    const int sms = num_sms();
    const long long cols = (p.vocab + BN - 1) / BN;
    const long long pairs = (p.rows_max + BM - 1) / BM * cols, lone = (p.rows_max + BM / 2 - 1) / (BM / 2) * cols;
    if ((lone + sms - 1) / sms >= (pairs + sms / 2 - 1) / (sms / 2))
        return vocab_gemm<LOGITS, true>(th, tw, p, what, s);
    static std::atomic<uint64_t> attr{0};
    if (set_smem_limit(reinterpret_cast<const void*>(k_vocab_teacher_gemm), SMEM, attr) != cudaSuccess)
        return fail(JNX_ERR_CUDA, "%s: smem attribute", what);
    static std::atomic<int> known{0};
    if (!vocab_registers(reinterpret_cast<const void*>(k_vocab_teacher_gemm), known))
        return fail(JNX_ERR_CUDA, "%s: the kernel's registers are not those that it shares out", what);
    pdl(k_vocab_teacher_gemm, (int)std::min<long long>(lone, sms), TEACHER_THREADS, SMEM, s)(th, tw, p);
    return launched(what);
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
    // (rows are counted in steps of 8,192 and padded by 256)
    if (vocab > 0x7fffff00 || n_rows > 0x7fffff00 - 8192 || d > 0x7fffff00)
        return fail(JNX_ERR_UNSUPPORTED, "%s: sizes", what);
    return JNX_OK;
}

// The gradients' arguments; with no rows dw is set to zero here.
static jnx_status vocab_grads(const float* row_weight, int n_rows, int vocab, int d,
                              const uint16_t* dh, int64_t lddh, uint16_t* dw, int64_t lddw,
                              const char* what, cudaStream_t s) {
    if (n_rows > 0 && (!row_weight || !dh || !aligned16(dh) || lddh % 8 || lddh < d))
        return fail(JNX_ERR_INVALID_ARG, "%s: null or misaligned gradients", what);
    if (dw && (!aligned16(dw) || lddw % 8 || lddw < d))
        return fail(JNX_ERR_INVALID_ARG, "%s: misaligned weight gradient", what);
    if (n_rows == 0 && dw && cudaMemset2DAsync(dw, lddw * 2, 0, (size_t)d * 2, vocab, s) != cudaSuccess)
        return launched(what);
    return JNX_OK;
}

static jnx_status teacher_check(const int32_t* ids, const float* logits, int top, float temperature,
                                int n_rows, const char* what) {
    if (top < 1 || !(temperature > 0.f) || !(temperature < INFINITY) || !(1.f / temperature < INFINITY))
        return fail(JNX_ERR_INVALID_ARG, "%s: %d entries, temperature %g", what, top, temperature);
    if (top > vocab::TOP)
        return fail(JNX_ERR_UNSUPPORTED, "%s: over %d entries a row", what, vocab::TOP);
    if (n_rows > 0 && (!ids || !logits)) return fail(JNX_ERR_INVALID_ARG, "%s: null teacher", what);
    return JNX_OK;
}

static int vocab_piece(int n_rows, int piece_rows) {
    return std::max(1, std::min(n_rows, piece_rows > 0 ? piece_rows : 8192));
}

// Parts of dh's contraction over the vocabulary: as many as bring its tiles, d being
// narrow, nearest to whole rounds of the SM pairs, a K step of a tile being 0.33 us and
// the parts' sums passing memory twice at 6 TB/s.  Alike for all rows of a block.
static int vocab_split(int rows, int vocab_size, int d) {
    using namespace vocab;
    const int row_blocks = (rows + BM - 1) / BM;
    const long long tiles = (long long)row_blocks * ((d + BN - 1) / BN);
    const int pairs = 76, ksteps = (vocab_size + BK - 1) / BK;
    int best = 1;
    double best_us = 1e30;
    for (int s = 1; s <= 16 && s <= std::max(1, ksteps / 8); ++s) {
        const double us = 0.33 * ksteps * (double)((tiles * s + pairs - 1) / pairs) / s +
                          (s > 1 ? 3.0 + (double)s * row_blocks * BM * d * 8 / 6e6 : 0.0);
        if (us < best_us - 1e-9) {
            best_us = us;
            best = s;
        }
    }
    return best;
}

// The workspace, in order: the call's packed rows, then one piece's.
struct VocabWs {
    int *count, *index, *packed, *place;
    uint16_t* h;
    float2* stats;
    float* at_target;
    uint16_t* G;
    float* parts;
    float* acc;
    // a teacher's rows
    int *words, *flag, *entries;
    float *prob, *log_prob;
    uint8_t* starts;
    size_t bytes;
};
// Rows of dh's parts of a piece, and the most that pieces of up to so many rows have: fewer
// rows can have more parts.
static size_t vocab_parts_rows(int piece, int vocab_size, int d) {
    const int split = vocab_split(piece, vocab_size, d);
    return split > 1 ? (size_t)split * piece : 0;
}
static size_t vocab_parts_rows_upto(int piece, int vocab_size, int d) {
    size_t most = 0;
    for (long long rows = vocab::BM; rows < piece + vocab::BM; rows += vocab::BM)
        most = std::max(most, vocab_parts_rows((int)std::min<long long>(rows, piece), vocab_size, d));
    return most;
}
static VocabWs vocab_ws(void* base, int n, int vocab_size, int d, int piece, bool train,
                        size_t parts_rows, int top = 0) {
    using namespace vocab;
    VocabWs w{};
    uint8_t* at = static_cast<uint8_t*>(base);
    size_t used = 0;
    auto take = [&](size_t bytes) {
        uint8_t* p = at + used;
        used += (bytes + 255) & ~(size_t)255;
        return p;
    };
    const size_t rows = pad_rows(piece);
    w.count = reinterpret_cast<int*>(take(4));
    w.index = reinterpret_cast<int*>(take((size_t)n * 4));
    w.packed = reinterpret_cast<int*>(take((size_t)n * 4));
    w.place = reinterpret_cast<int*>(take((size_t)n * 4));
    w.h = reinterpret_cast<uint16_t*>(take(((size_t)n + PAD) * d * 2));
    w.stats = reinterpret_cast<float2*>(take(rows * blocks(vocab_size) * 8));
    w.at_target = reinterpret_cast<float*>(take(rows * (top ? top : 1) * 4));
    if (top) {
        w.words = reinterpret_cast<int*>(take((size_t)n * top * 4));
        w.flag = reinterpret_cast<int*>(take((size_t)n * 4));
        w.entries = reinterpret_cast<int*>(take((size_t)n * 4));
        w.prob = reinterpret_cast<float*>(take((size_t)n * top * 4));
        w.log_prob = reinterpret_cast<float*>(take((size_t)n * top * 4));
        w.starts = take((size_t)n * (blocks(vocab_size) + 1));
    }
    if (train) {
        w.G = reinterpret_cast<uint16_t*>(take(rows * ld_g(vocab_size) * 2));
        w.parts = reinterpret_cast<float*>(take(parts_rows * d * 4));
        w.acc = reinterpret_cast<float*>(take(n > piece ? (size_t)vocab_size * d * 4 : 0));
    }
    w.bytes = used + 255;
    return w;
}

static void* align256(void* p) {
    return reinterpret_cast<void*>((reinterpret_cast<uintptr_t>(p) + 255) & ~(uintptr_t)255);
}

// What a call has in place of targets.
struct TeacherSpec {
    const int32_t* ids;
    const float* logits;
    int top;
    float inv_tau;
};

static jnx_status vocab_run(const uint16_t* h, int64_t ldh, const uint16_t* w, int64_t ldw,
                            const int32_t* targets, const float* weight, int n, int vocab_size,
                            int d, int piece, float* loss, uint16_t* dh, int64_t lddh,
                            uint16_t* dw, int64_t lddw, void* workspace, size_t ws_bytes,
                            int* status, const char* what, cudaStream_t s,
                            const TeacherSpec* teacher = nullptr) {
    using namespace vocab;
    const bool train = weight != nullptr;
    const VocabWs ws = vocab_ws(align256(workspace), n, vocab_size, d, piece, train,
                                train ? vocab_parts_rows(piece, vocab_size, d) : 0,
                                teacher ? teacher->top : 0);
    if (!workspace || ws_bytes < ws.bytes)
        return fail(JNX_ERR_WORKSPACE, "%s: workspace too small", what);
    TraceScope ts(JNX_K_VOCAB, 0.0, s);
    if (teacher) {
        const VocabTeacher t{teacher->ids, teacher->logits, n,       vocab_size, teacher->top,
                             teacher->inv_tau, ws.words,    ws.flag, ws.entries, ws.prob,
                             ws.log_prob,  ws.starts,       status};
        pdl(k_vocab_teacher, (n + 3) / 4, 128, 0, s)(t);
        targets = ws.flag;
    }
    const VocabRows vr{targets, n, vocab_size, d, ws.count, ws.index, ws.packed, ws.place, status};
    if (n <= kCountRows) {
        pdl(k_vocab_gather<true>, n + PAD, 256, 0, s)(h, ldh, vr, ws.h, loss, dh, lddh);
    } else {
        pdl(k_vocab_pack, 1, 1024, 0, s)(vr);
        pdl(k_vocab_gather<false>, n + PAD, 256, 0, s)(h, ldh, vr, ws.h, loss, dh, lddh);
    }
    CUtensorMap tw, twmn;
    if (!make_tmap_bf16(&tw, w, vocab_size, d, ldw, 128, 64) ||
        (train && !make_tmap_bf16(&twmn, w, vocab_size, d, ldw, 64, 64)))
        return fail(JNX_ERR_CUDA, "%s: tensor map encode failed", what);
    for (int r0 = 0, rows; r0 < n; r0 += rows) {
        rows = std::min(piece, n - r0);
        VocabGemm p{};
        p.rows_max = rows;
        p.count = ws.count;
        p.r0 = r0;
        p.vocab = vocab_size;
        p.d = d;
        p.split = 1;
        p.targets = ws.packed;
        p.G = ws.G;
        p.stats = ws.stats;
        p.at_target = ws.at_target;
        p.index = ws.index;
        p.status = status;
        // rows of the piece alone, and the zero rows behind the last
        const int map_rows = r0 + rows == n ? rows + PAD : rows;
        const uint16_t* hp = ws.h + (size_t)r0 * d;
        CUtensorMap th, tg, tgmn, thmn;
        if (!make_tmap_bf16(&th, hp, map_rows, d, d, 128, 64))
            return fail(JNX_ERR_CUDA, "%s: tensor map encode failed", what);
        if (teacher) {
            p.words = ws.words;
            p.starts = ws.starts;
            p.top = teacher->top;
            p.log2e = (float)std::min(1.4426950408889634 * teacher->inv_tau, 3e38);
            p.scale = teacher->inv_tau;
            if (jnx_status st = vocab_logits(th, tw, p, what, s)) return st;
            pdl(k_vocab_rows_teacher, rows, 256, 0, s)(ws.stats, p, ws.entries, ws.prob, ws.log_prob,
                                                       weight, teacher->inv_tau, loss);
        } else {
            if (jnx_status st = vocab_gemm<LOGITS>(th, tw, p, what, s)) return st;
            pdl(k_vocab_rows, rows, 256, 0, s)(ws.stats, ws.at_target, p, weight, loss);
        }
        if (jnx_status st = launched(what)) return st;
        if (!train) continue;
        const int gr = pad_rows(piece), gc = ld_g(vocab_size);
        if (!make_tmap_bf16(&tg, ws.G, gr, gc, gc, 128, 64) ||
            !make_tmap_bf16(&tgmn, ws.G, gr, gc, gc, 64, 64) ||
            !make_tmap_bf16(&thmn, hp, map_rows, d, d, 64, 64))
            return fail(JNX_ERR_CUDA, "%s: tensor map encode failed", what);
        p.out = dh;
        p.ldo = lddh;
        p.split = std::min(vocab_split(rows, vocab_size, d), vocab_split(piece, vocab_size, d));
        p.acc = ws.parts;
        if (jnx_status st = vocab_gemm<DH>(tg, twmn, p, what, s)) return st;
        if (p.split > 1) pdl(k_vocab_dh_sum, rows, 256, 0, s)(p);
        if (dw) {
            p.out = dw;
            p.ldo = lddw;
            p.split = 1;
            p.acc = ws.acc;
            p.first = r0 == 0;
            p.last = r0 + rows == n;
            if (jnx_status st = vocab_gemm<DW>(tgmn, thmn, p, what, s)) return st;
        }
    }
    return launched(what);
}

}  // namespace jnx

using namespace jnx;

extern "C" size_t jnx_op_vocab_loss_workspace_bytes(int32_t n_rows, int32_t vocab, int32_t d) {
    if (n_rows < 0 || vocab <= 0 || d <= 0) return 0;
    return vocab_ws(nullptr, n_rows, vocab, d, vocab_piece(n_rows, 0), false, 0).bytes;
}

extern "C" jnx_status jnx_op_vocab_loss(const uint16_t* h, int64_t ldh, const uint16_t* w,
                                        int64_t ldw, const int32_t* targets, int32_t n_rows,
                                        int32_t vocab, int32_t d, float* loss, void* workspace,
                                        size_t ws_bytes, int32_t* status, void* stream) {
    clear_error();
    const char* what = "vocab loss";
    if (jnx_status st = vocab_check(h, ldh, w, ldw, targets, n_rows, vocab, d, loss, what)) return st;
    if (n_rows == 0) return JNX_OK;
    return vocab_run(h, ldh, w, ldw, targets, nullptr, n_rows, vocab, d, vocab_piece(n_rows, 0), loss,
                     nullptr, 0, nullptr, 0, workspace, ws_bytes, status, what,
                     static_cast<cudaStream_t>(stream));
}

extern "C" size_t jnx_op_vocab_loss_train_workspace_bytes(int32_t n_rows, int32_t vocab, int32_t d,
                                                          int32_t piece_rows) {
    if (n_rows < 0 || vocab <= 0 || d <= 0) return 0;
    const int piece = vocab_piece(n_rows, piece_rows);
    return vocab_ws(nullptr, n_rows, vocab, d, piece, true,
                    vocab_parts_rows_upto(piece, vocab, d)).bytes;
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
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    if (jnx_status st = vocab_grads(row_weight, n_rows, vocab, d, dh, lddh, dw, lddw, what, s)) return st;
    if (n_rows == 0) return JNX_OK;
    return vocab_run(h, ldh, w, ldw, targets, row_weight, n_rows, vocab, d,
                     vocab_piece(n_rows, piece_rows), loss, dh, lddh, dw, lddw, workspace, ws_bytes,
                     status, what, s);
}

extern "C" size_t jnx_op_vocab_distill_workspace_bytes(int32_t n_rows, int32_t vocab, int32_t d,
                                                       int32_t top) {
    if (n_rows < 0 || vocab <= 0 || d <= 0 || top <= 0) return 0;
    return vocab_ws(nullptr, n_rows, vocab, d, vocab_piece(n_rows, 0), false, 0, top).bytes;
}

extern "C" jnx_status jnx_op_vocab_distill(const uint16_t* h, int64_t ldh, const uint16_t* w,
                                           int64_t ldw, const int32_t* ids, const float* teacher,
                                           int32_t top, float temperature, int32_t n_rows,
                                           int32_t vocab, int32_t d, float* loss, void* workspace,
                                           size_t ws_bytes, int32_t* status, void* stream) {
    clear_error();
    const char* what = "vocab distill";
    if (jnx_status st = vocab_check(h, ldh, w, ldw, ids, n_rows, vocab, d, loss, what)) return st;
    if (jnx_status st = teacher_check(ids, teacher, top, temperature, n_rows, what)) return st;
    if (n_rows == 0) return JNX_OK;
    const TeacherSpec t{ids, teacher, top, 1.f / temperature};
    return vocab_run(h, ldh, w, ldw, nullptr, nullptr, n_rows, vocab, d, vocab_piece(n_rows, 0), loss,
                     nullptr, 0, nullptr, 0, workspace, ws_bytes, status, what,
                     static_cast<cudaStream_t>(stream), &t);
}

extern "C" size_t jnx_op_vocab_distill_train_workspace_bytes(int32_t n_rows, int32_t vocab,
                                                             int32_t d, int32_t top,
                                                             int32_t piece_rows) {
    if (n_rows < 0 || vocab <= 0 || d <= 0 || top <= 0) return 0;
    const int piece = vocab_piece(n_rows, piece_rows);
    return vocab_ws(nullptr, n_rows, vocab, d, piece, true, vocab_parts_rows_upto(piece, vocab, d),
                    top).bytes;
}

extern "C" jnx_status jnx_op_vocab_distill_train(
    const uint16_t* h, int64_t ldh, const uint16_t* w, int64_t ldw, const int32_t* ids,
    const float* teacher, int32_t top, float temperature, const float* row_weight, int32_t n_rows,
    int32_t vocab, int32_t d, int32_t piece_rows, float* loss, uint16_t* dh, int64_t lddh,
    uint16_t* dw, int64_t lddw, void* workspace, size_t ws_bytes, int32_t* status, void* stream) {
    clear_error();
    const char* what = "vocab distill train";
    if (jnx_status st = vocab_check(h, ldh, w, ldw, ids, n_rows, vocab, d, loss, what)) return st;
    if (jnx_status st = teacher_check(ids, teacher, top, temperature, n_rows, what)) return st;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    if (jnx_status st = vocab_grads(row_weight, n_rows, vocab, d, dh, lddh, dw, lddw, what, s)) return st;
    if (n_rows == 0) return JNX_OK;
    const TeacherSpec t{ids, teacher, top, 1.f / temperature};
    return vocab_run(h, ldh, w, ldw, nullptr, row_weight, n_rows, vocab, d,
                     vocab_piece(n_rows, piece_rows), loss, dh, lddh, dw, lddw, workspace, ws_bytes,
                     status, what, s, &t);
}
