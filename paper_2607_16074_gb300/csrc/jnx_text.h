// What the operators of text tenants share: argument checks, the visibility rule and
// the tiles of packed prompts.
#pragma once
#include <cuda_runtime.h>
#include <stdint.h>

#include "../../include/jnx_ops.h"
#include "jnx_host.h"

namespace jnx {

inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

inline bool rows_ok(const jnx_head_rows* r) {
    return r && r->ptr && aligned16(r->ptr) && r->row_stride % 8 == 0 && r->head_stride % 8 == 0;
}

inline bool cache_ok(const jnx_kv_cache* c) {
    return c && c->k && c->v && aligned16(c->k) && aligned16(c->v) && c->n_slots >= 0 &&
           c->room >= 0 && c->slot_stride % 8 == 0 && c->row_stride % 8 == 0 &&
           c->head_stride % 8 == 0;
}

inline bool pages_ok(const jnx_pages* p) {
    return p && p->n_seqs >= 0 && p->max_pages >= 0 &&
           (p->n_seqs == 0 || p->max_pages == 0 || (p->table && p->ld >= 0));
}

// The page and row of a sequence's token; false: there is none.
struct Pages {
    const int* table;
    long long ld;
    int n_seqs, max_pages, n_pages, room;
    Pages() = default;
    Pages(const jnx_pages& p, const jnx_kv_cache& c)
        : table(p.table), ld(p.ld), n_seqs(p.n_seqs), max_pages(p.max_pages), n_pages(c.n_slots),
          room(c.room) {}
    __device__ __forceinline__ bool find(int seq, int token, int& page, int& row) const {
        if ((unsigned)seq >= (unsigned)n_seqs || token < 0 || room <= 0) return false;
        const int entry = token / room;
        row = token - entry * room;
        if (entry >= max_pages) return false;
        page = table[seq * ld + entry];
        return (unsigned)page < (unsigned)n_pages;
    }
};

constexpr int kMaxNodes = 64;  // of a sequence's tree

// A sequence's rows [first, first + n) among the call's; false: it is left out.
__device__ __forceinline__ bool tree_rows(const int* cu_nodes, int s, int n_rows, int most, int& first,
                                          int& n) {
    const int a = cu_nodes[s], b = cu_nodes[s + 1];
    first = a;
    n = b - a;
    return 0 <= a && a <= b && b <= n_rows && n <= most;
}

inline jnx_status launched(const char* what) {
    const cudaError_t e = cudaGetLastError();
    return e == cudaSuccess ? JNX_OK : fail(JNX_ERR_CUDA, "%s: %s", what, cudaGetErrorString(e));
}

// Keys that row i of a sequence's Lq query rows sees of its Lk keys.
__host__ __device__ inline int keys_seen(int i, int Lq, int Lk, int prefix) {
    const int causal = Lk - Lq + i + 1;
    const int n = causal > prefix ? causal : prefix;
    return n < 0 ? 0 : n < Lk ? n : Lk;
}

// First row of Lq that sees key j (Lq: none).
__host__ __device__ inline int first_row(int j, int Lq, int Lk, int prefix) {
    if (j < prefix) return 0;
    const int i = j - (Lk - Lq);
    return i < 0 ? 0 : i < Lq ? i : Lq;
}

// Rows of a 128-row tile are (token, query head of the group): whole tokens only.
__host__ __device__ inline int tile_tokens(int group) { return 128 / group; }

// Row tiles of one forward item, which share its keys.
__host__ __device__ inline int item_tiles(int head_dim) { return head_dim == 256 ? 1 : 2; }

constexpr int kMaxGroup = 64;

// Parts that the gradients' keys pass takes a 128-key tile's rows in: one where a sequence
// has a tile for every SM by itself, else 2,048 rows each (token, head of the group).  Of
// the sequence and the heads alone, so that a sequence's bits do not depend on others.  A
// part is item (sequence, first key + part): a tile's first key is a multiple of 128.
constexpr int kMaxParts = 64;
__host__ __device__ inline int key_parts(int at, int Lq, int Lk, int prefix, int group, int Hkv) {
    if ((long long)Hkv * ((Lk + 127) / 128) >= 152) return 1;
    const long long rows = (long long)(Lq - first_row(at, Lq, Lk, prefix)) * group;
    const long long n = (rows + 2047) / 2048;
    return n < 1 ? 1 : n < kMaxParts ? (int)n : kMaxParts;
}

// What a key tile's item costs, by which the keys' pass is sorted: rows of its part.
__host__ __device__ inline int part_rows(int at, int Lq, int Lk, int prefix, int np) {
    return (Lq - first_row(at, Lq, Lk, prefix)) / np;
}

// What a prompt's work list holds for a head layout: items of each pass, parts of a key tile
// at most, and items of the keys' pass up to the last one of a tile in parts.
struct PromptCounts {
    long long forward = 0, keys = 0, queries = 0, slabs = 0;
    int parts = 1;
};

// A sequence's place among the packed rows and keys, as the device's arrays have it.
struct PromptSeq {
    int q0, Lq, k0, Lk, pre;
};
// False: no such sequence, or one beyond the rows and keys that the call was launched for.
__device__ __forceinline__ bool prompt_seq(const int* cu_q, const int* cu_kv, const int* prefix, int n_seqs,
                                           int rows, int keys, int s, PromptSeq& x) {
    const int t = (unsigned)s < (unsigned)n_seqs ? s : 0;  // (no branch ahead of the loads)
    const int q0 = cu_q[t], q1 = cu_q[t + 1], k0 = cu_kv[t], k1 = cu_kv[t + 1];
    x = PromptSeq{q0, q1 - q0, k0, k1 - k0, prefix ? prefix[t] : 0};
    return t == s && 0 <= q0 && q0 <= q1 && q1 <= rows && 0 <= k0 && k0 <= k1 && k1 <= keys;
}

jnx_status heads_ok(int n_heads, int n_kv_heads, int head_dim, const char* what);

}  // namespace jnx
