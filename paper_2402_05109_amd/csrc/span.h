// Part of a paged KV cache (include/hydra.h, hydra_kv_span): which tiles of a row its nodes see, and which slots of a tile.
#pragma once

#include "device_common.h"
#include "internal.h"

namespace hydra {

struct SpanStat { float m, r; };                         // of a query: its largest unscaled score, and 1 / sum of 2^((score - m) c)

struct SpanArgs {
    const void *q;
    const void *kpages, *vpages;
    const int32_t *table, *seq_len, *first;              // first: NULL = 0
    const TreeDev *tree;
    float *apart;                                        // records of workgroups that share a head's keys
    SpanStat *stats;                                     // [B, H, Tq], or NULL
    float *z;                                            // the root's scores, by row and head, in the order of the row's tiles, z_slots of them; or NULL
    int z_slots;
    float *score;                                        // of the layer: [score_rows, H, 16 * max_pages]
    void *out;
    int32_t *flags;
    int max_pages, n_pages, layer, T, H, groups, key_wgs, n_sinks, window, n_scored;
    int plain;                                           // 16 bits: queries and result are half [B, T, H, Dh]; otherwise the packed query buffer and the next GEMM's input
    float c;                                             // log2(e) / sqrt(Dh)
};

// What the nodes of a row see, in tiles of W slots (W divides 32): tiles a0 .. a0 + na - 1 (sinks that do not touch the rest), then b0 .. b0 + nb - 1.
struct SpanRow {
    int L, F, S, low, total;                             // tokens, first slot, end of the sinks, first slot of the rest, L + T
    int a0, na, b0, n;                                   // n = na + nb
    bool ok;
    __device__ __forceinline__ int tile(int i) const { return i < na ? a0 + i : b0 + i - na; }
    // whether page lp holds a slot that some node sees
    __device__ __forceinline__ bool holds(int lp) const {
        const int s = lp * 16;
        return (s < total && s + 16 > low) || (S > F && s < S && s + 16 > F);
    }
};
template <int W>
__device__ __forceinline__ SpanRow span_row(const SpanArgs &p, int b) {
    SpanRow r;
    r.L = p.seq_len[b];
    r.F = p.first ? p.first[b] : 0;
    r.ok = r.L >= 0 && r.L <= p.max_pages * 16 - p.T && r.F >= 0 && r.F <= r.L;
    r.total = r.L + p.T;
    r.low = p.window > 0 ? max(r.F, r.L + 1 - p.window) : r.F;           // of the root: no node sees further back
    r.S = r.F + min(p.n_sinks, r.low - r.F);                              // sinks inside the rest are no part of their own
    r.b0 = r.low / W;
    r.a0 = r.F / W;
    r.na = r.S > r.F ? min((r.S + W - 1) / W, r.b0) - r.a0 : 0;
    r.n = r.na + (r.total + W - 1) / W - r.b0;
    return r;
}

// What one query sees: cached slots from `from` on or below `sinks` (never below F), and the tree slots that its ancestor mask names.
struct SpanQuery { int from, sinks; uint64_t anc0, anc1; };
struct SpanNode { int depth; uint64_t anc0, anc1; };                     // what the tree says of a query (behind the last node: of that one)
__device__ __forceinline__ SpanNode span_node(const SpanArgs &p, int query) {
    const int n = min(query, p.T - 1);
    return {p.tree->depth[n], p.tree->anc[n][0], p.tree->anc[n][1]};
}
__device__ __forceinline__ SpanQuery span_query(const SpanArgs &p, const SpanRow &r, int query, const SpanNode &node) {
    SpanQuery s = {0x7fffffff, 0, 0ull, 0ull};                            // behind the last node: nothing
    if (query >= p.T) return s;
    const int depth = node.depth;
    s.anc0 = node.anc0;
    s.anc1 = node.anc1;
    s.from = p.window > 0 ? max(r.F, r.L + depth + 1 - p.window) : r.F;
    s.sinks = r.F + min(p.n_sinks, r.total - r.F);
    if (p.window > 0 && p.window <= depth)                                // ancestors that are out of the window
        for (int a = p.tree->parent[query]; a >= 0; a = p.tree->parent[a]) {
            const int pos = r.L + p.tree->depth[a];
            if (pos < s.from && pos >= s.sinks) {
                if (a < 64) s.anc0 &= ~(1ull << a);
                else s.anc1 &= ~(1ull << (a - 64));
            }
        }
    return s;
}
__device__ __forceinline__ SpanQuery span_query(const SpanArgs &p, const SpanRow &r, int query) { return span_query(p, r, query, span_node(p, query)); }
// the low n bits, n clamped to [0, 32]
__device__ __forceinline__ uint32_t low_bits(int n) { return n <= 0 ? 0u : n >= 32 ? 0xffffffffu : (1u << n) - 1u; }

// Which of the 32 slots from slot0 on a query sees, one bit each.  Without a branch per slot.
__device__ __forceinline__ uint32_t span_seen(const SpanRow &r, const SpanQuery &q, int slot0) {
    const int rel = slot0 - r.L;                                          // node of the first slot; negative: cached slots first
    uint32_t tree;
    if (rel < 0) tree = -rel >= 32 ? 0u : (uint32_t)q.anc0 << -rel;
    else if (rel >= 64) tree = rel >= 128 ? 0u : (uint32_t)(q.anc1 >> (rel - 64));
    else tree = (uint32_t)(q.anc0 >> rel) | (rel > 32 ? (uint32_t)(q.anc1 << (64 - rel)) : 0u);
    const uint32_t held = low_bits(r.L - slot0) & ~low_bits(r.F - slot0);
    return tree | (held & (low_bits(q.sinks - slot0) | ~low_bits(q.from - slot0)));
}
// Which of the 32 slots from slot0 on some node of the row may see: what lies in the others may be anything.
__device__ __forceinline__ uint32_t span_held(const SpanRow &r, int slot0) {
    return (low_bits(r.total - slot0) & ~low_bits(r.low - slot0)) | (low_bits(r.S - slot0) & ~low_bits(r.F - slot0));
}
// Whether every query sees every slot of a tile of W: no mask is needed.
template <int W>
__device__ __forceinline__ bool span_whole(const SpanArgs &p, const SpanRow &r, int slot0) {
    if (slot0 < r.F || slot0 + W > r.L) return false;
    if (slot0 + W <= r.S) return true;
    return p.window == 0 || slot0 >= r.L + p.tree->max_depth + 1 - p.window;
}

// Where one node alone is counted, the root, its scores z are kept as the attention computes them, and once its maximum M and sum are known
//     score[s] += 2^((z_s - M) c) / l
// takes 12 bytes of a slot where another pass over K takes 64 to 512: 16 rows of 64 nodes behind 2048 tokens, 32 heads 158 -> 112 us, one row behind 32000, 40 heads 178 -> 124.
// by threads tid, tid + step, ... of the row's slots; dot(slot, page): the score of a slot for which z has no room
template <int W, class Dot>
__device__ __forceinline__ void span_add_root(const SpanArgs &p, const SpanRow &r, int b, int h, SpanStat st, int tid, int step, Dot dot) {
    const float *z = p.z + ((size_t)b * p.H + h) * p.z_slots;
    float *row = p.score + ((size_t)b * p.H + h) * ((size_t)p.max_pages * 16);
    for (uint32_t i = tid; i < (uint32_t)(r.n * W); i += step) {         // (the step behind the last slot may pass 2^31)
        const int slot0 = r.tile((int)(i / W)) * W, k = (int)(i % W), slot = slot0 + k;
        if (!((span_held(r, slot0) >> k) & 1u)) continue;
        float x;
        if (i < (uint32_t)p.z_slots) {
            x = z[i];
        } else {
            const SpanQuery q = span_query(p, r, 0);
            const int raw = p.table[(size_t)b * p.max_pages + (slot >> 4)];
            x = (span_seen(r, q, slot0) >> k) & 1u ? dot(slot, (unsigned)raw < (unsigned)p.n_pages ? raw : 0) : -INFINITY;
        }
        row[slot] = (slot < r.L ? row[slot] : 0.f) + __builtin_amdgcn_exp2f((x - st.m) * p.c) * st.r;
    }
}

enum { SPAN_MERGE_MAX = 16 };                            // records of a head
int launch_span_merge(hydra_ctx *c, hipStream_t s, const SpanArgs &a, int slots);                        // a.key_wgs > 1: joins the records of every head, and adds up the root's weights
int launch_span_f32(hydra_ctx *c, hipStream_t s, SpanArgs a, int slots, int units_max);                  // slots: host bound on what the nodes of a row see

}  // namespace hydra
