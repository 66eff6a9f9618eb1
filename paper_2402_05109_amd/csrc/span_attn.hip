// Tree attention over part of a 16-bit cache: a sliding window, the first tokens that stay in sight, what evictions have left; and the sums of
// the weights that every slot receives, by which tokens are evicted.
//
// A query is a column of both products, S^T = K Q^T and O^T = V^T P^T, as in bf16_attn.hip, so maxima, sums, masks and rescale factors are per-lane scalars
// and the weights are in the order that the second product needs.  With c = log2(e) / sqrt(Dh), M the running maximum of the unscaled scores z of a query,
//     w = 2^((z - M) c),   l = sum w,   O = sum half(w) V,   result = O / l
// (w <= 1 is rounded to half, by at most 2^-11 of itself, because the second product takes 16-bit operands; l adds up the unrounded ones.  The result's own rounding to half is as
// large: against 64 bits 2.1e-4 of it, 2.2e-4 over 16 rows, where 32 bits up to the result give 2.1e-4.)
// Only tiles that some node sees are read: those of the sinks and those from the root's window on (SpanRow); masks are made for the tiles at the edges.
#include <algorithm>
#include <climits>

#include "attn_bf16.h"
#include "span.h"

namespace hydra {

static constexpr float LOG2E = 1.44269504f;

// 16 bytes of a query: dims d0 .. d0 + 7 of column `col` of a query tile.  Queries past the last one: that one, or whatever the packed buffer holds, of which nobody writes those:
// they may be no numbers, and whoever adds over queries leaves them out by a select.
template <int DH>
__device__ __forceinline__ u32x4_t span_query_piece(const SpanArgs &p, int b, int h, int qtile, int QTtot, int col, int d0) {
    const size_t packed = ((((size_t)b * p.H + h) * QTtot + qtile) * (DH / 16) + (d0 >> 4)) * 64 + ((d0 >> 3) & 1) * 32 + col;
    const size_t plain = ((size_t)(b * p.T + min(qtile * 32 + col, p.T - 1)) * p.H + h) * (DH / 8) + (d0 >> 3);
    return reinterpret_cast<const u32x4_t *>(p.q)[p.plain ? plain : packed];
}
// the root's score for one slot
template <int DH>
__device__ __forceinline__ float span_root_dot(const SpanArgs &p, int b, int h, int slot, int page) {
    const u32x4_t *kp = reinterpret_cast<const u32x4_t *>(reinterpret_cast<const a16_t *>(p.kpages) + kv_block_base(p.layer, p.n_pages, page, p.H, h, DH)) + (slot & 15);
    float z = 0.f;
    for (int d = 0; d < DH; d += 8) {
        const a16x8_t k = __builtin_bit_cast(a16x8_t, kp[d * 2]), q = __builtin_bit_cast(a16x8_t, span_query_piece<DH>(p, b, h, 0, (p.T + 31) >> 5, 0, d));
#pragma unroll
        for (int e = 0; e < 8; ++e) z = fmaf((float)k[e], (float)q[e], z);
    }
    return z;
}
// four dims of a result
template <int DH>
__device__ __forceinline__ void span_store(const SpanArgs &p, int m, int h, int dim, f32x4_t v) {
    a16_t *to = reinterpret_cast<a16_t *>(p.out) + (p.plain ? ((size_t)m * p.H + h) * DH + dim : x_index<true>(m, h * DH + dim, p.H * DH));
    *reinterpret_cast<u32x2_t *>(to) = u32x2_t{f2a_pack(v[0], v[1]), f2a_pack(v[2], v[3])};
}

static size_t span_lds_bytes(int Dh, int qt, int nw) {        // queries and tiles, or maxima, sums and O of one query tile
    return std::max(((size_t)qt * (Dh / 16) + (size_t)nw * (Dh / 8)) * 1024, (size_t)qt * nw * 256 + (size_t)nw * Dh * 128);
}

// Masked slots leave a weight of 0, and V of slots that no node of the row may see is replaced by 0: those hold what was never written or has been
// evicted.  (Values that are held are finite: whatever writes the cache clamps them.)
// The bytes of K and V bound it where rows or heads are many (16 rows of 64 nodes, 32 heads, 1570 slots: 411 MB in 75 us, 5.5 TB/s); where they are few, the way from a
// length to a page number to K to a result (a node behind 1028 tokens: 8 us and 3 for the records, of which the bytes would be 2.6).
template <int DH, int QT, int NW, bool STREAM>
__global__ __launch_bounds__(NW * 64, 2) void span_attn_kernel(SpanArgs p) {
    constexpr int KS = DH / 16, DT = DH / 32, TILE = KS + 2 * DT;    // KiB of a K and V tile
    extern __shared__ float lds[];                          // queries [QT][KS] and a tile per wave [NW][TILE] of 1 KiB blocks; then maxima and sums, O of one query tile
    const int tid = (int)threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int hl = lane >> 5, col = lane & 31;
    const int T = p.T, H = p.H;
    const int QTtot = (T + 31) >> 5, QG = (QTtot + QT - 1) / QT, per = QG * p.key_wgs;
    const int seq = (int)blockIdx.x >> 3;
    const int group = seq / per * 8 + ((int)blockIdx.x & 7), j = seq % per;
    if (group >= p.groups) return;
    const int b = group / H, h = group - b * H, qg = j % QG, key_wg = j / QG;
    // what does not depend on the row's length, beside the load of that (a row of 64 nodes behind 1028 tokens 13.3 us; behind it 14.1)
    constexpr int PIECES = (QT * KS + NW - 1) / NW;
    u32x4_t piece[PIECES];
#pragma unroll
    for (int i = 0; i < PIECES; ++i) {
        const int at = min(wave + i * NW, QT * KS - 1), qtile = min(qg * QT + at / KS, QTtot - 1);       // a second tile behind the last query: the first one again, which nobody stores
        piece[i] = span_query_piece<DH>(p, b, h, qtile, QTtot, col, 16 * (at % KS) + 8 * hl);
    }
    SpanNode node[QT];
#pragma unroll
    for (int q = 0; q < QT; ++q) node[q] = span_node(p, (qg * QT + q) * 32 + col);
    const int units = p.key_wgs * NW, unit = key_wg * NW + wave;
    const SpanRow r = span_row<32>(p, b);
    if (!r.ok) {                                            // uniform over the workgroup
        if (tid == 0 && j == 0 && h == 0) atomicOr(p.flags, FLAG_CAPACITY);
        return;
    }
    const int32_t *pt = p.table + (size_t)b * p.max_pages;
    const int mine_n = unit < r.n ? (r.n - unit + units - 1) / units : 0;      // this wave's tiles: unit, unit + units, ...
    // page ids of this wave's next 32 tiles, two per tile, one per lane; a page that no node sees may have none: the other one of its tile then
    auto page_ids = [&](int first) {
        int lp = 2 * r.tile(min(unit + (first + (lane >> 1)) * units, r.n - 1)) + (lane & 1);
        if (!r.holds(lp)) lp ^= 1;
        return pt[min(lp, p.max_pages - 1)];
    };
    int pgs = page_ids(0);
    u32x4_t *qs = reinterpret_cast<u32x4_t *>(lds);
    SpanQuery sq[QT];
#pragma unroll
    for (int q = 0; q < QT; ++q) sq[q] = span_query(p, r, (qg * QT + q) * 32 + col, node[q]);
#pragma unroll
    for (int i = 0; i < PIECES; ++i)
        if (wave + i * NW < QT * KS) qs[(wave + i * NW) * 64 + lane] = piece[i];
    __syncthreads();

    u32x4_t *mine = qs + (QT * KS + wave * TILE) * 64;      // this wave's tile: K blocks, then V blocks [page][dims / 32]
    const uint32_t mine_at = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) void *)mine;
    auto dma = [&](const u32x4_t *src, int block) {
        __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void *)src,
                                         (__attribute__((address_space(3))) void *)(uintptr_t)(mine_at + (uint32_t)block * 1024u), 16, 0, STREAM ? 2 : 0);      // 2: nontemporal
    };
    const a16_t *kpages = reinterpret_cast<const a16_t *>(p.kpages), *vpages = reinterpret_cast<const a16_t *>(p.vpages);
    int p0 = 0, p1 = 0;                                     // pages of the tile that is requested next
    auto next_pages = [&](int it) {
        if (it > 0 && (it & 31) == 0) { pgs = page_ids(it); asm volatile("" : "+v"(pgs)); }      // awaited in here, not behind the branch
        p0 = checked_page(__builtin_amdgcn_readlane(pgs, 2 * (it & 31)), p.n_pages, p.flags);
        p1 = checked_page(__builtin_amdgcn_readlane(pgs, 2 * (it & 31) + 1), p.n_pages, p.flags);
    };
    auto request_k = [&] {
        const u32x4_t *kp = reinterpret_cast<const u32x4_t *>(kpages + kv_block_base(p.layer, p.n_pages, (col >> 4) ? p1 : p0, H, h, DH)) + hl * 16 + (col & 15);
#pragma unroll
        for (int s = 0; s < KS; ++s) dma(kp + s * 32, s);
    };
    auto request_v = [&] {
#pragma unroll
        for (int g = 0; g < 2; ++g) {
            const u32x4_t *vp = reinterpret_cast<const u32x4_t *>(vpages + kv_block_base(p.layer, p.n_pages, g ? p1 : p0, H, h, DH)) + col * 2 + hl;
#pragma unroll
            for (int dt = 0; dt < DT; ++dt) dma(vp + dt * 64, KS + g * DT + dt);
        }
    };
    f32x16_t o[QT][DT];
#pragma unroll
    for (int q = 0; q < QT; ++q)
#pragma unroll
        for (int dt = 0; dt < DT; ++dt)
#pragma unroll
            for (int v = 0; v < 16; ++v) o[q][dt][v] = 0.f;
    float m_run[QT], l_run[QT];
#pragma unroll
    for (int q = 0; q < QT; ++q) { m_run[q] = -INFINITY; l_run[q] = 0.f; }
    const bool root = p.z != nullptr && qg == 0;            // this workgroup holds the root, whose scores are wanted
    float *z0 = p.z + ((size_t)b * H + h) * p.z_slots;
    // these have arrived: nothing in the loop is to wait for an ordinary load, which would be a wait for the DMA as well
    asm volatile("" : "+v"(pgs));
#pragma unroll
    for (int q = 0; q < QT; ++q) asm volatile("" : "+v"(sq[q].from), "+v"(sq[q].sinks), "+v"(sq[q].anc0), "+v"(sq[q].anc1));
    if (mine_n > 0) { next_pages(0); request_k(); request_v(); }
    for (int it = 0; it < mine_n; ++it) {
        const bool more = it + 1 < mine_n;
        const int slot0 = r.tile(unit + it * units) * 32;
        const bool whole = span_whole<32>(p, r, slot0);     // uniform
        asm volatile("s_waitcnt vmcnt(%0)" ::"n"(2 * DT) : "memory");             // K has landed: of what was asked for only V may be missing
        f32x16_t sc[QT];
#pragma unroll
        for (int q = 0; q < QT; ++q)
#pragma unroll
            for (int v = 0; v < 16; ++v) sc[q][v] = 0.f;
        int at = lane;
        asm volatile("" : "+v"(at));                        // keeps the reads of the queries inside the loop
#pragma unroll
        for (int s = 0; s < KS; ++s) {
            const a16x8_t k = __builtin_bit_cast(a16x8_t, mine[s * 64 + lane]);
#pragma unroll
            for (int q = 0; q < QT; ++q) sc[q] = HYDRA_MFMA16(k, __builtin_bit_cast(a16x8_t, qs[at + (q * KS + s) * 64]), sc[q]);
        }
        if (more) {
            next_pages(it + 1);
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");                    // K is read
            request_k();
        }
        u32x4_t pb[QT][2];
        const bool kept = root && (unit + it * units) * 32 + 32 <= p.z_slots;
#pragma unroll
        for (int q = 0; q < QT; ++q) {
            if (!whole) {
                const uint32_t seen = span_seen(r, sq[q], slot0) >> (4 * hl);
#pragma unroll
                for (int v = 0; v < 16; ++v) sc[q][v] = (seen >> (8 * (v >> 2) + (v & 3))) & 1u ? sc[q][v] : -INFINITY;
            }
            if (q == 0 && kept) {                            // wave-uniform; four stores, which the wait for V counts
                if (col == 0) {
                    float *to = z0 + (unit + it * units) * 32 + 4 * hl;
#pragma unroll
                    for (int g = 0; g < 4; ++g) *reinterpret_cast<f32x4_t *>(to + 8 * g) = f32x4_t{sc[0][4 * g], sc[0][4 * g + 1], sc[0][4 * g + 2], sc[0][4 * g + 3]};
                }
                asm volatile("" ::: "memory");
            }
            float cmax = -INFINITY;
#pragma unroll
            for (int v = 0; v < 16; ++v) cmax = fmaxf(cmax, sc[q][v]);
            const HalfWaves cm = half_waves(cmax);
            cmax = fmaxf(cm.lo, cm.hi);
            if (__any(cmax > m_run[q])) {                                          // always on the first visible tile
                const float m_new = fmaxf(m_run[q], cmax);
                const float alpha = m_new == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((m_run[q] - m_new) * p.c);
                m_run[q] = m_new;
                l_run[q] *= alpha;
#pragma unroll
                for (int dt = 0; dt < DT; ++dt)
#pragma unroll
                    for (int v = 0; v < 16; ++v) o[q][dt][v] *= alpha;
            }
            const float ref = m_run[q] == -INFINITY ? 0.f : m_run[q];
            float rs = 0.f;
#pragma unroll
            for (int v = 0; v < 16; ++v) {
                const float w = __builtin_amdgcn_exp2f((sc[q][v] - ref) * p.c);   // 0 for masked slots, exactly 1 for the largest
                sc[q][v] = w;
                rs += w;
            }
            const HalfWaves rh = half_waves(rs);
            l_run[q] += rh.lo + rh.hi;
            // P^T operands: page g uses accumulator registers 8g .. 8g+7 in order
#pragma unroll
            for (int g = 0; g < 2; ++g)
#pragma unroll
                for (int w = 0; w < 4; ++w) pb[q][g][w] = half_pack(sc[q][8 * g + 2 * w], sc[q][8 * g + 2 * w + 1]);
        }
        // V has landed: only the next K, and the root's scores on their way out, may be missing
        if (!more)     asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        else if (kept) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(KS + 4) : "memory");
        else           asm volatile("s_waitcnt vmcnt(%0)" ::"n"(KS) : "memory");
        if (!whole) {
            const uint32_t held = span_held(r, slot0);
            if (held != 0xffffffffu) {
#pragma unroll
                for (int g = 0; g < 2; ++g) {
                    u32x4_t keep;
#pragma unroll
                    for (int w = 0; w < 4; ++w) {
                        // dword w holds keys i = 2w, 2w+1 of this half-wave: token = 8*(i/4) + 4*hl + i%4
                        const int i0 = 2 * w, i1 = 2 * w + 1;
                        const int s0 = 16 * g + 8 * (i0 >> 2) + 4 * hl + (i0 & 3), s1 = 16 * g + 8 * (i1 >> 2) + 4 * hl + (i1 & 3);
                        keep[w] = ((held >> s0) & 1u ? 0x0000ffffu : 0u) | ((held >> s1) & 1u ? 0xffff0000u : 0u);
                    }
#pragma unroll
                    for (int dt = 0; dt < DT; ++dt) mine[(KS + g * DT + dt) * 64 + lane] &= keep;      // each lane its own 16 bytes
                }
            }
        }
#pragma unroll
        for (int g = 0; g < 2; ++g)
#pragma unroll
            for (int dt = 0; dt < DT; ++dt) {
                const a16x8_t v = __builtin_bit_cast(a16x8_t, mine[(KS + g * DT + dt) * 64 + lane]);
#pragma unroll
                for (int q = 0; q < QT; ++q) o[q][dt] = HYDRA_MFMA16(v, __builtin_bit_cast(a16x8_t, pb[q][g]), o[q][dt]);
            }
        if (more) {
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");                    // V is read
            request_v();
        }
    }

    // ---- merge the waves through LDS, one query tile after the other: maxima and sums [QT][NW][2][32], then O[NW][DT * 4][64] of four dims each
    __syncthreads();                                         // every wave is done with queries and tiles
    float *ml = lds;
    f32x4_t *ob = reinterpret_cast<f32x4_t *>(lds + QT * NW * 64);
    if (hl == 0) {
#pragma unroll
        for (int q = 0; q < QT; ++q) {
            ml[(q * NW + wave) * 64 + col] = m_run[q];
            ml[(q * NW + wave) * 64 + 32 + col] = l_run[q];
        }
    }
    __syncthreads();
    const int Tq = QTtot * 32;
    float *rec = p.apart + (((size_t)b * H + h) * p.key_wgs + key_wg) * apart_record(Tq, DH);
#pragma unroll
    for (int q = 0; q < QT; ++q) {
        const int qtile = qg * QT + q, query = qtile * 32 + col;
        if (qtile >= QTtot) break;                           // uniform over the workgroup
        const float *mq = ml + q * NW * 64;
        float m_tot = -INFINITY;
#pragma unroll
        for (int w = 0; w < NW; ++w) m_tot = fmaxf(m_tot, mq[w * 64 + col]);
        const float m_safe = m_tot == -INFINITY ? 0.f : m_tot;
        float l_tot = 0.f;
#pragma unroll
        for (int w = 0; w < NW; ++w) l_tot += __builtin_amdgcn_exp2f((mq[w * 64 + col] - m_safe) * p.c) * mq[w * 64 + 32 + col];
        const float f = __builtin_amdgcn_exp2f((m_run[q] - m_safe) * p.c);
#pragma unroll
        for (int id = 0; id < DT * 4; ++id) {
            const f32x16_t &od = o[q][id >> 2];
            const int v = 4 * (id & 3);
            ob[(wave * DT * 4 + id) * 64 + lane] = f32x4_t{od[v] * f, od[v + 1] * f, od[v + 2] * f, od[v + 3] * f};
        }
        __syncthreads();
        // the (band, group of 4 registers = 4 consecutive dims) items are shared out over the waves
        const float inv = 1.0f / l_tot;
        for (int id = wave; id < DT * 4; id += NW) {
            const int dt = id >> 2, g4 = id & 3;
            f32x4_t acc = ob[id * 64 + lane];
#pragma unroll
            for (int w = 1; w < NW; ++w) acc += ob[(w * DT * 4 + id) * 64 + lane];
            const int dim = 32 * dt + 8 * g4 + 4 * hl;
            if (query >= T) continue;                        // columns behind the last node go nowhere (a node behind 1028 tokens 11.6 us; with them in the records 12.6)
            if (p.key_wgs > 1) *reinterpret_cast<f32x4_t *>(rec + (size_t)query * DH + dim) = acc;
            else span_store<DH>(p, b * T + query, h, dim, acc * inv);
        }
        if (wave == 0 && hl == 0) {
            if (p.key_wgs > 1) {
                rec[(size_t)Tq * DH + query] = m_tot;
                rec[(size_t)Tq * DH + Tq + query] = l_tot;
            } else if (p.stats) {
                p.stats[((size_t)b * H + h) * Tq + query] = SpanStat{m_tot, inv};
            }
        }
        if (q == 0 && root && p.key_wgs == 1) {              // uniform: the root's weights, by the whole workgroup
            if (tid == 0) *reinterpret_cast<SpanStat *>(ml) = SpanStat{m_tot, inv};          // the first maximum and sum are read
            __syncthreads();                                 // (and every wave's scores are written)
            const SpanStat st = *reinterpret_cast<const SpanStat *>(ml);
            span_add_root<32>(p, r, b, h, st, tid, NW * 64, [&](int slot, int page) { return span_root_dot<DH>(p, b, h, slot, page); });
        }
        if (q + 1 < QT) __syncthreads();                     // the next query tile's sums go where these were
    }
}

// out = sum_u 2^((m_u - m) c) O_u / sum_u 2^((m_u - m) c) l_u over the records of a head: one thread per (query, 4 dims), all its loads in one round trip.
// The workgroups behind the first `blocks` of a head add up the root's weights instead.
template <bool F32, int DH>
__global__ __launch_bounds__(256) void span_merge_kernel(SpanArgs p, int blocks) {
    const int h = blockIdx.y, b = blockIdx.z, T = p.T, H = p.H;
    constexpr int per_q = DH >> 2;
    const bool slots = (int)blockIdx.x >= blocks;           // uniform
    const int n = slots ? 0 : (int)blockIdx.x * (256 / per_q) + (int)threadIdx.x / per_q;
    const int dim = (int)threadIdx.x % per_q * 4;
    const int Tq = ((T + 31) >> 5) * 32;
    const size_t recsz = apart_record(Tq, DH);
    const float *base = p.apart + (((size_t)b * H + h) * p.key_wgs) * recsz;
    const bool live = n < T;
    float mu[SPAN_MERGE_MAX], lu[SPAN_MERGE_MAX];
    f32x4_t ou[SPAN_MERGE_MAX];
#pragma unroll
    for (int u = 0; u < SPAN_MERGE_MAX; ++u) {
        mu[u] = -INFINITY; lu[u] = 0.f; ou[u] = f32x4_t{0.f, 0.f, 0.f, 0.f};
        if (u < p.key_wgs && live) {
            const float *r = base + u * recsz;
            mu[u] = r[(size_t)Tq * DH + n];
            lu[u] = r[(size_t)Tq * DH + Tq + n];
            if (!slots) ou[u] = *reinterpret_cast<const f32x4_t *>(r + (size_t)n * DH + dim);
        }
    }
    constexpr int W = F32 ? 16 : 32;
    const SpanRow row = span_row<W>(p, b);
    if (!live || !row.ok) return;
    float mt = -INFINITY;
#pragma unroll
    for (int u = 0; u < SPAN_MERGE_MAX; ++u) mt = fmaxf(mt, mu[u]);
    const float m_safe = mt == -INFINITY ? 0.f : mt;
    float den = 0.f;
    f32x4_t acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int u = 0; u < SPAN_MERGE_MAX; ++u) {
        const float w = u < p.key_wgs ? __builtin_amdgcn_exp2f((mu[u] - m_safe) * p.c) : 0.f;
        den += w * lu[u];
        acc += ou[u] * w;
    }
    const float inv = 1.0f / den;
    if (slots) {
        const int first = ((int)blockIdx.x - blocks) * 256 + (int)threadIdx.x, step = ((int)gridDim.x - blocks) * 256;
        span_add_root<W>(p, row, b, h, SpanStat{mt, inv}, first, step, [&](int slot, int page) {
            if constexpr (F32) {
                const float *k = reinterpret_cast<const float *>(p.kpages) + kv_block_base(p.layer, p.n_pages, page, H, h, DH) + (slot & 15) * DH;
                const float *q = reinterpret_cast<const float *>(p.q) + ((size_t)b * T * H + h) * DH;
                float z = 0.f;
                for (int d = 0; d < DH; ++d) z = fmaf(k[d], q[d], z);
                return z;
            } else {
                return span_root_dot<DH>(p, b, h, slot, page);
            }
        });
        return;
    }
    if (F32) *reinterpret_cast<f32x4_t *>(reinterpret_cast<float *>(p.out) + ((size_t)(b * T + n) * H + h) * DH + dim) = acc * inv;
    else span_store<DH>(p, b * T + n, h, dim, acc * inv);
    if (p.stats && dim == 0) p.stats[((size_t)b * H + h) * Tq + n] = SpanStat{mt, inv};
}

// The weights that every slot receives from nodes 0 .. n_scored - 1, behind the attention that has left each query's maximum and sum:
//     score[s] += sum_n 2^((z_ns - M_n) c) / l_n = sum_n 2^((z_ns - M'_n) c),   M' = M + log2(l) / c
// A query that does not count begins with -infinity, which alone is no guard (-infinity + NaN): its weights are left out of the sum.
// Queries are the rows of S = Q K^T here, so that a lane holds one slot and adds over its registers, and -M' is what the accumulators of the product begin with: a score costs a
// multiplication, an exponential and an addition.  A wave takes 32-key tiles in turn, the next one's K under way, from the last tile down: those are what the attention has
// read last, and the masked ones are then no wave's last (a row of 64 behind 4000 tokens, 32 heads 30.5 us against 32.2 the other way round); no two waves hold the same slot, so no sum depends
// on an order of arrival.  K's bytes bound it: 40 heads x 128 queries x 16128 slots 44 us, 32 without the products and 35 without the exponentials, of which a tile per
// wave takes 9 and the bytes 26 at 6.4 TB/s; a second tile ahead, and queries read from LDS ahead of the products, change nothing.
enum { SCORE_WAVES = 8 };
template <int DH, int QS>
__global__ __launch_bounds__(SCORE_WAVES * 64, 2) void span_score_kernel(SpanArgs p) {
    constexpr int KS = DH / 16, NW = SCORE_WAVES;
    extern __shared__ float lds[];                          // queries [QS][KS] of 1 KiB, then -M' of each, a bit row per query for each wave, and what each query sees
    const int tid = (int)threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int hl = lane >> 5, col = lane & 31;
    const int T = p.T, H = p.H, QTtot = (T + 31) >> 5, Tq = QTtot * 32;
    const int seq = (int)blockIdx.x >> 3;
    const int group = seq / p.key_wgs * 8 + ((int)blockIdx.x & 7), key_wg = seq % p.key_wgs;
    if (group >= p.groups) return;
    const int b = group / H, h = group - b * H;
    // what does not depend on the row's length, beside the load of that
    constexpr int PIECES = (QS * KS + NW - 1) / NW;
    static_assert(QS * 32 <= NW * 64, "a thread per query");
    u32x4_t piece[PIECES];
#pragma unroll
    for (int i = 0; i < PIECES; ++i) {
        const int at = min(wave + i * NW, QS * KS - 1);
        piece[i] = span_query_piece<DH>(p, b, h, min(at / KS, QTtot - 1), QTtot, col, 16 * (at % KS) + 8 * hl);
    }
    const bool counts = tid < p.n_scored;
    const SpanStat stat = p.stats[((size_t)b * H + h) * Tq + min(tid, Tq - 1)];
    const SpanNode node = span_node(p, tid);
    const SpanRow r = span_row<32>(p, b);
    if (!r.ok) return;                                      // reported by the attention
    const int units = p.key_wgs * NW, unit = key_wg * NW + wave;
    const int32_t *pt = p.table + (size_t)b * p.max_pages;
    const a16_t *kpages = reinterpret_cast<const a16_t *>(p.kpages);
    auto page_id = [&](int u) {                             // of the lane's slot in this wave's tile u, from the row's last one down; behind them all: the first one again
        int lp = 2 * r.tile(max(r.n - 1 - u, 0)) + (col >> 4);
        if (!r.holds(lp)) lp ^= 1;
        const int raw = pt[min(lp, p.max_pages - 1)];
        return (unsigned)raw < (unsigned)p.n_pages ? raw : 0;                    // reported by the attention
    };
    auto load = [&](u32x4_t (&k)[KS], int page) {
        const u32x4_t *kp = reinterpret_cast<const u32x4_t *>(kpages + kv_block_base(p.layer, p.n_pages, page, H, h, DH)) + hl * 16 + (col & 15);
#pragma unroll
        for (int s = 0; s < KS; ++s) k[s] = kp[s * 32];
    };
    u32x4_t k[KS];
    load(k, page_id(unit));
    int page = page_id(unit + units);
    u32x4_t *qs = reinterpret_cast<u32x4_t *>(lds);
    float *begin = reinterpret_cast<float *>(qs + QS * KS * 64);          // -M' of the queries; no weight at all: -infinity
    uint32_t *sees = reinterpret_cast<uint32_t *>(begin + QS * 32) + wave * 32;
    SpanQuery *sq = reinterpret_cast<SpanQuery *>(begin + QS * 32 + NW * 32);
    if (tid < QS * 32) {
        begin[tid] = counts ? __builtin_amdgcn_logf(stat.r) / p.c - stat.m : -INFINITY;
        sq[tid] = span_query(p, r, counts ? tid : T, node);
    }
#pragma unroll
    for (int i = 0; i < PIECES; ++i)
        if (wave + i * NW < QS * KS) qs[(wave + i * NW) * 64 + lane] = piece[i];
    __syncthreads();
    auto begins = [&](int q) {                              // in the accumulators' rows
        f32x16_t z;
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            const f32x4_t v = *reinterpret_cast<const f32x4_t *>(begin + q * 32 + 8 * g + 4 * hl);
#pragma unroll
            for (int e = 0; e < 4; ++e) z[4 * g + e] = v[e];
        }
        return z;
    };
    f32x16_t start[QS];
#pragma unroll
    for (int q = 0; q < QS; ++q) start[q] = begins(q);
    float *row = p.score + ((size_t)b * H + h) * ((size_t)p.max_pages * 16);
    for (int u = unit; u < r.n; u += units) {
        const int slot0 = r.tile(r.n - 1 - u) * 32, slot = slot0 + col;
        const bool whole = span_whole<32>(p, r, slot0), mine = hl == 0 && ((span_held(r, slot0) >> col) & 1u);
        const float before = mine && slot < r.L ? row[slot] : 0.f;
        u32x4_t next[KS];
        load(next, page);
        page = page_id(u + 2 * units);
        float sum = 0.f;
        int at = lane;
        asm volatile("" : "+v"(at));                         // keeps the reads of the queries inside the loop
        auto product = [&](int from, f32x16_t z) {
#pragma unroll
            for (int s = 0; s < KS; ++s) z = HYDRA_MFMA16(__builtin_bit_cast(a16x8_t, qs[from + s * 64]), __builtin_bit_cast(a16x8_t, k[s]), z);
            return z;
        };
        if (whole) {                                         // no branch between the products: one query tile's reads and products go beside the other's exponentials
#pragma unroll
            for (int q = 0; q < QS; ++q) {
                const f32x16_t z = product(at + q * KS * 64, start[q]);
                float part[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int v = 0; v < 16; ++v) {
                    const float w = __builtin_amdgcn_exp2f(z[v] * p.c);
                    part[v & 3] += q + 1 == QS && start[q][v] == -INFINITY ? 0.f : w;        // the last tile alone has queries that do not count
                }
                sum += (part[0] + part[1]) + (part[2] + part[3]);
                if (q & 1) __builtin_amdgcn_sched_barrier(0);          // four tiles at once do not fit the registers
            }
        } else {
#pragma unroll 1
            for (int q = 0; q < QS; ++q) {
                const f32x16_t z = product(at + q * KS * 64, begins(q));
                // what each query sees is worked out once, by the lane of its number, and read by all through LDS, which is in order within a wave
                asm volatile("" ::: "memory");
                if (hl == 0) sees[col] = span_seen(r, sq[q * 32 + col], slot0);
                asm volatile("" ::: "memory");
#pragma unroll
                for (int g = 0; g < 4; ++g) {
                    const u32x4_t w = *reinterpret_cast<const u32x4_t *>(sees + 8 * g + 4 * hl);
#pragma unroll
                    for (int e = 0; e < 4; ++e) sum += (w[e] >> col) & 1u ? __builtin_amdgcn_exp2f(z[4 * g + e] * p.c) : 0.f;
                }
            }
        }
        const HalfWaves two = half_waves(sum);
        if (mine) row[slot] = before + (two.lo + two.hi);
#pragma unroll
        for (int s = 0; s < KS; ++s) k[s] = next[s];
    }
}

// (query tiles of a wave, waves, request policy) that the rules below choose from
#define SPAN_EACH_OF(X, DHv) X(DHv, 1, 8, true) X(DHv, 1, 8, false) X(DHv, 2, 8, true) X(DHv, 2, 8, false) X(DHv, 1, 4, true) X(DHv, 2, 4, true) X(DHv, 2, 4, false)
#define SPAN_EACH(X) SPAN_EACH_OF(X, 128) SPAN_EACH_OF(X, 64)

int span_max_dynamic_lds() {
    hipError_t e = hipSuccess;
#define ATTR(DHv, QTv, NWv, STv) \
    if (e == hipSuccess) e = hipFuncSetAttribute((const void *)span_attn_kernel<DHv, QTv, NWv, STv>, hipFuncAttributeMaxDynamicSharedMemorySize, 160 * 1024);
    SPAN_EACH(ATTR)
#undef ATTR
    if (e != hipSuccess) return hip_fail(e, "hipFuncSetAttribute(attention over part of a cache)");
    return HYDRA_OK;
}

int launch_span_merge(hydra_ctx *c, hipStream_t s, const SpanArgs &a, int slots) {
    const int Dh = c->m.head_dim, blocks = ceil_div(a.T, 256 / (Dh / 4)), adding = a.z ? std::min(ceil_div(slots, 512), std::max(1, 1024 / a.groups)) : 0;
    const dim3 grid(blocks + adding, a.H, a.groups / a.H);
#define LAUNCH(Fv, DHv) if (c->bf16 != Fv && Dh == DHv) hipLaunchKernelGGL((span_merge_kernel<Fv, DHv>), grid, dim3(256), 0, s, a, blocks);
    LAUNCH(false, 128) LAUNCH(false, 64) LAUNCH(true, 128) LAUNCH(true, 64)
#undef LAUNCH
    HYDRA_LAUNCH_CHECK("span_merge_kernel");
    return HYDRA_OK;
}

// host bound on the slots of a row that a call's nodes see
static int span_slots(const hydra_ctx *c, const hydra_kv_span *span) {
    int64_t len = span->span_hint > 0 ? span->span_hint : span->kv.seq_len_hint > 0 ? span->kv.seq_len_hint : c->m.max_pos;
    if (span->window > 0) len = std::min(len, (int64_t)span->window - 1 + std::min<int64_t>(span->n_sinks, len));
    return (int)std::min<int64_t>(len + c->tree.T, INT_MAX / 2);
}

static SpanArgs span_args(hydra_ctx *c, int B, int layer, const void *q, bool plain, const int32_t *seq_len, const hydra_kv_span *span, float *apart, float *stats, int z_slots,
                          void *out, int32_t *flags) {
    SpanArgs a;
    const int H = c->m.n_heads;
    a.q = q; a.kpages = span->kv.k_pages; a.vpages = span->kv.v_pages; a.table = span->kv.page_table; a.seq_len = seq_len; a.first = span->first;
    a.tree = tree_dev(c); a.apart = apart; a.out = out; a.flags = flags;
    a.max_pages = span->kv.max_pages; a.n_pages = span->kv.n_pages; a.layer = layer; a.T = c->tree.T; a.H = H; a.groups = H * B; a.key_wgs = 1;
    a.n_sinks = span->n_sinks; a.window = span->window; a.plain = plain ? 1 : 0; a.c = LOG2E / sqrtf((float)c->m.head_dim);
    a.n_scored = span->score ? span->n_scored : 0;
    const bool root = a.n_scored == 1;
    a.stats = span->score && !root ? reinterpret_cast<SpanStat *>(stats) : nullptr;
    a.z = root ? stats : nullptr;
    a.z_slots = z_slots;
    a.score = span->score ? span->score + (size_t)layer * span->score_rows * H * ((size_t)span->kv.max_pages * 16) : nullptr;
    return a;
}

int launch_span_attention(hydra_ctx *c, hipStream_t s, int B, int layer, const void *q, bool plain, const int32_t *seq_len, const hydra_kv_span *span,
                          float *apart, int units_max, float *stats, int z_slots, void *out, int32_t *flags) {
    SpanArgs a = span_args(c, B, layer, q, plain, seq_len, span, apart, stats, z_slots, out, flags);
    const int T = a.T, H = a.H, Dh = c->m.head_dim, QTtot = ceil_div(T, 32), slots = span_slots(c, span);
    if (!c->bf16) return launch_span_f32(c, s, a, slots, std::min(units_max, (int)SPAN_MERGE_MAX));
    const int tiles = ceil_div(slots, 32) + 2;
    // us, 16 bits, Dh 128, seen tokens in brackets; 32 heads unless said:
    // - two query tiles to a wave read K and V once for both, but leave half the workgroups: 16 rows of 64 nodes (1500) 79 against 94 with one, a row of 128, 40 heads (16000)
    //   88 against 137; but a row of 64 (600) 17 against 12, (4100) 27 against 22
    // - four waves to a workgroup, so that two or more share a compute unit, once there is a workgroup for each: 16 rows of 64 79 against 86 with eight, 16 rows of one node (1024)
    //   48.6 against 50.3; with fewer workgroups eight: a row of 64 (4100) 22 against 27
    // - K and V pass the caches by where one workgroup reads them: a node (32000), 40 heads 107 against 122, 16 rows of 64 79 against 89; not where several query tiles read
    //   them: a row of 128 (4100) 31 against 35
    // - one workgroup per head up to 20 tiles, 36 behind more than 32 nodes: a node (300) 8.4 against 9.7 with more of them and a second kernel, (570) 9.8 against 10.3, (640) 12.0
    //   against 10.5; a row of 64 (640) 11.9 against 13.5, (900) 13.8 against 14.4, (1200) 15.6 against 14.6.  Behind several nodes a wave takes two tiles, which is worth as
    //   much as one behind a single node (a node (1028) then 14.2 against 12.4)
    // - as many workgroups as compute units: twice as many leave twice the records, a row of 64 (4100) 28 against 22
    const int qt = QTtot > 1 && (H * B * QTtot > 256 || tiles >= (QTtot == 2 ? 400 : 200)) ? 2 : 1, qgroups = ceil_div(QTtot, qt), hb = H * B * qgroups;
    const int nw = hb > 256 ? 4 : 8;
    const bool stream = qgroups == 1;
    a.key_wgs = tiles <= (QTtot == 1 ? 20 : 36) ? 1 : std::max(1, std::min({ceil_div(tiles, QTtot == 1 ? nw : nw * 2), std::max(1, 256 / hb), units_max, (int)SPAN_MERGE_MAX}));
    const dim3 grid(ceil_div(H * B, 8) * 8 * qgroups * a.key_wgs), block(nw * 64);
    const size_t lds = span_lds_bytes(Dh, qt, nw);
#define LAUNCH(DHv, QTv, NWv, STv) \
    if (Dh == DHv && qt == QTv && nw == NWv && stream == STv) hipLaunchKernelGGL((span_attn_kernel<DHv, QTv, NWv, STv>), grid, block, lds, s, a);
    SPAN_EACH(LAUNCH)
#undef LAUNCH
    HYDRA_LAUNCH_CHECK("span_attn_kernel");
    if (a.key_wgs > 1)
        if (int rc = launch_span_merge(c, s, a, slots)) return rc;
    if (!a.score || a.z) return HYDRA_OK;
    const int QS = std::max(1, ceil_div(a.n_scored, 32));                       // 70 nodes, 40 heads (16000): 114 us with three query tiles, 119 with four
    // (twice as many workgroups, with the queries in LDS once more each: a row of 128, 40 heads (16000) 141 us against 134)
    a.key_wgs = std::max(1, std::min(ceil_div(tiles, SCORE_WAVES), std::max(1, 256 / (H * B))));
    const dim3 sgrid(ceil_div(H * B, 8) * 8 * a.key_wgs), sblock(SCORE_WAVES * 64);
    const size_t slds = (size_t)QS * ((Dh / 16) * 1024 + 32 * (4 + sizeof(SpanQuery))) + SCORE_WAVES * 128;
#define LAUNCH(DHv, QSv) if (Dh == DHv && QS == QSv) hipLaunchKernelGGL((span_score_kernel<DHv, QSv>), sgrid, sblock, slds, s, a);
    LAUNCH(128, 1) LAUNCH(128, 2) LAUNCH(128, 3) LAUNCH(128, 4) LAUNCH(64, 1) LAUNCH(64, 2) LAUNCH(64, 3) LAUNCH(64, 4)
#undef LAUNCH
    HYDRA_LAUNCH_CHECK("span_score_kernel");
    return HYDRA_OK;
}

}  // namespace hydra
