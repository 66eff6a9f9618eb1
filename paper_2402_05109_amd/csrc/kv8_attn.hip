// Tree attention behind the 8-bit cache, 16-bit family: the sealed pages of a row are read as codes, its last page and the tree nodes
// from the 16-bit tail.
//
// As in bf16_attn.hip a query is a column of both products, S^T = K Q^T and O^T = V^T P^T, so statistics, masks and rescale factors are
// per-lane scalars.  The scales never touch the tiles: codes become halves exactly, and with s_K, s_V the scales of a key's page and
// c = log2(e) / sqrt(Dh), z the product of codes and query,
//     w = 2^(c s_K z + log2 s_V - M),   O = sum half(w) code_V,   l = sum w / s_V,   result = O / l
// where M is the running maximum of the exponent.  Dequantising both K and V costs one multiply-add per score that the softmax
// needs anyway, and w, the only value that is rounded to 16 bits, is at most 1 whatever the scales are.  A key of the tail has
// s_K = s_V = 1.
//
// A wave holds one or two 32-query tiles and takes 32-key tiles (two pages) in turn.  Tiles go to LDS by the LDS DMA, two of them ahead
// per wave, and from there to registers without a wait for another wave; the waves of a workgroup meet at the end.
#include <algorithm>

#include "attn_bf16.h"
#include "kv8.h"

namespace hydra {

static constexpr float LOG2E = 1.44269504f;

struct TileScale { float k0, k1, v0, v1, r0, r1; };      // of a tile's two pages: c s_K, log2 s_V, 1 / s_V

// Products of one 32-key tile -> weights as the P^T operands of the two pages, the running maximum, and this half-wave's share of the sum.
// The maximum is exact at every tile, so the largest weight is a power of two, 1 in the end, which 16 bits hold: error against 64 bits 2.2e-4 of the
// 2-norm, of which 2.1e-4 is the rounding of the result.  A maximum that may trail by up to 2^8 saves most of the rescaling (16 rows x 64 nodes x 2048 tokens
// 63.6 us instead of 69.9, 32003 tokens 64.3 instead of 67.4), but the largest weights are then rounded too (2.6e-4 to 2.8e-4), and since a wave rescales all of
// its queries when one of them asks, a query's result depends on what the places behind the last query hold.
// The sum takes the weights in 32 bits, as they are before they are rounded: where V is small its page's weights are, and after the rounding
// nothing might be left of them, while the sum divides them by that scale again.
template <int DT>
__device__ __forceinline__ void kv8_softmax(const f32x16_t &z, const TileScale &ts, float &m_run, float &l_run, f32x16_t (&o)[DT], u32x4_t (&pb)[2]) {
    float a = z[0], b = z[8];
#pragma unroll
    for (int v = 1; v < 8; ++v) { a = fmaxf(a, z[v]); b = fmaxf(b, z[8 + v]); }
    float top = fmaxf(fmaf(a, ts.k0, ts.v0), fmaf(b, ts.k1, ts.v1));
    const HalfWaves h = half_waves(top);
    top = fmaxf(h.lo, h.hi);
    if (__any(top > m_run)) {
        const float m_new = fmaxf(m_run, top);
        const float alpha = m_new == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m_run - m_new);
        m_run = m_new;
        l_run *= alpha;
#pragma unroll
        for (int dt = 0; dt < DT; ++dt)
#pragma unroll
            for (int v = 0; v < 16; ++v) o[dt][v] *= alpha;
    }
    const float ref = m_run == -INFINITY ? 0.f : m_run;
    const float c0 = ts.v0 - ref, c1 = ts.v1 - ref;
    float s0 = 0.f, s1 = 0.f;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        const float a0 = __builtin_amdgcn_exp2f(fmaf(z[2 * w], ts.k0, c0)), a1 = __builtin_amdgcn_exp2f(fmaf(z[2 * w + 1], ts.k0, c0));
        const float b0 = __builtin_amdgcn_exp2f(fmaf(z[8 + 2 * w], ts.k1, c1)), b1 = __builtin_amdgcn_exp2f(fmaf(z[8 + 2 * w + 1], ts.k1, c1));
        s0 += a0; s0 += a1;
        s1 += b0; s1 += b1;
        pb[0][w] = half_pack(a0, a1);
        pb[1][w] = half_pack(b0, b1);
    }
    l_run += s0 * ts.r0 + s1 * ts.r1;
}

struct Kv8Args {
    const u32x4_t *q;
    const uint8_t *kcodes, *vcodes;
    const float *scales;
    const int32_t *table8, *n_sealed;
    const a16_t *kpages, *vpages;
    const int32_t *table16, *seq_len;
    const TreeDev *tree;
    float *apart;
    void *out;
    int32_t *flags;
    int max_pages8, n_pages8, max_pages, n_pages, layer, T, H, groups, key_wgs;
    int plain;                                               // queries and result are half [B, T, H, Dh]; otherwise the packed query buffer and the next GEMM's input
    float c;
};

// 16 bytes of a query: dims d0 .. d0 + 7 of column `col` of a query tile (queries past the last one: zeros, or whatever the packed buffer holds; nobody
// stores their result)
template <int DH>
__device__ __forceinline__ u32x4_t query_piece(const Kv8Args &p, int b, int h, int qtile, int QTtot, int col, int d0) {
    if (!p.plain) return p.q[((((size_t)b * p.H + h) * QTtot + qtile) * (DH / 16) + (d0 >> 4)) * 64 + ((d0 >> 3) & 1) * 32 + col];
    const int query = qtile * 32 + col;
    u32x4_t v = {0u, 0u, 0u, 0u};
    if (query < p.T) v = *reinterpret_cast<const u32x4_t *>(reinterpret_cast<const a16_t *>(p.q) + ((size_t)(b * p.T + query) * p.H + h) * DH + d0);
    return v;
}
// four dims of a result
template <int DH>
__device__ __forceinline__ void store_result(const Kv8Args &p, int m, int h, int dim, float a, float b, float c, float d) {
    a16_t *to = reinterpret_cast<a16_t *>(p.out) + (p.plain ? ((size_t)m * p.H + h) * DH + dim : x_index<true>(m, h * DH + dim, p.H * DH));
    *reinterpret_cast<u32x2_t *>(to) = u32x2_t{f2a_pack(a, b), f2a_pack(c, d)};
}

// queries and tiles, or maxima, sums and O of one query tile
static size_t kv8_lds_bytes(int Dh, int qt, int nw) { return std::max((size_t)qt * Dh * 64 + (size_t)nw * Dh * 128, (size_t)nw * 256 * qt + (size_t)nw * Dh * 128); }

// AUX: cache policy of the K/V requests, 2 = nontemporal
template <int DH, int QT, int NW, int FMT, int AUX>
__global__ __launch_bounds__(NW * 64, 2) void kv8_attn_kernel(Kv8Args p) {
    constexpr int KS = DH / 16, DT = DH / 32, KB = DH / 32, VB = DH / 32, TILE = KB + VB;     // KB, VB: KiB of a tile's K and V codes
    extern __shared__ float lds[];                          // queries [QT][KS], two tiles per wave [NW][2][TILE], of 1 KiB each; later sums
    const int tid = (int)threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int hl = lane >> 5, col = lane & 31;
    const int T = p.T, H = p.H;
    const int QTtot = (T + 31) >> 5, QG = (QTtot + QT - 1) / QT, per = QG * p.key_wgs;
    const int seq = (int)blockIdx.x >> 3;
    const int group = seq / per * 8 + ((int)blockIdx.x & 7), j = seq % per;
    if (group >= p.groups) return;
    const int b = group / H, h = group - b * H, qg = j % QG, key_wg = j / QG;
    const int units = p.key_wgs * NW, unit = key_wg * NW + wave;
    const int32_t *t8 = p.table8 + (size_t)b * p.max_pages8, *t16 = p.table16 + (size_t)b * p.max_pages;
    // ---- trip 1: whatever does not depend on the row's length.  Page ids of this wave's first 32 tiles, a page per lane (the table has max_pages8
    // entries for every row; those past the sealed pages are not used), ancestor masks, queries
    auto page_of = [&](int first) { return 2 * (unit + (first + (lane >> 1)) * units) + (lane & 1); };
    auto page_id = [&](int lp) { return t8[min(lp, p.max_pages8 - 1)]; };
    int ids = page_id(page_of(0));
    uint64_t anc[QT][2];
#pragma unroll
    for (int q = 0; q < QT; ++q) {
        const int query = (qg * QT + q) * 32 + col;
        anc[q][0] = anc[q][1] = 0ull;
        if (query < T) { anc[q][0] = p.tree->anc[query][0]; anc[q][1] = p.tree->anc[query][1]; }
    }
    const int L = p.seq_len[b], ns = p.n_sealed[b];
    // queries to LDS, in the order of the codes: block (i, e) holds, for half-wave hl, dims 32 i + 16 hl + 8 e .. + 7
    u32x4_t *qs = reinterpret_cast<u32x4_t *>(lds);
    constexpr int NQ = (QT * KS + NW - 1) / NW;
    u32x4_t qreg[NQ];
#pragma unroll
    for (int i = 0; i < NQ; ++i) {
        const int q = min(i * NW + wave, QT * KS - 1) / KS, blk = (i * NW + wave) % KS;
        const int qtile = min(qg * QT + q, QTtot - 1);       // a second tile behind the last query: the first one again, which nobody stores
        qreg[i] = query_piece<DH>(p, b, h, qtile, QTtot, col, 32 * (blk >> 1) + 16 * hl + 8 * (blk & 1));
    }
    if (L < 0 || L > p.max_pages * 16 - T || ns < 0 || ns > (L >> 4) || ns > p.max_pages8) {     // uniform over the workgroup
        if (tid == 0 && j == 0 && h == 0) atomicOr(p.flags, FLAG_CAPACITY);
        return;
    }
#pragma unroll
    for (int i = 0; i < NQ; ++i)
        if (i * NW + wave < QT * KS) qs[(i * NW + wave) * 64 + lane] = qreg[i];
    const int total = L + T, n8 = (ns + 1) >> 1, first16 = ns * 16, n16 = (total - first16 + 31) >> 5, row_pages = (total + 15) >> 4;
    const int mine8 = unit < n8 ? (n8 - unit + units - 1) / units : 0;           // this wave's tiles of codes: unit, unit + units, ...
    const int t0 = (unit - n8 % units + units) % units;      // and of the tail, which go on in the same turn: t0, t0 + units, ...
    const bool tail = t0 < n16;
    // pages outside the cache are replaced by page 0 and reported at the end: no branch between a page's number and the loads that it is for
    bool bad = false;
    auto page_in = [&](int page, int n_pages, bool used) {
        const bool good = (unsigned)page < (unsigned)n_pages;
        bad |= used && !good;
        return good ? page : 0;
    };
    int a0, a1;
    auto tail_pages = [&](int t) {                           // the second page may be missing: the first one is then read twice
        const int lp = ns + 2 * t, r0 = t16[min(lp, p.max_pages - 1)], r1 = t16[min(lp + 1, p.max_pages - 1)];
        const bool both = lp + 1 < row_pages;
        a0 = page_in(r0, p.n_pages, t < n16);
        a1 = both ? page_in(r1, p.n_pages, t < n16) : a0;
    };
    tail_pages(t0);

    // ---- trip 2: scales of the 32 tiles, and the first two tiles
    int pgs;
    float pk, pv, pr;
    auto scales_of = [&](int lp) {
        const bool there = lp < ns;
        const int page = page_in(ids, p.n_pages8, there);
        pgs = there ? page : -1;
        const float2 s = reinterpret_cast<const float2 *>(p.scales)[((size_t)p.layer * p.n_pages8 + page) * H + h];
        pk = there ? s.x : 0.f;
        pv = there ? s.y : 0.f;
    };
    auto scales_done = [&] {                                 // a page that is not there: exponent -infinity, weight 0
        pk *= p.c;
        pr = pv > 0.f ? __builtin_amdgcn_rcpf(pv) : 0.f;
        pv = __builtin_amdgcn_logf(pv);
        asm volatile("" : "+v"(pgs), "+v"(pk), "+v"(pv), "+v"(pr));               // awaited here: nothing in the loop waits for an ordinary load
    };
    scales_of(page_of(0));
#pragma unroll
    for (int q = 0; q < QT; ++q) asm volatile("" : "+v"(anc[q][0]), "+v"(anc[q][1]));

    u32x4_t *mine = qs + (QT * KS + wave * 2 * TILE) * 64;
    const uint32_t mine_at = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) void *)mine;
    auto dma = [&](const char *src, int block) {
        __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void *)src,
                                         (__attribute__((address_space(3))) void *)(uintptr_t)(mine_at + (uint32_t)block * 1024u), 16, 0, AUX);
    };
    auto lane_of = [](float v, int l) { return __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(v), l)); };
    auto tile_scale = [&](int it) {
        const int l = 2 * (it & 31);
        return TileScale{lane_of(pk, l), lane_of(pk, l + 1), lane_of(pv, l), lane_of(pv, l + 1), lane_of(pr, l), lane_of(pr, l + 1)};
    };
    auto tail_k = [&](int p0, int p1) {
        return reinterpret_cast<const char *>(p.kpages + kv_block_base(p.layer, p.n_pages, (col >> 4) ? p1 : p0, H, h, DH)) + (hl * 16 + (col & 15)) * 16;
    };
    auto tail_v = [&](int page) { return reinterpret_cast<const char *>(p.vpages + kv_block_base(p.layer, p.n_pages, page, H, h, DH)) + (col * 2 + hl) * 16; };
    // Half of what goes to a slot: K (part 0) or V (part 1) of tile `it` of codes; behind the last of those the first tile of the tail, its K as
    // the next, its V as the one after it (K: 16 DH bytes in each half; V: a page in each half); then one and the same 16 bytes in every lane, so
    // that the number of requests in flight is always the same.
    auto request = [&](int it, int part) {
        const char *a, *c;                                   // first and second half of the KB blocks
        int step = 1024;
        if (it < mine8) {
            const int l = 2 * (it & 31), p0 = max(__builtin_amdgcn_readlane(pgs, l), 0), q1 = __builtin_amdgcn_readlane(pgs, l + 1), p1 = q1 < 0 ? p0 : q1;
            if (part == 0) {
                step = 512;
                a = reinterpret_cast<const char *>(p.kcodes) + kv8_block_base(p.layer, p.n_pages8, (col >> 4) ? p1 : p0, H, h, DH) + (hl * 16 + (col & 15)) * 16;
                c = a + KB / 2 * 512;
            } else {
                a = reinterpret_cast<const char *>(p.vcodes) + kv8_block_base(p.layer, p.n_pages8, p0, H, h, DH) + lane * 16;
                c = reinterpret_cast<const char *>(p.vcodes) + kv8_block_base(p.layer, p.n_pages8, p1, H, h, DH) + lane * 16;
            }
        } else if (tail && it == mine8) {
            step = 512;
            a = tail_k(a0, a1) + part * KB * 512;
            c = a + KB / 2 * 512;
        } else if (tail && it == mine8 + 1) {
            a = tail_v(part ? a1 : a0);
            c = a + KB / 2 * 1024;
        } else {
            step = 0;
            a = c = reinterpret_cast<const char *>(p.kcodes) + kv8_block_base(p.layer, p.n_pages8, 0, H, h, DH);
        }
        const int to = (it & 1) * TILE + part * KB;
#pragma unroll
        for (int i = 0; i < KB; ++i) dma((i < KB / 2 ? a : c) + (i < KB / 2 ? i : i - KB / 2) * step, to + i);
    };
    request(0, 0); request(0, 1); request(1, 0); request(1, 1);
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
    scales_done();
    asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");              // the queries are in LDS; the tiles need not be

    auto scores = [&](int it, f32x16_t (&z)[QT]) {          // S^T of tile `it`, whose K has landed
        const u32x4_t *tile = mine + (it & 1) * TILE * 64 + lane;
#pragma unroll
        for (int q = 0; q < QT; ++q)
#pragma unroll
            for (int v = 0; v < 16; ++v) z[q][v] = 0.f;
        int at = lane;
        asm volatile("" : "+v"(at));                         // keeps the reads of the queries inside the loop
#pragma unroll
        for (int i = 0; i < KB; ++i) {
            const u32x4_t w = tile[i * 64];
            uint32_t k[8];
#pragma unroll
            for (int e = 0; e < 4; ++e) kv8_halves<FMT>(w[e], k[2 * e], k[2 * e + 1]);
            const u32x4_t ka = {k[0], k[1], k[2], k[3]}, kb = {k[4], k[5], k[6], k[7]};
#pragma unroll
            for (int q = 0; q < QT; ++q) {
                z[q] = HYDRA_MFMA16(__builtin_bit_cast(a16x8_t, ka), __builtin_bit_cast(a16x8_t, qs[at + (q * KS + 2 * i) * 64]), z[q]);
                z[q] = HYDRA_MFMA16(__builtin_bit_cast(a16x8_t, kb), __builtin_bit_cast(a16x8_t, qs[at + (q * KS + 2 * i + 1) * 64]), z[q]);
            }
        }
    };
    auto values = [&](int it, const u32x4_t (&pb)[QT][2]) { // O^T += V^T P^T of tile `it`, whose V has landed
        const u32x4_t *tile = mine + ((it & 1) * TILE + KB) * 64 + lane;
#pragma unroll
        for (int g = 0; g < 2; ++g)
#pragma unroll
            for (int i = 0; i < VB / 2; ++i) {
                const u32x4_t w = tile[(g * (VB / 2) + i) * 64];
                uint32_t v[8];
#pragma unroll
                for (int e = 0; e < 4; ++e) kv8_halves<FMT>(w[e], v[2 * e], v[2 * e + 1]);
                const u32x4_t va = {v[0], v[1], v[2], v[3]}, vb = {v[4], v[5], v[6], v[7]};
#pragma unroll
                for (int q = 0; q < QT; ++q) {
                    o[q][2 * i] = HYDRA_MFMA16(__builtin_bit_cast(a16x8_t, va), __builtin_bit_cast(a16x8_t, pb[q][g]), o[q][2 * i]);
                    o[q][2 * i + 1] = HYDRA_MFMA16(__builtin_bit_cast(a16x8_t, vb), __builtin_bit_cast(a16x8_t, pb[q][g]), o[q][2 * i + 1]);
                }
            }
    };
    auto new_pages = [&](int it) {                           // tile `it` is the first of another 32: the loads of their pages end every wait
        if ((it & 31) == 0 && it < mine8) {
            ids = page_id(page_of(it));
            scales_of(page_of(it));
            scales_done();
        }
    };
    TileScale ts = tile_scale(0), next = tile_scale(1);
    for (int it = 0; it < mine8; ++it) {
        asm volatile("s_waitcnt vmcnt(%0)" ::"n"(VB + TILE) : "memory");      // K has landed: younger are its V and the next tile
        f32x16_t z[QT];
        u32x4_t pb[QT][2];
        scores(it, z);
        new_pages(it + 2);
        const TileScale after = tile_scale(it + 2);
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");                    // K is read
        request(it + 2, 0);
#pragma unroll
        for (int q = 0; q < QT; ++q) kv8_softmax<DT>(z[q], ts, m_run[q], l_run[q], o[q], pb[q]);
        asm volatile("s_waitcnt vmcnt(%0)" ::"n"(TILE + KB) : "memory");      // V has landed: younger are the next tile and another K
        values(it, pb);
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");                    // V is read
        request(it + 2, 1);
        ts = next;
        next = after;
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");         // the tail's first tile, or what was requested past the last one, has landed

    // ---- the 16-bit tail: K in one slot, V in the other
    const TileScale one = {p.c, p.c, 0.f, 0.f, 1.f, 1.f};
    for (int t = t0, sk = mine8 & 1; t < n16; t += units) {
        if (t != t0) {                                       // a row with many pages that are not sealed
            tail_pages(t);
            const char *kp = tail_k(a0, a1), *v0 = tail_v(a0), *v1 = tail_v(a1);
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");                    // the tile before this one is read
#pragma unroll
            for (int s = 0; s < KS; ++s) dma(kp + s * 512, sk * TILE + s);
#pragma unroll
            for (int i = 0; i < DT; ++i) { dma(v0 + i * 1024, (sk ^ 1) * TILE + i); dma(v1 + i * 1024, (sk ^ 1) * TILE + DT + i); }
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        }
        const int slot0 = first16 + t * 32;
        const u32x4_t *kt = mine + sk * TILE * 64 + lane, *vt = mine + (sk ^ 1) * TILE * 64 + lane;
        f32x16_t z[QT];
        u32x4_t pb[QT][2];
#pragma unroll
        for (int q = 0; q < QT; ++q)
#pragma unroll
            for (int v = 0; v < 16; ++v) z[q][v] = 0.f;
#pragma unroll
        for (int s = 0; s < KS; ++s) {                       // 16-bit K has dims 16 s + 8 hl in step s: block (s / 2, e = hl), its half-wave s % 2
            const a16x8_t k = __builtin_bit_cast(a16x8_t, kt[s * 64]);
#pragma unroll
            for (int q = 0; q < QT; ++q)
                z[q] = HYDRA_MFMA16(k, __builtin_bit_cast(a16x8_t, qs[(q * KS + (s & ~1) + hl) * 64 + (s & 1) * 32 + col]), z[q]);
        }
#pragma unroll
        for (int q = 0; q < QT; ++q) {
            const uint32_t seen = keys_seen(slot0, L, anc[q][0], anc[q][1]) >> (4 * hl);
#pragma unroll
            for (int v = 0; v < 16; ++v) z[q][v] = (seen >> (8 * (v >> 2) + (v & 3))) & 1u ? z[q][v] : -INFINITY;
            kv8_softmax<DT>(z[q], one, m_run[q], l_run[q], o[q], pb[q]);
        }
#pragma unroll
        for (int g = 0; g < 2; ++g) {
            u32x4_t keep;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                // dword e holds keys i = 2e, 2e+1 of this half-wave: token = 8*(i/4) + 4*hl + i%4.  V of slots past the last node becomes 0: stale contents
                const int i0 = 2 * e, i1 = 2 * e + 1;
                const int s0 = slot0 + 16 * g + 8 * (i0 >> 2) + 4 * hl + (i0 & 3);
                const int s1 = slot0 + 16 * g + 8 * (i1 >> 2) + 4 * hl + (i1 & 3);
                keep[e] = (s0 < total ? 0x0000ffffu : 0u) | (s1 < total ? 0xffff0000u : 0u);
            }
#pragma unroll
            for (int dt = 0; dt < DT; ++dt) {
                const a16x8_t v = __builtin_bit_cast(a16x8_t, vt[(g * DT + dt) * 64] & keep);
#pragma unroll
                for (int q = 0; q < QT; ++q) o[q][dt] = HYDRA_MFMA16(v, __builtin_bit_cast(a16x8_t, pb[q][g]), o[q][dt]);
            }
        }
    }

    if (__any(bad) && lane == 0) atomicOr(p.flags, FLAG_BAD_PAGE);

    // ---- merge the waves through LDS, one query tile after the other: maxima and sums [QT][NW][2][32], then O[NW][DT * 4][64] of four dims each
    __syncthreads();                                         // every wave is done with queries and tiles
    float *ml = lds;
    f32x4_t *ob = reinterpret_cast<f32x4_t *>(lds + QT * NW * 64);
#pragma unroll
    for (int q = 0; q < QT; ++q) {
        const HalfWaves lh = half_waves(l_run[q]);           // each half-wave has summed its own keys
        if (hl == 0) {
            ml[(q * NW + wave) * 64 + col] = m_run[q];
            ml[(q * NW + wave) * 64 + 32 + col] = lh.lo + lh.hi;
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
        for (int w = 0; w < NW; ++w) l_tot += __builtin_amdgcn_exp2f(mq[w * 64 + col] - m_safe) * mq[w * 64 + 32 + col];
        const float f = __builtin_amdgcn_exp2f(m_run[q] - m_safe);
#pragma unroll
        for (int id = 0; id < DT * 4; ++id) {
            const f32x16_t &od = o[q][id >> 2];
            const int v = 4 * (id & 3);
            ob[(wave * DT * 4 + id) * 64 + lane] = f32x4_t{od[v] * f, od[v + 1] * f, od[v + 2] * f, od[v + 3] * f};
        }
        __syncthreads();
        // the (band, group of 4 registers = 4 consecutive dims) items are shared out over the waves
        const float inv = p.key_wgs == 1 ? 1.0f / l_tot : 1.0f;
        for (int id = wave; id < DT * 4; id += NW) {
            const int dt = id >> 2, g4 = id & 3;
            f32x4_t acc = ob[id * 64 + lane];
#pragma unroll
            for (int w = 1; w < NW; ++w) acc += ob[(w * DT * 4 + id) * 64 + lane];
            const int dim = 32 * dt + 8 * g4 + 4 * hl, m = b * T + query;
            if (p.key_wgs > 1) {
                *reinterpret_cast<f32x4_t *>(rec + (size_t)query * DH + dim) = acc;
            } else if (query < T) {
                store_result<DH>(p, m, h, dim, acc[0] * inv, acc[1] * inv, acc[2] * inv, acc[3] * inv);
            }
        }
        if (p.key_wgs > 1 && wave == 0 && hl == 0) {
            rec[(size_t)Tq * DH + query] = m_tot;
            rec[(size_t)Tq * DH + Tq + query] = l_tot;
        }
        if (q + 1 < QT) __syncthreads();                     // the next query tile's sums go where these were
    }
}

// Short contexts: a workgroup takes one 32-query tile of one (row, head) and 1 / DS of the head's dims, its eight waves split the keys and meet in LDS,
// and the result goes straight out.  A chain of round trips, so everything that can be is requested at once: the page ids before the length
// is known, then all tiles of a wave (20 registers each with DS = 4) and the first tile of its tail.
enum { KV8_SHORT_WAVES = 8 };
template <int DH, int DS>
struct Short8 { u32x4_t k[DH / 32]; uint32_t v[2][DH / DS / 16]; };       // V: 8 bytes for each 32 dims of a page

template <int DH, int DS>
struct ShortTail { u32x4_t k[DH / 16]; u32x4_t v[2][DH / 32 / DS]; };

static size_t kv8_short_lds_bytes(int Dh, int ds) {
    return ((size_t)KV8_SHORT_WAVES * 64 + std::max((size_t)KV8_SHORT_WAVES * (Dh / 32 / ds) * 16 * 64, (size_t)Dh * 16)) * 4;       // O, or the query tile
}

template <int DH, int DS, int FMT>
__global__ __launch_bounds__(KV8_SHORT_WAVES * 64, 2) void kv8_short_kernel(Kv8Args p) {
    constexpr int KS = DH / 16, KB = DH / 32, DT = DH / 32 / DS, NW = KV8_SHORT_WAVES, RING = DT == 4 ? 2 : 4;
    extern __shared__ float lds[];                          // [NW][2][32] maxima and sums, then the query tile and later O[NW][DT * 16][64]
    const int tid = (int)threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int hl = lane >> 5, col = lane & 31;
    const int T = p.T, H = p.H;
    const int QTtot = (T + 31) >> 5, per = QTtot * DS;
    const int seq = (int)blockIdx.x >> 3;
    const int group = seq / per * 8 + ((int)blockIdx.x & 7), j = seq % per;
    if (group >= p.groups) return;
    const int b = group / H, h = group - b * H, qtile = j / DS, ds = j % DS;
    const int32_t *t8 = p.table8 + (size_t)b * p.max_pages8, *t16 = p.table16 + (size_t)b * p.max_pages;
    u32x4_t *qs = reinterpret_cast<u32x4_t *>(lds + NW * 64);
    const int query = qtile * 32 + col;
    uint64_t anc0 = 0ull, anc1 = 0ull;
    if (query < T) { anc0 = p.tree->anc[query][0]; anc1 = p.tree->anc[query][1]; }
    int pg[RING][2];                                        // the table has max_pages8 entries for every row; those past the sealed pages are not used
#pragma unroll
    for (int i = 0; i < RING; ++i) {
        const int t = wave + i * NW;
        pg[i][0] = t8[min(2 * t, p.max_pages8 - 1)];
        pg[i][1] = t8[min(2 * t + 1, p.max_pages8 - 1)];
    }
    const int L = p.seq_len[b], ns = p.n_sealed[b];
    if (wave < KS) qs[wave * 64 + lane] = query_piece<DH>(p, b, h, qtile, QTtot, col, 32 * (wave >> 1) + 16 * hl + 8 * (wave & 1));
    if (L < 0 || L > p.max_pages * 16 - T || ns < 0 || ns > (L >> 4) || ns > p.max_pages8) {     // uniform over the workgroup
        if (tid == 0 && j == 0 && h == 0) atomicOr(p.flags, FLAG_CAPACITY);
        return;
    }
    const int total = L + T, n8 = (ns + 1) >> 1, first16 = ns * 16, n16 = (total - first16 + 31) >> 5, row_pages = (total + 15) >> 4;
    const int mine8 = wave < n8 ? (n8 - wave + NW - 1) / NW : 0;               // tiles of codes wave, wave + NW, ...; the tail's go on in the same turn
    const int t0 = (wave - n8 % NW + NW) % NW;
    const bool tail = t0 < n16;

    // Loads are never behind a condition: a tile past the last one reads one and the same piece of page 0 in every lane.
    auto load8 = [&](Short8<DH, DS> &kv, TileScale &ts, int it, int p0, int p1) {
        const int t = wave + it * NW;
        const bool live = t < n8, both = 2 * t + 1 < ns;
        p0 = live ? checked_page(p0, p.n_pages8, p.flags) : 0;
        p1 = both ? checked_page(p1, p.n_pages8, p.flags) : p0;
        const int ln = live ? lane : 0, lh = ln >> 5, lc = ln & 31;
        const float2 *sc = reinterpret_cast<const float2 *>(p.scales);
        const float2 s0 = sc[((size_t)p.layer * p.n_pages8 + p0) * H + h], s1 = sc[((size_t)p.layer * p.n_pages8 + p1) * H + h];
        ts.k0 = s0.x; ts.k1 = s1.x; ts.v0 = s0.y; ts.v1 = s1.y;                // raw; see scale8
        const uint8_t *kp = p.kcodes + kv8_block_base(p.layer, p.n_pages8, (lc >> 4) ? p1 : p0, H, h, DH) + (lh * 16 + (lc & 15)) * 16;
#pragma unroll
        for (int i = 0; i < KB; ++i) kv.k[i] = *reinterpret_cast<const u32x4_t *>(kp + i * 512);
#pragma unroll
        for (int g = 0; g < 2; ++g) {
            const uint8_t *vp = p.vcodes + kv8_block_base(p.layer, p.n_pages8, g ? p1 : p0, H, h, DH) + ln * 16;
#pragma unroll
            for (int dt = 0; dt < DT; ++dt) {
                const int d = ds * DT + dt;                  // (the 32 dims' place in the head)
                const u32x2_t w = *reinterpret_cast<const u32x2_t *>(vp + (d >> 1) * 1024 + (d & 1) * 8);
                kv.v[g][2 * dt] = w[0]; kv.v[g][2 * dt + 1] = w[1];
            }
        }
    };
    auto scale8 = [&](TileScale &ts, int it) {
        const bool both = 2 * (wave + it * NW) + 1 < ns;     // a page that is not there: exponent -infinity, weight 0
        const float v0 = ts.v0, v1 = ts.v1;
        ts.k0 *= p.c;
        ts.v0 = __builtin_amdgcn_logf(v0);
        ts.r0 = __builtin_amdgcn_rcpf(v0);
        ts.k1 = both ? ts.k1 * p.c : 0.f;
        ts.v1 = both ? __builtin_amdgcn_logf(v1) : -INFINITY;
        ts.r1 = both ? __builtin_amdgcn_rcpf(v1) : 0.f;
    };
    f32x16_t o[DT];
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
        for (int v = 0; v < 16; ++v) o[dt][v] = 0.f;
    float m_run = -INFINITY, l_run = 0.f;
    auto step8 = [&](const Short8<DH, DS> &kv, TileScale ts, int it) {
        f32x16_t z;
#pragma unroll
        for (int v = 0; v < 16; ++v) z[v] = 0.f;
        int at = lane;
        asm volatile("" : "+v"(at));                         // keeps the reads of the queries here (hoisted, they are registers)
#pragma unroll
        for (int i = 0; i < KB; ++i) {
            uint32_t k[8];
#pragma unroll
            for (int e = 0; e < 4; ++e) kv8_halves<FMT>(kv.k[i][e], k[2 * e], k[2 * e + 1]);
            const u32x4_t ka = {k[0], k[1], k[2], k[3]}, kb = {k[4], k[5], k[6], k[7]};
            z = HYDRA_MFMA16(__builtin_bit_cast(a16x8_t, ka), __builtin_bit_cast(a16x8_t, qs[at + 2 * i * 64]), z);
            z = HYDRA_MFMA16(__builtin_bit_cast(a16x8_t, kb), __builtin_bit_cast(a16x8_t, qs[at + (2 * i + 1) * 64]), z);
        }
        scale8(ts, it);
        u32x4_t pb[2];
        kv8_softmax<DT>(z, ts, m_run, l_run, o, pb);
#pragma unroll
        for (int g = 0; g < 2; ++g) {
#pragma unroll
            for (int dt = 0; dt < DT; ++dt) {
                uint32_t v[4];
                kv8_halves<FMT>(kv.v[g][2 * dt], v[0], v[1]);
                kv8_halves<FMT>(kv.v[g][2 * dt + 1], v[2], v[3]);
                const u32x4_t va = {v[0], v[1], v[2], v[3]};
                o[dt] = HYDRA_MFMA16(__builtin_bit_cast(a16x8_t, va), __builtin_bit_cast(a16x8_t, pb[g]), o[dt]);
            }
        }
    };
    // the 16-bit tail
    auto load16 = [&](ShortTail<DH, DS> &kv, int t, int p0, int p1, bool live) {
        p0 = live ? checked_page(p0, p.n_pages, p.flags) : 0;
        p1 = live && ns + 2 * t + 1 < row_pages ? checked_page(p1, p.n_pages, p.flags) : p0;
        const int ln = live ? lane : 0, lh = ln >> 5, lc = ln & 31;
        const u32x4_t *kp = reinterpret_cast<const u32x4_t *>(p.kpages + kv_block_base(p.layer, p.n_pages, (lc >> 4) ? p1 : p0, H, h, DH)) + lh * 16 + (lc & 15);
#pragma unroll
        for (int s = 0; s < KS; ++s) kv.k[s] = kp[s * 32];
#pragma unroll
        for (int g = 0; g < 2; ++g) {
            const u32x4_t *vp = reinterpret_cast<const u32x4_t *>(p.vpages + kv_block_base(p.layer, p.n_pages, g ? p1 : p0, H, h, DH)) + lc * 2 + lh;
#pragma unroll
            for (int dt = 0; dt < DT; ++dt) kv.v[g][dt] = vp[(ds * DT + dt) * 64];
        }
    };
    auto step16 = [&](ShortTail<DH, DS> &kv, int t) {
        const TileScale one = {p.c, p.c, 0.f, 0.f, 1.f, 1.f};
        const int slot0 = first16 + t * 32;
        f32x16_t z;
#pragma unroll
        for (int v = 0; v < 16; ++v) z[v] = 0.f;
#pragma unroll
        for (int s = 0; s < KS; ++s)                         // 16-bit K has dims 16 s + 8 hl in step s: block (s / 2, e = hl), its half-wave s % 2
            z = HYDRA_MFMA16(__builtin_bit_cast(a16x8_t, kv.k[s]), __builtin_bit_cast(a16x8_t, qs[((s & ~1) + hl) * 64 + (s & 1) * 32 + col]), z);
        const uint32_t seen = keys_seen(slot0, L, anc0, anc1) >> (4 * hl);
#pragma unroll
        for (int v = 0; v < 16; ++v) z[v] = (seen >> (8 * (v >> 2) + (v & 3))) & 1u ? z[v] : -INFINITY;
        u32x4_t pb[2];
        kv8_softmax<DT>(z, one, m_run, l_run, o, pb);
#pragma unroll
        for (int g = 0; g < 2; ++g) {
            u32x4_t keep;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                // dword e holds keys i = 2e, 2e+1 of this half-wave: token = 8*(i/4) + 4*hl + i%4.  V of slots past the last node becomes 0: stale contents
                const int i0 = 2 * e, i1 = 2 * e + 1;
                const int s0 = slot0 + 16 * g + 8 * (i0 >> 2) + 4 * hl + (i0 & 3);
                const int s1 = slot0 + 16 * g + 8 * (i1 >> 2) + 4 * hl + (i1 & 3);
                keep[e] = (s0 < total ? 0x0000ffffu : 0u) | (s1 < total ? 0xffff0000u : 0u);
            }
#pragma unroll
            for (int dt = 0; dt < DT; ++dt)
                o[dt] = HYDRA_MFMA16(__builtin_bit_cast(a16x8_t, kv.v[g][dt] & keep), __builtin_bit_cast(a16x8_t, pb[g]), o[dt]);
        }
    };
    const int lp0 = ns + 2 * t0;
    const int a0 = t16[min(lp0, p.max_pages - 1)], a1 = t16[min(lp0 + 1, p.max_pages - 1)];
    Short8<DH, DS> ring[RING];
    TileScale rs[RING];
#pragma unroll
    for (int i = 0; i < RING; ++i) load8(ring[i], rs[i], i, pg[i][0], pg[i][1]);
    ShortTail<DH, DS> last;
    load16(last, t0, a0, a1, tail);
    __syncthreads();                                         // the query tile is in LDS
    int it = 0;
    for (; it + RING < mine8; it += RING)                    // all of the ring's tiles exist
#pragma unroll
        for (int i = 0; i < RING; ++i) {
            const int next = it + i + RING, t = wave + next * NW;
            const int p0 = t8[min(2 * t, p.max_pages8 - 1)], p1 = t8[min(2 * t + 1, p.max_pages8 - 1)];
            step8(ring[i], rs[i], it + i);
            load8(ring[i], rs[i], next, p0, p1);
        }
#pragma unroll
    for (int i = 0; i < RING; ++i)
        if (it + i < mine8) step8(ring[i], rs[i], it + i);
    if (tail) step16(last, t0);
    for (int t = t0 + NW; t < n16; t += NW) {                // a row with many pages that are not sealed
        const int lp = ns + 2 * t;
        load16(last, t, t16[lp], t16[min(lp + 1, p.max_pages - 1)], true);
        step16(last, t);
    }

    // ---- merge the waves through LDS: ml[NW][2][32], then O[NW][DT * 4][64] of four dims each where the queries were
    float *ml = lds;
    f32x4_t *ob = reinterpret_cast<f32x4_t *>(lds + NW * 64);
    const HalfWaves lh2 = half_waves(l_run);                 // each half-wave has summed its own keys
    if (hl == 0) {
        ml[(wave * 2 + 0) * 32 + col] = m_run;
        ml[(wave * 2 + 1) * 32 + col] = lh2.lo + lh2.hi;
    }
    __syncthreads();
    float m_tot = -INFINITY;
#pragma unroll
    for (int w = 0; w < NW; ++w) m_tot = fmaxf(m_tot, ml[(w * 2 + 0) * 32 + col]);
    const float m_safe = m_tot == -INFINITY ? 0.f : m_tot;
    float l_tot = 0.f;
#pragma unroll
    for (int w = 0; w < NW; ++w) l_tot += __builtin_amdgcn_exp2f(ml[(w * 2 + 0) * 32 + col] - m_safe) * ml[(w * 2 + 1) * 32 + col];
    const float f = __builtin_amdgcn_exp2f(m_run - m_safe);
#pragma unroll
    for (int id = 0; id < DT * 4; ++id) {
        const f32x16_t &od = o[id >> 2];
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
        if (query < T) store_result<DH>(p, b * T + query, h, 32 * (ds * DT + dt) + 8 * g4 + 4 * hl, acc[0] * inv, acc[1] * inv, acc[2] * inv, acc[3] * inv);
    }
}

// out = sum_u 2^(M_u - M) O_u / sum_u 2^(M_u - M) l_u over the records of a head: one thread per (query, 4 dims), all its loads in one round trip.
enum { KV8_MERGE_MAX = 16 };
__global__ __launch_bounds__(256) void kv8_merge_kernel(const float *__restrict__ apart, const int32_t *__restrict__ seq_len, const int32_t *__restrict__ n_sealed,
                                                         int T, int H, int Dh, int units, int max_pages, int max_pages8, int plain, void *out) {
    const int h = blockIdx.y, b = blockIdx.z;
    const int per_q = Dh >> 2;
    const int n = blockIdx.x * (256 / per_q) + threadIdx.x / per_q;
    const int dim = (threadIdx.x % per_q) * 4;
    const int Tq = ((T + 31) >> 5) * 32;
    const size_t recsz = apart_record(Tq, Dh);
    const float *base = apart + (((size_t)b * H + h) * units) * recsz;
    const bool live = n < T;
    float mu[KV8_MERGE_MAX], lu[KV8_MERGE_MAX];
    f32x4_t ou[KV8_MERGE_MAX];
#pragma unroll
    for (int u = 0; u < KV8_MERGE_MAX; ++u) {
        mu[u] = -INFINITY; lu[u] = 0.f; ou[u] = f32x4_t{0.f, 0.f, 0.f, 0.f};
        if (u < units && live) {
            const float *r = base + u * recsz;
            mu[u] = r[(size_t)Tq * Dh + n];
            lu[u] = r[(size_t)Tq * Dh + Tq + n];
            ou[u] = *reinterpret_cast<const f32x4_t *>(r + (size_t)n * Dh + dim);
        }
    }
    const int L = seq_len[b], ns = n_sealed[b];
    if (L < 0 || L > max_pages * 16 - T || ns < 0 || ns > (L >> 4) || ns > max_pages8 || !live) return;
    float mt = -INFINITY;
#pragma unroll
    for (int u = 0; u < KV8_MERGE_MAX; ++u) mt = fmaxf(mt, mu[u]);
    float den = 0.f;
    f32x4_t acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int u = 0; u < KV8_MERGE_MAX; ++u) {
        const float w = u < units ? __builtin_amdgcn_exp2f(mu[u] - mt) : 0.f;
        den += w * lu[u];
        acc += ou[u] * w;
    }
    const float inv = 1.0f / den;
    const int m = b * T + n;
    const u32x2_t pk = {f2a_pack(acc[0] * inv, acc[1] * inv), f2a_pack(acc[2] * inv, acc[3] * inv)};
    a16_t *to = reinterpret_cast<a16_t *>(out) + (plain ? ((size_t)m * H + h) * Dh + dim : x_index<true>(m, h * Dh + dim, H * Dh));
    *reinterpret_cast<u32x2_t *>(to) = pk;
}

// (query tiles of a wave, waves, request policy) that the rules below choose from
#define KV8_EACH_OF(X, DHv, Fv) X(DHv, 1, 8, Fv, 0) X(DHv, 1, 4, Fv, 2) X(DHv, 2, 8, Fv, 0) X(DHv, 2, 8, Fv, 2) X(DHv, 2, 4, Fv, 0) X(DHv, 2, 4, Fv, 2)
#define KV8_EACH(X)                                                                                                                     \
    KV8_EACH_OF(X, 128, KV8_INT8) KV8_EACH_OF(X, 128, KV8_E4M3) KV8_EACH_OF(X, 64, KV8_INT8) KV8_EACH_OF(X, 64, KV8_E4M3)               \
    X(64, 1, 8, KV8_INT8, 2) X(64, 1, 8, KV8_E4M3, 2)
#define KV8_SHORT_EACH(X)                                                                                                               \
    X(128, 1, KV8_INT8) X(128, 2, KV8_INT8) X(128, 4, KV8_INT8) X(128, 1, KV8_E4M3) X(128, 2, KV8_E4M3) X(128, 4, KV8_E4M3)             \
    X(64, 1, KV8_INT8) X(64, 2, KV8_INT8) X(64, 1, KV8_E4M3) X(64, 2, KV8_E4M3)

int kv8_max_dynamic_lds() {
    hipError_t e = hipSuccess;
#define ATTR(DHv, QTv, NWv, Fv, AUXv) \
    if (e == hipSuccess) e = hipFuncSetAttribute((const void *)kv8_attn_kernel<DHv, QTv, NWv, Fv, AUXv>, hipFuncAttributeMaxDynamicSharedMemorySize, 160 * 1024);
    KV8_EACH(ATTR)
#undef ATTR
#define ATTR(DHv, DSv, Fv) \
    if (e == hipSuccess) e = hipFuncSetAttribute((const void *)kv8_short_kernel<DHv, DSv, Fv>, hipFuncAttributeMaxDynamicSharedMemorySize, 160 * 1024);
    KV8_SHORT_EACH(ATTR)
#undef ATTR
    if (e != hipSuccess) return hip_fail(e, "hipFuncSetAttribute(8-bit attention kernels)");
    return HYDRA_OK;
}

int launch_kv8_attention(hydra_ctx *c, hipStream_t s, int B, int layer, const void *q, bool plain, const int32_t *seq_len, const hydra_kv8 *kv,
                         float *apart, int units_max, void *out, int32_t *flags) {
    const int T = c->tree.T, H = c->m.n_heads, Dh = c->m.head_dim;
    const int QTtot = ceil_div(T, 32);
    const int len = kv->tail.seq_len_hint > 0 ? kv->tail.seq_len_hint : c->m.max_pos;
    const int tiles = ceil_div(len + T, 32) + 1;
    Kv8Args a;
    a.q = (const u32x4_t *)q; a.kcodes = (const uint8_t *)kv->k_codes; a.vcodes = (const uint8_t *)kv->v_codes; a.scales = kv->scales;
    a.table8 = kv->page_table; a.n_sealed = kv->n_sealed; a.kpages = (const a16_t *)kv->tail.k_pages; a.vpages = (const a16_t *)kv->tail.v_pages;
    a.table16 = kv->tail.page_table; a.seq_len = seq_len; a.tree = tree_dev(c); a.apart = apart; a.out = out; a.flags = flags;
    a.max_pages8 = kv->max_pages; a.n_pages8 = kv->n_pages; a.max_pages = kv->tail.max_pages; a.n_pages = kv->tail.n_pages; a.layer = layer;
    a.T = T; a.H = H; a.groups = H * B; a.plain = plain ? 1 : 0; a.c = LOG2E / sqrtf((float)Dh);
    // Short contexts, while a workgroup per (row, head, 32-query tile) fits one round of the chip: no records and no merge, and the head's dims shared out over
    // more workgroups while those fit the round too (us: 64 nodes behind 777 tokens, 32 heads 10.0 / 10.2 / 11.6 with 4 / 2 / 1 shares, 13.0 with records
    // and merge; 4 rows of it 14.8 against 14.6; beyond one round 16 rows of 400 tokens 38.5 against 25.4).  Up to 36 key tiles (one node, 32 heads,
    // 701 / 1100 / 1250 / 2000 tokens 8.7 / 10.7 / 12.3 / 15.3 against 9.8 / 10.8 / 11.0 / 11.9), 56 with more than one query tile (64 nodes, 1300 / 1650 / 2000 tokens
    // 13.7 / 15.7 / 16.9 against 13.9 / 14.5 / 15.0; 2 rows of 1500 16.5 against 17.7; 128 nodes, 1650 tokens 17.3 against 18.1).
    if (tiles <= (QTtot > 1 ? 56 : 36) && QTtot * H * B <= 256) {
        int ds = Dh / 32;
        while (ds > 1 && QTtot * H * B * ds > 256) ds >>= 1;
        a.key_wgs = 1;
        const dim3 grid(ceil_div(H * B, 8) * 8 * QTtot * ds), block(KV8_SHORT_WAVES * 64);
#define LAUNCH(DHv, DSv, Fv) \
        if (Dh == DHv && ds == DSv && kv->format == Fv) hipLaunchKernelGGL((kv8_short_kernel<DHv, DSv, Fv>), grid, block, kv8_short_lds_bytes(DHv, DSv), s, a);
        KV8_SHORT_EACH(LAUNCH)
#undef LAUNCH
        HYDRA_LAUNCH_CHECK("kv8_short_kernel");
        return HYDRA_OK;
    }
    // Beyond that the keys of a head are split over waves and, while the chip has room, over workgroups.
    //   query tiles of a wave: one while a workgroup for each fits one round (a tile then takes half as long and K/V come from L2 the second time: 64
    //     nodes, 32 heads, 2000 / 8000 tokens 15.2 / 27.2 us against 20.3 / 29.4, 4 rows of 2048 24.2 against 30.1), two beyond (16 rows of 2048 69.5
    //     against 81.8)
    //   waves of a workgroup: eight; four with more (row, head, query group)s than CUs, two or more workgroups to a CU, so that one's first
    //     round trips and merge lie under another's stream (16 rows of 2048 67.6 against 79.2; 8 rows of 128 nodes 61.7 against 70.9), and for up to 32 nodes with
    //     128 dims (32003 tokens, 40 heads 59.1 against 61.9; 8000 tokens 21.3 against 21.6; with 64 dims 16.2 against 15.1)
    const int qt = QTtot > 1 && H * B * QTtot > 256 ? 2 : 1, qgroups = ceil_div(QTtot, qt), hb = H * B * qgroups;
    const int nw = hb > 256 || (Dh == 128 && QTtot == 1) ? 4 : 8;
    const int wgs = std::max(1, std::min({ceil_div(tiles, nw * 2), std::max(1, 256 / hb), units_max, (int)KV8_MERGE_MAX}));
    a.key_wgs = wgs;
    // K and V that one workgroup alone reads are requested nontemporal (32003 tokens 62.0 -> 58.3 us, 16 rows of 2048 and 32 nodes 60.7 -> 57.6)
    const int aux = qgroups == 1 ? 2 : 0;
    const dim3 grid(ceil_div(H * B, 8) * 8 * qgroups * wgs), block(nw * 64);
    const size_t lds = kv8_lds_bytes(Dh, qt, nw);
#define LAUNCH(DHv, QTv, NWv, Fv, AUXv) \
    if (Dh == DHv && qt == QTv && nw == NWv && kv->format == Fv && aux == AUXv) hipLaunchKernelGGL((kv8_attn_kernel<DHv, QTv, NWv, Fv, AUXv>), grid, block, lds, s, a);
    KV8_EACH(LAUNCH)
#undef LAUNCH
    HYDRA_LAUNCH_CHECK("kv8_attn_kernel");
    if (wgs > 1) {
        const dim3 mgrid(ceil_div(T, 256 / (Dh / 4)), H, B), mblock(256);
        hipLaunchKernelGGL(kv8_merge_kernel, mgrid, mblock, 0, s, apart, seq_len, kv->n_sealed, T, H, Dh, wgs, kv->tail.max_pages, kv->max_pages, a.plain, out);
        HYDRA_LAUNCH_CHECK("kv8_merge_kernel");
    }
    return HYDRA_OK;
}

}  // namespace hydra
