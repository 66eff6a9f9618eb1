// Tree attention behind the 8-bit cache, 16-bit family: the sealed pages of a row are read as codes, its last page and the tree nodes
// from the 16-bit tail.
//
// As in bf16_attn.hip a query is a column of both products, S^T = K Q^T and O^T = V^T P^T, so statistics, masks and rescale factors are
// per-lane scalars.  The scales never touch the tiles: codes become halves exactly, and with s_K, s_V the scales of a key's page and
// c = log2(e) / sqrt(Dh), z the product of codes and query,
//     w = 2^(c s_K z + log2 s_V - M),   O = sum half(w) code_V,   l = sum w / s_V,   result = O / l
// where M is the running maximum of the exponent.  Dequantising both K and V costs one multiply-add per score that the softmax
// needs anyway, and w, the only value that is rounded to 16 bits, is at most one whatever the scales are.  A key of the tail has
// s_K = s_V = 1.
//
// A wave holds one or two 32-query tiles and takes 32-key tiles (two pages) in turn.  Tiles go to LDS by the LDS DMA, two of them ahead
// per wave, and from there to registers without a wait for another wave; the waves of a workgroup meet at the end.
#include <algorithm>

#include "attn_bf16.h"
#include "kv8.h"

namespace hydra {

static constexpr float LOG2E = 1.44269504f;

// Exponents of one 32-key tile -> weights, in place, the running maximum and the lane's share of the sum (its two pages apart).
struct TileScale { float k0, k1, v0, v1, r0, r1; };      // of its two pages: c s_K, log2 s_V, 1 / s_V
template <int DT>
__device__ __forceinline__ void kv8_softmax(f32x16_t &z, const TileScale &ts, float &m_run, float &l_run, f32x16_t (&o)[DT]) {
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
    for (int v = 0; v < 8; ++v) {
        z[v] = __builtin_amdgcn_exp2f(fmaf(z[v], ts.k0, c0));
        z[8 + v] = __builtin_amdgcn_exp2f(fmaf(z[8 + v], ts.k1, c1));
        s0 += z[v];
        s1 += z[8 + v];
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
    float c;
};

enum { KV8_WAVES = 8 };
static size_t kv8_lds_bytes(int Dh, int qt) { return (size_t)qt * Dh * 64 + (size_t)KV8_WAVES * Dh * 128 + KV8_WAVES * 64 * 4 * qt; }

// PLAIN: queries and result are half [B, T, H, Dh]; otherwise the packed query buffer and the next GEMM's input.
template <int DH, int QT, int FMT, bool PLAIN>
__global__ __launch_bounds__(KV8_WAVES * 64, 2) void kv8_attn_kernel(Kv8Args p) {
    constexpr int KS = DH / 16, DT = DH / 32, NW = KV8_WAVES, KB = DH / 32, VB = DH / 32, TILE = KB + VB;     // KB, VB: KiB of a tile's K and V codes
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
    const int L = p.seq_len[b], ns = p.n_sealed[b];
    const int32_t *t8 = p.table8 + (size_t)b * p.max_pages8, *t16 = p.table16 + (size_t)b * p.max_pages;
    if (L < 0 || L + T > p.max_pages * 16 || ns < 0 || ns > (L >> 4) || ns > p.max_pages8) {     // uniform over the workgroup
        if (tid == 0 && j == 0 && h == 0) atomicOr(p.flags, FLAG_CAPACITY);
        return;
    }
    // ---- queries to LDS, in the order of the codes: block (i, e) holds, for half-wave hl, dims 32 i + 16 hl + 8 e .. + 7
    u32x4_t *qs = reinterpret_cast<u32x4_t *>(lds);
    for (int i = wave; i < QT * KS; i += NW) {
        const int q = i / KS, blk = i % KS, i2 = blk >> 1, e = blk & 1;
        int qtile = qg * QT + q;
        if (qtile >= QTtot) qtile = QTtot - 1;               // a second tile behind the last query: the first one again, which nobody stores
        u32x4_t v = {0u, 0u, 0u, 0u};
        if (PLAIN) {
            const int query = qtile * 32 + col;
            if (query < T) v = *reinterpret_cast<const u32x4_t *>(reinterpret_cast<const a16_t *>(p.q) + ((size_t)(b * T + query) * H + h) * DH + 32 * i2 + 16 * hl + 8 * e);
        } else {
            v = p.q[((((size_t)b * H + h) * QTtot + qtile) * KS + 2 * i2 + hl) * 64 + e * 32 + col];
        }
        qs[i * 64 + lane] = v;
    }
    uint64_t anc[QT][2];
#pragma unroll
    for (int q = 0; q < QT; ++q) {
        const int query = (qg * QT + q) * 32 + col;
        anc[q][0] = anc[q][1] = 0ull;
        if (query < T) { anc[q][0] = p.tree->anc[query][0]; anc[q][1] = p.tree->anc[query][1]; }
    }
    const int total = L + T, n8 = (ns + 1) >> 1, first16 = ns * 16, n16 = (total - first16 + 31) >> 5, row_pages = (total + 15) >> 4;
    const int mine8 = unit < n8 ? (n8 - unit + units - 1) / units : 0;           // this wave's tiles of codes: unit, unit + units, ...

    // ---- pages and scales of the wave's next 32 tiles, a page per lane
    int pgs = 0;
    float pk = 0.f, pv = 0.f, pr = 0.f;
    auto page_ids = [&](int first) {
        const int lp = 2 * (unit + (first + (lane >> 1)) * units) + (lane & 1);
        const bool there = lp < ns;
        pgs = there ? checked_page(t8[lp], p.n_pages8, p.flags) : -1;
        const float2 s = reinterpret_cast<const float2 *>(p.scales)[((size_t)p.layer * p.n_pages8 + max(pgs, 0)) * H + h];
        pk = there ? s.x * p.c : 0.f;                        // a page that is not there: exponent -infinity, weight 0
        pv = there ? __builtin_amdgcn_logf(s.y) : -INFINITY;
        pr = there ? 1.0f / s.y : 0.f;
        asm volatile("" : "+v"(pgs), "+v"(pk), "+v"(pv), "+v"(pr));               // awaited here: nothing in the loop waits for an ordinary load
    };
    page_ids(0);
#pragma unroll
    for (int q = 0; q < QT; ++q) asm volatile("" : "+v"(anc[q][0]), "+v"(anc[q][1]));

    u32x4_t *mine = qs + (QT * KS + wave * 2 * TILE) * 64;
    const uint32_t mine_at = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) void *)mine;
    auto dma = [&](const void *src, int block) {
        __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void *)src,
                                         (__attribute__((address_space(3))) void *)(uintptr_t)(mine_at + (uint32_t)block * 1024u), 16, 0, 0);
    };
    // pages of tile `it`: the second one may be missing (then the first one is read twice), a tile behind the last one reads page 0
    auto tile_pages = [&](int it, int &p0, int &p1) {
        p0 = max(__builtin_amdgcn_readlane(pgs, 2 * (it & 31)), 0);
        p1 = __builtin_amdgcn_readlane(pgs, 2 * (it & 31) + 1);
        if (p1 < 0) p1 = p0;
    };
    auto lane_of = [](float v, int l) { return __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(v), l)); };
    auto tile_scale = [&](int it) {
        const int l = 2 * (it & 31);
        return TileScale{lane_of(pk, l), lane_of(pk, l + 1), lane_of(pv, l), lane_of(pv, l + 1), lane_of(pr, l), lane_of(pr, l + 1)};
    };
    auto request_k = [&](int p0, int p1, int slot) {
        const uint8_t *kp = p.kcodes + kv8_block_base(p.layer, p.n_pages8, (col >> 4) ? p1 : p0, H, h, DH) + (hl * 16 + (col & 15)) * 16;
#pragma unroll
        for (int i = 0; i < KB; ++i) dma(kp + i * 512, slot * TILE + i);
    };
    auto request_v = [&](int p0, int p1, int slot) {
#pragma unroll
        for (int g = 0; g < 2; ++g) {
            const uint8_t *vp = p.vcodes + kv8_block_base(p.layer, p.n_pages8, g ? p1 : p0, H, h, DH) + lane * 16;
#pragma unroll
            for (int i = 0; i < VB / 2; ++i) dma(vp + i * 1024, slot * TILE + KB + g * (VB / 2) + i);
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
    __syncthreads();                                         // the queries are in LDS

    if (mine8 > 0) {
        int p0, p1;
        tile_pages(0, p0, p1); request_k(p0, p1, 0); request_v(p0, p1, 0);
        tile_pages(min(1, mine8 - 1), p0, p1); request_k(p0, p1, 1); request_v(p0, p1, 1);
    }
    TileScale ts = tile_scale(0), next = tile_scale(1);
    for (int it = 0; it < mine8; ++it) {
        const int slot = it & 1;
        const u32x4_t *tile = mine + slot * TILE * 64 + lane;
        asm volatile("s_waitcnt vmcnt(%0)" ::"n"(VB + TILE) : "memory");          // K has landed: younger are its V and the next tile
        f32x16_t z[QT];
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
        // the tile after the next one; where it is the first of another 32, the loads of their pages end every wait
        const int nx = it + 2;
        int p0 = 0, p1 = 0;
        if ((nx & 31) == 0 && nx < mine8) page_ids(nx);
        if (nx < mine8) tile_pages(nx, p0, p1);
        const TileScale after = tile_scale(nx);
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");   // K is read
        request_k(p0, p1, slot);
        u32x4_t pb[QT][2];
#pragma unroll
        for (int q = 0; q < QT; ++q) {
            kv8_softmax<DT>(z[q], ts, m_run[q], l_run[q], o[q]);
#pragma unroll
            for (int g = 0; g < 2; ++g)
#pragma unroll
                for (int w = 0; w < 4; ++w) pb[q][g][w] = half_pack(z[q][8 * g + 2 * w], z[q][8 * g + 2 * w + 1]);
        }
        asm volatile("s_waitcnt vmcnt(%0)" ::"n"(TILE + KB) : "memory");          // V has landed: younger are the next tile and another K
#pragma unroll
        for (int g = 0; g < 2; ++g)
#pragma unroll
            for (int i = 0; i < VB / 2; ++i) {
                const u32x4_t w = tile[(KB + g * (VB / 2) + i) * 64];
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
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");   // V is read
        request_v(p0, p1, slot);
        ts = next;
        next = after;
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");         // what was requested past the last tile has landed

    // ---- the 16-bit tail: tiles n8, n8 + 1, ... in the same turn
    const TileScale one = {p.c, p.c, 0.f, 0.f, 1.f, 1.f};
    for (int t = (unit - n8 % units + units) % units; t < n16; t += units) {
        const int slot0 = first16 + t * 32, lp = ns + 2 * t;
        const int p0 = checked_page(t16[lp], p.n_pages, p.flags);
        const int p1 = lp + 1 < row_pages ? checked_page(t16[lp + 1], p.n_pages, p.flags) : p0;
        u32x4_t w[KS];
        const u32x4_t *kp = reinterpret_cast<const u32x4_t *>(p.kpages + kv_block_base(p.layer, p.n_pages, (col >> 4) ? p1 : p0, H, h, DH)) + hl * 16 + (col & 15);
#pragma unroll
        for (int s = 0; s < KS; ++s) w[s] = kp[s * 32];
#pragma unroll
        for (int g = 0; g < 2; ++g) {                        // V to LDS, each lane its own pieces
            const u32x4_t *vp = reinterpret_cast<const u32x4_t *>(p.vpages + kv_block_base(p.layer, p.n_pages, g ? p1 : p0, H, h, DH)) + col * 2 + hl;
            u32x4_t keep;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                // dword e holds keys i = 2e, 2e+1 of this half-wave: token = 8*(i/4) + 4*hl + i%4.  Slots past the last node become 0: stale contents
                const int i0 = 2 * e, i1 = 2 * e + 1;
                const int s0 = slot0 + 16 * g + 8 * (i0 >> 2) + 4 * hl + (i0 & 3);
                const int s1 = slot0 + 16 * g + 8 * (i1 >> 2) + 4 * hl + (i1 & 3);
                keep[e] = (s0 < total ? 0x0000ffffu : 0u) | (s1 < total ? 0xffff0000u : 0u);
            }
#pragma unroll
            for (int dt = 0; dt < DT; ++dt) mine[(g * DT + dt) * 64 + lane] = vp[dt * 64] & keep;
        }
        f32x16_t z[QT];
#pragma unroll
        for (int q = 0; q < QT; ++q)
#pragma unroll
            for (int v = 0; v < 16; ++v) z[q][v] = 0.f;
#pragma unroll
        for (int s = 0; s < KS; ++s)                         // 16-bit K has dims 16 s + 8 hl in step s: block (s / 2, e = hl), its half-wave s % 2
#pragma unroll
            for (int q = 0; q < QT; ++q)
                z[q] = HYDRA_MFMA16(__builtin_bit_cast(a16x8_t, w[s]), __builtin_bit_cast(a16x8_t, qs[(q * KS + (s & ~1) + hl) * 64 + (s & 1) * 32 + col]), z[q]);
#pragma unroll
        for (int q = 0; q < QT; ++q) {
            const uint32_t seen = keys_seen(slot0, L, anc[q][0], anc[q][1]) >> (4 * hl);
#pragma unroll
            for (int v = 0; v < 16; ++v) z[q][v] = (seen >> (8 * (v >> 2) + (v & 3))) & 1u ? z[q][v] : -INFINITY;
            kv8_softmax<DT>(z[q], one, m_run[q], l_run[q], o[q]);
        }
#pragma unroll
        for (int g = 0; g < 2; ++g) {
            u32x4_t pb[QT];
#pragma unroll
            for (int q = 0; q < QT; ++q)
#pragma unroll
                for (int e = 0; e < 4; ++e) pb[q][e] = half_pack(z[q][8 * g + 2 * e], z[q][8 * g + 2 * e + 1]);
#pragma unroll
            for (int dt = 0; dt < DT; ++dt) {
                const a16x8_t v = __builtin_bit_cast(a16x8_t, mine[(g * DT + dt) * 64 + lane]);
#pragma unroll
                for (int q = 0; q < QT; ++q) o[q][dt] = HYDRA_MFMA16(v, __builtin_bit_cast(a16x8_t, pb[q]), o[q][dt]);
            }
        }
    }

    // ---- merge the waves through LDS, one query tile after the other: maxima and sums [QT][NW][2][32], then O[NW][DT * 16][64]
    __syncthreads();                                         // every wave is done with queries and tiles
    float *ml = lds, *ob = lds + QT * NW * 64;
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
        float *dst = ob + (size_t)wave * DT * 16 * 64 + lane;
#pragma unroll
        for (int dt = 0; dt < DT; ++dt)
#pragma unroll
            for (int v = 0; v < 16; ++v) dst[(dt * 16 + v) * 64] = o[q][dt][v] * f;
        __syncthreads();
        // the (band, group of 4 registers = 4 consecutive dims) items are shared out over the waves
        const float inv = p.key_wgs == 1 ? 1.0f / l_tot : 1.0f;
        for (int id = wave; id < DT * 4; id += NW) {
            const int dt = id >> 2, g4 = id & 3;
            float acc[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int w = 0; w < NW; ++w) {
                const float *src = ob + (size_t)w * DT * 16 * 64 + lane;
#pragma unroll
                for (int e = 0; e < 4; ++e) acc[e] += src[(dt * 16 + 4 * g4 + e) * 64];
            }
            const int dim = 32 * dt + 8 * g4 + 4 * hl, m = b * T + query;
            if (p.key_wgs > 1) {
                *reinterpret_cast<f32x4_t *>(rec + (size_t)query * DH + dim) = f32x4_t{acc[0], acc[1], acc[2], acc[3]};
            } else if (query < T) {
                const u32x2_t pk2 = {f2a_pack(acc[0] * inv, acc[1] * inv), f2a_pack(acc[2] * inv, acc[3] * inv)};
                a16_t *to = reinterpret_cast<a16_t *>(p.out) + (PLAIN ? ((size_t)m * H + h) * DH + dim : x_index<true>(m, h * DH + dim, H * DH));
                *reinterpret_cast<u32x2_t *>(to) = pk2;
            }
        }
        if (p.key_wgs > 1 && wave == 0 && hl == 0) {
            rec[(size_t)Tq * DH + query] = m_tot;
            rec[(size_t)Tq * DH + Tq + query] = l_tot;
        }
        if (q + 1 < QT) __syncthreads();                     // the next query tile's sums go where these were
    }
}

// out = sum_u 2^(M_u - M) O_u / sum_u 2^(M_u - M) l_u over the records of a head: one thread per (query, 4 dims), all its loads in one round trip.
enum { KV8_MERGE_MAX = 16 };
template <bool PLAIN>
__global__ __launch_bounds__(256) void kv8_merge_kernel(const float *__restrict__ apart, const int32_t *__restrict__ seq_len, const int32_t *__restrict__ n_sealed,
                                                         int T, int H, int Dh, int units, int max_pages, int max_pages8, void *out) {
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
    if (L < 0 || L + T > max_pages * 16 || ns < 0 || ns > (L >> 4) || ns > max_pages8 || !live) return;
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
    a16_t *to = reinterpret_cast<a16_t *>(out) + (PLAIN ? ((size_t)m * H + h) * Dh + dim : x_index<true>(m, h * Dh + dim, H * Dh));
    *reinterpret_cast<u32x2_t *>(to) = pk;
}

#define KV8_EACH(X) X(128, 1, KV8_INT8) X(128, 2, KV8_INT8) X(128, 1, KV8_E4M3) X(128, 2, KV8_E4M3) X(64, 1, KV8_INT8) X(64, 2, KV8_INT8) X(64, 1, KV8_E4M3) X(64, 2, KV8_E4M3)

int kv8_max_dynamic_lds() {
    hipError_t e = hipSuccess;
#define ATTR(DHv, QTv, Fv)                                                                                                                                      \
    if (e == hipSuccess) e = hipFuncSetAttribute((const void *)kv8_attn_kernel<DHv, QTv, Fv, true>, hipFuncAttributeMaxDynamicSharedMemorySize, 160 * 1024);     \
    if (e == hipSuccess) e = hipFuncSetAttribute((const void *)kv8_attn_kernel<DHv, QTv, Fv, false>, hipFuncAttributeMaxDynamicSharedMemorySize, 160 * 1024);
    KV8_EACH(ATTR)
#undef ATTR
    if (e != hipSuccess) return hip_fail(e, "hipFuncSetAttribute(8-bit attention kernels)");
    return HYDRA_OK;
}

int launch_kv8_attention(hydra_ctx *c, hipStream_t s, int B, int layer, const void *q, bool q_plain, const int32_t *seq_len, const hydra_kv8 *kv,
                         float *apart, int units_max, void *out, bool out_plain, int32_t *flags) {
    (void)out_plain;                                         // queries and result are plain together or packed together
    const int T = c->tree.T, H = c->m.n_heads, Dh = c->m.head_dim;
    const int QTtot = ceil_div(T, 32), qt = QTtot > 1 ? 2 : 1, qgroups = ceil_div(QTtot, qt);
    const int len = kv->tail.seq_len_hint > 0 ? kv->tail.seq_len_hint : c->m.max_pos;
    const int tiles = ceil_div(len + T, 32) + 1, hb = H * B * qgroups;
    const int wgs = std::max(1, std::min({ceil_div(tiles, KV8_WAVES * 2), std::max(1, 256 / hb), units_max, (int)KV8_MERGE_MAX}));
    Kv8Args a;
    a.q = (const u32x4_t *)q; a.kcodes = (const uint8_t *)kv->k_codes; a.vcodes = (const uint8_t *)kv->v_codes; a.scales = kv->scales;
    a.table8 = kv->page_table; a.n_sealed = kv->n_sealed; a.kpages = (const a16_t *)kv->tail.k_pages; a.vpages = (const a16_t *)kv->tail.v_pages;
    a.table16 = kv->tail.page_table; a.seq_len = seq_len; a.tree = tree_dev(c); a.apart = apart; a.out = out; a.flags = flags;
    a.max_pages8 = kv->max_pages; a.n_pages8 = kv->n_pages; a.max_pages = kv->tail.max_pages; a.n_pages = kv->tail.n_pages; a.layer = layer;
    a.T = T; a.H = H; a.groups = H * B; a.key_wgs = wgs; a.c = LOG2E / sqrtf((float)Dh);
    const dim3 grid(ceil_div(H * B, 8) * 8 * qgroups * wgs), block(KV8_WAVES * 64);
    const size_t lds = kv8_lds_bytes(Dh, qt);
#define LAUNCH(DHv, QTv, Fv)                                                                                                     \
    if (Dh == DHv && qt == QTv && kv->format == Fv) {                                                                            \
        if (q_plain) hipLaunchKernelGGL((kv8_attn_kernel<DHv, QTv, Fv, true>), grid, block, lds, s, a);                          \
        else         hipLaunchKernelGGL((kv8_attn_kernel<DHv, QTv, Fv, false>), grid, block, lds, s, a);                         \
    }
    KV8_EACH(LAUNCH)
#undef LAUNCH
    HYDRA_LAUNCH_CHECK("kv8_attn_kernel");
    if (wgs > 1) {
        const dim3 mgrid(ceil_div(T, 256 / (Dh / 4)), H, B), mblock(256);
        if (q_plain) hipLaunchKernelGGL(kv8_merge_kernel<true>, mgrid, mblock, 0, s, apart, seq_len, kv->n_sealed, T, H, Dh, wgs, kv->tail.max_pages, kv->max_pages, out);
        else         hipLaunchKernelGGL(kv8_merge_kernel<false>, mgrid, mblock, 0, s, apart, seq_len, kv->n_sealed, T, H, Dh, wgs, kv->tail.max_pages, kv->max_pages, out);
        HYDRA_LAUNCH_CHECK("kv8_merge_kernel");
    }
    return HYDRA_OK;
}

}  // namespace hydra
