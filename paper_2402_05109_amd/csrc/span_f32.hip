// Tree attention over part of an fp32 cache, and the sums of the weights that every slot receives: span_attn.hip's operators for fp32 contexts.
//
// The products run on the fp32 matrix instruction (16x16x4, exact products and fp32 sums), one 16-token page at a time:
//   S^T[key][query] = K[key][:] . Q[query][:]       lane: key lane % 16, dims 16 i + 4 g .. + 3 with g = lane / 16 (any order of the dims will do for a sum)
//   O^T[dim][query] += V^T[dim][key] P^T[key][query]  step e takes keys 4 g + e, which is where the accumulator has them
// so K and V come in 16-byte loads straight from the page and a query is a column of both.  A wave holds 32 queries.
// 2 rows of 64 nodes behind 2000 tokens, 16 heads of 128: 34 us and 5 for the records, of which the products are 14 at the matrix units' rate: pages are
// short, and between a page's two products lie its maxima and exponentials.
#include <algorithm>

#include "span.h"

namespace hydra {

typedef __attribute__((ext_vector_type(4))) float f32x4_t;
#define SPAN_MFMA4(a, b, c) __builtin_amdgcn_mfma_f32_16x16x4f32(a, b, c, 0, 0, 0)

// over the four lanes that hold a query's keys; the same in all of them
template <class Op>
__device__ __forceinline__ float over_keys(float v, Op op) {
    const HalfWaves h = half_waves(v);
    v = op(h.lo, h.hi);
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return op(__uint_as_float(r[0]), __uint_as_float(r[1]));
}

enum { SPAN32_WAVES = 8, SPAN32_QT = 2 };
template <int DH>
__global__ __launch_bounds__(SPAN32_WAVES * 64) void span_f32_kernel(SpanArgs p) {
    constexpr int KS = DH / 16, J = DH / 64, NW = SPAN32_WAVES, QT = SPAN32_QT;
    __shared__ f32x4_t qs[QT * KS * 64];
    __shared__ f32x4_t ob[NW * J * 4 * 64];
    __shared__ float ml[QT * NW * 32];
    const int tid = (int)threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int g = lane >> 4, col = lane & 15;
    const int T = p.T, H = p.H, QG = (T + 16 * QT - 1) / (16 * QT), per = QG * p.key_wgs;
    const int seq = (int)blockIdx.x >> 3;
    const int group = seq / per * 8 + ((int)blockIdx.x & 7), j = seq % per;
    if (group >= p.groups) return;
    const int b = group / H, h = group - b * H, qg = j % QG, key_wg = j / QG;
    // what does not depend on the row's length, beside the load of that
    const float *q = reinterpret_cast<const float *>(p.q);
    constexpr int PIECES = (QT * KS + NW - 1) / NW;
    f32x4_t piece[PIECES];
#pragma unroll
    for (int i = 0; i < PIECES; ++i) {                       // queries behind the last one: that one again, which nobody stores
        const int at = min(wave + i * NW, QT * KS - 1), query = min((qg * QT + at / KS) * 16 + col, T - 1);
        piece[i] = *reinterpret_cast<const f32x4_t *>(q + ((size_t)(b * T + query) * H + h) * DH + 16 * (at % KS) + 4 * g);
    }
    SpanNode node[QT];
#pragma unroll
    for (int t = 0; t < QT; ++t) node[t] = span_node(p, (qg * QT + t) * 16 + col);
    const int units = p.key_wgs * NW, unit = key_wg * NW + wave;
    const SpanRow r = span_row<16>(p, b);
    if (!r.ok) {                                            // uniform over the workgroup
        if (tid == 0 && j == 0 && h == 0) atomicOr(p.flags, FLAG_CAPACITY);
        return;
    }
    const int32_t *pt = p.table + (size_t)b * p.max_pages;
    const float *kpages = reinterpret_cast<const float *>(p.kpages), *vpages = reinterpret_cast<const float *>(p.vpages);
    SpanQuery sq[QT];
#pragma unroll
    for (int t = 0; t < QT; ++t) sq[t] = span_query(p, r, (qg * QT + t) * 16 + col, node[t]);
#pragma unroll
    for (int i = 0; i < PIECES; ++i)
        if (wave + i * NW < QT * KS) qs[(wave + i * NW) * 64 + lane] = piece[i];
    __syncthreads();
    f32x4_t o[QT][J * 4];                                   // [4 jj + e]: dims 64 jj + 16 g + 4 rr + e, rr the place in the vector
#pragma unroll
    for (int t = 0; t < QT; ++t)
#pragma unroll
        for (int i = 0; i < J * 4; ++i) o[t][i] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    const int tiles = min(QT, (T - qg * QT * 16 + 15) >> 4);
    float m_run[QT], l_run[QT];
#pragma unroll
    for (int t = 0; t < QT; ++t) { m_run[t] = -INFINITY; l_run[t] = 0.f; }
    // K of the next tile is asked for behind this one's first product, V behind the second, page numbers a tile ahead; behind the last tile: the last one again
    auto tile_page = [&](int u) { return pt[r.tile(min(u, r.n - 1))]; };
    f32x4_t k[KS], v[4][J];
    auto load_k = [&](size_t base) {
#pragma unroll
        for (int i = 0; i < KS; ++i) k[i] = *reinterpret_cast<const f32x4_t *>(kpages + base + col * DH + 16 * i + 4 * g);
    };
    auto load_v = [&](size_t base) {
#pragma unroll
        for (int e = 0; e < 4; ++e)
#pragma unroll
            for (int jj = 0; jj < J; ++jj) v[e][jj] = *reinterpret_cast<const f32x4_t *>(vpages + base + (4 * g + e) * DH + 64 * jj + 4 * col);
    };
    auto base_of = [&](int page) { return kv_block_base(p.layer, p.n_pages, checked_page(page, p.n_pages, p.flags), H, h, DH); };
    size_t base = 0;
    int page = 0;
    if (unit < r.n) {
        base = base_of(tile_page(unit));
        page = tile_page(unit + units);
        load_k(base);
        load_v(base);
    }
    for (int u = unit; u < r.n; u += units) {
        const int slot0 = r.tile(u) * 16;
        const bool whole = span_whole<16>(p, r, slot0);     // uniform
        int at = lane;
        asm volatile("" : "+v"(at));                         // keeps the reads of the queries inside the loop
        f32x4_t st[QT];
#pragma unroll
        for (int t = 0; t < QT; ++t) {
            if (t >= tiles) break;                           // uniform over the workgroup: no node in it
            f32x4_t s = {0.f, 0.f, 0.f, 0.f}, s1 = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int i = 0; i < KS; ++i) {                   // two chains: a product waits for the one before it in its own
                const f32x4_t qv = qs[(t * KS + i) * 64 + at];
#pragma unroll
                for (int e = 0; e < 4; e += 2) {
                    s = SPAN_MFMA4(k[i][e], qv[e], s);
                    s1 = SPAN_MFMA4(k[i][e + 1], qv[e + 1], s1);
                }
            }
            st[t] = s + s1;
        }
        const size_t next = base_of(page);
        page = tile_page(u + 2 * units);
        load_k(next);
        bool odd = false;                                   // something that is not finite in a tile that not every query sees whole
        if (!whole) {
            const uint32_t held = span_held(r, slot0);
#pragma unroll
            for (int e = 0; e < 4; ++e)
#pragma unroll
                for (int jj = 0; jj < J; ++jj) {
                    if (!((held >> (4 * g + e)) & 1u)) v[e][jj] = f32x4_t{0.f, 0.f, 0.f, 0.f};      // never written, or evicted
#pragma unroll
                    for (int d = 0; d < 4; ++d) odd |= !(fabsf(v[e][jj][d]) < INFINITY);
                }
            odd = __any(odd);
        }
#pragma unroll
        for (int t = 0; t < QT; ++t) {
            if (t >= tiles) break;
            f32x4_t s = st[t];
            if (!whole) {
                const uint32_t seen = span_seen(r, sq[t], slot0) >> (4 * g);
#pragma unroll
                for (int e = 0; e < 4; ++e) s[e] = (seen >> e) & 1u ? s[e] : -INFINITY;
            }
            if (t == 0 && p.z && qg == 0 && col == 0 && u * 16 + 16 <= p.z_slots) *reinterpret_cast<f32x4_t *>(p.z + ((size_t)b * H + h) * p.z_slots + u * 16 + 4 * g) = s;
            const float top = over_keys(fmaxf(fmaxf(s[0], s[1]), fmaxf(s[2], s[3])), [](float a, float c) { return fmaxf(a, c); });
            const float m_new = fmaxf(m_run[t], top), ref = m_new == -INFINITY ? 0.f : m_new;
            const float alpha = __builtin_amdgcn_exp2f((m_run[t] - ref) * p.c);
            if (__any(m_new != m_run[t])) {
#pragma unroll
                for (int i = 0; i < J * 4; ++i) o[t][i] *= alpha;
            }
            m_run[t] = m_new;
#pragma unroll
            for (int e = 0; e < 4; ++e) s[e] = __builtin_amdgcn_exp2f((s[e] - ref) * p.c);       // 0 for masked slots
            l_run[t] = l_run[t] * alpha + over_keys((s[0] + s[1]) + (s[2] + s[3]), [](float a, float c) { return a + c; });
            if (!odd) {
#pragma unroll
                for (int e = 0; e < 4; ++e)
#pragma unroll
                    for (int jj = 0; jj < J; ++jj)
#pragma unroll
                        for (int d = 0; d < 4; ++d) o[t][4 * jj + d] = SPAN_MFMA4(v[e][jj][d], s[e], o[t][4 * jj + d]);
            } else {                                         // what a query does not see must not reach it as 0 * infinity: key by key
                for (int kk = 0; kk < 4; ++kk)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const float w = __shfl(s[e], kk * 16 + col, 64);
                        const float *vp = vpages + base + (4 * kk + e) * DH + 16 * g;
                        if (w == 0.f) continue;
#pragma unroll
                        for (int jj = 0; jj < J; ++jj)
#pragma unroll
                            for (int rr = 0; rr < 4; ++rr)
#pragma unroll
                                for (int d = 0; d < 4; ++d) o[t][4 * jj + d][rr] = fmaf(w, vp[64 * jj + 4 * rr + d], o[t][4 * jj + d][rr]);
                    }
            }
        }
        base = next;
        load_v(base);
    }
    // ---- merge the waves through LDS, one query tile after the other
    if (g == 0) {
#pragma unroll
        for (int t = 0; t < QT; ++t) {
            ml[(t * NW + wave) * 32 + col] = m_run[t];
            ml[(t * NW + wave) * 32 + 16 + col] = l_run[t];
        }
    }
    const int Tq = ((T + 31) >> 5) * 32;
    float *rec = p.apart + (((size_t)b * H + h) * p.key_wgs + key_wg) * ((size_t)Tq * DH + 2 * (size_t)Tq);
#pragma unroll
    for (int t = 0; t < QT; ++t) {
        const int query = (qg * QT + t) * 16 + col;
        if (t >= tiles) break;
        __syncthreads();                                     // maxima and sums are there; the tile before this one is stored
        float m_tot = -INFINITY;
#pragma unroll
        for (int w = 0; w < NW; ++w) m_tot = fmaxf(m_tot, ml[(t * NW + w) * 32 + col]);
        const float m_safe = m_tot == -INFINITY ? 0.f : m_tot;
        float l_tot = 0.f;
#pragma unroll
        for (int w = 0; w < NW; ++w) l_tot += __builtin_amdgcn_exp2f((ml[(t * NW + w) * 32 + col] - m_safe) * p.c) * ml[(t * NW + w) * 32 + 16 + col];
        const float f = __builtin_amdgcn_exp2f((m_run[t] - m_safe) * p.c);
#pragma unroll
        for (int jj = 0; jj < J; ++jj)
#pragma unroll
            for (int rr = 0; rr < 4; ++rr)
                ob[(wave * J * 4 + jj * 4 + rr) * 64 + lane] = f32x4_t{o[t][4 * jj][rr], o[t][4 * jj + 1][rr], o[t][4 * jj + 2][rr], o[t][4 * jj + 3][rr]} * f;
        __syncthreads();
        const float inv = 1.0f / l_tot;
        for (int id = wave; id < J * 4; id += NW) {
            f32x4_t acc = ob[id * 64 + lane];
#pragma unroll
            for (int w = 1; w < NW; ++w) acc += ob[(w * J * 4 + id) * 64 + lane];
            const int dim = 64 * (id >> 2) + 16 * g + 4 * (id & 3);
            if (query >= T) continue;                        // columns behind the last node go nowhere
            if (p.key_wgs > 1) *reinterpret_cast<f32x4_t *>(rec + (size_t)query * DH + dim) = acc;
            else *reinterpret_cast<f32x4_t *>(reinterpret_cast<float *>(p.out) + ((size_t)(b * T + query) * H + h) * DH + dim) = acc * inv;
        }
        if (wave == 0 && g == 0) {
            if (p.key_wgs > 1) {
                rec[(size_t)Tq * DH + query] = m_tot;
                rec[(size_t)Tq * DH + Tq + query] = l_tot;
            } else if (p.stats) {
                p.stats[((size_t)b * H + h) * Tq + query] = SpanStat{m_tot, inv};
            }
        }
        if (t == 0 && p.z && qg == 0 && p.key_wgs == 1) {    // uniform: the root's weights, by the whole workgroup
            if (tid == 0) *reinterpret_cast<SpanStat *>(ml) = SpanStat{m_tot, inv};
            __syncthreads();                                 // (and every wave's scores are written; the first maximum and sum had been read)
            const SpanStat st = *reinterpret_cast<const SpanStat *>(ml);
            span_add_root<16>(p, r, b, h, st, tid, NW * 64, [&](int slot, int page) {
                const float *kp = kpages + kv_block_base(p.layer, p.n_pages, page, H, h, DH) + (slot & 15) * DH, *q0 = q + ((size_t)b * T * H + h) * DH;
                float z = 0.f;
                for (int d = 0; d < DH; ++d) z = fmaf(kp[d], q0[d], z);
                return z;
            });
        }
    }
}

// The weights that every slot receives from nodes 0 .. n_scored - 1, behind the attention (span_attn.hip): queries are the rows of S = Q K^T here, a lane
// holds one slot, and the accumulators begin with -M' of the queries.
template <int DH>
__global__ __launch_bounds__(SPAN32_WAVES * 64) void span_score_f32_kernel(SpanArgs p) {
    constexpr int KS = DH / 16, NW = SPAN32_WAVES;
    extern __shared__ float lds[];                          // queries [tiles][KS] of 1 KiB, then of each query what it sees and -M'
    const int tid = (int)threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int g = lane >> 4, col = lane & 15;
    const int T = p.T, H = p.H, QS = (p.n_scored + 15) >> 4, Tq = ((T + 31) >> 5) * 32;
    const int seq = (int)blockIdx.x >> 3;
    const int group = seq / p.key_wgs * 8 + ((int)blockIdx.x & 7), key_wg = seq % p.key_wgs;
    if (group >= p.groups) return;
    const int b = group / H, h = group - b * H;
    const SpanRow r = span_row<16>(p, b);
    if (!r.ok) return;                                      // reported by the attention
    const int units = p.key_wgs * NW, unit = key_wg * NW + wave;
    const int32_t *pt = p.table + (size_t)b * p.max_pages;
    const float *q = reinterpret_cast<const float *>(p.q), *kpages = reinterpret_cast<const float *>(p.kpages);
    auto page_id = [&](int u) {                             // behind the last tile: the last one again
        const int raw = pt[r.tile(min(u, r.n - 1))];
        return (unsigned)raw < (unsigned)p.n_pages ? raw : 0;                    // reported by the attention
    };
    auto load = [&](f32x4_t (&k)[KS], int page) {
        const float *kp = kpages + kv_block_base(p.layer, p.n_pages, page, H, h, DH) + col * DH + 4 * g;
#pragma unroll
        for (int i = 0; i < KS; ++i) k[i] = *reinterpret_cast<const f32x4_t *>(kp + 16 * i);
    };
    f32x4_t k[KS];
    load(k, page_id(unit));
    int page = page_id(unit + units);
    f32x4_t *qs = reinterpret_cast<f32x4_t *>(lds);
    SpanQuery *sq = reinterpret_cast<SpanQuery *>(qs + QS * KS * 64);
    float *start = reinterpret_cast<float *>(sq + QS * 16);
    for (int i = wave; i < QS * KS; i += NW) {
        const int query = i / KS * 16 + col;
        f32x4_t v = {0.f, 0.f, 0.f, 0.f};
        if (query < T) v = *reinterpret_cast<const f32x4_t *>(q + ((size_t)(b * T + query) * H + h) * DH + 16 * (i % KS) + 4 * g);
        qs[i * 64 + lane] = v;
    }
    for (int i = tid; i < QS * 16; i += NW * 64) {
        const bool counts = i < p.n_scored;
        const SpanStat s = p.stats[((size_t)b * H + h) * Tq + (counts ? i : 0)];
        start[i] = counts ? __builtin_amdgcn_logf(s.r) / p.c - s.m : -INFINITY;
        sq[i] = span_query(p, r, counts ? i : T);
    }
    __syncthreads();
    float *row = p.score + ((size_t)b * H + h) * ((size_t)p.max_pages * 16);
    for (int u = unit; u < r.n; u += units) {
        const int slot0 = r.tile(u) * 16, slot = slot0 + col;
        const bool whole = span_whole<16>(p, r, slot0), mine = g == 0 && ((span_held(r, slot0) >> col) & 1u);
        const float before = mine && slot < r.L ? row[slot] : 0.f;
        f32x4_t next[KS];
        load(next, page);
        page = page_id(u + 2 * units);
        float sum = 0.f;
        for (int t = 0; t < QS; ++t) {
            const f32x4_t begin = *reinterpret_cast<const f32x4_t *>(start + t * 16 + 4 * g);
            f32x4_t z = begin, z1 = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int i = 0; i < KS; ++i) {                   // two chains: a product waits for the one before it in its own
                const f32x4_t qv = qs[(t * KS + i) * 64 + lane];
#pragma unroll
                for (int e = 0; e < 4; e += 2) {
                    z = SPAN_MFMA4(qv[e], k[i][e], z);
                    z1 = SPAN_MFMA4(qv[e + 1], k[i][e + 1], z1);
                }
            }
            z += z1;
            if (!whole) {
#pragma unroll
                for (int e = 0; e < 4; ++e) z[e] = (span_seen(r, sq[t * 16 + 4 * g + e], slot0) >> col) & 1u ? z[e] : -INFINITY;
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float w = __builtin_amdgcn_exp2f(z[e] * p.c);
                sum += begin[e] == -INFINITY ? 0.f : w;      // of a query that does not count, whose products may be infinite or no numbers
            }
        }
        sum = over_keys(sum, [](float a, float c) { return a + c; });
        if (mine) row[slot] = before + sum;
#pragma unroll
        for (int i = 0; i < KS; ++i) k[i] = next[i];
    }
}

int span_f32_max_dynamic_lds() {
    hipError_t e = hipFuncSetAttribute((const void *)span_score_f32_kernel<128>, hipFuncAttributeMaxDynamicSharedMemorySize, 160 * 1024);
    if (e == hipSuccess) e = hipFuncSetAttribute((const void *)span_score_f32_kernel<64>, hipFuncAttributeMaxDynamicSharedMemorySize, 160 * 1024);
    if (e != hipSuccess) return hip_fail(e, "hipFuncSetAttribute(attention over part of an fp32 cache)");
    return HYDRA_OK;
}

int launch_span_f32(hydra_ctx *c, hipStream_t s, SpanArgs a, int slots, int units_max) {
    const int T = a.T, Dh = c->m.head_dim, pages = ceil_div(slots, 16) + 2, hb = a.groups * ceil_div(T, 16 * SPAN32_QT);
    // two pages of a wave cost less than a second kernel (16 nodes, 4 heads of 64: a window of 100 7.8 us against 9.2; 330 tokens 8.8, by one workgroup with three pages of a
    // wave 9.9).  More workgroups than compute units leave more records only (2 rows of 64 nodes behind 2000 tokens, 16 heads of 128: 43 us instead of 37)
    a.key_wgs = pages <= 2 * SPAN32_WAVES ? 1 : std::max(1, std::min({ceil_div(pages, SPAN32_WAVES), std::max(1, 256 / hb), units_max}));
    const dim3 grid(ceil_div(a.groups, 8) * 8 * ceil_div(T, 16 * SPAN32_QT) * a.key_wgs), block(SPAN32_WAVES * 64);
    if (Dh == 128) hipLaunchKernelGGL(span_f32_kernel<128>, grid, block, 0, s, a);
    else           hipLaunchKernelGGL(span_f32_kernel<64>, grid, block, 0, s, a);
    HYDRA_LAUNCH_CHECK("span_f32_kernel");
    if (a.key_wgs > 1) {
        int rc = launch_span_merge(c, s, a, slots);
        if (rc) return rc;
    }
    if (!a.score || a.z) return HYDRA_OK;
    const int QS = ceil_div(a.n_scored, 16);
    a.key_wgs = std::max(1, std::min(ceil_div(pages, SPAN32_WAVES), std::max(1, 256 / a.groups)));
    const dim3 sgrid(ceil_div(a.groups, 8) * 8 * a.key_wgs);
    const size_t lds = (size_t)QS * ((Dh / 16) * 1024 + 16 * (sizeof(SpanQuery) + 4));
    if (Dh == 128) hipLaunchKernelGGL(span_score_f32_kernel<128>, sgrid, block, lds, s, a);
    else           hipLaunchKernelGGL(span_score_f32_kernel<64>, sgrid, block, lds, s, a);
    HYDRA_LAUNCH_CHECK("span_score_f32_kernel");
    return HYDRA_OK;
}

}  // namespace hydra
