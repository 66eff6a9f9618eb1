// Eviction from a cache by accumulated attention weight, and what goes with it: scores that follow accepted tokens, pages that nobody sees any more.
//
// A row that holds more than `keep` tokens keeps, for each layer and head on its own, its first ones, its last ones and those in between with the largest
// scores.  They move to the row's last slots, in their order, so that the last ones stay where they are, positions of tokens to come do not change and
// whole pages become free in front.
#include <algorithm>
#include <climits>

#include "device_common.h"
#include "internal.h"

namespace hydra {

typedef __attribute__((ext_vector_type(4))) uint32_t u32x4_t;

struct EvictArgs {
    const int32_t *table, *dst_table, *ref, *seq_len;       // dst_table: NULL = in place
    int32_t *first, *kept, *evicted, *flags;
    float *score;
    void *k, *v;
    int max_pages, n_pages, n_sinks, n_recent, keep, slack, score_rows, T;
};

// Larger scores have larger keys; a NaN has that of -infinity.  0 is below every key.
__device__ __forceinline__ uint32_t score_key(float v) {
    uint32_t b = __float_as_uint(v);
    if ((b & 0x7fffffffu) > 0x7f800000u) b = 0xff800000u;
    if (b == 0x80000000u) b = 0u;                           // -0 equals +0
    return (b & 0x80000000u) ? ~b : (b | 0x80000000u);
}

// the largest over the 64 lanes, the same in all of them
__device__ __forceinline__ uint32_t wave_max(uint32_t v) {
    const auto a = __builtin_amdgcn_permlane32_swap(v, v, false, false);
    v = max(a[0], a[1]);
    const auto b = __builtin_amdgcn_permlane16_swap(v, v, false, false);
    v = max(b[0], b[1]);
    v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x128, 0xf, 0xf, false));            // row_ror:8, 4, 2, 1
    v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x124, 0xf, 0xf, false));
    v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x122, 0xf, 0xf, false));
    return max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x121, 0xf, 0xf, false));
}
// sums over the lanes up to this one
__device__ __forceinline__ int wave_prefix(int v, int lane) {
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const int y = __shfl_up(v, d);
        if (lane >= d) v += y;
    }
    return v;
}

// One workgroup per (head, row, layer) finds what it keeps.  Between the smallest and the largest key, the bracket, lies the key of the last token that is kept
// (`want` tokens have it or a larger one): candidates are counted in BINS parts of the bracket, which then becomes the part that this key lies in, until all that
// is in it stays or it is one key; tokens with that very key are taken from the lowest slot on.  Keys are in the order of the scores but spread like their
// logarithms, so a second turn nearly always ends it (two bits of the key a turn, counted by comparisons with each candidate, took 38 us where this takes 19: 4 layers of 40 heads,
// 15487 candidates).  A thread holds PER neighbouring candidates in registers; rows that have more than THREADS * PER are read again in every turn.
template <int THREADS, int PER>
__global__ __launch_bounds__(THREADS) void evict_select_kernel(EvictArgs a) {
    constexpr int WAVES = THREADS / 64, PIECE = THREADS * PER;
    constexpr int BINS = THREADS * 4, LOG = THREADS == 256 ? 10 : THREADS == 512 ? 11 : 12;
    static_assert(1 << LOG == BINS, "");
    typedef __attribute__((ext_vector_type(4), may_alias)) int i32x4_t;
    __shared__ i32x4_t bins[THREADS];                        // of thread tid: the 4 from bin 4 * (THREADS - 1 - tid) on
    __shared__ int part[WAVES];
    __shared__ uint32_t ends[2][WAVES];
    __shared__ int found[3];                                 // a bin, how many candidates lie above it, how many in it
    const int tid = (int)threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int h = blockIdx.x, b = blockIdx.y, layer = blockIdx.z, H = gridDim.x, B = gridDim.y;
    const bool speaks = tid == 0 && h == 0 && layer == 0;
    const int L = a.seq_len[b], F = a.first[b];
    if (L < 0 || L > a.max_pages * 16 || F < 0 || F > L) {  // uniform over the workgroup, as all that follows up to the tokens
        if (speaks) { atomicOr(a.flags, FLAG_CAPACITY); a.evicted[b] = 0; }
        return;
    }
    if ((int64_t)L - F <= (int64_t)a.keep + a.slack) {
        if (speaks) a.evicted[b] = 0;
        return;
    }
    float *score = a.score + (((size_t)layer * a.score_rows + b) * H + h) * ((size_t)a.max_pages * 16);
    int32_t *kept = a.kept + (((size_t)layer * B + b) * H + h) * (size_t)a.keep;
    const int c0 = F + a.n_sinks, n = L - a.n_recent - c0, want = a.keep - a.n_sinks - a.n_recent;      // candidates, and how many of them stay: want < n
    const int pieces = (n - 1) / PIECE + 1;
    uint32_t key[PER];
    auto load = [&](int piece) {
        const uint32_t id = (uint32_t)piece * PIECE + tid * PER, end = (uint32_t)n;    // may pass 2^31 behind the last candidate
        float x[PER];
        typedef float f4u __attribute__((ext_vector_type(4), aligned(4)));
        if (id + PER <= end) {
#pragma unroll
            for (int e = 0; e < PER; e += 4) {
                const f4u v = *reinterpret_cast<const f4u *>(score + c0 + id + e);
#pragma unroll
                for (int q = 0; q < 4; ++q) x[e + q] = v[q];
            }
        } else {
#pragma unroll
            for (int e = 0; e < PER; ++e) x[e] = score[c0 + min(id + e, end - 1u)];
        }
#pragma unroll
        for (int e = 0; e < PER; ++e) key[e] = id + e < end ? score_key(x[e]) : 0u;
    };
    load(0);
    bins[tid] = i32x4_t{0, 0, 0, 0};
    const int32_t *pt = a.table + (size_t)b * a.max_pages;
    int bad = 0;                                            // 1: an entry that names no page, 2: a page that is shared
    for (int lp = (F >> 4) + tid; lp <= (L - 1) >> 4; lp += THREADS) {
        const int page = pt[lp];
        if ((unsigned)page >= (unsigned)a.n_pages) bad |= 1;
        else if (a.ref && !a.dst_table && a.ref[page] > 1) bad |= 2;
    }
    if (a.dst_table)
        for (int lp = ((L - a.keep) >> 4) + tid; lp <= (L - 1) >> 4; lp += THREADS)
            if ((unsigned)a.dst_table[(size_t)b * a.max_pages + lp] >= (unsigned)a.n_pages) bad |= 1;
    uint32_t top = 0u, low = 0u;                            // the largest key, and the complement of the smallest
    for (int pc = 0; pc < pieces; ++pc) {
        if (pc > 0) load(pc);
#pragma unroll
        for (int e = 0; e < PER; ++e) {
            top = max(top, key[e]);
            low = max(low, key[e] ? ~key[e] : 0u);
        }
    }
    top = wave_max(top);
    low = wave_max(low);
    if (lane == 0) { ends[0][wave] = top; ends[1][wave] = low; }
    const int none = __syncthreads_or(bad & 1), shared = __syncthreads_or(bad & 2);
    if (none || shared) {
        if (speaks) { atomicOr(a.flags, (none ? FLAG_BAD_PAGE : 0) | (shared ? FLAG_CAPACITY : 0)); a.evicted[b] = 0; }
        return;
    }
    if (speaks) a.evicted[b] = 1;

    for (uint32_t j = tid; j < (uint32_t)a.n_sinks; j += THREADS) kept[j] = F + (int)j;
    for (uint32_t j = tid; j < (uint32_t)a.n_recent; j += THREADS) kept[a.keep - a.n_recent + (int)j] = L - a.n_recent + (int)j;
    if (want > 0) {
#pragma unroll
        for (int w = 0; w < WAVES; ++w) {
            top = max(top, ends[0][w]);
            low = max(low, ends[1][w]);
        }
        uint32_t lo = ~low;                                 // the bracket: lo .. lo + 2^width - 1
        int width = 32 - __clz((int)(top - lo));
        int stay = want, inside = n;                        // of the bracket's candidates
        while (width > 0 && stay < inside) {                // uniform over the workgroup
            const int shift = max(width - LOG, 0);
            const uint32_t most = width == 32 ? 0xffffffffu : (1u << width) - 1u;
            for (int pc = 0; pc < pieces; ++pc) {
                if (pieces > 1) load(pc);
#pragma unroll
                for (int e = 0; e < PER; ++e) {
                    const uint32_t bin = (key[e] - lo) >> shift;
                    if (key[e] >= lo && key[e] - lo <= most) atomicAdd(reinterpret_cast<int *>(bins) + (bin ^ (BINS - 4)), 1);
                }
            }
            __syncthreads();
            const i32x4_t c = bins[tid];
            bins[tid] = i32x4_t{0, 0, 0, 0};
            const int sum = (c[0] + c[1]) + (c[2] + c[3]), upto = wave_prefix(sum, lane);
            if (lane == 63) part[wave] = upto;
            __syncthreads();
            int above = upto - sum;
#pragma unroll
            for (int w = 0; w < WAVES; ++w) above += w < wave ? part[w] : 0;
            if (above < stay && above + sum >= stay) {       // one thread's
                int i = 3;
#pragma unroll
                for (int q = 3; q > 0; --q)
                    if (i == q && above + c[q] < stay) { above += c[q]; i = q - 1; }
                found[0] = 4 * (THREADS - 1 - tid) + i;
                found[1] = above;
                found[2] = i == 3 ? c[3] : i == 2 ? c[2] : i == 1 ? c[1] : c[0];
            }
            __syncthreads();
            lo += (uint32_t)found[0] << shift;
            stay -= found[1];
            inside = found[2];
            width = shift;
        }
        const uint32_t last = stay == inside ? lo - 1u : lo;         // the smallest key is above 0
        const int equal = stay == inside ? 0 : stay;        // of those with the key `last`, the lowest slots
        int seen_gt = 0, seen_eq = 0;
        for (int pc = 0; pc < pieces; ++pc) {
            if (pieces > 1) load(pc);
            int mine = 0;
#pragma unroll
            for (int e = 0; e < PER; ++e) mine += (key[e] > last ? 1 : 0) + (key[e] == last && key[e] != 0u ? 0x10000 : 0);
            const int x = wave_prefix(mine, lane);          // two sums in one: a piece has at most 2^15 candidates
            __syncthreads();                                // `part` may still be read from the piece before
            if (lane == 63) part[wave] = x;
            __syncthreads();
            int before = x - mine, total = 0;
#pragma unroll
            for (int w = 0; w < WAVES; ++w) {
                const int p = part[w];
                if (w < wave) before += p;
                total += p;
            }
            int gt = seen_gt + (before & 0xffff), eq = seen_eq + (int)((unsigned)before >> 16);
#pragma unroll
            for (int e = 0; e < PER; ++e) {
                const bool is_gt = key[e] > last, is_eq = key[e] == last && key[e] != 0u;
                if (is_gt || (is_eq && eq < equal)) kept[a.n_sinks + gt + min(eq, equal)] = c0 + pc * PIECE + tid * PER + e;
                gt += is_gt ? 1 : 0;
                eq += is_eq ? 1 : 0;
            }
            seen_gt += total & 0xffff;
            seen_eq += (int)((unsigned)total >> 16);
        }
    }
    __syncthreads();                                        // `kept` is written
    // the scores follow, from the last one down: a source lies at or below its target, so below every target of the pieces before
    for (int top = a.keep - a.n_recent; top > 0; top -= THREADS) {
        const int j = top - THREADS + tid;
        float x = 0.f;
        if (j >= 0) x = score[kept[j]];
        asm volatile("" : "+v"(x));
        __syncthreads();                                    // every source of the piece is read
        if (j >= 0) score[L - a.keep + j] = x;
    }
}

// The contents follow.  A workgroup takes 64 dims of K or V of one (head, row, layer), a wave one page of targets at a time, from the last one down.  A source
// lies at or below its target, so the pages of one turn have to be read before any of them is written, and those of later turns lie below: their loads
// are under way while this turn's pages are stored.  Places of a page that no token moves to keep what they hold.
// Bytes bound it: 8 layers of 32 heads of 128, 2048 of 2560 tokens: 0.6 GB in 124 us, 4.9 TB/s.  Of 16003 tokens (4 layers of 40 heads) the 2048 that stay are an eighth, but
// a page's K holds 16 bytes of each token beside each other, and V two: with whole lines of 128 bytes that is 1.1 GB, in 242 us.
enum { EV_WAVES = 16, EV_GROUP = 2, EV_ROW_LDS = 272, EV_PAGE_LDS = 8 * EV_ROW_LDS };
struct EvictPlan { int to, slot, page; };                   // of a page of targets: its number, and for place lane % 16 the slot that moves there (-1: none) and its page
struct EvictMove {
    const int32_t *kept, *pt, *dt;
    int base, moved, low;
    __device__ __forceinline__ EvictPlan slots(int lp, int lane) const {
        EvictPlan p;
        const int j = lp * 16 + (lane & 15) - base;
        p.to = dt[max(lp, low)];
        p.slot = j >= 0 && j < moved ? kept[j] : -1;
        p.page = 0;
        return p;
    }
    __device__ __forceinline__ void look_up(EvictPlan &p) const { p.page = p.slot >= 0 ? pt[p.slot >> 4] : p.to; }
};

// fp32 rows, and 16-bit K (runs of 8 dims, [dim / 8][token]): they move as they lie, 16 bytes a lane.  block(page): the page's 64 dims.  They pass the caches by
// (13B, 2048 of 16003 tokens 277 -> 267 us in all, fp32 132 -> 126).
template <bool BF, class Block>
__device__ __forceinline__ void evict_move_rows(const EvictMove &m, int Dh, int last, int lane, int wave, Block block) {
    constexpr int N = BF ? 2 : 4;
    const int place = lane & 15, sub = lane >> 4;
    auto at = [&](int page, int tok, int i) -> u32x4_t * {
        if (BF) return reinterpret_cast<u32x4_t *>(block(page)) + (i * 4 + sub) * 16 + tok;                   // sub: the run of 8 dims
        return reinterpret_cast<u32x4_t *>(block(page) + tok * Dh) + place;                                    // 16 lanes to the 64 dims of token 4 i + sub
    };
    auto load = [&](const EvictPlan &p, u32x4_t (&x)[N]) {
        const int tok = p.slot >= 0 ? p.slot & 15 : place;
#pragma unroll
        for (int i = 0; i < N; ++i) x[i] = __builtin_nontemporal_load(BF ? at(p.page, tok, i) : at(__shfl(p.page, i * 4 + sub, 64), __shfl(tok, i * 4 + sub, 64), i));
    };
    EvictPlan now = m.slots(last - wave, lane), next = m.slots(last - wave - EV_WAVES, lane), after = m.slots(last - wave - 2 * EV_WAVES, lane);
    m.look_up(now);
    m.look_up(next);
    u32x4_t x[N], y[N];
    if (last - wave >= m.low) load(now, x);
    for (int lp = last - wave; lp + wave >= m.low; lp -= EV_WAVES) {            // uniform over the workgroup
        const bool live = lp >= m.low;                       // wave-uniform
        const int to = now.to;
        if (lp - EV_WAVES >= m.low) load(next, y);
        now = next;
        next = after;
        m.look_up(next);
        after = m.slots(lp - 3 * EV_WAVES, lane);
#pragma unroll
        for (int i = 0; i < N; ++i) asm volatile("" : "+v"(x[i]));               // this turn's sources have arrived
        __syncthreads();
        if (live) {
#pragma unroll
            for (int i = 0; i < N; ++i) __builtin_nontemporal_store(x[i], at(to, BF ? place : i * 4 + sub, i));
        }
#pragma unroll
        for (int i = 0; i < N; ++i) x[i] = y[i];
    }
}

// 16-bit V lies by dim: the 16 tokens of the 64 dims of a source page go to LDS as [dword][dim] (a dword: two tokens), loaded as whole lines, half a dim a lane; since every lane moves
// the same tokens, of one dim, one is picked by an offset that the wave shares, without bank conflicts.  (Neighbouring waves read the pages at their ends twice: through the caches;
// past them 7B took 165 us instead of 154 in all.)  Picked from registers, by a register number that the wave shares, a page of targets took
// twice as long as its loads and stores (7B, 8 layers, 2048 of 2560 tokens: 268 us).
template <class Block>
__device__ __forceinline__ void evict_move_v(const EvictMove &m, int last, int lane, int wave, char *lds, Block block) {
    typedef uint16_t __attribute__((may_alias)) half_word;   // of what is written as dwords
    const int place = lane & 15;
    u32x4_t s[EV_GROUP][2];
    uint32_t rest = 0;                                       // tokens that begin a source page which is not asked for yet
    int pick = 0;                                            // of token `place`: the group of its page, and where it will lie in LDS
    EvictPlan now;
    auto fetch = [&] {
#pragma unroll
        for (int g = 0; g < EV_GROUP; ++g)
            if (rest) {                                      // wave-uniform
                const u32x4_t *from = reinterpret_cast<const u32x4_t *>(block(__builtin_amdgcn_readlane(now.page, __builtin_ctz(rest)))) + lane;
                s[g][0] = from[0];
                s[g][1] = from[64];
                rest &= rest - 1u;
            }
    };
    auto begin = [&] {
        const int tok = now.slot >= 0 ? now.slot & 15 : place, before = __shfl_up(now.page, 1, 64);
        rest = (uint32_t)__ballot(lane < 16 && (lane == 0 || now.page != before));
        const int nth = __popc(rest & ((2u << place) - 1u)) - 1, at = v_perm(tok);
        pick = (nth / EV_GROUP) << 16 | (nth % EV_GROUP * EV_PAGE_LDS + (at >> 1) * EV_ROW_LDS + (at & 1) * 2);
        fetch();
    };
    now = m.slots(last - wave, lane);
    EvictPlan next = m.slots(last - wave - EV_WAVES, lane), after = m.slots(last - wave - 2 * EV_WAVES, lane);
    m.look_up(now);
    m.look_up(next);
    if (last - wave >= m.low) begin();
    for (int lp = last - wave; lp + wave >= m.low; lp -= EV_WAVES) {            // uniform over the workgroup
        const bool live = lp >= m.low;                       // wave-uniform
        const int to = now.to;
        uint32_t w[16];
        if (live) {
#pragma unroll
            for (int t = 0; t < 16; ++t) w[t] = 0u;
            for (int group = 0;; ++group) {
#pragma unroll
                for (int g = 0; g < EV_GROUP; ++g)
#pragma unroll
                    for (int d = 0; d < 8; ++d)
                        *reinterpret_cast<uint32_t *>(lds + g * EV_PAGE_LDS + ((lane & 1) * 4 + (d & 3)) * EV_ROW_LDS + ((lane >> 1) + (d >> 2) * 32) * 4) = s[g][d >> 2][d & 3];
                const bool more = rest != 0;
                if (more) fetch();
#pragma unroll
                for (int t = 0; t < 16; ++t) {
                    const int o = __builtin_amdgcn_readlane(pick, t);
                    if (o >> 16 == group) w[t] = *reinterpret_cast<const half_word *>(lds + (o & 0xffff) + lane * 4);
                }
                if (!more) break;
            }
        }
        now = next;
        next = after;
        m.look_up(next);
        after = m.slots(lp - 3 * EV_WAVES, lane);
        if (lp - EV_WAVES >= m.low) begin();
        u32x4_t x[2];
        if (live) {
            uint32_t y[16];
#pragma unroll
            for (int t = 0; t < 16; ++t) y[v_perm(t)] = w[t];
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e >> 2][e & 3] = y[2 * e] | (y[2 * e + 1] << 16);
        }
        asm volatile("" : "+v"(x[0]), "+v"(x[1]));
        __syncthreads();                                     // every wave's sources have gone through LDS
        if (live) {
            u32x4_t *out = reinterpret_cast<u32x4_t *>(block(to)) + lane * 2;
            out[0] = x[0];
            out[1] = x[1];
        }
    }
}

template <bool BF>
__global__ __launch_bounds__(EV_WAVES * 64, 8) void evict_move_kernel(EvictArgs a, int Dh) {
    __shared__ __attribute__((aligned(16))) char lds[BF ? EV_WAVES * EV_GROUP * EV_PAGE_LDS : 16];
    const int tid = (int)threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int parts = Dh >> 6, h = (int)blockIdx.x / (2 * parts), part = (int)blockIdx.x % parts, is_v = (int)blockIdx.x / parts & 1;
    const int b = blockIdx.y, layer = blockIdx.z, H = (int)gridDim.x / (2 * parts), B = gridDim.y;
    if (!a.evicted[b]) return;                              // uniform over the workgroup
    const int L = a.seq_len[b], base = L - a.keep, moved = a.dst_table ? a.keep : a.keep - a.n_recent;
    if (tid == 0 && blockIdx.x == 0 && layer == 0) a.first[b] = base;         // nobody reads it here
    if (moved == 0) return;
    EvictMove m;
    m.kept = a.kept + (((size_t)layer * B + b) * H + h) * (size_t)a.keep;
    m.pt = a.table + (size_t)b * a.max_pages;
    m.dt = (a.dst_table ? a.dst_table : a.table) + (size_t)b * a.max_pages;
    m.base = base; m.moved = moved; m.low = base >> 4;
    const int last = (base + moved - 1) >> 4;
    typedef typename Act<BF>::type elem;
    elem *pages = reinterpret_cast<elem *>(is_v ? a.v : a.k) + (BF ? part * 64 * 16 : part * 64);
    auto block = [&](int page) { return pages + kv_block_base(layer, a.n_pages, page, H, h, Dh); };
    if (BF && is_v) evict_move_v(m, last, lane, wave, lds + wave * EV_GROUP * EV_PAGE_LDS, block);
    else            evict_move_rows<BF>(m, Dh, last, lane, wave, block);
}

// Scores of accepted nodes: one thread walks the path for one head, as kv_compact walks it.
__global__ __launch_bounds__(256) void score_compact_kernel(const int32_t *n_acc, const int32_t *path, EvictArgs a, int H, int plen) {
    __shared__ int32_t walk[HYDRA_MAX_T];
    const int b = blockIdx.y, layer = blockIdx.z, h = blockIdx.x * 256 + (int)threadIdx.x;
    const int L = a.seq_len[b];
    for (int j = threadIdx.x; j < plen; j += 256) walk[j] = path[(size_t)b * plen + j];
    __syncthreads();
    if (L < 0 || L > a.max_pages * 16 - a.T || h >= H) return;                 // such a row was skipped by the attention
    float *score = a.score + (((size_t)layer * a.score_rows + b) * H + h) * ((size_t)a.max_pages * 16) + L;
    const int n = min(max(n_acc[b], 0), plen);
    int prev = -1;
    for (int j = 0; j < n; ++j) {
        const int from = walk[j];
        if (from <= prev || from < j || from >= a.T) {
            if (h == 0 && layer == 0) atomicOr(a.flags, FLAG_BAD_PATH);
            return;
        }
        if (from != j) score[j] = score[from];
        prev = from;
    }
}

// A page stays if it holds a slot from the root's window on, up to the last token, or one of the sinks in front of it.
__global__ __launch_bounds__(256) void release_span_kernel(int32_t *table, int32_t *ref, int n_pages, int max_pages, const int32_t *seq_len, const int32_t *first,
                                                            int n_sinks, int window, int32_t *lo, int32_t *flags) {
    const int b = blockIdx.y, i = blockIdx.x * 256 + threadIdx.x;
    const int L = seq_len[b], F = first ? first[b] : 0;
    if (L < 0 || F < 0 || F > L) {
        if (i == 0) { atomicOr(flags, FLAG_CAPACITY); if (lo) lo[b] = -1; }
        return;
    }
    const int low = window > 0 ? max(F, L + 1 - window) : F, S = F + min(n_sinks, low - F);
    if (i == 0 && lo) lo[b] = low;
    if (i >= max_pages) return;
    const int64_t s = (int64_t)i * 16;
    if ((low < L && s < L && s + 16 > low) || (S > F && s < S && s + 16 > F)) return;
    const int page = table[(size_t)b * max_pages + i];
    if (page < 0) return;
    table[(size_t)b * max_pages + i] = -1;
    if (page >= n_pages) { atomicOr(flags, FLAG_BAD_PAGE); return; }
    if (atomicSub(&ref[page], 1) <= 0) {                    // was free already: stays free
        atomicAdd(&ref[page], 1);
        atomicOr(flags, FLAG_BAD_PAGE);
    }
}

static EvictArgs evict_args(hydra_ctx *c, const int32_t *seq_len, const hydra_kv_span *span) {
    EvictArgs a = {};
    a.table = span->kv.page_table; a.seq_len = seq_len; a.first = span->first; a.flags = flags_dev(c);
    a.score = span->score; a.k = span->kv.k_pages; a.v = span->kv.v_pages;
    a.max_pages = span->kv.max_pages; a.n_pages = span->kv.n_pages; a.n_sinks = span->n_sinks; a.score_rows = span->score_rows; a.T = c->tree.T;
    return a;
}

int launch_kv_evict(hydra_ctx *c, hipStream_t s, int B, const int32_t *seq_len, const hydra_kv_span *span, int keep, int n_recent, int slack, const int32_t *dst_table,
                    const int32_t *ref, int32_t *kept, int32_t *evicted) {
    EvictArgs a = evict_args(c, seq_len, span);
    a.dst_table = dst_table; a.ref = ref; a.kept = kept; a.evicted = evicted; a.n_recent = n_recent; a.keep = keep; a.slack = slack;
    const int H = c->m.n_heads, NL = c->m.n_layers;
    const int64_t held = span->span_hint > 0 ? span->span_hint : span->kv.seq_len_hint > 0 ? span->kv.seq_len_hint : (int64_t)span->kv.max_pages * 16;
    const int64_t n = held - span->n_sinks - n_recent;       // candidates, as far as the host knows
    const dim3 sgrid(H, B, NL);
    if (n <= 1024)       hipLaunchKernelGGL((evict_select_kernel<256, 4>), sgrid, dim3(256), 0, s, a);
    else if (n <= 4096)  hipLaunchKernelGGL((evict_select_kernel<512, 8>), sgrid, dim3(512), 0, s, a);
    else if (n <= 16384) hipLaunchKernelGGL((evict_select_kernel<1024, 16>), sgrid, dim3(1024), 0, s, a);
    else                 hipLaunchKernelGGL((evict_select_kernel<1024, 32>), sgrid, dim3(1024), 0, s, a);
    HYDRA_LAUNCH_CHECK("evict_select_kernel");
    const dim3 grid(2 * H * (c->m.head_dim / 64), B, NL), block(EV_WAVES * 64);
    if (c->bf16) hipLaunchKernelGGL(evict_move_kernel<true>, grid, block, 0, s, a, c->m.head_dim);
    else         hipLaunchKernelGGL(evict_move_kernel<false>, grid, block, 0, s, a, c->m.head_dim);
    HYDRA_LAUNCH_CHECK("evict_move_kernel");
    return HYDRA_OK;
}

int launch_score_compact(hydra_ctx *c, hipStream_t s, int B, const int32_t *n_acc, const int32_t *path, const int32_t *seq_len, const hydra_kv_span *span) {
    const EvictArgs a = evict_args(c, seq_len, span);
    const int H = c->m.n_heads;
    hipLaunchKernelGGL(score_compact_kernel, dim3(ceil_div(H, 256), B, c->m.n_layers), dim3(256), 0, s, n_acc, path, a, H, c->tree.max_depth + 1);
    HYDRA_LAUNCH_CHECK("score_compact_kernel");
    return HYDRA_OK;
}

int launch_release_span(hydra_ctx *c, hipStream_t s, int B, const hydra_pages *pages, const int32_t *seq_len, const hydra_kv_span *span, int32_t *lo) {
    hipLaunchKernelGGL(release_span_kernel, dim3(ceil_div(pages->max_pages, 256), B), dim3(256), 0, s, pages->page_table, pages->ref, pages->n_pages, pages->max_pages,
                       seq_len, span->first, span->n_sinks, span->window, lo, flags_dev(c));
    HYDRA_LAUNCH_CHECK("release_span_kernel");
    return HYDRA_OK;
}

}  // namespace hydra
