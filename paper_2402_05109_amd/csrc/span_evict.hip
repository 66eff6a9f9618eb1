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

// One workgroup per (head, row, layer) finds what it keeps.  The key of the last token that is kept (`want` tokens have it or a larger one) is found from
// its upper bits down, two at a time, by counting; tokens with that very key are taken from the lowest slot on.  A thread holds EV_PER neighbouring
// candidates in registers, so up to EV_PIECE are read once; longer rows are read again for every count.
enum { EV_THREADS = 1024, EV_PER = 8, EV_PIECE = EV_THREADS * EV_PER };
__global__ __launch_bounds__(EV_THREADS) void evict_select_kernel(EvictArgs a) {
    __shared__ int cnt[3][3];
    __shared__ int part[EV_THREADS / 64];
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
    const int32_t *pt = a.table + (size_t)b * a.max_pages;
    int bad = 0;                                            // 1: an entry that names no page, 2: a page that is shared
    for (int lp = (F >> 4) + tid; lp <= (L - 1) >> 4; lp += EV_THREADS) {
        const int page = pt[lp];
        if ((unsigned)page >= (unsigned)a.n_pages) bad |= 1;
        else if (a.ref && !a.dst_table && a.ref[page] > 1) bad |= 2;
    }
    if (a.dst_table)
        for (int lp = ((L - a.keep) >> 4) + tid; lp <= (L - 1) >> 4; lp += EV_THREADS)
            if ((unsigned)a.dst_table[(size_t)b * a.max_pages + lp] >= (unsigned)a.n_pages) bad |= 1;
    const int none = __syncthreads_or(bad & 1), shared = __syncthreads_or(bad & 2);
    if (none || shared) {
        if (speaks) { atomicOr(a.flags, (none ? FLAG_BAD_PAGE : 0) | (shared ? FLAG_CAPACITY : 0)); a.evicted[b] = 0; }
        return;
    }
    if (speaks) a.evicted[b] = 1;

    float *score = a.score + (((size_t)layer * a.score_rows + b) * H + h) * ((size_t)a.max_pages * 16);
    int32_t *kept = a.kept + (((size_t)layer * B + b) * H + h) * (size_t)a.keep;
    const int c0 = F + a.n_sinks, n = L - a.n_recent - c0, want = a.keep - a.n_sinks - a.n_recent;      // candidates, and how many of them stay: want < n
    for (int j = tid; j < a.n_sinks; j += EV_THREADS) kept[j] = F + j;
    for (int j = tid; j < a.n_recent; j += EV_THREADS) kept[a.keep - a.n_recent + j] = L - a.n_recent + j;
    const int pieces = (n + EV_PIECE - 1) / EV_PIECE;
    uint32_t key[EV_PER];
    auto load = [&](int piece) {
        const int id = piece * EV_PIECE + tid * EV_PER;
        float x[EV_PER];
#pragma unroll
        for (int e = 0; e < EV_PER; ++e) x[e] = score[c0 + min(id + e, n - 1)];
#pragma unroll
        for (int e = 0; e < EV_PER; ++e) key[e] = id + e < n ? score_key(x[e]) : 0u;
    };
    if (want > 0) {
        load(0);
        if (tid < 9) cnt[tid / 3][tid % 3] = 0;
        __syncthreads();
        int turn = 0;
        // how many candidates have a key of at least t[0], t[1], t[2]
        auto count = [&](const uint32_t (&t)[3], int (&c)[3]) {
            int s[3] = {0, 0, 0};
            for (int pc = 0; pc < pieces; ++pc) {
                if (pieces > 1) load(pc);
#pragma unroll
                for (int e = 0; e < EV_PER; ++e)
#pragma unroll
                    for (int i = 0; i < 3; ++i) s[i] += __popcll(__ballot(key[e] >= t[i]));
            }
            if (lane == 0)
#pragma unroll
                for (int i = 0; i < 3; ++i) atomicAdd(&cnt[turn][i], s[i]);
            __syncthreads();
#pragma unroll
            for (int i = 0; i < 3; ++i) c[i] = cnt[turn][i];
            const int again = turn == 0 ? 2 : turn - 1;     // read by everybody before this barrier, next used behind the next one
            if (tid < 3) cnt[again][tid] = 0;
            turn = turn == 2 ? 0 : turn + 1;
        };
        uint32_t last = 0u;
        for (int bit = 30; bit >= 0; bit -= 2) {
            const uint32_t t[3] = {last | (1u << bit), last | (2u << bit), last | (3u << bit)};
            int c[3];
            count(t, c);
            last = c[2] >= want ? t[2] : c[1] >= want ? t[1] : c[0] >= want ? t[0] : last;
            if (c[2] == want || c[1] == want || c[0] == want) break;        // nothing is left to tell apart: the largest such bound has just these
        }
        int above = 0;
        if (last != 0xffffffffu) {
            const uint32_t t[3] = {last + 1u, last + 1u, last + 1u};
            int c[3];
            count(t, c);
            above = c[0];
        }
        const int equal = want - above;                     // of those with the key `last`, the lowest slots
        int seen_gt = 0, seen_eq = 0;
        for (int pc = 0; pc < pieces; ++pc) {
            if (pieces > 1) load(pc);
            int mine = 0;
#pragma unroll
            for (int e = 0; e < EV_PER; ++e) mine += (key[e] > last ? 1 : 0) + (key[e] == last && key[e] != 0u ? 0x10000 : 0);
            int x = mine;
#pragma unroll
            for (int d = 1; d < 64; d <<= 1) {
                const int y = __shfl_up(x, d);
                if (lane >= d) x += y;
            }
            __syncthreads();                                // `part` may still be read from the piece before
            if (lane == 63) part[wave] = x;
            __syncthreads();
            int before = x - mine, total = 0;
            for (int w = 0; w < EV_THREADS / 64; ++w) {
                const int p = part[w];
                if (w < wave) before += p;
                total += p;
            }
            int gt = seen_gt + (before & 0xffff), eq = seen_eq + (before >> 16);
#pragma unroll
            for (int e = 0; e < EV_PER; ++e) {
                const bool is_gt = key[e] > last, is_eq = key[e] == last && key[e] != 0u;
                if (is_gt || (is_eq && eq < equal)) kept[a.n_sinks + gt + min(eq, equal)] = c0 + pc * EV_PIECE + tid * EV_PER + e;
                gt += is_gt ? 1 : 0;
                eq += is_eq ? 1 : 0;
            }
            seen_gt += total & 0xffff;
            seen_eq += total >> 16;
        }
    }
    __syncthreads();                                        // `kept` is written
    // the scores follow, from the last one down: a source lies at or below its target, so below every target of the pieces before
    const int moved = a.keep - a.n_recent;
    for (int top = moved; top > 0; top -= EV_THREADS) {
        const int j = top - EV_THREADS + tid;
        float x = 0.f;
        if (j >= 0) x = score[kept[j]];
        asm volatile("" : "+v"(x));
        __syncthreads();                                    // every source of the piece is read
        if (j >= 0) score[L - a.keep + j] = x;
    }
}

// The contents follow: a wave takes a page of targets at a time, from the last one down, and a workgroup one of K and V of a (head, row, layer).  A source
// lies at or below its target, so the pages of one turn have to be read before any of them is written, and those of later turns lie below.
// Places of a page that no token moves to keep what they hold.
enum { EV_WAVES = 8 };
template <bool BF, int DH>
__global__ __launch_bounds__(EV_WAVES * 64) void evict_move_kernel(EvictArgs a) {
    const int tid = (int)threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int h = blockIdx.x >> 1, is_v = blockIdx.x & 1, b = blockIdx.y, layer = blockIdx.z, H = gridDim.x >> 1, B = gridDim.y;
    if (!a.evicted[b]) return;                              // uniform over the workgroup
    const int L = a.seq_len[b], base = L - a.keep, moved = a.dst_table ? a.keep : a.keep - a.n_recent;
    if (moved == 0) return;
    const int32_t *kept = a.kept + (((size_t)layer * B + b) * H + h) * (size_t)a.keep;
    const int32_t *pt = a.table + (size_t)b * a.max_pages, *dt = (a.dst_table ? a.dst_table : a.table) + (size_t)b * a.max_pages;
    const int last = (base + moved - 1) >> 4, low = base >> 4;
    typedef typename Act<BF>::type elem;
    elem *pages = reinterpret_cast<elem *>(is_v ? a.v : a.k);
    auto block = [&](int page) { return pages + kv_block_base(layer, a.n_pages, page, H, h, DH); };
    constexpr int N = BF ? DH / 32 : DH / 16;               // 16-byte pieces of a page per lane
    for (int p0 = last; p0 >= low; p0 -= EV_WAVES) {
        const int lp = p0 - wave;
        const bool live = lp >= low;                        // wave-uniform
        const int to = dt[max(lp, low)];
        u32x4_t x[N];
        if (live) {
            // lane t of the first 16 (and again of the others) knows where the token of place t comes from
            const int place = lane & 15, j = lp * 16 + place - base;
            const bool in = j >= 0 && j < moved;
            const int src = in ? kept[j] : 0;
            const int page = in ? pt[src >> 4] : to, tok = in ? src & 15 : place;
            if (BF && !is_v) {                              // runs of 8 dims, [dim / 8][token]
                const u32x4_t *from = reinterpret_cast<const u32x4_t *>(block(page)) + tok;
#pragma unroll
                for (int i = 0; i < N; ++i) x[i] = from[(i * 4 + (lane >> 4)) * 16];
            } else if (BF) {                                // 2 bytes, [dim][place]
#pragma unroll
                for (int i = 0; i < N / 2; ++i) {
                    uint32_t w[16];
#pragma unroll
                    for (int t = 0; t < 16; ++t)
                        w[v_perm(t)] = reinterpret_cast<const uint16_t *>(block(__builtin_amdgcn_readlane(page, t)))[(i * 64 + lane) * 16 + v_perm(__builtin_amdgcn_readlane(tok, t))];
#pragma unroll
                    for (int q = 0; q < 2; ++q)
#pragma unroll
                        for (int e = 0; e < 4; ++e) x[2 * i + q][e] = w[8 * q + 2 * e] | (w[8 * q + 2 * e + 1] << 16);
                }
            } else {                                        // a token's dims in a row
                constexpr int PER = DH / 4;                 // lanes of a token
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    const int t = (i * 64 + lane) / PER;
                    const int pg = __shfl(page, t, 64), tk = __shfl(tok, t, 64);
                    x[i] = reinterpret_cast<const u32x4_t *>(block(pg))[tk * PER + lane % PER];
                }
            }
        }
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __syncthreads();                                    // every source of this turn has arrived
        if (live) {
            u32x4_t *out = reinterpret_cast<u32x4_t *>(block(to));
            if (BF && !is_v) {
#pragma unroll
                for (int i = 0; i < N; ++i) out[(i * 4 + (lane >> 4)) * 16 + (lane & 15)] = x[i];
            } else if (BF) {
#pragma unroll
                for (int i = 0; i < N; ++i) out[((i >> 1) * 64 + lane) * 2 + (i & 1)] = x[i];
            } else {
#pragma unroll
                for (int i = 0; i < N; ++i) out[i * 64 + lane] = x[i];
            }
        }
    }
}

__global__ void evict_finish_kernel(const int32_t *seq_len, const int32_t *evicted, int32_t *first, int keep, int B) {
    const int b = blockIdx.x * blockDim.x + threadIdx.x;
    if (b < B && evicted[b]) first[b] = seq_len[b] - keep;
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
    hipLaunchKernelGGL(evict_select_kernel, dim3(H, B, NL), dim3(EV_THREADS), 0, s, a);
    HYDRA_LAUNCH_CHECK("evict_select_kernel");
    const dim3 grid(2 * H, B, NL), block(EV_WAVES * 64);
    if (c->bf16) {
        if (c->m.head_dim == 128) hipLaunchKernelGGL((evict_move_kernel<true, 128>), grid, block, 0, s, a);
        else                      hipLaunchKernelGGL((evict_move_kernel<true, 64>), grid, block, 0, s, a);
    } else {
        if (c->m.head_dim == 128) hipLaunchKernelGGL((evict_move_kernel<false, 128>), grid, block, 0, s, a);
        else                      hipLaunchKernelGGL((evict_move_kernel<false, 64>), grid, block, 0, s, a);
    }
    HYDRA_LAUNCH_CHECK("evict_move_kernel");
    hipLaunchKernelGGL(evict_finish_kernel, dim3(ceil_div(B, 256)), dim3(256), 0, s, seq_len, evicted, span->first, keep, B);
    HYDRA_LAUNCH_CHECK("evict_finish_kernel");
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
