// The pages of a cache as a pool: rows take pages, give them back, share them and move them; copies of whole pages.
//
// The tables and counts are small integers in device memory, so that no call waits for the host and all of them can be captured
// into a graph.  Every result is a function of the inputs alone: pages are handed out lowest first, by row, and counts are sums.
#include <algorithm>
#include <climits>

#include "device_common.h"
#include "internal.h"

namespace hydra {

typedef __attribute__((ext_vector_type(4))) uint32_t u32x4_t;

enum { PG_THREADS = 1024, PG_WAVES = PG_THREADS / 64 };

// Exclusive sum of v over the workgroup's threads, and the total.  `part`: PG_WAVES ints of shared memory; two barriers.
__device__ __forceinline__ int block_scan(int v, int *part, int &total) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int x = v;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const int y = __shfl_up(x, d);
        if (lane >= d) x += y;
    }
    __syncthreads();                                        // `part` may still be read from the call before
    if (lane == 63) part[wave] = x;
    __syncthreads();
    int before = 0;
    total = 0;
    for (int w = 0; w < PG_WAVES; ++w) {
        const int p = part[w];
        if (w < wave) before += p;
        total += p;
    }
    return before + x - v;
}

// The `want` lowest free pages into list[]; returns how many there are (at most want).  Uniform over the workgroup.  A thread looks at 16 counts at a
// time, all of them in one round trip.
__device__ __forceinline__ int lowest_free(const int32_t *ref, int n_pages, int want, int32_t *list, int *part) {
    typedef int32_t i4 __attribute__((ext_vector_type(4), aligned(4)));
    enum { PER = 16 };
    int found = 0;
    for (int p0 = 0; p0 < n_pages && found < want; p0 += PG_THREADS * PER) {
        const int p = p0 + (int)threadIdx.x * PER;
        uint32_t free_mask = 0;
        if (p + PER <= n_pages) {
            i4 v[PER / 4];
#pragma unroll
            for (int e = 0; e < PER / 4; ++e) v[e] = *reinterpret_cast<const i4 *>(ref + p + 4 * e);
#pragma unroll
            for (int e = 0; e < PER; ++e) free_mask |= (v[e >> 2][e & 3] == 0 ? 1u : 0u) << e;
        } else {
            for (int e = 0; p + e < n_pages; ++e) free_mask |= (ref[p + e] == 0 ? 1u : 0u) << e;
        }
        int total;
        int at = found + block_scan(__popc(free_mask), part, total);
        for (; free_mask && at < want; free_mask &= free_mask - 1) list[at++] = p + __ffs(free_mask) - 1;
        found += total;
    }
    return min(found, want);
}

struct PgRange { int first, last; bool ok; };
// logical pages [lo / 16, ceil(hi / 16)) of a row that is to hold slots lo .. hi - 1
__device__ __forceinline__ PgRange page_range(const int32_t *lo, const int32_t *hi, int extra, int b) {
    const int64_t a = lo ? lo[b] : 0, e = (int64_t)hi[b] + extra;
    PgRange r;
    r.ok = a >= 0 && hi[b] >= 0;
    r.first = (int)(a >> 4);
    r.last = (int)min((e + 15) >> 4, (int64_t)0x7fffffff);
    return r;
}

struct PgRow { int first, last, lacks, start; };             // its logical pages; how many have none (-1: no such range); where its pages begin among all
enum { PG_ROWS = 1024, PG_GROUP = 4 };

// How many entries each row lacks, and the first of them: a wave takes G rows and requests A pieces of 64 entries of each at a time.
template <int G, int A>
__device__ __forceinline__ void count_lacking(const int32_t *table, int max_pages, int B, PgRow *rows, int lane, int wave) {
    for (int b0 = wave; b0 < B; b0 += PG_WAVES * G) {
        int first[G], last[G], need[G], found[G], most = 0;
#pragma unroll
        for (int r = 0; r < G; ++r) {
            const int b = b0 + r * PG_WAVES;
            first[r] = last[r] = need[r] = 0;
            if (b < B) { first[r] = rows[b].first; last[r] = rows[b].last; }
            found[r] = last[r];
            most = max(most, last[r] - first[r]);
        }
        for (int i0 = 0; i0 < most; i0 += 64 * A) {
            int v[G][A];
#pragma unroll
            for (int r = 0; r < G; ++r)
#pragma unroll
                for (int u = 0; u < A; ++u) {
                    const int i = first[r] + i0 + u * 64 + lane, b = min(b0 + r * PG_WAVES, B - 1);      // no load behind a condition
                    v[r][u] = table[(size_t)b * max_pages + min(i, max_pages - 1)];
                    v[r][u] = i < last[r] ? v[r][u] : 0;
                }
#pragma unroll
            for (int r = 0; r < G; ++r)
#pragma unroll
                for (int u = 0; u < A; ++u) {
                    const uint64_t m = __ballot(v[r][u] < 0);
                    if (m && !need[r]) found[r] = first[r] + i0 + u * 64 + __builtin_ctzll(m);
                    need[r] += __popcll(m);
                }
        }
        if (lane == 0)
#pragma unroll
            for (int r = 0; r < G; ++r) {
                const int b = b0 + r * PG_WAVES;
                if (b < B && rows[b].lacks == 0) { rows[b].first = found[r]; rows[b].lacks = need[r]; }
            }
    }
}

// Four rows of a wave go together, their loads in flight at once, and what is known of a row (PgRow) lies in shared memory for up to PG_ROWS rows: a call
// is a chain of a dozen round trips whatever it hands out (64 rows of 2048 entries 39 us with a row after the other, 16 now).
// ws: PgRow [B], then the pages handed out (at most n_pages).
__global__ __launch_bounds__(PG_THREADS) void pages_reserve_kernel(int32_t *table, int32_t *ref, int n_pages, int max_pages, int B, const int32_t *lo,
                                                                    const int32_t *hi, int extra, int32_t *ws, int32_t *ok, int32_t *flags) {
    __shared__ int part[PG_WAVES];
    __shared__ PgRow in_lds[PG_ROWS];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    PgRow *rows = B <= PG_ROWS ? in_lds : reinterpret_cast<PgRow *>(ws);
    int32_t *list = ws + 4 * (size_t)B;
    for (int b = threadIdx.x; b < B; b += PG_THREADS) {
        const PgRange r = page_range(lo, hi, extra, b);
        const bool good = r.ok && (int64_t)(lo ? lo[b] : 0) <= (int64_t)hi[b] + extra && r.last <= max_pages;
        rows[b] = PgRow{good ? r.first : 0, good ? r.last : 0, good ? 0 : -1, 0};
    }
    __syncthreads();
    if (B <= PG_WAVES) count_lacking<1, 16>(table, max_pages, B, rows, lane, wave);
    else               count_lacking<PG_GROUP, 4>(table, max_pages, B, rows, lane, wave);
    __syncthreads();
    int all = 0;
    for (int b0 = 0; b0 < B; b0 += PG_THREADS) {
        const int b = b0 + (int)threadIdx.x;
        int total;
        const int at = block_scan(b < B ? max(rows[b].lacks, 0) : 0, part, total) + all;
        if (b < B) rows[b].start = at;
        all = min(all + total, 0x3fffffff);
    }
    const int found = lowest_free(ref, n_pages, min(all, n_pages), list, part);
    __syncthreads();
    for (int b = threadIdx.x; b < B; b += PG_THREADS) {
        const PgRow r = rows[b];
        const bool served = r.lacks == 0 || (r.lacks > 0 && r.start + r.lacks <= found);
        if (!served) { atomicOr(flags, FLAG_CAPACITY); rows[b].lacks = 0; }
        if (ok) ok[b] = served ? 1 : 0;
    }
    __syncthreads();
    for (int b0 = wave; b0 < B; b0 += PG_WAVES * PG_GROUP) {
        PgRow r[PG_GROUP];
        int most = 0;                                        // the longest way from a row's first entry without a page to its end
#pragma unroll
        for (int k = 0; k < PG_GROUP; ++k) {
            const int b = b0 + k * PG_WAVES;
            r[k] = b < B ? rows[b] : PgRow{0, 0, 0, 0};
            if (r[k].lacks > 0) most = max(most, r[k].last - r[k].first);
        }
        for (int i0 = 0; i0 < most; i0 += 64) {
            int page[PG_GROUP];
            bool lack[PG_GROUP];
#pragma unroll
            for (int k = 0; k < PG_GROUP; ++k) {
                const int i = r[k].first + i0 + lane;
                const int v = table[(size_t)min(b0 + k * PG_WAVES, B - 1) * max_pages + min(i, max_pages - 1)];
                lack[k] = r[k].lacks > 0 && i < r[k].last && v < 0;
            }
#pragma unroll
            for (int k = 0; k < PG_GROUP; ++k) {
                const uint64_t m = __ballot(lack[k]);
                page[k] = list[lack[k] ? r[k].start + __popcll(m & ((1ull << lane) - 1ull)) : 0];
                r[k].start += __popcll(m);
            }
#pragma unroll
            for (int k = 0; k < PG_GROUP; ++k)
                if (lack[k]) {
                    table[(size_t)(b0 + k * PG_WAVES) * max_pages + r[k].first + i0 + lane] = page[k];
                    ref[page[k]] = 1;
                }
        }
    }
}

// an entry gives its page back
__device__ __forceinline__ void drop_page(int32_t *ref, int n_pages, int page, int32_t *flags) {
    if ((unsigned)page >= (unsigned)n_pages) { atomicOr(flags, FLAG_BAD_PAGE); return; }
    if (atomicSub(&ref[page], 1) <= 0) {                    // was free already: stays free
        atomicAdd(&ref[page], 1);
        atomicOr(flags, FLAG_BAD_PAGE);
    }
}

__global__ __launch_bounds__(256) void pages_release_kernel(int32_t *table, int32_t *ref, int n_pages, int max_pages, const int32_t *lo, const int32_t *hi,
                                                             int32_t *flags) {
    const int b = blockIdx.y, i = blockIdx.x * 256 + threadIdx.x;
    PgRange r = page_range(lo, hi, 0, b);
    if (!r.ok) {
        if (i == 0) atomicOr(flags, FLAG_CAPACITY);
        return;
    }
    if ((lo ? lo[b] : 0) >= hi[b]) r.last = 0;              // the row is freed
    if (i >= max_pages || (i >= r.first && i < r.last)) return;
    const int page = table[(size_t)b * max_pages + i];
    if (page < 0) return;
    table[(size_t)b * max_pages + i] = -1;
    drop_page(ref, n_pages, page, flags);
}

// Entry i of row b in a fork: the page is named once more by each of the row's `copies` (own_whole: the row's whole pages); a row that becomes a copy itself
// (src != b, whole: the whole pages of src) takes its new entry and gives its old page back.  One addition for all copies: 31 rows that take over a
// prompt would queue up at its counts.
__device__ __forceinline__ void fork_entry(int32_t *table, int32_t *ref, int n_pages, int max_pages, int b, int i, int src, int copies, int own_whole, int whole,
                                           int fresh, const int32_t *old, int32_t *flags) {
    if (src == b && copies == 0) return;
    const int was = old[(size_t)b * max_pages + i];
    if (copies > 0 && was >= 0 && i < own_whole) {
        if (was < n_pages) atomicAdd(&ref[was], copies);
        else atomicOr(flags, FLAG_BAD_PAGE);
    }
    if (src == b) return;
    int page = -1;
    if (i < whole) page = old[(size_t)src * max_pages + i];
    else if (i == whole && fresh >= 0) { page = fresh; atomicAdd(&ref[page], 1); }
    table[(size_t)b * max_pages + i] = page;
    if (was >= 0) drop_page(ref, n_pages, was, flags);
}

// Which row a row becomes a copy of, by what the caller asks for (src) and the length of that row (L): itself where that is not possible.
__device__ __forceinline__ int fork_source(int b, int src, int L, int B, int max_pages, int32_t *flags) {
    if (src == -1 || src == b) return b;
    if (src < -1 || src >= B) { atomicOr(flags, FLAG_BAD_PATH); return b; }
    if (L < 0 || (L + 15LL) >> 4 > max_pages) { atomicOr(flags, FLAG_CAPACITY); return b; }
    return src;
}

// The whole fork in one workgroup, for tables that fit its shared memory: entries, lengths and sources come in one round trip, the counts in a second one.
enum { PG_SMALL = 8192 };
__global__ __launch_bounds__(PG_THREADS) void pages_fork_small_kernel(int32_t *table, int32_t *ref, int n_pages, int max_pages, int B, const int32_t *src_row,
                                                                       const int32_t *seq_len, int32_t *copy_src, int32_t *copy_dst, int32_t *forked, int32_t *flags) {
    __shared__ int part[PG_WAVES];
    __shared__ int32_t old[PG_SMALL], len[PG_ROWS], copies[PG_ROWS], row[PG_ROWS], fresh[PG_ROWS], list[PG_ROWS];      // B <= PG_ROWS
    const int tid = (int)threadIdx.x, entries = B * max_pages;
    int v[PG_SMALL / PG_THREADS];
#pragma unroll
    for (int u = 0; u < PG_SMALL / PG_THREADS; ++u) v[u] = table[min(tid + u * PG_THREADS, entries - 1)];
    const int b = min(tid, B - 1), want = src_row[b];
    len[tid] = seq_len[b];
    copies[tid] = 0;
#pragma unroll
    for (int u = 0; u < PG_SMALL / PG_THREADS; ++u)
        if (tid + u * PG_THREADS < entries) old[tid + u * PG_THREADS] = v[u];
    __syncthreads();
    int src = b, page = -1;
    if (tid < B) {
        src = fork_source(b, want, want >= 0 && want < B ? len[want] : 0, B, max_pages, flags);
        if (src != b && (len[src] & 15)) page = old[src * max_pages + (len[src] >> 4)];
    }
    int all;
    const int at = block_scan(page >= 0 ? 1 : 0, part, all);
    const int found = lowest_free(ref, n_pages, min(all, n_pages), list, part);
    __syncthreads();
    if (tid < B) {
        int mine = -1;
        if (page >= 0) {
            if (at < found) mine = list[at];
            else { atomicOr(flags, FLAG_CAPACITY); src = b; page = -1; }          // the pool is exhausted: the row stays as it is
        }
        row[b] = forked[b] = src;
        copy_src[b] = page;
        fresh[b] = copy_dst[b] = mine;
        if (src != b) atomicAdd(&copies[src], 1);
    }
    __syncthreads();
    for (int e = tid; e < entries; e += PG_THREADS) {
        const int r = e / max_pages, from = row[r];
        fork_entry(table, ref, n_pages, max_pages, r, e - r * max_pages, from, copies[r], len[r] >> 4, len[from] >> 4, fresh[r], old, flags);
    }
}

// Larger tables: block 0 plans while the others copy the tables, then pages_fork_kernel.  ws: fresh page of each row [B] (-1: none), list [B], copies of
// each row [B], tables [B, max_pages]
__global__ __launch_bounds__(PG_THREADS) void pages_fork_plan_kernel(const int32_t *table, const int32_t *ref, int n_pages, int max_pages, int B, const int32_t *src_row,
                                                                      const int32_t *seq_len, int32_t *ws, int32_t *copy_src, int32_t *copy_dst, int32_t *forked,
                                                                      int32_t *flags) {
    __shared__ int part[PG_WAVES];
    if (blockIdx.x > 0) {
        int32_t *old = ws + 3 * (size_t)B;
        const size_t n = (size_t)B * max_pages, step = (size_t)(gridDim.x - 1) * PG_THREADS;
        for (size_t i = (size_t)(blockIdx.x - 1) * PG_THREADS + threadIdx.x; i < n; i += step) old[i] = table[i];
        return;
    }
    int32_t *fresh = ws, *list = ws + B, *copies = ws + 2 * (size_t)B;
    int all = 0;
    for (int b0 = 0; b0 < B; b0 += PG_THREADS) {
        const int b = b0 + (int)threadIdx.x;
        int row = b, page = -1;
        if (b < B) {
            const int src = src_row[b], L = src >= 0 && src < B ? seq_len[src] : 0;
            row = fork_source(b, src, L, B, max_pages, flags);
            if (row != b && (L & 15)) page = table[(size_t)src * max_pages + (L >> 4)];
        }
        const bool need = page >= 0;
        int total;
        const int at = block_scan(need ? 1 : 0, part, total) + all;
        all += total;
        if (b < B) {
            forked[b] = row;
            copy_src[b] = page;
            fresh[b] = need ? at : -1;
            copies[b] = 0;
        }
    }
    const int found = lowest_free(ref, n_pages, min(all, n_pages), list, part);
    __syncthreads();
    for (int b = threadIdx.x; b < B; b += PG_THREADS) {
        const int at = fresh[b];
        int page = -1;
        if (at >= 0) {
            if (at < found) page = list[at];
            else {                                          // the pool is exhausted: the row stays as it is
                atomicOr(flags, FLAG_CAPACITY);
                forked[b] = b;
                copy_src[b] = -1;
            }
        }
        fresh[b] = page;
        copy_dst[b] = page;
        if (forked[b] != b) atomicAdd(&copies[forked[b]], 1);
    }
}

__global__ __launch_bounds__(256) void pages_fork_kernel(int32_t *table, int32_t *ref, int n_pages, int max_pages, int B, const int32_t *seq_len,
                                                          const int32_t *ws, const int32_t *forked, int32_t *flags) {
    const int b = blockIdx.y, i = blockIdx.x * 256 + threadIdx.x;
    if (i >= max_pages) return;
    const int src = forked[b];
    fork_entry(table, ref, n_pages, max_pages, b, i, src, ws[2 * (size_t)B + b], seq_len[b] >> 4, seq_len[src] >> 4, ws[b], ws + 3 * (size_t)B, flags);
}

__device__ __forceinline__ void remap_entry(int32_t *entry, int n_pages, int U, const int32_t *to, int32_t *flags) {
    const int page = *entry;
    if (page >= n_pages) atomicOr(flags, FLAG_BAD_PAGE);
    else if (page >= U) *entry = to[page];
}

// Moves of a compaction.  ws: where page p at or behind U goes [n_pages].  entries > 0: the tables (so many entries) follow at once.
__global__ __launch_bounds__(PG_THREADS) void pages_compact_plan_kernel(int32_t *table, int entries, int32_t *ref, int n_pages, int32_t *ws, int32_t *move_src,
                                                                         int32_t *move_dst, int32_t *counts, int32_t *flags) {
    __shared__ int part[PG_WAVES];
    enum { PER = 8 };
    int used = 0;
    for (int p0 = threadIdx.x; p0 < n_pages; p0 += PG_THREADS * PER) {
        int v[PER];
#pragma unroll
        for (int e = 0; e < PER; ++e) { const int p = p0 + e * PG_THREADS; v[e] = p < n_pages ? ref[p] : 0; }
#pragma unroll
        for (int e = 0; e < PER; ++e) used += v[e] > 0;
    }
    int U;
    block_scan(used, part, U);
    int holes = 0, moves = 0;
    for (int p0 = 0; p0 < n_pages; p0 += PG_THREADS * PER) {            // a thread looks at PER pages in a row
        const int p = p0 + (int)threadIdx.x * PER;
        int v[PER], hole = 0, move = 0;
#pragma unroll
        for (int e = 0; e < PER; ++e) v[e] = p + e < n_pages ? ref[p + e] : 0;
#pragma unroll
        for (int e = 0; e < PER; ++e) {
            if (p + e >= n_pages) continue;
            hole += p + e < U && v[e] <= 0;
            move += p + e >= U && v[e] > 0;
        }
        int nh, nm;
        int ah = holes + block_scan(hole, part, nh), am = moves + block_scan(move, part, nm);
#pragma unroll
        for (int e = 0; e < PER; ++e) {
            if (p + e >= n_pages) continue;
            if (p + e < U) { if (v[e] <= 0) move_dst[ah++] = p + e; }
            else {
                ws[p + e] = p + e;
                if (v[e] > 0) move_src[am++] = p + e;
            }
        }
        holes += nh;
        moves += nm;
    }
    __syncthreads();
    for (int i = threadIdx.x; i < n_pages; i += PG_THREADS) {
        if (i >= moves) { move_src[i] = move_dst[i] = -1; continue; }
        const int a = move_src[i], d = move_dst[i];
        ws[a] = d;
        ref[d] = ref[a];
        ref[a] = 0;
    }
    if (threadIdx.x == 0) { counts[0] = moves; counts[1] = U; }
    __syncthreads();
    for (int i = threadIdx.x; i < entries; i += PG_THREADS) remap_entry(table + i, n_pages, U, ws, flags);
}

__global__ __launch_bounds__(256) void pages_remap_kernel(int32_t *table, int n_pages, size_t entries, const int32_t *ws, const int32_t *counts, int32_t *flags) {
    const size_t i = (size_t)blockIdx.x * 256 + threadIdx.x;
    if (i < entries) remap_entry(table + i, n_pages, counts[1], ws, flags);
}

// Whole pages of up to three arrays ([layers][n_pages][bytes] each): a workgroup copies 16 KB pieces, all its loads before its stores.
struct CopyPlanes { char *base[3]; uint32_t bytes[3], pieces[3]; int n, n_pages, layers; };
enum { COPY_PIECE = 16384 };
__global__ __launch_bounds__(256) void copy_pages_kernel(CopyPlanes pl, int n, const int32_t *src, const int32_t *dst, const int32_t *count, int32_t *flags) {
    if (count) n = min(n, *count);
    uint32_t piece = blockIdx.x;
    int q = 0;
    while (piece >= pl.pieces[q]) piece -= pl.pieces[q++];
    const int layer = blockIdx.y;
    for (int i = blockIdx.z; i < n; i += gridDim.z) {
        const int a = src[i], d = dst[i];
        if (a < 0 || d < 0 || a == d) continue;
        if (a >= pl.n_pages || d >= pl.n_pages) {
            if (threadIdx.x == 0) atomicOr(flags, FLAG_BAD_PAGE);
            continue;
        }
        const char *from = pl.base[q] + ((size_t)layer * pl.n_pages + a) * pl.bytes[q];
        char *to = pl.base[q] + ((size_t)layer * pl.n_pages + d) * pl.bytes[q];
        const uint32_t at = piece * COPY_PIECE, end = min(at + (uint32_t)COPY_PIECE, pl.bytes[q]);
        typedef uint32_t u4 __attribute__((ext_vector_type(4), aligned(4)));     // the caller's pages: no more than 4 bytes' alignment is known
        u4 v[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const uint32_t o = at + (j * 256 + threadIdx.x) * 16;
            if (o + 16 <= end) v[j] = *reinterpret_cast<const u4 *>(from + o);
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const uint32_t o = at + (j * 256 + threadIdx.x) * 16;
            if (o + 16 <= end) *reinterpret_cast<u4 *>(to + o) = v[j];
        }
        const uint32_t rest = end & 15u;                    // scales of an odd number of heads end in half a piece
        if (rest && threadIdx.x < rest / 4) {
            const uint32_t o = (end & ~15u) + threadIdx.x * 4;
            *reinterpret_cast<uint32_t *>(to + o) = *reinterpret_cast<const uint32_t *>(from + o);
        }
    }
}

static int launch_copy(hydra_ctx *c, hipStream_t s, CopyPlanes pl, int n, const int32_t *src, const int32_t *dst, const int32_t *count) {
    uint32_t per = 0;
    for (int q = 0; q < pl.n; ++q) { pl.pieces[q] = (pl.bytes[q] + COPY_PIECE - 1) / COPY_PIECE; per += pl.pieces[q]; }
    const dim3 grid(per, c->m.n_layers, std::min(n, 64)), block(256);
    hipLaunchKernelGGL(copy_pages_kernel, grid, block, 0, s, pl, n, src, dst, count, flags_dev(c));
    HYDRA_LAUNCH_CHECK("copy_pages_kernel");
    return HYDRA_OK;
}

static int check_pages(hydra_ctx *c, int B, const hydra_pages *p) {
    if (!c) return fail(HYDRA_E_INVALID_ARG, "ctx is NULL");
    if (B < 1 || B > c->max_batch) return fail(HYDRA_E_CAPACITY, "B outside [1, max_batch]");
    if (!c->arena) return fail(HYDRA_E_STATE, "no weight arena bound (hydra_bind_weights)");
    if (!p || !p->page_table || !p->ref) return fail(HYDRA_E_INVALID_ARG, "pages or one of its pointers is NULL");
    if (p->n_pages < 1 || p->max_pages < 1) return fail(HYDRA_E_INVALID_ARG, "pages: n_pages and max_pages must be positive");
    // sums over entries and numbers of pages, with a workgroup's step behind them, are ints
    if (p->n_pages > (1 << 30) || (int64_t)B * p->max_pages > (1 << 30) || p->max_pages > INT_MAX / HYDRA_PAGE)
        return fail(HYDRA_E_CAPACITY, "pages: more than 2^30 pages or table entries, or a table of 2^31 slots");
    return HYDRA_OK;
}
static int check_ws(const void *ws) {
    if (!ws) return fail(HYDRA_E_INVALID_ARG, "workspace is NULL");
    if (((uintptr_t)ws) & 255) return fail(HYDRA_E_INVALID_ARG, "workspace must be 256-byte aligned");
    return HYDRA_OK;
}
static int check_copy(hydra_ctx *c, int n, const int32_t *src, const int32_t *dst) {
    if (!c) return fail(HYDRA_E_INVALID_ARG, "ctx is NULL");
    if (!c->arena) return fail(HYDRA_E_STATE, "no weight arena bound (hydra_bind_weights)");
    if (n < 0 || !src || !dst) return fail(HYDRA_E_INVALID_ARG, "copy_pages: n is negative or a list is NULL");
    return HYDRA_OK;
}

}  // namespace hydra

using namespace hydra;

extern "C" {

size_t hydra_pages_workspace_bytes(int B, int n_pages, int max_pages) {
    if (B < 1 || n_pages < 1 || max_pages < 1) return 0;
    const size_t reserve = 4 * (size_t)B + n_pages, fork = 3 * (size_t)B + (size_t)B * max_pages, compact = n_pages;
    return align_up(std::max(reserve, std::max(fork, compact)) * 4, 256);
}

int hydra_pages_reserve(hydra_ctx *c, void *stream, int B, void *ws, const hydra_pages *p, const int32_t *lo, const int32_t *hi, int extra, int32_t *ok) {
    int rc = check_pages(c, B, p);
    if (rc) return rc;
    if ((rc = check_ws(ws))) return rc;
    if (!hi || extra < 0) return fail(HYDRA_E_INVALID_ARG, "hydra_pages_reserve: hi is NULL or extra is negative");
    hipLaunchKernelGGL(pages_reserve_kernel, dim3(1), dim3(PG_THREADS), 0, (hipStream_t)stream, p->page_table, p->ref, p->n_pages, p->max_pages, B, lo, hi, extra,
                       (int32_t *)ws, ok, flags_dev(c));
    HYDRA_LAUNCH_CHECK("pages_reserve_kernel");
    return HYDRA_OK;
}

int hydra_pages_release(hydra_ctx *c, void *stream, int B, const hydra_pages *p, const int32_t *lo, const int32_t *hi) {
    int rc = check_pages(c, B, p);
    if (rc) return rc;
    if (!hi) return fail(HYDRA_E_INVALID_ARG, "hydra_pages_release: hi is NULL");
    hipLaunchKernelGGL(pages_release_kernel, dim3(ceil_div(p->max_pages, 256), B), dim3(256), 0, (hipStream_t)stream, p->page_table, p->ref, p->n_pages,
                       p->max_pages, lo, hi, flags_dev(c));
    HYDRA_LAUNCH_CHECK("pages_release_kernel");
    return HYDRA_OK;
}

int hydra_pages_fork(hydra_ctx *c, void *stream, int B, void *ws, const hydra_pages *p, const int32_t *src_row, const int32_t *seq_len, int32_t *copy_src,
                     int32_t *copy_dst, int32_t *forked) {
    int rc = check_pages(c, B, p);
    if (rc) return rc;
    if ((rc = check_ws(ws))) return rc;
    if (!src_row || !seq_len || !copy_src || !copy_dst || !forked) return fail(HYDRA_E_INVALID_ARG, "hydra_pages_fork: NULL argument");
    const size_t entries = (size_t)B * p->max_pages;
    if (entries <= PG_SMALL && B <= PG_ROWS) {
        hipLaunchKernelGGL(pages_fork_small_kernel, dim3(1), dim3(PG_THREADS), 0, (hipStream_t)stream, p->page_table, p->ref, p->n_pages, p->max_pages, B, src_row,
                           seq_len, copy_src, copy_dst, forked, flags_dev(c));
        HYDRA_LAUNCH_CHECK("pages_fork_small_kernel");
        return HYDRA_OK;
    }
    const int copiers = (int)std::min<size_t>(128, (entries + PG_THREADS - 1) / PG_THREADS);
    hipLaunchKernelGGL(pages_fork_plan_kernel, dim3(1 + copiers), dim3(PG_THREADS), 0, (hipStream_t)stream, p->page_table, p->ref, p->n_pages, p->max_pages, B,
                       src_row, seq_len, (int32_t *)ws, copy_src, copy_dst, forked, flags_dev(c));
    HYDRA_LAUNCH_CHECK("pages_fork_plan_kernel");
    hipLaunchKernelGGL(pages_fork_kernel, dim3(ceil_div(p->max_pages, 256), B), dim3(256), 0, (hipStream_t)stream, p->page_table, p->ref, p->n_pages, p->max_pages,
                       B, seq_len, (const int32_t *)ws, forked, flags_dev(c));
    HYDRA_LAUNCH_CHECK("pages_fork_kernel");
    return HYDRA_OK;
}

int hydra_pages_compact(hydra_ctx *c, void *stream, int B, void *ws, const hydra_pages *p, int32_t *move_src, int32_t *move_dst, int32_t *counts) {
    int rc = check_pages(c, B, p);
    if (rc) return rc;
    if ((rc = check_ws(ws))) return rc;
    if (!move_src || !move_dst || !counts) return fail(HYDRA_E_INVALID_ARG, "hydra_pages_compact: NULL argument");
    const size_t entries = (size_t)B * p->max_pages;
    const bool small = entries <= PG_SMALL;                 // one kernel; beyond, the tables are spread over the chip
    hipLaunchKernelGGL(pages_compact_plan_kernel, dim3(1), dim3(PG_THREADS), 0, (hipStream_t)stream, p->page_table, small ? (int)entries : 0, p->ref, p->n_pages,
                       (int32_t *)ws, move_src, move_dst, counts, flags_dev(c));
    HYDRA_LAUNCH_CHECK("pages_compact_plan_kernel");
    if (small) return HYDRA_OK;
    hipLaunchKernelGGL(pages_remap_kernel, dim3((unsigned)((entries + 255) / 256)), dim3(256), 0, (hipStream_t)stream, p->page_table, p->n_pages, entries,
                       (const int32_t *)ws, counts, flags_dev(c));
    HYDRA_LAUNCH_CHECK("pages_remap_kernel");
    return HYDRA_OK;
}

int hydra_kv_copy_pages(hydra_ctx *c, void *stream, const hydra_kv *kv, int n, const int32_t *src, const int32_t *dst, const int32_t *count) {
    int rc = check_copy(c, n, src, dst);
    if (rc) return rc;
    if (!kv || !kv->k_pages || !kv->v_pages || kv->n_pages < 1) return fail(HYDRA_E_INVALID_ARG, "kv or one of its page arrays is NULL, or n_pages is not positive");
    if (((uintptr_t)kv->k_pages | (uintptr_t)kv->v_pages) & 15) return fail(HYDRA_E_INVALID_ARG, "copy_pages: pages must be 16-byte aligned");
    if (n == 0) return HYDRA_OK;
    CopyPlanes pl = {};
    pl.n = 2; pl.n_pages = kv->n_pages; pl.layers = c->m.n_layers;
    pl.base[0] = (char *)kv->k_pages; pl.base[1] = (char *)kv->v_pages;
    pl.bytes[0] = pl.bytes[1] = (uint32_t)(c->m.d * HYDRA_PAGE * c->esz);
    return launch_copy(c, (hipStream_t)stream, pl, n, src, dst, count);
}

int hydra_kv8_copy_pages(hydra_ctx *c, void *stream, const hydra_kv8 *kv, int n, const int32_t *src, const int32_t *dst, const int32_t *count) {
    int rc = check_copy(c, n, src, dst);
    if (rc) return rc;
    if (!c->bf16) return fail(HYDRA_E_UNSUPPORTED, "the 8-bit cache is for HYDRA_BF16 contexts");
    if (!kv || !kv->k_codes || !kv->v_codes || !kv->scales || kv->n_pages < 1) return fail(HYDRA_E_INVALID_ARG, "kv8 or one of its arrays is NULL, or n_pages is not positive");
    if (((uintptr_t)kv->k_codes | (uintptr_t)kv->v_codes) & 15 || (uintptr_t)kv->scales & 7)
        return fail(HYDRA_E_INVALID_ARG, "copy_pages: codes must be 16-byte aligned, scales 8-byte");
    if (n == 0) return HYDRA_OK;
    CopyPlanes pl = {};
    pl.n = 3; pl.n_pages = kv->n_pages; pl.layers = c->m.n_layers;
    pl.base[0] = (char *)kv->k_codes; pl.base[1] = (char *)kv->v_codes; pl.base[2] = (char *)kv->scales;
    pl.bytes[0] = pl.bytes[1] = (uint32_t)(c->m.d * HYDRA_PAGE); pl.bytes[2] = (uint32_t)(c->m.n_heads * 8);
    return launch_copy(c, (hipStream_t)stream, pl, n, src, dst, count);
}

}  // extern "C"
