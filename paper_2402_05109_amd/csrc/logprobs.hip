// Log probabilities of given tokens, entropy and the most likely tokens of rows of logits (paper, section 6.3: p = softmax(logits / tau)).
//
// One pass over the logits.  With m the largest logit, z = (x - m) / tau, and the tokens that have m apart (there are `peaks` of them, each of weight 1):
//     rest = sum_{x < m} e^z      A = sum_{x < m} e^z z      ln Z = log1p(rest + peaks - 1)
//     log p(t) = z_t - ln Z       H = ln Z - A / Z
// Both terms of H are positive and log1p takes what is left beside the peak, so entropies and log probabilities near 0 keep their digits.
//
// A thread goes over its logits in portions of LP_PER, with a running maximum to which its sums are related; lanes, waves and pieces of a row are joined the
// same way.  The k most likely tokens come from the same pass: each wave puts what may be among them into a list of its own, about twice k entries (the k-th best
// of its lanes' largest logits so far is a bound that k logits reach), and what is left of the lists under a bound of all waves is ranked at the end.
#include <algorithm>

#include "device_common.h"
#include "internal.h"

namespace hydra {

enum { LP_PER = 32, LP_THREADS = 256, LP_LIST = 256, LP_MAX_PIECES = 64, LP_FLAT = LP_MAX_PIECES * HYDRA_MAX_TOPK };

// Monotone 32-bit key of a logit: larger logits have larger keys, -0 that of +0, a NaN that of -infinity; 0 is below every key.
__device__ __forceinline__ uint32_t logit_key(float v) {
    uint32_t b = __float_as_uint(v);
    if ((b & 0x7fffffffu) > 0x7f800000u) b = 0xff800000u;
    if (b == 0x80000000u) b = 0u;
    return (b & 0x80000000u) ? ~b : (b | 0x80000000u);
}
__device__ __forceinline__ float logit_of(uint32_t k) { return __uint_as_float((k & 0x80000000u) ? (k ^ 0x80000000u) : ~k); }

// Sums over some logits, relative to the largest of them: rest and A (in powers of two: A = sum 2^z2 z2) without the `peaks` that equal it.  A NaN among the
// logits makes `rest` one.
struct LpSums { float m, rest, A, peaks; };
struct LpRecord { LpSums s; int above, pad[3]; };         // of a piece; its k best entries follow, as (key, id) pairs
struct LogprobArgs {
    const float *logits;
    const int32_t *tokens;
    float *logprob, *entropy, *top_logprobs;
    int32_t *rank, *top_ids, *flags;
    float *records;                                         // [rows, pieces]
    int V, k, pieces, piece;                                // piece: logits of one, a multiple of 4
    float inv_tau;
};
__host__ __device__ inline size_t lp_record_floats(int k) { return sizeof(LpRecord) / 4 + 2 * (size_t)k; }

// the same sums relative to a maximum that is no less; the clamps are where an infinite difference would meet a weight of 0
__device__ __forceinline__ void lp_relate(LpSums &s, float m, float k2) {
    if (!(s.m < m)) return;
    const float d = fmaxf((s.m - m) * k2, -1e30f), w = __builtin_amdgcn_exp2f(d), all = s.rest + s.peaks;
    s.A = w * fmaf(d, all, s.A);
    s.rest = w * all;
    s.peaks = 0.f;
    s.m = m;
}
__device__ __forceinline__ void lp_wave(LpSums &s, float k2) {
    lp_relate(s, wave_max(s.m), k2);
    s.rest = wave_sum(s.rest);
    s.A = wave_sum(s.A);
    s.peaks = wave_sum(s.peaks);
}

__device__ __forceinline__ int sum_over_wave(int v) {
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) v += __shfl_xor(v, d, 64);
    return v;
}

// What is wanted of a row once its sums are known, but for the most likely tokens, from the thread that `writes`.  Returns ln Z.
__device__ __forceinline__ float lp_finish(const LogprobArgs &a, int row, const LpSums &s, int tok, float given, int above, bool writes) {
    // a largest logit that is infinite has no weights relative to it
    const float others = fabsf(s.m) < INFINITY ? s.rest + (s.peaks - 1.f) : __uint_as_float(0x7fc00000u);
    const float lnz = log1pf(others);
    if (!writes) return lnz;
    if (a.entropy) a.entropy[row] = lnz - 0.693147181f * s.A / (1.0f + others);
    if (a.logprob) a.logprob[row] = tok < 0 ? 0.f : (given - s.m) * a.inv_tau - lnz;
    if (a.rank) a.rank[row] = tok < 0 ? -1 : above;
    return lnz;
}
// the row's token and its logit (a NaN: -infinity, as in every order; the row's sums are no numbers then, nor is the log probability): -1 = none, others outside the vocabulary are
// reported and taken as 0
__device__ __forceinline__ int lp_token(const LogprobArgs &a, int row, float &given) {
    int tok = a.tokens ? a.tokens[row] : -1;
    if (tok != -1 && (tok < 0 || tok >= a.V)) { atomicOr(a.flags, FLAG_BAD_TOKEN); tok = 0; }
    given = tok >= 0 ? a.logits[(size_t)row * a.V + tok] : INFINITY;
    if (__builtin_isnan(given)) given = -INFINITY;
    return tok;
}

// A bound that at least k of the wave's logits reach: the k-th largest of its lanes' maxima, as far as its upper 16 bits tell.  The lowest finite value: fewer lanes
// have any.  (Scalar work for the most part: 64 lanes ranked against each other by broadcasts take twice the time of the sums.)
__device__ __forceinline__ float lp_bound(uint32_t best_key, int k) {
    uint32_t t = 0u;
#pragma unroll
    for (int bit = 30; bit >= 16; bit -= 2) {               // two bits at a time: three counts beside each other
        const uint32_t c1 = t | (1u << bit), c2 = t | (2u << bit), c3 = t | (3u << bit);
        const int n1 = __popcll(__ballot(best_key >= c1)), n2 = __popcll(__ballot(best_key >= c2)), n3 = __popcll(__ballot(best_key >= c3));
        t = n3 >= k ? c3 : n2 >= k ? c2 : n1 >= k ? c1 : t;
    }
    return t < 0x00800000u ? -3.402823466e38f : logit_of(t);
}

// The k best of the workgroup's entries e[] (key 0: none) among those with a key of at least `bound`, as put(rank, entry) by one thread each, by the (key descending,
// id ascending) order.  flat: LP_FLAT entries of LDS, which may be where e[] came from.  False, and nothing done, if there are fewer than k or more than LP_FLAT.
template <int PER, class Put>
__device__ __forceinline__ bool lp_place(const uint2 (&e)[PER], uint32_t bound, int k, uint2 *flat, int *counts, Put put) {
    const int tid = (int)threadIdx.x, wave = tid >> 6;
    int mine = 0;
#pragma unroll
    for (int i = 0; i < PER; ++i) mine += __popcll(__ballot(e[i].x >= bound));
    if ((tid & 63) == 0) counts[wave] = mine;
    __syncthreads();
    int at = 0, total = 0;
#pragma unroll
    for (int w = 0; w < LP_THREADS / 64; ++w) {
        if (w < wave) at += counts[w];
        total += counts[w];
    }
    if (total < k || total > LP_FLAT) return false;         // uniform
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const uint64_t has = __ballot(e[i].x >= bound);
        if (e[i].x >= bound) flat[at + (int)__builtin_amdgcn_mbcnt_hi((uint32_t)(has >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)has, 0u))] = e[i];
        at += __popcll(has);
    }
    if (tid < 8) flat[total + tid] = make_uint2(0u, 0xffffffffu);        // ranks are counted eight entries at a time
    __syncthreads();
    for (int i = tid; i < total; i += LP_THREADS) {
        const uint2 x = flat[i];
        int r = 0;
        for (int o = 0; o < total; o += 8) {
            uint2 y[8];
#pragma unroll
            for (int u = 0; u < 8; ++u) y[u] = flat[o + u];
#pragma unroll
            for (int u = 0; u < 8; ++u) r += (y[u].x > x.x || (y[u].x == x.x && y[u].y < x.y)) ? 1 : 0;
        }
        if (r < k) put(r, x);
    }
    return true;
}

// k rounds, each for the best of n entries behind the one before it; entry(i): its (key, id).  For rows with fewer than k logits over -infinity, or with more entries at
// the bound than the list holds (many equal ones).  list: an entry per wave.
template <class Entry, class Put>
__device__ __forceinline__ void lp_rounds(int n, int k, uint2 *list, Entry entry, Put put) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, waves = (int)blockDim.x >> 6;
    uint32_t pk = 0u, pi = 0u;
    for (int t = 0; t < k; ++t) {
        uint32_t bk = 0u, bi = 0xffffffffu;
        for (int i = (int)threadIdx.x; i < n; i += (int)blockDim.x) {
            const uint2 e = entry(i);
            const uint32_t key = e.x, id = e.y;
            if ((t == 0 || key < pk || (key == pk && id > pi)) && (key > bk || (key == bk && id < bi))) { bk = key; bi = id; }
        }
#pragma unroll
        for (int d = 32; d > 0; d >>= 1) {
            const uint32_t ok = (uint32_t)__shfl_xor((int)bk, d, 64), oi = (uint32_t)__shfl_xor((int)bi, d, 64);
            if (ok > bk || (ok == bk && oi < bi)) { bk = ok; bi = oi; }
        }
        __syncthreads();
        if (lane == 0) list[wave] = make_uint2(bk, bi);
        __syncthreads();
        bk = 0u; bi = 0xffffffffu;
        for (int w = 0; w < waves; ++w) {
            const uint2 y = list[w];
            if (y.x > bk || (y.x == bk && y.y < bi)) { bk = y.x; bi = y.y; }
        }
        pk = bk; pi = bi;
        if (threadIdx.x == 0) put(t, make_uint2(bk, bi));
    }
}

// One workgroup per piece of a row.  In a portion thread t holds groups of four neighbouring logits, group i at (i * threads + t) * 4: ids ascend with the portions.
template <bool TOP>
__global__ __launch_bounds__(LP_THREADS) void logprob_kernel(LogprobArgs a) {
    typedef float f4u __attribute__((ext_vector_type(4), aligned(4)));
    constexpr int WAVES = LP_THREADS / 64, PORTION = LP_THREADS * LP_PER;
    __shared__ LpSums sums[WAVES];
    __shared__ float bounds[2][WAVES];
    __shared__ int larger[WAVES], counts[WAVES], stay[WAVES];
    __shared__ uint2 lists[TOP ? LP_FLAT + 8 : 1];          // a list of LP_LIST per wave, then what is left of them
    const int tid = (int)threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int row = (int)blockIdx.x / a.pieces, pc = (int)blockIdx.x - row * a.pieces, from = pc * a.piece, n = min(a.piece, a.V - from);
    const float *x0 = a.logits + (size_t)row * a.V + from;
    const float k2 = a.inv_tau * 1.44269504f;
    // Logits pass the caches by (1024 rows x 32000, k = 0 / 5 / 32: 25.8 / 29.4 / 35.5 us; through them 28.5 / 32.3 / 37.4).  No load is behind a condition: a group
    // behind the last one reads the last four logits and holds none of them, the group that the end cuts reads them too and leaves out those that the one before it has.
    auto place = [&](int at0, int i) { return at0 + (i * LP_THREADS + tid) * 4; };
    auto load = [&](float (&x)[LP_PER], int at0) {
        if (n < 4) {                                         // uniform: a vocabulary of two or three tokens, or what is left of one
#pragma unroll
            for (int i = 0; i < LP_PER; ++i) x[i] = i < n && tid == 0 ? x0[i] : -INFINITY;
            return;
        }
#pragma unroll
        for (int i = 0; i < LP_PER / 4; ++i) {
            const f4u v = __builtin_nontemporal_load(reinterpret_cast<const f4u *>(x0 + min(place(at0, i), n - 4)));
#pragma unroll
            for (int e = 0; e < 4; ++e) x[4 * i + e] = v[e];
        }
    };
    float x[LP_PER];
    load(x, 0);
    float given;
    const int tok = lp_token(a, row, given);
    uint2 *list = lists + (TOP ? wave * LP_LIST : 0);
    int count = 0;                                          // of the wave's list; beyond LP_LIST: so many would have gone there
    float best = -INFINITY, thr = -INFINITY;                // the largest of the lane's logits so far, and what k of the wave's reach
    LpSums s = {-INFINITY, 0.f, 0.f, 0.f};
    int above = 0;
    for (int at0 = 0; at0 < n; at0 += PORTION) {
        const bool last = at0 + PORTION >= n;                // uniform
        if (at0 > 0) load(x, at0);
        if (last && n >= 4) {
#pragma unroll
            for (int i = 0; i < LP_PER / 4; ++i) {
                const int over = place(at0, i) - (n - 4);    // so many of the four are the group's before it
#pragma unroll
                for (int e = 0; e < 4; ++e) x[4 * i + e] = e < over ? -INFINITY : x[4 * i + e];
            }
        }
        float gm[LP_PER / 4], cm = -INFINITY;
#pragma unroll
        for (int i = 0; i < LP_PER / 4; ++i) {
            gm[i] = fmaxf(fmaxf(x[4 * i], x[4 * i + 1]), fmaxf(x[4 * i + 2], x[4 * i + 3]));
            cm = fmaxf(cm, gm[i]);
        }
        // the maximum is the wave's: groups that hold it, or logits over the given token's, are few
        lp_relate(s, fmaxf(s.m, wave_max(cm)), k2);
#pragma unroll
        for (int i = 0; i < LP_PER / 4; ++i) {
            float z[4], w[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                z[e] = (x[4 * i + e] - s.m) * k2;
                w[e] = __builtin_amdgcn_exp2f(z[e]);
            }
            if (__any(gm[i] == s.m)) {
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const bool peak = x[4 * i + e] == s.m;  // where both are infinite the difference is no number
                    w[e] = peak ? 0.f : w[e];
                    s.peaks += peak ? 1.f : 0.f;
                }
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                s.rest += w[e];
                s.A = fmaf(w[e], fmaxf(z[e], -1e30f), s.A);
            }
        }
#pragma unroll
        for (int i = 0; i < LP_PER / 4; ++i)                 // the given token's logit comes by two loads in a row: last
            if (__any(gm[i] > given)) {
#pragma unroll
                for (int e = 0; e < 4; ++e) above += x[4 * i + e] > given ? 1 : 0;
            }
        if constexpr (TOP) {
            best = fmaxf(best, cm);
            thr = lp_bound(logit_key(best), a.k);
#pragma unroll
            for (int i = 0; i < LP_PER / 4; ++i)
                if (__any(gm[i] >= thr)) {
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const float v = x[4 * i + e];
                        const uint64_t has = __ballot(v >= thr);
                        if (v >= thr) {
                            const int pos = count + (int)__builtin_amdgcn_mbcnt_hi((uint32_t)(has >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)has, 0u));
                            if (pos < LP_LIST) list[pos] = make_uint2(logit_key(v), (uint32_t)(from + (n < 4 ? 4 * i : min(place(at0, i), n - 4)) + e));
                        }
                        count += __popcll(has);
                    }
                }
        }
    }
    lp_wave(s, k2);
    above = sum_over_wave(above);
    if (lane == 0) { sums[wave] = s; larger[wave] = above; }
    if constexpr (TOP) {
        // a bound for the whole piece: k logits reach that of any wave, and a WAVES-th of k in every wave the lowest of theirs
        const float quarter = lp_bound(logit_key(best), (a.k + WAVES - 1) / WAVES);
        if (lane == 0) { bounds[0][wave] = thr; bounds[1][wave] = quarter; counts[wave] = count; }
    }
    __syncthreads();
    // every wave joins the waves' sums
    s = sums[min(lane, WAVES - 1)];
    if (lane >= WAVES) s.rest = s.A = s.peaks = 0.f;
    lp_wave(s, k2);
    int more = 0;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) more += larger[w];
    float *rec = a.records + (size_t)blockIdx.x * lp_record_floats(a.k);
    const bool done = a.pieces == 1;
    float lnz = 0.f;
    if (done) {
        if (TOP || tid == 0) lnz = lp_finish(a, row, s, tok, given, more, tid == 0);
    } else if (tid == 0) {
        *reinterpret_cast<LpRecord *>(rec) = LpRecord{s, more, {0, 0, 0}};
    }
    if constexpr (TOP) {
        float high = bounds[0][0], low = bounds[1][0];
        bool whole = counts[0] <= LP_LIST;                   // no list ran over
#pragma unroll
        for (int w = 1; w < WAVES; ++w) {
            high = fmaxf(high, bounds[0][w]);
            low = fminf(low, bounds[1][w]);
            whole = whole && counts[w] <= LP_LIST;
        }
        uint2 e[LP_LIST / 64];
#pragma unroll
        for (int i = 0; i < LP_LIST / 64; ++i) e[i] = i * 64 + lane < min(count, (int)LP_LIST) ? list[i * 64 + lane] : make_uint2(0u, 0u);
        const float m = s.m, inv_tau = a.inv_tau;
        const size_t first = (size_t)row * a.k;
        auto put = [=](int t, uint2 e) {
            if (done) {
                a.top_ids[first + t] = (int32_t)e.y;
                a.top_logprobs[first + t] = (logit_of(e.x) - m) * inv_tau - lnz;
            } else {
                reinterpret_cast<uint2 *>(rec + sizeof(LpRecord) / 4)[t] = e;
            }
        };
        if (!whole || !lp_place(e, logit_key(fmaxf(high, low)), a.k, lists, stay, put)) {
            __syncthreads();                                 // the lists give their place to the rounds
            lp_rounds(n, a.k, lists, [=](int i) { return make_uint2(logit_key(x0[i]), (uint32_t)(from + i)); }, put);
        }
    }
}

// Joins the records of a row: a piece per lane of every wave; the entries of all pieces are ranked.
template <bool TOP>
__global__ __launch_bounds__(LP_THREADS) void logprob_join_kernel(LogprobArgs a) {
    __shared__ uint2 flat[TOP ? LP_FLAT + 8 : 1];
    __shared__ int counts[LP_THREADS / 64];
    const int tid = (int)threadIdx.x, lane = tid & 63, row = blockIdx.x;
    const float k2 = a.inv_tau * 1.44269504f;
    const size_t step = lp_record_floats(a.k);
    const float *recs = a.records + (size_t)row * a.pieces * step;
    const float *mine = recs + (size_t)min(lane, a.pieces - 1) * step;
    LpRecord r = *reinterpret_cast<const LpRecord *>(mine);
    constexpr int PER = LP_FLAT / LP_THREADS;
    uint2 e[PER];
    uint32_t kth = 0u, part = 0u;
    if constexpr (TOP) {
        const uint2 *best = reinterpret_cast<const uint2 *>(mine + sizeof(LpRecord) / 4);
        kth = best[a.k - 1].x;
        part = best[(a.k + a.pieces - 1) / a.pieces - 1].x;
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const int q = i * LP_THREADS + tid, p = q / a.k;
            e[i] = make_uint2(0u, 0u);
            if (p < a.pieces) e[i] = reinterpret_cast<const uint2 *>(recs + (size_t)p * step + sizeof(LpRecord) / 4)[q - p * a.k];
        }
    }
    float given;
    const int tok = lp_token(a, row, given);
    if (lane >= a.pieces) { r.s.rest = r.s.A = r.s.peaks = 0.f; r.above = 0; }
    lp_wave(r.s, k2);
    r.above = sum_over_wave(r.above);
    const float lnz = lp_finish(a, row, r.s, tok, given, r.above, tid == 0);
    if constexpr (TOP) {
        // k entries reach the k-th of any piece, and the lowest of the pieces' ceil(k / pieces)-th; a piece may have fewer
        auto value = [](uint32_t k) { return k ? logit_of(k) : -INFINITY; };
        const float bound = fmaxf(wave_max(value(kth)), -wave_max(-value(part)));
        const float m = r.s.m, inv_tau = a.inv_tau;
        const size_t first = (size_t)row * a.k;
        lp_place(e, logit_key(bound), a.k, flat, counts, [=](int t, uint2 x) {
            a.top_ids[first + t] = (int32_t)x.y;
            a.top_logprobs[first + t] = (logit_of(x.x) - m) * inv_tau - lnz;
        });
    }
}

// Portions of a row that a workgroup takes: one while those are up to 768 in all, then as many as that needs; from 384 rows on all of a row, which then needs no second
// kernel.  A workgroup's fixed part (bounds, lists, ranks) is worth about a portion where tokens are wanted, and four of them fit a compute unit.  us, k = 0 / 5 / 32:
// 128 rows x 100003 15.3 / 24.6 / 35.5 with a portion, 16.2 / 21.9 / 29.8 with two; 256 rows x 131072 28.0 / 42.1 / 58.9 with one, 27.9 / 33.3 / 41.5 with four; 512 rows x 32000
// 18.1 / 23.1 / 29.9 with two, 15.5 / 20.7 / 27.3 with all four.  One row x 32000 takes 6.6 / 12 / 16 with pieces of 8192, 4096, 2048 or 1024.
static int logprob_pieces(int V, int rows) {
    const int portions = ceil_div(V, LP_THREADS * LP_PER);
    const int64_t per = rows >= 384 ? portions : std::max<int64_t>({1, ceil_div(portions, LP_MAX_PIECES), (int64_t)portions * rows / 768});
    return ceil_div(portions, (int)std::min<int64_t>(per, portions));
}
size_t logprob_scratch_bytes(const hydra_ctx *c, int rows) { return (size_t)rows * logprob_pieces(c->m.vocab, rows) * lp_record_floats(HYDRA_MAX_TOPK) * 4; }

int launch_token_logprobs(hydra_ctx *c, hipStream_t s, int rows, float *records, const float *logits, const int32_t *tokens, float tau, int k, float *logprob, int32_t *rank,
                          float *entropy, int32_t *top_ids, float *top_logprobs) {
    LogprobArgs a;
    const int V = c->m.vocab;
    a.logits = logits; a.tokens = tokens; a.logprob = logprob; a.entropy = entropy; a.top_logprobs = top_logprobs; a.rank = rank; a.top_ids = top_ids;
    a.flags = flags_dev(c); a.records = records; a.V = V; a.k = k; a.inv_tau = 1.0f / tau;
    a.piece = (int)align_up(ceil_div(V, logprob_pieces(V, rows)), 4);
    a.pieces = ceil_div(V, a.piece);
    if (k > 0) hipLaunchKernelGGL(logprob_kernel<true>, dim3(a.pieces * rows), dim3(LP_THREADS), 0, s, a);
    else       hipLaunchKernelGGL(logprob_kernel<false>, dim3(a.pieces * rows), dim3(LP_THREADS), 0, s, a);
    HYDRA_LAUNCH_CHECK("logprob_kernel");
    if (a.pieces > 1) {
        if (k > 0) hipLaunchKernelGGL(logprob_join_kernel<true>, dim3(rows), dim3(LP_THREADS), 0, s, a);
        else       hipLaunchKernelGGL(logprob_join_kernel<false>, dim3(rows), dim3(64), 0, s, a);
        HYDRA_LAUNCH_CHECK("logprob_join_kernel");
    }
    return HYDRA_OK;
}

}  // namespace hydra
