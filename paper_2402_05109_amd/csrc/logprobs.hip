// Log probabilities of given tokens, entropy and the most likely tokens of rows of logits (paper, section 6.3: p = softmax(logits / tau)).
//
// One pass over the logits.  With m the largest logit, z = (x - m) / tau, and the tokens that have m apart (there are `peaks` of them, each of weight 1):
//     rest = sum_{x < m} e^z      A = sum_{x < m} e^z (-z)      ln Z = log1p(rest + peaks - 1)
//     log p(t) = z_t - ln Z       H = ln Z + A / Z
// Both terms of H are positive and log1p takes what is left beside the peak, so entropies and log probabilities near 0 keep their digits.
// Bound by memory: the logits are read once.  A workgroup holds its piece of a row in registers, 32 logits to a thread.  Rows longer than a piece, or
// few rows, are cut into pieces whose records a second kernel joins.
#include <algorithm>

#include "device_common.h"
#include "internal.h"

namespace hydra {

enum { LP_PER = 32, LP_MAX_THREADS = 1024, LP_LIST = 1024, LP_MAX_PIECES = 64 };

// Monotone 32-bit key of a logit: larger logits have larger keys, -0 that of +0, a NaN that of -infinity; 0 is below every key.
__device__ __forceinline__ uint32_t logit_key(float v) {
    uint32_t b = __float_as_uint(v);
    if ((b & 0x7fffffffu) > 0x7f800000u) b = 0xff800000u;
    if (b == 0x80000000u) b = 0u;
    return (b & 0x80000000u) ? ~b : (b | 0x80000000u);
}
__device__ __forceinline__ float logit_of(uint32_t k) { return __uint_as_float((k & 0x80000000u) ? (k ^ 0x80000000u) : ~k); }

struct LogprobArgs {
    const float *logits;
    const int32_t *tokens;
    float *logprob, *entropy, *top_logprobs;
    int32_t *rank, *top_ids, *flags;
    float *records;                                         // [rows, pieces] of LpRecord, then k (key, id) pairs
    int V, k, pieces, piece;                                // piece: logits of one, a multiple of 4
    float inv_tau;
};
struct LpRecord { float m, rest, A; int peaks, above, pad[3]; };
__host__ __device__ inline size_t lp_record_floats(int k) { return sizeof(LpRecord) / 4 + 2 * (size_t)k; }

// What is wanted of a row once its sums are known; one thread.
__device__ __forceinline__ float lp_finish(const LogprobArgs &a, int row, float m, float rest, float A, int peaks, int above) {
    const float others = rest + (float)(peaks - 1);         // weights beside one of the peaks
    const float lnz = log1pf(others);
    if (a.entropy) a.entropy[row] = lnz + A / (1.0f + others);
    if (a.tokens) {
        int tok = a.tokens[row];
        if (tok != -1 && (tok < 0 || tok >= a.V)) { atomicOr(a.flags, FLAG_BAD_TOKEN); tok = 0; }
        if (a.logprob) a.logprob[row] = tok < 0 ? 0.f : (a.logits[(size_t)row * a.V + tok] - m) * a.inv_tau - lnz;
        if (a.rank) a.rank[row] = tok < 0 ? -1 : above;
    }
    return lnz;
}

// the k best of a workgroup's keys, in order, as put(place, key, id) by one thread each; entries are (key, id), key 0: none
template <int PER, class Id, class Put>
__device__ __forceinline__ void block_top_k(const uint32_t (&key)[PER], Id id_of, int k, uint2 *list, int *count, uint32_t *bounds, Put put) {
    const int tid = (int)threadIdx.x, lane = tid & 63, wave = tid >> 6, waves = (int)blockDim.x >> 6;
    // at least k of a wave's 64 lane maxima are no less than the k-th largest of them: a bound that k entries of the row reach
    uint32_t best = 0u;
#pragma unroll
    for (int i = 0; i < PER; ++i) best = max(best, key[i]);
    int rank = 0;
#pragma unroll 8
    for (int l = 0; l < 64; ++l) {
        const uint32_t o = (uint32_t)__builtin_amdgcn_readlane((int)best, l);
        rank += (o > best || (o == best && l < lane)) ? 1 : 0;
    }
    const uint64_t at = __ballot(rank == k - 1);            // k <= 32: exactly one lane
    const uint32_t mine = (uint32_t)__builtin_amdgcn_readlane((int)best, __builtin_ctzll(at));
    if (tid == 0) *count = 0;
    if (lane == 0) bounds[wave] = mine;
    __syncthreads();
    uint32_t bound = 1u;
    for (int w = 0; w < waves; ++w) bound = max(bound, bounds[w]);
#pragma unroll
    for (int i = 0; i < PER; ++i)
        if (key[i] >= bound) {
            const int pos = atomicAdd(count, 1);            // the order is settled by the ranks below
            if (pos < LP_LIST) list[pos] = make_uint2(key[i], (uint32_t)id_of(i));
        }
    __syncthreads();
    const int n = *count;
    if (n <= LP_LIST) {                                     // uniform
        for (int e = tid; e < n; e += (int)blockDim.x) {
            const uint2 x = list[e];
            int r = 0;
            for (int o = 0; o < n; ++o) {
                const uint2 y = list[o];
                r += (y.x > x.x || (y.x == x.x && y.y < x.y)) ? 1 : 0;
            }
            if (r < k) put(r, x.x, x.y);
        }
        for (int e = n + tid; e < k; e += (int)blockDim.x) put(e, 0u, 0xffffffffu);      // fewer entries than k
        return;
    }
    // many equal logits: k rounds, each for the best entry behind the one before it
    uint32_t pk = 0xffffffffu, pi = 0u;
    bool any = false;
    for (int t = 0; t < k; ++t) {
        uint32_t bk = 0u, bi = 0xffffffffu;
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const uint32_t id = (uint32_t)id_of(i);
            const bool behind = !any || key[i] < pk || (key[i] == pk && id > pi);
            if (key[i] != 0u && behind && (key[i] > bk || (key[i] == bk && id < bi))) { bk = key[i]; bi = id; }
        }
#pragma unroll
        for (int d = 32; d > 0; d >>= 1) {
            const uint32_t ok = (uint32_t)__shfl_xor((int)bk, d, 64), oi = (uint32_t)__shfl_xor((int)bi, d, 64);
            if (ok > bk || (ok == bk && oi < bi)) { bk = ok; bi = oi; }
        }
        __syncthreads();
        if (lane == 0) list[wave] = make_uint2(bk, bi);
        __syncthreads();
        for (int w = 0; w < waves; ++w) {
            const uint2 y = list[w];
            if (y.x > bk || (y.x == bk && y.y < bi)) { bk = y.x; bi = y.y; }
        }
        pk = bk; pi = bi; any = true;
        if (tid == 0) put(t, bk, bi);
    }
}

// One workgroup per piece of a row.  Thread t holds groups of four neighbouring logits, group i at (i * threads + t) * 4 of the piece.
template <bool TOP>
__global__ __launch_bounds__(LP_MAX_THREADS) void logprob_kernel(LogprobArgs a) {
    __shared__ float sh[3][16];
    __shared__ int shi[2][16];
    __shared__ uint2 list[TOP ? LP_LIST : 1];
    __shared__ int count;
    __shared__ uint32_t bounds[16];
    const int tid = (int)threadIdx.x, lane = tid & 63, wave = tid >> 6, threads = (int)blockDim.x, waves = threads >> 6;
    const int row = (int)blockIdx.x / a.pieces, pc = (int)blockIdx.x - row * a.pieces, from = pc * a.piece, n = min(a.piece, a.V - from);
    const float *x0 = a.logits + (size_t)row * a.V + from;
    typedef float f4u __attribute__((ext_vector_type(4), aligned(4)));
    float x[LP_PER];
    const int n4 = n & ~3;
#pragma unroll
    for (int i = 0; i < LP_PER / 4; ++i) {
        const int at = (i * threads + tid) * 4;
        f4u v = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
        if (at < n4) v = *reinterpret_cast<const f4u *>(x0 + at);
        else
#pragma unroll
            for (int e = 0; e < 3; ++e)
                if (at + e < n) v[e] = x0[at + e];           // the up to three logits behind the last whole group
#pragma unroll
        for (int e = 0; e < 4; ++e) x[4 * i + e] = v[e];
    }
    auto id_of = [&](int i) { return from + ((i >> 2) * threads + tid) * 4 + (i & 3); };
    float given = INFINITY;
    if (a.rank) {
        const int tok = a.tokens[row];
        if (tok != -1) given = a.logits[(size_t)row * a.V + (tok < 0 || tok >= a.V ? 0 : tok)];
    }
    float m = -INFINITY;
    bool nan = false;
#pragma unroll
    for (int i = 0; i < LP_PER; ++i) { m = fmaxf(m, x[i]); nan |= x[i] != x[i]; }
    m = wave_max(m);
    if (__any(nan)) m = __uint_as_float(0x7fc00000u);       // a NaN makes every sum one
    if (lane == 0) sh[0][wave] = m;
    __syncthreads();
    m = sh[0][0];
    for (int w = 1; w < waves; ++w) m = m != m || sh[0][w] != sh[0][w] ? __uint_as_float(0x7fc00000u) : fmaxf(m, sh[0][w]);
    float rest = 0.f, A = 0.f;
    int peaks = 0, above = 0;
#pragma unroll
    for (int i = 0; i < LP_PER; ++i) {
        const float z = (x[i] - m) * a.inv_tau, w = x[i] < m ? __expf(z) : 0.f;
        rest += w;
        A -= w > 0.f ? w * z : 0.f;
        peaks += x[i] == m ? 1 : 0;
        above += x[i] > given ? 1 : 0;
    }
    rest = wave_sum(rest);
    A = wave_sum(A);
    const float counts = wave_sum((float)peaks), more = wave_sum((float)above);      // up to 2048 each: exact
    if (lane == 0) { sh[1][wave] = rest; sh[2][wave] = A; shi[0][wave] = (int)counts; shi[1][wave] = (int)more; }
    __syncthreads();
    rest = A = 0.f;
    peaks = above = 0;
    for (int w = 0; w < waves; ++w) { rest += sh[1][w]; A += sh[2][w]; peaks += shi[0][w]; above += shi[1][w]; }
    // a largest logit that is no number, or infinite, has no weights relative to it
    if (!(fabsf(m) < INFINITY) && a.pieces == 1) rest = __uint_as_float(0x7fc00000u);
    if (a.pieces == 1) {
        if (tid == 0) {
            const float lnz = lp_finish(a, row, m, rest, A, peaks, above);
            sh[0][0] = lnz;                                  // read behind the barriers of block_top_k
        }
        if constexpr (TOP) {
            uint32_t key[LP_PER];
#pragma unroll
            for (int i = 0; i < LP_PER; ++i) key[i] = id_of(i) < from + n ? logit_key(x[i]) : 0u;
            block_top_k(key, id_of, a.k, list, &count, bounds, [&](int t, uint32_t k, uint32_t id) {
                a.top_ids[(size_t)row * a.k + t] = (int32_t)id;
                a.top_logprobs[(size_t)row * a.k + t] = (logit_of(k) - m) * a.inv_tau - sh[0][0];
            });
        }
    } else {
        float *rec = a.records + ((size_t)row * a.pieces + pc) * lp_record_floats(a.k);
        if (tid == 0) *reinterpret_cast<LpRecord *>(rec) = LpRecord{m, rest, A, peaks, above, {0, 0, 0}};
        if constexpr (TOP) {
            uint32_t key[LP_PER];
#pragma unroll
            for (int i = 0; i < LP_PER; ++i) key[i] = id_of(i) < from + n ? logit_key(x[i]) : 0u;
            uint2 *best = reinterpret_cast<uint2 *>(rec + sizeof(LpRecord) / 4);
            block_top_k(key, id_of, a.k, list, &count, bounds, [&](int t, uint32_t k, uint32_t id) { best[t] = make_uint2(k, id); });
        }
    }
}

// Joins the records of a row: one wave, a piece per lane in turn.
template <bool TOP>
__global__ __launch_bounds__(64) void logprob_join_kernel(LogprobArgs a) {
    __shared__ uint2 list[LP_LIST];
    __shared__ int count;
    __shared__ uint32_t bounds[1];
    const int lane = (int)threadIdx.x, row = blockIdx.x;
    const float *recs = a.records + (size_t)row * a.pieces * lp_record_floats(a.k);
    LpRecord r = {-INFINITY, 0.f, 0.f, 0, 0, {0, 0, 0}};
    if (lane < a.pieces) r = *reinterpret_cast<const LpRecord *>(recs + (size_t)lane * lp_record_floats(a.k));
    float m = wave_max(r.m);
    if (__any(r.m != r.m)) m = __uint_as_float(0x7fc00000u);
    // a piece whose largest logit is below the row's: all its weights are beside the peak
    const float z = (r.m - m) * a.inv_tau, w = r.m < m ? __expf(z) : 1.0f, all = r.rest + (float)r.peaks;
    float rest = r.m < m ? (w > 0.f ? w * all : 0.f) : r.rest, A = r.m < m ? (w > 0.f ? w * (r.A - z * all) : 0.f) : r.A;
    if (lane >= a.pieces) rest = A = 0.f;
    rest = wave_sum(rest);
    A = wave_sum(A);
    const int peaks = (int)wave_sum(r.m == m && lane < a.pieces ? (float)r.peaks : 0.f), above = (int)wave_sum((float)r.above);
    if (!(fabsf(m) < INFINITY)) rest = __uint_as_float(0x7fc00000u);
    float lnz = 0.f;
    if (lane == 0) lnz = lp_finish(a, row, m, rest, A, peaks, above);
    if constexpr (TOP) {
        lnz = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(lnz), 0));
        // 64 lanes over the pieces' lists, whose entries a lane takes in turn; up to 64 * 32 entries, 32 to a lane
        uint32_t key[HYDRA_MAX_TOPK], id[HYDRA_MAX_TOPK];
#pragma unroll
        for (int i = 0; i < HYDRA_MAX_TOPK; ++i) {
            uint2 e = make_uint2(0u, 0xffffffffu);
            const int q = i * 64 + lane, p = q % a.pieces, t = q / a.pieces;          // rank t of piece p: the lanes hold the heads of all lists
            if (t < a.k) e = reinterpret_cast<const uint2 *>(recs + (size_t)p * lp_record_floats(a.k) + sizeof(LpRecord) / 4)[t];
            key[i] = e.x; id[i] = e.y;
        }
        block_top_k(key, [&](int i) { return id[i]; }, a.k, list, &count, bounds, [&](int t, uint32_t k, uint32_t i) {
            a.top_ids[(size_t)row * a.k + t] = (int32_t)i;
            a.top_logprobs[(size_t)row * a.k + t] = (logit_of(k) - m) * a.inv_tau - lnz;
        });
    }
}

static int logprob_pieces(int V, int rows) {
    (void)rows;
    return ceil_div(V, LP_PER * LP_MAX_THREADS);
}
size_t logprob_scratch_bytes(const hydra_ctx *c, int rows) { return (size_t)rows * logprob_pieces(c->m.vocab, rows) * lp_record_floats(HYDRA_MAX_TOPK) * 4; }
bool logprob_fits(const hydra_ctx *c) { return c->m.vocab <= LP_PER * LP_MAX_THREADS * LP_MAX_PIECES; }

int launch_token_logprobs(hydra_ctx *c, hipStream_t s, int rows, float *records, const float *logits, const int32_t *tokens, float tau, int k, float *logprob, int32_t *rank,
                          float *entropy, int32_t *top_ids, float *top_logprobs) {
    LogprobArgs a;
    const int V = c->m.vocab;
    a.logits = logits; a.tokens = tokens; a.logprob = logprob; a.entropy = entropy; a.top_logprobs = top_logprobs; a.rank = rank; a.top_ids = top_ids;
    a.flags = flags_dev(c); a.records = records; a.V = V; a.k = k; a.inv_tau = 1.0f / tau;
    a.pieces = logprob_pieces(V, rows);
    a.piece = (int)align_up(ceil_div(V, a.pieces), 4);
    a.pieces = ceil_div(V, a.piece);
    const int threads = std::max(64, (int)align_up(ceil_div(a.piece, LP_PER), 64));
    const dim3 grid(a.pieces * rows), block(threads);
    if (k > 0) hipLaunchKernelGGL(logprob_kernel<true>, grid, block, 0, s, a);
    else       hipLaunchKernelGGL(logprob_kernel<false>, grid, block, 0, s, a);
    HYDRA_LAUNCH_CHECK("logprob_kernel");
    if (a.pieces > 1) {
        if (k > 0) hipLaunchKernelGGL(logprob_join_kernel<true>, dim3(rows), dim3(64), 0, s, a);
        else       hipLaunchKernelGGL(logprob_join_kernel<false>, dim3(rows), dim3(64), 0, s, a);
        HYDRA_LAUNCH_CHECK("logprob_join_kernel");
    }
    return HYDRA_OK;
}

}  // namespace hydra
