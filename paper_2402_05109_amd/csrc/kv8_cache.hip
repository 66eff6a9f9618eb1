// The KV cache in 8 bits: sealing pages, reading them back, copying whole pages (of either cache).
#include <algorithm>

#include "kv8.h"

namespace hydra {

typedef __attribute__((ext_vector_type(4))) uint32_t u32x4_t;
typedef __attribute__((ext_vector_type(4))) float f32x4_t;

// Which pages of a row are to be sealed: [n0, full).  False: the row is out of range.
__device__ __forceinline__ bool seal_range(int L, int n0, int max_pages8, int max_pages, int &full) {
    full = L >> 4;
    return L >= 0 && n0 >= 0 && n0 <= full && full <= max_pages8 && full <= max_pages;
}

// Scale of a block by its largest magnitude.  int8: top / 127 rounded up to 11 significant bits, so that x / scale (x has 11) is either
// a tie exactly or at least 2^-13 from one, and 32 bits decide every rounding as exact arithmetic does.
template <int FMT>
__device__ __forceinline__ float kv8_scale(float top) {
    if (top == 0.f) return 1.f;
    if (FMT == KV8_INT8) return __uint_as_float((__float_as_uint(top / 127.f) + 0x1fffu) & ~0x1fffu);
    const uint32_t u = __float_as_uint(top);                            // top in (1.75 2^(e - 1), 1.75 2^e] * 2^8 -> 2^e
    const int e = (int)(u >> 23) - 8 + ((u & 0x7fffffu) > 0x600000u ? 1 : 0);
    return __uint_as_float((uint32_t)e << 23);
}

// A lane's four values (finite: the cache saturates what is written) -> four codes.  r = 1 / scale.
template <int FMT>
__device__ __forceinline__ uint32_t kv8_codes(const float *x, float s, float r) {
    if (FMT == KV8_INT8) {
        uint32_t w = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            float y = x[i] * r;
            y = fmaf(fmaf(-y, s, x[i]), r, y);                          // the quotient to the last bit
            const int q = (int)rintf(fminf(fmaxf(y, -127.f), 127.f));
            w |= (uint32_t)(q + KV8_BIAS) << (8 * i);
        }
        return w;
    }
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(x[0] * r, x[1] * r, 0, false);          // r is a power of two
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(x[2] * r, x[3] * r, w, true);
}

// One wave seals the K or the V of one page and head: 16 * DH halves in, as many bytes out, one maximum in between.  All of a block is in
// registers (32 or 16 values a lane), so it is read once; bound by memory.
template <int DH, int FMT>
__global__ __launch_bounds__(256) void kv8_seal_kernel(const a16_t *__restrict__ kpages, const a16_t *__restrict__ vpages,
                                                        const int32_t *__restrict__ table16, int max_pages, int n_pages,
                                                        uint8_t *__restrict__ kcodes, uint8_t *__restrict__ vcodes, float *__restrict__ scales,
                                                        const int32_t *__restrict__ table8, int max_pages8, int n_pages8,
                                                        const int32_t *__restrict__ n_sealed, const int32_t *__restrict__ seq_len, int H, int32_t *flags) {
    constexpr int RUNS = DH / 64;                                        // 16-byte runs of codes per lane
    const int layer = blockIdx.y, b = blockIdx.z, lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int L = seq_len[b], n0 = n_sealed[b];
    int full;
    const bool first = blockIdx.x == 0 && layer == 0 && threadIdx.x == 0;
    if (!seal_range(L, n0, max_pages8, max_pages, full)) {
        if (first) atomicOr(flags, FLAG_CAPACITY);
        return;
    }
    const int tasks = (full - n0) * H * 2;
    for (int task = blockIdx.x * 4 + wave; task < tasks; task += gridDim.x * 4) {
        const int kv = task & 1, h = (task >> 1) % H, i = n0 + (task >> 1) / H;
        const int page = table16[(size_t)b * max_pages + i], page8 = table8[(size_t)b * max_pages8 + i];
        if ((unsigned)page >= (unsigned)n_pages || (unsigned)page8 >= (unsigned)n_pages8) {       // the row then keeps its n_sealed
            if (lane == 0) atomicOr(flags, FLAG_BAD_PAGE);
            continue;
        }
        const u32x4_t *src = reinterpret_cast<const u32x4_t *>((kv ? vpages : kpages) + kv_block_base(layer, n_pages, page, H, h, DH));
        u32x4_t in[RUNS][2];
#pragma unroll
        for (int r = 0; r < RUNS; ++r) {
            const int run = r * 64 + lane;                               // K: (dim / 16, token); V: (dim / 64, half-wave, dim % 32)
            const int a = kv ? (64 * r + (lane & 31)) * 2 + (lane >> 5) : (run >> 4) * 32 + (run & 15);
            in[r][0] = src[a];
            in[r][1] = src[a + (kv ? 64 : 16)];
        }
        float x[RUNS][16], top = 0.f;
#pragma unroll
        for (int r = 0; r < RUNS; ++r)
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const uint32_t w = in[r][e >> 2][e & 3];
                x[r][2 * e] = a2f((a16_t)w);
                x[r][2 * e + 1] = a2f((a16_t)(w >> 16));
                top = fmaxf(top, fmaxf(fabsf(x[r][2 * e]), fabsf(x[r][2 * e + 1])));
            }
        top = fminf(wave_max(top), 65504.f);
        const float s = kv8_scale<FMT>(top), inv = 1.0f / s;
        u32x4_t *dst = reinterpret_cast<u32x4_t *>((kv ? vcodes : kcodes) + kv8_block_base(layer, n_pages8, page8, H, h, DH));
#pragma unroll
        for (int r = 0; r < RUNS; ++r) {
            u32x4_t out;
#pragma unroll
            for (int e = 0; e < 4; ++e) out[e] = kv8_codes<FMT>(&x[r][4 * e], s, inv);
            dst[r * 64 + lane] = out;
        }
        if (lane == 0) scales[(((size_t)layer * n_pages8 + page8) * H + h) * 2 + kv] = s;
    }
}

// n_sealed follows once every page of the row is sealed; a row with a bad table entry keeps it.
__global__ __launch_bounds__(256) void kv8_sealed_kernel(const int32_t *__restrict__ table16, int max_pages, int n_pages, const int32_t *__restrict__ table8,
                                                          int max_pages8, int n_pages8, int32_t *n_sealed, const int32_t *__restrict__ seq_len) {
    const int b = blockIdx.x;
    const int L = seq_len[b], n0 = n_sealed[b];
    int full;
    if (!seal_range(L, n0, max_pages8, max_pages, full)) return;
    bool bad = false;
    for (int i = n0 + (int)threadIdx.x; i < full; i += 256)
        bad |= (unsigned)table16[(size_t)b * max_pages + i] >= (unsigned)n_pages || (unsigned)table8[(size_t)b * max_pages8 + i] >= (unsigned)n_pages8;
    if (__syncthreads_or(bad)) return;
    if (threadIdx.x == 0) n_sealed[b] = full;
}

int launch_kv8_seal(hydra_ctx *c, hipStream_t s, int B, const int32_t *seq_len, const hydra_kv8 *kv) {
    const int H = c->m.n_heads, Dh = c->m.head_dim;
    // As many waves as a step of the context's tree can complete pages (with twice as many, half of them without work, 16 rows x 8 layers of a page each
    // took 19 us instead of 15), but workgroups for all of the chip where layers and rows are few: a row with more pages goes round, and a whole cache
    // of 32000 tokens sealed at once, 40 heads, takes 203 us, 1090 with the waves of a 32-node tree
    const int step = ceil_div(ceil_div(c->tree.T, 16) * H * 2, 4), chip = ceil_div(2048, c->m.n_layers * B);
    const dim3 grid(std::max(step, chip), c->m.n_layers, B), block(256);
#define SEAL(DHv, Fv)                                                                                                                              \
    hipLaunchKernelGGL((kv8_seal_kernel<DHv, Fv>), grid, block, 0, s, (const a16_t *)kv->tail.k_pages, (const a16_t *)kv->tail.v_pages,            \
                       kv->tail.page_table, kv->tail.max_pages, kv->tail.n_pages, (uint8_t *)kv->k_codes, (uint8_t *)kv->v_codes, kv->scales,      \
                       kv->page_table, kv->max_pages, kv->n_pages, kv->n_sealed, seq_len, H, flags_dev(c))
    if (Dh == 128) { if (kv->format == KV8_INT8) SEAL(128, KV8_INT8); else SEAL(128, KV8_E4M3); }
    else           { if (kv->format == KV8_INT8) SEAL(64, KV8_INT8); else SEAL(64, KV8_E4M3); }
#undef SEAL
    HYDRA_LAUNCH_CHECK("kv8_seal_kernel");
    hipLaunchKernelGGL(kv8_sealed_kernel, dim3(B), dim3(256), 0, s, kv->tail.page_table, kv->tail.max_pages, kv->tail.n_pages, kv->page_table, kv->max_pages,
                       kv->n_pages, kv->n_sealed, seq_len);
    HYDRA_LAUNCH_CHECK("kv8_sealed_kernel");
    return HYDRA_OK;
}

// Plain values of the slots first .. first + n - 1: one wave per logical page, head and K or V.  Bound by the stores (four bytes for each code read),
// so a lane always holds four consecutive dims of a token and 32 (16) lanes write a token's whole 512 (256) bytes.
template <int DH, int FMT>
__global__ __launch_bounds__(256) void kv8_read_kernel(const a16_t *__restrict__ kpages, const a16_t *__restrict__ vpages,
                                                        const int32_t *__restrict__ table16, int max_pages, int n_pages,
                                                        const uint8_t *__restrict__ kcodes, const uint8_t *__restrict__ vcodes, const float *__restrict__ scales,
                                                        const int32_t *__restrict__ table8, int max_pages8, int n_pages8, const int32_t *__restrict__ n_sealed,
                                                        int layer0, int B, int first, int n, int H, float *__restrict__ plain, int32_t *flags) {
    constexpr int QUADS = DH / 4, TOKS = 64 / QUADS;         // lanes of a token, tokens of a wave's store
    const int lane = threadIdx.x & 63, task = (int)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int kv = task & 1, h = (task >> 1) % H, i = (first >> 4) + (task >> 1) / H, b = (int)blockIdx.y, l = (int)blockIdx.z, layer = layer0 + l;
    if (i > (first + n - 1) >> 4) return;
    const bool sealed = i < min(n_sealed[b], max_pages8);
    const int page = sealed ? table8[(size_t)b * max_pages8 + i] : table16[(size_t)b * max_pages + i];
    if ((unsigned)page >= (unsigned)(sealed ? n_pages8 : n_pages)) {
        if (lane == 0) atomicOr(flags, FLAG_BAD_PAGE);
        return;
    }
    const int dim = lane % QUADS * 4, t0 = lane / QUADS;
    float *const out = plain + (((((size_t)l * B + b) * n) * 2 + kv) * H + h) * DH + dim;          // of slot `first`
    const size_t stride = (size_t)2 * H * DH;
    auto put = [&](int tok, f32x4_t v) {
        const int slot = i * 16 + tok - first;
        if (slot >= 0 && slot < n) __builtin_nontemporal_store(v, reinterpret_cast<f32x4_t *>(out + slot * stride));
    };
    if (sealed) {
        const uint8_t *src = (kv ? vcodes : kcodes) + kv8_block_base(layer, n_pages8, page, H, h, DH);
        const float s = scales[(((size_t)layer * n_pages8 + page) * H + h) * 2 + kv];
        if (kv == 0) {
#pragma unroll
            for (int r = 0; r < 16 / TOKS; ++r) {
                const int tok = r * TOKS + t0;
                const uint32_t w = *reinterpret_cast<const uint32_t *>(src + k8_in_block(tok, dim));
                put(tok, f32x4_t{s * kv8_value<FMT>(w & 255u), s * kv8_value<FMT>((w >> 8) & 255u), s * kv8_value<FMT>((w >> 16) & 255u), s * kv8_value<FMT>(w >> 24)});
            }
        } else {
            typedef __attribute__((ext_vector_type(2))) uint32_t u2;
            // a lane's share of the 16 tokens: 16 / TOKS of them that lie together, tokens v_perm^-1 of TOKS-th parts of 0 .. 15
            constexpr int RUN = 16 / TOKS;                   // 8 with 128 dims, 4 with 64: bytes of one dim
            u2 w[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int d = dim + e, p0 = t0 * RUN, at = (((d >> 6) * 2 + (p0 >> 3)) * 32 + (d & 31)) * 16 + ((d >> 5) & 1) * 8 + (p0 & 7);
                w[e][0] = *reinterpret_cast<const uint32_t *>(src + at);
                w[e][1] = RUN == 8 ? *reinterpret_cast<const uint32_t *>(src + at + 4) : 0u;
            }
#pragma unroll
            for (int r = 0; r < RUN; ++r) {
                const int q = t0 * RUN + r, tok = ((q & 7) >> 2) * 8 + (q >> 3) * 4 + (q & 3);        // v_perm(tok) == q
                f32x4_t v;
#pragma unroll
                for (int e = 0; e < 4; ++e) v[e] = s * kv8_value<FMT>((w[e][r >> 2] >> (8 * (r & 3))) & 255u);
                put(tok, v);
            }
        }
    } else {
        const a16_t *src = (kv ? vpages : kpages) + kv_block_base(layer, n_pages, page, H, h, DH);
        for (int tok = t0; tok < 16; tok += TOKS) {
            f32x4_t v;
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = a2f(src[kv ? v_in_block<true>(tok, dim + e, DH) : k_in_block<true>(tok, dim + e, DH)]);
            put(tok, v);
        }
    }
}

int launch_kv8_read(hydra_ctx *c, hipStream_t s, int B, int layer, const hydra_kv8 *kv, int first_slot, int n_slots, float *plain) {
    const int H = c->m.n_heads, Dh = c->m.head_dim, NL = layer < 0 ? c->m.n_layers : 1;
    const int pages = (first_slot + n_slots - 1) / 16 - first_slot / 16 + 1;
    const dim3 grid(ceil_div(pages * H * 2, 4), B, NL), block(256);
#define READ(DHv, Fv)                                                                                                                               \
    hipLaunchKernelGGL((kv8_read_kernel<DHv, Fv>), grid, block, 0, s, (const a16_t *)kv->tail.k_pages, (const a16_t *)kv->tail.v_pages, kv->tail.page_table, \
                       kv->tail.max_pages, kv->tail.n_pages, (const uint8_t *)kv->k_codes, (const uint8_t *)kv->v_codes, kv->scales, kv->page_table,     \
                       kv->max_pages, kv->n_pages, kv->n_sealed, layer < 0 ? 0 : layer, B, first_slot, n_slots, H, plain, flags_dev(c))
    if (Dh == 128) { if (kv->format == KV8_INT8) READ(128, KV8_INT8); else READ(128, KV8_E4M3); }
    else           { if (kv->format == KV8_INT8) READ(64, KV8_INT8); else READ(64, KV8_E4M3); }
#undef READ
    HYDRA_LAUNCH_CHECK("kv8_read_kernel");
    return HYDRA_OK;
}

}  // namespace hydra
