// The KV cache in 8 bits: codes, scales and their placement (include/hydra.h, hydra_kv8).
//
// One block is a page (16 tokens) of one layer and head, 16 * Dh bytes for K and as many for V.  Placement inside a block: 16-byte runs
// that a lane of the attention kernel takes with one load, a wave's load touching 256-byte (K) or 512-byte (V) pieces:
//   K  [dim / 16][token][dim % 16]
//   V  [dim / 64][half-wave][dim % 32][(dim / 32) % 2][8 tokens], the half-wave and place of a token being those of v_perm()
// so that 8 bytes of a run are one lane's operand of a 32x32x16 product, once they are halves.
#pragma once

#include "device_common.h"
#include "internal.h"

namespace hydra {

enum { KV8_INT8 = HYDRA_KV8_INT8, KV8_E4M3 = HYDRA_KV8_E4M3 };
enum { KV8_BIAS = 128 };                 // int8 codes are kept as code + 128, in [1, 255]

typedef __attribute__((ext_vector_type(2))) _Float16 h16x2_t;

__device__ __forceinline__ size_t kv8_block_base(int layer, int n_pages, int page, int H, int head, int Dh) {
    return ((((size_t)layer * n_pages + page) * H) + head) * (size_t)(16 * Dh);
}
__device__ __forceinline__ int k8_in_block(int tok, int dim) { return ((dim >> 4) * 16 + tok) * 16 + (dim & 15); }
__device__ __forceinline__ int v8_in_block(int tok, int dim) {
    const int p = v_perm(tok);
    return (((dim >> 6) * 2 + (p >> 3)) * 32 + (dim & 31)) * 16 + ((dim >> 5) & 1) * 8 + (p & 7);
}

// Four codes of a dword -> two pairs of halves, exactly.  int8: byte b under the high byte 0x64 is the half 1024 + b, from which
// 1024 + 128 is taken.  e4m3: the hardware converter.
template <int FMT>
__device__ __forceinline__ void kv8_halves(uint32_t w, uint32_t &lo, uint32_t &hi) {
    if (FMT == KV8_INT8) {
        const h16x2_t bias = {(_Float16)(1024 + KV8_BIAS), (_Float16)(1024 + KV8_BIAS)};
        lo = __builtin_bit_cast(uint32_t, __builtin_bit_cast(h16x2_t, __builtin_amdgcn_perm(w, 0x64646464u, 0x00050004u)) - bias);
        hi = __builtin_bit_cast(uint32_t, __builtin_bit_cast(h16x2_t, __builtin_amdgcn_perm(w, 0x64646464u, 0x00070006u)) - bias);
    } else {
        lo = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, 1.0f, false));
        hi = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, 1.0f, true));
    }
}
// code byte -> its value before the scale
template <int FMT>
__device__ __forceinline__ float kv8_value(uint32_t byte) {
    if (FMT == KV8_INT8) return (float)((int)byte - KV8_BIAS);
    return __builtin_amdgcn_cvt_f32_fp8((int)byte, 0);
}

}  // namespace hydra
