// Pages of a paged cache (tkv_paged_desc): where a token's row lies, and the 4-bit blocks.
#pragma once

#include "tkv_common.h"

namespace tkv {

// A row of 4-bit pages: 64 bytes of codes, and 4 of scales behind the codes of all the page's tokens.
constexpr int kRow4 = TKV_D / 2, kScales4 = TKV_D / 32;

struct Pages {
  void* k;
  void* v;
  int64_t k_sp, k_sh, k_st, v_sp, v_sh, v_st;  // strides of pages, heads and tokens, in elements (16 bits) or bytes of codes (4)
  int32_t shift;                               // log2 of the page's tokens
  int32_t n_pages;
  int32_t hkv;
};

// The scale of a 4-bit block as a number: 2^(byte - 127), NaN for 255.
__device__ inline float scale_of(uint32_t byte) { return __builtin_bit_cast(float, byte == 255u ? 0x7FC00000u : byte << 23); }

// Eight codes (channel 2 i in the low half of byte i) to eight numbers of the type.  (Exact: see tkv_paged_append.)
template <typename T>
__device__ inline tkv_u32x4 values_of(uint32_t codes, float scale) {
  tkv_u32x4 r;
  if constexpr (__is_same(T, _Float16)) {
    r.x = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(codes, scale, 0));
    r.y = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(codes, scale, 1));
    r.z = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(codes, scale, 2));
    r.w = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(codes, scale, 3));
  } else {
    r.x = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 0));
    r.y = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 1));
    r.z = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 2));
    r.w = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 3));
  }
  return r;
}

// Smallest exponent of a 4-bit block: half of 2^lowest is the type's smallest number (fp16), or its smallest that is not subnormal (bf16).
inline int32_t lowest_exponent(int32_t dtype) { return dtype == TKV_F16 ? -23 : -125; }

int32_t check_paged_desc(const tkv_paged_desc* d);
// Addresses and strides for the kernels; TKV_E_INVAL where an address is NULL or not at a multiple of 16 bytes.
int32_t paged_view(const tkv_paged_desc* d, void* k_pages, void* v_pages, Pages* out);

}  // namespace tkv
