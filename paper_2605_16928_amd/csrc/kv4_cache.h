// The 4-bit K/V cache: where a token's bytes lie, and the checks of its descriptor (kv4_store.hip fills and reads it,
// kv4_attn.hip attends over it).
//
// A row of 128 values is four blocks of 32 consecutive ones; a block is a scale byte s, standing for 2^(s - 127), and 32 codes
// of e2m1 (sign, 2 exponent bits, 1 mantissa bit: 0, .5, 1, 1.5, 2, 3, 4, 6).  gfx950 converts between 16-bit values and such codes
// with the scale in one instruction per pair, which is why the cache is kept in this form and not in integers with an offset.
//
// One (page, KV head) holds page_size records of 128 bytes -- K in the first 64, V in the other 64, so that a gathered token is one
// cache line -- and page_size / 4 groups of 32 scale bytes: [K or V][block][token % 4].  The group form is for the attention: a lane
// of the PV product holds one block of four neighbouring tokens, whose scales it loads as one word.
#pragma once

#include "common.h"

namespace rtp {

constexpr int kKv4Row = 128;          // bytes of codes per token and KV head
constexpr int kKv4Group = 32;         // bytes of scales per four tokens and KV head

struct Kv4Cache {
  uint8_t* codes;
  uint8_t* scales;
  int64_t code_head_stride, scale_head_stride;     // bytes
  uint32_t code_page16, scale_page16;              // pages' strides in 16 bytes
  const int32_t* page_table;
  int64_t pt_stride;
  int32_t page_shift, n_pages;
};

// Checks the descriptor for sequences of up to max_tokens tokens (0: positions are known on the device only).
int32_t check_kv4_cache(const char* who, const rtp_layer_desc* L, const rtp_kv4_cache* c, int64_t max_tokens, Kv4Cache* out);

// The pool page that holds a position of the sequence whose table row is pt, or -1: a position behind the table and a page that is
// not one of the pool's are never followed.
__device__ __forceinline__ int kv4_page(const Kv4Cache& c, const int32_t* pt, int pos) {
  const int k = pos >> c.page_shift;
  if (pos < 0 || k >= c.pt_stride) return -1;
  const int page = pt[k];
  return (uint32_t)page < (uint32_t)c.n_pages ? page : -1;
}

// Scale byte of lane field i (0 .. 3) of a word of four, as the fp32 power of two that the conversions take (0 stands for 2^-127
// there, 255 makes every converted value NaN).
__device__ __forceinline__ float kv4_scale(uint32_t word, int i) {
  return __uint_as_float(((word >> (8 * i)) & 255u) << 23);      // (one instruction: a shift with a byte select)
}

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x2_t __attribute__((ext_vector_type(2)));
// Eight codes of one block as 16-bit values (bf16: exact; fp16: one rounding where the value is none of fp16's).
template <bool F16>
__device__ __forceinline__ u32x4 decode8(uint32_t codes, float scale) {
  u32x4 r;
  if constexpr (F16) {
    const f32x2_t a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, scale, 0), b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, scale, 1);
    const f32x2_t c = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, scale, 2), d = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, scale, 3);
    r[0] = f32_to_f16_rne(a.x) | ((uint32_t)f32_to_f16_rne(a.y) << 16);
    r[1] = f32_to_f16_rne(b.x) | ((uint32_t)f32_to_f16_rne(b.y) << 16);
    r[2] = f32_to_f16_rne(c.x) | ((uint32_t)f32_to_f16_rne(c.y) << 16);
    r[3] = f32_to_f16_rne(d.x) | ((uint32_t)f32_to_f16_rne(d.y) << 16);
  } else {
    r[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 0));
    r[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 1));
    r[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 2));
    r[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 3));
  }
  return r;
}

}  // namespace rtp
