// The 4-bit KV cache: its format, and what the kernels that write, read and attend over it share.
//
// A block of T tokens of one KV head is a run of T / 16 records, a record holds 16 tokens' K and V:
//   bytes    0 .. 1023   K codes      group g (32 dims), token t: 16 bytes at (g * 16 + t) * 16, dim g * 32 + e in the half byte e
//   bytes 1024 .. 2047   V codes      tokens 4q .. 4q+3, dims 8i .. 8i+7: 16 bytes at (q * 16 + i) * 16, token 4q + r in its word r
//   bytes 2048 .. 2111   K exponents  g * 16 + t
//   bytes 2112 .. 2175   V exponents  (q * 4 + g) * 4 + r
// Both orders are those of a 16x16x32 matrix instruction's operands: lane l reads the 16 bytes at l * 16 and holds 32 dims of
// one token of K (one group, one power), or 8 dims of 4 tokens of V, and no value ever moves between lanes.
//
// Elements are e2m1 codes under a power of two per group of 32, which the hardware's conversions take as they are
// (v_cvt_scalef32_pk_*_fp4 at the rate of any other vector instruction: 5.2 cycles a wave instruction with the clock taken as
// 2.4 GHz, a v_fma_f32 5.1); code * 2^x is exact in fp16 and bf16 alike, so that reading and attending see the same numbers.
#pragma once
#include <hip/hip_runtime.h>

#include "rc_common.hpp"

namespace rc {

constexpr int kRecordBytes = 2176, kRecordV = 1024, kRecordKExp = 2048, kRecordVExp = 2112;
constexpr int kNanByte = 255, kOneByte = 127;

typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));
typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));

// The exponent byte b as the fp32 number that the conversions take: they use its exponent field, which makes 255 a NaN, and nothing
// else of it (checked for all 256 exponents under any sign and fraction), so that byte `r` of a word takes one shift.
__device__ __forceinline__ float power_of(uint32_t b) { return __uint_as_float(b << 23); }
__device__ __forceinline__ float power_at(uint32_t w, int r) { return __uint_as_float(r == 3 ? w >> 1 : w << (23 - 8 * r)); }

// Byte `B` (0 .. 3) of w: two codes, low half byte first, as two 16-bit values.
template <bool BF16, int B>
__device__ __forceinline__ uint32_t unpack2(uint32_t w, float power) {
  if constexpr (BF16)
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, power, B));
  else
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, power, B));
}
// The eight codes of a word.
template <bool BF16>
__device__ __forceinline__ u32x4 unpack8(uint32_t w, float power) {
  return u32x4{unpack2<BF16, 0>(w, power), unpack2<BF16, 1>(w, power), unpack2<BF16, 2>(w, power), unpack2<BF16, 3>(w, power)};
}

// Checks of a cache's descriptor, shared by the entry points that take one.
inline rc_status check_cache(const rc_cache_desc* d, const char* who) {
  if (!d) return fail(RC_ERR_INVALID_ARG, "%s: cache descriptor is NULL", who);
  if (d->n_layers < 0 || d->n_blocks < 0) return fail(RC_ERR_INVALID_ARG, "%s: negative size", who);
  if (d->dtype != RC_F16 && d->dtype != RC_BF16) return fail(RC_ERR_UNSUPPORTED, "%s: dtype %d", who, d->dtype);
  if (d->head_dim != 128) return fail(RC_ERR_UNSUPPORTED, "%s: head_dim %d (only 128)", who, d->head_dim);
  if (d->block_tokens != 16 && d->block_tokens != 32)
    return fail(RC_ERR_UNSUPPORTED, "%s: block_tokens %d (only 16 or 32)", who, d->block_tokens);
  if (d->n_kv_heads < 1 || d->n_kv_heads > 16)
    return fail(RC_ERR_UNSUPPORTED, "%s: n_kv_heads %d (1..16)", who, d->n_kv_heads);
  if (d->n_layers > 65535) return fail(RC_ERR_UNSUPPORTED, "%s: more than 65535 layers", who);
  if (d->n_blocks > 0x7fffffffLL / d->block_tokens)
    return fail(RC_ERR_UNSUPPORTED, "%s: more than 2^31 - 1 slots (n_blocks * T)", who);
  const int64_t block = (int64_t)d->n_kv_heads * (d->block_tokens / 16) * kRecordBytes;
  if (d->layer_stride < d->n_blocks * block)
    return fail(RC_ERR_INVALID_ARG, "%s: layer_stride %lld smaller than n_blocks * rc_cache_block_bytes()", who,
                (long long)d->layer_stride);
  if (d->layer_stride % 16 != 0) return fail(RC_ERR_INVALID_ARG, "%s: layer_stride breaks 16-byte alignment", who);
  return RC_OK;
}

}  // namespace rc
