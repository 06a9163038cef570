// rc_cache_write and rc_cache_read: K and V of tokens quantised into the slots of a paged 4-bit cache, and blocks read back
// out of it into the layout that rc_block_norms and the searches take.  Both stream 16 bits and 4.25 bits a value and are bound by memory:
// 64 layers of 2.1k tokens written in 151 us (0.72 GB, 4.8 TB/s), a pool of 32 layers x 1013 blocks of 32 tokens read in 943 us (5.4 GB, 5.7 TB/s;
// a copy of 8 GB runs at 6.3).  Their smallest calls are a launch, 2 to 4 us.
#include <hip/hip_runtime.h>

#include "rc_cache.hpp"

namespace rc {
namespace {

constexpr int kCacheThreads = 256;
constexpr int64_t kCacheMostWaves = (1 << 26) - 4;  // a launch has fewer than 2^32 threads along its grid

struct WriteArgs {
  const char *k, *v;
  const int32_t* slots;
  char* cache;
  int64_t token_stride_b, kv_layer_stride_b, cache_layer_stride;
  int64_t n_slots;
  uint32_t waves;  // groups of 16 tokens x heads, of a layer
  int32_t N, H, tiles;
};

// Largest magnitude of eight 16-bit values as an fp32 bit pattern (their sign bits cleared, so that patterns order like
// magnitudes, and those of infinities and NaNs come last).
template <bool BF16>
__device__ __forceinline__ uint32_t magnitude8(u32x4 x) {
  uint32_t m = 0;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const uint32_t lo = x[j] & 0x7fffu, hi = (x[j] >> 16) & 0x7fffu;
    m = max(m, max(lo, hi));
  }
  return m;
}

// The exponent byte of a group whose largest magnitude has this 16-bit pattern: the smallest x with magnitude <= 7 * 2^x, within
// what the type holds (2^x / 2 is its smallest number, or normal, and 6 * 2^x finite).  7 * 2^x is where the half step above 6
// ends, so that no element within the limits is off by more than half the step of its code.
template <bool BF16>
__device__ __forceinline__ uint32_t exponent_byte(uint32_t m16) {
  constexpr uint32_t infinity = BF16 ? 0x7f80u : 0x7c00u;
  if (m16 >= infinity) return kNanByte;
  uint32_t bits;
  if constexpr (BF16)
    bits = m16 << 16;
  else
    bits = __float_as_uint((float)__builtin_bit_cast(_Float16, (unsigned short)m16));
  // magnitude = 1.f * 2^(E - 127); 7 * 2^(E - 129) = 1.75 * 2^(E - 127): a fraction above 0.75 carries into E
  const int e = (int)((bits + 0x1fffffu) >> 23) - 2;
  return (uint32_t)min(max(e, BF16 ? 2 : 104), BF16 ? 252 : 140);
}

// Two 16-bit values to byte B of w.  (By value: a bit cast of an element of a vector takes the vector's first one.)
template <bool BF16, int B>
__device__ __forceinline__ uint32_t pack2(uint32_t w, uint32_t x, float power) {
  if constexpr (BF16)
    return __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, __builtin_bit_cast(bf16x2, x), power, B);
  else
    return __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(w, __builtin_bit_cast(f16x2, x), power, B);
}
template <bool BF16>
__device__ __forceinline__ uint32_t pack8(u32x4 x, float power) {
  return pack2<BF16, 3>(pack2<BF16, 2>(pack2<BF16, 1>(pack2<BF16, 0>(0, x[0], power), x[1], power), x[2], power), x[3], power);
}

// Eight values of a lane to a word of codes and the exponent byte of its group (the four lanes of a quad hold a group).
template <bool BF16>
__device__ __forceinline__ uint32_t quantise(u32x4 x, uint32_t& byte) {
  uint32_t m = magnitude8<BF16>(x);
  m = max(m, (uint32_t)__builtin_amdgcn_mov_dpp((int)m, 0xb1, 0xf, 0xf, true));  // quad_perm 1 0 3 2
  m = max(m, (uint32_t)__builtin_amdgcn_mov_dpp((int)m, 0x4e, 0xf, 0xf, true));  // quad_perm 2 3 0 1
  byte = exponent_byte<BF16>(m);
  return byte == kNanByte ? 0u : pack8<BF16>(x, power_of(byte));
}

// A wave takes 16 tokens of one head: lane (q, i) holds dims 8i .. 8i+7 of tokens 4q .. 4q+3, so that every load of a wave
// covers 4 x 256 bytes and a group's maximum takes two exchanges within four lanes.
template <bool BF16>
__global__ __launch_bounds__(kCacheThreads) void cache_write_kernel(WriteArgs a) {
  const int lane = threadIdx.x & 63, q = lane >> 4, i = lane & 15;
  const uint32_t w = blockIdx.x * (kCacheThreads / 64) + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (w >= a.waves) return;
  const int h = (int)(w % (uint32_t)a.H);
  const int64_t n0 = (int64_t)(w / (uint32_t)a.H) * 16 + 4 * q, l = blockIdx.y;
  const int64_t off = l * a.kv_layer_stride_b + (int64_t)h * 256 + i * 16;
  u32x4 kx[4], vx[4];
  int slot[4];
#pragma unroll
  for (int r = 0; r < 4; ++r) {
    const bool there = n0 + r < a.N;
    slot[r] = there ? a.slots[n0 + r] : -1;
    if (slot[r] < 0 || slot[r] >= a.n_slots) slot[r] = -1;
    if (there) {
      kx[r] = *(const u32x4*)(a.k + off + (n0 + r) * a.token_stride_b);
      vx[r] = *(const u32x4*)(a.v + off + (n0 + r) * a.token_stride_b);
    } else {
      kx[r] = vx[r] = u32x4{0, 0, 0, 0};
    }
  }
  char* layer = a.cache + l * a.cache_layer_stride;
#pragma unroll
  for (int r = 0; r < 4; ++r) {
    uint32_t kb, vb;
    const uint32_t kw = quantise<BF16>(kx[r], kb), vw = quantise<BF16>(vx[r], vb);
    if (slot[r] >= 0) {
      const int tile = slot[r] >> 4, t = slot[r] & 15;
      const int64_t block = tile >> (a.tiles - 1);  // of one tile or two
      char* rec = layer + ((block * a.H + h) * a.tiles + (tile & (a.tiles - 1))) * kRecordBytes;
      *(uint32_t*)(rec + ((i >> 2) * 16 + t) * 16 + (i & 3) * 4) = kw;
      *(uint32_t*)(rec + kRecordV + ((t >> 2) * 16 + i) * 16 + (t & 3) * 4) = vw;
      if ((i & 3) == 0) {
        *(uint8_t*)(rec + kRecordKExp + (i >> 2) * 16 + t) = (uint8_t)kb;
        *(uint8_t*)(rec + kRecordVExp + ((t >> 2) * 4 + (i >> 2)) * 4 + (t & 3)) = (uint8_t)vb;
      }
    }
  }
}

struct ReadArgs {
  const char* cache;
  const int32_t* ids;
  char *k, *v;
  int64_t cache_layer_stride, kv_layer_stride_b, n_blocks;
  uint32_t waves;  // records of a layer
  int32_t H, tiles;
};

// A wave takes a record; lane (q, i) writes dims 8i .. 8i+7 of tokens 4q .. 4q+3: 256 consecutive bytes of a token per 16 lanes,
// and the waves of a workgroup are neighbouring heads.  The values go out without being kept in the caches: 986 us instead of 948 for the pool
// with ordinary stores.  (Four tokens of four heads to a wave, 1024 consecutive bytes at a time: 969.)
template <bool BF16>
__global__ __launch_bounds__(kCacheThreads) void cache_read_kernel(ReadArgs a) {
  const int lane = threadIdx.x & 63, q = lane >> 4, i = lane & 15;
  const uint32_t w = blockIdx.x * (kCacheThreads / 64) + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (w >= a.waves) return;
  const int h = (int)(w % (uint32_t)a.H);
  const int64_t row = w / (uint32_t)a.H, l = blockIdx.y;  // row: tile of the output
  const int tile = (int)row & (a.tiles - 1);               // of one tile or two
  const int id = a.ids[row >> (a.tiles - 1)];
  uint32_t kw[4] = {0, 0, 0, 0}, kb = 0, vb = 0;
  u32x4 vw = {0, 0, 0, 0};
  if (id >= 0 && id < a.n_blocks) {
    const char* rec = a.cache + l * a.cache_layer_stride + (((int64_t)id * a.H + h) * a.tiles + tile) * kRecordBytes;
#pragma unroll
    for (int r = 0; r < 4; ++r) kw[r] = *(const uint32_t*)(rec + ((i >> 2) * 16 + 4 * q + r) * 16 + (i & 3) * 4);
    vw = *(const u32x4*)(rec + kRecordV + lane * 16);
    kb = *(const uint32_t*)(rec + kRecordKExp + (i >> 2) * 16 + 4 * q);
    vb = *(const uint32_t*)(rec + kRecordVExp + (q * 4 + (i >> 2)) * 4);
  }
  const int64_t off = l * a.kv_layer_stride_b + ((row * 16 + 4 * q) * a.H + h) * 256 + i * 16;
#pragma unroll
  for (int r = 0; r < 4; ++r) {
    const u32x4 kx = unpack8<BF16>(kw[r], power_at(kb, r)), vx = unpack8<BF16>(vw[r], power_at(vb, r));
    __builtin_nontemporal_store(kx, (u32x4*)(a.k + off + (int64_t)r * a.H * 256));
    __builtin_nontemporal_store(vx, (u32x4*)(a.v + off + (int64_t)r * a.H * 256));
  }
}

}  // namespace
}  // namespace rc

extern "C" size_t rc_cache_block_bytes(int32_t block_tokens, int32_t n_kv_heads, int32_t head_dim) {
  rc_cache_desc d = {1, block_tokens, n_kv_heads, head_dim, RC_F16, 0, 0};
  if (rc::check_cache(&d, "rc_cache_block_bytes")) return 0;
  return (size_t)n_kv_heads * (block_tokens / 16) * rc::kRecordBytes;
}

extern "C" rc_status rc_cache_write(const rc_cache_desc* cdesc, const void* k, const void* v, int64_t n_tokens,
                                    int64_t token_stride, int64_t kv_layer_stride, const int32_t* slots, void* cache,
                                    void* hip_stream) {
  using namespace rc;
  const char* who = "rc_cache_write";
  clear_error();
  if (rc_status s = check_cache(cdesc, who)) return s;
  const int H = cdesc->n_kv_heads;
  if (n_tokens < 0) return fail(RC_ERR_INVALID_ARG, "%s: negative size", who);
  if (n_tokens > kCacheMostWaves / H * 16) return fail(RC_ERR_UNSUPPORTED, "%s: more than 2^30 / H tokens", who);
  if (n_tokens == 0 || cdesc->n_layers == 0 || cdesc->n_blocks == 0) return RC_OK;
  if (!k || !v || !slots || !cache) return fail(RC_ERR_INVALID_ARG, "%s: NULL pointer", who);
  if (!aligned16(k) || !aligned16(v) || !aligned16(cache)) return fail(RC_ERR_INVALID_ARG, "%s: pointer not 16-byte aligned", who);
  if (token_stride < (int64_t)H * 128 || token_stride > INT64_MAX / 4 / n_tokens || token_stride % 8 != 0 || kv_layer_stride % 8 != 0)
    return fail(RC_ERR_INVALID_ARG, "%s: token_stride smaller than H*Dh, or a stride that breaks 16-byte alignment", who);
  if (cdesc->n_layers > 1 && kv_layer_stride < H * 128) return fail(RC_ERR_INVALID_ARG, "%s: kv_layer_stride smaller than a token", who);
  WriteArgs a = {(const char*)k, (const char*)v, slots, (char*)cache, token_stride * 2, kv_layer_stride * 2, cdesc->layer_stride,
                 cdesc->n_blocks * cdesc->block_tokens, (uint32_t)((n_tokens + 15) / 16 * H), (int32_t)n_tokens, H, cdesc->block_tokens / 16};
  const dim3 grid((unsigned)((a.waves + 3) / 4), (unsigned)cdesc->n_layers);
  hipStream_t st = static_cast<hipStream_t>(hip_stream);
  if (cdesc->dtype == RC_BF16)
    cache_write_kernel<true><<<grid, kCacheThreads, 0, st>>>(a);
  else
    cache_write_kernel<false><<<grid, kCacheThreads, 0, st>>>(a);
  return check_launch(who);
}

extern "C" rc_status rc_cache_read(const rc_cache_desc* cdesc, const void* cache, const int32_t* ids, int64_t n,
                                   const rc_kv_desc* kvdesc, void* k, void* v, void* hip_stream) {
  using namespace rc;
  const char* who = "rc_cache_read";
  clear_error();
  if (rc_status s = check_cache(cdesc, who)) return s;
  if (rc_status s = check_desc(kvdesc, n, who)) return s;
  if (cdesc->n_layers != kvdesc->n_layers || cdesc->block_tokens != kvdesc->block_tokens || cdesc->n_kv_heads != kvdesc->n_kv_heads ||
      cdesc->head_dim != kvdesc->head_dim || cdesc->dtype != kvdesc->dtype)
    return fail(RC_ERR_INVALID_ARG, "%s: the descriptors of the cache and of the blocks differ", who);
  const int H = cdesc->n_kv_heads, tiles = cdesc->block_tokens / 16;
  if (n > kCacheMostWaves / (H * tiles)) return fail(RC_ERR_UNSUPPORTED, "%s: too many blocks", who);
  if (n == 0 || cdesc->n_layers == 0) return RC_OK;
  // a cache of no blocks has no address: every block lies outside it, none of it is read
  if ((!cache && cdesc->n_blocks > 0) || !ids || !k || !v) return fail(RC_ERR_INVALID_ARG, "%s: NULL pointer", who);
  if (!aligned16(cache) || !aligned16(k) || !aligned16(v)) return fail(RC_ERR_INVALID_ARG, "%s: pointer not 16-byte aligned", who);
  ReadArgs a = {(const char*)cache, ids, (char*)k, (char*)v, cdesc->layer_stride, kvdesc->layer_stride * 2, cdesc->n_blocks,
                (uint32_t)(n * tiles * H), H, tiles};
  const dim3 grid((unsigned)((a.waves + 3) / 4), (unsigned)cdesc->n_layers);
  hipStream_t st = static_cast<hipStream_t>(hip_stream);
  if (cdesc->dtype == RC_BF16)
    cache_read_kernel<true><<<grid, kCacheThreads, 0, st>>>(a);
  else
    cache_read_kernel<false><<<grid, kCacheThreads, 0, st>>>(a);
  return check_launch(who);
}
