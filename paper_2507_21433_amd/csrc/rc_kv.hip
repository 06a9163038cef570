// rc_kv_write: K and V of new tokens into the slots of 16-bit paged KV blocks.  rc_kv_evict: table entries whose blocks gathered the least attention leave.
#include <hip/hip_runtime.h>

#include "rc_kv.hpp"
#include "rc_vec.hpp"

namespace rc {
namespace {

constexpr int kKvThreads = 256;

// ---- rc_kv_write

// A copy, bound by memory: a thread moves 16 bytes of K and of V at a time, four of each, neighbouring threads neighbouring ones.
struct KvWriteArgs {
  const char *k_new, *v_new;
  const int32_t* slots;
  char *k, *v;
  int64_t token_stride_b, new_layer_stride_b, layer_stride_b, n_slots;
  uint32_t units, heads;  // of 16 bytes of a layer's K, KV heads
};
constexpr int kWriteEach = 4;

__global__ __launch_bounds__(kKvThreads) void kv_write_kernel(KvWriteArgs a) {
  const int64_t l = blockIdx.y;
  u32x4 x[kWriteEach], y[kWriteEach];
  int64_t to[kWriteEach];
#pragma unroll
  for (int i = 0; i < kWriteEach; ++i) {
    const uint32_t u = (blockIdx.x * kWriteEach + i) * kKvThreads + threadIdx.x;
    to[i] = -1;
    if (u < a.units) {
      const uint32_t row = u >> 4, n = row / a.heads, in_token = (row - n * a.heads) * 256 + (u & 15) * 16;
      const int32_t slot = a.slots[n];
      const int64_t from = l * a.new_layer_stride_b + (int64_t)n * a.token_stride_b + in_token;
      x[i] = *(const u32x4*)(a.k_new + from);
      y[i] = *(const u32x4*)(a.v_new + from);
      if (slot >= 0 && slot < a.n_slots) to[i] = l * a.layer_stride_b + (int64_t)slot * (a.heads * 256) + in_token;
    }
  }
#pragma unroll
  for (int i = 0; i < kWriteEach; ++i) {
    if (to[i] < 0) continue;
    *(u32x4*)(a.k + to[i]) = x[i];
    *(u32x4*)(a.v + to[i]) = y[i];
  }
}

// ---- rc_kv_evict

struct EvictArgs {
  const int32_t* tables_in;
  int32_t* tables_out;
  int64_t L, R, E, NB;
  int32_t T;
  const int32_t *ctx_len, *keep;
  const float* weights;
  int64_t n_first, n_last;
  int32_t *refcount, *n_evicted;
};

// The order of weights as that of whole numbers: -0 and 0 are equal, NaN is the largest.  What may not leave comes behind them all.
constexpr uint32_t kStays = 0xffffffffu;
__device__ __forceinline__ uint32_t weight_key(float w) {
  const uint32_t b = __float_as_uint(w + 0.f);
  if (w != w) return kStays - 1;
  return b >> 31 ? ~b : b | 0x80000000u;
}

// A row is the table of one request in one layer.  Its keys lie in registers where they fit (entry i * threads + thread at place i), else they are read
// again for every pass.  The n-th smallest key is found byte by byte from the top with a histogram of the entries that agree so far; of those equal to
// it the first ones leave.
template <int WAVES, int ITEMS>  // ITEMS: entries of a thread held in registers, 0: none
struct EvictRow {
  static constexpr int kRowThreads = 64 * WAVES;
  const EvictArgs& a;
  const int32_t* in;
  const float* weights;
  int32_t E;
  int32_t used, thread;
  uint32_t* histogram;  // LDS, 256
  uint32_t* scratch;    // LDS, 16 + a few
  uint32_t key[ITEMS ? ITEMS : 1];
  int32_t id[ITEMS ? ITEMS : 1];

  __device__ __forceinline__ void sync() const {
    if constexpr (WAVES > 1)
      __syncthreads();
    else
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  }
  __device__ __forceinline__ bool held(int32_t i, int32_t e) const { return e < used && i >= 0 && i < a.NB; }
  __device__ __forceinline__ uint32_t make_key(int32_t i, int32_t e) const {
    return held(i, e) && e >= a.n_first && e < used - a.n_last ? weight_key(weights[e]) : kStays;
  }
  // f(place, entry, id, key) for every entry of the thread; the same number of turns for all lanes of the row.
  template <class F>
  __device__ __forceinline__ void each(F f) {
    if constexpr (ITEMS) {
#pragma unroll
      for (int i = 0; i < ITEMS; ++i)
        if (i * kRowThreads < E) f(i * kRowThreads + thread, id[i], key[i]);
    } else {
      for (int32_t base = 0; base < E; base += kRowThreads) {
        const int32_t e = base + thread, j = e < E ? in[e] : -1;
        f(e, j, make_key(j, e));
      }
    }
  }
  __device__ __forceinline__ uint32_t sum(uint32_t x) {
#pragma unroll
    for (int d = 32; d; d >>= 1) x += __shfl_xor(x, d);
    if constexpr (WAVES > 1) {
      if ((thread & 63) == 0) scratch[thread >> 6] = x;
      __syncthreads();
      x = 0;
      for (int i = 0; i < WAVES; ++i) x += scratch[i];
      __syncthreads();
    }
    return x;
  }
};

template <int WAVES, int ITEMS>
__global__ __launch_bounds__(WAVES == 1 ? 256 : 64 * WAVES) void kv_evict_kernel(EvictArgs a) {
  constexpr int kRows = WAVES == 1 ? 4 : 1;
  using Row = EvictRow<WAVES, ITEMS>;
  __shared__ __attribute__((aligned(16))) uint32_t histogram[kRows][256], scratch[kRows][32];
  const int in_block = WAVES == 1 ? (int)(threadIdx.x >> 6) : 0;
  const int64_t lr = (int64_t)blockIdx.x * kRows + in_block;
  if (lr >= a.L * a.R) return;
  const int64_t l = lr / a.R, r = lr - l * a.R;
  Row row{a, a.tables_in + lr * a.E, a.weights + lr * a.E, (int32_t)a.E, 0, (int)(WAVES == 1 ? threadIdx.x & 63 : threadIdx.x), histogram[in_block], scratch[in_block], {}, {}};
  int32_t* out = a.tables_out + lr * a.E;
  const int32_t ctx = a.ctx_len[r], keep = a.keep[r];
  const int64_t blocks = ctx > 0 ? ((int64_t)ctx + a.T - 1) / a.T : 0;
  row.used = (int32_t)(blocks < a.E ? blocks : a.E);
  if constexpr (ITEMS) {
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
      const int32_t e = i * Row::kRowThreads + row.thread;
      row.id[i] = e < row.E ? row.in[e] : -1;
    }
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) row.key[i] = row.make_key(row.id[i], i * Row::kRowThreads + row.thread);
  }
  uint32_t held = 0, may = 0;
  row.each([&](int32_t e, int32_t i, uint32_t k) { held += row.held(i, e), may += k != kStays; });
  held = row.sum(held), may = row.sum(may);
  uint32_t n = held > (uint32_t)max(keep, 0) ? held - (uint32_t)max(keep, 0) : 0;
  n = min(n, may);
  if (row.thread == 0) a.n_evicted[lr] = (int32_t)n;
  const bool same = a.tables_in == a.tables_out;
  if (n == 0) {
    if (!same) row.each([&](int32_t e, int32_t i, uint32_t) { if (e < row.E) out[e] = i; });
    return;
  }
  // the n-th smallest key, and how many equal to it leave
  uint32_t prefix = 0, mask = 0, equal = n;
#pragma unroll 1
  for (int shift = 24; shift >= 0; shift -= 8) {
    for (int i = row.thread; i < 256; i += Row::kRowThreads) row.histogram[i] = 0;
    row.sync();
    row.each([&](int32_t, int32_t, uint32_t k) { if (k != kStays && (k & mask) == prefix) atomicAdd(&row.histogram[k >> shift & 255], 1u); });
    row.sync();
    // every wave finds the byte by itself: four bins a lane
    const int lane = row.thread & 63;
    const uint4 h = *(const uint4*)&row.histogram[4 * lane];
    const uint32_t four = h.x + h.y + h.z + h.w;
    uint32_t upto = four;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
      const uint32_t y = __shfl_up(upto, d);
      if (lane >= d) upto += y;
    }
    const int owner = __builtin_ctzll(__ballot(upto >= equal));
    uint32_t before = upto - four, byte = 4 * lane;
    if (before + h.x < equal) {
      before += h.x, ++byte;
      if (before + h.y < equal) {
        before += h.y, ++byte;
        if (before + h.z < equal) before += h.z, ++byte;
      }
    }
    equal -= __builtin_amdgcn_readlane(before, owner);
    prefix |= (uint32_t)__builtin_amdgcn_readlane(byte, owner) << shift;
    mask |= 255u << shift;
    row.sync();
  }
  uint32_t taken = 0;  // of those equal to the key, in the entries before
  row.each([&](int32_t e, int32_t i, uint32_t k) {
    const bool is = k == prefix;
    const uint64_t b = __ballot(is);
    uint32_t rank = taken + __builtin_amdgcn_mbcnt_hi((uint32_t)(b >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)b, 0));
    if constexpr (WAVES > 1) {
      if ((row.thread & 63) == 0) row.scratch[row.thread >> 6] = __popcll(b);
      __syncthreads();
      uint32_t all = 0;
      for (int v = 0; v < WAVES; ++v) {
        const uint32_t c = row.scratch[v];
        if (v < (row.thread >> 6)) rank += c;
        all += c;
      }
      __syncthreads();
      taken += all;
    } else {
      taken += __popcll(b);
    }
    const bool leaves = k < prefix || (is && rank < equal);
    if (leaves) atomicAdd(&a.refcount[l * a.NB + i], -1);
    if (e < row.E && (leaves || !same)) out[e] = leaves ? -1 : i;
  });
}

__global__ __launch_bounds__(kKvThreads) void copy_counts_kernel(const int32_t* in, int32_t* out, int64_t n) {
  for (int64_t i = (int64_t)blockIdx.x * kKvThreads + threadIdx.x; i < n; i += (int64_t)gridDim.x * kKvThreads) out[i] = in[i];
}

}  // namespace
}  // namespace rc

extern "C" rc_status rc_kv_write(const rc_kv_desc* desc, int64_t n_blocks, const void* k_new, const void* v_new, int64_t n_tokens, int64_t token_stride,
                                 int64_t new_layer_stride, const int32_t* slots, void* k, void* v, void* hip_stream) {
  using namespace rc;
  const char* who = "rc_kv_write";
  clear_error();
  if (rc_status e = check_paged(desc, n_blocks, who)) return e;
  if (n_tokens < 0) return fail(RC_ERR_INVALID_ARG, "%s: negative size", who);
  if (desc->n_layers == 0 || n_tokens == 0 || n_blocks == 0) return RC_OK;
  if (!k_new || !v_new || !slots || !k || !v) return fail(RC_ERR_INVALID_ARG, "%s: NULL pointer", who);
  if (!aligned16(k_new) || !aligned16(v_new) || !aligned16(k) || !aligned16(v)) return fail(RC_ERR_INVALID_ARG, "%s: pointer not 16-byte aligned", who);
  const int64_t token = (int64_t)desc->n_kv_heads * 128;
  if (n_tokens >= (1LL << 32) / (desc->n_kv_heads * 16)) return fail(RC_ERR_UNSUPPORTED, "%s: 2^28 heads of tokens or more", who);
  if (token_stride < token || token_stride > INT64_MAX / 4 / n_tokens || token_stride % 8 != 0 || new_layer_stride % 8 != 0)
    return fail(RC_ERR_INVALID_ARG, "%s: token_stride smaller than H*Dh, or a stride that breaks 16-byte alignment", who);
  if (desc->n_layers > 1 && new_layer_stride < token) return fail(RC_ERR_INVALID_ARG, "%s: new_layer_stride smaller than a token", who);
  KvWriteArgs a;
  a.k_new = (const char*)k_new, a.v_new = (const char*)v_new, a.slots = slots, a.k = (char*)k, a.v = (char*)v;
  a.token_stride_b = token_stride * 2, a.new_layer_stride_b = new_layer_stride * 2, a.layer_stride_b = desc->layer_stride * 2;
  a.n_slots = n_blocks * desc->block_tokens;
  a.heads = (uint32_t)desc->n_kv_heads, a.units = (uint32_t)(n_tokens * desc->n_kv_heads * 16);
  const uint32_t per = kKvThreads * kWriteEach;
  kv_write_kernel<<<dim3((unsigned)(((uint64_t)a.units + per - 1) / per), (unsigned)desc->n_layers), kKvThreads, 0, static_cast<hipStream_t>(hip_stream)>>>(a);
  return check_launch(who);
}

extern "C" rc_status rc_kv_evict(int32_t n_layers, const int32_t* tables_in, int32_t* tables_out, int64_t R, int64_t E, int64_t NB, int32_t block_tokens,
                                 const int32_t* ctx_len, const float* weights, const int32_t* keep, int64_t n_first, int64_t n_last,
                                 const int32_t* refcount_in, int32_t* refcount_out, int32_t* n_evicted, void* hip_stream) {
  using namespace rc;
  const char* who = "rc_kv_evict";
  clear_error();
  if (n_layers < 0 || R < 0 || E < 0 || NB < 0 || n_first < 0) return fail(RC_ERR_INVALID_ARG, "%s: negative size", who);
  if (n_last < 1) return fail(RC_ERR_INVALID_ARG, "%s: n_last must be 1 at least: a request's newest block is still being written", who);
  if (block_tokens != 16 && block_tokens != 32) return fail(RC_ERR_UNSUPPORTED, "%s: block_tokens %d (only 16 or 32)", who, block_tokens);
  if (E > 0x7fffffffLL - 1024 || NB > 0x7fffffffLL || R > (1 << 24) || (int64_t)n_layers * R > (1 << 24))
    return fail(RC_ERR_UNSUPPORTED, "%s: more than 2^24 tables, or 2^31 - 1024 entries or blocks", who);
  if (n_layers == 0 || (R == 0 && NB == 0)) return RC_OK;
  hipStream_t st = static_cast<hipStream_t>(hip_stream);
  if (NB > 0 && (!refcount_in || !refcount_out)) return fail(RC_ERR_INVALID_ARG, "%s: NULL pointer", who);
  if (R > 0 && (!ctx_len || !keep || !n_evicted || (E > 0 && (!tables_in || !tables_out || !weights)))) return fail(RC_ERR_INVALID_ARG, "%s: NULL pointer", who);
  if (NB > 0 && refcount_in != refcount_out) {
    const int64_t n = (int64_t)n_layers * NB, wgs = (n + kKvThreads - 1) / kKvThreads;
    copy_counts_kernel<<<dim3((unsigned)(wgs < 4096 ? wgs : 4096)), kKvThreads, 0, st>>>(refcount_in, refcount_out, n);
  }
  if (R > 0) {
    const EvictArgs a = {tables_in, tables_out, n_layers, R, E, NB, block_tokens, ctx_len, keep, weights, n_first, n_last, refcount_out, n_evicted};
    const int64_t rows = (int64_t)n_layers * R;
    if (E <= 1024)
      kv_evict_kernel<1, 16><<<dim3((unsigned)((rows + 3) / 4)), 256, 0, st>>>(a);
    else if (E <= 16384)
      kv_evict_kernel<16, 16><<<dim3((unsigned)rows), 1024, 0, st>>>(a);
    else
      kv_evict_kernel<16, 0><<<dim3((unsigned)rows), 1024, 0, st>>>(a);
  }
  return check_launch(who);
}
