// rc_kv_write: K and V of new tokens into the slots of 16-bit paged KV blocks.  rc_kv_evict: table entries whose blocks gathered the least attention leave.
#include <hip/hip_runtime.h>

#include "rc_kv.hpp"
#include "rc_vec.hpp"

namespace rc {
namespace {

constexpr int kKvThreads = 256;

// ---- rc_kv_write

// A copy, bound by memory: a thread moves 16 bytes of K and of V at a time, four of each, neighbouring threads neighbouring ones.  64 layers of 2.1k tokens
// 1.12 GB in 204 us (5.5 TB/s; a copy of 4 GB runs at 4.6); the smallest calls are a launch, 3 us.
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
  const int32_t* copied;  // what the only workgroup copies to refcount first, or NULL
  int32_t *refcount, *n_evicted;
};

// The order of weights as that of whole numbers: -0 and 0 are equal, NaN is the largest.  What may not leave comes behind them all.
constexpr uint32_t kStays = 0xffffffffu;
constexpr int kSmallRow = 1024;  // entries of a row that one wave takes
__device__ __forceinline__ uint32_t weight_key(float w) {
  const uint32_t b = __float_as_uint(w + 0.f);
  if (w != w) return kStays - 1;
  return b >> 31 ? ~b : b | 0x80000000u;
}

// A row is the table of one request in one layer.  The n entries that leave are those whose keys lie below a border, and of those that equal it the ones that
// lie before a place of the table: both are found bit by bit from the top, with a count of the entries below at every bit.  Keys lie in registers (entry
// i * threads + thread at place i), so that a count is a compare and a ballot for each; a row that they do not hold is counted by a histogram of
// each byte in turn, for which it is read again.
//
// 64 layers of 64 requests of up to 775 entries, 700 kept at most: 27 us and 5 for the copy of the reference counts; 11 of these are the 0.43M decrements, 11 the tables and
// weights going in and out, the borders the rest (a histogram by bytes for these as well: the same).  24 tables of 16384 entries cut down to a quarter: 45 us, 24 workgroups'
// work, 19 for the 0.22M decrements (with histograms 62).
template <int WAVES, int ITEMS>  // ITEMS: entries of a thread held in registers, 0: none
struct EvictRow {
  static constexpr int kRowThreads = 64 * WAVES;
  const EvictArgs& a;
  const int32_t* in;
  const float* weights;
  int32_t E, used, thread;
  uint32_t* lds;  // 2 * WAVES sums, and 256 more without registers
  int turn;
  static constexpr bool kIds = ITEMS && ITEMS <= 16;  // ids are held as well, else read again where they are written
  uint32_t key[ITEMS ? ITEMS : 1];
  int32_t id[kIds ? ITEMS : 1];

  __device__ __forceinline__ bool held(int32_t i, int32_t e) const { return e < used && i >= 0 && i < a.NB; }
  __device__ __forceinline__ uint32_t make_key(int32_t i, int32_t e) const {
    return held(i, e) && e >= a.n_first && e < used - a.n_last ? weight_key(weights[e]) : kStays;
  }
  // Of a number of every wave, the same for all its lanes.
  __device__ __forceinline__ uint32_t sum_waves(uint32_t x) {
    if constexpr (WAVES == 1) return x;
    uint32_t* at = lds + (turn++ & 1) * WAVES;  // (so that one barrier is enough: who still reads the last sums has not passed the next one)
    if ((thread & 63) == 0) at[thread >> 6] = x;
    __syncthreads();
    x = 0;
#pragma unroll
    for (int i = 0; i < WAVES; ++i) x += at[i];
    return __builtin_amdgcn_readfirstlane(x);
  }
  // f(entry, key) of every entry of the thread; the same number of turns for all lanes of the row.
  template <class F>
  __device__ __forceinline__ void each(F f) {
    each_id([&](int32_t e, uint32_t k, auto) { f(e, k); });
  }
  // ... and its id, asked for as a function
  template <class F>
  __device__ __forceinline__ void each_id(F f) {
    if constexpr (ITEMS) {
#pragma unroll
      for (int i = 0; i < ITEMS; ++i) {
        const int32_t e = i * kRowThreads + thread;
        if (i * kRowThreads < E) f(e, key[i], [&] { return kIds ? id[kIds ? i : 0] : in[e]; });
      }
    } else {
      for (int32_t base = 0; base < E; base += kRowThreads) {
        const int32_t e = base + thread;
        f(e, make_key(e < E ? in[e] : -1, e), [&] { return in[e]; });
      }
    }
  }
  template <class F>
  __device__ __forceinline__ uint32_t count(F f) {
    uint32_t n = 0;
    each([&](int32_t e, uint32_t k) { n += __popcll(__ballot(f(e, k))); });
    return sum_waves(n);
  }
  // The largest border of which fewer than n of the numbers x(entry, key) (in 32 bits, from `top` bits down) lie below; one with exactly n below it ends the
  // search.
  template <class F>
  __device__ __forceinline__ uint32_t border(int top, uint32_t n, bool& exact, F below) {
    uint32_t b = 0;
    exact = false;
#pragma unroll 1
    for (int bit = top - 1; bit >= 0 && !exact; --bit) {
      const uint32_t mid = b | 1u << bit, c = count([&](int32_t e, uint32_t k) { return below(e, k, mid); });
      if (c <= n) b = mid, exact = c == n;
    }
    return b;
  }
  // The n-th smallest key by bytes, and how many of those that equal it leave.
  __device__ __forceinline__ uint32_t nth(uint32_t n, uint32_t& equal) {
    uint32_t *histogram = lds + 2 * WAVES, prefix = 0, mask = 0;
    equal = n;
#pragma unroll 1
    for (int shift = 24; shift >= 0; shift -= 8) {
      if (thread < 256) histogram[thread] = 0;
      __syncthreads();
      each([&](int32_t, uint32_t k) { if (k != kStays && (k & mask) == prefix) atomicAdd(&histogram[k >> shift & 255], 1u); });
      __syncthreads();
      // every wave finds the byte by itself: four bins a lane
      const int lane = thread & 63;
      const uint4 h = *(const uint4*)&histogram[4 * lane];
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
      __syncthreads();
    }
    return prefix;
  }
};

template <int WAVES, int ITEMS>
__global__ __launch_bounds__(WAVES == 1 ? 256 : 64 * WAVES) void kv_evict_kernel(EvictArgs a) {
  constexpr int kRows = WAVES == 1 ? 4 : 1;
  using Row = EvictRow<WAVES, ITEMS>;
  __shared__ __attribute__((aligned(16))) uint32_t lds[2 * WAVES + (ITEMS ? 0 : 256)];
  const int in_block = WAVES == 1 ? (int)(threadIdx.x >> 6) : 0;
  if (a.copied) {
    for (int64_t i = threadIdx.x; i < a.L * a.NB; i += blockDim.x) a.refcount[i] = a.copied[i];
    __threadfence();
    __syncthreads();
  }
  const int64_t lr = ((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * kRows + in_block;
  if (lr >= a.L * a.R) return;
  const int64_t l = lr / a.R, r = lr - l * a.R;
  Row row{a, a.tables_in + lr * a.E, a.weights + lr * a.E, (int32_t)a.E, 0, (int)(WAVES == 1 ? threadIdx.x & 63 : threadIdx.x), lds, 0, {}, {}};
  int32_t* out = a.tables_out + lr * a.E;
  const int32_t ctx = a.ctx_len[r], keep = max(a.keep[r], 0);
  const int64_t blocks = ctx > 0 ? ((int64_t)ctx + a.T - 1) / a.T : 0;
  row.used = (int32_t)(blocks < a.E ? blocks : a.E);
  uint32_t held = 0;
  if constexpr (ITEMS) {
    int32_t id[ITEMS];
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
      const int32_t e = i * Row::kRowThreads + row.thread;
      id[i] = e < row.E ? row.in[e] : -1;
    }
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
      const int32_t e = i * Row::kRowThreads + row.thread;
      row.key[i] = row.make_key(id[i], e);
      if constexpr (Row::kIds) row.id[i] = id[i];
      held += __popcll(__ballot(row.held(id[i], e)));
    }
    held = row.sum_waves(held);
  } else {
    held = row.count([&](int32_t e, uint32_t) { return e < row.E && row.held(row.in[e], e); });
  }
  const uint32_t may = row.count([](int32_t, uint32_t k) { return k != kStays; });
  const uint32_t n = min(held > (uint32_t)keep ? held - (uint32_t)keep : 0, may);
  if (row.thread == 0) a.n_evicted[lr] = (int32_t)n;
  // keys below the border leave, and those that equal it at the entries before `place`
  uint32_t border = 0, place = 0;
  if (n) {
    if constexpr (ITEMS) {
      bool exact;
      border = row.border(32, n, exact, [](int32_t, uint32_t k, uint32_t mid) { return k < mid; });
      if (!exact) {
        const uint32_t left = n - row.count([&](int32_t, uint32_t k) { return k < border; });
        place = row.border(32 - __builtin_clz((uint32_t)row.E), left, exact, [&](int32_t e, uint32_t k, uint32_t mid) { return k == border && (uint32_t)e < mid; });
      }
    } else {
      uint32_t equal;
      border = row.nth(n, equal);
      bool exact;
      place = row.border(32 - __builtin_clz((uint32_t)row.E), equal, exact, [&](int32_t e, uint32_t k, uint32_t mid) { return k == border && (uint32_t)e < mid; });
    }
  }
  const bool same = a.tables_in == a.tables_out;
  if (n == 0 && same) return;
  row.each_id([&](int32_t e, uint32_t k, auto id) {
    const bool leaves = k < border || (k == border && (uint32_t)e < place);
    if (e >= row.E || (same && !leaves)) return;
    const int32_t i = id();
    if (leaves) atomicAdd(&a.refcount[l * a.NB + i], -1);
    out[e] = leaves ? -1 : i;
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
  const int64_t rows = (int64_t)n_layers * R, counts = (int64_t)n_layers * NB;
  const bool small = E <= kSmallRow, copy = counts > 0 && refcount_in != refcount_out;
  // a step of few short tables: one workgroup, one launch
  const bool one = small && rows > 0 && rows <= 4 && counts <= 4096;
  if (copy && !one) {
    const int64_t wgs = (counts + kKvThreads - 1) / kKvThreads;
    copy_counts_kernel<<<dim3((unsigned)(wgs < 4096 ? wgs : 4096)), kKvThreads, 0, st>>>(refcount_in, refcount_out, counts);
  }
  if (R > 0) {
    const EvictArgs a = {tables_in, tables_out, n_layers, R, E, NB, block_tokens, ctx_len, keep, weights, n_first, n_last, copy && one ? refcount_in : nullptr,
                         refcount_out, n_evicted};
    // (a launch has fewer than 2^32 threads in x)
    const int64_t wgs = small ? (rows + 3) / 4 : rows, x = wgs < (1 << 20) ? wgs : (1 << 20);
    const dim3 grid((unsigned)x, (unsigned)((wgs + x - 1) / x));
    if (small)
      kv_evict_kernel<1, kSmallRow / 64><<<grid, 256, 0, st>>>(a);
    else if (E <= 16 * 1024)
      kv_evict_kernel<16, 16><<<grid, 1024, 0, st>>>(a);
    else if (E <= 32 * 1024)
      kv_evict_kernel<16, 32><<<grid, 1024, 0, st>>>(a);
    else
      kv_evict_kernel<16, 0><<<grid, 1024, 0, st>>>(a);
  }
  return check_launch(who);
}
