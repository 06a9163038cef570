// What the attention kernels share (rc_cache_attend over the 4-bit cache, rc_kv_attend over 16-bit blocks): the walk along the line of units, the
// softmax of a row's scores with its running reference, and the launch that joins the parts of cut items.
//
// The softmax's reference is not the running maximum but a number at most 15 below it (in powers of two) and 7 below it when it is
// set: probabilities stay below 2^15, as fp16 holds them, and the sums are rescaled only where a score passes the reference by 15.
// bf16 values may be as large as fp32 numbers, and scores so large that an fp32 number is coarse: rescale().
#pragma once
#include <hip/hip_runtime.h>

#include "rc_attend_plan.hpp"
#include "rc_common.hpp"
#include "rc_vec.hpp"

namespace rc {
namespace {

constexpr int kThreads = 256, kWaves = 4;
constexpr float kNothing = -3e38f;  // the reference of a row that has seen nothing; -infinity would make NaNs of differences
constexpr float kRoom = 15.f, kBelow = 7.f;
// V's groups under a power of 2^65 and more, which only bf16 has: weights of 2^15 and the number of tokens would take their sums beyond fp32.
// From the first of them on a wave keeps weights to 2^-20 at most, and a lane's sum that has passed 2^-16 is set to 2^-24: a row's weights of a
// wave (four lanes, each with 16 more of a step) are 2^-13 at most, those of four waves and 768 parts 0.375, and 0.375 * 6 * 2^125 is an fp32
// number, however many tokens there are.  Below 2^65: 2^15 * 2^31 tokens * 7 * 2^64 is one.  (Lower limits throughout would cost small values their
// last bits.)
constexpr float kLowLimit = -20.f, kLowSum = 0x1p-16f, kLowSumExp = -24.f;

// What a call's kernels are told, whatever holds K and V.
struct AttendArgs {
  AttendShape s;
  const int32_t *tables, *ctx_len, *q_start;
  const char* q;
  char* out;
  float* lse;
  float2* ends;  // a row's last reference and its sum of weights, [L][n_q][heads], for those who weigh blocks; or NULL
  int64_t q_token_stride_b, q_layer_stride_b, n_blocks;
  float c;  // scale * log2(e)
  AttendBorder* borders;  // NULL where no item is cut
  char* parts;
};

template <bool BF16>
__device__ __forceinline__ f32x4 mfma(u32x4 a, u32x4 b, f32x4 c) {
  if constexpr (BF16)
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
  else
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
}

// Two fp32 numbers rounded to the nearest 16-bit ones.
template <bool BF16>
__device__ __forceinline__ uint32_t pack2(float a, float b) {
  if constexpr (BF16)
    return __builtin_bit_cast(uint32_t, bf16x2{(__bf16)a, (__bf16)b});
  else
    return __builtin_bit_cast(uint32_t, f16x2{(_Float16)a, (_Float16)b});
}
// Two fp32 numbers to 16-bit ones where the rest is kept as well, so that the direction does not matter.
template <bool BF16>
__device__ __forceinline__ uint32_t cut2(float a, float b) {
  if constexpr (BF16)
    return pack2<true>(a, b);
  else
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_pkrtz(a, b));
}
template <bool BF16>
__device__ __forceinline__ float low16(uint32_t w) {
  if constexpr (BF16)
    return __uint_as_float(w << 16);
  else
    return (float)__builtin_bit_cast(f16x2, w)[0];
}
template <bool BF16>
__device__ __forceinline__ float high16(uint32_t w) {
  if constexpr (BF16)
    return __uint_as_float(w & 0xffff0000u);
  else
    return (float)__builtin_bit_cast(f16x2, w)[1];
}

// Over the four lanes l, l + 16, l + 32, l + 48 that hold a row.
__device__ __forceinline__ float row_max(float x) {
  u32x2 y = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  x = fmaxf(__uint_as_float(y[0]), __uint_as_float(y[1]));
  y = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(y[0]), __uint_as_float(y[1]));
}
__device__ __forceinline__ float row_sum(float x) {
  u32x2 y = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  x = __uint_as_float(y[0]) + __uint_as_float(y[1]);
  y = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(y[0]) + __uint_as_float(y[1]);
}

__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }

__device__ __forceinline__ AttendRequest request(const AttendArgs& a, int r) {
  return a.q_start ? attend_request(a.s, a.ctx_len[r], a.q_start[r], a.q_start[r + 1]) : attend_request(a.s, a.ctx_len[r], r, r + 1);
}

// ---- Where a workgroup's stretch of the line of units begins, and the walk along it.

struct Walk {
  int at, end, begin, share;  // units of the line
  int l, r, h, t, rest;       // layer, request, head, row tile, unit of the row tile (or of the head's, before that is looked for)
  AttendRequest q;
  AttendItem item;
};

__device__ __forceinline__ void leave_border(const AttendArgs& a, int wg, int last, const Walk& w) {
  if (a.borders && threadIdx.x == 0) a.borders[wg] = {last, w.at == w.begin, w.l, w.h, w.t * a.s.rows, w.q.rows, w.q.first, 0};
}

// Sums over `lanes` neighbouring lanes, a power of two.
__device__ __forceinline__ int add_lanes(int x, int lanes) {
#pragma unroll 1
  for (int d = 1; d < lanes; d <<= 1) x += __shfl_xor(x, d);
  return x;
}
__device__ __forceinline__ int upto_lane(int x, int lane) {
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const int y = __shfl_up(x, d);
    if (lane >= d) x = attend_sum(x, y);
  }
  return x;
}
// Units of a request and KV head, counted by `lanes` lanes of which this one is number i.  ONE: a request has one row tile at most (and one lane counts it).
template <bool ONE>
__device__ __forceinline__ int units_of(const AttendArgs& a, const AttendRequest& q, int i, int lanes) {
  if constexpr (ONE) return q.tiles ? attend_only_item(a.s, q).units : 0;
  int n = 0;
#pragma unroll 1
  for (int t = i; t < q.tiles; t += lanes) n += attend_item(a.s, q, t).units;
  return n;
}

// Every wave counts the units of all requests by itself, every lane those of some requests in a row: three loads and a scan without
// a barrier, where a launch of its own would cost more than that.  What is run once here is read from memory once by every compute unit
// as well, instruction by instruction: it is kept short (2.0 us of a call of 8.3 went by before the first load, with everything
// inlined and unrolled 1000 instructions).
template <bool ONE>
__device__ inline bool find(const AttendArgs& a, int wg, Walk& w) {
  const int lane = threadIdx.x & 63, R = (int)a.s.R, H = a.s.H, lanes = ONE ? 1 : a.s.lanes, log = __builtin_ctz(lanes), sub = lane & (lanes - 1);
  const int each = (R + (64 >> log) - 1) >> (6 - log);
  int ctx = 0, start = 0, end = 0, mine = 0;
#pragma unroll 1
  for (int i = 0; i < each; ++i) {
    const int r = (lane >> log) * each + i;
    int units = 0;
    if (r < R) {
      ctx = a.ctx_len[r];
      start = a.q_start ? a.q_start[r] : r;
      end = a.q_start ? a.q_start[r + 1] : r + 1;
      units = units_of<ONE>(a, attend_request(a.s, ctx, start, end), sub, lanes);
    }
    if (!ONE) units = add_lanes(units, lanes);
    mine = attend_sum(mine, units * H);
  }
  if (!ONE && sub) mine = 0;
  const int upto = upto_lane(mine, lane);
  const int total = __builtin_amdgcn_readlane(upto, 63), line = uniform(attend_line(a.s, total));
  w.share = uniform(attend_share(a.s, line));
  w.begin = w.at = wg * w.share;
  w.end = min(w.at + w.share, line);
  w.l = w.r = w.h = w.t = 0;
  w.q = {0, 0, 0, 0, 0};
  if (w.at >= line) {
    leave_border(a, wg, -1, w);
    return false;
  }
  w.l = a.s.L == 1 ? 0 : uniform((int)((uint32_t)w.at / (uint32_t)total));
  const int off = w.at - w.l * total;
  // the lane whose requests hold the unit, and then the request
  const int owner = __builtin_ctzll(__ballot(off < upto));
  w.rest = off - (__builtin_amdgcn_readlane(upto, owner) - __builtin_amdgcn_readlane(mine, owner));
  w.r = (owner >> log) * each;
  w.q = attend_request(a.s, __builtin_amdgcn_readlane(ctx, owner), __builtin_amdgcn_readlane(start, owner), __builtin_amdgcn_readlane(end, owner));
  int units = __builtin_amdgcn_readlane(mine, owner);
  if (each > 1) {
    for (;; ++w.r) {
      w.q = request(a, w.r);
      const int n = units_of<ONE>(a, w.q, ONE ? 0 : lane, 64);
      units = uniform((ONE ? n : add_lanes(n, 64)) * H);
      if (w.rest < units) break;
      w.rest -= units;
    }
  }
  units = uniform((int)((uint32_t)units / (uint32_t)H));
  w.h = uniform((int)((uint32_t)w.rest / (uint32_t)units));
  w.rest -= w.h * units;
  // ... and the row tile, 64 at a time
  if constexpr (!ONE) {
    for (; w.t < w.q.tiles; w.t += 64) {
      const int n = w.t + lane < w.q.tiles ? attend_item(a.s, w.q, w.t + lane).units : 0, sum = upto_lane(n, lane), all = __builtin_amdgcn_readlane(sum, 63);
      if (w.rest < all) {
        const int tile = __builtin_ctzll(__ballot(w.rest < sum));
        w.rest -= __builtin_amdgcn_readlane(sum, tile) - __builtin_amdgcn_readlane(n, tile);
        w.t += tile;
        break;
      }
      w.rest -= all;
    }
  }
  return true;
}

// To the next item, a row tile of the same or another request, head and layer: only called where there is one.
template <bool ONE>
__device__ __forceinline__ void next_item(const AttendArgs& a, Walk& w) {
  if (!ONE && ++w.t < w.q.tiles) return;
  w.t = 0;
  if (++w.h < a.s.H) return;
  w.h = 0;
  do {
    if (++w.r == a.s.R) w.r = 0, ++w.l;
    w.q = request(a, w.r);
  } while (w.q.tiles == 0);
}

// A part of an item: units u0 to u1 of it, tokens of the runs pa to pb.
struct Part {
  int u0, u1, pa, pb;
  bool whole;
};
// The part that the walk stands before; false where it stands in an earlier row tile of the head, and has gone on to the next.
template <bool ONE>
__device__ __forceinline__ bool take_part(const AttendArgs& a, Walk& w, Part& p) {
  w.item = ONE ? attend_only_item(a.s, w.q) : attend_item(a.s, w.q, w.t);
  if (!ONE && w.rest >= w.item.units) {
    w.rest -= w.item.units;
    ++w.t;
    return false;
  }
  p.u0 = w.rest, p.u1 = min(w.item.units, w.rest + w.end - w.at);
  p.pa = uniform(attend_run(a.s, w.item, p.u0)), p.pb = uniform(attend_run(a.s, w.item, p.u1));
  p.whole = p.u0 <= w.item.free && p.u1 == w.item.units;
  return true;
}
// Nothing of the item falls to this stretch, whose end lies among its free units.
__device__ __forceinline__ bool only_free(const Walk& w, const Part& p) { return p.u1 <= w.item.free; }

// Behind a part: false at the end of the stretch.  If the part is the first of an item that goes on, the border says up to which
// workgroup the item's parts go.
template <bool ONE>
__device__ __forceinline__ bool go_on(const AttendArgs& a, int wg, Walk& w, const Part& p) {
  const int left = w.item.units - p.u1;
  if (w.at + (p.u1 - p.u0) >= w.end) {
    const bool first = p.u0 <= w.item.free && left;
    leave_border(a, wg, first ? wg + (int)((uint32_t)(left + w.share - 1) / (uint32_t)w.share) : -1, w);
    return false;
  }
  w.at += p.u1 - p.u0;
  w.rest = 0;
  next_item<ONE>(a, w);
  return true;
}

// ---- Loads.

// Block ids of the 64 tiles of 16 tokens that a wave will come to next: lane j holds that of the j-th, or -1 where there is no such
// block.  One load for 64 tiles; taken tile by tile, it would stand in front of the loads of the cache every time.
__device__ __forceinline__ int load_id(const AttendArgs& a, const int32_t* table, int tile, bool in) {
  const int e = a.s.T == 32 ? tile >> 1 : tile;
  const int id = in && e < a.s.E ? table[e] : -1;
  return id < a.n_blocks ? id : -1;
}

// ---- Softmax of a row's scores.

// How a wave takes the weights of its row tiles: 2^(score * times - ref), where no exponent passes `room`; else rescale() moves the references first.
// Odd: a bit for each row tile whose exponents rescale() leaves in place of its scores, under a reference of 0 and with times of 1, because of large V (`low`) or
// coarse scores.  From the first of either on, room is -infinity, and rescale() sees to every tile, so that the others have one comparison in front of
// them, as they would have without.  It costs a bf16 call 0 to 3 %, the look at V's powers with it (262143 tokens 59 us either way, drafts 32.4 -> 32.8, 256
// query tokens over 60000 268 -> 272), an fp16 call 0 to 2 % (1024 query tokens over 8192 256 either way, 64 requests of 12400 tokens 113 either way, 200
// tokens of 20 queries 12.0 -> 12.3).
struct Gate {
  float room, times[4];
  int odd;
  bool low;
  __device__ __forceinline__ Gate(float c) : room(kRoom), times{c, c, c, c}, odd(0), low(false) {}
  __device__ __forceinline__ void see(bool large) {
    low = low || large;
    room = large ? -__builtin_inff() : room;
  }
};
// Products score * c beyond this are so coarse that one taken exactly and one rounded may differ by whole powers of two: exponents are
// differences of rounded products there, so that the largest is what it was meant to be.
constexpr float kCoarse = 0x1p20f;

// Row tile t's scores s, the largest of the lane's ones in top; `kept`: in LDS, a place of the row's for the reference of an odd tile.  What decides is
// the exponent as it is taken for the largest score, so that no weight passes the limit.
template <bool BF16, int N>
__device__ __forceinline__ void rescale(f32x4 (&s)[N], f32x4 (&o)[8], float& ref, float& sum, float top, float c, int t, Gate& g, float& kept) {
  // a wave-wide decision: nearly always no row's score passes its reference by kRoom
  if (__builtin_expect(__any(fmaf(top, g.times[t], -ref) > g.room), 0)) {
    const bool low = BF16 && g.low;
    const float from = g.odd >> t & 1 ? kept : ref, most = row_max(top), limit = low ? kLowLimit : kRoom, below = low ? kLowLimit : kBelow;
    float to = fmaxf(from, fmaf(most, c, -below)), least = from;
    if (low) {
      const float all = row_max(sum);
      if (all > kLowSum) least = from + __builtin_amdgcn_logf(all) - kLowSumExp;
      to = fmaxf(to, least);
    }
    const bool coarse = fabsf(to) > kCoarse;
    if (low || uniform(__any(coarse && to != kNothing))) g.odd |= 1 << t;
    if (__builtin_expect(g.odd >> t & 1, 0)) {
#pragma clang fp contract(off)
      const float x = most * c;
      if (coarse) to = fmaxf(fmaxf(from, least), x - below);
#pragma unroll
      for (int i = 0; i < 4 * N; ++i) {
        const float y = s[i >> 2][i & 3], z = y * c, d = coarse ? z - to : fmaf(y, c, -to);
        s[i >> 2][i & 3] = d > limit ? limit : d;  // (NaN stays)
      }
      kept = to;
      ref = 0.f;
      g.times[t] = 1.f;
      g.room = -__builtin_inff();
    } else {
      ref = to;
    }
    const float f = __builtin_amdgcn_exp2f(from - to);
    sum *= f;
#pragma unroll
    for (int i = 0; i < 8; ++i) o[i] *= f;
  }
}

// ---- What a row leaves.

// Query token of row n of an item's first `rows` ones, n / g.  ONE: n is below 32 (and g as well, or n / g is 0).
template <bool ONE>
__device__ __forceinline__ int row_token(const AttendArgs& a, int n) {
  return ONE ? (int)((uint32_t)n * a.s.inverse >> 16) : (int)((uint32_t)n / (uint32_t)a.s.g);
}
// Row n of a request's rows of a layer and KV head, as a row of [L][n_q][n_heads]; `first` is the request's first query token.
template <bool ONE>
__device__ __forceinline__ int64_t row_place(const AttendArgs& a, int l, int h, int first, int n) {
  const int j = row_token<ONE>(a, n);
  return ((int64_t)l * a.s.n_q + first + j) * (int64_t)(a.s.H * a.s.g) + h * a.s.g + n - j * a.s.g;
}
template <bool ONE>
__device__ __forceinline__ int64_t row_place(const AttendArgs& a, const Walk& w, int n) {
  return row_place<ONE>(a, w.l, w.h, w.q.first, n);
}
__device__ __forceinline__ float row_lse(float ref, float sum) {
  return sum == 0.f ? -__builtin_inff() : (ref + __builtin_amdgcn_logf(sum)) * 0.6931471805599453f;
}
__device__ __forceinline__ float row_scale(float sum) { return sum == 0.f ? 0.f : 1.f / sum; }

// Its position.  Rows that the item does not have stand where its last one does: further on they would see tokens that nobody has written, and what
// lies there would decide when the wave moves the references of all its rows, and with these the last bits of the others' results.
template <bool ONE>
__device__ __forceinline__ int row_position(const AttendArgs& a, const Walk& w, int n) {
  return w.q.ctx - w.q.len + row_token<ONE>(a, min(n, w.q.rows - 1));
}
// Row n of q as lane (row, quarter) holds it for the four steps of K's dims; rows that the item does not have: its last one's.
template <bool ONE>
__device__ __forceinline__ void load_q(const AttendArgs& a, const Walk& w, int n, int quarter, u32x4 (&q)[4]) {
  n = min(n, w.q.rows - 1);
  const int j = row_token<ONE>(a, n), head = w.h * a.s.g + n - j * a.s.g;
  const u32x4* p = (const u32x4*)(a.q + (int64_t)w.l * a.q_layer_stride_b + (int64_t)(w.q.first + j) * a.q_token_stride_b + (head * 128 + quarter * 32) * 2);
#pragma unroll
  for (int s = 0; s < 4; ++s) q[s] = p[s];
}

// The rows of an item that sees nothing.  ENDS: a.ends may be there.  (Known when compiled: asked of a.ends alone, it costs the attention over the 4-bit
// cache scalar registers that it does not have, and 64 decoding requests of 12400 tokens take 115.6 us instead of 111.6.)
template <bool ONE, bool ENDS>
__device__ inline void store_nothing(const AttendArgs& a, const Walk& w) {
  const int rows = min(a.s.rows, w.q.rows - w.t * a.s.rows);
  for (int i = threadIdx.x; i < rows * 16; i += kThreads) {
    const int64_t at = row_place<ONE>(a, w, w.t * a.s.rows + (i >> 4));
    *(u32x4*)(a.out + (at * 128 + (i & 15) * 8) * 2) = u32x4{0, 0, 0, 0};
    if ((i & 15) == 0 && a.lse) a.lse[at] = -__builtin_inff();
    if (ENDS && (i & 15) == 0 && a.ends) a.ends[at] = float2{kNothing, 0.f};
  }
}

// ---- Items that were cut: a workgroup joins the parts of the item that begins in a stretch and goes on behind it, some rows at a time.

// Eight dims of a row and its softmax.
struct Joined {
  f32x4 x, y;
  float top, sum;
};
__device__ __forceinline__ void join(Joined& j, const Joined& k) {
  const float top = fmaxf(j.top, k.top), f = __builtin_amdgcn_exp2f(j.top - top), g = __builtin_amdgcn_exp2f(k.top - top);
  j.x = j.x * f + k.x * g;
  j.y = j.y * f + k.y * g;
  j.sum = j.sum * f + k.sum * g;
  j.top = top;
}
// Row m over the parts of workgroups g, g + step, .. up to the last: in one pass, so that all loads are on their way at once.
__device__ __forceinline__ Joined join_parts(const AttendArgs& a, const AttendBorder& b, int wg, int g, int step, int m, int d) {
  Joined j = {{0, 0, 0, 0}, {0, 0, 0, 0}, kNothing, 0.f};
#pragma unroll 4
  for (; g <= b.last; g += step) {
    const float* p = (const float*)(a.parts + attend_place(g, g > wg || b.begins) * (int64_t)attend_part_bytes(a.s.rows));
    const float2 s = *(const float2*)(p + a.s.rows * 128 + 2 * m);
    join(j, Joined{*(const f32x4*)(p + m * 128 + d), *(const f32x4*)(p + m * 128 + d + 4), s.x, s.y});
  }
  return j;
}
template <bool BF16>
__device__ __forceinline__ void join_store(const AttendArgs& a, const AttendBorder& b, int m, int d, const Joined& j) {
  const float f = row_scale(j.sum);
  const f32x4 x = j.x * f, y = j.y * f;
  const int64_t at = row_place<false>(a, b.l, b.h, b.first, b.row0 + m);
  *(u32x4*)(a.out + (at * 128 + d) * 2) = u32x4{pack2<BF16>(x[0], x[1]), pack2<BF16>(x[2], x[3]), pack2<BF16>(y[0], y[1]), pack2<BF16>(y[2], y[3])};
  if (d == 0 && a.lse) a.lse[at] = row_lse(j.top, j.sum);
  if (d == 0 && a.ends) a.ends[at] = float2{j.top, j.sum};
}

// Sixteen lanes hold a row.  An item of some parts takes sixteen lanes per row; where rows are few, one of many parts (a long context has up to a
// hundred) takes a workgroup per row, whose sixteen groups of lanes share the parts.
constexpr int kSomeParts = 8;

template <bool BF16, bool FEW>
__global__ __launch_bounds__(kThreads) void attend_join_kernel(AttendArgs a) {
  __shared__ Joined all[16][16];
  const int i = threadIdx.x & 15, group = threadIdx.x >> 4, d = i * 8, wg = blockIdx.x;
  const AttendBorder b = a.borders[wg];
  if (b.last < 0) return;
  const int rows = min(a.s.rows, b.rows - b.row0);
  if (FEW && b.last - wg >= kSomeParts) {
    const int m = blockIdx.y;
    if (m >= rows) return;
    all[group][i] = join_parts(a, b, wg, wg + group, 16, m, d);
    __syncthreads();
    if (group) return;
    Joined j = all[0][i];
#pragma unroll
    for (int v = 1; v < 16; ++v) join(j, all[v][i]);
    join_store<BF16>(a, b, m, d, j);
  } else {
    const int m = blockIdx.y * 16 + group;
    if (m < rows) join_store<BF16>(a, b, m, d, join_parts(a, b, wg, wg, 1, m, d));
  }
}

}  // namespace
}  // namespace rc
