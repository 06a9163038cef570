// rc_cache_attend: softmax attention over the 4-bit paged cache, one pass over the data with a running reference of the softmax.
//
// Scores are taken as S^T = K Q^T and outputs as O^T = V^T P^T on 16x16x32 matrix instructions: a row (a query token and head) is a
// column of both, so that its scores, its probabilities and its sums lie in the same four lanes and the probabilities go from
// one product into the next as they are.  K and V come from memory as codes in operand order (rc_cache.hpp); a wave turns 16 bytes
// of codes into 32 operand values with 16 conversions, V with 16 byte permutes more, which pair neighbouring tokens.
//
// The softmax's reference is not the running maximum but a number at most 15 below it (in powers of two) and 7 below it when it is
// set: probabilities stay below 2^15, as fp16 holds them, and the sums are rescaled only where a score passes the reference by 15.
// bf16 values may be as large as fp32 numbers, and scores so large that an fp32 number is coarse: rescale().
#include <hip/hip_runtime.h>

#include "rc_attend_plan.hpp"
#include "rc_cache.hpp"

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

struct AttendArgs {
  AttendShape s;
  const char* cache;
  const int32_t *tables, *ctx_len, *q_start;
  const char* q;
  char* out;
  float* lse;
  int64_t cache_layer_stride, q_token_stride_b, q_layer_stride_b, n_blocks;
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

// ONE: a request has one row tile at most.
template <bool ONE>
__device__ __forceinline__ int units_of(const AttendArgs& a, const AttendRequest& q) {
  if constexpr (ONE)
    return q.tiles ? attend_only_item(a.s, q).units : 0;
  else
    return attend_units(a.s, q);
}

// Every wave counts the units of all requests by itself, every lane those of some requests in a row: three loads and a scan without
// a barrier, where a launch of its own would cost more than that.  What is run once here is read from memory once by every compute unit
// as well, instruction by instruction: it is kept short (2.0 us of a call of 8.3 went by before the first load, with everything
// inlined and unrolled 1000 instructions).
template <bool ONE>
__device__ inline bool find(const AttendArgs& a, int wg, Walk& w) {
  const int lane = threadIdx.x & 63, R = (int)a.s.R, H = a.s.H, each = (R + 63) / 64;
  int ctx = 0, start = 0, end = 0, mine = 0;
#pragma unroll 1
  for (int i = 0; i < each; ++i) {
    const int r = lane * each + i;
    if (r < R) {
      ctx = a.ctx_len[r];
      start = a.q_start ? a.q_start[r] : r;
      end = a.q_start ? a.q_start[r + 1] : r + 1;
      mine = attend_sum(mine, units_of<ONE>(a, attend_request(a.s, ctx, start, end)) * H);
    }
  }
  int upto = mine;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const int y = __shfl_up(upto, d);
    if (lane >= d) upto = attend_sum(upto, y);
  }
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
  w.r = owner * each;
  w.q = attend_request(a.s, __builtin_amdgcn_readlane(ctx, owner), __builtin_amdgcn_readlane(start, owner), __builtin_amdgcn_readlane(end, owner));
  int units = __builtin_amdgcn_readlane(mine, owner);
  if (each > 1) {
    for (;; ++w.r) {
      w.q = request(a, w.r);
      units = uniform(units_of<ONE>(a, w.q) * H);
      if (w.rest < units) break;
      w.rest -= units;
    }
  }
  units = uniform((int)((uint32_t)units / (uint32_t)H));
  w.h = uniform((int)((uint32_t)w.rest / (uint32_t)units));
  w.rest -= w.h * units;
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

// What a wave holds of 16 tokens: codes in operand order, exponent bytes (K: the lane's token and group; V: four tokens of its group).
struct Tile {
  u32x4 k, v;
  uint32_t ke, ve;
};

// STREAM: codes that no other workgroup reads are not kept in the caches behind this one, where there are too many of them anyway.
template <bool STREAM>
__device__ __forceinline__ u32x4 load_codes(const char* p) {
  if constexpr (STREAM)
    return __builtin_nontemporal_load((const u32x4*)p);
  else
    return *(const u32x4*)p;
}
template <bool STREAM>
__device__ __forceinline__ void load_k(Tile& x, const char* rec, int lane) {
  x.k = load_codes<STREAM>(rec + lane * 16);
  x.ke = *(const uint8_t*)(rec + kRecordKExp + lane);
}
template <bool STREAM>
__device__ __forceinline__ void load_v(Tile& x, const char* rec, int lane) {
  x.v = load_codes<STREAM>(rec + kRecordV + lane * 16);
  x.ve = *(const uint32_t*)(rec + kRecordVExp + ((lane >> 4) * 4 + ((lane & 15) >> 2)) * 4);
}

// Block ids of the 64 tiles of 16 tokens that a wave will come to next: lane j holds that of the j-th, or -1 where there is no such
// block.  One load for 64 tiles; taken tile by tile, it would stand in front of the loads of the cache every time.
__device__ __forceinline__ int load_id(const AttendArgs& a, const int32_t* table, int tile, bool in) {
  const int e = a.s.T == 32 ? tile >> 1 : tile;
  const int id = in && e < a.s.E ? table[e] : -1;
  return id < a.n_blocks ? id : -1;
}
// The record of the tile whose id lane j holds (its parity chooses between the records of a block of 32); block 0's where there is no
// such block (`there` false): its values are replaced or masked.
__device__ __forceinline__ const char* record(const AttendArgs& a, const char* head, int ids, int j, int parity, bool& there) {
  const int id = __builtin_amdgcn_readlane(ids, j), tiles = a.s.T >> 4;
  there = id >= 0;
  return head + (uint64_t)(uint32_t)(there ? id : 0) * (uint32_t)(a.s.H * tiles * kRecordBytes) + (tiles == 2 ? parity * kRecordBytes : 0);
}

// V's exponent bytes with those of tokens that no row sees replaced by that of 1: whatever lies there (memory that was never
// written) gets a probability of 0, and 0 times infinity or NaN would not be 0.  Token r of the word stands at pos + r.
__device__ __forceinline__ uint32_t seen_only(uint32_t ve, int pos, bool there, const AttendItem& it) {
  const uint32_t span = there ? it.high_max - it.low_min : 0;  // (an item that sees no token has no run)
#pragma unroll
  for (int r = 0; r < 4; ++r) {
    const uint32_t m = 0xffu << (8 * r);
    if ((uint32_t)(pos + r - it.low_min) >= span) ve = (ve & ~m) | (kOneByte * 0x01010101u & m);
  }
  return ve;
}
// ... and those of NaN groups: where only some rows see a token, its NaNs are added to these (poison()).
__device__ __forceinline__ uint32_t nan_bytes(uint32_t ve) {
  uint32_t f = 0;
#pragma unroll
  for (int r = 0; r < 4; ++r)
    if ((ve >> (8 * r) & 255) == kNanByte) f |= 1u << r;
  return f;
}
__device__ __forceinline__ uint32_t without_nans(uint32_t ve, uint32_t flags) {
#pragma unroll
  for (int r = 0; r < 4; ++r)
    if (flags >> r & 1) ve = (ve & ~(0xffu << (8 * r))) | ((uint32_t)kOneByte << (8 * r));
  return ve;
}
// Two tokens' bits (b, b + 1 of f) as 16-bit ones and zeros.
template <bool BF16>
__device__ __forceinline__ uint32_t ones(uint32_t f, int b) {
  constexpr uint32_t one = BF16 ? 0x3f80u : 0x3c00u;
  return (f >> b & 1 ? one : 0) | (f >> (b + 1) & 1 ? one << 16 : 0);
}
// NaNs of 32 tokens (flags: bit 4 * tile + r, for the lane's group) into the sums of the rows that see them (seen: the same bits for the lane's row): the number
// of such tokens by row and lane of V's operand, whose 8 dims lie in the 8 sums of that place.
template <bool BF16>
__device__ inline void poison(f32x4 (&o)[8], uint32_t flags, uint32_t seen) {
  const u32x4 x = {ones<BF16>(flags, 0), ones<BF16>(flags, 2), ones<BF16>(flags, 4), ones<BF16>(flags, 6)};
  const u32x4 y = {ones<BF16>(seen, 0), ones<BF16>(seen, 2), ones<BF16>(seen, 4), ones<BF16>(seen, 6)};
  const f32x4 n = mfma<BF16>(x, y, f32x4{0, 0, 0, 0});
#pragma unroll
  for (int r = 0; r < 4; ++r)
    if (n[r] > 0) {
#pragma unroll
      for (int c = 0; c < 8; ++c) o[c][r] = __uint_as_float(0x7fc00000u);
    }
}

// V's operand of a pair of chunks (dims 8i + 2B and 8i + 2B + 1 for lane i of 16) from four tokens' words: tokens 0 and 1 to one
// register, 2 and 3 to the next.
template <bool BF16, int B>
__device__ __forceinline__ void unpack_v(u32x4 v, const float (&power)[4], uint32_t (&even)[2], uint32_t (&odd)[2]) {
#pragma unroll
  for (int p = 0; p < 2; ++p) {
    const uint32_t x = unpack2<BF16, B>(v[2 * p], power[2 * p]), y = unpack2<BF16, B>(v[2 * p + 1], power[2 * p + 1]);
    even[p] = __builtin_amdgcn_perm(y, x, 0x05040100u);
    odd[p] = __builtin_amdgcn_perm(y, x, 0x07060302u);
  }
}
__device__ __forceinline__ void powers(uint32_t ve, float (&p)[4]) {
#pragma unroll
  for (int r = 0; r < 4; ++r) p[r] = power_at(ve, r);
}

// ---- Softmax of a row's scores.

// Whether an exponent byte of either word is 192 or more.
__device__ __forceinline__ bool large_power(uint32_t a, uint32_t b) { return (((a & a << 1) | (b & b << 1)) & 0x80808080u) != 0; }

// How a wave takes the weights of its row tiles: 2^(score * times - ref), where no exponent passes `room`; else rescale() moves the references first.
// Odd: a bit for each row tile whose exponents rescale() leaves in place of its scores, under a reference of 0 and with times of 1, because of large V (`low`) or
// coarse scores.  From the first of either on, room is -infinity, and rescale() sees to every tile, so that the others have one comparison in front of
// them, as they would have without.  It costs a bf16 call 0 to 3 %, the look at V's powers with it (262143 tokens 59 us either way, drafts 32.4 -> 32.8, 256
// query tokens over 60000 268 -> 272), an fp16 call 0 to 2 % (1024 query tokens over 8192 256 either way, 64 requests of 12400 tokens 113 either way, 200
// tokens of 20 queries 12.0 -> 12.3).
struct Gate {
  float room, times[2];
  int odd;
  bool low;
  __device__ __forceinline__ Gate(float c) : room(kRoom), times{c, c}, odd(0), low(false) {}
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

// The rows of an item that sees nothing.
template <bool ONE>
__device__ inline void store_nothing(const AttendArgs& a, const Walk& w) {
  const int rows = min(a.s.rows, w.q.rows - w.t * a.s.rows);
  for (int i = threadIdx.x; i < rows * 16; i += kThreads) {
    const int64_t at = row_place<ONE>(a, w, w.t * a.s.rows + (i >> 4));
    *(u32x4*)(a.out + (at * 128 + (i & 15) * 8) * 2) = u32x4{0, 0, 0, 0};
    if ((i & 15) == 0 && a.lse) a.lse[at] = -__builtin_inff();
  }
}

// ---- Few rows: every wave has all of an item's rows and every fourth run of 32 tokens.

template <int RT>
struct RowsLds {
  float ref[kWaves][16 * RT], sum[kWaves][16 * RT];
  float o[kWaves][16][132];
};

// What bounds it is memory: 64 requests of up to 12.4k tokens 580 MB in 108 us (5.4 TB/s; a plain read of as much 113).  Three waves a SIMD of one
// row tile: with four (128 registers) 153 us instead of 118, with touches of the lines of the pairs to come 147: 32 KB of lines is all that a compute
// unit's cache holds on their way.  Each wave's K is loaded again where it is used up, and so is V; held twice, whole pairs ahead, 121.
template <bool BF16, int RT, bool STREAM>
__global__ __launch_bounds__(kThreads, RT == 1 ? 3 : 2) void attend_rows_kernel(AttendArgs a) {
  // Probabilities as sums of two 16-bit numbers: with one row tile the matrix cores have the time (1 to 5 % of a call), and the only rounding
  // that counts is that of the output; with two tiles it is 10 %, and they are rounded once, which in the output is as much as its own rounding.
  constexpr bool kTwo = RT == 1;
  __shared__ RowsLds<RT> lds;
  const int lane = threadIdx.x & 63, wave = uniform((int)(threadIdx.x >> 6)), quarter = lane >> 4, col = lane & 15;
  // neighbouring stretches to one XCD: row tiles of a request and head read the same cache
  const int wg = (blockIdx.x % 8) * (gridDim.x / 8) + blockIdx.x / 8;
  Walk w;
  if (!find<true>(a, wg, w)) return;
  for (;;) {
    Part part;
    take_part<true>(a, w, part);
    if (only_free(w, part)) {
      leave_border(a, wg, -1, w);
      return;
    }
    if (w.item.pairs == 0) {
      store_nothing<true>(a, w);
      if (!go_on<true>(a, wg, w, part)) return;
      continue;
    }
    const char* head = a.cache + (int64_t)w.l * a.cache_layer_stride + (int64_t)w.h * (a.s.T >> 4) * kRecordBytes;
    const int32_t* table = a.tables + ((int64_t)w.l * a.s.R + w.r) * a.s.E;

    // the wave's pairs of tiles: every fourth from pa + wave on
    const int mine = (part.pb - part.pa - wave + kWaves - 1) / kWaves;
    u32x4 q[RT][4];
    f32x4 o[RT][8];
    float ref[RT], sum[RT];
    int low[RT];
    uint32_t span[RT];  // of the positions that the lane's row sees, from low on
#pragma unroll
    for (int t = 0; t < RT; ++t) {
      load_q<true>(a, w, 16 * t + col, quarter, q[t]);
      const int pos = row_position<true>(a, w, 16 * t + col);
      low[t] = attend_low(a.s, pos), span[t] = max(attend_high(a.s, pos) - low[t], 0);
#pragma unroll
      for (int c = 0; c < 8; ++c) o[t][c] = f32x4{0, 0, 0, 0};
      ref[t] = kNothing, sum[t] = 0.f;
    }

    Tile x[2];
    const char* rec[2];
    bool there[2], there_next[2] = {false, false};
    Gate gate(a.c);
    int ids = -1;
    const auto find_records = [&](int n) {
      if ((n & 31) == 0) {
        const int pair = part.pa + wave + kWaves * (n + (lane >> 1));
        ids = load_id(a, table, 2 * pair + (lane & 1), pair < part.pb);
      }
#pragma unroll
      for (int j = 0; j < 2; ++j) rec[j] = record(a, head, ids, 2 * (n & 31) + j, j, there_next[j]);
    };
    if (mine) {
      find_records(0);
#pragma unroll
      for (int j = 0; j < 2; ++j) load_k<STREAM>(x[j], rec[j], lane), load_v<STREAM>(x[j], rec[j], lane);
    }
    // The next pair's K is on its way from where this one's is used up, and V likewise.  The loads are never left out (behind the
    // last pair that one is loaded again): where a branch goes round them, a wait for some of the loads becomes a wait for all.
#pragma unroll 1
    for (int n = 0; n < mine; ++n) {
      const int pair = part.pa + wave + kWaves * n, pos = pair * kPairTokens;
      there[0] = there_next[0], there[1] = there_next[1];
      f32x4 s[RT][2];
      const float power[2] = {power_of(x[0].ke), power_of(x[1].ke)};
#pragma unroll
      for (int d = 0; d < 4; ++d) {
        u32x4 k[2];
#pragma unroll
        for (int j = 0; j < 2; ++j) k[j] = unpack8<BF16>(x[j].k[d], power[j]);
#pragma unroll
        for (int t = 0; t < RT; ++t)
#pragma unroll
          for (int j = 0; j < 2; ++j) s[t][j] = mfma<BF16>(k[j], q[t][d], d ? s[t][j] : f32x4{0, 0, 0, 0});
      }
      if (n + 1 < mine) find_records(n + 1);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int j = 0; j < 2; ++j) load_k<STREAM>(x[j], rec[j], lane);
      // every row sees all 32 tokens, but at the ends of what the rows see and where the table has a hole
      if (pos < w.item.low_max || pos + kPairTokens > w.item.high_min || !there[0] || !there[1]) {
        uint32_t flags = 0, seen[RT];
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          x[j].ve = seen_only(x[j].ve, pos + 16 * j + 4 * quarter, there[j], w.item);
          const uint32_t f = nan_bytes(x[j].ve);
          x[j].ve = without_nans(x[j].ve, f);
          flags |= f << (4 * j);
        }
#pragma unroll
        for (int t = 0; t < RT; ++t) {
          seen[t] = 0;
#pragma unroll
          for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
              const bool is = (uint32_t)(pos + 16 * j + 4 * quarter + r - low[t]) < (there[j] ? span[t] : 0u);
              seen[t] |= (uint32_t)is << (4 * j + r);
              s[t][j][r] = is ? s[t][j][r] : -__builtin_inff();
            }
        }
        if (__any(flags != 0)) {
#pragma unroll
          for (int t = 0; t < RT; ++t) poison<BF16>(o[t], flags, seen[t]);
        }
      }
      if constexpr (BF16) {
        if (__builtin_expect(__any(large_power(x[0].ve, x[1].ve)), 0)) gate.see(true);
      }
      u32x4 hi[RT], lo[RT];
#pragma unroll
      for (int t = 0; t < RT; ++t) {
        float top = s[t][0][0];
#pragma unroll
        for (int j = 0; j < 8; ++j) top = fmaxf(top, s[t][j >> 2][j & 3]);
        rescale<BF16>(s[t], o[t], ref[t], sum[t], top, a.c, t, gate, lds.ref[wave][16 * t + col]);
        float p[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) p[j] = __builtin_amdgcn_exp2f(fmaf(s[t][j >> 2][j & 3], gate.times[t], -ref[t]));
        sum[t] += ((p[0] + p[1]) + (p[2] + p[3])) + ((p[4] + p[5]) + (p[6] + p[7]));
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const uint32_t two = kTwo ? cut2<BF16>(p[2 * j], p[2 * j + 1]) : pack2<BF16>(p[2 * j], p[2 * j + 1]);
          hi[t][j] = two;
          if (kTwo) lo[t][j] = cut2<BF16>(p[2 * j] - low16<BF16>(two), p[2 * j + 1] - high16<BF16>(two));
        }
      }
      float p0[4], p1[4];
      powers(x[0].ve, p0);
      powers(x[1].ve, p1);
      const auto chunks = [&](auto b) {
        constexpr int B = decltype(b)::value;
        uint32_t e0[2], d0[2], e1[2], d1[2];
        unpack_v<BF16, B>(x[0].v, p0, e0, d0);
        unpack_v<BF16, B>(x[1].v, p1, e1, d1);
        const u32x4 even = {e0[0], e0[1], e1[0], e1[1]}, odd = {d0[0], d0[1], d1[0], d1[1]};
#pragma unroll
        for (int t = 0; t < RT; ++t) {
          o[t][2 * B] = mfma<BF16>(even, hi[t], o[t][2 * B]);
          o[t][2 * B + 1] = mfma<BF16>(odd, hi[t], o[t][2 * B + 1]);
          if (kTwo) {
            o[t][2 * B] = mfma<BF16>(even, lo[t], o[t][2 * B]);
            o[t][2 * B + 1] = mfma<BF16>(odd, lo[t], o[t][2 * B + 1]);
          }
        }

      };
      chunks(std::integral_constant<int, 0>{});
      chunks(std::integral_constant<int, 1>{});
      chunks(std::integral_constant<int, 2>{});
      chunks(std::integral_constant<int, 3>{});
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int j = 0; j < 2; ++j) load_v<STREAM>(x[j], rec[j], lane);
    }

    // the four waves' sums, under the largest of their references
#pragma unroll
    for (int t = 0; t < RT; ++t) {
      sum[t] = row_sum(sum[t]);
      if (gate.odd >> t & 1) ref[t] = lds.ref[wave][16 * t + col];
      if (quarter == 0) lds.ref[wave][16 * t + col] = ref[t], lds.sum[wave][16 * t + col] = sum[t];
    }
    __syncthreads();
    float* to_part = (float*)(a.parts + attend_place(wg, w.at == w.begin) * (int64_t)attend_part_bytes(16 * RT));
#pragma unroll
    for (int t = 0; t < RT; ++t) {
      float top = kNothing;
#pragma unroll
      for (int v = 0; v < kWaves; ++v) top = fmaxf(top, lds.ref[v][16 * t + col]);
      const float f = __builtin_amdgcn_exp2f(ref[t] - top);
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        float* to = &lds.o[wave][col][(4 * quarter + r) * 8];
        *(f32x4*)to = f32x4{o[t][0][r], o[t][1][r], o[t][2][r], o[t][3][r]} * f;
        *(f32x4*)(to + 4) = f32x4{o[t][4][r], o[t][5][r], o[t][6][r], o[t][7][r]} * f;
      }
      __syncthreads();
      // a thread adds eight dims of a row
      const int row = threadIdx.x >> 4, d = (threadIdx.x & 15) * 8, n = 16 * t + row;
      if (n < w.q.rows) {
        float m = kNothing, all = 0.f;
#pragma unroll
        for (int v = 0; v < kWaves; ++v) m = fmaxf(m, lds.ref[v][n]);
        f32x4 y0 = {0, 0, 0, 0}, y1 = {0, 0, 0, 0};
#pragma unroll
        for (int v = 0; v < kWaves; ++v) {
          all += lds.sum[v][n] * __builtin_amdgcn_exp2f(lds.ref[v][n] - m);
          y0 += *(const f32x4*)&lds.o[v][row][d];
          y1 += *(const f32x4*)&lds.o[v][row][d + 4];
        }
        if (part.whole) {
          const float f1 = row_scale(all);
          const int64_t at = row_place<true>(a, w, n);
          y0 *= f1, y1 *= f1;
          *(u32x4*)(a.out + (at * 128 + d) * 2) = u32x4{pack2<BF16>(y0[0], y0[1]), pack2<BF16>(y0[2], y0[3]), pack2<BF16>(y1[0], y1[1]), pack2<BF16>(y1[2], y1[3])};
          if (d == 0 && a.lse) a.lse[at] = row_lse(m, all);
        } else {
          *(f32x4*)(to_part + n * 128 + d) = y0;
          *(f32x4*)(to_part + n * 128 + d + 4) = y1;
          if (d == 0) *(float2*)(to_part + 16 * RT * 128 + n * 2) = float2{m, all};
        }
      }
      __syncthreads();
    }
    if (!go_on<true>(a, wg, w, part)) return;
  }
}

// ---- Many rows: every wave has 32 of an item's 128 rows (16 of 64 with one row tile), and the workgroup turns 64 tokens at a time into operands
// in LDS, once for all of its rows: every wave the codes of 16 tokens, into the buffer that the step does not read.
//
// A step of a wave is 64 matrix instructions (1024 cycles), some 250 other vector instructions and 40 KB of LDS; by the counters each of them fills about a
// third of the time: two waves a SIMD, as many as the registers allow, do not cover each other's waits.  A chunk of 1024 query tokens over 8192: 242 us and
// 13 for the parts of its cut items, 220 GFLOP at 860 TFLOP/s with these (a library product of 8192^3 runs at 1170 to 1220).  What it took, us: every operand read by itself 293,
// four ahead of their products 262, products beside exponentials and unpacking 256.  Probabilities are rounded once to 16 bits (the output is then off
// by 1.3 times what its own rounding makes it).

struct ManyLds {
  u32x4 k[2][4][4][64];  // [buffer][16 tokens][step of the dims][lane]
  u32x2 v[2][2][8][64][2];  // [buffer][32 tokens][chunk][lane][16 tokens of the 32]
  uint32_t ve[2][4][16];    // V's exponent words of the tiles of a buffer at the ends of what the rows see
  int32_t there[2][4];      // of the tiles of a buffer: whether there is a block, and 16 for large V
  float ref[kWaves][32];    // references of odd row tiles
};

template <bool BF16, int RT>
__global__ __launch_bounds__(kThreads, 2) void attend_many_kernel(AttendArgs a) {
  constexpr int kStep = 64, kRows = kWaves * 16 * RT;
  __shared__ ManyLds lds;
  const int lane = threadIdx.x & 63, wave = uniform((int)(threadIdx.x >> 6)), quarter = lane >> 4, col = lane & 15;
  const int wg = (blockIdx.x % 8) * (gridDim.x / 8) + blockIdx.x / 8;
  Walk w;
  if (!find<false>(a, wg, w)) return;
  for (;;) {
    Part cut;
    if (!take_part<false>(a, w, cut)) continue;
    if (only_free(w, cut)) {
      leave_border(a, wg, -1, w);
      return;
    }
    if (w.item.pairs == 0) {
      store_nothing<false>(a, w);
      if (!go_on<false>(a, wg, w, cut)) return;
      continue;
    }
    const int pa = cut.pa, pb = cut.pb;
    const char* head = a.cache + (int64_t)w.l * a.cache_layer_stride + (int64_t)w.h * (a.s.T >> 4) * kRecordBytes;
    const int32_t* table = a.tables + ((int64_t)w.l * a.s.R + w.r) * a.s.E;
    const int steps = (pb - pa + 1) / 2, row0 = w.t * kRows + wave * 16 * RT;
    const bool busy = row0 < w.q.rows;

    u32x4 q[RT][4];
    f32x4 o[RT][8];
    float ref[RT], sum[RT];
    int low[RT];
    uint32_t span[RT];
#pragma unroll
    for (int t = 0; t < RT; ++t) {
      const int n = row0 + 16 * t + col;
      load_q<false>(a, w, n, quarter, q[t]);
      const int pos = row_position<false>(a, w, n);
      low[t] = attend_low(a.s, pos), span[t] = max(attend_high(a.s, pos) - low[t], 0);
#pragma unroll
      for (int c = 0; c < 8; ++c) o[t][c] = f32x4{0, 0, 0, 0};
      ref[t] = kNothing, sum[t] = 0.f;
    }

    const auto at_ends = [&](int pos) { return pos < w.item.low_max || pos + kStep > w.item.high_min; };
    Gate gate(a.c);
    // the wave's 16 tokens of a step
    int ids = -1;
    const auto load = [&](Tile& x, bool& there, int step) {
      if ((step & 63) == 0) {
        const int pair = pa + 2 * (step + lane) + (wave >> 1);
        ids = load_id(a, table, 2 * pair + (wave & 1), pair < pb);
      }
      const char* rec = record(a, head, ids, step & 63, wave & 1, there);
      load_k<false>(x, rec, lane);
      load_v<false>(x, rec, lane);
    };
    const auto check = [&](Tile& x, bool there, int step, int buf) {
      const int pos = (pa + 2 * step) * kPairTokens;
      if (at_ends(pos) || !there) {
        x.ve = seen_only(x.ve, pos + 16 * wave + 4 * quarter, there, w.item);
        if ((col & 3) == 0) lds.ve[buf][wave][quarter * 4 + (col >> 2)] = x.ve;
        x.ve = without_nans(x.ve, nan_bytes(x.ve));
      }
      int flags = there;
      if constexpr (BF16) flags |= __any(large_power(x.ve, 0)) ? 16 : 0;
      if (lane == 0) lds.there[buf][wave] = flags;
    };
    const auto unpack = [&](const Tile& x, int buf) {
      const float power = power_of(x.ke);
#pragma unroll
      for (int d = 0; d < 4; ++d) lds.k[buf][wave][d][lane] = unpack8<BF16>(x.k[d], power);
      float p[4];
      powers(x.ve, p);
      const auto chunks = [&](auto b) {
        constexpr int B = decltype(b)::value;
        uint32_t e[2], d[2];
        unpack_v<BF16, B>(x.v, p, e, d);
        lds.v[buf][wave >> 1][2 * B][lane][wave & 1] = u32x2{e[0], e[1]};
        lds.v[buf][wave >> 1][2 * B + 1][lane][wave & 1] = u32x2{d[0], d[1]};
      };
      chunks(std::integral_constant<int, 0>{});
      chunks(std::integral_constant<int, 1>{});
      chunks(std::integral_constant<int, 2>{});
      chunks(std::integral_constant<int, 3>{});
    };
    const auto attend = [&](Tile& x, bool there_next, int step, int buf) {
      const int pos = (pa + 2 * step) * kPairTokens;
      // Operands come from LDS four at a time, while the products of the four before them run: left to the compiler, every read is
      // waited for by itself.
      f32x4 s[RT][4];
#pragma unroll
      for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int t = 0; t < RT; ++t) s[t][j] = f32x4{0, 0, 0, 0};
      u32x4 k[2][4];
      const auto read_k = [&](int i) {  // tiles 2 (i / 2) and the next, steps 2 (i % 2) and the next
#pragma unroll
        for (int m = 0; m < 4; ++m) k[i & 1][m] = lds.k[buf][(i & 2) + (m & 1)][2 * (i & 1) + (m >> 1)][lane];
      };
      read_k(0);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if (i < 3) read_k(i + 1);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int m = 0; m < 4; ++m)
#pragma unroll
          for (int t = 0; t < RT; ++t) s[t][(i & 2) + (m & 1)] = mfma<BF16>(k[i & 1][m], q[t][2 * (i & 1) + (m >> 1)], s[t][(i & 2) + (m & 1)]);
        __builtin_amdgcn_sched_barrier(0);
      }
      int there = uniform(lds.there[buf][0] | lds.there[buf][1] << 1 | lds.there[buf][2] << 2 | lds.there[buf][3] << 3);
      if constexpr (BF16) {
        gate.see(there > 15);
        there &= 15;
      }
      const bool ends = at_ends(pos);
      if (ends || there != 15) {
        uint32_t flags = 0;
        if (ends) {
#pragma unroll
          for (int j = 0; j < 4; ++j) flags |= nan_bytes(lds.ve[buf][j][quarter * 4 + (col >> 2)]) << (4 * j);
        }
        const bool any = __any(flags != 0);
#pragma unroll
        for (int t = 0; t < RT; ++t) {
          uint32_t seen = 0;
#pragma unroll
          for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
              const bool is = (uint32_t)(pos + 16 * j + 4 * quarter + r - low[t]) < (there >> j & 1 ? span[t] : 0u);
              seen |= (uint32_t)is << (4 * j + r);
              s[t][j][r] = is ? s[t][j][r] : -__builtin_inff();
            }
          if (any) {
            poison<BF16>(o[t], flags & 255, seen & 255);
            poison<BF16>(o[t], flags >> 8, seen >> 8);
          }
        }
      }
#pragma unroll
      for (int t = 0; t < RT; ++t) {
        float top = s[t][0][0];
#pragma unroll
        for (int j = 0; j < 16; ++j) top = fmaxf(top, s[t][j >> 2][j & 3]);
        rescale<BF16>(s[t], o[t], ref[t], sum[t], top, a.c, t, gate, lds.ref[wave][16 * t + col]);
      }
      check(x, there_next, step + 1, buf ^ 1);
      u32x4 v[8], p16[RT][2];
      const auto read_v = [&](int i) {  // the chunks of tokens 32 i and the next
#pragma unroll
        for (int c = 0; c < 8; ++c) v[c] = *(const u32x4*)&lds.v[buf][i][c][lane][0];
      };
      const auto weigh = [&](int i) {
#pragma unroll
        for (int t = 0; t < RT; ++t) {
          float p[8];
#pragma unroll
          for (int j = 0; j < 8; ++j) p[j] = __builtin_amdgcn_exp2f(fmaf(s[t][2 * i + (j >> 2)][j & 3], gate.times[t], -ref[t]));
#pragma unroll
          for (int j = 0; j < 4; ++j) p16[t][i][j] = pack2<BF16>(p[2 * j], p[2 * j + 1]);
          sum[t] += ((p[0] + p[1]) + (p[2] + p[3])) + ((p[4] + p[5]) + (p[6] + p[7]));
        }
      };
      const auto add = [&](int i) {
#pragma unroll
        for (int c = 0; c < 8; ++c)
#pragma unroll
          for (int t = 0; t < RT; ++t) o[t][c] = mfma<BF16>(v[c], p16[t][i], o[t][c]);
      };
      // The products of the first 32 tokens run beside the exponentials of the other 32, and theirs beside the next step's unpacking.
      read_v(0);
      __builtin_amdgcn_sched_barrier(0);
      weigh(0);
      __builtin_amdgcn_sched_barrier(0);
      add(0);
      weigh(1);
#pragma unroll
      for (int i = 0; i < 8 * RT; ++i) {
        __builtin_amdgcn_sched_group_barrier(0x8, 1, 0);
        __builtin_amdgcn_sched_group_barrier(0x2, 4, 0);
      }
      __builtin_amdgcn_sched_barrier(0);
      read_v(1);
      add(1);
      unpack(x, buf ^ 1);
#pragma unroll
      for (int i = 0; i < 8 * RT; ++i) {
        __builtin_amdgcn_sched_group_barrier(0x8, 1, 1);
        __builtin_amdgcn_sched_group_barrier(0x2, 4, 1);
        __builtin_amdgcn_sched_group_barrier(0x200, 1, 1);
      }
      __builtin_amdgcn_sched_barrier(0);
    };

    Tile x;
    bool there;
    if (steps > 0) {
      load(x, there, 0);
      check(x, there, 0, 0);
      unpack(x, 0);
    }
    __syncthreads();
    // behind the last step a tile of no block is loaded and unpacked into the buffer that is free
    for (int step = 0; step < steps; ++step) {
      load(x, there, step + 1);
      if (busy) {
        attend(x, there, step, step & 1);
      } else {
        check(x, there, step + 1, ~step & 1);
        unpack(x, ~step & 1);
      }
      __syncthreads();
    }

    float* part = (float*)(a.parts + attend_place(wg, w.at == w.begin) * (int64_t)attend_part_bytes(kRows));
#pragma unroll
    for (int t = 0; t < RT; ++t) {
      const float all = row_sum(sum[t]);
      if (gate.odd >> t & 1) ref[t] = lds.ref[wave][16 * t + col];
      const int m = wave * 16 * RT + 16 * t + col, n = w.t * kRows + m;
      if (n >= w.q.rows) continue;
      if (cut.whole) {
        const float f = row_scale(all);
        const int64_t at = row_place<false>(a, w, n);
#pragma unroll
        for (int r = 0; r < 4; ++r)
          *(u32x4*)(a.out + (at * 128 + (4 * quarter + r) * 8) * 2) =
              u32x4{pack2<BF16>(o[t][0][r] * f, o[t][1][r] * f), pack2<BF16>(o[t][2][r] * f, o[t][3][r] * f),
                    pack2<BF16>(o[t][4][r] * f, o[t][5][r] * f), pack2<BF16>(o[t][6][r] * f, o[t][7][r] * f)};
        if (quarter == 0 && a.lse) a.lse[at] = row_lse(ref[t], all);
      } else {
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          *(f32x4*)(part + m * 128 + (4 * quarter + r) * 8) = f32x4{o[t][0][r], o[t][1][r], o[t][2][r], o[t][3][r]};
          *(f32x4*)(part + m * 128 + (4 * quarter + r) * 8 + 4) = f32x4{o[t][4][r], o[t][5][r], o[t][6][r], o[t][7][r]};
        }
        if (quarter == 0) part[kRows * 128 + m * 2] = ref[t], part[kRows * 128 + m * 2 + 1] = all;
      }
    }
    if (!go_on<false>(a, wg, w, cut)) return;
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

rc_status attend_check(const rc_cache_desc* d, int64_t R, int64_t E, int32_t n_heads, int64_t n_q, int64_t max_q, int64_t window, AttendShape* s,
                       const char* who) {
  if (rc_status e = check_cache(d, who)) return e;
  if (R < 0 || E < 0 || n_q < 0 || max_q < 0 || window < 0) return fail(RC_ERR_INVALID_ARG, "%s: negative size", who);
  if (n_heads < 1 || n_heads % d->n_kv_heads != 0)
    return fail(RC_ERR_INVALID_ARG, "%s: n_heads %d is not a multiple of n_kv_heads %d", who, n_heads, d->n_kv_heads);
  if (n_heads > 1024) return fail(RC_ERR_UNSUPPORTED, "%s: n_heads %d (at most 1024)", who, n_heads);
  if (!attend_shape(s, d->n_layers, R, d->n_blocks ? E : 0, d->block_tokens, d->n_kv_heads, n_heads, n_q, max_q, window))
    return fail(RC_ERR_UNSUPPORTED, "%s: a table of 2^31 positions or more, or more than 2^30 query tokens, requests or row tiles", who);
  return RC_OK;
}

template <bool BF16>
void attend_launch(const AttendArgs& a, hipStream_t st) {
  const dim3 grid(a.s.wgs);
  const bool stream = attend_streams(a.s);
  if (a.s.rows == 16)
    stream ? attend_rows_kernel<BF16, 1, true><<<grid, kThreads, 0, st>>>(a) : attend_rows_kernel<BF16, 1, false><<<grid, kThreads, 0, st>>>(a);
  else if (a.s.rows == 32)
    stream ? attend_rows_kernel<BF16, 2, true><<<grid, kThreads, 0, st>>>(a) : attend_rows_kernel<BF16, 2, false><<<grid, kThreads, 0, st>>>(a);
  else if (a.s.rows == 64)
    attend_many_kernel<BF16, 1><<<grid, kThreads, 0, st>>>(a);
  else
    attend_many_kernel<BF16, 2><<<grid, kThreads, 0, st>>>(a);
  if (!a.borders) return;
  const int64_t rows = (int64_t)a.s.max_q * a.s.g;
  if (a.s.rows <= 32)
    attend_join_kernel<BF16, true><<<dim3(a.s.wgs - 1, (unsigned)(rows < a.s.rows ? rows : a.s.rows)), kThreads, 0, st>>>(a);
  else
    attend_join_kernel<BF16, false><<<dim3(a.s.wgs - 1, 8), kThreads, 0, st>>>(a);
}

}  // namespace
}  // namespace rc

extern "C" size_t rc_cache_attend_workspace_size(const rc_cache_desc* desc, int64_t R, int64_t E, int32_t n_heads, int64_t max_q) {
  using namespace rc;
  clear_error();
  AttendShape s;
  const int64_t q = max_q < 1 ? max_q : 1;
  if (attend_check(desc, R, E, n_heads, q, q, 0, &s, "rc_cache_attend_workspace_size")) return 0;
  return attend_largest_workspace(s.L, R, s.E, s.T, s.H, n_heads, max_q);
}

extern "C" rc_status rc_cache_attend(const rc_cache_desc* desc, const void* cache, const int32_t* tables, int64_t R, int64_t E,
                                     const int32_t* ctx_len, const int32_t* q_start, const void* q, int64_t n_q, int32_t n_heads,
                                     int64_t q_token_stride, int64_t q_layer_stride, int64_t max_q, float scale, int64_t window,
                                     void* out, float* lse, void* workspace, size_t workspace_bytes, void* hip_stream) {
  using namespace rc;
  const char* who = "rc_cache_attend";
  clear_error();
  AttendArgs a;
  if (rc_status e = attend_check(desc, R, E, n_heads, n_q, max_q, window, &a.s, who)) return e;
  if (!q_start && (max_q > 1 || n_q < R)) return fail(RC_ERR_INVALID_ARG, "%s: without q_start there is one query token per request", who);
  a.c = scale * 1.4426950408889634f;
  if (!(scale > 0.f) || !(a.c < __builtin_inff()))
    return fail(RC_ERR_INVALID_ARG, "%s: scale must be positive, and scale * log2(e) an fp32 number", who);
  if (desc->n_layers == 0 || R == 0 || n_q == 0 || max_q == 0) return RC_OK;
  const bool empty = a.s.cap == 0;  // nothing to see: no table and no cache are read
  if (!ctx_len || !q || !out || (!empty && (!cache || !tables))) return fail(RC_ERR_INVALID_ARG, "%s: NULL pointer", who);
  if (!aligned16(q) || !aligned16(out) || (!empty && !aligned16(cache))) return fail(RC_ERR_INVALID_ARG, "%s: pointer not 16-byte aligned", who);
  if (q_token_stride < (int64_t)n_heads * 128 || q_token_stride > INT64_MAX / 4 / n_q || q_token_stride % 8 != 0 || q_layer_stride % 8 != 0)
    return fail(RC_ERR_INVALID_ARG, "%s: q_token_stride smaller than n_heads*Dh, or a stride that breaks 16-byte alignment", who);
  if (desc->n_layers > 1 && q_layer_stride < (int64_t)n_heads * 128) return fail(RC_ERR_INVALID_ARG, "%s: q_layer_stride smaller than a token", who);
  const size_t need = attend_workspace(a.s);
  if (need) {
    if (!workspace || workspace_bytes < need) return fail(RC_ERR_WORKSPACE, "%s: needs %zu bytes of workspace", who, need);
    if (!aligned16(workspace)) return fail(RC_ERR_WORKSPACE, "%s: workspace not 16-byte aligned", who);
  }
  a.cache = (const char*)cache, a.tables = tables, a.ctx_len = ctx_len, a.q_start = q_start;
  a.q = (const char*)q, a.out = (char*)out, a.lse = lse;
  a.cache_layer_stride = desc->layer_stride, a.q_token_stride_b = q_token_stride * 2, a.q_layer_stride_b = q_layer_stride * 2;
  a.n_blocks = desc->n_blocks;
  a.borders = need ? (AttendBorder*)workspace : nullptr;
  a.parts = need ? (char*)workspace + attend_header_bytes(a.s.wgs) : nullptr;
  hipStream_t st = static_cast<hipStream_t>(hip_stream);
  if (desc->dtype == RC_BF16)
    attend_launch<true>(a, st);
  else
    attend_launch<false>(a, st);
  return check_launch(who);
}
