// rc_kv_attend: softmax attention over 16-bit paged KV blocks, one pass over the data with a running reference of the softmax, and what
// every block gathers of it.
//
// Scores are taken as S^T = K Q^T and outputs as O^T = V^T P^T on 16x16x32 matrix instructions: a row (a query token and head) is a
// column of both, so that its scores, its probabilities and its sums lie in the same four lanes and the probabilities go from
// one product into the next as they are.  A token's head is 256 bytes in a row of memory.  K's operand (a lane: 8 dims of a token) is what a
// load of 16 bytes brings.  V's (a lane: 8 tokens of a dim) are, with few rows, eight such loads, of eight tokens, whose halves are paired by one byte
// permute for each two values, so that no value moves between lanes; with many rows V lies in LDS token by token and is read transposed.
#include <hip/hip_runtime.h>

#include "rc_attend.hpp"
#include "rc_kv.hpp"

// Lambdas of a kernel work on its registers: one that were called instead would put them into memory.
#define RC_INLINE __attribute__((always_inline))

namespace rc {
namespace {

struct KvAttendArgs : AttendArgs {
  const char *k, *v;
  int64_t layer_stride_b;
  uint32_t token_b, block_b;  // bytes of a token's heads, of a block
  f32x4* gathered;            // few rows: what the rows' weights of a run of 32 tokens come to, [L][R][H][runs][rows]: of its two tiles, and their reference
  int32_t runs, kept_rows;
};

// ---- Loads.

// What a wave holds of 16 tokens: K in operand order (lane: token lane % 16, dims 32 d + 8 (lane / 16) on), V as it lies (lane: dims 8 (lane % 16) on of
// tokens 4 (lane / 16) + r).
struct KvTile {
  u32x4 k[4], v[4];
};
struct KvLanes {
  uint32_t k, v[4];  // the lane's offsets into a tile
  __device__ __forceinline__ KvLanes(const KvAttendArgs& a, int lane) : k((lane & 15) * a.token_b + (lane >> 4) * 16) {
#pragma unroll
    for (int r = 0; r < 4; ++r) v[r] = (4 * (lane >> 4) + r) * a.token_b + (lane & 15) * 16;
  }
};
// STREAM: tokens that no other workgroup reads are not kept in the caches behind this one, where there are too many of them anyway.
typedef const __attribute__((address_space(1))) char* global_ptr;
template <bool STREAM>
__device__ __forceinline__ u32x4 load16(global_ptr p) {
  typedef const __attribute__((address_space(1))) u32x4* vector_ptr;
  if constexpr (STREAM)
    return __builtin_nontemporal_load((vector_ptr)p);
  else
    return *(vector_ptr)p;
}
// An address that all lanes have in common, kept in scalar registers: left to the compiler, each lane's offset is added to the first part of it outside of
// the loop, in vector registers.
__device__ __forceinline__ global_ptr scalar(const char* p) {
  asm volatile("" : "+s"(p));
  return (global_ptr)p;
}
template <bool STREAM>
__device__ __forceinline__ void load_k(KvTile& x, const char* k, const KvLanes& at) {
  const global_ptr p = scalar(k);
#pragma unroll
  for (int d = 0; d < 4; ++d) x.k[d] = load16<STREAM>(p + at.k + d * 64);
}
template <bool STREAM>
__device__ __forceinline__ void load_v(KvTile& x, const char* v, const KvLanes& at) {
  const global_ptr p = scalar(v);
#pragma unroll
  for (int r = 0; r < 4; ++r) x.v[r] = load16<STREAM>(p + at.v[r]);
}
// Where the tile whose id lane j holds lies behind the layer's and head's first byte (its parity chooses between the halves of a block of 32); in block 0
// where there is no such block (`there` false): its values are replaced or masked.
__device__ __forceinline__ uint64_t tile_offset(const KvAttendArgs& a, int id, int parity, bool& there) {
  there = id >= 0;
  return (uint64_t)(uint32_t)(there ? id : 0) * a.block_b + (a.s.T == 32 ? parity * 16 * a.token_b : 0);
}

// Row n of q as lane (row, quarter) holds it for the four steps of K's dims; rows that the item does not have: its last one's.
template <bool ONE>
__device__ __forceinline__ void load_rows(const AttendArgs& a, const Walk& w, int n, int quarter, u32x4 (&q)[4]) {
  n = min(n, w.q.rows - 1);
  const int j = row_token<ONE>(a, n), head = w.h * a.s.g + n - j * a.s.g;
  const char* p = a.q + (int64_t)w.l * a.q_layer_stride_b + (int64_t)(w.q.first + j) * a.q_token_stride_b + head * 256 + quarter * 16;
#pragma unroll
  for (int s = 0; s < 4; ++s) q[s] = *(const u32x4*)(p + s * 64);
}

// V's operands of dims 8i + 2B and 8i + 2B + 1 (lane i of 16) from word B of four tokens: tokens 0 and 1 to one register, 2 and 3 to the next.
template <int B>
__device__ __forceinline__ void pair_v(const u32x4 (&v)[4], uint32_t (&even)[2], uint32_t (&odd)[2]) {
#pragma unroll
  for (int p = 0; p < 2; ++p) {
    even[p] = __builtin_amdgcn_perm(v[2 * p + 1][B], v[2 * p][B], 0x05040100u);
    odd[p] = __builtin_amdgcn_perm(v[2 * p + 1][B], v[2 * p][B], 0x07060302u);
  }
}

// Whether any of a lane's values is a bf16 number of 2^65 or more (its exponent byte 192 or more).
__device__ __forceinline__ uint32_t large_bits(const u32x4 (&v)[4]) {
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < 16; ++i) m |= v[i >> 2][i & 3] & v[i >> 2][i & 3] << 1;
  return m & 0x40004000u;
}
// Infinities and NaNs among two 16-bit values: their halves' bits.
template <bool BF16>
__device__ __forceinline__ uint32_t strange_half(uint32_t w) {
  constexpr uint32_t inf = BF16 ? 0x7f80u : 0x7c00u;
  return ((w & inf) == inf ? 0xffffu : 0u) | ((w >> 16 & inf) == inf ? 0xffff0000u : 0u);
}
// V of tokens that no row sees replaced by 0: whatever lies there (memory that was never written) gets a probability of 0, and 0 times infinity or NaN would
// not be 0.  So are infinities and NaNs of tokens that only some rows may see: strange() adds them to these.  Token r of the lane stands at pos + r.  True if
// there were such.
template <bool BF16, int N>
__device__ inline bool seen_only(u32x4 (&v)[N], int pos, bool there, const AttendItem& it) {
  const uint32_t span = there ? it.high_max - it.low_min : 0;  // (an item that sees no token has no run)
  uint32_t found = 0;
#pragma unroll
  for (int r = 0; r < N; ++r) {
    const uint32_t keep = (uint32_t)(pos + r - it.low_min) < span ? ~0u : 0u;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t x = v[r][i] & keep, bad = strange_half<BF16>(x);
      found |= bad;
      v[r][i] = x & ~bad;
    }
  }
  return found != 0;
}
// Infinities and NaNs of a tile's V (16 tokens from position pos on) into the sums of the rows that see them: the lane's row sees `span` positions from
// low on.  o[c][r] is the sum of dim 32 * quarter + 8 r + c, FOURS: 4 c + r.
template <bool BF16, bool FOURS>
__device__ __forceinline__ void strange(f32x4 (&o)[8], const char* v, uint32_t token_b, int pos, int low, uint32_t span, int quarter) {
#pragma unroll 1
  for (int t = 0; t < 16; ++t) {
    const bool seen = (uint32_t)(pos + t - low) < span;
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      __builtin_amdgcn_sched_barrier(0);
      const u32x4 x = *(const u32x4*)(v + t * token_b + (4 * quarter + r) * 16);
#pragma unroll
      for (int c = 0; c < 8; ++c) {
        const uint32_t w = x[c >> 1], bad = strange_half<BF16>(w);
        const float add = seen && (c & 1 ? bad >> 16 : bad & 0xffffu) ? c & 1 ? high16<BF16>(w) : low16<BF16>(w) : 0.f;
        if constexpr (FOURS)
          o[2 * r + (c >> 2)][c & 3] += add;
        else
          o[c][r] += add;
      }
    }
  }
}

// ---- Few rows: every wave has all of an item's rows and every fourth run of 32 tokens.

template <int RT>
struct RowsLds {
  float ref[kWaves][16 * RT], sum[kWaves][16 * RT];
  float o[kWaves][16][132];
};

// What bounds it is memory: 64 requests of up to 12400 tokens 2.18 GB in 381 us (5.7 TB/s; a read of 4 GB runs at 5.9), one of
// 262143 tokens 1.07 GB in 194 (5.5).  Two waves a SIMD: for three (168 registers, some of a run's values in memory) 470 us and 247.  Calls of few rows and short contexts
// are bound by what comes one after the other: 300 tokens 9.5 us, a launch, the lengths, the block ids, three runs of 32 tokens a wave, the joining of four
// waves.  With weights a wave leaves the sums of the two tiles of a run and its reference for every row, 16 bytes beside the run's 16384.
template <bool BF16, int RT, bool STREAM, bool WEIGH>
__global__ __launch_bounds__(kThreads, 2) void kv_rows_kernel(KvAttendArgs a) {
  // Probabilities are sums of two 16-bit numbers: the matrix cores have the time, and the only rounding that counts is that of the output.  24 rows over
  // 305 MB, two numbers and one: bf16 78 and 89 us (184 and 328 B a thread in memory), fp16 90 and 90 (336 B either way); with weights 102 and 111 in
  // both types (188 and 340).  Against 64 bits the outputs of one number are 1.3 times as far off.
  __shared__ RowsLds<RT> lds;
  const int lane = threadIdx.x & 63, wave = uniform((int)(threadIdx.x >> 6)), quarter = lane >> 4, col = lane & 15;
  const int wg = (blockIdx.x % 8) * (gridDim.x / 8) + blockIdx.x / 8;
  const KvLanes lanes(a, lane);
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
      store_nothing<true, true>(a, w);
      if (!go_on<true>(a, wg, w, part)) return;
      continue;
    }
    const int64_t head = (int64_t)w.l * a.layer_stride_b + w.h * 256;
    const char *head_k = a.k + head, *head_v = a.v + head;
    const int32_t* table = a.tables + ((int64_t)w.l * a.s.R + w.r) * a.s.E;
    f32x4* gathered = nullptr;
    if constexpr (WEIGH) gathered = a.gathered + (((int64_t)w.l * a.s.R + w.r) * a.s.H + w.h) * (int64_t)a.runs * a.kept_rows;

    // the wave's runs of 32 tokens: every fourth from pa + wave on
    const int mine = (part.pb - part.pa - wave + kWaves - 1) / kWaves;
    u32x4 q[RT][4];
    f32x4 o[RT][8];
    float ref[RT], sum[RT];
    int low[RT];
    uint32_t span[RT];  // of the positions that the lane's row sees, from low on
#pragma unroll
    for (int t = 0; t < RT; ++t) {
      load_rows<true>(a, w, 16 * t + col, quarter, q[t]);
      const int pos = row_position<true>(a, w, 16 * t + col);
      low[t] = attend_low(a.s, pos), span[t] = max(attend_high(a.s, pos) - low[t], 0);
#pragma unroll
      for (int c = 0; c < 8; ++c) o[t][c] = f32x4{0, 0, 0, 0};
      ref[t] = kNothing, sum[t] = 0.f;
    }

    KvTile x[2];
    uint64_t at[2] = {0, 0};
    bool there[2], there_next[2] = {false, false};
    Gate gate(a.c);
    // Runs whose blocks are all gone are passed over: block ids of 32 runs at a time, a bit of `left` for each that has a block.
    int ids = -1, batch = -32, n = 0;
    uint64_t left = 0;
    const auto next = [&]() -> bool {
      while (left == 0) {
        batch += 32;
        if (batch >= mine) return false;
        const int pair = part.pa + wave + kWaves * (batch + (lane >> 1));
        ids = load_id(a, table, 2 * pair + (lane & 1), pair < part.pb);
        const uint64_t b = __ballot(ids >= 0);
        left = (b | b >> 1) & 0x5555555555555555ull;
      }
      const int bit = __builtin_ctzll(left);
      left &= left - 1;
      n = batch + (bit >> 1);
#pragma unroll
      for (int j = 0; j < 2; ++j) at[j] = tile_offset(a, __builtin_amdgcn_readlane(ids, bit + j), j, there_next[j]);
      return true;
    };
    bool more = next();
    if (more) {
#pragma unroll
      for (int j = 0; j < 2; ++j) load_k<STREAM>(x[j], head_k + at[j], lanes);
    }
    // A run's V is on its way from where its K is used, the next one's K from where this one's is used up: more at a time (V behind the last run's
    // products) is slower, 390 us for 381 (64 requests of up to 12400 tokens) and 97 for 87 (24 rows).  The loads are never left out (behind the
    // last run that one is loaded again): where a branch goes round them, a wait for some of the loads becomes a wait for all.
#pragma unroll 1
    while (more) {
      const int pair = part.pa + wave + kWaves * n, pos = pair * kPairTokens;
      const uint64_t here[2] = {at[0], at[1]};
      there[0] = there_next[0], there[1] = there_next[1];
#pragma unroll
      for (int j = 0; j < 2; ++j) load_v<STREAM>(x[j], head_v + here[j], lanes);
      __builtin_amdgcn_sched_barrier(0);
      f32x4 s[RT][2];
#pragma unroll
      for (int d = 0; d < 4; ++d)
#pragma unroll
        for (int t = 0; t < RT; ++t)
#pragma unroll
          for (int j = 0; j < 2; ++j) s[t][j] = mfma<BF16>(x[j].k[d], q[t][d], d ? s[t][j] : f32x4{0, 0, 0, 0});
      more = next();
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int j = 0; j < 2; ++j) load_k<STREAM>(x[j], head_k + at[j], lanes);
      // every row sees all 32 tokens, but at the ends of what the rows see and where the table has a hole
      if (pos < w.item.low_max || pos + kPairTokens > w.item.high_min || !there[0] || !there[1]) {
        bool odd[2];
#pragma unroll
        for (int j = 0; j < 2; ++j) odd[j] = __any(seen_only<BF16>(x[j].v, pos + 16 * j + 4 * quarter, there[j], w.item));
#pragma unroll
        for (int t = 0; t < RT; ++t) {
#pragma unroll
          for (int j = 0; j < 2; ++j) {
#pragma unroll
            for (int r = 0; r < 4; ++r) {
              const bool is = (uint32_t)(pos + 16 * j + 4 * quarter + r - low[t]) < (there[j] ? span[t] : 0u);
              s[t][j][r] = is ? s[t][j][r] : -__builtin_inff();
            }
            if (__builtin_expect(odd[j], 0)) strange<BF16, false>(o[t], head_v + here[j], a.token_b, pos + 16 * j, low[t], span[t], quarter);
          }
        }
      }
      if constexpr (BF16) {
        if (__builtin_expect(__any((large_bits(x[0].v) | large_bits(x[1].v)) != 0), 0)) gate.see(true);
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
        const float first = (p[0] + p[1]) + (p[2] + p[3]), second = (p[4] + p[5]) + (p[6] + p[7]);
        sum[t] += first + second;
        if constexpr (WEIGH) {
          const float a0 = row_sum(first), a1 = row_sum(second);
          if (quarter == 0 && 16 * t + col < w.q.rows)
            gathered[(int64_t)pair * a.kept_rows + 16 * t + col] = f32x4{a0, a1, gate.odd >> t & 1 ? lds.ref[wave][16 * t + col] : ref[t], 0};
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const uint32_t two = cut2<BF16>(p[2 * j], p[2 * j + 1]);
          hi[t][j] = two;
          lo[t][j] = cut2<BF16>(p[2 * j] - low16<BF16>(two), p[2 * j + 1] - high16<BF16>(two));
        }
      }
      const auto chunks = [&](auto b) {
        constexpr int B = decltype(b)::value;
        uint32_t e0[2], d0[2], e1[2], d1[2];
        pair_v<B>(x[0].v, e0, d0);
        pair_v<B>(x[1].v, e1, d1);
        const u32x4 even = {e0[0], e0[1], e1[0], e1[1]}, odd = {d0[0], d0[1], d1[0], d1[1]};
#pragma unroll
        for (int t = 0; t < RT; ++t) {
          o[t][2 * B] = mfma<BF16>(even, hi[t], o[t][2 * B]);
          o[t][2 * B + 1] = mfma<BF16>(odd, hi[t], o[t][2 * B + 1]);
          o[t][2 * B] = mfma<BF16>(even, lo[t], o[t][2 * B]);
          o[t][2 * B + 1] = mfma<BF16>(odd, lo[t], o[t][2 * B + 1]);
        }
      };
      chunks(std::integral_constant<int, 0>{});
      chunks(std::integral_constant<int, 1>{});
      chunks(std::integral_constant<int, 2>{});
      chunks(std::integral_constant<int, 3>{});
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
      const int row = threadIdx.x >> 4, d = (threadIdx.x & 15) * 8, m = 16 * t + row;
      if (m < w.q.rows) {
        float most = kNothing, all = 0.f;
#pragma unroll
        for (int v = 0; v < kWaves; ++v) most = fmaxf(most, lds.ref[v][m]);
        f32x4 y0 = {0, 0, 0, 0}, y1 = {0, 0, 0, 0};
#pragma unroll
        for (int v = 0; v < kWaves; ++v) {
          all += lds.sum[v][m] * __builtin_amdgcn_exp2f(lds.ref[v][m] - most);
          y0 += *(const f32x4*)&lds.o[v][row][d];
          y1 += *(const f32x4*)&lds.o[v][row][d + 4];
        }
        if (part.whole) {
          const float f1 = row_scale(all);
          const int64_t place = row_place<true>(a, w, m);
          y0 *= f1, y1 *= f1;
          *(u32x4*)(a.out + (place * 128 + d) * 2) = u32x4{pack2<BF16>(y0[0], y0[1]), pack2<BF16>(y0[2], y0[3]), pack2<BF16>(y1[0], y1[1]), pack2<BF16>(y1[2], y1[3])};
          if (d == 0 && a.lse) a.lse[place] = row_lse(most, all);
          if (WEIGH && d == 0) a.ends[place] = float2{most, all};
        } else {
          *(f32x4*)(to_part + m * 128 + d) = y0;
          *(f32x4*)(to_part + m * 128 + d + 4) = y1;
          if (d == 0) *(float2*)(to_part + 16 * RT * 128 + m * 2) = float2{most, all};
        }
      }
      __syncthreads();
    }
    if (!go_on<true>(a, wg, w, part)) return;
  }
}

// ---- Many rows: every wave has 16 RT of an item's rows, and the workgroup takes runs of 32 tokens into LDS, once for all of its rows: straight from
// memory, three runs ahead of the one that is computed.  K comes in operand order: a lane asks for the 16 bytes that it will hold.
// V comes token by token, and reads that transpose give a lane four tokens of a dim; the 16-byte units of a token's 256 are exchanged by its
// number (unit u lies at u ^ token % 4), so that the sixteen lanes of such a read, four tokens and four units of each, find different banks.
//
// A run of a wave with 48 rows is 48 matrix instructions (768 cycles), some 110 other vector instructions, 24 of them exponentials, and 16 KB of LDS.  A chunk of
// 1024 query tokens over 8192: 220 GFLOP in 237 us at the card's steady speed (930 TFLOP/s; a library product of 8192^3 runs at 1155) and 16 for the parts of cut items; a
// SIMD's matrix unit is busy for 39 % of the time, its other vector instructions take 28 % at four cycles each and more where they are exponentials, a compute unit's LDS 20 %.  Two waves a SIMD, each a chain of reads, products, exponentials and products, do not cover each other's waits:
// workgroups of equal work end between 190 and 286 us.  What was tried against that (us before the card has reached its speed, 256 as it is): wave tiles of 32 rows 280 us, steps of 64 tokens to a barrier 258, products
// woven between exponentials 260, K and V through registers 293, two groups of four waves that take turns at the matrix cores with a barrier at each turn 320 to 385.
// Without the loads it takes 8 % less, without the exponentials 14 %.

constexpr int kRuns = 4;  // buffers

template <int RT>
struct ManyLds {
  u32x4 k[kRuns][2][4][64];    // [buffer][16 tokens][step of the dims][lane]
  u32x4 v[kRuns][2][4][64];    // [buffer][16 tokens][4 tokens][unit]
  int32_t odd[kWaves];         // infinities or NaNs that only some rows may see, in the part of a run that a wave looked through
  float ref[kWaves][16 * RT];  // references of odd row tiles
};

// 16 bytes a lane from memory into LDS, lane l's to to + 16 l, past the registers: counted by vmcnt, waited for by hand.
__device__ __forceinline__ void to_lds(const char* base, uint32_t offset, uint32_t to) {
  asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1" : : "v"(offset), "s"(base), "s"(to) : "memory", "m0");
}
__device__ __forceinline__ uint32_t lds_offset(const void* p) { return (uint32_t)(uintptr_t)(const __attribute__((address_space(3))) char*)p; }

// Four tokens of a dim: lane 4 k + m of sixteen names dims 4 m' .. 4 m' + 3 of token k, lane l gets dim l % 4 of those that the lanes l / 4 named.
__device__ __forceinline__ u32x2 read_transposed(uint32_t at) {
  typedef short s4 __attribute__((ext_vector_type(4)));
  typedef __attribute__((address_space(3))) s4* lds_ptr;
  return __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr)(uintptr_t)at));
}

// Sums of this size and more of bf16 values might overflow, here or where parts are joined: the item is computed again under lower limits (rescale()).
constexpr float kLargeSum = 0x1p100f;

template <bool BF16, int RT>
__global__ __launch_bounds__(kThreads, 2) void kv_many_kernel(KvAttendArgs a) {
  constexpr int kRows = kWaves * 16 * RT;
  __shared__ ManyLds<RT> lds;
  const int lane = threadIdx.x & 63, wave = uniform((int)(threadIdx.x >> 6)), quarter = lane >> 4, col = lane & 15;
  const int wg = (blockIdx.x % 8) * (gridDim.x / 8) + blockIdx.x / 8;
  Walk w;
  if (!find<false>(a, wg, w)) return;
  // A wave brings half of a run's K and V of 16 tokens: steps 2 part and the next of K's dims, tokens 8 part .. 8 part + 7 of V.
  const int tile = wave >> 1, part = wave & 1;
  const uint32_t from_k = col * a.token_b + quarter * 16 + part * 128, from_v = (8 * part + quarter) * a.token_b + (col ^ quarter) * 16;
  // where the lane's transposed reads of chunk pairs begin: the four tokens of its quarter, token (lane / 4) % 4, unit 4 (lane % 4) + i
  uint32_t read_at[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) read_at[i] = lds_offset(&lds.v[0][0][quarter][(col >> 2) * 16 + (lane & 3) * 4 + (i ^ (col >> 2))]);
  for (;;) {
    Part cut;
    if (!take_part<false>(a, w, cut)) continue;
    if (only_free(w, cut)) {
      leave_border(a, wg, -1, w);
      return;
    }
    if (w.item.pairs == 0) {
      store_nothing<false, true>(a, w);
      if (!go_on<false>(a, wg, w, cut)) return;
      continue;
    }
    const int64_t head = (int64_t)w.l * a.layer_stride_b + w.h * 256;
    const char *head_k = a.k + head, *head_v = a.v + head;
    const int32_t* table = a.tables + ((int64_t)w.l * a.s.R + w.r) * a.s.E;
    const int mine = cut.pb - cut.pa, row0 = w.t * kRows + wave * 16 * RT;
    const bool busy = row0 < w.q.rows;

    u32x4 q[RT][4];
    f32x4 o[RT][8];
    float ref[RT], sum[RT];
    int low[RT];
    uint32_t span[RT];
#pragma unroll
    for (int t = 0; t < RT; ++t) {
      const int n = row0 + 16 * t + col;
      load_rows<false>(a, w, n, quarter, q[t]);
      const int pos = row_position<false>(a, w, n);
      low[t] = attend_low(a.s, pos), span[t] = max(attend_high(a.s, pos) - low[t], 0);
    }
    // (waited for here: in the loop a wait for them would be one for the runs on their way as well)
#pragma unroll
    for (int t = 0; t < RT; ++t)
#pragma unroll
      for (int d = 0; d < 4; ++d) asm volatile("" : "+v"(q[t][d]));

    Gate gate(a.c);
    // Runs whose blocks are all gone are passed over: block ids of 32 runs at a time, a bit of `left` for each that has a block.
    int ids = -1, batch = -32;
    uint64_t left = 0;
    // of the runs in the buffers: position (-1: there is no further run), and whether its tiles have blocks (bits 0 and 1)
    int pos[kRuns], there[kRuns];
    const auto load = [&](int b) RC_INLINE {
      pos[b] = -1;
      while (left == 0) {
        batch += 32;
        if (batch >= mine) return;
        const int pair = cut.pa + batch + (lane >> 1);
        ids = load_id(a, table, 2 * pair + (lane & 1), pair < cut.pb);
        const uint64_t x = __ballot(ids >= 0);
        left = (x | x >> 1) & 0x5555555555555555ull;
      }
      const int bit = __builtin_ctzll(left);
      left &= left - 1;
      pos[b] = (cut.pa + batch + (bit >> 1)) * kPairTokens;
      const int id0 = __builtin_amdgcn_readlane(ids, bit), id1 = __builtin_amdgcn_readlane(ids, bit + 1);
      there[b] = (id0 >= 0) | (id1 >= 0) << 1;
      bool is;
      const uint64_t at = tile_offset(a, tile ? id1 : id0, tile, is);
      const uint32_t k = lds_offset(&lds.k[b][tile][2 * part][0]), v = lds_offset(&lds.v[b][tile][2 * part][0]);
#pragma unroll
      for (int i = 0; i < 2; ++i) to_lds(head_k + at, from_k + i * 64, k + i * 1024);
#pragma unroll
      for (int i = 0; i < 2; ++i) to_lds(head_v + at, from_v + 4 * i * a.token_b, v + i * 1024);
    };
    // What no row sees of the wave's part of a run, and what only some rows may see, is made 0 where it lies.  Bits of tiles with such.
    const auto clean = [&](int b) RC_INLINE {
      bool odd = false;
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        u32x4* p = &lds.v[b][tile][2 * part + i][lane];
        u32x4 one[1] = {*p};
        odd |= seen_only<BF16>(one, pos[b] + 16 * tile + 4 * (2 * part + i) + quarter, there[b] >> tile & 1, w.item);
        *p = one[0];
      }
      const bool any = __any(odd);
      if (lane == 0) lds.odd[wave] = any;
      __syncthreads();
      return uniform((lds.odd[0] | lds.odd[1]) | (lds.odd[2] | lds.odd[3]) << 1);
    };
    const auto attend = [&](int b, bool masked, int odd) RC_INLINE {
      f32x4 s[RT][2];
      // Operands come from LDS ahead of their products: left to the compiler, nearly every read is waited for by itself.
      u32x4 k[2][2];
      const auto read_k = [&](int d) RC_INLINE {
#pragma unroll
        for (int j = 0; j < 2; ++j) k[d & 1][j] = lds.k[b][j][d][lane];
      };
      read_k(0);
#pragma unroll
      for (int d = 0; d < 4; ++d) {
        if (d < 3) read_k(d + 1);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
          for (int t = 0; t < RT; ++t) s[t][j] = mfma<BF16>(k[d & 1][j], q[t][d], d ? s[t][j] : f32x4{0, 0, 0, 0});
        __builtin_amdgcn_sched_barrier(0);
      }
      if (__builtin_expect(masked, 0)) {
#pragma unroll
        for (int t = 0; t < RT; ++t)
#pragma unroll
          for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
              const bool is = (uint32_t)(pos[b] + 16 * j + 4 * quarter + r - low[t]) < (there[b] >> j & 1 ? span[t] : 0u);
              s[t][j][r] = is ? s[t][j][r] : -__builtin_inff();
            }
#pragma unroll 1
        for (int j = 0; odd >> j; ++j) {
          if (!(odd >> j & 1)) continue;
          bool is;
          const uint64_t at = tile_offset(a, uniform(load_id(a, table, pos[b] / 16 + j, true)), j, is);
#pragma unroll
          for (int t = 0; t < RT; ++t) strange<BF16, true>(o[t], head_v + at, a.token_b, pos[b] + 16 * j, low[t], span[t], quarter);
        }
      }
      float top[RT];
      bool over = false;
#pragma unroll
      for (int t = 0; t < RT; ++t) {
        top[t] = s[t][0][0];
#pragma unroll
        for (int j = 0; j < 8; ++j) top[t] = fmaxf(top[t], s[t][j >> 2][j & 3]);
        over |= fmaf(top[t], gate.times[t], -ref[t]) > gate.room;
      }
      if (__builtin_expect(__any(over), 0)) {
#pragma unroll
        for (int t = 0; t < RT; ++t) rescale<BF16>(s[t], o[t], ref[t], sum[t], top[t], a.c, t, gate, lds.ref[wave][16 * t + col]);
      }
      // A probability is rounded once to the 16-bit type, as an operand of the second product (the sums of weights take it in fp32).  As the sum of two
      // such numbers it takes half of this loop's matrix instructions again: the chunk of 1024 336 us for 254, prompts of 2500 tokens 191 for 153, for outputs that are
      // off by 6.2e-6 instead of 8.6e-6 in the mean square of the chunk (fp16; bf16 4.9e-5 and 6.8e-5), where the rounding of the output itself is most of the former.
      u32x4 v[2][4], p16[RT];
      const auto read_v = [&](int i) RC_INLINE {  // chunks 4 i to 4 i + 3
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          const uint32_t at = read_at[2 * i + (c >> 1)] + b * (uint32_t)sizeof(lds.v[0]) + (c & 1) * 8;
          const u32x2 x = read_transposed(at), y = read_transposed(at + (uint32_t)sizeof(lds.v[0][0]));
          v[i][c] = u32x4{x[0], x[1], y[0], y[1]};
        }
      };
      read_v(0);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int t = 0; t < RT; ++t) {
        float p[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) p[j] = __builtin_amdgcn_exp2f(fmaf(s[t][j >> 2][j & 3], gate.times[t], -ref[t]));
#pragma unroll
        for (int j = 0; j < 4; ++j) p16[t][j] = pack2<BF16>(p[2 * j], p[2 * j + 1]);
        sum[t] += ((p[0] + p[1]) + (p[2] + p[3])) + ((p[4] + p[5]) + (p[6] + p[7]));
      }
      __builtin_amdgcn_sched_barrier(0);
      read_v(1);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int c = 0; c < 8; ++c)
#pragma unroll
        for (int t = 0; t < RT; ++t) o[t][c] = mfma<BF16>(v[c >> 2][c & 3], p16[t], o[t][c]);
    };

    for (;;) {
#pragma unroll
      for (int t = 0; t < RT; ++t) {
#pragma unroll
        for (int c = 0; c < 8; ++c) o[t][c] = f32x4{0, 0, 0, 0};
        ref[t] = kNothing, sum[t] = 0.f;
      }
      ids = -1, batch = -32, left = 0;
      // (the buffers are free: whoever read them last has passed a barrier since, or is behind the loop's last one and reads no more)
      __syncthreads();
#pragma unroll
      for (int b = 0; b + 1 < kRuns; ++b) load(b);
      bool more = true;
      while (more) {
#pragma unroll
        for (int b = 0; b < kRuns; ++b) {
          if (pos[b] < 0) {
            more = false;
            break;
          }
          // this run has landed where the two behind it may still be on their way, and nobody reads the buffer before it any more
          if (pos[(b + 2) % kRuns] >= 0)
            asm volatile("s_waitcnt vmcnt(8) lgkmcnt(0)\n\ts_barrier" ::: "memory");
          else
            asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
          load((b + 3) % kRuns);
          const bool masked = pos[b] < w.item.low_max || pos[b] + kPairTokens > w.item.high_min || there[b] != 3;
          const int odd = masked ? clean(b) : 0;
          if (busy) attend(b, masked, odd);
        }
      }
      if constexpr (!BF16) break;
      bool large = false;
#pragma unroll
      for (int t = 0; t < RT; ++t)
#pragma unroll
        for (int i = 0; i < 32; ++i) large |= !(fabsf(o[t][i >> 2][i & 3]) < kLargeSum);
      if (gate.low || !__syncthreads_or(large && busy)) break;
      gate = Gate(a.c);
      gate.see(true);
    }

    float* to_part = (float*)(a.parts + attend_place(wg, w.at == w.begin) * (int64_t)attend_part_bytes(kRows));
#pragma unroll
    for (int t = 0; t < RT; ++t) {
      const float all = row_sum(sum[t]);
      if (gate.odd >> t & 1) ref[t] = lds.ref[wave][16 * t + col];
      const int m = wave * 16 * RT + 16 * t + col, n = w.t * kRows + m;
      if (n >= w.q.rows) continue;
      if (cut.whole) {
        const float f = row_scale(all);
        const int64_t place = row_place<false>(a, w, n);
#pragma unroll
        for (int i = 0; i < 4; ++i)
          *(u32x4*)(a.out + (place * 128 + quarter * 32 + i * 8) * 2) =
              u32x4{pack2<BF16>(o[t][2 * i][0] * f, o[t][2 * i][1] * f), pack2<BF16>(o[t][2 * i][2] * f, o[t][2 * i][3] * f),
                    pack2<BF16>(o[t][2 * i + 1][0] * f, o[t][2 * i + 1][1] * f), pack2<BF16>(o[t][2 * i + 1][2] * f, o[t][2 * i + 1][3] * f)};
        if (quarter == 0 && a.lse) a.lse[place] = row_lse(ref[t], all);
        if (quarter == 0 && a.ends) a.ends[place] = float2{ref[t], all};
      } else {
#pragma unroll
        for (int c = 0; c < 8; ++c) *(f32x4*)(to_part + m * 128 + quarter * 32 + c * 4) = o[t][c];
        if (quarter == 0) to_part[kRows * 128 + m * 2] = ref[t], to_part[kRows * 128 + m * 2 + 1] = all;
      }
    }
    if (!go_on<false>(a, wg, w, cut)) return;
  }
}

// ---- What blocks gather.

struct WeighArgs {
  KvAttendArgs a;
  const float* in;
  float* out;
  float* sums;  // many rows: of the rows of a share and KV head, [share][L][R][H][tiles of 16 tokens]
  int32_t tiles, shares;
};

// Many rows: the probabilities are taken once more, from K, Q and the rows' final references and sums: a wave holds the K of 128 tokens and goes through a
// share of the rows that see them.  (Kept from the first time they would be a number for each row and 16 tokens: 10 GB for a prompt of 32k tokens and 40 heads.)
// Prompts of 2500 tokens and 32 heads: 51 GFLOP in 103 us at the card's steady speed (115 before it).  Nothing is busy all the time: the matrix units are for 19 % of it, other
// vector instructions take 31 % at four cycles each, and more where they are exponentials.  Without the loads of rows, which every wave takes from the L2 for itself,
// a pass takes 18 us less, without the exponentials 8.  64 tokens a wave 142 us for 117, 32 and 64 shares of the rows instead of 16 122 and 149;
// with the rows read when they are needed 228, two tiles ahead 116 for 115, with one tile's products after another's 147, four tiles' products beside the powers of the
// last four 123 for 115.
constexpr int kWeighTiles = 8;

template <bool BF16>
__global__ __launch_bounds__(kThreads, 2) void weigh_many_kernel(WeighArgs g) {
  const KvAttendArgs& a = g.a;
  const int lane = threadIdx.x & 63, quarter = lane >> 4, col = lane & 15, chunks = (g.tiles + kWeighTiles - 1) / kWeighTiles;
  const int64_t heads = a.s.L * a.s.R * a.s.H, tasks = heads * chunks * g.shares;
  for (int64_t task = (int64_t)blockIdx.x * kWaves + uniform((int)(threadIdx.x >> 6)); task < tasks; task += (int64_t)gridDim.x * kWaves) {
    // shares beside each other: they read the same K; the first chunks, which most rows see, before the later ones
    const int64_t i = task / g.shares;
    const int share = (int)(task - i * g.shares), chunk = (int)(i / heads);
    int64_t at = i - chunk * heads;
    Walk w;
    w.h = (int)(at % a.s.H);
    at /= a.s.H;
    w.r = (int)(at % a.s.R), w.l = (int)(at / a.s.R), w.t = 0;
    w.q = request(a, w.r);
    const int pos0 = chunk * kWeighTiles * 16, pos1 = pos0 + (kWeighTiles * 16 - 1), first = w.q.ctx - w.q.len;  // (pos1 + 1 may be 2^31)
    if (w.q.rows == 0) continue;
    // the rows that see any of these tokens
    const int last = first + (w.q.rows - 1) / a.s.g;
    if (attend_high(a.s, last) <= pos0 || attend_low(a.s, first) > pos1) continue;
    // the row tiles that see any of these tokens, and the task's share of them
    const int g_ = a.s.g;
    const int64_t beyond = a.s.window ? ((int64_t)pos1 + a.s.window - first) * g_ : w.q.rows;
    const int t0 = pos0 > first ? (int)(((int64_t)pos0 - first) * g_ / 16) : 0, t1 = (int)((min(beyond, (int64_t)w.q.rows) + 15) / 16);
    const int64_t all = max(t1 - t0, 0);
    const int from = t0 + (int)(all * share / g.shares), to = t0 + (int)(all * (share + 1) / g.shares);
    const int32_t* table = a.tables + ((int64_t)w.l * a.s.R + w.r) * a.s.E;
    const char* head_k = a.k + (int64_t)w.l * a.layer_stride_b + w.h * 256 + (lane & 15) * a.token_b + quarter * 16;
    u32x4 k[kWeighTiles][4];
    int there = 0;
    const int ids = from < to ? load_id(a, table, chunk * kWeighTiles + (lane & (kWeighTiles - 1)), true) : -1;
    if (from < to) {
#pragma unroll
      for (int j = 0; j < kWeighTiles; ++j) {
        bool is;
        const uint64_t at = tile_offset(a, __builtin_amdgcn_readlane(ids, j), j & 1, is);
        there |= (int)is << j;
#pragma unroll
        for (int d = 0; d < 4; ++d) k[j][d] = *(const u32x4*)(head_k + at + d * 64);
      }
    }
    float sum[kWeighTiles];
#pragma unroll
    for (int j = 0; j < kWeighTiles; ++j) sum[j] = 0.f;
    struct Rows {
      u32x4 q[4];
      float2 end;
      int pos;
    };
    const auto load = [&](Rows& x, int t) RC_INLINE {
      const int n = t * 16 + col, m = min(n, w.q.rows - 1), j = (int)((uint32_t)m / (uint32_t)g_), row = w.h * g_ + m - j * g_;
      x.pos = first + j;
      x.end = a.ends[((int64_t)w.l * a.s.n_q + w.q.first + j) * (int64_t)(a.s.H * g_) + row];
      const char* p = a.q + (int64_t)w.l * a.q_layer_stride_b + (int64_t)(w.q.first + j) * a.q_token_stride_b + row * 256 + quarter * 16;
#pragma unroll
      for (int d = 0; d < 4; ++d) x.q[d] = *(const u32x4*)(p + d * 64);
    };
    const auto add_rows = [&](const Rows& x, int t) RC_INLINE {
      const int p0 = __builtin_amdgcn_readlane(x.pos, 0), p1 = __builtin_amdgcn_readlane(x.pos, 15);
      // a row that is not there, or that sees nothing: no weight, and a reference that no score comes near
      const bool none = t * 16 + col >= w.q.rows || x.end.y == 0.f;
      // a row that is not finite has a NaN where it sees a token, and only there
      const bool bad = !none && !(fabsf(x.end.x) < __builtin_inff() && x.end.y < __builtin_inff());
      const bool ends = attend_low(a.s, p1) > pos0 || attend_high(a.s, p0) <= pos1 || there != (1 << kWeighTiles) - 1;
      const float f = none ? 0.f : bad ? 1.f : 1.f / x.end.y, ref = none ? -kNothing : bad ? ends ? 0.f : __builtin_nanf("") : x.end.x;
      const int low = attend_low(a.s, x.pos);
      const uint32_t span = max(attend_high(a.s, x.pos) - low, 0);
      const bool coarse = uniform(__any(f != 0.f && fabsf(ref) > kCoarse));
      // four tiles at a time: a product waits for the one before it of the same tile
#pragma unroll
      for (int j0 = 0; j0 < kWeighTiles; j0 += 4) {
        f32x4 s[4];
#pragma unroll
        for (int d = 0; d < 4; ++d)
#pragma unroll
          for (int j = 0; j < 4; ++j) s[j] = mfma<BF16>(k[j0 + j][d], x.q[d], d ? s[j] : f32x4{0, 0, 0, 0});
        __builtin_amdgcn_sched_barrier(0);
        if (__builtin_expect(ends, 0)) {
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            const int j = j0 + (i >> 2);
            const bool is = (uint32_t)(pos0 + 16 * j + 4 * quarter + (i & 3) - low) < (there >> j & 1 ? span : 0u);
            s[i >> 2][i & 3] = !is ? -__builtin_inff() : bad ? __builtin_nanf("") : s[i >> 2][i & 3];
          }
        }
        if (__builtin_expect(coarse, 0)) {
#pragma unroll
          for (int i = 0; i < 16; ++i) {
#pragma clang fp contract(off)
            const float z = s[i >> 2][i & 3] * a.c, d = z - ref;
            s[i >> 2][i & 3] = fabsf(ref) > kCoarse ? d : fmaf(s[i >> 2][i & 3], a.c, -ref);
          }
        } else {
#pragma unroll
          for (int i = 0; i < 16; ++i) s[i >> 2][i & 3] = fmaf(s[i >> 2][i & 3], a.c, -ref);
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          float p[4];
#pragma unroll
          for (int r = 0; r < 4; ++r) p[r] = __builtin_amdgcn_exp2f(s[j][r]);
          sum[j0 + j] = fmaf((p[0] + p[1]) + (p[2] + p[3]), f, sum[j0 + j]);
        }
      }
    };
    // the next rows are on their way beside the products of these
    Rows x, y;
    if (from < to) load(x, from);
#pragma unroll 1
    for (int t = from; t < to; t += 2) {
      load(y, min(t + 1, to - 1));
      add_rows(x, t);
      load(x, min(t + 2, to - 1));
      if (t + 1 < to) add_rows(y, t + 1);
    }
    float* sums = g.sums + ((((int64_t)share * a.s.L + w.l) * a.s.R + w.r) * a.s.H + w.h) * (int64_t)g.tiles + chunk * kWeighTiles;
#pragma unroll
    for (int j = 0; j < kWeighTiles; ++j) {
      float x = row_sum(sum[j]);
#pragma unroll
      for (int d = 8; d; d >>= 1) x += __shfl_xor(x, d);
      if (lane == 0 && chunk * kWeighTiles + j < g.tiles) sums[j] = x;
    }
  }
}

// Eight lanes add up what the rows of an entry's KV heads left, every lane of every eighth of them.
template <bool FEW>
__global__ __launch_bounds__(kThreads) void weigh_entries_kernel(WeighArgs g) {
  const KvAttendArgs& a = g.a;
  const int64_t E = a.s.E, total = a.s.L * a.s.R * E;
  const int part = threadIdx.x & 7;
  for (int64_t at = (int64_t)blockIdx.x * 32 + (threadIdx.x >> 3); at < total; at += (int64_t)gridDim.x * 32) {
    const int e = (int)(at % E);
    const int64_t lr = at / E;
    const int r = (int)(lr % a.s.R), l = (int)(lr / a.s.R);
    const AttendRequest q = request(a, r);
    float sum = 0.f;
    if (q.rows) {
      const int first = q.ctx - q.len, last = first + (q.rows - 1) / a.s.g;
      const int low = attend_low(a.s, first), high = attend_high(a.s, last);
      const int id = a.tables[at];
      const int64_t begin = (int64_t)e * a.s.T;
      if (id >= 0 && id < a.n_blocks && begin < high && begin + a.s.T > low) {
        const int per = a.s.T >> 4;
        if constexpr (FEW) {
          const int pair = per == 2 ? e : e >> 1;
          // where some rows do not see the entry: what these left may be a NaN
          const bool some = begin < attend_low(a.s, last) || begin + a.s.T > attend_high(a.s, first);
          const f32x4* gathered = a.gathered + (lr * a.s.H * (int64_t)a.runs + pair) * a.kept_rows;
          for (int i = part; i < a.s.H * q.rows; i += 8) {
            const int h = i / q.rows, n = i - h * q.rows;
            if (some && (begin >= attend_high(a.s, first + n / a.s.g) || begin + a.s.T <= attend_low(a.s, first + n / a.s.g))) continue;
            const f32x4 x = gathered[(int64_t)h * a.runs * a.kept_rows + n];
            const float2 end = a.ends[row_place<false>(a, l, h, q.first, n)];
            const float w = per == 2 ? x[0] + x[1] : e & 1 ? x[1] : x[0];
            const float p = w * __builtin_amdgcn_exp2f(x[2] - end.x) * row_scale(end.y);
            sum += end.y == 0.f ? 0.f : p;
          }
        } else {
          const float* sums = g.sums + lr * a.s.H * (int64_t)g.tiles + (int64_t)e * per;
          const int64_t step = a.s.L * a.s.R * a.s.H * (int64_t)g.tiles;
          for (int i = part; i < a.s.H * g.shares; i += 8) {
            const int share = i / a.s.H, h = i - share * a.s.H;
            const float* x = sums + share * step + (int64_t)h * g.tiles;
            sum += per == 2 ? x[0] + x[1] : x[0];
          }
        }
      }
    }
#pragma unroll
    for (int d = 4; d; d >>= 1) sum += __shfl_xor(sum, d);
    if (part == 0) g.out[at] = g.in ? g.in[at] + sum : sum;
  }
}

// ---- The call.

// What the workspace holds behind the parts of cut items, where blocks are weighed.
struct WeighRoom {
  int64_t ends, gathered, sums;  // bytes
  int32_t shares;
  int64_t bytes() const { return ends + gathered + sums; }
};
constexpr int64_t up16(int64_t n) { return (n + 15) / 16 * 16; }
constexpr int kFewRows = 32, kMostShares = 16, kMostWaves = 4096;
constexpr int64_t kMostSharedBytes = 2 * kMostWaves * kWeighTiles * 4;
constexpr int64_t kMostEntries = 1 << 29;  // table entries of a call that weighs them

inline int64_t runs_of(const AttendShape& s) { return ((int64_t)s.cap + 31) / 32; }
inline WeighRoom few_room(int64_t L, int64_t R, int64_t H, int64_t runs, int64_t rows) { return {0, L * R * H * runs * rows * 16, 0, 0}; }
inline WeighRoom many_room(int64_t L, int64_t R, int64_t H, int64_t runs, int64_t rows) {
  // A few thousand waves, of 8 row tiles at least.  (By the tables' width: those of contexts that fill a small part of their table are fewer.  Prompts of 2500 tokens
  // in tables for 131072 have one share instead of 16, and their weights take 994 us instead of 103.)
  const double chunks = (double)L * R * H * ((runs * 2 + kWeighTiles - 1) / kWeighTiles);
  int64_t shares = 1;
  while (shares < kMostShares && shares * 2 * 128 <= rows && chunks * shares < kMostWaves) shares *= 2;
  return {0, 0, up16(shares * L * R * H * runs * 2 * 4), (int32_t)shares};
}
inline WeighRoom weigh_room(const AttendShape& s) {
  const int64_t rows = (int64_t)s.max_q * s.g, runs = runs_of(s);
  WeighRoom r = rows <= kFewRows ? few_room(s.L, s.R, s.H, runs, rows) : many_room(s.L, s.R, s.H, runs, rows);
  r.ends = up16(s.L * s.n_q * s.H * s.g * 8);
  return r;
}

rc_status kv_check(const rc_kv_desc* d, int64_t n_blocks, int64_t R, int64_t E, int32_t n_heads, int64_t n_q, int64_t max_q, int64_t window, bool weigh,
                   AttendShape* s, const char* who) {
  if (rc_status e = check_paged(d, n_blocks, who)) return e;
  if (R < 0 || E < 0 || n_q < 0 || max_q < 0 || window < 0) return fail(RC_ERR_INVALID_ARG, "%s: negative size", who);
  if (n_heads < 1 || n_heads % d->n_kv_heads != 0)
    return fail(RC_ERR_INVALID_ARG, "%s: n_heads %d is not a multiple of n_kv_heads %d", who, n_heads, d->n_kv_heads);
  if (n_heads > 1024) return fail(RC_ERR_UNSUPPORTED, "%s: n_heads %d (at most 1024)", who, n_heads);
  if (!attend_shape(s, d->n_layers, R, n_blocks ? E : 0, d->block_tokens, d->n_kv_heads, n_heads, n_q, max_q, window, kv_kernel))
    return fail(RC_ERR_UNSUPPORTED, "%s: a table of 2^31 positions or more, or more than 2^30 query tokens, requests or row tiles", who);
  if (weigh && (double)d->n_layers * R * E > (double)kMostEntries) return fail(RC_ERR_UNSUPPORTED, "%s: more than 2^29 table entries to weigh", who);
  return RC_OK;
}

// Whether a call's tables can hold more than the last-level cache keeps from one pass over them to the next.
inline bool kv_streams(const AttendShape& s) {
  const double seen = s.window && (double)s.window + s.max_q < s.cap ? (double)s.window + s.max_q : s.cap;
  return (double)s.L * s.R * s.H * seen * 512 > 384e6;
}

template <bool BF16, bool STREAM, bool WEIGH>
void kv_rows_launch(const KvAttendArgs& a, hipStream_t st) {
  if (a.s.rows == 16)
    kv_rows_kernel<BF16, 1, STREAM, WEIGH><<<dim3(a.s.wgs), kThreads, 0, st>>>(a);
  else
    kv_rows_kernel<BF16, 2, STREAM, WEIGH><<<dim3(a.s.wgs), kThreads, 0, st>>>(a);
}

template <bool BF16>
void kv_launch(const WeighArgs& g, hipStream_t st) {
  const KvAttendArgs& a = g.a;
  const bool stream = kv_streams(a.s), few = a.s.rows <= kFewRows;
  if (few && g.out)
    stream ? kv_rows_launch<BF16, true, true>(a, st) : kv_rows_launch<BF16, false, true>(a, st);
  else if (few)
    stream ? kv_rows_launch<BF16, true, false>(a, st) : kv_rows_launch<BF16, false, false>(a, st);
  else if (a.s.rows == 64)
    kv_many_kernel<BF16, 1><<<dim3(a.s.wgs), kThreads, 0, st>>>(a);
  else if (a.s.rows == 128)
    kv_many_kernel<BF16, 2><<<dim3(a.s.wgs), kThreads, 0, st>>>(a);
  else
    kv_many_kernel<BF16, 3><<<dim3(a.s.wgs), kThreads, 0, st>>>(a);
  if (a.borders) {
    const int64_t rows = (int64_t)a.s.max_q * a.s.g;
    if (few)
      attend_join_kernel<BF16, true><<<dim3(a.s.wgs - 1, (unsigned)(rows < a.s.rows ? rows : a.s.rows)), kThreads, 0, st>>>(a);
    else
      attend_join_kernel<BF16, false><<<dim3(a.s.wgs - 1, (a.s.rows + 15) / 16), kThreads, 0, st>>>(a);
  }
  if (!g.out) return;
  const int64_t entries = a.s.L * a.s.R * a.s.E;
  if (!few) {
    const int64_t tasks = a.s.L * a.s.R * a.s.H * ((g.tiles + kWeighTiles - 1) / kWeighTiles) * (int64_t)g.shares, wgs = (tasks + kWaves - 1) / kWaves;
    weigh_many_kernel<BF16><<<dim3((unsigned)(wgs < (1 << 22) ? wgs : (1 << 22))), kThreads, 0, st>>>(g);
  }
  const int64_t wgs = (entries + 31) / 32;
  const dim3 grid((unsigned)(wgs < (1 << 22) ? wgs : (1 << 22)));
  few ? weigh_entries_kernel<true><<<grid, kThreads, 0, st>>>(g) : weigh_entries_kernel<false><<<grid, kThreads, 0, st>>>(g);
}

// Nothing was asked: what was gathered before is what there is.
__global__ __launch_bounds__(kThreads) void weigh_nothing_kernel(const float* in, float* out, int64_t n) {
  const int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x;
  if (i < n) out[i] = in ? in[i] : 0.f;
}

}  // namespace
}  // namespace rc

extern "C" size_t rc_kv_attend_workspace_size(const rc_kv_desc* desc, int64_t n_blocks, int64_t R, int64_t E, int32_t n_heads, int64_t n_q, int64_t max_q,
                                              int32_t weigh) {
  using namespace rc;
  clear_error();
  AttendShape s;
  const int64_t q = max_q < 1 ? max_q : 1;
  if (n_q < 0) return 0;
  if (kv_check(desc, n_blocks, R, E, n_heads, q, q, 0, weigh != 0, &s, "rc_kv_attend_workspace_size")) return 0;
  size_t n = attend_largest_workspace(s.L, R, s.E, s.T, s.H, n_heads, max_q, kv_kernel);
  if (weigh && max_q > 0) {
    if ((double)s.L * n_q * n_heads > 1e15) return 0;
    const int64_t runs = runs_of(s), few = max_q < kFewRows / s.g ? max_q : kFewRows / s.g;
    // many rows: more shares than one are taken while there are fewer than 8192 waves, of kWeighTiles sums each
    const int64_t one = many_room(s.L, R, s.H, runs, 1).bytes(), shared = kMostShares * one < kMostSharedBytes ? kMostShares * one : kMostSharedBytes;
    const int64_t a = few_room(s.L, R, s.H, runs, few * s.g).bytes(), b = one > shared ? one : shared;
    n = (size_t)up16((int64_t)n) + (size_t)up16(s.L * n_q * n_heads * 8) + (size_t)(max_q > kFewRows / s.g && b > a ? b : a);
  }
  return n;
}

extern "C" rc_status rc_kv_attend(const rc_kv_desc* desc, int64_t n_blocks, const void* k, const void* v, const int32_t* tables, int64_t R, int64_t E,
                                  const int32_t* ctx_len, const int32_t* q_start, const void* q, int64_t n_q, int32_t n_heads, int64_t q_token_stride,
                                  int64_t q_layer_stride, int64_t max_q, float scale, int64_t window, void* out, float* lse, const float* weights_in,
                                  float* weights_out, void* workspace, size_t workspace_bytes, void* hip_stream) {
  using namespace rc;
  const char* who = "rc_kv_attend";
  clear_error();
  WeighArgs g;
  KvAttendArgs& a = g.a;
  if (rc_status e = kv_check(desc, n_blocks, R, E, n_heads, n_q, max_q, window, weights_out != nullptr, &a.s, who)) return e;
  if (!q_start && (max_q > 1 || n_q < R)) return fail(RC_ERR_INVALID_ARG, "%s: without q_start there is one query token per request", who);
  a.c = scale * 1.4426950408889634f;
  if (!(scale > 0.f) || !(a.c < __builtin_inff()))
    return fail(RC_ERR_INVALID_ARG, "%s: scale must be positive, and scale * log2(e) an fp32 number", who);
  if (weights_in && !weights_out) return fail(RC_ERR_INVALID_ARG, "%s: weights_in without weights_out", who);
  hipStream_t st = static_cast<hipStream_t>(hip_stream);
  const int64_t entries = weights_out ? (int64_t)desc->n_layers * R * E : 0;
  const auto keep_weights = [&] {
    if (entries == 0 || weights_in == weights_out) return RC_OK;
    weigh_nothing_kernel<<<dim3((unsigned)((entries + kThreads - 1) / kThreads)), kThreads, 0, st>>>(weights_in, weights_out, entries);
    return check_launch(who);
  };
  if (desc->n_layers == 0 || R == 0 || n_q == 0 || max_q == 0) return keep_weights();
  const bool empty = a.s.cap == 0;  // nothing to see: no table and no blocks are read
  if (!ctx_len || !q || !out || (!empty && (!k || !v || !tables))) return fail(RC_ERR_INVALID_ARG, "%s: NULL pointer", who);
  if (!aligned16(q) || !aligned16(out) || (!empty && (!aligned16(k) || !aligned16(v)))) return fail(RC_ERR_INVALID_ARG, "%s: pointer not 16-byte aligned", who);
  if (q_token_stride < (int64_t)n_heads * 128 || q_token_stride > INT64_MAX / 4 / n_q || q_token_stride % 8 != 0 || q_layer_stride % 8 != 0)
    return fail(RC_ERR_INVALID_ARG, "%s: q_token_stride smaller than n_heads*Dh, or a stride that breaks 16-byte alignment", who);
  if (desc->n_layers > 1 && q_layer_stride < (int64_t)n_heads * 128) return fail(RC_ERR_INVALID_ARG, "%s: q_layer_stride smaller than a token", who);
  const size_t parts = attend_workspace(a.s);
  WeighRoom room = {0, 0, 0, 0};
  if (weights_out) {
    if ((double)a.s.L * n_q * n_heads > 1e15) return fail(RC_ERR_UNSUPPORTED, "%s: too many rows to weigh", who);
    room = weigh_room(a.s);
  }
  const size_t need = parts && weights_out ? (size_t)up16((int64_t)parts) + (size_t)room.bytes() : parts + (size_t)room.bytes();
  if (need) {
    if (!workspace || workspace_bytes < need) return fail(RC_ERR_WORKSPACE, "%s: needs %zu bytes of workspace", who, need);
    if (!aligned16(workspace)) return fail(RC_ERR_WORKSPACE, "%s: workspace not 16-byte aligned", who);
  }
  a.k = (const char*)k, a.v = (const char*)v, a.tables = tables, a.ctx_len = ctx_len, a.q_start = q_start;
  a.q = (const char*)q, a.out = (char*)out, a.lse = lse;
  a.layer_stride_b = desc->layer_stride * 2, a.q_token_stride_b = q_token_stride * 2, a.q_layer_stride_b = q_layer_stride * 2;
  a.token_b = (uint32_t)desc->n_kv_heads * 256, a.block_b = a.token_b * (uint32_t)desc->block_tokens;
  a.n_blocks = n_blocks;
  a.borders = parts ? (AttendBorder*)workspace : nullptr;
  a.parts = parts ? (char*)workspace + attend_header_bytes(a.s.wgs) : nullptr;
  char* at = (char*)workspace + up16((int64_t)parts);
  a.ends = weights_out ? (float2*)at : nullptr;
  a.gathered = (f32x4*)(at + room.ends);
  a.runs = (int32_t)runs_of(a.s), a.kept_rows = (int32_t)a.s.max_q * a.s.g;
  g.sums = (float*)(at + room.ends + room.gathered);
  g.in = weights_in, g.out = empty ? nullptr : weights_out, g.tiles = a.runs * 2, g.shares = room.shares;
  if (desc->dtype == RC_BF16)
    kv_launch<true>(g, st);
  else
    kv_launch<false>(g, st);
  if (rc_status e = check_launch(who)) return e;
  return empty ? keep_weights() : RC_OK;
}
