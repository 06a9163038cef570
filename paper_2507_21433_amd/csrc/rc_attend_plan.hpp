// How the work of rc_cache_attend is cut into equal shares.  Plain C++ (host and device), so that the arithmetic can be checked
// where there is no GPU.
//
// The query tokens of a request times the query heads of one KV head are its rows, in tiles of `rows` rows.  An item is one row
// tile of one request and KV head of one layer; its work is the run of cached tokens that its rows see, in units of
// `unit` tokens.  All units of a call, item after item (layer, request, head, tile), are one line, and every workgroup
// takes an equal stretch of it, whatever the lengths of the requests are.  Where a stretch ends inside an item, the parts are
// joined by a second launch.
#pragma once
#include <cstddef>
#include <cstdint>
#include <initializer_list>

#ifdef __HIPCC__
#define RC_HD __host__ __device__
#else
#define RC_HD
#endif

namespace rc {

constexpr int kPairTokens = 32;  // what a wave takes at a time; items begin at a multiple of it

// The shape of a call, and of its kernel's tiles.
struct AttendShape {
  int64_t L, R, E;
  int32_t T, H, g;     // tokens of a block, KV heads, query heads of a KV head
  int32_t n_q, max_q;  // query tokens of a layer, of a request at most
  int32_t window;      // 0: none
  int32_t rows, unit;  // rows of a tile, tokens of a unit
  int32_t cap;         // positions of a table, E * T
  int32_t least;       // units of a stretch, at least; more than `free`
  int32_t free;        // units that an item costs whatever its length
  int32_t wgs;         // workgroups
  uint32_t inverse;    // n * inverse >> 16 is n / g for n below 32
  int32_t longest;     // units of a layer, at most
};

// A request's query tokens, row tiles and cached tokens, from what the device arrays hold (anything at all).
struct AttendRequest {
  int32_t first, len, rows, tiles, ctx;
};
RC_HD inline AttendRequest attend_request(const AttendShape& s, int32_t ctx, int32_t start, int32_t end) {
  AttendRequest q;
  q.first = start < 0 ? 0 : start > s.n_q ? s.n_q : start;
  const int32_t stop = end < q.first ? q.first : end > s.n_q ? s.n_q : end;
  q.len = stop - q.first;
  q.ctx = ctx < 0 ? 0 : ctx;
  // tokens beyond the longest that the host told of keep their places but are not computed
  q.rows = (q.len < s.max_q ? q.len : s.max_q) * s.g;
  q.tiles = (q.rows + s.rows - 1) / s.rows;
  return q;
}

// The cached tokens of a row tile.  Row n of a request is query token n / g, at position ctx - len + n / g.
struct AttendItem {
  int32_t pair0, pairs;      // first run of 32 tokens, number of runs
  int32_t free, units;       // units of the line: the first `free` of them stand for what an item costs whatever its length
  int32_t low_min, low_max;  // first position seen by the first and by the last row
  int32_t high_min, high_max;  // one past the last position seen by the first and by the last row
};
RC_HD inline int32_t attend_low(const AttendShape& s, int32_t pos) {
  return s.window && pos >= s.window ? pos - s.window + 1 : 0;
}
RC_HD inline int32_t attend_high(const AttendShape& s, int32_t pos) { return pos < 0 ? 0 : pos < s.cap ? pos + 1 : s.cap; }
// Of rows at positions p0 to p1.
RC_HD inline AttendItem attend_span(const AttendShape& s, int32_t p0, int32_t p1) {
  AttendItem i;
  i.low_min = attend_low(s, p0), i.low_max = attend_low(s, p1);
  i.high_min = attend_high(s, p0), i.high_max = attend_high(s, p1);
  i.pair0 = i.low_min / kPairTokens;
  const int32_t end = (int32_t)(((uint32_t)i.high_max + kPairTokens - 1) / kPairTokens);
  // (where a window lies behind the table's end, both may fall into the last run: it sees nothing all the same)
  i.pairs = i.high_max > i.low_min ? end - i.pair0 : 0;
  // an item that sees nothing has a unit as well: it still has to say so
  i.free = i.pairs ? s.free : 0;
  const uint32_t per = s.unit / kPairTokens;
  i.units = i.pairs ? i.free + (int32_t)((i.pairs + per - 1) / per) : 1;
  return i;
}
RC_HD inline AttendItem attend_item(const AttendShape& s, const AttendRequest& q, int32_t tile) {
  const int32_t n0 = tile * s.rows, n1 = (q.rows - n0 < s.rows ? q.rows : n0 + s.rows) - 1;
  return attend_span(s, q.ctx - q.len + n0 / s.g, q.ctx - q.len + n1 / s.g);
}
// The same where a request has one tile at most.
RC_HD inline AttendItem attend_only_item(const AttendShape& s, const AttendRequest& q) {
  const int32_t p0 = q.ctx - q.len;
  return attend_span(s, p0, p0 + (q.len < s.max_q ? q.len : s.max_q) - 1);
}

// Units of a request and KV head.
RC_HD inline int32_t attend_units(const AttendShape& s, const AttendRequest& q) {
  int32_t n = 0;
  for (int32_t t = 0; t < q.tiles; ++t) n += attend_item(s, q, t).units;
  return n;
}

// The runs of 32 tokens of the part of an item from unit u0 to u1 of its units: [first, last).  A stretch that ends among the free ones
// leaves the item to the next, which begins it then.
RC_HD inline int32_t attend_run(const AttendShape& s, const AttendItem& i, int32_t u) {
  const int64_t n = u > i.free ? (int64_t)(u - i.free) * (s.unit / kPairTokens) : 0;
  return i.pair0 + (n < i.pairs ? (int32_t)n : i.pairs);
}

// The line of units is counted in 32 bits, and has fewer than 2^30 of them: a layer's sums stay at that number, and a line that is longer is none
// (only starts of query tokens that do not ascend can make it so: attend_shape() has seen to the others).  So no count overflows, whatever the arrays
// hold.
constexpr int32_t kLongestLine = 1 << 30;
RC_HD inline int32_t attend_sum(int32_t a, int32_t b) {
  const uint32_t n = (uint32_t)a + (uint32_t)b;
  return n < (uint32_t)kLongestLine ? (int32_t)n : kLongestLine;
}
RC_HD inline int32_t attend_line(const AttendShape& s, int32_t total) { return total <= s.longest ? total * (int32_t)s.L : 0; }

// Units of a workgroup's stretch where there are `total` of them.
RC_HD inline int32_t attend_share(const AttendShape& s, int32_t total) {
  const int32_t n = (int32_t)((uint32_t)(total + s.wgs - 1) / (uint32_t)s.wgs);
  return n < s.least ? s.least : n;
}

// Where a part of an item that is cut is kept: two places per workgroup, one for the part that its stretch begins with, one for a
// part that begins later (and that the stretch then ends with).
RC_HD inline int64_t attend_place(int64_t wg, bool begins) { return 2 * wg + (begins ? 0 : 1); }

// What a workgroup says of the item that its stretch ends in: where it lies, and up to which workgroup its parts go, if the item begins
// in this stretch and goes on behind it (else last is -1).
struct AttendBorder {
  int32_t last, begins, l, h;
  int32_t row0, rows, first, unused;  // the row tile's first row and the request's rows, the request's first query token
};

// The workspace: a border per workgroup, then the parts, rows x (128 sums, reference, sum of weights) in fp32.
RC_HD inline size_t attend_header_bytes(int32_t wgs) { return (size_t)wgs * sizeof(AttendBorder); }
RC_HD inline size_t attend_part_bytes(int32_t rows) { return (size_t)rows * 130 * 4; }

// Tables of up to so many tokens: items are not cut, and no second launch joins them.  us, not cut -> cut: 64 requests of up to 1000 tokens
// 19.2 -> 21.3, one of 900 11.6 -> 13.9; of 2000: 8 requests 18.7 -> 15.8, 40 requests 26.9 -> 23.6.
constexpr int kWholeTokens = 1024;

struct AttendKernel {
  int32_t rows, unit, wgs, least, free;
};
// Kernels by the rows of a request and KV head (query tokens times heads of a KV head): tiles of 16 and 32 rows, where every wave
// of a workgroup has all rows and a quarter of the tokens, and of 64 and 128, where every wave has a quarter of the rows.  64 also for
// more rows where tiles of 128 would be few and their work small (`pairs` (layers, requests and heads) times `steps` of 64 tokens): more
// workgroups with less to do each.  us, tiles of 128 -> 64, by tiles times steps: 2000 29.8 -> 25.9, 4000 44.5 -> 37.5 (46.2 -> 40.4 and 52.8 -> 57.0 with 5 and
// 8 heads a KV head), 6000 47.6 -> 46.4, 50.1 -> 46.1 and 57.6 -> 64.4, 8000 51.5 -> 51.8 and 53.8 -> 52.0, 10000 58.1 -> 61.0, 16000 74.1 -> 84.1, 74.8 -> 84.8 and
// 98.1 -> 118.7; with more tiles, 192 of 1000 tokens 30.3 -> 30.2, 256 of 900 38.7 -> 46.0, 256 of 2000 53.2 -> 55.9.
// A stretch has `least` units at least (2, 4, 8 and 16 tried: one request of 4096 tokens 14.1, 13.4, 15.2 and 19.6), an item costs `free` units more
// than its tokens (0, 1 and 2: 40 requests of 2000 tokens 23.6, 23.6 and 22.3; drafts of 20 requests 33.7, 31.4 and 31.8).
inline AttendKernel attend_kernel(int64_t rows, double pairs, int64_t steps) {
  if (rows <= 16) return {16, 128, 768, 4, 2};
  if (rows <= 32) return {32, 128, 512, 4, 1};
  const double tiles = pairs * (double)((rows + 127) / 128);
  if (rows <= 64 || (tiles <= 128 && tiles * (double)steps <= 8192)) return {64, 64, 512, 8, 1};
  return {128, 64, 512, 8, 1};
}

// Most units of an item, whatever the lengths.
inline int64_t attend_most_units(const AttendShape& s) {
  const int64_t pairs = ((int64_t)s.cap + kPairTokens - 1) / kPairTokens, per = s.unit / kPairTokens;
  const int64_t n = (pairs + per - 1) / per;
  return n < 1 ? 1 : n + s.free;
}

constexpr int64_t kMostTokens = 0x7fffffffLL / 2;  // query tokens of a layer, and requests

// The shape of a call; false where it is beyond what the kernels count in 32 bits.
inline bool attend_shape(AttendShape* s, int64_t L, int64_t R, int64_t E, int32_t T, int32_t H, int32_t n_heads, int64_t n_q, int64_t max_q,
                         int64_t window) {
  const int32_t g = n_heads / H;
  if (max_q > n_q) max_q = n_q;
  if (E > (0x7fffffffLL - 64) / T || n_q > kMostTokens || R > kMostTokens || (max_q > 0 && max_q > 0x7fffff00LL / g)) return false;
  const AttendKernel k = attend_kernel(max_q * g, (double)L * R * H, E * T / 64);
  // a window longer than any position is none
  *s = {L, R, E, T, H, g, (int32_t)n_q, (int32_t)max_q, (int32_t)(window > 0x7fffffffLL ? 0 : window), k.rows, k.unit, (int32_t)(E * T), k.least, k.free, k.wgs,
        65536u / (uint32_t)g + 1, (int32_t)(L > 0 ? (kLongestLine - 1) / L : 0)};
  // a short table: items are not cut, and nothing has to be joined
  if (s->cap <= kWholeTokens) s->unit = (s->cap + k.unit - 1) / k.unit * k.unit + k.unit, s->least = 1, s->free = 0;
  // Row tiles of a layer and KV head: as many as every request's longest step has, but no more than all query tokens together fill (those of one
  // request of many tokens and of hundreds with one are far fewer than the first).  Tables long enough for more than 2^30 units have longer ones.
  const int64_t asked = R < n_q ? R : n_q;
  const double each = (double)asked * (double)((max_q * g + k.rows - 1) / k.rows), all = ((double)n_q * g + (double)asked * (k.rows - 1)) / k.rows;
  const double items = (double)L * H * (each < all ? each : all);
  if (items >= kLongestLine) return false;
  while (items * attend_most_units(*s) >= kLongestLine) {
    if (s->unit >= 1 << 29) return false;
    s->unit *= 2;
  }
  // no more workgroups than there can be stretches
  const double most = items * attend_most_units(*s) / s->least + 1;
  if (most < s->wgs) s->wgs = ((int32_t)most + 8) / 8 * 8;
  return true;
}
// Whether a call's tables can hold more than the last-level cache (256 MB on an MI355X) keeps from one pass over them to the next: its codes
// are then loaded without being kept.  us, kept -> not: 580 MB 118 -> 113, 416 MB 87.5 -> 84.7, 285 MB 62.7 -> 63.1, 160 MB 39.6 -> 43.3, 94 MB 35.3 -> 37.0.
inline bool attend_streams(const AttendShape& s) {
  const double seen = s.window && (double)s.window + s.max_q < s.cap ? (double)s.window + s.max_q : s.cap;
  return (double)s.L * s.R * s.H * seen * 136 > 384e6;
}
// Parts of a call, at most, and its workspace.
inline int64_t attend_most_parts(const AttendShape& s) { return attend_most_units(s) > 1 ? 2 * (int64_t)s.wgs : 0; }
inline size_t attend_workspace(const AttendShape& s) {
  const int64_t parts = attend_most_parts(s);
  return parts ? attend_header_bytes(s.wgs) + (size_t)parts * attend_part_bytes(s.rows) : 0;
}
// The workspace of calls of up to max_q query tokens a request, however many there are in all: the largest of the kernels that fewer of them would take
// as well.  Where so many requests of max_q tokens each are more than a call can have, calls of fewer tokens may have all workgroups.
inline size_t attend_largest_workspace(int64_t L, int64_t R, int64_t E, int32_t T, int32_t H, int32_t n_heads, int64_t max_q) {
  const int32_t g = n_heads / H;
  size_t most = 0;
  for (const int64_t rows : {(int64_t)16, (int64_t)32, (int64_t)64, max_q > kMostTokens ? kMostTokens * g : max_q * g}) {
    const int64_t q = rows / g;
    if ((q < 1 && max_q > 0) || q > max_q) continue;
    AttendShape s;
    size_t n;
    if (attend_shape(&s, L, R, E, T, H, n_heads, q && R > kMostTokens / q ? kMostTokens : R * q, q, 0)) {
      n = attend_workspace(s);
    } else {
      const AttendKernel k = attend_kernel(rows, 1e18, 1);
      n = attend_header_bytes(k.wgs) + 2 * (size_t)k.wgs * attend_part_bytes(k.rows);
    }
    if (n > most) most = n;
  }
  return most;
}

}  // namespace rc
