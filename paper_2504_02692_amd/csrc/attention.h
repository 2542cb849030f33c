// What the kernels of gptaq_attention share: which keys a row sees, how they are dealt out, and the arithmetic of a softmax taken in one pass.
#pragma once
#include "cache.h"

namespace gptaq {

// A row is a query: one head of one new token.  The rows of a sequence and a key head are numbered token by token, the `group` heads of a token that share the
// key head side by side, so that a block of rows reads its keys once for all of them.
struct AttentionArgs {
  CacheShape c;
  const uint16_t *q, *keys, *values; int64_t ldq, hq;
  uint16_t* out; int64_t ldo, ho;
  float scale;                         // times log2(e): exponentials are powers of two
  int32_t window, sinks;               // window 0: none
  int32_t parts;                       // the keys of a block of rows in so many parts at most, each of min_tiles tiles at least
  int32_t min_tiles, rows_bits;        // rows of a block (log2)
  int64_t first_block;
  int32_t mixed;                       // sequences of kFewMixed rows and fewer are taken by blocks of few rows, one a sequence, the others by blocks of many;
  int32_t target;                      // mixed, of few rows: so many blocks and parts together, where there are not more blocks
  float *partial, *stats;              // [part][row of the call][d], [part][row of the call][maximum, sum]; mixed, of few rows: [part][block][key head][row of 16]..
};

constexpr int kTile = 64;              // keys to a tile: what is dealt out
// Tiles that some row between positions pmin and pmax sees: 0 .. sink_tiles - 1, then first .. first + rest - 1.
struct Tiles {
  int32_t sink_tiles, first, count;
  __device__ __forceinline__ int at(int i) const { return i < sink_tiles ? i : first + i - sink_tiles; }
};
__device__ __forceinline__ Tiles attention_tiles(const AttentionArgs& a, int pmin, int pmax) {
  Tiles t{0, 0, 0};
  const int64_t room = (int64_t)a.c.table_pages << a.c.page_bits;
  if (pmax >= room) pmax = (int)room - 1;
  if (pmax < 0) return t;
  const int end = pmax / kTile + 1;
  if (a.window) {
    const int lo = pmin - a.window + 1;
    t.first = lo > 0 ? lo / kTile : 0;
    t.sink_tiles = a.sinks > 0 ? (a.sinks - 1) / kTile + 1 : 0;
    if (t.sink_tiles > t.first) t.sink_tiles = t.first;
  }
  t.count = t.sink_tiles + max(0, end - t.first);
  if (t.first > end) t.count = min(t.sink_tiles, end);
  return t;
}
// The token of a row that is the same in all lanes (a division is vector work).
__device__ __forceinline__ int at_token(int row, int group) { return __builtin_amdgcn_readfirstlane(row / group); }
// Tiles a part has, and how many parts there are.  Blocks of few rows have no more than 20 parts unless these have 20 tiles: joining more takes longer than they save.  us,
// one token, 64 heads over 8, with no such bound / with it: 8000 positions 15.6 / 14.6, 16000 23.2 / 19.7, 32000 33.2 / 29.7, 130000 107 / 107.
struct Parts { int32_t each, count; };
constexpr int kFewBits = 4, kFewMixed = 16;      // blocks of few rows have 16
__device__ __forceinline__ Deal attention_deal(const AttentionArgs& a) {
  const bool few = a.rows_bits == kFewBits;
  return Deal{a.rows_bits, a.mixed && !few ? kFewMixed : 0, a.mixed && few ? kFewMixed : 0x7fffffff, a.parts, a.target};
}
__device__ __forceinline__ Parts attention_parts(const AttentionArgs& a, int tiles, int parts) {
  const int least = a.rows_bits == kFewBits ? max(a.min_tiles, min(tiles / 20, 20)) : a.min_tiles;
  const int each = max(least, (tiles + parts - 1) / parts);
  return Parts{each, (tiles + each - 1) / each};
}

// A tile that some row does not see whole may hold anything where it is not seen, and a weight of zero lets an infinity or NaN through.  What lies behind the
// last position that a row sees, which nobody may have written, is taken for zeros.  Elsewhere such values are rare, so a block whose sums
// are not all finite takes them again with care: the values' entries that are not finite are taken out, and added to the rows that do see them from a second
// product, of marks: 1 for infinity, 2^7 for minus infinity, 2^14 for NaN, summed over at most 64 keys (exact).
__device__ __forceinline__ void attention_marks(u32x4& v, u32x4& marks) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    uint32_t clean = 0, mark = 0;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const uint32_t b = (v[i] >> (16 * h)) & 0xffffu;
      const uint32_t m = (b & 0x7f80u) != 0x7f80u ? 0u : (b & 0x7fu) ? 0x4680u : (b >> 15) ? 0x4300u : 0x3f80u;
      clean |= (m ? 0u : b) << (16 * h);
      mark |= m << (16 * h);
    }
    v[i] = clean;
    marks[i] = mark;
  }
}
__device__ __forceinline__ float attention_strange_sum(float count) {
  const int n = (int)count;
  if (n >> 14 || ((n & 127) && ((n >> 7) & 127))) return __builtin_nanf("");
  return (n & 127) ? __builtin_inff() : (n >> 7) ? -__builtin_inff() : 0.f;
}
__device__ __forceinline__ uint32_t at_bf16x2(float lo, float hi) {
  typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
  return __builtin_bit_cast(uint32_t, bf16x2{(__bf16)lo, (__bf16)hi});
}
__device__ __forceinline__ float at_exp2(float x) { return __builtin_amdgcn_exp2f(x); }
// The running maximum is raised only when a score passes it by 2^8: a softmax does not depend on what is taken off its exponents, and weights up to 256 times
// larger change no rounding of bf16 or fp32, so most tiles scale nothing.
constexpr float kSlack = 8.f;
// The score of a key that is not seen.  (One that is, with a score of minus infinity, has the same weight: none.)
constexpr float kUnseen = -__builtin_inff();
// A maximum to take off: rows that have seen nothing have none.
__device__ __forceinline__ float at_origin(float m) { return m == -__builtin_inff() ? 0.f : m; }

// What sums taken with the maximum `was` are multiplied by when it is `now`.  (Sums without a maximum are zero, or NaN.)
__device__ __forceinline__ float at_factor(float was, float now) { return was == -__builtin_inff() ? 1.f : at_exp2(was - now); }

// attention_many.hip: blocks of 32 kManyWaves rows, `blocks` of them (a.rows_bits is set).
constexpr int kManyWaves = 4, kManyBits = 7;
hipError_t launch_attention_many(const AttentionArgs& a, int64_t blocks, hipStream_t s);

}  // namespace gptaq
