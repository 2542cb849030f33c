// A paged cache of keys and values as gptaq_cache_append writes it and gptaq_attention reads it.
#pragma once
#include "common.h"

namespace gptaq {

// keys (pages, kv_heads, d / 8, page, 8), values (pages, kv_heads, page / 8, d, 8), both bf16: eight contraction elements (of a key's entries; of
// positions) are 16 bytes, so a lane's operand of a matrix instruction is one 16-byte load, lanes side by side read bytes side by side, and neither product
// needs a transposition.
struct CacheShape {
  const int32_t* table; int64_t ld_table; int32_t table_pages;      // pages of a sequence, in order; entries outside 0 .. pages - 1: no page there
  const int32_t *starts, *lengths;                                  // seqs + 1 first rows; tokens of each sequence, the new ones among them
  int32_t seqs, tokens, heads, kv_heads, group, d, page_bits;       // group: heads / kv_heads; a page has 1 << page_bits positions
  int64_t pages;
};
// A sequence's new tokens: rows first .. first + count - 1, positions before .. before + count - 1 (before may be negative where `lengths` says less than
// `starts`; positions below 0 are no tokens).  Whatever the arrays hold, rows stay inside the tensors and positions inside 31 bits.
struct Sequence { int32_t first, count, before; };
// What one address serves all lanes is read through the scalar cache (nothing of it changes while a kernel runs), and waited for apart from loads to LDS.
typedef const __attribute__((address_space(4))) int32_t* ConstantInts;
__device__ __forceinline__ ConstantInts cache_constant(const int32_t* p) { return (ConstantInts)(uintptr_t)p; }
__device__ __forceinline__ int cache_clamp(int v, int lo, int hi) { return v < lo ? lo : v > hi ? hi : v; }
__device__ __forceinline__ Sequence cache_sequence(const CacheShape& c, int s) {
  Sequence q;
  q.first = cache_clamp(cache_constant(c.starts)[s], 0, c.tokens);
  q.count = cache_clamp(cache_constant(c.starts)[s + 1], q.first, c.tokens) - q.first;
  q.before = cache_clamp(cache_constant(c.lengths)[s], 0, 1 << 30) - q.count;
  return q;
}
// Work is dealt out without the host knowing the lengths: with `units` pieces a token and 2^bits of them to a block, sequence s has the blocks from starts[s] units / 2^bits + s * extra
// on, which leaves each sequence room for ceil(count units / 2^bits) + extra - 1 at least.  This finds the sequence of a block: 64 are tried at a time, one a lane, so up to 64
// sequences are one load.
__device__ __forceinline__ int64_t cache_block_of(const CacheShape& c, int s, int units, int bits, int extra) {
  return (((int64_t)cache_clamp(c.starts[s], 0, c.tokens) * units) >> bits) + (int64_t)s * extra;
}
__device__ __forceinline__ int cache_find(const CacheShape& c, int64_t block, int units, int bits, int extra) {
  const int lane = threadIdx.x & 63;
  int lo = 0, n = c.seqs;
  while (n > 1) {
    const int step = (n + 63) >> 6, at = lane * step;
    const bool here = at < n && cache_block_of(c, lo + (at < n ? at : 0), units, bits, extra) <= block;
    const uint64_t mask = __ballot(here);
    const int k = mask ? 63 - __builtin_clzll(mask) : 0;
    lo += k * step;
    n = n - k * step < step ? n - k * step : step;
  }
  return __builtin_amdgcn_readfirstlane(lo);
}
// The same without gaps, for work that fills the GPU once or a few times: sequence s has ceil(rows / 2^bits) blocks of its count * group rows where these are more than `above` and at
// most `most`, and a block is found by sums over the lanes, each of which has a run of sequences; then over that lane's sequences.  Workgroup `at` of those that deal out blocks
// first .. first + n - 1, counted from the last block on, and `parts` parts of each: first parts before second ones, or, with a `target`, a block's side by side, as many as make no more than that
// together.  Behind them all come the workgroups that find nothing to do (block -1).  They go to the shader engines in turn, and between others they would leave CUs idle: two sequences' 16 tokens behind 16000, 64 heads over 8, 52 us with two of
// four blocks empty in every part, 32 this way.
struct Dealt { int32_t sequence, block, part, parts, index, all; };      // index: of all blocks
struct Deal { int32_t bits, above, most, parts, target; };
__device__ __forceinline__ int cache_parts(const Deal& d, int all) { return d.target ? max(1, min(d.parts, d.target / all)) : d.parts; }
__device__ __forceinline__ int64_t cache_blocks(const CacheShape& c, int s, const Deal& d) {
  const int first = cache_clamp(c.starts[s], 0, c.tokens), count = cache_clamp(c.starts[s + 1], first, c.tokens) - first;
  const int64_t rows = (int64_t)count * c.group;
  return rows > d.above && rows <= d.most ? (rows + (1 << d.bits) - 1) >> d.bits : 0;
}
__device__ __forceinline__ int cache_prefix(int v) {                 // sums over this lane and those below
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int d = 1; d < 64; d *= 2) {
    const int below = __shfl_up(v, d);
    v += lane >= d ? below : 0;
  }
  return v;
}
__device__ __forceinline__ Dealt cache_deal(const CacheShape& c, uint32_t at, int64_t first, int n, const Deal& d) {
  const int lane = threadIdx.x & 63, per = (c.seqs + 63) >> 6, mine0 = lane * per, mine1 = mine0 + per < c.seqs ? mine0 + per : c.seqs;
  int mine = 0;                                                      // (blocks are 2^23 at most; starts that do not ascend could say more than 31 bits)
  for (int s = mine0; s < mine1; ++s) mine = min(mine + (int)cache_blocks(c, s, d), 1 << 24);
  int sums = cache_prefix(mine);
  const int all = __builtin_amdgcn_readlane(sums, 63);
  const int here_all = (int)(all - first < n ? all - first : n);
  if (here_all <= 0) return Dealt{0, -1, 0, 0, 0, 0};
  const int parts = cache_parts(d, all);
  const uint32_t by = d.target ? (uint32_t)parts : (uint32_t)here_all, q = at / by, r = at - q * by;
  const int part = (int)(d.target ? r : q), which = (int)(d.target ? q : r);
  if (part >= parts || which >= here_all) return Dealt{0, -1, 0, 0, 0, 0};
  const int index = all - 1 - (int)(first + which);
  int block = index;
  uint64_t mask = __ballot(sums > block);
  int k = __builtin_ctzll(mask);
  block -= __builtin_amdgcn_readlane(sums, k) - __builtin_amdgcn_readlane(mine, k);
  int s0 = k * per;
  if (per > 1) {
    const int end = s0 + per < c.seqs ? s0 + per : c.seqs;
    for (;; s0 += 64) {                                              // (ends: the lane's sequences have the block among them)
      mine = s0 + lane < end ? (int)cache_blocks(c, s0 + lane, d) : 0;
      sums = cache_prefix(mine);
      const int here = __builtin_amdgcn_readlane(sums, 63);
      if (block < here || s0 + 64 >= end) break;
      block -= here;
    }
    mask = __ballot(sums > block);
    k = mask ? __builtin_ctzll(mask) : 63;
    block -= __builtin_amdgcn_readlane(sums, k) - __builtin_amdgcn_readlane(mine, k);
    s0 = s0 + k < end ? s0 + k : end - 1;
  }
  auto same = [](int v) { return __builtin_amdgcn_readfirstlane(v); };
  return Dealt{same(s0), same(block), same(part), same(parts), same(index), same(all)};
}
// The page of a position, or -1.
__device__ __forceinline__ int cache_page(const CacheShape& c, int s, int position) {
  const int at = position >> c.page_bits;
  if (at >= c.table_pages) return -1;
  const int id = cache_constant(c.table + s * c.ld_table)[at];
  return (uint32_t)id < (uint64_t)c.pages ? id : -1;
}

// What both calls refuse; fills `c`.
constexpr int64_t kMostSequences = 65536;
inline int cache_shape(CacheShape& c, const gptaq_cache* cache, int64_t tokens, int64_t heads) {
  if (!cache) return GPTAQ_ENULL;
  const auto [keys, values, pages, kv_heads, page, d, table, ld_table, table_pages, starts, lengths, seqs] = *cache;
  if (tokens != 0 && seqs != 0 && (!starts || !lengths || (table_pages != 0 && !table) || (pages != 0 && (!keys || !values)))) return GPTAQ_ENULL;
  if (((uintptr_t)keys | (uintptr_t)values) & 15) return GPTAQ_EDIM;
  if (seqs < 0 || seqs > kMostSequences || tokens < 0 || tokens > (1 << 24) || heads <= 0 || kv_heads <= 0 || heads > 4096 || heads % kv_heads || tokens * heads > (1 << 30) || pages < 0 ||
      pages > (1 << 30) || table_pages < 0 || ld_table < table_pages || (((uintptr_t)table | (uintptr_t)starts | (uintptr_t)lengths) & 3))
    return GPTAQ_EDIM;
  if (page < 16 || page > 256 || (page & (page - 1))) return GPTAQ_EUNSUPPORTED;
  if (table_pages > (((int64_t)1 << 30) / page)) return GPTAQ_EDIM;
  c.table = table; c.ld_table = ld_table; c.table_pages = (int32_t)table_pages;
  c.starts = starts; c.lengths = lengths;
  c.seqs = (int32_t)seqs; c.tokens = (int32_t)tokens; c.heads = (int32_t)heads; c.kv_heads = (int32_t)kv_heads; c.group = (int32_t)(heads / kv_heads);
  c.d = (int32_t)d; c.page_bits = __builtin_ctzll(page); c.pages = pages;
  return GPTAQ_OK;
}

// Whether the heads of an output's rows lie apart, in either order.
inline bool cache_rows_apart(int64_t tokens, int64_t ld, int64_t heads, int64_t h, int64_t d) {
  constexpr int64_t kMost = (int64_t)1 << 40;                        // (no stride of a real tensor)
  return ld >= 0 && h >= 0 && ld <= kMost && h <= kMost && (heads == 1 || h >= d) && (tokens <= 1 || ld >= d) &&
         (tokens <= 1 || heads == 1 || ld >= (heads - 1) * h + d || h >= (tokens - 1) * ld + d);
}

}  // namespace gptaq
