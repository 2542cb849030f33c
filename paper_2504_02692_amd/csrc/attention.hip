// Attention of new tokens over a paged cache: y_i = sum_j softmax_j(scale q_i k_j) v_j over the keys that token i sees, with an optional window and first
// tokens that stay visible.  In one pass over the keys, with the running maximum and sum of the softmax in fp32.
#include "attention.h"
#include <type_traits>

namespace gptaq {

// ---- few rows: a block is 16 rows (a step of decoding: the heads that share a key head).  Bound by memory: keys and values go from the cache straight to the
// registers of the lanes that feed v_mfma 16x16x32, and nothing is read twice.  Both products are taken transposed: S^T = K Q^T leaves a lane the scores of one
// row (l % 16), and O^T = V^T P^T takes them from there, with the keys in such an order that a lane's scores of 32 keys are what the second product wants of it: row
// 4 a + i of the first product's tile T has key 8 a + 4 T + i.  The four wavefronts of a block take 32 keys each in turn and join through LDS.
// Weights are rounded to bf16 for the second product (2^-9 each, as the output is once more); their sum is taken of the fp32 values.
// 64 sequences of up to 8192 positions, 64 heads over 8 of 128: 212 to 217 us, 5.3 TB/s, with two loads of 16 KB in flight a wavefront and two blocks a CU.  One of 2000 in a
// window of 1024: 7.6 to 8 us in 160 blocks, and 4.7 for the join.
template <int D>
__global__ __launch_bounds__(256, 2) void attention_few_kernel(AttentionArgs a) {
  constexpr int KS = D / 32, VT = D / 16, PAD = D + 4;
  __shared__ __attribute__((aligned(16))) float joined[4][16][PAD];
  __shared__ float maxima[4][16], sums[4][16];
  const CacheShape& c = a.c;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), l16 = lane & 15, quad = lane >> 4;
  const int head = (int)(blockIdx.x % (unsigned)c.kv_heads), rest = (int)(blockIdx.x / (unsigned)c.kv_heads);
  int part, s, parts_most = a.parts, index = 0, indexes = 0;
  int64_t in_seq;
  if (a.mixed) {
    const Dealt dealt = cache_deal(c, (uint32_t)(a.first_block + rest), 0, 0x7fffffff, attention_deal(a));
    if (dealt.block < 0) return;
    part = dealt.part, s = dealt.sequence, in_seq = 0, parts_most = dealt.parts, index = dealt.index, indexes = dealt.all;
  } else {
    part = rest % a.parts;
    const int64_t block = a.first_block + rest / a.parts;
    s = cache_find(c, block, c.group, 4, 1);
    in_seq = block - cache_block_of(c, s, c.group, 4, 1);
  }
  const Sequence seq = cache_sequence(c, s);
  const int rows = seq.count * c.group;
  if (in_seq < 0 || in_seq * 16 >= rows) return;
  const int row0 = (int)in_seq * 16, last = min(row0 + 15, rows - 1);
  const int pmin = seq.before + at_token(row0, c.group), pmax = seq.before + at_token(last, c.group);
  const Tiles tiles = attention_tiles(a, pmin, pmax);
  const Parts parts = attention_parts(a, tiles.count, parts_most);
  if (part > 0 && part >= parts.count) return;                       // (part 0 writes the zeros of rows that see nothing)
  const int begin = part * parts.each, end = min(begin + parts.each, tiles.count);

  const int row = min(row0 + l16, last), token = row / c.group, p_row = seq.before + token;
  const uint16_t* const qrow = a.q + (int64_t)(seq.first + token) * a.ldq + (int64_t)(head * c.group + row % c.group) * a.hq;
  typedef u32x4 __attribute__((aligned(2))) u32x4_at2;
  bf16x8 qf[KS];
#pragma unroll
  for (int i = 0; i < KS; ++i) qf[i] = __builtin_bit_cast(bf16x8, (u32x4) * reinterpret_cast<const u32x4_at2*>(qrow + i * 32 + quad * 8));

  const int page = 1 << c.page_bits;
  const int64_t head_elements = (int64_t)D << c.page_bits;           // of a page, of one head
  const int kslot = 8 * (l16 >> 2) + (l16 & 3);                      // key of 32 that lane has in tile 0 (4 more in tile 1)
  struct Stage { u32x4 k[2][KS], v[VT]; int j0; int ok; };          // ok: bit 0, 1: keys 0 .. 15, 16 .. 31 have a page
  auto load = [&](Stage& g, int step) {
    g.j0 = tiles.at(begin + (step >> 1)) * kTile + (step & 1) * 32;
    const int id0 = cache_page(c, s, g.j0), id1 = cache_page(c, s, g.j0 + 16);
    g.ok = (id0 >= 0 ? 1 : 0) | (id1 >= 0 ? 2 : 0);
    const int64_t at0 = ((int64_t)max(id0, 0) * c.kv_heads + head) * head_elements, at1 = ((int64_t)max(id1, 0) * c.kv_heads + head) * head_elements;
    const int off = g.j0 & (page - 1);
    const uint16_t* kfrom = a.keys + (l16 < 8 ? at0 : at1) + (((off + kslot) & (page - 1)) + quad * page) * 8;
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int i = 0; i < KS; ++i) g.k[t][i] = *reinterpret_cast<const u32x4*>(kfrom + t * 32 + i * 32 * page);
    const uint16_t* vfrom = a.values + (quad < 2 ? at0 : at1) + (int64_t)(((off + quad * 8) & (page - 1)) >> 3) * (D * 8) + l16 * 8;
#pragma unroll
    for (int i = 0; i < VT; ++i) g.v[i] = *reinterpret_cast<const u32x4*>(vfrom + i * 128);
  };

  f32x4 acc[VT];
  float top, total;                                                  // total: this lane's keys alone
  auto work = [&](auto careful, Stage& g) {
    constexpr bool CAREFUL = decltype(careful)::value;
    f32x4 sc[2] = {f32x4{0.f, 0.f, 0.f, 0.f}, f32x4{0.f, 0.f, 0.f, 0.f}};
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int i = 0; i < KS; ++i) sc[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, g.k[t][i]), qf[i], sc[t], 0, 0, 0);
    const bool whole = g.ok == 3 && g.j0 + 31 <= pmin && (a.window == 0 || g.j0 > pmax - a.window || g.j0 + 31 < a.sinks);
    float v[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = sc[e >> 2][e & 3] * a.scale;
    if (!whole) {
      const int j = g.j0 + quad * 8, after = a.window ? p_row - a.window - j : -1 << 30, sinks = a.sinks - j;
      const int until = (quad < 2 ? (g.ok & 1) : (g.ok & 2)) ? p_row - j : -1;
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = e <= until && (e > after || e < sinks) ? v[e] : kUnseen;
    }
    float most = fmaxf(fmaxf(fmaxf(v[0], v[1]), fmaxf(v[2], v[3])), fmaxf(fmaxf(v[4], v[5]), fmaxf(v[6], v[7])));
    if (__ballot(most > top + kSlack)) {
      most = fmaxf(most, __shfl_xor(most, 16));
      most = fmaxf(most, __shfl_xor(most, 32));
      const float now = fmaxf(top, most), factor = at_factor(top, now);
      top = now;
      total *= factor;
#pragma unroll
      for (int i = 0; i < VT; ++i) acc[i] *= factor;
    }
    const float from = at_origin(top);
    float w[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) { w[e] = at_exp2(v[e] - from); total += w[e]; }
    const u32x4 wp = {at_bf16x2(w[0], w[1]), at_bf16x2(w[2], w[3]), at_bf16x2(w[4], w[5]), at_bf16x2(w[6], w[7])};
    if (CAREFUL) {
      u32x4 ones;
#pragma unroll
      for (int i = 0; i < 4; ++i) ones[i] = (v[2 * i] != kUnseen ? 0x3f80u : 0u) | (v[2 * i + 1] != kUnseen ? 0x3f800000u : 0u);
#pragma unroll
      for (int i = 0; i < VT; ++i) {
        u32x4 marks;
        attention_marks(g.v[i], marks);
        const f32x4 n = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, marks), __builtin_bit_cast(bf16x8, ones), f32x4{0.f, 0.f, 0.f, 0.f}, 0, 0, 0);
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[i][e] += attention_strange_sum(n[e]);
      }
    } else if (g.j0 + 31 > pmax) {                                   // behind the last position that some row sees: zeros
      u32x4 ends;
#pragma unroll
      for (int h = 0; h < 4; ++h) {
        const int left = pmax - g.j0 - quad * 8 - 2 * h;
        ends[h] = left >= 1 ? ~0u : left == 0 ? 0xffffu : 0u;
      }
#pragma unroll
      for (int i = 0; i < VT; ++i) g.v[i] &= ends;
    }
#pragma unroll
    for (int i = 0; i < VT; ++i)
      acc[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, g.v[i]), __builtin_bit_cast(bf16x8, wp), acc[i], 0, 0, 0);
  };
  const int steps = 2 * max(0, end - begin);
  auto pass = [&](auto careful) {
#pragma unroll
    for (int i = 0; i < VT; ++i) acc[i] = f32x4{0.f, 0.f, 0.f, 0.f};
    top = -__builtin_inff();
    total = 0.f;
    Stage x, y;
    int step = wave;
    if (step < steps) load(x, step);
    if (decltype(careful)::value) {
#pragma unroll 1
      for (; step < steps; step += 4) {
        work(careful, x);
        if (step + 4 < steps) load(x, step + 4);
      }
      return;
    }
    for (; step < steps; step += 8) {
      if (step + 4 < steps) load(y, step + 4);
      work(careful, x);
      if (step + 8 < steps) load(x, step + 8);
      if (step + 4 < steps) work(careful, y);
    }
  };
  pass(std::false_type{});
  float bad = 0.f;                                                   // NaN if a sum is not finite
#pragma unroll
  for (int i = 0; i < VT; ++i)
#pragma unroll
    for (int e = 0; e < 4; ++e) bad = fmaf(acc[i][e], 0.f, bad);
  if (__ballot(bad != 0.f)) pass(std::true_type{});

  // ---- the wavefronts' sums: a lane has row l % 16, entries 16 i + 4 quad + e
  total += __shfl_xor(total, 16);
  total += __shfl_xor(total, 32);
  if (quad == 0) { maxima[wave][l16] = top; sums[wave][l16] = total; }
#pragma unroll
  for (int i = 0; i < VT; ++i) *reinterpret_cast<f32x4*>(&joined[wave][l16][i * 16 + quad * 4]) = acc[i];
  __syncthreads();
  const int r = threadIdx.x >> 4, e0 = threadIdx.x & 15;
  if (row0 + r > last) return;
  float m = maxima[0][r];
#pragma unroll
  for (int w = 1; w < 4; ++w) m = fmaxf(m, maxima[w][r]);
  float sum = 0.f, factor[4];
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    factor[w] = at_factor(maxima[w][r], m);
    sum += factor[w] * sums[w][r];
  }
  const int rr = row0 + r, tok = rr / c.group;
  const int64_t call_row = (int64_t)(seq.first + tok) * c.heads + head * c.group + rr % c.group;
  const float inv = sum == 0.f ? 0.f : 1.f / sum;
  uint16_t* const to = a.out + (int64_t)(seq.first + tok) * a.ldo + (int64_t)(head * c.group + rr % c.group) * a.ho;
  const int64_t part_row = a.mixed ? (((int64_t)part * indexes + index) * c.kv_heads + head) * kFewMixed + r : (int64_t)part * c.tokens * c.heads + call_row;
  float* const to_part = a.partial + part_row * D;
#pragma unroll
  for (int i = 0; i < D / 32; ++i) {
    const int e = i * 32 + e0 * 2;
    float o[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      o[h] = 0.f;
#pragma unroll
      for (int w = 0; w < 4; ++w) o[h] += factor[w] * joined[w][r][e + h];
    }
    if (parts.count > 1) {
      to_part[e] = o[0];
      to_part[e + 1] = o[1];
    } else {
      typedef uint32_t __attribute__((aligned(2))) u32_at2;
      *reinterpret_cast<u32_at2*>(to + e) = at_bf16x2(o[0] * inv, o[1] * inv);
    }
  }
  if (parts.count > 1 && e0 == 0) {
    float* st = a.stats + part_row * 2;
    st[0] = m;
    st[1] = sum;
  }
}

// The parts of a row, L lanes a row; a wavefront has 64 / L heads of a token.  Bound by the instructions of a row, and by latency where rows are few.  us, 64 / 32 / 16 lanes: 16384 rows of two
// parts 11.7 / 9.6 / 8.6, 32768 21.4 / 12.2 / 10.4; with the kernel before it, one token of 64 heads over 8 behind 8000 14.5 / 14.8 / 16.2, of 32 heads in a window of 1024 10.7 / 10.7 / 10.9.
template <int D, int L>
__global__ __launch_bounds__(256) void attention_join_kernel(AttentionArgs a, int64_t first, int64_t items) {
  const CacheShape& c = a.c;
  const int lane = threadIdx.x & 63, in_row = lane & (L - 1);
  const int64_t item = first + (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (item >= items) return;
  int s, token, h, parts_most = a.parts;
  int64_t row, step;                                                 // in the partial sums; from a part to the next
  if (a.mixed && a.rows_bits == kFewBits) {                          // 16 rows of each sequence and key head; rows are 2^30 at most
    constexpr uint32_t kItems = kFewMixed * L / 64;
    const uint32_t block = (uint32_t)item / kItems, head = block % (uint32_t)c.kv_heads;
    const int at = (int)((uint32_t)item % kItems) * (64 / L) + lane / L;
    const Deal deal = attention_deal(a);
    const Dealt dealt = cache_deal(c, block / (uint32_t)c.kv_heads, 0, 0x7fffffff, Deal{deal.bits, deal.above, deal.most, 1, 0});
    if (dealt.block < 0) return;
    s = dealt.sequence, parts_most = cache_parts(deal, dealt.all);
    token = at / c.group;
    h = (int)head * c.group + at % c.group;
    row = ((int64_t)dealt.index * c.kv_heads + head) * kFewMixed + at;
    step = (int64_t)dealt.all * c.kv_heads * kFewMixed;
  } else {                                                           // 64 / L heads of a token
    const uint32_t groups = (c.heads + 64 / L - 1) / (64 / L);
    token = (int)((uint32_t)item / groups);
    h = (int)((uint32_t)item % groups) * (64 / L) + lane / L;
    s = cache_find(c, token, 1, 0, 0);
    row = (int64_t)token * c.heads + h;
    step = (int64_t)c.tokens * c.heads;
  }
  const Sequence seq = cache_sequence(c, s);
  const int rows_seq = seq.count * c.group;
  if (a.mixed && a.rows_bits == kFewBits) token += seq.first;
  const int in_seq = token - seq.first;
  if (in_seq < 0 || in_seq >= seq.count || h >= c.heads) return;     // (no sequence's)
  if (a.mixed && (rows_seq <= kFewMixed) != (a.rows_bits == kFewBits)) return;
  // as the block of this row dealt its tiles out
  const int row0 = (in_seq * c.group + h % c.group) >> a.rows_bits << a.rows_bits;
  const int last = min(row0 + (1 << a.rows_bits) - 1, rows_seq - 1);
  const Parts parts = attention_parts(a, attention_tiles(a, seq.before + row0 / c.group, seq.before + last / c.group).count, parts_most);
  if (parts.count <= 1) return;
  // a lane has the statistics of every L-th part (there are 64 at most), and a share of every part's sums
  typedef __attribute__((ext_vector_type(2))) float f32x2;
  constexpr int S = 64 / L;
  f32x2 st[S];
  float m = -__builtin_inff(), sum = 0.f, mine[S];
#pragma unroll
  for (int k = 0; k < S; ++k) {
    st[k] = f32x2{-__builtin_inff(), 0.f};
    if (L * k + in_row < parts.count) st[k] = *reinterpret_cast<const f32x2*>(a.stats + ((L * k + in_row) * step + row) * 2);
    m = fmaxf(m, st[k][0]);
  }
#pragma unroll
  for (int k = 1; k < L; k *= 2) m = fmaxf(m, __shfl_xor(m, k));
#pragma unroll
  for (int k = 0; k < S; ++k) {
    mine[k] = L * k + in_row < parts.count ? at_factor(st[k][0], m) : 0.f;
    sum += mine[k] * st[k][1];
  }
#pragma unroll
  for (int k = 1; k < L; k *= 2) sum += __shfl_xor(sum, k);
  constexpr int E = D / L % 4 == 0 ? 4 : D / L % 2 == 0 ? 2 : 1, N = D / L / E;
  typedef __attribute__((ext_vector_type(E))) float Entries;
  Entries o[N];
#pragma unroll
  for (int k = 0; k < N; ++k) o[k] = Entries(0.f);
  const float* const from = a.partial + row * D + in_row * (D / L);
  auto add = [&](int count) {
    for (int i0 = 0; i0 < count; i0 += 8) {
      Entries v[8][N];
#pragma unroll
      for (int i = 0; i < 8; ++i)
#pragma unroll
        for (int k = 0; k < N; ++k)
          v[i][k] = i0 + i < count ? *reinterpret_cast<const Entries*>(from + (i0 + i) * step * D + E * k) : Entries(0.f);
      float factors = mine[0];
#pragma unroll
      for (int k = 1; k < S; ++k) factors = i0 >= L * k ? mine[k] : factors;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float factor = __shfl(factors, (lane & -L) + (i0 & (L - 1)) + i);
#pragma unroll
        for (int k = 0; k < N; ++k)
          if (i0 + i < count) o[k] += factor * v[i][k];
      }
    }
  };
  const int count = __builtin_amdgcn_readfirstlane(parts.count);      // (a token's heads mostly are of one block, or of blocks alike)
  if (__ballot(parts.count != count)) add(parts.count);
  else add(count);
  const float inv = sum == 0.f ? 0.f : 1.f / sum;
  uint16_t* const to = a.out + (int64_t)token * a.ldo + (int64_t)h * a.ho + in_row * (D / L);
  typedef uint32_t __attribute__((aligned(2))) u32_at2;
  float y[D / L];
#pragma unroll
  for (int k = 0; k < D / L; ++k) y[k] = ((const float*)o)[k] * inv;
  if (D / L % 2 == 0) {
#pragma unroll
    for (int k = 0; k < D / L; k += 2) *reinterpret_cast<u32_at2*>(to + k) = at_bf16x2(y[k], y[k + 1]);
  } else {
#pragma unroll
    for (int k = 0; k < D / L; ++k) to[k] = __builtin_bit_cast(uint16_t, (__bf16)y[k]);
  }
}

// ---- how a call is dealt out.  The host knows neither the lengths nor the tokens of a sequence, so it plans with what it knows: tokens, sequences, heads.
constexpr int64_t kMostParts = 64, kMostFewMixed = 32, kPartialRows = 65536, kFewMixedRows = 1024 * kFewMixed;
static int64_t attention_blocks(int64_t tokens, int64_t seqs, int64_t group, int bits) { return ((tokens * group) >> bits) + seqs; }
// Blocks of few rows read the keys once for 16 rows, and little else bounds them; blocks of many read them once for 128, and take longer to begin and end.
// So calls are of few as long as the tiles of their blocks, with nine for what a block costs besides, are kFewWork at most.
//   us a call of few / many, by rows of a sequence and key head (in brackets the number that the rule goes by):
//     32 heads behind 2000 positions           96 19.6 / 25.6 (8k)      256 25.8 / 32.5 (23k)    512 51 / 46 (50k)
//     32 heads behind none                     512 14.5 / 19 (17k)      768 23 / 24.5 (32k)
//     64 heads over 8 behind 8000              256 27.7 / 29.5 (17k)    384 47 / 35 (26k)
//     four sequences of these behind 4000      128 30 / 31 (18k)        256 44 / 41 (37k)
//     sixteen, 32 heads over 8 behind 2000     64 29.5 / 33.5 (21k)     96 45 / 37 (31k)
//     64 behind 500                            32 26 / 22 (17k)         48 37 / 24 (26k)
//     64 behind 8000, 64 heads over 8          16 324 / 301             32 408 / 319             96 724 / 342
// Tiles are those of the table: one much wider than the sequences are long plans for the longest that it has room for.  us a call in a graph, in a table of
// 512 positions (or 300) / of 128000: a prompt of 512, 32 heads 16.1 / 23.8; four of up to 300, 32 heads over 8 17.3 / 25.1.
//
// In calls of many, sequences of 16 rows at most (a step's tokens beside a prompt) are blocks of few all the same, dealt out by themselves, where there may be
// more than kMixedTiles tiles, which a block of many takes one after the other, and too few sequences to fill the chip that way.
//   us a call, 64 heads over 8, all in blocks of many / this way (steps and prompt in calls of their own):
//     7 tokens behind 32000 and 512 of a prompt       734 / 197 (175 and 20)
//     16 behind 8000 and 2048 behind 2048             393 / 320 (102 and 214)
//     31 behind 4000 and 512                          134 / 128
//     63 behind 4000 and 1000                         222 / 227
//     100 behind 1000 and 300                         91 / 102
//   Prompts alone take 3 to 5 us longer, for launches that find nothing.
constexpr int64_t kFewWork = 22000, kMixedTiles = 96, kMixedRows = 256;      // (kMixedRows: smaller calls need no room for both)
struct Plan { int bits; int64_t parts; int min_tiles; };
// Rows of a block, and parts of the keys.
// Blocks of many rows: the parts, of 8 tiles at least, that take the least time by what calls were measured to take: a tile 1.6 us where no CU has two blocks,
// 2.35 where all have; sums that are joined 3.5 us, and their rows' and bytes' time.
//   us a call, as many parts as make two blocks a CU / these:
//     three sequences of 256 tokens behind 600, 32 heads       37 (2) / 29 (1)
//     sixteen of 64 behind 2000, 32 heads over 8               60 (2) / 55 (1)
//     1024 tokens of 32 heads                                  41 (2) / 30 (1)
//     96 of 64 heads over 8 behind 8000                        47 / 47 (8)
// Blocks of few rows: for two a CU, of 4 tiles at least, or, which evens sequences of different lengths out, for eight a CU of 32 tiles at least.
//   us a call, room for 512 / 1024 / 2048 workgroups of 4 tiles:
//     64 heads over 8 of 128, 64 sequences of up to 1000       30.0 / 35.5 / 43.7 (those that find nothing to do take a microsecond, too)
//     64 of up to 8191                                         245 / 241 / 234
//     8 heads, 8 of up to 16000                                70.8 / 73.7 / 73.4
//   tiles at least, 2 / 4 / 9:
//     32 heads, one sequence of 200                            8.1 / 5.8 / 7.5
//     32 heads, a window of 1024                               11.4 / 10.7 / 12.9
//     64 heads over 8, one of 8000                             18.4 / 16.0 / 15.4
static Plan many_plan(int64_t blocks, int64_t rows, int64_t tiles, int64_t d) {
  int64_t best = 1;
  double least = 1e30;
  for (int64_t parts = 1; parts <= kMostParts && (parts == 1 || (parts * blocks <= 512 && tiles / parts >= 8)); ++parts) {
    const double each = (double)((tiles + parts - 1) / parts), groups = (double)(parts * blocks);
    const double us = (groups <= 256 ? 1.6 : groups <= 512 ? 2.35 : 2.35 * groups / 512) * each + (parts > 1 ? 3.5 + (double)rows * (2e-4 + (double)(parts * d) * 4 / 7.3e6) : 0);
    if (us < least) { least = us; best = parts; }
  }
  return Plan{kManyBits, best, 8};
}
static Plan few_plan(int64_t blocks, int64_t most_tiles) {
  int64_t parts = 512 / blocks, even = 2048 / blocks;
  if (parts > (most_tiles + 3) / 4) parts = (most_tiles + 3) / 4;
  if (even > most_tiles / 32) even = most_tiles / 32;
  if (parts < even) parts = even;
  return Plan{kFewBits, parts < 1 ? 1 : parts > kMostParts ? kMostParts : parts, 4};
}
static int64_t attention_blocks_of(int64_t tokens, int64_t seqs, int64_t group, int bits) {      // of sequences of one length
  const int64_t rows = (tokens * group - 1) / seqs + 1;
  return (((rows - 1) >> bits) + 1) * seqs;
}
// Room for the parts' sums: parts times blocks times their rows is 65536 at most, and parts are kMostParts at most; in calls that mix blocks, behind these the sums of blocks of few rows,
// of which there are 1024 at most where they have parts.  (More tokens never take less, so a workspace serves all smaller calls.)
static int64_t partial_rows(int64_t tokens, int64_t heads) {
  return (kMostParts * tokens * heads < kPartialRows ? kMostParts * tokens * heads : kPartialRows) + (tokens * heads > kMixedRows ? kFewMixedRows : 0);
}

template <int D>
static hipError_t launch_attention(const AttentionArgs& many, const AttentionArgs& few, hipStream_t s) {
  const CacheShape& c = many.c;
  const bool is_many = many.rows_bits == kManyBits, is_few = !is_many || many.mixed;
  if (is_many)
    if (const hipError_t e = launch_attention_many(many, attention_blocks(c.tokens, c.seqs, c.group, kManyBits), s); e != hipSuccess) return e;
  AttentionArgs a = few;
  // (mixed: of blocks and parts together)
  const int64_t blocks = !is_few ? 0 : a.mixed ? (c.seqs > a.target ? c.seqs : a.target) : attention_blocks(c.tokens, c.seqs, c.group, kFewBits);
  const int64_t each = (int64_t)(a.mixed ? 1 : a.parts) * c.kv_heads;
  const int64_t most = ((int64_t)1 << 23) / each;                    // (a grid has less than 2^32 threads)
  for (int64_t first = 0; first < blocks; first += most) {
    a.first_block = first;
    const int64_t n = blocks - first < most ? blocks - first : most;
    hipLaunchKernelGGL(attention_few_kernel<D>, dim3((unsigned)(n * each)), dim3(256), 0, s, a);
    if (const hipError_t e = hipGetLastError(); e != hipSuccess) return e;
  }
  constexpr int kLanes = 32;
  auto join = [&](const AttentionArgs& of, int64_t items) -> hipError_t {
    const int64_t each_launch = (int64_t)1 << 25;
    for (int64_t first = 0; first < items; first += each_launch) {
      const int64_t n = items - first < each_launch ? items - first : each_launch;
      hipLaunchKernelGGL((attention_join_kernel<D, kLanes>), dim3((unsigned)((n + 3) / 4)), dim3(256), 0, s, of, first, items);
      if (const hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    }
    return hipSuccess;
  };
  if (many.mixed && few.parts > 1)
    if (const hipError_t e = join(few, (int64_t)c.seqs * c.kv_heads * (kFewMixed * kLanes / 64)); e != hipSuccess) return e;
  return many.parts > 1 ? join(many, (int64_t)c.tokens * ((c.heads + 64 / kLanes - 1) / (64 / kLanes))) : hipSuccess;
}

static bool attention_size(int64_t tokens, int64_t seqs, int64_t heads, int64_t kv_heads, int64_t d) {
  return tokens >= 0 && tokens <= (1 << 24) && seqs >= 0 && seqs <= kMostSequences && heads > 0 && heads <= 4096 && tokens * heads <= (1 << 30) && kv_heads > 0 && heads % kv_heads == 0 &&
         (d == 64 || d == 96 || d == 128);
}

}  // namespace gptaq

using namespace gptaq;

extern "C" size_t gptaq_attention_workspace_bytes(int64_t tokens, int64_t seqs, int64_t heads, int64_t kv_heads, int64_t d) {
  if (!attention_size(tokens, seqs, heads, kv_heads, d) || tokens == 0 || seqs == 0) return 0;
  return ((size_t)partial_rows(tokens, heads) * (d + 2) * 4 + 255) / 256 * 256;
}

extern "C" int gptaq_attention(const uint16_t* q, int64_t ldq, int64_t hq, const gptaq_cache* cache, int64_t tokens, int64_t heads, int64_t window, int64_t sinks,
                               float scale, uint16_t* out, int64_t ldo, int64_t ho, void* ws, size_t ws_bytes, void* stream) {
  AttentionArgs a{};
  if (const int rc = cache_shape(a.c, cache, tokens, heads)) return rc;
  const int64_t d = cache->d, kv_heads = cache->kv_heads, seqs = cache->seqs;
  if (tokens != 0 && seqs != 0 && (!q || !out || !ws)) return GPTAQ_ENULL;
  if (d != 64 && d != 96 && d != 128) return GPTAQ_EUNSUPPORTED;
  if ((((uintptr_t)q | (uintptr_t)out) & 1) || ldq < 0 || hq < 0 || window < 0 || sinks < 0 ||
      !cache_rows_apart(tokens, ldo, heads, ho, d))
    return GPTAQ_EDIM;
  if (out == q && tokens != 0 && ((tokens > 1 && ldo != ldq) || (heads > 1 && ho != hq))) return GPTAQ_EUNSUPPORTED;
  const float scale2 = scale * 1.4426950408889634f;
  if (!(fabsf(scale2) < __builtin_inff())) return GPTAQ_EUNSUPPORTED;
  if (tokens == 0 || seqs == 0) return GPTAQ_OK;
  if (((uintptr_t)ws & 255) || ws_bytes < gptaq_attention_workspace_bytes(tokens, seqs, heads, kv_heads, d)) return GPTAQ_EWORKSPACE;
  constexpr int64_t kFar = (int64_t)1 << 30;                          // (positions are below this)
  a.q = q; a.keys = cache->keys; a.values = cache->values; a.ldq = ldq; a.hq = hq;
  a.out = out; a.ldo = ldo; a.ho = ho;
  a.scale = scale2;
  a.window = (int32_t)(window < kFar ? window : 0);
  a.sinks = (int32_t)(sinks < kFar ? sinks : kFar);
  // Tiles that a row can see: those of the table, or of the window (which begins and ends inside a tile, as the block's other rows have theirs) and the sinks.
  int64_t most_tiles = (cache->table_pages * cache->page + kTile - 1) / kTile;
  if (a.window && a.window / kTile + a.sinks / kTile + 4 < most_tiles) most_tiles = a.window / kTile + a.sinks / kTile + 4;
  if (cache->pages == 0) a.c.table_pages = 0;                                // no key anywhere: zeros
  // For all that is known here sequences may be of one length, or have a token each but for one.
  const int64_t group = heads / kv_heads, longest = (tokens > seqs ? tokens - seqs + 1 : 1) * group;
  int64_t blocks = longest > kFewMixed ? ((longest - 1) >> kFewBits) + 1 : 0;
  if (tokens * group > kFewMixed * seqs) { const int64_t like = attention_blocks_of(tokens, seqs, group, kFewBits); blocks = blocks > like ? blocks : like; }
  const bool many = blocks * kv_heads * (most_tiles + 9) > kFewWork;
  AttentionArgs f = a;
  auto take = [&](AttentionArgs& x, const Plan& plan, float* at, int64_t part_rows) {
    x.rows_bits = plan.bits; x.parts = (int32_t)plan.parts; x.min_tiles = plan.min_tiles;
    const int64_t sums = plan.parts > 1 ? plan.parts * part_rows : 0;
    x.partial = at;
    x.stats = at + sums * d;
    return at + (sums * (d + 2) + 3) / 4 * 4;                         // (vectors of four; a full workspace's sums are a multiple of four)
  };
  float* const at = (float*)ws;
  if (!many) {
    take(a, few_plan(attention_blocks_of(tokens, seqs, group, kFewBits) * kv_heads, most_tiles), at, tokens * heads);
    f = a;
  } else {
    a.mixed = f.mixed = seqs > 1 && most_tiles > kMixedTiles && most_tiles * 4 > seqs * kv_heads && tokens * heads > kMixedRows;
    float* const next = take(a, many_plan(attention_blocks_of(tokens, seqs, group, kManyBits) * kv_heads, tokens * heads, most_tiles, d), at, tokens * heads);
    if (a.mixed) {
      f.target = (int32_t)(kv_heads < 1024 ? 1024 / kv_heads : 1);   // four a CU: sequences' lengths differ
      int64_t parts = (most_tiles + 3) / 4;
      if (parts > kMostFewMixed) parts = kMostFewMixed;
      take(f, Plan{kFewBits, parts < 1 ? 1 : parts, 4}, next, 0);
      f.stats = f.partial + kFewMixedRows * d;
    } else {
      f = a;
    }
  }
  const hipError_t e = d == 64 ? launch_attention<64>(a, f, (hipStream_t)stream) : d == 96 ? launch_attention<96>(a, f, (hipStream_t)stream)
                                                                               : launch_attention<128>(a, f, (hipStream_t)stream);
  if (e != hipSuccess) { set_last_hip_error(e); return GPTAQ_ELAUNCH; }
  return GPTAQ_OK;
}
