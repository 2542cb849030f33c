// Attention over a paged cache for many rows: prompts, and pieces of prompts behind what the cache has of them.
#include "attention.h"
#include "linear.h"
#include <type_traits>

namespace gptaq {

// A block is 32 NW rows, NW wavefronts of 32 rows each.  Keys and values come in pieces of 32 (half a tile) straight from memory to LDS, as they lie in the pages, into a ring
// of kRing pieces with one barrier a piece.  Both products are taken transposed, with v_mfma 32x32x16: S^T = K Q^T leaves a lane the scores of one row (l % 32), and O^T = V^T P^T
// takes the weights from there without an exchange, if the first product's row 16 s + 8 b + 4 a + i has key 16 s + 8 a + 4 b + i (bits 2 and 3 change places).
// Reads of either from LDS are runs of 512 bytes: no bank is met twice.
// 2048 tokens behind 14336, 32 heads of 128: 528 us, 0.98 PFLOP/s; 8192 tokens, 64 heads over 8: 1.08 ms, 1.0; in a window of 2048, 32 heads: 314 to 323 us, of which a tenth is
// masked.  No unit is busy throughout: the matrix unit for 51 % of the cycles (48 behind 14336, 41 in the window), vector instructions issue in 40 to 45 %, LDS is read
// for a quarter, at a clock of 1.80 to 1.93 GHz.  Of a wavefront's time 46 % are its instructions, 27 to 30 % wait for a turn at a unit, and 23 to 28 % wait for loads, LDS or a
// barrier: it is the steps' own chain, two wavefronts a SIMD, at the clock that there is.  Two blocks of 128 rows share a CU, so that one works while the other begins, ends or waits; one block of 256 with pieces of 64 reads keys half as
// often, which takes 2 to 4 % off the largest calls, and adds 3 to 10 % to those in a window or of a few rounds (8192 tokens, window 2048: 296 / 306 us; 512 tokens
// of 32 heads 19 / 24; of 64 heads over 8 behind 8000, 40 / 58).
// PB: bits of a page as far as they matter to a piece's layout (4, 5: pages of 16, and more).
constexpr int kRing = 4, kPiece = 32;                  // (five, with two pieces in flight: the same times)
template <int D, int NW> struct ManyShape {
  static constexpr int kPieceBytes = kPiece * D * 2, kLoads = kPieceBytes / 1024;      // of keys, or of values
  static constexpr int kPerWave = 2 * kLoads / NW;
  static constexpr int kOutRow = D * 2 + 16;                                        // results in LDS
  static constexpr int kRingBytes = kRing * 2 * kPieceBytes, kOutBytes = 32 * NW * kOutRow;
  static constexpr int kLds = kRingBytes > kOutBytes ? kRingBytes : kOutBytes;
  static_assert(2 * kLoads % NW == 0, "every wavefront has as many loads");
};
__device__ __forceinline__ void am_barrier() {            // no memory fence: loads stay in flight across it
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}
template <int N> __device__ __forceinline__ void am_wait() {        // vmcnt <= N, lgkmcnt == 0
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt((N & 15) | ((N >> 4) << 14) | (7 << 4));
  asm volatile("" ::: "memory");
}

// No finite score is lower than this; with it as the origin every weight of one that is not as low is infinite.  A step's 16 weights of a lane may sum up to 2^12: a softmax does not depend on its origin,
// and weights that much larger change no rounding of bf16 or fp32.
constexpr float kNoOrigin = -3.402823466e38f, kMostSum = 4096.f;

template <int D, int PB, int NW>
__global__ __launch_bounds__(64 * NW, 2) void attention_many_kernel(AttentionArgs a, int blocks) {
  using Shape = ManyShape<D, NW>;
  extern __shared__ __attribute__((aligned(256))) unsigned char smem[];
  constexpr int KS = D / 16, VT = D / 32, P = 1 << PB, PIECE = Shape::kPieceBytes;
  const CacheShape& c = a.c;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), l32 = lane & 31, half = lane >> 5;
  // The heads of a block side by side, so that with eight key heads each XCD has one; late blocks first, which see the most.
  const int head = (int)(blockIdx.x % (unsigned)c.kv_heads), rest = (int)(blockIdx.x / (unsigned)c.kv_heads);
  const Dealt dealt = cache_deal(c, rest, a.first_block, blocks, attention_deal(a));
  if (dealt.block < 0) return;
  const int s = dealt.sequence, part = dealt.part;
  const Sequence seq = cache_sequence(c, s);
  const int rows = seq.count * c.group;
  if (((int64_t)dealt.block << a.rows_bits) >= rows) return;         // (starts that do not ascend)
  const int row0 = dealt.block << a.rows_bits, last = min(row0 + 32 * NW - 1, rows - 1);
  const Tiles tiles = attention_tiles(a, seq.before + at_token(row0, c.group), seq.before + at_token(last, c.group));
  const Parts parts = attention_parts(a, tiles.count, a.parts);
  if (part > 0 && part >= parts.count) return;                       // (part 0 writes the zeros of rows that see nothing)
  const int begin = part * parts.each, end = min(begin + parts.each, tiles.count);

  // the wavefront's rows
  const int wave0 = row0 + wave * 32, wave1 = min(wave0 + 31, last);
  const bool idle = wave0 > last;
  const int row = min(wave0 + l32, last), token = row / c.group, p_row = seq.before + token;
  const int pmin = seq.before + at_token(min(wave0, last), c.group), pmax = idle ? -1 : seq.before + at_token(wave1, c.group);
  const uint16_t* const qrow = a.q + (int64_t)(seq.first + token) * a.ldq + (int64_t)(head * c.group + row % c.group) * a.hq;
  typedef u32x4 __attribute__((aligned(2))) u32x4_at2;
  // (A negative scale goes to the queries' signs, so that the largest score is that of the largest product.)
  const uint32_t flip = a.scale < 0.f ? 0x80008000u : 0u;
  const float scale = fabsf(a.scale);
  bf16x8 qf[KS];
#pragma unroll
  for (int i = 0; i < KS; ++i) qf[i] = __builtin_bit_cast(bf16x8, *reinterpret_cast<const u32x4_at2*>(qrow + i * 16 + half * 8) ^ flip);

  // ---- loads: a piece's keys, then its values, 1 KB each; a wavefront's are neighbours.  Of a page of up to 32 positions they are one run, of a larger one the keys' are
  // two rows of 32 positions each.
  constexpr int PAGES = PB == 4 ? 4 : 2, PER = Shape::kLoads * 2 / PAGES;      // pages of a tile (that of each half of it at least), loads of a page
  const int64_t head_bytes = (int64_t)(D * 2) << c.page_bits;        // of a page, of one head
  const int64_t page_bytes = head_bytes * c.kv_heads;
  static_assert(PER % Shape::kPerWave == 0, "a wavefront's loads of a piece are of one page");
  const int first_load = wave * Shape::kPerWave;                     // keys' loads, then values'
  const bool loads_values = first_load >= Shape::kLoads;
  const int load0 = loads_values ? first_load - Shape::kLoads : first_load, own_page = load0 / PER;
  const unsigned char* const base = (const unsigned char*)(loads_values ? a.values : a.keys) + head * head_bytes;
  const int load_step = loads_values || PB < 5 ? 1024 : 32 << c.page_bits, load_from = load0 % PER * load_step;      // from one load of a page to the next
  const int load_lane = loads_values || PB < 5 ? lane * 16 : l32 * 16 + half * (16 << c.page_bits);
  const int place_bytes = loads_values ? D * 2 : 16, off_mask = (1 << c.page_bits) - 1;
  const int last_tile = tiles.at(max(end - 1, 0));
  auto tile_of = [&](int i) { return i < end ? tiles.at(i) : last_tile; };      // (behind the last that again)
  struct Ids { int page[2], there; };                                // of a tile: the wavefront's own page of either half, a bit for each that there is
  // A tile's pages are asked for a tile before its loads, lane k for the k-th, by a vector load: what waits for it waits for what was asked for before it alone.
  auto ask_pages = [&](int tile) {
    const int at = (tile * kTile + lane % PAGES * (kTile / PAGES)) >> c.page_bits;
    return at < c.table_pages ? c.table[(int64_t)s * c.ld_table + at] : -1;
  };
  auto pages_of = [&](Ids& g, int asked) {
    const bool there = (uint32_t)asked < (uint32_t)c.pages;
    g.there = (int)(__ballot(there) & ((1 << PAGES) - 1));
    g.page[0] = __builtin_amdgcn_readlane(there ? asked : 0, own_page);
    g.page[1] = __builtin_amdgcn_readlane(there ? asked : 0, own_page + PAGES / 2);
  };
  auto load_piece = [&](const Ids& g, int tile, int b, int slot) {
    const int from = load_from + (PB < 5 ? 0 : ((tile * kTile + b * kPiece) & off_mask) * place_bytes);
    unsigned char* const to = smem + slot * 2 * PIECE + first_load * 1024;
    const LdsLoader loader(base + g.page[b] * page_bytes);
#pragma unroll
    for (int n = 0; n < Shape::kPerWave; ++n) loader.load(to + n * 1024, load_lane, from + n * load_step);
  };
  auto valid = [&](const Ids& g) { return PAGES == 4 ? g.there : (g.there & 1) * 3 | (g.there >> 1) * 12; };      // a bit for each 16 keys

  f32x16 acc[VT];
#pragma unroll
  for (int i = 0; i < VT; ++i)
#pragma unroll
    for (int e = 0; e < 16; ++e) acc[i][e] = 0.f;
  float origin = kNoOrigin, total = 0.f;                             // what is taken off scaled scores; total: this lane's keys alone
  const int key = (l32 & 0x13) | (l32 & 4) << 1 | (l32 & 8) >> 1;    // of 32 that the lane reads
  const int kread = (key >> PB) * (D * 2 * P) + (key & (P - 1)) * 16 + half * P * 16, vread = PIECE + (half * D + l32) * 16;

  // The weights of a step's scores are taken with the origin as it is.  Where their sum says that some score is far above it (or that there is none yet, which
  // makes every weight infinite), the origin becomes the largest score so far, sums are to be scaled by `factor`, and the weights are taken again.
  // `seen`: a bit for each of the lane's 16 keys, at the key's place in 24.
  auto place = [](int e) { return 16 * (e >> 3) + (e & 7); };
  auto only = [&](float w, uint32_t seen, int e) { return __uint_as_float(__float_as_uint(w) & (uint32_t)((int32_t)(seen << (31 - place(e))) >> 31)); };
  auto seen_of = [&](int j) {                                        // j: the first of the lane's keys
    auto first = [](int n) { return (1u << cache_clamp(n, 0, 24)) - 1u; };
    const int p = p_row - j;
    return first(p + 1) & (a.window ? ~first(p - a.window + 1) | first(a.sinks - j) : ~0u);
  };
  float factor = 1.f;
  auto raise = [&](const f32x16& now, float (&w)[16], float& sum, uint32_t seen) {
    if (!__ballot(sum > kMostSum)) return false;
    float most = kUnseen;
#pragma unroll
    for (int e = 0; e < 16; ++e) most = fmaxf(most, seen >> place(e) & 1 ? now[e] : kUnseen);
    most = most == kUnseen ? kUnseen : most * scale;                 // (a scale of 0 would make NaN of it)
    most = fmaxf(most, __shfl_xor(most, 32));
    if (most == kUnseen) most = kNoOrigin;
    const float to = fmaxf(origin, most);
    factor = origin == kNoOrigin ? 1.f : at_exp2(origin - to);       // (sums without an origin are zero, or NaN)
    origin = to;
    total *= factor;
    sum = 0.f;
#pragma unroll
    for (int e = 0; e < 16; ++e) { w[e] = only(at_exp2(fmaf(now[e], scale, -origin)), seen, e); sum += w[e]; }
    return true;
  };
  auto scale_sums = [&]() {
#pragma unroll
    for (int t = 0; t < VT; ++t) acc[t] *= factor;
  };
  auto pack = [&](const float* w) {
    return __builtin_bit_cast(bf16x8, u32x4{at_bf16x2(w[0], w[1]), at_bf16x2(w[2], w[3]), at_bf16x2(w[4], w[5]), at_bf16x2(w[6], w[7])});
  };
  auto keys_of = [&](const unsigned char* at, int k) { return *reinterpret_cast<const bf16x8*>(at + kread + k * (2 * P * 16)); };
  auto values_of = [&](const unsigned char* at, int h16, int t) { return *reinterpret_cast<const u32x4*>(at + vread + (h16 * 2 * D + t * 32) * 16); };
  f32x16 sc[2];                                                      // scores of 32 keys; element e: key 16 (e / 8) + 8 half + e % 8
  bf16x8 weight[2][2];                                               // [step & 1][16 keys]
  // A piece of a tile of which parts are not there; what is behind the last position that some row sees is taken for zeros.  CAREFUL (see
  // attention_marks) takes any piece, and every sum in the same order as where it is not needed.
  auto work = [&](auto careful, const unsigned char* at_piece, int j0, int ok) {
    constexpr bool CAREFUL = decltype(careful)::value;
    f32x16& s32 = sc[0];
#pragma unroll
    for (int e = 0; e < 16; ++e) s32[e] = 0.f;
#pragma unroll
    for (int k = 0; k < KS; ++k) s32 = __builtin_amdgcn_mfma_f32_32x32x16_bf16(keys_of(at_piece, k), qf[k], s32, 0, 0, 0);
    const int j = j0 + 8 * half;
    const uint32_t seen = seen_of(j) & ((ok & 1 ? 0xffu : 0u) | (ok & 2 ? 0xff0000u : 0u));
    float w[16], sum = 0.f;
#pragma unroll
    for (int e = 0; e < 16; ++e) { w[e] = only(at_exp2(fmaf(s32[e], scale, -origin)), seen, e); sum += w[e]; }
    if (raise(s32, w, sum, seen)) scale_sums();
    total += sum;
#pragma unroll
    for (int h16 = 0; h16 < 2; ++h16) {
      weight[1][h16] = pack(w + 8 * h16);
      u32x4 ones, ends;
#pragma unroll
      for (int h = 0; h < 4; ++h) {
        const int at = 8 * h16 + 2 * h, left = pmax - j - 16 * h16 - 2 * h;      // keys of the lane's pair that are not behind the last
        if (CAREFUL) ones[h] = (seen >> place(at) & 1 ? 0x3f80u : 0u) | (seen >> place(at + 1) & 1 ? 0x3f800000u : 0u);
        ends[h] = left >= 1 ? ~0u : left == 0 ? 0xffffu : 0u;
      }
#pragma unroll
      for (int t = 0; t < VT; ++t) {
        u32x4 v = values_of(at_piece, h16, t);
        if (CAREFUL) {
          u32x4 marks;
          attention_marks(v, marks);
          f32x16 n;
#pragma unroll
          for (int e = 0; e < 16; ++e) n[e] = 0.f;
          n = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, marks), __builtin_bit_cast(bf16x8, ones), n, 0, 0, 0);
#pragma unroll
          for (int e = 0; e < 16; ++e) acc[t][e] += attention_strange_sum(n[e]);
        } else if (j0 + kPiece > pmax) {
          v &= ends;
        }
        acc[t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, v), weight[1][h16], acc[t], 0, 0, 0);
      }
    }
  };

  // All other tiles go through in steps of 32 keys, each with three parts that do not wait for each other: the next step's scores, this one's
  // weights, and the product of the last one's weights with its values.  So the matrix unit works while the vector unit takes exponentials.  Groups of one
  // instruction of either product, the reads of the group after the next, and the group's share of the weights; the barriers keep the compiler to this order.
  auto scores_alone = [&](f32x16& next, const unsigned char* at) {
#pragma unroll
    for (int e = 0; e < 16; ++e) next[e] = 0.f;
#pragma unroll
    for (int k = 0; k < KS; ++k) next = __builtin_amdgcn_mfma_f32_32x32x16_bf16(keys_of(at, k), qf[k], next, 0, 0, 0);
  };
  auto product_alone = [&](const bf16x8 (&w)[2], const unsigned char* at) {
#pragma unroll
    for (int k = 0; k < KS; ++k)
      acc[k % VT] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, values_of(at, k / VT, k % VT)), w[k / VT], acc[k % VT], 0, 0, 0);
  };
  auto step = [&](const f32x16& now, f32x16& next, const unsigned char* at_next, const bf16x8 (&before)[2], const unsigned char* at_before, bf16x8 (&packed)[2],
                  bool parts_seen, int j) {
    constexpr int AHEAD = 2;
    u32x4 kf[AHEAD + 1], vf[AHEAD + 1];
    auto read = [&](int k) {
      kf[k % (AHEAD + 1)] = __builtin_bit_cast(u32x4, keys_of(at_next, k));
      vf[k % (AHEAD + 1)] = values_of(at_before, k / VT, k % VT);
    };
#pragma unroll
    for (int k = 0; k < AHEAD; ++k) read(k);
    float w[16], sum = 0.f;
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int k = 0; k < KS; ++k) {
      if (k + AHEAD < KS) read(k + AHEAD);
      const f32x16 zero = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
      next = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, kf[k % (AHEAD + 1)]), qf[k], k == 0 ? zero : next, 0, 0, 0);
#pragma unroll
      for (int e = k * 16 / KS; e < (k + 1) * 16 / KS; ++e) {
        w[e] = at_exp2(fmaf(now[e], scale, -origin));
        sum += w[e];
        asm volatile("" : "+v"(w[e]), "+v"(sum));                    // (here, not behind the products)
      }
      acc[k % VT] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, vf[k % (AHEAD + 1)]), before[k / VT], acc[k % VT], 0, 0, 0);
      __builtin_amdgcn_sched_barrier(0);
    }
    uint32_t seen = ~0u;
    if (parts_seen) {
      seen = seen_of(j);
      sum = 0.f;
#pragma unroll
      for (int e = 0; e < 16; ++e) { w[e] = only(w[e], seen, e); sum += w[e]; }
    }
    if (raise(now, w, sum, seen)) scale_sums();
    total += sum;
#pragma unroll
    for (int h = 0; h < 2; ++h) packed[h] = pack(w + 8 * h);
  };

  // Tiles of which the wavefront's rows see something are seen_from .. seen_to and those below seen_sinks; tiles that all of them see whole likewise.
  const int seen_to = pmax >> 6, seen_from = a.window ? max(pmin - a.window + 1, 0) >> 6 : 0, seen_sinks = a.window ? (a.sinks + kTile - 1) / kTile : 0;
  const int whole_to = ((pmin + 1) >> 6) - 1, whole_from = a.window ? (max(pmax - a.window + 1, 0) + kTile - 1) >> 6 : 0, whole_sinks = a.window ? a.sinks / kTile : 0;
  enum { kNothing, kOdd, kParts, kWhole };                           // kOdd: some of it is not there, or behind the sequence's end
  const int end_tile = (seq.before + seq.count) >> 6;
  auto kind_of = [&](const Ids& g, int tile) {
    const bool some = tile <= seen_to && (tile >= seen_from || tile < seen_sinks);
    const bool all = tile <= whole_to && (tile >= whole_from || tile < whole_sinks);
    return idle || !some ? kNothing : valid(g) != 15 || tile >= end_tile ? kOdd : all ? kWhole : kParts;
  };
  auto pass = [&](auto careful) {
    constexpr bool CAREFUL = decltype(careful)::value;
    Ids ids[3];                                                      // pages of tiles i .. i + 2
    int i = begin, slot = 0, tile[3], asked[3];                      // slot: of the piece
    auto slot_of = [&](int ahead) { return (slot + ahead) % kRing; };
    auto at_slot = [&](int ahead) { return smem + slot_of(ahead) * 2 * PIECE; };
#pragma unroll
    for (int k = 0; k < 3; ++k) {
      tile[k] = tile_of(i + k);
      asked[k] = ask_pages(tile[k]);
    }
    pages_of(ids[0], asked[0]);
    pages_of(ids[1], asked[1]);
    __builtin_amdgcn_sched_barrier(0);
    load_piece(ids[0], tile[0], 0, 0);
    load_piece(ids[0], tile[0], 1, 1);
    auto top_of = [&](int b) {                                       // before half b of tile i
      am_wait<0>();                                                  // the wavefront's loads of the next piece are there ..
      am_barrier();                                                  // .. and everyone's; and the piece before the last is no longer read
      if (b == 1) {
        pages_of(ids[2], asked[2]);
        asked[2] = ask_pages(tile_of(i + 3));
        __builtin_amdgcn_sched_barrier(0);
      }
      load_piece(ids[1], tile[1], b, slot_of(2));
      __builtin_amdgcn_sched_barrier(0);
    };
    auto middle = [&]() {
      slot = slot_of(1);
      top_of(1);
    };
    auto advance = [&]() {
      ++i;
      slot = slot_of(1);
#pragma unroll
      for (int k = 0; k < 2; ++k) { ids[k] = ids[k + 1]; tile[k] = tile[k + 1]; }
      tile[2] = tile_of(i + 2);
      if (i < end) top_of(0);
    };
    top_of(0);
    while (i < end) {
      int kind = __builtin_amdgcn_readfirstlane(kind_of(ids[0], tile[0]));
      if (!CAREFUL && kind >= kParts) {
        const unsigned char* before = at_slot(0);                    // (the first product is with weights of zero)
        scores_alone(sc[0], before);
        weight[1][0] = weight[1][1] = bf16x8{};
        for (;;) {
          const int j = tile[0] * kTile + 8 * half;
          step(sc[0], sc[1], at_slot(1), weight[1], before, weight[0], kind == kParts, j);
          before = at_slot(0);
          middle();
          step(sc[1], sc[0], at_slot(1), weight[0], before, weight[1], kind == kParts, j + 32);
          before = at_slot(0);
          kind = i + 1 < end ? __builtin_amdgcn_readfirstlane(kind_of(ids[1], tile[1])) : kNothing;
          if (kind < kParts) break;
          advance();
        }
        product_alone(weight[1], before);
      } else {
#pragma unroll 1
        for (int b = 0;; ++b) {
          if (kind != kNothing) work(careful, at_slot(0), tile[0] * kTile + b * kPiece, valid(ids[0]) >> (2 * b));
          if (b == 1) break;
          middle();
        }
      }
      advance();
    }
    am_wait<0>();                                                    // (no load writes to LDS from here on)
  };
  if (begin < end) {
    pass(std::false_type{});
    float bad = 0.f;                                                 // NaN if a sum is not finite
#pragma unroll
    for (int t = 0; t < VT; ++t)
#pragma unroll
      for (int e = 0; e < 16; ++e) bad = fmaf(acc[t][e], 0.f, bad);
    // (All of LDS is the ring's.)
    int* const again = reinterpret_cast<int*>(smem);
    __syncthreads();
    if (threadIdx.x == 0) *again = 0;
    __syncthreads();
    if (bad != 0.f) *again = 1;
    __syncthreads();
    const bool careful = *again != 0;
    __syncthreads();
    if (careful) {
#pragma unroll
      for (int t = 0; t < VT; ++t)
#pragma unroll
        for (int e = 0; e < 16; ++e) acc[t][e] = 0.f;
      origin = kNoOrigin;
      total = 0.f;
      pass(std::true_type{});
      __syncthreads();
    }
  }
  if (idle) return;

  // ---- results: a lane has row l % 32, entries 32 t + 8 (e / 4) + 4 half + e % 4
  total += __shfl_xor(total, 32);
  const int64_t rows_call = (int64_t)c.tokens * c.heads;
  if (parts.count > 1) {
    if (wave0 + l32 > last) return;
    const int64_t call_row = part * rows_call + (int64_t)(seq.first + token) * c.heads + head * c.group + row % c.group;
    float* const to = a.partial + call_row * D;
#pragma unroll
    for (int t = 0; t < VT; ++t)
#pragma unroll
      for (int e = 0; e < 16; e += 4)
        *reinterpret_cast<f32x4*>(to + 32 * t + 2 * e + 4 * half) = f32x4{acc[t][e], acc[t][e + 1], acc[t][e + 2], acc[t][e + 3]};
    if (half == 0) { a.stats[call_row * 2] = origin == kNoOrigin ? -__builtin_inff() : origin; a.stats[call_row * 2 + 1] = total; }
    return;
  }
  // through the wavefront's own rows of LDS, so that a row leaves in one run
  typedef __attribute__((ext_vector_type(2))) uint32_t u32x2;
  const float inv = total == 0.f ? 0.f : 1.f / total;
  unsigned char* const own = smem + wave * 32 * Shape::kOutRow;
#pragma unroll
  for (int t = 0; t < VT; ++t)
#pragma unroll
    for (int e = 0; e < 16; e += 4)
      *reinterpret_cast<u32x2*>(own + l32 * Shape::kOutRow + (32 * t + 2 * e + 4 * half) * 2) =
          u32x2{at_bf16x2(acc[t][e] * inv, acc[t][e + 1] * inv), at_bf16x2(acc[t][e + 2] * inv, acc[t][e + 3] * inv)};
  am_wait<0>();
  constexpr int PIECES = D / 8;
  for (int at = lane; at < 32 * PIECES; at += 64) {
    const int r = wave0 + at / PIECES, piece = at % PIECES;
    if (r > last) break;
    const u32x4 v = *reinterpret_cast<const u32x4*>(own + (at / PIECES) * Shape::kOutRow + piece * 16);
    *reinterpret_cast<u32x4_at2*>(a.out + (int64_t)(seq.first + r / c.group) * a.ldo + (int64_t)(head * c.group + r % c.group) * a.ho + piece * 8) = v;
  }
}

template <int D, int PB, int NW> static hipError_t launch_many_as(const AttentionArgs& all, int64_t blocks, hipStream_t s) {
  static LdsLimitOnce once;
  if (const hipError_t e = once.ensure((const void*)&attention_many_kernel<D, PB, NW>, ManyShape<D, NW>::kLds); e != hipSuccess) return e;
  AttentionArgs a = all;
  const int64_t each = (int64_t)a.parts * a.c.kv_heads, most = ((int64_t)1 << 22) / each;      // (a grid has less than 2^32 threads)
  for (int64_t first = 0; first < blocks; first += most) {
    a.first_block = first;
    const int64_t n = blocks - first < most ? blocks - first : most;
    hipLaunchKernelGGL((attention_many_kernel<D, PB, NW>), dim3((unsigned)(n * each)), dim3(64 * NW), (ManyShape<D, NW>::kLds), s, a, (int)n);
    if (const hipError_t e = hipGetLastError(); e != hipSuccess) return e;
  }
  return hipSuccess;
}
template <int D> static hipError_t launch_many_of(const AttentionArgs& a, int64_t blocks, hipStream_t s) {
  return a.c.page_bits == 4 ? launch_many_as<D, 4, kManyWaves>(a, blocks, s) : launch_many_as<D, 5, kManyWaves>(a, blocks, s);
}
hipError_t launch_attention_many(const AttentionArgs& a, int64_t blocks, hipStream_t s) {
  return a.c.d == 64 ? launch_many_of<64>(a, blocks, s) : a.c.d == 96 ? launch_many_of<96>(a, blocks, s) : launch_many_of<128>(a, blocks, s);
}

}  // namespace gptaq
