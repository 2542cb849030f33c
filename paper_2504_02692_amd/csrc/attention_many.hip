// Attention over a paged cache for many rows: prompts, and pieces of prompts behind what the cache has of them.
#include "attention.h"
#include "linear.h"

namespace gptaq {

// A block is 32 NW rows, NW wavefronts of 32 rows each.  Keys and values come in tiles of 64 straight from memory to LDS, as they lie in the pages, into a ring of
// kRing tiles with one barrier a tile.  Both products are taken transposed, with v_mfma 32x32x16: S^T = K Q^T leaves a lane the scores of one row (l % 32), and O^T = V^T P^T
// takes the weights from there without an exchange, if the first product's row 16 s + 8 b + 4 a + i has key 16 s + 8 a + 4 b + i (bits 2 and 3 change places).
// Reads of either from LDS are runs of 512 bytes: no bank is met twice.
// PB: bits of a page as far as they matter to a tile's layout (4, 5, 6: pages of 16, 32, and more).
constexpr int kRing = 4;
template <int D, int NW> struct ManyShape {
  static constexpr int kTileBytes = kTile * D * 2, kLoads = kTileBytes / 1024;      // of keys, or of values
  static constexpr int kPerWave = 2 * kLoads / NW;
  static constexpr int kOutRow = D * 2 + 16;                                        // results in LDS
  static constexpr int kRingBytes = kRing * 2 * kTileBytes, kOutBytes = 32 * NW * kOutRow;
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

template <int D, int PB, int NW>
__global__ __launch_bounds__(64 * NW, 2) void attention_many_kernel(AttentionArgs a, int64_t blocks) {
  using Shape = ManyShape<D, NW>;
  extern __shared__ __attribute__((aligned(256))) unsigned char smem[];
  constexpr int KS = D / 16, VT = D / 32, P = 1 << PB, TILE = Shape::kTileBytes;
  const CacheShape& c = a.c;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), l32 = lane & 31, half = lane >> 5;
  // The heads of a block side by side, so that with eight key heads each XCD has one; late blocks first, which see the most.
  const int head = (int)(blockIdx.x % (unsigned)c.kv_heads), rest = (int)(blockIdx.x / (unsigned)c.kv_heads);
  const int part = rest % a.parts;
  const int64_t block = blocks - 1 - (a.first_block + rest / a.parts);
  const int s = cache_find(c, block, c.group, a.rows_bits, 1);
  const Sequence seq = cache_sequence(c, s);
  const int64_t in_seq = block - cache_block_of(c, s, c.group, a.rows_bits, 1);
  const int rows = seq.count * c.group;
  if (in_seq < 0 || (in_seq << a.rows_bits) >= rows) return;
  const int row0 = (int)in_seq << a.rows_bits, last = min(row0 + 32 * NW - 1, rows - 1);
  const Tiles tiles = attention_tiles(a, seq.before + row0 / c.group, seq.before + last / c.group);
  const Parts parts = attention_parts(a, tiles.count);
  if (part > 0 && part >= parts.count) return;                       // (part 0 writes the zeros of rows that see nothing)
  const int begin = part * parts.each, end = min(begin + parts.each, tiles.count);

  // the wavefront's rows
  const int wave0 = row0 + wave * 32, wave1 = min(wave0 + 31, last);
  const bool idle = wave0 > last;
  const int row = min(wave0 + l32, last), token = row / c.group, p_row = seq.before + token;
  const int pmin = seq.before + min(wave0, last) / c.group, pmax = idle ? -1 : seq.before + wave1 / c.group;
  const uint16_t* const qrow = a.q + (int64_t)(seq.first + token) * a.ldq + (int64_t)(head * c.group + row % c.group) * a.hq;
  typedef u32x4 __attribute__((aligned(2))) u32x4_at2;
  // (A negative scale goes to the queries' signs, so that the largest score is that of the largest product.)
  const uint32_t flip = a.scale < 0.f ? 0x80008000u : 0u;
  const float scale = fabsf(a.scale);
  bf16x8 qf[KS];
#pragma unroll
  for (int i = 0; i < KS; ++i) qf[i] = __builtin_bit_cast(bf16x8, *reinterpret_cast<const u32x4_at2*>(qrow + i * 16 + half * 8) ^ flip);

  // ---- loads: a tile of keys, then of values, 1 KB each
  const int64_t head_bytes = (int64_t)(D * 2) << c.page_bits;        // of a page, of one head
  const int32_t* const table = c.table + (int64_t)s * c.ld_table;
  struct Ids { int id[1 << (6 - PB)]; };
  auto pages_of = [&](Ids& g, int i) {                               // of the i-th tile of this part (behind the last: that again)
    const int at = (tiles.at(min(i, end - 1)) * kTile) >> c.page_bits;
#pragma unroll
    for (int k = 0; k < (1 << (6 - PB)); ++k) {
      const int id = at + k < c.table_pages ? table[at + k] : -1;
      g.id[k] = __builtin_amdgcn_readfirstlane((uint32_t)id < (uint64_t)c.pages ? id : -1);
    }
  };
  auto load_tile = [&](const Ids& g, int i) {
    const int off = (tiles.at(min(i, end - 1)) * kTile) & ((1 << c.page_bits) - 1);      // (in a page of more than 64)
    constexpr int PER = Shape::kLoads >> (6 - PB);                   // loads of a page
#pragma unroll
    for (int n = 0; n < Shape::kPerWave; ++n) {
      const int at = wave * Shape::kPerWave + n, load = at % Shape::kLoads;
      const bool value = at >= Shape::kLoads;
      const int which = load / PER, in_page = load % PER;
      int id = g.id[0];
#pragma unroll
      for (int k = 1; k < (1 << (6 - PB)); ++k) id = which == k ? g.id[k] : id;
      const int64_t from = ((int64_t)max(id, 0) * c.kv_heads + head) * head_bytes +
                           (PB < 6 ? in_page * 1024 : value ? off * (D * 2) + in_page * 1024 : ((in_page << c.page_bits) + off) * 16);
      const LdsLoader loader((const unsigned char*)(value ? a.values : a.keys) + from);
      loader.load(smem + ((i % kRing) * 2 + (value ? 1 : 0)) * TILE + load * 1024, lane * 16, 0);
    }
  };
  auto valid = [&](const Ids& g) {                                   // a bit for each 16 keys
    int ok = 0;
#pragma unroll
    for (int k = 0; k < 4; ++k) ok |= (g.id[k >> (PB - 4)] >= 0 ? 1 : 0) << k;
    return ok;
  };

  f32x16 acc[VT];
#pragma unroll
  for (int i = 0; i < VT; ++i)
#pragma unroll
    for (int e = 0; e < 16; ++e) acc[i][e] = 0.f;
  float top = -__builtin_inff(), total = 0.f;                        // top: of scaled scores; total: this lane's keys alone
  const int key = (l32 & 0x13) | (l32 & 4) << 1 | (l32 & 8) >> 1;    // of 32 that the lane reads
  int kread[2];
#pragma unroll
  for (int b = 0; b < 2; ++b) {
    const int k = b * 32 + key;
    kread[b] = (k >> PB) * (D * 2 * P) + (k & (P - 1)) * 16 + half * P * 16;
  }
  const int vread = (half * D + l32) * 16;

  auto work = [&](auto whole_tile, int i, int j0, int ok) {
    constexpr bool WHOLE = decltype(whole_tile)::value;
    const unsigned char* const kt = smem + (i % kRing) * 2 * TILE;
    const unsigned char* const vt = kt + TILE;
    f32x16 sc[2];
#pragma unroll
    for (int b = 0; b < 2; ++b) {
#pragma unroll
      for (int e = 0; e < 16; ++e) sc[b][e] = 0.f;
#pragma unroll
      for (int k = 0; k < KS; ++k)
        sc[b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(*reinterpret_cast<const bf16x8*>(kt + kread[b] + k * (2 * P * 16)), qf[k], sc[b], 0, 0, 0);
    }
    // element e of block b: key 32 b + 16 (e / 8) + 8 half + e % 8
    if (!WHOLE) {
      const int j = j0 + 8 * half, until = p_row - j, after = a.window ? p_row - a.window - j : -1 << 30, sinks = a.sinks - j;
#pragma unroll
      for (int b = 0; b < 2; ++b)
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          const int at = 32 * b + 16 * (e >> 3) + (e & 7);
          const bool here = (ok >> (at >> 4) & 1) && at <= until && (at > after || at < sinks);
          sc[b][e] = here ? sc[b][e] : kUnseen;
        }
    }
    float most = sc[0][0];
#pragma unroll
    for (int e = 1; e < 32; ++e) most = fmaxf(most, sc[e >> 4][e & 15]);
    most *= scale;
    if (__ballot(most > top + kSlack)) {
      most = fmaxf(most, __shfl_xor(most, 32));
      const float now = fmaxf(top, most), factor = at_factor(top, now);
      top = now;
      total *= factor;
#pragma unroll
      for (int t = 0; t < VT; ++t) acc[t] *= factor;
    }
    const float from = at_origin(top);
#pragma unroll
    for (int b = 0; b < 2; ++b) {
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        float w[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          w[e] = at_exp2(fmaf(sc[b][8 * k + e], scale, -from));
          total += w[e];
        }
        const u32x4 wp = {at_bf16x2(w[0], w[1]), at_bf16x2(w[2], w[3]), at_bf16x2(w[4], w[5]), at_bf16x2(w[6], w[7])};
        u32x4 v[VT];
#pragma unroll
        for (int t = 0; t < VT; ++t) v[t] = *reinterpret_cast<const u32x4*>(vt + vread + ((b * 4 + k * 2) * D + t * 32) * 16);
        if (!WHOLE) {
          bool any = false;
#pragma unroll
          for (int t = 0; t < VT; ++t) any |= attention_strange(v[t]);
          if (__ballot(any)) {
            u32x4 ones;
#pragma unroll
            for (int h = 0; h < 4; ++h) ones[h] = (sc[b][8 * k + 2 * h] != kUnseen ? 0x3f80u : 0u) | (sc[b][8 * k + 2 * h + 1] != kUnseen ? 0x3f800000u : 0u);
#pragma unroll
            for (int t = 0; t < VT; ++t) {
              u32x4 marks;
              attention_marks(v[t], marks);
              f32x16 n;
#pragma unroll
              for (int e = 0; e < 16; ++e) n[e] = 0.f;
              n = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, marks), __builtin_bit_cast(bf16x8, ones), n, 0, 0, 0);
#pragma unroll
              for (int e = 0; e < 16; ++e) acc[t][e] += attention_strange_sum(n[e]);
            }
          }
        }
#pragma unroll
        for (int t = 0; t < VT; ++t)
          acc[t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, v[t]), __builtin_bit_cast(bf16x8, wp), acc[t], 0, 0, 0);
      }
    }
  };

  if (begin < end) {
    Ids ids[kRing];                                                  // of the tiles in flight: ids[k] of tile i + k
#pragma unroll
    for (int k = 0; k < kRing - 1; ++k) {
      pages_of(ids[k], begin + k);
      load_tile(ids[k], begin + k);
    }
    pages_of(ids[kRing - 1], begin + kRing - 1);
    for (int i = begin; i < end; ++i) {
      am_wait<(kRing - 2) * Shape::kPerWave>();                      // the wavefront's loads of tile i are there ..
      am_barrier();                                                  // .. and everyone's; and tile i - 1 is no longer read
      load_tile(ids[kRing - 1], i + kRing - 1);
      const int ok = valid(ids[0]);
#pragma unroll
      for (int k = 0; k < kRing - 1; ++k) ids[k] = ids[k + 1];
      pages_of(ids[kRing - 1], i + kRing);
      const int j0 = tiles.at(i) * kTile;
      if (j0 > pmax || (a.window && j0 + kTile - 1 <= pmin - a.window && j0 >= a.sinks)) continue;
      if (ok == 15 && j0 + kTile - 1 <= pmin && (a.window == 0 || j0 > pmax - a.window || j0 + kTile - 1 < a.sinks)) work(std::true_type{}, i, j0, ok);
      else work(std::false_type{}, i, j0, ok);
    }
    am_wait<0>();                                                    // (no load writes to LDS from here on)
    am_barrier();
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
    if (half == 0) { a.stats[call_row * 2] = top; a.stats[call_row * 2 + 1] = total; }
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
    hipLaunchKernelGGL((attention_many_kernel<D, PB, NW>), dim3((unsigned)(n * each)), dim3(64 * NW), (ManyShape<D, NW>::kLds), s, a, blocks);
    if (const hipError_t e = hipGetLastError(); e != hipSuccess) return e;
  }
  return hipSuccess;
}
template <int D> static hipError_t launch_many_of(const AttentionArgs& a, int64_t blocks, hipStream_t s) {
  return a.c.page_bits == 4 ? launch_many_as<D, 4, kManyWaves>(a, blocks, s) : a.c.page_bits == 5 ? launch_many_as<D, 5, kManyWaves>(a, blocks, s)
                                                                                              : launch_many_as<D, 6, kManyWaves>(a, blocks, s);
}
hipError_t launch_attention_many(const AttentionArgs& a, int64_t blocks, hipStream_t s) {
  return a.c.d == 64 ? launch_many_of<64>(a, blocks, s) : a.c.d == 96 ? launch_many_of<96>(a, blocks, s) : launch_many_of<128>(a, blocks, s);
}

}  // namespace gptaq
