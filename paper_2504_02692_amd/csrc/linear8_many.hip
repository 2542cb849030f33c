// y = x W^T for many tokens, codes of 8 bits on both sides.
#include "linear8.h"

namespace gptaq {

// A workgroup takes 32 TT WT tokens x 32 RT WR rows of W, a wavefront 32 TT tokens and 32 RT rows of these, as TT RT results of v_mfma 32x32x32.  W goes straight from memory
// to the lanes that feed the matrix unit, 128 columns (a stage) two stages ahead; activations straight to LDS, in a ring of four stages with one barrier a stage, in its
// middle: it publishes the next stage (whose first fragments are read before the stage ends) and retires the one before.  With 128 x 64 a wavefront LDS is
// read for half of the time that the matrix unit works.
// The left operand is W, so that a lane has four rows of a token side by side.  The activations' sums (linear8.h) are taken by dot products of four of the fragments that
// the wavefront has, each fragment by one of the wavefronts that share the tokens.
// 8192 tokens, 28672 x 8192, tiles of 256 x 256: 1.65 ms, 2.3 POP/s, with the matrix unit busy for 60 % of the cycles at 1.74 to 1.81 GHz; of a wavefront's time 43 % waits
// for its turn at the unit and 32 % for loads and barriers.  Small calls are bound by their stages, each of which waits for loads that were asked for two
// stages before: 257 tokens, 4096 x 1024, eight stages of 160 tiles, 8.3 us.
constexpr int kX8Ring = 4;
template <int TT, int RT, int WT, int WR> struct Many8 {
  static constexpr int kTokens = 32 * TT * WT, kRows = 32 * RT * WR, kWaves = WT * WR;
  static constexpr int kStage = kTokens * 128, kLoads = kStage / 1024 / kWaves;       // loads of activations, per wavefront and stage
  static constexpr int kOutRow = 32 * RT * 4 + 16;                                    // results in LDS, 32 tokens of a wavefront at a time
  static constexpr int kRing = kX8Ring * kStage, kOut = kWaves * 32 * kOutRow, kSums = WR * kTokens * 4;
  static constexpr int kLds = (kRing > kOut ? kRing : kOut) + kSums;
  static_assert(kLoads * 1024 * kWaves == kStage && 4 % WR == 0, "");
};
template <int N> __device__ __forceinline__ void many8_wait() {      // vmcnt <= N, lgkmcnt == 0
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt((N & 15) | ((N >> 4) << 14) | (7 << 4));
  asm volatile("" ::: "memory");
}
__device__ __forceinline__ void many8_barrier() {         // no memory fence: loads stay in flight across it
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

template <int TT, int RT, int WT, int WR>
__global__ __launch_bounds__(64 * WT * WR, 2) void linear8_many_kernel(Linear8Args p, int token_tiles, int row_tiles) {
  using Tile = Many8<TT, RT, WT, WR>;
  extern __shared__ __attribute__((aligned(256))) unsigned char smem[];
  constexpr int NL = Tile::kLoads;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wt = wave / WR, wr = wave % WR;
  const int l32 = lane & 31, half = lane >> 5, l16 = lane & 15;
  // Workgroups go to the eight XCDs in turn: each gets one run of the list of tiles, and the list takes eight tiles of tokens against
  // one tile of rows after the other, so that what an XCD works on at a time shares both operands in its L2.
  const int grid = gridDim.x, xcd = blockIdx.x & 7, tiles = token_tiles * row_tiles;
  const int of_list = xcd * (grid >> 3) + min(xcd, grid & 7) + (int)(blockIdx.x >> 3);
  const int part = of_list / tiles, at = of_list - part * tiles;
  const int band = at / (8 * row_tiles), in_band = at - band * 8 * row_tiles, wide = min(8, token_tiles - band * 8);
  const int tok0 = (band * 8 + in_band % wide) * Tile::kTokens, row0 = in_band / wide * Tile::kRows;
  const int k_begin = (int)((int64_t)p.kt * part / p.parts), k_end = (int)((int64_t)p.kt * (part + 1) / p.parts);   // stages of this part

  // ---- activations: the wavefront's share of a stage's rows.  The 16-byte chunks of a row are permuted so that 16 consecutive rows of one chunk lie in 16
  // different places of 256 bytes (all banks once).
  auto swizzle = [](int row) { return (row >> 1) & 7; };
  const LdsLoader xfrom((const unsigned char*)p.x + (int64_t)tok0 * p.ldx);
  int xsrc[NL];
#pragma unroll
  for (int j = 0; j < NL; ++j) {
    const int row = (wave * NL + j) * 8 + lane / 8, chunk = lane % 8 ^ swizzle(row);
    const int tok = tok0 + row < p.tokens ? row : p.tokens - 1 - tok0;         // (their results are not stored)
    xsrc[j] = tok * (int)p.ldx + chunk * 16;
  }
  auto load_x = [&](int k) {
    const int from = (k < k_end ? k : k_end - 1) * 128;                        // (behind the last stage that again: the counts stay the same)
#pragma unroll
    for (int j = 0; j < NL; ++j) xfrom.load(smem + k % kX8Ring * Tile::kStage + (wave * NL + j) * 1024, xsrc[j], from);
  };
  int foff[4];                                            // of the steps
#pragma unroll
  for (int s = 0; s < 4; ++s) foff[s] = (wt * TT * 32 + l32) * 128 + ((((half ^ swizzle(l32)) << 4)) ^ (s << 5));
  u32x4 xf[2][TT];                                        // [step & 1][tile of 32 tokens]
  auto read_x = [&](int stage, int s, int i) {
    xf[s & 1][i] = *reinterpret_cast<const u32x4*>(smem + stage % kX8Ring * Tile::kStage + foff[s] + i * 32 * 128);
  };
  // ---- weights: lane l has row l % 32 of 32; step s has chunks 2 s and 2 s + 1 of the stage's eight
  // (Buffer loads: the place in the row is a scalar.)
  const int tr0 = row0 / 16;
  const __amdgpu_buffer_rsrc_t codes = __builtin_amdgcn_make_buffer_rsrc((void*)(p.codes + (int64_t)tr0 * p.kt * 2048), 0, 0x7fffffff, 0x00020000);
  int wsrc[RT];
#pragma unroll
  for (int j = 0; j < RT; ++j) {
    const int tr = (wr * RT + j) * 2 + (l32 >> 4);
    wsrc[j] = (tr0 + tr < p.mt ? tr : p.mt - 1 - tr0) * p.kt * 2048 + half * 256 + l16 * 16;
  }
  struct Codes { u32x4 w[4][RT]; };
  auto load_w = [&](Codes& c, int k, int s) {
    const int from = (k < k_end ? k : k_end - 1) * 2048 + s * 512;
#pragma unroll
    for (int j = 0; j < RT; ++j) c.w[s][j] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(codes, wsrc[j], from, 0));
  };

  i32x16 acc[RT][TT];
  int sums[TT];
#pragma unroll
  for (int i = 0; i < TT; ++i) {
    sums[i] = 0;
#pragma unroll
    for (int j = 0; j < RT; ++j)
#pragma unroll
      for (int e = 0; e < 16; ++e) acc[j][i][e] = 0;
  }
  // (The dot products are written out: the compiler would take all, and keep one of WR.)  Behind each fragment's matrix instructions: the same fragment of the next step; behind a step's, its weights of the stage after the next.
  auto stage = [&](Codes& c, int k) {
#pragma unroll
    for (int s = 0; s < 4; ++s) {
#pragma unroll
      for (int i = 0; i < TT; ++i) {
#pragma unroll
        for (int j = 0; j < RT; ++j)
          acc[j][i] = __builtin_amdgcn_mfma_i32_32x32x32_i8(__builtin_bit_cast(i32x4, c.w[s][j]), __builtin_bit_cast(i32x4, xf[s & 1][i]), acc[j][i], 0, 0, 0);
        if (s % WR == wr) {
#pragma unroll
          for (int e = 0; e < 4; ++e) asm volatile("v_dot4_i32_i8 %0, %1, %2, %0" : "+v"(sums[i]) : "v"(xf[s & 1][i][e]), "s"(0x01010101));
        }
        __builtin_amdgcn_sched_barrier(0);
        if (s < 3) read_x(k, s + 1, i);
        else read_x(k + 1, 0, i);
        __builtin_amdgcn_sched_barrier(0);
      }
      load_w(c, k + 2, s);
      __builtin_amdgcn_sched_barrier(0);
      if (s == 1) {
        many8_wait<6 * RT + NL>();                        // stage k + 1 is there: behind it have been asked for 2 RT loads of W three times, and stage k + 2
        many8_barrier();
        load_x(k + 3);
        __builtin_amdgcn_sched_barrier(0);
      }
    }
  };
  Codes ca, cb;
  load_x(k_begin);
  load_x(k_begin + 1);
  __builtin_amdgcn_sched_barrier(0);
#pragma unroll
  for (int s = 0; s < 4; ++s) load_w(ca, k_begin, s);
  __builtin_amdgcn_sched_barrier(0);
  load_x(k_begin + 2);
  __builtin_amdgcn_sched_barrier(0);
#pragma unroll
  for (int s = 0; s < 4; ++s) load_w(cb, k_begin + 1, s);
  __builtin_amdgcn_sched_barrier(0);
  many8_wait<2 * NL + 8 * RT>();                          // the first stage is there
  many8_barrier();
#pragma unroll
  for (int i = 0; i < TT; ++i) read_x(k_begin, 0, i);
  int k = k_begin;
  for (; k + 1 < k_end; k += 2) {
    stage(ca, k);
    stage(cb, k + 1);
  }
  if (k < k_end) stage(ca, k);

  // ---- results, 32 tokens of a wavefront after the other, through its own place in LDS, so that a token's outputs leave in runs
  many8_wait<0>();                                        // (no load writes to LDS from here on)
  int32_t* const sx = reinterpret_cast<int32_t*>(smem + Tile::kLds - Tile::kSums);
#pragma unroll
  for (int i = 0; i < TT; ++i) {
    const int all = sums[i] + __shfl_xor(sums[i], 32);
    if (half == 0) sx[wr * Tile::kTokens + (wt * TT + i) * 32 + l32] = all;
  }
  __syncthreads();
  unsigned char* const own = smem + wave * 32 * Tile::kOutRow;
  constexpr int RUNS = 4 * RT;                            // of eight rows
  const int col = lane % RUNS * 8, row = row0 + wr * RT * 32 + col;
  float scale[8], bias[8];
  int shift[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const bool real = row + e < p.out.m;
    scale[e] = real ? p.scales[row + e] : 0.f;
    shift[e] = real ? p.shifts[row + e] : 0;
    bias[e] = real && p.out.bias ? p.out.bias[row + e] : 0.f;
  }
#pragma unroll
  for (int i = 0; i < TT; ++i) {
#pragma unroll
    for (int j = 0; j < RT; ++j)
#pragma unroll
      for (int e = 0; e < 16; e += 4)
        *reinterpret_cast<i32x4*>(own + l32 * Tile::kOutRow + (32 * j + 2 * e + 4 * half) * 4) = i32x4{acc[j][i][e], acc[j][i][e + 1], acc[j][i][e + 2], acc[j][i][e + 3]};
    many8_wait<0>();
#pragma unroll
    for (int t = lane / RUNS; t < 32; t += 64 / RUNS) {
      const int in_tile = (wt * TT + i) * 32 + t, tok = tok0 + in_tile;
      if (tok >= p.tokens || row >= p.out.m) continue;
      uint32_t sum = 0;
#pragma unroll
      for (int w = 0; w < WR; ++w) sum += (uint32_t)sx[w * Tile::kTokens + in_tile];
      const i32x4 lo = *reinterpret_cast<const i32x4*>(own + t * Tile::kOutRow + col * 4), hi = *reinterpret_cast<const i32x4*>(own + t * Tile::kOutRow + col * 4 + 16);
      int v[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = (int)((uint32_t)(e < 4 ? lo[e] : hi[e - 4]) + (uint32_t)shift[e] * sum);
      if (p.parts > 1) {                                  // (whole runs: rows of p.partial have room for them)
        int32_t* to = p.partial + ((int64_t)part * p.tokens + tok) * p.ld_partial + row;
        *reinterpret_cast<i32x4*>(to) = i32x4{v[0], v[1], v[2], v[3]};
        *reinterpret_cast<i32x4*>(to + 4) = i32x4{v[4], v[5], v[6], v[7]};
      } else {
        const float xs = p.xs[tok];
        float y[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) y[e] = fmaf((float)v[e], xs * scale[e], bias[e]);
        linear_store(p.out, tok, row, y);
      }
    }
    many8_wait<0>();                                      // (before the next tokens' results take the place)
  }
}

// The parts' sums of eight outputs of a token: whole numbers, in any order the same.
__global__ __launch_bounds__(256) void linear8_join_kernel(Linear8Args p) {
  const int runs = (int)(p.ld_partial / 8);
  const int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const int tok = (int)(at / runs), row = (int)(at % runs) * 8;
  if (tok >= p.tokens) return;
  i32x4 v[2] = {i32x4{0, 0, 0, 0}, i32x4{0, 0, 0, 0}};
  for (int k = 0; k < p.parts; ++k) {
    const int32_t* from = p.partial + ((int64_t)k * p.tokens + tok) * p.ld_partial + row;
    v[0] += *reinterpret_cast<const i32x4*>(from);
    v[1] += *reinterpret_cast<const i32x4*>(from + 4);
  }
  const float xs = p.xs[tok];
  float y[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const bool real = row + e < p.out.m;
    y[e] = fmaf((float)v[e >> 2][e & 3], xs * (real ? p.scales[row + e] : 0.f), real && p.out.bias ? p.out.bias[row + e] : 0.f);
  }
  linear_store(p.out, tok, row, y);
}

template <int TT, int RT, int WT, int WR> static hipError_t launch_many8_as(const Linear8Args& p, hipStream_t s) {
  using Tile = Many8<TT, RT, WT, WR>;
  static LdsLimitOnce once;
  if (const hipError_t e = once.ensure((const void*)&linear8_many_kernel<TT, RT, WT, WR>, Tile::kLds); e != hipSuccess) return e;
  const int tt = (p.tokens + Tile::kTokens - 1) / Tile::kTokens, rt = (p.out.m + Tile::kRows - 1) / Tile::kRows;
  hipLaunchKernelGGL((linear8_many_kernel<TT, RT, WT, WR>), dim3((unsigned)((int64_t)tt * rt * p.parts)), dim3(64 * WT * WR), Tile::kLds, s, p, tt, rt);
  if (const hipError_t e = hipGetLastError(); e != hipSuccess || p.parts == 1) return e;
  hipLaunchKernelGGL(linear8_join_kernel, dim3((unsigned)((p.tokens * (p.ld_partial / 8) + 255) / 256)), dim3(256), 0, s, p);
  return hipGetLastError();
}

// Tile of a call, 64 x 128, 128 x 128 or 256 x 256, and the parts that the columns of the smallest are taken in.  The rule is the least of what the calls were measured to
// take, us: a stage of the smaller tiles takes 0.5 and 0.7 while every CU has one at most, and 0.37 and 0.69 for each 256 tiles from there on, more where a few CUs
// have one more than the others; one of the largest 1.6 while half of the CUs have one, and 1.9 for each round of 256; parts save stages, and cost a launch and their sums' way through memory; and the weights are read at
// 5 TB/s at best.  us a call, 64 x 128 / 128 x 128 / 256 x 256, one part: 4096 x 4096, 512 tokens 18.5 / 24.7 / 51.9, 2048 46.7 / 42.9 / 56.2, 4096 91.6 / 82.4 / 70.0;
// 28672 x 8192, 257 122 / 121 / 121, 512 179 / 168 / 132, 2048 615 / 545 / 465; 11008 x 4096, 257 22.9 / 33.5 / 52.3, 1500 94 / 95 / 112, 4096 255 / 225 / 193.  One part /
// parts: 4096 x 11008, 33 tokens 34.0 / 16.3 (5), 257 35.6 / 29.7 (3), 512 38.7 / 41.7 (2); 1024 x 8192, 257 27.1 / 16.4 (4), 2048 29.8 / 34.5 (2); 4096 x 4096, 257 17.1 / 23.2 (3).
struct Many8Plan { int tile; int64_t parts; };
static constexpr int64_t kTileTokens[3] = {64, 128, 256}, kTileRows[3] = {128, 128, 256}, kRoom = 512;
static int64_t tiles_of(int tile, int64_t tokens, int64_t m) {
  return (tokens + kTileTokens[tile] - 1) / kTileTokens[tile] * ((m + kTileRows[tile] - 1) / kTileRows[tile]);
}
static int64_t most_parts8(int64_t n) { return (n + 127) / 128 / 4; }       // of at least four stages each
static Many8Plan many8_plan(int64_t tokens, int64_t m, int64_t n) {
  const double kt = (double)((n + 127) / 128), t0 = (double)tiles_of(0, tokens, m) / 256, t1 = (double)tiles_of(1, tokens, m) / 256;
  const int64_t t2 = tiles_of(2, tokens, m);
  auto greater = [](double a, double b) { return a > b ? a : b; };
  Many8Plan plan{0, 1};
  double least = kt * (t0 <= 2 ? greater(0.5, 0.38 * t0) : greater(1.0, 0.37 * t0));
  if (const double us = kt * (t1 <= 1 ? 0.7 : greater(1.15, 0.69 * t1)); us < least) { least = us; plan.tile = 1; }
  if (const double us = kt * (t2 <= 128 ? 1.6 : 1.9 * (double)((t2 + 255) / 256)); us < least) { least = us; plan.tile = 2; }
  const double read = (double)m * (double)n / 5e6;
  least = greater(least, read);
  for (int64_t parts = 2; parts <= most_parts8(n) && parts * tiles_of(0, tokens, m) <= kRoom; ++parts) {
    const double us = greater(read, kt / (double)parts * greater(0.5, 0.36 * t0 * (double)parts)) + 4 + (double)(parts * tokens * m) * 8 / 2.5e6;
    if (us < least) { least = us; plan = Many8Plan{0, parts}; }
  }
  return plan;
}
// Room for the partial sums of every call with at most so many tokens: parts times tiles is at most kRoom, and parts at most so many.
size_t linear8_partial_bytes(int64_t tokens, int64_t m, int64_t n) {
  const int64_t ld = (m + 7) / 8 * 8, each = kRoom / ((m + kTileRows[0] - 1) / kTileRows[0]);
  if (most_parts8(n) < 2 || each < 2) return 0;
  const int64_t rows = each * kTileTokens[0] < most_parts8(n) * tokens ? each * kTileTokens[0] : most_parts8(n) * tokens;      // of ld values
  return (size_t)(rows * ld) * 4;
}
hipError_t launch_linear8_many(Linear8Args p, int32_t* partial, hipStream_t s) {
  const Many8Plan plan = many8_plan(p.tokens, p.out.m, (int64_t)p.kt * 128);
  p.parts = (int32_t)plan.parts;
  p.partial = partial;
  p.ld_partial = (p.out.m + 7) / 8 * 8;
  return plan.tile == 0 ? launch_many8_as<2, 1, 1, 4>(p, s) : plan.tile == 1 ? launch_many8_as<2, 2, 2, 2>(p, s) : launch_many8_as<4, 2, 2, 4>(p, s);
}

}  // namespace gptaq
