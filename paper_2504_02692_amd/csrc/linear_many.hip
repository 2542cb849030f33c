// y = x W^T for many tokens: matrix products with weights that are made from their 4-bit codes on the way.
#include "linear.h"

namespace gptaq {

typedef __attribute__((ext_vector_type(4))) int32_t i32x4;
typedef __attribute__((ext_vector_type(16))) int32_t i32x16;

// A workgroup of eight wavefronts takes 128 tokens x 256 rows of W; a wavefront all the tokens and 32 rows, as four results of
// v_mfma 32x32, twice: the sum of the current group of columns and the fp32 total it is scaled into.  These 128 registers a lane
// are what limits the tile.  The right operand of a matrix instruction is made of codes in the registers of the lanes that feed it:
// the rows of W belong to one wavefront each, so every code is unpacked once per workgroup and W never passes through LDS.
// A byte of W feeds four times the products that a byte of bf16 activations does, so the tile is taller in W.
// Activations go from memory straight to LDS, 128 columns (a stage) at a time, in a ring of four stages with one barrier a stage, in
// its middle: it publishes the next stage (whose first fragments are read before the stage ends) and retires the one before.
// 2048 x 11008 x 4096 bf16 181 to 198 us on two cards, 0.93 to 1.0 PFLOP/s (the library's bf16 product of this card: 1.46), 8192 x 28672 x 8192 8-bit 2.25 to 2.4 ms, 1.6 to 1.7 POP/s (2.43).
// A 32x32 matrix instruction takes 32 cycles of the matrix unit and 16 of the SIMD's vector issue, a vector instruction 4: with n of these to each it is
// max(32, 16 + 4 n) cycles.  bf16 has 7 (5 of them unpack codes, 2 scale sums), 8 bits 12 (4 and 8), and the chip's power holds bf16 to about 2.1 GHz:
// with inputs of zeros the same products take four fifths of the time.
// TT tiles of 32 tokens (4, or 2 where there are few tokens or tiles) and WV wavefronts; with fewer tokens than 128 several workgroups
// share a CU.  A result that too few workgroups would share is taken in parts of the columns, each by workgroups of its own: their sums
// go to p.partial, and linear_join_kernel adds them in order.
constexpr int kXRing = 4;
template <int TT, int WV> struct ManyTile {
  static constexpr int kTokens = 32 * TT, kRows = 32 * WV;
  static constexpr int kOutRow = kRows + 4;               // results in LDS: fp32, and 16 bytes so that tokens start at different banks
  static constexpr int kRingBytes = kXRing * kTokens * 256, kOutBytes = kTokens * kOutRow * 4;
  static constexpr int kLds = kRingBytes > kOutBytes ? kRingBytes : kOutBytes;
};

__device__ __forceinline__ void many_barrier() {          // no memory fence: loads stay in flight across it
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}
template <int N> __device__ __forceinline__ void many_wait() {      // vmcnt <= N, lgkmcnt == 0
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt((N & 15) | ((N >> 4) << 14) | (7 << 4));
}

template <bool I8, int GS, int TT, int WV>
__global__ __launch_bounds__(64 * WV, 2) void linear_many_kernel(LinearArgs p, int token_tiles, int row_tiles) {
  using Tile = ManyTile<TT, WV>;
  extern __shared__ __attribute__((aligned(256))) unsigned char smem[];
  constexpr int ST = I8 ? 4 : 8;                        // steps (matrix instructions along the columns) per stage
  constexpr int SPG = GS ? ST / (GS ? GS : 1) : ST;                // steps per group
  constexpr int NG = GS ? GS : 1;
  constexpr int XROW = I8 ? 128 : 256, XSTAGE = Tile::kTokens * XROW, CHUNKS = XROW / 16;
  constexpr int NL = XSTAGE / (1024 * WV);              // loads of 1 KB per wavefront and stage
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int l32 = lane & 31, half = lane >> 5, l16 = lane & 15;
  // Workgroups go to the eight XCDs in turn: each gets one run of the list of tiles, and the list takes eight tiles of tokens against
  // one tile of rows after the other, so that what an XCD works on at a time shares both operands in its L2.
  const int grid = gridDim.x, xcd = blockIdx.x & 7, tiles = token_tiles * row_tiles;
  const int of_list = xcd * (grid >> 3) + min(xcd, grid & 7) + (int)(blockIdx.x >> 3);
  const int part = of_list / tiles, at = of_list - part * tiles;
  const int band = at / (8 * row_tiles), in_band = at - band * 8 * row_tiles, wide = min(8, token_tiles - band * 8);
  const int tile_t = band * 8 + in_band % wide, tile_r = in_band / wide;
  const int tok0 = tile_t * Tile::kTokens, row0 = tile_r * Tile::kRows;
  const int k_begin = (int)((int64_t)p.kt * part / p.parts), k_end = (int)((int64_t)p.kt * (part + 1) / p.parts);   // stages of this part

  // ---- activations: the wavefront's share of a stage's rows in NL loads.  The 16-byte chunks of a row are permuted so that 16
  // consecutive rows of one chunk lie in 16 different places of 256 bytes (all banks once).
  auto swizzle = [](int row) { return I8 ? (row >> 1) & 7 : row & 15; };
  const LdsLoader xfrom((const unsigned char*)p.x + (int64_t)tok0 * p.ldx * (I8 ? 1 : 2));
  int xsrc[NL];
#pragma unroll
  for (int j = 0; j < NL; ++j) {
    const int row = (wave * NL + j) * (1024 / XROW) + lane / CHUNKS, chunk = lane % CHUNKS ^ swizzle(row);
    const int tok = tok0 + row < p.tokens ? row : p.tokens - 1 - tok0;         // (their results are not stored)
    xsrc[j] = tok * (int)p.ldx * (I8 ? 1 : 2) + chunk * 16;
  }
  int xload = k_begin;                                  // next stage to load
  auto load_x = [&]() {
    const int from = (xload < k_end ? xload : k_end - 1) * XROW;                 // (behind the last stage that again: the counts stay the same)
#pragma unroll
    for (int j = 0; j < NL; ++j)
      xfrom.load(smem + xload % kXRing * XSTAGE + (wave * NL + j) * 1024, xsrc[j], from);
    ++xload;
  };
  const int foff = l32 * XROW + ((half ^ swizzle(l32)) << 4);
  u32x4 xf[2][TT];                                      // [step & 1][tile of 32 tokens]
  auto read_x = [&](int stage, int s, int i) {
    xf[s & 1][i] = *reinterpret_cast<const u32x4*>(smem + ((stage % kXRing * XSTAGE + foff) ^ (s << 5)) + i * 32 * XROW);
  };

  // ---- weights: lane l has row l % 32 of the wavefront's; of a tile's columns the pieces that its steps need (linear.h): bf16: word s / 2
  // of piece s % 2 in step s; int8: word s of both
  int tr = row0 / 16 + wave * 2 + (l32 >> 4);
  tr = tr < p.mt ? tr : p.mt - 1;
  const uint8_t* const codes = p.codes + (int64_t)tr * p.kt * 1024 + l16 * 16;
  const int piece0 = (I8 ? 2 * half : half) * 256, piece1 = (I8 ? 2 * half + 1 : half + 2) * 256;
  const int64_t group0 = (int64_t)tr * p.groups * 16 + l16;
  struct Codes { u32x4 w[2]; uint32_t zero[NG]; float scale[NG]; };
  auto load_codes = [&](Codes& c, int k) {
    k = k < k_end ? k : k_end - 1;
    c.w[0] = *reinterpret_cast<const u32x4*>(codes + (int64_t)k * 1024 + piece0);
    c.w[1] = *reinterpret_cast<const u32x4*>(codes + (int64_t)k * 1024 + piece1);
    if (GS) {
#pragma unroll
      for (int g = 0; g < NG; ++g) {
        c.zero[g] = p.zeros[group0 + (int64_t)(k * GS + g) * 16];
        c.scale[g] = p.scales[group0 + (int64_t)(k * GS + g) * 16];
      }
    }
  };
  uint32_t off = GS ? 0u : linear_offset(p.zeros[group0]);       // of the group being unpacked
  u32x4 wf[2];                                          // [step & 1]
  u32x2 bytes;
  // Bytes 0, 1 or 2, 3 as bf16.  (Left to itself the compiler shifts the odd bytes down first.)
  auto pair = [](uint32_t b, bool high) {
    float f0, f1;
    if (high) {
      asm("v_cvt_f32_i32_sdwa %0, sext(%1) dst_sel:DWORD dst_unused:UNUSED_PAD src0_sel:BYTE_2" : "=v"(f0) : "v"(b));
      asm("v_cvt_f32_i32_sdwa %0, sext(%1) dst_sel:DWORD dst_unused:UNUSED_PAD src0_sel:BYTE_3" : "=v"(f1) : "v"(b));
    } else {
      asm("v_cvt_f32_i32_sdwa %0, sext(%1) dst_sel:DWORD dst_unused:UNUSED_PAD src0_sel:BYTE_0" : "=v"(f0) : "v"(b));
      asm("v_cvt_f32_i32_sdwa %0, sext(%1) dst_sel:DWORD dst_unused:UNUSED_PAD src0_sel:BYTE_1" : "=v"(f1) : "v"(b));
    }
    typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
    return __builtin_bit_cast(uint32_t, bf16x2{(__bf16)f0, (__bf16)f1});
  };
  // step s's operand, in four parts
  auto unpack = [&](const Codes& c, int s, int part) {
    if (GS && s % SPG == 0 && part == 0) {
      uint32_t z = c.zero[s / SPG];
      asm volatile("" : "+v"(z));                       // (here, not right behind its load)
      off = linear_offset(z);
    }
    if (I8) {
      if (part < 2) {
        const u32x2 b = linear_bytes(c.w[part][s], off);
        wf[s & 1][2 * part] = b[0];
        wf[s & 1][2 * part + 1] = b[1];
      }
    } else {
      if (part == 0) bytes = linear_bytes(c.w[s & 1][s >> 1], off);
      if (part == 1) { wf[s & 1][0] = pair(bytes[0], false); wf[s & 1][1] = pair(bytes[0], true); }
      if (part == 2) { wf[s & 1][2] = pair(bytes[1], false); wf[s & 1][3] = pair(bytes[1], true); }
    }
  };

  // ---- products
  f32x16 acc[TT], total[TT];                            // I8: acc holds the bits of int32
#pragma unroll
  for (int i = 0; i < TT; ++i)
#pragma unroll
    for (int e = 0; e < 16; ++e) { acc[i][e] = 0.f; total[i][e] = 0.f; }
  auto add_scaled = [&](int i, float s) {
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      const float v = I8 ? (float)__float_as_int(acc[i][e]) : acc[i][e];
      total[i][e] = fmaf(s, v, total[i][e]);
    }
  };
  auto product = [&](int s, int i, bool first) {
    const f32x16 zero = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    const f32x16 c = first ? zero : acc[i];
    if (I8)
      acc[i] = __builtin_bit_cast(f32x16, __builtin_amdgcn_mfma_i32_32x32x32_i8(__builtin_bit_cast(i32x4, xf[s & 1][i]),
                                  __builtin_bit_cast(i32x4, wf[s & 1]), __builtin_bit_cast(i32x16, c), 0, 0, 0));
    else
      acc[i] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, xf[s & 1][i]), __builtin_bit_cast(bf16x8, wf[s & 1]), c, 0, 0, 0);
  };

  // Behind each of a step's matrix instructions: one fragment of the next step's activations, a share of its weights.  A group's sum goes
  // to the total just before the first instruction of the next group replaces it.
  float last_scale = 0.f;
  auto stage = [&](Codes& c, Codes& next, int k) {
#pragma unroll
    for (int s = 0; s < ST; ++s) {
      const bool first = GS && s % SPG == 0;
#pragma unroll
      for (int i = 0; i < TT; ++i) {
        if (first) add_scaled(i, s == 0 ? last_scale : c.scale[s == 0 ? 0 : s / SPG - 1]);
        product(s, i, first);
        __builtin_amdgcn_sched_barrier(0);
        if (s + 1 < ST) read_x(k, s + 1, i);
        else read_x(k + 1, 0, i);
#pragma unroll
        for (int part = i * (4 / TT); part < (i + 1) * (4 / TT); ++part) {
          if (s + 1 < ST) unpack(c, s + 1, part);
          else unpack(next, 0, part);
        }
        __builtin_amdgcn_sched_barrier(0);
      }
      if (s == ST / 2 - 1) {
        many_wait<NL>();                                // stage k + 1 is there: all but the youngest loads, those of stage k + 2
        many_barrier();
        load_x();
        __builtin_amdgcn_sched_barrier(0);
      }
    }
    if (GS) {
      last_scale = c.scale[NG - 1];
      asm volatile("" : "+v"(last_scale));              // (here, not behind the loads that replace it)
    }
    __builtin_amdgcn_sched_barrier(0);
    load_codes(c, k + 2);
    __builtin_amdgcn_sched_barrier(0);
  };
  Codes ca, cb;
  load_codes(ca, k_begin);
  load_codes(cb, k_begin + 1);
  __builtin_amdgcn_sched_barrier(0);
  load_x();
  load_x();
  load_x();
#pragma unroll
  for (int part = 0; part < 3; ++part) unpack(ca, 0, part);
  many_wait<2 * NL>();
  many_barrier();
#pragma unroll
  for (int i = 0; i < TT; ++i) read_x(k_begin, 0, i);
  int k = k_begin;
  for (; k + 1 < k_end; k += 2) {
    stage(ca, cb, k);
    stage(cb, ca, k + 1);
  }
  if (k < k_end) stage(ca, cb, k);
  if (!GS) last_scale = p.scales[group0];
#pragma unroll
  for (int i = 0; i < TT; ++i) add_scaled(i, last_scale);

  // ---- results: through LDS, so that a token's outputs leave in runs.  The lane has row l32 of a tile, tokens 8 (e / 4) + 4 half + e % 4.
  many_wait<0>();                                       // (no load writes to LDS from here on)
  many_barrier();
  float* out = reinterpret_cast<float*>(smem);
#pragma unroll
  for (int i = 0; i < TT; ++i)
#pragma unroll
    for (int e = 0; e < 16; ++e) out[(i * 32 + 8 * (e >> 2) + 4 * half + (e & 3)) * Tile::kOutRow + wave * 32 + l32] = total[i][e];
  __syncthreads();
  constexpr int RUNS = Tile::kRows / 8;                  // runs of eight rows
  const int col = tid % RUNS * 8, row = row0 + col;
  float b[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) b[e] = p.bias && p.parts == 1 && row + e < p.m ? p.bias[row + e] : 0.f;
  for (int t = tid / RUNS; t < Tile::kTokens; t += 64 * WV / RUNS) {
    const int tok = tok0 + t;
    if (tok >= p.tokens || row >= p.m) break;
    float v[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = out[t * Tile::kOutRow + col + e];
    if (p.parts > 1) {                                   // (whole runs: rows of p.partial have room for them)
      float* to = p.partial + ((int64_t)part * p.tokens + tok) * p.ld_partial + row;
      *reinterpret_cast<f32x4*>(to) = f32x4{v[0], v[1], v[2], v[3]};
      *reinterpret_cast<f32x4*>(to + 4) = f32x4{v[4], v[5], v[6], v[7]};
    } else {
      const float sx = I8 ? p.xs[tok] : 1.f;
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = I8 ? fmaf(v[e], sx, b[e]) : v[e] + b[e];
      linear_store(p, tok, row, v);
    }
  }
}

// The parts' sums of eight outputs of a token, in order.
__global__ __launch_bounds__(256) void linear_join_kernel(LinearArgs p) {
  const int runs = (int)(p.ld_partial / 8);
  const int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const int tok = (int)(at / runs), row = (int)(at % runs) * 8;
  if (tok >= p.tokens) return;
  f32x4 v[2] = {f32x4{0.f, 0.f, 0.f, 0.f}, f32x4{0.f, 0.f, 0.f, 0.f}};
  for (int k = 0; k < p.parts; ++k) {
    const float* from = p.partial + ((int64_t)k * p.tokens + tok) * p.ld_partial + row;
    v[0] += *reinterpret_cast<const f32x4*>(from);
    v[1] += *reinterpret_cast<const f32x4*>(from + 4);
  }
  const float sx = p.xs ? p.xs[tok] : 1.f;
  float y[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) y[e] = fmaf(v[e >> 2][e & 3], sx, p.bias && row + e < p.m ? p.bias[row + e] : 0.f);
  linear_store(p, tok, row, y);
}

template <bool I8, int GS, int TT, int WV> static hipError_t launch_many_as(const LinearArgs& p, hipStream_t s) {
  using Tile = ManyTile<TT, WV>;
  static LdsLimitOnce once;
  if (const hipError_t e = once.ensure((const void*)&linear_many_kernel<I8, GS, TT, WV>, Tile::kLds); e != hipSuccess) return e;
  const int tt = (p.tokens + Tile::kTokens - 1) / Tile::kTokens, rt = (p.m + Tile::kRows - 1) / Tile::kRows;
  hipLaunchKernelGGL((linear_many_kernel<I8, GS, TT, WV>), dim3((unsigned)((int64_t)tt * rt * p.parts)), dim3(64 * WV), Tile::kLds, s, p, tt, rt);
  if (const hipError_t e = hipGetLastError(); e != hipSuccess || p.parts == 1) return e;
  hipLaunchKernelGGL(linear_join_kernel, dim3((unsigned)((p.tokens * (p.ld_partial / 8) + 255) / 256)), dim3(256), 0, s, p);
  return hipGetLastError();
}
template <int TT, int WV> static hipError_t launch_many_of(const LinearArgs& p, int gs, bool i8, hipStream_t s) {
  switch (gs) {
    case 0: return i8 ? launch_many_as<true, 0, TT, WV>(p, s) : launch_many_as<false, 0, TT, WV>(p, s);
    case 1: return i8 ? launch_many_as<true, 1, TT, WV>(p, s) : launch_many_as<false, 1, TT, WV>(p, s);
    case 2: return i8 ? launch_many_as<true, 2, TT, WV>(p, s) : launch_many_as<false, 2, TT, WV>(p, s);
    default: return i8 ? launch_many_as<true, 4, TT, WV>(p, s) : launch_many_as<false, 4, TT, WV>(p, s);
  }
}

// Tile of a call: tiles of 32 tokens, and wavefronts.  Small tiles where the large ones are few: us a call with 128 x 256 / 64 x 128, bf16,
// tiles of the larger kind times 128 columns in brackets: 4096 x 4096, 65 tokens 20.0 / 16.8 (512), 384 31.2 / 30.7 (1536), 768 43.6 / 43.6 (3072), 2048 70 /
// 96 (8192); 4096 x 11008, 192 tokens 37.6 / 34.7 (2752), 384 49.9 / 61.4 (4128); 11008 x 4096, 128 tokens 30.4 / 31.4 (1376), 512 58.7 / 72.5 (5504);
// 4096 x 1024, 257 tokens 17.0 / 10.6 (384), 1024 19.2 / 16.4 (1024), 2048 23.2 / 28.5 (2048, 256 tiles); 8-bit activations a little more for the small ones.
static void many_tile(int64_t tokens, int64_t m, int64_t n, int& tt, int& wv) {
  const int64_t large = (tokens + 127) / 128 * ((m + 255) / 256), kt = (n + 127) / 128;
  tt = tokens <= 64 || (large <= 128 && large * kt <= 3072) ? 2 : 4;
  wv = tt == 4 ? 8 : 4;
}
// Parts that the columns are taken in: as many as leave room for 512 workgroups of four wavefronts (two a CU) or 256 of eight, of at least eight
// stages each (four up to 64 tokens, where joining them is cheap).  On 4096 x 4096, 11008 x 4096, 4096 x 11008, 28672 x 8192 and 1024 x 8192, 33 to 1024
// tokens: room for 256 (128) instead takes 1.0 to 1.7 times as long, for 1024 (512) 0.9 to 1.8 times.  Stages, 8 / 4: 4096 x 4096, 33 tokens 15.0 /
// 13.9, 4096 x 1024, 512 tokens 12.0 / 19.2, 1024 x 4096, 512 tokens 17.6 / 19.1.
static int64_t many_room(int tt) { return tt == 4 ? 256 : 512; }
static int64_t most_parts(int64_t tokens, int64_t n) { return (n + 127) / 128 / (tokens <= 64 ? 4 : 8); }
static int64_t many_parts(int64_t tokens, int64_t m, int64_t n) {
  int tt, wv;
  many_tile(tokens, m, n, tt, wv);
  const int64_t tiles = (tokens + 32 * tt - 1) / (32 * tt) * ((m + 32 * wv - 1) / (32 * wv)), most = most_parts(tokens, n);
  const int64_t want = many_room(tt) / tiles;
  return want < 1 || most < 1 ? 1 : want < most ? want : most;
}
// Room for the partial sums of every call with at most so many tokens: parts times tiles of tokens is at most room / tiles of rows.
size_t linear_partial_bytes(int64_t tokens, int64_t m, int64_t n) {
  const int64_t ld = (m + 7) / 8 * 8;
  int64_t rows = 0;                                        // of ld floats
  for (const int tt : {2, 4}) {
    const int64_t least = 16 * tt + 1, each = many_room(tt) / ((m + 64 * (tt == 4 ? 4 : 2) - 1) / (64 * (tt == 4 ? 4 : 2)));
    for (const int64_t t : {tokens < 64 ? tokens : (int64_t)64, tokens}) {
      if (t < least || each < 2 || most_parts(t, n) < 2) continue;
      const int64_t need = each * 32 * tt < most_parts(t, n) * t ? each * 32 * tt : most_parts(t, n) * t;
      rows = need > rows ? need : rows;
    }
  }
  return (size_t)(rows * ld) * 4;
}

hipError_t launch_linear_many(LinearArgs p, int gs, bool i8, float* partial, hipStream_t s) {
  int tt, wv;
  many_tile(p.tokens, p.m, (int64_t)p.kt * 128, tt, wv);
  p.parts = (int32_t)many_parts(p.tokens, p.m, (int64_t)p.kt * 128);
  p.partial = partial;
  p.ld_partial = (p.m + 7) / 8 * 8;
  return tt == 2 ? launch_many_of<2, 4>(p, gs, i8, s) : launch_many_of<4, 8>(p, gs, i8, s);
}

}  // namespace gptaq
