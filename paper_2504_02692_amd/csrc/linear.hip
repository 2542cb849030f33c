// y = x W^T + bias for layers whose weights the solve has quantised: W[r][j] = scale[r][g] * (code[r][j] - zero[r][g]), g the group
// of column j, codes of at most 4 bits.
//
// code - zero is an integer between -15 and 15, exact in bfloat16 and in 8 bits, so the matrix instructions multiply exact weights:
// per group of columns the sum of (code - zero) x is taken in fp32 (bf16 activations) or exactly in int32 (8-bit activations),
// multiplied by the group's fp32 scale, and added to the fp32 total.  No weight is rounded.  With up to 16 tokens, many rows, and bf16 in and
// out it is the sum of (16 + code) x less (16 + zero) times that of x: exact weights too, but larger sums (linear_few_kernel).
#include "linear.h"
#include <type_traits>

namespace gptaq {

typedef __attribute__((ext_vector_type(4))) int32_t i32x4;

// ---- laying out the weights

__global__ __launch_bounds__(256) void linear_pack_codes_kernel(const uint8_t* codes, int64_t ldc, int m, int n, int kt, uint32_t* out,
                                                                int32_t* info) {
  const int tile_c = blockIdx.x % kt, tile_r = blockIdx.x / kt;
  const int lane = threadIdx.x >> 2, i = threadIdx.x & 3;
  const int row = tile_r * 16 + (lane & 15), col = tile_c * 128 + i * 32 + (lane >> 4) * 8;
  uint32_t w = 0, all = 0;
  if (row < m) {
    const uint8_t* c = codes + (int64_t)row * ldc;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const uint32_t v = col + j < n ? c[col + j] : 0u;
      all |= v;
      w |= (v & 15u) << (j < 4 ? 8 * j : 8 * (j - 4) + 4);
    }
  }
  out[(int64_t)blockIdx.x * 256 + threadIdx.x] = w;
  if (all > 15u) atomicMax(info, row + 1);
}

__global__ __launch_bounds__(256) void linear_pack_groups_kernel(const float* scales, const float* zeros, int m, int given, int groups,
                                                                 int64_t count, float* out_scales, uint8_t* out_zeros, int32_t* info) {
  const int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (at >= count) return;
  const int64_t g = at / 16 % groups, row = at / 16 / groups * 16 + at % 16;
  float s = 0.f, z = 0.f;
  if (row < m && g < given) {
    s = scales[row * given + g];
    z = zeros[row * given + g];
  }
  if (!(z >= 0.f && z <= 15.f && z == rintf(z))) { atomicMax(info, (int)row + 1); z = 0.f; }
  out_scales[at] = s;
  out_zeros[at] = (uint8_t)z;
}

// info, and the bytes between the end of the zeros and that of the weights (less than 256)
__global__ void linear_clear_kernel(int32_t* info, uint8_t* tail, int count) {
  if (threadIdx.x == 0) *info = 0;
  if ((int)threadIdx.x < count) tail[threadIdx.x] = 0;
}

// ---- activations that the products cannot read as they are: columns in another order, rows that do not start at 16 bytes or end
// inside a piece of 16.  Rows of `out` have `ldo` elements, zeros behind the n-th.  A workgroup a row, each thread's loads one behind the other: 5 us for
// one row of 4096, 18 to 19 for one to 2048 rows of 8192 or 11008, latency throughout; more than the product of few tokens behind it.
template <typename T>
__global__ __launch_bounds__(256) void linear_gather_kernel(const T* x, int64_t ldx, const int32_t* perm, int n, T* out, int64_t ldo) {
  const T* row = x + (int64_t)blockIdx.x * ldx;
  T* to = out + (int64_t)blockIdx.x * ldo;
  for (int c = threadIdx.x; c < (int)ldo; c += 256) {
    const int from = c < n ? (perm ? perm[c] : c) : -1;
    to[c] = (uint32_t)from < (uint32_t)n ? row[from] : T(0);
  }
}

// ---- few tokens
//
// TT = 1 or 2 tiles of v_mfma 16x16: 16 or 32 tokens at a time.  A workgroup takes RT tiles of 16 rows; its wavefronts share the tiles of 128 columns out
// among themselves and add their sums through LDS, in the wavefronts' order.  The weights go straight from memory to the lanes that
// feed the matrix unit, two tiles of columns ahead (three or four ahead were slower: registers): nothing of W is read twice, and with everything of a
// wavefront independent many loads are in flight.  The left operand is 16 tokens (lane l: token l % 16), the right 16 rows of W (lane l: row l % 16), the
// result has the row of W in l % 16 and tokens 4 (l / 16) .. + 3 in the lane's four values, so one scale per lane serves a result.
// Bound by the weights' bytes where there are many: 28672 x 8192, one token, 8-bit activations 23 to 25 us, 5.0 to 5.4 TB/s; bf16 26 to 31 us, where unpacking the codes
// takes most of the time that the bytes leave.  4096 x 4096 4.3 us, 2.1 TB/s: the launch, one trip to memory and the join.
// Activations go to LDS in runs of a token's whole 128 columns, to a place of the wavefront's own, so that no wavefront waits for another.  (A load of
// 16 tokens by 64 bytes to registers takes about four times as long as one of 1 KB in one run: 4096 x 11008, 16 tokens, 14.5 us; through LDS 9.2.)
// GS: groups per 128 columns (1, 2, 4), 0: one group per row.

// Most wavefronts of a workgroup: 16 leave a lane 128 registers.
constexpr int few_waves(int gs, int rt, int tt) { return rt > 1 || tt > 1 || gs == 4 ? 8 : 16; }

template <bool I8, int GS, int RT, int TT>
__global__ __launch_bounds__(64 * few_waves(GS, RT, TT)) void linear_few_kernel(LinearArgs p) {
  extern __shared__ __attribute__((aligned(256))) float lds[];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), waves = blockDim.x >> 6;
  const int l16 = lane & 15, q = lane >> 4;
  const int rt0 = blockIdx.x * RT, tok0 = blockIdx.y * TT * 16, tokens = min(p.tokens - tok0, TT * 16);
  constexpr int G = GS ? GS : 1;       // groups per tile of 128 columns

  f32x4 total[TT][RT], acc[TT][RT];    // I8: acc holds the bits of int32
  const uint8_t* codes[RT];
  int64_t group[RT];
#pragma unroll
  for (int r = 0; r < RT; ++r) {
    const int64_t tr = rt0 + r < p.mt ? rt0 + r : p.mt - 1;      // (past the last tile of rows: that one again; nothing of it is stored)
    codes[r] = p.codes + tr * p.kt * 1024 + lane * 16;
    group[r] = tr * p.groups * 16 + l16;
  }
  // The 16-byte chunks of a token's 128 columns are permuted so that 16 tokens' same chunk lies in 16 different places of 256 bytes.  Places of
  // tokens that there are not hold anything: their results are not stored.
  constexpr int XROW = I8 ? 128 : 256, XSTAGE = TT * 16 * XROW, CHUNKS = XROW / 16, PER_LOAD = 1024 / XROW, NL = TT * 16 / PER_LOAD;
  auto swizzle = [](int row) { return I8 ? (row >> 1) & 7 : row & 15; };
  unsigned char* const xlds = reinterpret_cast<unsigned char*>(lds) + wave * 2 * XSTAGE;
  const LdsLoader xfrom((const unsigned char*)p.x + (int64_t)tok0 * p.ldx * (I8 ? 1 : 2));
  int xsrc[NL];
#pragma unroll
  for (int j = 0; j < NL; ++j) {
    const int row = j * PER_LOAD + lane / CHUNKS;
    xsrc[j] = min(row, tokens - 1) * (int)p.ldx * (I8 ? 1 : 2) + ((lane % CHUNKS ^ swizzle(row)) << 4);
  }

  struct Stage { u32x4 w[RT]; uint32_t zero[RT][G]; float scale[RT][G]; };
  auto load = [&](Stage& s, int k, int place) {
    // The activations first: where the weights are there, so are they.  The place's last reads are over.
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt(0xc07f);          // lgkmcnt == 0
#pragma unroll
    for (int j = 0; j < NL; ++j)
      if (j == 0 || j * PER_LOAD < tokens) xfrom.load(xlds + place * XSTAGE + j * 1024, xsrc[j], __builtin_amdgcn_readfirstlane(k * XROW));
    asm volatile("" ::: "memory");
#pragma unroll
    for (int r = 0; r < RT; ++r) {
      if (GS) {
#pragma unroll
        for (int g = 0; g < G; ++g) {
          s.zero[r][g] = p.zeros[group[r] + (int64_t)(k * GS + g) * 16];
          s.scale[r][g] = p.scales[group[r] + (int64_t)(k * GS + g) * 16];
        }
      }
      s.w[r] = *reinterpret_cast<const u32x4*>(codes[r] + (int64_t)k * 1024);
    }
  };
  uint32_t row_zero[RT];
  if (!GS) {
#pragma unroll
    for (int r = 0; r < RT; ++r) row_zero[r] = p.zeros[group[r]];
  }
  const u32x4 ones = {0x3f803f80u, 0x3f803f80u, 0x3f803f80u, 0x3f803f80u};
  uint32_t sixteen = 0x41804180u;
  asm volatile("" : "+v"(sixteen));    // (in a register, where the mask and it are one instruction)
  f32x4 accx[TT];                      // sums of the group's activations (the same in all of a token's lanes)
  // EXACT: the products are those of code - zero.  Else: of 16 + code, which is two instructions for two codes where the difference takes
  // five, and (16 + zero) times the activations' sum, one more matrix instruction for all RT, is taken off each group's sum, of a group as long as the row
  // off each 128 columns': what is subtracted stays below 31 times the 128 columns' sum |x|, so its rounding does, and does not grow with the row.
  // A bf16 output's own rounding hides that; outputs in fp32 are EXACT, and where a result is not finite the subtraction may be why, and the workgroup takes
  // its sums again with EXACT.
  // One matrix instruction for an operand (TT 1) and one sum of activations for several operands (RT) is where it pays: us a call, EXACT / else, one token:
  // 28672 x 8192 33 / 29 (groups of 32 40 / 41), 22016 x 4096 15.9 / 12.9, 11008 x 4096 10.3 / 9.1; RT 1: 4096 x 11008 7.7 / 7.8, 16 tokens 9.2 / 9.7; TT 2, 32 tokens:
  // 4096 x 11008 13.1 / 14.3, 11008 x 4096 13.5 / 14.0, 28672 x 8192 42 / 49 (registers spill).
  constexpr bool kSixteen = !I8 && TT == 1 && RT > 1;
  auto add_scaled = [&](auto exact, int r, float s, uint32_t zero) {
    const float z = -16.f - (float)zero;
#pragma unroll
    for (int t = 0; t < TT; ++t)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        float v = I8 ? (float)__float_as_int(acc[t][r][e]) : acc[t][r][e];
        if (!exact) v = fmaf(z, accx[t][e], v);
        total[t][r][e] = fmaf(s, v, total[t][r][e]);
      }
  };
  auto multiply = [&](auto exact, const Stage& s, int place) {
    const f32x4 nothing = {0.f, 0.f, 0.f, 0.f};
    asm volatile("" :: "v"(s.w[RT - 1]) : "memory");
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      constexpr bool kGrouped = GS || !decltype(exact)::value;       // (else the sum runs over the row)
      const bool first = kGrouped && i % (4 / G) == 0, last = kGrouped && (i + 1) % (4 / G) == 0;
      u32x4 x[TT];
#pragma unroll
      for (int t = 0; t < TT; ++t) {
        const unsigned char* row = xlds + place * XSTAGE + (t * 16 + l16) * XROW;
        if (I8) {
          const u32x2 v = *reinterpret_cast<const u32x2*>(row + (((2 * i + (q >> 1)) ^ swizzle(l16)) << 4) + (q & 1) * 8);
          x[t] = u32x4{v[0], v[1], 0u, 0u};
        } else {
          x[t] = *reinterpret_cast<const u32x4*>(row + (((4 * i + q) ^ swizzle(l16)) << 4));
        }
      }
      if (!exact) {
#pragma unroll
        for (int t = 0; t < TT; ++t) {  // columns 0 2 4 6 1 3 5 7, as the codes come out of a word
          x[t] = u32x4{__builtin_amdgcn_perm(x[t][1], x[t][0], 0x05040100u), __builtin_amdgcn_perm(x[t][3], x[t][2], 0x05040100u),
                       __builtin_amdgcn_perm(x[t][1], x[t][0], 0x07060302u), __builtin_amdgcn_perm(x[t][3], x[t][2], 0x07060302u)};
          accx[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, x[t]), __builtin_bit_cast(bf16x8, ones), first ? nothing : accx[t], 0, 0, 0);
        }
      }
#pragma unroll
      for (int r = 0; r < RT; ++r) {
        const uint32_t w = s.w[r][i], zero = GS ? s.zero[r][i * G / 4] : row_zero[r];
        u32x4 v;                         // the right operand (I8: two words)
        if (I8) {
          const u32x2 b = linear_bytes(w, linear_offset(zero));
          v[0] = b[0]; v[1] = b[1];
        } else if (exact) {
          v = __builtin_bit_cast(u32x4, linear_bf16(w, linear_offset(zero)));
        } else {                         // the code in the upper bits of the mantissa of 16
          const uint32_t shifted[4] = {w << 3, w >> 1, w >> 5, w >> 9};
#pragma unroll
          for (int e = 0; e < 4; ++e) v[e] = (shifted[e] & 0x00780078u) | sixteen;
        }
#pragma unroll
        for (int t = 0; t < TT; ++t) {
          const f32x4 c = first ? nothing : acc[t][r];
          if (I8)
            acc[t][r] = __builtin_bit_cast(f32x4, __builtin_amdgcn_mfma_i32_16x16x32_i8(__builtin_bit_cast(long, u32x2{x[t][0], x[t][1]}),
                                                  __builtin_bit_cast(long, u32x2{v[0], v[1]}), __builtin_bit_cast(i32x4, c), 0, 0, 0));
          else
            acc[t][r] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, x[t]), __builtin_bit_cast(bf16x8, v), c, 0, 0, 0);
        }
        if (last) add_scaled(exact, r, GS ? s.scale[r][i * G / 4] : 1.f, zero);
      }
    }
  };
  auto sums = [&](auto exact) {
#pragma unroll
    for (int t = 0; t < TT; ++t) {
      accx[t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int r = 0; r < RT; ++r) total[t][r] = acc[t][r] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    Stage a, b, c;
    int k = wave;                      // (a workgroup has no more wavefronts than there are tiles)
    load(a, k, 0);
    if (k + waves < p.kt) load(b, k + waves, 1);
    for (; k + 3 * waves < p.kt; k += 2 * waves) {
      multiply(exact, a, 0);
      load(a, k + 2 * waves, 0);
      multiply(exact, b, 1);
      load(b, k + 3 * waves, 1);
    }
    multiply(exact, a, 0);
    if (k + 2 * waves < p.kt) load(c, k + 2 * waves, 0);
    if (k + waves < p.kt) multiply(exact, b, 1);
    if (k + 2 * waves < p.kt) multiply(exact, c, 0);
    __syncthreads();                   // (the sums go where other wavefronts' activations are)
    if (!GS) {
#pragma unroll
      for (int r = 0; r < RT; ++r) {
        const float s = p.scales[group[r]];
        if (exact) add_scaled(exact, r, s, row_zero[r]);
#pragma unroll
        for (int t = 0; t < TT; ++t)
          if (!exact) total[t][r] *= s;
      }
    }
  };
  // Joins the wavefronts' sums, [wave][t][r][lane][4], and stores those of this thread's results that `wanted` has a bit for; returns which are not
  // finite.  (A second pass replaces these alone: the other tokens' results do not depend on them.)
  auto finish = [&](uint64_t wanted) {
#pragma unroll
    for (int t = 0; t < TT; ++t)
#pragma unroll
      for (int r = 0; r < RT; ++r) *reinterpret_cast<f32x4*>(&lds[(((wave * TT + t) * RT + r) * 64 + lane) * 4]) = total[t][r];
    __syncthreads();
    uint64_t lost = 0;
    int bit = 0;
    for (int at = threadIdx.x; at < TT * RT * 256; at += blockDim.x, ++bit) {
      // 16 RT rows of W in a run of threads, so that a token's outputs are written together
      const int r = at % (16 * RT), tok = at / (16 * RT), row = rt0 * 16 + r;
      if (row >= p.m || tok >= tokens || !(wanted >> bit & 1)) continue;
      const int slot = (((tok >> 4) * RT + (r >> 4)) * 64 + (tok & 15) / 4 * 16 + (r & 15)) * 4 + (tok & 3);
      float v = 0.f;
      for (int w = 0; w < waves; ++w) v += lds[w * TT * RT * 256 + slot];
      if (!(fabsf(v) < __builtin_inff())) lost |= 1ull << bit;
      if (I8) v *= p.xs[tok0 + tok];
      if (p.bias) v += p.bias[row];
      const int64_t o = (int64_t)(tok0 + tok) * p.ldy + row;
      if (p.y_f32) ((float*)p.y)[o] = v;
      else ((uint16_t*)p.y)[o] = __builtin_bit_cast(uint16_t, (__bf16)v);
    }
    return lost;
  };
  static_assert(TT * RT * 256 / 64 <= 64, "a bit for each of a thread's results");
  uint64_t wanted = ~0ull;
  if constexpr (kSixteen) {
    if (!p.y_f32) {
      sums(std::false_type{});
      wanted = finish(wanted);
      if (!__syncthreads_or(wanted != 0)) return;
    }
  }
  sums(std::true_type{});
  finish(wanted);
}

template <bool I8, int GS, int RT, int TT>
static hipError_t launch_few_as(const LinearArgs& p, int waves, hipStream_t s) {
  if (waves > few_waves(GS, RT, TT)) waves = few_waves(GS, RT, TT);
  while (waves > 1 && waves > p.kt) waves /= 2;
  constexpr int kStages = 2 * TT * 16 * (I8 ? 128 : 256), kSums = TT * RT * 1024, kPerWave = kStages > kSums ? kStages : kSums;
  static LdsLimitOnce once;
  if (const hipError_t e = once.ensure((const void*)&linear_few_kernel<I8, GS, RT, TT>, few_waves(GS, RT, TT) * kPerWave); e != hipSuccess) return e;
  hipLaunchKernelGGL((linear_few_kernel<I8, GS, RT, TT>), dim3((unsigned)((p.mt + RT - 1) / RT), (unsigned)((p.tokens + TT * 16 - 1) / (TT * 16))), dim3(64 * waves), (size_t)(waves * kPerWave), s, p);
  return hipGetLastError();
}
// Tiles of rows per workgroup: the more, the less often the activations are read, the fewer workgroups.  us a call, RT 1 (8 wavefronts) / 2 (4, 8) / 4 (4):
//              4096 x 4096          11008 x 4096               8192 x 8192                28672 x 8192
//   1, bf16    4.3 / 7.1 5.5 / 8.8  8.4 / 8.6  8.3  / 9.2      10.4 / 12.0 9.4 / 15.6     34.4 / 28.3 28.7 / 27.2
//   1, int8    3.4 / 5.7 4.6 / 7.6  6.6 / 7.0  7.2  / 8.2      8.1 / 9.4  8.1  / 13.1     23.3 / 25.3 24.4 / 25.1
//   16, bf16   5.2 / 7.8 6.2 / 10   9.7 / 10.0 9.8  / 10.8     12.1 / 13.2 10.7 / 17.5    44.7 / 37.0 37.0 / 31.8
//   16, int8   3.7 / 6.1 4.9 / 8.6  6.8 / 7.6  7.8  / 9.4      8.6 / 10.1 8.7  / 14.2     32.8 / 28.1 28.1 / 27.4
//   32, bf16   6.8 / 9.9 8.3 / 15   16.5 / 13.6 15.4 / 15.2    18.4 / 16.6 13.7 / 24.4    73.9 / 50.5 54.2 / 42.8
//   32, int8   5.2 / 7.8 6.2 / 11   9.4 / 9.8  9.6  / 12.0     10.9 / 12.6 10.5 / 18.7    43.0 / 35.5 35.2 / 32.5
// 16 wavefronts instead of 8, RT 1, one token: 4096 x 11008 8.3 -> 7.6, 1024 x 8192 5.7 -> 5.3, 4096 x 4096 4.4 -> 4.2, 11008 x 4096 8.3 -> 10.5.
// With more scales a tile, fewer tiles fit in the registers: 242 of 256 with two groups a tile (RT 4, one tile of tokens), 208 with one group and two tiles of tokens.
template <bool I8, int GS, int TT>
static hipError_t launch_few_rows(const LinearArgs& p, hipStream_t s) {
  constexpr int kMost = GS <= 1 ? 4 : GS == 2 ? (TT == 1 ? 4 : 2) : (TT == 1 ? 2 : 1), kTwo = kMost < 2 ? kMost : 2;
  if (p.mt >= 1024 && !(I8 && p.tokens <= 8)) return launch_few_as<I8, GS, kMost, TT>(p, kMost == 1 ? 8 : 4, s);
  if constexpr (!I8)
    if (p.mt >= 512) return launch_few_as<I8, GS, kTwo, TT>(p, kTwo == 1 || p.kt >= 64 ? 8 : 4, s);
  return launch_few_as<I8, GS, 1, TT>(p, p.mt < 512 && p.kt >= 64 ? 16 : 8, s);
}
template <bool I8, int GS>
static hipError_t launch_few_of(const LinearArgs& p, hipStream_t s) {
  return p.tokens <= 16 ? launch_few_rows<I8, GS, 1>(p, s) : launch_few_rows<I8, GS, 2>(p, s);
}
template <bool I8>
static hipError_t launch_few(const LinearArgs& p, int gs, hipStream_t s) {
  return gs == 0 ? launch_few_of<I8, 0>(p, s) : gs == 1 ? launch_few_of<I8, 1>(p, s) : gs == 2 ? launch_few_of<I8, 2>(p, s) : launch_few_of<I8, 4>(p, s);
}

// Above 32 tokens, in blocks of 32, as far as few workgroups have the work: us a call with this kernel / with that for many tokens, bf16 (workgroups times
// tiles of columns): 4096 x 4096, 64 tokens 11.8 / 14.5 (512 x 32), 96 16.7 / 16.4; 1024 x 8192, 128 tokens 9.8 / 16.3 (256 x 64), 192 17.6 / 16.7;
// 2048 x 2048, 192 tokens 10.9 / 13.5 (768 x 16), 256 15.2 / 15.0; 4096 x 11008, 64 tokens 23.9 / 22.7 (512 x 86).  8-bit: 4096 x 4096, 128 tokens 12.9 / 14.6
// (1024 x 32), 256 22.2 / 19.0; 4096 x 11008, 64 tokens 14.1 / 19.4 (512 x 86), 128 26.2 / 20.8; 4096 x 1024, 128 tokens 5.7 / 6.6 (1024 x 8), 192 7.8 / 6.7.
static bool few_tokens(const LinearArgs& p, bool i8) {
  const int64_t workgroups = (int64_t)p.mt * ((p.tokens + 31) / 32);
  return p.tokens <= 32 || (workgroups <= (i8 ? 1280 : 768) && workgroups * p.kt <= (i8 ? 49152 : 16384));
}

static hipError_t launch_linear(const LinearArgs& p, int gs, bool i8, float* partial, hipStream_t s) {
  if (!few_tokens(p, i8)) return launch_linear_many(p, gs, i8, partial, s);
  return i8 ? launch_few<true>(p, gs, s) : launch_few<false>(p, gs, s);
}

// ---- argument checks

constexpr int64_t kMaxSide = (int64_t)1 << 20, kMaxTokens = (int64_t)1 << 23, kMaxTiles = (int64_t)1 << 23;
// (A workgroup a tile lays the weights out, and a grid has less than 2^32 threads.)
static bool good_size(int64_t m, int64_t n) {
  return m > 0 && n > 0 && m <= kMaxSide && n <= kMaxSide && ((m + 15) / 16) * ((n + 127) / 128) <= kMaxTiles;
}
static bool good_group(int64_t n, int group) {
  return group <= 0 || ((group == 32 || group == 64 || group == 128) && n % group == 0);
}
// Elements of a row of activations in the workspace: whole tiles of columns.
static int64_t padded_columns(int64_t n) { return (n + 127) / 128 * 128; }

static size_t gather_bytes(int64_t tokens, int64_t n) { return ((size_t)tokens * padded_columns(n) * 2 + 255) / 256 * 256; }

static int run_linear(bool i8, const void* X, const float* xs, int64_t tokens, int64_t ldx, const int32_t* perm, const void* weights, size_t weights_bytes,
                      int64_t m, int64_t n, int group, const float* bias, void* Y, int64_t ldy, int y_f32, void* ws, size_t ws_bytes, void* stream) {
  if (!weights || (tokens != 0 && (!X || !Y || !ws || (i8 && !xs)))) return GPTAQ_ENULL;      // (no tokens: nothing to point to)
  const uintptr_t y_align = y_f32 ? 3 : 1;
  if (tokens < 0 || tokens > kMaxTokens || !good_size(m, n) || ldx < n || ldy < m ||
      ((uintptr_t)weights & 255) || ((uintptr_t)Y & y_align) || (!i8 && ((uintptr_t)X & 1)) || (((uintptr_t)xs | (uintptr_t)bias | (uintptr_t)perm) & 3))
    return GPTAQ_EDIM;
  if (!good_group(n, group)) return GPTAQ_EUNSUPPORTED;
  if (weights_bytes < linear_layout(m, n, group > 0 ? group : 0).bytes) return GPTAQ_EWORKSPACE;
  if (tokens == 0) return GPTAQ_OK;
  if (((uintptr_t)ws & 255) || ws_bytes < gptaq_linear_workspace_bytes(tokens, m, n)) return GPTAQ_EWORKSPACE;
  if (group < 0) group = 0;
  const LinearLayout l = linear_layout(m, n, group);
  const hipStream_t s = (hipStream_t)stream;
  LinearArgs p{};
  p.x = X; p.xs = xs; p.ldx = ldx;
  p.codes = (const uint8_t*)weights;
  p.scales = (const float*)(p.codes + l.scales);
  p.zeros = p.codes + l.zeros;
  p.bias = bias; p.y = Y; p.ldy = ldy; p.y_f32 = y_f32 ? 1 : 0;
  p.tokens = (int32_t)tokens; p.m = (int32_t)m; p.n = (int32_t)n;
  p.mt = (int32_t)l.mt; p.kt = (int32_t)l.kt; p.groups = (int32_t)l.groups;
  if (perm || n % 128 || ldx % (i8 ? 16 : 8) || ((uintptr_t)X & 15) || ldx * (i8 ? 1 : 2) > kManyMaxRow) {
    const int64_t ld = padded_columns(n);
    if (i8) hipLaunchKernelGGL(linear_gather_kernel<int8_t>, dim3((unsigned)tokens), dim3(256), 0, s, (const int8_t*)X, ldx, perm, (int)n, (int8_t*)ws, ld);
    else hipLaunchKernelGGL(linear_gather_kernel<uint16_t>, dim3((unsigned)tokens), dim3(256), 0, s, (const uint16_t*)X, ldx, perm, (int)n, (uint16_t*)ws, ld);
    GPTAQ_LAUNCH_CHECK();
    p.x = ws; p.ldx = ld;
    p.n = (int32_t)ld;                 // (the columns behind n are zeros here)
  }
  float* const partial = (float*)((uint8_t*)ws + gather_bytes(tokens, n));
  // A grid has less than 2^32 threads: more tokens than that takes are several launches.
  const int64_t most = (((int64_t)1 << 22) / p.mt) * 64;
  for (int64_t first = 0; first < tokens; first += most) {
    LinearArgs part = p;
    part.tokens = (int32_t)(tokens - first < most ? tokens - first : most);
    part.x = (const uint8_t*)p.x + first * p.ldx * (i8 ? 1 : 2);
    part.y = (uint8_t*)p.y + first * p.ldy * (y_f32 ? 4 : 2);
    if (i8) part.xs = p.xs + first;
    if (const hipError_t e = launch_linear(part, group ? 128 / group : 0, i8, partial, s); e != hipSuccess) { set_last_hip_error(e); return GPTAQ_ELAUNCH; }
  }
  return GPTAQ_OK;
}

}  // namespace gptaq

using namespace gptaq;

extern "C" size_t gptaq_linear_weights_bytes(int64_t m, int64_t n, int group) {
  if (!good_size(m, n) || !good_group(n, group)) return 0;
  return linear_layout(m, n, group > 0 ? group : 0).bytes;
}

extern "C" int gptaq_linear_pack(const uint8_t* codes, int64_t ldc, const float* scales, const float* zeros, int64_t m, int64_t n, int group,
                                 void* weights, size_t weights_bytes, int32_t* info, void* stream) {
  if (!codes || !scales || !zeros || !weights || !info) return GPTAQ_ENULL;
  if (!good_size(m, n) || ldc < n || (((uintptr_t)scales | (uintptr_t)zeros | (uintptr_t)info) & 3)) return GPTAQ_EDIM;
  if (!good_group(n, group)) return GPTAQ_EUNSUPPORTED;
  const LinearLayout l = linear_layout(m, n, group > 0 ? group : 0);
  if (((uintptr_t)weights & 255) || weights_bytes < l.bytes) return GPTAQ_EWORKSPACE;
  const hipStream_t s = (hipStream_t)stream;
  uint8_t* to = (uint8_t*)weights;
  const size_t end = l.zeros + (size_t)(l.mt * l.groups) * 16;
  hipLaunchKernelGGL(linear_clear_kernel, dim3(1), dim3(256), 0, s, info, to + end, (int)(l.bytes - end));
  hipLaunchKernelGGL(linear_pack_codes_kernel, dim3((unsigned)(l.mt * l.kt)), dim3(256), 0, s, codes, ldc, (int)m, (int)n, (int)l.kt,
                     (uint32_t*)to, info);
  const int64_t count = l.mt * l.groups * 16;
  hipLaunchKernelGGL(linear_pack_groups_kernel, dim3((unsigned)((count + 255) / 256)), dim3(256), 0, s, scales, zeros, (int)m,
                     (int)(group > 0 ? n / group : 1), (int)l.groups, count, (float*)(to + l.scales), to + l.zeros, info);
  GPTAQ_LAUNCH_CHECK();
  return GPTAQ_OK;
}

extern "C" size_t gptaq_linear_workspace_bytes(int64_t tokens, int64_t m, int64_t n) {
  if (tokens <= 0 || tokens > kMaxTokens || !good_size(m, n)) return 0;
  return gather_bytes(tokens, n) + (linear_partial_bytes(tokens, m, n) + 255) / 256 * 256;
}

extern "C" int gptaq_linear(const uint16_t* X, int64_t tokens, int64_t ldx, const int32_t* perm, const void* weights, size_t weights_bytes,
                            int64_t m, int64_t n, int group, const float* bias, void* Y, int64_t ldy, int y_f32, void* ws, size_t ws_bytes, void* stream) {
  return run_linear(false, X, nullptr, tokens, ldx, perm, weights, weights_bytes, m, n, group, bias, Y, ldy, y_f32, ws, ws_bytes, stream);
}

extern "C" int gptaq_linear_i8(const int8_t* X, const float* x_scales, int64_t tokens, int64_t ldx, const int32_t* perm, const void* weights,
                               size_t weights_bytes, int64_t m, int64_t n, int group, const float* bias, void* Y, int64_t ldy, int y_f32, void* ws, size_t ws_bytes,
                               void* stream) {
  return run_linear(true, X, x_scales, tokens, ldx, perm, weights, weights_bytes, m, n, group, bias, Y, ldy, y_f32, ws, ws_bytes, stream);
}
