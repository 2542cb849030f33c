// y = x W^T for many tokens: matrix products with weights that are made from their 4-bit codes on the way.
#include "linear.h"

namespace gptaq {

typedef __attribute__((ext_vector_type(4))) int32_t i32x4;
typedef __attribute__((ext_vector_type(16))) int32_t i32x16;

// A workgroup of eight wavefronts takes 128 tokens x 256 rows of W; a wavefront 64 x 64 of it as 2 x 2 results of
// v_mfma 32x32, twice: the sum of the current group of columns and the fp32 total it is scaled into.  These 128 registers a lane
// are what limits the tile.  A byte of W feeds four times the products that a byte of bf16 activations does, so the tile is
// taller in W: 24 KB come in for every 64 columns of bf16.
// A stage is 128 bytes of each row (64 columns of bf16, 128 of int8): activations go from memory straight to LDS, codes to
// registers, code - zero from there to LDS, once per workgroup.  Rings of three stages, one barrier a stage, in its middle: it
// publishes the next stage (whose first fragments are read before the stage ends) and retires the one before.
constexpr int kManyTokens = 128, kManyRows = 256;
constexpr int kXStage = kManyTokens * 128, kWStage = kManyRows * 128, kRing = 3;
constexpr int kManyLds = kRing * (kXStage + kWStage);

__device__ __forceinline__ void many_barrier() {          // no memory fence: loads stay in flight across it
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}
template <int N> __device__ __forceinline__ void many_wait() {      // vmcnt <= N, lgkmcnt == 0
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt((N & 15) | ((N >> 4) << 14) | (7 << 4));
}

template <bool I8, int GS>
__global__ __launch_bounds__(512, 2) void linear_many_kernel(LinearArgs p, int token_tiles, int row_tiles) {
  extern __shared__ __attribute__((aligned(128))) unsigned char smem[];
  constexpr int NST = I8 ? 1 : 2;                       // stages per 128 columns
  constexpr int WPS = I8 ? 4 : 2;                       // words of a tile per stage
  constexpr int SPG = GS ? 4 * NST / GS : 0;            // steps (four a stage) per group
  constexpr int NG = GS ? GS : 1;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int l32 = lane & 31, half = lane >> 5, l16 = lane & 15, q = lane >> 4;
  const int tile_t = blockIdx.x % token_tiles, tile_r = blockIdx.x / token_tiles;
  const int tok0 = tile_t * kManyTokens, row0 = tile_r * kManyRows;
  const int wt = (wave & 1) * 64, wr = (wave >> 1) * 64;
  unsigned char* const xs_lds = smem + kRing * kWStage;

  // ---- activations: the wavefront's 16 rows of a stage in two loads of 1 KB.  LDS rows are 128 bytes, their 16-byte chunks
  // permuted so that 16 consecutive rows of one chunk lie in 16 different places of two rows' 256 bytes (all banks once).
  const unsigned char* xsrc[2];
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    const int row = wave * 16 + j * 8 + (lane >> 3), chunk = (lane & 7) ^ ((row >> 1) & 7);
    const int tok = tok0 + row < p.tokens ? tok0 + row : p.tokens - 1;         // (their results are not stored)
    xsrc[j] = (const unsigned char*)p.x + (int64_t)tok * p.ldx * (I8 ? 1 : 2) + chunk * 16;
  }
  const int nstage = p.kt * NST;
  int xload = 0, xslot = 0;                             // next stage to load, its place
  auto load_x = [&]() {
#pragma unroll
    for (int j = 0; j < 2; ++j)
      __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)xsrc[j],
                                       (__attribute__((address_space(3))) void*)(xs_lds + xslot * kXStage + wave * 2048 + j * 1024), 16, 0, 0);
    ++xload;
    xslot = xslot == kRing - 1 ? 0 : xslot + 1;
    const int step = xload < nstage ? 128 : 0;          // (behind the last stage it is loaded again, so that the counts stay the same)
    xsrc[0] += step;
    xsrc[1] += step;
  };

  // ---- weights: the wavefront unpacks two tiles of 16 rows
  const uint8_t* csrc[2];
  int64_t zat[2], sat[2];
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    int tr = row0 / 16 + wave * 2 + j;
    tr = tr < p.mt ? tr : p.mt - 1;
    csrc[j] = p.codes + (int64_t)tr * p.kt * 1024 + lane * 16;
    zat[j] = (int64_t)tr * p.groups * 16 + l16;
    int sr = (row0 + wr + j * 32 + l32) / 16;           // the results' rows
    sr = sr < p.mt ? sr : p.mt - 1;
    sat[j] = (int64_t)sr * p.groups * 16 + l16;
  }
  struct Codes { u32x4 w[2]; uint32_t z[2][NG]; };
  auto load_codes = [&](Codes& c, int k) {
    k = k < p.kt ? k : p.kt - 1;
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      c.w[j] = *reinterpret_cast<const u32x4*>(csrc[j] + (int64_t)k * 1024);
#pragma unroll
      for (int g = 0; g < NG; ++g) c.z[j][g] = p.zeros[zat[j] + (GS ? (int64_t)(k * GS + g) * 16 : 0)];
    }
  };
  const int wrow = wave * 32 + l16;                     // of the first tile; the second is 16 rows on
  const int wswz = (l16 >> 1) & 7;
  // word i of tile j to the stage at `slot`
  auto unpack = [&](const Codes& c, int j, int i, int slot) {
    const uint32_t z = c.z[j][GS ? i * GS / 4 : 0], z4 = __builtin_amdgcn_perm(z, z, 0u);
    unsigned char* row = smem + slot * kWStage + (wrow + j * 16) * 128;
    if (I8) {
      *reinterpret_cast<u32x2*>(row + (((2 * i + (q >> 1)) ^ wswz) << 4) + (q & 1) * 8) = linear_bytes(c.w[j][i], z4);
    } else {
      *reinterpret_cast<u32x4*>(row + (((4 * (i & 1) + q) ^ wswz) << 4)) = __builtin_bit_cast(u32x4, linear_bf16(c.w[j][i], z4));
    }
  };

  // ---- products
  f32x16 acc[2][2], total[2][2];                        // I8: acc holds the bits of int32
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
      for (int e = 0; e < 16; ++e) { acc[i][j][e] = 0.f; total[i][j][e] = 0.f; }
  int off[4];
#pragma unroll
  for (int s = 0; s < 4; ++s) off[s] = l32 * 128 + (((2 * s + half) ^ ((l32 >> 1) & 7)) << 4);
  u32x4 xf[2][2], wf[2][2];                             // [set][tile]
  auto read_frags = [&](int set, int s, int slot) {
    const unsigned char* xb = xs_lds + slot * kXStage + wt * 128 + off[s];
    const unsigned char* wb = smem + slot * kWStage + wr * 128 + off[s];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      xf[set][i] = *reinterpret_cast<const u32x4*>(xb + i * 4096);
      wf[set][i] = *reinterpret_cast<const u32x4*>(wb + i * 4096);
    }
  };
  auto add_scaled = [&](int i, int j, float s) {
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      const float v = I8 ? (float)__float_as_int(acc[i][j][e]) : acc[i][j][e];
      total[i][j][e] = fmaf(s, v, total[i][j][e]);
    }
  };
  auto product = [&](int set, int i, int j, bool first) {
    const f32x16 zero = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    const f32x16 c = first ? zero : acc[i][j];
    if (I8)
      acc[i][j] = __builtin_bit_cast(f32x16, __builtin_amdgcn_mfma_i32_32x32x32_i8(__builtin_bit_cast(i32x4, xf[set][i]),
                                     __builtin_bit_cast(i32x4, wf[set][j]), __builtin_bit_cast(i32x16, c), 0, 0, 0));
    else
      acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, xf[set][i]), __builtin_bit_cast(bf16x8, wf[set][j]), c, 0, 0, 0);
  };
  float s_old[2] = {0.f, 0.f}, s_cur[2][NG], s_next[2][NG];
  auto load_scales = [&](float (&s)[2][NG], int k) {
    k = k < p.kt ? k : p.kt - 1;
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
      for (int g = 0; g < NG; ++g) s[j][g] = p.scales[sat[j] + (GS ? (int64_t)(k * GS + g) * 16 : 0)];
  };

  // ---- start: stages 0 and 1 unpacked and on their way
  Codes cur, next;
  load_codes(cur, 0);
  load_codes(next, 1);
  load_scales(s_cur, 0);
  load_scales(s_next, 1);
  __builtin_amdgcn_sched_barrier(0);
  load_x();
  load_x();
  constexpr int kWords = 2 * WPS;                       // per stage: tile w / WPS, word w % WPS
#pragma unroll
  for (int w = 0; w < kWords; ++w) unpack(cur, w / WPS, w % WPS, 0);
  if (NST == 2) {
#pragma unroll
    for (int w = 0; w < kWords; ++w) unpack(cur, w / WPS, WPS * (NST - 1) + w % WPS, 1);
  } else {
#pragma unroll
    for (int w = 0; w < kWords; ++w) unpack(next, w / WPS, w % WPS, 1);
    load_codes(next, 2);
  }
  many_wait<0>();
  many_barrier();
  int slot = 0;
  read_frags(0, 0, 0);
  // Stage t = k * NST + h; behind its barrier stage t + 2 is unpacked (words 0 .. half of them in this stage, the rest in the next).
  for (int k = 0; k < p.kt; ++k) {
#pragma unroll
    for (int h = 0; h < NST; ++h) {
      const int slot1 = slot == kRing - 1 ? 0 : slot + 1, slot2 = slot1 == kRing - 1 ? 0 : slot1 + 1;
#pragma unroll
      for (int s = 0; s < 4; ++s) {
        const int set = s & 1;
        const int gstep = h * 4 + s;                    // step in the 128 columns
        if (s < 3) read_frags(set ^ 1, s + 1, slot);
        else read_frags(set ^ 1, 0, slot1);
        const bool first = GS ? gstep % (SPG ? SPG : 1) == 0 : false;
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            if (first) add_scaled(i, j, gstep == 0 ? s_old[j] : s_cur[j][GS ? (gstep - 1) / (SPG ? SPG : 1) : 0]);
            product(set, i, j, first);
          }
        // unpacking: steps 2, 3 the first half of stage t + 2, steps 0, 1 the second half of stage t + 1
        constexpr int PER = kWords / 4;
        if (s == 2) {
          if (h == 0) { cur = next; load_codes(next, k + (I8 ? 3 : 2)); }
        }
        if (s >= 2) {
#pragma unroll
          for (int w = (s - 2) * PER; w < (s - 1) * PER; ++w) unpack(cur, w / WPS, (I8 ? 0 : WPS * h) + w % WPS, slot2);
        } else {
          // (the stage before this one began it, from the same registers)
          const int hw = NST == 2 ? 1 - h : 0;
          if (h != 0 || k != 0) {
#pragma unroll
            for (int w = (s + 2) * PER; w < (s + 3) * PER; ++w) unpack(cur, w / WPS, (I8 ? 0 : WPS * hw) + w % WPS, slot1);
          }
        }
        if (s == 1) {
          many_wait<0>();
          many_barrier();
          load_x();
        }
      }
      slot = slot1;
    }
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      s_old[j] = s_cur[j][NG - 1];
#pragma unroll
      for (int g = 0; g < NG; ++g) s_cur[j][g] = s_next[j][g];
    }
    load_scales(s_next, k + 2);
  }
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int j = 0; j < 2; ++j) add_scaled(i, j, GS ? s_old[j] : s_cur[j][0]);

  many_wait<0>();                                       // (nothing writes to LDS behind the workgroup's end)

  // ---- results: the lane has row l32 of a tile, tokens 8 (e / 4) + 4 half + e % 4
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    const int row = row0 + wr + j * 32 + l32;
    const float b = p.bias && row < p.m ? p.bias[row] : 0.f;
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        const int tok = tok0 + wt + i * 32 + 8 * (e >> 2) + 4 * half + (e & 3);
        if (row >= p.m || tok >= p.tokens) continue;
        float v = total[i][j][e];
        if (I8) v *= p.xs[tok];
        v += b;
        const int64_t o = (int64_t)tok * p.ldy + row;
        if (p.y_f32) ((float*)p.y)[o] = v;
        else ((uint16_t*)p.y)[o] = __builtin_bit_cast(uint16_t, (__bf16)v);
      }
  }
}

template <bool I8, int GS> static hipError_t launch_many_as(const LinearArgs& p, hipStream_t s) {
  static LdsLimitOnce once;
  if (const hipError_t e = once.ensure((const void*)&linear_many_kernel<I8, GS>, kManyLds); e != hipSuccess) return e;
  const int tt = (p.tokens + kManyTokens - 1) / kManyTokens, rt = (p.m + kManyRows - 1) / kManyRows;
  hipLaunchKernelGGL((linear_many_kernel<I8, GS>), dim3((unsigned)(tt * rt)), dim3(512), kManyLds, s, p, tt, rt);
  return hipGetLastError();
}

hipError_t launch_linear_many(const LinearArgs& p, int gs, bool i8, hipStream_t s) {
  switch (gs) {
    case 0: return i8 ? launch_many_as<true, 0>(p, s) : launch_many_as<false, 0>(p, s);
    case 1: return i8 ? launch_many_as<true, 1>(p, s) : launch_many_as<false, 1>(p, s);
    case 2: return i8 ? launch_many_as<true, 2>(p, s) : launch_many_as<false, 2>(p, s);
    default: return i8 ? launch_many_as<true, 4>(p, s) : launch_many_as<false, 4>(p, s);
  }
}

}  // namespace gptaq
