// y = x W^T + bias for layers whose weights the solve has quantised: W[r][j] = scale[r][g] * (code[r][j] - zero[r][g]), g the group
// of column j, codes of at most 4 bits.
//
// code - zero is an integer between -15 and 15, exact in bfloat16 and in 8 bits, so the matrix instructions multiply exact weights:
// per group of columns the sum of (code - zero) x is taken in fp32 (bf16 activations) or exactly in int32 (8-bit activations),
// multiplied by the group's fp32 scale, and added to the fp32 total.  No weight is rounded.
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
// inside a piece of 16.  Rows of `out` have `ldo` elements, zeros behind the n-th.
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
// Up to 16 tokens, one tile of v_mfma 16x16.  A workgroup takes RT tiles of 16 rows; its wavefronts share the tiles of 128 columns out
// among themselves and add their sums through LDS, in the wavefronts' order.  The weights go straight from memory to the lanes that
// feed the matrix unit, two tiles of columns ahead: nothing of W is read twice, and with everything of a wavefront independent many
// loads are in flight.  The left operand is 16 tokens (lane l: token l % 16), the right 16 rows of W (lane l: row l % 16), the result has the
// row of W in l % 16 and tokens 4 (l / 16) .. + 3 in the lane's four values, so one scale per lane serves a result.
// A load of 16 bytes a lane costs the same whether its lanes want it or not, and a token fills 4 of 64 lanes: so up to XT = 4 (8) tokens
// one load brings 4 (2) of the 4 steps of 128 columns, each to XT lanes of 16 of its own; the others are zeros for that step, the result has
// the steps in different rows, and the join adds them.
// GS: groups per 128 columns (1, 2, 4), 0: one group per row.
// Most wavefronts of a workgroup: 16 leave a lane 128 registers.
constexpr int few_waves(int gs, int rt, int xt) { return rt > 1 || (gs == 4 && xt == 16) ? 8 : 16; }

template <bool I8, int GS, int RT, int XT>
__global__ __launch_bounds__(64 * few_waves(GS, RT, XT)) void linear_few_kernel(LinearArgs p) {
  extern __shared__ float lds[];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, waves = blockDim.x >> 6;
  const int l16 = lane & 15, q = lane >> 4;
  const int rt0 = blockIdx.x * RT;
  constexpr int G = GS ? GS : 1;       // groups per tile of 128 columns

  f32x4 total[RT], acc[RT];            // I8: acc holds the bits of int32
  const uint8_t* codes[RT];
  int64_t group[RT];
#pragma unroll
  for (int r = 0; r < RT; ++r) {
    total[r] = acc[r] = f32x4{0.f, 0.f, 0.f, 0.f};
    const int64_t tr = rt0 + r < p.mt ? rt0 + r : p.mt - 1;      // (past the last tile of rows: that one again; nothing of it is stored)
    codes[r] = p.codes + tr * p.kt * 1024 + lane * 16;
    group[r] = tr * p.groups * 16 + l16;
  }
  constexpr int SP = 16 / XT, NX = 4 / SP;       // steps per load of activations, loads per 128 columns
  const int sub = l16 / XT, tok_lane = l16 % XT;
  const bool here = tok_lane < p.tokens;
  const int x_col = sub * 32 + q * 8;
  const uint8_t* x0 = (const uint8_t*)p.x + ((int64_t)(here ? tok_lane : 0) * p.ldx + x_col) * (I8 ? 1 : 2);

  struct Stage { u32x4 w[RT]; uint32_t zero[RT][G]; float scale[RT][G]; u32x4 x[NX]; };
  auto load = [&](Stage& s, int k) {
    if (k >= p.kt) return;
#pragma unroll
    for (int r = 0; r < RT; ++r) {
      s.w[r] = *reinterpret_cast<const u32x4*>(codes[r] + (int64_t)k * 1024);
      if (GS) {
#pragma unroll
        for (int g = 0; g < G; ++g) {
          s.zero[r][g] = p.zeros[group[r] + (int64_t)(k * GS + g) * 16];
          s.scale[r][g] = p.scales[group[r] + (int64_t)(k * GS + g) * 16];
        }
      }
    }
#pragma unroll
    for (int i = 0; i < NX; ++i) {
      const int col = k * 128 + i * SP * 32;
      s.x[i] = u32x4{0u, 0u, 0u, 0u};
      if (here && col + x_col < p.n) {
        if (I8) {
          const u32x2 v = *reinterpret_cast<const u32x2*>(x0 + col);
          s.x[i][0] = v[0]; s.x[i][1] = v[1];
        } else {
          s.x[i] = *reinterpret_cast<const u32x4*>(x0 + 2 * col);
        }
      }
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
  f32x4 accx;                          // sums of the group's activations (the same in all of a token's lanes)
  // EXACT: the products are those of code - zero.  Else (bf16 only): of 16 + code, which is two instructions for two codes where the difference
  // takes five, and (16 + zero) times the activations' sum, one more matrix instruction for all RT, is taken off each group's sum.
  // Where a result is not finite this subtraction may be why, and the workgroup takes its sums again with EXACT.
  auto add_scaled = [&](auto exact, int r, float s, uint32_t zero) {
    const float z = -16.f - (float)zero;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      float v = I8 ? (float)__float_as_int(acc[r][e]) : acc[r][e];
      if (!exact) v = fmaf(z, accx[e], v);
      total[r][e] = fmaf(s, v, total[r][e]);
    }
  };
  auto multiply = [&](auto exact, const Stage& s) {
    const f32x4 nothing = {0.f, 0.f, 0.f, 0.f};
    u32x4 all[NX];
#pragma unroll
    for (int i = 0; i < NX; ++i) {
      all[i] = s.x[i];
      if (!exact)                      // columns 0 2 4 6 1 3 5 7, as the codes come out of a word
        all[i] = u32x4{__builtin_amdgcn_perm(s.x[i][1], s.x[i][0], 0x05040100u), __builtin_amdgcn_perm(s.x[i][3], s.x[i][2], 0x05040100u),
                       __builtin_amdgcn_perm(s.x[i][1], s.x[i][0], 0x07060302u), __builtin_amdgcn_perm(s.x[i][3], s.x[i][2], 0x07060302u)};
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const bool first = GS && i % (4 / G) == 0, last = GS && (i + 1) % (4 / G) == 0;
      u32x4 x = all[i / SP];
      if (SP > 1) {
#pragma unroll
        for (int e = 0; e < (I8 ? 2 : 4); ++e) x[e] = sub == i % SP ? x[e] : 0u;
      }
      if (!exact)
        accx = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, x), __builtin_bit_cast(bf16x8, ones), first ? nothing : accx, 0, 0, 0);
#pragma unroll
      for (int r = 0; r < RT; ++r) {
        const f32x4 c = first ? nothing : acc[r];
        const uint32_t w = s.w[r][i], zero = GS ? s.zero[r][i * G / 4] : row_zero[r];
        if (I8) {
          acc[r] = __builtin_bit_cast(f32x4, __builtin_amdgcn_mfma_i32_16x16x32_i8(
              __builtin_bit_cast(long, u32x2{x[0], x[1]}), __builtin_bit_cast(long, linear_bytes(w, linear_offset(zero))),
              __builtin_bit_cast(i32x4, c), 0, 0, 0));
        } else if (exact) {
          acc[r] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, x), linear_bf16(w, linear_offset(zero)), c, 0, 0, 0);
        } else {
          u32x4 v;                     // the code in the upper bits of the mantissa of 16
          const uint32_t shifted[4] = {w << 3, w >> 1, w >> 5, w >> 9};
#pragma unroll
          for (int e = 0; e < 4; ++e) v[e] = (shifted[e] & 0x00780078u) | sixteen;
          acc[r] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, x), __builtin_bit_cast(bf16x8, v), c, 0, 0, 0);
        }
        if (last) add_scaled(exact, r, s.scale[r][i * G / 4], zero);
      }
    }
  };
  auto sums = [&](auto exact) {
    accx = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int r = 0; r < RT; ++r) total[r] = acc[r] = f32x4{0.f, 0.f, 0.f, 0.f};
    Stage a, b;
    load(a, wave);
    load(b, wave + waves);
    for (int k = wave; k < p.kt; k += 2 * waves) {
      multiply(exact, a);
      load(a, k + 2 * waves);
      if (k + waves >= p.kt) break;
      multiply(exact, b);
      load(b, k + 3 * waves);
    }
    if (!GS) {
#pragma unroll
      for (int r = 0; r < RT; ++r) add_scaled(exact, r, p.scales[group[r]], row_zero[r]);
    }
  };
  // Joins the wavefronts' sums, [wave][r][lane][4], and stores; returns whether a sum of this thread's is not finite.
  auto finish = [&]() {
#pragma unroll
    for (int r = 0; r < RT; ++r) *reinterpret_cast<f32x4*>(&lds[((wave * RT + r) * 64 + lane) * 4]) = total[r];
    __syncthreads();
    bool lost = false;
    for (int at = threadIdx.x; at < RT * 16 * XT; at += blockDim.x) {
      // 16 RT rows of W in a run of threads, so that a token's outputs are written together
      const int r = at % (16 * RT), tok = at / (16 * RT), row = rt0 * 16 + r;
      if (row >= p.m || tok >= p.tokens) continue;
      float v = 0.f;
      for (int w = 0; w < waves; ++w)
#pragma unroll
        for (int st = 0; st < SP; ++st) {
          const int t = st * XT + tok;
          v += lds[w * RT * 256 + ((r >> 4) * 64 + (t >> 2) * 16 + (r & 15)) * 4 + (t & 3)];
        }
      lost |= !(fabsf(v) < __builtin_inff());
      if (I8) v *= p.xs[tok];
      if (p.bias) v += p.bias[row];
      const int64_t o = (int64_t)tok * p.ldy + row;
      if (p.y_f32) ((float*)p.y)[o] = v;
      else ((uint16_t*)p.y)[o] = __builtin_bit_cast(uint16_t, (__bf16)v);
    }
    return lost;
  };
  sums(std::integral_constant<bool, I8>{});
  const bool lost = finish();
  if (!I8 && __syncthreads_or(lost)) {
    sums(std::true_type{});
    finish();
  }
}

template <bool I8, int GS, int RT, int XT>
static hipError_t launch_few_as(const LinearArgs& p, int waves, hipStream_t s) {
  if (waves > few_waves(GS, RT, XT)) waves = few_waves(GS, RT, XT);
  while (waves > 1 && waves > p.kt) waves /= 2;
  hipLaunchKernelGGL((linear_few_kernel<I8, GS, RT, XT>), dim3((unsigned)((p.mt + RT - 1) / RT)), dim3(64 * waves), (size_t)waves * RT * 1024, s, p);
  return hipGetLastError();
}
// Tiles of rows per workgroup: the more, the less often the activations are read, the fewer workgroups.  us a call, bf16, RT 1 / 2 / 4: 1 token
// 4096 x 4096 4.5 / 5.8 / 9.5, 28672 x 8192 31.8 / 30.0 / 37; 16 tokens 4096 x 4096 7.1 / 7.9 / 11, 11008 x 4096 15.6 / 14.6 / 10.4, 28672 x 8192
// 61 / 49 / 34.  (With four groups to 128 columns, four tiles of rows have more scales than registers.)
// Wavefronts, RT 1, 8 / 16: 4096 x 11008 8.7 / 8.1, 1024 x 8192 5.8 / 5.7, 11008 x 4096 8.9 / 9.5; RT 4, 4 / 8: 28672 x 8192, 16 tokens 34 / 42,
// 11008 x 4096 14.9 / 10.4.
template <bool I8, int GS>
static hipError_t launch_few_of(const LinearArgs& p, hipStream_t s) {
  if (p.tokens > 8) {
    if (p.mt < 512) return launch_few_as<I8, GS, 1, 16>(p, 16, s);
    if (GS == 4) return launch_few_as<I8, GS, 2, 16>(p, 8, s);
    return launch_few_as<I8, GS, GS == 4 ? 2 : 4, 16>(p, p.mt >= 1024 ? 4 : 8, s);
  }
  const int waves = p.mt < 512 ? 16 : 8;
  if (p.tokens > 4) return p.mt >= 1024 ? launch_few_as<I8, GS, 2, 8>(p, waves, s) : launch_few_as<I8, GS, 1, 8>(p, waves, s);
  return p.mt >= 1024 ? launch_few_as<I8, GS, 2, 4>(p, waves, s) : launch_few_as<I8, GS, 1, 4>(p, waves, s);
}
template <bool I8>
static hipError_t launch_few(const LinearArgs& p, int gs, hipStream_t s) {
  return gs == 0 ? launch_few_of<I8, 0>(p, s) : gs == 1 ? launch_few_of<I8, 1>(p, s) : gs == 2 ? launch_few_of<I8, 2>(p, s) : launch_few_of<I8, 4>(p, s);
}

static hipError_t launch_linear(const LinearArgs& p, int gs, bool i8, float* partial, hipStream_t s) {
  if (p.tokens > 16) return launch_linear_many(p, gs, i8, partial, s);
  return i8 ? launch_few<true>(p, gs, s) : launch_few<false>(p, gs, s);
}

// ---- argument checks

constexpr int64_t kMaxSide = (int64_t)1 << 20, kMaxTokens = (int64_t)1 << 23;
static bool good_group(int64_t n, int group) {
  return group <= 0 || ((group == 32 || group == 64 || group == 128) && n % group == 0);
}
// Elements of a row of activations in the workspace: whole tiles of columns.
static int64_t padded_columns(int64_t n) { return (n + 127) / 128 * 128; }

static size_t gather_bytes(int64_t tokens, int64_t n) { return ((size_t)tokens * padded_columns(n) * 2 + 255) / 256 * 256; }

static int run_linear(bool i8, const void* X, const float* xs, int64_t tokens, int64_t ldx, const int32_t* perm, const void* weights, int64_t m,
                      int64_t n, int group, const float* bias, void* Y, int64_t ldy, int y_f32, void* ws, size_t ws_bytes, void* stream) {
  if (!weights || (tokens != 0 && (!X || !Y || !ws || (i8 && !xs)))) return GPTAQ_ENULL;      // (no tokens: nothing to point to)
  const uintptr_t y_align = y_f32 ? 3 : 1;
  if (tokens < 0 || tokens > kMaxTokens || m <= 0 || n <= 0 || m > kMaxSide || n > kMaxSide || ldx < n || ldy < m ||
      ((uintptr_t)weights & 255) || ((uintptr_t)Y & y_align) || (!i8 && ((uintptr_t)X & 1)) || (((uintptr_t)xs | (uintptr_t)bias | (uintptr_t)perm) & 3))
    return GPTAQ_EDIM;
  if (!good_group(n, group)) return GPTAQ_EUNSUPPORTED;
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
  const int piece = tokens > 16 ? 128 : i8 ? 16 : 8;
  if (perm || n % piece || ldx % (i8 ? 16 : 8) || ((uintptr_t)X & 15) || (tokens > 16 && ldx * (i8 ? 1 : 2) > kManyMaxRow)) {
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
  if (m <= 0 || n <= 0 || m > kMaxSide || n > kMaxSide || !good_group(n, group)) return 0;
  return linear_layout(m, n, group > 0 ? group : 0).bytes;
}

extern "C" int gptaq_linear_pack(const uint8_t* codes, int64_t ldc, const float* scales, const float* zeros, int64_t m, int64_t n, int group,
                                 void* weights, size_t weights_bytes, int32_t* info, void* stream) {
  if (!codes || !scales || !zeros || !weights || !info) return GPTAQ_ENULL;
  if (m <= 0 || n <= 0 || m > kMaxSide || n > kMaxSide || ldc < n || (((uintptr_t)scales | (uintptr_t)zeros | (uintptr_t)info) & 3)) return GPTAQ_EDIM;
  if (!good_group(n, group)) return GPTAQ_EUNSUPPORTED;
  const LinearLayout l = linear_layout(m, n, group > 0 ? group : 0);
  if (((uintptr_t)weights & 255) || weights_bytes < l.bytes) return GPTAQ_EWORKSPACE;
  if (l.mt * l.kt > ((int64_t)1 << 23)) return GPTAQ_EDIM;
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
  if (tokens <= 0 || tokens > kMaxTokens || m <= 0 || n <= 0 || m > kMaxSide || n > kMaxSide) return 0;
  return gather_bytes(tokens, n) + (linear_partial_bytes(tokens, m, n) + 255) / 256 * 256;
}

extern "C" int gptaq_linear(const uint16_t* X, int64_t tokens, int64_t ldx, const int32_t* perm, const void* weights, int64_t m, int64_t n,
                            int group, const float* bias, void* Y, int64_t ldy, int y_f32, void* ws, size_t ws_bytes, void* stream) {
  return run_linear(false, X, nullptr, tokens, ldx, perm, weights, m, n, group, bias, Y, ldy, y_f32, ws, ws_bytes, stream);
}

extern "C" int gptaq_linear_i8(const int8_t* X, const float* x_scales, int64_t tokens, int64_t ldx, const int32_t* perm, const void* weights,
                               int64_t m, int64_t n, int group, const float* bias, void* Y, int64_t ldy, int y_f32, void* ws, size_t ws_bytes,
                               void* stream) {
  return run_linear(true, X, x_scales, tokens, ldx, perm, weights, m, n, group, bias, Y, ldy, y_f32, ws, ws_bytes, stream);
}
