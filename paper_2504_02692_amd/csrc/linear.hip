// y = x W^T + bias for layers whose weights the solve has quantised: W[r][j] = scale[r][g] * (code[r][j] - zero[r][g]), g the group
// of column j, codes of at most 4 bits.
//
// code - zero is an integer between -15 and 15, exact in bfloat16 and in 8 bits, so the matrix instructions multiply exact weights:
// per group of columns the sum of (code - zero) x is taken in fp32 (bf16 activations) or exactly in int32 (8-bit activations),
// multiplied by the group's fp32 scale, and added to the fp32 total.  No weight is rounded.
#include "linear.h"

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
// GS: groups per 128 columns (1, 2, 4), 0: one group per row.
template <bool I8, int GS, int RT>
__global__ __launch_bounds__(RT == 1 ? 1024 : 512) void linear_few_kernel(LinearArgs p) {
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
  const bool here = l16 < p.tokens;
  const uint8_t* x0 = (const uint8_t*)p.x + ((int64_t)(here ? l16 : 0) * p.ldx + q * 8) * (I8 ? 1 : 2);

  struct Stage { u32x4 w[RT]; uint32_t zero[RT][G]; float scale[RT][G]; u32x4 x[4]; };
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
    for (int i = 0; i < 4; ++i) {
      const int col = k * 128 + i * 32;
      s.x[i] = u32x4{0u, 0u, 0u, 0u};
      if (here && col + q * 8 < p.n) {
        if (I8) {
          const u32x2 v = *reinterpret_cast<const u32x2*>(x0 + col);
          s.x[i][0] = v[0]; s.x[i][1] = v[1];
        } else {
          s.x[i] = *reinterpret_cast<const u32x4*>(x0 + 2 * col);
        }
      }
    }
  };
  auto add_scaled = [&](int r, float s) {
#pragma unroll
    for (int e = 0; e < 4; ++e) total[r][e] = fmaf(s, I8 ? (float)__float_as_int(acc[r][e]) : acc[r][e], total[r][e]);
  };
  uint32_t row_off[RT];
  if (!GS) {
#pragma unroll
    for (int r = 0; r < RT; ++r) row_off[r] = linear_offset(p.zeros[group[r]]);
  }
  auto multiply = [&](const Stage& s) {
#pragma unroll
    for (int r = 0; r < RT; ++r) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint32_t off = GS ? linear_offset(s.zero[r][i * G / 4]) : row_off[r];
        const f32x4 c = GS && i % (4 / G) == 0 ? f32x4{0.f, 0.f, 0.f, 0.f} : acc[r];
        if (I8)
          acc[r] = __builtin_bit_cast(f32x4, __builtin_amdgcn_mfma_i32_16x16x32_i8(
              __builtin_bit_cast(long, u32x2{s.x[i][0], s.x[i][1]}), __builtin_bit_cast(long, linear_bytes(s.w[r][i], off)),
              __builtin_bit_cast(i32x4, c), 0, 0, 0));
        else
          acc[r] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, s.x[i]), linear_bf16(s.w[r][i], off), c, 0, 0, 0);
        if (GS && (i + 1) % (4 / G) == 0) add_scaled(r, s.scale[r][i * G / 4]);
      }
    }
  };
  Stage a, b;
  load(a, wave);
  load(b, wave + waves);
  for (int k = wave; k < p.kt; k += 2 * waves) {
    multiply(a);
    load(a, k + 2 * waves);
    if (k + waves >= p.kt) break;
    multiply(b);
    load(b, k + 3 * waves);
  }
  if (!GS) {
#pragma unroll
    for (int r = 0; r < RT; ++r) add_scaled(r, p.scales[group[r]]);
  }
  // [wave][r][lane][4]
#pragma unroll
  for (int r = 0; r < RT; ++r) *reinterpret_cast<f32x4*>(&lds[((wave * RT + r) * 64 + lane) * 4]) = total[r];
  __syncthreads();
  for (int at = threadIdx.x; at < RT * 256; at += blockDim.x) {
    // 16 RT rows of W in a run of threads, so that a token's outputs are written together
    const int r = at % (16 * RT), tok = at / (16 * RT), row = rt0 * 16 + r;
    if (row >= p.m || tok >= p.tokens) continue;
    const int slot = ((r >> 4) * 64 + (tok >> 2) * 16 + (r & 15)) * 4 + (tok & 3);
    float v = 0.f;
    for (int w = 0; w < waves; ++w) v += lds[w * RT * 256 + slot];
    if (I8) v *= p.xs[tok];
    if (p.bias) v += p.bias[row];
    const int64_t o = (int64_t)tok * p.ldy + row;
    if (p.y_f32) ((float*)p.y)[o] = v;
    else ((uint16_t*)p.y)[o] = __builtin_bit_cast(uint16_t, (__bf16)v);
  }
}

template <bool I8, int RT>
static hipError_t launch_few_as(const LinearArgs& p, int gs, int waves, hipStream_t s) {
  const auto kernel = gs == 0 ? &linear_few_kernel<I8, 0, RT> : gs == 1 ? &linear_few_kernel<I8, 1, RT>
                    : gs == 2 ? &linear_few_kernel<I8, 2, RT> : &linear_few_kernel<I8, RT == 4 ? 2 : 4, RT>;
  hipLaunchKernelGGL(kernel, dim3((unsigned)((p.mt + RT - 1) / RT)), dim3(64 * waves), (size_t)waves * RT * 1024, s, p);
  return hipGetLastError();
}
// Tiles of rows per workgroup: the more, the less often the activations are read, the fewer workgroups.  us a call, 1 token, RT 1 / 2 / 4:
// 4096 x 4096 5.1 / 7.4 / 10.3, 11008 x 4096 10.7 / 11.3 / 11.5, 28672 x 8192 43.2 / 38.3 / 40.9; 16 tokens 6.7 / 8.4 / 11.8, 15.2 / 13.7 / 12.5,
// 60.8 / 45.7 / 42.3.  (With four groups to 128 columns, four tiles of rows have more scales than registers.)
// Wavefronts, RT 1, 8 / 16: 4096 x 11008 11.3 / 9.3, 1024 x 8192 7.1 / 6.6, 11008 x 4096 10.7 / 11.7.  RT 4, 4 / 8: 28672 x 8192, 16 tokens 40.2 / 42.3,
// 11008 x 4096 15.0 / 12.5.
template <bool I8>
static hipError_t launch_few(const LinearArgs& p, int gs, hipStream_t s) {
  const int rt = p.tokens > 8 ? (p.mt >= 512 ? (gs == 4 ? 2 : 4) : 1) : p.mt >= 1024 ? 2 : 1;
  int waves = rt == 1 ? (p.mt < 512 ? 16 : 8) : rt == 4 && p.mt >= 1024 ? 4 : 8;
  while (waves > 1 && waves > p.kt) waves /= 2;
  if (rt == 4) return launch_few_as<I8, 4>(p, gs, waves, s);
  if (rt == 2) return launch_few_as<I8, 2>(p, gs, waves, s);
  return launch_few_as<I8, 1>(p, gs, waves, s);
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
