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
// A workgroup takes RT tiles of 16 rows and TT of 16 tokens; its wavefronts share the tiles of 128 columns out among themselves and
// add their sums through LDS, in the wavefronts' order.  The weights go straight from memory to the lanes that feed the matrix
// unit: nothing is read twice, and with all of a wavefront's tiles independent many loads are in flight.  v_mfma 16x16: the left
// operand is 16 tokens (lane l: token l % 16), the right 16 rows of W (lane l: row l % 16), the result has the row of W in l % 16
// and tokens 4 (l / 16) .. + 3 in the lane's four values, so one scale per lane serves a result.
// GS: groups per 128 columns (1, 2, 4), 0: one group per row.
template <bool I8, int GS, int TT, int RT>
__global__ __launch_bounds__(512) void linear_few_kernel(LinearArgs p) {
  extern __shared__ float lds[];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, waves = blockDim.x >> 6;
  const int l16 = lane & 15, q = lane >> 4;
  const int row_blocks = (p.mt + RT - 1) / RT;
  const int rb = blockIdx.x % row_blocks, tb = blockIdx.x / row_blocks;
  const int rt0 = rb * RT, tok0 = tb * TT * 16;

  f32x4 total[TT][RT];
  f32x4 acc[TT][RT];                   // I8: the bits of int32
#pragma unroll
  for (int t = 0; t < TT; ++t)
#pragma unroll
    for (int r = 0; r < RT; ++r) { total[t][r] = f32x4{0.f, 0.f, 0.f, 0.f}; acc[t][r] = f32x4{0.f, 0.f, 0.f, 0.f}; }

  int64_t tile_row[RT];                // (past the last tile of rows: that one again; nothing of it is stored)
#pragma unroll
  for (int r = 0; r < RT; ++r) tile_row[r] = rt0 + r < p.mt ? rt0 + r : p.mt - 1;
  auto add_scaled = [&](int t, int r, float s) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float v = I8 ? (float)__float_as_int(acc[t][r][e]) : acc[t][r][e];
      total[t][r][e] = fmaf(s, v, total[t][r][e]);
    }
    acc[t][r] = f32x4{0.f, 0.f, 0.f, 0.f};
  };
  constexpr int G = GS ? GS : 1;       // groups per tile of 128 columns
  for (int k = wave; k < p.kt; k += waves) {
    u32x4 w[RT];
    float s[RT][G];
    uint32_t off[RT][G];
#pragma unroll
    for (int r = 0; r < RT; ++r) {
      w[r] = *reinterpret_cast<const u32x4*>(p.codes + (tile_row[r] * p.kt + k) * 1024 + lane * 16);
#pragma unroll
      for (int g = 0; g < G; ++g) {
        const int64_t at = (tile_row[r] * p.groups + (GS ? k * GS + g : 0)) * 16 + l16;
        s[r][g] = p.scales[at];
        off[r][g] = linear_offset(p.zeros[at]);
      }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int col = k * 128 + i * 32 + q * 8;
      u32x4 x[TT];                     // I8: two words
#pragma unroll
      for (int t = 0; t < TT; ++t) {
        const int tok = tok0 + t * 16 + l16;
        x[t] = u32x4{0u, 0u, 0u, 0u};
        if (tok < p.tokens && col < p.n) {
          if (I8) {
            const u32x2 v = *reinterpret_cast<const u32x2*>((const int8_t*)p.x + (int64_t)tok * p.ldx + col);
            x[t][0] = v[0]; x[t][1] = v[1];
          } else {
            x[t] = *reinterpret_cast<const u32x4*>((const uint16_t*)p.x + (int64_t)tok * p.ldx + col);
          }
        }
      }
#pragma unroll
      for (int r = 0; r < RT; ++r) {
        const uint32_t z = off[r][GS ? i * GS / 4 : 0];
        if (I8) {
          const u32x2 b = linear_bytes(w[r][i], z);
#pragma unroll
          for (int t = 0; t < TT; ++t)
            acc[t][r] = __builtin_bit_cast(f32x4, __builtin_amdgcn_mfma_i32_16x16x32_i8(
                __builtin_bit_cast(long, u32x2{x[t][0], x[t][1]}), __builtin_bit_cast(long, b), __builtin_bit_cast(i32x4, acc[t][r]), 0, 0, 0));
        } else {
          const bf16x8 b = linear_bf16(w[r][i], z);
#pragma unroll
          for (int t = 0; t < TT; ++t)
            acc[t][r] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, x[t]), b, acc[t][r], 0, 0, 0);
        }
        if (GS && (i + 1) % (4 / G) == 0) {
#pragma unroll
          for (int t = 0; t < TT; ++t) add_scaled(t, r, s[r][i * G / 4]);
        }
      }
    }
  }
  if (!GS) {
#pragma unroll
    for (int r = 0; r < RT; ++r) {
      const float s = p.scales[tile_row[r] * 16 + l16];
#pragma unroll
      for (int t = 0; t < TT; ++t) add_scaled(t, r, s);
    }
  }
  // [wave][t][r][lane][4]
#pragma unroll
  for (int t = 0; t < TT; ++t)
#pragma unroll
    for (int r = 0; r < RT; ++r) *reinterpret_cast<f32x4*>(&lds[(((wave * TT + t) * RT + r) * 64 + lane) * 4]) = total[t][r];
  __syncthreads();
  for (int at = threadIdx.x; at < TT * RT * 256; at += blockDim.x) {
    // 16 rows of W in a run of threads, so that a token's outputs are written together
    const int r = at & 15, rt = at / 16 % RT, tok_in = at / (16 * RT);
    const int t = tok_in >> 4, row = (rt0 + rt) * 16 + r, tok = tok0 + tok_in;
    if (rt0 + rt >= p.mt || row >= p.m || tok >= p.tokens) continue;
    const int slot = ((t * RT + rt) * 64 + (tok_in & 15) / 4 * 16 + r) * 4 + (tok_in & 3);
    float v = 0.f;
    for (int w = 0; w < waves; ++w) v += lds[w * TT * RT * 256 + slot];
    if (I8) v *= p.xs[tok];
    if (p.bias) v += p.bias[row];
    const int64_t o = (int64_t)tok * p.ldy + row;
    if (p.y_f32) ((float*)p.y)[o] = v;
    else ((uint16_t*)p.y)[o] = __builtin_bit_cast(uint16_t, (__bf16)v);
  }
}

template <bool I8, int TT, int RT>
static hipError_t launch_few(const LinearArgs& p, int gs, hipStream_t s) {
  int waves = 8;
  while (waves > 1 && waves > p.kt) waves /= 2;
  const int64_t blocks = (int64_t)((p.mt + RT - 1) / RT) * ((p.tokens + TT * 16 - 1) / (TT * 16));
  const auto kernel = gs == 0 ? &linear_few_kernel<I8, 0, TT, RT> : gs == 1 ? &linear_few_kernel<I8, 1, TT, RT>
                    : gs == 2 ? &linear_few_kernel<I8, 2, TT, RT> : &linear_few_kernel<I8, 4, TT, RT>;
  hipLaunchKernelGGL(kernel, dim3((unsigned)blocks), dim3(64 * waves), (size_t)waves * TT * RT * 1024, s, p);
  return hipGetLastError();
}

static hipError_t launch_linear(const LinearArgs& p, int gs, bool i8, hipStream_t s) {
  if (p.tokens > 128) return launch_linear_many(p, gs, i8, s);
  if (p.tokens <= 16) return i8 ? launch_few<true, 1, 1>(p, gs, s) : launch_few<false, 1, 1>(p, gs, s);
  return i8 ? launch_few<true, 4, 2>(p, gs, s) : launch_few<false, 4, 2>(p, gs, s);
}

// ---- argument checks

constexpr int64_t kMaxSide = (int64_t)1 << 20, kMaxTokens = (int64_t)1 << 23;
static bool good_group(int64_t n, int group) {
  return group <= 0 || ((group == 32 || group == 64 || group == 128) && n % group == 0);
}
// Elements of a row of activations in the workspace: whole tiles of columns.
static int64_t padded_columns(int64_t n) { return (n + 127) / 128 * 128; }

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
  const int piece = tokens > 128 ? 128 : i8 ? 16 : 8;
  if (perm || n % piece || ldx % (i8 ? 16 : 8) || ((uintptr_t)X & 15) || (tokens > 128 && ldx * (i8 ? 1 : 2) > kManyMaxRow)) {
    const int64_t ld = padded_columns(n);
    if (i8) hipLaunchKernelGGL(linear_gather_kernel<int8_t>, dim3((unsigned)tokens), dim3(256), 0, s, (const int8_t*)X, ldx, perm, (int)n, (int8_t*)ws, ld);
    else hipLaunchKernelGGL(linear_gather_kernel<uint16_t>, dim3((unsigned)tokens), dim3(256), 0, s, (const uint16_t*)X, ldx, perm, (int)n, (uint16_t*)ws, ld);
    GPTAQ_LAUNCH_CHECK();
    p.x = ws; p.ldx = ld;
    p.n = (int32_t)ld;                 // (the columns behind n are zeros here)
  }
  // A grid has less than 2^32 threads: more tokens than that takes are several launches.
  const int64_t most = (((int64_t)1 << 22) / p.mt) * 64;
  for (int64_t first = 0; first < tokens; first += most) {
    LinearArgs part = p;
    part.tokens = (int32_t)(tokens - first < most ? tokens - first : most);
    part.x = (const uint8_t*)p.x + first * p.ldx * (i8 ? 1 : 2);
    part.y = (uint8_t*)p.y + first * p.ldy * (y_f32 ? 4 : 2);
    if (i8) part.xs = p.xs + first;
    if (const hipError_t e = launch_linear(part, group ? 128 / group : 0, i8, s); e != hipSuccess) { set_last_hip_error(e); return GPTAQ_ELAUNCH; }
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
  return ((size_t)tokens * padded_columns(n) * 2 + 255) / 256 * 256;
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
