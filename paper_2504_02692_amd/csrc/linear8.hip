// y = x W^T + bias for layers whose weights the solve has quantised to 5 .. 8 bits with one scale and zero a row, and 8-bit activations:
// y[t][r] = xs[t] scale[r] sum_j (code[r][j] - zero[r]) x[t][j] + bias[r].  The sum is exact (linear8.h); it is converted to fp32 once, multiplied by the product of
// the two scales, and the bias is added with the same rounding.
#include "linear8.h"

namespace gptaq {

// ---- laying out the weights

// inverse[perm[j]] = j, and -1 where no j goes: what is missing or met twice shows as a column without a source.
__global__ __launch_bounds__(256) void linear8_clear_kernel(int32_t* inverse, int n, const int32_t* perm, int32_t* info, uint8_t* tail, int count) {
  const int at = blockIdx.x * 256 + threadIdx.x;
  if (at < n) inverse[at] = perm ? -1 : at;
  if (blockIdx.x == 0 && threadIdx.x == 0) *info = 0;
  if (blockIdx.x == 0 && (int)threadIdx.x < count) tail[threadIdx.x] = 0;
}
__global__ __launch_bounds__(256) void linear8_invert_kernel(int32_t* inverse, int n, const int32_t* perm) {
  const int at = blockIdx.x * 256 + threadIdx.x;
  if (at < n && (uint32_t)perm[at] < (uint32_t)n) atomicMax(inverse + perm[at], at);
}
// R rows of a tile of 16 per workgroup, by way of LDS, where their bytes are picked out in the columns' order; a thread writes 16 columns of each.  (Picked from memory
// they are a load of a byte each: 4096 x 11008 in act_order's order 377 us, this way 72.)  Bound by those reads of LDS, one for every byte, in any order: 28672 x 8192 288 us,
// three times what its bytes take.  It runs once a layer.
constexpr int kPack8Lds = 65536;
template <int R>
__global__ __launch_bounds__(256) void linear8_pack_kernel(const uint8_t* codes, int64_t ldc, const float* scales, const float* zeros, int m, int n, int kt,
                                                           const int32_t* inverse, uint8_t* out, float* out_scales, int32_t* out_shifts, int32_t* info) {
  extern __shared__ __attribute__((aligned(16))) uint8_t row_codes[];
  const int row0 = blockIdx.x * R, ld = (n + 15) / 16 * 16;
  typedef u32x4 __attribute__((aligned(1))) u32x4_at_byte;
#pragma unroll
  for (int r = 0; r < R; ++r) {
    if (row0 + r >= m) break;
    const uint8_t* from = codes + (int64_t)(row0 + r) * ldc;
    for (int c = threadIdx.x * 16; c < n; c += 256 * 16) {
      if (c + 16 <= n) *reinterpret_cast<u32x4*>(row_codes + r * ld + c) = *reinterpret_cast<const u32x4_at_byte*>(from + c);
      else
        for (int j = c; j < n; ++j) row_codes[r * ld + j] = from[j];
    }
  }
  __syncthreads();
  for (int chunk = threadIdx.x; chunk < kt * 8; chunk += 256) {
    int source[16];
#pragma unroll
    for (int j = 0; j < 16; ++j) {
      const int col = chunk * 16 + j;
      source[j] = col < n ? inverse[col] : -1;
      if (col < n && source[j] < 0) atomicMin(info, -1 - col);
    }
#pragma unroll
    for (int r = 0; r < R; ++r) {
      u32x4 w = {0u, 0u, 0u, 0u};
      if (row0 + r < m) {
#pragma unroll
        for (int j = 0; j < 16; ++j)
          if (source[j] >= 0) w[j >> 2] |= (uint32_t)(row_codes[r * ld + source[j]] ^ 0x80u) << (8 * (j & 3));
      }
      *reinterpret_cast<u32x4*>(out + ((int64_t)(row0 / 16) * kt * 8 + chunk) * 256 + ((row0 & 15) + r) * 16) = w;
    }
  }
  if ((int)threadIdx.x < R) {
    const int row = row0 + threadIdx.x;
    float s = 0.f, z = 128.f;
    if (row < m) { s = scales[row]; z = zeros[row]; }
    if (!(z >= 0.f && z <= 255.f && z == rintf(z))) { atomicMax(info, row + 1); z = 128.f; }
    out_scales[row] = s;
    out_shifts[row] = 128 - (int)z;
  }
}

// ---- activations whose rows do not start at 16 bytes or end inside 128 columns: to rows of `ldo` columns, zeros behind the n-th.  Bound by memory, and by its launch where tokens are few.
typedef u32x4 __attribute__((aligned(1))) u32x4_at1;
__global__ __launch_bounds__(256) void linear8_align_kernel(const int8_t* x, int64_t ldx, int n, int8_t* out, int ldo, int64_t pieces) {
  for (int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x; at < pieces; at += (int64_t)gridDim.x * 256) {
    const int64_t t = at / (ldo / 16);
    const int c = (int)(at % (ldo / 16)) * 16;
    const int8_t* from = x + t * ldx + c;
    u32x4 v = {0u, 0u, 0u, 0u};
    if (c + 16 <= n) {
      v = *reinterpret_cast<const u32x4_at1*>(from);
    } else {
#pragma unroll
      for (int j = 0; j < 16; ++j)
        if (c + j < n) v[j >> 2] |= (uint32_t)(uint8_t)from[j] << (8 * (j & 3));
    }
    *reinterpret_cast<u32x4*>(out + t * ldo + c) = v;
  }
}

__device__ __forceinline__ i32x4 linear8_mfma(u32x4 a, u32x4 b, i32x4 c) {
  return __builtin_amdgcn_mfma_i32_16x16x64_i8(__builtin_bit_cast(i32x4, a), __builtin_bit_cast(i32x4, b), c, 0, 0, 0);
}

// ---- few tokens: TT tiles of v_mfma 16x16x64, 16 tokens each.  A workgroup takes RT tiles of 16 rows, its wavefronts share the runs of 128 columns out
// among themselves.  Weights go straight from memory to the lanes that feed the matrix unit, two runs ahead; activations through LDS in runs of a token's 128
// columns, to a place of the wavefront's own.  The activations' sum comes from one more matrix instruction, with ones.
// The left operand is 16 tokens (lane l: token l % 16), the right 16 rows of W, the result has the row in l % 16 and tokens 4 (l / 16) .. + 3.
// Bound by the weights' bytes, small layers by a launch and a trip to memory: 28672 x 8192, 17 tokens 51 us (4.6 TB/s); 4096 x 11008, 37 tokens 12.7 us (3.7 TB/s);
// 4096 x 4096, one token 5.2 to 5.7 us.
constexpr int kFew8Waves = 16;
template <int RT, int TT>
__global__ __launch_bounds__(64 * kFew8Waves) void linear8_few_kernel(Linear8Args p) {
  extern __shared__ __attribute__((aligned(256))) int32_t lds[];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), waves = blockDim.x >> 6;
  const int l16 = lane & 15, q = lane >> 4;
  const int rt0 = blockIdx.x * RT, tok0 = blockIdx.y * TT * 16, tokens = min(p.tokens - tok0, TT * 16);

  const uint8_t* codes[RT];
#pragma unroll
  for (int r = 0; r < RT; ++r) {
    const int64_t tr = rt0 + r < p.mt ? rt0 + r : p.mt - 1;      // (past the last tile of rows: that one again; nothing of it is stored)
    codes[r] = p.codes + tr * p.kt * 2048 + lane * 16;
  }
  // The 16-byte chunks of a token's 128 columns are permuted so that 16 tokens' same chunk lies in 16 different places of 256 bytes.  Places of
  // tokens that there are not hold anything: their results are not stored.
  constexpr int XSTAGE = TT * 2048, NL = TT * 2;
  auto swizzle = [](int row) { return (row >> 1) & 7; };
  unsigned char* const xlds = reinterpret_cast<unsigned char*>(lds) + wave * 2 * XSTAGE;
  const LdsLoader xfrom((const unsigned char*)p.x + (int64_t)tok0 * p.ldx);
  int xsrc[NL];
#pragma unroll
  for (int j = 0; j < NL; ++j) {
    const int row = j * 8 + lane / 8;
    xsrc[j] = min(row, tokens - 1) * (int)p.ldx + ((lane % 8 ^ swizzle(row)) << 4);
  }
  struct Stage { u32x4 w[RT][2]; };
  auto load = [&](Stage& s, int k, int place) {
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt(0xc07f);          // lgkmcnt == 0: the place's last reads are over
#pragma unroll
    for (int j = 0; j < NL; ++j)
      if (j == 0 || j * 8 < tokens) xfrom.load(xlds + place * XSTAGE + j * 1024, xsrc[j], __builtin_amdgcn_readfirstlane(k * 128));
    asm volatile("" ::: "memory");
#pragma unroll
    for (int r = 0; r < RT; ++r)
#pragma unroll
      for (int i = 0; i < 2; ++i) s.w[r][i] = *reinterpret_cast<const u32x4*>(codes[r] + (int64_t)k * 2048 + i * 1024);
  };
  i32x4 acc[TT][RT], accx[TT];
#pragma unroll
  for (int t = 0; t < TT; ++t) {
    accx[t] = i32x4{0, 0, 0, 0};
#pragma unroll
    for (int r = 0; r < RT; ++r) acc[t][r] = i32x4{0, 0, 0, 0};
  }
  const u32x4 ones = {0x01010101u, 0x01010101u, 0x01010101u, 0x01010101u};
  auto multiply = [&](const Stage& s, int place) {
    asm volatile("" :: "v"(s.w[RT - 1][1]) : "memory");     // (where the weights are there, so are the activations, which were asked for before)
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int t = 0; t < TT; ++t) {
        const u32x4 x = *reinterpret_cast<const u32x4*>(xlds + place * XSTAGE + (t * 16 + l16) * 128 + (((4 * i + q) ^ swizzle(l16)) << 4));
        accx[t] = linear8_mfma(x, ones, accx[t]);
#pragma unroll
        for (int r = 0; r < RT; ++r) acc[t][r] = linear8_mfma(x, s.w[r][i], acc[t][r]);
      }
  };
  Stage a, b, c;
  int k = wave;                        // (a workgroup has no more wavefronts than there are runs)
  load(a, k, 0);
  if (k + waves < p.kt) load(b, k + waves, 1);
  for (; k + 3 * waves < p.kt; k += 2 * waves) {
    multiply(a, 0);
    load(a, k + 2 * waves, 0);
    multiply(b, 1);
    load(b, k + 3 * waves, 1);
  }
  multiply(a, 0);
  if (k + 2 * waves < p.kt) load(c, k + 2 * waves, 0);
  if (k + waves < p.kt) multiply(b, 1);
  if (k + 2 * waves < p.kt) multiply(c, 0);
  __syncthreads();                     // (the sums go where other wavefronts' activations are)
#pragma unroll
  for (int r = 0; r < RT; ++r) {
    const int shift = p.shifts[(rt0 + r < p.mt ? rt0 + r : p.mt - 1) * 16 + l16];
#pragma unroll
    for (int t = 0; t < TT; ++t) {
      i32x4 v;
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] = (int)((uint32_t)acc[t][r][e] + (uint32_t)shift * (uint32_t)accx[t][e]);
      *reinterpret_cast<i32x4*>(&lds[(((wave * TT + t) * RT + r) * 64 + lane) * 4]) = v;
    }
  }
  __syncthreads();
  for (int at = threadIdx.x; at < TT * RT * 256; at += blockDim.x) {
    // 16 RT rows of W in a run of threads, so that a token's outputs are written together
    const int r = at % (16 * RT), tok = at / (16 * RT), row = rt0 * 16 + r;
    if (row >= p.out.m || tok >= tokens) continue;
    const int slot = (((tok >> 4) * RT + (r >> 4)) * 64 + (tok & 15) / 4 * 16 + (r & 15)) * 4 + (tok & 3);
    uint32_t sum = 0;
    for (int w = 0; w < waves; ++w) sum += (uint32_t)lds[w * TT * RT * 256 + slot];
    const float v = fmaf((float)(int)sum, p.xs[tok0 + tok] * p.scales[row], p.out.bias ? p.out.bias[row] : 0.f);
    const int64_t o = (int64_t)(tok0 + tok) * p.out.ldy + row;
    if (p.out.y_f32) ((float*)p.out.y)[o] = v;
    else ((uint16_t*)p.out.y)[o] = __builtin_bit_cast(uint16_t, (__bf16)v);
  }
}

template <int RT, int TT>
static hipError_t launch_few8_as(const Linear8Args& p, int waves, hipStream_t s) {
  while (waves > 1 && waves > p.kt) waves /= 2;
  constexpr int kPerWave = TT * 4096 > TT * RT * 1024 ? TT * 4096 : TT * RT * 1024;
  static LdsLimitOnce once;
  if (const hipError_t e = once.ensure((const void*)&linear8_few_kernel<RT, TT>, kFew8Waves * kPerWave); e != hipSuccess) return e;
  hipLaunchKernelGGL((linear8_few_kernel<RT, TT>), dim3((unsigned)((p.mt + RT - 1) / RT), (unsigned)((p.tokens + TT * 16 - 1) / (TT * 16))), dim3(64 * waves),
                     (size_t)(waves * kPerWave), s, p);
  return hipGetLastError();
}
// Two tiles of rows a workgroup, which read the activations half as often, where enough workgroups are left: us a call, one / two, 32 tokens a block: 28672 x 8192, 17 tokens 56.7 /
// 53.6; 4096 x 4096, 64 8.3 / 7.2, 128 13.4 / 10.1; 4096 x 11008, 64 19.8 / 13.0, 128 36.2 / 20.3; 4096 x 1024, 128 5.7 / 4.9; but 1024 x 8192, 128 7.6 / 9.1 and 11008 x 4096, 32 11.3 /
// 12.0 (344 workgroups).
// Blocks of 32 tokens as far as they are few and small; more go to the tiles of linear8_many.hip: us a call, this / that: 4096 x 4096, 128 tokens 10.1 / 16.5, 257 24.4 / 17.1;
// 4096 x 11008, 64 13.0 / 16.6, 96 19.7 / 19.9, 128 20.3 / 21.3; 28672 x 8192, 33 84 / 54; 11008 x 4096, 64 16.1 / 16.4, 96 22.7 / 17.1; 4096 x 1024, 128 4.9 / 7.6; 1024 x 8192, 257
// 15.8 / 16.4.
static hipError_t launch_linear8(const Linear8Args& p, int32_t* partial, hipStream_t s) {
  const int64_t blocks = (p.tokens + 31) / 32, workgroups = blocks * p.mt;
  if (blocks > 1 && (workgroups > 2048 || workgroups * p.kt > 57344)) return launch_linear8_many(p, partial, s);
  const int waves = p.mt < 512 && p.kt >= 64 ? 16 : 8;
  if (p.tokens <= 16) return launch_few8_as<1, 1>(p, waves, s);
  return workgroups >= 512 && (blocks > 1 || p.mt >= 1024) ? launch_few8_as<2, 2>(p, 8, s) : launch_few8_as<1, 2>(p, waves, s);
}

// ---- argument checks

constexpr int64_t kMaxRow8 = (int64_t)1 << 22;          // bytes between rows: 256 of them take 31 bits of offset
constexpr int64_t kMaxRows8 = (int64_t)1 << 20, kMaxColumns8 = (int64_t)1 << 16, kMaxTokens8 = (int64_t)1 << 23, kMaxTiles8 = (int64_t)1 << 23;
static bool good_size8(int64_t m, int64_t n) {
  return m > 0 && n > 0 && m <= kMaxRows8 && n <= kMaxColumns8 && ((m + 15) / 16) * ((n + 127) / 128) <= kMaxTiles8;
}
static size_t aligned_bytes(int64_t tokens, int64_t n) { return ((size_t)tokens * ((n + 127) / 128 * 128) + 255) / 256 * 256; }

}  // namespace gptaq

using namespace gptaq;

extern "C" size_t gptaq_linear8_weights_bytes(int64_t m, int64_t n) { return good_size8(m, n) ? linear8_layout(m, n).bytes : 0; }

extern "C" int gptaq_linear8_pack(const uint8_t* codes, int64_t ldc, const float* scales, const float* zeros, int64_t m, int64_t n, const int32_t* perm,
                                  void* weights, size_t weights_bytes, int32_t* info, void* stream) {
  if (!codes || !scales || !zeros || !weights || !info) return GPTAQ_ENULL;
  if (!good_size8(m, n) || ldc < n || (((uintptr_t)scales | (uintptr_t)zeros | (uintptr_t)perm | (uintptr_t)info) & 3)) return GPTAQ_EDIM;
  const Linear8Layout l = linear8_layout(m, n);
  if (((uintptr_t)weights & 255) || weights_bytes < l.bytes) return GPTAQ_EWORKSPACE;
  const hipStream_t s = (hipStream_t)stream;
  uint8_t* const to = (uint8_t*)weights;
  int32_t* const inverse = (int32_t*)(to + l.inverse);
  const size_t end = l.inverse + (size_t)n * 4;
  const unsigned columns = (unsigned)((n + 255) / 256);
  hipLaunchKernelGGL(linear8_clear_kernel, dim3(columns), dim3(256), 0, s, inverse, (int)n, perm, info, to + end, (int)(l.bytes - end));
  if (perm) hipLaunchKernelGGL(linear8_invert_kernel, dim3(columns), dim3(256), 0, s, inverse, (int)n, perm);
  const int64_t row_bytes = (n + 15) / 16 * 16, rows = 4 * row_bytes <= kPack8Lds ? 4 : 1;
  hipLaunchKernelGGL(rows == 4 ? &linear8_pack_kernel<4> : &linear8_pack_kernel<1>, dim3((unsigned)(l.mt * 16 / rows)), dim3(256), (size_t)(rows * row_bytes), s, codes, ldc,
                     scales, zeros, (int)m, (int)n, (int)l.kt, inverse, to, (float*)(to + l.scales), (int32_t*)(to + l.shifts), info);
  GPTAQ_LAUNCH_CHECK();
  return GPTAQ_OK;
}

extern "C" size_t gptaq_linear8_workspace_bytes(int64_t tokens, int64_t m, int64_t n) {
  if (tokens <= 0 || tokens > kMaxTokens8 || !good_size8(m, n)) return 0;
  return aligned_bytes(tokens, n) + (linear8_partial_bytes(tokens, m, n) + 255) / 256 * 256;
}

extern "C" int gptaq_linear8_i8(const int8_t* X, const float* x_scales, int64_t tokens, int64_t ldx, const void* weights, size_t weights_bytes, int64_t m, int64_t n,
                                const float* bias, void* Y, int64_t ldy, int y_f32, void* ws, size_t ws_bytes, void* stream) {
  if (!weights || (tokens != 0 && (!X || !x_scales || !Y || !ws))) return GPTAQ_ENULL;      // (no tokens: nothing to point to)
  if (tokens < 0 || tokens > kMaxTokens8 || !good_size8(m, n) || ldx < n || ldy < m || ((uintptr_t)weights & 255) || ((uintptr_t)Y & (y_f32 ? 3 : 1)) ||
      (((uintptr_t)x_scales | (uintptr_t)bias) & 3))
    return GPTAQ_EDIM;
  const Linear8Layout l = linear8_layout(m, n);
  if (weights_bytes < l.bytes) return GPTAQ_EWORKSPACE;
  if (tokens == 0) return GPTAQ_OK;
  if (((uintptr_t)ws & 255) || ws_bytes < gptaq_linear8_workspace_bytes(tokens, m, n)) return GPTAQ_EWORKSPACE;
  const hipStream_t s = (hipStream_t)stream;
  const uint8_t* const from = (const uint8_t*)weights;
  Linear8Args p{};
  p.out.bias = bias; p.out.y = Y; p.out.ldy = ldy; p.out.y_f32 = y_f32 ? 1 : 0; p.out.m = (int32_t)m;
  p.x = X; p.xs = x_scales; p.ldx = ldx;
  p.codes = from; p.scales = (const float*)(from + l.scales); p.shifts = (const int32_t*)(from + l.shifts);
  p.mt = (int32_t)l.mt; p.kt = (int32_t)l.kt;
  if (n % 128 || ldx % 16 || ((uintptr_t)X & 15) || ldx > kMaxRow8) {
    const int64_t ld = l.kt * 128, pieces = tokens * (ld / 16), blocks = (pieces + 255) / 256;
    hipLaunchKernelGGL(linear8_align_kernel, dim3((unsigned)(blocks < 16384 ? blocks : 16384)), dim3(256), 0, s, X, ldx, (int)n, (int8_t*)ws, (int)ld, pieces);
    GPTAQ_LAUNCH_CHECK();
    p.x = (const int8_t*)ws;
    p.ldx = ld;
  }
  int32_t* const partial = (int32_t*)((uint8_t*)ws + aligned_bytes(tokens, n));
  // A grid has less than 2^32 threads, and 2^16 blocks along its second axis: more tokens than that takes are several launches.
  int64_t most = (((int64_t)1 << 22) / l.mt) * 16;
  if (most > 65535 * 16) most = 65535 * 16;
  for (int64_t first = 0; first < tokens; first += most) {
    Linear8Args part = p;
    part.tokens = (int32_t)(tokens - first < most ? tokens - first : most);
    part.x = p.x + first * p.ldx;
    part.xs = p.xs + first;
    part.out.y = (uint8_t*)Y + first * ldy * (y_f32 ? 4 : 2);
    if (const hipError_t e = launch_linear8(part, partial, s); e != hipSuccess) { set_last_hip_error(e); return GPTAQ_ELAUNCH; }
  }
  return GPTAQ_OK;
}
