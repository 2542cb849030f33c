// What lies between the products of a quantised layer set: the root-mean-square norm with the residual's addition, and the gated
// activation, each with its output in bfloat16 or as 8-bit codes with one scale per token; and rows that are in bfloat16 already as such codes.
#include "common.h"

namespace gptaq {

__device__ __forceinline__ float ro_lo(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float ro_hi(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }
__device__ __forceinline__ uint32_t ro_bf16(float f) { return __builtin_bit_cast(uint16_t, (__bf16)f); }

// Eight values of a row.  Rows may start at any multiple of 2 bytes (an odd number of columns): global memory takes wide accesses
// at any address, so only the last, ragged piece of a row goes value by value.
typedef u32x4 __attribute__((aligned(2))) u32x4_any;
typedef __attribute__((ext_vector_type(2))) uint32_t u32x2;
typedef u32x2 __attribute__((aligned(1))) u32x2_any;

__device__ __forceinline__ void ro_load(const uint16_t* row, int c, int n, float (&v)[8]) {
  u32x4 a = {0u, 0u, 0u, 0u};
  if (c + 8 <= n) {
    a = *reinterpret_cast<const u32x4_any*>(row + c);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (c + i < n) a[i >> 1] |= (uint32_t)row[c + i] << (16 * (i & 1));
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) { v[2 * i] = ro_lo(a[i]); v[2 * i + 1] = ro_hi(a[i]); }
}
__device__ __forceinline__ void ro_store(uint16_t* row, int c, int n, const float (&v)[8]) {
  u32x4 a;
#pragma unroll
  for (int i = 0; i < 4; ++i) a[i] = ro_bf16(v[2 * i]) | (ro_bf16(v[2 * i + 1]) << 16);
  if (c + 8 <= n) {
    *reinterpret_cast<u32x4_any*>(row + c) = a;
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (c + i < n) row[c + i] = (uint16_t)(a[i >> 1] >> (16 * (i & 1)));
  }
}
__device__ __forceinline__ void ro_store_codes(int8_t* row, int c, int n, const int (&q)[8]) {
  u32x2 a = {0u, 0u};
#pragma unroll
  for (int i = 0; i < 8; ++i) a[i >> 2] |= (uint32_t)(q[i] & 255) << (8 * (i & 3));
  if (c + 8 <= n) {
    *reinterpret_cast<u32x2_any*>(row + c) = a;
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (c + i < n) row[c + i] = (int8_t)(a[i >> 2] >> (8 * (i & 3)));
  }
}

// Sum and maximum over 16 lanes, by exchanges inside the row of lanes that need no LDS.
__device__ __forceinline__ int ro_lanes(int v, int step) {
  switch (step) {
    case 0: return __builtin_amdgcn_update_dpp(0, v, 0xB1, 0xf, 0xf, true);       // quad_perm 1 0 3 2
    case 1: return __builtin_amdgcn_update_dpp(0, v, 0x4E, 0xf, 0xf, true);       // quad_perm 2 3 0 1
    case 2: return __builtin_amdgcn_update_dpp(0, v, 0x141, 0xf, 0xf, true);      // row_half_mirror
    default: return __builtin_amdgcn_update_dpp(0, v, 0x140, 0xf, 0xf, true);     // row_mirror
  }
}
__device__ __forceinline__ void ro_reduce16(float& sum, uint32_t& top) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    sum += __int_as_float(ro_lanes(__float_as_int(sum), i));
    const uint32_t t = (uint32_t)ro_lanes((int)top, i);
    top = top > t ? top : t;
  }
}
// Sum and maximum over the workgroup's threads of one row; the maximum of absolute values as bit patterns, so that a NaN, whose
// pattern is above infinity's, is not lost.  `part` holds 2 x 64 words; every thread of the workgroup calls this.
__device__ __forceinline__ void ro_reduce(float& sum, uint32_t& top, int waves, float* part) {
  ro_reduce16(sum, top);
  if (waves == 1) {
    const float s = sum;
    const uint32_t t = top;
    sum = 0.f;
    top = 0u;
#pragma unroll
    for (int l = 0; l < 64; l += 16) {
      sum += __int_as_float(__builtin_amdgcn_readlane(__float_as_int(s), l));
      const uint32_t u = (uint32_t)__builtin_amdgcn_readlane((int)t, l);
      top = top > u ? top : u;
    }
    return;
  }
  // four sums a wavefront: lane l of every row of 16 lanes takes those of places l, l + 16, ..
  uint32_t* tops = reinterpret_cast<uint32_t*>(part + 64);
  if ((threadIdx.x & 15) == 0) { part[threadIdx.x >> 4] = sum; tops[threadIdx.x >> 4] = top; }
  __syncthreads();
  sum = 0.f;
  top = 0u;
  for (int at = threadIdx.x & 15; at < 4 * waves; at += 16) {
    sum += part[at];
    top = top > tops[at] ? top : tops[at];
  }
  ro_reduce16(sum, top);
}

// g / (1 + exp(-g)).  The reciprocal instruction returns 0 where its result is below fp32's normal range, that is for a sum above 2^126 (g about -87):
// so it takes a quarter of the sum.
__device__ __forceinline__ float ro_silu(float g) {
  const float quarter = fmaf(0.25f, __expf(-g), 0.25f);
  return g * __builtin_amdgcn_rcpf(quarter) * 0.25f;
}

struct RowArgs {
  const uint16_t *a, *b, *weight;      // norm: x, residual (or NULL), weight (or NULL); gated: gate, up; plain: x
  int64_t lda, ldb;
  uint16_t* sum; int64_t lds;          // norm with a residual: bf16(x + residual)
  uint16_t* y; int8_t* codes; int64_t ldy;
  float* scales;
  int first, tokens, n;                // rows first .. first + tokens - 1
  float eps, clip;
};

// Bound by memory: 16384 x 8192 with residual 190 us, 5.7 TB/s read and written (a plain copy reaches 5.0); gated 16384 x 11008 187 us, 5.8 TB/s; one
// row of 4096 4 us, most of it the launch.
// One row per workgroup (T threads) or, rows of one wavefront, several rows per workgroup.  A thread keeps its first KEEP pieces of
// eight columns between the pass that takes the row's sums and the one that writes; later pieces are read again.  Outputs in bf16 may be
// the inputs' own memory: a thread writes only columns that it has read, and reads no others.  (Codes take half the bytes: not where other threads' columns were.)
// 8 bits: scale = clip * max|y| / 127, code = rint(y / scale); the maximum is taken of |h w| and multiplied by the positive 1 / rms
// afterwards, so one pass and one reduction give both.
// Plain rows take the nearest code to the quotient itself: their values have eight bits, so quotients between two codes are common where
// the scale has few bits, and a product with the reciprocal would break those ties at random.  The product is within 2 ulp of the quotient: it is
// divided only where a tie is as near as that, which few wavefronts meet (16384 x 8192 85 us, 4.7 TB/s).
enum RowKind { kGated = 0, kNorm = 1, kPlain = 2 };
template <int KIND, bool CODES>
__global__ __launch_bounds__(1024) void row_kernel(RowArgs p) {
  constexpr bool NORM = KIND == kNorm;
  __shared__ float part[128];
  constexpr int KEEP = 4;
  const int T = blockDim.x, waves = T >> 6;
  const int in_grid = blockIdx.x * blockDim.y + threadIdx.y;
  if (in_grid >= p.tokens) return;                     // (blockDim.y > 1: one wavefront a row and no barrier; else never)
  const int64_t t = p.first + in_grid;
  const uint16_t* a = p.a + t * p.lda;
  const uint16_t* b = p.b ? p.b + t * p.ldb : nullptr;
  const int n = p.n;
  float keep[KEEP][8];
  float ss = 0.f;
  uint32_t top = 0u;
  auto value = [&](int c, float (&v)[8]) {             // norm: h; gated: y
    float u[8];
    ro_load(a, c, n, v);
    if (NORM) {
      if (b) {
        ro_load(b, c, n, u);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] += u[i];
      }
    } else if (KIND == kGated) {
      ro_load(b, c, n, u);
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = ro_silu(v[i]) * u[i];
    }
  };
  auto weight = [&](int c, float (&w)[8]) {
    if (p.weight) {
      ro_load(p.weight, c, n, w);
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) w[i] = 1.f;
    }
  };
  auto sums = [&](int c, const float (&v)[8]) {
    float w[8];
    if (NORM && CODES) weight(c, w);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      if (NORM) ss = fmaf(v[i], v[i], ss);
      if (CODES) {
        const uint32_t bits = __float_as_uint(fabsf(NORM ? v[i] * w[i] : v[i]));
        top = bits > top ? bits : top;
      }
    }
  };
  if (NORM || CODES) {
#pragma unroll
    for (int k = 0; k < KEEP; ++k) {
      const int c = (threadIdx.x + k * T) * 8;
      if (c < n) { value(c, keep[k]); sums(c, keep[k]); }
    }
    for (int c = (threadIdx.x + KEEP * T) * 8; c < n; c += T * 8) {
      float v[8];
      value(c, v);
      sums(c, v);
    }
    ro_reduce(ss, top, waves, part);
  }
  float r = 1.f;
  if (NORM) {
    const float square = ss / (float)n + p.eps;
    r = square == 0.f ? 0.f : 1.f / sqrtf(square);     // (eps = 0 and a row of zeros: zeros, as for every other eps)
  }
  float scale = 0.f, inv = 0.f;
  bool divide = false;
  if (CODES) {
    scale = __uint_as_float(top) * r * (p.clip / 127.f);
    inv = scale > 0.f ? 1.f / scale : 0.f;
    divide = !(inv < __builtin_inff());                // a scale below 2^-128 has no reciprocal
    if (!(scale < __builtin_inff())) { scale = __builtin_nanf(""); inv = 0.f; divide = false; }
    if (threadIdx.x == 0) p.scales[t] = scale;
  }
  auto put = [&](int c, float (&v)[8]) {
    if (NORM) {
      if (p.sum) ro_store(p.sum + t * p.lds, c, n, v);
      float w[8];
      weight(c, w);
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = v[i] * r * w[i];
    }
    if (CODES) {
      int q[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        float f = divide ? v[i] / scale : v[i] * inv;
        if (KIND == kPlain && !divide && fabsf(f - rintf(f)) > 0.4999f) f = v[i] / scale;
        q[i] = (int)rintf(fminf(fmaxf(f, -127.f), 127.f));     // (a row that is not finite: inv is 0, NaN becomes -127)
      }
      ro_store_codes(p.codes + t * p.ldy, c, n, q);
    } else {
      ro_store(p.y + t * p.ldy, c, n, v);
    }
  };
#pragma unroll
  for (int k = 0; k < KEEP; ++k) {
    const int c = (threadIdx.x + k * T) * 8;
    if (c < n) {
      if (!NORM && !CODES) value(c, keep[k]);
      put(c, keep[k]);
    }
  }
  for (int c = (threadIdx.x + KEEP * T) * 8; c < n; c += T * 8) {
    float v[8];
    value(c, v);
    put(c, v);
  }
}

static int launch_rows(RowArgs p, RowKind kind, void* stream) {
  const int pieces = (p.n + 7) / 8;
  // Threads of a row.  With few rows, or nothing to reduce, one piece each: a row takes the least time.  With many rows two to four pieces, and 512
  // threads as far as these hold a row, so that three rows share a CU (76 to 79 registers: six wavefronts a SIMD) and one reads while another waits in its reduction.
  // 16384 x 8192, norm / 8 bits, 1024, 512, 256 threads: 237 / 254, 194 / 197, 203 / 191 us; 16384 x 11008, 1024, 704, 512: 338 / 388, 277 / 307, 265 / 268.
  const bool reduces = kind == kNorm || p.codes;
  int T = p.tokens < 512 || !reduces ? pieces : pieces <= 2048 ? (pieces + 1) / 2 : (pieces + 3) / 4;
  if (p.tokens >= 512 && reduces && pieces <= 2048 && T > 512) T = 512;
  T = (T + 63) / 64 * 64;
  if (T > 1024) T = 1024;
  const int rows = T == 64 ? 4 : 1;
  const auto kernel = kind == kNorm ? (p.codes ? &row_kernel<kNorm, true> : &row_kernel<kNorm, false>)
                      : kind == kGated ? (p.codes ? &row_kernel<kGated, true> : &row_kernel<kGated, false>) : &row_kernel<kPlain, true>;
  constexpr int kRowsPerLaunch = 1 << 21;              // (a grid has less than 2^32 threads)
  const int tokens = p.tokens;
  for (int64_t first = 0; first < tokens; first += kRowsPerLaunch) {
    p.first = (int)first;
    p.tokens = (int)(tokens - first < kRowsPerLaunch ? tokens - first : kRowsPerLaunch);
    hipLaunchKernelGGL(kernel, dim3((unsigned)((p.tokens + rows - 1) / rows)), dim3(T, rows), 0, (hipStream_t)stream, p);
    GPTAQ_LAUNCH_CHECK();
  }
  return GPTAQ_OK;
}

constexpr int64_t kMaxTokens = ((int64_t)1 << 31) - 8, kMaxColumns = (int64_t)1 << 24;
static bool odd(const void* a) { return ((uintptr_t)a & 1) != 0; }
static bool same(const void* a, const void* b) { return a == b; }

static int norm_args(RowArgs& p, const uint16_t* X, const uint16_t* residual, const uint16_t* weight, int64_t tokens, int64_t n,
                     int64_t ldx, int64_t ldr, float eps, uint16_t* sum, int64_t lds, int64_t ldy) {
  if (tokens < 0 || tokens > kMaxTokens || n <= 0 || n > kMaxColumns || ldx < n || ldy < n || (residual && ldr < n) || (sum && lds < n) ||
      odd(X) || odd(residual) || odd(weight) || odd(sum))
    return GPTAQ_EDIM;
  if (!(eps >= 0.f) || !(eps < __builtin_inff())) return GPTAQ_EUNSUPPORTED;
  p = RowArgs{};
  p.a = X; p.b = residual; p.weight = weight;
  p.lda = ldx; p.ldb = ldr;
  p.sum = sum; p.lds = lds; p.ldy = ldy;
  p.tokens = (int)tokens; p.n = (int)n; p.eps = eps;
  return GPTAQ_OK;
}

static int gated_args(RowArgs& p, const uint16_t* gate, const uint16_t* up, int64_t tokens, int64_t n, int64_t ldg, int64_t ldu, int64_t ldy) {
  if (tokens < 0 || tokens > kMaxTokens || n <= 0 || n > kMaxColumns || ldg < n || ldu < n || ldy < n || odd(gate) || odd(up)) return GPTAQ_EDIM;
  p = RowArgs{};
  p.a = gate; p.b = up;
  p.lda = ldg; p.ldb = ldu; p.ldy = ldy;
  p.tokens = (int)tokens; p.n = (int)n;
  return GPTAQ_OK;
}

}  // namespace gptaq

using namespace gptaq;

extern "C" int gptaq_rms_norm(const uint16_t* X, const uint16_t* residual, const uint16_t* weight, int64_t tokens, int64_t n, int64_t ldx,
                              int64_t ldr, float eps, uint16_t* sum, int64_t lds, uint16_t* Y, int64_t ldy, void* stream) {
  if (tokens != 0 && (!X || !Y)) return GPTAQ_ENULL;
  RowArgs p;
  if (const int rc = norm_args(p, X, residual, weight, tokens, n, ldx, ldr, eps, sum, lds, ldy)) return rc;
  if (odd(Y)) return GPTAQ_EDIM;
  p.y = Y;
  return launch_rows(p, kNorm, stream);
}

extern "C" int gptaq_rms_norm_i8(const uint16_t* X, const uint16_t* residual, const uint16_t* weight, int64_t tokens, int64_t n, int64_t ldx,
                                 int64_t ldr, float eps, uint16_t* sum, int64_t lds, float clip, int8_t* codes, int64_t ldc, float* scales,
                                 void* stream) {
  if (tokens != 0 && (!X || !codes || !scales)) return GPTAQ_ENULL;
  RowArgs p;
  if (const int rc = norm_args(p, X, residual, weight, tokens, n, ldx, ldr, eps, sum, lds, ldc)) return rc;
  if (!(clip > 0.f && clip <= 1.f)) return GPTAQ_EUNSUPPORTED;
  if (tokens != 0 && (same(codes, X) || same(codes, residual) || same(codes, sum))) return GPTAQ_EUNSUPPORTED;
  p.codes = codes; p.scales = scales; p.clip = clip;
  return launch_rows(p, kNorm, stream);
}

extern "C" int gptaq_silu_mul(const uint16_t* gate, const uint16_t* up, int64_t tokens, int64_t n, int64_t ldg, int64_t ldu, uint16_t* Y,
                              int64_t ldy, void* stream) {
  if (tokens != 0 && (!gate || !up || !Y)) return GPTAQ_ENULL;
  RowArgs p;
  if (const int rc = gated_args(p, gate, up, tokens, n, ldg, ldu, ldy)) return rc;
  if (odd(Y)) return GPTAQ_EDIM;
  p.y = Y;
  return launch_rows(p, kGated, stream);
}

extern "C" int gptaq_silu_mul_i8(const uint16_t* gate, const uint16_t* up, int64_t tokens, int64_t n, int64_t ldg, int64_t ldu, float clip,
                                 int8_t* codes, int64_t ldc, float* scales, void* stream) {
  if (tokens != 0 && (!gate || !up || !codes || !scales)) return GPTAQ_ENULL;
  RowArgs p;
  if (const int rc = gated_args(p, gate, up, tokens, n, ldg, ldu, ldc)) return rc;
  if (!(clip > 0.f && clip <= 1.f)) return GPTAQ_EUNSUPPORTED;
  if (tokens != 0 && (same(codes, gate) || same(codes, up))) return GPTAQ_EUNSUPPORTED;
  p.codes = codes; p.scales = scales; p.clip = clip;
  return launch_rows(p, kGated, stream);
}

extern "C" int gptaq_quant_activations_i8(const uint16_t* X, int64_t tokens, int64_t n, int64_t ldx, float clip, int8_t* codes, int64_t ldc, float* scales,
                                          void* stream) {
  if (tokens != 0 && (!X || !codes || !scales)) return GPTAQ_ENULL;
  if (tokens < 0 || tokens > kMaxTokens || n <= 0 || n > kMaxColumns || ldx < n || ldc < n || odd(X) || ((uintptr_t)scales & 3)) return GPTAQ_EDIM;
  if (!(clip > 0.f && clip <= 1.f)) return GPTAQ_EUNSUPPORTED;
  if (tokens != 0 && same(codes, X)) return GPTAQ_EUNSUPPORTED;
  RowArgs p{};
  p.a = X; p.lda = ldx; p.ldy = ldc;
  p.tokens = (int)tokens; p.n = (int)n;
  p.codes = codes; p.scales = scales; p.clip = clip;
  return launch_rows(p, kPlain, stream);
}
