// Layout of a quantised layer's weights as the products read them (gptaq_linear_pack).
#pragma once
#include "common.h"

namespace gptaq {

// Codes lie in tiles of 16 rows by 128 columns, 1 KB each, the tiles of 16 rows one after the other.  A tile is four words for each
// of 64 lanes: word i of lane l holds row l % 16, columns 32 i + 8 (l / 16) .. + 7, which is what the lane feeds to the i-th matrix
// instruction of 32 columns; columns 0 .. 3 of the eight in the even nibbles, 4 .. 7 in the odd ones.  So a wavefront reads a tile
// as one run of 16 bytes a lane.  Behind the codes: scales [tile row][group][16] in fp32, then zeros likewise, one byte each.
// Rows are padded to 16 and columns to 128 with codes, scales and zeros of 0, so padding adds nothing.
struct LinearLayout {
  int64_t mt, kt, groups;              // tiles of rows, tiles of columns, groups (padded to whole column tiles; 1: one per row)
  size_t scales, zeros, bytes;         // offsets of the scales and zeros, total size
};
// group: 32, 64, 128, or 0 for one group per row.
inline LinearLayout linear_layout(int64_t m, int64_t n, int group) {
  LinearLayout l;
  l.mt = (m + 15) / 16;
  l.kt = (n + 127) / 128;
  l.groups = group > 0 ? l.kt * (128 / group) : 1;
  l.scales = (size_t)(l.mt * l.kt) * 1024;
  l.zeros = l.scales + (size_t)(l.mt * l.groups) * 64;
  l.bytes = (l.zeros + (size_t)(l.mt * l.groups) * 16 + 255) / 256 * 256;
  return l;
}

typedef __attribute__((ext_vector_type(2))) uint32_t u32x2;

// code - zero of the eight codes of a word as signed bytes: columns 0 .. 3, then 4 .. 7.  `off` is linear_offset(zero): the differences
// are taken with 128 more in every byte, which keeps a byte's borrow from the next, and flipping bit 7 makes them signed.
__device__ __forceinline__ uint32_t linear_offset(uint32_t zero) { return __builtin_amdgcn_perm(zero, zero, 0u) - 0x80808080u; }
__device__ __forceinline__ u32x2 linear_bytes(uint32_t w, uint32_t off) {
  u32x2 b;
  b[0] = ((w & 0x0f0f0f0fu) - off) ^ 0x80808080u;
  b[1] = (((w >> 4) & 0x0f0f0f0fu) - off) ^ 0x80808080u;
  return b;
}
// The same as bfloat16: integers of at most four bits and a sign, so the conversion is exact.
__device__ __forceinline__ bf16x8 linear_bf16(uint32_t w, uint32_t off) {
  const u32x2 b = linear_bytes(w, off);
  bf16x8 v;
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = (__bf16)(float)(int8_t)(b[i >> 2] >> (8 * (i & 3)));
  return v;
}

// 16 bytes a lane from base + lane offset + scalar offset to 1 KB of LDS.  (A buffer load: behind a global load to LDS the compiler takes LDS reads to
// return in any order, and waits for all of them each time.)
struct LdsLoader {
  __amdgpu_buffer_rsrc_t rsrc;
  __device__ __forceinline__ LdsLoader(const unsigned char* base) : rsrc(__builtin_amdgcn_make_buffer_rsrc((void*)base, 0, 0x7fffffff, 0x00020000)) {}
  __device__ __forceinline__ void load(unsigned char* to, int lane, int scalar) const {
    __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc, (__attribute__((address_space(3))) void*)to, 16, lane, scalar, 0, 0);
  }
};

struct LinearArgs {
  const void* x;                       // tokens x n bf16, or int8 codes
  const float* xs;                     // int8: a scale per token
  int64_t ldx;
  const uint8_t* codes; const float* scales; const uint8_t* zeros;
  const float* bias;
  void* y; int64_t ldy;
  int32_t y_f32;
  int32_t tokens, m, n;
  int32_t mt, kt, groups;
  int32_t parts;                       // linear_many.hip: the columns in so many parts, whose sums (more than one) go to
  float* partial; int64_t ld_partial;  // partial[part][token][row]
};

// Outputs row .. row + 7 of a token, as far as there are so many.  Rows of Y start at any element: global memory takes wide accesses at any address.
typedef u32x4 __attribute__((aligned(2))) u32x4_at2;
typedef u32x4 __attribute__((aligned(4))) u32x4_at4;
__device__ __forceinline__ void linear_store(const LinearArgs& p, int tok, int row, const float (&v)[8]) {
  const int64_t o = (int64_t)tok * p.ldy + row;
  if (p.y_f32) {
    float* y = (float*)p.y + o;
    if (row + 8 <= p.m) {
#pragma unroll
      for (int h = 0; h < 2; ++h)
        *reinterpret_cast<u32x4_at4*>(y + 4 * h) = u32x4{__float_as_uint(v[4 * h]), __float_as_uint(v[4 * h + 1]), __float_as_uint(v[4 * h + 2]), __float_as_uint(v[4 * h + 3])};
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (row + e < p.m) y[e] = v[e];
    }
  } else {
    uint16_t* y = (uint16_t*)p.y + o;
    u32x4 a;
#pragma unroll
    for (int e = 0; e < 4; ++e)
      a[e] = (uint32_t)__builtin_bit_cast(uint16_t, (__bf16)v[2 * e]) | (uint32_t)__builtin_bit_cast(uint16_t, (__bf16)v[2 * e + 1]) << 16;
    if (row + 8 <= p.m) {
      *reinterpret_cast<u32x4_at2*>(y) = a;
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (row + e < p.m) y[e] = (uint16_t)(a[e >> 1] >> (16 * (e & 1)));
    }
  }
}

// linear_many.hip: rows of activations start at 16 bytes, have a multiple of 128 columns, and lie at most kManyMaxRow bytes apart (its
// loads take 31 bits of offset inside 128 rows).
constexpr int64_t kManyMaxRow = ((int64_t)1 << 24) - 16;
hipError_t launch_linear_many(LinearArgs p, int gs, bool i8, float* partial, hipStream_t s);
size_t linear_partial_bytes(int64_t tokens, int64_t m, int64_t n);

}  // namespace gptaq
