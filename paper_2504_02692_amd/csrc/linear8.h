// Layout of a layer's weights with codes of up to 8 bits as the products read them (gptaq_linear8_pack).
#pragma once
#include "linear.h"

namespace gptaq {

typedef __attribute__((ext_vector_type(4))) int32_t i32x4;
typedef __attribute__((ext_vector_type(16))) int32_t i32x16;

// code - zero has nine bits, so the matrix instructions multiply code - 128, and
//   sum_j (code_j - zero) x_j = sum_j (code_j - 128) x_j + (128 - zero) sum_j x_j,
// all in int32: every partial sum may wrap, the result is below 255 * 128 * 65536 < 2^31 and exact in any order.  128 - zero is the row's `shift`.
// Codes lie in tiles of 16 rows by 64 columns, 1 KB each, the tiles of 16 rows one after the other: 16 columns of a row are 16 bytes, the rows of 16
// columns one run of 256.  So lane l of a wavefront, 16 bytes each, has row l % 16 and columns 16 (l / 16) .. + 15, the operand of v_mfma 16x16x64; two tiles of
// rows likewise make that of 32x32x32.  Columns are in the order of the activations, whatever order the solve took them in (one scale a row: nothing depends on
// it), so a product reads its activations as they are.  Rows are padded to 16 and columns to 128 with bytes, scales and shifts of 0.
// Behind the codes: scales, shifts (int32), and the inverse of the columns' order, which only the layout itself needs.
struct Linear8Layout {
  int64_t mt, kt;                      // tiles of 16 rows, runs of 128 columns
  size_t scales, shifts, inverse, bytes;
};
inline Linear8Layout linear8_layout(int64_t m, int64_t n) {
  Linear8Layout l;
  l.mt = (m + 15) / 16;
  l.kt = (n + 127) / 128;
  l.scales = (size_t)(l.mt * l.kt) * 2048;
  l.shifts = l.scales + (size_t)l.mt * 64;
  l.inverse = l.shifts + (size_t)l.mt * 64;
  l.bytes = (l.inverse + (size_t)n * 4 + 255) / 256 * 256;
  return l;
}

struct Linear8Args {
  LinearArgs out;                      // what linear_store reads: bias, y, ldy, y_f32, m
  const int8_t* x; const float* xs; int64_t ldx;
  const uint8_t* codes; const float* scales; const int32_t* shifts;
  int32_t tokens, mt, kt;
  int32_t parts;                       // linear8_many.hip: the columns in so many parts, whose sums (more than one) go to
  int32_t* partial; int64_t ld_partial;                             // partial[part][token][row]
};

// linear8_many.hip
hipError_t launch_linear8_many(Linear8Args p, int32_t* partial, hipStream_t s);
size_t linear8_partial_bytes(int64_t tokens, int64_t m, int64_t n);

}  // namespace gptaq
