// Keys and values of new tokens into a paged cache, keys and queries rotated by their positions on the way.
#include "cache.h"

namespace gptaq {

typedef u32x4 __attribute__((aligned(2))) u32x4_at2;

struct AppendArgs {
  CacheShape c;
  const uint16_t *q, *k, *v; int64_t ldq, hq, ldk, hk, ldv, hv;     // rows of tokens, heads of a row
  uint16_t *keys, *values, *out; int64_t ldo, ho;
  const double* freqs;
  int32_t half, interleaved;                                        // rotated pairs of a head
};

__device__ __forceinline__ float ca_f32(uint32_t h) { return __uint_as_float(h << 16); }
__device__ __forceinline__ uint32_t ca_bf16(float f) { return __builtin_bit_cast(uint16_t, (__bf16)f); }
__device__ __forceinline__ u32x4 ca_pack(const float (&v)[8]) {
  u32x4 a;
#pragma unroll
  for (int i = 0; i < 4; ++i) a[i] = ca_bf16(v[2 * i]) | ca_bf16(v[2 * i + 1]) << 16;
  return a;
}
__device__ __forceinline__ void ca_unpack(u32x4 a, float (&v)[8]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) { v[2 * i] = ca_f32(a[i] & 0xffffu); v[2 * i + 1] = __uint_as_float(a[i] & 0xffff0000u); }
}

// A block is eight positions of a sequence that begin at a multiple of eight: the values' layout has them in one run of 16 bytes, which is
// written whole where all eight are new, and so many tokens share the cosines and sines.  grid.y shares out the block's pieces of 16 entries where there are few blocks.
// (a, b) -> (a cos - b sin, b cos + a sin) in fp32, rounded once; the angle, position * frequency, is reduced to a fraction of a turn in fp64, as positions
// times the largest frequency pass what fp32 resolves, and its sine and cosine are taken in fp32 from there (2^-24 of a turn, a 2^-13th of a bf16 rounding).
// Bound by memory: five prompts of up to 4096 tokens, 32 heads of 128, 373 MB in 87 to 89 us (4.2 to 4.3 TB/s); 37 tokens by the launch and two trips to memory, 4.3 us.
__global__ __launch_bounds__(256) void append_kernel(AppendArgs p) {
  __shared__ float turn[8 * 256];                                   // [position in the block][pair][cos, sin], 128 pairs at most
  const CacheShape& c = p.c;
  const int s = cache_find(c, blockIdx.x, 1, 3, 2);
  const Sequence seq = cache_sequence(c, s);
  const int end = seq.before + seq.count;
  const int64_t from = ((int64_t)(seq.before >> 3) + ((int64_t)blockIdx.x - cache_block_of(c, s, 1, 3, 2))) * 8;
  if (seq.count == 0 || from >= end || from + 8 <= 0) return;
  const int first = max(max((int)from, seq.before), 0), n = min((int)from + 8, end) - first;      // positions of this block that are new
  if (n <= 0) return;
  const int half = p.half;
  for (int i = threadIdx.x; i < n * half; i += 256) {
    const int at = i / half, j = i - at * half;
    const double turns = (double)(first + at) * p.freqs[j] * 0.15915494309189533577;
    float sn, cs;
    sincospif(2.f * (float)(turns - rint(turns)), &sn, &cs);
    turn[(at * 128 + j) * 2] = cs;
    turn[(at * 128 + j) * 2 + 1] = sn;
  }
  __syncthreads();
  const int id = cache_page(c, s, first);                           // (eight positions are of one page)
  const int slot = first & ((1 << c.page_bits) - 1), page = 1 << c.page_bits, d = c.d;
  const int64_t row0 = seq.first + (first - seq.before);
  const int64_t kv_page = (int64_t)id * c.kv_heads;
  // ---- queries and keys: 16 entries a thread, the tokens of a block side by side
  const int pieces = d / 16, heads = c.heads + c.kv_heads, items = n * pieces * heads;
  for (int i = blockIdx.y * 256 + threadIdx.x; i < items; i += gridDim.y * 256) {
    const int at = i % n, rest = i / n, piece = rest % pieces, head = rest / pieces;
    const bool is_key = head >= c.heads;
    const int h = is_key ? head - c.heads : head;
    if (is_key && id < 0) continue;
    const uint16_t* from_row = is_key ? p.k + (row0 + at) * p.ldk + h * p.hk : p.q + (row0 + at) * p.ldq + h * p.hq;
    const bool turned = piece * 8 < half, apart = turned && !p.interleaved;
    const int c0 = apart ? piece * 8 : piece * 16, c1 = apart ? half + piece * 8 : c0 + 8;
    float a[8], b[8];
    ca_unpack(*reinterpret_cast<const u32x4_at2*>(from_row + c0), a);
    ca_unpack(*reinterpret_cast<const u32x4_at2*>(from_row + c1), b);
    if (turned) {
      const float* t = turn + (at * 128 + piece * 8) * 2;
      if (apart) {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const float cs = t[2 * j], sn = t[2 * j + 1], x = a[j], y = b[j];
          a[j] = x * cs - y * sn;
          b[j] = y * cs + x * sn;
        }
      } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const float cs = t[2 * j], sn = t[2 * j + 1];
          float& first_of = j < 4 ? a[2 * j & 7] : b[2 * j & 7];
          float& second_of = j < 4 ? a[(2 * j + 1) & 7] : b[(2 * j + 1) & 7];
          const float x = first_of, y = second_of;
          first_of = x * cs - y * sn;
          second_of = y * cs + x * sn;
        }
      }
    }
    if (is_key) {
      uint16_t* to = p.keys + ((kv_page + h) * (d / 8) * page + slot + at) * 8;
      *reinterpret_cast<u32x4*>(to + (int64_t)(c0 / 8) * page * 8) = ca_pack(a);
      *reinterpret_cast<u32x4*>(to + (int64_t)(c1 / 8) * page * 8) = ca_pack(b);
    } else {
      uint16_t* to = p.out + (row0 + at) * p.ldo + h * p.ho;
      *reinterpret_cast<u32x4_at2*>(to + c0) = ca_pack(a);
      *reinterpret_cast<u32x4_at2*>(to + c1) = ca_pack(b);
    }
  }
  if (id < 0) return;
  // ---- values: eight entries of all the block's tokens a thread, turned so that an entry's tokens are side by side
  const int eights = d / 8, slot8 = slot & 7;
  for (int i = blockIdx.y * 256 + threadIdx.x; i < eights * c.kv_heads; i += gridDim.y * 256) {
    const int e0 = i % eights * 8, h = i / eights;
    const uint16_t* row = p.v + row0 * p.ldv + h * p.hv + e0;
    uint16_t* to = p.values + ((kv_page + h) * (page / 8) + slot / 8) * d * 8 + (int64_t)e0 * 8;
    if (n == 8) {
      u32x4 r[8];
#pragma unroll
      for (int t = 0; t < 8; ++t) r[t] = *reinterpret_cast<const u32x4_at2*>(row + t * p.ldv);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        u32x4 w;
#pragma unroll
        for (int t = 0; t < 4; ++t)
          w[t] = __builtin_amdgcn_perm(r[2 * t + 1][e >> 1], r[2 * t][e >> 1], e & 1 ? 0x07060302u : 0x05040100u);
        *reinterpret_cast<u32x4*>(to + e * 8) = w;
      }
    } else {
      for (int t = 0; t < n; ++t) {
        const u32x4 r = *reinterpret_cast<const u32x4_at2*>(row + t * p.ldv);
#pragma unroll
        for (int e = 0; e < 8; ++e) to[e * 8 + slot8 + t] = (uint16_t)(r[e >> 1] >> (16 * (e & 1)));
      }
    }
  }
}

}  // namespace gptaq

using namespace gptaq;

extern "C" int gptaq_cache_append(const uint16_t* q, int64_t ldq, int64_t hq, const uint16_t* k, int64_t ldk, int64_t hk, const uint16_t* v, int64_t ldv, int64_t hv,
                                  const gptaq_cache* cache, int64_t tokens, int64_t heads, const double* freqs, int64_t pairs, int interleaved, uint16_t* out,
                                  int64_t ldo, int64_t ho, void* stream) {
  AppendArgs p{};
  if (const int rc = cache_shape(p.c, cache, tokens, heads)) return rc;
  const int64_t d = cache->d, kv_heads = cache->kv_heads, seqs = cache->seqs;
  if (tokens != 0 && seqs != 0 && (!q || !k || !v || !out || (pairs != 0 && !freqs))) return GPTAQ_ENULL;
  if (d <= 0 || d % 16 || d > 256 || pairs < 0 || pairs % 8 || 2 * pairs > d) return GPTAQ_EUNSUPPORTED;
  if ((((uintptr_t)q | (uintptr_t)k | (uintptr_t)v | (uintptr_t)out) & 1) || ((uintptr_t)freqs & 7) ||
      ldq < 0 || hq < 0 || ldk < 0 || hk < 0 || ldv < 0 || hv < 0 || !cache_rows_apart(tokens, ldo, heads, ho, d))
    return GPTAQ_EDIM;
  if (out == q && tokens != 0 && (ldo != ldq || ho != hq)) return GPTAQ_EUNSUPPORTED;
  if (tokens == 0 || seqs == 0) return GPTAQ_OK;
  p.q = q; p.k = k; p.v = v; p.ldq = ldq; p.hq = hq; p.ldk = ldk; p.hk = hk; p.ldv = ldv; p.hv = hv;
  p.keys = cache->keys; p.values = cache->values; p.out = out; p.ldo = ldo; p.ho = ho;
  p.freqs = freqs; p.half = (int32_t)pairs; p.interleaved = interleaved ? 1 : 0;
  const int64_t blocks = tokens / 8 + 2 * seqs;
  const int64_t items = (heads + kv_heads) * (d / 16);              // of a token
  int64_t share = blocks < 1024 ? (items + 255) / 256 : 1;
  if (share > 64) share = 64;
  hipLaunchKernelGGL(append_kernel, dim3((unsigned)blocks, (unsigned)share), dim3(256), 0, (hipStream_t)stream, p);
  GPTAQ_LAUNCH_CHECK();
  return GPTAQ_OK;
}
