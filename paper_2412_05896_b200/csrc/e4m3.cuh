// Cache rows stored as 8-bit floats (1-4-3, "e4m3") with one power-of-two scale per block of 16 slots and KV head:
// the encoding every writer of such a cache shares (compaction, append, rows stored by slot).
//
// A block's scale s is the smallest power of two (exponent within [-100, 120]) with max|x| <= 448 s over the finite
// values of its rows; a stored code is x / s rounded to nearest, ties to even, saturating at +-448 (a NaN stays a NaN).
// The scale is a power of two so that x / s is exact and a block whose scale has to grow (a later row is larger)
// re-expresses its earlier codes by an exponent shift: exact unless the code falls below the normal range 2^-6, where
// it is rounded once more (at most half of that range's step 2^-9, in units of the new scale).
#pragma once

#include "common.cuh"

namespace xkv {

constexpr int kScaleBlock = 16;                 // slots that share a scale; page_size is a multiple

// Smallest power of two s with amax <= 448 s; amax finite and >= 0 (zero and subnormals take the smallest scale).
__device__ __forceinline__ float e4m3_block_scale(float amax) {
  const uint32_t u = __float_as_uint(amax);
  int e = (int)(u >> 23) - 127;                              // amax = f 2^e, f in [1, 2);  448 = 1.75 2^8
  e = (u & 0x7fffffu) > 0x600000u ? e - 7 : e - 8;
  e = max(-100, min(120, e));
  return __uint_as_float((uint32_t)(e + 127) << 23);
}

// Two fp32 -> two codes, `lo` in the low byte; nearest, ties to even, saturating, NaN -> 0x7f.
__device__ __forceinline__ uint32_t e4m3x2_from_f32(float lo, float hi) {
  uint16_t r;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(hi), "f"(lo));
  return r;
}
// Two codes (low 16 bits of w) -> two fp32, exact.
__device__ __forceinline__ float2 f32_from_e4m3x2(uint32_t w) {
  uint32_t h;
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"((uint16_t)w));
  float2 f;
  asm("{\n\t.reg .b16 a, b;\n\tmov.b32 {a, b}, %2;\n\tcvt.f32.f16 %0, a;\n\tcvt.f32.f16 %1, b;\n\t}"
      : "=f"(f.x), "=f"(f.y)
      : "r"(h));
  return f;
}
// Two bf16 times a power of two (exact, or below every code's reach), in one instruction.
__device__ __forceinline__ uint32_t bf16x2_scale(uint32_t v, __nv_bfloat162 f) {
  const __nv_bfloat162 r = __hmul2(*reinterpret_cast<const __nv_bfloat162*>(&v), f);
  return *reinterpret_cast<const uint32_t*>(&r);
}
// Sixteen bf16 (two 16-byte pieces) times inv, a power of two, -> sixteen codes.
__device__ __forceinline__ uint4 e4m3x16_from_bf16(const uint4& a, const uint4& b, float inv) {
  const uint32_t w[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
  const __nv_bfloat162 f = __float2bfloat162_rn(inv);
  uint32_t r[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t x = bf16x2_scale(w[2 * i], f), y = bf16x2_scale(w[2 * i + 1], f);
    r[i] = __byte_perm(e4m3x2_from_f32(bf16_lo(x), bf16_hi(x)), e4m3x2_from_f32(bf16_lo(y), bf16_hi(y)), 0x5410);
  }
  return make_uint4(r[0], r[1], r[2], r[3]);
}
// Sixteen codes times a power of two <= 1, rounded back to codes.
__device__ __forceinline__ uint32_t e4m3x4_shift(uint32_t w, float factor) {
  const float2 lo = f32_from_e4m3x2(w & 0xffffu), hi = f32_from_e4m3x2(w >> 16);
  return e4m3x2_from_f32(lo.x * factor, lo.y * factor) | (e4m3x2_from_f32(hi.x * factor, hi.y * factor) << 16);
}
// Largest finite magnitude of two bf16 as bf16 bits in both halves (non-finite values count as zero).
__device__ __forceinline__ uint32_t finite_abs_bf16x2(uint32_t v) {
  const uint32_t m = v & 0x7fff7fffu;
  return m & ~__vcmpgeu2(m, 0x7f807f80u);
}

// Stores n_new rows behind the n_old rows that the block already holds; all 32 lanes of a warp take part.
//   codes   first byte of the block: 16 rows of D bytes, contiguous
//   scale   the block's scale; read only when n_old > 0
//   row_of  i -> the bf16 values of new row i (16-byte aligned)
// n_old >= 0, n_new >= 1, n_old + n_new <= 16.  Rows behind the new ones keep their bytes.
template <int D, class RowOf>
__device__ __forceinline__ void e4m3_store_block(uint8_t* codes, float* scale, int n_old, int n_new, RowOf row_of) {
  constexpr int kLanesPerRow = D / 16;                       // a lane carries 16 consecutive values of a row
  constexpr int kRowsPerPass = 32 / kLanesPerRow;
  constexpr int kPasses = kScaleBlock / kRowsPerPass;
  const int lane = threadIdx.x & 31;
  const int lr = lane / kLanesPerRow, lc = lane % kLanesPerRow;
  uint4 x[kPasses][2];
#pragma unroll
  for (int p = 0; p < kPasses; ++p) {
    const int i = p * kRowsPerPass + lr - n_old;
    x[p][0] = x[p][1] = make_uint4(0u, 0u, 0u, 0u);
    if (i >= 0 && i < n_new) {
      const uint4* src = reinterpret_cast<const uint4*>(row_of(i)) + 2 * lc;
      x[p][0] = __ldg(src);
      x[p][1] = __ldg(src + 1);
    }
  }
  auto largest = [&](auto magnitude) -> uint32_t {           // over the block's new rows, as bf16 bits
    uint32_t m = 0;
#pragma unroll
    for (int p = 0; p < kPasses; ++p)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        m = __vmaxu2(m, magnitude(x[p][h].x));
        m = __vmaxu2(m, magnitude(x[p][h].y));
        m = __vmaxu2(m, magnitude(x[p][h].z));
        m = __vmaxu2(m, magnitude(x[p][h].w));
      }
    return __reduce_max_sync(0xffffffffu, max(m & 0xffffu, m >> 16));
  };
  uint32_t top = largest([](uint32_t v) { return v & 0x7fff7fffu; });
  if (top >= 0x7f80u) top = largest([](uint32_t v) { return finite_abs_bf16x2(v); });   // infinities or NaN: leave them out
  float s = e4m3_block_scale(__uint_as_float(top << 16));
  if (n_old > 0) {
    const float was = *scale;
    if (was >= s) {
      s = was;
    } else {                                                 // the earlier rows move to the larger scale
      const float factor = was / s;
#pragma unroll
      for (int p = 0; p < kPasses; ++p) {
        const int r = p * kRowsPerPass + lr;
        if (r < n_old) {
          uint4* at = reinterpret_cast<uint4*>(codes + r * D) + lc;
          uint4 c = *at;
          c.x = e4m3x4_shift(c.x, factor);
          c.y = e4m3x4_shift(c.y, factor);
          c.z = e4m3x4_shift(c.z, factor);
          c.w = e4m3x4_shift(c.w, factor);
          *at = c;
        }
      }
    }
  }
  __syncwarp();                                              // every lane has read the scale before lane 0 replaces it
  const float inv = 1.0f / s;
#pragma unroll
  for (int p = 0; p < kPasses; ++p) {
    const int r = p * kRowsPerPass + lr;
    if (r >= n_old && r < n_old + n_new)
      *(reinterpret_cast<uint4*>(codes + r * D) + lc) = e4m3x16_from_bf16(x[p][0], x[p][1], inv);
  }
  if (lane == 0) *scale = s;
}

}  // namespace xkv
