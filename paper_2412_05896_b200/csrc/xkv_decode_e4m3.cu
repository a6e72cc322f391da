// Decode attention over caches of 8-bit floats with one scale per block of 16 slots and KV head (Eq. 1).
//
// One CTA per (layer, sequence, KV head); a warp takes every fourth cached row, its lanes share the row's columns, and
// the four warps' softmax states are joined at the end.  All arithmetic in fp32.
#include <cmath>

#include "common.cuh"
#include "e4m3.cuh"
#include "ops.h"

namespace xkv {
namespace {

constexpr int kMaxGroup = 8;
constexpr int kWarps = 4;

struct Params {
  const __nv_bfloat16* q;
  __nv_bfloat16* out;
  float* lse;
  const uint8_t* k_pages;
  const uint8_t* v_pages;
  const float* k_scales;
  const float* v_scales;
  const int32_t* block_table;
  const int32_t* seq_lens;
  int32_t layer_begin, batch, n_q_heads, n_kv_heads, group, page_size, max_pages_per_seq, n_pages;
  float scale_log2;
};

template <int D>
__global__ void __launch_bounds__(32 * kWarps) decode_rows_kernel(const Params p) {
  constexpr int kCols = D / 32;
  __shared__ float s_o[kWarps][kMaxGroup][D];
  __shared__ float s_ml[kWarps][kMaxGroup][2];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int e = blockIdx.x / p.n_kv_heads, h = blockIdx.x % p.n_kv_heads;
  const size_t le = (size_t)p.layer_begin * p.batch + e;
  const int n = min(max(p.seq_lens[le], 0), p.max_pages_per_seq * p.page_size);
  const size_t row0 = (size_t)e * p.n_q_heads + (size_t)h * p.group;
  float q[kMaxGroup][kCols], o[kMaxGroup][kCols], m[kMaxGroup], l[kMaxGroup], lost[kMaxGroup];
#pragma unroll
  for (int g = 0; g < kMaxGroup; ++g) {
    m[g] = -INFINITY;
    l[g] = 0.f;
    lost[g] = 0.f;                              // what the running sum l has rounded off (thousands of rows per warp)
#pragma unroll
    for (int j = 0; j < kCols; ++j) {
      o[g][j] = 0.f;
      q[g][j] = g < p.group ? __bfloat162float(p.q[(row0 + g) * D + lane * kCols + j]) * p.scale_log2 : 0.f;
    }
  }
  for (int r = warp; r < n; r += kWarps) {
    int page = p.block_table[le * p.max_pages_per_seq + r / p.page_size];
    page = min(max(page, 0), p.n_pages - 1);
    const size_t row = ((size_t)page * p.n_kv_heads + h) * p.page_size + r % p.page_size;
    const float ks = p.k_scales[row / kScaleBlock], vs = p.v_scales[row / kScaleBlock];
    float k[kCols], v[kCols];
#pragma unroll
    for (int j = 0; j < kCols; j += 2) {
      const float2 a = f32_from_e4m3x2(*reinterpret_cast<const uint16_t*>(p.k_pages + row * D + lane * kCols + j));
      const float2 b = f32_from_e4m3x2(*reinterpret_cast<const uint16_t*>(p.v_pages + row * D + lane * kCols + j));
      k[j] = a.x; k[j + 1] = a.y;
      v[j] = b.x; v[j + 1] = b.y;
    }
#pragma unroll
    for (int g = 0; g < kMaxGroup; ++g) {
      if (g >= p.group) break;
      float s = 0.f;
#pragma unroll
      for (int j = 0; j < kCols; ++j) s += q[g][j] * k[j];
#pragma unroll
      for (int x = 16; x > 0; x >>= 1) s += __shfl_xor_sync(0xffffffffu, s, x);
      s *= ks;
      const float mn = fmaxf(m[g], s);
      const float al = m[g] == mn ? 1.f : exp2f(m[g] - mn), w = exp2f(s - mn);
      m[g] = mn;
      l[g] *= al;
      const float y = w - lost[g] * al, t = l[g] + y;
      lost[g] = (t - l[g]) - y;
      l[g] = t;
#pragma unroll
      for (int j = 0; j < kCols; ++j) o[g][j] = o[g][j] * al + w * vs * v[j];
    }
  }
#pragma unroll
  for (int g = 0; g < kMaxGroup; ++g) {
    if (g >= p.group) break;
#pragma unroll
    for (int j = 0; j < kCols; ++j) s_o[warp][g][lane * kCols + j] = o[g][j];
    if (lane == 0) {
      s_ml[warp][g][0] = m[g];
      s_ml[warp][g][1] = l[g];
    }
  }
  __syncthreads();
  for (int i = threadIdx.x; i < p.group * D; i += 32 * kWarps) {
    const int g = i / D, c = i % D;
    float mx = -INFINITY;
    for (int w = 0; w < kWarps; ++w) mx = fmaxf(mx, s_ml[w][g][0]);
    float den = 0.f, acc = 0.f;
    for (int w = 0; w < kWarps; ++w) {
      if (s_ml[w][g][1] == 0.f) continue;                    // this warp saw no row
      const float f = exp2f(s_ml[w][g][0] - mx);
      den += f * s_ml[w][g][1];
      acc += f * s_o[w][g][c];
    }
    p.out[(row0 + g) * D + c] = __float2bfloat16(n > 0 ? acc / den : 0.f);
    if (c == 0 && p.lse != nullptr) p.lse[row0 + g] = n > 0 ? (mx + log2f(den)) * 0.6931471805599453f : -INFINITY;
  }
}

}  // namespace

xkv_status decode_attn_e4m3(const xkv_dims* d, const xkv_cache* c, int layer_begin, int n_layers, const void* q,
                            const void* k_new, const void* v_new, void* out, float* lse, int chunk_rows,
                            const DecodeScratch& ws, cudaStream_t st) {
  (void)chunk_rows;
  const int n_units = n_layers * d->batch;
  if (k_new != nullptr) {
    const xkv_status s = append_e4m3(d, c, layer_begin, n_units, k_new, v_new, ws.header, st);
    if (s != XKV_OK) return s;
  }
  Params p;
  p.q = static_cast<const __nv_bfloat16*>(q);
  p.out = static_cast<__nv_bfloat16*>(out);
  p.lse = lse;
  p.k_pages = static_cast<const uint8_t*>(c->k_pages);
  p.v_pages = static_cast<const uint8_t*>(c->v_pages);
  p.k_scales = c->k_scales;
  p.v_scales = c->v_scales;
  p.block_table = c->block_table;
  p.seq_lens = c->seq_lens;
  p.layer_begin = layer_begin;
  p.batch = d->batch;
  p.n_q_heads = d->n_q_heads;
  p.n_kv_heads = d->n_kv_heads;
  p.group = d->n_q_heads / d->n_kv_heads;
  p.page_size = c->page_size;
  p.max_pages_per_seq = c->max_pages_per_seq;
  p.n_pages = c->n_pages;
  p.scale_log2 = (d->scale != 0.f ? d->scale : 1.0f / sqrtf((float)d->head_dim)) * 1.4426950408889634f;
  const int grid = n_units * d->n_kv_heads;
  if (d->head_dim == 128) decode_rows_kernel<128><<<grid, 32 * kWarps, 0, st>>>(p);
  else                    decode_rows_kernel<64><<<grid, 32 * kWarps, 0, st>>>(p);
  count_launch();
  return check_launch();
}

}  // namespace xkv
