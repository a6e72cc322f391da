// Differential attention of single tokens where there is little to read: few caches that their tables bound to few rows.
//
// Mathematics: that of xkv_diff_decode_attn.  With a head's query row [q1 | q2], cache rows [k1 | k2] and v,
//   z_s[c] = scale q_s . k_s[c],  p_s = exp(z_s - max z_s),  o_s = sum_c p_s[c] v[c]          s = 1, 2
// per chunk of rows, joined over the chunks of a cache by their maxima and sums; then the difference of the two maps and its norm.
//
// The streaming kernel is made for caches that keep every SM busy for many tiles; here a call is a chain of latencies, so everything
// is laid out for few of them: one launch that needs nothing cleared before it, one CTA per chunk of a KV head's cache, and all
// of a chunk's K and V bytes asked for at once as soon as its page ids are known (a thread keeps its share of both in registers), on
// CUDA cores.  The last CTA of a cache to finish joins the chunks (in their order, so the result does not depend on who that is)
// and sets the cache's ticket back to zero.
// Measured (device time): four layers x four heads of 64, 49 to 146 rows: SMALL_TIME (streaming kernel 18.5 us).
#include <algorithm>

#include "common.cuh"
#include "ops.h"

namespace xkv {
namespace {

constexpr int kThreads = 256;
constexpr int kWarps = kThreads / 32;
constexpr int kChunk = 128;           // rows of a CTA
constexpr int kMaxCtas = 2 * 148;     // one wave: two CTAs an SM
constexpr int kTickets = sizeof(WorkspaceHeader::few_tickets) / 4;

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
  int32_t layer_begin, batch, n_q_heads, n_kv_heads, group, page_size, max_pages_per_seq, n_pages, max_chunks;
  float scale_log2, eps;
  const float* lambda;
  const float* gain;
  int32_t* tickets;                   // [units * n_kv_heads], zero between calls; not used where max_chunks is 1
  float* part_o;                      // [CTAs][2 G][D]
  float2* part_ml;                    // [CTAs][2 G] largest logit (log2), sum
};

// Eight consecutive elements of a cached row.
template <bool Q8>
struct Piece;
template <>
struct Piece<false> {
  uint4 raw;
  __device__ __forceinline__ void load(const uint8_t* pages, size_t element) {
    raw = __ldg(reinterpret_cast<const uint4*>(pages + element * 2));
  }
  __device__ __forceinline__ void values(float (&x)[8]) const { bf16x8_to_f32(raw, x); }
};
template <>
struct Piece<true> {
  uint2 raw;
  __device__ __forceinline__ void load(const uint8_t* pages, size_t element) {
    raw = __ldg(reinterpret_cast<const uint2*>(pages + element));
  }
  __device__ __forceinline__ void values(float (&x)[8]) const {
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = (float)(int)(((i < 4 ? raw.x : raw.y) >> (8 * (i & 3))) & 0xffu) - 128.f;
  }
};

template <int D, bool Q8, int GP>     // GP: heads per KV head, rounded up to a power of two
__global__ void __launch_bounds__(kThreads) diff_decode_few_kernel(const Params p) {
  constexpr int kLanes = D / 8;                      // lanes of a row, eight elements each
  constexpr int kRowsAtOnce = kThreads / kLanes;     // rows that the CTA holds a piece of at a time
  constexpr int kPer = kChunk / kRowsAtOnce;         // pieces of K, and of V, a thread
  __shared__ float s_z[kChunk][2 * GP];              // logits (log2), then weights; of V: times the row's scale
  __shared__ float s_o[2 * GP][D];
  __shared__ float s_m[2 * GP], s_l[2 * GP];
  __shared__ float s_w[2 * GP][32];                  // a batch of chunks' weights
  __shared__ int s_last;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, G = p.group;
  const int chunk = blockIdx.x % p.max_chunks, unit_head = blockIdx.x / p.max_chunks;
  const int h = unit_head % p.n_kv_heads, e = unit_head / p.n_kv_heads;
  const size_t le = (size_t)p.layer_begin * p.batch + e;
  const int n = min(max(__ldg(&p.seq_lens[le]), 0), p.max_pages_per_seq * p.page_size);
  const int n_chunks = max((n + kChunk - 1) / kChunk, 1);
  if (chunk >= n_chunks) return;
  const int row0 = chunk * kChunk, rows = min(kChunk, n - row0);
  const int c = tid % kLanes, r0 = tid / kLanes;     // this thread's columns 8 c .. 8 c + 7 of rows r0, r0 + kRowsAtOnce, ..
  const size_t q_row = (size_t)e * p.n_q_heads + (size_t)h * G;
  float q[GP][8];
#pragma unroll
  for (int g = 0; g < GP; ++g)
    if (g < G) bf16x8_to_f32(__ldg(reinterpret_cast<const uint4*>(p.q + (q_row + g) * D + c * 8)), q[g]);
  // ---- all of the chunk at once: page ids, then rows and scales
  const int32_t* table = p.block_table + le * p.max_pages_per_seq;
  int page[kPer];
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    const int r = row0 + r0 + i * kRowsAtOnce;
    page[i] = r < n ? __ldg(&table[r / p.page_size]) : -1;
  }
  Piece<Q8> k[kPer], v[kPer];
  float ks[kPer], vs[kPer];
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    const int r = row0 + r0 + i * kRowsAtOnce;
    const size_t row = ((size_t)min(max(page[i], 0), p.n_pages - 1) * p.n_kv_heads + h) * p.page_size + r % p.page_size;
    ks[i] = vs[i] = 1.f;
    k[i].raw = {};
    v[i].raw = {};
    if (page[i] < 0 && r >= n) continue;             // (rows behind the last one: zero)
    k[i].load(p.k_pages, row * D + c * 8);
    v[i].load(p.v_pages, row * D + c * 8);
    if constexpr (Q8) {
      ks[i] = __ldg(&p.k_scales[row]);
      vs[i] = __ldg(&p.v_scales[row]);
    }
  }
  // ---- logits: the lanes of a row's first half have map 1, those of its second half map 2
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    const int r = r0 + i * kRowsAtOnce;
    float x[8];
    k[i].values(x);
#pragma unroll
    for (int g = 0; g < GP; ++g) {
      float z = 0.f;
      if (g < G) {
#pragma unroll
        for (int y = 0; y < 8; ++y) z = fmaf(q[g][y], x[y], z);
      }
#pragma unroll
      for (int o = 1; o < kLanes / 2; o <<= 1) z += __shfl_xor_sync(0xffffffffu, z, o);
      if (c % (kLanes / 2) == 0) s_z[r][2 * g + c / (kLanes / 2)] = r < rows ? z * ks[i] * p.scale_log2 : -INFINITY;
    }
  }
  __syncthreads();
  // ---- weights: a warp a map of a head
  for (int m = warp; m < 2 * GP; m += kWarps) {
    float z[kChunk / 32], top = -INFINITY, sum = 0.f;
#pragma unroll
    for (int i = 0; i < kChunk / 32; ++i) {
      z[i] = s_z[32 * i + lane][m];
      top = fmaxf(top, z[i]);
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
    const float ref = top == -INFINITY ? 0.f : top;
#pragma unroll
    for (int i = 0; i < kChunk / 32; ++i) {
      z[i] = fast_exp2(z[i] - ref);
      sum += z[i];
      s_z[32 * i + lane][m] = z[i];
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    if (lane == 0) {
      s_m[m] = top;
      s_l[m] = sum;
    }
  }
  for (int i = tid; i < 2 * GP * D; i += kThreads) (&s_o[0][0])[i] = 0.f;
  __syncthreads();
  // ---- products with V: a thread its columns of its rows, then over the rows of a warp, then over the warps
  {
    float o[2 * GP][8];
#pragma unroll
    for (int m = 0; m < 2 * GP; ++m)
#pragma unroll
      for (int y = 0; y < 8; ++y) o[m][y] = 0.f;
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      const int r = r0 + i * kRowsAtOnce;
      if (r >= rows) continue;                       // (0 * what lies behind the last row)
      float x[8];
      v[i].values(x);
#pragma unroll
      for (int m = 0; m < 2 * GP; ++m) {
        const float w = s_z[r][m] * vs[i];
#pragma unroll
        for (int y = 0; y < 8; ++y) o[m][y] = fmaf(w, x[y], o[m][y]);
      }
    }
#pragma unroll
    for (int m = 0; m < 2 * GP; ++m)
#pragma unroll
      for (int y = 0; y < 8; ++y)
#pragma unroll
        for (int s = kLanes; s < 32; s <<= 1) o[m][y] += __shfl_xor_sync(0xffffffffu, o[m][y], s);
    // one warp after the other, so that the sum's order is fixed
    for (int w = 0; w < kWarps; ++w) {
      if (warp == w && lane < kLanes) {
#pragma unroll
        for (int m = 0; m < 2 * GP; ++m)
#pragma unroll
          for (int y = 0; y < 8; ++y) s_o[m][c * 8 + y] += o[m][y];
      }
      __syncthreads();
    }
  }
  // ---- a cache of several chunks: the last CTA joins them
  if (n_chunks > 1) {
    for (int i = tid; i < 2 * G * D; i += kThreads) __stcg(&p.part_o[(size_t)blockIdx.x * 2 * G * D + i], (&s_o[0][0])[i]);
    if (tid < 2 * G) __stcg(&p.part_ml[(size_t)blockIdx.x * 2 * G + tid], make_float2(s_m[tid], s_l[tid]));
    __threadfence();
    __syncthreads();
    if (tid == 0) {
      const int was = atomicAdd(&p.tickets[unit_head], 1);
      s_last = was == n_chunks - 1;
      if (s_last) p.tickets[unit_head] = 0;
    }
    __syncthreads();
    if (!s_last) return;
    __threadfence();
    const size_t first = (size_t)unit_head * p.max_chunks;
    for (int m = warp; m < 2 * G; m += kWarps) {     // maxima and sums over all chunks
      float top = -INFINITY;
      for (int i = lane; i < n_chunks; i += 32) top = fmaxf(top, __ldcg(&p.part_ml[(first + i) * 2 * G + m]).x);
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
      float sum = 0.f;
      for (int i = lane; i < n_chunks; i += 32) {
        const float2 ml = __ldcg(&p.part_ml[(first + i) * 2 * G + m]);
        sum = fmaf(fast_exp2(ml.x - top), ml.y, sum);
      }
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
      if (lane == 0) {
        s_m[m] = top;
        s_l[m] = sum;
      }
    }
    constexpr int kMine = (2 * GP * D + kThreads - 1) / kThreads;
    float o[kMine];
#pragma unroll
    for (int x = 0; x < kMine; ++x) o[x] = 0.f;
    for (int c0 = 0; c0 < n_chunks; c0 += 32) {
      __syncthreads();
      const int nb = min(32, n_chunks - c0);
      for (int i = tid; i < 2 * G * 32; i += kThreads)
        if (i % 32 < nb) s_w[i / 32][i % 32] = fast_exp2(__ldcg(&p.part_ml[(first + c0 + i % 32) * 2 * G + i / 32]).x - s_m[i / 32]);
      __syncthreads();
#pragma unroll
      for (int x = 0; x < kMine; ++x) {
        const int i = x * kThreads + tid;
        if (i >= 2 * G * D) continue;
#pragma unroll 8
        for (int y = 0; y < nb; ++y) o[x] = fmaf(s_w[i / D][y], __ldcg(&p.part_o[(first + c0 + y) * 2 * G * D + i]), o[x]);
      }
    }
    __syncthreads();
#pragma unroll
    for (int x = 0; x < kMine; ++x)
      if (x * kThreads + tid < 2 * G * D) (&s_o[0][0])[x * kThreads + tid] = o[x];
    __syncthreads();
  }
  // ---- the difference and its norm: a warp a head
  for (int g = warp; g < G; g += kWarps) {
    const int layer = e / p.batch;
    const float l1 = s_l[2 * g], l2 = s_l[2 * g + 1];
    const float w1 = l1 > 0.f ? 1.f / l1 : 0.f;
    const float w2 = l2 > 0.f ? -__ldg(&p.lambda[(size_t)layer * p.n_q_heads + h * G + g]) / l2 : 0.f;
    float y[D / 32], sq = 0.f;
#pragma unroll
    for (int i = 0; i < D / 32; ++i) {
      y[i] = fmaf(s_o[2 * g + 1][lane * (D / 32) + i], w2, s_o[2 * g][lane * (D / 32) + i] * w1);
      sq = fmaf(y[i], y[i], sq);
    }
    if (p.gain != nullptr) {
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) sq += __shfl_xor_sync(0xffffffffu, sq, o);
      const float r = diff_norm<D>(sq, p.eps);
#pragma unroll
      for (int i = 0; i < D / 32; ++i) y[i] *= r * __ldg(&p.gain[(size_t)layer * D + lane * (D / 32) + i]);
    }
#pragma unroll
    for (int i = 0; i < D / 32; i += 2)
      *reinterpret_cast<uint32_t*>(p.out + (q_row + g) * D + lane * (D / 32) + i) = pack_bf16(y[i], y[i + 1]);
    if (lane < 2 && p.lse != nullptr) {
      const float l = lane == 0 ? l1 : l2;
      p.lse[2 * (q_row + g) + lane] = l > 0.f ? (s_m[2 * g + lane] + log2f(l)) * 0.6931471805599453f : -INFINITY;
    }
  }
}

template <int D, bool Q8>
xkv_status launch(const Params& p, int ctas, cudaStream_t st) {
  if (p.group == 1)      diff_decode_few_kernel<D, Q8, 1><<<ctas, kThreads, 0, st>>>(p);
  else if (p.group == 2) diff_decode_few_kernel<D, Q8, 2><<<ctas, kThreads, 0, st>>>(p);
  else if (p.group <= 4) diff_decode_few_kernel<D, Q8, 4><<<ctas, kThreads, 0, st>>>(p);
  else                   diff_decode_few_kernel<D, Q8, 8><<<ctas, kThreads, 0, st>>>(p);
  count_launch();
  return check_launch();
}

int64_t few_ctas(const xkv_dims* d, int n_layers, int max_cache_len) {
  return (int64_t)n_layers * d->batch * d->n_kv_heads * std::max(1, (max_cache_len + kChunk - 1) / kChunk);
}

}  // namespace

bool diff_decode_is_few(const xkv_dims* d, int n_layers, int max_cache_len, int64_t max_rows) {
  const int64_t ctas = few_ctas(d, n_layers, max_cache_len);
  if (ctas > kMaxCtas) return false;
  return max_cache_len <= kChunk ||
         ((int64_t)n_layers * d->batch * d->n_kv_heads <= kTickets && ctas * 2 * (d->n_q_heads / d->n_kv_heads) <= max_rows);
}

xkv_status diff_decode_few(const xkv_dims* d, const xkv_cache* c, int layer_begin, int n_layers, const void* q, void* out,
                           float* lse, const DiffHeads& diff, const DecodeScratch& ws, cudaStream_t st) {
  const int max_cache_len = c->max_pages_per_seq * c->page_size;
  const int64_t ctas = few_ctas(d, n_layers, max_cache_len);
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
  p.max_chunks = std::max(1, (max_cache_len + kChunk - 1) / kChunk);
  p.scale_log2 = (d->scale != 0.f ? d->scale : 1.0f / sqrtf((float)(d->head_dim / 2))) * 1.4426950408889634f;
  p.eps = diff.eps;
  p.lambda = diff.lambda;
  p.gain = diff.gain;
  p.tickets = static_cast<WorkspaceHeader*>(ws.header)->few_tickets;
  p.part_o = ws.part_o;
  p.part_ml = reinterpret_cast<float2*>(ws.part_ml);
  const bool q8 = c->kv_format == XKV_KV_INT8;
  if (d->head_dim == 128) return q8 ? launch<128, true>(p, (int)ctas, st) : launch<128, false>(p, (int)ctas, st);
  return q8 ? launch<64, true>(p, (int)ctas, st) : launch<64, false>(p, (int)ctas, st);
}

}  // namespace xkv
