// Differential attention of single tokens where there is little to read: few caches that their tables bound to few rows.
//
// Mathematics: that of xkv_diff_decode_attn.  With a head's query row [q1 | q2], cache rows [k1 | k2] and v,
//   z_s[c] = scale q_s . k_s[c],  p_s = exp(z_s - max z_s),  o_s = sum_c p_s[c] v[c]          s = 1, 2
// per chunk of rows, joined over the chunks of a cache by their maxima and sums; then the difference of the two maps and its norm.
//
// The streaming kernel is made for caches that keep every SM busy for many tiles; here a call is a chain of latencies, so everything
// is laid out for few of them: one launch that needs nothing cleared before it, one CTA per chunk of a streamed cache, and all of a
// chunk's K and V bytes asked for at once as soon as its page ids are known.  A warp has 16 rows in registers and multiplies them with
// mma.sync m16n8k16, rows on M and the (at most eight) query rows on N.  A lane's 16 bytes of a row are eight consecutive columns, so
// no fragment goes through shared memory: of the logits the columns' order does not matter as long as the query has the same, and
// of the outputs it only says where a value is stored (V's fragments are transposed in registers, 8 x 8 at a time).  The last CTA
// of a cache to finish joins the chunks (in their order, so the result does not depend on who that is) and sets the ticket back to
// zero.
#include <algorithm>

#include "common.cuh"
#include "ops.h"

namespace xkv {
namespace {

constexpr int kThreads = 256;
constexpr int kWarps = kThreads / 32;
constexpr int kChunk = 16 * kWarps;   // rows of a CTA
constexpr int kRows = 8;              // query rows at most: the N of the products
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
  int32_t layer_begin, batch, n_q_heads, n_kv_heads, n_heads, page_size, max_pages_per_seq, n_pages, max_chunks;
  float scale_log2;
  DiffHeads diff;
  int32_t* tickets;                   // [units * n_heads], zero between calls; not used where max_chunks is 1
  float* part_o;                      // [CTAs][kRows][D]
  float2* part_ml;                    // [CTAs][kRows] largest logit (log2), sum
};

__device__ __forceinline__ void mma_f16(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
template <bool Q8>
__device__ __forceinline__ void mma(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  if constexpr (Q8) mma_f16(c, a, b0, b1);
  else              mma_bf16_16816(c, a, b0, b1);
}
template <bool Q8>
__device__ __forceinline__ uint32_t pack16(float lo, float hi) {
  if constexpr (!Q8) return pack_bf16(lo, hi);
  uint32_t r;
  asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}
// Eight consecutive elements of a cached row as four pairs: bf16 as they lie, 8-bit integers as fp16.
template <bool Q8>
__device__ __forceinline__ void load_piece(uint32_t (&x)[4], const uint8_t* pages, size_t element) {
  if constexpr (Q8) {
    const uint2 r = __ldg(reinterpret_cast<const uint2*>(pages + element));
    x[0] = r.x, x[1] = r.y;           // (expanded where it is used, so that the load does not have to be waited for here)
  } else {
    const uint4 r = __ldg(reinterpret_cast<const uint4*>(pages + element * 2));
    x[0] = r.x, x[1] = r.y, x[2] = r.z, x[3] = r.w;
  }
}
template <bool Q8>
__device__ __forceinline__ void expand(uint32_t (&x)[4]) {
  if constexpr (Q8) {
    const uint32_t lo = x[0], hi = x[1];
    x[0] = int8x2_to_f16x2<0x5140>(lo);
    x[1] = int8x2_to_f16x2<0x5342>(lo);
    x[2] = int8x2_to_f16x2<0x5140>(hi);
    x[3] = int8x2_to_f16x2<0x5342>(hi);
  }
}

template <int D, bool Q8>
__global__ void __launch_bounds__(kThreads, 2) diff_decode_few_kernel(const Params p) {
  constexpr int kPieces = D / 32;                    // pieces of eight columns that a lane has of a row
  __shared__ float s_o[kWarps][kRows][D];            // the warps' outputs, then in [0] the CTA's
  __shared__ float s_m[kWarps][kRows], s_l[kWarps][kRows];
  __shared__ float s_top[kRows], s_sum[kRows];
  __shared__ float s_w[kRows][32];                   // a batch of chunks' weights
  __shared__ int s_last;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, gid = lane >> 2, tig = lane & 3;
  const int chunk = blockIdx.x % p.max_chunks, unit_head = blockIdx.x / p.max_chunks;
  const int h = unit_head % p.n_heads, e = unit_head / p.n_heads, kvh = h / p.diff.subs;
  const size_t le = (size_t)p.layer_begin * p.batch + e;
  const int n = min(max(__ldg(&p.seq_lens[le]), 0), p.max_pages_per_seq * p.page_size);
  const int n_chunks = max((n + kChunk - 1) / kChunk, 1);
  if (chunk >= n_chunks) return;
  const int n_rows = 2 * p.diff.heads(h);            // row 2 j + s is map s of head j
  const size_t head0 = (size_t)e * p.n_q_heads + p.diff.first_head(h);
  // ---- page ids of this warp's 16 rows, then everything at once: rows gid and gid + 8, columns 8 (tig + 4 j) .. + 7
  const int row0 = chunk * kChunk + 16 * warp, rows = min(16, n - row0);
  uint32_t k[2][kPieces][4], v[2][kPieces][4];
  float ks[2] = {1.f, 1.f}, vs[2] = {1.f, 1.f};
  if (rows > 0) {
    // (page_size is a multiple of 16: the 16 rows share a page)
    const int page = min(max(__ldg(&p.block_table[le * p.max_pages_per_seq + row0 / p.page_size]), 0), p.n_pages - 1);
    const size_t first = ((size_t)page * p.n_kv_heads + kvh) * p.page_size + row0 % p.page_size;
#pragma unroll
    for (int y = 0; y < 2; ++y) {
      const size_t row = first + gid + 8 * y;
#pragma unroll
      for (int j = 0; j < kPieces; ++j) load_piece<Q8>(k[y][j], p.k_pages, row * D + 8 * (tig + 4 * j));
#pragma unroll
      for (int j = 0; j < kPieces; ++j) load_piece<Q8>(v[y][j], p.v_pages, row * D + 8 * (tig + 4 * j));
      if constexpr (Q8) {
        ks[y] = __ldg(&p.k_scales[row]);
        vs[y] = __ldg(&p.v_scales[row]);
      }
    }
  }
  // ---- the query row of this lane: the half that is not its map's is zero
  uint32_t q[kPieces][4];
#pragma unroll
  for (int j = 0; j < kPieces; ++j) {
    uint4 r = make_uint4(0u, 0u, 0u, 0u);
    if (gid < n_rows && (j >= kPieces / 2) == ((gid & 1) != 0))
      r = __ldg(reinterpret_cast<const uint4*>(p.q + (head0 + (gid >> 1)) * D + 8 * (tig + 4 * j)));
    q[j][0] = r.x, q[j][1] = r.y, q[j][2] = r.z, q[j][3] = r.w;
    if constexpr (Q8) {
#pragma unroll
      for (int i = 0; i < 4; ++i) q[j][i] = pack16<true>(bf16_lo(q[j][i]), bf16_hi(q[j][i]));
    }
  }
  float m[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f};     // of query rows 2 tig and 2 tig + 1
  float o[D / 16][4];
#pragma unroll
  for (int x = 0; x < D / 16; ++x) o[x][0] = o[x][1] = o[x][2] = o[x][3] = 0.f;
  if (rows > 0) {
    float z[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int j = 0; j < kPieces; ++j) {
      expand<Q8>(k[0][j]);
      expand<Q8>(k[1][j]);
      const uint32_t a0[4] = {k[0][j][0], k[1][j][0], k[0][j][1], k[1][j][1]};
      const uint32_t a1[4] = {k[0][j][2], k[1][j][2], k[0][j][3], k[1][j][3]};
      mma<Q8>(z, a0, q[j][0], q[j][1]);
      mma<Q8>(z, a1, q[j][2], q[j][3]);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) z[i] = gid + 8 * (i >> 1) < rows ? z[i] * ks[i >> 1] * p.scale_log2 : -INFINITY;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      m[i] = fmaxf(z[i], z[i + 2]);
#pragma unroll
      for (int x = 4; x < 32; x <<= 1) m[i] = fmaxf(m[i], __shfl_xor_sync(0xffffffffu, m[i], x));
    }
    float w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = fast_exp2(z[i] - (m[i & 1] == -INFINITY ? 0.f : m[i & 1]));
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      l[i] = w[i] + w[i + 2];
#pragma unroll
      for (int x = 4; x < 32; x <<= 1) l[i] += __shfl_xor_sync(0xffffffffu, l[i], x);
    }
    // the weights as the B operand (rounded to 16 bits, 8-bit rows: times the row's scale); rows behind the last one: no weight
    // and no value, whatever lies there
#pragma unroll
    for (int y = 0; y < 2; ++y)
      if (gid + 8 * y >= rows) {
        vs[y] = 0.f;
#pragma unroll
        for (int j = 0; j < kPieces; ++j) v[y][j][0] = v[y][j][1] = v[y][j][2] = v[y][j][3] = Q8 ? 0x80808080u : 0u;
      }
    const uint32_t b0 = movmatrix_trans(pack16<Q8>(Q8 ? w[0] * vs[0] : w[0], Q8 ? w[1] * vs[0] : w[1]));
    const uint32_t b1 = movmatrix_trans(pack16<Q8>(Q8 ? w[2] * vs[1] : w[2], Q8 ? w[3] * vs[1] : w[3]));
#pragma unroll
    for (int j = 0; j < kPieces; ++j) {
      expand<Q8>(v[0][j]);
      expand<Q8>(v[1][j]);
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const uint32_t a[4] = {movmatrix_trans(v[0][j][2 * i]), movmatrix_trans(v[0][j][2 * i + 1]),
                               movmatrix_trans(v[1][j][2 * i]), movmatrix_trans(v[1][j][2 * i + 1])};
        mma<Q8>(o[2 * j + i], a, b0, b1);
      }
    }
  }
  // accumulator row gid (+ 8) of block (j, i) is column 8 (gid / 2 + 4 j) + 4 i + gid % 2 (+ 2)
#pragma unroll
  for (int x = 0; x < D / 16; ++x)
#pragma unroll
    for (int i = 0; i < 4; ++i)
      s_o[warp][2 * tig + (i & 1)][8 * ((gid >> 1) + 4 * (x >> 1)) + 4 * (x & 1) + 2 * (i >> 1) + (gid & 1)] = o[x][i];
  if (gid == 0) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      s_m[warp][2 * tig + i] = m[i];
      s_l[warp][2 * tig + i] = l[i];
    }
  }
  __syncthreads();
  // ---- the warps' results joined
  if (tid < kRows) {
    float top = -INFINITY, sum = 0.f;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) top = fmaxf(top, s_m[w][tid]);
#pragma unroll
    for (int w = 0; w < kWarps; ++w) {
      const float x = s_m[w][tid] == -INFINITY ? 0.f : fast_exp2(s_m[w][tid] - top);
      sum = fmaf(x, s_l[w][tid], sum);
      s_m[w][tid] = x;
    }
    s_top[tid] = top;
    s_sum[tid] = sum;
  }
  __syncthreads();
  constexpr int kMine = kRows * D / kThreads;
#pragma unroll
  for (int x = 0; x < kMine; ++x) {
    const int i = x * kThreads + tid, r = i / D, col = i % D;
    float sum = 0.f;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) sum = fmaf(s_m[w][r], s_o[w][r][col], sum);
    s_o[0][r][col] = sum;             // (no other thread reads this column of any warp)
  }
  __syncthreads();
  // ---- a cache of several chunks: the last CTA joins them
  if (n_chunks > 1) {
    float* part = p.part_o + (size_t)blockIdx.x * kRows * D;
#pragma unroll
    for (int x = 0; x < kMine; ++x) __stcg(&part[x * kThreads + tid], (&s_o[0][0][0])[x * kThreads + tid]);
    if (tid < kRows) __stcg(&p.part_ml[(size_t)blockIdx.x * kRows + tid], make_float2(s_top[tid], s_sum[tid]));
    __threadfence();
    __syncthreads();
    if (tid == 0) {
      s_last = atomicAdd(&p.tickets[unit_head], 1) == n_chunks - 1;
      if (s_last) p.tickets[unit_head] = 0;
    }
    __syncthreads();
    if (!s_last) return;
    __threadfence();
    const size_t first = (size_t)unit_head * p.max_chunks;
    {                                                // a warp a query row: maximum and sum over all chunks
      float top = -INFINITY, sum = 0.f;
      for (int i = lane; i < n_chunks; i += 32) top = fmaxf(top, __ldcg(&p.part_ml[(first + i) * kRows + warp]).x);
#pragma unroll
      for (int x = 16; x > 0; x >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, x));
      for (int i = lane; i < n_chunks; i += 32) {
        const float2 ml = __ldcg(&p.part_ml[(first + i) * kRows + warp]);
        sum = fmaf(fast_exp2(ml.x - top), ml.y, sum);
      }
#pragma unroll
      for (int x = 16; x > 0; x >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, x);
      if (lane == 0) {
        s_top[warp] = top;
        s_sum[warp] = sum;
      }
    }
    static_assert(kWarps == kRows, "a warp a query row");
    float acc[kMine];
#pragma unroll
    for (int x = 0; x < kMine; ++x) acc[x] = 0.f;
    for (int c0 = 0; c0 < n_chunks; c0 += 32) {
      const int nb = min(32, n_chunks - c0);
      __syncthreads();
      if (lane < nb) s_w[warp][lane] = fast_exp2(__ldcg(&p.part_ml[(first + c0 + lane) * kRows + warp]).x - s_top[warp]);
      __syncthreads();
#pragma unroll
      for (int x = 0; x < kMine; ++x) {
        const int i = x * kThreads + tid;
#pragma unroll 8
        for (int y = 0; y < nb; ++y)
          acc[x] = fmaf(s_w[i / D][y], __ldcg(&p.part_o[(first + c0 + y) * kRows * D + i]), acc[x]);
      }
    }
#pragma unroll
    for (int x = 0; x < kMine; ++x) (&s_o[0][0][0])[x * kThreads + tid] = acc[x];
    __syncthreads();
  }
  // ---- the difference and its norm: a warp a head
  for (int g = warp; 2 * g < n_rows; g += kWarps) {
    const int layer = e / p.batch;
    const float l1 = s_sum[2 * g], l2 = s_sum[2 * g + 1];
    const float w1 = l1 > 0.f ? 1.f / l1 : 0.f;
    const float w2 = l2 > 0.f ? -__ldg(&p.diff.lambda[(size_t)layer * p.n_q_heads + p.diff.first_head(h) + g]) / l2 : 0.f;
    float y[D / 32], sq = 0.f;
#pragma unroll
    for (int i = 0; i < D / 32; ++i) {
      y[i] = fmaf(s_o[0][2 * g + 1][lane * (D / 32) + i], w2, s_o[0][2 * g][lane * (D / 32) + i] * w1);
      sq = fmaf(y[i], y[i], sq);
    }
    if (p.diff.gain != nullptr) {
#pragma unroll
      for (int x = 16; x > 0; x >>= 1) sq += __shfl_xor_sync(0xffffffffu, sq, x);
      const float r = diff_norm<D>(sq, p.diff.eps);
#pragma unroll
      for (int i = 0; i < D / 32; ++i) y[i] *= r * __ldg(&p.diff.gain[(size_t)layer * D + lane * (D / 32) + i]);
    }
#pragma unroll
    for (int i = 0; i < D / 32; i += 2)
      *reinterpret_cast<uint32_t*>(p.out + (head0 + g) * D + lane * (D / 32) + i) = pack_bf16(y[i], y[i + 1]);
    if (lane < 2 && p.lse != nullptr) {
      const float x = lane == 0 ? l1 : l2;
      p.lse[2 * (head0 + g) + lane] = x > 0.f ? (s_top[2 * g + lane] + log2f(x)) * 0.6931471805599453f : -INFINITY;
    }
  }
}

template <int D, bool Q8>
xkv_status launch(const Params& p, int ctas, cudaStream_t st) {
  diff_decode_few_kernel<D, Q8><<<ctas, kThreads, 0, st>>>(p);
  count_launch();
  return check_launch();
}

int64_t few_ctas(const xkv_dims& streamed, int n_layers, int max_cache_len) {
  return (int64_t)n_layers * streamed.batch * streamed.n_kv_heads * std::max(1, (max_cache_len + kChunk - 1) / kChunk);
}

}  // namespace

bool diff_decode_is_few(const xkv_dims* streamed, int n_layers, int max_cache_len, int64_t max_rows) {
  const int64_t ctas = few_ctas(*streamed, n_layers, max_cache_len);
  if (ctas > kMaxCtas) return false;
  return max_cache_len <= kChunk ||
         ((int64_t)n_layers * streamed->batch * streamed->n_kv_heads <= kTickets && ctas * kRows <= max_rows);
}

xkv_status diff_decode_few(const xkv_dims* d, const xkv_cache* c, int layer_begin, int n_layers, const void* q, void* out,
                           float* lse, const DiffHeads& diff, const DecodeScratch& ws, cudaStream_t st) {
  const int max_cache_len = c->max_pages_per_seq * c->page_size;
  const xkv_dims streamed = streamed_dims(d, diff);
  const int64_t ctas = few_ctas(streamed, n_layers, max_cache_len);
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
  p.n_heads = streamed.n_kv_heads;
  p.page_size = c->page_size;
  p.max_pages_per_seq = c->max_pages_per_seq;
  p.n_pages = c->n_pages;
  p.max_chunks = std::max(1, (max_cache_len + kChunk - 1) / kChunk);
  p.scale_log2 = (d->scale != 0.f ? d->scale : 1.0f / sqrtf((float)(d->head_dim / 2))) * 1.4426950408889634f;
  p.diff = diff;
  p.tickets = static_cast<WorkspaceHeader*>(ws.header)->few_tickets;
  p.part_o = ws.part_o;
  p.part_ml = reinterpret_cast<float2*>(ws.part_ml);
  const bool q8 = c->kv_format == XKV_KV_INT8;
  if (d->head_dim == 128) return q8 ? launch<128, true>(p, (int)ctas, st) : launch<128, false>(p, (int)ctas, st);
  return q8 ? launch<64, true>(p, (int)ctas, st) : launch<64, false>(p, (int)ctas, st);
}

}  // namespace xkv
