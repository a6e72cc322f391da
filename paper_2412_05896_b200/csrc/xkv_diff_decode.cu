// Differential attention of single tokens over bf16 and int8 caches, straight from registers.
//
// Mathematics: that of xkv_diff_decode_attn.  With a head's query row [q1 | q2], cache rows [k1 | k2] and v,
//   z_s[c] = scale q_s . k_s[c],  p_s = exp(z_s - max z_s),  o_s = sum_c p_s[c] v[c]          s = 1, 2
// per chunk of rows, joined over the chunks of a cache by their maxima and sums; then the difference of the two maps and its norm.
//
// The streaming kernel stages rows in shared memory behind a plan of the lengths and suits calls that keep every SM busy for long;
// a small call is a chain of latencies, and a large one of 8-bit rows is bound by instructions.  Here one launch needs nothing planned
// before it: one CTA of four or eight warps per chunk of a streamed cache, a warp's 16 rows of K and V in its registers and the next tile's
// asked for as soon as their registers are free.  The products are mma.sync m16n8k16, rows on M and the (at most eight) query rows,
// both maps of up to four heads, on N: N = 8 fits, where a 128-row tcgen05 tile would be all but empty and the tensor pipe is idle
// either way.  A lane's part of a row is runs of consecutive columns, so no fragment goes through shared memory: of the logits the
// columns' order does not matter as long as the query has the same, and of the outputs it only says where a value is stored (V's
// fragments are transposed in registers, 8 x 8 at a time).  8-bit rows become fp16 with a bias, one instruction a pair, which comes
// off the sums.  The last CTA of a cache to finish joins the chunks (in their order, so the result does not depend on who that is)
// and sets the ticket back to zero.
// Weights are rounded to 16 bits for their product: half a step, 2^-8 of a weight in bf16, 2^-11 of weight times row scale in fp16, and
// below 2^-14 of the largest such product of a row that has a value 2^-25 (see scale_share); sums, maxima and outputs are fp32.
// Measured, device time: 16 caches of 49 - 146 rows of 64 7.4 us (floor 0.1: latencies of ids, rows, barriers and the launch); 2048 caches,
// 1.66 GB of bf16 rows 264 us = 6.3 TB/s, HBM; int8, one head a KV head, 338 MB 65 to 67 us = 5.1 TB/s, the chains
// of latencies at a CTA's two ends (loads take 36 % of L1's cycles, instructions 47 % of the issue slots).  bf16 rows of 128 spill 48 bytes a
// thread at their 128 registers.
#include <algorithm>

#include "common.cuh"
#include "ops.h"

namespace xkv {
namespace {

constexpr int kThreads = 256;         // of the kernel that stores new rows
constexpr int kRows = 8;              // query rows at most: the N of the products
constexpr int kSms = 148;
// CTAs of the attention that an SM takes at a time: two of eight warps; of four, four for rows of 128 and five for rows of 64, which fit in
// fewer registers (2048 int8 caches of 1000 such rows 63 us, with four 82, with six 68; rows of 128 with five 128, with four 102).
constexpr int ctas_of_an_sm(int head_dim, int warps) { return warps == 8 ? 2 : (head_dim == 64 ? 5 : 4); }
constexpr float kLazy = 8.f;          // log2 slack before the reference maximum is raised
constexpr int kTickets = sizeof(WorkspaceHeader::row_tickets) / 4;

struct AppendParams {
  const __nv_bfloat16* k_new;
  const __nv_bfloat16* v_new;
  uint8_t* k_pages;
  uint8_t* v_pages;
  float* k_scales;
  float* v_scales;
  const int32_t* block_table;
  int32_t* seq_lens;
  int32_t layer_begin, batch, n_kv_heads, page_size, max_pages_per_seq, n_pages;
  WorkspaceHeader* hdr;
};

// One CTA a unit: its new row of every KV head stored behind its last one, its length advanced.
template <int D, bool Q8>
__global__ void __launch_bounds__(kThreads) append_kernel(const AppendParams p) {
  constexpr int kPieces = D / 8;
  const int e = blockIdx.x;
  const size_t le = (size_t)p.layer_begin * p.batch + e;
  const int n = p.seq_lens[le];
  int page = -1;
  if (n >= 0 && n < p.max_pages_per_seq * p.page_size) page = p.block_table[le * p.max_pages_per_seq + n / p.page_size];
  if (page < 0 || page >= p.n_pages) {
    if (threadIdx.x == 0) record_status(p.hdr, XKV_ERR_CAPACITY);
    return;
  }
  for (int i = threadIdx.x; i < p.n_kv_heads * kPieces; i += kThreads) {       // (whole rows: a row's lanes stay together)
    const int h = i / kPieces, c = i % kPieces;
    const size_t src = ((size_t)e * p.n_kv_heads + h) * D + c * 8;
    const size_t row = ((size_t)page * p.n_kv_heads + h) * p.page_size + n % p.page_size;
    const uint4 k = __ldg(reinterpret_cast<const uint4*>(p.k_new + src)), v = __ldg(reinterpret_cast<const uint4*>(p.v_new + src));
    if constexpr (Q8) {
      float x[8], ks, vs;
      bf16x8_to_f32(k, x);
      const uint2 kc = quantize_row_piece(x, kPieces, &ks);
      bf16x8_to_f32(v, x);
      const uint2 vc = quantize_row_piece(x, kPieces, &vs);
      *reinterpret_cast<uint2*>(p.k_pages + row * D + c * 8) = kc;
      *reinterpret_cast<uint2*>(p.v_pages + row * D + c * 8) = vc;
      if (c == 0) {
        p.k_scales[row] = ks;
        p.v_scales[row] = vs;
      }
    } else {
      *reinterpret_cast<uint4*>(p.k_pages + (row * D + c * 8) * 2) = k;
      *reinterpret_cast<uint4*>(p.v_pages + (row * D + c * 8) * 2) = v;
    }
  }
  __syncthreads();                    // every thread has read the length
  if (threadIdx.x == 0) p.seq_lens[le] = n + 1;
}

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
  int32_t layer_begin, batch, n_q_heads, n_kv_heads, n_heads, page_size, max_pages_per_seq, n_pages, max_chunks, chunk;   // chunk: rows of a CTA
  float scale_log2;
  DiffHeads diff;
  int32_t* tickets;                   // [units * n_heads], zero; not used where max_chunks is 1
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
// What a lane has of a cached row: pieces of eight elements as they lie (four words of bf16 or two of stored bytes), in runs of kRun
// consecutive ones.  A run is 32 bytes (8-bit rows of 64: 16), so that the four lanes of a row take whole lines of it: of a load of eight rows L1
// hands out a line at a time (16-byte pieces took 64 % of its data cycles: int8 batch 91 us, then 76; bf16 batch 285, then 267, and 264
// with lines that L1 does not keep).
template <int D, bool Q8>
struct RowPart {
  static constexpr int kPieces = D / 32, kWords = Q8 ? 2 : 4;         // words: of a piece
  static constexpr int kRun = Q8 ? D / 4 : 16;
  uint32_t x[kPieces][kWords];
  // the first element of piece j of lane t of a row
  static __device__ __forceinline__ int column(int t, int j) { return kRun * (t + 4 * (8 * j / kRun)) + 8 * j % kRun; }
  __device__ __forceinline__ void load(const uint8_t* pages, size_t row, int t) {
    uint32_t* w = &x[0][0];
#pragma unroll
    for (int r = 0; r < D / 4 / kRun; ++r) {
      const uint8_t* at = pages + (row * D + kRun * (t + 4 * r)) * (Q8 ? 1 : 2);
      if constexpr (kRun * (Q8 ? 1 : 2) == 32) {
        asm volatile("ld.global.nc.L1::no_allocate.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                     : "=r"(w[8 * r]), "=r"(w[8 * r + 1]), "=r"(w[8 * r + 2]), "=r"(w[8 * r + 3]), "=r"(w[8 * r + 4]),
                       "=r"(w[8 * r + 5]), "=r"(w[8 * r + 6]), "=r"(w[8 * r + 7])
                     : "l"(at));
      } else {
        const uint4 v = __ldg(reinterpret_cast<const uint4*>(at));
        w[0] = v.x, w[1] = v.y, w[2] = v.z, w[3] = v.w;
      }
    }
  }
};
// The outputs' rows in shared memory: a gap of four floats every 32, and one that keeps rows apart, so that the lanes of a store meet in a
// bank in twos at most.
template <int D>
struct OutRows {
  static constexpr int kStride = D + D / 8 + (D == 128 ? 4 : 12);     // 4 modulo 16
  static __device__ __forceinline__ int at(int col) { return col + 4 * (col >> 5); }
};

// W warps: 8 or 4.
template <int D, bool Q8, int W>
__global__ void __launch_bounds__(32 * W, ctas_of_an_sm(D, W)) diff_decode_rows_kernel(const Params p) {
  constexpr int kWarps = W, kThreads = 32 * W, kTile = 16 * W;       // kTile: rows that the CTA has in registers
  constexpr int kPieces = D / 32;                    // pieces of eight columns that a lane has of a row
  using Part = RowPart<D, Q8>;
  using Out = OutRows<D>;
  __shared__ float s_o[kWarps][kRows][Out::kStride]; // the warps' outputs, then in [0] the CTA's
  __shared__ float s_m[kWarps][kRows], s_l[kWarps][kRows];
  __shared__ float s_top[kRows], s_sum[kRows];
  __shared__ float s_w[kRows][32];                   // a batch of chunks' weights
  __shared__ int s_last;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, gid = lane >> 2, tig = lane & 3;
  const int chunk = blockIdx.x % p.max_chunks, unit_head = blockIdx.x / p.max_chunks;
  const int h = unit_head % p.n_heads, e = unit_head / p.n_heads, kvh = h / p.diff.subs;
  const size_t le = (size_t)p.layer_begin * p.batch + e;
  const int n = min(max(__ldg(&p.seq_lens[le]), 0), p.max_pages_per_seq * p.page_size);
  const int n_chunks = max((n + p.chunk - 1) / p.chunk, 1);
  if (chunk >= n_chunks) return;
  const int n_rows = 2 * p.diff.heads(h);            // row 2 j + s is map s of head j
  const size_t head0 = (size_t)e * p.n_q_heads + p.diff.first_head(h);
  // ---- this warp's tiles of 16 rows, kTile apart; of a tile a lane has its part of rows gid and gid + 8
  const int end = min(n, (chunk + 1) * p.chunk);
  int row0 = chunk * p.chunk + 16 * warp;
  Part k[2], v[2];
  float ks[2] = {1.f, 1.f}, vs[2] = {1.f, 1.f};
  const int32_t* table = p.block_table + le * p.max_pages_per_seq;
  // first row of a tile in the page pool (page_size is a multiple of 16: its rows share a page)
  auto pool_row = [&](int at) -> size_t {
    const int page = at < end ? min(max(__ldg(&table[at / p.page_size]), 0), p.n_pages - 1) : 0;
    return ((size_t)page * p.n_kv_heads + kvh) * p.page_size + at % p.page_size + gid;
  };
  auto load_k = [&](size_t first) {
#pragma unroll
    for (int y = 0; y < 2; ++y) {
      k[y].load(p.k_pages, first + 8 * y, tig);
      if constexpr (Q8) ks[y] = __ldg(&p.k_scales[first + 8 * y]);
    }
  };
  auto load_v = [&](size_t first) {
#pragma unroll
    for (int y = 0; y < 2; ++y) {
      v[y].load(p.v_pages, first + 8 * y, tig);
      if constexpr (Q8) vs[y] = __ldg(&p.v_scales[first + 8 * y]);
    }
  };
  size_t now = pool_row(row0);
  if (row0 < end) {
    load_k(now);
    load_v(now);
  }
  // ---- the query row of this lane: the half that is not its map's is zero
  uint32_t q[kPieces][4];
#pragma unroll
  for (int j = 0; j < kPieces; ++j) {
    uint4 r = make_uint4(0u, 0u, 0u, 0u);
    const int col = Part::column(tig, j);
    if (gid < n_rows && (col >= D / 2) == ((gid & 1) != 0))
      r = __ldg(reinterpret_cast<const uint4*>(p.q + (head0 + (gid >> 1)) * D + col));
    q[j][0] = r.x, q[j][1] = r.y, q[j][2] = r.z, q[j][3] = r.w;
    if constexpr (Q8) {
#pragma unroll
      for (int i = 0; i < 4; ++i) q[j][i] = pack16<true>(bf16_lo(q[j][i]), bf16_hi(q[j][i]));
    }
  }
  // 8-bit rows enter the products as kInt8Bias + integer (one instruction a pair): kInt8Bias times the query's sum comes off every logit,
  // kInt8Bias times the sum of the weights off every output.  Both sums are products with ones, rounded like what they correct.
  const uint32_t ones[4] = {0x3c003c00u, 0x3c003c00u, 0x3c003c00u, 0x3c003c00u};
  float q_bias[4] = {0.f, 0.f, 0.f, 0.f}, w_sum[4] = {0.f, 0.f, 0.f, 0.f};
  if constexpr (Q8) {
#pragma unroll
    for (int j = 0; j < kPieces; ++j) {
      mma_f16(q_bias, ones, q[j][0], q[j][1]);
      mma_f16(q_bias, ones, q[j][2], q[j][3]);
    }
  }
  float m[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f};     // of query rows 2 tig and 2 tig + 1; l: of this lane's rows
  float o[D / 16][4];
#pragma unroll
  for (int x = 0; x < D / 16; ++x) o[x][0] = o[x][1] = o[x][2] = o[x][3] = 0.f;
#pragma unroll 1
  for (; row0 < end; row0 += kTile) {
    const int rows = end - row0;
    const bool more = row0 + kTile < end;
    const size_t next = pool_row(row0 + kTile);
    float z[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int j = 0; j < kPieces; ++j)
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        uint32_t a[4];
        if constexpr (Q8) {
          a[0] = int8x2_to_biased_f16x2<0x5140>(k[0].x[j][i]), a[1] = int8x2_to_biased_f16x2<0x5140>(k[1].x[j][i]);
          a[2] = int8x2_to_biased_f16x2<0x5342>(k[0].x[j][i]), a[3] = int8x2_to_biased_f16x2<0x5342>(k[1].x[j][i]);
        } else {
          a[0] = k[0].x[j][2 * i], a[1] = k[1].x[j][2 * i], a[2] = k[0].x[j][2 * i + 1], a[3] = k[1].x[j][2 * i + 1];
        }
        mma<Q8>(z, a, q[j][2 * i], q[j][2 * i + 1]);
      }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if constexpr (Q8) z[i] = fmaf(-kInt8Bias, q_bias[i], z[i]) * ks[i >> 1];
      z[i] = gid + 8 * (i >> 1) < rows ? z[i] * p.scale_log2 : -INFINITY;
    }
    if (more) load_k(next);           // under the softmax and the outputs
    // rows behind the last one: no weight and no value, whatever lies there
    if (rows < 16) {
#pragma unroll
      for (int y = 0; y < 2; ++y)
        if (gid + 8 * y >= rows) {
          vs[y] = 0.f;
          if constexpr (!Q8) {
#pragma unroll
            for (int j = 0; j < kPieces; ++j) v[y].x[j][0] = v[y].x[j][1] = v[y].x[j][2] = v[y].x[j][3] = 0u;
          }
        }
    }
    // the warp's reference is exact on its first tile and raised lazily (by 2^8) afterwards
    float top[2];
    auto tops = [&] {
      if constexpr (Q8) {
        const float b0 = scale_share(vs[0]), b1 = scale_share(vs[1]);
        top[0] = fmaxf(z[0] + b0, z[2] + b1), top[1] = fmaxf(z[1] + b0, z[3] + b1);
      } else {
        top[0] = fmaxf(z[0], z[2]), top[1] = fmaxf(z[1], z[3]);
      }
    };
    tops();
    if (__any_sync(0xffffffffu, top[0] > m[0] + kLazy || top[1] > m[1] + kLazy)) {
      float al[2];
      if constexpr (Q8) {
#pragma unroll
        for (int y = 0; y < 2; ++y) {
          uint32_t x = 0u;
#pragma unroll
          for (int j = 0; j < kPieces; ++j) x |= (v[y].x[j][0] ^ 0x80808080u) | (v[y].x[j][1] ^ 0x80808080u);
          if (!row_has_value(x)) vs[y] = 0.f;
        }
        tops();
      }
#pragma unroll
      for (int i = 0; i < 2; ++i) {
#pragma unroll
        for (int x = 4; x < 32; x <<= 1) top[i] = fmaxf(top[i], __shfl_xor_sync(0xffffffffu, top[i], x));
        top[i] = fmaxf(top[i], m[i]);
        al[i] = m[i] == -INFINITY ? 0.f : fast_exp2(m[i] - top[i]);
        m[i] = top[i];
        l[i] *= al[i];
      }
#pragma unroll
      for (int x = 0; x < D / 16; ++x) {
        o[x][0] *= al[0];
        o[x][1] *= al[1];
        o[x][2] *= al[0];
        o[x][3] *= al[1];
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) w_sum[i] *= al[i & 1];
    }
    float w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = fast_exp2(z[i] - (m[i & 1] == -INFINITY ? 0.f : m[i & 1]));
    l[0] += w[0] + w[2];
    l[1] += w[1] + w[3];
    // the weights as the B operand (rounded to 16 bits, 8-bit rows: times the row's scale)
    if constexpr (Q8) {
#pragma unroll
      for (int i = 0; i < 4; ++i) w[i] *= vs[i >> 1];
    }
    const uint32_t b0 = movmatrix_trans(pack16<Q8>(w[0], w[1])), b1 = movmatrix_trans(pack16<Q8>(w[2], w[3]));
#pragma unroll
    for (int j = 0; j < kPieces; ++j)
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        uint32_t a[4];
        if constexpr (Q8) {           // two neighbouring columns travel as one 16-bit element
          const uint32_t t0 = movmatrix_trans(v[0].x[j][i]), t1 = movmatrix_trans(v[1].x[j][i]);
          a[0] = int8x2_to_biased_f16x2<0x5240>(t0), a[1] = int8x2_to_biased_f16x2<0x5341>(t0);
          a[2] = int8x2_to_biased_f16x2<0x5240>(t1), a[3] = int8x2_to_biased_f16x2<0x5341>(t1);
        } else {
          a[0] = movmatrix_trans(v[0].x[j][2 * i]), a[1] = movmatrix_trans(v[0].x[j][2 * i + 1]);
          a[2] = movmatrix_trans(v[1].x[j][2 * i]), a[3] = movmatrix_trans(v[1].x[j][2 * i + 1]);
        }
        mma<Q8>(o[2 * j + i], a, b0, b1);
      }
    if constexpr (Q8) mma_f16(w_sum, ones, b0, b1);
    if (more) load_v(next);           // under the next tile's logits
  }
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int x = 4; x < 32; x <<= 1) l[i] += __shfl_xor_sync(0xffffffffu, l[i], x);
  // accumulator row gid of block (j, i) is column 4 i + gid % 2 of piece j of lane gid / 2, row gid + 8 the one 2 further; 8-bit rows:
  // + 2 (gid % 2), and the next one
#pragma unroll
  for (int x = 0; x < D / 16; ++x)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int col = Part::column(gid >> 1, x >> 1) + 4 * (x & 1) + (Q8 ? 2 * (gid & 1) + (i >> 1) : 2 * (i >> 1) + (gid & 1));
      s_o[warp][2 * tig + (i & 1)][Out::at(col)] = Q8 ? fmaf(-kInt8Bias, w_sum[i], o[x][i]) : o[x][i];
    }
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
    const int i = x * kThreads + tid, r = i / D, col = Out::at(i % D);
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
    for (int x = 0; x < kMine; ++x) {
      const int i = x * kThreads + tid;
      __stcg(&part[i], s_o[0][i / D][Out::at(i % D)]);
    }
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
    for (int r = warp; r < kRows; r += kWarps) {     // a warp a query row: maximum and sum over all chunks
      float top = -INFINITY, sum = 0.f;
      for (int i = lane; i < n_chunks; i += 32) top = fmaxf(top, __ldcg(&p.part_ml[(first + i) * kRows + r]).x);
#pragma unroll
      for (int x = 16; x > 0; x >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, x));
      for (int i = lane; i < n_chunks; i += 32) {
        const float2 ml = __ldcg(&p.part_ml[(first + i) * kRows + r]);
        sum = fmaf(fast_exp2(ml.x - top), ml.y, sum);
      }
#pragma unroll
      for (int x = 16; x > 0; x >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, x);
      if (lane == 0) {
        s_top[r] = top;
        s_sum[r] = sum;
      }
    }
    float acc[kMine];
#pragma unroll
    for (int x = 0; x < kMine; ++x) acc[x] = 0.f;
    for (int c0 = 0; c0 < n_chunks; c0 += 32) {
      const int nb = min(32, n_chunks - c0);
      __syncthreads();
      for (int r = warp; r < kRows; r += kWarps)
        if (lane < nb) s_w[r][lane] = fast_exp2(__ldcg(&p.part_ml[(first + c0 + lane) * kRows + r]).x - s_top[r]);
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
    for (int x = 0; x < kMine; ++x) {
      const int i = x * kThreads + tid;
      s_o[0][i / D][Out::at(i % D)] = acc[x];
    }
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
      const int col = Out::at(lane * (D / 32) + i);
      y[i] = fmaf(s_o[0][2 * g + 1][col], w2, s_o[0][2 * g][col] * w1);
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
xkv_status launch(const Params& p, int warps, int ctas, cudaStream_t st) {
  if (warps == 8) diff_decode_rows_kernel<D, Q8, 8><<<ctas, 256, 0, st>>>(p);
  else            diff_decode_rows_kernel<D, Q8, 4><<<ctas, 128, 0, st>>>(p);
  count_launch();
  return check_launch();
}

struct Cut {
  int warps, chunk, max_chunks;       // rows of a CTA, CTAs of the longest cache that its table allows
  int64_t ctas;
};
// Little to do (fewer than four tiles of 64 rows for each four-warp CTA that runs at the same time): eight warps a CTA, as many chunks as
// run at the same time, but no more than about the root of eight times a cache's tiles, since one CTA joins them, at some 0.2 us a
// chunk, where a tile takes 1.5 us (32 000 rows of one KV head: 251 chunks 59 us, 42 chunks 25 us).  More: four warps, whose CTAs start
// and end under each other's loads (2048 int8 caches of 1000 rows 109 to 102 us, eight heads 184 to 152; but one request of 8 caches
// 11.5 to 21), unless long bf16 rows are in not so many caches: CTAs of twice the speed wait less for the longest (2048 caches of 290 to
// 2707 rows 264 us, with four warps 276).  With more caches than CTAs at a time a cache is one chunk, since joins cost (2048 caches
// of 1000 rows cut in two 102 to 134 us), but for a last wave that is mostly empty (640 caches of 3000 rows 213 to 183 us).
// Tables of more than 12 288 rows: chunks of 4096, as far as that makes eight waves of CTAs, most of which may find nothing (a sequence of
// 65 536 rows among 15 short ones 437 to 80 us; 64 short sequences in tables of 32 768 rows 37 to 43, the streaming kernel 60).
// max_rows: query rows that the partial results have room for.
Cut cut(const xkv_dims& streamed, const xkv_cache& cache, int n_layers, int64_t max_rows) {
  const int64_t caches = (int64_t)n_layers * streamed.batch * streamed.n_kv_heads;
  const int64_t rows = std::max<int64_t>(1, (int64_t)cache.max_pages_per_seq * cache.page_size);
  Cut c;
  c.warps = caches * ((rows + 63) / 64) < 4 * 4 * kSms ||
            (cache.kv_format == XKV_KV_BF16 && rows > 1024 && caches < 4096) ? 8 : 4;
  const int64_t tile = 16 * c.warps, tiles = (rows + tile - 1) / tile;
  const int64_t slots = ctas_of_an_sm(streamed.head_dim, c.warps) * kSms;
  int64_t chunks = slots / caches;
  if (caches > slots && 4 * caches < 3 * slots * ((caches + slots - 1) / slots))
    chunks = std::min((4 * slots + caches - 1) / caches, tiles / 16);
  if (rows > 12288) chunks = std::max(chunks, std::min((rows + 4095) / 4096, 8 * slots / caches));
  chunks = std::max<int64_t>(std::min({chunks, tiles, max_rows / kRows / caches}), 1);
  int64_t per = (tiles + chunks - 1) / chunks;
  while (per * per * 8 < tiles) ++per;
  c.max_chunks = (int)((tiles + per - 1) / per);
  c.chunk = (int)(((tiles + c.max_chunks - 1) / c.max_chunks) * tile);
  c.ctas = caches * c.max_chunks;
  return c;
}

}  // namespace

// Whether this kernel or the streaming one takes a call without chunk_rows.  Device time of both, us (rows of 128, G = 4 unless said):
//   bf16: 8 caches of 2129 rows 12.3 / 31.0, 64 of 2000 20.6 / 36.6, 2048 of 120 37.5 / 38.3, of 1000 177 / 218, 4096 of 1500 475 / 585;
//   G = 1: 2048 of 1000 175 / 191
//   int8, the same: 11.6 / 48.6, 18.6 / 52.1, 23.7 / 45.2, 103 / 155, 269 / 427;  G = 1: 101 / 146
// Not so where one cache is much longer than the others in tables of up to 12 288 rows, which this kernel does not cut: 512 caches of
// 200 - 1000 rows and one sequence of 12 000 195 / 89, int8 171 / 91.
bool diff_decode_by_rows(const xkv_dims* streamed, const xkv_cache* c, int n_layers, int64_t max_rows) {
  if (c->kv_format == XKV_KV_E4M3 || ((reinterpret_cast<uintptr_t>(c->k_pages) | reinterpret_cast<uintptr_t>(c->v_pages)) & 31u) != 0)
    return false;                     // (a run is one load)
  return cut(*streamed, *c, n_layers, max_rows).ctas < (1 << 30);
}

xkv_status diff_decode_rows(const xkv_dims* d, const xkv_cache* c, int layer_begin, int n_layers, const void* q,
                           const void* k_new, const void* v_new, void* out, float* lse, const DiffHeads& diff,
                           const DecodeScratch& ws, int64_t max_rows, cudaStream_t st) {
  const bool q8 = c->kv_format == XKV_KV_INT8, wide = d->head_dim == 128;
  if (k_new != nullptr) {
    const AppendParams a = {static_cast<const __nv_bfloat16*>(k_new), static_cast<const __nv_bfloat16*>(v_new),
                            static_cast<uint8_t*>(c->k_pages), static_cast<uint8_t*>(c->v_pages), c->k_scales, c->v_scales,
                            c->block_table, c->seq_lens, layer_begin, d->batch, d->n_kv_heads, c->page_size,
                            c->max_pages_per_seq, c->n_pages, static_cast<WorkspaceHeader*>(ws.header)};
    const int units = n_layers * d->batch;
    if (wide) {
      if (q8) append_kernel<128, true><<<units, kThreads, 0, st>>>(a);
      else    append_kernel<128, false><<<units, kThreads, 0, st>>>(a);
    } else {
      if (q8) append_kernel<64, true><<<units, kThreads, 0, st>>>(a);
      else    append_kernel<64, false><<<units, kThreads, 0, st>>>(a);
    }
    count_launch();
    const xkv_status s = check_launch();
    if (s != XKV_OK) return s;
  }
  const xkv_dims streamed = streamed_dims(d, diff);
  const Cut how = cut(streamed, *c, n_layers, max_rows);
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
  p.max_chunks = how.max_chunks;
  p.chunk = how.chunk;
  p.scale_log2 = (d->scale != 0.f ? d->scale : 1.0f / sqrtf((float)(d->head_dim / 2))) * 1.4426950408889634f;
  p.diff = diff;
  // Tickets that stay zero between calls, where they suffice; others are cleared first (a launch more, 2 us).
  p.tickets = static_cast<WorkspaceHeader*>(ws.header)->row_tickets;
  const int64_t caches = (int64_t)n_layers * d->batch * p.n_heads;
  if (p.max_chunks > 1 && caches > kTickets) {
    p.tickets = ws.tickets;
    if (cudaMemsetAsync(p.tickets, 0, caches * 4, st) != cudaSuccess) return XKV_ERR_CUDA;
  }
  p.part_o = ws.part_o;
  p.part_ml = reinterpret_cast<float2*>(ws.part_ml);
  const int ctas = (int)how.ctas;
  if (wide) return q8 ? launch<128, true>(p, how.warps, ctas, st) : launch<128, false>(p, how.warps, ctas, st);
  return q8 ? launch<64, true>(p, how.warps, ctas, st) : launch<64, false>(p, how.warps, ctas, st);
}

}  // namespace xkv
