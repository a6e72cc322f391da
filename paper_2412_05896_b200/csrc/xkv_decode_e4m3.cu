// Decode attention over caches of 8-bit floats with one scale per block of 16 slots and KV head (Eq. 1, one query row
// per head), on the 5th-generation tensor cores without converting a cached byte.
//
// Mathematics.  With stored codes k, v (e4m3), block scales s_k, s_v and the G query heads of a KV head:
//   logits  S[c, h] = (codes k_c . q_h) s_k[c] scale          M = 128 cache rows, N = heads, K = d
//   output  O[j, h] = sum_c v[c, j] (s_v[c] P[c, h])          M = d, N = heads, K = a tile's cache rows
// Both products are tcgen05.mma kind::f8f6f4 with the cache tile as the A operand exactly as it lies in the page (K rows
// are K-major, V rows are M-major), fp32 accumulators in tensor memory.  The small operand has more bits than one code
// holds, so it enters as two codes side by side on the N axis: q = a1 + a2 / 32 and p = b1 + b2 / 32, each part rounded to
// nearest.  The query is scaled so that its largest element lies in [128, 256): a bf16 value (8 significant bits) is
// exactly such a sum down to 2^-15, 2^-22 of the largest.  The products s_v P of a tile are scaled so that the largest is 256:
// the sum keeps 2^-8 of one (the rounding of bf16) down to 2^-15, 2^-23 of the tile's largest.  For that the softmax's
// reference is not the tile's largest logit but its largest S + log2(s_v / max s_v), whichever row has it (a row of a large s_v and
// no weight costs the others no bits); a weight may then exceed 1, by 2^80 at most, to where s_v / max s_v counts in it.
// Because the range is per tile, every tile's product goes to fresh accumulators and is added in fp32 registers with the
// tile's own factor; nothing in tensor memory is ever rescaled.
//
// Shape of the launch: two CTAs of eight warps per SM, no CTA waits for another one.  All (layer, sequence, KV head) caches
// lie on one line, a cache as long as the blocks of its tiles plus a constant for what a cache costs besides them (by tiles,
// not by rows: 7168 caches of 84 to 157 rows with G = 7 take 107 us, by rows 116 us, other shapes the same), and the line
// is cut into equal segments, one per CTA, that every CTA derives for itself from the lengths.  A tile belongs to
// the segment in which it starts.  A cache cut by a boundary leaves partial results (m, l, O), at most two pieces a CTA, and
// the CTA that finishes the last piece joins them in the order of the pieces, so the result does not depend on who
// was when.  (Small segments at the ends of the shares that go to whoever is done first level the finishing times, but
// what they add in pieces and joins costs more: 74.6 against 70.2 us for 363 MB, 150.8 against 140.2 us for 814 MB.)
// Bound by HBM where caches are long, else by what a launch costs before the first and after the last byte (about 8 us: the
// lengths, page ids and first tiles one after the other; the last tile's softmax, output, count and join).  Measured, device
// time a call: 538 MB in two caches of 131 000 rows x 8 heads 92.6 us (0.88 of the measured copy rate; 7.4 TB/s between
// the first tile and the last), 814 MB ragged batch 133.3 us (0.93), 363 MB of 2048 short caches 63.8 us (0.87), one request
// of 2129 rows 12.5 us.  With five to eight heads a group the softmax warps bound it where caches are short or d = 64 (a
// third of the issue slots, the rest waits on what comes before): 246 MB in 7168 caches of 84-157 rows, G = 7, 105 us;
// 214 MB of d = 64, G = 5, 53.3 us.  A call that also appends (two launches in series) takes 2 us more for one request, 14 us more
// for the ragged batch (146 us).
//
//   warp 6     finds the CTA's pieces of caches ("items") and lays out their queries as two codes per element
//   warp 4     copies: TMA boxes of K and V, block scales
//   warp 5     issues the MMAs: logits up to two tiles ahead of the outputs
//   warps 0-3  one thread per cache row (two rows with d = 64): logits out of tensor memory, the tile's maximum (one exchange among the four
//              warps), weights back as codes; then, as one thread per output column, O of the tile before
//   warp 7     counts finished pieces of cut caches and joins those that are complete, by query heads; warps that
//              have run out of tiles help
#include <cuda.h>

#include <atomic>
#include <cmath>

#include "common.cuh"
#include "e4m3.cuh"
#include "ops.h"
#include "tc_common.cuh"

namespace xkv {
namespace {

using tc::tc_fence_after_sync;
using tc::tc_fence_before_sync;
using tc::tmem_alloc;
using tc::tmem_dealloc;
using tc::tmem_relinquish;
using tc::tmem_wait_ld;
using tc::umma_commit;

constexpr int kN = 16;                // N of both MMAs: two codes x up to eight heads, the rest zero rows
constexpr int kThreads = 256;
constexpr int kSoftThreads = 128;
constexpr int kFifo = 3;              // items between the walk and the last reader
constexpr int kCtasPerSm = 2;
constexpr float kPart = 32.f;         // weight of the second code
constexpr float kMinShare = -80.f;    // log2 of the smallest s_v / max s_v of a tile that counts in the softmax's reference
constexpr int kBarSoft = 1;           // named barrier of warps 0-3
constexpr int kCacheCost = 12;        // what a cache costs besides its tiles, in blocks of 16 rows (2048 caches of 203 to 1101 rows
                                      // laid out by rows: 66.6 us with 4, 64.9 with 8, 64.2 with 12, 64.9 with 16)
constexpr int kJobs = 2;              // joins of a CTA: only the pieces at the two ends of its share are of cut caches

template <int D>
struct Cfg {
  // A tile is 16 KB of K and of V: 128 rows of 128 elements or 256 of 64.  What the softmax warps spend on a tile is mostly
  // waits and exchanges that do not grow with its rows.
  static constexpr int kTile = 128 * (128 / D);                 // cache rows per tile
  static constexpr int kSpans = kTile / 128;                    // M = 128 products per tile of logits, rows per softmax thread
  static constexpr int kTileBlocks = kTile / kScaleBlock;
  static constexpr int kMinSegment = kTileBlocks;               // shortest segment, in blocks: a tile, so that a cache has a
                                                                // tile in every segment between its first and its last one
  static constexpr int kTmemCols = kSpans == 1 ? 64 : 128;      // two logit buffers, two output buffers; 16 columns a product
  static constexpr int kStages = 3;                             // 96 KB a CTA
  static constexpr int kTileBytes = kTile * D;
  static constexpr int kQBytes = kN * D;
  static constexpr int kPBytes = kN * kTile;                    // 16 bytes a cache row
  static constexpr int kOffV = kStages * kTileBytes;
  static constexpr int kOffQ = 2 * kStages * kTileBytes;
  static constexpr int kOffP = kOffQ + kFifo * kQBytes;
  static constexpr int kOffScales = kOffP + 2 * kPBytes;         // [kStages][2 * kTileBlocks]: of K, of V
  static constexpr int kSmemBytes = 1024 + kOffScales + kStages * 8 * kTileBlocks;
};

struct Params {
  const __nv_bfloat16* q;
  __nv_bfloat16* out;
  float* lse;
  const float* k_scales;
  const float* v_scales;
  const int32_t* block_table;
  const int32_t* seq_lens;
  int32_t layer_begin, batch, n_units, n_q_heads, n_kv_heads, group, page_size, max_pages_per_seq, n_pages;
  // row -> page: page_size is 8 n with n even, 2 <= n <= 32, and x / n = (x * ceil(2^32 / n)) >> 32 for x <= 2^27 + 32
  uint32_t page_mul;                  // ceil(2^32 / n)
  __device__ __forceinline__ int page_of(int row) const { return (int)__umulhi((uint32_t)row >> 3, page_mul); }
  int32_t box_rows;                   // rows of a TMA box: the largest power of two up to a tile's that divides page_size
  int32_t box_shift;                  // its logarithm
  int32_t max_ctas;                   // CTAs that the partial results have room for
  int32_t withhold_cta;               // test hook: this CTA's copies are never issued, so that waits expire (-1: none)
  int32_t wait_first;                 // the launch before this one appends rows: wait for it before reading a length
  float scale_log2;
  uint64_t wait_ns;
  WorkspaceHeader* hdr;
  int32_t* tickets;                   // [units * n_kv_heads] pieces of a cache that are done
  float* part_o;                      // [2 * CTAs][G][D]
  float* part_ml;                     // [2 * CTAs][G][2]
};

// a / b for 0 <= a < 2^31, 0 < b: two steps of a reciprocal and a correction, half the instructions of the general
// division.  (What a CTA runs once it runs out of a cold instruction cache, at some seven clocks an instruction.)
__device__ __forceinline__ int quotient(int a, int b) {
  const float inv = __frcp_rn((float)b);
  int q = (int)((float)a * inv);                  // off by at most a / b * 2^-22 + 1
  q += (int)((float)(a - q * b) * inv);           // off by at most one
  const int r = a - q * b;
  return r < 0 ? q - 1 : (r >= b ? q + 1 : q);
}

// [0, n) cut into `parts` runs that differ by at most one.
struct Cut {
  int32_t q, r;
  __device__ __forceinline__ Cut(int n, int parts) : q(quotient(n, parts)), r(n - q * parts) {}
  __device__ __forceinline__ int begin(int i) const { return i * q + min(i, r); }
  __device__ __forceinline__ int part_of(int x) const {
    const bool longer = x < r * (q + 1);
    return longer ? quotient(x, q + 1) : r + quotient(x - r * (q + 1), q);
  }
};

struct Item {                         // one CTA's piece of one cache
  int32_t e, h, row0, rows;           // unit, KV head, first row, rows; e < 0: no more
  int32_t first_cta, n_pieces;        // the CTAs that share the cache
};

// D[tmem] (+)= A[smem] B[smem]^T, e4m3 x e4m3 -> fp32; issued by one thread.
__device__ __forceinline__ void umma_e4m3(uint32_t tmem_d, uint64_t adesc, uint64_t bdesc, uint32_t idesc,
                                          uint32_t accumulate) {
  asm volatile(
      "{\n\t"
      ".reg .pred p;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], %1, %2, %3, {%5, %5, %5, %5}, p;\n\t"
      "}\n" ::"r"(tmem_d),
      "l"(adesc), "l"(bdesc), "r"(idesc), "r"(accumulate), "r"(0u)
      : "memory");
}

// One lane of a converged warp.
__device__ __forceinline__ bool elect_one() {
  uint32_t r;
  asm volatile("{\n\t.reg .pred q;\n\telect.sync _|q, 0xffffffff;\n\tselp.u32 %0, 1, 0, q;\n\t}" : "=r"(r));
  return r != 0;
}

// Shared-memory matrix descriptor: rows of kRowBytes (128: 128-byte swizzle, 64: 64-byte swizzle), groups of eight rows
// 8 * kRowBytes apart.  The same for a K-major operand (rows = M or N) and an M-major one (rows = K) whose M extent is
// the row.
template <int kRowBytes>
__device__ __forceinline__ uint64_t smem_desc(uint32_t addr) {
  uint64_t d = (uint64_t)((addr & 0x3ffffu) >> 4);
  d |= (uint64_t)1 << 16;
  d |= (uint64_t)((8 * kRowBytes) >> 4) << 32;
  d |= (uint64_t)1 << 46;
  d |= (uint64_t)(kRowBytes == 128 ? 2 : 4) << 61;
  return d;
}
// An N-major operand of 16 N values of one byte: 16 bytes a row of K, no swizzle (groups of eight rows 128 bytes apart).
__device__ __forceinline__ uint64_t smem_desc_rows16(uint32_t addr) {
  return (uint64_t)((addr & 0x3ffffu) >> 4) | (uint64_t)(128 >> 4) << 16 | (uint64_t)(128 >> 4) << 32 | (uint64_t)1 << 46;
}
// e4m3 x e4m3 -> fp32, M x N; mn: the operands are M-major and N-major, else both K-major
__host__ __device__ constexpr uint32_t idesc_e4m3(int M, int N, bool mn) {
  return (1u << 4) | (mn ? 3u << 15 : 0u) | ((uint32_t)(N >> 3) << 17) | ((uint32_t)(M >> 4) << 24);
}
// byte offset of (row, column byte) in a swizzled operand
template <int kRowBytes>
__device__ __forceinline__ uint32_t swizzled(int row, int col) {
  const int x = kRowBytes == 128 ? (row & 7) : ((row >> 1) & 3);
  return (uint32_t)(row * kRowBytes + (((col >> 4) ^ x) << 4) + (col & 15));
}

template <int N>
__device__ __forceinline__ void tmem_ld(uint32_t taddr, float (&v)[N]) {
  uint32_t r[N];
  if constexpr (N == 2) {
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x2.b32 {%0, %1}, [%2];" : "=r"(r[0]), "=r"(r[1]) : "r"(taddr) : "memory");
  } else if constexpr (N == 4) {
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x4.b32 {%0, %1, %2, %3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
                 : "r"(taddr)
                 : "memory");
  } else if constexpr (N == 8) {
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7])
                 : "r"(taddr)
                 : "memory");
  } else {
    static_assert(N == 16, "2, 4, 8 or 16 columns");
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, "
        "[%16];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
          "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
        : "r"(taddr)
        : "memory");
  }
  tmem_wait_ld();
#pragma unroll
  for (int i = 0; i < N; ++i) v[i] = __uint_as_float(r[i]);
}

__device__ __forceinline__ float warp_max(float x) {
  float r;
  asm volatile("redux.sync.max.f32 %0, %1, 0xffffffff;" : "=f"(r) : "f"(x));
  return r;
}
// 1 / x within 2^-23, one instruction
__device__ __forceinline__ float fast_rcp(float x) {
  float r;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}
// A value per head to and from shared memory (16-byte aligned), in as few accesses as there are.
template <int GP>
__device__ __forceinline__ void put_heads(float* dst, const float (&v)[GP]) {
  if constexpr (GP >= 4) {
#pragma unroll
    for (int g = 0; g < GP; g += 4) *reinterpret_cast<float4*>(dst + g) = make_float4(v[g], v[g + 1], v[g + 2], v[g + 3]);
  } else if constexpr (GP == 2) {
    *reinterpret_cast<float2*>(dst) = make_float2(v[0], v[1]);
  } else {
    dst[0] = v[0];
  }
}
template <int GP>
__device__ __forceinline__ void get_heads(const float* src, float (&v)[GP]) {
  if constexpr (GP >= 4) {
#pragma unroll
    for (int g = 0; g < GP; g += 4) {
      const float4 x = *reinterpret_cast<const float4*>(src + g);
      v[g] = x.x, v[g + 1] = x.y, v[g + 2] = x.z, v[g + 3] = x.w;
    }
  } else if constexpr (GP == 2) {
    const float2 x = *reinterpret_cast<const float2*>(src);
    v[0] = x.x, v[1] = x.y;
  } else {
    v[0] = src[0];
  }
}
// Barrier of the four softmax warps that also tells whether any of its threads passed a true predicate.
__device__ __forceinline__ bool soft_any(bool x) {
  uint32_t r;
  asm volatile(
      "{\n\t.reg .pred p, q;\n\t"
      "setp.ne.b32 p, %1, 0;\n\t"
      "barrier.cta.red.or.pred q, %2, %3, p;\n\t"
      "selp.u32 %0, 1, 0, q;\n\t}"
      : "=r"(r)
      : "r"((uint32_t)x), "n"(kBarSoft), "n"(kSoftThreads)
      : "memory");
  return r != 0;
}
// Bounded wait for the phase with the given parity; gives up when another role has raised the abort flag.  A short rolled
// loop: the kernel waits in two dozen places, and its roles share the instruction cache.
__device__ __forceinline__ bool wait_bar(uint64_t* bar, uint32_t parity, volatile int* abort_flag, uint64_t limit_ns) {
  if (mbar_try_wait(bar, parity)) return true;
  const uint64_t t0 = global_timer_ns();
#pragma unroll 1
  while (!mbar_try_wait(bar, parity)) {
    if (*abort_flag) return false;
    if (global_timer_ns() - t0 > limit_ns) {
      *abort_flag = 1;
      return false;
    }
  }
  return true;
}
__device__ __forceinline__ int add_acq_rel(int32_t* at, int v) {
  int was;
  asm volatile("atom.add.acq_rel.gpu.global.s32 %0, [%1], %2;" : "=r"(was) : "l"(at), "r"(v) : "memory");
  return was;
}
// Whether the phase with the given parity is over, without waiting.
__device__ __forceinline__ bool mbar_test(uint64_t* bar, uint32_t parity) {
  uint32_t ok;
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "mbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
      "selp.u32 %0, 1, 0, p;\n\t}"
      : "=r"(ok)
      : "r"(smem_u32(bar)), "r"(parity)
      : "memory");
  return ok != 0;
}
// 4-byte asynchronous copy global -> shared, zero when !valid
__device__ __forceinline__ void cp_async_4(void* dst, const void* src, bool valid) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(smem_u32(dst)), "l"(src), "r"(valid ? 4 : 0) : "memory");
}
// the barrier gets one arrival once this thread's copies so far have landed
__device__ __forceinline__ void cp_async_arrive(uint64_t* bar) {
  asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(smem_u32(bar)) : "memory");
}

// Programmatic dependent launch: returns once the launch before this one has completed and its writes are visible.
__device__ __forceinline__ void grid_dependency_wait() { asm volatile("griddepcontrol.wait;" ::: "memory"); }

__device__ __forceinline__ int unit_rows(const Params& p, int e) {
  // (not through the read-only path: the launch before this one may write lengths while this one is resident already)
  const int n = p.seq_lens[(size_t)p.layer_begin * p.batch + e];
  return min(max(n, 0), p.max_pages_per_seq * p.page_size);
}
template <int D>
__device__ __forceinline__ int tiles_of(int rows) {
  constexpr int kTile = Cfg<D>::kTile;
  return (rows + kTile - 1) / kTile;
}
// length of a cache on the line
template <int D>
__device__ __forceinline__ int cost_of(int rows) {
  return rows > 0 ? tiles_of<D>(rows) * Cfg<D>::kTileBlocks + kCacheCost : 0;
}

// Caches that this CTA has found complete and is to join.
struct Joins {
  int4 job[kJobs];                    // {unit, KV head, first CTA, pieces}
  int n_jobs, claimed;                // jobs so far, heads claimed
  int all;                            // no more jobs to come
};

// Joins kHeads query heads from g on (those behind the last one are left out) of a cut cache, kPieces pieces at a time,
// all loads of a batch in flight together; the lanes share the columns.
template <int D, int kHeads, int kPieces>
__device__ __forceinline__ void join_heads(const Params& p, const int4 job, int g) {
  constexpr int kCols = D / 32;
  const int lane = threadIdx.x & 31, G = p.group;
  const float2* ml_at = reinterpret_cast<const float2*>(p.part_ml);
  const float* o_at = p.part_o + lane * kCols;
  float mx[kHeads], den[kHeads], o[kHeads][kCols];
#pragma unroll
  for (int x = 0; x < kHeads; ++x) {
    mx[x] = -INFINITY;
    den[x] = 0.f;
#pragma unroll
    for (int c = 0; c < kCols; ++c) o[x][c] = 0.f;
  }
#pragma unroll 1
  for (int i0 = 0; i0 < job.w; i0 += kPieces) {
    const int nb = min(kPieces, job.w - i0);
    // Row of (piece i of the batch, head g + x).  Rounds past the last piece or head read that one: loads under a
    // condition would be taken one after the other.
    auto row_of = [&](int i, int x) -> int {
      i = i0 + min(i, nb - 1);
      return (2 * (job.z + i) + (i == 0 ? 1 : 0)) * G + min(g + x, G - 1);
    };
    float2 ml[kHeads];
    float v[kHeads][kPieces][kCols];
#pragma unroll
    for (int x = 0; x < kHeads; ++x) ml[x] = __ldcg(ml_at + row_of(lane, x));
#pragma unroll
    for (int x = 0; x < kHeads; ++x)
#pragma unroll
      for (int k = 0; k < kPieces; ++k) {
        const float* src = o_at + (size_t)row_of(k, x) * D;
        if constexpr (kCols == 4) {
          const float4 q = __ldcg(reinterpret_cast<const float4*>(src));
          v[x][k][0] = q.x, v[x][k][1] = q.y, v[x][k][2] = q.z, v[x][k][3] = q.w;
        } else {
          const float2 q = __ldcg(reinterpret_cast<const float2*>(src));
          v[x][k][0] = q.x, v[x][k][1] = q.y;
        }
      }
#pragma unroll
    for (int x = 0; x < kHeads; ++x) {
      const float mn = fmaxf(mx[x], warp_max(ml[x].x));
      const float al = fast_exp2(mx[x] - mn), wgt = lane < nb ? fast_exp2(ml[x].x - mn) : 0.f;
      float ds = wgt * ml[x].y;
#pragma unroll
      for (int y = 16; y > 0; y >>= 1) ds += __shfl_xor_sync(0xffffffffu, ds, y);
      den[x] = fmaf(den[x], al, ds);
      mx[x] = mn;
#pragma unroll
      for (int c = 0; c < kCols; ++c) o[x][c] *= al;
#pragma unroll
      for (int k = 0; k < kPieces; ++k) {
        const float wk = __shfl_sync(0xffffffffu, wgt, k);
#pragma unroll
        for (int c = 0; c < kCols; ++c) o[x][c] = k < nb ? fmaf(wk, v[x][k][c], o[x][c]) : o[x][c];
      }
    }
  }
#pragma unroll
  for (int x = 0; x < kHeads; ++x) {
    if (g + x >= G) break;
    const size_t row = (size_t)job.x * p.n_q_heads + (size_t)job.y * G + g + x;
    const float inv = __frcp_rn(den[x]);
#pragma unroll
    for (int c = 0; c < kCols; c += 2)
      *reinterpret_cast<uint32_t*>(p.out + row * D + lane * kCols + c) = pack_bf16(o[x][c] * inv, o[x][c + 1] * inv);
    if (lane == 0 && p.lse != nullptr) p.lse[row] = (mx[x] + __log2f(den[x])) * 0.6931471805599453f;
  }
}

// Takes query heads of open jobs, up to four of one job at a time, until none is left (a whole warp).
template <int D>
__device__ __noinline__ void join_open(const Params& p, Joins* joins) {
  const int lane = threadIdx.x & 31, G = p.group;
#pragma unroll 1
  while (true) {
    int claim = -1, n = 0;
    if (lane == 0) {
      int at = *(volatile int*)&joins->claimed;
      const int open = *(volatile int*)&joins->n_jobs * G;
      __threadfence_block();                      // n_jobs before the jobs and, behind them, the pieces
      while (at < open) {
        // few pieces: four heads in one go; many: one head a warp, so that several warps share the job
        n = joins->job[at / G].w <= 4 ? min(4, G - at % G) : 1;
        const int was = atomicCAS(&joins->claimed, at, at + n);
        if (was == at) {
          claim = at;
          break;
        }
        at = was;
      }
    }
    claim = __shfl_sync(0xffffffffu, claim, 0);
    if (claim < 0) return;
    n = __shfl_sync(0xffffffffu, n, 0);
    __syncwarp();                                 // what lane 0 has seen, all lanes see
    const int4 job = joins->job[claim / G];
    if (job.w <= 4) join_heads<D, 4, 4>(p, job, claim % G);
    else            join_heads<D, 1, 16>(p, job, claim % G);
  }
}

template <int D, int GP>              // GP: query heads per KV head, rounded up to a power of two
__global__ void __launch_bounds__(kThreads, kCtasPerSm)
decode_e4m3_kernel(const __grid_constant__ CUtensorMap tmap_k, const __grid_constant__ CUtensorMap tmap_v,
                   const __grid_constant__ Params p) {
  using C = Cfg<D>;
  constexpr int kTile = C::kTile, kTileBlocks = C::kTileBlocks;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  __shared__ uint64_t s_k_full[C::kStages], s_k_empty[C::kStages], s_v_full[C::kStages], s_v_empty[C::kStages],
      s_scale_full[C::kStages], s_s_full[2], s_p_full[2], s_d_full[2], s_fifo_full[kFifo], s_fifo_empty[kFifo],
      s_q_full[kFifo], s_done_full[kFifo], s_wake;
  __shared__ Item s_item[kFifo];
  __shared__ __align__(16) float s_qscale[kFifo][8];              // heads from G on are never read for a result
  __shared__ __align__(16) float s_max[2][4][8];
  __shared__ __align__(16) float s_head[4][3][8];
  __shared__ __align__(16) float s_sum[2][16];    // reciprocal denominators, or (one or two heads) the warps' sums from [8] on
  __shared__ int s_scan[kThreads / 32];
  __shared__ int4 s_first;                        // the unit in which the share begins: unit, rows, where it begins on the line
  __shared__ int4 s_end_cut;                      // the cache that the share's end cuts: unit, KV head, where it begins, rows
  __shared__ uint32_t s_tmem;
  __shared__ int s_abort_store;
  __shared__ Joins s_joins;
  volatile int* s_abort = &s_abort_store;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int Hkv = p.n_kv_heads, G = p.group;

  if (p.wait_first) grid_dependency_wait();
  // ---- the plan: each thread a run of units, and their length on the line
  const int per = (p.n_units + kThreads - 1) / kThreads;
  int mine = 0;
#pragma unroll 8
  for (int i = 0; i < per; ++i) {
    const int e = tid * per + i;
    if (e < p.n_units) mine += cost_of<D>(unit_rows(p, e));
  }
  if (tid == 0) {
    for (int i = 0; i < C::kStages; ++i) {
      mbar_init(&s_k_full[i], 1);
      mbar_init(&s_k_empty[i], 1);
      mbar_init(&s_v_full[i], 1);
      mbar_init(&s_v_empty[i], 1);
      mbar_init(&s_scale_full[i], 32);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(&s_s_full[i], 1);
      mbar_init(&s_p_full[i], 4);
      mbar_init(&s_d_full[i], 1);
    }
    for (int i = 0; i < kFifo; ++i) {
      mbar_init(&s_fifo_full[i], 1);
      mbar_init(&s_fifo_empty[i], 7);             // copies, logit MMAs, four softmax warps, warp 7
      mbar_init(&s_q_full[i], 1);
      mbar_init(&s_done_full[i], 4);
    }
    mbar_init(&s_wake, 1);
    s_abort_store = 0;
    s_joins.n_jobs = s_joins.claimed = s_joins.all = 0;
    fence_mbar_init();
    prefetch_tmap(&tmap_k);
    prefetch_tmap(&tmap_v);
  }
  if (warp == 5) {
    tmem_alloc(&s_tmem, C::kTmemCols);
    tmem_relinquish();
  }
  // operand rows that no head fills stay zero
#pragma unroll 1
  for (int i = tid; i < (kFifo * C::kQBytes + 2 * C::kPBytes) / 16; i += kThreads)
    reinterpret_cast<uint4*>(smem + C::kOffQ)[i] = make_uint4(0u, 0u, 0u, 0u);
  fence_proxy_async_smem();

  int incl = mine;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int x = __shfl_up_sync(0xffffffffu, incl, o);
    if (lane >= o) incl += x;
  }
  if (lane == 31) s_scan[warp] = incl;
  tc_fence_before_sync();
  __syncthreads();
  tc_fence_after_sync();
  int line = 0, before = incl - mine;
#pragma unroll
  for (int w = 0; w < kThreads / 32; ++w) {
    if (w < warp) before += s_scan[w];
    line += s_scan[w];
  }
  line *= Hkv;
  const int n_ctas = min(min((int)gridDim.x, p.max_ctas), max(line / C::kMinSegment, 1));
  const Cut share(line, n_ctas);
  const bool works = (int)blockIdx.x < n_ctas && line > 0;
  const int begin = works ? share.begin(blockIdx.x) : 0, stop_at = works ? share.begin(blockIdx.x + 1) : 0;
  const int my_begin = before * Hkv, my_end = (before + mine) * Hkv;
  if (works && my_begin < my_end && ((my_begin <= begin && begin < my_end) || (my_begin <= stop_at && stop_at < my_end))) {
    int at = my_begin;                            // this thread's run of units holds the begin or the end of the share
#pragma unroll 1
    for (int i = 0; i < per; ++i) {
      const int e = tid * per + i, rows = e < p.n_units ? unit_rows(p, e) : 0, cost = cost_of<D>(rows), next = at + cost * Hkv;
      if (at <= begin && begin < next) s_first = make_int4(e, rows, at, 0);
      if (at <= stop_at && stop_at < next) {
        const int h = quotient(stop_at - at, cost), g0 = at + h * cost;
        // cut: some of its tiles start before the end, others behind it (and none in the piece that the begin cuts)
        const bool cut = g0 > begin && g0 < stop_at && stop_at - g0 <= (tiles_of<D>(rows) - 1) * kTileBlocks;
        s_end_cut = make_int4(e, h, g0, cut ? rows : 0);
      }
      at = next;
    }
  }
  if (tid == 0 && (!works || stop_at >= line)) s_end_cut = make_int4(0, 0, 0, 0);
  __syncthreads();
  const uint32_t tmem = s_tmem;

  if (warp == 4) {
    // ================================================================ the copies
    const int R = p.box_rows, boxes_per_tile = kTile >> p.box_shift;
    // page of box `lane` of a batch of 32 boxes of an item
    auto load_pages = [&](const Item& it, int box0) -> int {
      const int r = it.row0 + (box0 + lane) * R;
      int page = 0;
      if (it.e >= 0 && r < it.row0 + it.rows)
        page = __ldg(&p.block_table[((size_t)p.layer_begin * p.batch + it.e) * p.max_pages_per_seq + p.page_of(r)]);
      return page;
    };
    uint32_t j = 0;                               // tiles issued
    Item nxt = {-1, 0, 0, 0, 0, 0};
    // Page ids of the share's first tile, on their way before the first item is known: it begins in this unit (unless no
    // tile starts there any more).
    Item guess = {-1, 0, 0, 0, 0, 0};
    if (works) {
      guess.e = s_first.x;
      const int cost = cost_of<D>(s_first.y), off = begin - s_first.z;
      guess.row0 = (off - quotient(off, cost) * cost + kTileBlocks - 1) / kTileBlocks * kTile;
      guess.rows = s_first.y - guess.row0;
      if (s_end_cut.w > 0) {
        guess.e = s_end_cut.x;
        guess.row0 = 0;
        guess.rows = s_end_cut.w;
      }
    }
    const int guess_pages = load_pages(guess, 0);
    int nxt_pages = 0;
    bool have_next = false, ok = true;
#pragma unroll 1
    for (uint32_t n_item = 0; ok; ++n_item) {
      const int slot = n_item % kFifo;
      if (!have_next) {
        ok = __all_sync(0xffffffffu, wait_bar(&s_fifo_full[slot], (n_item / kFifo) & 1, s_abort, p.wait_ns));
        if (!ok) break;
        nxt = s_item[slot];
        nxt_pages = n_item == 0 && nxt.e == guess.e && nxt.row0 == guess.row0 ? guess_pages : load_pages(nxt, 0);
      }
      const Item cur = nxt;
      if (cur.e < 0 || (int)blockIdx.x == p.withhold_cta) break;
      int pages = nxt_pages, ahead = 0;
      have_next = false;
      const int n_tiles = tiles_of<D>(cur.rows);
#pragma unroll 1
      for (int t = 0; t < n_tiles; ++t, ++j) {
        const int box0 = t * boxes_per_tile;
        if ((box0 & 31) == 0) {                   // a new batch of page ids; the next one is on its way meanwhile
          if (t > 0) pages = ahead;
          ahead = load_pages(cur, box0 + 32);
        }
        const int stage = j % C::kStages;
        const uint32_t ph = ((j / C::kStages) - 1) & 1;
        const int left = min(kTile, cur.rows - t * kTile);
        const int n_box = (left + R - 1) >> p.box_shift, n_blk = (left + kScaleBlock - 1) / kScaleBlock;
        // first row of this lane's box in the page pool (lanes past the last box: not used)
        const int row_of_box = cur.row0 + t * kTile + lane * R;
        int page = __shfl_sync(0xffffffffu, pages, (box0 + lane) & 31);
        page = min(max(page, 0), p.n_pages - 1);
        const int grow = (page * Hkv + cur.h - p.page_of(row_of_box)) * p.page_size + row_of_box;
        if (j >= C::kStages) ok = wait_bar(&s_k_empty[stage], ph, s_abort, p.wait_ns);
        ok = __all_sync(0xffffffffu, ok);
        if (!ok) break;
        if (lane == 0) mbar_arrive_expect_tx(&s_k_full[stage], (uint32_t)(n_box * R * D));
        __syncwarp();
        if (lane < n_box)
          tma_load_2d(smem + stage * C::kTileBytes + lane * R * D, &tmap_k, 0, grow, &s_k_full[stage]);
        if (j >= C::kStages) ok = wait_bar(&s_v_empty[stage], ph, s_abort, p.wait_ns);
        ok = __all_sync(0xffffffffu, ok);
        if (!ok) break;
        if (lane == 0) mbar_arrive_expect_tx(&s_v_full[stage], (uint32_t)(n_box * R * D));
        __syncwarp();
        if (lane < n_box)
          tma_load_2d(smem + C::kOffV + stage * C::kTileBytes + lane * R * D, &tmap_v, 0, grow, &s_v_full[stage]);
        {
          // the first lanes: scales of the tile's blocks of K rows, the next ones: of V rows
          const int blk = lane % kTileBlocks;
          const int in_box = (blk * kScaleBlock) >> p.box_shift;
          int bg = __shfl_sync(0xffffffffu, grow, in_box);
          bg = bg / kScaleBlock + blk - (in_box << p.box_shift) / kScaleBlock;
          if (lane < 2 * kTileBlocks) {
            const bool live = blk < n_blk;
            float* dst = reinterpret_cast<float*>(smem + C::kOffScales) + stage * 2 * kTileBlocks + lane;
            cp_async_4(dst, (lane < kTileBlocks ? p.k_scales : p.v_scales) + (live ? bg : 0), live);
          }
          cp_async_arrive(&s_scale_full[stage]);
        }
        if (!have_next) {                         // the next item's first page ids, if that item is known already
          const int ns = (n_item + 1) % kFifo;
          if (__all_sync(0xffffffffu, mbar_test(&s_fifo_full[ns], ((n_item + 1) / kFifo) & 1))) {
            nxt = s_item[ns];
            nxt_pages = load_pages(nxt, 0);
            have_next = true;
          }
        }
      }
      if (!ok) break;
      __syncwarp();
      if (lane == 0) mbar_arrive(&s_fifo_empty[slot]);
    }
  } else if (warp == 5) {
    // ================================================================ the MMAs
    // The whole warp walks, one elected lane issues: a branch on elect.sync costs 49 clocks an MMA, one on the lane
    // index 78 (measured, whatever the shape; the 128 x 16 x 32 product itself takes 42).
    constexpr uint32_t kIdescS = idesc_e4m3(128, kN, false), kIdescO = idesc_e4m3(D, kN, true);
    uint32_t js = 0, jo = 0, n_item = 0;          // logit tiles issued, output tiles issued, items begun
    int slot = 0, t = 0, n_tiles = 0, last_rows = 0;   // of the logits
    int rows0 = kTile, rows1 = kTile;             // rows of the even and the odd tile between the two products
    bool more = true;
#pragma unroll 1
    while (true) {
      if (more && js - jo < 2) {
        if (t == n_tiles) {                       // next item
          slot = n_item % kFifo;
          if (!__all_sync(0xffffffffu, wait_bar(&s_fifo_full[slot], (n_item / kFifo) & 1, s_abort, p.wait_ns))) break;
          const int e = s_item[slot].e, rows = s_item[slot].rows;
          if (e < 0) {
            more = false;
            continue;
          }
          if (!__all_sync(0xffffffffu, wait_bar(&s_q_full[slot], (n_item / kFifo) & 1, s_abort, p.wait_ns))) break;
          ++n_item;
          t = 0;
          n_tiles = tiles_of<D>(rows);
          last_rows = rows - (n_tiles - 1) * kTile;
        }
        const int stage = js % C::kStages;
        if (!__all_sync(0xffffffffu, wait_bar(&s_k_full[stage], (js / C::kStages) & 1, s_abort, p.wait_ns))) break;
        tc_fence_after_sync();
        ++t;
        const bool last = t == n_tiles;
        if (elect_one()) {
          const uint64_t a = smem_desc<D>(smem_u32(smem + stage * C::kTileBytes));
          const uint64_t b = smem_desc<D>(smem_u32(smem + C::kOffQ + slot * C::kQBytes));
          const uint32_t d = tmem + (js & 1) * C::kSpans * kN;
#pragma unroll
          for (int x = 0; x < C::kSpans; ++x)
            if (x == 0 || !last || last_rows > 128 * x)
#pragma unroll
              for (int k = 0; k < D / 32; ++k) umma_e4m3(d + x * kN, a + x * (128 * D / 16) + 2 * k, b + 2 * k, kIdescS, k > 0);
          umma_commit(&s_s_full[js & 1]);
          umma_commit(&s_k_empty[stage]);
          if (last) umma_commit(&s_fifo_empty[slot]);
        }
        __syncwarp();
        if (js & 1) rows1 = last ? last_rows : kTile;
        else        rows0 = last ? last_rows : kTile;
        ++js;
      } else if (jo < js) {
        const int stage = jo % C::kStages;
        if (!__all_sync(0xffffffffu, wait_bar(&s_v_full[stage], (jo / C::kStages) & 1, s_abort, p.wait_ns) &&
                                         wait_bar(&s_p_full[jo & 1], (jo / 2) & 1, s_abort, p.wait_ns)))
          break;
        tc_fence_after_sync();
        const int rows = (jo & 1) ? rows1 : rows0;
        if (elect_one()) {
          const uint64_t a = smem_desc<D>(smem_u32(smem + C::kOffV + stage * C::kTileBytes));
          const uint64_t b = smem_desc_rows16(smem_u32(smem + C::kOffP + (jo & 1) * C::kPBytes));
          const uint32_t d = tmem + (2 * C::kSpans + (jo & 1)) * kN;
#pragma unroll
          for (int k = 0; k < kTile / 32; ++k)    // whole groups of 32 rows; those behind the last row stay out
            if (32 * k < rows) umma_e4m3(d, a + 2 * D * k, b + 32 * k, kIdescO, k > 0);
          umma_commit(&s_d_full[jo & 1]);
          umma_commit(&s_v_empty[stage]);
        }
        __syncwarp();
        ++jo;
      } else {
        break;                                    // no more logits, every output issued
      }
    }
  } else if (warp == 6) {
    // ================================================================ the walk, and the queries as two codes per element
    int at = begin;                               // next position of the share
    int e = s_first.x, rows = s_first.y, unit_at = s_first.z;      // unit_at: where (e, head 0) begins
    int cost = cost_of<D>(rows), h = works ? quotient(begin - unit_at, cost) : 0;
    // The piece that the end of the share cuts comes first, then the one that its begin cuts, then the whole caches: counting
    // and joining pieces takes microseconds, which then lie under the copies of what follows.
    const int walk_end = s_end_cut.w > 0 ? s_end_cut.z : stop_at;
    bool end_first = s_end_cut.w > 0;
    // The next piece: the tiles of (e, h) that start in [at, walk_end).
    auto next_item = [&]() -> Item {
      Item it = {-1, 0, 0, 0, 0, 0};
      if (end_first) {
        end_first = false;
        const int g0 = s_end_cut.z;
        it.e = s_end_cut.x;
        it.h = s_end_cut.y;
        it.rows = (stop_at - g0 + kTileBlocks - 1) / kTileBlocks * kTile;
        it.first_cta = (int)blockIdx.x;
        it.n_pieces = share.part_of(g0 + (tiles_of<D>(s_end_cut.w) - 1) * kTileBlocks) - it.first_cta + 1;
        return it;
      }
#pragma unroll 1
      while (at < walk_end) {
#pragma unroll 1
        while (h == Hkv || rows == 0) {           // on to the next cache that holds rows
          unit_at += cost * Hkv;
          ++e;
          h = 0;
          if (e >= p.n_units) return it;
          rows = unit_rows(p, e);
          cost = cost_of<D>(rows);
        }
        const int g0 = unit_at + h * cost, nt = tiles_of<D>(rows);
        const int t0 = (at - g0 + kTileBlocks - 1) / kTileBlocks;                       // first tile that starts at or behind `at`
        const int t1 = min(nt, (min(walk_end, g0 + cost) - g0 + kTileBlocks - 1) / kTileBlocks);   // first one behind the piece
        const int this_h = h;
        at = min(walk_end, g0 + cost);
        if (at == g0 + cost) ++h;
        if (t0 >= t1) continue;                   // no tile starts here
        it.e = e;
        it.h = this_h;
        it.row0 = t0 * kTile;
        it.rows = min(rows, t1 * kTile) - it.row0;
        const bool whole = t0 == 0 && t1 == nt;
        it.first_cta = whole ? (int)blockIdx.x : share.part_of(g0);
        it.n_pieces = whole ? 1 : share.part_of(g0 + (nt - 1) * kTileBlocks) - it.first_cta + 1;
        return it;
      }
      return it;
    };
#pragma unroll 1
    for (uint32_t n_item = 0;; ++n_item) {
      const int slot = n_item % kFifo;
      const Item it = next_item();
      if (n_item >= kFifo &&
          !__all_sync(0xffffffffu, wait_bar(&s_fifo_empty[slot], ((n_item / kFifo) - 1) & 1, s_abort, p.wait_ns)))
        break;
      if (lane == 0) {
        s_item[slot] = it;
        mbar_arrive(&s_fifo_full[slot]);
      }
      if (it.e < 0) break;
      // D / 16 lanes a head, sixteen elements a lane, as many heads at a time as the warp holds
      constexpr int kLanes = D / 16, kHeads = 32 / kLanes, kPasses = (GP + kHeads - 1) / kHeads;
      const int c = lane % kLanes;
      const __nv_bfloat16* q = p.q + ((size_t)it.e * p.n_q_heads + (size_t)it.h * G) * D + c * 16;
      uint8_t* dst = smem + C::kOffQ + slot * C::kQBytes;
      uint4 raw[kPasses][2];
#pragma unroll
      for (int x = 0; x < kPasses; ++x) {
        const int g = min(x * kHeads + lane / kLanes, G - 1);
        raw[x][0] = __ldg(reinterpret_cast<const uint4*>(q + (size_t)g * D));
        raw[x][1] = __ldg(reinterpret_cast<const uint4*>(q + (size_t)g * D) + 1);
      }
#pragma unroll
      for (int x = 0; x < kPasses; ++x) {
        const int g = x * kHeads + lane / kLanes;
        const uint32_t v[8] = {raw[x][0].x, raw[x][0].y, raw[x][0].z, raw[x][0].w,
                               raw[x][1].x, raw[x][1].y, raw[x][1].z, raw[x][1].w};
        uint32_t top = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) top = __vmaxu2(top, v[i] & 0x7fff7fffu);
        top = max(top & 0xffffu, top >> 16);
#pragma unroll
        for (int o = 1; o < kLanes; o <<= 1) top = max(top, __shfl_xor_sync(0xffffffffu, top, o));
        const bool bad = top >= 0x7f80u;                       // an infinity or NaN in the row: every code a NaN
        const int ex = min(max((int)(top >> 7), 20), 254);     // exponent field; largest element in [128, 256) after scaling
        const __nv_bfloat162 inv = __float2bfloat162_rn(__uint_as_float((uint32_t)(261 - ex) << 23));
        uint32_t c1[4], c2[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          uint32_t a[2], b[2];
#pragma unroll
          for (int k = 0; k < 2; ++k) {
            const uint32_t y = bf16x2_scale(v[2 * i + k], inv);
            const float lo = bf16_lo(y), hi = bf16_hi(y);
            a[k] = e4m3x2_from_f32(lo, hi);
            const float2 f = f32_from_e4m3x2(a[k]);
            b[k] = e4m3x2_from_f32((lo - f.x) * kPart, (hi - f.y) * kPart);
          }
          c1[i] = bad ? 0x7f7f7f7fu : __byte_perm(a[0], a[1], 0x5410);
          c2[i] = bad ? 0x7f7f7f7fu : __byte_perm(b[0], b[1], 0x5410);
        }
        if (g < G) {
          *reinterpret_cast<uint4*>(dst + swizzled<D>(g, c * 16)) = make_uint4(c1[0], c1[1], c1[2], c1[3]);
          *reinterpret_cast<uint4*>(dst + swizzled<D>(GP + g, c * 16)) = make_uint4(c2[0], c2[1], c2[2], c2[3]);
          if (c == 0) s_qscale[slot][g] = __uint_as_float((uint32_t)(ex - 7) << 23) * p.scale_log2;
        }
      }
      fence_proxy_async_smem();
      __syncwarp();
      if (lane == 0) mbar_arrive(&s_q_full[slot]);
    }
  } else if (warp == 7) {
    // ================================================================ finished pieces of cut caches
    bool woken = false;                           // warps that are out of tiles wait for the first job or for the end
    // first the rows of empty caches
#pragma unroll 1
    for (int e = blockIdx.x; e < p.n_units; e += gridDim.x) {
      if (unit_rows(p, e) != 0) continue;
      const size_t row0 = (size_t)e * p.n_q_heads;
#pragma unroll 1
      for (int i = lane; i < p.n_q_heads * D / 8; i += 32)
        reinterpret_cast<uint4*>(p.out + row0 * D)[i] = make_uint4(0u, 0u, 0u, 0u);
      if (p.lse != nullptr)
#pragma unroll 1
        for (int i = lane; i < p.n_q_heads; i += 32) p.lse[row0 + i] = -INFINITY;
    }
    if (!p.wait_first) grid_dependency_wait();    // the tickets are cleared by the launch before this one
#pragma unroll 1
    for (uint32_t n_item = 0;; ++n_item) {
      const int slot = n_item % kFifo;
      if (!__all_sync(0xffffffffu, wait_bar(&s_fifo_full[slot], (n_item / kFifo) & 1, s_abort, p.wait_ns))) break;
      const Item it = s_item[slot];
      if (it.e < 0) break;
      if (!__all_sync(0xffffffffu, wait_bar(&s_done_full[slot], (n_item / kFifo) & 1, s_abort, p.wait_ns))) break;
      __syncwarp();
      if (lane == 0) mbar_arrive(&s_fifo_empty[slot]);
      if (it.n_pieces == 1) continue;
      int last = 0;
      if (lane == 0) {
        // counted once it is visible; whoever counts the last one sees all
        last = add_acq_rel(&p.tickets[(size_t)it.e * Hkv + it.h], 1) == it.n_pieces - 1;
      }
      if (__shfl_sync(0xffffffffu, last, 0)) {
        const int n = *(volatile int*)&s_joins.n_jobs;
        if (lane == 0) {
          s_joins.job[n] = make_int4(it.e, it.h, it.first_cta, it.n_pieces);
          __threadfence_block();
          *(volatile int*)&s_joins.n_jobs = n + 1;
          if (!woken) mbar_arrive(&s_wake);
        }
        woken = true;
        __syncwarp();
        join_open<D>(p, &s_joins);
      }
    }
    if (lane == 0) {
      *(volatile int*)&s_joins.all = 1;
      if (!woken) mbar_arrive(&s_wake);
    }
  } else {
    // ================================================================ softmax and output
    const uint32_t lane_base = (uint32_t)warp << 21;            // tensor-memory lanes 32 * warp ..
    const bool holds_col = D == 128 || lane < 16;               // M = 64 accumulators lie in lanes 0-15 of each quarter
    const int col = D == 128 ? warp * 32 + lane : warp * 16 + lane;
    const int blk = tid / kScaleBlock;
    uint32_t j = 0;                                              // tiles begun
#pragma unroll 1
    for (uint32_t n_item = 0;; ++n_item) {
      const int slot = n_item % kFifo;
      bool bad = !wait_bar(&s_fifo_full[slot], (n_item / kFifo) & 1, s_abort, p.wait_ns);
      if (!bad) bad = *s_abort != 0;
      if (soft_any(bad)) break;
      const Item it = s_item[slot];
      if (it.e < 0) break;
      // From here to the end of the item every thread takes every barrier, also when a wait has expired.
      wait_bar(&s_q_full[slot], (n_item / kFifo) & 1, s_abort, p.wait_ns);
      float qs[GP], l[GP], acc[GP], f[GP];
      float m[GP];                                               // four heads and more: m[0] of lane g is that of head g
#pragma unroll
      for (int g = 0; g < GP; ++g) {
        m[g] = -INFINITY;
        l[g] = acc[g] = f[g] = 0.f;
      }
      get_heads<GP>(s_qscale[slot], qs);
      auto add_output = [&](uint32_t jd) {                       // O of tile jd
        wait_bar(&s_d_full[jd & 1], (jd / 2) & 1, s_abort, p.wait_ns);
        tc_fence_after_sync();
        float d[2 * GP];
        tmem_ld<2 * GP>(tmem + (2 * C::kSpans + (jd & 1)) * kN + lane_base, d);
#pragma unroll
        for (int g = 0; g < GP; ++g) acc[g] = fmaf(fmaf(d[GP + g], 1.f / kPart, d[g]), f[g], acc[g]);
      };
      const int n_tiles = tiles_of<D>(it.rows);
#pragma unroll 1
      for (int t = 0; t < n_tiles; ++t, ++j) {
        const int stage = j % C::kStages;
        const int left = it.rows - t * kTile;
        wait_bar(&s_scale_full[stage], (j / C::kStages) & 1, s_abort, p.wait_ns);
        const float* sc = reinterpret_cast<const float*>(smem + C::kOffScales) + stage * 2 * kTileBlocks;
        const float vmax = fmaxf(warp_max(sc[kTileBlocks + lane % kTileBlocks]), 0x1p-110f);
        const float inv_vmax = fast_rcp(vmax);
        wait_bar(&s_s_full[j & 1], (j / 2) & 1, s_abort, p.wait_ns);
        tc_fence_after_sync();
        float s[C::kSpans][GP], mt[GP];                           // logits, then weights, of rows tid and tid + 128; the reference
#pragma unroll
        for (int x = 0; x < C::kSpans; ++x) {
          const bool live = x * 128 + tid < left;
          if (x == 0 || left > 128 * x) {
            float r[2 * GP];
            tmem_ld<2 * GP>(tmem + ((j & 1) * C::kSpans + x) * kN + lane_base, r);
            const float ks = sc[x * 8 + blk];
            const float share = fmaxf(__log2f(sc[kTileBlocks + x * 8 + blk] * inv_vmax), kMinShare);
#pragma unroll
            for (int g = 0; g < GP; ++g) {
              s[x][g] = fmaf(r[GP + g], 1.f / kPart, r[g]) * (ks * qs[g]);
              if (!live) s[x][g] = -INFINITY;
              mt[g] = x == 0 ? s[x][g] + share : fmaxf(mt[g], s[x][g] + share);
            }
          } else {
#pragma unroll
            for (int g = 0; g < GP; ++g) s[x][g] = -INFINITY;
          }
        }
        // (heads from G on: no maximum, weight 0, codes 0; a branch a pair of heads would keep the codes of all pairs apart,
        // 106 against 103 us for 7168 caches with G = 7)
#pragma unroll
        for (int g = 0; g < GP; ++g) mt[g] = g < G ? warp_max(mt[g]) : 0.f;
        if (lane == 0) put_heads<GP>(s_max[j & 1][warp], mt);
        named_bar_sync(kBarSoft, kSoftThreads);
        // The tile's reference of a head, and how the running sums move to the new running reference, the largest so far: for
        // four heads and more lane g works for head g and hands the results round (the same arithmetic in every thread is six
        // times the code).
        bool grows_any;                                           // the running reference of some head has grown
        if constexpr (GP >= 4) {
          bool grows = false;
          if (lane < GP) {
            const float top = fmaxf(fmaxf(s_max[j & 1][0][lane], s_max[j & 1][1][lane]),
                                    fmaxf(s_max[j & 1][2][lane], s_max[j & 1][3][lane]));
            const float up = top - m[0];                          // +inf at the first tile
            grows = up > 0.f;
            const float ex = fast_exp2(grows ? -up : up);
            m[0] = grows ? top : m[0];
            s_head[warp][0][lane] = top;
            s_head[warp][1][lane] = grows ? ex : 1.f;             // what the sums so far are multiplied by
            s_head[warp][2][lane] = grows ? 1.f : ex;             // and the tile's
          }
          grows_any = __any_sync(0xffffffffu, grows);
          __syncwarp();                                           // the stores before the loads below
          get_heads<GP>(s_head[warp][0], mt);
        } else {
#pragma unroll
          for (int g = 0; g < GP; ++g)
            mt[g] = fmaxf(fmaxf(s_max[j & 1][0][g], s_max[j & 1][1][g]), fmaxf(s_max[j & 1][2][g], s_max[j & 1][3][g]));
          grows_any = true;
        }
        // weights relative to the tile's reference; the codes also carry the V scale relative to the tile's largest
        uint8_t* pb = smem + C::kOffP + (j & 1) * C::kPBytes;
        float w[GP];                                              // sum of the weights of this thread's rows
#pragma unroll
        for (int x = 0; x < C::kSpans; ++x) {
          if (x > 0 && left <= 128 * x) break;                    // the output's product does not reach this span
          const float vr = sc[kTileBlocks + x * 8 + blk] * inv_vmax * 256.f;
#pragma unroll
          for (int g = 0; g < GP; ++g) {
            s[x][g] = g < G ? fast_exp2(s[x][g] - mt[g]) : 0.f;
            w[g] = x == 0 ? s[x][g] : w[g] + s[x][g];
          }
          uint32_t c[GP < 4 ? 2 : GP / 2] = {};                   // pairs of first codes, then of second codes
#pragma unroll
          for (int g = 0; g < GP; g += 2) {
            const float a = s[x][g] * vr, b = GP > 1 ? s[x][g + (GP > 1)] * vr : 0.f;
            const uint32_t c1 = e4m3x2_from_f32(a, b);
            const float2 y = f32_from_e4m3x2(c1);
            const uint32_t c2 = e4m3x2_from_f32((a - y.x) * kPart, (b - y.y) * kPart);
            if constexpr (GP < 4) {
              c[0] = c1, c[1] = c2;
            } else {
              c[g / 4] |= c1 << (g % 4 * 8);
              c[GP / 4 + g / 4] |= c2 << (g % 4 * 8);
            }
          }
          uint8_t* row = pb + (x * 128 + tid) * kN;
          if constexpr (GP == 8)      *reinterpret_cast<uint4*>(row) = make_uint4(c[0], c[1], c[2], c[3]);
          else if constexpr (GP == 4) *reinterpret_cast<uint2*>(row) = make_uint2(c[0], c[1]);
          else if constexpr (GP == 2) *reinterpret_cast<uint32_t*>(row) = __byte_perm(c[0], c[1], 0x5410);
          else                        *reinterpret_cast<uint16_t*>(row) = (uint16_t)__byte_perm(c[0], c[1], 0x0040);
        }
        if (left < kTile) {
          // rows behind the last one hold whatever the page or the stage held before; the product runs over whole
          // groups of 32 rows, so clear V there (0 * NaN)
          wait_bar(&s_v_full[stage], (j / C::kStages) & 1, s_abort, p.wait_ns);
          uint4* z = reinterpret_cast<uint4*>(smem + C::kOffV + stage * C::kTileBytes);
#pragma unroll 1
          for (int i = left * (D / 16) + tid; i < (left + 31) / 32 * 32 * (D / 16); i += kSoftThreads)
            z[i] = make_uint4(0u, 0u, 0u, 0u);
        }
        fence_proxy_async_smem();
        tc_fence_before_sync();
        __syncwarp();
        if (lane == 0) mbar_arrive(&s_p_full[j & 1]);
        if (t > 0) add_output(j - 1);
        // on to the new running reference
        if constexpr (GP >= 4) {
          float fw[GP];
          if (grows_any) {
            float al[GP];
            get_heads<GP>(s_head[warp][1], al);
#pragma unroll
            for (int g = 0; g < GP; ++g) {
              l[g] *= al[g];
              acc[g] *= al[g];
            }
          }
          get_heads<GP>(s_head[warp][2], fw);
#pragma unroll
          for (int g = 0; g < GP; ++g) {
            l[g] = fmaf(w[g], fw[g], l[g]);
            f[g] = fw[g] * (vmax * (1.f / 256.f));
          }
        } else {
#pragma unroll
          for (int g = 0; g < GP; ++g) {
            const float up = mt[g] - m[g];                        // +inf at the first tile
            const bool grows = up > 0.f;
            const float ex = fast_exp2(grows ? -up : up);
            const float al = grows ? ex : 1.f, fw = grows ? 1.f : ex;
            l[g] = fmaf(l[g], al, w[g] * fw);
            acc[g] *= al;
            f[g] = fw * (vmax * (1.f / 256.f));
            m[g] = grows ? mt[g] : m[g];
          }
        }
      }
      // ---- denominators over the 128 rows' threads, while the last tile's output is on its way; the thread that has head
      // g's also writes its statistics
      const size_t row0 = (size_t)it.e * p.n_q_heads + (size_t)it.h * G;
      const size_t piece = 2 * (size_t)blockIdx.x + ((int)blockIdx.x == it.first_cta ? 1 : 0);
      auto write_stats = [&](int g, float mg, float lg) {
        if (it.n_pieces > 1) __stcg(reinterpret_cast<float2*>(p.part_ml) + piece * G + g, make_float2(mg, lg));
        else if (p.lse != nullptr && !*s_abort) p.lse[row0 + g] = (mg + __log2f(lg)) * 0.6931471805599453f;
      };
      float* sum_at = s_sum[n_item & 1];
      if constexpr (GP >= 4) {
        // Through shared memory (the weights' buffer that the last tile does not use): 128 / GP threads a head.  (What
        // runs once an item runs out of a cold instruction cache: shuffles of every head take four times the code.)
        constexpr int kPer = 128 / GP, kRow = GP == 8 ? 64 : 128;
        static_assert(GP * kRow * 4 <= C::kPBytes && kRow == 4 * kPer, "fits, four values a thread");
        float* part = reinterpret_cast<float*>(smem + C::kOffP + (j & 1) * C::kPBytes);
        if constexpr (GP == 8) {                                  // each half of a warp takes four heads of both
          const bool upper = lane >= 16;
#pragma unroll
          for (int g = 0; g < 4; ++g) {
            const float theirs = __shfl_xor_sync(0xffffffffu, upper ? l[g] : l[(g + 4) % GP], 16);
            part[(g + (upper ? 4 : 0)) * kRow + warp * 16 + (lane & 15)] = (upper ? l[(g + 4) % GP] : l[g]) + theirs;
          }
        } else {
#pragma unroll
          for (int g = 0; g < GP; ++g) part[g * kRow + tid] = l[g];
        }
        if (lane < GP) s_head[warp][0][lane] = m[0];
        named_bar_sync(kBarSoft, kSoftThreads);
        const int g = tid / kPer;
        const float4 v = *reinterpret_cast<const float4*>(part + 4 * tid);
        float x = (v.x + v.y) + (v.z + v.w);
#pragma unroll
        for (int o = kPer / 2; o > 0; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
        if (tid % kPer == 0 && g < G) {
          sum_at[g] = fast_rcp(x);
          write_stats(g, s_head[warp][0][g], x);
        }
      } else {
#pragma unroll
        for (int g = 0; g < GP; ++g) {
#pragma unroll
          for (int o = 16; o > 0; o >>= 1) l[g] += __shfl_xor_sync(0xffffffffu, l[g], o);
          if (lane == 0) sum_at[8 + 4 * g + warp] = l[g];
        }
      }
      add_output(j - 1);
      const bool drop = *s_abort != 0;
      named_bar_sync(kBarSoft, kSoftThreads);
      if constexpr (GP < 4) {
#pragma unroll
        for (int g = 0; g < GP; ++g) {
          const float4 v = *reinterpret_cast<const float4*>(sum_at + 8 + 4 * g);
          l[g] = (v.x + v.y) + (v.z + v.w);
          if (tid == g) write_stats(g, m[g], l[g]);
        }
      }
      tc_fence_before_sync();
      __syncwarp();
      if (lane == 0) mbar_arrive(&s_fifo_empty[slot]);
      if (it.n_pieces == 1) {
        float inv[GP];
        if constexpr (GP >= 4) {
          get_heads<GP>(sum_at, inv);
        } else {
#pragma unroll
          for (int g = 0; g < GP; ++g) inv[g] = fast_rcp(l[g]);
        }
        if (holds_col && !drop) {
          __nv_bfloat16* o = p.out + row0 * D + col;
#pragma unroll
          for (int g = 0; g < GP; ++g) {
            if (g >= G) break;
            o[g * D] = __float2bfloat16(acc[g] * inv[g]);
          }
        }
      } else if (holds_col) {                                     // a piece; warp 7 counts it
        float* o = p.part_o + piece * G * D + col;
#pragma unroll
        for (int g = 0; g < GP; ++g) {
          if (g >= G) break;
          __stcg(o + g * D, acc[g]);
        }
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(&s_done_full[slot]);
    }
  }
  // ---- out of tiles: help with the joins until warp 7 has counted its last piece
  if (warp != 7) wait_bar(&s_wake, 0, s_abort, p.wait_ns);
#pragma unroll 1
  while (warp != 7) {
    const bool over = __any_sync(0xffffffffu, *(volatile int*)&s_joins.all != 0);   // set on every way out of warp 7's loop
    join_open<D>(p, &s_joins);
    if (over) break;
    __nanosleep(40);
  }
  __syncthreads();
  if (*s_abort) {
    if (tid == 0) record_status(p.hdr, XKV_ERR_TIMEOUT);
    // let copies already issued land before this CTA's shared memory can be handed on
    for (int i = 0; i < 1000; ++i) __nanosleep(1000);
  }
  tc_fence_after_sync();
  if (warp == 5) tmem_dealloc(tmem, C::kTmemCols);
}

bool make_tmap(CUtensorMap* tmap, void* base, int D, uint64_t rows, int box_rows) {
  tc::EncodeTiledFn enc = tc::tc_encode_fn();
  if (enc == nullptr) return false;
  const cuuint64_t dims[2] = {(cuuint64_t)D, (cuuint64_t)rows};
  const cuuint64_t strides[1] = {(cuuint64_t)D};
  const cuuint32_t box[2] = {(cuuint32_t)D, (cuuint32_t)box_rows};
  const cuuint32_t estr[2] = {1u, 1u};
  return enc(tmap, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, base, dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
             D == 128 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
             CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int D, int GP>
xkv_status launch(const CUtensorMap& tk, const CUtensorMap& tv, const Params& p, int grid, cudaStream_t st) {
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return XKV_ERR_CUDA;
  static std::atomic<bool> done[64];   // idempotent set-up: two threads doing it twice is harmless
  if (!done[dev].load(std::memory_order_acquire)) {
    if (cudaFuncSetAttribute(decode_e4m3_kernel<D, GP>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                             Cfg<D>::kSmemBytes) != cudaSuccess)
      return XKV_ERR_CUDA;
    done[dev].store(true, std::memory_order_release);
  }
  cudaEvent_t start, stop;
  get_profile_events(&start, &stop);
  const bool timed = start != nullptr && stop != nullptr;
  if (timed) cudaEventRecord(start, st);
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)grid);
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = Cfg<D>::kSmemBytes;
  cfg.stream = st;
  // its CTAs may start while the launch before (counters cleared, rows appended) is still running
  cudaLaunchAttribute attr;
  attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr.val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = &attr;
  cfg.numAttrs = timed ? 0 : 1;
  const cudaError_t err = cudaLaunchKernelEx(&cfg, decode_e4m3_kernel<D, GP>, tk, tv, p);
  if (timed) cudaEventRecord(stop, st);
  count_launch();
  if (err != cudaSuccess) {
    (void)cudaGetLastError();
    return XKV_ERR_CUDA;
  }
  return check_launch();
}

// Clears the call's counters and tickets.
__global__ void clear_kernel(int32_t* words, int n) {
  asm volatile("griddepcontrol.launch_dependents;");
  for (int i = blockIdx.x * blockDim.x + threadIdx.x; i < n; i += gridDim.x * blockDim.x) words[i] = 0;
}

}  // namespace

xkv_status decode_attn_e4m3(const xkv_dims* d, const xkv_cache* c, int layer_begin, int n_layers, const void* q,
                            const void* k_new, const void* v_new, void* out, float* lse, const DecodeScratch& ws,
                            cudaStream_t st) {
  const int n_units = n_layers * d->batch;
  int box = 16;
  const int tile = d->head_dim == 128 ? Cfg<128>::kTile : Cfg<64>::kTile;
  while (box < tile && c->page_size % (2 * box) == 0) box *= 2;
  const uint64_t page_rows = (uint64_t)c->n_pages * d->n_kv_heads * c->page_size;
  // the line of all caches, as long as their tables allow, has 31-bit places
  const int64_t max_rows = (int64_t)c->max_pages_per_seq * c->page_size;
  const int64_t caches = (int64_t)n_units * d->n_kv_heads, most = caches * ((max_rows + tile - 1) / tile);
  if (caches * ((max_rows + tile) / kScaleBlock + kCacheCost) >= (1ll << 31)) return XKV_ERR_UNSUPPORTED;
  CUtensorMap tk, tv;
  if (!make_tmap(&tk, c->k_pages, d->head_dim, page_rows, box) || !make_tmap(&tv, c->v_pages, d->head_dim, page_rows, box))
    return XKV_ERR_CUDA;
  xkv_status s;
  if (k_new != nullptr) {
    s = append_e4m3(d, c, layer_begin, n_units, k_new, v_new, ws.header, ws.clear, ws.n_clear, st);
  } else {
    const int blocks = (ws.n_clear + 1023) / 1024;
    clear_kernel<<<blocks < 64 ? blocks : 64, 256, 0, st>>>(ws.clear, ws.n_clear);
    count_launch();
    s = check_launch();
  }
  if (s != XKV_OK) return s;
  Params p;
  p.q = static_cast<const __nv_bfloat16*>(q);
  p.out = static_cast<__nv_bfloat16*>(out);
  p.lse = lse;
  p.k_scales = c->k_scales;
  p.v_scales = c->v_scales;
  p.block_table = c->block_table;
  p.seq_lens = c->seq_lens;
  p.layer_begin = layer_begin;
  p.batch = d->batch;
  p.n_units = n_units;
  p.n_q_heads = d->n_q_heads;
  p.n_kv_heads = d->n_kv_heads;
  p.group = d->n_q_heads / d->n_kv_heads;
  p.page_size = c->page_size;
  p.max_pages_per_seq = c->max_pages_per_seq;
  p.n_pages = c->n_pages;
  const uint32_t n8 = (uint32_t)c->page_size / 8;
  p.page_mul = (uint32_t)(((1ull << 32) + n8 - 1) / n8);
  p.box_rows = box;
  p.box_shift = 31 - __builtin_clz((unsigned)box);
  const int64_t room = ws.max_items / 2;
  p.max_ctas = (int32_t)(room < 1 ? 1 : (room < (1 << 20) ? room : 1 << 20));
  p.wait_first = k_new != nullptr ? 1 : 0;
  p.scale_log2 = (d->scale != 0.f ? d->scale : 1.0f / sqrtf((float)d->head_dim)) * 1.4426950408889634f;
  p.withhold_cta = debug_withhold_item();
  p.wait_ns = wait_limit_ns();
  p.hdr = static_cast<WorkspaceHeader*>(ws.header);
  p.tickets = ws.tickets;
  p.part_o = ws.part_o;
  p.part_ml = ws.part_ml;
  // no more CTAs than tiles there can be
  const int64_t full = (int64_t)kCtasPerSm * sm_count();
  const int grid = (int)(most < full ? most : full);
  const int G = p.group;
  if (d->head_dim == 128) {
    if (G == 1) return launch<128, 1>(tk, tv, p, grid, st);
    if (G == 2) return launch<128, 2>(tk, tv, p, grid, st);
    if (G <= 4) return launch<128, 4>(tk, tv, p, grid, st);
    return launch<128, 8>(tk, tv, p, grid, st);
  }
  if (G == 1) return launch<64, 1>(tk, tv, p, grid, st);
  if (G == 2) return launch<64, 2>(tk, tv, p, grid, st);
  if (G <= 4) return launch<64, 4>(tk, tv, p, grid, st);
  return launch<64, 8>(tk, tv, p, grid, st);
}

}  // namespace xkv
