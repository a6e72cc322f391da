// xkv_diff_prefill_attn: causal attention of the whole prompt by heads whose weights are the difference of two softmax maps, on
// the 5th-generation tensor cores.
//
// Mathematics.  A head's query tile is [Q1 | Q2], a KV head's key tile [K1 | K2] (halves of d/2 columns), its values V (d columns):
//   S_s = scale Q_s K_s^T,  P_s = exp(S_s - m_s),  O_s = P_s V,  l_s = row sums of P_s          s = 1, 2
//   y = O_1 / l_1 - lambda O_2 / l_2,  out = y or y / sqrt(mean y^2 + eps) * gain
// The two maps share every K and V tile: one pass over the keys, four products a tile.  Per visible pair and head that is 2 d + 4 d
// flops and two exponentials; for a tile of 128 rows x 64 keys the tensor pipe needs 896 clocks (d = 128; the logits' products read
// both operands from shared memory, which at N = 64 sets their pace), the exponentials 1024 at 16 a clock.
//
// Shape of the launch: one persistent CTA per SM takes (query tile, head) items, long ones first and in alternating direction, so
// that the CTAs' sums differ by little; the heads of a tile lie next to each other, so that a KV head's tiles meet in L2.  Tensor
// memory holds per map O_s (d columns), one 64-column buffer of logits and two 32-column buffers of weights: the next tile's logits
// are formed as soon as this tile's are in registers, so the softmax warps wait for no product.  (Weights over their logits, and
// two such buffers, or one of 128 keys: the chain weights - product - logits is then in the way, 980 and 1010 us for the largest case.)
//   warps 0-3  softmax of map 1, warps 4-7 of map 2: thread = query row = tensor-memory lane.  A row's 64 logits leave tensor memory
//              once; the reference maximum is exact on the first tile and raised lazily (by 2^8) afterwards, which is when O_s is
//              rescaled; P_s goes back as bf16 pairs to one of its two buffers, the A operand of O_s += P_s V.  At the end of an item
//              each map's warps take half of the columns of both O_1 and O_2.
//   warp 8     Q tiles (two buffers, so that the next item's logits start under this item's last products) and K tiles by TMA
//   warps 9, 10   issue the logits of map 1 and of map 2, warps 12, 13 the outputs (a warp of its own each: what runs once a tile runs out
//              of a cold instruction cache, and one warp for both took longer than the softmax); warp 12 clears the V rows
//              behind a prompt's last token (the next prompt's, or 0 * NaN)
//   warp 11    finds the items, V tiles by TMA
// Every wait is bounded and ends when another role has given up; an expired one sets the status word and lets the CTA drain.
//
// Measured (device time, clock under the power limit 1.65 - 1.8 GHz): four prompts of 2399 - 4428 tokens, 32 heads of 128 over 8 KV heads 864
// us = 840 TFLOP/s (773 to 884 from GPU to GPU); one of 32 768 tokens, 8 heads 1020 TFLOP/s; one of 487 tokens, 4 heads of 64 13.4 us.  What bounds it is
// latency in the softmax, at d = 64 as at 128 (four prompts of 4096 tokens, 32 heads: 755 and 934 us): 1550 clocks a tile where the
// tensor pipe would take 896 and the exponentials 1024, since two warps an SM sub-partition do not cover each other's waits (issue
// slots 42 % taken, exponentials 59 %, tensor pipe 44 %), and some 7000 clocks at an item's end, when the tensor pipe has nothing to do (the
// same warps form the output; four warps of their own for it left the softmax 96 registers a thread instead of 128: 1010 us).
#include <atomic>

#include "ops.h"
#include "tc_common.cuh"

namespace xkv {
namespace {

using namespace tc;

constexpr int kThreads = 512;
constexpr int kSoftWarps = 8;
constexpr int kRows = 128;            // query rows of an item
constexpr int kKeys = 64;             // keys of a tile
constexpr int kStages = 4;            // K tiles, and V tiles
constexpr int kItems = 4;             // items between the walk and the last reader
constexpr int kItemReaders = 5 + kSoftWarps;   // all but the walk itself
constexpr float kLazy = 8.f;          // log2 slack before the reference maximum is raised
// Registers a thread: the launch has 128 for each of its 512; a softmax thread, which holds a row's logits, takes 192 and leaves the
// other roles' threads 64 (a prompt of 32 768 tokens 3.23 ms, with 176 and 80 3.28; heads of 64 750 and 788 us).
constexpr int kLaunchRegs = 128, kSoftRegs = 192, kRoleRegs = 64;
static_assert(256 * kSoftRegs + 256 * kRoleRegs <= kThreads * kLaunchRegs, "no more than the launch has");

struct Params {
  const int32_t* cu_seqlens;
  const float* lambda;                // [Hq]
  const float* gain;                  // [D], nullptr: no norm
  __nv_bfloat16* out;                 // [T][Hq][D]
  float* lse;                         // [Hq][2][T]
  WorkspaceHeader* hdr;
  int64_t total_tokens;
  int32_t batch, n_q_heads, group, max_seqlen;
  int32_t withhold_cta;               // test hook: this CTA's Q and K tiles are never asked for, so that waits expire (-1: none)
  float scale_log2, eps;
  uint64_t wait_ns;
};

struct Item {
  int32_t cu, t, q0, h;               // first token and length of the sequence, first row, query head; h < 0: no more
};

template <int D>
struct Cfg {
  static constexpr int kHalves = D / 64;                     // 128-byte columns of a row
  static constexpr int kMapSteps = D / 32;                   // k-steps of a map's logits
  static constexpr int kQHalfBytes = kRows * 128;
  static constexpr int kQBytes = kHalves * kQHalfBytes;
  static constexpr int kKvHalfBytes = kKeys * 128;
  static constexpr int kKvBytes = kHalves * kKvHalfBytes;
  static constexpr uint32_t kTmemCols = 512;
  // of a map's 256 columns: O_s, logits, weights of even and of odd tiles
  static constexpr uint32_t kMapCols = 256, kSCol = 128, kPCol = 192;
  static constexpr size_t kSmemBytes = 1024 + 2 * (size_t)kQBytes + 2 * (size_t)kStages * kKvBytes;
};

__device__ __forceinline__ bool elect_one() {
  uint32_t r;
  asm volatile("{\n\t.reg .pred q;\n\telect.sync _|q, 0xffffffff;\n\tselp.u32 %0, 1, 0, q;\n\t}" : "=r"(r));
  return r != 0;
}

__device__ __forceinline__ float max3(float a, float b, float c) {
  float r;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
  return r;
}

// Two fp32 operations in one instruction.
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
  float2 r;
  asm("{\n\t.reg .b64 x, y, z, w;\n\t"
      "mov.b64 x, {%2, %3};\n\tmov.b64 y, {%4, %5};\n\tmov.b64 z, {%6, %7};\n\t"
      "fma.rn.f32x2 w, x, y, z;\n\t"
      "mov.b64 {%0, %1}, w;\n\t}"
      : "=f"(r.x), "=f"(r.y)
      : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y), "f"(c.x), "f"(c.y));
  return r;
}
__device__ __forceinline__ float2 add2(float2 a, float2 b) {
  float2 r;
  asm("{\n\t.reg .b64 x, y, w;\n\t"
      "mov.b64 x, {%2, %3};\n\tmov.b64 y, {%4, %5};\n\t"
      "add.rn.f32x2 w, x, y;\n\t"
      "mov.b64 {%0, %1}, w;\n\t}"
      : "=f"(r.x), "=f"(r.y)
      : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
  return r;
}

// The slow side of a bounded wait, a short rolled loop: the kernel waits in two dozen places, and its roles share the instruction
// cache.
__device__ __forceinline__ bool wait_on(uint64_t* bar, uint32_t parity, volatile int* abort_flag, uint64_t limit_ns) {
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

// Item number idx: query tiles in the order of their rows, last rows first, over all sequences; the heads of a tile one after
// the other.  A whole warp.
__device__ Item find_item(const Params& p, int idx) {
  const int lane = threadIdx.x & 31;
  const int tile = idx / p.n_q_heads;
  auto tiles_of = [&](int b) -> int {
    if (b >= p.batch) return 0;
    return (min(__ldg(&p.cu_seqlens[b + 1]) - __ldg(&p.cu_seqlens[b]), p.max_seqlen) + kRows - 1) / kRows;
  };
  const int first = tiles_of(lane);
  // tiles whose place in their sequence is `from` or later
  auto tiles_from = [&](int from) -> int {
    int n = max(first - from, 0);
    for (int b = 32 + lane; b < p.batch; b += 32) n += max(tiles_of(b) - from, 0);
    return __reduce_add_sync(0xffffffffu, n);
  };
  Item it = {0, 0, 0, -1};
  if (tile >= tiles_from(0)) return it;
  int lo = 0, hi = (p.max_seqlen + kRows - 1) / kRows;       // tiles_from(hi) <= tile < tiles_from(lo)
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (tiles_from(mid) <= tile) hi = mid;
    else lo = mid;
  }
  int rank = tile - tiles_from(hi);                          // among the sequences that have a tile at place lo
  for (int base = 0; base < p.batch; base += 32) {
    const unsigned has = __ballot_sync(0xffffffffu, tiles_of(base + lane) > lo);
    const int n = __popc(has);
    if (rank < n) {
      const int b = base + (int)__fns(has, 0, rank + 1);
      it.cu = __ldg(&p.cu_seqlens[b]);
      it.t = min(__ldg(&p.cu_seqlens[b + 1]) - it.cu, p.max_seqlen);
      it.q0 = lo * kRows;
      it.h = idx % p.n_q_heads;
      return it;
    }
    rank -= n;
  }
  return it;
}

// key tiles up to the last one that a row of the item sees
__device__ __forceinline__ int key_tiles(const Item& it) { return (min(it.q0 + kRows, it.t) + kKeys - 1) / kKeys; }

template <int D>
__global__ void __launch_bounds__(kThreads, 1)
diff_prefill_kernel(const __grid_constant__ CUtensorMap tmap_q, const __grid_constant__ CUtensorMap tmap_k,
                    const __grid_constant__ CUtensorMap tmap_v, const __grid_constant__ Params p) {
  using C = Cfg<D>;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  uint8_t* q_s = smem;
  uint8_t* k_s = q_s + 2 * C::kQBytes;
  uint8_t* v_s = k_s + kStages * C::kKvBytes;
  __shared__ uint64_t s_item_full[kItems], s_item_empty[kItems], s_q_full[2], s_q_empty[2], s_k_full[kStages], s_k_empty[kStages],
      s_v_full[kStages], s_v_clear, s_v_empty[kStages], s_s_full[2], s_s_free[2], s_p_full[2][2], s_o_full[2][2], s_o_free, s_inv_full,
      s_sq_full;
  __shared__ Item s_item[kItems];
  __shared__ uint4 s_stage[kSoftWarps][32][5];               // rows of 64 bytes, a piece apart: no two lanes of a phase share a bank
  __shared__ float s_inv[2][2][kRows], s_sq[2][kRows];      // s_inv: of even and of odd items, a warp may still read the item before
  __shared__ uint32_t s_tmem;
  __shared__ int s_abort_store;
  volatile int* s_abort = &s_abort_store;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;

  if (tid == 0) {
    for (int i = 0; i < kItems; ++i) {
      mbar_init(&s_item_full[i], 1);
      mbar_init(&s_item_empty[i], kItemReaders);
    }
    for (int i = 0; i < kStages; ++i) {
      mbar_init(&s_k_full[i], 1);
      mbar_init(&s_k_empty[i], 2);
      mbar_init(&s_v_full[i], 1);
      mbar_init(&s_v_empty[i], 2);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(&s_q_full[i], 1);
      mbar_init(&s_q_empty[i], 2);
      mbar_init(&s_s_full[i], 1);
      mbar_init(&s_s_free[i], kSoftWarps / 2);
      for (int b = 0; b < 2; ++b) {
        mbar_init(&s_p_full[i][b], kSoftWarps / 2);
        mbar_init(&s_o_full[i][b], 1);
      }
    }
    mbar_init(&s_v_clear, 1);
    mbar_init(&s_o_free, kSoftWarps);
    mbar_init(&s_inv_full, kSoftWarps);
    mbar_init(&s_sq_full, kSoftWarps);
    s_abort_store = 0;
    fence_mbar_init();
    prefetch_tmap(&tmap_q);
    prefetch_tmap(&tmap_k);
    prefetch_tmap(&tmap_v);
  }
  if (warp == 9) {
    tmem_alloc(&s_tmem, C::kTmemCols);
    tmem_relinquish();
  }
  tc_fence_before_sync();
  __syncthreads();
  tc_fence_after_sync();
  const uint32_t tmem = s_tmem;

  auto wait = [&](uint64_t* bar, uint32_t parity) -> bool {
    bool ok = true;
    if (__builtin_expect(!mbar_try_wait(bar, parity & 1u), 0)) ok = wait_on(bar, parity & 1u, s_abort, p.wait_ns);
    __syncwarp();
    return ok;
  };
  // the n-th item; false when there is none (or a wait has expired)
  auto get_item = [&](uint32_t n, Item* it) -> bool {
    if (!wait(&s_item_full[n % kItems], n / kItems)) return false;
    *it = s_item[n % kItems];
    return it->h >= 0;
  };
  auto done_item = [&](uint32_t n) {
    __syncwarp();
    if (lane == 0) mbar_arrive(&s_item_empty[n % kItems]);
  };

  if (warp >= kSoftWarps) {
  asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kRoleRegs));
  if (warp == 8) {
    // ================================================================ Q and K tiles
    uint32_t jj = 0;
    Item it;
    for (uint32_t n = 0; get_item(n, &it); ++n) {
      done_item(n);
      if ((int)blockIdx.x == p.withhold_cta) break;
      const int n_kt = key_tiles(it), g = it.h / p.group;
      if (n >= 2 && !wait(&s_q_empty[n & 1], (n / 2) - 1)) break;
      if (elect_one()) {
        mbar_arrive_expect_tx(&s_q_full[n & 1], (uint32_t)C::kQBytes);
#pragma unroll
        for (int hf = 0; hf < C::kHalves; ++hf)
          tma_load_3d(q_s + (n & 1) * C::kQBytes + hf * C::kQHalfBytes, &tmap_q, hf * 64, it.h, it.cu + it.q0, &s_q_full[n & 1]);
      }
      __syncwarp();
      bool ok = true;
      for (int j = 0; j < n_kt; ++j, ++jj) {
        const uint32_t s = jj % kStages;
        if (jj >= kStages) ok = wait(&s_k_empty[s], jj / kStages - 1);
        if (!ok) break;
        if (elect_one()) {
          mbar_arrive_expect_tx(&s_k_full[s], (uint32_t)C::kKvBytes);
#pragma unroll
          for (int hf = 0; hf < C::kHalves; ++hf)
            tma_load_3d(k_s + s * C::kKvBytes + hf * C::kKvHalfBytes, &tmap_k, hf * 64, g, it.cu + j * kKeys, &s_k_full[s]);
        }
        __syncwarp();
      }
      if (!ok) break;
    }
  } else if (warp == 11) {
    // ================================================================ the walk, and V tiles
    auto publish = [&](uint32_t n) -> Item {
      const int at = (n & 1) ? (int)(gridDim.x - 1 - blockIdx.x) : (int)blockIdx.x;
      const Item it = find_item(p, (int)(n * gridDim.x) + at);
      if (n >= kItems && !wait(&s_item_empty[n % kItems], n / kItems - 1)) return {0, 0, 0, -1};
      if (lane == 0) {
        s_item[n % kItems] = it;
        mbar_arrive(&s_item_full[n % kItems]);
      }
      __syncwarp();
      return it;
    };
    uint32_t jj = 0;
    Item it = publish(0);
    for (uint32_t n = 0; it.h >= 0; ++n) {
      const Item next = publish(n + 1);
      const int n_kt = key_tiles(it), g = it.h / p.group;
      bool ok = true;
      for (int j = 0; j < n_kt; ++j, ++jj) {
        const uint32_t s = jj % kStages;
        if (jj >= kStages) ok = wait(&s_v_empty[s], jj / kStages - 1);
        if (!ok) break;
        if (elect_one()) {
          mbar_arrive_expect_tx(&s_v_full[s], (uint32_t)C::kKvBytes);
#pragma unroll
          for (int hf = 0; hf < C::kHalves; ++hf)
            tma_load_3d(v_s + s * C::kKvBytes + hf * C::kKvHalfBytes, &tmap_v, hf * 64, g, it.cu + j * kKeys, &s_v_full[s]);
        }
        __syncwarp();
      }
      if (!ok) break;
      it = next;
    }
  } else if (warp == 9 || warp == 10) {
    // ================================================================ the logits of a map
    const int map = warp - 9;
    constexpr uint32_t kIdesc = umma_idesc(kRows, kKeys);
    const uint32_t s_at = tmem + map * C::kMapCols + C::kSCol;
    uint32_t jj = 0;
    Item it;
    bool ok = true;
    for (uint32_t n = 0; ok && get_item(n, &it); ++n) {
      done_item(n);
      const int n_kt = key_tiles(it);
      ok = wait(&s_q_full[n & 1], n / 2);
      const uint64_t q_desc = umma_desc_k128(smem_u32(q_s + (n & 1) * C::kQBytes));
      for (int j = 0; j < n_kt; ++j, ++jj) {
        const uint32_t s = jj % kStages;
        ok = ok && wait(&s_k_full[s], jj / kStages);
        if (jj > 0) ok = ok && wait(&s_s_free[map], jj - 1);            // the tile before is in registers
        // the product of the tile before that has read its weights, whose buffer this tile's go to
        if (jj > 1) ok = ok && wait(&s_o_full[map][jj & 1], jj / 2 - 1);
        if (!ok) break;
        tc_fence_after_sync();
        if (elect_one()) {
          const uint64_t k_desc = umma_desc_k128(smem_u32(k_s + s * C::kKvBytes));
#pragma unroll
          for (int x = 0; x < C::kMapSteps; ++x) {
            const int k = map * C::kMapSteps + x;
            const uint64_t q_off = (uint64_t)(((k / 4) * C::kQHalfBytes + (k % 4) * 32) >> 4);
            const uint64_t k_off = (uint64_t)(((k / 4) * C::kKvHalfBytes + (k % 4) * 32) >> 4);
            umma_bf16(s_at, q_desc + q_off, k_desc + k_off, kIdesc, x > 0 ? 1u : 0u);
          }
          umma_commit(&s_s_full[map]);
          umma_commit(&s_k_empty[s]);
          if (j == n_kt - 1) umma_commit(&s_q_empty[n & 1]);
        }
        __syncwarp();
      }
    }
  } else if (warp == 12 || warp == 13) {
    // ================================================================ the outputs of a map
    const int map = warp - 12;
    constexpr uint32_t kIdesc = umma_idesc_b_mn(kRows, D);
    const uint32_t o_at = tmem + map * C::kMapCols, p_at = o_at + C::kPCol;
    uint32_t jj = 0, n_clear = 0;
    Item it;
    bool ok = true;
    for (uint32_t n = 0; ok && get_item(n, &it); ++n) {
      done_item(n);
      const int n_kt = key_tiles(it);
      // the item before has read its O (which also keeps the two warps within one clearing of each other)
      if (n > 0) ok = wait(&s_o_free, n - 1);
      for (int j = 0; j < n_kt; ++j, ++jj) {
        const uint32_t s = jj % kStages, b = jj & 1;
        ok = ok && wait(&s_v_full[s], jj / kStages);
        if (!ok) break;
        const int left = it.t - j * kKeys;
        if (left < kKeys) {                                  // rows behind the prompt's last one
          if (map == 0) {
            uint4* v = reinterpret_cast<uint4*>(v_s + s * C::kKvBytes);
            for (int i = left * 8 + lane; i < kKeys * 8; i += 32)
#pragma unroll
              for (int hf = 0; hf < C::kHalves; ++hf) v[hf * (C::kKvHalfBytes / 16) + i] = make_uint4(0u, 0u, 0u, 0u);
            fence_proxy_async_smem();
            __syncwarp();
            if (lane == 0) mbar_arrive(&s_v_clear);
          } else {
            ok = wait(&s_v_clear, n_clear);
            fence_proxy_async_smem();
          }
          ++n_clear;
        }
        ok = ok && wait(&s_p_full[map][b], jj / 2);
        if (!ok) break;
        tc_fence_after_sync();
        if (elect_one()) {
          const uint64_t v_desc = umma_desc_mn128(smem_u32(v_s + s * C::kKvBytes), C::kKvHalfBytes);
#pragma unroll
          for (int k = 0; k < kKeys / 16; ++k)
            umma_bf16_a_tmem(o_at, p_at + b * 32 + k * 8, v_desc + (uint64_t)(k * 16 * 128 >> 4), kIdesc,
                             (j > 0 || k > 0) ? 1u : 0u);
          umma_commit(&s_o_full[map][b]);
          umma_commit(&s_v_empty[s]);
        }
        __syncwarp();
      }
    }
  }
  } else {
    // ================================================================ softmax of map `map`
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kSoftRegs));
    const int map = warp >> 2, r = tid & (kRows - 1);
    const uint32_t lanes = tmem + ((uint32_t)(32 * (warp & 3)) << 16);
    const uint32_t o_at = lanes + map * C::kMapCols, s_at = o_at + C::kSCol, p_at = o_at + C::kPCol;
    uint32_t jj = 0;
    Item it;
    for (uint32_t n = 0; get_item(n, &it); ++n) {
      done_item(n);
      const int n_kt = key_tiles(it), row = it.q0 + r;
      float m_ref = -INFINITY, l = 0.f;
      const float lambda = __ldg(&p.lambda[it.h]);
      bool ok = true;
      for (int j = 0; j < n_kt; ++j, ++jj) {
        const uint32_t b = jj & 1;
        ok = wait(&s_s_full[map], jj);
        if (!ok) break;
        tc_fence_after_sync();
        float v[2][32];
        tmem_ld32(s_at, v[0]);
        tmem_ld32(s_at + 32, v[1]);
        tmem_wait_ld();
        tc_fence_before_sync();
        __syncwarp();
        if (lane == 0) mbar_arrive(&s_s_free[map]);
        const int c0 = j * kKeys;
        if (c0 + kKeys - 1 > it.q0) {                        // the tile holds keys behind some row
#pragma unroll
          for (int i = 0; i < kKeys; ++i)
            if (c0 + i > row) v[i >> 5][i & 31] = -INFINITY;
        }
        float m4[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
        for (int i = 0; i < kKeys; i += 8)
#pragma unroll
          for (int x = 0; x < 4; ++x) m4[x] = max3(m4[x], v[i >> 5][(i & 31) + x], v[i >> 5][(i & 31) + x + 4]);
        const float mx = fmaxf(fmaxf(m4[0], m4[1]), fmaxf(m4[2], m4[3])) * p.scale_log2;   // key 0 is visible to every row
        const bool grow = mx > m_ref + kLazy;                // also on the first tile
        float alpha = 1.f;
        if (grow) {
          alpha = j == 0 ? 0.f : fast_exp2(m_ref - mx);
          m_ref = mx;
          l *= alpha;
        }
        if (j > 0 && __any_sync(0xffffffffu, grow)) {        // O_s of the tiles so far is complete, then rescaled
          ok = wait(&s_o_full[map][(jj - 1) & 1], (jj - 1) / 2);
          if (!ok) break;
          tc_fence_after_sync();
#pragma unroll
          for (int c = 0; c < D; c += 16) {
            float o[16];
            tmem_ld16(o_at + c, o);
            tmem_wait_ld();
#pragma unroll
            for (int i = 0; i < 16; ++i) o[i] *= alpha;
            tmem_st16(o_at + c, o);
          }
          tmem_wait_st();
        }
        float2 sm[2] = {{0.f, 0.f}, {0.f, 0.f}};
        const float2 scale2 = {p.scale_log2, p.scale_log2}, ref2 = {-m_ref, -m_ref};
        uint32_t packed[32];
#pragma unroll
        for (int c = 0; c < kKeys; c += 4) {
#pragma unroll
          for (int x = 0; x < 2; ++x) {
            const int i = c + 2 * x;
            float2 e = fma2({v[i >> 5][i & 31], v[i >> 5][(i & 31) + 1]}, scale2, ref2);
            e = {fast_exp2(e.x), fast_exp2(e.y)};
            sm[x] = add2(sm[x], e);
            packed[i >> 1] = pack_bf16(e.x, e.y);
          }
        }
        // (the buffer is free: this tile's logits were issued after the product of the tile before the last)
        tmem_st32u(p_at + b * 32, packed);
        l += (sm[0].x + sm[0].y) + (sm[1].x + sm[1].y);
        tmem_wait_st();
        tc_fence_before_sync();
        __syncwarp();
        if (lane == 0) mbar_arrive(&s_p_full[map][b]);
      }
      if (!ok) break;
      // ---- both maps' O are complete; this map's warps take columns [map D/2, (map + 1) D/2) of their rows
      const uint32_t last = jj - 1;
      s_inv[n & 1][map][r] = l > 0.f ? 1.f / l : 0.f;
      __syncwarp();
      if (lane == 0) mbar_arrive(&s_inv_full);
      if (row < it.t && p.lse != nullptr)
        p.lse[((size_t)it.h * 2 + map) * p.total_tokens + it.cu + row] = (m_ref + log2f(l)) * 0.6931471805599453f;
      // First that every warp has come to its last tile: the other map may be tiles behind, and a wait by parity would then take
      // the phase two back for the one meant.
      ok = wait(&s_inv_full, n) && wait(&s_o_full[0][last & 1], last / 2) && wait(&s_o_full[1][last & 1], last / 2);
      if (!ok) break;
      tc_fence_after_sync();
      const float w1 = s_inv[n & 1][0][r], w2 = -lambda * s_inv[n & 1][1][r];
      float y[D / 2], sq = 0.f;
#pragma unroll
      for (int c = 0; c < D / 2; c += 32) {
        float a[32], x[32];
        tmem_ld32(lanes + map * (D / 2) + c, a);
        tmem_ld32(lanes + C::kMapCols + map * (D / 2) + c, x);
        tmem_wait_ld();
#pragma unroll
        for (int i = 0; i < 32; ++i) {
          y[c + i] = fmaf(x[i], w2, a[i] * w1);
          sq = fmaf(y[c + i], y[c + i], sq);
        }
      }
      tc_fence_before_sync();
      if (p.gain != nullptr) {
        s_sq[map][r] = sq;
        __syncwarp();
        if (lane == 0) {
          mbar_arrive(&s_o_free);
          mbar_arrive(&s_sq_full);
        }
        ok = wait(&s_sq_full, n);
        if (!ok) break;
        const float norm = diff_norm<D>(s_sq[0][r] + s_sq[1][r], p.eps);
        const float4* gain = reinterpret_cast<const float4*>(p.gain + map * (D / 2));
#pragma unroll
        for (int c = 0; c < D / 2; c += 4) {
          const float4 gv = __ldg(&gain[c / 4]);
          y[c] *= norm * gv.x, y[c + 1] *= norm * gv.y, y[c + 2] *= norm * gv.z, y[c + 3] *= norm * gv.w;
        }
      } else {
        __syncwarp();
        if (lane == 0) mbar_arrive(&s_o_free);
      }
      // 32 columns at a time through shared memory, so that a store takes eight rows of 64 bytes instead of 32 of 16
#pragma unroll
      for (int c = 0; c < D / 2; c += 32) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float* x = y + c + 8 * i;
          s_stage[warp][lane][i] =
              make_uint4(pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]), pack_bf16(x[4], x[5]), pack_bf16(x[6], x[7]));
        }
        __syncwarp();
        const int first = it.q0 + 32 * (warp & 3) + (lane >> 2);
        __nv_bfloat16* o = p.out + ((size_t)(it.cu + first) * p.n_q_heads + it.h) * D + map * (D / 2) + c + 8 * (lane & 3);
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (first + 8 * i < it.t)
            *reinterpret_cast<uint4*>(o + (size_t)(8 * i) * p.n_q_heads * D) = s_stage[warp][8 * i + (lane >> 2)][lane & 3];
        __syncwarp();
      }
    }
  }

  // ---- teardown
  __syncthreads();
  if (*s_abort) {
    if (tid == 0) record_status(p.hdr, XKV_ERR_TIMEOUT);
    for (int i = 0; i < 1000; ++i) __nanosleep(1000);   // let copies and MMAs already issued finish
  }
  tc_fence_after_sync();
  if (warp == 9) tmem_dealloc(tmem, C::kTmemCols);
}

template <int D>
xkv_status launch(const CUtensorMap& tq, const CUtensorMap& tk, const CUtensorMap& tv, const Params& p, int grid,
                  cudaStream_t st) {
  static std::atomic<bool> done[64];   // idempotent set-up: two threads doing it twice is harmless
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return XKV_ERR_CUDA;
  if (!done[dev].load(std::memory_order_acquire)) {
    cudaFuncAttributes attr;           // the split of the registers counts on the launch's
    if (cudaFuncGetAttributes(&attr, diff_prefill_kernel<D>) != cudaSuccess || attr.numRegs != kLaunchRegs ||
        cudaFuncSetAttribute(diff_prefill_kernel<D>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)Cfg<D>::kSmemBytes) !=
            cudaSuccess) {
      (void)cudaGetLastError();
      return XKV_ERR_CUDA;
    }
    done[dev].store(true, std::memory_order_release);
  }
  diff_prefill_kernel<D><<<grid, kThreads, Cfg<D>::kSmemBytes, st>>>(tq, tk, tv, p);
  count_launch();
  return check_launch();
}

}  // namespace

xkv_status diff_prefill_attn(const xkv_dims* d, const void* q, const void* k, const void* v, const float* lambda,
                             const float* gain, float eps, const int32_t* cu_seqlens, int64_t total_tokens, int max_seqlen,
                             void* out, float* lse, void* workspace, cudaStream_t st) {
  Params p;
  p.cu_seqlens = cu_seqlens;
  p.lambda = lambda;
  p.gain = gain;
  p.out = static_cast<__nv_bfloat16*>(out);
  p.lse = lse;
  p.hdr = reinterpret_cast<WorkspaceHeader*>(workspace);
  p.total_tokens = total_tokens;
  p.batch = d->batch;
  p.n_q_heads = d->n_q_heads;
  p.group = d->n_q_heads / d->n_kv_heads;
  p.max_seqlen = max_seqlen;
  p.scale_log2 = (d->scale != 0.f ? d->scale : 1.0f / sqrtf((float)(d->head_dim / 2))) * 1.4426950408889634f;
  p.eps = eps;
  p.wait_ns = wait_limit_ns();
  p.withhold_cta = debug_withhold_item();
  CUtensorMap tq, tk, tv;
  if (!tc_make_token_tmap(&tq, q, d->head_dim, d->n_q_heads, total_tokens, (int64_t)d->n_q_heads * d->head_dim, d->head_dim,
                          kRows) ||
      !tc_make_token_tmap(&tk, k, d->head_dim, d->n_kv_heads, total_tokens, d->kv_stride_token, d->kv_stride_head, kKeys) ||
      !tc_make_token_tmap(&tv, v, d->head_dim, d->n_kv_heads, total_tokens, d->kv_stride_token, d->kv_stride_head, kKeys))
    return XKV_ERR_CUDA;
  // every sequence adds at most one partial tile; items are counted in 32 bits, the last round's and the look-ahead included
  const int64_t items = (total_tokens / kRows + d->batch) * d->n_q_heads;
  if (items > 0x7fffffffll - 4 * 1024) return XKV_ERR_UNSUPPORTED;
  const int grid = (int)(items < sm_count() ? items : sm_count());
  return d->head_dim == 128 ? launch<128>(tq, tk, tv, p, grid, st) : launch<64>(tq, tk, tv, p, grid, st);
}

}  // namespace xkv
