// Serving on a reduced cache: the plan of a step (xkv_plan_append) and rows stored by slot (xkv_store_rows).
//
//   plan_small_kernel   the plan of up to 4096 (layer, sequence) caches by one CTA: pages asked for, their scan, new
//                       lengths; for a decode step's few tokens also their slots and table entries
//   slots_kernel        slots and table entries of many tokens, from what plan_small_kernel found (programmatic dependent
//                       launch): a stretch of tokens per warp, the page ids of eight rounds in flight together.  Bound by
//                       its 8 bytes written per layer and token and by the instructions that make them: 64 prompts in 32
//                       layers, 84 MB: 25.7 us, of which about 7 us are the first launch (a plain fill takes 13 us)
//   plan_kernel         more caches than that, in one launch: grid = (slices, layers), no CTA waits for another one: each
//                       forms the pages asked for by the layers before its own and the scan over its layer's sequences by
//                       itself (integers out of L2), and the last CTA to leave writes the lengths, so that they may
//                       be advanced in place.
//   store_block_kernel  caches of 8-bit floats: one warp per (run of tokens within a block of 16 slots, KV head, K or V),
//                       which reads the run once, finds its largest magnitude and stores the codes: HBM-bound, 3 bytes a
//                       value (K and V of 9160 tokens, 32 heads of 128: 225 MB in 38 us, 0.90 of the copy rate)
//   store_row_kernel    caches of bf16 or of 8-bit integers: D/8 lanes per (token, KV head)
//   append_block_kernel one new row per (layer, sequence) and KV head of a cache of 8-bit floats, lengths advanced
#include <algorithm>
#include <atomic>

#include "common.cuh"
#include "e4m3.cuh"
#include "ops.h"

namespace xkv {
namespace {

// ---------------------------------------------------------------------------------------------
// Plan of a step
// ---------------------------------------------------------------------------------------------
constexpr int kPlanThreads = 256;
constexpr int kSmallThreads = 1024;           // one CTA plans up to kSmallUnits sequences of all layers
constexpr int kSmallUnits = 4096;
constexpr int kSlotRun = 64;                  // ... and hands its tokens to its warps in runs of so many
constexpr int64_t kSmallTokens = 4096;        // ... where they are no more than this (by the slot maps' sizes)
constexpr int kStepTokens = 2;                // ... unless no cache takes more than so many: then by its threads
constexpr int kPlanMaxBatch = 16384;          // sequences of a layer: two 4-byte table entries each in shared memory

struct PlanParams {
  const int32_t* n_new;
  int64_t n_new_stride;
  const int32_t* lens_before;   // null: all zero
  int32_t* lens_after;
  const int32_t* free_pages;    // null: page id = position
  int32_t n_free;
  const int32_t* used_before;   // null: 0
  int32_t* used_after;
  int32_t* block_table;
  int64_t* slots;
  int64_t slots_stride;
  int32_t n_layers, batch, page_size, max_pages_per_seq, n_pages;
  WorkspaceHeader* hdr;
  // in the workspace
  int32_t* new_lens;            // [n_layers][batch]: one launch of many CTAs: until the last of them copies them out
  int32_t* ws_tok;              // [n_layers][batch + 1], [n_layers][batch] twice: two launches: what the first one found
  int32_t* ws_start;
  int32_t* ws_len;
  int32_t two_launches;
  // row -> page: page_size is 8 D with D even, 2 <= D <= 32, and n / D = (n * ceil(2^32 / D)) >> 32 for n <= 2^27 + 32
  // (exact: n times what the ceiling adds, at most 29 where D is no power of two and else nothing, stays below 2^32)
  uint32_t page_mul;            // ceil(2^32 / D)
  __device__ __forceinline__ int page_of(int row) const { return (int)__umulhi((uint32_t)row >> 3, page_mul); }
};

struct Ask {
  int32_t len, add;             // rows before, rows to add (both clamped at 0)
  int32_t pages;                // pages to take; -1: the cache cannot hold that many rows
  bool bad;                     // a negative count was found
};

// e = l * batch + b
__device__ __forceinline__ Ask plan_ask(const PlanParams& p, int l, int e, int b) {
  Ask a;
  const int len = p.lens_before != nullptr ? p.lens_before[e] : 0;      // (not through the read-only path: may be seq_lens)
  const int add = __ldg(&p.n_new[l * p.n_new_stride + b]);
  a.bad = len < 0 || add < 0;
  a.len = max(len, 0);
  a.add = max(add, 0);
  const int64_t total = (int64_t)a.len + a.add;
  if (total > (int64_t)p.max_pages_per_seq * p.page_size) {
    a.pages = -1;
  } else {
    a.pages = p.page_of((int)total + p.page_size - 1) - p.page_of(a.len + p.page_size - 1);
  }
  return a;
}

__device__ __forceinline__ long long warp_sum(long long v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}

// A page id of the free list: position `at`.
__device__ __forceinline__ int free_page(const PlanParams& p, int at) {
  return p.free_pages != nullptr ? __ldg(&p.free_pages[at]) : at;
}

constexpr int kRounds = 8;                    // tokens a lane takes at a time

// 32 * kRounds tokens from t on, or those of them before `end` (kAll: all), of one sequence and in new pages.  Row `x +
// shift` of the sequence is token x; id(i): its page i.
template <bool kAll, class Id>
__device__ __forceinline__ void write_batch(const PlanParams& p, int32_t* row, int64_t* out, int t, int end, int shift, Id id) {
  const int lane = threadIdx.x & 31;
  const int pos0 = t + shift + lane, n = end - t - lane;          // rounds 32 k < n of this lane hold a token
  int64_t* dst = out + t + lane;
  int page[kRounds];
  uint32_t top = 0;
#pragma unroll
  for (int k = 0; k < kRounds; ++k) page[k] = id(p.page_of(kAll || 32 * k < n ? pos0 + 32 * k : end - 1 + shift));
#pragma unroll
  for (int k = 0; k < kRounds; ++k) top = max(top, (uint32_t)page[k]);
  if (top >= (uint32_t)p.n_pages) {                               // an id outside the pool: no slot
    record_status(p.hdr, XKV_ERR_INVALID_ARG);
#pragma unroll 1
    for (int k = 0; k < kRounds && 32 * k < n; ++k) {
      const int i = p.page_of(pos0 + 32 * k), in_page = pos0 + 32 * k - i * p.page_size, pg = id(i);
      dst[32 * k] = (uint32_t)pg < (uint32_t)p.n_pages ? (int64_t)pg * p.page_size + in_page : -1;
      if (in_page == 0) row[i] = pg;
    }
    return;
  }
#pragma unroll
  for (int k = 0; k < kRounds; ++k) {
    const int i = p.page_of(pos0 + 32 * k), in_page = pos0 + 32 * k - i * p.page_size;
    if (kAll || 32 * k < n) {
      dst[32 * k] = (int64_t)page[k] * p.page_size + in_page;
      if (in_page == 0) row[i] = page[k];
    }
  }
}

template <class Id>
__device__ __forceinline__ void write_stretch(const PlanParams& p, int32_t* row, int64_t* out, int t, int end, int shift,
                                              Id id) {
#pragma unroll 1
  for (; end - t >= 32 * kRounds; t += 32 * kRounds) write_batch<true>(p, row, out, t, end, shift, id);
  if (t < end) write_batch<false>(p, row, out, t, end, shift, id);
}

// The new tokens [t, t_end) of a layer (a whole warp), all of which have a place in `out`: their slots, and the table
// entries of the pages that begin with one of them (every new page begins with a new token).  tok(b): tokens of the layer
// before sequence b (b <= batch; more than 2^31 - 1 count as that many), start(b): where its new pages begin in the free
// list (-1: it cannot grow), len(b): its rows before the step.  t_end may be 2^31 - 1: no token number behind it is formed.
template <class Tok, class Start, class Len>
__device__ __forceinline__ void write_range(const PlanParams& p, int32_t* table, int64_t* out, int t, int t_end, Tok tok,
                                            Start start, Len len) {
  const int lane = threadIdx.x & 31;
  constexpr int kMix = 2;
  auto search = [&](int lo, int x) -> int {    // the sequence that holds token x; lo: one at or before it
    int hi = p.batch;                          // tok(lo) <= x < tok(hi)
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (tok(mid) <= x) lo = mid;
      else hi = mid;
    }
    return lo;
  };
  int lo = t < t_end ? search(0, t) : 0;
#pragma unroll 1
  while (t < t_end) {
    const int seq_end = (int)min((long long)tok(lo + 1), (long long)t_end);
    if (seq_end - t >= 32 * kMix && start(lo) >= 0) {
      // a stretch of one sequence (prompts), in new pages: the page ids of eight rounds in flight together
      const int n = len(lo), shift = n - (int)tok(lo), have = p.page_of(n + p.page_size - 1), first = start(lo) - have;
      if (t + shift >= have * p.page_size) {
        int32_t* row = table + (size_t)lo * p.max_pages_per_seq;
        if (p.free_pages != nullptr) write_stretch(p, row, out, t, seq_end, shift, [&](int i) { return __ldg(p.free_pages + first + i); });
        else                         write_stretch(p, row, out, t, seq_end, shift, [&](int i) { return first + i; });
        t = seq_end;
        if (t < t_end) lo = search(lo, t);
        continue;
      }
    }
    // any mixture: every lane its own search (a decode step has one token per sequence)
    const int left = t_end - t;
    int seq[kMix], page[kMix];
#pragma unroll
    for (int k = 0; k < kMix; ++k) {
      seq[k] = -1;
      page[k] = -1;
      if (32 * k + lane < left) {
        const int at = t + 32 * k + lane;
        if (tok(lo + 1) <= at) lo = search(lo, at);
        const int st = start(lo);
        if (st >= 0) {
          const int n = len(lo), i = p.page_of(n + (int)(at - tok(lo))), have = p.page_of(n + p.page_size - 1);
          seq[k] = lo;
          page[k] = i < have ? table[(size_t)lo * p.max_pages_per_seq + i] : free_page(p, st + i - have);
        }
      }
    }
#pragma unroll
    for (int k = 0; k < kMix; ++k) {
      if (32 * k + lane >= left) continue;
      const int at = t + 32 * k + lane, b = seq[k];
      int64_t slot = -1;
      if (b >= 0) {
        const int pos = len(b) + (int)(at - tok(b)), i = p.page_of(pos), in_page = pos - i * p.page_size;
        if (in_page == 0) table[(size_t)b * p.max_pages_per_seq + i] = page[k];
        if ((unsigned)page[k] < (unsigned)p.n_pages) slot = (int64_t)page[k] * p.page_size + in_page;
        else record_status(p.hdr, XKV_ERR_INVALID_ARG);
      }
      out[at] = slot;
    }
    if (left <= 32 * kMix) break;
    t += 32 * kMix;
    lo = search(__shfl_sync(0xffffffffu, lo, 0), t);
  }
}

// Entries lane, lane + 32, .. of a sequence's new pages (a whole warp).
__device__ __forceinline__ void write_pages(const PlanParams& p, int32_t* at, int pages, int start) {
  for (int i = threadIdx.x & 31; i < pages; i += 32) {
    const int page = free_page(p, start + i);
    if ((unsigned)page >= (unsigned)p.n_pages) record_status(p.hdr, XKV_ERR_INVALID_ARG);
    at[i] = page;
  }
}

__global__ void __launch_bounds__(kPlanThreads) plan_kernel(const PlanParams p) {
  extern __shared__ int32_t s_plan[];
  int32_t* s_tok = s_plan;                    // [batch + 1] tokens of the layer before each sequence
  int32_t* s_start = s_plan + p.batch + 1;    // [batch] position in the free list, -1: the pages do not fit
  __shared__ long long s_red[32], s_red2[32];
  __shared__ int s_last;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  constexpr int kWarps = kPlanThreads / 32;
  const int layer = blockIdx.y, slice = blockIdx.x, n_slices = gridDim.x;
  int used = p.used_before != nullptr ? *p.used_before : 0;
  if (used < 0 || used > p.n_free) {
    if (tid == 0) record_status(p.hdr, XKV_ERR_INVALID_ARG);
    used = p.n_free;                          // nothing can be handed out
  }

  // ---- pages asked for by the layers before this one
  long long before = 0;
#pragma unroll 8
  for (int e = tid; e < layer * p.batch; e += kPlanThreads) {
    const Ask a = plan_ask(p, e / p.batch, e, e % p.batch);
    before += max(a.pages, 0);
  }
  before = warp_sum(before);
  if (lane == 0) s_red[warp] = before;
  __syncthreads();
  before = used;
#pragma unroll
  for (int w = 0; w < kWarps; ++w) before += s_red[w];

  // ---- scan over the layer's sequences
  long long carry = before, tok_carry = 0;
  int end_max = 0;
  for (int b0 = 0; b0 < p.batch; b0 += kPlanThreads) {
    const int b = b0 + tid;
    Ask a = {0, 0, 0, false};
    if (b < p.batch) a = plan_ask(p, layer, layer * p.batch + b, b);
    const long long ask = max(a.pages, 0), add = a.add;
    long long incl = ask, tincl = add;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const long long x = __shfl_up_sync(0xffffffffu, incl, o), y = __shfl_up_sync(0xffffffffu, tincl, o);
      if (lane >= o) {
        incl += x;
        tincl += y;
      }
    }
    __syncthreads();
    if (lane == 31) {
      s_red[warp] = incl;
      s_red2[warp] = tincl;
    }
    __syncthreads();
    long long base = carry, tbase = tok_carry, all = 0, tall = 0;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) {
      if (w < warp) {
        base += s_red[w];
        tbase += s_red2[w];
      }
      all += s_red[w];
      tall += s_red2[w];
    }
    if (b < p.batch) {
      const long long start = base + incl - ask;
      const bool fits = a.pages >= 0 && (ask == 0 || start + ask <= p.n_free);
      s_start[b] = fits ? (int)min(start, (long long)p.n_free) : -1;
      s_tok[b] = (int)min(tbase + tincl - add, 0x7fffffffll);
      if (fits && ask > 0) end_max = max(end_max, (int)(start + ask));
      if (slice == 0) {
        p.new_lens[(size_t)layer * p.batch + b] = fits ? a.len + a.add : a.len;
        if (a.bad) record_status(p.hdr, XKV_ERR_INVALID_ARG);
        else if (!fits) record_status(p.hdr, XKV_ERR_CAPACITY);
      }
    }
    carry += all;
    tok_carry += tall;
  }
  if (tid == 0) s_tok[p.batch] = (int)min(tok_carry, 0x7fffffffll);
  if (slice == 0) {
    end_max = __reduce_max_sync(0xffffffffu, end_max);
    if (lane == 0 && end_max > 0) atomicMax(&p.hdr->plan_used, end_max);
    __threadfence();                          // the new lengths, for the last CTA; what follows is not waited for
  }
  __syncthreads();

  int32_t* table = p.block_table + (size_t)layer * p.batch * p.max_pages_per_seq;
  if (p.slots != nullptr) {
    // ---- slots and new table entries, by runs of tokens
    const int total = s_tok[p.batch], n_slots = (int)min((int64_t)total, p.slots_stride);
    if (slice == 0 && tid == 0 && total > p.slots_stride) record_status(p.hdr, XKV_ERR_CAPACITY);
    int64_t* out = p.slots + layer * p.slots_stride;
    const int32_t* lens = p.lens_before != nullptr ? p.lens_before + (size_t)layer * p.batch : nullptr;
    // every warp one stretch: it looks up a sequence once and finds its page ids in the L1 cache
    const int64_t stretch = ((int64_t)n_slots + n_slices * kWarps - 1) / (n_slices * kWarps);
    const int64_t t0 = (slice * kWarps + warp) * stretch;
    write_range(p, table, out, (int)min(t0, (int64_t)n_slots), (int)min(t0 + stretch, (int64_t)n_slots),
                [&](int b) { return s_tok[b]; }, [&](int b) { return s_start[b]; },
                [&](int b) { return lens != nullptr ? max(lens[b], 0) : 0; });
  }
  if (p.slots == nullptr || s_tok[p.batch] > p.slots_stride) {
    // ---- the new table entries of sequences that have tokens without a place in the slot map: a warp per sequence
    for (int b = slice * kWarps + warp; b < p.batch; b += n_slices * kWarps) {
      const int start = s_start[b];
      if (start < 0 || (p.slots != nullptr && s_tok[b + 1] <= p.slots_stride)) continue;
      const Ask a = plan_ask(p, layer, layer * p.batch + b, b);
      write_pages(p, table + (size_t)b * p.max_pages_per_seq + p.page_of(a.len + p.page_size - 1), a.pages, start);
    }
  }

  // ---- the last CTA to get here writes the lengths (every other one has read them) and the list position
  __syncthreads();
  const int n_ctas = gridDim.x * gridDim.y;
  if (tid == 0) s_last = (atomicAdd(&p.hdr->plan_ticket, 1) == n_ctas - 1) ? 1 : 0;
  __syncthreads();
  if (!s_last) return;
  __threadfence();
#pragma unroll 8
  for (int e = tid; e < p.n_layers * p.batch; e += kPlanThreads) p.lens_after[e] = __ldcg(&p.new_lens[e]);
  if (tid == 0) {
    const int end = atomicExch(&p.hdr->plan_used, 0);
    if (p.used_after != nullptr) *p.used_after = max(end, used);
    p.hdr->plan_ticket = 0;
  }
}

// The same by one CTA, for a decode step's sizes: all lengths are read before any is written by a barrier instead of a
// count of CTAs, and nothing is read twice.  Where the tokens are many (two_launches) it leaves their slots and table
// entries to slots_kernel.
__global__ void __launch_bounds__(kSmallThreads) plan_small_kernel(const PlanParams p) {
  extern __shared__ long long s_tok64[];      // [units + 1] new tokens before each (layer, sequence)
  const int n_units = p.n_layers * p.batch;
  int32_t* s_start = reinterpret_cast<int32_t*>(s_tok64 + n_units + 1);   // [units]
  int32_t* s_len = s_start + n_units;                                     // [units]
  __shared__ long long s_red[32], s_red2[32];
  __shared__ int s_end[32];
  asm volatile("griddepcontrol.launch_dependents;");
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  constexpr int kPer = kSmallUnits / kSmallThreads;
  const int per = (n_units + kSmallThreads - 1) / kSmallThreads;
  int used = p.used_before != nullptr ? *p.used_before : 0;
  Ask a[kPer];
  long long ask = 0, add = 0;
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    const int e = tid * per + i;
    a[i] = {0, 0, 0, false};
    if (i < per && e < n_units) a[i] = plan_ask(p, e / p.batch, e, e % p.batch);
    ask += max(a[i].pages, 0);
    add += a[i].add;
  }
  if (used < 0 || used > p.n_free) {
    if (tid == 0) record_status(p.hdr, XKV_ERR_INVALID_ARG);
    used = p.n_free;
  }
  long long incl = ask, tincl = add;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const long long x = __shfl_up_sync(0xffffffffu, incl, o), y = __shfl_up_sync(0xffffffffu, tincl, o);
    if (lane >= o) {
      incl += x;
      tincl += y;
    }
  }
  if (lane == 31) {
    s_red[warp] = incl;
    s_red2[warp] = tincl;
  }
  __syncthreads();                            // also: every length has been read
  if (warp == 0) {
    long long x = s_red[lane], y = s_red2[lane];
    const long long x0 = x, y0 = y;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const long long u = __shfl_up_sync(0xffffffffu, x, o), v = __shfl_up_sync(0xffffffffu, y, o);
      if (lane >= o) {
        x += u;
        y += v;
      }
    }
    s_red[lane] = x - x0;
    s_red2[lane] = y - y0;
    if (lane == 31) s_tok64[n_units] = y;
  }
  __syncthreads();
  long long start = used + s_red[warp] + incl - ask, tok = s_red2[warp] + tincl - add;
  int end_max = used;
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    const int e = tid * per + i;
    if (i >= per || e >= n_units) break;
    const int pages = max(a[i].pages, 0);
    const bool fits = a[i].pages >= 0 && (pages == 0 || start + pages <= p.n_free);
    s_start[e] = fits ? (int)min(start, (long long)p.n_free) : -1;
    s_tok64[e] = tok;
    s_len[e] = a[i].len;
    if (p.two_launches) {
      p.ws_start[e] = s_start[e];
      p.ws_len[e] = a[i].len;
    }
    p.lens_after[e] = fits ? a[i].len + a[i].add : a[i].len;
    if (fits && pages > 0) end_max = max(end_max, (int)(start + pages));
    if (a[i].bad) record_status(p.hdr, XKV_ERR_INVALID_ARG);
    else if (!fits) record_status(p.hdr, XKV_ERR_CAPACITY);
    start += pages;
    tok += a[i].add;
    if (!fits) a[i].pages = 0;
  }
  end_max = (int)__reduce_max_sync(0xffffffffu, (unsigned)end_max);
  if (lane == 0) s_end[warp] = end_max;
  bool few = true;                            // no cache takes more than kStepTokens
#pragma unroll
  for (int i = 0; i < kPer; ++i) few = few && a[i].add <= kStepTokens;
  few = __syncthreads_and(few) != 0;
  if (tid == 0 && p.used_after != nullptr) {
    int end = s_end[0];
    for (int w = 1; w < 32; ++w) end = max(end, s_end[w]);
    *p.used_after = end;
  }
  // the new table entries of those of a warp's caches that have tokens without a place in the slot map, one after the other
  auto write_tables = [&]() {
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      const int e = tid * per + i;
      const bool mine = i < per && e < n_units &&
                        (p.slots == nullptr || s_tok64[e] + a[i].add - s_tok64[e / p.batch * p.batch] > p.slots_stride);
      const int pages = mine ? max(a[i].pages, 0) : 0;
      int32_t* at = p.block_table;
      if (pages > 0) at += (size_t)e * p.max_pages_per_seq + p.page_of(a[i].len + p.page_size - 1);
      unsigned todo = __ballot_sync(0xffffffffu, pages > 0);
      const int st = pages > 0 ? s_start[e] : 0;
      while (todo != 0) {
        const int w = __ffs(todo) - 1;
        todo &= todo - 1;
        write_pages(p, reinterpret_cast<int32_t*>(__shfl_sync(0xffffffffu, reinterpret_cast<unsigned long long>(at), w)),
                    __shfl_sync(0xffffffffu, pages, w), __shfl_sync(0xffffffffu, st, w));
      }
    }
  };
  if (p.slots == nullptr) {
    write_tables();
    return;
  }
  if (few && !p.two_launches) {
    // a decode step: every thread the tokens of its own caches, all page ids in flight together
    int page[kPer][kStepTokens];
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      const int e = tid * per + i, st = i < per && e < n_units ? s_start[e] : -1;
      const int have = p.page_of(a[i].len + p.page_size - 1);
#pragma unroll
      for (int k = 0; k < kStepTokens; ++k) {
        page[i][k] = -1;
        if (st < 0 || k >= a[i].add) continue;
        const int at = p.page_of(a[i].len + k);
        page[i][k] = at < have ? p.block_table[(size_t)e * p.max_pages_per_seq + at] : free_page(p, st + at - have);
      }
    }
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      const int e = tid * per + i;
      if (i >= per || e >= n_units) break;
      const int l = e / p.batch, st = s_start[e];
      const long long first = s_tok64[e] - s_tok64[l * p.batch];
      if (e - l * p.batch == p.batch - 1 && first + a[i].add > p.slots_stride) record_status(p.hdr, XKV_ERR_CAPACITY);
#pragma unroll
      for (int k = 0; k < kStepTokens; ++k) {
        if (k >= a[i].add) break;
        const int pos = a[i].len + k, at = p.page_of(pos), in_page = pos - at * p.page_size;
        const bool ok = (unsigned)page[i][k] < (unsigned)p.n_pages;
        if (st >= 0 && in_page == 0) p.block_table[(size_t)e * p.max_pages_per_seq + at] = page[i][k];   // the page is new
        if (st >= 0 && !ok) record_status(p.hdr, XKV_ERR_INVALID_ARG);
        if (first + k < p.slots_stride)
          p.slots[l * p.slots_stride + first + k] = ok ? (int64_t)page[i][k] * p.page_size + in_page : -1;
      }
    }
    return;
  }
  if (p.two_launches) {
    for (int i = tid; i < p.n_layers * (p.batch + 1); i += kSmallThreads) {
      const int l = i / (p.batch + 1), b = i - l * (p.batch + 1);
      p.ws_tok[i] = (int32_t)min(s_tok64[l * p.batch + b] - s_tok64[l * p.batch], 0x7fffffffll);
    }
    return;
  }
  write_tables();
  // the runs of the layers' slot maps, dealt out to the warps
  const int runs = (int)((p.slots_stride + kSlotRun - 1) / kSlotRun);
#pragma unroll 1
  for (int w = warp; w < p.n_layers * runs; w += kSmallThreads / 32) {
    const int l = w / runs, r = w % runs, e0 = l * p.batch;
    const long long first = s_tok64[e0], total = s_tok64[e0 + p.batch] - first;
    if (r == 0 && lane == 0 && total > p.slots_stride) record_status(p.hdr, XKV_ERR_CAPACITY);
    const int n_slots = (int)min(total, (long long)p.slots_stride);
    if (r * kSlotRun >= n_slots) continue;
    write_range(p, p.block_table + (size_t)e0 * p.max_pages_per_seq, p.slots + l * p.slots_stride, r * kSlotRun,
                min((r + 1) * kSlotRun, n_slots), [&](int b) { return s_tok64[e0 + b] - first; },
                [&](int b) { return s_start[e0 + b]; }, [&](int b) { return s_len[e0 + b]; });
  }
}

// Slots and new table entries from what plan_small_kernel found.  grid = (slices, layers), a stretch of tokens per warp.
__global__ void __launch_bounds__(kPlanThreads) slots_kernel(const PlanParams p) {
  extern __shared__ int32_t s_plan[];
  int32_t* s_tok = s_plan;                    // [batch + 1]
  int32_t* s_start = s_plan + p.batch + 1;    // [batch]
  int32_t* s_len = s_start + p.batch;         // [batch]
  const int tid = threadIdx.x, layer = blockIdx.y, n_warps = gridDim.x * (kPlanThreads / 32);
  asm volatile("griddepcontrol.wait;" ::: "memory");
  // (not through the read-only path: plan_small_kernel may write them while this kernel is resident already)
  for (int i = tid; i <= p.batch; i += kPlanThreads) {
    s_tok[i] = p.ws_tok[(size_t)layer * (p.batch + 1) + i];
    if (i < p.batch) {
      s_start[i] = p.ws_start[(size_t)layer * p.batch + i];
      s_len[i] = p.ws_len[(size_t)layer * p.batch + i];
    }
  }
  __syncthreads();
  const int total = s_tok[p.batch], n_slots = (int)min((int64_t)total, p.slots_stride);
  if (blockIdx.x == 0 && tid == 0 && total > p.slots_stride) record_status(p.hdr, XKV_ERR_CAPACITY);
  const int64_t stretch = ((int64_t)n_slots + n_warps - 1) / n_warps;
  const int64_t t0 = (blockIdx.x * (kPlanThreads / 32) + (tid >> 5)) * stretch;
  write_range(p, p.block_table + (size_t)layer * p.batch * p.max_pages_per_seq, p.slots + layer * p.slots_stride,
              (int)min(t0, (int64_t)n_slots), (int)min(t0 + stretch, (int64_t)n_slots),
              [&](int b) { return s_tok[b]; }, [&](int b) { return s_start[b]; }, [&](int b) { return s_len[b]; });
  if (total > p.slots_stride) {
    // the new table entries of sequences that have tokens without a place in the slot map: a warp per sequence
    for (int b = blockIdx.x * (kPlanThreads / 32) + (tid >> 5); b < p.batch; b += n_warps) {
      if (s_start[b] < 0 || s_tok[b + 1] <= p.slots_stride) continue;
      const int add = max(__ldg(&p.n_new[layer * p.n_new_stride + b]), 0);
      const int have = p.page_of(s_len[b] + p.page_size - 1), need = p.page_of(s_len[b] + add + p.page_size - 1);
      write_pages(p, p.block_table + ((size_t)layer * p.batch + b) * p.max_pages_per_seq + have, need - have, s_start[b]);
    }
  }
}

// ---------------------------------------------------------------------------------------------
// Rows stored by slot
// ---------------------------------------------------------------------------------------------
constexpr int kStoreThreads = 256;

struct StoreParams {
  const __nv_bfloat16* k;
  const __nv_bfloat16* v;
  const int64_t* slots;
  int64_t n_tokens, n_slots;
  int64_t stride_token, stride_head;
  uint8_t* k_pages;
  uint8_t* v_pages;
  float* k_scales;
  float* v_scales;
  int32_t n_kv_heads, page_size, tokens_per_warp;
  WorkspaceHeader* hdr;
};

// Whether up to 31 tokens of padding part token t, of slot s, from a token of the same block: another warp may be storing that
// one.  (Not inlined: nothing that runs often asks.)
__device__ __noinline__ bool behind_padding_of_its_block(const int64_t* slots, int64_t t, int64_t s) {
  if (s % kScaleBlock == 0) return false;
#pragma unroll 1
  for (int64_t i = t - 2; i >= 0 && i >= t - 32; --i) {
    const int64_t before = __ldg(&slots[i]);
    if (before >= 0) return before / kScaleBlock == s / kScaleBlock;
  }
  return false;
}

// One warp: the runs that begin among tokens_per_warp consecutive tokens, of one KV head of K or of V.  A run is the
// longest stretch of tokens whose slots follow each other inside one block; rows of the block before the run are there
// already, rows behind it are not in use.
template <int D>
__global__ void __launch_bounds__(kStoreThreads, 4) store_block_kernel(const StoreParams p) {
  const int lane = threadIdx.x & 31;
  const int64_t w = (int64_t)blockIdx.x * (kStoreThreads / 32) + (threadIdx.x >> 5);
  const int n_jobs = 2 * p.n_kv_heads;                        // (head, K or V) of a token
  const int64_t t0 = w / n_jobs * p.tokens_per_warp;
  const int job = (int)(w % n_jobs);
  const int h = job >> 1, is_v = job & 1;
  if (t0 >= p.n_tokens) return;
  // lane i: the slots of token t0 + i and of the one before it
  const int64_t ti = t0 + lane;
  int64_t s = -1, prev = -1;
  if (lane < p.tokens_per_warp && ti < p.n_tokens) {
    s = __ldg(&p.slots[ti]);
    if (ti > 0) prev = __ldg(&p.slots[ti - 1]);
    if (s >= p.n_slots) {
      if (job == 0) record_status(p.hdr, XKV_ERR_CAPACITY);
      s = -1;
    }
    if (s >= 0 && prev >= 0 && prev / kScaleBlock == s / kScaleBlock && prev + 1 != s) {
      if (job == 0) record_status(p.hdr, XKV_ERR_INVALID_ARG);   // a block's tokens are not in slot order
      s = -1;
    }
    if (s >= 0 && prev < 0 && behind_padding_of_its_block(p.slots, ti, s)) {
      if (job == 0) record_status(p.hdr, XKV_ERR_INVALID_ARG);
      s = -1;
    }
  }
  unsigned heads = __ballot_sync(0xffffffffu, s >= 0 && (s % kScaleBlock == 0 || prev + 1 != s));
  const __nv_bfloat16* src = is_v ? p.v : p.k;
  while (heads != 0) {
    const int first = __ffs(heads) - 1;
    heads &= heads - 1;
    const int64_t t = t0 + first;
    const int64_t slot = __shfl_sync(0xffffffffu, s, first);
    const int n_old = (int)(slot % kScaleBlock);
    // tokens of the run
    bool follows = false;
    if (lane < kScaleBlock - n_old && t + lane < p.n_tokens) follows = __ldg(&p.slots[t + lane]) == slot + lane;
    const int n_new = __ffs(~__ballot_sync(0xffffffffu, follows)) - 1;
    const int64_t page = slot / p.page_size, in_page = slot % p.page_size - n_old;
    const int64_t row = (page * p.n_kv_heads + h) * p.page_size + in_page;
    const __nv_bfloat16* rows = src + t * p.stride_token + h * p.stride_head;
    e4m3_store_block<D>((is_v ? p.v_pages : p.k_pages) + row * D, (is_v ? p.v_scales : p.k_scales) + row / kScaleBlock,
                        n_old, n_new, [&](int i) { return rows + i * p.stride_token; });
    __syncwarp();
  }
}

template <int D, bool Q8>
__global__ void __launch_bounds__(kStoreThreads) store_row_kernel(const StoreParams p) {
  constexpr int kPieces = D / 8;
  const int64_t idx = (int64_t)blockIdx.x * kStoreThreads + threadIdx.x;
  const int c = (int)(idx % kPieces);
  const int64_t r = idx / kPieces;
  const int h = (int)(r % p.n_kv_heads);
  const int64_t t = r / p.n_kv_heads;
  if (t >= p.n_tokens) return;                                // whole rows: a row's lanes leave together
  const int64_t slot = __ldg(&p.slots[t]);
  if (slot < 0) return;
  if (slot >= p.n_slots) {
    if (c == 0) record_status(p.hdr, XKV_ERR_CAPACITY);
    return;
  }
  const size_t src = (size_t)t * p.stride_token + (size_t)h * p.stride_head + c * 8;
  const uint4 kv = __ldg(reinterpret_cast<const uint4*>(p.k + src));
  const uint4 vv = __ldg(reinterpret_cast<const uint4*>(p.v + src));
  const size_t row = ((size_t)(slot / p.page_size) * p.n_kv_heads + h) * p.page_size + slot % p.page_size;
  if constexpr (Q8) {
    float x[8], ks, vs;
    bf16x8_to_f32(kv, x);
    const uint2 kc = quantize_row_piece(x, kPieces, &ks);
    bf16x8_to_f32(vv, x);
    const uint2 vc = quantize_row_piece(x, kPieces, &vs);
    *reinterpret_cast<uint2*>(p.k_pages + row * D + c * 8) = kc;
    *reinterpret_cast<uint2*>(p.v_pages + row * D + c * 8) = vc;
    if (c == 0) {
      p.k_scales[row] = ks;
      p.v_scales[row] = vs;
    }
  } else {
    *reinterpret_cast<uint4*>(p.k_pages + (row * D + c * 8) * 2) = kv;
    *reinterpret_cast<uint4*>(p.v_pages + (row * D + c * 8) * 2) = vv;
  }
}

// ---------------------------------------------------------------------------------------------
// One new row per (layer, sequence): grid = units, a warp per (KV head, K or V)
// ---------------------------------------------------------------------------------------------
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
  int32_t* clear;              // words that the attention launch behind this one wants at zero
  int32_t n_clear;
};

template <int D>
__global__ void __launch_bounds__(kStoreThreads) append_block_kernel(const AppendParams p) {
  asm volatile("griddepcontrol.launch_dependents;");          // that launch waits for this one before it reads a length
  for (int i = blockIdx.x * kStoreThreads + threadIdx.x; i < p.n_clear; i += gridDim.x * kStoreThreads) p.clear[i] = 0;
  const int e = blockIdx.x;
  const size_t le = (size_t)p.layer_begin * p.batch + e;
  const int n = p.seq_lens[le];
  int page = -1;
  if (n >= 0 && n < p.max_pages_per_seq * p.page_size) page = p.block_table[le * p.max_pages_per_seq + n / p.page_size];
  if (page < 0 || page >= p.n_pages) {
    if (threadIdx.x == 0) record_status(p.hdr, XKV_ERR_CAPACITY);
    return;
  }
  const int n_old = n % kScaleBlock;
  for (int job = threadIdx.x >> 5; job < 2 * p.n_kv_heads; job += kStoreThreads / 32) {
    const int h = job >> 1, is_v = job & 1;
    const int64_t row = ((int64_t)page * p.n_kv_heads + h) * p.page_size + (n % p.page_size - n_old);
    const __nv_bfloat16* src = (is_v ? p.v_new : p.k_new) + ((size_t)e * p.n_kv_heads + h) * D;
    e4m3_store_block<D>((is_v ? p.v_pages : p.k_pages) + row * D, (is_v ? p.v_scales : p.k_scales) + row / kScaleBlock,
                        n_old, 1, [&](int) { return src; });
  }
  __syncthreads();                                           // every warp has read the length
  if (threadIdx.x == 0) p.seq_lens[le] = n + 1;
}

// Shared memory of the plan kernels.
size_t small_smem(int n_units) { return (size_t)(n_units + 1) * 8 + (size_t)n_units * 8; }
size_t slots_smem(int batch) { return (size_t)(3 * batch + 1) * 4; }
size_t plan_smem(int batch) { return (size_t)(2 * batch + 1) * 4; }

// Opts in to the most shared memory that any call takes, once per device: the limit is one for all host threads, so that a
// call that set it to its own size could take away another thread's between that one's setting and its launch.
bool plan_set_up() {
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return false;
  static std::atomic<bool> done[64];   // idempotent: two threads doing it twice is harmless
  if (done[dev].load(std::memory_order_acquire)) return true;
  constexpr cudaFuncAttribute kMost = cudaFuncAttributeMaxDynamicSharedMemorySize;
  if (cudaFuncSetAttribute(plan_small_kernel, kMost, (int)small_smem(kSmallUnits)) != cudaSuccess ||
      cudaFuncSetAttribute(slots_kernel, kMost, (int)slots_smem(kSmallUnits)) != cudaSuccess ||
      cudaFuncSetAttribute(plan_kernel, kMost, (int)plan_smem(kPlanMaxBatch)) != cudaSuccess) {
    (void)cudaGetLastError();
    return false;
  }
  done[dev].store(true, std::memory_order_release);
  return true;
}

}  // namespace

size_t plan_workspace_bytes(int n_layers, int batch) {
  return kHeaderBytes + align_up(((size_t)n_layers * batch * 4 + n_layers) * 4, 256);
}

int plan_max_batch() { return kPlanMaxBatch; }

xkv_status plan_append(const xkv_cache* c, int batch, const int32_t* n_new, int n_new_stride, const int32_t* lens_before,
                       const int32_t* free_pages, int n_free, const int32_t* pages_used_before, int32_t* pages_used_after,
                       int64_t* slots, int64_t slots_stride, void* workspace, cudaStream_t st) {
  if (!plan_set_up()) return XKV_ERR_CUDA;
  PlanParams p;
  p.n_new = n_new;
  p.n_new_stride = n_new_stride;
  p.lens_before = lens_before;
  p.lens_after = c->seq_lens;
  p.free_pages = free_pages;
  p.n_free = n_free;
  p.used_before = pages_used_before;
  p.used_after = pages_used_after;
  p.block_table = c->block_table;
  p.slots = slots;
  p.slots_stride = slots_stride;
  p.n_layers = c->n_layers;
  p.batch = batch;
  p.page_size = c->page_size;
  p.max_pages_per_seq = c->max_pages_per_seq;
  p.n_pages = c->n_pages;
  const uint32_t d8 = (uint32_t)c->page_size / 8;
  p.page_mul = (uint32_t)(((1ull << 32) + d8 - 1) / d8);
  p.hdr = static_cast<WorkspaceHeader*>(workspace);
  p.two_launches = 0;
  p.new_lens = reinterpret_cast<int32_t*>(static_cast<uint8_t*>(workspace) + kHeaderBytes);
  const int64_t n_units = (int64_t)c->n_layers * batch;
  p.ws_tok = p.new_lens + n_units;
  p.ws_start = p.ws_tok + n_units + c->n_layers;
  p.ws_len = p.ws_start + n_units;
  const int64_t tokens = slots != nullptr ? slots_stride : 0;
  int64_t slices = (tokens + 4 * kPlanThreads - 1) / (4 * kPlanThreads);
  const int64_t most = std::max<int64_t>(1, 4 * (int64_t)sm_count() / c->n_layers);     // one wave
  slices = slices < 1 ? 1 : (slices > most ? most : slices);
  const dim3 grid((unsigned)slices, (unsigned)c->n_layers);
  if (n_units <= kSmallUnits) {
    // One CTA finds out who gets what; it also writes the slots where they are few.  One launch against two, device time
    // of layers x sequences x new tokens: steps 4 x 1 x 1: 3.2 / 4.3 us, 32 x 8 x 1: 3.3 / 4.7, 32 x 64 x 1: 5.5 / 7.0, 32 x 120 x 1:
    // 9.1 / 10.1; more tokens a cache 4 x 1 x 300: 4.2 / 4.5, 32 x 4 x 16: 5.0 / 4.5, 4 x 1 x 1000: 6.5 / 4.7, 32 x 64 x 4: 15.2 / 6.8.
    p.two_launches = c->n_layers * tokens > kSmallTokens ? 1 : 0;
    plan_small_kernel<<<1, kSmallThreads, small_smem((int)n_units), st>>>(p);
    count_launch();
    xkv_status s = check_launch();
    if (s != XKV_OK || !p.two_launches) return s;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = dim3(kPlanThreads);
    cfg.dynamicSmemBytes = slots_smem(batch);
    cfg.stream = st;
    cudaLaunchAttribute attr;                 // its CTAs are in place when the first launch ends
    attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr.val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = &attr;
    cfg.numAttrs = 1;
    if (cudaLaunchKernelEx(&cfg, slots_kernel, p) != cudaSuccess) {
      (void)cudaGetLastError();
      return XKV_ERR_CUDA;
    }
    count_launch();
    return check_launch();
  }
  plan_kernel<<<grid, kPlanThreads, plan_smem(batch), st>>>(p);
  count_launch();
  return check_launch();
}

size_t store_workspace_bytes() { return kHeaderBytes; }

xkv_status store_rows(const xkv_dims* d, const xkv_cache* c, const void* k, const void* v, const int64_t* slots,
                      int64_t n_tokens, void* workspace, cudaStream_t st) {
  StoreParams p;
  p.k = static_cast<const __nv_bfloat16*>(k);
  p.v = static_cast<const __nv_bfloat16*>(v);
  p.slots = slots;
  p.n_tokens = n_tokens;
  p.n_slots = (int64_t)c->n_pages * c->page_size;
  p.stride_token = d->kv_stride_token;
  p.stride_head = d->kv_stride_head;
  p.k_pages = static_cast<uint8_t*>(c->k_pages);
  p.v_pages = static_cast<uint8_t*>(c->v_pages);
  p.k_scales = c->k_scales;
  p.v_scales = c->v_scales;
  p.n_kv_heads = d->n_kv_heads;
  p.page_size = c->page_size;
  p.hdr = static_cast<WorkspaceHeader*>(workspace);
  if (c->kv_format == XKV_KV_E4M3) {
    // A warp looks for runs among 1, 4 or 16 tokens and takes them one after the other.  Few tokens: one each (a decode
    // step: every token is a run of its own); many: more, so that few warps start only to find no run (a prompt: one run
    // in 16 tokens).  Measured with 1 / 4 / 16, 8 heads of 128: step of 64 tokens 2.9 / 6.3 / 19.6 us, of 600 7.7 / 8.4 / 20.5, of
    // 4000 37 / 31 / 36; prompts of 1000 tokens 5.8 / 4.1 / 3.0 us, of 4 x 2048 26.0 / 12.3 / 7.4.
    const int64_t jobs = n_tokens * 2 * d->n_kv_heads;
    p.tokens_per_warp = jobs <= 64 * (int64_t)sm_count() ? 1 : (jobs <= 448 * (int64_t)sm_count() ? 4 : kScaleBlock);
    const int64_t warps = (n_tokens + p.tokens_per_warp - 1) / p.tokens_per_warp * 2 * d->n_kv_heads;
    const int64_t grid = (warps + kStoreThreads / 32 - 1) / (kStoreThreads / 32);
    if (grid > 0x7fffffffll) return XKV_ERR_UNSUPPORTED;
    if (d->head_dim == 128) store_block_kernel<128><<<(unsigned)grid, kStoreThreads, 0, st>>>(p);
    else                    store_block_kernel<64><<<(unsigned)grid, kStoreThreads, 0, st>>>(p);
  } else {
    p.tokens_per_warp = 0;
    const int64_t threads = n_tokens * d->n_kv_heads * (d->head_dim / 8);
    const int64_t grid = (threads + kStoreThreads - 1) / kStoreThreads;
    if (grid > 0x7fffffffll) return XKV_ERR_UNSUPPORTED;
    const bool q8 = c->kv_format == XKV_KV_INT8;
    if (d->head_dim == 128) {
      if (q8) store_row_kernel<128, true><<<(unsigned)grid, kStoreThreads, 0, st>>>(p);
      else    store_row_kernel<128, false><<<(unsigned)grid, kStoreThreads, 0, st>>>(p);
    } else {
      if (q8) store_row_kernel<64, true><<<(unsigned)grid, kStoreThreads, 0, st>>>(p);
      else    store_row_kernel<64, false><<<(unsigned)grid, kStoreThreads, 0, st>>>(p);
    }
  }
  count_launch();
  return check_launch();
}

xkv_status append_e4m3(const xkv_dims* d, const xkv_cache* c, int layer_begin, int n_units, const void* k_new,
                       const void* v_new, void* workspace, int32_t* clear, int n_clear, cudaStream_t st) {
  AppendParams p;
  p.clear = clear;
  p.n_clear = n_clear;
  p.k_new = static_cast<const __nv_bfloat16*>(k_new);
  p.v_new = static_cast<const __nv_bfloat16*>(v_new);
  p.k_pages = static_cast<uint8_t*>(c->k_pages);
  p.v_pages = static_cast<uint8_t*>(c->v_pages);
  p.k_scales = c->k_scales;
  p.v_scales = c->v_scales;
  p.block_table = c->block_table;
  p.seq_lens = c->seq_lens;
  p.layer_begin = layer_begin;
  p.batch = d->batch;
  p.n_kv_heads = d->n_kv_heads;
  p.page_size = c->page_size;
  p.max_pages_per_seq = c->max_pages_per_seq;
  p.n_pages = c->n_pages;
  p.hdr = static_cast<WorkspaceHeader*>(workspace);
  if (d->head_dim == 128) append_block_kernel<128><<<n_units, kStoreThreads, 0, st>>>(p);
  else                    append_block_kernel<64><<<n_units, kStoreThreads, 0, st>>>(p);
  count_launch();
  return check_launch();
}

}  // namespace xkv
