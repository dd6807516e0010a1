// Attention of ragged prompts over expanded keys and values (include/qmla.h,
// qmla_mla_prefill): 128 content channels and 64 shared RoPE channels in QK, 128
// in PV.
//
// plan_kernel cuts every sequence into items of 256 query rows and orders them,
// the longest first; prefill_kernel (persistent, one CTA per SM) draws (item, head)
// pairs from that list. A short call (kUnplanned, kUnplannedRows, kUnplannedKeys) has
// no plan: its CTAs work their items out of the offsets. In a CTA the two 128-row tiles
// of an item take turns on the tensor core: while one tile's scores are turned into
// weights, the other's MMAs run (PV of the old keys, QK of the next). An item of one
// tile (a short prompt, a sequence's last rows) has its keys dealt to the two in turn
// instead: both hold the same rows, every other key step each, and are merged at the
// end.
//
//   warps 0..3 / 4..7   softmax of tile 0 / 1, a query row per thread
//   warps 8..11         epilogue of both tiles
//   warps 12, 14        one thread each, which issues tile 0's / tile 1's MMAs
//   warp 13             TMA loads of queries, keys and values
//   warp 15             draws the pairs
//
// The roles run through the pairs without a stop between them: a pair's first QK and
// softmax run while the O of the one before is read out, and only its first PV waits
// for that (o_free).
//
// Shared memory: the queries (2 x 3 chunks of 128 rows x 64 channels, 96 KB) and a
// ring of eight 16 KB slots for keys (three slots per 128 tokens: two content
// chunks, one RoPE chunk) and values (two slots, 64 tokens x 128 channels each).
// TMEM: S0, S1 (fp32, 128 columns each; the bf16 weights overwrite the first half
// of their scores) and O0, O1.
//
// Mathematics: online softmax. Row r keeps a reference m and the sum l of
// 2^(s - m) over the keys seen; O accumulates P V with P = RN_bf16(2^(s - m)). m is
// raised, and O and l rescaled, only when a score exceeds it by more than 2^8: the
// weights then stay below 2^8, which fp32 sums and bf16 weights, being floating point,
// hold as well as weights below one.
#include <cuda.h>
#include <cuda_runtime.h>

#include <algorithm>

#include "common.cuh"
#include "kernels.h"
#include "ptx.cuh"

namespace qmla {
namespace {

constexpr int kDn = 128;               // content channels of a query and key head
constexpr int kDv = 128;               // channels of a value head
constexpr int kTile = 128;             // query rows of a tile, keys of a step
constexpr int kItemRows = 2 * kTile;   // query rows of an item
constexpr int kSlotBytes = 16384;      // 128 rows of 64 channels, or 64 tokens of 128
constexpr int kQChunks = 3, kKChunks = 3, kVSlots = 2;
constexpr int kRing = 8;
constexpr int kInFlight = 3;  // entries (a step's keys or values) that the ring holds at once
constexpr int kSoftWarps = 8;
constexpr int kEpiWarp = 8, kMmaWarp = 12, kLoadWarp = 13, kDrawWarp = 15;  // (and 14: MMAs)
constexpr int kThreads = 16 * 32;
// 128 registers a thread at launch: 2 x 160 + 96 + 96 = 4 x 128.
constexpr int kSoftRegs = 160, kEpiRegs = 96, kOtherRegs = 96;
constexpr int kRingOff = 2 * kQChunks * kSlotBytes;
constexpr int kCtlOff = kRingOff + kRing * kSlotBytes;
constexpr uint32_t kColO = 256;  // O0; O1 128 columns on
constexpr uint64_t kLimitNs = 2000000000ull;  // of every wait (a pair of 2^26 keys takes 0.8 s)
constexpr int kAhead = 4;  // steps before the end of a pair at which the next is drawn
constexpr float kRaise = 8.0f;  // log2 of the growth that raises a reference

// Wait sites in the error word (bits 8 ..), after the decode's.
enum : uint32_t { kSiteLoad = 10, kSiteMma, kSiteSoftmax, kSiteEpilogue, kSiteEnd };

struct Ctl {
  uint64_t q_full[2], q_free[2];
  uint64_t full[4], freed[4];  // of entry e: [e & 3]
  uint64_t s_full[2], p_full[2][2], o_full[2];  // p_full: of the halves, 64 keys each
  uint64_t l_full[2], o_free[2];  // a tile's (m, l) are in `sums`; they and O have been read
  uint64_t sched_full[2], sched_free[2], ask;  // ask: the load warp wants the next pair
  uint64_t tail, fin;
  uint32_t tmem_base, abort;
  int turn;  // 1: a tile's MMAs are being issued
  int4 work[2][4];
  float2 sums[2][kTile];  // (m, l) of the tiles' rows
};
constexpr int kSmem = kCtlOff + static_cast<int>(sizeof(Ctl));
static_assert(kSmem <= 232448, "shared memory of a CTA");

// Two tiles of one sequence: rows q_row .. of q, `rows` of them (at most 256); keys
// kv_start .. + kv_len. Row r sees the first min(kv_len, vis0 + r * step) keys.
// Items that lie side by side in a sequence form bundles: the list holds a bundle's
// items for one head, then for the next, so that they meet the same keys in L2.
struct Item {
  int q_row, rows, kv_start, kv_len;
  int vis0, step, n0, n1;  // n0, n1: key steps of the tiles (dealt: of the one tile, 0)
  int first, bundle;       // the bundle's first item and its length
  int head;                // (of a pair; -1: no more)
  int dealt;               // one tile, whose key steps the two tiles share out
  int part, parts;         // a long item's keys go in parts, each an item of its own
  int slot;                // parts > 1: first of the heads x parts partial results
  int unused;
};
static_assert(sizeof(Item) == 64, "four 16-byte loads");

// Keys are cut into parts where one pair would take half as long again as the SMs' fair
// share of the whole call: parts of at most L rounds, L >= W / kShares, W all the rounds,
// and kLeastPart at least. An item of R > L rounds makes ceil(R / L) < 2 R / L parts, so
// there are never more than 2 kShares partial results, nor more than kShares items cut up.
// L itself: parts of W / SMs rounds can be a few more than SMs, which then takes two turns
// of L, so some longer ones are weighed against it (kLengths). What that does, us, with L alone
// and weighed: 16 heads, 512 rows over 16,896 keys 114 / 84 (160 parts, then 128), 200 over
// 20,200 80 / 61, 1 over 50,001 106 / 78, 50 over 9,050 29.2 / 31.2 (the weighing does not count
// what a longer part costs where the parts are few rounds); 24 heads, 700 over 9,700 122 / 97;
// 32 heads, two of 128 over 12,128 103 / 88; 8 heads, 300 over 30,300 68.1 / 68.6.
constexpr int kShares = 160, kSlots = 2 * kShares, kLeastPart = 4, kLengths = 4;
struct Join {  // an item cut up
  int q_row, rows, slot, parts;
};
struct Partial {  // of a part and head: rows of the item
  float o[kItemRows][kDv];   // unnormalised
  float2 ml[kItemRows];      // reference (log2) and sum
};

struct Workspace {
  size_t prefix_off, items_off, join_off, part_off, total;
  int max_items, max_entries;
};
Workspace workspace_layout(int batch, int n_q) {
  Workspace w;
  w.max_items = n_q / kItemRows + batch;  // disjoint sequences have no more
  w.prefix_off = 256;                     // ints: items written, pairs drawn beyond one per CTA, joins
  w.items_off = (w.prefix_off + 4 * (static_cast<size_t>(batch) + 1) + 255) / 256 * 256;
  w.max_entries = w.max_items + kSlots;
  w.join_off = w.items_off + sizeof(Item) * static_cast<size_t>(w.max_entries);
  w.part_off = (w.join_off + sizeof(Join) * kShares + 255) / 256 * 256;
  w.total = w.part_off + sizeof(Partial) * kSlots;
  return w;
}

// ------------------------------------------------------------------------- plan
// One block of kPlanThreads, or of kSmallPlan where that many sequences and items at
// most can come up: a small call's time is the plan's chain of latencies.
constexpr int kPlanThreads = 1024, kSmallPlan = 64;
// Sequences, rows and keys of a call without a plan, at most.
constexpr int kUnplanned = 64, kUnplannedRows = 65536, kUnplannedKeys = 2048;
constexpr int kPlanOnChip = 2048;  // sequences whose prefix is kept in shared memory

struct Sum {
  __device__ __forceinline__ int operator()(int a, int b) const { return a + b; }
};
struct Largest {
  __device__ __forceinline__ int operator()(int a, int b) const { return max(a, b); }
};
// Exclusive prefix of v >= 0 over the block under op, and the total.
template <class Op>
__device__ __forceinline__ int block_scan(int v, int* warp_totals, int& total, Op op) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
  int x = v;
#pragma unroll
  for (int off = 1; off < 32; off <<= 1) {
    const int y = __shfl_up_sync(0xffffffffu, x, off);
    if (lane >= off) x = op(x, y);
  }
  if (lane == 31) warp_totals[warp] = x;
  __syncthreads();
  int s = lane < warps ? warp_totals[lane] : 0;
#pragma unroll
  for (int off = 1; off < 32; off <<= 1) {
    const int y = __shfl_up_sync(0xffffffffu, s, off);
    if (lane >= off) s = op(s, y);
  }
  total = __shfl_sync(0xffffffffu, s, 31);
  const int before = __shfl_sync(0xffffffffu, s, warp == 0 ? 0 : warp - 1);
  const int in_warp = __shfl_up_sync(0xffffffffu, x, 1);
  __syncthreads();
  return op(warp == 0 ? 0 : before, lane == 0 ? 0 : in_warp);
}

// The item of rows r0 .. of a sequence of lq queries and lk keys.
__device__ __forceinline__ Item make_item(int q0, int lq, int k0, int lk, int r0, int causal) {
  Item it = {};
  it.q_row = q0 + r0;
  it.rows = min(lq - r0, kItemRows);
  it.kv_start = k0;
  it.kv_len = lk;
  it.vis0 = causal ? r0 + lk - lq + 1 : lk;
  it.step = causal ? 1 : 0;
  const int last0 = min(it.rows, kTile) - 1, last1 = it.rows - 1;
  it.n0 = (max(min(lk, it.vis0 + it.step * last0), 0) + kTile - 1) / kTile;
  it.n1 = it.rows > kTile ? (max(min(lk, it.vis0 + it.step * last1), 0) + kTile - 1) / kTile : 0;
  it.dealt = it.rows <= kTile && it.n0 > 1 ? 1 : 0;
  it.parts = 1;
  return it;
}
// Whether a sequence's offsets are within the rows given. Where a sequence's offsets
// decrease, good ones can overlap: of those, what begins before an earlier one's end is left
// out, so that the sequences worked on are disjoint, and have no more items than there is
// room for.
__device__ __forceinline__ bool good_offsets(int q0, int q1, int k0, int k1, int n_q, int n_kv) {
  return q0 >= 0 && q1 >= q0 && q1 <= n_q && k0 >= 0 && k1 >= k0 && k1 <= n_kv;
}

// Rounds of an item: key steps of its longer tile. Dealt, two of one tile's steps make a
// round, but they load twice as many keys and take half as long again.
__device__ __forceinline__ int rounds_of(const Item& it) {
  return it.rows <= kTile ? (3 * it.n0 + 3) >> 2 : max(it.n0, it.n1);
}

// One block. A sequence has ceil(Lq / 256) items, in bundles of `bundle`; a counting
// sort by key steps puts the longest bundles first (the order among equals is free:
// items do not meet). Passes: the rounds of all items; the parts that each length in
// question makes; the sizes of the buckets; the list.
__global__ void __launch_bounds__(kPlanThreads) plan_kernel(const int32_t* __restrict__ cu_q,
                                                            const int32_t* __restrict__ cu_kv, int batch, int n_q,
                                                            int n_kv, int heads, int causal, int sms, int bundle,
                                                            int shift, int* __restrict__ count,
                                                            int* __restrict__ prefix_far, Item* __restrict__ items,
                                                            Join* __restrict__ joins, uint32_t* dev_err) {
  __shared__ int warp_totals[32];
  __shared__ int bucket[kPlanThreads];  // (as many as threads)
  __shared__ int prefix_near[kPlanOnChip];
  __shared__ unsigned long long rounds;
  __shared__ int entries, slots, cut, most;  // most: rounds of the longest item
  __shared__ unsigned long long cut_rounds[kLengths], cut_parts[kLengths];
  griddep_launch_dependents();  // prefill_kernel may start its set-up meanwhile
  const int tid = threadIdx.x, threads = blockDim.x;
  int* prefix = batch <= kPlanOnChip ? prefix_near : prefix_far;
  bucket[tid] = 0;
  if (tid == 0) {
    rounds = 0;
    entries = slots = cut = most = 0;
  }
  if (tid < kLengths) cut_rounds[tid] = cut_parts[tid] = 0;
  int bundles = 0, reach = 0;  // reach: where the earlier sequences with good offsets end
  bool any_bad = false;
  for (int b0 = 0; b0 < batch; b0 += threads) {
    const int b = b0 + tid;
    int q0 = 0, q1 = 0;
    bool good = false;
    if (b < batch) {
      q0 = cu_q[b], q1 = cu_q[b + 1];
      good = good_offsets(q0, q1, cu_kv[b], cu_kv[b + 1], n_q, n_kv);
    }
    if (__syncthreads_or(b < batch && !good) || any_bad) {
      if (!any_bad && b0 > 0) reach = cu_q[b0];  // (none was bad: they do not decrease)
      any_bad = true;
      int end;
      const int before = block_scan(good ? q1 : 0, warp_totals, end, Largest{});
      good = good && q0 >= max(reach, before);
      reach = max(reach, end);
      if (b < batch && !good) report(dev_err, QMLA_DEVERR_BAD_OFFSETS);
    }
    const int tiles = good ? (q1 - q0 + kItemRows - 1) / kItemRows : 0;
    int sum;
    const int at = block_scan((tiles + bundle - 1) / bundle, warp_totals, sum, Sum{});
    if (b < batch) prefix[b] = bundles + at;
    bundles += sum;
  }
  __syncthreads();
  int longest = INT32_MAX;  // rounds of a part
  // W / SMs and 1.15, 1.35 and 1.7 times that (in fp32: off by less than the step from
  // kShares - 1 to kShares)
  auto length = [&](int x) {
    const float f = x == 0 ? 1.0f : (x == 1 ? 1.15f : (x == 2 ? 1.35f : 1.7f));
    const float l = __ull2float_rn(rounds) * f / static_cast<float>(min(sms, kShares - 1));
    return max(static_cast<int>(fminf(l, 1e9f)) + 1, kLeastPart);
  };
  auto parts_at = [](int r, int l) { return r - l > l >> 1 ? (r + l - 1) / l : 1; };
  struct Place {  // of a bundle: its sequence, first item and length
    int q0, lq, k0, lk, t0, k;
  };
  auto find = [&](int i) {
    int lo = 0, hi = batch - 1;  // the last sequence with prefix <= i: it has items
    while (lo < hi) {
      const int mid = (lo + hi + 1) >> 1;
      if (prefix[mid] <= i) {
        lo = mid;
      } else {
        hi = mid - 1;
      }
    }
    Place x;
    x.q0 = cu_q[lo];
    x.lq = cu_q[lo + 1] - x.q0;
    x.k0 = cu_kv[lo];
    x.lk = cu_kv[lo + 1] - x.k0;
    x.t0 = (i - prefix[lo]) * bundle;
    x.k = min(bundle, (x.lq + kItemRows - 1) / kItemRows - x.t0);
    return x;
  };
  const Place first_place = tid < bundles ? find(tid) : Place{};
#pragma unroll 1
  for (int pass = 0; pass < 4; ++pass) {
    unsigned long long mine = 0;
    for (int i = tid; i < bundles; i += threads) {
      const Place at_i = i == tid ? first_place : find(i);
      const int q0 = at_i.q0, lq = at_i.lq, k0 = at_i.k0, lk = at_i.lk, t0 = at_i.t0, k = at_i.k;
      // (the last item stands first: it has the most keys. With one tile, whose rounds count
      // 3/4, it can still be shorter than the one before it, which then is the longest.)
      auto item = [&](int x) { return make_item(q0, lq, k0, lk, (t0 + k - 1 - x) * kItemRows, causal); };
      auto parts_of = [&](const Item& it) { return parts_at(rounds_of(it), longest); };
      int all = 0;  // entries of the bundle
      for (int x = 0; x < k; ++x) {
        const Item it = item(x);
        const int r = rounds_of(it);
        if (pass == 0) {
          mine += static_cast<unsigned long long>(r) * heads;
          if (x < 2) atomicMax(&most, r);
        } else if (pass == 1) {
#pragma unroll 1
          for (int c = 0; c < kLengths; ++c) {
            const int parts = parts_at(r, length(c));
            if (parts > 1) {
              atomicAdd(&cut_rounds[c], static_cast<unsigned long long>(r) * heads);
              atomicAdd(&cut_parts[c], static_cast<unsigned long long>(parts) * heads);
            }
          }
        } else {
          all += parts_of(it);
        }
      }
      if (pass < 2) continue;
      const int top = k > 1 ? max(rounds_of(item(0)), rounds_of(item(1))) : rounds_of(item(0));
      const int key = threads - 1 - min(min(top, longest) >> shift, threads - 1);
      int at = atomicAdd(&bucket[key], all);
      if (pass == 2) {
        atomicAdd(&entries, all);
        continue;
      }
      const int first = at;
      for (int x = 0; x < k; ++x) {
        const Item whole = item(x);
        // (dealt: an even number of steps, so that both tiles have as many)
        const int parts = parts_of(whole), steps = max(whole.n0, whole.n1);
        const int per = whole.rows <= kTile ? ((steps + 2 * parts - 1) / (2 * parts)) * 2 : (steps + parts - 1) / parts;
        int slot = 0;
        if (parts > 1) {
          slot = atomicAdd(&slots, parts * heads);
          joins[atomicAdd(&cut, 1)] = Join{whole.q_row, whole.rows, slot, parts};
        }
        for (int y = 0; y < parts; ++y, ++at) {
          // A part is the item without the keys before it.
          Item it = whole;
          const int skip = parts > 1 ? y * per : 0;
          it.kv_start += skip * kTile;
          it.kv_len -= skip * kTile;
          it.vis0 -= skip * kTile;
          it.n0 = max(0, min(whole.n0 - skip, parts > 1 ? per : whole.n0));
          it.n1 = max(0, min(whole.n1 - skip, parts > 1 ? per : whole.n1));
          it.first = first;
          it.bundle = all;
          it.head = 0;
          it.dealt = it.rows <= kTile && it.n0 > 1 ? 1 : 0;
          it.part = y;
          it.parts = parts;
          it.slot = slot;
          it.unused = 0;
          items[at] = it;
        }
      }
    }
    if (pass == 0) {
#pragma unroll
      for (int off = 16; off > 0; off >>= 1) mine += __shfl_xor_sync(0xffffffffu, mine, off);
      if ((tid & 31) == 0) atomicAdd(&rounds, mine);
    }
    __syncthreads();
    if (pass == 0) {
      longest = length(0);
      if (parts_at(most, longest) == 1) ++pass;  // (no item is cut up)
    } else if (pass == 1) {
      // Turns of the SMs times the length; items that stay whole fill the last turn up.
      float best = INFINITY;
#pragma unroll 1
      for (int c = 0; c < kLengths; ++c) {
        const int l = length(c);
        const unsigned long long parts = cut_parts[c];
        const float turns = parts == 0 || (rounds - cut_rounds[c]) * 4 > rounds
                                ? 1.0f
                                : static_cast<float>((static_cast<int>(parts) + sms - 1) / sms);
        if (turns * static_cast<float>(l) < best) {
          best = turns * static_cast<float>(l);
          longest = l;
        }
      }
    } else if (pass == 2) {
      int sum;
      const int before = block_scan(bucket[tid], warp_totals, sum, Sum{});
      bucket[tid] = before;
      __syncthreads();
    }
  }
  if (tid == 0) {
    count[0] = entries;
    count[1] = 0;
    count[2] = cut;
  }
}

// ------------------------------------------------------------------------ main
struct PrefillParams {
  int* count;  // [0] items, [1] pairs drawn beyond one per CTA, [2] joins
  const Item* items;
  int heads;
  float scale_log2;
  uint16_t* out;
  float* lse;
  Partial* partial;
  bool join;  // join_kernel follows
  bool unplanned;  // no plan_kernel: the draw warps work the pairs out (at most kUnplanned sequences)
  const int32_t* cu_q;
  const int32_t* cu_kv;
  int batch, n_q, n_kv, causal;
  uint32_t* dev_err;
};

__device__ __forceinline__ void give_up(Ctl& c, uint32_t* dev_err, uint32_t site) {
  report(dev_err, QMLA_DEVERR_TIMEOUT | (0x100u << site));
  *reinterpret_cast<volatile uint32_t*>(&c.abort) = 1u;
}
// One thread's bounded wait. (Each probe sleeps for up to 100 us; the clock is read
// between them only.)
__device__ __forceinline__ bool wait1(uint64_t* bar, uint32_t parity, Ctl& c, uint32_t site, uint32_t* dev_err) {
  uint64_t t0 = 0;
#pragma unroll 1
  while (!mbar_try_wait(bar, parity & 1u)) {
    if (*reinterpret_cast<volatile uint32_t*>(&c.abort) != 0u) return false;
    const uint64_t t = globaltimer_ns();
    if (t0 == 0) t0 = t;
    if (t - t0 > kLimitNs) {
      give_up(c, dev_err, site);
      return false;
    }
  }
  return true;
}
// A whole warp's (every lane waits on the barrier itself).
__device__ __forceinline__ bool wait_warp(uint64_t* bar, uint32_t parity, Ctl& c, uint32_t site, uint32_t* dev_err) {
  return __all_sync(0xffffffffu, wait1(bar, parity, c, site, dev_err));
}

// The pair at hand, k-th of this CTA: read from shared memory, where the draw warp
// leaves it. For whole warps (LANES) and single threads.
template <bool LANES>
__device__ __forceinline__ bool next_pair(Ctl& c, uint32_t k, Item& it, uint32_t site, uint32_t* dev_err) {
  uint64_t* bar = &c.sched_full[k & 1u];
  if (!(LANES ? wait_warp(bar, k >> 1, c, site, dev_err) : wait1(bar, k >> 1, c, site, dev_err))) return false;
  const int4 x = c.work[k & 1u][0], y = c.work[k & 1u][1], z = c.work[k & 1u][2], v = c.work[k & 1u][3];
  it = Item{x.x, x.y, x.z, x.w, y.x, y.y, y.z, y.w, z.x, z.y, z.z, z.w, v.x, v.y, v.z, v.w};
  if (LANES) __syncwarp();
  mbar_arrive_if(!LANES || (threadIdx.x & 31) == 0 ? 1u : 0u, &c.sched_free[k & 1u]);
  return it.head >= 0;
}

// An entry of the ring: the keys (three slots) or the values (two) of a key step.
// Three entries are on their way at once; no three in a row are all keys, so they
// fit into the eight slots.
struct Entry {
  uint32_t e = 0, slot = 0;
  __device__ __forceinline__ void next(uint32_t slots) {
    ++e;
    slot = (slot + slots) & 7u;
  }
};

// The item that is the i-th of all (64 sequences at most, two to a lane: tiles and
// prefix are their items and the prefix's end), or none.
struct Few {
  int q0[2], lq[2], k0[2], lk[2], tiles[2], end[2];
  __device__ __forceinline__ int init(const PrefillParams& p, int lane) {
    int total = 0, reach = 0;  // reach: as in plan_kernel
    bool any_bad = false;
    int q1[2];
    bool in_range[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {  // (all loads first)
      const int b = 32 * h + lane;
      q0[h] = lq[h] = k0[h] = lk[h] = tiles[h] = q1[h] = 0;
      in_range[h] = false;
      if (b < p.batch) {
        q1[h] = p.cu_q[b + 1];
        const int k1 = p.cu_kv[b + 1];
        q0[h] = p.cu_q[b];
        k0[h] = p.cu_kv[b];
        lq[h] = q1[h] - q0[h];
        lk[h] = k1 - k0[h];
        in_range[h] = good_offsets(q0[h], q1[h], k0[h], k1, p.n_q, p.n_kv);
      }
    }
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int b = 32 * h + lane;
      bool good = in_range[h];
      if (__any_sync(0xffffffffu, b < p.batch && !good) || any_bad) {
        if (!any_bad && h > 0) reach = __shfl_sync(0xffffffffu, q0[h], 0);
        any_bad = true;
        int x = good ? q1[h] : 0;
#pragma unroll
        for (int off = 1; off < 32; off <<= 1) {
          const int y = __shfl_up_sync(0xffffffffu, x, off);
          if (lane >= off) x = max(x, y);
        }
        const int before = __shfl_up_sync(0xffffffffu, x, 1);
        good = good && q0[h] >= max(reach, lane == 0 ? 0 : before);
        reach = max(reach, __shfl_sync(0xffffffffu, x, 31));
        if (b < p.batch && !good && blockIdx.x == 0) report(p.dev_err, QMLA_DEVERR_BAD_OFFSETS);
      }
      if (good) tiles[h] = (lq[h] + kItemRows - 1) / kItemRows;
      int x = tiles[h];
#pragma unroll
      for (int off = 1; off < 32; off <<= 1) {
        const int y = __shfl_up_sync(0xffffffffu, x, off);
        if (lane >= off) x += y;
      }
      end[h] = total + x;
      total = __shfl_sync(0xffffffffu, end[h], 31);
    }
    return total;
  }
  __device__ __forceinline__ Item item(int i, int causal) const {
    Item it = {};
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const uint32_t behind = __ballot_sync(0xffffffffu, end[h] > i);
      if (behind == 0u || (h == 1 && it.parts != 0)) continue;
      const int from = __ffs(behind) - 1;
      auto of = [&](int v) { return __shfl_sync(0xffffffffu, v, from); };
      // (a sequence's last item, the longest, first)
      it = make_item(of(q0[h]), of(lq[h]), of(k0[h]), of(lk[h]), (of(end[h]) - 1 - i) * kItemRows, causal);
    }
    return it;
  }
};

// Draws the CTA's pairs: pair c first, then whichever is next when the load warp asks
// for it. (A draw is three round trips to L2.) Without a plan every SMs-th pair.
__device__ void draw_role(const PrefillParams& p, Ctl& ctl, int lane) {
  const int4* list = reinterpret_cast<const int4*>(p.items);
  Few few;
  const int pairs = (p.unplanned ? few.init(p, lane) : p.count[0]) * p.heads;
  int at = static_cast<int>(blockIdx.x);
  for (uint32_t k = 0;; ++k) {
    if (k > 0) {
      if (!wait_warp(&ctl.ask, k - 1, ctl, kSiteLoad, p.dev_err)) return;
      if (p.unplanned) {
        at += static_cast<int>(gridDim.x);
      } else {
        if (lane == 0) at = static_cast<int>(gridDim.x) + atomicAdd(p.count + 1, 1);
        at = __shfl_sync(0xffffffffu, at, 0);
      }
    }
    int4 w = make_int4(0, 0, -1, 0);  // lane l < 4: the l-th quarter of the item
    const bool more = at < pairs;
    if (more && p.unplanned) {
      Item it = few.item(at / p.heads, p.causal);
      it.head = at % p.heads;
      w = lane == 0   ? make_int4(it.q_row, it.rows, it.kv_start, it.kv_len)
          : lane == 1 ? make_int4(it.vis0, it.step, it.n0, it.n1)
          : lane == 2 ? make_int4(it.first, it.bundle, it.head, it.dealt)
                      : make_int4(it.part, it.parts, it.slot, it.unused);
    } else if (more) {
      const int4 place = list[at / p.heads * 4 + 2];  // {the bundle's first item, its length, ..}
      const int rem = at - place.x * p.heads, head = rem / place.y;
      w = list[(place.x + rem - head * place.y) * 4 + (lane & 3)];
      if (lane == 2) w.z = head;
    }
    if (k >= 2 && !wait_warp(&ctl.sched_free[k & 1u], (k - 2) >> 1, ctl, kSiteLoad, p.dev_err)) return;
    if (lane < 4) ctl.work[k & 1u][lane] = w;
    __syncwarp();
    mbar_arrive_if(lane == 0 ? 1u : 0u, &ctl.sched_full[k & 1u]);
    if (!more) return;
  }
}

__device__ void load_role(const PrefillParams& p, const CUtensorMap& tq, const CUtensorMap& tk, const CUtensorMap& tv,
                          const CUtensorMap& tpe, uint8_t* sm, Ctl& ctl, int lane) {
  uint8_t* ring = sm + kRingOff;
  Entry en;
  uint32_t nq[2] = {0, 0}, tails = 0;
  bool ok = true;
  Item it;
  auto load_q = [&](int i) {
    if (nq[i] > 0 && !(ok = wait_warp(&ctl.q_free[i], nq[i] - 1, ctl, kSiteLoad, p.dev_err))) return;
    if (lane == 0) {
      mbar_arrive_expect_tx(&ctl.q_full[i], kQChunks * kSlotBytes);
      for (int c = 0; c < kQChunks; ++c)
        tma_load_3d(sm + (i * kQChunks + c) * kSlotBytes, &tq, c * 64, it.head, it.q_row + i * kTile, &ctl.q_full[i]);
    }
    ++nq[i];
  };
  auto room = [&]() {
    if (en.e >= kInFlight)
      ok = wait_warp(&ctl.freed[(en.e - kInFlight) & 3u], (en.e - kInFlight) >> 2, ctl, kSiteLoad, p.dev_err);
    return ok;
  };
  auto load_k = [&](int j) {
    if (!room()) return;
    if (lane == 0) {
      const int row = it.kv_start + j * kTile;
      uint64_t* bar = &ctl.full[en.e & 3u];
      mbar_arrive_expect_tx(bar, kKChunks * kSlotBytes);
      for (int c = 0; c < 2; ++c)
        tma_load_3d(ring + ((en.slot + c) & 7u) * kSlotBytes, &tk, c * 64, it.head, row, bar);
      tma_load_2d(ring + ((en.slot + 2) & 7u) * kSlotBytes, &tpe, 0, row, bar);
    }
    en.next(kKChunks);
  };
  auto load_v = [&](int j) {
    if (!room()) return;
    const int row = it.kv_start + j * kTile;
    uint64_t* bar = &ctl.full[en.e & 3u];
    uint8_t* s0 = ring + en.slot * kSlotBytes;
    uint8_t* s1 = ring + ((en.slot + 1) & 7u) * kSlotBytes;
    // Rows behind the sequence's last token belong to others: their weights are 0,
    // but 0 x inf is not, so they are cleared before the tensor core sees them.
    const int left = it.kv_len - j * kTile;
    uint64_t* on = left < kTile ? &ctl.tail : bar;
    if (lane == 0) {
      mbar_arrive_expect_tx(on, kVSlots * kSlotBytes);
      for (int c = 0; c < 2; ++c) {
        tma_load_3d(s0 + c * 8192, &tv, c * 64, it.head, row, on);
        tma_load_3d(s1 + c * 8192, &tv, c * 64, it.head, row + 64, on);
      }
    }
    if (left < kTile) {
      if (!(ok = wait_warp(&ctl.tail, tails, ctl, kSiteLoad, p.dev_err))) {
        if (lane == 0) mbar_wait(&ctl.tail, tails & 1u, kLimitNs, nullptr);  // (its copy may be on its way)
        return;
      }
      ++tails;
      for (int x = lane; x < (kTile - left) * 16; x += 32) {  // 16-byte pieces: 8 per row and half
        const int t = left + (x >> 4), c = (x >> 3) & 1;
        uint8_t* dst = (t < 64 ? s0 : s1) + c * 8192 + (t & 63) * 128 + (x & 7) * 16;
        *reinterpret_cast<uint4*>(dst) = make_uint4(0, 0, 0, 0);
      }
      fence_proxy_async_smem();
      __syncwarp();
      mbar_arrive_if(lane == 0 ? 1u : 0u, bar);
    }
    en.next(kVSlots);
  };
  for (uint32_t pair = 0; ok && next_pair<true>(ctl, pair, it, kSiteLoad, p.dev_err); ++pair) {
    // In the order in which mma_role uses them up, but that the first keys do not wait for
    // the queries: a pair's query tiles can only be loaded once the last QKs of the pair
    // before are through. (The next pair is asked for kAhead steps before the end.)
    const int n = max(it.n0, it.n1), when = max(n - 1 - kAhead, 0);
    const int per = it.dealt != 0 ? 2 : 1;  // key steps in a round
    if (n == 0) mbar_arrive_if(lane == 0 ? 1u : 0u, &ctl.ask);
    for (int j = 0; ok && j < n; j += per) {
      for (int x = 0; ok && x < per && j + x < n; ++x) {
        load_k(j + x);
        if (ok && j + x == 0 && it.n0 > 0) load_q(0);
      }
      if (ok && j == 0 && it.n1 > 0) load_q(1);
      for (int x = 0; ok && x < per && j + x < n; ++x) load_v(j + x);
      if (when >= j && when < j + per) mbar_arrive_if(lane == 0 ? 1u : 0u, &ctl.ask);
    }
  }
  if (lane != 0) return;
  // No copy may be on its way when the CTA's shared memory is released; these waits
  // ignore the abort flag.
  for (int i = 0; i < 2; ++i)
    if (nq[i] > 0 && mbar_wait(&ctl.q_full[i], (nq[i] - 1) & 1u, kLimitNs, nullptr) != 1) give_up(ctl, p.dev_err, kSiteEnd);
  for (uint32_t k = 1; k <= kInFlight && k <= en.e; ++k)
    if (mbar_wait(&ctl.full[(en.e - k) & 3u], ((en.e - k) >> 2) & 1u, kLimitNs, nullptr) != 1)
      give_up(ctl, p.dev_err, kSiteEnd);
}

// Tile i's MMAs, from one thread. What a thread does around them (waits, commits of 70
// cycles, addresses: about 650 cycles per step) is more than the tensor core's queue
// covers; with a thread for each tile it falls into the other's MMAs.
__device__ void mma_role(const PrefillParams& p, uint32_t smem, Ctl& ctl, uint32_t tmem, int i) {
  constexpr uint32_t kIdQK = idesc_bf16_f32(kTile, kTile, false, false);
  constexpr uint32_t kIdPV = idesc_bf16_f32(kTile, kDv, false, true);
  // Low words of the descriptors of the first chunks; a slot is 1,024 units on.
  constexpr uint32_t kSlotUnits = kSlotBytes >> 4;
  const uint32_t hi = static_cast<uint32_t>(smem_desc(0, 16, 1024, SWZ_128B) >> 32);
  const uint32_t lo_q = static_cast<uint32_t>(smem_desc(smem, 16, 1024, SWZ_128B));
  const uint32_t lo_k = static_cast<uint32_t>(smem_desc(smem + kRingOff, 16, 1024, SWZ_128B));
  const uint32_t lo_v = static_cast<uint32_t>(smem_desc(smem + kRingOff, 8192, 1024, SWZ_128B));
  const uint32_t t_s = tmem + i * 128, t_o = tmem + kColO + i * 128;
  Entry en;
  uint32_t nq[2] = {0, 0}, np = 0, no = 0;
  bool ok = true;
  auto wait = [&](uint64_t* bar, uint32_t phase) { return ok = wait1(bar, phase, ctl, kSiteMma, p.dev_err); };
  // One tile's PV and QK are issued without the other's in between: mixed, both tiles'
  // scores would be ready at the same time, and the tensor core would idle through
  // both softmaxes.
  bool mine = false;
  auto take = [&]() {
    if (mine) return true;
    uint64_t t0 = 0;
    for (uint32_t k = 0; atomicCAS(&ctl.turn, 0, 1) != 0; ++k) {
      if (*reinterpret_cast<volatile uint32_t*>(&ctl.abort) != 0u) return ok = false;
      if ((k & 1023u) != 1023u) continue;
      const uint64_t t = globaltimer_ns();
      if (t0 == 0) t0 = t;
      if (t - t0 > kLimitNs) {
        give_up(ctl, p.dev_err, kSiteMma);
        return ok = false;
      }
    }
    return mine = true;
  };
  auto give = [&]() {
    if (mine) atomicExch(&ctl.turn, 0);
    mine = false;
  };
  // An entry of the other tile's: given back by this one as soon as it is there.
  auto skip = [&](uint32_t slots) {
    uint64_t* bar = &ctl.full[en.e & 3u];
    if (!mbar_test(bar, (en.e >> 2) & 1u)) {
      give();
      if (!wait(bar, en.e >> 2)) return;
    }
    mbar_arrive_if(1u, &ctl.freed[en.e & 3u]);
    en.next(slots);
  };
  // S = Q (tile q of shared memory) K^T
  auto qk = [&](int q, bool last) {
    uint64_t* bar = &ctl.full[en.e & 3u];
    if (!mbar_test(bar, (en.e >> 2) & 1u)) {
      give();  // (the keys are late)
      if (!wait(bar, en.e >> 2)) return;
    }
    if (!take()) return;
#pragma unroll
    for (int c = 0; c < kKChunks; ++c)
      umma_f16_ss_x4(t_s, lo_q + (q * kQChunks + c) * kSlotUnits, lo_k + ((en.slot + c) & 7u) * kSlotUnits, hi, kIdQK,
                     c != 0 ? 1u : 0u);
    umma_commit(&ctl.s_full[i]);
    give();
    umma_commit(&ctl.freed[en.e & 3u]);
    if (last) umma_commit(&ctl.q_free[q]);
    en.next(kKChunks);
  };
  // O (+)= P V
  auto pv = [&](bool first, bool last) {
    if (!wait(&ctl.full[en.e & 3u], en.e >> 2)) return;
    if (first && no > 0 && !wait(&ctl.o_free[i], no - 1)) return;  // (the pair before's has been read)
#pragma unroll
    for (int h = 0; h < kVSlots; ++h) {
      if (!wait(&ctl.p_full[i][h], np)) return;
      if (h == 0 && !take()) return;
      tc_fence_after();
      umma_f16_ts_x4(t_o, t_s + h * 32, lo_v + ((en.slot + h) & 7u) * kSlotUnits, hi, kIdPV, first && h == 0 ? 0u : 1u);
    }
    ++np;
    umma_commit(&ctl.freed[en.e & 3u]);
    if (last) {
      umma_commit(&ctl.o_full[i]);
      ++no;
      give();
    }
    en.next(kVSlots);
  };
  Item it;
  for (uint32_t pair = 0; ok && next_pair<false>(ctl, pair, it, kSiteMma, p.dev_err); ++pair) {
    // Entries: K0, V0, K1, V1, .., all for both tiles; dealt: K0, K1, V0, V1, K2, K3, ..,
    // the even ones tile 0's and the odd ones tile 1's. Query tile 0 is given back by
    // both threads, by one that does not use it once the first values are there: they are
    // loaded after it, so it is this pair's, and the one before has been given back.
    // (One place for each kind of entry: the roles' code has to share the SM's instruction
    // caches.)
    const bool dealt = it.dealt != 0;
    const int q = dealt ? 0 : i, all = max(it.n0, it.n1);
    const int n = dealt ? (it.n0 + 1 - i) >> 1 : (i == 0 ? it.n0 : it.n1);  // of this tile
    const int rounds = dealt ? (all + 1) >> 1 : all;
    if (n > 0 && !wait(&ctl.q_full[q], nq[q])) break;
    nq[0] += it.n0 > 0 ? 1u : 0u;
    nq[1] += !dealt && it.n1 > 0 ? 1u : 0u;
#pragma unroll 1
    for (int x = 0; ok && x < 2 * rounds; ++x) {
      const int j = x >> 1;
      const uint32_t slots = (x & 1) == 0 ? kKChunks : kVSlots;
      if (dealt ? i == 1 : j >= n) skip(slots);
      if (ok && j < n) {
        if ((x & 1) == 0) {
          qk(q, j + 1 == n);
        } else {
          pv(j == 0, j + 1 == n);
        }
      }
      if (ok && dealt && i == 0 && 2 * j + 1 < all) skip(slots);
      if (x == 1 && i == 1 && !dealt && it.n0 > 0) mbar_arrive_if(1u, &ctl.q_free[0]);
    }
  }
  give();
  // Every MMA must have landed before TMEM and shared memory are released.
  umma_commit(&ctl.fin);
  if (mbar_wait(&ctl.fin, 0, kLimitNs, nullptr) != 1) give_up(ctl, p.dev_err, kSiteEnd);
}

__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

__device__ __forceinline__ float max3(float a, float b, float c) {
  float y;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(y) : "f"(a), "f"(b), "f"(c));
  return y;
}

// Holds the registers of a TMEM load whose values are not used until here: the load
// writes them some time before its wait.
__device__ __forceinline__ void keep64(float (&s)[64]) {
#pragma unroll
  for (int c = 0; c < 64; c += 8)
    asm volatile("" ::"f"(s[c]), "f"(s[c + 1]), "f"(s[c + 2]), "f"(s[c + 3]), "f"(s[c + 4]), "f"(s[c + 5]), "f"(s[c + 6]),
                 "f"(s[c + 7]));
}

// Hides the scores from key `lim` on (lim >= 64: none).
__device__ __forceinline__ void hide64(float (&s)[64], int lim) {
#pragma unroll
  for (int c = 0; c < 64; ++c) s[c] = c < lim ? s[c] : -INFINITY;
}

// 2^(s scale - ref) of 64 scores as pairs of bf16, and the sum (of the unrounded ones). The
// weights meet values in bf16 in one MMA, whose operands have to be of one type, and values in
// fp16 would lose range; so each is off by up to 2^-8, as a value is. Their sum is taken
// before that rounding: it is the exact one's to fp32, and the roundings of many weights,
// which are as often up as down, do not enter the log-sum-exp.
__device__ __forceinline__ float weights64(const float (&s)[64], float scale, float ref, uint32_t (&w)[32]) {
  const uint64_t sl = f32x2(scale, scale), mm = f32x2(-ref, -ref);
  uint64_t sum[4] = {0, 0, 0, 0};  // (pairs of zeros)
#pragma unroll
  for (int c = 0; c < 32; ++c) {
    const uint64_t x = fma2(f32x2(s[2 * c], s[2 * c + 1]), sl, mm);
    const float a = ex2(lo2(x)), b = ex2(hi2(x));
    sum[c & 3] = add2(sum[c & 3], f32x2(a, b));
    w[c] = pack_bf16(a, b);
  }
  const uint64_t t = add2(add2(sum[0], sum[1]), add2(sum[2], sum[3]));
  return lo2(t) + hi2(t);
}

// Softmax of tile i, a query row per thread.
__device__ void softmax_role(const PrefillParams& p, Ctl& ctl, uint32_t tmem, int i, int warp, int lane) {
  const uint32_t lanes = static_cast<uint32_t>((warp & 3) * 32) << 16;
  const uint32_t t_s = tmem + lanes + i * 128, t_o = tmem + lanes + kColO + i * 128;
  const int row_in = (warp & 3) * 32 + lane;  // of the tile
  uint32_t ns = 0, no = 0;
  Item it;
  for (uint32_t pair = 0; next_pair<true>(ctl, pair, it, kSiteSoftmax, p.dev_err); ++pair) {
    const bool dealt = it.dealt != 0;
    const int n = dealt ? (it.n0 + 1 - i) / 2 : (i == 0 ? it.n0 : it.n1);
    const int row = dealt ? row_in : row_in + i * kTile;  // of the item
    float m = -INFINITY, l = 0.0f;                        // m in units of log2
    const int vis = min(it.kv_len, it.vis0 + it.step * row);
    const int vis_warp = min(it.kv_len, it.vis0 + it.step * (row - lane));  // of the warp's first row
    for (int j = 0; j < n; ++j) {
      if (!wait_warp(&ctl.s_full[i], ns, ctl, kSiteSoftmax, p.dev_err)) return;
      ++ns;
      tc_fence_after();
      // The row's maximum comes with the load, but for rows that hide keys of this step.
      // (Loops stay loops and the second half of the scores is read again: unrolled,
      // with everything in registers, the code outgrows the instruction caches that the
      // roles share, and every second issue slot waits for instructions.)
      const int key0 = (dealt ? 2 * j + i : j) * kTile;
      const bool masked = vis_warp < key0 + kTile;
      float s[64], top;
      {
        float u[64], t[4];
        tmem_ld32_max(t_s, s, t[0]);
        tmem_ld32_max(t_s + 32, s + 32, t[1]);
        tmem_ld32_max(t_s + 64, u, t[2]);
        tmem_ld32_max(t_s + 96, u + 32, t[3]);
        tmem_ld_wait();
        keep64(u);
        top = fmaxf(max3(t[0], t[1], t[2]), t[3]);
      }
      if (masked) {
        top = -INFINITY;
#pragma unroll 1
        for (int c = 0; c < 4; ++c) {
          float u[32];
          tmem_ld32(t_s + 32 * c, reinterpret_cast<uint32_t*>(u));
          tmem_ld_wait();
          const int lim = vis - key0 - 32 * c;
#pragma unroll
          for (int x = 0; x < 32; ++x) top = fmaxf(top, x < lim ? u[x] : -INFINITY);
        }
      }
      top *= p.scale_log2;
      const bool raise = top > m + kRaise;  // (m = -inf: the first visible key)
      if (__any_sync(0xffffffffu, raise)) {
        const float factor = raise ? ex2(m - top) : 1.0f;  // 0 where nothing has been seen yet
        if (raise) m = top;
        l *= factor;
        // (the scores' arrival says that PV of the keys before has completed too)
#pragma unroll 1
        for (int c = j > 0 ? 0 : 16; c < 16; ++c) {
          uint32_t o[8];
          tmem_ld(t_o + 8 * c, o);
          tmem_ld_wait();
#pragma unroll
          for (int x = 0; x < 8; ++x) o[x] = __float_as_uint(__uint_as_float(o[x]) * factor);
          tmem_st(t_o + 8 * c, o);
        }
      }
      const float ref = m == -INFINITY ? 0.0f : m;
#pragma unroll 1
      for (int h = 0; h < 2; ++h) {
        if (masked) hide64(s, vis - key0 - 64 * h);
        uint32_t w[32];
        l += weights64(s, p.scale_log2, ref, w);
        tmem_st32(t_s + 32 * h, w);
        if (h == 0) {
          tmem_ld32(t_s + 64, reinterpret_cast<uint32_t*>(s));
          tmem_ld32(t_s + 96, reinterpret_cast<uint32_t*>(s + 32));
        }
        tmem_st_wait();
        tc_fence_before();
        __syncwarp();
        mbar_arrive_if(lane == 0 ? 1u : 0u, &ctl.p_full[i][h]);
        tmem_ld_wait();
      }
    }
    if (n > 0) {
      if (no > 0 && !wait_warp(&ctl.o_free[i], no - 1, ctl, kSiteSoftmax, p.dev_err)) return;
      ++no;
      ctl.sums[i][row_in] = make_float2(m, l);
      __syncwarp();
      mbar_arrive_if(lane == 0 ? 1u : 0u, &ctl.l_full[i]);
    }
  }
}

// 32 bytes of a row.
__device__ __forceinline__ void st_v8(void* dst, const uint32_t* w) {
  asm volatile("st.global.v8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"l"(dst), "r"(w[0]), "r"(w[1]), "r"(w[2]),
               "r"(w[3]), "r"(w[4]), "r"(w[5]), "r"(w[6]), "r"(w[7])
               : "memory");
}

// O / l and the log-sum-exp of both tiles, a query row per thread. A part's O goes to
// the workspace as it is, in fp32 with its (m, l), for join_kernel.
__device__ void epilogue_role(const PrefillParams& p, Ctl& ctl, uint32_t tmem, int warp, int lane) {
  const uint32_t t_o = tmem + (static_cast<uint32_t>((warp & 3) * 32) << 16) + kColO;
  const int row_in = (warp & 3) * 32 + lane;
  uint32_t no[2] = {0, 0};
  Item it;
  for (uint32_t pair = 0; next_pair<true>(ctl, pair, it, kSiteEpilogue, p.dev_err); ++pair) {
    const bool dealt = it.dealt != 0, whole = it.parts == 1;
    Partial* part = whole ? nullptr : p.partial + it.slot + static_cast<size_t>(it.head) * it.parts + it.part;
#pragma unroll 1
    for (int i = 0; i < 2; ++i) {
      if (i * kTile >= it.rows) break;
      const int n = i == 0 ? it.n0 : it.n1, row = i * kTile + row_in;
      float m = -INFINITY, l = 0.0f, mine = 0.0f, theirs = 0.0f;
      if (n > 0) {
        // (dealt: tile 1's as well)
#pragma unroll 1
        for (int x = i; x <= (dealt ? 1 : i); ++x) {
          if (!wait_warp(&ctl.l_full[x], no[x], ctl, kSiteEpilogue, p.dev_err)) return;
          if (!wait_warp(&ctl.o_full[x], no[x], ctl, kSiteEpilogue, p.dev_err)) return;
          ++no[x];
        }
        tc_fence_after();
        const float2 a = ctl.sums[i][row_in];
        m = a.x, l = a.y, mine = 1.0f;
        if (dealt) {
          const float2 c = ctl.sums[1][row_in];
          m = fmaxf(a.x, c.x);
          const float ref = m == -INFINITY ? 0.0f : m;
          mine = ex2(a.x - ref);
          theirs = ex2(c.x - ref);
          l = a.y * mine + c.y * theirs;
        }
        if (whole) {
          const float inv = 1.0f / l;  // (l = 0, a row that sees no key: not used)
          mine *= inv;
          theirs *= inv;
        }
      }
      const bool write = row < it.rows;
      const bool none = l == 0.0f;  // the row sees no key (a visible one leaves l >= 1, or NaN)
      const size_t at = static_cast<size_t>(it.q_row + row) * p.heads + it.head;
#pragma unroll 1
      for (int c = 0; c < (whole || n > 0 ? 4 : 0); ++c) {
        uint32_t o[32], w[16];
        if (n > 0) {
          tmem_ld32(t_o + i * 128 + 32 * c, o);
          tmem_ld_wait();
#pragma unroll
          for (int x = 0; x < 16; ++x) {
            const uint64_t v = mul2(f32x2(__uint_as_float(o[2 * x]), __uint_as_float(o[2 * x + 1])), f32x2(mine, mine));
            o[2 * x] = __float_as_uint(lo2(v));
            o[2 * x + 1] = __float_as_uint(hi2(v));
          }
          if (dealt) {
#pragma unroll
            for (int y = 0; y < 2; ++y) {
              uint32_t e[16];
              tmem_ld(t_o + 128 + 32 * c + 16 * y, e);
              tmem_ld_wait();
#pragma unroll
              for (int x = 0; x < 16; ++x)
                o[16 * y + x] = __float_as_uint(fmaf(__uint_as_float(e[x]), theirs, __uint_as_float(o[16 * y + x])));
            }
          }
          if (c == 3) {
            tc_fence_before();
            __syncwarp();
            mbar_arrive_if(lane == 0 ? 1u : 0u, &ctl.o_free[i]);
            if (dealt) mbar_arrive_if(lane == 0 ? 1u : 0u, &ctl.o_free[1]);
          }
        }
        if (!write) continue;
        if (whole) {
#pragma unroll
          for (int x = 0; x < 16; ++x)
            w[x] = none ? 0u : pack_bf16(__uint_as_float(o[2 * x]), __uint_as_float(o[2 * x + 1]));
          st_v8(p.out + at * kDv + 32 * c, w);
          st_v8(p.out + at * kDv + 32 * c + 16, w + 8);
        } else {
#pragma unroll
          for (int x = 0; x < 4; ++x) st_v8(part->o[row] + 32 * c + 8 * x, o + 8 * x);
        }
      }
      if (!write) continue;
      if (!whole) {
        part->ml[row] = make_float2(m, l);
      } else if (p.lse != nullptr) {
        p.lse[at] = none ? -INFINITY : m * 0.6931471805599453f + logf(l);
      }
    }
  }
}

__global__ void __launch_bounds__(kThreads, 1)
    prefill_kernel(const __grid_constant__ CUtensorMap tq, const __grid_constant__ CUtensorMap tk,
                   const __grid_constant__ CUtensorMap tv, const __grid_constant__ CUtensorMap tpe,
                   const PrefillParams p) {
  extern __shared__ __align__(1024) uint8_t sm[];
  Ctl& ctl = *reinterpret_cast<Ctl*>(sm + kCtlOff);
  const int warp = __shfl_sync(0xffffffffu, static_cast<int>(threadIdx.x) >> 5, 0), lane = threadIdx.x & 31;
  if (threadIdx.x == 0) {
    for (int i = 0; i < 2; ++i) {
      mbar_init(&ctl.q_full[i], 1);
      mbar_init(&ctl.q_free[i], i == 0 ? 2 : 1);  // (query tile 0 can serve both tiles)
      mbar_init(&ctl.s_full[i], 1);
      for (int h = 0; h < 2; ++h) mbar_init(&ctl.p_full[i][h], 4);
      mbar_init(&ctl.o_full[i], 1);
    }
    for (int i = 0; i < 4; ++i) {
      mbar_init(&ctl.full[i], 1);
      mbar_init(&ctl.freed[i], 2);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(&ctl.sched_full[i], 1);
      mbar_init(&ctl.sched_free[i], kSoftWarps + 4 + 2 + 1);
      mbar_init(&ctl.l_full[i], 4);
      mbar_init(&ctl.o_free[i], 4);
    }
    mbar_init(&ctl.ask, 1);
    mbar_init(&ctl.tail, 1);
    mbar_init(&ctl.fin, 2);
    ctl.abort = 0u;
    ctl.turn = 0;
    fence_mbar_init();
  }
  if (warp == 0) {
    tmem_alloc(&ctl.tmem_base, 512);
    tmem_relinquish();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = __shfl_sync(0xffffffffu, ctl.tmem_base, 0);
  griddep_wait();  // the plan, and with it everything before it in the stream
  if (warp < kSoftWarps) {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kSoftRegs));
    softmax_role(p, ctl, tmem, warp >> 2, warp, lane);
  } else if (warp < kMmaWarp) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kEpiRegs));
    epilogue_role(p, ctl, tmem, warp - kEpiWarp, lane);
  } else {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kOtherRegs));
    if (warp == kLoadWarp) {
      load_role(p, tq, tk, tv, tpe, sm, ctl, lane);
    } else if (warp == kDrawWarp) {
      draw_role(p, ctl, lane);
    } else if (elect_one()) {
      mma_role(p, smem_u32(sm), ctl, tmem, warp == kMmaWarp ? 0 : 1);
    } else {
      asm volatile("exit;");
    }
  }
  if (p.join) griddep_launch_dependents();  // it may be scheduled as CTAs finish
  tc_fence_before();
  __syncthreads();  // (exited lanes do not take part)
  if (warp == 0) {
    tc_fence_after();
    tmem_dealloc(tmem, 512);
  }
}

// The items that were cut up: a row of one head per warp and turn, a lane four
// channels. A row's parts are added in their order; eight of them are on their way at
// once, and the first eight while the maximum is found.
constexpr int kJoinThreads = 256, kJoinRows = kJoinThreads / 32, kJoinAhead = 8;
__global__ void __launch_bounds__(kJoinThreads) join_kernel(const PrefillParams p, const Join* __restrict__ joins) {
  griddep_wait();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int units = p.count[2] * p.heads * (kItemRows / kJoinRows);
  for (int u = blockIdx.x; u < units; u += gridDim.x) {
    const int pair = u / (kItemRows / kJoinRows), head = pair % p.heads;
    const int row = u % (kItemRows / kJoinRows) * kJoinRows + warp;
    const Join j = joins[pair / p.heads];
    if (row >= j.rows) continue;
    const Partial* part = p.partial + j.slot + static_cast<size_t>(head) * j.parts;
    float4 v[kJoinAhead];
    float2 x[kJoinAhead];
    auto load = [&](int y0) {
#pragma unroll
      for (int k = 0; k < kJoinAhead; ++k) {
        if (y0 + k < j.parts) {
          x[k] = part[y0 + k].ml[row];
          v[k] = *reinterpret_cast<const float4*>(part[y0 + k].o[row] + 4 * lane);
        }
      }
    };
    load(0);
    float m = -INFINITY;
    for (int y = lane; y < j.parts; y += 32) {
      const float2 z = part[y].ml[row];
      if (z.y != 0.0f) m = fmaxf(m, z.x);  // (a sum of 0: the row sees no key of this part)
    }
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, off));
    const float ref = m == -INFINITY ? 0.0f : m;
    float l = 0.0f;
    float4 o = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    for (int y0 = 0; y0 < j.parts; y0 += kJoinAhead) {
      if (y0 > 0) load(y0);
#pragma unroll
      for (int k = 0; k < kJoinAhead; ++k) {
        if (y0 + k >= j.parts || x[k].y == 0.0f) continue;  // (then v was not written)
        const float f = ex2(x[k].x - ref);
        l = fmaf(x[k].y, f, l);
        o = make_float4(fmaf(v[k].x, f, o.x), fmaf(v[k].y, f, o.y), fmaf(v[k].z, f, o.z), fmaf(v[k].w, f, o.w));
      }
    }
    const bool none = l == 0.0f;
    const float inv = 1.0f / l;
    const size_t at = static_cast<size_t>(j.q_row + row) * p.heads + head;
    *reinterpret_cast<uint2*>(p.out + at * kDv + 4 * lane) =
        none ? make_uint2(0u, 0u) : make_uint2(pack_bf16(o.x * inv, o.y * inv), pack_bf16(o.z * inv, o.w * inv));
    if (lane == 0 && p.lse != nullptr) p.lse[at] = none ? -INFINITY : m * 0.6931471805599453f + logf(l);
  }
}

// ------------------------------------------------------------------------ host
using EncodeFn = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*,
                              const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                              CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

cudaError_t encode_fn(EncodeFn& fn) {
  static EncodeFn found = nullptr;
  if (found == nullptr) {
    void* f = nullptr;
    cudaDriverEntryPointQueryResult r;
    const cudaError_t e = cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &f, 12000, cudaEnableDefault, &r);
    if (e != cudaSuccess) return e;
    if (r != cudaDriverEntryPointSuccess || f == nullptr) return cudaErrorNotSupported;
    found = reinterpret_cast<EncodeFn>(f);
  }
  fn = found;
  return cudaSuccess;
}

// Boxes of 64 channels x `rows` tokens of one head, 128-byte swizzled. heads = 0: a
// tensor without a head axis.
cudaError_t make_map(CUtensorMap& m, const void* base, int channels, int heads, int tokens, long long token_stride,
                     long long head_stride, int rows) {
  EncodeFn fn;
  const cudaError_t e = encode_fn(fn);
  if (e != cudaSuccess) return e;
  const cuuint32_t rank = heads > 0 ? 3 : 2;
  cuuint64_t dims[3] = {static_cast<cuuint64_t>(channels), static_cast<cuuint64_t>(heads), static_cast<cuuint64_t>(tokens)};
  cuuint64_t strides[2] = {static_cast<cuuint64_t>(head_stride) * 2, static_cast<cuuint64_t>(token_stride) * 2};
  cuuint32_t box[3] = {64, 1, static_cast<cuuint32_t>(rows)}, steps[3] = {1, 1, 1};
  if (rank == 2) {
    dims[1] = dims[2];
    strides[0] = strides[1];
    box[1] = box[2];
  }
  const CUresult r = fn(&m, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, rank, const_cast<void*>(base), dims, strides, box, steps,
                        CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                        CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  return r == CUDA_SUCCESS ? cudaSuccess : cudaErrorInvalidValue;
}

}  // namespace

size_t prefill_workspace_bytes(int batch, int n_q) { return workspace_layout(batch, n_q).total; }

cudaError_t launch_prefill(const qmla_prefill_desc& d, int sms, cudaStream_t stream) {
  const Workspace w = workspace_layout(d.batch, d.n_q);
  uint8_t* ws = static_cast<uint8_t*>(d.workspace);
  PrefillParams p;
  p.count = reinterpret_cast<int*>(ws);
  p.items = reinterpret_cast<const Item*>(ws + w.items_off);
  p.heads = d.heads;
  Join* joins = reinterpret_cast<Join*>(ws + w.join_off);
  p.partial = reinterpret_cast<Partial*>(ws + w.part_off);
  p.scale_log2 = d.softmax_scale * 1.4426950408889634f;
  p.out = d.out;
  p.lse = d.lse;
  p.dev_err = d.dev_err;
  CUtensorMap tq, tk, tv, tpe;
  // A stride of an axis of one element is never used; a valid one stands in its place.
  // Without keys no copy of one is issued, and none of their strides is looked at.
  const bool keys = d.n_kv > 0;
  const int key_heads = keys ? d.heads : 1;
  auto stride = [](int n, long long s, long long least) { return n > 1 ? s : least; };
  cudaError_t e = make_map(tq, d.q, kDn + kDr, d.heads, d.n_q, stride(d.n_q, d.q_token_stride, kDn + kDr),
                           stride(d.heads, d.q_head_stride, kDn + kDr), kTile);
  const void* any = d.q;
  if (e == cudaSuccess)
    e = make_map(tk, keys ? d.k : any, kDn, d.heads, std::max(d.n_kv, 1), stride(d.n_kv, d.k_token_stride, kDn),
                 stride(key_heads, d.k_head_stride, kDn), kTile);
  if (e == cudaSuccess)
    e = make_map(tv, keys ? d.v : any, kDv, d.heads, std::max(d.n_kv, 1), stride(d.n_kv, d.v_token_stride, kDv),
                 stride(key_heads, d.v_head_stride, kDv), 64);
  if (e == cudaSuccess)
    e = make_map(tpe, keys ? d.k_pe : any, kDr, 0, std::max(d.n_kv, 1), stride(d.n_kv, d.k_pe_stride, kDr), 0, kTile);
  if (e != cudaSuccess) return e;
  static int configured_device = -1;
  int dev = 0;
  if ((e = cudaGetDevice(&dev)) != cudaSuccess) return e;
  if (configured_device != dev) {
    if ((e = cudaFuncSetAttribute(prefill_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmem)) != cudaSuccess)
      return e;
    configured_device = dev;
  }
  const long long pairs = static_cast<long long>(w.max_items) * d.heads;
  // A plan (and the join of what it cuts up) is worth its launches where items are long
  // or many. With it and without, in us: 16 heads x 37 rows 11.6 and 8.2, over 1,037 keys
  // 22.3 and 16.4, over 2,037 22.2 and 23.2, over 4,037 25.0 and 41.5; 128 heads x 500 rows
  // 28.5 and 24.8, x 1,000 55.7 and 55.4, x 2,000 151 and 154; 16 heads x 2,000 rows 43.4
  // and 36.9; 16 heads x 8 prompts of 20 to 110 rows 13.7 and 9.6.
  p.unplanned = d.n_kv <= kUnplannedKeys && d.batch <= kUnplanned && d.n_q <= kUnplannedRows;
  const bool parts = !p.unplanned && d.n_kv > kLeastPart * kTile;  // (else no item is cut up)
  p.join = parts;
  p.cu_q = d.cu_q;
  p.cu_kv = d.cu_kv;
  p.batch = d.batch;
  p.n_q = d.n_q;
  p.n_kv = d.n_kv;
  p.causal = d.causal;
  // Items per bundle: with few pairs per SM single items even the load out better.
  const int bundle = pairs >= 8ll * sms ? 4 : 1;
  if (!p.unplanned) {
    const int threads = w.max_items <= kSmallPlan && d.batch <= kSmallPlan ? kSmallPlan : kPlanThreads;
    int shift = 0;
    while (((d.n_kv / kTile + 1) >> shift) >= threads) ++shift;
    plan_kernel<<<1, threads, 0, stream>>>(d.cu_q, d.cu_kv, d.batch, d.n_q, d.n_kv, d.heads, d.causal != 0, sms, bundle,
                                           shift, p.count, reinterpret_cast<int*>(ws + w.prefix_off),
                                           reinterpret_cast<Item*>(ws + w.items_off), joins, d.dev_err);
    if ((e = cudaGetLastError()) != cudaSuccess) return e;
  }
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(static_cast<unsigned>(std::min<long long>(sms, pairs + (parts ? kSlots : 0))));
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = kSmem;
  cfg.stream = stream;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = p.unplanned ? 0 : 1;  // (behind whatever the caller launched: in full)
  if ((e = cudaLaunchKernelEx(&cfg, prefill_kernel, tq, tk, tv, tpe, p)) != cudaSuccess) return e;
  if (!parts) return cudaSuccess;
  cfg.gridDim = dim3(static_cast<unsigned>(2 * sms));
  cfg.blockDim = dim3(kJoinThreads);
  cfg.dynamicSmemBytes = 0;
  return cudaLaunchKernelEx(&cfg, join_kernel, p, static_cast<const Join*>(joins));
}

}  // namespace qmla
