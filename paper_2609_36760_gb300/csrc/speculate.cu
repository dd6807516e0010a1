// Verification of a tree of drafted tokens (qmla_tree_verify) and what its result does to a
// cache (qmla_cache_keep).
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <cstddef>
#include <cstdint>
#include <type_traits>

#include "common.cuh"
#include "kernels.h"
#include "ptx.cuh"

namespace qmla {
namespace {

constexpr int kMaxNodes = QMLA_MAX_TREE_NODES;

// ------------------------------------------------------------- error-free sums
// hi + lo with |lo| at most half a unit of hi: about 48 bits. A draw from 10^5 tokens has that
// many borders a sum may fall on the wrong side of, and a decision that depended on the order
// of a sum would differ from run to run of another launch shape; with an error of 2^-46 (an emulation of
// rows' sums: 2^-45 at most, for up to 2^22 tokens a warp) that is one draw in 5 10^8. (In double the
// additions alone would take 40 us for 64 x 131,072 tokens: the card adds 1.25 T doubles a second.)
struct Pair {
  float hi, lo;
};
__device__ __forceinline__ Pair two_sum(float a, float b) {
  const float s = __fadd_rn(a, b), bb = __fadd_rn(s, -a);
  return {s, __fadd_rn(__fadd_rn(a, -__fadd_rn(s, -bb)), __fadd_rn(b, -bb))};
}
__device__ __forceinline__ Pair normal(float s, float e) {  // |s| >= |e|
  const float h = __fadd_rn(s, e);
  return {h, __fadd_rn(e, -__fadd_rn(h, -s))};
}
__device__ __forceinline__ Pair add(Pair a, Pair b) {
  const Pair s = two_sum(a.hi, b.hi);
  return normal(s.hi, __fadd_rn(s.lo, __fadd_rn(a.lo, b.lo)));
}
__device__ __forceinline__ Pair times(Pair a, float u) {
  const float h = __fmul_rn(a.hi, u);
  return normal(h, __fmaf_rn(a.lo, u, __fmaf_rn(a.hi, u, -h)));
}
__device__ __forceinline__ bool above(Pair a, Pair b) { return a.hi > b.hi || (a.hi == b.hi && a.lo > b.lo); }
__device__ __forceinline__ Pair product(Pair a, Pair b) {
  const float h = __fmul_rn(a.hi, b.hi);
  return normal(h, __fmaf_rn(a.hi, b.lo, __fmaf_rn(a.lo, b.hi, __fmaf_rn(a.hi, b.hi, -h))));
}
__device__ __forceinline__ Pair shfl_up(Pair a, int d) {
  return {__shfl_up_sync(0xffffffffu, a.hi, d), __shfl_up_sync(0xffffffffu, a.lo, d)};
}
// Sum over the lanes up to this one.
__device__ __forceinline__ Pair warp_scan(Pair x, int lane) {
#pragma unroll
  for (int d = 1; d < 32; d *= 2) {
    const Pair y = shfl_up(x, d);
    if (lane >= d) x = add(y, x);
  }
  return x;
}

// --------------------------------------------------------------- verification
__device__ __forceinline__ float as_float(float x) { return x; }
__device__ __forceinline__ float as_float(__nv_bfloat16 x) { return __bfloat162float(x); }

__device__ __forceinline__ float max_nan(float a, float b) {  // (a NaN stays one)
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}

// What the terms of a sum are made of: p alone, p and q after a first refusal, p and q after more.
enum Mode { kWhole, kOnce, kMore };

// What is left of p after refusals, max(p - a q, 0), of two tokens at a time (packed fp32), as
// hi + lo. The first refusal takes q itself (R is 1 until then), and p - q is exact as a pair,
// the larger coming first. The later ones take b q of that, b = a - 1. So where a draft is nearly the
// target, and what is left are units of p's last place, they are known to 2^-46 of themselves.
// (From p - a q, with a q to 2^-48 of it, draws went wrong there, and what was left came out below 0.
// That took 53 us for 64 x 131,072 tokens and walks of up to six passes, this 60.) A NaN in p stays
// one where p is alone and after one refusal, and so in b.
struct Pairs {
  uint64_t hi, lo;
};
struct Taken {  // b
  uint64_t hi, lo, minus_hi;
  __device__ explicit Taken(Pair b) : hi(f32x2(b.hi, b.hi)), lo(f32x2(b.lo, b.lo)), minus_hi(f32x2(-b.hi, -b.hi)) {}
};
template <Mode M>
__device__ __forceinline__ Pairs left_over(float p0, float p1, float q0, float q1, const Taken& b) {
  if constexpr (M == kWhole) return {f32x2(max_nan(p0, 0.0f), max_nan(p1, 0.0f)), 0};
  const uint64_t minus = f32x2(-1.0f, -1.0f), p = f32x2(p0, p1), q = f32x2(q0, q1);
  const uint64_t m = M == kOnce ? f32x2(fminf(p0, q0), fminf(p1, q1)) : q;
  const uint64_t s = fma2(m, minus, p), rounding = add2(m, fma2(p, minus, s));  // (s - p) + m, the minus of it
  if constexpr (M == kOnce) return {s, mul2(rounding, minus)};
  // (b q = l - h; t + e is s + h, or t is far below 0. The pair is not normal: lo may be more than t, and
  // decides the sign then. Where q is more than p, or no number, hi is below 0 or a NaN.)
  const uint64_t h = mul2(b.minus_hi, q), l = fma2(b.lo, q, fma2(b.hi, q, h));
  const uint64_t t = add2(s, h), e = add2(fma2(t, minus, s), h);
  const uint64_t lo = fma2(add2(rounding, l), minus, e), hi = add2(t, lo);
  const bool some0 = lo2(hi) > 0.0f, some1 = hi2(hi) > 0.0f;
  return {f32x2(some0 ? lo2(t) : 0.0f, some1 ? hi2(t) : 0.0f), f32x2(some0 ? lo2(lo) : 0.0f, some1 ? hi2(lo) : 0.0f)};
}
// Of one token, as a normal pair; q and b 0 where nothing was refused.
__device__ __forceinline__ Pair left_over(float p, float q, const Taken& b) {
  const Pairs r = left_over<kMore>(p, 0.0f, q, 0.0f, b);
  return two_sum(lo2(r.hi), lo2(r.lo));
}

// Two running sums of pairs, of the even and the odd terms.
struct Sums {
  uint64_t hi = 0, lo = 0;
  __device__ __forceinline__ void add(Pairs x) {
    const uint64_t minus = f32x2(-1.0f, -1.0f);
    const uint64_t s = add2(hi, x.hi), bb = fma2(hi, minus, s);
    const uint64_t e = add2(fma2(fma2(bb, minus, s), minus, hi), fma2(bb, minus, x.hi));
    hi = s;
    lo = add2(lo, add2(e, x.lo));
  }
  // lo back below half a unit of hi: left to grow, it takes errors in with every term (2^-41 of a sum after
  // 16,384 of them; kept small 2^-46).
  __device__ __forceinline__ void renormalise() {
    const uint64_t minus = f32x2(-1.0f, -1.0f), s = add2(hi, lo);
    lo = fma2(fma2(hi, minus, s), minus, lo);
    hi = s;
  }
  __device__ __forceinline__ Pair total() const {
    return qmla::add(two_sum(lo2(hi), lo2(lo)), two_sum(hi2(hi), hi2(lo)));
  }
};

constexpr int kVerifyThreads = 512, kVerifyWarps = kVerifyThreads / 32;
constexpr int kMaxCluster = 8;

struct VerifyShared {
  int token[kMaxNodes], parent[kMaxNodes];
  float u[kMaxNodes], p[kMaxNodes], q[kMaxNodes];  // a node's token in its parent's distributions
  Pair part[2][kMaxCluster * kVerifyWarps];        // every warp's sum, of every CTA
  Pair before[kMaxCluster * kVerifyWarps];         // sum of the warps before
  Pair total;
  Pair scan[kVerifyWarps];
  // the walk's state, written by warp 0
  int cur, last, refused_n;
  bool taken;  // a is 1 + b, not 0
  Pair b;
  int refused[kMaxNodes];
  unsigned long long found;
};

// Sum of the terms v0 .. v1 - 1 of a node (p and q its rows), a share of it in each lane. kFlight
// values of each row are on their way at a time: in 16 bytes where both rows lie on such
// borders (VEC; v0 and v1 are multiples of their values then), else one by one. SOME: the n tokens
// `gone` count as 0. (Taken off the sum afterwards they leave its rounding behind, from which a
// token of probability 0 would be drawn where nothing else is left.)
template <typename T, Mode M, bool VEC, bool SOME = false>
__device__ __forceinline__ Pair row_sum(const T* p, const T* q, const Taken& b, int v0, int v1, int lane,
                                        const int* gone = nullptr, int n = 0) {
  constexpr int kFlight = M == kMore ? 8 : 16;
  constexpr int kWide = VEC ? 16 / static_cast<int>(sizeof(T)) : 1, kLoads = kFlight / kWide;
  using Load = typename std::conditional<VEC, uint4, T>::type;
  Sums sums;
#pragma unroll 1
  for (int v = v0 + lane * kWide; v < v1; v += 32 * kFlight) {
    Load x[kLoads], y[kLoads];
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const int at = v + i * 32 * kWide;
      x[i] = y[i] = Load{};
      if (at < v1) {
        x[i] = __ldg(reinterpret_cast<const Load*>(p + at));
        if (M != kWhole) y[i] = __ldg(reinterpret_cast<const Load*>(q + at));
      }
    }
    if constexpr (SOME) {
      uint32_t zero = 0u;  // of this lane's values, in the order in which they are added
      for (int i = 0; i < n; ++i) {
        const uint32_t d = static_cast<uint32_t>(gone[i] - (v - lane * kWide));
        if (d < 32 * kFlight && d / kWide % 32 == static_cast<uint32_t>(lane)) zero |= 1u << (d / (32 * kWide) * kWide + d % kWide);
      }
      if (zero != 0u) {
#pragma unroll
        for (int e = 0; e < kFlight; ++e)
          if ((zero >> e) & 1u) reinterpret_cast<T*>(&x[e / kWide])[e % kWide] = T(0.0f);
      }
    }
    auto value = [&](const Load* from, int e) { return as_float(reinterpret_cast<const T*>(&from[e / kWide])[e % kWide]); };
#pragma unroll
    for (int e = 0; e < kFlight; e += 2)
      sums.add(left_over<M>(value(x, e), value(x, e + 1), M == kWhole ? 0.0f : value(y, e),
                            M == kWhole ? 0.0f : value(y, e + 1), b));
    sums.renormalise();
  }
  return sums.total();
}

// A piece of a row that refused certain drafts lie in. (A call of its own: in line, its registers cost every
// pass; 16 x 50,001 tokens, none refused: 34.3 us instead of 32.5.)
template <typename T, bool VEC>
__device__ __noinline__ Pair row_sum_without(const T* p, int v0, int v1, int lane, const int* gone, int n) {
  return row_sum<T, kWhole, VEC, true>(p, nullptr, Taken({0.0f, 0.0f}), v0, v1, lane, gone, n);
}

// One cluster a sequence. The walk itself is a warp's, done alike in every CTA; the sums over
// the vocabulary are all warps', warp w of the cluster taking the w-th piece of the row.
template <typename T>
__global__ void __launch_bounds__(kVerifyThreads, 2) verify_kernel(const qmla_verify_desc d, int ctas) {
  __shared__ VerifyShared sh;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int rank = static_cast<int>(cluster_ctarank()), b = blockIdx.y;
  const size_t first = static_cast<size_t>(b) * d.nodes;
  griddep_wait();
  int n = d.tree_lens != nullptr ? d.tree_lens[b] : d.nodes;
  if (n < 0 || n > d.nodes) {
    if (tid == 0 && rank == 0) report(d.dev_err, QMLA_DEVERR_BAD_TREE);
    n = 0;
  }
  if (n == 0) {  // (alike in all CTAs of the cluster)
    if (rank == 0 && tid < d.nodes) d.path[first + tid] = -1;
    if (rank == 0 && tid == 0) {
      d.kept[b] = 0;
      d.next_token[b] = -1;
    }
    return;
  }
  const T* const target = static_cast<const T*>(d.target) + static_cast<size_t>(b) * d.target_seq_stride;
  const T* const draft =
      d.draft == nullptr ? nullptr : static_cast<const T*>(d.draft) + static_cast<size_t>(b) * d.draft_seq_stride;
  if (tid < kMaxNodes) {
    int token = -1, parent = -1;
    float u = 0.0f, p = 0.0f, q = 0.0f;
    if (tid < n) {
      token = d.tokens[first + tid];
      parent = d.parents[first + tid];
      u = fminf(fmaxf(d.uniforms[first + tid], 0.0f), 1.0f - 0x1p-24f);
      if (tid > 0) {
        if (parent < -1 || parent >= tid || token < 0 || token >= d.vocab) {
          if (rank == 0) report(d.dev_err, QMLA_DEVERR_BAD_TREE);
          parent = -1;
        }
        if (parent >= 0) {
          p = as_float(target[static_cast<size_t>(parent) * d.target_row_stride + token]);
          if (draft != nullptr) q = as_float(draft[static_cast<size_t>(parent) * d.draft_row_stride + token]);
        }
      } else {
        if (parent != -1 && rank == 0) report(d.dev_err, QMLA_DEVERR_BAD_TREE);
        parent = -1;
      }
    }
    sh.token[tid] = token;
    sh.parent[tid] = parent;
    sh.u[tid] = u;
    sh.p[tid] = p;
    sh.q[tid] = q;
  }
  __syncthreads();

  // (pieces of whole vectors)
  const int chunk = ((d.vocab + ctas * kVerifyWarps - 1) / (ctas * kVerifyWarps) + 63) / 64 * 64;
  const bool vec = d.vocab % (16 / sizeof(T)) == 0 && d.target_row_stride % (16 / sizeof(T)) == 0 &&
                   d.draft_row_stride % (16 / sizeof(T)) == 0 && (reinterpret_cast<uintptr_t>(target) & 15) == 0 &&
                   (reinterpret_cast<uintptr_t>(draft) & 15) == 0;
  // Warp 0's state: the node, its children not yet looked at, the refusals so far.
  int cur = 0, kept = 1;
  uint64_t children = 0ull;
  bool taken = false;
  Pair more = {0.0f, 0.0f}, mass = {1.0f, 0.0f};  // a = 1 + more once taken, R
  int my_path = lane == 0 ? 0 : -1, my_path2 = -1;  // entries lane and lane + 32
  auto enter = [&](int node) {
    cur = node;
    taken = false;
    more = {0.0f, 0.0f};
    mass = {1.0f, 0.0f};
    const uint32_t lo = __ballot_sync(0xffffffffu, sh.parent[lane] == node);
    const uint32_t hi = __ballot_sync(0xffffffffu, sh.parent[lane + 32] == node);
    children = static_cast<uint64_t>(hi) << 32 | lo;
  };
  if (warp == 0) {
    enter(0);
    if (lane == 0) sh.refused_n = 0;
    __syncwarp();
  }
  cluster_sync_all();  // every CTA of the cluster runs before another writes into it
  for (int pass = 0;; ++pass) {
    if (warp == 0) {
      // On to the next sum that is needed: after a refusal, or where the walk ends.
      bool refusal = false;
      while (children != 0ull && !refusal) {
        const int t = __ffsll(static_cast<long long>(children)) - 1;
        children &= children - 1;
        const float u = sh.u[t], p = sh.p[t], q = sh.q[t];
        if (draft != nullptr) {
          // (u q is exact as a pair)
          const float uq = __fmul_rn(u, q);
          const Pair need = product({uq, __fmaf_rn(u, q, -uq)}, mass);
          const Pair r = taken ? left_over(p, q, Taken(more)) : Pair{fmaxf(p, 0.0f), 0.0f};
          if (above(r, need)) {
            if (lane == (kept & 31)) (kept < 32 ? my_path : my_path2) = t;
            ++kept;
            enter(t);
          } else {
            if (taken) more = add(more, mass);
            taken = refusal = true;
          }
        } else {
          bool gone = false;
          const int m = sh.refused_n;
          for (int i = 0; i < m; ++i) gone |= sh.refused[i] == sh.token[t];
          const float r = gone ? 0.0f : fmaxf(p, 0.0f);
          __syncwarp();
          if (above({r, 0.0f}, times(mass, u))) {
            if (lane == (kept & 31)) (kept < 32 ? my_path : my_path2) = t;
            ++kept;
            enter(t);
            if (lane == 0) sh.refused_n = 0;
          } else if (!gone) {
            mass = add(mass, {-r, 0.0f});
            if (lane == 0) {
              sh.refused[m] = sh.token[t];
              sh.refused_n = m + 1;
            }
          }
          __syncwarp();
        }
      }
      if (lane == 0) {
        sh.cur = cur;
        sh.last = children == 0ull;
        sh.taken = taken;
        sh.b = more;
        sh.found = ~0ull;
      }
    }
    __syncthreads();
    const T* const p = target + static_cast<size_t>(sh.cur) * d.target_row_stride;
    const T* const q = draft == nullptr ? nullptr : draft + static_cast<size_t>(sh.cur) * d.draft_row_stride;
    const Taken took(sh.b);
    const Mode mode = !sh.taken ? kWhole : (sh.b.hi == 0.0f ? kOnce : kMore);
    const int refusals = sh.refused_n;  // (of certain drafts)
    const bool last = sh.last;
    auto counted = [&](int v, Pair r) {  // what is left of token v
      for (int i = 0; i < refusals; ++i)
        if (sh.refused[i] == v) r = {0.0f, 0.0f};
      return r;
    };
    // ---- this warp's piece of the sum
    const int w = rank * kVerifyWarps + warp;
    const int v0 = min(w * chunk, d.vocab), v1 = min(v0 + chunk, d.vocab);
    Pair sum;
    if (mode == kWhole) {
      auto mine = [&](int i) { return i < refusals && sh.refused[i] >= v0 && sh.refused[i] < v1; };
      if (__any_sync(0xffffffffu, mine(lane) || mine(lane + 32))) {
        sum = vec ? row_sum_without<T, true>(p, v0, v1, lane, sh.refused, refusals)
                  : row_sum_without<T, false>(p, v0, v1, lane, sh.refused, refusals);
      } else {
        sum = vec ? row_sum<T, kWhole, true>(p, q, took, v0, v1, lane) : row_sum<T, kWhole, false>(p, q, took, v0, v1, lane);
      }
    } else if (mode == kOnce) {
      sum = vec ? row_sum<T, kOnce, true>(p, q, took, v0, v1, lane) : row_sum<T, kOnce, false>(p, q, took, v0, v1, lane);
    } else {
      sum = vec ? row_sum<T, kMore, true>(p, q, took, v0, v1, lane) : row_sum<T, kMore, false>(p, q, took, v0, v1, lane);
    }
    sum = warp_scan(sum, lane);
    Pair* const part = sh.part[pass & 1];
    if (lane == 31) {
      for (int r = 0; r < ctas; ++r) {
        const uint32_t to = cluster_map(smem_u32(&part[w]), r);
        st_cluster_u32(to, __float_as_uint(sum.hi));
        st_cluster_u32(to + 4, __float_as_uint(sum.lo));
      }
    }
    cluster_sync_all();
    if (warp == 0) {  // every lane a few of the partial sums in a row
      constexpr int kEach = kMaxCluster * kVerifyWarps / 32;
      const int warps = ctas * kVerifyWarps;
      Pair run = {0.0f, 0.0f}, upto[kEach];
#pragma unroll
      for (int i = 0; i < kEach; ++i) {
        upto[i] = run;
        if (lane * kEach + i < warps) run = add(run, part[lane * kEach + i]);
      }
      const Pair incl = warp_scan(run, lane);
      Pair excl = shfl_up(incl, 1);
      if (lane == 0) excl = {0.0f, 0.0f};
      const Pair total = {__shfl_sync(0xffffffffu, incl.hi, 31), __shfl_sync(0xffffffffu, incl.lo, 31)};
      mass = total;
      if (last) {
        if (lane == 0) sh.total = total;
#pragma unroll
        for (int i = 0; i < kEach; ++i)
          if (lane * kEach + i < warps) sh.before[lane * kEach + i] = add(excl, upto[i]);
      }
    }
    if (!last) continue;
    __syncthreads();

    // ---- the draw: the warp whose piece the threshold lies in, then its tokens
    const Pair total = sh.total;
    const Pair cut = times(total, sh.u[0]);
    const bool fine = total.hi > 0.0f && total.hi < INFINITY;
    const int warps = ctas * kVerifyWarps;
    // (One with anything in it, for the sums up to a piece and up to the one before it are rounded apart;
    // the last such where rounding leaves no piece above the cut.)
    if (fine && tid < warps && part[tid].hi > 0.0f) {
      const Pair end = add(sh.before[tid], part[tid]);
      if (above(end, cut)) atomicMin(&sh.found, static_cast<unsigned long long>(tid));
    }
    __syncthreads();
    int piece = static_cast<int>(sh.found);
    if (fine && sh.found == ~0ull)
      for (piece = warps - 1; piece > 0 && !(part[piece].hi > 0.0f); --piece) {}
    __syncthreads();
    if (fine && piece / kVerifyWarps == rank) {
      if (tid == 0) sh.found = ~0ull;
      // A few tokens in a row for each thread; then those of the thread whose sum passes the cut,
      // a lane each.
      const int each = (chunk + kVerifyThreads - 1) / kVerifyThreads;
      const int p0 = min(piece * chunk, d.vocab), p1 = min(p0 + chunk, d.vocab);
      const int t0 = min(p0 + tid * each, p1), t1 = min(t0 + each, p1);
      Pair s = {0.0f, 0.0f};
      for (int v = t0; v < t1; v += 8) {
        float x[8], y[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          x[i] = y[i] = 0.0f;
          if (v + i < t1) {
            x[i] = as_float(p[v + i]);
            if (mode != kWhole) y[i] = as_float(q[v + i]);
          }
        }
#pragma unroll
        for (int i = 0; i < 8; i += 2) {
          const Pairs r = left_over<kMore>(x[i], x[i + 1], y[i], y[i + 1], took);
          s = add(s, counted(v + i, two_sum(lo2(r.hi), lo2(r.lo))));
          s = add(s, counted(v + i + 1, two_sum(hi2(r.hi), hi2(r.lo))));
        }
      }
      const Pair incl = warp_scan(s, lane);
      if (lane == 31) sh.scan[warp] = incl;
      Pair excl = shfl_up(incl, 1);
      if (lane == 0) excl = {0.0f, 0.0f};
      __syncthreads();
      const Pair ends = warp_scan(lane < kVerifyWarps ? sh.scan[lane] : Pair{0.0f, 0.0f}, lane);
      const int w1 = max(warp - 1, 0);
      const Pair below = {__shfl_sync(0xffffffffu, ends.hi, w1), __shfl_sync(0xffffffffu, ends.lo, w1)};
      const Pair run = add(warp > 0 ? add(sh.before[piece], below) : sh.before[piece], excl);
      // (the first thread above the cut, else, where rounding leaves none, the last with anything)
      if (s.hi > 0.0f) atomicMin(&sh.found, above(add(run, s), cut) ? tid : (1ull << 40) - tid);
      __syncthreads();
      const unsigned long long found = sh.found;
      const bool passes = found < (1ull << 32);
      const int who = static_cast<int>(passes ? found : (1ull << 40) - found);
      if (warp == who / 32) {
        const int from = who & 31, first_v = __shfl_sync(0xffffffffu, t0, from), end_v = __shfl_sync(0xffffffffu, t1, from);
        Pair upto = {__shfl_sync(0xffffffffu, run.hi, from), __shfl_sync(0xffffffffu, run.lo, from)};
        int token = -1;
        bool done = false;
        for (int v = first_v; v < end_v && !done; v += 32) {
          const int mine = v + lane;
          Pair x = {0.0f, 0.0f};
          if (mine < end_v)
            x = counted(mine, left_over(as_float(p[mine]), mode != kWhole ? as_float(q[mine]) : 0.0f, took));
          const Pair sum_to = add(upto, warp_scan(x, lane));
          const uint32_t any = __ballot_sync(0xffffffffu, x.hi > 0.0f);
          const uint32_t over = __ballot_sync(0xffffffffu, x.hi > 0.0f && above(sum_to, cut));
          if (any != 0u) token = v + 31 - __clz(any);
          if (over != 0u) {
            token = v + __ffs(over) - 1;
            done = true;
          }
          upto = {__shfl_sync(0xffffffffu, sum_to.hi, 31), __shfl_sync(0xffffffffu, sum_to.lo, 31)};
        }
        if (lane == 0) d.next_token[b] = token;
      }
    }
    if (rank == 0 && warp == 0) {
      if (lane < d.nodes) d.path[first + lane] = my_path;
      if (lane + 32 < d.nodes) d.path[first + lane + 32] = my_path2;
      if (lane == 0) {
        d.kept[b] = kept;
        if (!fine) {
          d.next_token[b] = -1;
          report(d.dev_err, QMLA_DEVERR_BAD_PROBS);
        }
      }
    }
    break;
  }
}

// ----------------------------------------------------------------- kept rows
// The bytes of a slot: pieces of 16, 4, 2 and 1 bytes, and where each lies.
template <int CB>
struct Slot;
template <>
struct Slot<4> {
  using L = BlockLayout<4>;
  static constexpr int n16 = 18, n4 = 9, n2 = 0, n1 = 0, bytes = L::kBytes;
  __device__ static int at16(int k, int slot) { return L::code_off(k >> 1, slot) + 16 * (k & 1); }
  __device__ static int at4(int k, int slot) { return L::sz_off(k, slot); }
  __device__ static int at2(int, int) { return 0; }
  __device__ static int at1(int, int) { return 0; }
};
template <>
struct Slot<2> {
  using L = BlockLayout<2>;
  static constexpr int n16 = 10, n4 = 9, n2 = 0, n1 = 0, bytes = L::kBytes;
  __device__ static int at16(int k, int slot) {
    return k < 8 ? L::code_off(k, slot) : L::code_off(8, slot) + 16 * (k - 8);
  }
  __device__ static int at4(int k, int slot) { return L::sz_off(k, slot); }
  __device__ static int at2(int, int) { return 0; }
  __device__ static int at1(int, int) { return 0; }
};
template <>
struct Slot<kC4R4> {
  using L = BlockLayout<kC4R4>;
  static constexpr int n16 = 18, n4 = 1, n2 = 8, n1 = 9, bytes = L::kBytes;
  __device__ static int at16(int k, int slot) { return L::code_off(k >> 1, slot) + 16 * (k & 1); }
  __device__ static int at4(int, int slot) { return L::pe_scale_off(slot); }
  __device__ static int at2(int k, int slot) { return L::c_scale_off(k, slot); }
  __device__ static int at1(int k, int slot) { return L::zero_off(k, slot); }
};
template <>
struct Slot<16> {
  static constexpr int n16 = 72, n4 = 0, n2 = 0, n1 = 0, bytes = kBf16BlockBytes;
  __device__ static int at16(int k, int slot) { return slot * (kDqk * 2) + 16 * k; }
  __device__ static int at4(int, int) { return 0; }
  __device__ static int at2(int, int) { return 0; }
  __device__ static int at1(int, int) { return 0; }
};

constexpr int kKeepThreads = 256;

// One block a sequence. All rows are in registers before any is written: a row may lie where
// another goes to.
template <int CB>
__global__ void __launch_bounds__(kKeepThreads) keep_kernel(const qmla_keep_desc d) {
  using S = Slot<CB>;
  __shared__ uint8_t* from[kMaxNodes];  // block of the row to move, or null
  __shared__ uint8_t* to[kMaxNodes];
  __shared__ int from_slot[kMaxNodes], to_slot[kMaxNodes], node[kMaxNodes];
  const int tid = threadIdx.x, b = blockIdx.x;
  griddep_wait();
  const int len = d.seq_lens[b], n = d.tree_lens != nullptr ? d.tree_lens[b] : d.nodes, kept = d.kept[b];
  const bool bad_len = len < 0 || len > d.max_blocks * kBlockTokens;
  bool good = !bad_len && n >= 0 && n <= d.nodes && n <= len && kept >= 0 && kept <= n;
  if (good && tid < kept) {
    const int32_t* path = d.path + static_cast<size_t>(b) * d.nodes;
    const int me = path[tid], before = tid > 0 ? path[tid - 1] : -1;
    good = me > before && me < n;
    node[tid] = me;
  }
  good = __syncthreads_and(good);
  if (tid == 0) {
    if (bad_len) report(d.dev_err, QMLA_DEVERR_BAD_POSITION);
    else if (!good) report(d.dev_err, QMLA_DEVERR_BAD_TREE);
    d.new_lens[b] = good ? len - n + kept : len;
  }
  if (!good) return;
  const int ctx = len - n;
  uint8_t* const pool = static_cast<uint8_t*>(d.pool);
  if (tid < kept) {
    const int32_t* row = d.block_table + static_cast<size_t>(b) * d.max_blocks;
    const int src = ctx + node[tid], dst = ctx + tid;
    uint8_t *f = nullptr, *t = nullptr;
    if (src != dst) {
      const int sb = row[src / kBlockTokens], db = row[dst / kBlockTokens];
      if (sb < 0 || sb >= d.num_blocks || db < 0 || db >= d.num_blocks) {
        report(d.dev_err, QMLA_DEVERR_BAD_BLOCK);
      } else {
        f = pool + static_cast<size_t>(sb) * S::bytes;
        t = pool + static_cast<size_t>(db) * S::bytes;
      }
    }
    from[tid] = f;
    to[tid] = t;
    from_slot[tid] = src % kBlockTokens;
    to_slot[tid] = dst % kBlockTokens;
  }
  __syncthreads();
  constexpr int r16 = (kMaxNodes * S::n16 + kKeepThreads - 1) / kKeepThreads;
  constexpr int r4 = (kMaxNodes * S::n4 + kKeepThreads - 1) / kKeepThreads;
  constexpr int r2 = (kMaxNodes * S::n2 + kKeepThreads - 1) / kKeepThreads;
  constexpr int r1 = (kMaxNodes * S::n1 + kKeepThreads - 1) / kKeepThreads;
  uint4 x16[r16 > 0 ? r16 : 1];
  uint32_t x4[r4 > 0 ? r4 : 1];
  uint16_t x2[r2 > 0 ? r2 : 1];
  uint8_t x1[r1 > 0 ? r1 : 1];
#define QMLA_EACH(R, N, AT, TYPE, X, BASE, SLOT, BODY)                          \
  _Pragma("unroll") for (int e = 0; e < (R); ++e) {                             \
    const int item = e * kKeepThreads + tid;                                    \
    const int i = item / ((N) > 0 ? (N) : 1), k = item - i * (N);               \
    if (i < kept && from[i] != nullptr) {                                       \
      TYPE* const at = reinterpret_cast<TYPE*>(BASE[i] + S::AT(k, SLOT[i]));    \
      BODY;                                                                     \
    }                                                                           \
  }
  QMLA_EACH(r16, S::n16, at16, uint4, x16, from, from_slot, x16[e] = *at)
  QMLA_EACH(r4, S::n4, at4, uint32_t, x4, from, from_slot, x4[e] = *at)
  QMLA_EACH(r2, S::n2, at2, uint16_t, x2, from, from_slot, x2[e] = *at)
  QMLA_EACH(r1, S::n1, at1, uint8_t, x1, from, from_slot, x1[e] = *at)
  __syncthreads();
  QMLA_EACH(r16, S::n16, at16, uint4, x16, to, to_slot, *at = x16[e])
  QMLA_EACH(r4, S::n4, at4, uint32_t, x4, to, to_slot, *at = x4[e])
  QMLA_EACH(r2, S::n2, at2, uint16_t, x2, to, to_slot, *at = x2[e])
  QMLA_EACH(r1, S::n1, at1, uint8_t, x1, to, to_slot, *at = x1[e])
#undef QMLA_EACH
  if (CB != 16 && d.prot != nullptr) {
    // (64 positions at most, so no two in a ring row)
    constexpr int kPieces = kDqk * 2 / 16;
    const uint4* rows = reinterpret_cast<const uint4*>(d.draft_rows) + static_cast<size_t>(b) * kMaxNodes * kPieces;
    uint4* const keep = static_cast<uint4*>(d.prot) + static_cast<size_t>(b) * kProtRows * kPieces;
    for (int item = tid; item < kept * kPieces; item += kKeepThreads) {
      const int i = item / kPieces, k = item - i * kPieces, pos = ctx + i;
      const uint4 x = rows[node[i] * kPieces + k];
      keep[(kSinkTokens + pos % kRecentTokens) * kPieces + k] = x;
      if (pos < kSinkTokens) keep[pos * kPieces + k] = x;
    }
  }
}

// (Programmatic launches: the kernels' own start overlaps the end of what is before them, which
// they wait for at once.)
template <typename... Args>
cudaError_t launch(void (*kern)(Args...), dim3 grid, int threads, int cluster, cudaStream_t stream, Args... args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = dim3(threads);
  cfg.stream = stream;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim = {static_cast<unsigned>(cluster), 1, 1};
  cfg.attrs = attr;
  cfg.numAttrs = cluster > 0 ? 2 : 1;
  return cudaLaunchKernelEx(&cfg, kern, args...);
}

}  // namespace

cudaError_t launch_tree_verify(const qmla_verify_desc& d, int sms, cudaStream_t stream) {
  // More CTAs a row while each has 4,096 tokens and all of them run at once (two an SM).
  int ctas = 1;
  while (ctas < kMaxCluster && d.vocab > 4096 * ctas && 2 * ctas * d.batch <= 2 * sms) ctas *= 2;
  auto* const kern = d.probs == QMLA_PROBS_F32 ? verify_kernel<float> : verify_kernel<__nv_bfloat16>;
  return launch(kern, dim3(ctas, d.batch), kVerifyThreads, ctas, stream, d, ctas);
}

cudaError_t launch_cache_keep(const qmla_keep_desc& d, cudaStream_t stream) {
  auto* const kern = d.cache_kind == 4 ? keep_kernel<4>
                                       : (d.cache_kind == 2 ? keep_kernel<2>
                                                            : (d.cache_kind == kC4R4 ? keep_kernel<kC4R4> : keep_kernel<16>));
  return launch(kern, dim3(d.batch), kKeepThreads, 0, stream, d);
}

}  // namespace qmla
