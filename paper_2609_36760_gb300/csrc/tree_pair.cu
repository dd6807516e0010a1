// Attention of a tree's nodes for many query rows: a cluster of two CTAs handles 128 rows, 64
// per CTA, with tcgen05 cta_group::2, over the context as fp16 tiles that the prep kernel has
// laid out in memory once for all rows (decode_tree.cu, expand_block).
//
// A tile is one 64-token block, as M = 128 MMAs over the pair:
//   S[r, t] = q[r, :] . C[t, :]     A: each CTA's 64 rows of q, B: each CTA's 32 tokens (N = 64), K = 576
//   O[r, c] += P[r, :] C[:, c]      A: each CTA's 64 rows of P, B: each CTA's 256 channels (2 x N = 256),
//                                   K = 64 tokens
// Its operands come by bulk copies of the swizzled images: 36 KB of a CTA's own tokens for the
// scores, 32 KB of its own channels for the values, two stages of each. So a block is
// dequantised once for all row groups of its sequence instead of once (and a half) for each, and
// the SM's warps only do the softmax: decode_pair, which dequantises, spends 3.35k cycles a tile
// of which the MMAs are 1.5k.
//
// Short sequences (at most kExactTokens) also have images of what rounding to fp16 left off their
// rows (C - RN_f16(C)), and their scores are the sum of both products: with few keys the
// roundings do not average out of lse (200 INT4 tokens: 2e-5 of it against 1e-7).
//
// TMEM (per CTA; lanes 0..63 hold the first half of N for rows 0..63, lanes 64..127 the second):
// O 2 x 128 columns, S 4 buffers of 32.
#include <cuda_runtime.h>

#include <cstddef>

#include "decode_common.cuh"

namespace qmla {
namespace {

constexpr int kTok = 64;        // tokens per tile: one cache block
constexpr int kSoftWarps = 4;   // warps 0..3, one per TMEM lane quarter
constexpr int kLoadWarp = 5;    // bulk copies; warp 4: MMAs (leader), or arrivals on the leader for the copies
constexpr int kThreads = 6 * 32;
constexpr uint32_t kRows = 64;                        // query rows per CTA
constexpr uint32_t kQBytes = kNumChunks * kRows * 128;
constexpr uint32_t kKBytes = kHalfImage;              // own 32 tokens, K-major B of QK
constexpr uint32_t kKChunk = 32 * 128;
constexpr uint32_t kVChunk = kTok * 128, kVBytes = 4 * kVChunk;  // own channels, MN-major B of PV
constexpr uint32_t kPTile = kRows * 128;              // P, K-major A of PV
constexpr uint32_t kKOff = kQBytes, kVOff = kKOff + 2 * kKBytes, kPOff = kVOff + 2 * kVBytes;
constexpr uint32_t kCtrlOff = kPOff + 2 * kPTile;
constexpr uint32_t kColS = 256, kTmemCols = 512;

struct __align__(16) TreeCtrl {
  // Completed by this CTA's own copies (transaction counts).
  uint64_t k_bar[2], v_bar[2], q_bar;
  // The leader's: the other CTA's copies have landed; P written, S read (4 warps per CTA), O read.
  uint64_t k_peer[2], v_peer[2], q_peer;
  uint64_t p_full[2], s_free[4], o_free;
  // Arrived on by MMA commits, multicast to both CTAs: scores complete, K stage free, PV complete
  // (V stage and P free), every QK of a segment done.
  uint64_t s_full[4], k_free[2], pv_done[2], q_free;
  uint64_t halves[2];  // the two warps that share rows, [warp & 1]
  uint64_t fin;
  uint32_t tmem_base, abort;
  float xch[2][128];
};
constexpr int kSmem = 1024 + kCtrlOff + static_cast<int>(sizeof(TreeCtrl));
static_assert(kSmem <= 232448, "shared memory per CTA");

// The tiles of one pair: its range of the plan's list of 128-token tiles, cut into segments at
// unit ends. Tile q is 64-token block q of a sequence.
struct TreeSched {
  int q, qend, q0;    // current tile, end and first tile of the segment
  int unit, pu0, pu1; // unit and its 128-token tiles in the plan's list
  int b, g, len;
  int t0, t1;
  bool live;
  __device__ void enter(const Params& p, int j) {
    b = unit / p.n_hg;
    g = unit - b * p.n_hg;
    len = p.seq_lens[b];
    q = q0 = 2 * j;
    qend = min(2 * (min(t1, pu1) - pu0), (len + kTok - 1) / kTok);
  }
  __device__ void init(const Params& p, int pair) {
    const int4 info = p.cta_info[pair];
    t0 = p.cta_t0[pair];
    t1 = p.cta_t0[pair + 1];
    unit = info.x;
    pu0 = info.y;
    pu1 = info.z;
    live = t0 < t1;
    q = qend = q0 = b = g = len = 0;
    if (live) enter(p, t0 - pu0);
  }
  __device__ bool first() const { return q == q0; }
  __device__ bool last() const { return q + 1 == qend; }
  __device__ void next(const Params& p) {
    if (++q < qend) return;
    const int t = min(t1, pu1);
    if (t >= t1) {
      live = false;
      return;
    }
    const int units = p.batch * p.n_hg;
    while (t >= pu1 && unit + 1 < units) {
      ++unit;
      pu0 = pu1;
      pu1 = p.prefix[unit + 1];
    }
    enter(p, 0);
  }
  // Products that make up the scores: of the images, and of what they leave off.
  __device__ int parts(const Params& p) const { return p.rest_images != nullptr && len <= kExactTokens ? 2 : 1; }
};

// The order in which the issuer takes QK and PV, and the copies come: QK of a tile goes before PV
// of the tile before it, unless it starts a segment, whose query waits for the last QK of the
// segment before. (QK of tile i so goes after PV of tile i - 2: who has its scores knows that
// its P tile is free.)
struct TreeOrder {
  TreeSched k, v;  // at tiles nk and nv
  uint32_t nk = 0, nv = 0;
  __device__ bool live() const { return v.live; }
  __device__ bool score_next() const { return k.live && nk < nv + 2 && !(k.first() && nk > nv); }
};

__device__ __forceinline__ bool pwait(uint64_t* bar, uint32_t parity, TreeCtrl& c, uint32_t site, uint32_t* dev_err) {
  return wait_ok(mbar_wait(bar, parity, kWaitNs, &c.abort), site, c, dev_err);
}
// The same for a barrier of the leader that the other CTA arrives on: acquired from the cluster.
__device__ __forceinline__ bool pwait_cluster(uint64_t* bar, uint32_t parity, TreeCtrl& c, uint32_t site,
                                              uint32_t* dev_err) {
  if (mbar_test_cluster(bar, parity)) return true;
  const uint64_t t0 = globaltimer_ns();
  for (;;) {
    if (mbar_test_cluster(bar, parity)) return true;
    if (*reinterpret_cast<volatile uint32_t*>(&c.abort) != 0u) return false;
    if (globaltimer_ns() - t0 > kWaitNs) return wait_ok(0, site, c, dev_err);
  }
}

// ------------------------------------------------------------------- copies
__device__ void load_role(const Params& p, const TreeSched& sc, uint8_t* sm, TreeCtrl& ctl, int rank) {
  TreeOrder o;
  o.k = o.v = sc;
  uint32_t kk = 0, seg = 0;
  bool ok = true;
  while (ok && o.live()) {
    if (o.score_next()) {
      const size_t img = static_cast<size_t>(o.k.b) * p.img_width + o.k.q;
      const int parts = o.k.parts(p);
      for (int part = 0; ok && part < parts; ++part, ++kk) {
        const uint32_t st = kk & 1u;
        if (kk >= 2 && !(ok = pwait(&ctl.k_free[st], ((kk >> 1) - 1) & 1u, ctl, kSiteDqSlot, p.dev_err))) break;
        mbar_arrive_expect_tx(&ctl.k_bar[st], kKBytes);
        const uint8_t* src = part == 0 ? p.images + img * kImage
                                       : p.rest_images + (static_cast<size_t>(o.k.b) * p.rest_width + o.k.q) * kImage;
        bulk_g2s(sm + kKOff + st * kKBytes, src + rank * kHalfImage, kKBytes, &ctl.k_bar[st]);
      }
      if (ok && o.k.first()) {
        if (seg > 0 && !(ok = pwait(&ctl.q_free, (seg - 1) & 1u, ctl, kSiteMmaQFull, p.dev_err))) break;
        mbar_arrive_expect_tx(&ctl.q_bar, kQBytes);
        bulk_g2s(sm, p.qimg + (static_cast<size_t>(o.k.b) * p.n_img + 2 * o.k.g + rank) * kQBytes, kQBytes, &ctl.q_bar);
        ++seg;
      }
      ++o.nk;
      o.k.next(p);
    } else {
      const uint32_t st = o.nv & 1u;
      if (o.nv >= 2 && !(ok = pwait(&ctl.pv_done[st], ((o.nv >> 1) - 1) & 1u, ctl, kSiteDqSlot, p.dev_err))) break;
      mbar_arrive_expect_tx(&ctl.v_bar[st], kVBytes);
      const uint8_t* src = p.images + (static_cast<size_t>(o.v.b) * p.img_width + o.v.q) * kImage + 4 * rank * kKChunk;
#pragma unroll 1
      for (int i = 0; i < 8; ++i)  // chunk i / 2, tokens 32 (i & 1) ..
        bulk_g2s(sm + kVOff + st * kVBytes + (i >> 1) * kVChunk + (i & 1) * kKChunk,
                 src + (i & 1) * kHalfImage + (i >> 1) * kKChunk, kKChunk, &ctl.v_bar[st]);
      ++o.nv;
      o.v.next(p);
    }
  }
  if (!ok) set_abort(ctl, p.dev_err);
  // No copy and no commit may reach this CTA once it has left; these waits ignore the abort flag.
  for (uint32_t st = 0; st < 2; ++st) {
    const uint32_t nk = (kk + 1 - st) >> 1, nv = (o.nv + 1 - st) >> 1;  // phases begun on stage st
    if (nk > 0) mbar_wait(&ctl.k_bar[st], (nk - 1) & 1u, kWaitNs, nullptr);
    if (nv > 0) mbar_wait(&ctl.v_bar[st], (nv - 1) & 1u, kWaitNs, nullptr);
    if (ok && nk > 0) mbar_wait(&ctl.k_free[st], (nk - 1) & 1u, kWaitNs, nullptr);
  }
  if (seg > 0) mbar_wait(&ctl.q_bar, (seg - 1) & 1u, kWaitNs, nullptr);
  if (ok && seg > 0) mbar_wait(&ctl.q_free, (seg - 1) & 1u, kWaitNs, nullptr);
}

// The other CTA: tells the leader of each of its copies, in the order in which the issuer asks.
__device__ void relay_role(const Params& p, const TreeSched& sc, TreeCtrl& ctl) {
  TreeOrder o;
  o.k = o.v = sc;
  uint32_t kk = 0, seg = 0;
  bool ok = true;
  const uint32_t kpeer = cluster_map(smem_u32(&ctl.k_peer[0]), 0), vpeer = cluster_map(smem_u32(&ctl.v_peer[0]), 0);
  const uint32_t qpeer = cluster_map(smem_u32(&ctl.q_peer), 0);
  while (ok && o.live()) {
    if (o.score_next()) {
      if (o.k.first()) {
        if (!(ok = pwait(&ctl.q_bar, seg & 1u, ctl, kSiteMmaQFull, p.dev_err))) break;
        mbar_arrive_cluster(qpeer, true);
        ++seg;
      }
      const int parts = o.k.parts(p);
      for (int part = 0; part < parts; ++part, ++kk) {
        if (!(ok = pwait(&ctl.k_bar[kk & 1u], (kk >> 1) & 1u, ctl, kSiteMmaChunk, p.dev_err))) break;
        mbar_arrive_cluster(kpeer + (kk & 1u) * 8, true);
      }
      ++o.nk;
      o.k.next(p);
    } else {
      if (!(ok = pwait(&ctl.v_bar[o.nv & 1u], (o.nv >> 1) & 1u, ctl, kSiteMmaChunk, p.dev_err))) break;
      mbar_arrive_cluster(vpeer + (o.nv & 1u) * 8, true);
      ++o.nv;
      o.v.next(p);
    }
  }
  if (!ok) set_abort(ctl, p.dev_err);
}

// --------------------------------------------------------------------- MMAs
__device__ void issue_role(const Params& p, const TreeSched& sc, uint32_t smem, TreeCtrl& ctl, uint32_t tmem) {
  constexpr uint32_t kIdQK = idesc_f16_f32(128, kTok, false, false);
  constexpr uint32_t kIdPV = idesc_f16_f32(128, 256, false, true);
  const uint64_t qa = smem_desc(smem, 16, 1024, SWZ_128B), kb = smem_desc(smem + kKOff, 16, 1024, SWZ_128B);
  const uint64_t pa = smem_desc(smem + kPOff, 16, 1024, SWZ_128B);
  const uint64_t vb = smem_desc(smem + kVOff, kVChunk, 1024, SWZ_128B);
  TreeOrder o;
  o.k = o.v = sc;
  uint32_t kk = 0, qseg = 0, pseg = 0;
  bool ok = true;
  while (ok && o.live()) {
    if (o.score_next()) {
      const uint32_t n = o.nk;
      if (o.k.first()) {
        if (!(ok = pwait(&ctl.q_bar, qseg & 1u, ctl, kSiteMmaQFull, p.dev_err) &&
                   pwait_cluster(&ctl.q_peer, qseg & 1u, ctl, kSiteMmaQFull, p.dev_err)))
          break;
        ++qseg;
      }
      if (n >= 4 && !(ok = pwait_cluster(&ctl.s_free[n & 3u], ((n >> 2) - 1) & 1u, ctl, kSiteSmSFull, p.dev_err))) break;
      const uint32_t ts = tmem + kColS + (n & 3u) * 32;
      const int parts = o.k.parts(p);
      for (int part = 0; part < parts; ++part, ++kk) {
        const uint32_t st = kk & 1u;
        if (!(ok = pwait(&ctl.k_bar[st], (kk >> 1) & 1u, ctl, kSiteMmaChunk, p.dev_err) &&
                   pwait_cluster(&ctl.k_peer[st], (kk >> 1) & 1u, ctl, kSiteMmaChunk, p.dev_err)))
          break;
        tc_fence_after();
        const uint64_t b1 = kb + ((st * kKBytes) >> 4);
#pragma unroll
        for (int k = 0; k < kNumChunks; ++k) {
#pragma unroll
          for (int s = 0; s < 4; ++s)
            umma2_f16_ss(ts, qa + ((k * kRows * 128 + s * 32) >> 4), b1 + ((k * kKChunk + s * 32) >> 4), kIdQK,
                         k == 0 && s == 0 && part == 0 ? 0u : 1u);
        }
        umma2_commit(&ctl.k_free[st]);
      }
      if (!ok) break;
      umma2_commit(&ctl.s_full[n & 3u]);
      if (o.k.last()) umma2_commit(&ctl.q_free);
      ++o.nk;
      o.k.next(p);
    } else {
      const uint32_t st = o.nv & 1u, ph = (o.nv >> 1) & 1u;
      const bool first = o.v.first();
      if (!(ok = pwait(&ctl.v_bar[st], ph, ctl, kSiteMmaChunk, p.dev_err) &&
                 pwait_cluster(&ctl.v_peer[st], ph, ctl, kSiteMmaChunk, p.dev_err) &&
                 pwait_cluster(&ctl.p_full[st], ph, ctl, kSiteMmaPFull, p.dev_err) &&
                 (!first || pseg == 0 || pwait_cluster(&ctl.o_free, (pseg - 1) & 1u, ctl, kSiteMmaOFree, p.dev_err))))
        break;
      tc_fence_after();
      const uint64_t a1 = pa + ((st * kPTile) >> 4), b1 = vb + ((st * kVBytes) >> 4);
#pragma unroll
      for (int blk = 0; blk < 2; ++blk) {
#pragma unroll
        for (int s = 0; s < 4; ++s)
          umma2_f16_ss(tmem + blk * 128, a1 + ((s * 32) >> 4), b1 + ((blk * 2 * kVChunk + s * 2048) >> 4), kIdPV,
                       first && s == 0 ? 0u : 1u);
      }
      umma2_commit(&ctl.pv_done[st]);
      if (o.v.last()) ++pseg;
      ++o.nv;
      o.v.next(p);
    }
  }
  if (!ok) set_abort(ctl, p.dev_err);
  // Every MMA must have landed before TMEM and shared memory are released; this wait ignores
  // the abort flag.
  umma2_commit_local(&ctl.fin);
  wait_ok(mbar_wait(&ctl.fin, 0, kWaitNs, nullptr), kSiteMmaFin, ctl, p.dev_err);
}

// ------------------------------------------------------------------- softmax
__device__ __forceinline__ void arrive_leader(int lane, uint32_t bar_addr) { mbar_arrive_remote(bar_addr, lane == 0); }

// Thread (row, half): query row `row` of the CTA and half the tokens of a tile; in O, half the
// channels. P = 2^(S scale log2e - m) in fp16 with a reference m per row, raised when a score
// exceeds it by 2^8; l sums the weights before their rounding.
__device__ void softmax_role(const Params& p, TreeSched sc, uint32_t smem, TreeCtrl& ctl, uint32_t tmem, int rank,
                             int warp, int lane, int pair) {
  const int half = warp >> 1, row = (warp & 1) * 32 + lane;
  const uint32_t lanes = static_cast<uint32_t>(warp * 32) << 16;
  const uint32_t t_o = tmem + lanes;
  const float sl2 = p.scale_log2;
  const uint32_t sfree = cluster_map(smem_u32(&ctl.s_free[0]), 0), pfull = cluster_map(smem_u32(&ctl.p_full[0]), 0);
  const uint32_t ofree = cluster_map(smem_u32(&ctl.o_free), 0);
  uint64_t* const both = &ctl.halves[warp & 1];
  uint32_t n = 0, ex = 0;
  bool ok = true, whole = false;
  float m = -INFINITY, l = 0.0f;
  int ctx = 0;            // positions before the tree that this row sees (all or none)
  uint64_t line = 0ull;   // nodes that it sees

  // The other half's value of a per-row quantity.
  auto exchange = [&](float mine, float& other) {
    const uint32_t buf = ex & 1u;
    ctl.xch[buf][half * 64 + row] = mine;
    __syncwarp();
    mbar_arrive_if(lane == 0 ? 1u : 0u, both);
    ok = wwait(both, buf, ctl, kSiteGrp, p.dev_err);
    other = ctl.xch[buf][(1 - half) * 64 + row];
    ++ex;
    return ok;
  };

  for (; ok && sc.live; sc.next(p)) {
    const bool first = sc.first();
    if (first) {
      const int t = ((sc.g * 2 + rank) * static_cast<int>(kRows) + row) / p.hpt;
      const TreeSeq& tree = p.trees[sc.b];
      const bool alive = t < kMaxNodes && ((tree.alive >> t) & 1ull);
      ctx = tree.ctx;
      line = alive ? tree.line[t] : 0ull;
      m = -INFINITY;
      l = 0.0f;
      whole = sc.q == 0;
    }
    // which of the 32 columns the row sees
    const int pos = kTok * sc.q + 32 * half, d = pos - ctx;
    uint32_t mask = 0u;
    if (line != 0ull) {
      mask = d <= -32 ? ~0u : (d < 0 ? (1u << -d) - 1u : 0u);
      if (d >= 0 && d < 64) mask |= static_cast<uint32_t>(line >> d);
      if (d < 0 && d > -32) mask |= static_cast<uint32_t>(line << -d);
    }
    const bool full = __all_sync(0xffffffffu, mask == ~0u);
    if (!(ok = wwait(&ctl.s_full[n & 3u], (n >> 2) & 1u, ctl, kSiteSmSFull, p.dev_err))) break;
    tc_fence_after();
    float x[32], top;
    tmem_ld32_max(tmem + kColS + (n & 3u) * 32 + lanes, x, top);
    tmem_ld_wait();
    tc_fence_before();
    __syncwarp();
    arrive_leader(lane, sfree + (n & 3u) * 8);
    if (!full) {
      top = -INFINITY;
#pragma unroll
      for (int i = 0; i < 32; ++i) top = fmaxf(top, (mask >> i) & 1u ? x[i] : -INFINITY);
    }
    float mine = top * sl2, other = 0.0f;
    if (!exchange(mine, other)) break;
    mine = fmaxf(mine, other);
    const bool raise = first ? mine > m : mine > m + kRescaleLog2;
    if (__any_sync(0xffffffffu, raise)) {
      const float a = raise && m != -INFINITY ? exp2f(m - mine) : 1.0f;
      if (raise) m = mine;
      l *= a;
      if (!first && __any_sync(0xffffffffu, a != 1.0f)) {
        if (!(ok = wwait(&ctl.pv_done[(n - 1) & 1u], ((n - 1) >> 1) & 1u, ctl, kSitePvEpi, p.dev_err))) break;
        tc_fence_after();
#pragma unroll 1
        for (int c = 0; c < 256; c += 32) {
          uint32_t r[32];
          tmem_ld32(t_o + c, r);
          tmem_ld_wait();
#pragma unroll
          for (int e = 0; e < 32; ++e) r[e] = __float_as_uint(__uint_as_float(r[e]) * a);
          tmem_st32(t_o + c, r);
        }
        tmem_st_wait();
      }
    }
    // (a row that has seen no key has no reference: its columns are all masked)
    const float ref = m == -INFINITY ? 0.0f : m;
    const uint32_t st = n & 1u;
    const uint32_t ptile = smem + kPOff + st * kPTile;
    float s0 = 0.0f, s1 = 0.0f, s2 = 0.0f, s3 = 0.0f;
#pragma unroll
    for (int i = 0; i < 32; i += 8) {
      float w[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float y = __fmaf_rn(x[i + e], sl2, -ref);
        w[e] = ex2_approx(full || ((mask >> (i + e)) & 1u) ? y : -INFINITY);
      }
      s0 += w[0] + w[4];
      s1 += w[1] + w[5];
      s2 += w[2] + w[6];
      s3 += w[3] + w[7];
      sts_v4(ptile + swz_off(row, half * 4 + i / 8, 128), pack_h2(w[0], w[1]), pack_h2(w[2], w[3]), pack_h2(w[4], w[5]),
             pack_h2(w[6], w[7]));
    }
    fence_proxy_async_smem();
    tc_fence_before();
    __syncwarp();
    arrive_leader(lane, pfull + st * 8);
    l += (s0 + s1) + (s2 + s3);
    ++n;
    if (!sc.last()) continue;

    // ---- segment end: out = O / l in bf16, or the partial (m, l, o)
    whole = whole && sc.t1 >= sc.pu1;
    float lo = 0.0f;
    if (!exchange(l, lo)) break;
    const float lt = half == 0 ? l + lo : lo + l;
    const float inv = lt > 0.0f ? 1.0f / lt : 0.0f;
    if (!(ok = wwait(&ctl.pv_done[(n - 1) & 1u], ((n - 1) >> 1) & 1u, ctl, kSitePvEpi, p.dev_err))) break;
    tc_fence_after();
    // Through the P tiles, 128 bytes of a row at a time, so that a warp stores whole lines. The
    // two warps that share 32 rows of both tiles take one tile each; the weights of the next
    // segment come after the exchange of its first tile, when both are through.
    const int h0 = (sc.g * 2 + rank) * static_cast<int>(kRows) + (warp & 1) * 32;  // the warp's first row
    const int rows = min(32, p.heads - h0);
    const uint32_t buf = smem + kPOff + half * kPTile + (warp & 1) * 4096;
    if (whole) {
      __nv_bfloat16* const dst = reinterpret_cast<__nv_bfloat16*>(p.out) +
                                 (static_cast<size_t>(sc.b) * p.heads + h0) * kDc + half * 256 + (lane & 7) * 8;
#pragma unroll 1
      for (int c = 0; c < 256; c += 64) {
#pragma unroll
        for (int part = 0; part < 2; ++part) {
          uint32_t r[32];
          tmem_ld32(t_o + c + 32 * part, r);
          tmem_ld_wait();
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            uint32_t w[4];
#pragma unroll
            for (int e = 0; e < 4; ++e)
              w[e] = pack_bf16(__uint_as_float(r[8 * q + 2 * e]) * inv, __uint_as_float(r[8 * q + 2 * e + 1]) * inv);
            sts_v4(buf + swz_off(lane, 4 * part + q, 128), w[0], w[1], w[2], w[3]);
          }
        }
        __syncwarp();
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const int rr = 4 * i + (lane >> 3);
          const uint4 o = lds_v4(buf + swz_off(rr, lane & 7, 128));
          if (rr < rows) *reinterpret_cast<uint4*>(dst + static_cast<size_t>(rr) * kDc + c) = o;
        }
        __syncwarp();
      }
      if (half == 0 && lane < rows && p.lse != nullptr)
        p.lse[static_cast<size_t>(sc.b) * p.heads + h0 + lane] = (m + log2f(lt)) * kLn2;
    } else {
      const size_t row0 = (static_cast<size_t>(pair) + sc.unit) * 128 + rank * kRows + (warp & 1) * 32;
      float* const dst = p.part_o + row0 * kDc + half * 256 + (lane & 7) * 4;
#pragma unroll 1
      for (int c = 0; c < 256; c += 32) {
        uint32_t r[32];
        tmem_ld32(t_o + c, r);
        tmem_ld_wait();
#pragma unroll
        for (int q = 0; q < 8; ++q) sts_v4(buf + swz_off(lane, q, 128), r[4 * q], r[4 * q + 1], r[4 * q + 2], r[4 * q + 3]);
        __syncwarp();
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const int rr = 4 * i + (lane >> 3);
          const uint4 o = lds_v4(buf + swz_off(rr, lane & 7, 128));
          if (rr < rows) *reinterpret_cast<uint4*>(dst + static_cast<size_t>(rr) * kDc + c) = o;
        }
        __syncwarp();
      }
      if (half == 0 && lane < rows) {
        p.part_ml[(row0 + lane) * 2] = m;
        p.part_ml[(row0 + lane) * 2 + 1] = lt;
      }
    }
    tc_fence_before();
    __syncwarp();
    arrive_leader(lane, ofree);
  }
  if (!ok && lane == 0) set_abort(ctl, p.dev_err);
}

__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kThreads, 1) tree_pair(const __grid_constant__ Params p) {
  extern __shared__ uint8_t smem_raw[];
  uint8_t* sm = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  const uint32_t smem = smem_u32(sm);
  TreeCtrl& ctl = *reinterpret_cast<TreeCtrl*>(sm + kCtrlOff);
  const int warp = __shfl_sync(0xffffffffu, static_cast<int>(threadIdx.x) >> 5, 0);
  const int lane = threadIdx.x & 31;
  const int rank = static_cast<int>(cluster_ctarank());
  const int pair = static_cast<int>(blockIdx.x >> 1);
  if (threadIdx.x == 0) {
    for (int i = 0; i < 2; ++i) {
      mbar_init(&ctl.k_bar[i], 1);
      mbar_init(&ctl.v_bar[i], 1);
      mbar_init(&ctl.k_peer[i], 1);
      mbar_init(&ctl.v_peer[i], 1);
      mbar_init(&ctl.p_full[i], 2 * kSoftWarps);
      mbar_init(&ctl.s_free[i], 2 * kSoftWarps);
      mbar_init(&ctl.s_free[i + 2], 2 * kSoftWarps);
      mbar_init(&ctl.s_full[i], 1);
      mbar_init(&ctl.s_full[i + 2], 1);
      mbar_init(&ctl.k_free[i], 1);
      mbar_init(&ctl.pv_done[i], 1);
      mbar_init(&ctl.halves[i], 2);
    }
    mbar_init(&ctl.q_bar, 1);
    mbar_init(&ctl.q_peer, 1);
    mbar_init(&ctl.q_free, 1);
    mbar_init(&ctl.o_free, 2 * kSoftWarps);
    mbar_init(&ctl.fin, 1);
    ctl.abort = 0u;
    fence_mbar_init();
  }
  if (warp == 0) {
    tmem_alloc2(&ctl.tmem_base, kTmemCols);
    tmem_relinquish2();
  }
  tc_fence_before();
  __syncthreads();
  cluster_sync_all();  // the other CTA's barriers are initialised
  tc_fence_after();
  const uint32_t tmem = __shfl_sync(0xffffffffu, ctl.tmem_base, 0);
  // The set-up above may overlap the prep kernel; everything below reads what it produced.
  griddep_wait();
  if (warp < kSoftWarps) {
    TreeSched sc;
    sc.init(p, pair);
    softmax_role(p, sc, smem, ctl, tmem, rank, warp, lane, pair);
  } else if (elect_one()) {  // (single threads; the other lanes leave, see decode_pair)
    TreeSched sc;
    sc.init(p, pair);
    if (warp == kLoadWarp) {
      load_role(p, sc, sm, ctl, rank);
    } else if (rank == 0) {
      issue_role(p, sc, smem, ctl, tmem);
    } else {
      relay_role(p, sc, ctl);
    }
  } else {
    asm volatile("exit;");
  }
  griddep_launch_dependents();  // the merge may be scheduled as CTAs finish
  tc_fence_before();
  // Neither CTA leaves while the other may still arrive on its barriers or its tensor core
  // reads this CTA's operands (exited threads do not take part).
  cluster_arrive_wait();
  if (warp == 0) {
    tc_fence_after();
    tmem_dealloc2(tmem, kTmemCols);
  }
}

}  // namespace

cudaError_t launch_tree_pair(const Params& prm, cudaStream_t stream) {
  static int configured_device = -1;
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  if (configured_device != dev) {
    e = cudaFuncSetAttribute(tree_pair, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmem);
    if (e != cudaSuccess) return e;
    configured_device = dev;
  }
  return launch_k(tree_pair, dim3(2 * prm.grid), dim3(kThreads), kSmem, stream, true, prm);
}

}  // namespace qmla
