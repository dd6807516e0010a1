// Attention of a tree's nodes for many query rows: a cluster of two CTAs handles 128 rows, 64
// per CTA, with tcgen05 cta_group::2, over the context as fp16 tiles that the prep kernel has
// laid out in memory once for all rows (decode_tree.cu, expand_block).
//
// A tile is 128 tokens, two cache blocks, as M = 128 MMAs over the pair:
//   S[r, t] = q[r, :] . C[t, :]     A: each CTA's 64 rows of q, B: each CTA's block (N = 128), K = 576
//   O[r, c] += P[r, :] C[:, c]      A: each CTA's 64 rows of P, B: each CTA's 256 channels (2 x N = 256),
//                                   K = 128 tokens
// Its operands come by bulk copies of the swizzled images: 72 KB of a CTA's own block for the
// scores, 64 KB of its own channels of both blocks for the values. So a block is dequantised
// once for all row groups of its sequence instead of once (and a half) for each, and the SM's
// warps only do the softmax (decode_pair, which dequantises, spends 6.7k cycles on 128 tokens).
//
// There is room for one tile of each operand. Its parts (three of the keys', four of the
// values') are filled, used and freed one by one: the scores of a tile take half of the time
// that its values leave them, so that a part's copy has most of a tile's time to arrive.
//
// Where lse is asked for, there are also images of what rounding to fp16 left off the rows
// (C - RN_f16(C)), and the scores are the sum of both products. The roundings average out of lse
// over many keys of like weight, but not where a few keys have most of it: 2e-6 to 4e-5 of it,
// at any length, against 1e-7. (The results, in bf16, do not need it.)
//
// TMEM (per CTA; lanes 0..63 hold the first half of N for rows 0..63, lanes 64..127 the second):
// O 2 x 128 columns, S 2 buffers of 64.
#include <cuda_runtime.h>

#include <cstddef>

#include "decode_common.cuh"

namespace qmla {
namespace {

constexpr int kSoftWarps = 4;   // warps 0..3, one per TMEM lane quarter
constexpr int kLoadWarp = 5;    // bulk copies; warp 4: MMAs (leader), or arrivals on the leader for the copies
constexpr int kThreads = 6 * 32;
constexpr uint32_t kRows = 64;                        // query rows per CTA
constexpr uint32_t kChunk = 64 * 128;                 // 64 rows or tokens x 64 channels
constexpr uint32_t kQBytes = kNumChunks * kChunk;
constexpr uint32_t kKBytes = kImage;                  // own block, K-major B of QK
constexpr uint32_t kVChunk = 2 * kChunk, kVBytes = 4 * kVChunk;  // own channels, MN-major B of PV
constexpr uint32_t kPBytes = 2 * kRows * 128;         // P, K-major A of PV: 64 tokens, then the others
constexpr uint32_t kKOff = kQBytes, kVOff = kKOff + kKBytes, kPOff = kVOff + kVBytes;
constexpr uint32_t kCtrlOff = kPOff + kPBytes;
constexpr uint32_t kColS = 256, kTmemCols = 512;
// Parts of the operands: three chunks of the keys (and of the query, where a segment starts);
// 128 channels of 64 tokens of the values.
constexpr int kKeyParts = 3, kValueParts = 4;
constexpr uint32_t kKeyPart = 3 * kChunk, kValuePart = 2 * kChunk;

struct __align__(16) TreeCtrl {
  // A part is there: this CTA's own copies (transaction counts), in the leader also an arrival
  // for the other CTA's.
  uint64_t k_bar[kKeyParts], v_bar[kValueParts];
  // The leader's: P written (4 warps per CTA), and before it, where a segment starts, O read.
  uint64_t p_full;
  // Arrived on by MMA commits, multicast to both CTAs: scores complete, a part free (the last of
  // the values': PV complete, P free).
  uint64_t s_full[2], k_free[kKeyParts], v_free[kValueParts];
  uint64_t fin;
  uint32_t tmem_base, abort;
  float xch[2][128];
};
constexpr int kSmem = 1024 + kCtrlOff + static_cast<int>(sizeof(TreeCtrl));
static_assert(kSmem <= 232448, "shared memory per CTA");

// The tiles of one pair: its range of the plan's list of 128-token tiles, cut into segments at
// unit ends. Tile q is blocks 2 q and 2 q + 1 of a sequence.
struct TreeSched {
  int q, qend, q0;    // current tile, end and first tile of the segment
  int unit, pu0, pu1; // unit and its tiles in the plan's list
  int b, g;
  int t0, t1;
  bool live;
  __device__ void enter(const Params& p, int j) {
    tree_unit(p, unit, b, g);
    q = q0 = j;
    qend = min(t1, pu1) - pu0;
  }
  __device__ void init(const Params& p, int pair) {
    const int4 info = p.cta_info[pair];
    t0 = p.cta_t0[pair];
    t1 = p.cta_t0[pair + 1];
    unit = info.x;
    pu0 = info.y;
    pu1 = info.z;
    live = t0 < t1;
    q = qend = q0 = b = g = 0;
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
};

// The order in which the issuer takes QK and PV, and the copies come: QK of a tile goes before PV
// of the tile before it. (So the softmax of a tile has the QK of the next one to work under, and
// QK of tile i goes after PV of tile i - 2, whose P shows that its scores have been read.)
// A tile has one or two passes of QK, over the images and over what they leave off, and two halves
// of PV, of 128 of a CTA's channels each. Two passes are kept apart by halves,
//   QK(i + 1), PV(i) first half, rest of QK(i + 1), PV(i) second half, QK(i + 2) ..,
// for each pass has all of the keys' room, and its copies have half a PV to arrive in (2 x 30,000
// tokens, 64 nodes x 64 heads: 442 to 434 us).
// (One pass and whole PVs are a kernel of their own: the counting of halves cost it 3%.)
template <int PASSES>
struct TreeOrder {
  static constexpr int kParts = kValueParts / PASSES;  // of the values, in a step of PV
  TreeSched k, v;                                      // tiles of the next pass and step of PV
  uint32_t pass = 0, step = 0;                         // counted
  __device__ explicit TreeOrder(const TreeSched& sc) : k(sc), v(sc) {}
  __device__ bool live() const { return v.live; }
  __device__ bool score_next() const { return k.live && pass < step + 1 + PASSES; }
  __device__ bool rest() const { return PASSES == 2 && (pass & 1u); }
  __device__ bool ends() const { return PASSES == 1 || (pass & 1u); }  // last pass of its tile
  __device__ uint32_t scored() const { return pass / PASSES; }         // tile of the pass
  __device__ uint32_t summed() const { return step / PASSES; }         // and of the step
  __device__ int half() const { return PASSES == 1 ? 0 : step & 1u; }
  __device__ void pass_done(const Params& p) {
    if (ends()) k.next(p);
    ++pass;
  }
  __device__ void step_done(const Params& p) {
    if (PASSES == 1 || (step & 1u)) v.next(p);
    ++step;
  }
};

__device__ __forceinline__ bool pwait(uint64_t* bar, uint32_t parity, TreeCtrl& c, uint32_t site, uint32_t* dev_err) {
  return wait_ok(mbar_wait(bar, parity, kWaitNs, &c.abort), site, c, dev_err);
}
// The same for a barrier of the leader that the other CTA arrives on: acquired from the cluster.
__device__ __forceinline__ bool try_wait_cluster(uint64_t* bar, uint32_t parity) {
  uint32_t ok;
  asm volatile(
      "{\n\t.reg .pred p;\n\tmbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2;\n\t"
      "selp.u32 %0, 1, 0, p;\n\t}"
      : "=r"(ok)
      : "r"(smem_u32(bar)), "r"(parity)
      : "memory");
  return ok != 0;
}
__device__ __forceinline__ bool pwait_cluster(uint64_t* bar, uint32_t parity, TreeCtrl& c, uint32_t site,
                                              uint32_t* dev_err) {
  if (mbar_test_cluster(bar, parity)) return true;
  const uint64_t t0 = globaltimer_ns();
  for (;;) {
    if (try_wait_cluster(bar, parity)) return true;
    if (*reinterpret_cast<volatile uint32_t*>(&c.abort) != 0u) return false;
    if (globaltimer_ns() - t0 > kWaitNs) return wait_ok(0, site, c, dev_err);
  }
}

// ------------------------------------------------------------------- copies
template <int PASSES>
__device__ void load_role(const Params& p, const TreeSched& sc, uint8_t* sm, TreeCtrl& ctl, int rank) {
  TreeOrder<PASSES> o(sc);
  uint32_t copies = 0, values = 0;  // parts asked for
  bool ok = true;
  while (ok && o.live()) {
    if (o.score_next()) {
      const int block = 2 * o.k.q + rank;
      const uint8_t* q = p.qimg + (static_cast<size_t>(o.k.b) * p.n_img + 2 * o.k.g + rank) * kQBytes;
      const uint8_t* src = (o.rest() ? p.rest_images : p.images) + (static_cast<size_t>(o.k.b) * p.img_width + block) * kImage;
      const bool query = !o.rest() && o.k.first();  // (its part's last reader was that of the keys')
#pragma unroll 1
      for (int part = 0; part < kKeyParts; ++part) {
        uint64_t* const bar = &ctl.k_bar[part];
        if (o.pass > 0 && !(ok = pwait(&ctl.k_free[part], (o.pass - 1) & 1u, ctl, kSiteDqSlot, p.dev_err))) break;
        mbar_arrive_expect_tx(bar, query ? 2 * kKeyPart : kKeyPart);
        if (query) bulk_g2s(sm + part * kKeyPart, q + part * kKeyPart, kKeyPart, bar);
        bulk_g2s(sm + kKOff + part * kKeyPart, src + part * kKeyPart, kKeyPart, bar);
        ++copies;
      }
      o.pass_done(p);
    } else {
      const uint8_t* src = p.images + (static_cast<size_t>(o.v.b) * p.img_width + 2 * o.v.q) * kImage + 4 * rank * kChunk;
#pragma unroll 1
      for (int i = 0; i < o.kParts; ++i) {  // channels 128 (part / 2) .., block part & 1
        const int part = o.kParts * o.half() + i;
        uint64_t* const bar = &ctl.v_bar[part];
        if (o.summed() > 0 && !(ok = pwait(&ctl.v_free[part], (o.summed() - 1) & 1u, ctl, kSiteDqSlot, p.dev_err))) break;
        mbar_arrive_expect_tx(bar, kValuePart);
#pragma unroll
        for (int c = part & ~1; c < (part & ~1) + 2; ++c)
          bulk_g2s(sm + kVOff + c * kVChunk + (part & 1) * kChunk, src + (part & 1) * kImage + c * kChunk, kChunk, bar);
        ++values;
      }
      o.step_done(p);
    }
  }
  if (!ok) set_abort(ctl, p.dev_err);
  // No copy and no commit may reach this CTA once it has left; these waits ignore the abort flag.
  for (uint32_t i = 0; i < kKeyParts; ++i) {
    const uint32_t n = (copies + kKeyParts - 1 - i) / kKeyParts;  // phases begun
    if (n > 0) mbar_wait(&ctl.k_bar[i], (n - 1) & 1u, kWaitNs, nullptr);
    if (ok && n > 0) mbar_wait(&ctl.k_free[i], (n - 1) & 1u, kWaitNs, nullptr);
  }
  for (uint32_t i = 0; i < kValueParts; ++i) {
    const uint32_t n = (values + kValueParts - 1 - i) / kValueParts;
    if (n > 0) mbar_wait(&ctl.v_bar[i], (n - 1) & 1u, kWaitNs, nullptr);
    if (ok && n > 0) mbar_wait(&ctl.v_free[i], (n - 1) & 1u, kWaitNs, nullptr);
  }
}

// The other CTA: tells the leader of each of its copies, in the order in which the issuer asks.
// (The tensor core of this SM reads what they brought, and this thread has written nothing, so
// the arrivals release nothing to the cluster: with that release each took more than a
// thousand cycles, 4,700 instead of 1,830 for 64 tokens.)
template <int PASSES>
__device__ void relay_role(const Params& p, const TreeSched& sc, TreeCtrl& ctl) {
  TreeOrder<PASSES> o(sc);
  bool ok = true;
  const uint32_t kbar = cluster_map(smem_u32(&ctl.k_bar[0]), 0), vbar = cluster_map(smem_u32(&ctl.v_bar[0]), 0);
  while (ok && o.live()) {
    if (o.score_next()) {
#pragma unroll 1
      for (int part = 0; part < kKeyParts; ++part) {
        if (!(ok = pwait(&ctl.k_bar[part], o.pass & 1u, ctl, kSiteMmaChunk, p.dev_err))) break;
        mbar_arrive_remote(kbar + part * 8, true);
      }
      o.pass_done(p);
    } else {
#pragma unroll 1
      for (int i = 0; i < o.kParts; ++i) {
        const int part = o.kParts * o.half() + i;
        if (!(ok = pwait(&ctl.v_bar[part], o.summed() & 1u, ctl, kSiteMmaChunk, p.dev_err))) break;
        mbar_arrive_remote(vbar + part * 8, true);
      }
      o.step_done(p);
    }
  }
  if (!ok) set_abort(ctl, p.dev_err);
}

// --------------------------------------------------------------------- MMAs
template <int PASSES>
__device__ void issue_role(const Params& p, const TreeSched& sc, uint32_t smem, TreeCtrl& ctl, uint32_t tmem) {
  constexpr uint32_t kIdQK = idesc_f16_f32(128, 128, false, false);
  constexpr uint32_t kIdPV = idesc_f16_f32(128, 256, false, true);
  const uint64_t qa = smem_desc(smem, 16, 1024, SWZ_128B), kb = smem_desc(smem + kKOff, 16, 1024, SWZ_128B);
  const uint64_t pa = smem_desc(smem + kPOff, 16, 1024, SWZ_128B);
  const uint64_t vb = smem_desc(smem + kVOff, kVChunk, 1024, SWZ_128B);
  TreeOrder<PASSES> o(sc);
  bool ok = true;
  while (ok && o.live()) {
    if (o.score_next()) {
      const uint32_t s_at = o.scored() & 1u, ts = tmem + kColS + s_at * 64;
      const bool adds = o.rest();
#pragma unroll(PASSES == 1 ? kKeyParts : 1)
      for (int part = 0; part < kKeyParts; ++part) {
        if (!(ok = pwait_cluster(&ctl.k_bar[part], o.pass & 1u, ctl, kSiteMmaChunk, p.dev_err))) break;
        tc_fence_after();
#pragma unroll
        for (int k = 3 * part; k < 3 * part + 3; ++k) {
#pragma unroll
          for (int s = 0; s < 4; ++s)
            umma2_f16_ss(ts, qa + ((k * kChunk + s * 32) >> 4), kb + ((k * kChunk + s * 32) >> 4), kIdQK,
                         k == 0 && s == 0 && !adds ? 0u : 1u);
        }
        umma2_commit(&ctl.k_free[part]);
      }
      if (!ok) break;
      if (o.ends()) umma2_commit(&ctl.s_full[s_at]);
      o.pass_done(p);
    } else {
      const uint32_t ph = o.summed() & 1u;
      const bool first = o.v.first();
      if (o.half() == 0 && !(ok = pwait_cluster(&ctl.p_full, ph, ctl, kSiteMmaPFull, p.dev_err))) break;
#pragma unroll(PASSES == 1 ? kValueParts : 1)
      for (int i = 0; i < o.kParts; ++i) {
        const int part = o.kParts * o.half() + i;
        if (!(ok = pwait_cluster(&ctl.v_bar[part], ph, ctl, kSiteMmaChunk, p.dev_err))) break;
        tc_fence_after();
#pragma unroll
        for (int s = 0; s < 4; ++s)
          umma2_f16_ss(tmem + (part >> 1) * 128, pa + (((part & 1) * kRows * 128 + s * 32) >> 4),
                       vb + (((part >> 1) * 2 * kVChunk + (part & 1) * kChunk + s * 2048) >> 4), kIdPV,
                       first && (part & 1) == 0 && s == 0 ? 0u : 1u);
        umma2_commit(&ctl.v_free[part]);
      }
      if (!ok) break;
      o.step_done(p);
    }
  }
  if (!ok) set_abort(ctl, p.dev_err);
  // Every MMA must have landed before TMEM and shared memory are released; this wait ignores
  // the abort flag.
  umma2_commit_local(&ctl.fin);
  wait_ok(mbar_wait(&ctl.fin, 0, kWaitNs, nullptr), kSiteMmaFin, ctl, p.dev_err);
}

// ------------------------------------------------------------------- softmax
__device__ __forceinline__ void stg_v8(void* ptr, const uint32_t* w) {
  asm volatile("st.global.v8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"l"(ptr), "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]),
               "r"(w[4]), "r"(w[5]), "r"(w[6]), "r"(w[7])
               : "memory");
}
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
  const uint32_t pfull = cluster_map(smem_u32(&ctl.p_full), 0);
  uint32_t n = 0, ex = 0;
  bool ok = true, whole = false, all_alive = false;
  float m = -INFINITY, l = 0.0f;
  int ctx = 0;            // positions before the tree that this row sees (all or none)
  uint64_t line = 0ull;   // nodes that it sees

  // A per-row quantity for the thread of the other half, and that one's. (The two warps that
  // share rows meet at a barrier of theirs; one that gives up arrives there too, after it has
  // set the abort word, which is therefore read behind the barrier.)
  auto give = [&](float mine) { ctl.xch[ex & 1u][half * 64 + row] = mine; };
  auto take = [&](float& other) {
    asm volatile("bar.sync %0, 64;" ::"r"(1 + (warp & 1)) : "memory");
    other = ctl.xch[ex & 1u][(1 - half) * 64 + row];
    ok = *reinterpret_cast<volatile uint32_t*>(&ctl.abort) == 0u;
    ++ex;
    return ok;
  };
  // PV of tile i has completed: its P may be overwritten, O moved or read.
  auto wait_pv = [&](uint32_t i) {
    ok = wwait(&ctl.v_free[kValueParts - 1], i & 1u, ctl, kSitePvEpi, p.dev_err);
    tc_fence_after();
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
      all_alive = __all_sync(0xffffffffu, line != 0ull);
    }
    const int d = kTileTokens * sc.q + 64 * half - ctx;  // node in the first of the 64 columns
    const bool full = all_alive && d <= -64;
    if (!(ok = wwait(&ctl.s_full[n & 1u], (n >> 1) & 1u, ctl, kSiteSmSFull, p.dev_err))) break;
    tc_fence_after();
    float x[64], top, top2;
    tmem_ld32_max(tmem + kColS + (n & 1u) * 64 + lanes, x, top);
    tmem_ld32_max(tmem + kColS + (n & 1u) * 64 + 32 + lanes, x + 32, top2);
    tmem_ld_wait();
    top = fmaxf(top, top2);
    if (!full) {  // the columns that the row sees: the context's, and the nodes of its line
      uint64_t mask = 0ull;
      if (line != 0ull) {
        if (d <= -64) mask = ~0ull;
        else if (d < 0) mask = ((1ull << -d) - 1ull) | (line << -d);
        else if (d < 64) mask = line >> d;
      }
      const uint32_t lo = static_cast<uint32_t>(mask), hi = static_cast<uint32_t>(mask >> 32);
      top = -INFINITY;
#pragma unroll
      for (int i = 0; i < 64; ++i) {
        x[i] = ((i < 32 ? lo : hi) >> (i & 31)) & 1u ? x[i] : -INFINITY;
        top = fmaxf(top, x[i]);
      }
    }
    uint32_t pk[32];
    float sum = 0.0f;
    // (a row that has seen no key has no reference: its columns are all masked)
    auto weights = [&]() {
      const float ref = m == -INFINITY ? 0.0f : m;
      float s[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
      for (int i = 0; i < 64; i += 2) {
        const float w0 = ex2_approx(__fmaf_rn(x[i], sl2, -ref)), w1 = ex2_approx(__fmaf_rn(x[i + 1], sl2, -ref));
        s[i & 3] += w0;
        s[(i & 3) + 1] += w1;
        pk[i / 2] = pack_h2(w0, w1);
      }
      sum = (s[0] + s[1]) + (s[2] + s[3]);
    };
    // The weights go by the reference as it is while the other half's largest score is on its
    // way, and once more in the rare tile that raises it.
    float mine = top * sl2, other = 0.0f;
    give(mine);
    if (!first) weights();
    if (!take(other)) break;
    mine = fmaxf(mine, other);
    const bool raise = first ? mine > m : mine > m + kRescaleLog2;
    if (n > 0 && !wait_pv(n - 1)) break;
    if (first || __any_sync(0xffffffffu, raise)) {
      const float a = raise && m != -INFINITY ? exp2f(m - mine) : 1.0f;
      if (raise) m = mine;
      l *= a;
      if (!first && __any_sync(0xffffffffu, a != 1.0f)) {
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
      weights();
    }
    const uint32_t ptile = smem + kPOff + half * (kRows * 128);
#pragma unroll
    for (int i = 0; i < 8; ++i)
      sts_v4(ptile + swz_off(row, i, 128), pk[4 * i], pk[4 * i + 1], pk[4 * i + 2], pk[4 * i + 3]);
    fence_proxy_async_smem();
    tc_fence_before();
    __syncwarp();
    arrive_leader(lane, pfull);
    l += sum;
    ++n;
    if (!sc.last()) continue;

    // ---- segment end: out = O / l in bf16, or the partial (m, l, o)
    whole = whole && sc.t1 >= sc.pu1;
    float lo = 0.0f;
    give(l);
    if (!take(lo)) break;
    const float lt = half == 0 ? l + lo : lo + l;
    const float inv = lt > 0.0f ? 1.0f / lt : 0.0f;
    // (32 bytes at a time, a whole sector of the thread's own row. The pieces of a partial result lie
    // row by row, so that a warp's store is 8 lines: laid out by rows it was 32, and a segment's
    // end 6k cycles.)
    const int h0 = (sc.g * 2 + rank) * static_cast<int>(kRows) + (warp & 1) * 32;  // the warp's first row
    const bool mine_out = h0 + lane < p.heads;
    const size_t out_row = static_cast<size_t>(sc.b) * p.heads + h0 + lane;
    const int unit_row = rank * static_cast<int>(kRows) + (warp & 1) * 32 + lane;
    const size_t piece = static_cast<size_t>(pair) + sc.unit;
    __nv_bfloat16* const dst = reinterpret_cast<__nv_bfloat16*>(p.out) + out_row * kDc + half * 256;
    float* const part = p.part_o + tree_part_at(piece, unit_row, half * 256);
    if (!wait_pv(n - 1)) break;
    auto put = [&](int c, const uint32_t* o) {
      if (!mine_out) return;
      if (whole) {
#pragma unroll
        for (int q = 0; q < 2; ++q) {
          uint32_t w[8];
#pragma unroll
          for (int e = 0; e < 8; ++e)
            w[e] = pack_bf16(__uint_as_float(o[16 * q + 2 * e]) * inv, __uint_as_float(o[16 * q + 2 * e + 1]) * inv);
          stg_v8(dst + c + 16 * q, w);
        }
      } else {
#pragma unroll
        for (int q = 0; q < 4; ++q) stg_v8(part + (c + 8 * q) * 128, o + 8 * q);
      }
    };
    // (the next columns are read while these are stored; a short loop, for its code is cold)
    uint32_t r0[32], r1[32];
    tmem_ld32(t_o, r0);
#pragma unroll 1
    for (int c = 0; c < 256; c += 64) {
      tmem_ld_wait();
      tmem_ld32(t_o + c + 32, r1);
      put(c, r0);
      tmem_ld_wait();
      if (c < 192) tmem_ld32(t_o + c + 64, r0);
      put(c + 32, r1);
    }
    if (half == 0 && mine_out) {
      if (!whole) {
        p.part_ml[(piece * 128 + unit_row) * 2] = m;
        p.part_ml[(piece * 128 + unit_row) * 2 + 1] = lt;
      } else if (p.lse != nullptr) {
        p.lse[out_row] = (m + log2f(lt)) * kLn2;
      }
    }
    __syncwarp();
  }
  if (!ok) {
    if (lane == 0) set_abort(ctl, p.dev_err);
    __syncwarp();
    asm volatile("bar.arrive %0, 64;" ::"r"(1 + (warp & 1)) : "memory");
  }
}

template <int PASSES>
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
    const uint32_t copies = rank == 0 ? 2 : 1;  // (own, and in the leader the other CTA's)
    for (int i = 0; i < kKeyParts; ++i) {
      mbar_init(&ctl.k_bar[i], copies);
      mbar_init(&ctl.k_free[i], 1);
    }
    for (int i = 0; i < kValueParts; ++i) {
      mbar_init(&ctl.v_bar[i], copies);
      mbar_init(&ctl.v_free[i], 1);
    }
    for (int i = 0; i < 2; ++i) mbar_init(&ctl.s_full[i], 1);
    mbar_init(&ctl.p_full, 2 * kSoftWarps);
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
      load_role<PASSES>(p, sc, sm, ctl, rank);
    } else if (rank == 0) {
      issue_role<PASSES>(p, sc, smem, ctl, tmem);
    } else {
      relay_role<PASSES>(p, sc, ctl);
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

// ---------------------------------------------------------------------- merge
// A row's share of a partial result: (m, l) and 16 channels of o; the merge of two (App. C.5).
struct Piece {
  float2 ml;
  float o[16];
  __device__ __forceinline__ void load(const Params& p, size_t piece, int row, int channel) {
    ml = *reinterpret_cast<const float2*>(p.part_ml + (piece * 128 + row) * 2);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float4 v = *reinterpret_cast<const float4*>(p.part_o + tree_part_at(piece, row, channel + 4 * i));
      o[4 * i] = v.x, o[4 * i + 1] = v.y, o[4 * i + 2] = v.z, o[4 * i + 3] = v.w;
    }
  }
  __device__ __forceinline__ void add(const Piece& x) {
    const float m = fmaxf(ml.x, x.ml.x);
    const float s = ml.x == m ? 1.0f : exp2f(ml.x - m), t = x.ml.x == m ? 1.0f : exp2f(x.ml.x - m);
    ml = make_float2(m, ml.y * s + x.ml.y * t);
#pragma unroll
    for (int i = 0; i < 16; ++i) o[i] = o[i] * s + x.o[i] * t;
  }
  __device__ __forceinline__ void store(const Params& p, int b, int head_row, int channel) const {
    const float inv = ml.y > 0.0f ? 1.0f / ml.y : 0.0f;
    uint32_t w[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) w[i] = pack_bf16(o[2 * i] * inv, o[2 * i + 1] * inv);
    const size_t at = static_cast<size_t>(b) * p.heads + head_row;
    stg_v8(reinterpret_cast<__nv_bfloat16*>(p.out) + at * kDc + channel, w);
    if (channel == 0 && p.lse != nullptr) p.lse[at] = (ml.x + log2f(ml.y)) * kLn2;
  }
};
constexpr int kMergeThreads = 256, kMergeWarps = kMergeThreads / 32;

// The unit that begins in range c and goes on behind its end. A lane per row, 16 channels a warp;
// nearly always two pieces, both of which are on their way before the first is used. (A warp a
// row, a piece after the other and the pieces' number by division took 7 to 14 us.)
__global__ void __launch_bounds__(kMergeThreads) tree_merge(const Params p) {
  const int c = blockIdx.x, row = blockIdx.y * 32 + (threadIdx.x & 31);
  const int channel = (blockIdx.z * kMergeWarps + (threadIdx.x >> 5)) * 16;
  griddep_wait();  // the partials of the main kernel
  const int4 next = p.cta_info[c + 1];
  const int begin = p.cta_t0[c], end = p.cta_t0[c + 1];
  const int u = next.x, P0 = next.y, P1 = next.z;
  if (P0 < begin || P0 >= end || end >= P1) return;
  int b, g;
  tree_unit(p, u, b, g);
  if (g * 128 + row >= p.heads) return;
  Piece sum;
  sum.load(p, static_cast<size_t>(c) + u, row, channel);
  for (int d = c + 1, at = end; at < P1; ++d) {
    if (next.w < p.grid) d = cta_of(at, next.w, p.grid);  // (fewer tiles than ranges: past the empty ones)
    at = p.cta_t0[d + 1];
    Piece x;
    x.load(p, static_cast<size_t>(d) + u, row, channel);
    sum.add(x);
  }
  sum.store(p, b, g * 128 + row, channel);
}

// The same for few units of many pieces each: a block per unit, 32 rows and 16 channels, its
// warps taking every eighth piece.
__global__ void __launch_bounds__(kMergeThreads) tree_merge_wide(const Params p) {
  __shared__ Piece part[kMergeWarps][32];
  const int u = blockIdx.x, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int row = blockIdx.y * 32 + lane, channel = blockIdx.z * 16;
  griddep_wait();  // the partials of the main kernel
  const int P0 = p.prefix[u], P1 = p.prefix[u + 1], T = p.prefix[p.batch * p.n_hg];
  if (P0 == P1) return;  // (prep wrote the results)
  const int c0 = cta_of(P0, T, p.grid), c1 = cta_of(P1 - 1, T, p.grid);
  if (c0 == c1) return;
  Piece sum;
  sum.ml = make_float2(-INFINITY, 0.0f);
#pragma unroll
  for (int i = 0; i < 16; ++i) sum.o[i] = 0.0f;
#pragma unroll 2
  for (int d = c0 + warp; d <= c1; d += kMergeWarps) {
    if (p.cta_t0[d] == p.cta_t0[d + 1]) continue;  // an empty range wrote nothing
    Piece x;
    x.load(p, static_cast<size_t>(d) + u, row, channel);
    sum.add(x);
  }
  part[warp][lane] = sum;
  __syncthreads();
  int b, g;
  tree_unit(p, u, b, g);
  if (warp != 0 || g * 128 + row >= p.heads) return;
#pragma unroll
  for (int w = 1; w < kMergeWarps; ++w) sum.add(part[w][lane]);
  sum.store(p, b, g * 128 + row, channel);
}

}  // namespace

cudaError_t launch_tree_merge(const Params& prm, cudaStream_t stream) {
  if (prm.grid < 2) return cudaSuccess;
  // Few units (a unit in more than four ranges), of more than eight tiles.
  const int units = prm.batch * prm.n_hg;
  if (units * 4 < prm.grid && prm.img_width > 16)
    return launch_k(tree_merge_wide, dim3(units, 4, kDc / 16), dim3(kMergeThreads), 0, stream, true, prm);
  return launch_k(tree_merge, dim3(prm.grid - 1, 4, kDc / 16 / kMergeWarps), dim3(kMergeThreads), 0, stream, true, prm);
}

cudaError_t launch_tree_pair(const Params& prm, cudaStream_t stream) {
  static int configured_device = -1;
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  if (configured_device != dev) {
    for (auto* kern : {tree_pair<1>, tree_pair<2>}) {
      e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmem);
      if (e != cudaSuccess) return e;
    }
    configured_device = dev;
  }
  return launch_k(prm.rest_images != nullptr ? tree_pair<2> : tree_pair<1>, dim3(2 * prm.grid), dim3(kThreads), kSmem, stream, true, prm);
}

}  // namespace qmla
