// Quantise-and-pack cache writer (App. C.4 quantiser; App. C.5 cache update:
// content- and RoPE-cache quantisation, integer packing and slot-mapped page
// insertion) for this library's block and for the paper's own page, and the
// plain BF16 writer for the comparison cache. The fused form takes the rows as the
// projections leave them: it normalises the latent and rotates the RoPE key on
// the way into any of the four caches.
//
// A block of nine warps writes a few tokens: warp g quantises group g (64
// coordinates) of four or sixteen tokens, eight lanes per token with eight
// coordinates (16 bytes) each. (The fused form for many tokens has another layout, a
// whole token in eight lanes: wide_append_kernel.) A warp then reads four whole 128-byte lines and,
// where the tokens take consecutive slots (a prefill), writes their code rows
// and scales as contiguous runs; the bit width and the scale format are uniform
// in a warp. See quant_append_kernel for what bounds it.
#include <cuda_runtime.h>

#include "common.cuh"
#include "kernels.h"
#include "ptx.cuh"
#include "rope.cuh"

namespace qmla {
namespace {

// Stored fp16 scale and integer zero point of one group (App. C.4 with the
// fp16 staging of include/qmla.h): s = RN_f16(RN_f32(max(d, 1e-8) / m)),
// clamped to [2^-24, 65504]; z = clip(rne(-x_min / s), 0, m).
__device__ __forceinline__ void group_scale(float xmin, float xmax, int m, float& s, float& z) {
  const float d = xmax - xmin;
  const float s32 = __fdiv_rn(fmaxf(d, 1e-8f), static_cast<float>(m));
  s = __half2float(__float2half_rn(s32));
  if (s == 0.0f) s = 5.9604644775390625e-08f;  // 2^-24, the smallest fp16 subnormal
  if (isinf(s)) s = 65504.0f;
  z = fminf(fmaxf(rintf(__fdiv_rn(-xmin, s)), 0.0f), static_cast<float>(m));
}

// Scales of the paper's page (App. C.4 with that format's staging): content
// s = RN_bf16(RN_f32(max(d, 1e-8) / 15)), RoPE s = RN_f32(max(d, 1e-8) / 15);
// z = clip(rne(-x_min / s), 0, 15) from an fp32 quotient. A bf16 scale and a
// bf16 input carry 8 significant bits each, so the fp32 quotients of the
// content path round to the same codes as exact arithmetic would.
__device__ __forceinline__ void paper_scale(float xmin, float xmax, bool content, float& s, float& z) {
  const float s32 = __fdiv_rn(fmaxf(xmax - xmin, 1e-8f), 15.0f);
  s = content ? __bfloat162float(__float2bfloat16_rn(s32)) : s32;
  z = fminf(fmaxf(rintf(__fdiv_rn(-xmin, s)), 0.0f), 15.0f);
}

__device__ __forceinline__ uint32_t quant_code(float x, float s, float z, float m) {
  // q = clip(rne(x / s + z), 0, m): z is added before rounding.
  return static_cast<uint32_t>(fminf(fmaxf(rintf(__fdiv_rn(x, s) + z), 0.0f), m));
}

// The codes clip(rne(x / s + z), 0, m) of eight bf16 values (four words of two),
// as four words with one code in each half, without a division per value: y =
// RN(1 / s), q = RN(x y) corrected once by its exact residual x - q s (P.
// Markstein, IBM J. Res. Dev. 34(1), 1990) is within 2^-22 relative of x / s and
// exact where x / s is representable. The codes need no more: s has at most 11
// and x 8 significant bits, so an x / s of magnitude 16 or less is a half-integer
// (representable) or at least 2^-12 away from one, and what lies outside is
// clipped. Adding 1.5 * 2^23 leaves the integer nearest to q + z (ties to even)
// in the low bits, for |q| <= 2^14 in the low 16 as a signed number, and a NaN as
// -1, which is clipped to 0.
__device__ __forceinline__ void codes8(const uint32_t (&w)[4], float s, float y, float z, uint32_t m, uint32_t (&c)[4]) {
  const uint64_t yy = f32x2(y, y), ns = f32x2(-s, -s), zz = f32x2(z, z), magic = f32x2(12582912.0f, 12582912.0f);
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const uint64_t x = f32x2(__uint_as_float(w[e] << 16), __uint_as_float(w[e] & 0xFFFF0000u));
    uint64_t q = mul2(x, yy);
    q = fma2(fma2(q, ns, x), yy, q);
    q = add2(add2(q, zz), magic);
    c[e] = __vimin_s16x2_relu(__byte_perm(static_cast<uint32_t>(q), static_cast<uint32_t>(q >> 32), 0x5410),
                              m | (m << 16));
  }
}

// Extrema of a group's 64 values, eight in each of eight lanes: (min, -max) as a bf16
// pair, so that one packed minimum per shuffle serves both. bf16 minima are exact, and
// NaNs lose against numbers as in fminf / fmaxf. All lanes of the warp take part.
__device__ __forceinline__ uint32_t extrema64(const uint32_t (&w)[4]) {
  __nv_bfloat162 lo = *reinterpret_cast<const __nv_bfloat162*>(&w[0]), hi = lo;
#pragma unroll
  for (int e = 1; e < 4; ++e) {
    const __nv_bfloat162 v = *reinterpret_cast<const __nv_bfloat162*>(&w[e]);
    lo = __hmin2(lo, v);
    hi = __hmax2(hi, v);
  }
  lo = __hmin2(lo, __lowhigh2highlow(lo));
  hi = __hmax2(hi, __lowhigh2highlow(hi));
  uint32_t pk =
      __byte_perm(*reinterpret_cast<uint32_t*>(&lo), *reinterpret_cast<uint32_t*>(&hi) ^ 0x80008000u, 0x7610);
#pragma unroll
  for (int off = 1; off < 8; off <<= 1) {
    const uint32_t o = __shfl_xor_sync(0xffffffffu, pk, off);
    const __nv_bfloat162 r = __hmin2(*reinterpret_cast<const __nv_bfloat162*>(&pk),
                                     *reinterpret_cast<const __nv_bfloat162*>(&o));
    pk = *reinterpret_cast<const uint32_t*>(&r);
  }
  return pk;
}

// Scale, zero point and 1 / s of a group from its extrema; 1 / s is 0 for a group whose
// values divide one by one (an infinite or NaN quotient among them; 1 / s is 0 when s is
// infinite, and for the paper's fp32 RoPE scale).
template <int CB>
__device__ __forceinline__ void scale_of(uint32_t ext, bool content, int m, float& s, float& z, float& y) {
  const float xmin = __uint_as_float(ext << 16), xmax = -__uint_as_float(ext & 0xFFFF0000u);
  if constexpr (CB == kC4R4) {
    paper_scale(xmin, xmax, content, s, z);
  } else {
    group_scale(xmin, xmax, m, s, z);
  }
  y = __frcp_rn(s);
  if (!(fmaxf(fabsf(xmin), fabsf(xmax)) * y <= 16384.0f) || (CB == kC4R4 && !content)) y = 0.0f;
}

template <int CB>
__device__ __forceinline__ void store_scale(uint8_t* blk, int g, int slot, float s, float z) {
  using L = BlockLayout<CB>;
  if constexpr (CB == kC4R4) {
    if (g < 8) {
      *reinterpret_cast<__nv_bfloat16*>(blk + L::c_scale_off(g, slot)) = __float2bfloat16_rn(s);  // exact
    } else {
      *reinterpret_cast<float*>(blk + L::pe_scale_off(slot)) = s;
    }
    blk[L::zero_off(g, slot)] = static_cast<uint8_t>(z);
  } else {
    *reinterpret_cast<__half2*>(blk + L::sz_off(g, slot)) =
        __halves2half2(__float2half_rn(s), __float2half_rn(z));
  }
}

// The codes of eight values, packed low bits first: INT4 byte j = code 2 j | code 2 j + 1
// << 4 (four bytes), INT2 byte j = codes 4 j .. 4 j + 3 (two).
__device__ __forceinline__ uint32_t pack_codes(const uint32_t (&w)[4], float s, float y, float z, int bits) {
  const uint32_t m = (1u << bits) - 1u;
  uint32_t c[4];  // codes 2 e and 2 e + 1 in the halves of c[e]
  if (y > 0.0f) {
    codes8(w, s, y, z, m, c);
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      c[e] = quant_code(__uint_as_float(w[e] << 16), s, z, static_cast<float>(m)) |
             quant_code(__uint_as_float(w[e] & 0xFFFF0000u), s, z, static_cast<float>(m)) << 16;
  }
  if (bits == 4) {
    const uint32_t a = c[0] | c[1] << 8, b = c[2] | c[3] << 8;
    return __byte_perm(a | a >> 12, b | b >> 12, 0x5410);
  }
  const uint32_t a = c[0] | c[1] << 4 | c[2] << 8 | c[3] << 12;
  return a | a >> 14;
}

// Looks up and validates the destination of token i: its block id, or -1 (after
// recording the error) when the token cannot be written. turns: the positions that the
// fused writer takes the angles of, all below rope_len.
__device__ __forceinline__ int token_block(int num_blocks, const int32_t* seq_ids, const int32_t* positions, int i,
                                           const int32_t* table, int num_seqs, int max_blocks, uint32_t* dev_err,
                                           int& seq, int& pos, const int32_t* turns = nullptr, int rope_len = 0) {
  seq = seq_ids != nullptr ? seq_ids[i] : i;
  pos = positions[i];
  const bool turned = turns == nullptr || static_cast<unsigned>(turns[i]) < static_cast<unsigned>(rope_len);
  if (seq < 0 || seq >= num_seqs) {
    report(dev_err, QMLA_DEVERR_BAD_SEQ);
    return -1;
  }
  if (pos < 0 || pos >= max_blocks * kBlockTokens || !turned) {
    report(dev_err, QMLA_DEVERR_BAD_POSITION);
    return -1;
  }
  const int blk = table[static_cast<size_t>(seq) * max_blocks + pos / kBlockTokens];
  if (blk < 0 || blk >= num_blocks) {
    report(dev_err, QMLA_DEVERR_BAD_BLOCK);
    return -1;
  }
  return blk;
}

// Sink/recent BF16 protection rows (App. C.5, "BF16 protection and cache
// lifecycle"): position p of a request whose length after this write is L goes
// to row p when p < 4 and to row 4 + p mod 128 when p >= L - 128; each lane stores
// its own 16 bytes of the token's 1152.

constexpr int kAppendThreads = kGroups * 32;

// What the fused writer does to a row on its way into the cache.
struct RowTransform {
  size_t latent_words, k_pe_words;  // row strides in 4-byte words
  const uint4* weight;              // [512] bf16, or null: all ones
  bool norm;
  float eps;
  const float* cos_sin;  // [rope_len][64]: cos[32] | sin[32]
  int rope_len;
  const int32_t* turns;  // [n] position of each token's angles
  bool interleaved;
};

// Warp g's piece of four tokens (eight lanes each) normalised (g < 8) or rotated
// (g = 8) in registers. The row's sum of squares needs all eight content warps: each
// leaves its 64 channels' share in shared memory and every warp adds the eight shares in
// the same order, so the result does not depend on the launch, and all eight come to the
// same answer about far rows. Every thread of the block takes part; the eight content
// warps meet at a barrier of their own.
__device__ __forceinline__ void content_barrier() { asm volatile("bar.sync 1, 256;" ::: "memory"); }
__device__ __forceinline__ void transform_rows(uint4& raw, const RowTransform& tr, int n, int tok, int g, int lane) {
  __shared__ float2 share[8][4];
  __shared__ uint32_t tops[8][4];
  const int piece = lane & 7, sub = lane >> 3;
  uint32_t w[4] = {raw.x, raw.y, raw.z, raw.w};
  if (g == 8) {
    const int pos = tok < n ? tr.turns[tok] : -1;
    Angles a;
    load_angles(a, pos >= 0 && pos < tr.rope_len ? tr.cos_sin + static_cast<size_t>(pos) * kDr : nullptr, piece,
                tr.interleaved);
    rotate_row<true>(w, a, piece, tr.interleaved);
    raw = make_uint4(w[0], w[1], w[2], w[3]);
    return;
  }
  if (!tr.norm) return;
  auto row_sum = [&]() {
    F2 s = square_sum8(w);
#pragma unroll
    for (int off = 1; off < 8; off <<= 1)
      s = add_f2(s, {__shfl_xor_sync(0xffffffffu, s.hi, off), __shfl_xor_sync(0xffffffffu, s.lo, off)});
    if (piece == 0) share[g][sub] = make_float2(s.hi, s.lo);
    content_barrier();
    // The row's sum: four shares here, the other four in the lane four away.
    F2 sum = {0.0f, 0.0f};
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const float2 v = share[(piece & 4) + k][sub];
      sum = k == 0 ? F2{v.x, v.y} : add_f2(sum, {v.x, v.y});
    }
    const F2 o = {__shfl_xor_sync(0xffffffffu, sum.hi, 4), __shfl_xor_sync(0xffffffffu, sum.lo, 4)};
    return (piece & 4) == 0 ? add_f2(sum, o) : add_f2(o, sum);
  };
  F2 sum = row_sum(), rs;
  const bool far = tok < n && far_row(sum, tr.eps);
  if (!__any_sync(0xffffffffu, far)) {
    rs = row_rstd(sum, tr.eps);
  } else {
    uint32_t top = largest8(w);
#pragma unroll
    for (int off = 1; off < 8; off <<= 1) top = max(top, __shfl_xor_sync(0xffffffffu, top, off));
    if (piece == 0) tops[g][sub] = top;
    content_barrier();  // (the shares have been read as well)
#pragma unroll
    for (int k = 0; k < 8; ++k) top = max(top, tops[k][sub]);
    const float f = far ? far_factor(top, tr.eps) : 1.0f;
    scale_words(w, f);
    sum = row_sum();
    rs = far_rstd(sum, tr.eps, f, top);
  }
  const uint4 ones = make_uint4(0x3F803F80u, 0x3F803F80u, 0x3F803F80u, 0x3F803F80u);
  const uint4 gv = tr.weight != nullptr ? tr.weight[g * 8 + piece] : ones;
  const uint64_t gw[4] = {f32x2(bf16_low(gv.x), bf16_high(gv.x)), f32x2(bf16_low(gv.y), bf16_high(gv.y)),
                          f32x2(bf16_low(gv.z), bf16_high(gv.z)), f32x2(bf16_low(gv.w), bf16_high(gv.w))};
  scale_row(w, gw, rs);
  raw = make_uint4(w[0], w[1], w[2], w[3]);
}
constexpr int kBf16Rows = 16;  // cache kind of the BF16 cache

// Quantises and packs n tokens. CB: content bits (4, 2) or kC4R4 for the paper's
// page (INT4 codes). NT: tokens per lane, 1 or 4 (a block writes 4 NT). VEC: latent
// and k_pe are 16-byte aligned (one 16-byte load per lane, else four 4-byte ones).
// prot / lens: the protection buffer [num_seqs][132][576] bf16 and the requests'
// lengths after this write, or null for an unprotected cache.
// FUSED: the rows are normalised and rotated first (RowTransform), which also gives
// their strides; then CB may be kBf16Rows, which stores them as they are.
//
// What bounds it: for a prefill the issue slots, then the HBM traffic (1152 bytes
// read and 324 written per token, INT4); for a decode step's few tokens the latency
// of load -> extrema -> scale -> codes -> store. So one pass holds eight coordinates
// per lane, the extrema take three packed shuffles for minimum and maximum together,
// and the codes take two values per instruction (codes8). With four tokens per lane
// the eight lanes of a token share what is per token: lane i of four looks token i's
// destination up and works out its scale, and shuffles hand them round. Groups
// outside codes8's argument (quotients above 2^14, infinite values or scales) and
// the fp32 RoPE scale of the paper's page, whose codes are defined by the rounded
// fp32 quotient, divide value by value. 32,797 tokens of eight ragged prompts (INT4, calls
// on buffers larger together than L2) take 16.5 us, 2.9 TB/s of 6.8; a warp per (token,
// group) with two coordinates per lane and a division per code took 61.5.
template <int CB, int NT, bool VEC, bool FUSED>
__global__ void __launch_bounds__(kAppendThreads) quant_append_kernel(
    uint8_t* __restrict__ pool, int num_blocks, const uint32_t* __restrict__ latent,
    const uint32_t* __restrict__ k_pe, const int32_t* __restrict__ seq_ids,
    const int32_t* __restrict__ positions, int n, const int32_t* __restrict__ table, int num_seqs,
    int max_blocks, uint32_t* dev_err, uint4* __restrict__ prot, const int32_t* __restrict__ lens,
    const RowTransform tr) {
  static_assert(NT == 1 || NT == 4, "tokens per lane");
  static_assert(FUSED || CB != kBf16Rows, "bf16 rows have a writer of their own");
  static_assert(!FUSED || NT == 1, "many tokens have a fused writer of their own");
  using L = BlockLayout<CB == kBf16Rows ? 4 : CB>;
  // The decode's prep kernel may start meanwhile: it does not read the cache, and it
  // neither writes anything nor ends before this kernel has ended. (A decode step with
  // prep after the writer / beside it, us: 8 sequences x 128 heads, 300..2,500 tokens,
  // protected 36.9 / 35.2; 64 x 4,097 INT4 116.8 / 115.5; 128 x 16 heads 186.9 / 185.4.)
  griddep_launch_dependents();
  const int g = threadIdx.x >> 5;  // this warp's group
  const int lane = threadIdx.x & 31;
  const int piece = lane & 7;
  const int tok0 = blockIdx.x * (4 * NT) + (lane >> 3);  // token i of the lane: tok0 + 4 i
  const int bits = g < 8 ? (CB == kC4R4 ? 4 : CB) : kPeBits;
  const int m = (1 << bits) - 1;
  // The groups' loads do not wait for the seq_ids -> block-table lookups, which
  // only the stores need.
  uint4 raw[NT];
#pragma unroll
  for (int i = 0; i < NT; ++i) {
    const int tok = tok0 + 4 * i;
    raw[i] = make_uint4(0, 0, 0, 0);
    if (tok < n) {
      const size_t row = static_cast<size_t>(tok);
      const uint32_t* src = g < 8 ? latent + row * (FUSED ? tr.latent_words : kDc / 2) + g * 32 + piece * 4
                                  : k_pe + row * (FUSED ? tr.k_pe_words : kDr / 2) + piece * 4;
      if constexpr (VEC) {
        raw[i] = *reinterpret_cast<const uint4*>(src);
      } else {
        raw[i] = make_uint4(src[0], src[1], src[2], src[3]);
      }
    }
  }
  // This lane's share: token `own` of the lane's NT. dst is the block's slot, the
  // block id times 64 plus the slot, or -1; rows the protection rows (sink, ring), or
  // -1. Errors are reported once per token, by its group-0 warp.
  const int own = piece & (NT - 1);
  int dst = -1, sink = -1, ring = -1;
  if (tok0 + 4 * own < n) {
    const int tok = tok0 + 4 * own;
    int seq = 0, pos = 0;
    const int blk = token_block(num_blocks, seq_ids, positions, tok, table, num_seqs, max_blocks,
                                piece == own && g == 0 ? dev_err : nullptr, seq, pos, FUSED ? tr.turns : nullptr, tr.rope_len);
    if (blk >= 0) {
      dst = blk * kBlockTokens + pos % kBlockTokens;
      if (prot != nullptr) {
        if (pos < kSinkTokens) sink = seq * kProtRows + pos;
        if (pos >= lens[seq] - kRecentTokens) ring = seq * kProtRows + kSinkTokens + pos % kRecentTokens;
      }
    }
  }
  if constexpr (FUSED) {
    transform_rows(raw[0], tr, n, tok0, g, lane);
    if constexpr (CB == kBf16Rows) {
      if (dst >= 0)
        reinterpret_cast<uint4*>(pool + static_cast<size_t>(dst / kBlockTokens) * kBf16BlockBytes +
                                 dst % kBlockTokens * (kDqk * 2))[g * 8 + piece] = raw[0];
      return;
    }
  }
  uint32_t ext = 0;  // of token `own`
#pragma unroll
  for (int i = 0; i < NT; ++i) {
    const uint32_t w[4] = {raw[i].x, raw[i].y, raw[i].z, raw[i].w};
    const uint32_t pk = extrema64(w);
    if (i == own) ext = pk;
  }
  float s_own, z_own, y_own;
  scale_of<CB>(ext, g < 8, m, s_own, z_own, y_own);
  if (piece == own && dst >= 0)
    store_scale<CB == kBf16Rows ? 4 : CB>(pool + static_cast<size_t>(dst / kBlockTokens) * L::kBytes, g,
                                          dst % kBlockTokens, s_own, z_own);
#pragma unroll
  for (int i = 0; i < NT; ++i) {
    const uint32_t w[4] = {raw[i].x, raw[i].y, raw[i].z, raw[i].w};
    // (the token's values from its lane i)
    const int from = (lane & 24) | i;
    const float s = NT == 1 ? s_own : __shfl_sync(0xffffffffu, s_own, from);
    const float y = NT == 1 ? y_own : __shfl_sync(0xffffffffu, y_own, from);
    const float z = NT == 1 ? z_own : __shfl_sync(0xffffffffu, z_own, from);
    const int d = NT == 1 ? dst : __shfl_sync(0xffffffffu, dst, from);
    const uint32_t word = pack_codes(w, s, y, z, bits);
    if (prot != nullptr) {
      const int rows[2] = {NT == 1 ? sink : __shfl_sync(0xffffffffu, sink, from),
                           NT == 1 ? ring : __shfl_sync(0xffffffffu, ring, from)};
#pragma unroll
      for (int r = 0; r < 2; ++r)
        if (rows[r] >= 0) prot[static_cast<size_t>(rows[r]) * (kDqk * 2 / 16) + g * 8 + piece] = raw[i];
    }
    if (d < 0) continue;
    uint8_t* code = pool + static_cast<size_t>(d / kBlockTokens) * L::kBytes + L::code_off(g, d % kBlockTokens);
    if (bits == 4) {
      reinterpret_cast<uint32_t*>(code)[piece] = word;
    } else {
      reinterpret_cast<uint16_t*>(code)[piece] = static_cast<uint16_t>(word);
    }
  }
}

// A row's sum of squares from its eight lanes' pairs.
__device__ __forceinline__ F2 wide_sum(F2x2 sum) {
  F2 s = add_f2({lo2(sum.hi), lo2(sum.lo)}, {hi2(sum.hi), hi2(sum.lo)});
#pragma unroll
  for (int off = 1; off < 8; off <<= 1)
    s = add_f2(s, {__shfl_xor_sync(0xffffffffu, s.hi, off), __shfl_xor_sync(0xffffffffu, s.lo, off)});
  return s;
}
// Group g's eight values of a lane normalised; weight: the 512 in shared memory, fp32.
__device__ __forceinline__ void scale_wide(uint32_t (&w)[4], const float4* weight, int g, int piece, F2 rs) {
  const ulonglong2 wa = reinterpret_cast<const ulonglong2*>(weight)[g * 16 + piece * 2];
  const ulonglong2 wb = reinterpret_cast<const ulonglong2*>(weight)[g * 16 + piece * 2 + 1];
  const uint64_t gw[4] = {wa.x, wa.y, wb.x, wb.y};
  scale_row(w, gw, rs);
}
// The four tokens of a warp of wide_append_kernel where a row is far: everything from the
// norm on, from memory once more and a group at a time. (Led back into the kernel, scaled
// rows cost all others 3%.)
// row: the latent, or null; pe: the rotated RoPE key; dst, sink and ring as there.
template <int CB>
__device__ __noinline__ void far_tokens(const uint32_t* row, uint4 pe, const float4* weight, bool far, float eps, int piece,
                                        uint8_t* pool, int dst, uint4* prot, int sink, int ring) {
  using L = BlockLayout<CB == kBf16Rows ? 4 : CB>;
  uint32_t w[4], top = 0;
  auto load = [&](int g) {
    const uint4 v = g == 8 ? pe : (row != nullptr ? *reinterpret_cast<const uint4*>(row + g * 32 + piece * 4) : make_uint4(0, 0, 0, 0));
    w[0] = v.x, w[1] = v.y, w[2] = v.z, w[3] = v.w;
  };
#pragma unroll 1
  for (int g = 0; g < 8; ++g) {
    load(g);
    top = max(top, largest8(w));
  }
#pragma unroll
  for (int off = 1; off < 8; off <<= 1) top = max(top, __shfl_xor_sync(0xffffffffu, top, off));
  const float f = far ? far_factor(top, eps) : 1.0f;
  F2x2 sum = {0, 0};
#pragma unroll 1
  for (int g = 0; g < 8; ++g) {
    load(g);
    scale_words(w, f);
    add_squares8(sum, w);
  }
  const F2 rs = far_rstd(wide_sum(sum), eps, f, top);
#pragma unroll 1
  for (int g = 0; g < kGroups; ++g) {
    load(g);
    if (g < 8) {
      scale_words(w, f);
      scale_wide(w, weight, g, piece, rs);
    }
    const uint4 v = make_uint4(w[0], w[1], w[2], w[3]);
    if (sink >= 0) prot[static_cast<size_t>(sink) * (kDqk * 2 / 16) + g * 8 + piece] = v;
    if (ring >= 0) prot[static_cast<size_t>(ring) * (kDqk * 2 / 16) + g * 8 + piece] = v;
    const int slot = max(dst, 0) % kBlockTokens;
    const size_t id = static_cast<size_t>(max(dst, 0) / kBlockTokens);
    if constexpr (CB == kBf16Rows) {
      if (dst >= 0) reinterpret_cast<uint4*>(pool + id * kBf16BlockBytes + slot * (kDqk * 2))[g * 8 + piece] = v;
    } else {
      const int bits = g < 8 && CB != kC4R4 ? CB : kPeBits;
      float s, z, y;
      scale_of<CB>(extrema64(w), g < 8, (1 << bits) - 1, s, z, y);
      const uint32_t word = pack_codes(w, s, y, z, bits);
      if (dst < 0) continue;
      uint8_t* blk = pool + id * L::kBytes;
      if (piece == 0) store_scale<CB>(blk, g, slot, s, z);
      if (bits == 4) {
        reinterpret_cast<uint32_t*>(blk + L::code_off(g, slot))[piece] = word;
      } else {
        reinterpret_cast<uint16_t*>(blk + L::code_off(g, slot))[piece] = static_cast<uint16_t>(word);
      }
    }
  }
}

// The fused writer for many tokens: eight lanes hold a whole token, lane l the eight
// channels l of each of its nine groups, so that a warp writes four tokens without a
// word to the others. The row's sum takes three shuffles instead of a way through shared
// memory, and lane l works out the scale of group l, which shuffles hand round.
//
// What bounds it: neither the issue slots (57% busy) nor the HBM traffic (1,152 bytes of the
// row and 256 of its angles read, 324 written) by itself. A warp loads its tokens, works and
// stores, once; at 93 registers an SM has 20 warps, too few to cover each other's loads
// (long scoreboard 1.8 and math pipe 1.1 of 7.8 cycles per instruction). Most of the work is
// the norm: INT4 rows as they are take 16.7 us. 32,797 tokens take 22.7 us, 2.5 TB/s of 6.8,
// of which about 4.5 are the launch and the first loads; 116,736 take 67.6, 3.0 TB/s. Five
// blocks per SM: with six the registers spill (23.7 and 69.7).
constexpr int kWideThreads = 128;
template <int CB>
__global__ void __launch_bounds__(kWideThreads, 5) wide_append_kernel(
    uint8_t* __restrict__ pool, int num_blocks, const uint32_t* __restrict__ latent,
    const uint32_t* __restrict__ k_pe, const int32_t* __restrict__ seq_ids,
    const int32_t* __restrict__ positions, int n, const int32_t* __restrict__ table, int num_seqs,
    int max_blocks, uint32_t* dev_err, uint4* __restrict__ prot, const int32_t* __restrict__ lens,
    const RowTransform tr) {
  using L = BlockLayout<CB == kBf16Rows ? 4 : CB>;
  constexpr int kBits = CB == kC4R4 || CB == kBf16Rows ? 4 : CB;
  griddep_launch_dependents();  // as in quant_append_kernel
  __shared__ float4 weight[kDc / 4];
  static_assert(kWideThreads == kDc / 4, "a thread fetches four weights");
  if (tr.norm) {
    uint2 v = make_uint2(0x3F803F80u, 0x3F803F80u);
    if (tr.weight != nullptr) v = reinterpret_cast<const uint2*>(tr.weight)[threadIdx.x];
    weight[threadIdx.x] = make_float4(bf16_low(v.x), bf16_high(v.x), bf16_low(v.y), bf16_high(v.y));
    __syncthreads();
  }
  const int lane = threadIdx.x & 31, piece = lane & 7;
  const int tok = (blockIdx.x * (kWideThreads / 32) + (threadIdx.x >> 5)) * 4 + (lane >> 3);
  uint32_t raw[kGroups][4];
#pragma unroll
  for (int g = 0; g < kGroups; ++g) {
    uint4 v = make_uint4(0, 0, 0, 0);
    if (tok < n) {
      const size_t row = static_cast<size_t>(tok);
      v = *reinterpret_cast<const uint4*>(g < 8 ? latent + row * tr.latent_words + g * 32 + piece * 4
                                                : k_pe + row * tr.k_pe_words + piece * 4);
    }
    raw[g][0] = v.x, raw[g][1] = v.y, raw[g][2] = v.z, raw[g][3] = v.w;
  }
  int dst = -1, sink = -1, ring = -1;
  const float* angles = nullptr;
  if (tok < n) {
    int seq = 0, pos = 0;
    const int blk = token_block(num_blocks, seq_ids, positions, tok, table, num_seqs, max_blocks,
                                piece == 0 ? dev_err : nullptr, seq, pos, tr.turns, tr.rope_len);
    if (blk >= 0) {
      dst = blk * kBlockTokens + pos % kBlockTokens;
      if (prot != nullptr) {
        if (pos < kSinkTokens) sink = seq * kProtRows + pos;
        if (pos >= lens[seq] - kRecentTokens) ring = seq * kProtRows + kSinkTokens + pos % kRecentTokens;
      }
    }
    const int turn = tr.turns[tok];
    if (turn >= 0 && turn < tr.rope_len) angles = tr.cos_sin + static_cast<size_t>(turn) * kDr;
  }
  {
    Angles a;
    load_angles(a, angles, piece, tr.interleaved);
    rotate_row<true>(raw[8], a, piece, tr.interleaved);
  }
  if (tr.norm) {
    F2x2 sum = {0, 0};
#pragma unroll
    for (int g = 0; g < 8; ++g) add_squares8(sum, raw[g]);
    const F2 s = wide_sum(sum);
    const bool far = tok < n && far_row(s, tr.eps);
    if (__any_sync(0xffffffffu, far)) {
      far_tokens<CB>(tok < n ? latent + static_cast<size_t>(tok) * tr.latent_words : nullptr,
                     make_uint4(raw[8][0], raw[8][1], raw[8][2], raw[8][3]), weight, far, tr.eps, piece, pool, dst, prot,
                     sink, ring);
      return;
    }
    const F2 rs = row_rstd(s, tr.eps);
#pragma unroll
    for (int g = 0; g < 8; ++g) scale_wide(raw[g], weight, g, piece, rs);
  }
  if (prot != nullptr) {
#pragma unroll
    for (int g = 0; g < kGroups; ++g) {
      const uint4 v = make_uint4(raw[g][0], raw[g][1], raw[g][2], raw[g][3]);
      if (sink >= 0) prot[static_cast<size_t>(sink) * (kDqk * 2 / 16) + g * 8 + piece] = v;
      if (ring >= 0) prot[static_cast<size_t>(ring) * (kDqk * 2 / 16) + g * 8 + piece] = v;
    }
  }
  if constexpr (CB == kBf16Rows) {
    if (dst < 0) return;
    uint4* row = reinterpret_cast<uint4*>(pool + static_cast<size_t>(dst / kBlockTokens) * kBf16BlockBytes +
                                          dst % kBlockTokens * (kDqk * 2)) + piece;
#pragma unroll
    for (int g = 0; g < kGroups; ++g) row[g * 8] = make_uint4(raw[g][0], raw[g][1], raw[g][2], raw[g][3]);
  } else {
    uint8_t* blk = pool + static_cast<size_t>(max(dst, 0) / kBlockTokens) * L::kBytes;
    const int slot = max(dst, 0) % kBlockTokens;
    // Extrema; lane l keeps group l's (and every lane the RoPE key's).
    uint32_t ext = 0, ext_pe = 0;
#pragma unroll
    for (int g = 0; g < kGroups; ++g) {
      const uint32_t pk = extrema64(raw[g]);
      if (g == piece) ext = pk;
      if (g == 8) ext_pe = pk;
    }
    float s, z, y;
    scale_of<CB>(ext, true, (1 << kBits) - 1, s, z, y);
    float s_pe, z_pe, y_pe;
    scale_of<CB>(ext_pe, false, 15, s_pe, z_pe, y_pe);
    if (dst >= 0) {
      store_scale<CB>(blk, piece, slot, s, z);
      if (piece == 0) store_scale<CB>(blk, 8, slot, s_pe, z_pe);
    }
#pragma unroll
    for (int g = 0; g < kGroups; ++g) {
      const int from = (lane & 24) | g;
      const float sg = g < 8 ? __shfl_sync(0xffffffffu, s, from) : s_pe;
      const float yg = g < 8 ? __shfl_sync(0xffffffffu, y, from) : y_pe;
      const float zg = g < 8 ? __shfl_sync(0xffffffffu, z, from) : z_pe;
      const int bits = g < 8 ? kBits : kPeBits;
      const uint32_t word = pack_codes(raw[g], sg, yg, zg, bits);
      if (dst < 0) continue;
      uint8_t* code = blk + L::code_off(g, slot);
      if (bits == 4) {
        reinterpret_cast<uint32_t*>(code)[piece] = word;
      } else {
        reinterpret_cast<uint16_t*>(code)[piece] = static_cast<uint16_t>(word);
      }
    }
  }
}

// Copies each token's 72 16-byte pieces (64 of the latent, 8 of the RoPE key)
// unchanged, one piece per thread. Bound by HBM for a prefill: whole 16-byte
// accesses on both sides, neighbouring threads on neighbouring pieces.
template <bool VEC>
__global__ void __launch_bounds__(256) bf16_append_kernel(
    uint8_t* __restrict__ pool, int num_blocks, const uint32_t* __restrict__ latent,
    const uint32_t* __restrict__ k_pe, const int32_t* __restrict__ seq_ids,
    const int32_t* __restrict__ positions, int n, const int32_t* __restrict__ table, int num_seqs,
    int max_blocks, uint32_t* dev_err) {
  constexpr int kPieces = kDqk * 2 / 16;
  griddep_launch_dependents();  // as in quant_append_kernel
  const long long idx = static_cast<long long>(blockIdx.x) * blockDim.x + threadIdx.x;
  const int tok = static_cast<int>(idx / kPieces);
  const int piece = static_cast<int>(idx - static_cast<long long>(tok) * kPieces);
  if (tok >= n) return;
  const uint32_t* src = piece < kDc / 8 ? latent + static_cast<size_t>(tok) * (kDc / 2) + piece * 4
                                        : k_pe + static_cast<size_t>(tok) * (kDr / 2) + (piece - kDc / 8) * 4;
  uint4 v;
  if constexpr (VEC) {
    v = *reinterpret_cast<const uint4*>(src);
  } else {
    v = make_uint4(src[0], src[1], src[2], src[3]);
  }
  int seq = 0, pos = 0;
  const int blk = token_block(num_blocks, seq_ids, positions, tok, table, num_seqs, max_blocks,
                              piece == 0 ? dev_err : nullptr, seq, pos);
  if (blk < 0) return;
  reinterpret_cast<uint4*>(pool + static_cast<size_t>(blk) * kBf16BlockBytes + pos % kBlockTokens * (kDqk * 2))[piece] =
      v;
}

bool aligned16(const void* a, const void* b) {
  return ((reinterpret_cast<uintptr_t>(a) | reinterpret_cast<uintptr_t>(b)) & 15) == 0;
}

struct AppendArgs {
  void* pool;
  int num_blocks;
  const uint16_t *latent, *k_pe;
  const int32_t *seq_ids, *positions;
  int n;
  const int32_t* table;
  int num_seqs, max_blocks;
  uint32_t* dev_err;
  void* prot;
  const int32_t* lens;
};

template <int CB, int NT, bool VEC, bool FUSED>
void launch_quant(const AppendArgs& a, const RowTransform& tr, cudaStream_t stream) {
  const unsigned grid = static_cast<unsigned>((static_cast<long long>(a.n) + 4 * NT - 1) / (4 * NT));
  quant_append_kernel<CB, NT, VEC, FUSED><<<grid, kAppendThreads, 0, stream>>>(
      static_cast<uint8_t*>(a.pool), a.num_blocks, reinterpret_cast<const uint32_t*>(a.latent),
      reinterpret_cast<const uint32_t*>(a.k_pe), a.seq_ids, a.positions, a.n, a.table, a.num_seqs, a.max_blocks,
      a.dev_err, static_cast<uint4*>(a.prot), a.lens, tr);
}

// Tokens from which a lane takes four: below, one token per lane spreads the
// tokens over more SMs and ends sooner. One GB300, INT4 / the paper's page, eight
// prompts of equal length, buffers larger together than L2, four against one: 4,096
// tokens 4.1 against 3.9 / 5.4 against 4.5 us, 8,192 5.8 against 6.3 / 7.1 against 7.1,
// 32,768 15.1 against 19.5 / 19.8 against 20.7.
constexpr int kFourPerLane = 8192;

// Tokens up to which the fused writer gives a warp to a group; above, eight lanes to a
// token. The border is one wave of the former: 152 SMs with five blocks of 288 threads (40
// registers; seven where nothing is quantised, 32) of four tokens. A warp to a group / eight
// lanes to a token, us, buffers larger together than L2:
//                                  3,040          3,041          4,256          4,257
//   INT4, normalised            5.64 / 6.25    6.42 / 6.28
//   INT4, as it is              4.22 / 4.50    4.99 / 4.63
//   INT4 / INT2, protected      5.9 / 6.5      6.7 / 6.5
//   the paper's page            5.74 / 6.43    7.38 / 7.30
//   BF16, normalised            4.84 / 5.37                   5.79 / 5.63    6.01 / 5.68
//   BF16, as it is              3.51 / 3.76                   3.96 / 4.13    4.39 / 4.14
template <int CB>
constexpr int kOneWave = 152 * 4 * (CB == kBf16Rows ? 7 : 5);

template <int CB, bool FUSED>
void launch_quant(const AppendArgs& a, const RowTransform& tr, bool vec, cudaStream_t stream) {
  if constexpr (FUSED) {
    if (vec && a.n > kOneWave<CB>) {
      constexpr long long kPerBlock = kWideThreads / 8;
      wide_append_kernel<CB><<<static_cast<unsigned>((a.n + kPerBlock - 1) / kPerBlock), kWideThreads, 0, stream>>>(
          static_cast<uint8_t*>(a.pool), a.num_blocks, reinterpret_cast<const uint32_t*>(a.latent),
          reinterpret_cast<const uint32_t*>(a.k_pe), a.seq_ids, a.positions, a.n, a.table, a.num_seqs, a.max_blocks,
          a.dev_err, static_cast<uint4*>(a.prot), a.lens, tr);
      return;
    }
    auto* f = vec ? launch_quant<CB, 1, true, true> : launch_quant<CB, 1, false, true>;
    f(a, tr, stream);
  } else {
    auto* f = !vec ? launch_quant<CB, 1, false, false>
                   : (a.n >= kFourPerLane ? launch_quant<CB, 4, true, false> : launch_quant<CB, 1, true, false>);
    f(a, tr, stream);
  }
}

}  // namespace

cudaError_t launch_quant_append(void* pool, int c_bits, int num_blocks, const uint16_t* latent,
                                const uint16_t* k_pe, const int32_t* seq_ids,
                                const int32_t* positions, int n, const int32_t* table, int num_seqs,
                                int max_blocks, uint32_t* dev_err, cudaStream_t stream, void* prot,
                                const int32_t* lens) {
  if (n == 0) return cudaSuccess;
  const AppendArgs a = {pool,     num_blocks, latent, k_pe,       seq_ids, positions,
                        n,        table,      num_seqs, max_blocks, dev_err, prot, lens};
  auto* f = c_bits == kC4R4 ? launch_quant<kC4R4, false> : (c_bits == 4 ? launch_quant<4, false> : launch_quant<2, false>);
  f(a, RowTransform{}, aligned16(latent, k_pe), stream);
  return cudaGetLastError();
}

cudaError_t launch_rope_append(const qmla_append_desc& d, const int32_t* rope_positions, cudaStream_t stream) {
  const AppendArgs a = {d.pool,        d.num_blocks, d.latent,     d.k_pe,    d.seq_ids, d.positions, d.n,
                        d.block_table, d.num_seqs,   d.max_blocks, d.dev_err, d.prot,    d.prot != nullptr ? d.seq_lens : nullptr};
  RowTransform tr;
  tr.latent_words = static_cast<size_t>(d.latent_stride) / 2;
  tr.k_pe_words = static_cast<size_t>(d.k_pe_stride) / 2;
  tr.norm = d.norm != 0;
  tr.weight = reinterpret_cast<const uint4*>(d.norm_weight);
  tr.eps = d.norm_eps;
  tr.cos_sin = d.cos_sin;
  tr.rope_len = d.rope_len;
  tr.turns = rope_positions != nullptr ? rope_positions : d.positions;
  tr.interleaved = d.interleaved != 0;
  const bool vec = aligned16(d.latent, d.k_pe) && d.latent_stride % 8 == 0 && d.k_pe_stride % 8 == 0;
  auto* f = d.cache_kind == kC4R4
                ? launch_quant<kC4R4, true>
                : (d.cache_kind == 4 ? launch_quant<4, true> : (d.cache_kind == 2 ? launch_quant<2, true> : launch_quant<kBf16Rows, true>));
  f(a, tr, vec, stream);
  return cudaGetLastError();
}

cudaError_t launch_bf16_append(void* pool, int num_blocks, const uint16_t* latent,
                               const uint16_t* k_pe, const int32_t* seq_ids,
                               const int32_t* positions, int n, const int32_t* table, int num_seqs,
                               int max_blocks, uint32_t* dev_err, cudaStream_t stream) {
  if (n == 0) return cudaSuccess;
  const unsigned grid = static_cast<unsigned>((static_cast<long long>(n) * (kDqk * 2 / 16) + 255) / 256);
  auto* f = aligned16(latent, k_pe) ? bf16_append_kernel<true> : bf16_append_kernel<false>;
  f<<<grid, 256, 0, stream>>>(static_cast<uint8_t*>(pool), num_blocks, reinterpret_cast<const uint32_t*>(latent),
                              reinterpret_cast<const uint32_t*>(k_pe), seq_ids, positions, n, table, num_seqs,
                              max_blocks, dev_err);
  return cudaGetLastError();
}

}  // namespace qmla
