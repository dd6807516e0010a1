// Cached tokens back as bf16 rows (the inverse of the cache writers' last step)
// and the rotation of queries.
#include <cuda_runtime.h>

#include "common.cuh"
#include "kernels.h"
#include "ptx.cuh"
#include "rope.cuh"

namespace qmla {
namespace {

constexpr int kBf16Rows = 16;  // cache kind of the BF16 cache
constexpr int kReadThreads = 128;

__device__ __forceinline__ uint4 load16(const void* p) {
  uint4 r;
  asm volatile("ld.global.nc.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];"
               : "=r"(r.x), "=r"(r.y), "=r"(r.z), "=r"(r.w)
               : "l"(p));
  return r;
}

// RN_bf16(RN_f32(s (q - z))) of two codes: 2^23 + q has q in its low mantissa bits
// and (2^23 + q) - (2^23 + z) is exact; for scales of at most 20 significant bits
// (all but the paper's RoPE scale) the product is exact too.
__device__ __forceinline__ uint32_t value2(uint32_t q0, uint32_t q1, uint64_t zz, uint64_t ss) {
  const uint64_t q = f32x2(__uint_as_float(0x4B000000u | q0), __uint_as_float(0x4B000000u | q1));
  const uint64_t v = mul2(add2(q, zz), ss);
  return pack_bf16(lo2(v), hi2(v));
}

// Reads n tokens: eight lanes a token, lane l the eight channels l of each of its nine
// groups (4 or 2 bytes of codes, a 16-byte store), so that a token's place is looked up
// once, all its loads are on their way together, and lane l fetches the scale of group l,
// which a shuffle hands round.
//
// What bounds it: the chain position -> block table -> codes -> store, which a warp goes
// through once (32,797 INT4 tokens 10.4 us, where 1,152 bytes written and 332 read a token are
// 7.2 at the copy's rate); over long BF16 contexts the HBM traffic (98,821 tokens 5.5 TB/s).
template <int CB>
__global__ void __launch_bounds__(kReadThreads) cache_read_kernel(
    const uint8_t* __restrict__ pool, int num_blocks, const int32_t* __restrict__ seq_ids,
    const int32_t* __restrict__ positions, int n, const int32_t* __restrict__ table, int num_seqs, int max_blocks,
    const int32_t* __restrict__ lens, const uint4* __restrict__ prot, uint16_t* __restrict__ rows, size_t row_stride,
    uint32_t* dev_err) {
  using L = BlockLayout<CB == kBf16Rows ? 4 : CB>;
  const int lane = threadIdx.x & 31, piece = lane & 7;
  const int tok = (blockIdx.x * (kReadThreads / 32) + (threadIdx.x >> 5)) * 4 + (lane >> 3);
  // Where the token is: in the pool (blk), in the protection buffer (kept), or nowhere.
  const uint8_t* blk = nullptr;
  const uint4* kept = nullptr;
  int slot = 0;
  if (tok < n) {
    const int seq = seq_ids != nullptr ? seq_ids[tok] : tok;
    const int pos = positions[tok];
    uint32_t bad = 0;
    if (seq < 0 || seq >= num_seqs) {
      bad = QMLA_DEVERR_BAD_SEQ;
    } else if (pos < 0 || pos >= max_blocks * kBlockTokens || (prot != nullptr && pos >= lens[seq])) {
      bad = QMLA_DEVERR_BAD_POSITION;
    } else if (prot != nullptr && (pos < kSinkTokens || pos >= lens[seq] - kRecentTokens)) {
      const int row = pos < kSinkTokens ? pos : kSinkTokens + pos % kRecentTokens;
      kept = prot + (static_cast<size_t>(seq) * kProtRows + row) * (kDqk * 2 / 16) + piece;
    } else {
      const int id = table[static_cast<size_t>(seq) * max_blocks + pos / kBlockTokens];
      if (id < 0 || id >= num_blocks) {
        bad = QMLA_DEVERR_BAD_BLOCK;
      } else {
        blk = pool + static_cast<size_t>(id) * (CB == kBf16Rows ? kBf16BlockBytes : L::kBytes);
        slot = pos % kBlockTokens;
      }
    }
    if (bad != 0 && piece == 0) report(dev_err, bad);
  }
  uint4* out = reinterpret_cast<uint4*>(rows + static_cast<size_t>(max(tok < n ? tok : 0, 0)) * row_stride) + piece;
  if (CB == kBf16Rows || kept != nullptr) {  // whole pieces
    const uint4* src = kept;
    if (CB == kBf16Rows && blk != nullptr) src = reinterpret_cast<const uint4*>(blk + slot * (kDqk * 2)) + piece;
    if (src != nullptr) {
      uint4 v[kGroups];
#pragma unroll
      for (int g = 0; g < kGroups; ++g) v[g] = load16(src + g * 8);
#pragma unroll
      for (int g = 0; g < kGroups; ++g) out[g * 8] = v[g];
    }
  }
  if constexpr (CB != kBf16Rows) {
    // Codes, and the scales of group `piece` (own) and of the RoPE key (pe).
    uint32_t c[kGroups];
    float s_own = 0.0f, z_own = 0.0f, s_pe = 0.0f, z_pe = 0.0f;
    if (blk != nullptr) {
#pragma unroll
      for (int g = 0; g < kGroups; ++g) {
        const uint8_t* at = blk + L::code_off(g, slot);
        c[g] = CB == 2 && g < 8 ? reinterpret_cast<const uint16_t*>(at)[piece] : reinterpret_cast<const uint32_t*>(at)[piece];
      }
      if constexpr (CB == kC4R4) {
        s_own = __uint_as_float(static_cast<uint32_t>(*reinterpret_cast<const uint16_t*>(blk + L::c_scale_off(piece, slot))) << 16);
        z_own = static_cast<float>(blk[L::zero_off(piece, slot)]);
        s_pe = *reinterpret_cast<const float*>(blk + L::pe_scale_off(slot));
        z_pe = static_cast<float>(blk[L::zero_off(8, slot)]);
      } else {
        const float2 own = __half22float2(*reinterpret_cast<const __half2*>(blk + L::sz_off(piece, slot)));
        const float2 pe = __half22float2(*reinterpret_cast<const __half2*>(blk + L::sz_off(8, slot)));
        s_own = own.x, z_own = own.y, s_pe = pe.x, z_pe = pe.y;
      }
    }
#pragma unroll
    for (int g = 0; g < kGroups; ++g) {
      const int from = (lane & 24) | (g & 7);
      const float s = g < 8 ? __shfl_sync(0xffffffffu, s_own, from) : s_pe;
      const float z = g < 8 ? __shfl_sync(0xffffffffu, z_own, from) : z_pe;
      if (blk == nullptr) continue;
      const uint64_t zz = f32x2(-8388608.0f - z, -8388608.0f - z), ss = f32x2(s, s);
      const uint32_t q = c[g];
      if (CB != 2 || g == 8) {
        out[g * 8] = make_uint4(value2(q & 15u, (q >> 4) & 15u, zz, ss), value2((q >> 8) & 15u, (q >> 12) & 15u, zz, ss),
                                value2((q >> 16) & 15u, (q >> 20) & 15u, zz, ss), value2((q >> 24) & 15u, q >> 28, zz, ss));
      } else {
        out[g * 8] = make_uint4(value2(q & 3u, (q >> 2) & 3u, zz, ss), value2((q >> 4) & 3u, (q >> 6) & 3u, zz, ss),
                                value2((q >> 8) & 3u, (q >> 10) & 3u, zz, ss), value2((q >> 12) & 3u, (q >> 14) & 3u, zz, ss));
      }
    }
  }
}

template <int CB>
void launch_read(const qmla_read_desc& d, cudaStream_t stream) {
  constexpr long long kPerBlock = kReadThreads / 8;
  cache_read_kernel<CB><<<static_cast<unsigned>((d.n + kPerBlock - 1) / kPerBlock), kReadThreads, 0, stream>>>(
      static_cast<const uint8_t*>(d.pool), d.num_blocks, d.seq_ids, d.positions, d.n, d.block_table, d.num_seqs,
      d.max_blocks, d.seq_lens, static_cast<const uint4*>(d.prot), d.rows, static_cast<size_t>(d.row_stride), d.dev_err);
}

// Rotates rows of 64 channels, `heads` of them per token: eight lanes a row, each
// with 16 bytes. A lane group takes kQueryRows rows, kQueryStep apart, whose loads are all
// issued first; neighbouring rows share a token, so the angles are loaded again
// only where the token changes. One division per thread finds the first row's token;
// step_tokens and step_heads are what kQueryStep rows are in tokens and heads.
//
// What bounds it: the HBM traffic (256 bytes per row). 8,184 tokens x 128 heads, the RoPE
// part of [n, heads, 192] queries, take 43.0 us, 6.3 TB/s of 6.8. Ten blocks per SM: with
// the eight that the registers would leave 46.4 (a 64-bit division per row 55; two rows
// per lane group 53, eight 61; blocks of 256 threads 47.8), with twelve 42.4, but 80
// rows, which are all latency, 4.1 instead of 3.4.
constexpr int kQueryThreads = 128;
constexpr int kQueryRows = 4, kQueryStep = kQueryThreads / 8;

__global__ void __launch_bounds__(kQueryThreads, 10) rope_query_kernel(
    const uint16_t* q, size_t q_token, size_t q_head, const int32_t* __restrict__ positions, long long rows, int heads,
    int step_tokens, int step_heads, const float* __restrict__ cos_sin, int rope_len, bool interleaved, uint16_t* out,
    size_t out_token, size_t out_head, uint32_t* dev_err) {
  const int piece = threadIdx.x & 7;
  const long long row0 = static_cast<long long>(blockIdx.x) * (kQueryStep * kQueryRows) + (threadIdx.x >> 3);
  int tok[kQueryRows], head[kQueryRows];
  if (rows <= UINT32_MAX) {
    tok[0] = static_cast<int>(static_cast<uint32_t>(row0) / static_cast<uint32_t>(heads));
  } else {
    tok[0] = static_cast<int>(row0 / heads);
  }
  head[0] = static_cast<int>(row0 - static_cast<long long>(tok[0]) * heads);
  uint4 raw[kQueryRows];
#pragma unroll
  for (int i = 0; i < kQueryRows; ++i) {
    if (i > 0) {
      tok[i] = tok[i - 1] + step_tokens;
      head[i] = head[i - 1] + step_heads;
      if (head[i] >= heads) {
        head[i] -= heads;
        ++tok[i];
      }
    }
    raw[i] = make_uint4(0, 0, 0, 0);
    if (row0 + i * kQueryStep < rows)
      raw[i] = *reinterpret_cast<const uint4*>(q + tok[i] * q_token + head[i] * q_head + piece * 8);
  }
  int have = -1;
  bool good = false;
  Angles a;
  load_angles(a, nullptr, piece, interleaved);
#pragma unroll
  for (int i = 0; i < kQueryRows; ++i) {
    const bool live = row0 + i * kQueryStep < rows;
    if (live && tok[i] != have) {
      have = tok[i];
      const int pos = positions[have];
      good = pos >= 0 && pos < rope_len;
      load_angles(a, good ? cos_sin + static_cast<size_t>(pos) * kDr : nullptr, piece, interleaved);
    }
    if (live && !good && piece == 0 && head[i] == 0) report(dev_err, QMLA_DEVERR_BAD_POSITION);
    uint32_t w[4] = {raw[i].x, raw[i].y, raw[i].z, raw[i].w};
    rotate_row<false>(w, a, piece, interleaved);
    if (live && good)
      *reinterpret_cast<uint4*>(out + tok[i] * out_token + head[i] * out_head + piece * 8) =
          make_uint4(w[0], w[1], w[2], w[3]);
  }
}

}  // namespace

cudaError_t launch_cache_read(const qmla_read_desc& d, cudaStream_t stream) {
  auto* f = d.cache_kind == kC4R4 ? launch_read<kC4R4>
                                  : (d.cache_kind == 4 ? launch_read<4> : (d.cache_kind == 2 ? launch_read<2> : launch_read<kBf16Rows>));
  f(d, stream);
  return cudaGetLastError();
}

cudaError_t launch_rope_query(const uint16_t* q, long long q_token, long long q_head, const int32_t* positions, int n,
                              int heads, const float* cos_sin, int rope_len, bool interleaved, uint16_t* out,
                              long long out_token, long long out_head, uint32_t* dev_err, cudaStream_t stream) {
  const long long rows = static_cast<long long>(n) * heads;
  constexpr long long kPerBlock = kQueryStep * kQueryRows;
  rope_query_kernel<<<static_cast<unsigned>((rows + kPerBlock - 1) / kPerBlock), kQueryThreads, 0, stream>>>(
      q, static_cast<size_t>(q_token), static_cast<size_t>(q_head), positions, rows, heads, kQueryStep / heads,
      kQueryStep % heads, cos_sin, rope_len, interleaved, out, static_cast<size_t>(out_token), static_cast<size_t>(out_head), dev_err);
  return cudaGetLastError();
}

}  // namespace qmla
