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
constexpr int kReadThreads = kGroups * 32;

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

// Reads n tokens: warp g of a block the 64 channels of group g of 4 NT tokens, eight
// lanes a token with eight channels (a 16-byte store) each, as the writer has them.
// Lane i of a token's NT looks the place of token i up; shuffles hand it round.
//
// What bounds it: the HBM traffic, 1,152 bytes written and 196 to 1,152 read per
// token, once enough tokens are in flight to cover the chain position -> block
// table -> codes.
template <int CB, int NT>
__global__ void __launch_bounds__(kReadThreads) cache_read_kernel(
    const uint8_t* __restrict__ pool, int num_blocks, const int32_t* __restrict__ seq_ids,
    const int32_t* __restrict__ positions, int n, const int32_t* __restrict__ table, int num_seqs, int max_blocks,
    const int32_t* __restrict__ lens, const uint4* __restrict__ prot, uint16_t* __restrict__ rows, size_t row_stride,
    uint32_t* dev_err) {
  using L = BlockLayout<CB == kBf16Rows ? 4 : CB>;
  const int g = threadIdx.x >> 5, lane = threadIdx.x & 31, piece = lane & 7;
  const int tok0 = blockIdx.x * (4 * NT) + (lane >> 3);
  const int own = piece & (NT - 1);
  // >= 0: block id times 64 plus the slot; -1: nothing to read; -2 - r: protection row r
  long long src = -1;
  if (const int tok = tok0 + 4 * own; tok < n) {
    const int seq = seq_ids != nullptr ? seq_ids[tok] : tok;
    const int pos = positions[tok];
    uint32_t bad = 0;
    if (seq < 0 || seq >= num_seqs) {
      bad = QMLA_DEVERR_BAD_SEQ;
    } else if (pos < 0 || pos >= max_blocks * kBlockTokens || (prot != nullptr && pos >= lens[seq])) {
      bad = QMLA_DEVERR_BAD_POSITION;
    } else if (prot != nullptr && (pos < kSinkTokens || pos >= lens[seq] - kRecentTokens)) {
      const int row = pos < kSinkTokens ? pos : kSinkTokens + pos % kRecentTokens;
      src = -2 - (static_cast<long long>(seq) * kProtRows + row);
    } else {
      const int blk = table[static_cast<size_t>(seq) * max_blocks + pos / kBlockTokens];
      if (blk < 0 || blk >= num_blocks) {
        bad = QMLA_DEVERR_BAD_BLOCK;
      } else {
        src = static_cast<long long>(blk) * kBlockTokens + pos % kBlockTokens;
      }
    }
    if (bad != 0 && g == 0 && piece == own) report(dev_err, bad);
  }
  const bool four = CB != 2 || g == 8;  // codes of four bits (uniform in the warp)
  long long at[NT];
  uint4 full[NT];  // a whole piece (bf16 rows, protection rows), or {codes, scale, zero, -}
#pragma unroll
  for (int i = 0; i < NT; ++i) {
    at[i] = NT == 1 ? src : __shfl_sync(0xffffffffu, src, (lane & 24) | i);
    full[i] = make_uint4(0, 0, 0, 0);
    if (at[i] <= -2) {
      full[i] = load16(prot + static_cast<size_t>(-2 - at[i]) * (kDqk * 2 / 16) + g * 8 + piece);
    } else if (at[i] >= 0) {
      const size_t blk = static_cast<size_t>(at[i]) / kBlockTokens;
      const int slot = static_cast<int>(at[i] % kBlockTokens);
      if constexpr (CB == kBf16Rows) {
        full[i] = load16(pool + blk * kBf16BlockBytes + slot * (kDqk * 2) + (g * 8 + piece) * 16);
      } else {
        const uint8_t* b = pool + blk * L::kBytes;
        const uint8_t* c = b + L::code_off(g, slot);
        full[i].x = four ? reinterpret_cast<const uint32_t*>(c)[piece] : reinterpret_cast<const uint16_t*>(c)[piece];
        if constexpr (CB == kC4R4) {
          full[i].y = g < 8 ? static_cast<uint32_t>(*reinterpret_cast<const uint16_t*>(b + L::c_scale_off(g, slot))) << 16
                            : *reinterpret_cast<const uint32_t*>(b + L::pe_scale_off(slot));
          full[i].z = b[L::zero_off(g, slot)];
        } else {
          full[i].y = *reinterpret_cast<const uint32_t*>(b + L::sz_off(g, slot));
        }
      }
    }
  }
#pragma unroll
  for (int i = 0; i < NT; ++i) {
    if (at[i] == -1) continue;
    uint4 out = full[i];
    if constexpr (CB != kBf16Rows) {
      if (at[i] >= 0) {
        float s, z;
        if constexpr (CB == kC4R4) {
          s = __uint_as_float(full[i].y);
          z = static_cast<float>(full[i].z);
        } else {
          const float2 sz = __half22float2(*reinterpret_cast<const __half2*>(&full[i].y));
          s = sz.x;
          z = sz.y;
        }
        const uint64_t zz = f32x2(-8388608.0f - z, -8388608.0f - z), ss = f32x2(s, s);
        const uint32_t c = full[i].x;
        if (four) {
          out = make_uint4(value2(c & 15u, (c >> 4) & 15u, zz, ss), value2((c >> 8) & 15u, (c >> 12) & 15u, zz, ss),
                           value2((c >> 16) & 15u, (c >> 20) & 15u, zz, ss), value2((c >> 24) & 15u, c >> 28, zz, ss));
        } else {
          out = make_uint4(value2(c & 3u, (c >> 2) & 3u, zz, ss), value2((c >> 4) & 3u, (c >> 6) & 3u, zz, ss),
                           value2((c >> 8) & 3u, (c >> 10) & 3u, zz, ss), value2((c >> 12) & 3u, (c >> 14) & 3u, zz, ss));
        }
      }
    }
    *reinterpret_cast<uint4*>(rows + static_cast<size_t>(tok0 + 4 * i) * row_stride + g * 64 + piece * 8) = out;
  }
}

template <int CB, int NT>
void launch_read_nt(const qmla_read_desc& d, cudaStream_t stream) {
  const unsigned grid = static_cast<unsigned>((static_cast<long long>(d.n) + 4 * NT - 1) / (4 * NT));
  cache_read_kernel<CB, NT><<<grid, kReadThreads, 0, stream>>>(
      static_cast<const uint8_t*>(d.pool), d.num_blocks, d.seq_ids, d.positions, d.n, d.block_table, d.num_seqs,
      d.max_blocks, d.seq_lens, static_cast<const uint4*>(d.prot), d.rows, static_cast<size_t>(d.row_stride), d.dev_err);
}

// Tokens from which a lane takes four.
constexpr int kFourPerLane = 4096;

template <int CB>
void launch_read(const qmla_read_desc& d, cudaStream_t stream) {
  if (d.n >= kFourPerLane) {
    launch_read_nt<CB, 4>(d, stream);
  } else {
    launch_read_nt<CB, 1>(d, stream);
  }
}

// Rotates rows of 64 channels, `heads` of them per token: eight lanes a row, each
// with 16 bytes. A lane group takes kQueryRows rows, 32 apart, whose loads are all
// issued first; neighbouring rows share a token, so the angles are loaded again
// only where the token changes.
constexpr int kQueryThreads = 256;
constexpr int kQueryRows = 4;

__global__ void __launch_bounds__(kQueryThreads) rope_query_kernel(
    const uint16_t* q, size_t q_token, size_t q_head, const int32_t* __restrict__ positions, long long rows, int heads,
    const float* __restrict__ cos_sin, int rope_len, bool interleaved, uint16_t* out, size_t out_token, size_t out_head,
    uint32_t* dev_err) {
  constexpr int kStep = kQueryThreads / 8;
  const int piece = threadIdx.x & 7;
  const long long row0 = static_cast<long long>(blockIdx.x) * (kStep * kQueryRows) + (threadIdx.x >> 3);
  uint4 raw[kQueryRows];
  long long tok[kQueryRows];
#pragma unroll
  for (int i = 0; i < kQueryRows; ++i) {
    const long long row = row0 + i * kStep;
    raw[i] = make_uint4(0, 0, 0, 0);
    tok[i] = -1;
    if (row < rows) {
      tok[i] = row / heads;
      raw[i] = *reinterpret_cast<const uint4*>(q + tok[i] * q_token + (row - tok[i] * heads) * q_head + piece * 8);
    }
  }
  long long have = -1;
  bool good = false;
  Angles a;
  load_angles(a, nullptr, piece, interleaved);
#pragma unroll
  for (int i = 0; i < kQueryRows; ++i) {
    const long long row = row0 + i * kStep;
    if (tok[i] >= 0 && tok[i] != have) {
      have = tok[i];
      const int pos = positions[have];
      good = pos >= 0 && pos < rope_len;
      load_angles(a, good ? cos_sin + static_cast<size_t>(pos) * kDr : nullptr, piece, interleaved);
    }
    if (tok[i] >= 0 && !good && piece == 0 && row == tok[i] * heads) report(dev_err, QMLA_DEVERR_BAD_POSITION);
    uint32_t w[4] = {raw[i].x, raw[i].y, raw[i].z, raw[i].w};
    rotate_row<false>(w, a, piece, interleaved);
    if (tok[i] >= 0 && good)
      *reinterpret_cast<uint4*>(out + tok[i] * out_token + (row - tok[i] * heads) * out_head + piece * 8) =
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
  constexpr long long kPerBlock = kQueryThreads / 8 * kQueryRows;
  rope_query_kernel<<<static_cast<unsigned>((rows + kPerBlock - 1) / kPerBlock), kQueryThreads, 0, stream>>>(
      q, static_cast<size_t>(q_token), static_cast<size_t>(q_head), positions, rows, heads, cos_sin, rope_len,
      interleaved, out, static_cast<size_t>(out_token), static_cast<size_t>(out_head), dev_err);
  return cudaGetLastError();
}

}  // namespace qmla
