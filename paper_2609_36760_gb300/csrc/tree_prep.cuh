// What prep does for a tree's decode beside the plan and the query rows: the nodes' sets, and the
// context as fp16 images for tree_pair. Included by decode.cu inside its namespaces, where it
// is compiled for trees (decode_tree.cu).
#pragma once

// Sets of nodes of kTreesPerBlock sequences from b0 on, a thread per node: each finds the
// nodes above its own by doubling (after step i it holds 2^i of them, and its 2^i-th
// ancestor). kMaxNodes stands for "none above".
__device__ __forceinline__ void make_trees(const Params& p, int b0) {
  __shared__ uint64_t line[kTreesPerBlock][kMaxNodes + 1];
  __shared__ uint8_t up[kTreesPerBlock][kMaxNodes + 1], bad[kTreesPerBlock][kMaxNodes + 1];
  const int i = threadIdx.x / kMaxNodes, t = threadIdx.x % kMaxNodes, b = b0 + i;
  const bool any = b < p.batch;
  int n = 0, parent = -1;
  if (any) {
    n = p.tree_lens != nullptr ? p.tree_lens[b] : p.q_tokens;
    if (n < 0 || n > p.q_tokens || n > p.seq_lens[b]) n = 0;  // (reported with the lengths)
    if (t < n) parent = p.parents[static_cast<size_t>(b) * p.q_tokens + t];
  }
  const bool wrong = t < n && (parent < -1 || parent >= t);
  if (wrong) report(p.dev_err, QMLA_DEVERR_BAD_TREE);
  line[i][t] = t < n ? 1ull << t : 0ull;
  up[i][t] = static_cast<uint8_t>(wrong || parent < 0 ? kMaxNodes : parent);
  bad[i][t] = wrong ? 1 : 0;
  if (t == 0) {
    line[i][kMaxNodes] = 0ull;
    up[i][kMaxNodes] = kMaxNodes;
    bad[i][kMaxNodes] = 0;
  }
  __syncthreads();
#pragma unroll 1
  for (int s = 1; s < kMaxNodes; s *= 2) {
    const int a = up[i][t];
    const uint64_t l = line[i][t] | line[i][a];
    const uint8_t w = bad[i][t] | bad[i][a], a2 = up[i][a];
    __syncthreads();
    line[i][t] = l;
    bad[i][t] = w;
    up[i][t] = a2;
    __syncthreads();
  }
  const bool ok = t < n && bad[i][t] == 0;
  const uint64_t mine = ok ? line[i][t] : 0ull;
  __syncthreads();
  line[i][t] = mine;
  __syncthreads();
  uint64_t below = 0ull, alive = 0ull;
#pragma unroll 4
  for (int u = 0; u < kMaxNodes; ++u) {
    const uint64_t l = line[i][u];
    if ((l >> t) & 1ull) below |= 1ull << u;
    if (l != 0ull) alive |= 1ull << u;
  }
  griddep_wait();  // (see prep_kernel)
  if (!any) return;
  TreeSeq& o = p.trees[b];
  o.seen_by[t] = below;
  o.line[t] = mine;
  if (t == 0) {
    o.alive = alive;
    o.ctx = p.seq_lens[b] - n;
  }
}

// One 16-byte piece of a cache row as it is loaded, and its eight values.
struct RowPiece {
  uint4 raw;    // bf16 values, or codes in x and scale and zero in y, z
};
// Piece i of chunk k of the packed row in `slot` of blk (the BF16 cache: of its values).
template <int CB>
__device__ __forceinline__ RowPiece load_piece(const uint8_t* blk, int slot, int k, int i) {
  RowPiece r;
  r.raw = make_uint4(0, 0, 0, 0);
  if constexpr (CB == 16) {
    r.raw = ldg_nc_v4(blk + slot * (kDqk * 2) + k * 128 + i * 16);
  } else {
    using L = BlockLayout<CB>;
    const uint8_t* codes = blk + L::code_off(k, slot);
    r.raw.x = CB == 2 && k < 8 ? ldg_nc_u16(codes + 2 * i) : ldg_nc_u32(codes + 4 * i);
    if constexpr (CB == kC4R4) {
      r.raw.y = k < 8 ? ldg_nc_u16(blk + L::c_scale_off(k, slot)) : ldg_nc_u32(blk + L::pe_scale_off(slot));
      r.raw.z = ldg_nc_u8(blk + L::zero_off(k, slot));
    } else {
      r.raw.y = ldg_nc_u32(blk + L::sz_off(k, slot));
    }
  }
  return r;
}
__device__ __forceinline__ void bf16_values(const uint4& raw, float (&f)[8]) {
  const uint32_t w[4] = {raw.x, raw.y, raw.z, raw.w};
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    f[2 * e] = bf16_lo(w[e]);
    f[2 * e + 1] = bf16_hi(w[e]);
  }
}
template <int CB>
__device__ __forceinline__ void piece_values(const RowPiece& r, int k, float (&f)[8]) {
  if constexpr (CB == 16) {
    bf16_values(r.raw, f);
  } else {
    float s, z;
    if constexpr (CB == kC4R4) {
      s = __uint_as_float(k < 8 ? r.raw.y << 16 : r.raw.y);
      z = static_cast<float>(r.raw.z);
    } else {
      const __half2 h = *reinterpret_cast<const __half2*>(&r.raw.y);
      s = __low2float(h);
      z = __high2float(h);
    }
    constexpr uint32_t kNarrow = 2, kWide = 4;
    const uint32_t bits = CB == 2 && k < 8 ? kNarrow : kWide;
#pragma unroll
    for (int e = 0; e < 8; ++e)
      f[e] = s * (static_cast<float>((r.raw.x >> (bits * e)) & ((1u << bits) - 1u)) - z);
  }
}
__device__ __forceinline__ uint4 half_piece(const float (&f)[8]) {
  return make_uint4(pack_h2(f[0], f[1]), pack_h2(f[2], f[3]), pack_h2(f[4], f[5]), pack_h2(f[6], f[7]));
}
// What rounding to fp16 leaves off.
__device__ __forceinline__ uint4 rest_piece(const float (&f)[8]) {
  float d[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) d[e] = f[e] - __half2float(__float2half_rn(f[e]));
  return half_piece(d);
}

// Largest magnitude of fp16 pieces so far; an infinity or NaN stays one.
__device__ __forceinline__ void widen(__half2& top, uint4 v) {
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int e = 0; e < 4; ++e) top = __hmax2_nan(top, __habs2(*reinterpret_cast<const __half2*>(&w[e])));
}
// Whether one of the eight threads of a row (whole warps call) met such a value.
__device__ __forceinline__ bool row_not_finite(__half2 top) {
  const bool finite = __low2float(top) <= 65504.0f && __high2float(top) <= 65504.0f;
  return (__ballot_sync(0xffffffffu, !finite) >> (threadIdx.x & 24) & 0xffu) != 0u;
}

// The nodes of sequence b whose cache row has a value that is not finite, eight threads a row.
template <int CB>
__device__ void find_not_finite(const Params& p, int b) {
  __shared__ unsigned long long found;
  if (threadIdx.x == 0) found = 0ull;
  __syncthreads();
  int groups;
  tree_tiles(p, b, 1, groups, nullptr);
  const int t = threadIdx.x >> 3, i = threadIdx.x & 7;
  const int n = groups == 0 ? 0 : (p.tree_lens != nullptr ? p.tree_lens[b] : p.q_tokens);
  const int pos = p.seq_lens[b] - n + t, slot = pos & (kBlockTokens - 1);
  const int entry = t < n ? p.table[static_cast<size_t>(b) * p.max_blocks + pos / kBlockTokens] : -1;
  __half2 top = __float2half2_rn(0.0f);
  griddep_wait();  // (the cache may still be written until here)
  if (t < n) {
    float f[8];
    if (CB != 16 && p.prot != nullptr) {
      const uint8_t* const src = p.draft_rows + (static_cast<size_t>(b) * kMaxNodes + t) * (kDqk * 2);
#pragma unroll
      for (int k = 0; k < kNumChunks; ++k) {
        bf16_values(ldg_nc_v4(src + k * 128 + i * 16), f);
        widen(top, half_piece(f));
      }
    } else if (entry >= 0 && entry < p.num_blocks) {
      constexpr size_t kBlk = CB == 16 ? static_cast<size_t>(kBf16BlockBytes) : BlockLayout<CB == 16 ? 4 : CB>::kBytes;
      const uint8_t* const blk = p.pool + static_cast<size_t>(entry) * kBlk;
#pragma unroll
      for (int k = 0; k < kNumChunks; ++k) {
        const RowPiece r = load_piece<CB>(blk, slot, k, i);
        piece_values<CB>(r, k, f);
        widen(top, half_piece(f));
        // (a scale beyond fp16: the tile's product with a difference of 0 is NaN)
        if (CB == kC4R4) top = __hmax2_nan(top, __float2half2_rn(k < 8 ? __uint_as_float(r.raw.y << 16) : __uint_as_float(r.raw.y)));
      }
    }
  }
  if (row_not_finite(top) && t < n && i == 0) atomicOr(&found, 1ull << t);
  __syncthreads();
  if (threadIdx.x == 0) p.trees[b].not_finite = found;
}

// Block j of sequence b as an fp16 image (see Params::images), zero
// behind the sequence's end up to a whole tile, and perhaps the image of C - RN_f16(C). A thread has
// the same eight channels of one row's nine chunks, all loaded before any is stored. A row with a
// value that is not finite is 0 with NaN in the RoPE channels, which are keys alone: so it makes
// NaN of the queries that see it, and its weight of 0 nothing of the others. False: behind the
// sequence's end.
template <int CB>
__device__ bool expand_block(const Params& p, int b, int j) {
  static_assert(!kTree || kPrepThreads == kBlockTokens * 8, "a thread per row and piece");
  const size_t idx = static_cast<size_t>(b) * p.img_width + j;
  const int entry = j < p.max_blocks ? p.table[static_cast<size_t>(b) * p.max_blocks + j] : -1;
  int groups;
  if (j >= tree_tiles(p, b, 1, groups, nullptr) * (kTileTokens / kBlockTokens) || groups == 0) return false;
  const int len = p.seq_lens[b], ctx = len - (p.tree_lens != nullptr ? p.tree_lens[b] : p.q_tokens);
  constexpr size_t kBlk = CB == 16 ? static_cast<size_t>(kBf16BlockBytes) : BlockLayout<CB == 16 ? 4 : CB>::kBytes;
  griddep_wait();  // (the cache may still be written until here)
  const bool known = entry >= 0 && entry < p.num_blocks;
  const uint8_t* const blk = p.pool + static_cast<size_t>(known ? entry : 0) * kBlk;
  const int i = threadIdx.x & 7, slot = threadIdx.x >> 3, pos = j * kBlockTokens + slot;
  const size_t at = swz_off(slot, i, 128);
  uint8_t* const img = p.images + idx * kImage + at;
  uint8_t* const rest = p.rest_images != nullptr ? p.rest_images + idx * kImage + at : nullptr;
  const uint8_t* src = nullptr;
  if (CB != 16 && p.prot != nullptr) {
    RowRef r;
    r.has = true;
    r.j = pos / kTileTokens;
    r.len = len;
    r.b = b;
    src = prot_row_tree(p, r, pos % kTileTokens, ctx);
  }
  float f[8];
  __half2 top = __float2half2_rn(0.0f);
  auto put = [&](int k) {
    const uint4 v = half_piece(f);
    widen(top, v);
    *reinterpret_cast<uint4*>(img + k * (64 * 128)) = v;
    if (rest != nullptr) *reinterpret_cast<uint4*>(rest + k * (64 * 128)) = rest_piece(f);
  };
  if (CB != 16 && src != nullptr) {
    uint4 raw[kNumChunks];
#pragma unroll
    for (int k = 0; k < kNumChunks; ++k) raw[k] = ldg_nc_v4(src + k * 128 + i * 16);
#pragma unroll
    for (int k = 0; k < kNumChunks; ++k) {
      bf16_values(raw[k], f);
      put(k);
    }
  } else if (known && pos < len) {
    RowPiece r[kNumChunks];
#pragma unroll
    for (int k = 0; k < kNumChunks; ++k) r[k] = load_piece<CB>(blk, slot, k, i);
#pragma unroll
    for (int k = 0; k < kNumChunks; ++k) {
      piece_values<CB>(r[k], k, f);
      put(k);
    }
  } else {
    if (pos < len) report(p.dev_err, QMLA_DEVERR_BAD_BLOCK);
#pragma unroll 1
    for (int k = 0; k < kNumChunks; ++k) {
      *reinterpret_cast<uint4*>(img + k * (64 * 128)) = make_uint4(0, 0, 0, 0);
      if (rest != nullptr) *reinterpret_cast<uint4*>(rest + k * (64 * 128)) = make_uint4(0, 0, 0, 0);
    }
  }
  if (row_not_finite(top)) {
#pragma unroll 1
    for (int k = 0; k < kNumChunks; ++k) {
      const uint32_t w = k < 8 ? 0u : 0x7fff7fffu;
      *reinterpret_cast<uint4*>(img + k * (64 * 128)) = make_uint4(w, w, w, w);
      if (rest != nullptr) *reinterpret_cast<uint4*>(rest + k * (64 * 128)) = make_uint4(0, 0, 0, 0);
    }
  }
  return true;
}

// The image of 64 query rows (see query_piece), in channel order; a thread's work as above. Rows
// of a group without a node get their results.
__device__ __forceinline__ void query_image(const Params& p, int u) {
  const int b = u / p.n_img, i = threadIdx.x & 7, h = threadIdx.x >> 3;
  const int row = (u - b * p.n_img) * 64 + h;
  int groups;
  const int tiles = tree_tiles(p, b, 128, groups, nullptr);
  if (tiles == 0 || (u - b * p.n_img) / 2 >= groups) {
    // No node has a row here: nothing runs for them but this.
    if (row >= p.heads) return;
    griddep_wait();
    uint4* const out = reinterpret_cast<uint4*>(reinterpret_cast<__nv_bfloat16*>(p.out) +
                                                (static_cast<size_t>(b) * p.heads + row) * kDc) + i * (kDc / 64);
#pragma unroll
    for (int e = 0; e < kDc / 64; ++e) out[e] = make_uint4(0, 0, 0, 0);
    if (i == 0 && p.lse != nullptr) p.lse[static_cast<size_t>(b) * p.heads + row] = -INFINITY;
    return;
  }
  uint4 raw[kNumChunks];
#pragma unroll
  for (int k = 0; k < kNumChunks; ++k) raw[k] = make_uint4(0, 0, 0, 0);
  if (row < p.heads) {
    const size_t r = static_cast<size_t>(b) * p.heads + row;
#pragma unroll
    for (int k = 0; k < kNumChunks; ++k)
      raw[k] = ldg_nc_v4(k < 8 ? p.q_lat + r * kDc + k * 64 + i * 8 : p.q_pe + r * kDr + i * 8);
  }
  griddep_wait();  // (see prep_kernel)
  uint8_t* const img = p.qimg + static_cast<size_t>(u) * (kNumChunks * 64 * 128) + swz_off(h, i, 128);
  float f[8];
#pragma unroll
  for (int k = 0; k < kNumChunks; ++k) {
    bf16_values(raw[k], f);
    *reinterpret_cast<uint4*>(img + k * 64 * 128) = half_piece(f);
  }
}
