// Attention of a tree of drafted tokens over a paged cache: query row (t, h), node t and
// head h, sees the context and the nodes on its path (Eq. mla_compact, with a mask of nodes
// in the place of the causal one).
//
// With few query rows over long contexts the kernels are the decode's (decode.cu, compiled here
// for trees: masks, bf16 results); prep also finds the sets of nodes above and below each node.
// Else prep lays the context out as fp16 images, once for all rows of a sequence, and
// tree_pair and tree_merge (tree_pair.cu) work over those.
#define QMLA_DECODE_TREE 1
#include "decode.cu"

namespace qmla {
namespace {

constexpr size_t round_up(size_t x) { return (x + 255) & ~static_cast<size_t>(255); }

struct TreeWorkspace {
  DecodeWorkspace decode;
  size_t trees_off, images_off;  // images: what is left
};
TreeWorkspace tree_workspace_layout(int batch, int rows, int grid) {
  TreeWorkspace w;
  // (units of 128 rows have images for an even number of 64-row groups)
  w.decode = decode_workspace_layout(batch, rows <= 64 ? 128 : (rows + 127) / 128 * 128, grid);
  w.trees_off = round_up(w.decode.total);
  w.images_off = round_up(w.trees_off + static_cast<size_t>(batch) * sizeof(TreeSeq));
  return w;
}
int image_blocks(long long tokens) {  // of whole tiles
  return static_cast<int>((tokens + kTileTokens - 1) / kTileTokens * (kTileTokens / kBlockTokens));
}
size_t image_bytes(int blocks, bool rest) { return static_cast<size_t>(blocks) * (rest ? 2 : 1) * kImage; }  // a sequence's

// Whether the context is laid out as images for tree_pair (where the workspace has room for them):
// where lse is asked for of a quantised cache, for its precision (with the second pass for it 8 x
// 8,000 tokens and 16 rows take 69 us, 64 x 4,000 217); else for more than 64 rows, and up to
// 40,960 tokens of the batch, counted by the table's width or the caller's bound. Measured on one GB300
// (INT4 without lse, one call replayed, us, decode_main's rows against the images; protected and BF16
// rows gain more from them):
//                 16 rows         64         128         256       1,024
//   1 x    500  21.6 / 15.4  30.2 / 16.9  27.3 / 17.2  26.6 / 18.5  30.3 / 19.6
//   8 x    500  17.9 / 16.3  26.8 / 18.1  29.7 / 19.0  36.9 / 22.4  55.9 / 31.3
//   8 x  4,000  22.7 / 27.1  31.7 / 30.2  43.9 / 31.2  64.7 / 38.4   145 / 66
//  64 x    500  23.8 / 27.2  38.7 / 32.1  54.0 / 35.5  85.8 / 51.3   261 / 120
//   1 x 40,000  33.3 / 31.6  43.5 / 37.4  46.8 / 38.8  60.0 / 38.9   158 / 70
//   8 x  8,000  28.5 / 42.6  39.4 / 45.2  59.0 / 45.3  87.2 / 54.7   250 / 109
//   1 x 100,000 42.5 / 63.7  55.9 / 64.8  70.9 / 61.3   109 / 73     354 / 150
//  64 x  4,000  61.9 / 130   95.5 / 135    152 / 139    273 / 176  1,004 / 420
bool on_images(int rows, long long tokens, bool rest) { return rest || rows > 64 || tokens <= 40960; }

template <int CB, bool PROT>
cudaError_t launch_rows(int hg, const Params& prm, cudaStream_t stream) {
  if (hg == 16) return launch_impl<CB, 16, PROT, false>(prm, stream, nullptr, nullptr);
  if (hg == 32) return launch_impl<CB, 32, PROT, false>(prm, stream, nullptr, nullptr);
  return launch_impl<CB, 64, PROT, false>(prm, stream, nullptr, nullptr);
}

// Images that L2 does not hold are read by all row groups of a sequence at once: the plan
// goes group by group, with as many ranges to each, which then keep step (64 x 4,096 tokens, 4
// groups: the main kernel 221 to 181 us), unless that leaves over a twelfth of the pairs idle.
bool keep_step(int pairs, int groups) {
  const int teams = pairs / groups;
  return teams > 0 && (pairs - teams * groups) * 12 <= pairs;
}

// The n sequences from b on over images at `images`, blocks of them a sequence.
cudaError_t launch_images(const qmla_tree_desc& d, Params prm, uint8_t* images, int b, int n, int blocks, bool rest,
                          cudaStream_t stream) {
  const size_t rows = static_cast<size_t>(b) * prm.heads;  // query rows before them
  prm.batch = n;
  prm.q_lat += rows * kDc;
  prm.q_pe += rows * kDr;
  prm.out = reinterpret_cast<float*>(d.out + rows * kDc);
  if (prm.lse != nullptr) prm.lse += rows;
  prm.table += static_cast<size_t>(b) * prm.max_blocks;
  prm.seq_lens += b;
  prm.parents += static_cast<size_t>(b) * prm.q_tokens;
  if (prm.tree_lens != nullptr) prm.tree_lens += b;
  if (prm.prot != nullptr) {
    prm.prot += static_cast<size_t>(b) * kProtRows * (kDqk * 2);
    prm.draft_rows += static_cast<size_t>(b) * kMaxNodes * (kDqk * 2);
  }
  prm.images = images;
  prm.img_width = blocks;
  if (rest) prm.rest_images = images + static_cast<size_t>(n) * blocks * kImage;
  prm.n_hg = (prm.heads + 127) / 128;
  prm.n_img = 2 * prm.n_hg;
  prm.grid = prm.sms / 2;
  if (n * image_bytes(blocks, rest) > (96u << 20) && keep_step(prm.grid, prm.n_hg)) {
    prm.by_group = true;
    prm.grid = prm.grid / prm.n_hg * prm.n_hg;
  }
  switch (d.cache_kind) {
    case 4: return launch_impl<4, 64, false, true>(prm, stream, nullptr, nullptr);
    case 2: return launch_impl<2, 64, false, true>(prm, stream, nullptr, nullptr);
    case kC4R4: return launch_impl<kC4R4, 64, false, true>(prm, stream, nullptr, nullptr);
    default: return launch_impl<16, 64, false, true>(prm, stream, nullptr, nullptr);
  }
}

}  // namespace

size_t tree_workspace_bytes(int batch, int rows, int max_tokens, int grid) {
  return tree_workspace_layout(batch, rows, grid).images_off + batch * image_bytes(image_blocks(max_tokens), true);
}

cudaError_t launch_decode_tree(const qmla_tree_desc& d, int grid, cudaStream_t stream) {
  const int rows = d.nodes * d.heads, hg = head_group_size(rows);
  const TreeWorkspace w = tree_workspace_layout(d.batch, rows, grid);
  uint8_t* ws = static_cast<uint8_t*>(d.workspace);
  Params prm{};
  prm.pool = static_cast<const uint8_t*>(d.pool);
  prm.prot = static_cast<const uint8_t*>(d.prot);
  prm.num_blocks = d.num_blocks;
  prm.q_lat = reinterpret_cast<const __nv_bfloat16*>(d.q_latent);
  prm.q_pe = reinterpret_cast<const __nv_bfloat16*>(d.q_pe);
  prm.batch = d.batch;
  prm.heads = rows;
  prm.n_img = prm.n_hg = (rows + hg - 1) / hg;
  prm.grid = prm.sms = grid;
  prm.q_tokens = d.nodes;
  prm.hpt = d.heads;
  prm.table = d.block_table;
  prm.max_blocks = d.max_blocks;
  prm.seq_lens = d.seq_lens;
  prm.scale_log2 = d.softmax_scale * 1.4426950408889634f;
  prm.out = reinterpret_cast<float*>(d.out);  // (bf16)
  prm.lse = d.lse;
  prm.prefix = reinterpret_cast<const int32_t*>(ws + w.decode.prefix_off);
  prm.prefix_w = reinterpret_cast<int32_t*>(ws + w.decode.prefix_off);
  prm.cta_info = reinterpret_cast<int4*>(ws + w.decode.cta_off);
  prm.cta_first = prm.cta_info + grid;
  prm.cta_t0 = reinterpret_cast<int32_t*>(prm.cta_first + grid);
  prm.part_o = reinterpret_cast<float*>(ws + w.decode.part_o_off);
  prm.part_ml = reinterpret_cast<float*>(ws + w.decode.part_ml_off);
  prm.qimg = ws + w.decode.qimg_off;
  prm.dev_err = d.dev_err;
  prm.parents = d.parents;
  prm.tree_lens = d.tree_lens;
  prm.draft_rows = reinterpret_cast<const uint8_t*>(d.draft_rows);
  prm.trees = reinterpret_cast<TreeSeq*>(ws + w.trees_off);
  prm.max_tokens = d.max_blocks * kBlockTokens;
  if (d.max_len > 0) prm.max_tokens = std::min(prm.max_tokens, d.max_len);
  const int blocks = image_blocks(prm.max_tokens);
  // lse needs the scores of the values before their rounding to fp16, of which BF16 ones have none
  // (but the very small, and those beyond 65,504, which are infinite).
  const bool rest = d.lse != nullptr && d.cache_kind != QMLA_CACHE_BF16;
  const size_t room = d.workspace_bytes > w.images_off ? d.workspace_bytes - w.images_off : 0;
  int fit = static_cast<int>(std::min<size_t>(d.batch, blocks > 0 ? room / image_bytes(blocks, rest) : 0));
  if (fit > 0 && on_images(rows, static_cast<long long>(d.batch) * blocks * kBlockTokens, rest)) {
    // As many sequences at a time as there is room for; and as L2 holds, where many row groups that
    // do not keep step read their images (16 x 4,096 tokens, 32 groups, both passes: 714 us at once, 630
    // by 80 MB, 598 by 60, 588 by 40; 2 x 30,000 435 and 398; 57 MB by 40 instead of at once 100 and 116;
    // between 57 and 151 MB nothing was measured).
    // Not over six launches for that: the lengths may be far below their bound.
    const int groups = (rows + 127) / 128;
    if (groups >= 8 && !keep_step(grid / 2, groups) && d.batch * image_bytes(blocks, rest) > (112u << 20))
      fit = std::min(fit, std::max((d.batch + 5) / 6, static_cast<int>((56u << 20) / image_bytes(blocks, rest))));
    const int parts = (d.batch + fit - 1) / fit, per = (d.batch + parts - 1) / parts;
    for (int b = 0; b < d.batch; b += per) {
      const cudaError_t e = launch_images(d, prm, ws + w.images_off, b, std::min(per, d.batch - b), blocks, rest, stream);
      if (e != cudaSuccess) return e;
    }
    return cudaSuccess;
  }
  const bool prot = prm.prot != nullptr;
  switch (d.cache_kind) {
    case 4: return prot ? launch_rows<4, true>(hg, prm, stream) : launch_rows<4, false>(hg, prm, stream);
    case 2: return prot ? launch_rows<2, true>(hg, prm, stream) : launch_rows<2, false>(hg, prm, stream);
    case kC4R4: return prot ? launch_rows<kC4R4, true>(hg, prm, stream) : launch_rows<kC4R4, false>(hg, prm, stream);
    default: return launch_rows<16, false>(hg, prm, stream);
  }
}

}  // namespace qmla
