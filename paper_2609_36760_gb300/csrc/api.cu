// Host side of the C ABI declared in include/qmla.h: argument validation,
// device checks and kernel launches. Nothing here allocates device memory.
#include <cuda_runtime.h>

#include <cstdint>

#include "common.cuh"
#include "kernels.h"
#include "qmla.h"

namespace {

thread_local int g_last_cuda_error = 0;

// (The runtime keeps the error until it is read: the next launch that looks for one of its
// own would report it again.)
int cuda_fail(cudaError_t e) {
  g_last_cuda_error = static_cast<int>(e);
  (void)cudaGetLastError();
  return QMLA_ERR_CUDA;
}

bool aligned(const void* p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

// SM count and architecture of each device, looked up once.
struct DevInfo {
  int sms = -1;
  bool supported = false;
};
DevInfo g_dev[64];

int current_device_info(DevInfo& out) {
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return cuda_fail(e);
  if (dev < 0 || dev >= 64) return QMLA_ERR_UNSUPPORTED;
  if (g_dev[dev].sms < 0) {
    int major = 0, minor = 0, sms = 0;
    if ((e = cudaDeviceGetAttribute(&major, cudaDevAttrComputeCapabilityMajor, dev)) != cudaSuccess) return cuda_fail(e);
    if ((e = cudaDeviceGetAttribute(&minor, cudaDevAttrComputeCapabilityMinor, dev)) != cudaSuccess) return cuda_fail(e);
    if ((e = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev)) != cudaSuccess) return cuda_fail(e);
    g_dev[dev].supported = (major == 10 && minor == 3);
    g_dev[dev].sms = sms;
  }
  out = g_dev[dev];
  return out.supported ? QMLA_OK : QMLA_ERR_UNSUPPORTED;
}

bool known_cache(int kind) { return kind == 4 || kind == 2 || kind == QMLA_CACHE_C4R4 || kind == QMLA_CACHE_BF16; }

// The protection buffer and the rows of a tree's nodes come together.
bool bad_node_rows(int kind, const void* prot, const void* draft_rows) {
  return (prot == nullptr) != (draft_rows == nullptr) || !aligned(prot, 16) || !aligned(draft_rows, 16) ||
         (prot != nullptr && kind == QMLA_CACHE_BF16);
}

int append_common_checks(const void* pool, int num_blocks, const uint16_t* latent, const uint16_t* k_pe,
                         const int32_t* positions, int n, const int32_t* table, int num_seqs,
                         int max_blocks) {
  if (n < 0 || num_blocks <= 0 || num_seqs <= 0 || max_blocks <= 0) return QMLA_ERR_INVALID_ARG;
  if (n == 0) return QMLA_OK;
  if (pool == nullptr || latent == nullptr || k_pe == nullptr || positions == nullptr || table == nullptr)
    return QMLA_ERR_INVALID_ARG;
  if (!aligned(pool, 32) || !aligned(latent, 4) || !aligned(k_pe, 4) || !aligned(positions, 4) ||
      !aligned(table, 4))
    return QMLA_ERR_INVALID_ARG;
  if (static_cast<long long>(max_blocks) * qmla::kBlockTokens > INT32_MAX) return QMLA_ERR_INVALID_ARG;
  return QMLA_OK;
}

// Host checks of a decode call (no device access). heads counts every query
// row of a sequence (q_tokens x heads per token).
int decode_checks(const void* pool, int num_blocks, const uint16_t* q_latent, const uint16_t* q_pe, int batch,
                  int heads, const int32_t* table, int max_blocks, const int32_t* seq_lens, float softmax_scale,
                  const float* out, const float* lse, const void* workspace, const void* prot, int q_tokens,
                  bool need_workspace = true) {
  if (pool == nullptr || q_latent == nullptr || q_pe == nullptr || table == nullptr || seq_lens == nullptr ||
      out == nullptr || (need_workspace && workspace == nullptr))
    return QMLA_ERR_INVALID_ARG;
  if (prot != nullptr && !aligned(prot, 16)) return QMLA_ERR_INVALID_ARG;
  if (q_tokens < 1 || q_tokens > QMLA_MAX_Q_TOKENS || heads % q_tokens != 0) return QMLA_ERR_INVALID_ARG;
  if (batch <= 0 || heads < 1 || heads / q_tokens > 128 || num_blocks <= 0 || max_blocks <= 0)
    return QMLA_ERR_INVALID_ARG;
  if (!(softmax_scale > 0.0f) || softmax_scale > 1e30f) return QMLA_ERR_INVALID_ARG;
  if (!aligned(pool, 32) || !aligned(q_latent, 16) || !aligned(q_pe, 16) || !aligned(table, 4) ||
      !aligned(seq_lens, 4) || !aligned(out, 16) || (lse != nullptr && !aligned(lse, 4)) ||
      (need_workspace && !aligned(workspace, 256)))
    return QMLA_ERR_INVALID_ARG;
  if (static_cast<long long>(max_blocks) * qmla::kBlockTokens > INT32_MAX) return QMLA_ERR_INVALID_ARG;
  return QMLA_OK;
}

int decode_common(const void* pool, int kind, int num_blocks, const uint16_t* q_latent, const uint16_t* q_pe,
                  int batch, int heads, const int32_t* table, int max_blocks, const int32_t* seq_lens,
                  float softmax_scale, float* out, float* lse, void* workspace, size_t workspace_bytes,
                  uint32_t* dev_err, qmla_stream_t stream, const void* prot = nullptr, int q_tokens = 1,
                  void* ev_before_main = nullptr, void* ev_after_main = nullptr, int max_len = 0) {
  int st = decode_checks(pool, num_blocks, q_latent, q_pe, batch, heads, table, max_blocks, seq_lens, softmax_scale,
                         out, lse, workspace, prot, q_tokens);
  if (st != QMLA_OK) return st;
  DevInfo di;
  st = current_device_info(di);
  if (st != QMLA_OK) return st;
  const qmla::DecodeWorkspace w = qmla::decode_workspace_layout(batch, heads, di.sms);
  if (workspace_bytes < w.total) return QMLA_ERR_WORKSPACE_TOO_SMALL;
  qmla::DecodeArgs a;
  a.pool = pool;
  a.cache_kind = kind;
  a.num_blocks = num_blocks;
  a.q_latent = q_latent;
  a.q_pe = q_pe;
  a.batch = batch;
  a.heads = heads;
  a.table = table;
  a.max_blocks = max_blocks;
  a.max_len = max_len;
  a.seq_lens = seq_lens;
  a.softmax_scale = softmax_scale;
  a.out = out;
  a.lse = lse;
  a.workspace = workspace;
  a.dev_err = dev_err;
  a.grid = di.sms;
  a.prot = prot;
  a.q_tokens = q_tokens;
  a.ev_before_main = static_cast<cudaEvent_t>(ev_before_main);
  a.ev_after_main = static_cast<cudaEvent_t>(ev_after_main);
  cudaError_t e = qmla::launch_decode(a, reinterpret_cast<cudaStream_t>(stream));
  return e == cudaSuccess ? QMLA_OK : cuda_fail(e);
}

// Descriptor-level checks of qmla_mla_decode_ex before the common ones.
int desc_checks(const qmla_decode_desc* d) {
  if (d == nullptr) return QMLA_ERR_INVALID_ARG;
  const int kind = d->cache_kind;
  if (kind != 4 && kind != 2 && kind != QMLA_CACHE_C4R4 && kind != QMLA_CACHE_BF16) return QMLA_ERR_INVALID_ARG;
  if (kind == QMLA_CACHE_BF16 && (d->prot != nullptr || d->q_tokens != 1)) return QMLA_ERR_INVALID_ARG;
  if (kind == QMLA_CACHE_C4R4 && d->q_tokens != 1) return QMLA_ERR_INVALID_ARG;
  if (d->q_tokens < 1 || d->q_tokens > QMLA_MAX_Q_TOKENS || d->heads < 1 || d->heads > 128)
    return QMLA_ERR_INVALID_ARG;
  return QMLA_OK;
}

}  // namespace

namespace qmla {
void record_cuda_error(int err) { cuda_fail(static_cast<cudaError_t>(err)); }

int check_decode_desc(const qmla_decode_desc* d, bool check_workspace) {
  int st = desc_checks(d);
  if (st != QMLA_OK) return st;
  return decode_checks(d->pool, d->num_blocks, d->q_latent, d->q_pe, d->batch, d->q_tokens * d->heads,
                       d->block_table, d->max_blocks, d->seq_lens, d->softmax_scale, d->out, d->lse, d->workspace,
                       d->prot, d->q_tokens, check_workspace);
}
}  // namespace qmla

extern "C" {

size_t qmla_block_bytes(int c_bits) {
  if (c_bits == 4) return qmla::BlockLayout<4>::kBytes;
  if (c_bits == 2) return qmla::BlockLayout<2>::kBytes;
  return 0;
}

size_t qmla_bf16_block_bytes(void) { return qmla::kBf16BlockBytes; }

int qmla_quant_append(void* pool_dev, int c_bits, int num_blocks, const uint16_t* latent_dev,
                      const uint16_t* k_pe_dev, const int32_t* seq_ids_dev, const int32_t* positions_dev,
                      int n, const int32_t* block_table_dev, int num_seqs, int max_blocks,
                      uint32_t* dev_err_dev, qmla_stream_t stream) {
  if (c_bits != 4 && c_bits != 2) return QMLA_ERR_INVALID_ARG;
  int st = append_common_checks(pool_dev, num_blocks, latent_dev, k_pe_dev, positions_dev, n, block_table_dev,
                                num_seqs, max_blocks);
  if (st != QMLA_OK || n == 0) return st;
  DevInfo di;
  if ((st = current_device_info(di)) != QMLA_OK) return st;
  cudaError_t e = qmla::launch_quant_append(pool_dev, c_bits, num_blocks, latent_dev, k_pe_dev, seq_ids_dev,
                                            positions_dev, n, block_table_dev, num_seqs, max_blocks,
                                            dev_err_dev, reinterpret_cast<cudaStream_t>(stream));
  return e == cudaSuccess ? QMLA_OK : cuda_fail(e);
}

size_t qmla_protect_bytes_per_seq(void) { return static_cast<size_t>(qmla::kProtRows) * qmla::kDqk * 2; }

int qmla_quant_append_protected(void* pool_dev, int c_bits, int num_blocks, const uint16_t* latent_dev,
                                const uint16_t* k_pe_dev, const int32_t* seq_ids_dev,
                                const int32_t* positions_dev, int n, const int32_t* block_table_dev,
                                int num_seqs, int max_blocks, const int32_t* seq_lens_dev, void* prot_dev,
                                uint32_t* dev_err_dev, qmla_stream_t stream) {
  if (c_bits != 4 && c_bits != 2) return QMLA_ERR_INVALID_ARG;
  int st = append_common_checks(pool_dev, num_blocks, latent_dev, k_pe_dev, positions_dev, n, block_table_dev,
                                num_seqs, max_blocks);
  if (st != QMLA_OK) return st;
  if (prot_dev == nullptr || seq_lens_dev == nullptr || !aligned(prot_dev, 16) || !aligned(seq_lens_dev, 4) ||
      !aligned(latent_dev, 16) || !aligned(k_pe_dev, 16))
    return QMLA_ERR_INVALID_ARG;
  if (n == 0) return QMLA_OK;
  DevInfo di;
  if ((st = current_device_info(di)) != QMLA_OK) return st;
  cudaError_t e = qmla::launch_quant_append(pool_dev, c_bits, num_blocks, latent_dev, k_pe_dev, seq_ids_dev,
                                            positions_dev, n, block_table_dev, num_seqs, max_blocks,
                                            dev_err_dev, reinterpret_cast<cudaStream_t>(stream), prot_dev,
                                            seq_lens_dev);
  return e == cudaSuccess ? QMLA_OK : cuda_fail(e);
}

int qmla_bf16_append(void* pool_dev, int num_blocks, const uint16_t* latent_dev, const uint16_t* k_pe_dev,
                     const int32_t* seq_ids_dev, const int32_t* positions_dev, int n,
                     const int32_t* block_table_dev, int num_seqs, int max_blocks, uint32_t* dev_err_dev,
                     qmla_stream_t stream) {
  int st = append_common_checks(pool_dev, num_blocks, latent_dev, k_pe_dev, positions_dev, n, block_table_dev,
                                num_seqs, max_blocks);
  if (st != QMLA_OK || n == 0) return st;
  DevInfo di;
  if ((st = current_device_info(di)) != QMLA_OK) return st;
  cudaError_t e = qmla::launch_bf16_append(pool_dev, num_blocks, latent_dev, k_pe_dev, seq_ids_dev, positions_dev,
                                           n, block_table_dev, num_seqs, max_blocks, dev_err_dev,
                                           reinterpret_cast<cudaStream_t>(stream));
  return e == cudaSuccess ? QMLA_OK : cuda_fail(e);
}

size_t qmla_decode_workspace_bytes(int batch, int heads) {
  if (batch <= 0 || heads < 1 || heads > 128 * QMLA_MAX_Q_TOKENS) return 0;
  DevInfo di;
  if (current_device_info(di) != QMLA_OK) return 0;
  return qmla::decode_workspace_layout(batch, heads, di.sms).total;
}

int qmla_mla_decode(const void* pool_dev, int c_bits, int num_blocks, const uint16_t* q_latent_dev,
                    const uint16_t* q_pe_dev, int batch, int heads, const int32_t* block_table_dev, int max_blocks,
                    const int32_t* seq_lens_dev, float softmax_scale, float* out_dev, float* lse_dev,
                    void* workspace_dev, size_t workspace_bytes, uint32_t* dev_err_dev, qmla_stream_t stream) {
  if (c_bits != 4 && c_bits != 2) return QMLA_ERR_INVALID_ARG;
  return decode_common(pool_dev, c_bits, num_blocks, q_latent_dev, q_pe_dev, batch, heads, block_table_dev,
                       max_blocks, seq_lens_dev, softmax_scale, out_dev, lse_dev, workspace_dev, workspace_bytes,
                       dev_err_dev, stream);
}

int qmla_mla_decode_protected(const void* pool_dev, int c_bits, int num_blocks, const uint16_t* q_latent_dev,
                              const uint16_t* q_pe_dev, int batch, int heads, const int32_t* block_table_dev,
                              int max_blocks, const int32_t* seq_lens_dev, const void* prot_dev,
                              float softmax_scale, float* out_dev, float* lse_dev, void* workspace_dev,
                              size_t workspace_bytes, uint32_t* dev_err_dev, qmla_stream_t stream) {
  if (c_bits != 4 && c_bits != 2) return QMLA_ERR_INVALID_ARG;
  if (prot_dev == nullptr) return QMLA_ERR_INVALID_ARG;
  return decode_common(pool_dev, c_bits, num_blocks, q_latent_dev, q_pe_dev, batch, heads, block_table_dev,
                       max_blocks, seq_lens_dev, softmax_scale, out_dev, lse_dev, workspace_dev, workspace_bytes,
                       dev_err_dev, stream, prot_dev);
}

size_t qmla_c4r4_page_bytes(void) { return qmla::BlockLayout<qmla::kC4R4>::kBytes; }

int qmla_quant_append_c4r4(void* pool_dev, int num_blocks, const uint16_t* latent_dev, const uint16_t* k_pe_dev,
                           const int32_t* seq_ids_dev, const int32_t* positions_dev, int n,
                           const int32_t* block_table_dev, int num_seqs, int max_blocks,
                           const int32_t* seq_lens_dev, void* prot_dev, uint32_t* dev_err_dev,
                           qmla_stream_t stream) {
  int st = append_common_checks(pool_dev, num_blocks, latent_dev, k_pe_dev, positions_dev, n, block_table_dev,
                                num_seqs, max_blocks);
  if (st != QMLA_OK) return st;
  if (prot_dev != nullptr &&
      (seq_lens_dev == nullptr || !aligned(prot_dev, 16) || !aligned(seq_lens_dev, 4) ||
       !aligned(latent_dev, 16) || !aligned(k_pe_dev, 16)))
    return QMLA_ERR_INVALID_ARG;
  if (n == 0) return QMLA_OK;
  DevInfo di;
  if ((st = current_device_info(di)) != QMLA_OK) return st;
  cudaError_t e = qmla::launch_quant_append(pool_dev, qmla::kC4R4, num_blocks, latent_dev, k_pe_dev, seq_ids_dev,
                                            positions_dev, n, block_table_dev, num_seqs, max_blocks,
                                            dev_err_dev, reinterpret_cast<cudaStream_t>(stream), prot_dev,
                                            prot_dev != nullptr ? seq_lens_dev : nullptr);
  return e == cudaSuccess ? QMLA_OK : cuda_fail(e);
}

int qmla_mla_decode_c4r4(const void* pool_dev, int num_blocks, const uint16_t* q_latent_dev,
                         const uint16_t* q_pe_dev, int batch, int heads, const int32_t* block_table_dev,
                         int max_blocks, const int32_t* seq_lens_dev, const void* prot_dev, float softmax_scale,
                         float* out_dev, float* lse_dev, void* workspace_dev, size_t workspace_bytes,
                         uint32_t* dev_err_dev, qmla_stream_t stream) {
  return decode_common(pool_dev, qmla::kC4R4, num_blocks, q_latent_dev, q_pe_dev, batch, heads, block_table_dev,
                       max_blocks, seq_lens_dev, softmax_scale, out_dev, lse_dev, workspace_dev, workspace_bytes,
                       dev_err_dev, stream, prot_dev);
}

int qmla_mla_decode_multi(const void* pool_dev, int c_bits, int num_blocks, const uint16_t* q_latent_dev,
                          const uint16_t* q_pe_dev, int batch, int q_tokens, int heads,
                          const int32_t* block_table_dev, int max_blocks, const int32_t* seq_lens_dev,
                          const void* prot_dev, float softmax_scale, float* out_dev, float* lse_dev,
                          void* workspace_dev, size_t workspace_bytes, uint32_t* dev_err_dev, qmla_stream_t stream) {
  if (c_bits != 4 && c_bits != 2) return QMLA_ERR_INVALID_ARG;
  if (q_tokens < 1 || q_tokens > QMLA_MAX_Q_TOKENS || heads < 1 || heads > 128) return QMLA_ERR_INVALID_ARG;
  return decode_common(pool_dev, c_bits, num_blocks, q_latent_dev, q_pe_dev, batch, q_tokens * heads,
                       block_table_dev, max_blocks, seq_lens_dev, softmax_scale, out_dev, lse_dev, workspace_dev,
                       workspace_bytes, dev_err_dev, stream, prot_dev, q_tokens);
}

int qmla_mla_decode_bf16cache(const void* pool_dev, int num_blocks, const uint16_t* q_latent_dev,
                              const uint16_t* q_pe_dev, int batch, int heads, const int32_t* block_table_dev,
                              int max_blocks, const int32_t* seq_lens_dev, float softmax_scale, float* out_dev,
                              float* lse_dev, void* workspace_dev, size_t workspace_bytes, uint32_t* dev_err_dev,
                              qmla_stream_t stream) {
  return decode_common(pool_dev, 16, num_blocks, q_latent_dev, q_pe_dev, batch, heads, block_table_dev, max_blocks,
                       seq_lens_dev, softmax_scale, out_dev, lse_dev, workspace_dev, workspace_bytes, dev_err_dev,
                       stream);
}

int qmla_debug_tile(const void* pool_dev, int cache_kind, int num_blocks, const int32_t* block_table_dev,
                    int max_blocks, const int32_t* seq_lens_dev, int batch, int b, int j, const void* prot_dev,
                    uint16_t* tile_dev, uint32_t* dev_err_dev, qmla_stream_t stream) {
  static_assert(QMLA_CACHE_C4R4 == qmla::kC4R4, "kind code of the paper's page");
  if (cache_kind != 4 && cache_kind != 2 && cache_kind != QMLA_CACHE_C4R4 && cache_kind != QMLA_CACHE_BF16)
    return QMLA_ERR_INVALID_ARG;
  if (pool_dev == nullptr || block_table_dev == nullptr || seq_lens_dev == nullptr || tile_dev == nullptr)
    return QMLA_ERR_INVALID_ARG;
  if (num_blocks <= 0 || max_blocks <= 0 || batch <= 0 || b < 0 || b >= batch || j < 0 ||
      static_cast<long long>(j) * 2 >= max_blocks)
    return QMLA_ERR_INVALID_ARG;
  if (!aligned(pool_dev, 32) || !aligned(tile_dev, 16) || (prot_dev != nullptr && !aligned(prot_dev, 16)))
    return QMLA_ERR_INVALID_ARG;
  if (prot_dev != nullptr && cache_kind == QMLA_CACHE_BF16) return QMLA_ERR_INVALID_ARG;
  DevInfo di;
  int st = current_device_info(di);
  if (st != QMLA_OK) return st;
  qmla::DecodeArgs a;
  a.pool = pool_dev;
  a.cache_kind = cache_kind;
  a.num_blocks = num_blocks;
  a.batch = batch;
  a.table = block_table_dev;
  a.max_blocks = max_blocks;
  a.seq_lens = seq_lens_dev;
  a.dev_err = dev_err_dev;
  a.prot = prot_dev;
  cudaError_t e = qmla::launch_tile_dump(a, b, j, tile_dev, reinterpret_cast<cudaStream_t>(stream));
  return e == cudaSuccess ? QMLA_OK : cuda_fail(e);
}

int qmla_debug_decode_route(const qmla_decode_desc* d, int sms) {
  if (desc_checks(d) != QMLA_OK || d->batch < 1 || d->max_blocks < 1 || sms < 1) return -1;
  qmla::DecodeArgs a;
  a.cache_kind = d->cache_kind;
  a.batch = d->batch;
  a.heads = d->q_tokens * d->heads;
  a.max_blocks = d->max_blocks;
  a.max_len = d->max_len;
  a.prot = d->prot;
  a.grid = sms;
  return qmla::decode_on_pairs(a) ? 1 : 0;
}

int qmla_debug_wait_timeout(uint32_t limit_us, uint32_t* dev_err_dev, qmla_stream_t stream) {
  if (dev_err_dev == nullptr || limit_us < 1u || limit_us > 1000000u) return QMLA_ERR_INVALID_ARG;
  DevInfo di;
  int st = current_device_info(di);
  if (st != QMLA_OK) return st;
  cudaError_t e = qmla::launch_wait_timeout(dev_err_dev, static_cast<unsigned long long>(limit_us) * 1000ull,
                                            reinterpret_cast<cudaStream_t>(stream));
  return e == cudaSuccess ? QMLA_OK : cuda_fail(e);
}

int qmla_read_dev_err(const uint32_t* dev_err_dev, uint32_t* host_out, qmla_stream_t stream) {
  if (dev_err_dev == nullptr || host_out == nullptr) return QMLA_ERR_INVALID_ARG;
  cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  cudaError_t e = cudaMemcpyAsync(host_out, dev_err_dev, sizeof(uint32_t), cudaMemcpyDeviceToHost, s);
  if (e == cudaSuccess) e = cudaStreamSynchronize(s);
  return e == cudaSuccess ? QMLA_OK : cuda_fail(e);
}

int qmla_mla_decode_ex(const qmla_decode_desc* d, qmla_stream_t stream) {
  const int st = desc_checks(d);
  if (st != QMLA_OK) return st;
  return decode_common(d->pool, d->cache_kind, d->num_blocks, d->q_latent, d->q_pe, d->batch, d->q_tokens * d->heads,
                       d->block_table, d->max_blocks, d->seq_lens, d->softmax_scale, d->out, d->lse, d->workspace,
                       d->workspace_bytes, d->dev_err, stream, d->prot, d->q_tokens, d->ev_before_main,
                       d->ev_after_main, d->max_len);
}

int qmla_rope_append(const qmla_append_desc* desc, qmla_stream_t stream) {
  return qmla_rope_append_at(desc, nullptr, stream);
}

int qmla_rope_append_at(const qmla_append_desc* desc, const int32_t* rope_positions_dev, qmla_stream_t stream) {
  if (desc == nullptr || !known_cache(desc->cache_kind)) return QMLA_ERR_INVALID_ARG;
  qmla_append_desc own = *desc;  // (a single row's strides are not used)
  if (own.n == 1) own.latent_stride = qmla::kDc, own.k_pe_stride = qmla::kDr;
  const qmla_append_desc* d = &own;
  int st = append_common_checks(d->pool, d->num_blocks, d->latent, d->k_pe, d->positions, d->n, d->block_table,
                                d->num_seqs, d->max_blocks);
  if (st != QMLA_OK) return st;
  if (d->rope_len < 1 || (d->interleaved != 0 && d->interleaved != 1)) return QMLA_ERR_INVALID_ARG;
  if (d->norm != 0 && (!(d->norm_eps >= 0.0f) || d->norm_eps > 1e30f || !aligned(d->norm_weight, 16)))
    return QMLA_ERR_INVALID_ARG;
  if (d->prot != nullptr && (d->cache_kind == QMLA_CACHE_BF16 || d->seq_lens == nullptr || !aligned(d->prot, 16) ||
                             !aligned(d->seq_lens, 4)))
    return QMLA_ERR_INVALID_ARG;
  if (d->n == 0) return QMLA_OK;
  if (d->cos_sin == nullptr || !aligned(d->cos_sin, 16) || !aligned(d->seq_ids, 4) || !aligned(rope_positions_dev, 4))
    return QMLA_ERR_INVALID_ARG;
  if (d->latent_stride % 2 != 0 || d->k_pe_stride % 2 != 0 || (d->n > 1 && (d->latent_stride < qmla::kDc || d->k_pe_stride < qmla::kDr)))
    return QMLA_ERR_INVALID_ARG;
  DevInfo di;
  if ((st = current_device_info(di)) != QMLA_OK) return st;
  cudaError_t e = qmla::launch_rope_append(*d, rope_positions_dev, reinterpret_cast<cudaStream_t>(stream));
  return e == cudaSuccess ? QMLA_OK : cuda_fail(e);
}

int qmla_rope_query(const uint16_t* q_pe_dev, long long q_token_stride, long long q_head_stride,
                    const int32_t* positions_dev, int n, int heads, const float* cos_sin_dev, int rope_len,
                    int interleaved, uint16_t* out_dev, long long out_token_stride, long long out_head_stride,
                    uint32_t* dev_err_dev, qmla_stream_t stream) {
  // (a block takes 64 rows, a grid has 2^31 - 1 blocks)
  if (n < 0 || heads < 1 || heads > (1 << 24) || static_cast<long long>(n) * heads > (1ll << 36) || rope_len < 1 ||
      (interleaved != 0 && interleaved != 1))
    return QMLA_ERR_INVALID_ARG;
  if (n == 0) return QMLA_OK;
  if (q_pe_dev == nullptr || positions_dev == nullptr || cos_sin_dev == nullptr || out_dev == nullptr)
    return QMLA_ERR_INVALID_ARG;
  if (!aligned(q_pe_dev, 16) || !aligned(out_dev, 16) || !aligned(cos_sin_dev, 16) || !aligned(positions_dev, 4))
    return QMLA_ERR_INVALID_ARG;
  if (n == 1) q_token_stride = out_token_stride = qmla::kDr;  // (not used)
  if (heads == 1) q_head_stride = out_head_stride = qmla::kDr;
  for (long long s : {q_token_stride, q_head_stride, out_token_stride, out_head_stride})
    if (s < 0 || s % 8 != 0 || s >= (1ll << 38)) return QMLA_ERR_INVALID_ARG;
  // Rows of out that overlap would race: one axis has to step over all of the other.
  const long long in_token = heads > 1 ? (heads - 1) * out_head_stride + qmla::kDr : qmla::kDr;
  if (out_token_stride > (1ll << 56) / n) return QMLA_ERR_INVALID_ARG;  // (more than there are addresses)
  const long long in_head = n > 1 ? (n - 1) * out_token_stride + qmla::kDr : qmla::kDr;
  if ((n > 1 && out_token_stride < qmla::kDr) || (heads > 1 && out_head_stride < qmla::kDr) ||
      (n > 1 && heads > 1 && out_token_stride < in_token && out_head_stride < in_head))
    return QMLA_ERR_INVALID_ARG;
  DevInfo di;
  int st = current_device_info(di);
  if (st != QMLA_OK) return st;
  cudaError_t e = qmla::launch_rope_query(q_pe_dev, q_token_stride, q_head_stride, positions_dev, n, heads, cos_sin_dev,
                                          rope_len, interleaved != 0, out_dev, out_token_stride, out_head_stride,
                                          dev_err_dev, reinterpret_cast<cudaStream_t>(stream));
  return e == cudaSuccess ? QMLA_OK : cuda_fail(e);
}

int qmla_cache_read(const qmla_read_desc* d, qmla_stream_t stream) {
  if (d == nullptr || !known_cache(d->cache_kind)) return QMLA_ERR_INVALID_ARG;
  if (d->n < 0 || d->num_blocks <= 0 || d->num_seqs <= 0 || d->max_blocks <= 0 ||
      static_cast<long long>(d->max_blocks) * qmla::kBlockTokens > INT32_MAX)
    return QMLA_ERR_INVALID_ARG;
  if (d->prot != nullptr && (d->cache_kind == QMLA_CACHE_BF16 || d->seq_lens == nullptr || !aligned(d->prot, 16) ||
                             !aligned(d->seq_lens, 4)))
    return QMLA_ERR_INVALID_ARG;
  if (d->n == 0) return QMLA_OK;
  if (d->pool == nullptr || d->positions == nullptr || d->block_table == nullptr || d->rows == nullptr)
    return QMLA_ERR_INVALID_ARG;
  if (!aligned(d->pool, 32) || !aligned(d->rows, 16) || !aligned(d->seq_ids, 4) || !aligned(d->positions, 4) ||
      !aligned(d->block_table, 4) || (d->n > 1 && (d->row_stride % 8 != 0 || d->row_stride < qmla::kDqk)))
    return QMLA_ERR_INVALID_ARG;
  DevInfo di;
  int st = current_device_info(di);
  if (st != QMLA_OK) return st;
  cudaError_t e = qmla::launch_cache_read(*d, reinterpret_cast<cudaStream_t>(stream));
  return e == cudaSuccess ? QMLA_OK : cuda_fail(e);
}

size_t qmla_prefill_workspace_bytes(int batch, int n_q) {
  if (batch < 1 || batch > 65536 || n_q < 0 || n_q > (1 << 26)) return 0;
  return qmla::prefill_workspace_bytes(batch, n_q);
}

int qmla_mla_prefill(const qmla_prefill_desc* d, qmla_stream_t stream) {
  if (d == nullptr) return QMLA_ERR_INVALID_ARG;
  if (d->n_q < 0 || d->n_kv < 0 || d->n_q > (1 << 26) || d->n_kv > (1 << 26) || d->heads < 1 || d->heads > 1024 ||
      d->batch < 1 || d->batch > 65536 || (d->causal != 0 && d->causal != 1))
    return QMLA_ERR_INVALID_ARG;
  if (!(d->softmax_scale > 0.0f) || d->softmax_scale > 1e30f) return QMLA_ERR_INVALID_ARG;
  if (d->n_q == 0) return QMLA_OK;
  if (d->q == nullptr || d->cu_q == nullptr || d->cu_kv == nullptr || d->out == nullptr || d->workspace == nullptr ||
      (d->n_kv > 0 && (d->k == nullptr || d->v == nullptr || d->k_pe == nullptr)))
    return QMLA_ERR_INVALID_ARG;
  if (!aligned(d->q, 16) || !aligned(d->out, 32) || !aligned(d->cu_q, 4) || !aligned(d->cu_kv, 4) ||
      !aligned(d->lse, 4) || !aligned(d->workspace, 256) ||
      (d->n_kv > 0 && (!aligned(d->k, 16) || !aligned(d->v, 16) || !aligned(d->k_pe, 16))))
    return QMLA_ERR_INVALID_ARG;
  auto bad = [](int n, long long s) { return n > 1 && (s < 8 || s % 8 != 0 || s >= (1ll << 38)); };
  if (bad(d->n_q, d->q_token_stride) || bad(d->heads, d->q_head_stride) || bad(d->n_kv, d->k_token_stride) ||
      bad(d->n_kv, d->v_token_stride) || bad(d->n_kv, d->k_pe_stride) ||
      (d->n_kv > 0 && (bad(d->heads, d->k_head_stride) || bad(d->heads, d->v_head_stride))))
    return QMLA_ERR_INVALID_ARG;
  if (d->workspace_bytes < qmla::prefill_workspace_bytes(d->batch, d->n_q)) return QMLA_ERR_WORKSPACE_TOO_SMALL;
  DevInfo di;
  int st = current_device_info(di);
  if (st != QMLA_OK) return st;
  cudaError_t e = qmla::launch_prefill(*d, di.sms, reinterpret_cast<cudaStream_t>(stream));
  return e == cudaSuccess ? QMLA_OK : cuda_fail(e);
}

size_t qmla_tree_workspace_bytes(int batch, int nodes, int heads, int max_tokens) {
  if (batch <= 0 || max_tokens < 0 || nodes < 1 || nodes > QMLA_MAX_TREE_NODES || heads < 1 || heads > 128) return 0;
  DevInfo di;
  if (current_device_info(di) != QMLA_OK) return 0;
  return qmla::tree_workspace_bytes(batch, nodes * heads, max_tokens, di.sms);
}

int qmla_mla_decode_tree(const qmla_tree_desc* d, qmla_stream_t stream) {
  if (d == nullptr || !known_cache(d->cache_kind)) return QMLA_ERR_INVALID_ARG;
  if (d->batch <= 0 || d->nodes < 1 || d->nodes > QMLA_MAX_TREE_NODES || d->heads < 1 || d->heads > 128 ||
      d->num_blocks <= 0 || d->max_blocks <= 0 || d->max_len < 0 ||
      static_cast<long long>(d->max_blocks) * qmla::kBlockTokens > INT32_MAX)
    return QMLA_ERR_INVALID_ARG;
  if (!(d->softmax_scale > 0.0f) || d->softmax_scale > 1e30f) return QMLA_ERR_INVALID_ARG;
  if (d->pool == nullptr || d->q_latent == nullptr || d->q_pe == nullptr || d->parents == nullptr ||
      d->block_table == nullptr || d->seq_lens == nullptr || d->out == nullptr || d->workspace == nullptr)
    return QMLA_ERR_INVALID_ARG;
  if (!aligned(d->pool, 32) || !aligned(d->q_latent, 16) || !aligned(d->q_pe, 16) || !aligned(d->parents, 4) ||
      !aligned(d->tree_lens, 4) || !aligned(d->block_table, 4) || !aligned(d->seq_lens, 4) || !aligned(d->out, 32) ||
      !aligned(d->lse, 4) || !aligned(d->workspace, 256))
    return QMLA_ERR_INVALID_ARG;
  if (bad_node_rows(d->cache_kind, d->prot, d->draft_rows)) return QMLA_ERR_INVALID_ARG;
  // (the plan counts 128-token tiles of 64-row groups in 32 bits)
  const int groups = (d->nodes * d->heads + qmla::head_group_size(d->nodes * d->heads) - 1) / qmla::head_group_size(d->nodes * d->heads);
  if (static_cast<long long>(d->batch) * groups * ((d->max_blocks + 1ll) / 2) > INT32_MAX) return QMLA_ERR_INVALID_ARG;
  DevInfo di;
  int st = current_device_info(di);
  if (st != QMLA_OK) return st;
  if (d->workspace_bytes < qmla::tree_workspace_bytes(d->batch, d->nodes * d->heads, 0, di.sms))
    return QMLA_ERR_WORKSPACE_TOO_SMALL;
  cudaError_t e = qmla::launch_decode_tree(*d, di.sms, reinterpret_cast<cudaStream_t>(stream));
  return e == cudaSuccess ? QMLA_OK : cuda_fail(e);
}

int qmla_tree_verify(const qmla_verify_desc* desc, qmla_stream_t stream) {
  if (desc == nullptr || (desc->probs != QMLA_PROBS_F32 && desc->probs != QMLA_PROBS_BF16)) return QMLA_ERR_INVALID_ARG;
  if (desc->batch < 1 || desc->batch > 65535 || desc->nodes < 1 || desc->nodes > QMLA_MAX_TREE_NODES ||
      desc->vocab < 1 || desc->vocab > (1 << 24))
    return QMLA_ERR_INVALID_ARG;
  if (desc->target == nullptr || desc->tokens == nullptr || desc->parents == nullptr || desc->uniforms == nullptr ||
      desc->path == nullptr || desc->kept == nullptr || desc->next_token == nullptr)
    return QMLA_ERR_INVALID_ARG;
  const uintptr_t size = desc->probs == QMLA_PROBS_F32 ? 4 : 2;
  if (!aligned(desc->target, size) || !aligned(desc->draft, size) || !aligned(desc->tokens, 4) ||
      !aligned(desc->parents, 4) || !aligned(desc->tree_lens, 4) || !aligned(desc->uniforms, 4) ||
      !aligned(desc->path, 4) || !aligned(desc->kept, 4) || !aligned(desc->next_token, 4))
    return QMLA_ERR_INVALID_ARG;
  qmla_verify_desc d = *desc;  // (a single row's strides are not used)
  if (d.batch == 1) d.target_seq_stride = d.draft_seq_stride = 0;
  if (d.nodes == 1) d.target_row_stride = d.draft_row_stride = 0;
  if (d.draft == nullptr) d.draft_seq_stride = d.draft_row_stride = 0;
  for (long long s : {d.target_seq_stride, d.target_row_stride, d.draft_seq_stride, d.draft_row_stride})
    if (s < 0 || s >= (1ll << 40)) return QMLA_ERR_INVALID_ARG;
  DevInfo di;
  int st = current_device_info(di);
  if (st != QMLA_OK) return st;
  cudaError_t e = qmla::launch_tree_verify(d, di.sms, reinterpret_cast<cudaStream_t>(stream));
  return e == cudaSuccess ? QMLA_OK : cuda_fail(e);
}

int qmla_cache_keep(const qmla_keep_desc* d, qmla_stream_t stream) {
  if (d == nullptr || !known_cache(d->cache_kind)) return QMLA_ERR_INVALID_ARG;
  if (d->batch <= 0 || d->nodes < 1 || d->nodes > QMLA_MAX_TREE_NODES || d->num_blocks <= 0 || d->max_blocks <= 0 ||
      static_cast<long long>(d->max_blocks) * qmla::kBlockTokens > INT32_MAX)
    return QMLA_ERR_INVALID_ARG;
  if (d->pool == nullptr || d->block_table == nullptr || d->seq_lens == nullptr || d->path == nullptr ||
      d->kept == nullptr || d->new_lens == nullptr)
    return QMLA_ERR_INVALID_ARG;
  if (!aligned(d->pool, 32) || !aligned(d->block_table, 4) || !aligned(d->seq_lens, 4) || !aligned(d->tree_lens, 4) ||
      !aligned(d->path, 4) || !aligned(d->kept, 4) || !aligned(d->new_lens, 4))
    return QMLA_ERR_INVALID_ARG;
  if (bad_node_rows(d->cache_kind, d->prot, d->draft_rows)) return QMLA_ERR_INVALID_ARG;
  DevInfo di;
  int st = current_device_info(di);
  if (st != QMLA_OK) return st;
  cudaError_t e = qmla::launch_cache_keep(*d, reinterpret_cast<cudaStream_t>(stream));
  return e == cudaSuccess ? QMLA_OK : cuda_fail(e);
}

int qmla_last_cuda_error(void) { return g_last_cuda_error; }

#ifdef QMLA_TRACE_BUILD
// Trace builds only (libqmla_trace.so): device buffer that receives the
// decode kernel's per-CTA event timeline; NULL disables.
int qmla_trace_set(void* buf_dev) {
  cudaError_t e = qmla::set_trace_buffer(buf_dev);
  return e == cudaSuccess ? QMLA_OK : cuda_fail(e);
}
#endif

const char* qmla_status_string(int status) {
  switch (status) {
    case QMLA_OK: return "ok";
    case QMLA_ERR_INVALID_ARG: return "invalid argument";
    case QMLA_ERR_UNSUPPORTED: return "unsupported device or shape";
    case QMLA_ERR_WORKSPACE_TOO_SMALL: return "workspace too small";
    case QMLA_ERR_CUDA: return "CUDA error";
    default: return "unknown status";
  }
}

int qmla_num_sms(void) {
  DevInfo di;
  if (current_device_info(di) != QMLA_OK) return -1;
  return di.sms;
}

}  // extern "C"
