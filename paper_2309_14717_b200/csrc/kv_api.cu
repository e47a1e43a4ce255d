// C-ABI entry points of the key/value cache: argument checks and scratch layout.
#define QALORA_TU 13
#include "kv.cuh"

namespace qalora {

int check_kv_desc(const qalora_kv_desc* d, KvShape* sh) {
  if (d == nullptr) return QALORA_ERR_NULL_POINTER;
  if (d->heads <= 0 || d->kv_heads <= 0 || d->head_dim <= 0 || d->block_tokens <= 0 || d->num_blocks <= 0)
    return QALORA_ERR_INVALID_ARG;
  if (d->heads % d->kv_heads != 0 || d->heads > 1024) return QALORA_ERR_UNSUPPORTED_SHAPE;
  if (d->head_dim != 64 && d->head_dim != 128) return QALORA_ERR_UNSUPPORTED_SHAPE;
  if (d->block_tokens != 16 && d->block_tokens != 32 && d->block_tokens != 64 && d->block_tokens != 128)
    return QALORA_ERR_UNSUPPORTED_SHAPE;
  if ((long long)d->num_blocks * 2 * d->kv_heads > 0x7fffffffll / d->block_tokens) return QALORA_ERR_UNSUPPORTED_SHAPE;
  sh->heads = d->heads; sh->kv_heads = d->kv_heads; sh->group = d->heads / d->kv_heads;
  sh->dim = d->head_dim; sh->block = d->block_tokens; sh->log_block = d->block_tokens == 16 ? 4 : d->block_tokens == 32 ? 5 : d->block_tokens == 64 ? 6 : 7;
  sh->num_blocks = d->num_blocks;
  return QALORA_OK;
}

namespace {

bool aligned4(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }
bool stride_ok(int64_t stride, int64_t row) { return stride >= row && stride % 8 == 0 && stride <= (int64_t)1 << 40; }

// The sizes of a batch; what is empty needs no pointers.
int check_batch(int32_t batch, int64_t m, int32_t max_new, int32_t max_blocks) {
  if (batch < 0 || batch > 65535 || m < 0 || m > QALORA_MAX_ROWS || max_new < 0 || max_new > m) return QALORA_ERR_INVALID_ARG;
  if (max_blocks < 0) return QALORA_ERR_INVALID_ARG;
  return QALORA_OK;
}

KvBatch make_batch(const KvShape& sh, const int32_t* starts, const int32_t* lens, const int32_t* table, int32_t batch,
                   int32_t max_blocks, int64_t m, int32_t max_new, int64_t max_len) {
  // (the kernels' positions, a step of a loop behind the last one included, stay below 2^31)
  const int64_t capacity = (int64_t)max_blocks * sh.block, most = capacity < 0x7fff0000 ? capacity : 0x7fff0000;
  KvBatch b{};
  b.starts = starts; b.lens = lens; b.table = table;
  b.batch = batch; b.max_blocks = max_blocks;
  b.m = (int)m; b.max_new = max_new;
  b.max_len = (int)(max_len < most ? max_len : most);
  b.n_lo = 0;
  b.n_hi = max_new;
  return b;
}

}  // namespace
}  // namespace qalora

using namespace qalora;

extern "C" {

int qalora_kv_cache_bytes(const qalora_kv_desc* desc, size_t* code_bytes, size_t* scale_bytes, size_t* score_bytes) {
  KvShape sh;
  const int st = check_kv_desc(desc, &sh);
  if (st != QALORA_OK) return st;
  if (code_bytes == nullptr || scale_bytes == nullptr || score_bytes == nullptr) return QALORA_ERR_NULL_POINTER;
  const size_t planes = (size_t)sh.num_blocks * sh.kv_heads;
  *code_bytes = planes * 2 * sh.block * sh.dim;
  *scale_bytes = planes * 2 * sizeof(float);
  *score_bytes = planes * sh.block * sizeof(float);
  return QALORA_OK;
}

int qalora_kv_append(const qalora_kv_desc* desc, int32_t batch, int64_t m, int32_t max_new,
                     const int32_t* starts, const int32_t* lens, const int32_t* table, int32_t max_blocks,
                     const void* k, int64_t k_stride, const void* v, int64_t v_stride,
                     void* codes, float* scales, float* score, int32_t* dev_status, void* cuda_stream) {
  KvShape sh;
  int st = check_kv_desc(desc, &sh);
  if (st == QALORA_OK) st = check_batch(batch, m, max_new, max_blocks);
  if (st != QALORA_OK) return st;
  const int64_t row = (int64_t)sh.kv_heads * sh.dim;
  if (!stride_ok(k_stride, row) || !stride_ok(v_stride, row)) return QALORA_ERR_INVALID_ARG;
  if (batch == 0 || m == 0 || max_new == 0 || max_blocks == 0) return QALORA_OK;
  if (starts == nullptr || lens == nullptr || table == nullptr || k == nullptr || v == nullptr || codes == nullptr || scales == nullptr)
    return QALORA_ERR_NULL_POINTER;
  if (!aligned4(starts) || !aligned4(lens) || !aligned4(table) || !aligned4(dev_status) || !aligned16(k) || !aligned16(v) ||
      !aligned16(codes) || !aligned16(scales) || !aligned16(score))
    return QALORA_ERR_MISALIGNED;
  return launch_kv_append(sh, make_batch(sh, starts, lens, table, batch, max_blocks, m, max_new, INT64_MAX),
                          static_cast<const __nv_bfloat16*>(k), k_stride, static_cast<const __nv_bfloat16*>(v), v_stride,
                          static_cast<int8_t*>(codes), scales, score, dev_status, static_cast<cudaStream_t>(cuda_stream));
}

int qalora_kv_read(const qalora_kv_desc* desc, int32_t batch, int64_t m, int32_t max_new,
                   const int32_t* starts, const int32_t* first, const int32_t* table, int32_t max_blocks,
                   const void* codes, const float* scales, void* k, void* v, int out_bf16, void* cuda_stream) {
  KvShape sh;
  int st = check_kv_desc(desc, &sh);
  if (st == QALORA_OK) st = check_batch(batch, m, max_new, max_blocks);
  if (st != QALORA_OK) return st;
  if (batch == 0 || m == 0 || max_new == 0 || max_blocks == 0 || (k == nullptr && v == nullptr)) return QALORA_OK;
  if (starts == nullptr || first == nullptr || table == nullptr || codes == nullptr || scales == nullptr)
    return QALORA_ERR_NULL_POINTER;
  if (!aligned4(starts) || !aligned4(first) || !aligned4(table) || !aligned16(codes) || !aligned16(scales) || !aligned16(k) ||
      !aligned16(v))
    return QALORA_ERR_MISALIGNED;
  return launch_kv_read(sh, make_batch(sh, starts, first, table, batch, max_blocks, m, max_new, INT64_MAX),
                        static_cast<const int8_t*>(codes), scales, k, v, out_bf16 != 0, static_cast<cudaStream_t>(cuda_stream));
}

int qalora_kv_attention_workspace_bytes(const qalora_kv_desc* desc, int32_t batch, int64_t m, int32_t max_new,
                                        int32_t max_len, int with_score, size_t* bytes) {
  KvShape sh;
  int st = check_kv_desc(desc, &sh);
  if (st == QALORA_OK) st = check_batch(batch, m, max_new, 0);
  if (st != QALORA_OK) return st;
  if (max_len < 0) return QALORA_ERR_INVALID_ARG;
  if (bytes == nullptr) return QALORA_ERR_NULL_POINTER;
  *bytes = kv_attention_workspace(sh, batch, m, max_new, max_len, with_score != 0, nullptr);
  return QALORA_OK;
}

int qalora_kv_attention(const qalora_kv_desc* desc, int32_t batch, int64_t m, int32_t max_new, int32_t max_len,
                        const int32_t* starts, const int32_t* lens, const int32_t* table, int32_t max_blocks,
                        const void* q, int64_t q_stride, const void* codes, const float* scales, float softmax_scale,
                        void* out, float* lse, const float* score_in, float* score_out,
                        void* workspace, size_t workspace_bytes, void* cuda_stream) {
  KvShape sh;
  int st = check_kv_desc(desc, &sh);
  if (st == QALORA_OK) st = check_batch(batch, m, max_new, max_blocks);
  if (st != QALORA_OK) return st;
  if (max_len < 0 || !(softmax_scale > 0.f && softmax_scale <= 3.0e38f)) return QALORA_ERR_INVALID_ARG;
  if (!stride_ok(q_stride, (int64_t)sh.heads * sh.dim)) return QALORA_ERR_INVALID_ARG;
  if (score_in != nullptr && score_out == nullptr) return QALORA_ERR_NULL_POINTER;
  if (batch == 0 || m == 0 || max_new == 0) return QALORA_OK;
  if (starts == nullptr || lens == nullptr || (table == nullptr && max_blocks > 0) || q == nullptr || codes == nullptr ||
      scales == nullptr || out == nullptr || workspace == nullptr)
    return QALORA_ERR_NULL_POINTER;
  if (!aligned4(starts) || !aligned4(lens) || !aligned4(table) || !aligned16(q) || !aligned16(codes) || !aligned16(scales) ||
      !aligned16(out) || !aligned16(lse) || !aligned16(score_in) || !aligned16(score_out) || !aligned16(workspace))
    return QALORA_ERR_MISALIGNED;
  Workspace guards{};
  if (workspace_bytes < kv_attention_workspace(sh, batch, m, max_new, max_len, score_out != nullptr, &guards))
    return QALORA_ERR_WORKSPACE_TOO_SMALL;
  cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
  const KvAttention a{static_cast<const __nv_bfloat16*>(q), q_stride, static_cast<const int8_t*>(codes), scales, softmax_scale,
                      static_cast<__nv_bfloat16*>(out), lse, score_in, score_out};
  if ((st = debug_fill_guards(guards, workspace, stream)) != QALORA_OK) return st;
  st = launch_kv_attention(sh, make_batch(sh, starts, lens, table, batch, max_blocks, m, max_new, max_len), a, workspace, max_len,
                           stream);
  if (st != QALORA_OK) return st;
  return debug_verify_guards(guards, workspace, stream);
}

int qalora_kv_evict(const qalora_kv_desc* desc, int32_t batch, int32_t max_len, int32_t budget, int32_t recent,
                    const int32_t* lens, const int32_t* table, int32_t max_blocks,
                    void* codes, float* scales, float* score, const int32_t* dst_table, int32_t dst_max_blocks,
                    int32_t* dst_lens, int32_t* kept, void* cuda_stream) {
  KvShape sh;
  int st = check_kv_desc(desc, &sh);
  if (st != QALORA_OK) return st;
  if (batch < 0 || batch > 65535 || max_len < 0 || max_blocks < 0 || dst_max_blocks < 0 || budget < 1 || recent < 0 || recent > budget)
    return QALORA_ERR_INVALID_ARG;
  const KvBatch b = make_batch(sh, nullptr, lens, table, batch, max_blocks, 0, 0, max_len);
  if ((int64_t)dst_max_blocks * sh.block < (b.max_len < budget ? b.max_len : budget)) return QALORA_ERR_INVALID_ARG;
  if (batch == 0) return QALORA_OK;
  if (lens == nullptr || (table == nullptr && max_blocks > 0) || codes == nullptr || scales == nullptr || score == nullptr ||
      (dst_table == nullptr && dst_max_blocks > 0) || dst_lens == nullptr || kept == nullptr)
    return QALORA_ERR_NULL_POINTER;
  if (!aligned4(lens) || !aligned4(table) || !aligned4(dst_table) || !aligned4(dst_lens) || !aligned4(kept) || !aligned16(codes) ||
      !aligned16(scales) || !aligned16(score))
    return QALORA_ERR_MISALIGNED;
  return launch_kv_evict(sh, b, budget, recent, static_cast<int8_t*>(codes), scales, score, dst_table, dst_max_blocks, dst_lens,
                         kept, static_cast<cudaStream_t>(cuda_stream));
}

}  // extern "C"
