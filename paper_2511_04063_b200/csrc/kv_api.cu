// C entry points of the key/value cache in 4 bits: checks of arguments, then the launches of qk_rope.cu, kv_cache.cu and
// kv_attention.cu.
#include "kv_common.cuh"

using namespace dq;

namespace {
constexpr int64_t MAX_TOKENS = ((int64_t)1 << 31) - 256, MAX_STRIDE = (int64_t)1 << 40, MAX_SLOTS = (int64_t)1 << 30;
inline bool is_float(int t) { return t == DQ_FP32 || t == DQ_BF16 || t == DQ_FP16; }
inline bool aligned(const void* p, uintptr_t to) { return ((uintptr_t)p & (to - 1)) == 0; }

// heads of a tensor [token][head][dim]
dq_status heads(const dq_heads_t* x, int dtype, int64_t tokens, int dim, kv::Heads& out) {
  if (!x || x->heads <= 0 || x->heads > 65536 || x->token_stride < 0 || x->head_stride < 0) return DQ_ERR_INVALID_ARG;
  if ((x->heads > 1 && x->head_stride < dim) || (tokens > 1 && x->token_stride < dim)) return DQ_ERR_INVALID_ARG;
  if (x->token_stride > MAX_STRIDE || x->head_stride > MAX_STRIDE) return DQ_ERR_UNSUPPORTED;
  if (tokens > 0 && (!x->d_data || !aligned(x->d_data, dtype == DQ_FP32 ? 4 : 2))) return DQ_ERR_INVALID_ARG;
  out.p = x->d_data;
  out.token = x->token_stride;
  out.head = x->head_stride;
  out.heads = x->heads;
  out.vec = kv::pieces(x->d_data, x->token_stride, x->head_stride, dtype);
  return DQ_OK;
}
inline bool log2_of(int v, int& shift) {
  for (shift = 4; shift <= 12; ++shift) if (v == 1 << shift) return true;
  return false;
}
inline bool cache_dim(int dim) { return dim == 64 || dim == 128 || dim == 256; }
dq_status cache_of(const dq_kv_cache_t* c, kv::Cache& out) {
  int shift;
  if (!c || c->n_seqs < 0 || c->heads <= 0 || c->heads > 65536 || c->table_width <= 0 || c->n_pages < 0) return DQ_ERR_INVALID_ARG;
  if (!cache_dim(c->head_dim) || !log2_of(c->page_size, shift)) return DQ_ERR_UNSUPPORTED;
  if ((int64_t)c->table_width << shift > MAX_SLOTS || (int64_t)c->n_seqs * c->heads > MAX_TOKENS) return DQ_ERR_UNSUPPORTED;
  if (c->n_pages > MAX_TOKENS) return DQ_ERR_UNSUPPORTED;
  if (c->n_seqs > 0 && (!c->d_table || !c->d_lengths || (c->n_pages > 0 && !c->d_pages))) return DQ_ERR_INVALID_ARG;
  if (!aligned(c->d_table, 4) || !aligned(c->d_lengths, 4)) return DQ_ERR_INVALID_ARG;
  if (!aligned(c->d_pages, 128)) return DQ_ERR_UNSUPPORTED;
  out = kv::Cache{(uint8_t*)c->d_pages, c->n_pages, dq_kv_page_bytes(c->page_size, c->head_dim), c->d_table, c->d_lengths,
                  c->n_seqs, c->table_width, c->heads, shift};
  return DQ_OK;
}
dq_status batch_of(const dq_kv_cache_t* c, const int32_t* starts, int64_t tokens, kv::Batch& out) {
  if (tokens < 0 || !aligned(starts, 4)) return DQ_ERR_INVALID_ARG;
  if (tokens > MAX_TOKENS) return DQ_ERR_UNSUPPORTED;
  if (!starts && c->n_seqs > 0 && tokens % c->n_seqs) return DQ_ERR_INVALID_ARG;
  out = kv::Batch{starts, tokens, c->n_seqs ? (int)(tokens / c->n_seqs) : 0, c->n_seqs};
  return DQ_OK;
}
dq_status appended(const dq_heads_t* K, const dq_heads_t* V, int dtype, int64_t tokens, const dq_kv_cache_t* cache, const int32_t* starts,
                   kv::AppendArgs& a) {
  if (!is_float(dtype)) return DQ_ERR_INVALID_ARG;
  DQ_CHECK(cache_of(cache, a.cache));
  DQ_CHECK(batch_of(cache, starts, tokens, a.batch));
  DQ_CHECK(heads(K, dtype, tokens, cache->head_dim, a.k));
  DQ_CHECK(heads(V, dtype, tokens, cache->head_dim, a.v));
  return a.k.heads == cache->heads && a.v.heads == cache->heads ? DQ_OK : DQ_ERR_INVALID_ARG;
}
dq_status attended(const dq_heads_t* Q, int dtype, int64_t tokens, const dq_kv_cache_t* cache, const int32_t* starts, float scale,
                   kv::AttentionArgs& a) {
  if (!is_float(dtype)) return DQ_ERR_INVALID_ARG;
  if (dtype == DQ_FP32) return DQ_ERR_UNSUPPORTED;
  DQ_CHECK(cache_of(cache, a.cache));
  DQ_CHECK(batch_of(cache, starts, tokens, a.batch));
  DQ_CHECK(heads(Q, dtype, tokens, cache->head_dim, a.q));
  if (a.q.heads % cache->heads || !(scale > -INFINITY && scale < INFINITY)) return DQ_ERR_INVALID_ARG;
  a.group = a.q.heads / cache->heads;
  a.group_shift = a.group & (a.group - 1) ? -1 : __builtin_ctz((unsigned)a.group);
  if (tokens * a.group > MAX_TOKENS) return DQ_ERR_UNSUPPORTED;
  a.scale = scale;
  return DQ_OK;
}
}  // namespace

extern "C" {

int64_t dq_kv_page_bytes(int32_t page_size, int32_t head_dim) {
  int shift;
  return cache_dim(head_dim) && log2_of(page_size, shift) ? (int64_t)page_size * (head_dim + 8) : -1;
}

int64_t dq_kv_attention_workspace(int32_t head_dim) { return cache_dim(head_dim) ? kv::attention_workspace(head_dim) : -1; }

int64_t dq_kv_evict_workspace(int32_t n_seqs, int32_t heads, int32_t keep) {
  if (n_seqs < 0 || heads <= 0 || heads > 65536 || keep <= 0) return -1;
  const int64_t rows = (int64_t)n_seqs * heads, each = kv::evict_stride(keep) * 4;
  return rows > MAX_TOKENS || rows > INT64_MAX / each ? -1 : rows * each;
}

dq_status dq_qk_norm_rope(const dq_heads_t* Q, const dq_heads_t* K, int32_t dtype, int64_t tokens, int32_t head_dim,
                          const int32_t* d_positions, const float* d_inv_freq, int32_t rot_dim, const void* d_q_gamma,
                          const void* d_k_gamma, int32_t gamma_dtype, float eps, int32_t flags, const dq_heads_t* Q_out,
                          const dq_heads_t* K_out, void* cuda_stream) {
  kv::RopeArgs a{};
  if (!is_float(dtype) || tokens < 0 || head_dim <= 0 || rot_dim < 0 || rot_dim > head_dim || !K != !K_out) return DQ_ERR_INVALID_ARG;
  if (flags & ~(DQ_QK_NORM | DQ_QK_NEIGHBOURS | DQ_QK_HADAMARD)) return DQ_ERR_INVALID_ARG;
  const bool norm = flags & DQ_QK_NORM;
  if (!norm && (d_q_gamma || d_k_gamma)) return DQ_ERR_INVALID_ARG;
  if (norm && (!(eps >= 0.f) || ((d_q_gamma || d_k_gamma) && gamma_dtype != DQ_FP32 && gamma_dtype != dtype))) return DQ_ERR_INVALID_ARG;
  if (tokens > MAX_TOKENS || head_dim % 16 || head_dim > 256 || rot_dim % 16) return DQ_ERR_UNSUPPORTED;
  if ((flags & DQ_QK_HADAMARD) && !cache_dim(head_dim)) return DQ_ERR_UNSUPPORTED;
  DQ_CHECK(heads(Q, dtype, tokens, head_dim, a.q));
  DQ_CHECK(heads(Q_out, dtype, tokens, head_dim, a.q_out));
  if (a.q.heads != a.q_out.heads) return DQ_ERR_INVALID_ARG;
  if (K) {
    DQ_CHECK(heads(K, dtype, tokens, head_dim, a.k));
    DQ_CHECK(heads(K_out, dtype, tokens, head_dim, a.k_out));
    if (a.k.heads != a.k_out.heads) return DQ_ERR_INVALID_ARG;
  }
  const uintptr_t g = gamma_dtype == DQ_FP32 ? 4 : 2;
  if (!aligned(d_q_gamma, g) || !aligned(d_k_gamma, g) || !aligned(d_positions, 4) || !aligned(d_inv_freq, 4)) return DQ_ERR_INVALID_ARG;
  if (tokens == 0) return DQ_OK;
  if (rot_dim && (!d_positions || !d_inv_freq)) return DQ_ERR_INVALID_ARG;
  mx::Device dev;
  DQ_CHECK(mx::current_device(dev));
  a.tokens = tokens; a.dim = head_dim; a.rot = rot_dim;
  a.positions = d_positions; a.inv_freq = d_inv_freq;
  a.q_gamma = d_q_gamma; a.k_gamma = d_k_gamma; a.gamma_fp32 = gamma_dtype == DQ_FP32;
  a.eps = eps; a.flags = flags;
  return kv::rope((cudaStream_t)cuda_stream, dev, dtype, a);
}

dq_status dq_kv_append(const dq_heads_t* K, const dq_heads_t* V, int32_t dtype, int64_t tokens, const dq_kv_cache_t* cache,
                       const int32_t* d_starts, const dq_heads_t* k_values, const dq_heads_t* v_values, const int32_t* d_positions,
                       int32_t* d_slot_positions, int64_t ld_slots, void* cuda_stream) {
  kv::AppendArgs a{};
  DQ_CHECK(appended(K, V, dtype, tokens, cache, d_starts, a));
  if (k_values) DQ_CHECK(heads(k_values, dtype, tokens, cache->head_dim, a.k_values));
  if (v_values) DQ_CHECK(heads(v_values, dtype, tokens, cache->head_dim, a.v_values));
  if ((k_values && a.k_values.heads != cache->heads) || (v_values && a.v_values.heads != cache->heads)) return DQ_ERR_INVALID_ARG;
  if (!aligned(d_positions, 4) || !aligned(d_slot_positions, 4)) return DQ_ERR_INVALID_ARG;
  if (d_slot_positions && ld_slots < (int64_t)cache->table_width * cache->page_size) return DQ_ERR_INVALID_ARG;
  if (tokens == 0 || cache->n_seqs == 0) return DQ_OK;
  mx::Device dev;
  DQ_CHECK(mx::current_device(dev));
  a.positions = d_positions; a.slot_positions = d_slot_positions; a.ld_slots = ld_slots;
  return kv::append((cudaStream_t)cuda_stream, dev, dtype, cache->head_dim, a);
}

dq_status dq_kv_dequantize(const dq_kv_cache_t* cache, const int32_t* d_starts, int64_t tokens, const dq_heads_t* K,
                           const dq_heads_t* V, int32_t dtype, void* cuda_stream) {
  kv::AppendArgs a{};
  DQ_CHECK(appended(K, V, dtype, tokens, cache, d_starts, a));
  if (tokens == 0 || cache->n_seqs == 0) return DQ_OK;
  mx::Device dev;
  DQ_CHECK(mx::current_device(dev));
  return kv::dequantize((cudaStream_t)cuda_stream, dev, dtype, cache->head_dim, a);
}

dq_status dq_kv_attention(const dq_heads_t* Q, int32_t dtype, int64_t tokens, const dq_kv_cache_t* cache, const int32_t* d_starts,
                          float scale, const dq_heads_t* out, float* d_lse, void* d_workspace, void* cuda_stream) {
  kv::AttentionArgs a{};
  DQ_CHECK(attended(Q, dtype, tokens, cache, d_starts, scale, a));
  DQ_CHECK(heads(out, dtype, tokens, cache->head_dim, a.out));
  if (a.out.heads != a.q.heads || !aligned(d_lse, 4)) return DQ_ERR_INVALID_ARG;
  if (tokens == 0 || cache->n_seqs == 0) return DQ_OK;
  if (!d_workspace) return DQ_ERR_INVALID_ARG;
  if (!aligned(d_workspace, 16)) return DQ_ERR_UNSUPPORTED;
  mx::Device dev;
  DQ_CHECK(mx::current_device(dev));
  a.lse = d_lse; a.workspace = (uint8_t*)d_workspace; a.d_status = dev.d_status;
  return kv::attention((cudaStream_t)cuda_stream, dev, dtype, cache->head_dim, a);
}

dq_status dq_kv_attention_weights(const dq_heads_t* Q, int32_t dtype, int64_t tokens, const float* d_lse, const dq_kv_cache_t* cache,
                                  const int32_t* d_starts, float scale, const float* d_weights, float* d_weights_out,
                                  int64_t ld_slots, void* cuda_stream) {
  kv::AttentionArgs a{};
  DQ_CHECK(attended(Q, dtype, tokens, cache, d_starts, scale, a));
  if (ld_slots < (int64_t)cache->table_width * cache->page_size || !aligned(d_lse, 4) || !aligned(d_weights, 4) || !aligned(d_weights_out, 4))
    return DQ_ERR_INVALID_ARG;
  if (cache->n_seqs == 0) return DQ_OK;
  if ((tokens > 0 && !d_lse) || !d_weights_out) return DQ_ERR_INVALID_ARG;
  mx::Device dev;
  DQ_CHECK(mx::current_device(dev));
  a.lse = const_cast<float*>(d_lse); a.weights = d_weights; a.weights_out = d_weights_out; a.ld_slots = ld_slots;
  a.d_status = dev.d_status;
  return kv::attention_weights((cudaStream_t)cuda_stream, dev, dtype, cache->head_dim, a);
}

dq_status dq_kv_evict(const dq_kv_cache_t* cache, const float* d_weights, const int32_t* d_positions, int64_t ld_slots, int32_t keep,
                      int32_t recent, float* d_weights_out, int32_t* d_positions_out, int32_t* d_lengths_out, void* d_workspace,
                      void* cuda_stream) {
  kv::EvictArgs a{};
  DQ_CHECK(cache_of(cache, a.cache));
  if (keep <= 0 || recent < 0 || recent > keep || ld_slots < (int64_t)cache->table_width * cache->page_size) return DQ_ERR_INVALID_ARG;
  if (cache->n_seqs == 0) return DQ_OK;
  if (dq_kv_evict_workspace(cache->n_seqs, cache->heads, keep) < 0) return DQ_ERR_UNSUPPORTED;
  if (!d_weights || !d_positions || !d_weights_out || !d_positions_out || !d_lengths_out || !d_workspace) return DQ_ERR_INVALID_ARG;
  if (!aligned(d_weights, 4) || !aligned(d_positions, 4) || !aligned(d_weights_out, 4) || !aligned(d_positions_out, 4) ||
      !aligned(d_lengths_out, 4) || !aligned(d_workspace, 4))
    return DQ_ERR_INVALID_ARG;
  mx::Device dev;
  DQ_CHECK(mx::current_device(dev));
  a.weights = d_weights; a.positions = d_positions; a.ld_slots = ld_slots; a.keep = keep; a.recent = recent;
  a.weights_out = d_weights_out; a.positions_out = d_positions_out; a.lengths_out = d_lengths_out; a.workspace = (int*)d_workspace;
  return kv::evict((cudaStream_t)cuda_stream, dev, cache->head_dim, a);
}

}  // extern "C"
