// C ABI: argument validation, workspace layout and dispatch.  No arithmetic of the method lives here.
#include <math.h>

#include "fc_common.h"

using namespace fc;

namespace {

constexpr int64_t kMaxUnits = 32767;   // grid.y / grid.z limits of the launches below

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

fc_status check_desc(const fc_kv_desc* d) {
  if (!d) return FC_EINVAL;
  if (d->batch < 0 || d->layers < 1 || d->kv_heads < 1 || d->n_tokens < 1 || d->head_dim < 1)
    return FC_EINVAL;
  if (d->dtype != FC_F32 && d->dtype != FC_BF16) return FC_EINVAL;
  const int64_t eb = d->dtype == FC_BF16 ? 2 : 4;
  if ((d->head_dim * eb) % 16 != 0) return FC_EINVAL;
  if (d->stride_n < d->head_dim) return FC_EINVAL;
  if (d->stride_l < 0 || d->stride_b < 0 || d->stride_h < 0) return FC_EINVAL;
  if ((d->stride_n * eb) % 16 || (d->stride_h * eb) % 16 || (d->stride_l * eb) % 16 ||
      (d->stride_b * eb) % 16)
    return FC_EINVAL;
  if ((int64_t)d->batch * d->layers * d->kv_heads > kMaxUnits) return FC_EUNSUPPORTED;
  if (d->layers > 1024) return FC_EUNSUPPORTED;
  return FC_OK;
}

bool basis_supported(const fc_kv_desc& d) { return d.head_dim <= 256; }   // (the kernels pad rows to 64 columns)

// What FC_PATH_AUTO resolves to; every other path that applies stays as it is; 0 if unsupported
int32_t resolve(const fc_kv_desc& d, int32_t r, int32_t path) {
  switch (path) {
    case FC_PATH_AUTO: return fft_supported(d, r) ? FC_PATH_FFT : (basis_supported(d) ? FC_PATH_DENSE : 0);
    case FC_PATH_DENSE: case FC_PATH_BASIS: return basis_supported(d) ? path : 0;
    case FC_PATH_FFT: case FC_PATH_STREAM: return fft_supported(d, r) ? path : 0;
    case FC_PATH_RESAMPLE: return resample_supported(d, r) ? path : 0;
    default: return 0;
  }
}

// The realisation behind a path: FC_PATH_BASIS, FC_PATH_STREAM, FC_PATH_RESAMPLE, or 0
int32_t realisation(const fc_kv_desc& d, int32_t r, int32_t path) {
  const int32_t p = resolve(d, r, path);
  if (p != FC_PATH_DENSE && p != FC_PATH_FFT) return p;
  if (resample_supported(d, r)) return FC_PATH_RESAMPLE;
  return p == FC_PATH_FFT ? FC_PATH_STREAM : FC_PATH_BASIS;
}

size_t score_workspace(const fc_kv_desc& d, int32_t r, int32_t path) {
  if (resolve(d, r, path) == FC_PATH_FFT) return fft_layout(d, r).total + resample_reserve(d);
  switch (realisation(d, r, path)) {
    case FC_PATH_BASIS: return dense_layout(d, r).total;
    case FC_PATH_STREAM: return fft_layout(d, r).total;
    case FC_PATH_RESAMPLE: return resample_layout(d, r).total;
    default: return 0;
  }
}

}  // namespace

extern "C" {

int32_t flashcache_cutoff_r(int32_t n_tokens, double gamma) {
  if (n_tokens < 1) return 0;
  double w = floor(gamma * (double)n_tokens);
  if (!(w >= 0.0)) w = 0.0;                       // also catches NaN
  if (w > (double)n_tokens) w = (double)n_tokens;
  int64_t r = (int64_t)w + 1;
  if (r > n_tokens) r = n_tokens;
  return (int32_t)r;
}

int64_t flashcache_total_budget(int32_t layers, int32_t n_tokens, double rho) {
  if (layers < 1 || n_tokens < 1) return 0;
  const int64_t full = (int64_t)layers * n_tokens;
  double t = floor(rho * (double)layers * (double)n_tokens);
  if (!(t >= (double)layers)) return layers;      // also catches NaN
  if (t > (double)full) return full;
  return (int64_t)t;
}

int32_t flashcache_resolve_path(const fc_kv_desc* desc, int32_t r, int32_t path) {
  if (check_desc(desc) != FC_OK || r < 1 || r > desc->n_tokens) return 0;
  return resolve(*desc, r, path);
}

int32_t flashcache_realisation(const fc_kv_desc* desc, int32_t r, int32_t path) {
  if (check_desc(desc) != FC_OK || r < 1 || r > desc->n_tokens) return 0;
  return realisation(*desc, r, path);
}

size_t flashcache_workspace_bytes(const fc_kv_desc* desc, int32_t r, int32_t path) {
  if (check_desc(desc) != FC_OK || r < 1 || r > desc->n_tokens) return 0;
  return score_workspace(*desc, r, path);
}

size_t flashcache_select_workspace_bytes(const fc_kv_desc* desc) {
  (void)desc;
  return 0;
}

fc_status flashcache_prepare(const fc_kv_desc* desc, int32_t r, int32_t path, void* workspace,
                             size_t workspace_bytes, void* hip_stream) {
  fc_status st = check_desc(desc);
  if (st != FC_OK) return st;
  if (r < 1 || r > desc->n_tokens) return FC_EINVAL;
  const int32_t real = realisation(*desc, r, path);
  if (real == 0) return FC_EUNSUPPORTED;
  if (!workspace || (reinterpret_cast<uintptr_t>(workspace) % kWsAlign) != 0) return FC_EWORKSPACE;
  hipStream_t s = static_cast<hipStream_t>(hip_stream);
  hipError_t e;
  if (real == FC_PATH_BASIS) {
    DenseLayout lay = dense_layout(*desc, r);
    if (workspace_bytes < lay.total) return FC_EWORKSPACE;
    e = dense_prepare(*desc, r, lay, workspace, s);
  } else if (real == FC_PATH_RESAMPLE) {
    ResampleLayout lay = resample_layout(*desc, r);
    if (workspace_bytes < lay.total) return FC_EWORKSPACE;
    e = resample_prepare(*desc, r, lay, workspace, s);
  } else {
    FftLayout lay = fft_layout(*desc, r);
    if (workspace_bytes < lay.total) return FC_EWORKSPACE;
    e = fft_prepare(*desc, r, lay, workspace, s);
  }
  return e == hipSuccess ? FC_OK : FC_EHIP;
}

fc_status flashcache_workspace_error(const void* workspace, int32_t* flag_out, void* hip_stream) {
  if (!workspace || !flag_out) return FC_EINVAL;
  hipStream_t s = static_cast<hipStream_t>(hip_stream);
  WsHeader h;
  if (hipMemcpyAsync(&h, workspace, sizeof(h), hipMemcpyDeviceToHost, s) != hipSuccess) return FC_EHIP;
  if (hipStreamSynchronize(s) != hipSuccess) return FC_EHIP;
  *flag_out = (h.magic != kWsMagic) ? 2 : h.error;
  return FC_OK;
}

static fc_status score_common(const void* K, const void* V, const fc_kv_desc* desc, int32_t r, int32_t path,
                              float* scores, double* energy, void* workspace, size_t workspace_bytes,
                              UnitMap um, void* hip_stream) {
  fc_status st = check_desc(desc);
  if (st != FC_OK) return st;
  if (r < 1 || r > desc->n_tokens) return FC_EINVAL;
  const int32_t real = realisation(*desc, r, path);
  if (real == 0) return FC_EUNSUPPORTED;
  if (desc->batch == 0) return FC_OK;
  if (!K || !V || !scores || !energy) return FC_EINVAL;
  if (!aligned16(K) || !aligned16(V) || !aligned16(scores) || !aligned16(energy)) return FC_EINVAL;
  if (!workspace || (reinterpret_cast<uintptr_t>(workspace) % kWsAlign) != 0) return FC_EWORKSPACE;
  hipStream_t s = static_cast<hipStream_t>(hip_stream);
  hipError_t e;
  if (real == FC_PATH_BASIS) {
    DenseLayout lay = dense_layout(*desc, r);
    if (workspace_bytes < lay.total) return FC_EWORKSPACE;
    e = dense_score(K, V, *desc, r, lay, scores, energy, workspace, um, s);
  } else if (real == FC_PATH_RESAMPLE) {
    ResampleLayout lay = resample_layout(*desc, r);
    if (workspace_bytes < lay.total) return FC_EWORKSPACE;
    e = resample_score(K, V, *desc, r, lay, scores, energy, workspace, um, s);
  } else {
    FftLayout lay = fft_layout(*desc, r);
    if (workspace_bytes < lay.total) return FC_EWORKSPACE;
    e = fft_score(K, V, *desc, r, lay, scores, energy, workspace, um, s);
  }
  return e == hipSuccess ? FC_OK : FC_EHIP;
}

fc_status flashcache_score(const void* K, const void* V, const fc_kv_desc* desc, int32_t r, int32_t path,
                           float* scores, double* energy, void* workspace, size_t workspace_bytes,
                           void* hip_stream) {
  return score_common(K, V, desc, r, path, scores, energy, workspace, workspace_bytes, UnitMap{0, 0, 0},
                      hip_stream);
}

fc_status flashcache_score_layer(const void* K, const void* V, const fc_kv_desc* desc, int32_t layer,
                                 int32_t total_layers, int32_t r, int32_t path, float* scores,
                                 double* energy, void* workspace, size_t workspace_bytes,
                                 void* hip_stream) {
  if (!desc || desc->layers != 1 || total_layers < 1 || layer < 0 || layer >= total_layers) return FC_EINVAL;
  return score_common(K, V, desc, r, path, scores, energy, workspace, workspace_bytes,
                      UnitMap{desc->kv_heads, total_layers, layer}, hip_stream);
}

fc_status flashcache_lowpass_energy(const fc_kv_desc* desc, int32_t r, int32_t path, void* workspace,
                                    size_t workspace_bytes, double* lowpass_energy, void* hip_stream) {
  fc_status st = check_desc(desc);
  if (st != FC_OK) return st;
  if (r < 1 || r > desc->n_tokens) return FC_EINVAL;
  const int32_t real = realisation(*desc, r, path);
  if (real == 0) return FC_EUNSUPPORTED;
  if (desc->batch == 0) return FC_OK;
  if (!lowpass_energy || (reinterpret_cast<uintptr_t>(lowpass_energy) & 7u)) return FC_EINVAL;
  if (!workspace || (reinterpret_cast<uintptr_t>(workspace) % kWsAlign) != 0) return FC_EWORKSPACE;
  hipStream_t s = static_cast<hipStream_t>(hip_stream);
  hipError_t e;
  if (real == FC_PATH_BASIS) {
    DenseLayout lay = dense_layout(*desc, r);
    if (workspace_bytes < lay.total) return FC_EWORKSPACE;
    e = dense_lowpass(*desc, lay, workspace, lowpass_energy, s);
  } else if (real == FC_PATH_RESAMPLE) {
    ResampleLayout lay = resample_layout(*desc, r);
    if (workspace_bytes < lay.total) return FC_EWORKSPACE;
    e = resample_lowpass(*desc, lay, workspace, lowpass_energy, s);
  } else {
    FftLayout lay = fft_layout(*desc, r);
    if (workspace_bytes < lay.total) return FC_EWORKSPACE;
    e = fft_lowpass(*desc, r, lay, workspace, lowpass_energy, s);
  }
  return e == hipSuccess ? FC_OK : FC_EHIP;
}

fc_status flashcache_allocate(const double* energy, int32_t batch, int32_t layers, int32_t kv_heads,
                              int32_t n_tokens, int64_t total_budget, int32_t b_min, int32_t b_max,
                              int32_t* budgets, int64_t* layer_offsets, void* hip_stream) {
  if (batch < 0 || layers < 1 || kv_heads < 1 || n_tokens < 1) return FC_EINVAL;
  if (layers > 1024) return FC_EUNSUPPORTED;
  if (b_min < 1 || b_max < b_min || b_max > n_tokens) return FC_EBUDGET;
  if ((int64_t)layers * b_min > total_budget || (int64_t)layers * b_max < total_budget) return FC_EBUDGET;
  if (batch == 0) return FC_OK;
  if (!energy || !budgets || !layer_offsets) return FC_EINVAL;
  if ((reinterpret_cast<uintptr_t>(energy) & 7u) || (reinterpret_cast<uintptr_t>(layer_offsets) & 7u) ||
      (reinterpret_cast<uintptr_t>(budgets) & 3u))
    return FC_EINVAL;
  hipError_t e = allocate_launch(energy, batch, layers, kv_heads, n_tokens, total_budget, b_min, b_max,
                                 budgets, layer_offsets, static_cast<hipStream_t>(hip_stream));
  return e == hipSuccess ? FC_OK : FC_EHIP;
}

static fc_status select_gather_common(const void* K, const void* V, const fc_kv_desc* desc,
                                      const float* scores, const int32_t* budgets,
                                      const int64_t* layer_offsets, int64_t rows_per_seq, bool shared,
                                      int32_t* idx_out, void* K_out, void* V_out,
                                      const int32_t* block_table, int32_t page_size, int32_t max_pages,
                                      int64_t num_pages, void* hip_stream, bool copies = true) {
  fc_status st = check_desc(desc);
  if (st != FC_OK) return st;
  if (rows_per_seq < 0 || rows_per_seq > (int64_t)desc->layers * desc->kv_heads * desc->n_tokens)
    return FC_EINVAL;
  if (desc->batch == 0 || rows_per_seq == 0) return FC_OK;
  if (!K || !V || !scores || !budgets || !layer_offsets || !idx_out || (copies && (!K_out || !V_out))) return FC_EINVAL;
  if (!aligned16(K) || !aligned16(V) || !aligned16(K_out) || !aligned16(V_out)) return FC_EINVAL;
  if ((reinterpret_cast<uintptr_t>(scores) & 3u) || (reinterpret_cast<uintptr_t>(budgets) & 3u) ||
      (reinterpret_cast<uintptr_t>(idx_out) & 3u) || (reinterpret_cast<uintptr_t>(layer_offsets) & 7u))
    return FC_EINVAL;
  hipError_t e = select_gather_launch(K, V, *desc, scores, budgets, layer_offsets, rows_per_seq, shared,
                                      idx_out, K_out, V_out, block_table, page_size, max_pages, num_pages,
                                      static_cast<hipStream_t>(hip_stream));
  return e == hipSuccess ? FC_OK : FC_EHIP;
}

fc_status flashcache_select_gather(const void* K, const void* V, const fc_kv_desc* desc, const float* scores,
                                   const int32_t* budgets, const int64_t* layer_offsets,
                                   int64_t rows_per_seq, int32_t* idx_out, void* K_out, void* V_out,
                                   void* workspace, size_t workspace_bytes, void* hip_stream) {
  (void)workspace; (void)workspace_bytes;
  return select_gather_common(K, V, desc, scores, budgets, layer_offsets, rows_per_seq, false, idx_out,
                              K_out, V_out, nullptr, 0, 0, 0, hip_stream);
}

fc_status flashcache_select_gather_shared(const void* K, const void* V, const fc_kv_desc* desc,
                                          const float* scores, const int32_t* budgets,
                                          const int64_t* layer_offsets, int64_t rows_per_seq,
                                          int32_t* idx_out, void* K_out, void* V_out, void* workspace,
                                          size_t workspace_bytes, void* hip_stream) {
  (void)workspace; (void)workspace_bytes;
  return select_gather_common(K, V, desc, scores, budgets, layer_offsets, rows_per_seq, true, idx_out,
                              K_out, V_out, nullptr, 0, 0, 0, hip_stream);
}

fc_status flashcache_select_gather_paged(const void* K, const void* V, const fc_kv_desc* desc,
                                         const float* scores, const int32_t* budgets,
                                         const int64_t* layer_offsets, int64_t rows_per_seq, int32_t shared,
                                         int32_t* idx_out, const int32_t* block_table, int32_t page_size,
                                         int32_t max_pages, int64_t num_pages, void* K_cache, void* V_cache,
                                         void* workspace, size_t workspace_bytes, void* hip_stream) {
  (void)workspace; (void)workspace_bytes;
  if (page_size < 1 || max_pages < 1 || num_pages < 1) return FC_EINVAL;
  if (!block_table || (reinterpret_cast<uintptr_t>(block_table) & 3u)) return FC_EINVAL;
  return select_gather_common(K, V, desc, scores, budgets, layer_offsets, rows_per_seq, shared != 0, idx_out,
                              K_cache, V_cache, block_table, page_size, max_pages, num_pages, hip_stream);
}

size_t flashcache_decode_workspace_bytes(int32_t batch, int32_t layers, int32_t kv_heads, int32_t q_heads,
                                         int32_t head_dim) {
  if (batch < 0 || layers < 1 || kv_heads < 1 || q_heads < kv_heads || q_heads % kv_heads) return 0;
  const int group = q_heads / kv_heads;      // the same size serves both storage types
  if (!decode_supported(group, head_dim, FC_BF16) && !decode_supported(group, head_dim, FC_F32)) return 0;
  if ((int64_t)batch * layers * kv_heads > kMaxUnits) return 0;
  return decode_workspace_bytes(batch, layers, kv_heads, q_heads / kv_heads, head_dim);
}

fc_status flashcache_decode_attention(const void* Q, const void* K_cache, const void* V_cache, int32_t batch,
                                      int32_t layers, int32_t kv_heads, int32_t q_heads, int32_t head_dim,
                                      int32_t dtype, const int32_t* budgets, const int64_t* layer_offsets,
                                      int64_t rows_per_seq, float scale, float* out, void* workspace,
                                      size_t workspace_bytes, void* hip_stream) {
  if (batch < 0 || layers < 1 || kv_heads < 1 || q_heads < kv_heads || q_heads % kv_heads || head_dim < 1)
    return FC_EINVAL;
  if (dtype != FC_F32 && dtype != FC_BF16) return FC_EINVAL;
  if (rows_per_seq < 0 || !(scale == scale)) return FC_EINVAL;
  if (!decode_supported(q_heads / kv_heads, head_dim, dtype)) return FC_EUNSUPPORTED;
  if ((int64_t)batch * layers * kv_heads > kMaxUnits) return FC_EUNSUPPORTED;
  if (batch == 0) return FC_OK;
  if (!Q || !K_cache || !V_cache || !budgets || !layer_offsets || !out) return FC_EINVAL;
  if (!aligned16(Q) || !aligned16(K_cache) || !aligned16(V_cache) || !aligned16(out)) return FC_EINVAL;
  if ((reinterpret_cast<uintptr_t>(budgets) & 3u) || (reinterpret_cast<uintptr_t>(layer_offsets) & 7u))
    return FC_EINVAL;
  const size_t need = decode_workspace_bytes(batch, layers, kv_heads, q_heads / kv_heads, head_dim);
  if (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 15u) || workspace_bytes < need)
    return FC_EWORKSPACE;
  hipError_t e = decode_launch(Q, K_cache, V_cache, batch, layers, kv_heads, q_heads / kv_heads, head_dim,
                               dtype, budgets, layer_offsets, rows_per_seq, scale, out, workspace, nullptr, 0, 0,
                               0, static_cast<hipStream_t>(hip_stream));
  return e == hipSuccess ? FC_OK : FC_EHIP;
}

size_t flashcache_decode_static_scratch_bytes(void) { return decode_static_scratch_bytes(); }

fc_status flashcache_decode_attention_static(const void* Q, const void* K_cache, const void* V_cache,
                                             int32_t batch, int32_t layers, int32_t kv_heads,
                                             int32_t q_heads, int32_t head_dim, int32_t dtype,
                                             const int32_t* budgets, const int64_t* layer_offsets,
                                             int64_t rows_per_seq, float scale, float* out,
                                             void* hip_stream) {
  if (batch < 0 || layers < 1 || kv_heads < 1 || q_heads < kv_heads || q_heads % kv_heads || head_dim < 1)
    return FC_EINVAL;
  if (dtype != FC_F32 && dtype != FC_BF16) return FC_EINVAL;
  if (rows_per_seq < 0 || !(scale == scale)) return FC_EINVAL;
  if (!decode_supported(q_heads / kv_heads, head_dim, dtype)) return FC_EUNSUPPORTED;
  if ((int64_t)batch * layers * kv_heads > kMaxUnits) return FC_EUNSUPPORTED;
  // the partial results must fit the static array: larger problems need the workspace variant
  if (decode_workspace_bytes(batch, layers, kv_heads, q_heads / kv_heads, head_dim) >
      decode_static_scratch_bytes())
    return FC_EWORKSPACE;
  if (batch == 0) return FC_OK;
  if (!Q || !K_cache || !V_cache || !budgets || !layer_offsets || !out) return FC_EINVAL;
  if (!aligned16(Q) || !aligned16(K_cache) || !aligned16(V_cache) || !aligned16(out)) return FC_EINVAL;
  if ((reinterpret_cast<uintptr_t>(budgets) & 3u) || (reinterpret_cast<uintptr_t>(layer_offsets) & 7u))
    return FC_EINVAL;
  void* scratch_ptr = nullptr;
  if (decode_static_scratch(&scratch_ptr) != hipSuccess) return FC_EHIP;
  hipError_t e = decode_launch(Q, K_cache, V_cache, batch, layers, kv_heads, q_heads / kv_heads, head_dim,
                               dtype, budgets, layer_offsets, rows_per_seq, scale, out, scratch_ptr, nullptr, 0,
                               0, 0, static_cast<hipStream_t>(hip_stream));
  return e == hipSuccess ? FC_OK : FC_EHIP;
}

fc_status flashcache_decode_attention_paged(const void* Q, const void* K_pages, const void* V_pages,
                                            const int32_t* block_table, int32_t page_size,
                                            int32_t max_pages, int64_t num_pages, int32_t batch,
                                            int32_t layers, int32_t kv_heads, int32_t q_heads,
                                            int32_t head_dim, int32_t dtype, const int32_t* budgets,
                                            float scale, float* out, void* workspace, size_t workspace_bytes,
                                            void* hip_stream) {
  if (batch < 0 || layers < 1 || kv_heads < 1 || q_heads < kv_heads || q_heads % kv_heads || head_dim < 1)
    return FC_EINVAL;
  if (dtype != FC_F32 && dtype != FC_BF16) return FC_EINVAL;
  if (page_size < 1 || max_pages < 1 || num_pages < 1 || !(scale == scale)) return FC_EINVAL;
  if (!decode_supported(q_heads / kv_heads, head_dim, dtype)) return FC_EUNSUPPORTED;
  if ((int64_t)batch * layers * kv_heads > kMaxUnits) return FC_EUNSUPPORTED;
  if (batch == 0) return FC_OK;
  if (!Q || !K_pages || !V_pages || !block_table || !budgets || !out) return FC_EINVAL;
  if (!aligned16(Q) || !aligned16(K_pages) || !aligned16(V_pages) || !aligned16(out)) return FC_EINVAL;
  if ((reinterpret_cast<uintptr_t>(budgets) & 3u) || (reinterpret_cast<uintptr_t>(block_table) & 3u))
    return FC_EINVAL;
  const size_t need = decode_workspace_bytes(batch, layers, kv_heads, q_heads / kv_heads, head_dim);
  if (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 15u) || workspace_bytes < need)
    return FC_EWORKSPACE;
  hipError_t e = decode_launch(Q, K_pages, V_pages, batch, layers, kv_heads, q_heads / kv_heads, head_dim,
                               dtype, budgets, nullptr, 0, scale, out, workspace, block_table, page_size,
                               max_pages, num_pages, static_cast<hipStream_t>(hip_stream));
  return e == hipSuccess ? FC_OK : FC_EHIP;
}

static fc_status check_heads(const fc_rotary_plan& plan, const fc_heads_desc& d, const void* in, const void* out) {
  if (d.batch < 0 || d.tokens < 0 || d.heads < 0 || d.head_dim < 1) return FC_EINVAL;
  if (d.dtype != FC_F32 && d.dtype != FC_BF16) return FC_EINVAL;
  if (d.head_dim % 2 || d.head_dim < plan.rotary_dim) return FC_EINVAL;
  if (d.head_dim > 512) return FC_EUNSUPPORTED;
  if (d.stride_b < 0 || d.stride_t < 0 || d.stride_h < 0) return FC_EINVAL;
  if (d.out_stride_b < 0 || d.out_stride_t < 0 || d.out_stride_h < 0) return FC_EINVAL;
  // (a workgroup of 256 threads has a token at least, and a launch fewer than 2^32 threads)
  if ((int64_t)d.batch * d.tokens >= (1 << 24) || d.heads > 65535) return FC_EUNSUPPORTED;
  if ((int64_t)d.batch * d.tokens * d.heads == 0) return FC_OK;
  const uintptr_t e = d.dtype == FC_BF16 ? 2 : 4;
  if (!in || !out || reinterpret_cast<uintptr_t>(in) % e || reinterpret_cast<uintptr_t>(out) % e) return FC_EINVAL;
  // rows of the output must not lie on one another
  if ((d.batch > 1 && d.out_stride_b < d.head_dim) || (d.tokens > 1 && d.out_stride_t < d.head_dim) ||
      (d.heads > 1 && d.out_stride_h < d.head_dim))
    return FC_EINVAL;
  if (in == out && ((d.batch > 1 && d.stride_b != d.out_stride_b) || (d.tokens > 1 && d.stride_t != d.out_stride_t) ||
                    (d.heads > 1 && d.stride_h != d.out_stride_h)))
    return FC_EINVAL;
  return FC_OK;
}

fc_status flashcache_rotary(const fc_rotary_plan* plan, const int32_t* positions, const void* Q, void* Q_out,
                            const fc_heads_desc* q_desc, const void* K, void* K_out, const fc_heads_desc* k_desc,
                            int32_t inverse, void* hip_stream) {
  if (!plan || !q_desc || plan->magic != kWsMagic) return FC_EINVAL;
  if (plan->rotary_dim < 2 || plan->rotary_dim % 2 || plan->rotary_dim > 2 * FC_ROTARY_MAX_PAIRS || plan->streams < 1 || plan->streams > 4) return FC_EINVAL;
  fc_status st = check_heads(*plan, *q_desc, Q, Q_out);
  if (st != FC_OK) return st;
  if (k_desc) {
    st = check_heads(*plan, *k_desc, K, K_out);
    if (st != FC_OK) return st;
    if (k_desc->batch != q_desc->batch || k_desc->tokens != q_desc->tokens || k_desc->head_dim != q_desc->head_dim ||
        k_desc->dtype != q_desc->dtype)
      return FC_EINVAL;
  }
  const int64_t heads = (int64_t)q_desc->heads + (k_desc ? k_desc->heads : 0);
  if (heads > 65535) return FC_EUNSUPPORTED;
  if ((int64_t)q_desc->batch * q_desc->tokens * heads == 0) return FC_OK;
  if (!positions || (reinterpret_cast<uintptr_t>(positions) & 3u)) return FC_EINVAL;
  hipError_t e = rotary_launch(*plan, positions, Q, Q_out, *q_desc, K, K_out, k_desc, inverse != 0, static_cast<hipStream_t>(hip_stream));
  return e == hipSuccess ? FC_OK : FC_EHIP;
}

fc_status flashcache_assign_pages(const int32_t* rows, const int32_t* add, int32_t add_each, int32_t batch, int32_t layers,
                                  int32_t kv_heads, int32_t page_size, int32_t max_pages, const int32_t* free_pages,
                                  int64_t num_free, const int64_t* cursor, int32_t* block_table, int64_t* slots,
                                  int64_t slots_per_seq, int32_t* rows_out, int64_t* cursor_out, void* hip_stream) {
  if (batch < 0 || layers < 1 || kv_heads < 1 || page_size < 1 || max_pages < 1 || num_free < 0 || slots_per_seq < 0) return FC_EINVAL;
  if (layers > 1024 || page_size > (1 << 25) || (int64_t)batch * layers * kv_heads > kMaxUnits) return FC_EUNSUPPORTED;
  if (batch == 0) return FC_OK;
  if (!rows || !cursor || !block_table || !rows_out || !cursor_out || (slots_per_seq > 0 && !slots)) return FC_EINVAL;
  auto misaligned = [](const void* p, uintptr_t to) { return reinterpret_cast<uintptr_t>(p) % to != 0; };
  if (misaligned(rows, 4) || misaligned(add, 4) || misaligned(free_pages, 4) || misaligned(block_table, 4) || misaligned(rows_out, 4) ||
      misaligned(cursor, 8) || misaligned(cursor_out, 8) || misaligned(slots, 8))
    return FC_EINVAL;
  if (rows_out == add || rows_out == free_pages || block_table == rows || block_table == add || block_table == free_pages) return FC_EINVAL;
  hipError_t e = assign_pages_launch(rows, add, add_each, batch, layers, kv_heads, page_size, max_pages, free_pages, num_free, block_table,
                                     cursor, slots, slots_per_seq, rows_out, cursor_out, static_cast<hipStream_t>(hip_stream));
  return e == hipSuccess ? FC_OK : FC_EHIP;
}

static fc_status check_mx_pages(int32_t page_size, int32_t head_dim, int64_t num_pages) {
  if (page_size < 1 || num_pages < 1 || head_dim < 1) return FC_EINVAL;
  if (head_dim != 64 && head_dim != 128) return FC_EUNSUPPORTED;
  if (page_size % 16 || page_size > (1 << 25)) return FC_EUNSUPPORTED;
  if (num_pages * (page_size / 16) > 0x7FFFFFFFll) return FC_EUNSUPPORTED;      // (2 TB and more)
  return FC_OK;
}

size_t flashcache_mx_page_bytes(int32_t page_size, int32_t head_dim) {
  return check_mx_pages(page_size, head_dim, 1) == FC_OK ? (size_t)(page_size / 16) * 17 * head_dim : 0;
}

static fc_status check_mx_rows(const fc_rows_desc* d, const void* K, const void* V, const int64_t* slots, const void* pages,
                               int32_t page_size, int64_t num_pages) {
  if (!d || d->batch < 0 || d->rows < 0 || d->head_dim < 1) return FC_EINVAL;
  if (d->dtype != FC_F32 && d->dtype != FC_BF16) return FC_EINVAL;
  fc_status st = check_mx_pages(page_size, d->head_dim, num_pages);
  if (st != FC_OK) return st;
  const int64_t e = d->dtype == FC_BF16 ? 2 : 4;
  if (d->stride_b < 0 || d->stride_r < 0 || (d->batch > 1 && (d->stride_b * e) % 16) || (d->rows > 1 && (d->stride_r * e) % 16)) return FC_EINVAL;
  // (a workgroup of 256 threads has 32 rows, the last one fewer, and a launch fewer than 2^32 threads)
  if (d->batch > 65535 || d->rows > (1 << 29) - 32) return FC_EUNSUPPORTED;
  if (d->batch == 0 || d->rows == 0) return FC_OK;
  if (!K || !V || !slots || !pages) return FC_EINVAL;
  if (!aligned16(K) || !aligned16(V) || !aligned16(pages) || (reinterpret_cast<uintptr_t>(slots) & 7u)) return FC_EINVAL;
  return FC_OK;
}

fc_status flashcache_mx_store(const void* K, const void* V, const fc_rows_desc* desc, const int64_t* slots, int32_t page_size,
                              int64_t num_pages, void* pages, void* hip_stream) {
  fc_status st = check_mx_rows(desc, K, V, slots, pages, page_size, num_pages);
  if (st != FC_OK || desc->batch == 0 || desc->rows == 0) return st;
  hipError_t e = mx_store_launch(K, V, *desc, slots, pages, num_pages * page_size, static_cast<hipStream_t>(hip_stream));
  return e == hipSuccess ? FC_OK : FC_EHIP;
}

fc_status flashcache_mx_load(const int64_t* slots, const void* pages, int32_t page_size, int64_t num_pages,
                             const fc_rows_desc* desc, void* K, void* V, void* hip_stream) {
  fc_status st = check_mx_rows(desc, K, V, slots, pages, page_size, num_pages);
  if (st != FC_OK || desc->batch == 0 || desc->rows == 0) return st;
  // rows of the output must not lie on one another
  if ((desc->rows > 1 && desc->stride_r < desc->head_dim) || (desc->batch > 1 && desc->stride_b < desc->head_dim)) return FC_EINVAL;
  hipError_t e = mx_load_launch(*desc, slots, pages, num_pages * page_size, K, V, static_cast<hipStream_t>(hip_stream));
  return e == hipSuccess ? FC_OK : FC_EHIP;
}

fc_status flashcache_select_gather_mx(const void* K, const void* V, const fc_kv_desc* desc, const float* scores,
                                      const int32_t* budgets, const int64_t* layer_offsets, int64_t rows_per_seq,
                                      int32_t shared, int32_t* idx_out, const int32_t* block_table, int32_t page_size,
                                      int32_t max_pages, int64_t num_pages, void* pages, void* hip_stream) {
  fc_status st = check_desc(desc);
  if (st != FC_OK) return st;
  if (max_pages < 1) return FC_EINVAL;
  st = check_mx_pages(page_size, desc->head_dim, num_pages);
  if (st != FC_OK) return st;
  if ((int64_t)desc->kv_heads * desc->n_tokens > 0xFFFFFFFFll || desc->batch > 65535 || rows_per_seq >= (1 << 29)) return FC_EUNSUPPORTED;
  if (!block_table || (reinterpret_cast<uintptr_t>(block_table) & 3u)) return FC_EINVAL;
  if (desc->batch > 0 && rows_per_seq > 0 && (!pages || !aligned16(pages))) return FC_EINVAL;
  st = select_gather_common(K, V, desc, scores, budgets, layer_offsets, rows_per_seq, shared != 0, idx_out, nullptr, nullptr, nullptr, 0, 0,
                            0, hip_stream, false);
  if (st != FC_OK || desc->batch == 0 || rows_per_seq == 0) return st;
  hipError_t e = mx_gather_launch(K, V, *desc, budgets, layer_offsets, rows_per_seq, idx_out, block_table, page_size, max_pages, pages,
                                  num_pages * page_size, static_cast<hipStream_t>(hip_stream));
  return e == hipSuccess ? FC_OK : FC_EHIP;
}

static bool mx_decode_shape(int32_t batch, int32_t layers, int32_t kv_heads, int32_t q_heads) {
  return batch >= 0 && layers >= 1 && kv_heads >= 1 && q_heads >= kv_heads && q_heads % kv_heads == 0;
}

size_t flashcache_mx_decode_workspace_bytes(int32_t batch, int32_t layers, int32_t kv_heads, int32_t q_heads, int32_t head_dim) {
  if (!mx_decode_shape(batch, layers, kv_heads, q_heads) || !mx_decode_supported(q_heads / kv_heads, head_dim)) return 0;
  if ((int64_t)batch * layers * kv_heads > kMaxUnits) return 0;
  return mx_decode_workspace_bytes(batch * layers * kv_heads, q_heads / kv_heads, head_dim);
}

fc_status flashcache_mx_decode_attention(const void* Q, const void* pages, const int32_t* block_table, int32_t page_size,
                                         int32_t max_pages, int64_t num_pages, int32_t batch, int32_t layers,
                                         int32_t kv_heads, int32_t q_heads, int32_t head_dim, int32_t dtype,
                                         const int32_t* rows, float scale, float* out, void* workspace,
                                         size_t workspace_bytes, void* hip_stream) {
  if (!mx_decode_shape(batch, layers, kv_heads, q_heads) || head_dim < 1) return FC_EINVAL;
  if (dtype != FC_F32 && dtype != FC_BF16) return FC_EINVAL;
  if (max_pages < 1 || !(scale == scale)) return FC_EINVAL;
  fc_status st = check_mx_pages(page_size, head_dim, num_pages);
  if (st != FC_OK) return st;
  if (!mx_decode_supported(q_heads / kv_heads, head_dim)) return FC_EUNSUPPORTED;
  if ((int64_t)batch * layers * kv_heads > kMaxUnits) return FC_EUNSUPPORTED;
  if (!mx_decode_reach((int64_t)batch * layers * kv_heads, max_pages, page_size)) return FC_EUNSUPPORTED;
  if (batch == 0) return FC_OK;
  if (!Q || !pages || !block_table || !rows || !out) return FC_EINVAL;
  if (!aligned16(Q) || !aligned16(pages) || !aligned16(out)) return FC_EINVAL;
  if ((reinterpret_cast<uintptr_t>(rows) & 3u) || (reinterpret_cast<uintptr_t>(block_table) & 3u)) return FC_EINVAL;
  const size_t need = mx_decode_workspace_bytes(batch * layers * kv_heads, q_heads / kv_heads, head_dim);
  if (!workspace || !aligned16(workspace) || workspace_bytes < need) return FC_EWORKSPACE;
  hipError_t e = mx_decode_launch(Q, pages, block_table, page_size, max_pages, num_pages, batch, layers, kv_heads, q_heads / kv_heads,
                                  head_dim, dtype, rows, scale, out, workspace, static_cast<hipStream_t>(hip_stream));
  return e == hipSuccess ? FC_OK : FC_EHIP;
}

// A paged cache's shape; what is of a sequence has to fit between one and the next unless it is the same for all.
static fc_status check_paged(const fc_paged_kv* kv) {
  if (!kv || kv->batch < 0 || kv->layers < 1 || kv->kv_heads < 1 || kv->head_dim < 1 || kv->page_size < 1 || kv->max_pages < 1 || kv->num_pages < 1) return FC_EINVAL;
  if (kv->dtype != FC_F32 && kv->dtype != FC_BF16) return FC_EINVAL;
  if (kv->batch > 1 && (kv->rows_stride_b < 0 || kv->table_stride_b < 0)) return FC_EINVAL;
  if (((int64_t)kv->head_dim * (kv->dtype == FC_BF16 ? 2 : 4)) % 16) return FC_EINVAL;
  if (kv->head_dim > 512) return FC_EUNSUPPORTED;
  if ((int64_t)kv->batch * kv->layers * kv->kv_heads > kMaxUnits) return FC_EUNSUPPORTED;
  if (kv->page_size > (1 << 25) || kv->num_pages > 0x7FFFFFFFll || kv->num_pages * kv->page_size >= 0xFFFFFFFFll) return FC_EUNSUPPORTED;
  return FC_OK;
}

static fc_status check_paged_pointers(const fc_paged_kv* kv, bool rows_alone) {
  if (!kv->rows || !kv->block_table || (reinterpret_cast<uintptr_t>(kv->rows) & 3u) || (reinterpret_cast<uintptr_t>(kv->block_table) & 3u)) return FC_EINVAL;
  if (!rows_alone && (!kv->K || !kv->V || !aligned16(kv->K) || !aligned16(kv->V))) return FC_EINVAL;
  return FC_OK;
}

fc_status flashcache_append_paged(const fc_rotary_plan* plan, const int32_t* positions, const void* Q, void* Q_out, const fc_heads_desc* q_desc,
                                  const void* K, const fc_heads_desc* k_desc, const void* V, const fc_heads_desc* v_desc, const int64_t* slots,
                                  int64_t slots_stride_b, int64_t slots_stride_h, int32_t page_size, int64_t num_pages, void* K_pages,
                                  void* V_pages, void* bounds, void* hip_stream) {
  if (!plan || !q_desc || !k_desc || !v_desc || plan->magic != kWsMagic) return FC_EINVAL;
  if (plan->rotary_dim < 2 || plan->rotary_dim % 2 || plan->rotary_dim > 2 * FC_ROTARY_MAX_PAIRS || plan->streams < 1 || plan->streams > 4) return FC_EINVAL;
  fc_status st = check_heads(*plan, *q_desc, Q, Q_out);
  if (st != FC_OK) return st;
  // (rows of K and V go to slots: of their descriptors the input's part counts)
  for (int i = 0; i < 2; ++i) {
    fc_heads_desc d = i ? *v_desc : *k_desc;
    const void* const in = i ? V : K;
    void* const to = i ? V_pages : K_pages;
    d.out_stride_b = d.out_stride_t = d.out_stride_h = d.head_dim;
    st = check_heads(*plan, d, in, to);
    if (st != FC_OK) return st;
    if (d.batch != q_desc->batch || d.tokens != q_desc->tokens || d.head_dim != q_desc->head_dim || d.dtype != q_desc->dtype || in == to) return FC_EINVAL;
  }
  if (k_desc->heads != v_desc->heads) return FC_EINVAL;
  if (page_size < 1 || num_pages < 1) return FC_EINVAL;
  if (page_size > (1 << 25) || num_pages > 0x7FFFFFFFll || num_pages * page_size >= 0xFFFFFFFFll) return FC_EUNSUPPORTED;
  if ((int64_t)q_desc->heads + 2 * (int64_t)k_desc->heads > 65535) return FC_EUNSUPPORTED;
  if ((int64_t)q_desc->batch * q_desc->tokens == 0 || q_desc->heads + k_desc->heads == 0) return FC_OK;
  if (!positions || (reinterpret_cast<uintptr_t>(positions) & 3u)) return FC_EINVAL;
  if (reinterpret_cast<uintptr_t>(bounds) % (q_desc->dtype == FC_BF16 ? 2 : 4)) return FC_EINVAL;
  if (k_desc->heads > 0 && (!slots || (reinterpret_cast<uintptr_t>(slots) & 7u) || K_pages == V_pages || slots_stride_b < 0 || slots_stride_h < 0)) return FC_EINVAL;
  hipError_t e = append_launch(*plan, positions, Q, Q_out, *q_desc, K, *k_desc, V, *v_desc, slots, slots_stride_b, slots_stride_h, page_size, num_pages, K_pages,
                               V_pages, bounds, static_cast<hipStream_t>(hip_stream));
  return e == hipSuccess ? FC_OK : e == hipErrorInvalidConfiguration ? FC_EUNSUPPORTED : FC_EHIP;
}

fc_status flashcache_page_bounds(const fc_paged_kv* kv, void* bounds, void* hip_stream) {
  fc_status st = check_paged(kv);
  if (st != FC_OK) return st;
  if (kv->head_dim * (kv->dtype == FC_BF16 ? 2 : 4) > 1024) return FC_EUNSUPPORTED;
  if (kv->batch == 0) return FC_OK;
  st = check_paged_pointers(kv, true);
  if (st != FC_OK) return st;
  if (!kv->K || !aligned16(kv->K) || !bounds || !aligned16(bounds)) return FC_EINVAL;
  hipError_t e = page_bounds_launch(*kv, bounds, static_cast<hipStream_t>(hip_stream));
  return e == hipSuccess ? FC_OK : FC_EHIP;
}

// What the attention kernels and the choice of pages take.
static fc_status check_attended(const fc_paged_kv* kv, int32_t q_heads) {
  fc_status st = check_paged(kv);
  if (st != FC_OK) return st;
  if (q_heads < kv->kv_heads || q_heads % kv->kv_heads) return FC_EINVAL;
  return attend_supported(q_heads / kv->kv_heads, kv->head_dim) ? FC_OK : FC_EUNSUPPORTED;
}

size_t flashcache_choose_pages_workspace_bytes(const fc_paged_kv* kv) {
  return check_paged(kv) == FC_OK ? choose_workspace_bytes((int64_t)kv->batch * kv->layers * kv->kv_heads, kv->max_pages) : 0;
}

fc_status flashcache_choose_pages(const void* Q, int32_t q_heads, const fc_paged_kv* kv, const void* bounds, int32_t count, int32_t first,
                                  int32_t last, int32_t* chosen, void* workspace, size_t workspace_bytes, void* hip_stream) {
  fc_status st = check_attended(kv, q_heads);
  if (st != FC_OK) return st;
  if (count < 1 || first < 0 || last < 0 || (int64_t)first + last > count) return FC_EINVAL;
  if (count >= 1 << 30) return FC_EUNSUPPORTED;
  if (kv->batch == 0) return FC_OK;
  st = check_paged_pointers(kv, true);
  if (st != FC_OK) return st;
  if (!Q || !bounds || !chosen || !aligned16(Q) || !aligned16(bounds) || (reinterpret_cast<uintptr_t>(chosen) & 3u)) return FC_EINVAL;
  if (!workspace || !aligned16(workspace) || workspace_bytes < flashcache_choose_pages_workspace_bytes(kv)) return FC_EWORKSPACE;
  hipError_t e = choose_launch(Q, q_heads / kv->kv_heads, *kv, bounds, count, first, last, chosen, workspace, static_cast<hipStream_t>(hip_stream));
  return e == hipSuccess ? FC_OK : FC_EHIP;
}

size_t flashcache_decode_chosen_workspace_bytes(const fc_paged_kv* kv, int32_t q_heads, int32_t count) {
  if (check_attended(kv, q_heads) != FC_OK || kv->batch == 0 || count < 1 || (int64_t)count * kv->page_size >= (1 << 30)) return 0;
  return attend_chosen_workspace_bytes(kv->batch * kv->layers * kv->kv_heads, q_heads / kv->kv_heads, kv->head_dim, kv->dtype, kv->page_size, count);
}

fc_status flashcache_decode_attention_chosen(const void* Q, int32_t q_heads, const fc_paged_kv* kv, const int32_t* chosen, int32_t count, float scale,
                                             float* out, void* workspace, size_t workspace_bytes, void* hip_stream) {
  fc_status st = check_attended(kv, q_heads);
  if (st != FC_OK) return st;
  if (count < 1 || !(scale == scale)) return FC_EINVAL;
  if ((int64_t)count * kv->page_size >= (1 << 30)) return FC_EUNSUPPORTED;
  if (kv->batch == 0) return FC_OK;
  st = check_paged_pointers(kv, false);
  if (st != FC_OK) return st;
  if (!Q || !out || !chosen || !aligned16(Q) || !aligned16(out) || (reinterpret_cast<uintptr_t>(chosen) & 3u)) return FC_EINVAL;
  const size_t need = flashcache_decode_chosen_workspace_bytes(kv, q_heads, count);
  if (need && (!workspace || !aligned16(workspace) || workspace_bytes < need)) return FC_EWORKSPACE;
  hipError_t e = attend_chosen_launch(Q, q_heads / kv->kv_heads, *kv, chosen, count, scale, out, workspace, static_cast<hipStream_t>(hip_stream));
  return e == hipSuccess ? FC_OK : FC_EHIP;
}

size_t flashcache_decode_shared_workspace_bytes(int32_t prompts, int32_t batch, int32_t layers, int32_t kv_heads, int32_t q_heads, int32_t head_dim,
                                                int32_t dtype) {
  if (prompts < 0 || batch < 1 || layers < 1 || kv_heads < 1 || q_heads < kv_heads || q_heads % kv_heads || (dtype != FC_F32 && dtype != FC_BF16)) return 0;
  if (!attend_supported(q_heads / kv_heads, head_dim) || (int64_t)batch * layers * kv_heads > kMaxUnits || (int64_t)prompts * layers * kv_heads > kMaxUnits)
    return 0;
  return attend_shared_workspace_bytes(prompts, batch, layers, kv_heads, q_heads / kv_heads, head_dim, dtype);
}

fc_status flashcache_decode_attention_shared(const void* Q, int32_t q_heads, const fc_paged_kv* common, const int32_t* starts, const fc_paged_kv* own,
                                             float scale, float* out, void* workspace, size_t workspace_bytes, void* hip_stream) {
  fc_status st = check_attended(own, q_heads);
  if (st == FC_OK) st = check_attended(common, q_heads);
  if (st != FC_OK) return st;
  if (common->layers != own->layers || common->kv_heads != own->kv_heads || common->head_dim != own->head_dim || common->dtype != own->dtype) return FC_EINVAL;
  if (!(scale == scale)) return FC_EINVAL;
  if (own->batch == 0) return FC_OK;
  st = check_paged_pointers(own, false);
  if (st == FC_OK && common->batch > 0) st = check_paged_pointers(common, false);
  if (st != FC_OK) return st;
  if (!Q || !out || !starts || !aligned16(Q) || !aligned16(out) || (reinterpret_cast<uintptr_t>(starts) & 3u)) return FC_EINVAL;
  const size_t need = flashcache_decode_shared_workspace_bytes(common->batch, own->batch, own->layers, own->kv_heads, q_heads, own->head_dim, own->dtype);
  if (!workspace || !aligned16(workspace) || workspace_bytes < need) return FC_EWORKSPACE;
  hipError_t e = attend_shared_launch(Q, q_heads / own->kv_heads, *common, starts, *own, scale, out, workspace, static_cast<hipStream_t>(hip_stream));
  return e == hipSuccess ? FC_OK : FC_EHIP;
}

const char* flashcache_status_string(int32_t status) {
  switch (status) {
    case FC_OK: return "FC_OK";
    case FC_EINVAL: return "FC_EINVAL: invalid argument";
    case FC_EUNSUPPORTED: return "FC_EUNSUPPORTED: no kernel for this request";
    case FC_EWORKSPACE: return "FC_EWORKSPACE: workspace missing, misaligned or too small";
    case FC_EBUDGET: return "FC_EBUDGET: infeasible budget";
    case FC_EHIP: return "FC_EHIP: HIP error";
    default: return "unknown status";
  }
}

}  // extern "C"
