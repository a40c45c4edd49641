// Internal host-side launchers (C++ linkage, not exported).  Arguments are
// validated by the C entry points in api.hip before any of these run.
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

namespace pair {

// Compute units of the current device (cached per device).
int device_cu_count();

// Whether a launch is of 2^32 threads or more: HIP counts them in 32 bits and
// starts the remainder without an error.
inline bool too_many_threads(int64_t groups, int64_t threads) {
  return groups > (int64_t)0xffffffff / threads;
}

int launch_design(int64_t B, int64_t nv, int32_t gmax, const int64_t* offsets, const float* p,
                  uint64_t seed, int64_t rep0, int64_t R, uint8_t* mask, float* pi,
                  int32_t* edge_count, int32_t* completed, int32_t* d_status, hipStream_t stream);

int launch_coeffs(int64_t B, int64_t nv, int32_t gmax, const int64_t* offsets,
                  const float* rewards, const uint8_t* mask, const float* pi, int32_t rule,
                  float wmax, float* coeff, int32_t* edge_count, float* ess, float* max_weight,
                  int32_t* d_status, hipStream_t stream);

int launch_design_coeffs(int64_t B, int64_t nv, int32_t gmax, const int64_t* offsets,
                         const float* p, const float* rewards, uint64_t seed, int64_t rep,
                         uint8_t* mask, float* pi, float* coeff, int32_t* edge_count,
                         int32_t* completed, int32_t* d_status, hipStream_t stream);

int launch_wgrad(int64_t B, int64_t nv, const int64_t* offsets, int64_t D, const void* scores,
                 int32_t dtype, int64_t ld, const float* coeff, float* out, int32_t reduce,
                 int32_t* d_status, hipStream_t stream);

// The workspace a caller is asked for, and the part of it that is written.
size_t audit_workspace_bytes(int64_t B, int32_t gmax, int64_t D, int64_t R);
size_t audit_need_bytes(int64_t B, int32_t gmax, int64_t D, int64_t R);

// Prompt b of the call is prompt pbase + b of the generator's counter (its
// design draws are those of that prompt index); 0 for a whole batch.
int launch_audit(int64_t B, int64_t nv, int32_t gmax, const int64_t* offsets, int64_t D,
                 const void* scores, int64_t ld, const float* rewards, const float* p,
                 const float* pi_w, int32_t rule, float wmax, uint64_t seed, int64_t rep0,
                 int64_t pbase, int64_t R, double* mse, double* bias_norm, float* rep_sqerr,
                 int32_t* edge_count, void* workspace, int32_t* d_status, hipStream_t stream);

// pair_audit with the library's static scratch as the workspace, the prompts
// in chunks that fit it (PAIR_ESCRATCH if one prompt does not).
int64_t audit_noalloc_chunk(int64_t B, int32_t gmax, int64_t D, int64_t R);
int launch_audit_noalloc(int64_t B, int64_t nv, int32_t gmax, const int64_t* offsets, int64_t D,
                         const void* scores, int64_t ld, const float* rewards, const float* p,
                         const float* pi_w, uint64_t seed, int64_t rep0, int64_t R, double* mse,
                         double* bias_norm, float* rep_sqerr, int32_t* edge_count,
                         int32_t* d_status, hipStream_t stream);

// max_sweeps <= 0: the library's default cap on a prompt's coordinate sweeps.
int launch_alloc(int64_t B, int64_t nv, int32_t gmax, const int64_t* offsets, const float* p_hat,
                 const float* c_hat, const float* m_hat, const float* budget, float pi_min,
                 int32_t design, const float* pi_prev, int32_t max_sweeps, float* pi,
                 double* objective, int32_t* iters, double* residual, int32_t* d_status,
                 hipStream_t stream);

int launch_cps_fit(int64_t B, int64_t nv, int32_t gmax, const int64_t* offsets,
                   const float* pi_target, double* w, int32_t* n_out, float* pi_joint,
                   int32_t* iters, int32_t* d_status, hipStream_t stream);

int launch_cps_draw(int64_t B, int64_t nv, int32_t gmax, const int64_t* offsets, const double* w,
                    const int32_t* n, uint64_t seed, int64_t rep0, int64_t R, uint8_t* mask,
                    int32_t* edge_count, int32_t* d_status, hipStream_t stream);

size_t exact_workspace_bytes(int64_t B, int32_t gmax, int64_t D);

int launch_audit_exact(int64_t B, int64_t nv, int32_t gmax, const int64_t* offsets, int64_t D,
                       const void* scores, int64_t ld, const float* rewards, const float* p,
                       const float* pi_w, int32_t rule, float wmax, double* mse,
                       double* bias_norm, double* gram, void* workspace, int32_t* d_status,
                       hipStream_t stream);

size_t direction_workspace_bytes(int64_t B, int32_t gmax, int64_t D, int64_t R);

int launch_audit_direction(int64_t B, int64_t nv, int32_t gmax, const int64_t* offsets, int64_t D,
                           const void* scores, int64_t ld, const float* rewards, const float* p,
                           const float* pi_w, int32_t rule, float wmax, uint64_t seed,
                           int64_t rep0, int64_t R, double* cosine, double* target_norm,
                           void* workspace, int32_t* d_status, hipStream_t stream);

size_t clip_workspace_bytes(int64_t count);

int launch_clip(int64_t count, const void* const* grads, void* const* outs, const int64_t* sizes,
                const int32_t* dtypes, const int32_t* out_dtypes, float max_norm, float* norm,
                float* coef, void* workspace, int32_t* d_status, hipStream_t stream);

size_t page_plan_workspace_bytes(int64_t n);

int launch_page_plan(int64_t n, const int32_t* cached, const int32_t* fresh, const uint8_t* mask,
                     int32_t page, int32_t* table, int64_t ldt, int64_t capacity,
                     const int32_t* free_pages, const int64_t* free_count, int64_t max_tokens,
                     int64_t* q_offsets, int32_t* lens, int64_t* slots, int32_t* positions,
                     int32_t* free_out, int64_t* free_count_out, void* workspace,
                     int32_t* d_status, hipStream_t stream);

// A paged cache: strides in elements, of 16 bits, or (in 8 and 4 bits) in bytes.
struct PagedCache {
  int64_t page_stride, slot_stride, head_stride;
  int32_t page;
  int64_t n_pages;
};

int launch_cache_store(int64_t tokens, int32_t kv_heads, int32_t dim, const void* k, const void* v,
                       int64_t token_stride, int64_t new_head_stride, void* k_cache,
                       void* v_cache, const PagedCache& cache, const int64_t* slots,
                       int32_t* d_status, hipStream_t stream);

// The scales of a cache in 8 or 4 bits: strides in bytes.
struct PagedScales {
  const unsigned char* k;
  const unsigned char* v;
  int64_t page, slot, head;
};

// A paged cache in 8 or 4 bits, strides in bytes.
struct MxCache {
  void* k;
  void* v;
  void* k_scale;
  void* v_scale;
  int64_t page_stride, slot_stride, head_stride;
  int64_t scale_page, scale_slot, scale_head;
  int64_t n_pages;
  int32_t page, kv_heads, dim, bits;
};

// New rows into the cache (`store`), or cached ones out of it.
int launch_mx_move(bool store, const MxCache& cache, int64_t tokens, bool bf16, void* k, void* v,
                   int64_t token_stride, int64_t row_head_stride, const int64_t* slots,
                   int32_t* d_status, hipStream_t stream);

struct AttnCall {
  int64_t n, tokens;
  int32_t q_heads, kv_heads, dim;
  int32_t bits;           // of an element of the cache: 16, 8, 4
  bool bf16;
  const void* q;
  int64_t q_token, q_head;
  const void* k_cache;
  const void* v_cache;
  PagedCache cache;
  PagedScales scales;     // where bits < 16
  const int32_t* table;
  int64_t ldt;
  const int64_t* q_offsets;
  const int32_t* lens;
  int32_t max_q, max_len;
  float scale;
  void* out;
  int64_t out_token, out_head;
  float* lse;
  int32_t* d_status;
};

// Workgroups of a call's largest launch.
int64_t attention_groups(int64_t n, int64_t tokens, int32_t q_heads, int32_t kv_heads,
                         int32_t dim, int32_t bits, int32_t max_q, int32_t max_len);

size_t attention_workspace_bytes(int64_t n, int64_t tokens, int32_t q_heads, int32_t kv_heads,
                                 int32_t dim, int32_t bits, int32_t max_q, int32_t max_len);

int launch_attention(const AttnCall& call, void* workspace, hipStream_t stream);

}  // namespace pair
