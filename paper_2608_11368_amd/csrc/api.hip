// C entry points of libpair.  Every argument a host can check is checked
// here, before anything is enqueued; the kernels only see validated sizes
// and re-check device-resident offsets themselves.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <atomic>

#include "../../include/pair.h"
#include "launch.hpp"

namespace pair {

int device_cu_count() {
  static std::atomic<int> cached[64];
  int dev = 0;
  if (hipGetDevice(&dev) != hipSuccess || dev < 0) return 256;
  if (dev < 64) {
    int v = cached[dev].load(std::memory_order_relaxed);
    if (v > 0) return v;
  }
  int cus = 0;
  if (hipDeviceGetAttribute(&cus, hipDeviceAttributeMultiprocessorCount, dev) != hipSuccess ||
      cus <= 0)
    cus = 256;
  if (dev < 64) cached[dev].store(cus, std::memory_order_relaxed);
  return cus;
}

}  // namespace pair

namespace {

constexpr int64_t kMaxCount = (int64_t)1 << 40;
constexpr int64_t kMaxTensors = (int64_t)1 << 20;
constexpr int64_t kMaxRequests = (int64_t)1 << 24;
constexpr int64_t kMaxSlots = 0x7fffffff;
constexpr int32_t kMaxHeads = 1024;

bool aligned16(const void* ptr) { return (reinterpret_cast<uintptr_t>(ptr) & 15u) == 0; }

int check_groups(int64_t B, int64_t nv, int32_t gmax, const int64_t* offsets) {
  if (offsets == nullptr) return PAIR_EINVAL;
  if (B < 1 || B > 0x7fffffffLL || nv < 2 || nv > kMaxCount) return PAIR_EINVAL;
  if (gmax < 2 || gmax > PAIR_GMAX_LIMIT) return PAIR_ERANGE;
  return PAIR_OK;
}

int check_scores(const void* scores, int32_t dtype, int64_t D, int64_t ld) {
  if (scores == nullptr) return PAIR_EINVAL;
  if (dtype != PAIR_F32 && dtype != PAIR_BF16) return PAIR_EDTYPE;
  if (D < 1 || ld < D || D > kMaxCount || ld > kMaxCount) return PAIR_ERANGE;
  const int64_t elt = dtype == PAIR_BF16 ? 2 : 4;
  if (!aligned16(scores) || (ld * elt) % 16 != 0) return PAIR_EALIGN;
  return PAIR_OK;
}

// A caller's array, as the checks of overlaps see it.
struct Extent {
  const void* at;
  int64_t bytes;
};

bool overlap(const Extent& a, const Extent& b) {
  const uintptr_t x = reinterpret_cast<uintptr_t>(a.at), y = reinterpret_cast<uintptr_t>(b.at);
  return a.at != nullptr && b.at != nullptr && a.bytes > 0 && b.bytes > 0 &&
         x < y + (uint64_t)b.bytes && y < x + (uint64_t)a.bytes;
}

// Whether rows of `width` elements at all multiples of the strides, `count` of
// each, may share elements: every dimension has to reach past the smaller ones
// together (as those of any permuted or padded array do).
struct Strided {
  int64_t count, stride;
};

template <int N>
bool rows_overlap(Strided (&dims)[N], int64_t width) {
  std::sort(dims, dims + N, [](const Strided& a, const Strided& b) { return a.stride < b.stride; });
  __int128 extent = width;
  for (const Strided& d : dims) {
    if (d.count <= 1) continue;
    if (d.stride < extent) return true;
    extent += (__int128)(d.count - 1) * d.stride;
  }
  return false;
}

// Rows of `width` bytes at all multiples of the strides, in bytes, from `at` on.
struct Rows {
  const void* at;
  int64_t width;
  Strided dims[3];
};

// Steps of a distance between two rows: j * stride, least <= j <= most.
struct Steps {
  int64_t stride, least, most;
};

// Whether some choice of a step of each (those of `n`, by falling stride) brings a
// distance x to -before < x < after.  For nested arrays two or three steps of a stride
// come near at most; a search that `left` more steps do not end counts as a yes.
bool comes_near(const Steps* s, int n, __int128 x, int64_t before, int64_t after, int* left) {
  if (n == 0) return -before < x && x < after;
  __int128 low = 0, high = 0;                     // of the further steps together
  for (int k = 1; k < n; ++k) {
    low += (__int128)s[k].least * s[k].stride;
    high += (__int128)s[k].most * s[k].stride;
  }
  auto floor_div = [&](__int128 a) {
    const __int128 q = a / s->stride;
    return q * s->stride > a ? q - 1 : q;
  };
  __int128 j = floor_div(-before - x - high) + 1, last = floor_div(after - 1 - x - low);
  if (j < s->least) j = s->least;
  if (last > s->most) last = s->most;
  for (; j <= last; ++j)
    if (--*left < 0 || comes_near(s + 1, n - 1, x + j * s->stride, before, after, left)) return true;
  return false;
}

// Whether two arrays of rows share bytes; arrays that lie between each other's rows
// (a page's keys, values and scales side by side, say) do not.
bool share_bytes(const Rows& a, const Rows& b) {
  Steps steps[6];
  int n = 0;
  auto add = [&](int64_t stride, int64_t least, int64_t most) {
    if (stride > 0 && least < most) steps[n++] = {stride, least, most};
  };
  __int128 a_bytes = a.width, b_bytes = b.width;
  for (int k = 0; k < 3; ++k) {
    const Strided &x = a.dims[k], &y = b.dims[k];
    if (x.count > 1) a_bytes += (__int128)(x.count - 1) * x.stride;
    if (y.count > 1) b_bytes += (__int128)(y.count - 1) * y.stride;
    if (x.stride == y.stride) {
      add(x.stride, 1 - x.count, y.count - 1);
    } else {
      add(x.stride, 1 - x.count, 0);
      add(y.stride, 0, y.count - 1);
    }
  }
  const __int128 apart = (__int128)reinterpret_cast<uintptr_t>(b.at) -
                         (__int128)reinterpret_cast<uintptr_t>(a.at);
  if (apart >= a_bytes || -apart >= b_bytes) return false;
  std::sort(steps, steps + n, [](const Steps& x, const Steps& y) { return x.stride > y.stride; });
  int left = 4096;
  return comes_near(steps, n, apart, b.width, a.width, &left);
}

hipStream_t as_stream(void* s) { return static_cast<hipStream_t>(s); }

}  // namespace

extern "C" {

int pair_design_inclusion(int64_t B, int64_t nv, int32_t gmax, const int64_t* offsets,
                          const float* p, uint64_t seed, int64_t rep0, int64_t R, uint8_t* mask,
                          float* pi, int32_t* edge_count, int32_t* completed, int32_t* d_status,
                          void* stream) {
  int st = check_groups(B, nv, gmax, offsets);
  if (st) return st;
  if (p == nullptr) return PAIR_EINVAL;
  if (R < 1 || rep0 < 0 || R > kMaxCount || rep0 > kMaxCount) return PAIR_ERANGE;
  if (mask == nullptr && pi == nullptr && edge_count == nullptr && completed == nullptr)
    return PAIR_EINVAL;
  if (mask != nullptr && R > kMaxCount / nv) return PAIR_ERANGE;
  if ((edge_count != nullptr || completed != nullptr) && R > kMaxCount / B) return PAIR_ERANGE;
  return pair::launch_design(B, nv, gmax, offsets, p, seed, rep0, R, mask, pi, edge_count,
                             completed, d_status, as_stream(stream));
}

static int check_rule(int32_t rule, float wmax) {
  if (rule < PAIR_RULE_HT || rule > PAIR_RULE_MARGINAL) return PAIR_EINVAL;
  if (rule == PAIR_RULE_CLIPPED && !(wmax > 0.0f && wmax <= 3.4e38f)) return PAIR_EINVAL;
  return PAIR_OK;
}

int pair_edge_coeffs_rule(int64_t B, int64_t nv, int32_t gmax, const int64_t* offsets,
                          const float* rewards, const uint8_t* mask, const float* pi,
                          int32_t rule, float wmax, float* coeff, int32_t* edge_count, float* ess,
                          float* max_weight, int32_t* d_status, void* stream) {
  int st = check_groups(B, nv, gmax, offsets);
  if (st) return st;
  st = check_rule(rule, wmax);
  if (st) return st;
  if (rewards == nullptr || coeff == nullptr) return PAIR_EINVAL;
  return pair::launch_coeffs(B, nv, gmax, offsets, rewards, mask, pi, rule, wmax, coeff,
                             edge_count, ess, max_weight, d_status, as_stream(stream));
}

int pair_design_coeffs(int64_t B, int64_t nv, int32_t gmax, const int64_t* offsets,
                       const float* p, const float* rewards, uint64_t seed, int64_t rep,
                       uint8_t* mask, float* pi, float* coeff, int32_t* edge_count,
                       int32_t* completed, int32_t* d_status, void* stream) {
  int st = check_groups(B, nv, gmax, offsets);
  if (st) return st;
  if (p == nullptr || rewards == nullptr || coeff == nullptr) return PAIR_EINVAL;
  if (rep < 0 || rep > kMaxCount) return PAIR_ERANGE;
  return pair::launch_design_coeffs(B, nv, gmax, offsets, p, rewards, seed, rep, mask, pi, coeff,
                                    edge_count, completed, d_status, as_stream(stream));
}

int pair_edge_coeffs(int64_t B, int64_t nv, int32_t gmax, const int64_t* offsets,
                     const float* rewards, const uint8_t* mask, const float* pi, float* coeff,
                     int32_t* edge_count, int32_t* d_status, void* stream) {
  return pair_edge_coeffs_rule(B, nv, gmax, offsets, rewards, mask, pi, PAIR_RULE_HT, 0.0f, coeff,
                               edge_count, nullptr, nullptr, d_status, stream);
}

int pair_weighted_grad(int64_t B, int64_t nv, const int64_t* offsets, int64_t D,
                       const void* scores, int32_t dtype, int64_t ld, const float* coeff,
                       float* out, int32_t reduce, int32_t* d_status, void* stream) {
  if (offsets == nullptr || coeff == nullptr || out == nullptr) return PAIR_EINVAL;
  if (reduce != 0 && reduce != 1) return PAIR_EINVAL;
  if (B < 1 || B > 0x7fffffffLL || nv < 0 || nv > kMaxCount) return PAIR_EINVAL;
  int st = check_scores(scores, dtype, D, ld);
  if (st) return st;
  if (B > kMaxCount / D) return PAIR_ERANGE;
  return pair::launch_wgrad(B, nv, offsets, D, scores, dtype, ld, coeff, out, reduce, d_status,
                            as_stream(stream));
}

size_t pair_audit_workspace_bytes(int64_t B, int32_t gmax, int64_t D, int64_t R) {
  if (B < 1 || gmax < 2 || gmax > PAIR_GMAX_LIMIT || D < 1 || R < 1 || R > kMaxCount ||
      B > kMaxCount / (R + 1))
    return 0;
  return pair::audit_workspace_bytes(B, gmax, D, R);
}

int pair_audit_rule(int64_t B, int64_t nv, int32_t gmax, const int64_t* offsets, int64_t D,
                    const void* scores, int32_t dtype, int64_t ld, const float* rewards,
                    const float* p, const float* pi_w, int32_t rule, float wmax, uint64_t seed,
                    int64_t rep0, int64_t R, double* mse, double* bias_norm, float* rep_sqerr,
                    int32_t* edge_count, void* workspace, size_t ws_bytes, int32_t* d_status,
                    void* stream) {
  int st = check_groups(B, nv, gmax, offsets);
  if (st) return st;
  st = check_rule(rule, wmax);
  if (st) return st;
  if (dtype != PAIR_BF16) return PAIR_EDTYPE;
  st = check_scores(scores, dtype, D, ld);
  if (st) return st;
  if (rewards == nullptr || p == nullptr || mse == nullptr || bias_norm == nullptr)
    return PAIR_EINVAL;
  if (R < 1 || rep0 < 0 || R > kMaxCount || rep0 > kMaxCount) return PAIR_ERANGE;
  const size_t need = pair_audit_workspace_bytes(B, gmax, D, R);
  if (need == 0) return PAIR_ERANGE;
  if (workspace == nullptr || (reinterpret_cast<uintptr_t>(workspace) & 255u) != 0 ||
      ws_bytes < need)
    return PAIR_EWORKSPACE;
  return pair::launch_audit(B, nv, gmax, offsets, D, scores, ld, rewards, p, pi_w, rule, wmax,
                            seed, rep0, 0, R,
                            mse, bias_norm, rep_sqerr, edge_count, workspace, d_status,
                            as_stream(stream));
}

size_t pair_audit_direction_workspace_bytes(int64_t B, int32_t gmax, int64_t D, int64_t R) {
  if (B < 1 || gmax < 2 || gmax > PAIR_GMAX_LIMIT || D < 1 || D > kMaxCount || R < 1 ||
      R > kMaxCount || B > kMaxCount / (R + 1))
    return 0;
  return pair::direction_workspace_bytes(B, gmax, D, R);
}

int pair_audit_direction(int64_t B, int64_t nv, int32_t gmax, const int64_t* offsets, int64_t D,
                         const void* scores, int32_t dtype, int64_t ld, const float* rewards,
                         const float* p, const float* pi_w, int32_t rule, float wmax,
                         uint64_t seed, int64_t rep0, int64_t R, double* cosine,
                         double* target_norm, void* workspace, size_t ws_bytes,
                         int32_t* d_status, void* stream) {
  int st = check_groups(B, nv, gmax, offsets);
  if (st) return st;
  st = check_rule(rule, wmax);
  if (st) return st;
  if (dtype != PAIR_BF16) return PAIR_EDTYPE;
  st = check_scores(scores, dtype, D, ld);
  if (st) return st;
  if (rewards == nullptr || p == nullptr || cosine == nullptr || target_norm == nullptr)
    return PAIR_EINVAL;
  if (R < 1 || rep0 < 0 || R > kMaxCount || rep0 > kMaxCount) return PAIR_ERANGE;
  const size_t need = pair_audit_direction_workspace_bytes(B, gmax, D, R);
  if (need == 0) return PAIR_ERANGE;
  if (workspace == nullptr || (reinterpret_cast<uintptr_t>(workspace) & 255u) != 0 ||
      ws_bytes < need)
    return PAIR_EWORKSPACE;
  return pair::launch_audit_direction(B, nv, gmax, offsets, D, scores, ld, rewards, p, pi_w, rule,
                                      wmax, seed, rep0, R, cosine, target_norm, workspace,
                                      d_status, as_stream(stream));
}

int pair_design_alloc_ex(int64_t B, int64_t nv, int32_t gmax, const int64_t* offsets,
                         const float* p_hat, const float* c_hat, const float* m_hat,
                         const float* budget, float pi_min, int32_t design, const float* pi_prev,
                         int32_t max_sweeps, float* pi, double* objective, int32_t* iters,
                         double* residual, int32_t* d_status, void* stream) {
  if (offsets == nullptr || p_hat == nullptr || c_hat == nullptr || budget == nullptr ||
      pi == nullptr)
    return PAIR_EINVAL;
  if (B < 1 || B > 0x7fffffffLL || nv < 0 || nv > kMaxCount) return PAIR_EINVAL;
  if (gmax < 1 || gmax > PAIR_GMAX_LIMIT) return PAIR_ERANGE;
  if (design < PAIR_DESIGN_PAIR || design > PAIR_DESIGN_UNIFORM) return PAIR_EINVAL;
  if (!(pi_min > 0.0f && pi_min <= 1.0f)) return PAIR_ERANGE;
  if (max_sweeps < 0) return PAIR_ERANGE;
  return pair::launch_alloc(B, nv, gmax, offsets, p_hat, c_hat, m_hat, budget, pi_min, design,
                            pi_prev, max_sweeps, pi, objective, iters, residual, d_status,
                            as_stream(stream));
}

int pair_design_alloc(int64_t B, int64_t nv, int32_t gmax, const int64_t* offsets,
                      const float* p_hat, const float* c_hat, const float* m_hat,
                      const float* budget, float pi_min, int32_t design, float* pi,
                      double* objective, int32_t* iters, int32_t* d_status, void* stream) {
  return pair_design_alloc_ex(B, nv, gmax, offsets, p_hat, c_hat, m_hat, budget, pi_min, design,
                              nullptr, 0, pi, objective, iters, nullptr, d_status, stream);
}

int pair_cps_fit(int64_t B, int64_t nv, int32_t gmax, const int64_t* offsets,
                 const float* pi_target, double* w, int32_t* n_out, float* pi_joint,
                 int32_t* iters, int32_t* d_status, void* stream) {
  int st = check_groups(B, nv, gmax, offsets);
  if (st) return st;
  if (pi_target == nullptr || w == nullptr) return PAIR_EINVAL;
  return pair::launch_cps_fit(B, nv, gmax, offsets, pi_target, w, n_out, pi_joint, iters,
                              d_status, as_stream(stream));
}

int pair_cps_draw(int64_t B, int64_t nv, int32_t gmax, const int64_t* offsets, const double* w,
                  const int32_t* n, uint64_t seed, int64_t rep0, int64_t R, uint8_t* mask,
                  int32_t* edge_count, int32_t* d_status, void* stream) {
  if (offsets == nullptr || w == nullptr || n == nullptr || mask == nullptr) return PAIR_EINVAL;
  if (B < 1 || B > 0x7fffffffLL || nv < 0 || nv > kMaxCount) return PAIR_EINVAL;
  if (gmax < 1 || gmax > PAIR_GMAX_LIMIT) return PAIR_ERANGE;
  if (R < 1 || rep0 < 0 || R > kMaxCount || rep0 > kMaxCount || R > kMaxCount / (nv > 0 ? nv : 1))
    return PAIR_ERANGE;
  return pair::launch_cps_draw(B, nv, gmax, offsets, w, n, seed, rep0, R, mask, edge_count,
                               d_status, as_stream(stream));
}

size_t pair_audit_exact_workspace_bytes(int64_t B, int32_t gmax, int64_t D) {
  if (B < 1 || gmax < 2 || gmax > PAIR_GMAX_LIMIT || D < 1 || D > kMaxCount) return 0;
  return pair::exact_workspace_bytes(B, gmax, D);
}

int pair_audit_exact(int64_t B, int64_t nv, int32_t gmax, const int64_t* offsets, int64_t D,
                     const void* scores, int32_t dtype, int64_t ld, const float* rewards,
                     const float* p, const float* pi_w, int32_t rule, float wmax, double* mse,
                     double* bias_norm, double* gram, void* workspace, size_t ws_bytes,
                     int32_t* d_status, void* stream) {
  int st = check_groups(B, nv, gmax, offsets);
  if (st) return st;
  st = check_rule(rule, wmax);
  if (st) return st;
  if (rule == PAIR_RULE_RATIO_KE || rule == PAIR_RULE_SELFNORM) return PAIR_EINVAL;
  if (dtype != PAIR_BF16) return PAIR_EDTYPE;
  st = check_scores(scores, dtype, D, ld);
  if (st) return st;
  if (rewards == nullptr || p == nullptr || mse == nullptr || bias_norm == nullptr)
    return PAIR_EINVAL;
  const size_t need = pair_audit_exact_workspace_bytes(B, gmax, D);
  if (need == 0) return PAIR_ERANGE;
  if (workspace == nullptr || (reinterpret_cast<uintptr_t>(workspace) & 255u) != 0 ||
      ws_bytes < need)
    return PAIR_EWORKSPACE;
  return pair::launch_audit_exact(B, nv, gmax, offsets, D, scores, ld, rewards, p, pi_w, rule,
                                  wmax, mse, bias_norm, gram, workspace, d_status,
                                  as_stream(stream));
}

int pair_audit(int64_t B, int64_t nv, int32_t gmax, const int64_t* offsets, int64_t D,
               const void* scores, int32_t dtype, int64_t ld, const float* rewards,
               const float* p, const float* pi_w, uint64_t seed, int64_t rep0, int64_t R,
               double* mse, double* bias_norm, float* rep_sqerr, int32_t* edge_count,
               void* workspace, size_t ws_bytes, int32_t* d_status, void* stream) {
  return pair_audit_rule(B, nv, gmax, offsets, D, scores, dtype, ld, rewards, p, pi_w,
                         PAIR_RULE_HT, 0.0f, seed, rep0, R, mse, bias_norm, rep_sqerr, edge_count,
                         workspace, ws_bytes, d_status, stream);
}

int pair_audit_noalloc(int64_t B, int64_t nv, int32_t gmax, const int64_t* offsets, int64_t D,
                       const void* scores, int32_t dtype, int64_t ld, const float* rewards,
                       const float* p, const float* pi_w, uint64_t seed, int64_t rep0, int64_t R,
                       double* mse, double* bias_norm, float* rep_sqerr, int32_t* edge_count,
                       int32_t* d_status, void* stream) {
  int st = check_groups(B, nv, gmax, offsets);
  if (st) return st;
  if (dtype != PAIR_BF16) return PAIR_EDTYPE;
  st = check_scores(scores, dtype, D, ld);
  if (st) return st;
  if (rewards == nullptr || p == nullptr || mse == nullptr || bias_norm == nullptr)
    return PAIR_EINVAL;
  if (R < 1 || rep0 < 0 || R > kMaxCount || rep0 > kMaxCount) return PAIR_ERANGE;
  if (pair_audit_workspace_bytes(B, gmax, D, R) == 0) return PAIR_ERANGE;
  return pair::launch_audit_noalloc(B, nv, gmax, offsets, D, scores, ld, rewards, p, pi_w, seed,
                                    rep0, R, mse, bias_norm, rep_sqerr, edge_count, d_status,
                                    as_stream(stream));
}

static bool bad_workspace(const void* workspace, size_t ws_bytes, size_t need) {
  return workspace == nullptr || (reinterpret_cast<uintptr_t>(workspace) & 255u) != 0 ||
         ws_bytes < need;
}

size_t pair_clip_grads_workspace_bytes(int64_t count) {
  return count < 0 || count > kMaxTensors ? 0 : pair::clip_workspace_bytes(count);
}

int pair_clip_grads(int64_t count, const void* const* grads, void* const* outs,
                    const int64_t* sizes, const int32_t* dtypes, const int32_t* out_dtypes,
                    float max_norm, float* norm, float* coef, void* workspace, size_t ws_bytes,
                    int32_t* d_status, void* stream) {
  if (count < 0 || count > kMaxTensors) return PAIR_ERANGE;
  if (norm == nullptr || coef == nullptr) return PAIR_EINVAL;
  if (count > 0 && (grads == nullptr || sizes == nullptr || dtypes == nullptr)) return PAIR_EINVAL;
  if (count > 0 && outs != nullptr && out_dtypes == nullptr) return PAIR_EINVAL;
  if (!(max_norm > 0.0f)) return PAIR_ERANGE;
  int64_t total = 0;
  for (int64_t i = 0; i < count; ++i) {
    const int32_t t = dtypes[i];
    if (t != PAIR_F32 && t != PAIR_BF16 && t != PAIR_F16) return PAIR_EDTYPE;
    if (outs != nullptr && out_dtypes[i] != t && out_dtypes[i] != PAIR_F32) return PAIR_EDTYPE;
    if (sizes[i] < 0 || sizes[i] > kMaxCount || (total += sizes[i]) > kMaxCount) return PAIR_ERANGE;
    if (sizes[i] == 0) continue;
    if (grads[i] == nullptr || (outs != nullptr && outs[i] == nullptr)) return PAIR_EINVAL;
    const uintptr_t unit = t == PAIR_F32 ? 4 : 2;
    if (reinterpret_cast<uintptr_t>(grads[i]) % unit != 0) return PAIR_EALIGN;
    if (outs != nullptr &&
        reinterpret_cast<uintptr_t>(outs[i]) % (out_dtypes[i] == PAIR_F32 ? 4 : 2) != 0)
      return PAIR_EALIGN;
  }
  if (bad_workspace(workspace, ws_bytes, pair::clip_workspace_bytes(count))) return PAIR_EWORKSPACE;
  return pair::launch_clip(count, grads, outs, sizes, dtypes, out_dtypes, max_norm, norm, coef,
                           workspace, d_status, as_stream(stream));
}

size_t pair_page_plan_workspace_bytes(int64_t n) {
  return n < 1 || n > kMaxRequests ? 0 : pair::page_plan_workspace_bytes(n);
}

int pair_page_plan(int64_t n, const int32_t* cached, const int32_t* fresh, const uint8_t* mask,
                   int32_t page, int32_t* table, int64_t ldt, int64_t capacity,
                   const int32_t* free_pages, const int64_t* free_count, int64_t max_tokens,
                   int64_t* q_offsets, int32_t* lens, int64_t* slots, int32_t* positions,
                   int32_t* free_out, int64_t* free_count_out, void* workspace, size_t ws_bytes,
                   int32_t* d_status, void* stream) {
  if (cached == nullptr || fresh == nullptr || table == nullptr || free_count == nullptr ||
      q_offsets == nullptr || lens == nullptr || free_count_out == nullptr)
    return PAIR_EINVAL;
  if (n < 1 || n > kMaxRequests || page < 1 || ldt < 1 || ldt > kMaxSlots / n) return PAIR_ERANGE;
  if (capacity < 0 || capacity > kMaxSlots / page || max_tokens < 0 || max_tokens > kMaxSlots)
    return PAIR_ERANGE;
  if (capacity > 0 && (free_pages == nullptr || free_out == nullptr || free_pages == free_out))
    return PAIR_EINVAL;
  if (max_tokens > 0 && slots == nullptr) return PAIR_EINVAL;
  if (bad_workspace(workspace, ws_bytes, pair::page_plan_workspace_bytes(n)))
    return PAIR_EWORKSPACE;
  // Every workgroup reads all lengths and the pool while others write.
  const Extent in[] = {{cached, n * 4}, {fresh, n * 4}, {mask, n}, {free_pages, capacity * 4},
                       {free_count, 8}};
  const Extent out[] = {{table, n * ldt * 4},   {q_offsets, (n + 1) * 8},
                        {lens, n * 4},          {slots, max_tokens * 8},
                        {positions, max_tokens * 4}, {free_out, capacity * 4},
                        {free_count_out, 8},    {workspace, (int64_t)pair::page_plan_workspace_bytes(n)},
                        {d_status, 4}};
  constexpr int kOuts = sizeof(out) / sizeof(out[0]);
  for (int i = 0; i < kOuts; ++i) {
    for (const Extent& e : in)
      if (overlap(out[i], e)) return PAIR_EINVAL;
    for (int k = 0; k < i; ++k)
      if (overlap(out[i], out[k])) return PAIR_EINVAL;
  }
  return pair::launch_page_plan(n, cached, fresh, mask, page, table, ldt, capacity, free_pages,
                                free_count, max_tokens, q_offsets, lens, slots, positions,
                                free_out, free_count_out, workspace, d_status, as_stream(stream));
}

// Layout of a paged cache: 16-byte pieces, slots numbered in 31 bits.
static int check_cache(const void* k_cache, const void* v_cache, int64_t page_stride,
                       int64_t slot_stride, int64_t head_stride, int32_t page, int64_t n_pages) {
  if (k_cache == nullptr || v_cache == nullptr) return PAIR_EINVAL;
  if (page < 1 || n_pages < 1 || n_pages > kMaxSlots / page) return PAIR_ERANGE;
  if (page_stride < 0 || slot_stride < 0 || head_stride < 0 || page_stride > kMaxCount ||
      slot_stride > kMaxCount || head_stride > kMaxCount)
    return PAIR_ERANGE;
  if (!aligned16(k_cache) || !aligned16(v_cache) || page_stride % 8 != 0 || slot_stride % 8 != 0 ||
      head_stride % 8 != 0)
    return PAIR_EALIGN;
  return PAIR_OK;
}

int pair_cache_store(int64_t tokens, int32_t kv_heads, int32_t dim, int32_t dtype, const void* k,
                     const void* v, int64_t token_stride, int64_t new_head_stride, void* k_cache,
                     void* v_cache, int64_t page_stride, int64_t slot_stride, int64_t head_stride,
                     int32_t page, int64_t n_pages, const int64_t* slots, int32_t* d_status,
                     void* stream) {
  if (dtype != PAIR_BF16 && dtype != PAIR_F16) return PAIR_EDTYPE;
  if (tokens < 0 || tokens > kMaxSlots || kv_heads < 1 || kv_heads > kMaxHeads || dim < 8 ||
      dim > 256 || dim % 8 != 0)
    return PAIR_ERANGE;
  const int st = check_cache(k_cache, v_cache, page_stride, slot_stride, head_stride, page, n_pages);
  if (st) return st;
  if (tokens == 0) return PAIR_OK;
  if (k == nullptr || v == nullptr || slots == nullptr) return PAIR_EINVAL;
  if (token_stride < 0 || new_head_stride < 0 || token_stride > kMaxCount ||
      new_head_stride > kMaxCount)
    return PAIR_ERANGE;
  if (!aligned16(k) || !aligned16(v) || token_stride % 8 != 0 || new_head_stride % 8 != 0)
    return PAIR_EALIGN;
  Strided places[] = {{n_pages, page_stride}, {page, slot_stride}, {kv_heads, head_stride}};
  if (rows_overlap(places, dim)) return PAIR_EINVAL;
  const pair::PagedCache cache = {page_stride, slot_stride, head_stride, page, n_pages};
  return pair::launch_cache_store(tokens, kv_heads, dim, k, v, token_stride, new_head_stride,
                                  k_cache, v_cache, cache, slots, d_status, as_stream(stream));
}

static int check_attention(int64_t n, int64_t tokens, int32_t q_heads, int32_t kv_heads,
                           int32_t dim, int32_t bits, int32_t max_q, int32_t max_len) {
  if (n < 1 || n > kMaxRequests || tokens < 0 || tokens > kMaxSlots) return PAIR_ERANGE;
  if (kv_heads < 1 || kv_heads > kMaxHeads || q_heads < kv_heads || q_heads % kv_heads != 0 ||
      q_heads / kv_heads > 64)
    return PAIR_ERANGE;
  if (dim != 64 && dim != 128) return PAIR_ERANGE;
  // rows and key positions are counted in 31 bits, with room for a window ahead
  if (tokens > kMaxSlots / q_heads || max_len > kMaxSlots / 2) return PAIR_ERANGE;
  if (max_q < 0 || max_len < 0 || (tokens > 0 && max_q < 1)) return PAIR_ERANGE;
  // Not counted where two workgroups a request and head and one for 64 rows, more
  // than a call has beside some thousands, are far from a launch's 2^24.
  if ((2 * n + tokens) * q_heads > (int64_t)1 << 22 &&
      pair::too_many_threads(
          pair::attention_groups(n, tokens, q_heads, kv_heads, dim, bits, max_q, max_len), 256))
    return PAIR_ERANGE;
  return PAIR_OK;
}

size_t pair_paged_attention_workspace_bytes(int64_t n, int64_t tokens, int32_t q_heads,
                                            int32_t kv_heads, int32_t dim, int32_t max_q,
                                            int32_t max_len) {
  if (check_attention(n, tokens, q_heads, kv_heads, dim, 16, max_q, max_len)) return 0;
  return pair::attention_workspace_bytes(n, tokens, q_heads, kv_heads, dim, 16, max_q, max_len);
}

// What the attention's calls share: `c` has the cache, already checked, and dim,
// kv_heads and bits.
static int attention(pair::AttnCall c, int64_t n, int64_t tokens, int32_t q_heads, int32_t dtype,
                     const void* q, int64_t q_token, int64_t q_head, const int32_t* table,
                     int64_t ldt, const int64_t* q_offsets, const int32_t* lens, int32_t max_q,
                     int32_t max_len, float scale, void* out, int64_t out_token, int64_t out_head,
                     float* lse, void* workspace, size_t ws_bytes, int32_t* d_status,
                     void* stream) {
  if (table == nullptr || q_offsets == nullptr || lens == nullptr) return PAIR_EINVAL;
  if (ldt < 1 || ldt > kMaxSlots / n) return PAIR_ERANGE;
  if (!(scale > 0.0f && scale <= 3.4e38f)) return PAIR_ERANGE;
  if (tokens == 0) return PAIR_OK;
  if (q == nullptr || out == nullptr) return PAIR_EINVAL;
  if (q_token < 0 || q_head < 0 || out_token < 0 || out_head < 0 || q_token > kMaxCount ||
      q_head > kMaxCount || out_token > kMaxCount || out_head > kMaxCount)
    return PAIR_ERANGE;
  if (!aligned16(q) || !aligned16(out) || q_token % 8 != 0 || q_head % 8 != 0 ||
      out_token % 8 != 0 || out_head % 8 != 0)
    return PAIR_EALIGN;
  Strided results[] = {{tokens, out_token}, {q_heads, out_head}};
  if (rows_overlap(results, c.dim)) return PAIR_EINVAL;
  if (bad_workspace(workspace, ws_bytes,
                    pair::attention_workspace_bytes(n, tokens, q_heads, c.kv_heads, c.dim, c.bits,
                                                    max_q, max_len)))
    return PAIR_EWORKSPACE;
  c.n = n;
  c.tokens = tokens;
  c.q_heads = q_heads;
  c.bf16 = dtype == PAIR_BF16;
  c.q = q;
  c.q_token = q_token;
  c.q_head = q_head;
  c.table = table;
  c.ldt = ldt;
  c.q_offsets = q_offsets;
  c.lens = lens;
  c.max_q = max_q;
  c.max_len = max_len;
  c.scale = scale;
  c.out = out;
  c.out_token = out_token;
  c.out_head = out_head;
  c.lse = lse;
  c.d_status = d_status;
  return pair::launch_attention(c, workspace, as_stream(stream));
}

int pair_paged_attention(int64_t n, int64_t tokens, int32_t q_heads, int32_t kv_heads, int32_t dim,
                         int32_t dtype, const void* q, int64_t q_token, int64_t q_head,
                         const void* k_cache, const void* v_cache, int64_t page_stride,
                         int64_t slot_stride, int64_t head_stride, int32_t page, int64_t n_pages,
                         const int32_t* table, int64_t ldt, const int64_t* q_offsets,
                         const int32_t* lens, int32_t max_q, int32_t max_len, float scale,
                         void* out, int64_t out_token, int64_t out_head, float* lse,
                         void* workspace, size_t ws_bytes, int32_t* d_status, void* stream) {
  if (dtype != PAIR_BF16 && dtype != PAIR_F16) return PAIR_EDTYPE;
  int st = check_attention(n, tokens, q_heads, kv_heads, dim, 16, max_q, max_len);
  if (st) return st;
  st = check_cache(k_cache, v_cache, page_stride, slot_stride, head_stride, page, n_pages);
  if (st) return st;
  pair::AttnCall c = {};
  c.kv_heads = kv_heads;
  c.dim = dim;
  c.bits = 16;
  c.k_cache = k_cache;
  c.v_cache = v_cache;
  c.cache = {page_stride, slot_stride, head_stride, page, n_pages};
  return attention(c, n, tokens, q_heads, dtype, q, q_token, q_head, table, ldt, q_offsets, lens,
                   max_q, max_len, scale, out, out_token, out_head, lse, workspace, ws_bytes,
                   d_status, stream);
}

// A cache in 8 or 4 bits; `out` is what the launches take.
static int check_mx(const pair_mx_cache* c, pair::MxCache* out) {
  if (c == nullptr || c->k == nullptr || c->v == nullptr || c->k_scale == nullptr ||
      c->v_scale == nullptr)
    return PAIR_EINVAL;
  if (c->format != PAIR_MXFP8 && c->format != PAIR_MXFP4) return PAIR_EDTYPE;
  if (c->kv_heads < 1 || c->kv_heads > kMaxHeads || c->dim < 32 || c->dim > 256 || c->dim % 32 != 0)
    return PAIR_ERANGE;
  if (c->page < 1 || c->n_pages < 1 || c->n_pages > kMaxSlots / c->page) return PAIR_ERANGE;
  const int64_t codes[] = {c->page_stride, c->slot_stride, c->head_stride};
  const int64_t scales[] = {c->scale_page, c->scale_slot, c->scale_head};
  const int blocks = c->dim / 32;
  const int unit = (blocks & -blocks) < 4 ? blocks & -blocks : 4;
  for (int64_t s : codes)
    if (s < 0 || s > kMaxCount) return PAIR_ERANGE;
  for (int64_t s : scales)
    if (s < 0 || s > kMaxCount) return PAIR_ERANGE;
  for (int64_t s : codes)
    if (s % 16 != 0) return PAIR_EALIGN;
  for (int64_t s : scales)
    if (s % unit != 0) return PAIR_EALIGN;
  if (!aligned16(c->k) || !aligned16(c->v) ||
      reinterpret_cast<uintptr_t>(c->k_scale) % unit != 0 ||
      reinterpret_cast<uintptr_t>(c->v_scale) % unit != 0)
    return PAIR_EALIGN;
  *out = {c->k,           c->v,           c->k_scale,    c->v_scale,  c->page_stride,
          c->slot_stride, c->head_stride, c->scale_page, c->scale_slot, c->scale_head,
          c->n_pages,     c->page,        c->kv_heads,   c->dim,      c->format == PAIR_MXFP8 ? 8 : 4};
  return PAIR_OK;
}

// The cache's arrays, as the checks of overlaps see them.
static void mx_arrays(const pair::MxCache& c, Rows (&to)[4]) {
  const Rows codes = {nullptr, c.dim * c.bits / 8,
                      {{c.n_pages, c.page_stride}, {c.page, c.slot_stride}, {c.kv_heads, c.head_stride}}};
  const Rows scales = {nullptr, c.dim / 32,
                       {{c.n_pages, c.scale_page}, {c.page, c.scale_slot}, {c.kv_heads, c.scale_head}}};
  to[0] = to[1] = codes;
  to[2] = to[3] = scales;
  to[0].at = c.k;
  to[1].at = c.v;
  to[2].at = c.k_scale;
  to[3].at = c.v_scale;
}

// The 16-bit rows of `at` that a call moves.
static Rows half_rows(const pair::MxCache& c, const void* at, int64_t tokens, int64_t token_stride,
                      int64_t head_stride) {
  return {at, 2 * c.dim, {{tokens, 2 * token_stride}, {1, 0}, {c.kv_heads, 2 * head_stride}}};
}

// The 16-bit rows that a call of an mx cache moves.
static int check_rows(int64_t tokens, const void* k, const void* v, int64_t token_stride,
                      int64_t head_stride, const int64_t* slots) {
  if (k == nullptr || v == nullptr || slots == nullptr) return PAIR_EINVAL;
  if (token_stride < 0 || head_stride < 0 || token_stride > kMaxCount || head_stride > kMaxCount)
    return PAIR_ERANGE;
  if (!aligned16(k) || !aligned16(v) || token_stride % 8 != 0 || head_stride % 8 != 0)
    return PAIR_EALIGN;
  return PAIR_OK;
}

int pair_cache_store_mx(const pair_mx_cache* cache, int64_t tokens, int32_t dtype, const void* k,
                        const void* v, int64_t token_stride, int64_t new_head_stride,
                        const int64_t* slots, int32_t* d_status, void* stream) {
  if (dtype != PAIR_BF16 && dtype != PAIR_F16) return PAIR_EDTYPE;
  pair::MxCache c;
  int st = check_mx(cache, &c);
  if (st) return st;
  if (tokens < 0 || tokens > kMaxSlots) return PAIR_ERANGE;
  if (tokens == 0) return PAIR_OK;
  st = check_rows(tokens, k, v, token_stride, new_head_stride, slots);
  if (st) return st;
  Strided codes[] = {{c.n_pages, c.page_stride}, {c.page, c.slot_stride}, {c.kv_heads, c.head_stride}};
  Strided scales[] = {{c.n_pages, c.scale_page}, {c.page, c.scale_slot}, {c.kv_heads, c.scale_head}};
  if (rows_overlap(codes, c.dim * c.bits / 8) || rows_overlap(scales, c.dim / 32)) return PAIR_EINVAL;
  Rows arrays[4];
  mx_arrays(c, arrays);
  for (int i = 0; i < 4; ++i) {
    for (int j = 0; j < i; ++j)
      if (share_bytes(arrays[j], arrays[i])) return PAIR_EINVAL;
    for (const void* from : {k, v})
      if (share_bytes(half_rows(c, from, tokens, token_stride, new_head_stride), arrays[i]))
        return PAIR_EINVAL;
  }
  return pair::launch_mx_move(true, c, tokens, dtype == PAIR_BF16, const_cast<void*>(k),
                              const_cast<void*>(v), token_stride, new_head_stride, slots, d_status,
                              as_stream(stream));
}

int pair_cache_load_mx(const pair_mx_cache* cache, int64_t tokens, const int64_t* slots,
                       int32_t dtype, void* k, void* v, int64_t token_stride,
                       int64_t out_head_stride, int32_t* d_status, void* stream) {
  if (dtype != PAIR_BF16 && dtype != PAIR_F16) return PAIR_EDTYPE;
  pair::MxCache c;
  int st = check_mx(cache, &c);
  if (st) return st;
  if (tokens < 0 || tokens > kMaxSlots) return PAIR_ERANGE;
  if (tokens == 0) return PAIR_OK;
  st = check_rows(tokens, k, v, token_stride, out_head_stride, slots);
  if (st) return st;
  Strided rows[] = {{tokens, token_stride}, {c.kv_heads, out_head_stride}};
  if (rows_overlap(rows, c.dim)) return PAIR_EINVAL;
  const Rows out[] = {half_rows(c, k, tokens, token_stride, out_head_stride),
                      half_rows(c, v, tokens, token_stride, out_head_stride)};
  if (share_bytes(out[0], out[1])) return PAIR_EINVAL;
  Rows arrays[4];
  mx_arrays(c, arrays);
  for (const Rows& a : arrays)
    if (share_bytes(out[0], a) || share_bytes(out[1], a)) return PAIR_EINVAL;
  return pair::launch_mx_move(false, c, tokens, dtype == PAIR_BF16, k, v, token_stride,
                              out_head_stride, slots, d_status, as_stream(stream));
}

size_t pair_paged_attention_mx_workspace_bytes(int64_t n, int64_t tokens, int32_t q_heads,
                                               int32_t kv_heads, int32_t dim, int32_t format,
                                               int32_t max_q, int32_t max_len) {
  if (format != PAIR_MXFP8 && format != PAIR_MXFP4) return 0;
  const int32_t bits = format == PAIR_MXFP8 ? 8 : 4;
  if (check_attention(n, tokens, q_heads, kv_heads, dim, bits, max_q, max_len)) return 0;
  return pair::attention_workspace_bytes(n, tokens, q_heads, kv_heads, dim, bits, max_q, max_len);
}

int pair_paged_attention_mx(const pair_mx_cache* cache, int64_t n, int64_t tokens, int32_t q_heads,
                            int32_t dtype, const void* q, int64_t q_token, int64_t q_head,
                            const int32_t* table, int64_t ldt, const int64_t* q_offsets,
                            const int32_t* lens, int32_t max_q, int32_t max_len, float scale,
                            void* out, int64_t out_token, int64_t out_head, float* lse,
                            void* workspace, size_t ws_bytes, int32_t* d_status, void* stream) {
  if (dtype != PAIR_BF16 && dtype != PAIR_F16) return PAIR_EDTYPE;
  pair::MxCache m;
  int st = check_mx(cache, &m);
  if (st) return st;
  st = check_attention(n, tokens, q_heads, m.kv_heads, m.dim, m.bits, max_q, max_len);
  if (st) return st;
  pair::AttnCall c = {};
  c.kv_heads = m.kv_heads;
  c.dim = m.dim;
  c.bits = m.bits;
  c.k_cache = m.k;
  c.v_cache = m.v;
  c.cache = {m.page_stride, m.slot_stride, m.head_stride, m.page, m.n_pages};
  c.scales = {static_cast<const unsigned char*>(m.k_scale),
              static_cast<const unsigned char*>(m.v_scale), m.scale_page, m.scale_slot,
              m.scale_head};
  return attention(c, n, tokens, q_heads, dtype, q, q_token, q_head, table, ldt, q_offsets, lens,
                   max_q, max_len, scale, out, out_token, out_head, lse, workspace, ws_bytes,
                   d_status, stream);
}

const char* pair_strerror(int code) {
  switch (code) {
    case PAIR_OK: return "ok";
    case PAIR_EINVAL: return "invalid argument (null pointer, malformed size or overlapping arrays)";
    case PAIR_EDTYPE: return "unsupported dtype";
    case PAIR_ERANGE: return "size out of the supported range";
    case PAIR_EALIGN: return "base pointer or row stride misaligned (16 bytes; gradients: an element; scales: their blocks)";
    case PAIR_EHIP: return "HIP launch or runtime error";
    case PAIR_EWORKSPACE: return "workspace missing, misaligned or too small";
    case PAIR_ESCRATCH:
      return "one prompt's audit workspace exceeds the no-alloc entry point's static scratch";
    default: return "unknown error code";
  }
}

int pair_version(void) { return 500; }   // 0.5.0: paged cache in 8 and 4 bits added

}  // extern "C"
