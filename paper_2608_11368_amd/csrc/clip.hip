// Global gradient norm over many tensors, and clipping:
//     norm = sqrt(sum g^2),  coef = norm > max ? max / norm : 1,  out = coef g.
//
// HBM-bound: the gradients are read for the norm and again for the product
// (the factor is known only after the last element), and written once.  Two
// launches for up to kNormBatch tensors: the first leaves one fp64 partial per
// workgroup, the second sums the partials in every workgroup (the same order,
// so the same bits) and scales.  Squares and sums are fp64: no overflow of a
// large fp32 gradient, no dependence of the error on the element count; at two
// fp64 operations per element they stay hidden behind the loads.
//
// A batch's tensors are cut into chunks of kChunkBytes, and each workgroup
// takes a run of consecutive chunks.  The second launch walks its run
// backwards: what the first read last is what the 256 MiB memory-side cache
// still holds.  A lane has a whole chunk's 64 bytes in flight before it uses any
// (32 bytes: 4.2 TB/s for the norm of bf16, 64 bytes: 6.3), and gradients larger
// than that cache are read and written past the caches (5 to 10% faster).  The
// tensor table travels in the kernel's arguments, so nothing is copied to the
// device or kept between calls.
//
// Measured: norm of 600M bf16 or 455M fp32 elements 187 and 269 us (6.4 and 6.8
// TB/s); clipping 600M bf16 into fp32 898 us, into bf16 663 us, 455M fp32 998 us
// (5.3 to 5.5 TB/s of two reads and a write); 301 tensors of 40M bf16 elements
// into fp32, two launches for the norm (11 us each) and three for the product
// (15 to 21 us), 77 us in all.
#include <math.h>

#include "paged.hpp"

namespace pair {

namespace {

constexpr int kThreads = 256;
constexpr int kLaneBytes = 64;                      // of a lane per chunk: what is in flight
constexpr int kChunkBytes = kThreads * kLaneBytes;
constexpr int kNormBatch = 160;
constexpr int kScaleBatch = 120;
constexpr int kNormGroups = 1024;                   // most workgroups of a launch
constexpr int kScaleGroups = 2048;
constexpr int64_t kCached = (int64_t)192 << 20;     // of the 256 MiB memory-side cache
// Partials that every workgroup of the second pass sums itself (2048 of them:
// 1.1 us a launch more than reading one sum); more of them (beyond about 600
// tensors, so six such launches) are summed once by a launch in between (2 us).
constexpr int64_t kMaxOwnSum = 4096;

template <int N>
struct TensorTable {
  const void* in[N];
  int64_t size[N];
  uint32_t first[N + 1];   // first chunk of each tensor, and the chunk count
  uint8_t type[N];
  int32_t count;
};
struct OutTable {
  void* out[kScaleBatch];
  uint8_t type[kScaleBatch];
};
static_assert(sizeof(TensorTable<kNormBatch>) + 64 <= 4096, "kernel arguments");
static_assert(sizeof(TensorTable<kScaleBatch>) + sizeof(OutTable) + 128 <= 4096,
              "kernel arguments");

__device__ __forceinline__ float half_to_f32(uint32_t bits) {
  return (float)__builtin_bit_cast(_Float16, (uint16_t)bits);
}

__device__ __forceinline__ uint32_t bf16_bits(float v) {   // round to nearest even
  const uint32_t u = __float_as_uint(v);
  if ((u & 0x7fffffffu) > 0x7f800000u) return (u >> 16) | 0x40u;
  return (u + 0x7fffu + ((u >> 16) & 1u)) >> 16;
}

__device__ __forceinline__ uint32_t f16_bits(float v) {
  return __builtin_bit_cast(uint16_t, (_Float16)v);
}

// Pieces of N elements of a type: one vector access, which may start at any
// element (a view does).
template <int DWORDS>
struct Dwords;
template <>
struct Dwords<4> {
  typedef u32x4_t Wide;
};
template <>
struct Dwords<2> {
  typedef u32x2_t Wide;
};

template <int TYPE>
struct Elements {          // PAIR_F32
  static constexpr int kBytes = 4;
  __device__ static float get(const uint32_t* w, int e) { return __uint_as_float(w[e]); }
  __device__ static float one(const void* p, int64_t i) { return static_cast<const float*>(p)[i]; }
  __device__ static void put(void* p, int64_t i, float v) { static_cast<float*>(p)[i] = v; }
  template <int N>
  __device__ static void pack(const float (&v)[N], uint32_t* w) {
#pragma unroll
    for (int e = 0; e < N; ++e) w[e] = __float_as_uint(v[e]);
  }
};
template <bool BF16>
struct Halves {
  static constexpr int kBytes = 2;
  __device__ static float wide(uint32_t b) {
    return BF16 ? __uint_as_float(b << 16) : half_to_f32(b & 0xffffu);
  }
  __device__ static uint32_t narrow(float v) { return BF16 ? bf16_bits(v) : f16_bits(v); }
  __device__ static float get(const uint32_t* w, int e) {
    return wide(e & 1 ? w[e >> 1] >> 16 : w[e >> 1]);
  }
  __device__ static float one(const void* p, int64_t i) {
    return wide(static_cast<const uint16_t*>(p)[i]);
  }
  __device__ static void put(void* p, int64_t i, float v) {
    static_cast<uint16_t*>(p)[i] = (uint16_t)narrow(v);
  }
  template <int N>
  __device__ static void pack(const float (&v)[N], uint32_t* w) {
#pragma unroll
    for (int e = 0; e < N; e += 2) w[e / 2] = narrow(v[e]) | (narrow(v[e + 1]) << 16);
  }
};
template <>
struct Elements<PAIR_BF16> : Halves<true> {};
template <>
struct Elements<PAIR_F16> : Halves<false> {};

template <int TYPE, int N, bool STREAM>
struct Piece {
  static constexpr int kDwords = N * Elements<TYPE>::kBytes / 4;
  typedef typename Dwords<kDwords>::Wide Wide __attribute__((aligned(2)));
  uint32_t w[kDwords];
  __device__ __forceinline__ void load(const void* p, int64_t i) {
    const Wide* q = reinterpret_cast<const Wide*>(static_cast<const unsigned char*>(p) +
                                                  i * Elements<TYPE>::kBytes);
    const typename Dwords<kDwords>::Wide x = STREAM ? __builtin_nontemporal_load(q) : *q;
#pragma unroll
    for (int d = 0; d < kDwords; ++d) w[d] = x[d];
  }
  __device__ __forceinline__ void store(void* p, int64_t i) const {
    Wide* q =
        reinterpret_cast<Wide*>(static_cast<unsigned char*>(p) + i * Elements<TYPE>::kBytes);
    typename Dwords<kDwords>::Wide x;
#pragma unroll
    for (int d = 0; d < kDwords; ++d) x[d] = w[d];
    if (STREAM)
      __builtin_nontemporal_store(x, q);
    else
      *q = x;
  }
};

// The tensor that holds chunk c (wave-uniform): the number of tensors that end
// at or before it, counted by the lanes.  Tensors without elements are not in
// the table.
template <int N>
__device__ __forceinline__ int find_tensor(const TensorTable<N>& t, uint32_t c) {
  const int lane = threadIdx.x & (kWave - 1);
  int k = 0;
#pragma unroll
  for (int w = 0; w < N; w += kWave) {
    const int i = w + lane;
    const bool before = i < N && i < t.count && t.first[i < N ? i + 1 : N] <= c;
    k += __popcll(__ballot(before));
  }
  return uniform(k);
}

// Sum over a workgroup in a fixed order, in thread 0 (and every other one).
__device__ __forceinline__ double group_sum(double v) {
  __shared__ double part[kThreads / kWave];
  v = wave_sum_d(v);
  if ((threadIdx.x & (kWave - 1)) == 0) part[threadIdx.x / kWave] = v;
  __syncthreads();
  double s = part[0];
#pragma unroll
  for (int w = 1; w < kThreads / kWave; ++w) s += part[w];
  return s;
}

// Squares of a chunk's `left` elements at p, added to this thread's sums.
template <int TYPE, bool STREAM>
__device__ __forceinline__ void add_squares(const void* p, int64_t left, double (&acc)[4]) {
  typedef Elements<TYPE> E;
  constexpr int N = 16 / E::kBytes, P = kLaneBytes / 16;   // 16-byte pieces
  if (left >= kThreads * N * P) {
    Piece<TYPE, N, STREAM> x[P];
#pragma unroll
    for (int s = 0; s < P; ++s) x[s].load(p, (s * kThreads + (int)threadIdx.x) * N);
#pragma unroll
    for (int s = 0; s < P; ++s)
#pragma unroll
      for (int e = 0; e < N; ++e) {
        const double v = E::get(x[s].w, e);
        acc[e & 3] = fma(v, v, acc[e & 3]);
      }
    return;
  }
  for (int s = 0; s < P; ++s) {
    const int64_t i = (s * kThreads + (int)threadIdx.x) * N;
    if (i + N <= left) {
      Piece<TYPE, N, STREAM> x;
      x.load(p, i);
#pragma unroll
      for (int e = 0; e < N; ++e) {
        const double v = E::get(x.w, e);
        acc[e & 3] = fma(v, v, acc[e & 3]);
      }
    } else {
      for (int64_t j = i; j < left; ++j) {
        const double v = E::one(p, j);
        acc[0] = fma(v, v, acc[0]);
      }
    }
  }
}

template <bool STREAM>
__global__ __launch_bounds__(kThreads) void clip_norm_kernel(TensorTable<kNormBatch> t,
                                                             double* partial) {
  const uint32_t chunks = t.first[t.count];
  const uint32_t lo = (uint32_t)((uint64_t)chunks * blockIdx.x / gridDim.x);
  const uint32_t hi = (uint32_t)((uint64_t)chunks * (blockIdx.x + 1) / gridDim.x);
  double acc[4] = {0.0, 0.0, 0.0, 0.0};
  int k = lo < hi ? find_tensor(t, lo) : 0;
  for (uint32_t c = lo; c < hi; ++c) {
    while (c >= t.first[k + 1]) ++k;
    const int type = t.type[k], unit = type == PAIR_F32 ? 4 : 2;
    const int64_t at = (int64_t)(c - t.first[k]) * kChunkBytes;
    const int64_t left = t.size[k] - at / unit;
    const void* p = static_cast<const unsigned char*>(t.in[k]) + at;
    if (type == PAIR_F32)
      add_squares<PAIR_F32, STREAM>(p, left, acc);
    else if (type == PAIR_BF16)
      add_squares<PAIR_BF16, STREAM>(p, left, acc);
    else
      add_squares<PAIR_F16, STREAM>(p, left, acc);
  }
  const double s = group_sum((acc[0] + acc[1]) + (acc[2] + acc[3]));
  if (threadIdx.x == 0) partial[blockIdx.x] = s;
}

__device__ __forceinline__ double sum_partials(const double* partial, int64_t n) {
  double s = 0.0;
  for (int64_t i0 = threadIdx.x; i0 < n; i0 += 4 * kThreads) {   // four loads in flight
    double v[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = i0 + e * kThreads < n ? partial[i0 + e * kThreads] : 0.0;
    s += (v[0] + v[1]) + (v[2] + v[3]);
  }
  return group_sum(s);
}

__global__ __launch_bounds__(kThreads) void clip_sum_kernel(double* partial, int64_t n) {
  const double s = sum_partials(partial, n);
  if (threadIdx.x == 0) partial[n] = s;
}

// A chunk's product.  Pieces are of four elements where the result is fp32, so
// that a wave's stores cover whole cache lines.
template <int FROM, int TO, bool STREAM>
__device__ __forceinline__ void scale_chunk(const void* p, void* q, int64_t left, float coef) {
  typedef Elements<FROM> E;
  constexpr int N = 16 / Elements<TO>::kBytes, P = kLaneBytes / E::kBytes / N;
  auto scale = [&](const Piece<FROM, N, STREAM>& x, int64_t i) {
    float v[N];
#pragma unroll
    for (int e = 0; e < N; ++e) v[e] = E::get(x.w, e) * coef;
    Piece<TO, N, STREAM> y;
    Elements<TO>::template pack<N>(v, y.w);
    y.store(q, i);
  };
  if (left >= kThreads * N * P) {
    Piece<FROM, N, STREAM> x[P];
#pragma unroll
    for (int s = 0; s < P; ++s) x[s].load(p, (s * kThreads + (int)threadIdx.x) * N);
#pragma unroll
    for (int s = 0; s < P; ++s) scale(x[s], (s * kThreads + (int)threadIdx.x) * N);
    return;
  }
  for (int s = 0; s < P; ++s) {
    const int64_t i = (s * kThreads + (int)threadIdx.x) * N;
    if (i + N <= left) {
      Piece<FROM, N, STREAM> x;
      x.load(p, i);
      scale(x, i);
    } else {
      for (int64_t j = i; j < left; ++j) Elements<TO>::put(q, j, E::one(p, j) * coef);
    }
  }
}

// `sum` holds `n` partials of the squared norm.  `report`: this launch writes
// the norm and the factor (workgroup 0).
template <bool STREAM>
__global__ __launch_bounds__(kThreads) void clip_scale_kernel(
    TensorTable<kScaleBatch> t, OutTable o, const double* sum, int64_t n, float max_norm,
    int in_place, int report, float* norm_out, float* coef_out, int32_t* d_status) {
  const double norm = sqrt(sum_partials(sum, n));
  const bool finite = norm < INFINITY;             // false for NaN too
  const bool clip = finite && norm > (double)max_norm;
  const float coef = clip ? (float)((double)max_norm / norm) : 1.0f;
  if (report && blockIdx.x == 0 && threadIdx.x == 0) {
    *norm_out = (float)norm;
    *coef_out = coef;
    if (!finite) raise_status(d_status, PAIR_ST_NONFINITE);
  }
  if (in_place && !clip) return;
  const uint32_t chunks = t.first[t.count];
  const uint32_t lo = (uint32_t)((uint64_t)chunks * blockIdx.x / gridDim.x);
  uint32_t c = (uint32_t)((uint64_t)chunks * (blockIdx.x + 1) / gridDim.x);
  if (c <= lo) return;
  int k = find_tensor(t, c - 1);
  while (c-- > lo) {
    while (c < t.first[k]) --k;
    const int type = t.type[k], to = o.type[k], unit = type == PAIR_F32 ? 4 : 2;
    const int64_t at = (int64_t)(c - t.first[k]) * kChunkBytes;
    const int64_t left = t.size[k] - at / unit;
    const void* p = static_cast<const unsigned char*>(t.in[k]) + at;
    void* q = static_cast<unsigned char*>(o.out[k]) + at / unit * (to == PAIR_F32 ? 4 : 2);
    if (type == PAIR_F32)
      scale_chunk<PAIR_F32, PAIR_F32, STREAM>(p, q, left, coef);
    else if (type == PAIR_BF16 && to == PAIR_BF16)
      scale_chunk<PAIR_BF16, PAIR_BF16, STREAM>(p, q, left, coef);
    else if (type == PAIR_BF16)
      scale_chunk<PAIR_BF16, PAIR_F32, STREAM>(p, q, left, coef);
    else if (to == PAIR_F16)
      scale_chunk<PAIR_F16, PAIR_F16, STREAM>(p, q, left, coef);
    else
      scale_chunk<PAIR_F16, PAIR_F32, STREAM>(p, q, left, coef);
  }
}

uint32_t chunks_of(int64_t size, int32_t type) {
  return (uint32_t)((size * (type == PAIR_F32 ? 4 : 2) + kChunkBytes - 1) / kChunkBytes);
}

unsigned groups_of(uint32_t chunks, int most) {
  return chunks < (uint32_t)most ? (chunks ? chunks : 1u) : (unsigned)most;
}

// Fills a table from tensor i0 on, skipping empty ones; returns the next tensor.
// A batch stays below 2^31 chunks, so that a launch can count them.
template <int N>
int64_t fill(TensorTable<N>* t, OutTable* o, int64_t i0, int64_t count, const void* const* grads,
             void* const* outs, const int64_t* sizes, const int32_t* dtypes,
             const int32_t* out_dtypes) {
  t->count = 0;
  t->first[0] = 0;
  int64_t i = i0;
  for (; i < count && t->count < N; ++i) {
    if (sizes[i] == 0) continue;
    const int k = t->count;
    t->in[k] = grads[i];
    t->size[k] = sizes[i];
    t->type[k] = (uint8_t)dtypes[i];
    t->first[k + 1] = t->first[k] + chunks_of(sizes[i], dtypes[i]);
    if (o != nullptr) {
      o->out[k] = outs != nullptr ? outs[i] : const_cast<void*>(grads[i]);
      o->type[k] = (uint8_t)(outs != nullptr ? out_dtypes[i] : dtypes[i]);
    }
    t->count = k + 1;
  }
  return i;
}

}  // namespace

// One partial per workgroup of the first pass, and one sum.
size_t clip_workspace_bytes(int64_t count) {
  const int64_t batches = count / kNormBatch + 1;
  return ((size_t)(batches * kNormGroups + 1) * sizeof(double) + 255) / 256 * 256;
}

int launch_clip(int64_t count, const void* const* grads, void* const* outs, const int64_t* sizes,
                const int32_t* dtypes, const int32_t* out_dtypes, float max_norm, float* norm,
                float* coef, void* workspace, int32_t* d_status, hipStream_t stream) {
  double* partial = static_cast<double*>(workspace);
  // Gradients that the memory-side cache does not hold are streamed past it.
  int64_t bytes = 0;
  for (int64_t i = 0; i < count; ++i) bytes += sizes[i] * (dtypes[i] == PAIR_F32 ? 4 : 2);
  const bool stream_past = bytes > kCached;
  int64_t n = 0;
  for (int64_t i = 0; i < count;) {
    TensorTable<kNormBatch> t;
    i = fill(&t, nullptr, i, count, grads, nullptr, sizes, dtypes, nullptr);
    if (t.count == 0) break;
    const unsigned g = groups_of(t.first[t.count], kNormGroups);
    if (stream_past)
      hipLaunchKernelGGL(clip_norm_kernel<true>, dim3(g), dim3(kThreads), 0, stream, t, partial + n);
    else
      hipLaunchKernelGGL(clip_norm_kernel<false>, dim3(g), dim3(kThreads), 0, stream, t, partial + n);
    n += g;
  }
  if (hipGetLastError() != hipSuccess) return PAIR_EHIP;
  if (n > kMaxOwnSum) {
    hipLaunchKernelGGL(clip_sum_kernel, dim3(1), dim3(kThreads), 0, stream, partial, n);
    partial += n;
    n = 1;
  }
  // With an infinite bound and no outputs the norm is all there is to write.
  const bool norm_only = outs == nullptr && max_norm > 3.4028235e38f;
  int report = 1;
  for (int64_t i = 0; i < count || report;) {
    TensorTable<kScaleBatch> t;
    OutTable o;
    i = fill(&t, &o, norm_only ? count : i, count, grads, outs, sizes, dtypes, out_dtypes);
    if (t.count == 0 && !report) break;
    const unsigned g = groups_of(t.first[t.count], kScaleGroups);
    if (stream_past)
      hipLaunchKernelGGL(clip_scale_kernel<true>, dim3(g), dim3(kThreads), 0, stream, t, o, partial,
                         n, max_norm, outs == nullptr ? 1 : 0, report, norm, coef, d_status);
    else
      hipLaunchKernelGGL(clip_scale_kernel<false>, dim3(g), dim3(kThreads), 0, stream, t, o, partial,
                         n, max_norm, outs == nullptr ? 1 : 0, report, norm, coef, d_status);
    report = 0;
  }
  return hipGetLastError() == hipSuccess ? PAIR_OK : PAIR_EHIP;
}

}  // namespace pair
