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
// A batch's tensors are cut into chunks of kChunk elements, and each workgroup
// takes a run of consecutive chunks.  The second launch walks its run
// backwards: what the first read last is what the 256 MiB memory-side cache
// still holds.  The tensor table travels in the kernel's arguments, so nothing
// is copied to the device or kept between calls.
#include <math.h>

#include "paged.hpp"

namespace pair {

namespace {

constexpr int kThreads = 256;
constexpr int kVec = 8;                             // elements of a lane's piece
constexpr int kPieces = 2;                          // pieces of a lane per chunk
constexpr int kChunk = kThreads * kVec * kPieces;
constexpr int kNormBatch = 160;
constexpr int kScaleBatch = 120;
constexpr int kMaxGroups = 2048;                    // workgroups of a launch
// Partials that every workgroup of the second pass sums itself; more of them
// (beyond about 2000 tensors) are summed once by a launch in between.
constexpr int64_t kMaxOwnSum = 16384;

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

typedef u32x4_t u32x4_a2 __attribute__((aligned(2)));   // a view may start at any element
typedef f32x4_t f32x4_a4 __attribute__((aligned(4)));

__device__ __forceinline__ float half_to_f32(uint32_t bits) {
  return (float)__builtin_bit_cast(_Float16, (uint16_t)bits);
}

__device__ __forceinline__ float load_one(const void* p, int type, int64_t i) {
  if (type == PAIR_F32) return static_cast<const float*>(p)[i];
  const uint32_t b = static_cast<const uint16_t*>(p)[i];
  return type == PAIR_BF16 ? __uint_as_float(b << 16) : half_to_f32(b);
}

// A piece of 8 elements of one type as raw 16-byte parts (two for fp32).
struct Piece {
  u32x4_t a, b;
};

__device__ __forceinline__ Piece load_piece(const void* p, int type, int64_t i) {
  Piece r;
  if (type == PAIR_F32) {
    const float* q = static_cast<const float*>(p) + i;
    r.a = *reinterpret_cast<const u32x4_a2*>(q);
    r.b = *reinterpret_cast<const u32x4_a2*>(q + 4);
  } else {
    r.a = *reinterpret_cast<const u32x4_a2*>(static_cast<const uint16_t*>(p) + i);
    r.b = r.a;
  }
  return r;
}

__device__ __forceinline__ void unpack(const Piece& x, int type, float (&v)[kVec]) {
  if (type == PAIR_F32) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      v[e] = __uint_as_float(x.a[e]);
      v[e + 4] = __uint_as_float(x.b[e]);
    }
  } else if (type == PAIR_BF16) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      v[2 * e] = bf16lo_to_f32(x.a[e]);
      v[2 * e + 1] = bf16hi_to_f32(x.a[e]);
    }
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      v[2 * e] = half_to_f32(x.a[e] & 0xffffu);
      v[2 * e + 1] = half_to_f32(x.a[e] >> 16);
    }
  }
}

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

__global__ __launch_bounds__(kThreads) void clip_norm_kernel(TensorTable<kNormBatch> t,
                                                             double* partial) {
  const uint32_t chunks = t.first[t.count];
  const uint32_t lo = (uint32_t)((uint64_t)chunks * blockIdx.x / gridDim.x);
  const uint32_t hi = (uint32_t)((uint64_t)chunks * (blockIdx.x + 1) / gridDim.x);
  double acc[4] = {0.0, 0.0, 0.0, 0.0};
  int k = lo < hi ? find_tensor(t, lo) : 0;
  for (uint32_t c = lo; c < hi; ++c) {
    while (c >= t.first[k + 1]) ++k;
    const int64_t base = (int64_t)(c - t.first[k]) * kChunk;
    const int64_t left = t.size[k] - base;
    const int type = t.type[k];
    const void* p = static_cast<const unsigned char*>(t.in[k]) + base * (type == PAIR_F32 ? 4 : 2);
    if (left >= kChunk) {
      Piece x[kPieces];
#pragma unroll
      for (int s = 0; s < kPieces; ++s)
        x[s] = load_piece(p, type, (int64_t)(s * kThreads + threadIdx.x) * kVec);
#pragma unroll
      for (int s = 0; s < kPieces; ++s) {
        float v[kVec];
        unpack(x[s], type, v);
#pragma unroll
        for (int e = 0; e < kVec; ++e) acc[e & 3] = fma((double)v[e], (double)v[e], acc[e & 3]);
      }
    } else {
      for (int s = 0; s < kPieces; ++s) {
        const int64_t i = (int64_t)(s * kThreads + threadIdx.x) * kVec;
        if (i + kVec <= left) {
          float v[kVec];
          unpack(load_piece(p, type, i), type, v);
#pragma unroll
          for (int e = 0; e < kVec; ++e) acc[e & 3] = fma((double)v[e], (double)v[e], acc[e & 3]);
        } else {
          for (int64_t j = i; j < left; ++j) {
            const double v = load_one(p, type, j);
            acc[0] = fma(v, v, acc[0]);
          }
        }
      }
    }
  }
  const double s = group_sum((acc[0] + acc[1]) + (acc[2] + acc[3]));
  if (threadIdx.x == 0) partial[blockIdx.x] = s;
}

__device__ __forceinline__ double sum_partials(const double* partial, int64_t n) {
  double s = 0.0;
  for (int64_t i = threadIdx.x; i < n; i += kThreads) s += partial[i];
  return group_sum(s);
}

__global__ __launch_bounds__(kThreads) void clip_sum_kernel(double* partial, int64_t n) {
  const double s = sum_partials(partial, n);
  if (threadIdx.x == 0) partial[n] = s;
}

__device__ __forceinline__ uint32_t bf16_bits(float v) {   // round to nearest even
  const uint32_t u = __float_as_uint(v);
  if ((u & 0x7fffffffu) > 0x7f800000u) return (u >> 16) | 0x40u;
  return (u + 0x7fffu + ((u >> 16) & 1u)) >> 16;
}

__device__ __forceinline__ uint32_t f16_bits(float v) {
  return __builtin_bit_cast(uint16_t, (_Float16)v);
}

__device__ __forceinline__ void store_one(void* p, int type, int64_t i, float v) {
  if (type == PAIR_F32)
    static_cast<float*>(p)[i] = v;
  else
    static_cast<uint16_t*>(p)[i] = (uint16_t)(type == PAIR_BF16 ? bf16_bits(v) : f16_bits(v));
}

__device__ __forceinline__ void store_piece(void* p, int type, int64_t i, const float (&v)[kVec]) {
  if (type == PAIR_F32) {
    float* q = static_cast<float*>(p) + i;
    const f32x4_t a = {v[0], v[1], v[2], v[3]}, b = {v[4], v[5], v[6], v[7]};
    *reinterpret_cast<f32x4_a4*>(q) = a;
    *reinterpret_cast<f32x4_a4*>(q + 4) = b;
  } else {
    u32x4_t w;
#pragma unroll
    for (int e = 0; e < 4; ++e)
      w[e] = type == PAIR_BF16 ? bf16_bits(v[2 * e]) | (bf16_bits(v[2 * e + 1]) << 16)
                               : f16_bits(v[2 * e]) | (f16_bits(v[2 * e + 1]) << 16);
    *reinterpret_cast<u32x4_a2*>(static_cast<uint16_t*>(p) + i) = w;
  }
}

// `sum` holds `n` partials of the squared norm.  `report`: this launch writes
// the norm and the factor (workgroup 0).
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
    const int64_t base = (int64_t)(c - t.first[k]) * kChunk;
    const int64_t left = t.size[k] - base;
    const int type = t.type[k], to = o.type[k];
    const void* p = static_cast<const unsigned char*>(t.in[k]) + base * (type == PAIR_F32 ? 4 : 2);
    void* q = static_cast<unsigned char*>(o.out[k]) + base * (to == PAIR_F32 ? 4 : 2);
    if (left >= kChunk) {
      Piece x[kPieces];
#pragma unroll
      for (int s = 0; s < kPieces; ++s)
        x[s] = load_piece(p, type, (int64_t)(s * kThreads + threadIdx.x) * kVec);
#pragma unroll
      for (int s = 0; s < kPieces; ++s) {
        float v[kVec];
        unpack(x[s], type, v);
#pragma unroll
        for (int e = 0; e < kVec; ++e) v[e] *= coef;
        store_piece(q, to, (int64_t)(s * kThreads + threadIdx.x) * kVec, v);
      }
    } else {
      for (int s = 0; s < kPieces; ++s) {
        const int64_t i = (int64_t)(s * kThreads + threadIdx.x) * kVec;
        if (i + kVec <= left) {
          float v[kVec];
          unpack(load_piece(p, type, i), type, v);
#pragma unroll
          for (int e = 0; e < kVec; ++e) v[e] *= coef;
          store_piece(q, to, i, v);
        } else {
          for (int64_t j = i; j < left; ++j) store_one(q, to, j, load_one(p, type, j) * coef);
        }
      }
    }
  }
}

uint32_t chunks_of(int64_t size) { return (uint32_t)((size + kChunk - 1) / kChunk); }

unsigned groups_of(uint32_t chunks) {
  return chunks < (uint32_t)kMaxGroups ? (chunks ? chunks : 1u) : (unsigned)kMaxGroups;
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
    t->first[k + 1] = t->first[k] + chunks_of(sizes[i]);
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
  return ((size_t)(batches * kMaxGroups + 1) * sizeof(double) + 255) / 256 * 256;
}

int launch_clip(int64_t count, const void* const* grads, void* const* outs, const int64_t* sizes,
                const int32_t* dtypes, const int32_t* out_dtypes, float max_norm, float* norm,
                float* coef, void* workspace, int32_t* d_status, hipStream_t stream) {
  double* partial = static_cast<double*>(workspace);
  int64_t n = 0;
  for (int64_t i = 0; i < count;) {
    TensorTable<kNormBatch> t;
    i = fill(&t, nullptr, i, count, grads, nullptr, sizes, dtypes, nullptr);
    if (t.count == 0) break;
    const unsigned g = groups_of(t.first[t.count]);
    hipLaunchKernelGGL(clip_norm_kernel, dim3(g), dim3(kThreads), 0, stream, t, partial + n);
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
    const unsigned g = groups_of(t.first[t.count]);
    hipLaunchKernelGGL(clip_scale_kernel, dim3(g), dim3(kThreads), 0, stream, t, o, partial, n,
                       max_norm, outs == nullptr ? 1 : 0, report, norm, coef, d_status);
    report = 0;
  }
  return hipGetLastError() == hipSuccess ? PAIR_OK : PAIR_EHIP;
}

}  // namespace pair
