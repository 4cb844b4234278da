// Divergence of a student's logits from a teacher's top logits, and its
// gradient (ssd_distill_forward, _backward, _step of ssd_ops.h).
//
// Per row, with x_i = z_i / T and p the softmax of the teacher's slots:
//   m = max x, s = sum exp(x_i - m), lse = m + log s,
//   loss = w sum_j p_j (log p_j - (x_{id_j} - lse)),
//   dz_i = w / T (exp(x_i - lse) - sum_{j: id_j = i} p_j).
// Bound: memory.  The forward pass has to read the row, the step to read and to
// write it.
#include <type_traits>

#include "ops_common.h"

namespace ssd {
namespace {

constexpr int kMaxSlots = 128;  // teacher slots of a row

typedef unsigned u32x4 __attribute__((ext_vector_type(4)));
// rows begin where the caller's stride puts them: at any element
typedef unsigned u32x4_a2 __attribute__((ext_vector_type(4), aligned(2)));

template <typename T> struct Vec;  // 16 bytes of elements
template <> struct Vec<float> {
  static constexpr int E = 4;
  static constexpr unsigned kNone = 0xff800000u;  // -infinity
  static __device__ __forceinline__ float get(const u32x4& r, int e) { return __uint_as_float(r[e]); }
  static __device__ __forceinline__ u32x4 pack(const float (&v)[4]) {
    return (u32x4){__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3])};
  }
};
template <> struct Vec<bf16_t> {
  static constexpr int E = 8;
  static constexpr unsigned kNone = 0xff80ff80u;
  static __device__ __forceinline__ float get(const u32x4& r, int e) {
    return __uint_as_float(e & 1 ? r[e >> 1] & 0xffff0000u : r[e >> 1] << 16);
  }
  static __device__ __forceinline__ u32x4 pack(const float (&v)[8]) {
    typedef __bf16 b2 __attribute__((ext_vector_type(2)));
    typedef float f2 __attribute__((ext_vector_type(2)));
    u32x4 r;
#pragma unroll
    for (int i = 0; i < 4; ++i)
      r[i] = __builtin_bit_cast(unsigned, __builtin_convertvector((f2){v[2 * i], v[2 * i + 1]}, b2));
    return r;
  }
};

// chunk c of a row (elements c E .. c E + E - 1); -infinity past its end
template <typename T>
__device__ __forceinline__ u32x4 load_chunk(const T* row, int c, int V) {
  constexpr int E = Vec<T>::E;
  u32x4 r = {Vec<T>::kNone, Vec<T>::kNone, Vec<T>::kNone, Vec<T>::kNone};
  const int at = c * E;
  if (at + E <= V) {
    r = *(const u32x4_a2*)(row + at);
  } else if (at < V) {
    float v[E];
#pragma unroll
    for (int e = 0; e < E; ++e) v[e] = at + e < V ? op_ld(row, at + e) : -INFINITY;
    r = Vec<T>::pack(v);
  }
  return r;
}

template <typename T>
__device__ __forceinline__ void store_chunk(T* row, int c, int V, const float (&v)[Vec<T>::E]) {
  constexpr int E = Vec<T>::E;
  const int at = c * E;
  if (at + E <= V) {
    *(u32x4_a2*)(row + at) = Vec<T>::pack(v);
  } else {
#pragma unroll
    for (int e = 0; e < E; ++e)
      if (at + e < V) op_st(row, at + e, v[e]);
  }
}

__device__ __forceinline__ float wave_max(float v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor(v, o));
  return v;
}
__device__ __forceinline__ float wave_sum(float v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o);
  return v;
}

struct DistillArgs {
  const void* logits;
  int64_t ld;
  int V;
  const int* ids;
  const float* vals;
  int K;
  const float* weight;
  float inv_t;
  float* loss;
  float* lse;           // backward: read
  void* grad;
  int64_t ld_d;
};

// the row's slots, in LDS: a slot that is left out has id -1 and p 0
struct Slots {
  int id[kMaxSlots];
  float p[kMaxSlots];
  int live;  // whether the row counts
};

// By one wave; lane l has slots l and l + 64.  lp: their log p.
__device__ __forceinline__ void teacher(const DistillArgs& a, int n, Slots& s, float (&lp)[2]) {
  const int lane = threadIdx.x & 63;
  int id[2];
  float x[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int j = lane + 64 * i;
    id[i] = -1;
    x[i] = -INFINITY;
    if (j < a.K) {
      const int t = a.ids[(size_t)n * a.K + j];
      const float v = a.vals[(size_t)n * a.K + j];
      if (t >= 0 && t < a.V && !(v == -INFINITY)) {
        id[i] = t;
        x[i] = v * a.inv_t;
      }
    }
  }
  const bool any = __builtin_amdgcn_ballot_w64(id[0] >= 0 || id[1] >= 0) != 0;
  const float m = any ? wave_max(fmaxf(x[0], x[1])) : 0.f;
  const float e0 = __expf(x[0] - m), e1 = __expf(x[1] - m);
  const float total = wave_sum(e0 + e1), ls = logf(total);
  const float w = a.weight ? a.weight[n] : 1.f;
  lp[0] = x[0] - m - ls;
  lp[1] = x[1] - m - ls;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int j = lane + 64 * i;
    s.id[j] = id[i];
    s.p[j] = id[i] >= 0 ? (i ? e1 : e0) / total : 0.f;
  }
  if (lane == 0) s.live = any && w != 0.f;
}

// marks, for every thread, which of its chunks (bit i: chunk c0 + i TPB + t)
// hold a teacher's token; by the wave that ran teacher(), after the marks are 0
template <int E, int TPB>
__device__ __forceinline__ void mark(const Slots& s, int K, int c0, int C, unsigned* marks) {
  for (int j = threadIdx.x & 63; j < K; j += 64) {
    const int c = s.id[j] / E - c0;
    if (s.id[j] >= 0 && c >= 0 && c < C * TPB) atomicOr(&marks[c % TPB], 1u << (c / TPB));
  }
}

// subtracts the teacher's probabilities of a marked chunk's tokens, in the slots' order
template <int E>
__device__ __forceinline__ void subtract(const Slots& s, int K, int c, float (&g)[E]) {
  for (int j = 0; j < K; ++j) {
    const int at = s.id[j] - c * E;
#pragma unroll
    for (int e = 0; e < E; ++e)
      if (at == e) g[e] -= s.p[j];
  }
}

template <int TPB, bool MAX>
__device__ __forceinline__ float block_reduce(float v, float* red) {
  constexpr int W = TPB / 64;
  v = MAX ? wave_max(v) : wave_sum(v);
  if (W == 1) return v;
  __syncthreads();
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
  __syncthreads();
  v = red[0];
#pragma unroll
  for (int i = 1; i < W; ++i) v = MAX ? fmaxf(v, red[i]) : v + red[i];
  return v;
}

// One workgroup per row, two sweeps over it: the running maximum and sum, then
// the gradient.
template <typename T, bool GRAD>
__global__ __launch_bounds__(1024) void distill_sweep_kernel(DistillArgs a) {
  constexpr int TPB = 1024, E = Vec<T>::E, SEG = 32;
  __shared__ Slots slots;
  __shared__ unsigned marks[TPB];
  __shared__ float red[TPB / 64];
  const int n = blockIdx.x, t = threadIdx.x;
  const T* row = (const T*)a.logits + (size_t)n * a.ld;
  const int chunks = (a.V + E - 1) / E;
  float lp[2] = {0.f, 0.f}, z[2] = {0.f, 0.f};
  if (t < 64) {
    teacher(a, n, slots, lp);
#pragma unroll
    for (int i = 0; i < 2; ++i)
      if (slots.id[t + 64 * i] >= 0) z[i] = op_ld(row, slots.id[t + 64 * i]);
  }
  float m = -INFINITY, s = 0.f;
  for (int c = t; c < chunks; c += TPB) {
    const u32x4 r = load_chunk(row, c, a.V);
    float top = m;
#pragma unroll
    for (int e = 0; e < E; ++e) top = fmaxf(top, Vec<T>::get(r, e) * a.inv_t);
    const float ref = top == -INFINITY ? 0.f : top;
    s *= __expf(m - ref);
#pragma unroll
    for (int e = 0; e < E; ++e) s += __expf(Vec<T>::get(r, e) * a.inv_t - ref);
    m = top;
  }
  const float top = block_reduce<TPB, true>(m, red), ref = top == -INFINITY ? 0.f : top;
  const float total = block_reduce<TPB, false>(s * __expf(m - ref), red);
  const float lse = top + logf(total);
  if (t < 64) {
    float l = 0.f;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const float p = slots.p[t + 64 * i];
      if (p != 0.f) l += p * (lp[i] - (z[i] * a.inv_t - lse));
    }
    l = wave_sum(l);
    if (t == 0) {
      a.loss[n] = slots.live ? l * (a.weight ? a.weight[n] : 1.f) : 0.f;
      a.lse[n] = lse;
    }
  }
  if (!GRAD) return;
  T* out = (T*)a.grad + (size_t)n * a.ld_d;
  const bool live = slots.live;
  const float f = (a.weight ? a.weight[n] : 1.f) * a.inv_t, inv = 1.f / total;
  for (int c0 = 0; c0 < chunks; c0 += SEG * TPB) {
    __syncthreads();
    marks[t] = 0;
    __syncthreads();
    if (t < 64) mark<E, TPB>(slots, a.K, c0, SEG, marks);
    __syncthreads();
    const unsigned mk = marks[t];
    for (int i = 0; i < SEG; ++i) {
      const int c = c0 + i * TPB + t;
      if (c >= chunks) break;
      const u32x4 r = load_chunk(row, c, a.V);
      float g[E];
#pragma unroll
      for (int e = 0; e < E; ++e) g[e] = __expf(Vec<T>::get(r, e) * a.inv_t - top) * inv;
      if (mk >> i & 1) subtract<E>(slots, a.K, c, g);
#pragma unroll
      for (int e = 0; e < E; ++e) g[e] = live ? g[e] * f : 0.f;
      store_chunk(out, c, a.V, g);
    }
  }
}

// The gradient from a known log-sum-exp: a workgroup per row and 8 chunks a thread.
template <typename T>
__global__ __launch_bounds__(256) void distill_grad_kernel(DistillArgs a) {
  constexpr int TPB = 256, E = Vec<T>::E, C = 8;
  __shared__ Slots slots;
  __shared__ unsigned marks[TPB];
  const int n = blockIdx.x, c0 = blockIdx.y * (C * TPB), t = threadIdx.x;
  const T* row = (const T*)a.logits + (size_t)n * a.ld;
  T* out = (T*)a.grad + (size_t)n * a.ld_d;
  const int chunks = (a.V + E - 1) / E;
  u32x4 r[C];
#pragma unroll
  for (int i = 0; i < C; ++i) r[i] = load_chunk(row, c0 + i * TPB + t, a.V);
  marks[t] = 0;
  float lp[2];
  if (t < 64) teacher(a, n, slots, lp);
  __syncthreads();
  if (t < 64) mark<E, TPB>(slots, a.K, c0, C, marks);
  __syncthreads();
  const unsigned mk = marks[t];
  const bool live = slots.live;
  const float f = (a.weight ? a.weight[n] : 1.f) * a.inv_t, lse = a.lse[n];
#pragma unroll
  for (int i = 0; i < C; ++i) {
    const int c = c0 + i * TPB + t;
    float g[E];
#pragma unroll
    for (int e = 0; e < E; ++e) g[e] = __expf(Vec<T>::get(r[i], e) * a.inv_t - lse);
    if (mk >> i & 1) subtract<E>(slots, a.K, c, g);
#pragma unroll
    for (int e = 0; e < E; ++e) g[e] = live ? g[e] * f : 0.f;
    if (c < chunks) store_chunk(out, c, a.V, g);
  }
}

ssd_status check(int dtype, const void* logits, int64_t ld, int n, int V, const int* ids, const float* vals, int k,
                 float temperature) {
  OP_REQUIRE(op_dtype(dtype), SSD_E_INVALID_ARG, "dtype must be SSD_F32 or SSD_BF16");
  OP_REQUIRE(n >= 0, SSD_E_INVALID_ARG, "n_rows is negative");
  OP_REQUIRE(V >= 1 && V <= 1 << 24, SSD_E_INVALID_ARG, "vocab outside [1, 2^24]");
  OP_REQUIRE(k >= 1 && k <= kMaxSlots, SSD_E_INVALID_ARG, "k outside [1, 128]");
  OP_REQUIRE(temperature > 0.f && temperature < INFINITY, SSD_E_INVALID_ARG, "temperature must be positive and finite");
  OP_REQUIRE(ld >= V, SSD_E_INVALID_ARG, "the logits' row stride is below vocab");
  OP_REQUIRE(n == 0 || (logits && ids && vals), SSD_E_INVALID_ARG, "null argument");
  OP_REQUIRE((uintptr_t)logits % op_size(dtype) == 0, SSD_E_INVALID_ARG, "logits not aligned to their type");
  return SSD_OK;
}

ssd_status check_grad(int dtype, const void* logits, int64_t ld, int n, int V, const void* grad, int64_t ld_d) {
  OP_REQUIRE(ld_d >= V, SSD_E_INVALID_ARG, "dlogits' row stride is below vocab");
  OP_REQUIRE(n == 0 || grad, SSD_E_INVALID_ARG, "null argument");
  OP_REQUIRE((uintptr_t)grad % op_size(dtype) == 0, SSD_E_INVALID_ARG, "dlogits not aligned to their type");
  OP_REQUIRE((grad == logits && ld == ld_d) || !op_overlap(logits, op_span(n, ld, V, op_size(dtype)), grad,
                                                           op_span(n, ld_d, V, op_size(dtype))),
             SSD_E_INVALID_ARG, "dlogits overlaps the logits without being them");
  return SSD_OK;
}

template <typename T>
void launch_rows(const DistillArgs& a, int n, bool grad, hipStream_t s) {
  if (grad) distill_sweep_kernel<T, true><<<n, 1024, 0, s>>>(a);
  else distill_sweep_kernel<T, false><<<n, 1024, 0, s>>>(a);
}

}  // namespace
}  // namespace ssd

using namespace ssd;

extern "C" ssd_status ssd_distill_forward(ssd_dtype dtype, const void* logits, int64_t ld, int32_t n_rows,
                                          int32_t vocab, const int32_t* ids, const float* vals, int32_t k,
                                          const float* weight, float temperature, float* loss, float* lse,
                                          void* stream) {
  ssd_status st = check(dtype, logits, ld, n_rows, vocab, ids, vals, k, temperature);
  if (st != SSD_OK) return st;
  if (n_rows == 0) return SSD_OK;
  OP_REQUIRE(loss && lse, SSD_E_INVALID_ARG, "null argument");
  DistillArgs a{logits, ld, vocab, ids, vals, k, weight, 1.f / temperature, loss, lse, nullptr, 0};
  if (dtype == SSD_F32) launch_rows<float>(a, n_rows, false, (hipStream_t)stream);
  else launch_rows<bf16_t>(a, n_rows, false, (hipStream_t)stream);
  OP_LAUNCHED();
  return SSD_OK;
}

extern "C" ssd_status ssd_distill_step(ssd_dtype dtype, const void* logits, int64_t ld, int32_t n_rows, int32_t vocab,
                                       const int32_t* ids, const float* vals, int32_t k, const float* weight,
                                       float temperature, float* loss, float* lse, void* dlogits, int64_t ld_d,
                                       void* stream) {
  ssd_status st = check(dtype, logits, ld, n_rows, vocab, ids, vals, k, temperature);
  if (st == SSD_OK) st = check_grad(dtype, logits, ld, n_rows, vocab, dlogits, ld_d);
  if (st != SSD_OK) return st;
  if (n_rows == 0) return SSD_OK;
  OP_REQUIRE(loss && lse, SSD_E_INVALID_ARG, "null argument");
  DistillArgs a{logits, ld, vocab, ids, vals, k, weight, 1.f / temperature, loss, lse, dlogits, ld_d};
  if (dtype == SSD_F32) launch_rows<float>(a, n_rows, true, (hipStream_t)stream);
  else launch_rows<bf16_t>(a, n_rows, true, (hipStream_t)stream);
  OP_LAUNCHED();
  return SSD_OK;
}

extern "C" ssd_status ssd_distill_backward(ssd_dtype dtype, const void* logits, int64_t ld, int32_t n_rows,
                                           int32_t vocab, const int32_t* ids, const float* vals, int32_t k,
                                           const float* lse, const float* weight, float temperature, void* dlogits,
                                           int64_t ld_d, void* stream) {
  ssd_status st = check(dtype, logits, ld, n_rows, vocab, ids, vals, k, temperature);
  if (st == SSD_OK) st = check_grad(dtype, logits, ld, n_rows, vocab, dlogits, ld_d);
  if (st != SSD_OK) return st;
  if (n_rows == 0) return SSD_OK;
  OP_REQUIRE(lse, SSD_E_INVALID_ARG, "null argument");
  DistillArgs a{logits, ld, vocab, ids, vals, k, weight, 1.f / temperature, nullptr, (float*)lse, dlogits, ld_d};
  const int per = 8 * 256 * (16 / op_size(dtype));
  const dim3 grid(n_rows, (vocab + per - 1) / per);
  if (dtype == SSD_F32) distill_grad_kernel<float><<<grid, 256, 0, (hipStream_t)stream>>>(a);
  else distill_grad_kernel<bf16_t><<<grid, 256, 0, (hipStream_t)stream>>>(a);
  OP_LAUNCHED();
  return SSD_OK;
}
