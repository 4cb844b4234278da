// Divergence of a student's logits from a teacher's top logits, and its
// gradient (ssd_distill_forward, _backward, _step of ssd_ops.h).
//
// Per row, with x_i = z_i / T and p the softmax of the teacher's slots:
//   m = max x, s = sum exp(x_i - m), lse = m + log s,
//   loss = w sum_j p_j (log p_j - (x_{id_j} - lse)),
//   dz_i = w / T (exp(x_i - lse) - sum_{j: id_j = i} p_j).
// Bound: memory.  The forward pass has to read the row, the step to read and to
// write it.
#include "ops_common.h"

namespace ssd {
namespace {

constexpr int kMaxSlots = 128;  // teacher slots of a row
constexpr int kCUs = 256;
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

typedef unsigned u32x4 __attribute__((ext_vector_type(4)));
// for outputs that lie differently from the logits
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

// A row's body is its 16-byte chunks at multiples of 16 bytes; up to E - 1
// elements lie before it and after it.  (Rows of an odd number of elements begin
// anywhere.)  Thread t < 2 E also takes edge element t, the ones before the
// body, then the ones after it.
template <typename T>
struct Row {
  static constexpr int E = Vec<T>::E;
  int head, chunks, tail, V;
  __device__ __forceinline__ Row(const T* row, int V_) : V(V_) {
    head = min((int)((16 - (uintptr_t)row % 16) % 16 / sizeof(T)), V);
    chunks = (V - head) / E;
    tail = V - head - chunks * E;
  }
  // chunk c0 + thread; -infinity where there is none.  LAST: it is not read
  // again, and need not stay in the caches.
  template <bool LAST>
  __device__ __forceinline__ u32x4 load(const T* row, int c0) const {
    u32x4 r = {Vec<T>::kNone, Vec<T>::kNone, Vec<T>::kNone, Vec<T>::kNone};
    if (c0 + (int)threadIdx.x < chunks) {
      const u32x4* at = (const u32x4*)((const char*)(row + head + (size_t)c0 * E) + 16u * threadIdx.x);
      r = LAST ? __builtin_nontemporal_load(at) : *at;
    }
    return r;
  }
  // the index of edge element t, or -1
  __device__ __forceinline__ int edge(int t) const {
    if (t < E) return t < head ? t : -1;
    return t - E < tail ? V - tail + t - E : -1;
  }
};

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
  float sum[kMaxSlots];  // of the p of all slots that name this one's token, in the first of them; 0 in the others
  float z[kMaxSlots];    // the token's logit
  float lp[kMaxSlots];   // log p
  int live;              // whether the row counts
};

// Lane l of the first wave has slots l and l + 64: their tokens (-1: left out),
// the teacher's logits and the student's.
struct Mine {
  int id[2];
  float x[2], z[2];
};

template <typename T>
__device__ __forceinline__ void fetch(const DistillArgs& a, int n, const T* row, Mine& m) {
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int j = lane + 64 * i;
    m.id[i] = -1;
    m.x[i] = -INFINITY;
    if (j < a.K) {
      const int t = a.ids[(size_t)n * a.K + j];
      const float v = a.vals[(size_t)n * a.K + j];
      if (t >= 0 && t < a.V && !(v == -INFINITY)) {
        m.id[i] = t;
        m.x[i] = v;
      }
    }
  }
#pragma unroll
  for (int i = 0; i < 2; ++i) m.z[i] = m.id[i] >= 0 ? op_ld(row, m.id[i]) : 0.f;
}

// the teacher's probabilities, by the wave that fetched
__device__ __forceinline__ void teacher(const DistillArgs& a, int n, const Mine& mine, Slots& s) {
  const int lane = threadIdx.x & 63;
  const int(&id)[2] = mine.id;
  const float(&x)[2] = mine.x;
  const bool any = __builtin_amdgcn_ballot_w64(id[0] >= 0 || id[1] >= 0) != 0;
  const float m = any ? wave_max(fmaxf(x[0], x[1])) : 0.f;
  const float c = a.inv_t * kLog2e;
  const float e0 = __builtin_amdgcn_exp2f((x[0] - m) * c), e1 = __builtin_amdgcn_exp2f((x[1] - m) * c);
  const float total = wave_sum(e0 + e1), ls = logf(total);
  const float w = a.weight ? a.weight[n] : 1.f;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int j = lane + 64 * i;
    s.id[j] = id[i];
    s.z[j] = mine.z[i];
    s.lp[j] = (x[i] - m) * a.inv_t - ls;
    s.p[j] = id[i] >= 0 ? (i ? e1 : e0) / total : 0.f;
  }
  if (lane == 0) s.live = any && w != 0.f;
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  float sum[2] = {s.p[lane], s.p[lane + 64]};
  for (int k = 0; k < a.K; ++k) {
    const int ik = s.id[k];
    const float pk = s.p[k];
#pragma unroll
    for (int i = 0; i < 2; ++i)
      if (ik == id[i] && k != lane + 64 * i) sum[i] = k < lane + 64 * i ? -INFINITY : sum[i] + pk;
  }
  // (a token named before: -infinity, whatever was added)
#pragma unroll
  for (int i = 0; i < 2; ++i) s.sum[lane + 64 * i] = sum[i] == -INFINITY ? 0.f : sum[i];
}

// Every thread's list of the teacher's tokens among its elements of a run: the
// edge element it has, and chunks c0 + i TPB + t.
template <int TPB>
struct __align__(16) Lists {
  int head[TPB];
  int next[kMaxSlots];

  // By the wave that ran teacher().  A list's order does not matter, its tokens differ.
  template <typename T>
  __device__ __forceinline__ void fill(const Slots& s, int K, const Row<T>& body, int c0, int C) {
    constexpr int E = Vec<T>::E;
#pragma unroll
    for (int i = 0; i < TPB / 256; ++i) ((int4*)head)[64 * i + threadIdx.x] = make_int4(-1, -1, -1, -1);
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    for (int j = threadIdx.x; j < K; j += 64) {
      const int id = s.id[j];
      if (id < 0 || s.sum[j] == 0.f) continue;
      int t;
      if (id < body.head || id >= body.V - body.tail) {
        if (c0) continue;
        t = id < body.head ? id : E + id - (body.V - body.tail);
      } else {
        const int c = (id - body.head) / E - c0;
        if (c < 0 || c >= C * TPB) continue;
        t = c % TPB;
      }
      next[j] = atomicExch(&head[t], j);
    }
  }
};

// A reference m and the sum of 2^(c z - m), c = log2 e / T: with m the largest
// c z for the sums of one thread, which agree on one later.
struct Stat {
  float m, s;
};
// References from here on are not used: 2^(c z - m) by one rounding (fmaf) leaves the
// row's largest entry 2^r with r the rounding of m, below 1/2 here, 2^128 for m around
// 2^32, and c z itself may overflow.  Such a row is found by its reference and
// done again by sweep().
constexpr float kFar = 16777216.f;
__device__ __forceinline__ float near_(float x) { return fminf(fmaxf(x, -kFar), kFar); }

// Keeps the compiler from holding the chunk's elements unpacked from one use
// to the next (twice the registers for bfloat16).
__device__ __forceinline__ void repack(u32x4& r) { asm volatile("" : "+v"(r)); }

// Adds a row's chunks, four at a time as their loads arrive: the arithmetic of a
// row takes about as long as its loads.
template <typename T, int FROM, int N>
__device__ __forceinline__ void add_all(Stat& a, u32x4 (&r)[N], float c) {
  if constexpr (FROM < N) {
    constexpr int E = Vec<T>::E, TO = FROM + 4 < N ? FROM + 4 : N;
    float top = -INFINITY;
#pragma unroll
    for (int i = FROM; i < TO; ++i) {
#pragma unroll
      for (int e = 0; e < E; ++e) top = fmaxf(top, Vec<T>::get(r[i], e));
      repack(r[i]);
    }
    const float m = fmaxf(a.m, near_(top * c));
    float s = a.s * __builtin_amdgcn_exp2f(a.m - m);
#pragma unroll
    for (int i = FROM; i < TO; ++i) {
#pragma unroll
      for (int e = 0; e < E; ++e) s += __builtin_amdgcn_exp2f(fmaf(Vec<T>::get(r[i], e), c, -m));
      repack(r[i]);
    }
    a.m = m;
    a.s = s;
    __builtin_amdgcn_sched_barrier(0);
    add_all<T, TO>(a, r, c);
  }
}

// Joins the workgroup's; one barrier.  c: 1, or the factor of sums whose
// references are not in units of log 2 yet.
template <int TPB>
__device__ __forceinline__ Stat block_stat(Stat a, float c, Stat* red) {
  constexpr int W = TPB / 64;
  const float top = wave_max(a.m);
  // (a thread, or a wave, all of whose entries are -infinity adds 0)
  a.s = wave_sum(a.m == -INFINITY ? a.s : a.s * __builtin_amdgcn_exp2f((a.m - top) * c));
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = (Stat){top, a.s};
  __syncthreads();
  Stat r = red[0];
#pragma unroll
  for (int i = 1; i < W; ++i) r.m = fmaxf(r.m, red[i].m);
  float t = 0.f;
#pragma unroll
  for (int i = 0; i < W; ++i)
    t += red[i].m == -INFINITY ? red[i].s : red[i].s * __builtin_amdgcn_exp2f((red[i].m - r.m) * c);
  r.s = t;
  return r;
}

// Chunk c0 + thread of the gradient, mul q' with q' its exponentials, as if the teacher had
// none of its tokens; aligned: whether out's chunks begin at multiples of 16 bytes
// as the logits' do.  The stores pass by the caches (512 float32 rows of
// 131072, step: 151 us with plain ones, 121 with these).
template <typename T>
__device__ __forceinline__ void put_chunk(T* out, const Row<T>& body, int c0, bool aligned, float mul,
                                          float (&q)[Vec<T>::E]) {
  constexpr int E = Vec<T>::E;
#pragma unroll
  for (int e = 0; e < E; ++e) q[e] *= mul;
  const u32x4 r = Vec<T>::pack(q);
  char* at = (char*)(out + body.head + (size_t)c0 * E) + 16u * threadIdx.x;
  if (aligned) __builtin_nontemporal_store(r, (u32x4*)at);
  else *(u32x4_a2*)at = r;
}

// The gradient of the thread's tokens, mul q' - f p, over what its own stores
// have put there; q(z): q' of a logit.
template <typename T, int TPB, typename Q>
__device__ __forceinline__ void put_tokens(T* out, const Slots& s, const Lists<TPB>& lists, float mul, float f, Q q) {
  for (int j = lists.head[threadIdx.x]; j >= 0; j = lists.next[j])
    op_st(out, s.id[j], q(s.z[j]) * mul - s.sum[j] * f);
}

// the gradient of a row that does not count: chunks c0 .. c1 - 1, and edge element `edge`
template <typename T, int TPB>
__device__ __forceinline__ void put_zeros(T* out, const Row<T>& row, int c0, int c1, int edge) {
  for (int c = c0 + threadIdx.x; c < min(c1, row.chunks); c += TPB)
    *(u32x4_a2*)(out + row.head + (size_t)c * Vec<T>::E) = (u32x4){0, 0, 0, 0};
  if (edge >= 0) op_st(out, edge, 0.f);
}

// The row's loss, by the wave that ran teacher().  logq(z): log q of a logit, from its
// difference to the reference (log q = z / T - lse would carry the rounding of two large numbers).
template <typename Q>
__device__ __forceinline__ void put_loss(const DistillArgs& a, int n, const Slots& s, float lse, Q logq) {
  const int lane = threadIdx.x & 63;
  float l = 0.f;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const float p = s.p[lane + 64 * i];
    if (p != 0.f) l += p * (s.lp[lane + 64 * i] - logq(s.z[lane + 64 * i]));
  }
  l = wave_sum(l);
  if (lane == 0) {
    a.loss[n] = s.live ? l * (a.weight ? a.weight[n] : 1.f) : 0.f;
    a.lse[n] = lse;
  }
}

// what is taken from z: the maximum, or 0 where all entries are -infinity
__device__ __forceinline__ float ref_of(float m) { return m == -INFINITY ? 0.f : m; }

// A row by two sweeps over it: the maximum and sum, then the gradient.  The
// difference z - maximum comes before the factor c, for logits of any size.
// The first wave has run teacher().
template <typename T, int TPB, bool GRAD>
__device__ void sweep(const DistillArgs& a, int n, const Row<T>& body, int edge, float ze, const Slots& slots,
                      Lists<TPB>& lists, Stat* red) {
  constexpr int E = Vec<T>::E, U = 4, SEG = 64;
  const int t = threadIdx.x, chunks = body.chunks;
  const T* row = (const T*)a.logits + (size_t)n * a.ld;
  const float c2 = a.inv_t * kLog2e;
  Stat st = {ze, edge >= 0 && ze != -INFINITY ? 1.f : 0.f};
  for (int c = 0; c < chunks; c += U * TPB) {
    u32x4 r[U];
#pragma unroll
    for (int i = 0; i < U; ++i) r[i] = body.template load<!GRAD>(row, c + i * TPB);
    float top = st.m;
#pragma unroll
    for (int i = 0; i < U; ++i)
#pragma unroll
      for (int e = 0; e < E; ++e) top = fmaxf(top, Vec<T>::get(r[i], e));
    const float ref = ref_of(top);
    float s = st.s * __builtin_amdgcn_exp2f((st.m - ref) * c2);
#pragma unroll
    for (int i = 0; i < U; ++i)
#pragma unroll
      for (int e = 0; e < E; ++e) s += __builtin_amdgcn_exp2f((Vec<T>::get(r[i], e) - ref) * c2);
    st.m = top;
    st.s = s;
  }
  __syncthreads();  // (red may still be read)
  st = block_stat<TPB>(st, c2, red);
  const float ref = ref_of(st.m);
  if (GRAD) {
    T* out = (T*)a.grad + (size_t)n * a.ld_d;
    const bool aligned = (uintptr_t)out % 16 == (uintptr_t)row % 16;
    const float f = (a.weight ? a.weight[n] : 1.f) * a.inv_t, mul = f / st.s;
    if (!slots.live) put_zeros<T, TPB>(out, body, 0, chunks, edge);
    else
      for (int c0 = 0; c0 == 0 || c0 < chunks; c0 += SEG * TPB) {
        __syncthreads();
        if (t < 64) lists.fill(slots, a.K, body, c0, SEG);
        __syncthreads();
        auto q1 = [&](float x) { return __builtin_amdgcn_exp2f((x - ref) * c2); };
        if (c0 == 0 && edge >= 0) op_st(out, edge, q1(ze) * mul);
        for (int i0 = 0; i0 < SEG && c0 + i0 * TPB < chunks; i0 += U) {
          u32x4 r[U];
#pragma unroll
          for (int i = 0; i < U; ++i) r[i] = body.template load<true>(row, c0 + (i0 + i) * TPB);
#pragma unroll
          for (int i = 0; i < U; ++i) {
            const int c = c0 + (i0 + i) * TPB;
            if (c + t >= chunks) continue;
            float q[E];
#pragma unroll
            for (int e = 0; e < E; ++e) q[e] = q1(Vec<T>::get(r[i], e));
            put_chunk(out, body, c, aligned, mul, q);
          }
        }
        put_tokens(out, slots, lists, mul, f, q1);
      }
  }
  const float ls = logf(st.s);
  if (t < 64) put_loss(a, n, slots, ref * a.inv_t + ls, [&](float z) { return (z - ref) * a.inv_t - ls; });
}

// One workgroup per row of any length, read twice for the gradient (512 float32 rows of
// 140000: 127 us; 4096 of 65000, loss alone: 159, 6.7 TB/s).
template <typename T, bool GRAD>
__global__ __launch_bounds__(1024) void distill_sweep_kernel(DistillArgs a) {
  constexpr int TPB = 1024, E = Vec<T>::E;
  __shared__ Slots slots;
  __shared__ Lists<TPB> lists;
  __shared__ Stat red[TPB / 64];
  const int n = blockIdx.x, t = threadIdx.x;
  const T* row = (const T*)a.logits + (size_t)n * a.ld;
  const Row<T> body(row, a.V);
  const int edge = t < 2 * E ? body.edge(t) : -1;
  const float ze = edge >= 0 ? op_ld(row, edge) : -INFINITY;
  Mine mine;
  if (t < 64) {
    fetch(a, n, row, mine);
    teacher(a, n, mine, slots);
  }
  sweep<T, TPB, GRAD>(a, n, body, edge, ze, slots, lists, red);
}

// One workgroup per row, which its registers hold: C chunks a thread.
// W: waves per SIMD that its registers leave room for.  Bound: memory (4096 bfloat16
// rows of 50257, step: 162 us, 5.1 TB/s).
template <typename T, int TPB, int C, int W, bool GRAD>
__global__ __launch_bounds__(TPB, W) void distill_row_kernel(DistillArgs a) {
  constexpr int E = Vec<T>::E;
  __shared__ Slots slots;
  __shared__ Lists<TPB> lists;
  __shared__ Stat red[TPB / 64];
  const int n = blockIdx.x, t = threadIdx.x;
  const T* row = (const T*)a.logits + (size_t)n * a.ld;
  const Row<T> body(row, a.V);
  const int edge = t < 2 * E ? body.edge(t) : -1;
  const float ze = edge >= 0 ? op_ld(row, edge) : -INFINITY;
  Mine mine;
  if (t < 64) fetch(a, n, row, mine);  // (first: all else waits for it less long than it would for the row)
  u32x4 r[C];
#pragma unroll
  for (int i = 0; i < C; ++i) r[i] = body.template load<true>(row, i * TPB);
  if (t < 64) {
    teacher(a, n, mine, slots);
    if (GRAD) lists.fill(slots, a.K, body, 0, C);
  }
  const float c2 = a.inv_t * kLog2e;
  Stat st;
  st.m = near_(ze * c2);
  st.s = __builtin_amdgcn_exp2f(fmaf(ze, c2, -st.m));
  add_all<T, 0>(st, r, c2);
  st = block_stat<TPB>(st, 1.f, red);
  if (!(fabsf(st.m) < kFar)) return sweep<T, TPB, GRAD>(a, n, body, edge, ze, slots, lists, red);
  if (GRAD) {
    T* out = (T*)a.grad + (size_t)n * a.ld_d;
    const float f = (a.weight ? a.weight[n] : 1.f) * a.inv_t, mul = f / st.s;
    if (slots.live) {
      const bool aligned = (uintptr_t)out % 16 == (uintptr_t)row % 16;
      auto q1 = [&](float x) { return __builtin_amdgcn_exp2f(fmaf(x, c2, -st.m)); };
      if (edge >= 0) op_st(out, edge, q1(ze) * mul);
#pragma unroll
      for (int i = 0; i < C; ++i) {
        if (i * TPB + t >= body.chunks) continue;
        float q[E];
#pragma unroll
        for (int e = 0; e < E; ++e) q[e] = q1(Vec<T>::get(r[i], e));
        put_chunk(out, body, i * TPB, aligned, mul, q);
      }
      put_tokens(out, slots, lists, mul, f, q1);
    } else {
      put_zeros<T, TPB>(out, body, 0, body.chunks, edge);
    }
  }
  const float ls = __log2f(st.s);
  if (t < 64) put_loss(a, n, slots, (st.m + ls) * kLn2, [&](float z) { return (fmaf(z, c2, -st.m) - ls) * kLn2; });
}

// The gradient from a known log-sum-exp: a workgroup per row and C chunks a thread.
// Rows of more than one part: 512 threads (3000 bfloat16 rows of 50257: 127 us with
// 256 threads, 117 with 512; 1500 float32 rows 127 and 125), shorter ones 256 (4096
// bfloat16 rows of 8000: 30 and 39).
constexpr int kGradChunks = 8;
template <typename T, int TPB>
__global__ __launch_bounds__(TPB) void distill_grad_kernel(DistillArgs a) {
  constexpr int E = Vec<T>::E, C = kGradChunks;
  __shared__ Slots slots;
  __shared__ Lists<TPB> lists;
  const int n = blockIdx.x, c0 = blockIdx.y * (C * TPB), t = threadIdx.x;
  const T* row = (const T*)a.logits + (size_t)n * a.ld;
  T* out = (T*)a.grad + (size_t)n * a.ld_d;
  const Row<T> body(row, a.V);
  const int chunks = body.chunks, edge = blockIdx.y == 0 && t < 2 * E ? body.edge(t) : -1;
  if (c0 >= chunks && blockIdx.y) return;
  const float ze = edge >= 0 ? op_ld(row, edge) : 0.f;
  Mine mine;
  if (t < 64) fetch(a, n, row, mine);
  u32x4 r[C];
#pragma unroll
  for (int i = 0; i < C; ++i) r[i] = body.template load<true>(row, c0 + i * TPB);
  if (t < 64) {
    teacher(a, n, mine, slots);
    lists.fill(slots, a.K, body, c0, C);
  }
  __syncthreads();
  const bool aligned = (uintptr_t)out % 16 == (uintptr_t)row % 16;
  const float f = (a.weight ? a.weight[n] : 1.f) * a.inv_t, lse = a.lse[n];
  if (!slots.live) return put_zeros<T, TPB>(out, body, c0, c0 + C * TPB, edge);
  // (the difference before the factor log2 e: 2^(c z - lse log2 e) would carry the rounding of two large numbers)
  auto q1 = [&](float x) { return __expf(fmaf(x, a.inv_t, -lse)); };
  if (edge >= 0) op_st(out, edge, q1(ze) * f);
#pragma unroll
  for (int i = 0; i < C; ++i) {
    const int c = c0 + i * TPB;
    if (c + t >= chunks) continue;
    float q[E];
#pragma unroll
    for (int e = 0; e < E; ++e) q[e] = q1(Vec<T>::get(r[i], e));
    put_chunk(out, body, c, aligned, f, q);
  }
  put_tokens(out, slots, lists, f, f, q1);
}

ssd_status check(int dtype, const void* logits, int64_t ld, int n, int V, const int* ids, const float* vals, int k,
                 float temperature) {
  OP_REQUIRE(op_dtype(dtype), SSD_E_INVALID_ARG, "dtype must be SSD_F32 or SSD_BF16");
  OP_REQUIRE(n >= 0, SSD_E_INVALID_ARG, "n_rows is negative");
  OP_REQUIRE(V >= 1 && V <= 1 << 24, SSD_E_INVALID_ARG, "vocab outside [1, 2^24]");
  OP_REQUIRE(k >= 1 && k <= kMaxSlots, SSD_E_INVALID_ARG, "k outside [1, 128]");
  OP_REQUIRE(temperature > 0.f && temperature < INFINITY && 1.f / temperature * kLog2e < INFINITY, SSD_E_INVALID_ARG,
             "temperature and its reciprocal, times log2 e, must be positive and finite");
  OP_REQUIRE(ld >= V, SSD_E_INVALID_ARG, "the logits' row stride is below vocab");
  OP_REQUIRE(n == 0 || (logits && ids && vals), SSD_E_INVALID_ARG, "null argument");
  OP_REQUIRE((uintptr_t)logits % op_size(dtype) == 0, SSD_E_INVALID_ARG, "logits not aligned to their type");
  return SSD_OK;
}

ssd_status check_grad(int dtype, const void* logits, int64_t ld, int n, int V, const void* grad, int64_t ld_d) {
  OP_REQUIRE(ld_d >= V, SSD_E_INVALID_ARG, "dlogits' row stride is below vocab");
  OP_REQUIRE(n == 0 || grad, SSD_E_INVALID_ARG, "null argument");
  OP_REQUIRE((uintptr_t)grad % op_size(dtype) == 0, SSD_E_INVALID_ARG, "dlogits not aligned to their type");
  OP_REQUIRE((grad == logits && ld == ld_d) || op_apart(op_matrix(logits, n, ld, V, op_size(dtype)),
                                                        op_matrix(grad, n, ld_d, V, op_size(dtype))),
             SSD_E_INVALID_ARG, "dlogits overlaps the logits without being them");
  return SSD_OK;
}

// How a row is held: TPB threads with up to C chunks each.  One row a CU at most:
// more threads are sooner done with it (64 float32 rows of 50257, step: 15.5 us with
// 256 threads, 11.9 with 512, 11.1 with 1024).  More rows: few threads with many
// chunks, so that two to four rows are on a CU and one's loads and stores run beside
// another's arithmetic and waits (4096 bfloat16 rows of 32000, step: 98 us with 256
// threads, 101 with 512, 147 with 1024), up to what their registers hold with few
// spilled (the step's instances of 13 chunks and more than 512 threads, of 16 and of 48
// spill 3 to 10 each, 256 threads of 16 chunks of float32 none; 4096 bfloat16 rows of
// 50257: 170, 157, 197; float32: 332, 325, 316).  The step of longer rows keeps them in 512
// threads, few rows too (4096 float32 rows of 65000: 427 us, 465 in two sweeps; 256 rows
// 29, 4.6 TB/s, of 90000 36, 5.1).  The loss alone reads a row once either way: long rows are swept
// (4096 float32 rows of 65000: 193 us with 512 threads, 159 swept; of 20000: 54 with 256, 68).
template <typename T, bool GRAD>
void launch_rows(const DistillArgs& a, int n, hipStream_t s) {
  const int chunks = a.V / Vec<T>::E;
#define ROWS(TPB, C, W) \
  if (chunks <= TPB * C) return distill_row_kernel<T, TPB, C, W, GRAD><<<n, TPB, 0, s>>>(a);
  ROWS(256, 4, 6)
  if (n <= kCUs) {
    ROWS(1024, 4, 4)
    ROWS(1024, 7, 4)
    ROWS(1024, 13, 4)
  }
  ROWS(256, 10, 4)
  ROWS(256, 16, 4)
  if constexpr (GRAD) {
    ROWS(512, 13, 4)
    ROWS(512, 16, 4)
    ROWS(1024, 13, 4)
    ROWS(512, 32, 2)
    ROWS(512, 48, 2)
  } else {
    ROWS(256, 25, 3)
  }
#undef ROWS
  return distill_sweep_kernel<T, GRAD><<<n, 1024, 0, s>>>(a);
}

template <typename T>
void launch_grad(const DistillArgs& a, int n, hipStream_t s) {
  constexpr int per = kGradChunks * Vec<T>::E;  // elements a thread
  if (a.V <= 256 * per) distill_grad_kernel<T, 256><<<dim3(n, 1), 256, 0, s>>>(a);
  else distill_grad_kernel<T, 512><<<dim3(n, (a.V + 512 * per - 1) / (512 * per)), 512, 0, s>>>(a);
}

// Calls launch(arguments, rows) for at most kSlice rows at a time: a grid holds
// fewer than 2^32 threads.
constexpr int kSlice = 1 << 21;
template <typename T, typename Launch>
hipError_t by_slices(DistillArgs a, int n, Launch launch) {
  for (;;) {
    const int rows = n < kSlice ? n : kSlice;
    launch(a, rows);
    const hipError_t e = hipGetLastError();
    n -= rows;
    if (e != hipSuccess || n == 0) return e;
    a.logits = (const T*)a.logits + (size_t)rows * a.ld;
    a.ids += (size_t)rows * a.K;
    a.vals += (size_t)rows * a.K;
    a.lse += rows;
    if (a.weight) a.weight += rows;
    if (a.loss) a.loss += rows;
    if (a.grad) a.grad = (T*)a.grad + (size_t)rows * a.ld_d;
  }
}

template <typename T, bool GRAD>
hipError_t rows(const DistillArgs& a, int n, hipStream_t s) {
  return by_slices<T>(a, n, [s](const DistillArgs& x, int m) { launch_rows<T, GRAD>(x, m, s); });
}
template <typename T>
hipError_t gradient(const DistillArgs& a, int n, hipStream_t s) {
  return by_slices<T>(a, n, [s](const DistillArgs& x, int m) { launch_grad<T>(x, m, s); });
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
  const hipError_t e = dtype == SSD_F32 ? rows<float, false>(a, n_rows, (hipStream_t)stream)
                                        : rows<bf16_t, false>(a, n_rows, (hipStream_t)stream);
  if (e != hipSuccess) return op_fail(SSD_E_DEVICE, hipGetErrorString(e));
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
  const hipError_t e = dtype == SSD_F32 ? rows<float, true>(a, n_rows, (hipStream_t)stream)
                                        : rows<bf16_t, true>(a, n_rows, (hipStream_t)stream);
  if (e != hipSuccess) return op_fail(SSD_E_DEVICE, hipGetErrorString(e));
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
  const hipError_t e = dtype == SSD_F32 ? gradient<float>(a, n_rows, (hipStream_t)stream)
                                        : gradient<bf16_t>(a, n_rows, (hipStream_t)stream);
  if (e != hipSuccess) return op_fail(SSD_E_DEVICE, hipGetErrorString(e));
  return SSD_OK;
}
