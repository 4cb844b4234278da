// Attention of a batch of sequences over a prefix they share and over their
// own rows (ssd_prefix_attn of ssd_ops.h).
//
// With x_j the scaled score of row j, in units of log 2, and a set c of rows:
//   m_c >= max x_j - 8,  l_c = sum 2^(x_j - m_c),  o_c = sum 2^(x_j - m_c) v_j;
// out = sum_c 2^(m_c - M) o_c / sum_c 2^(m_c - M) l_c with M the largest m_c.
// The shared rows are read once for all queries of a kv head: the queries of
// every sequence and of the head's group are the columns of one product.
//
// A workgroup of four waves takes a tile of queries (16 per matrix tile) and a
// chunk of rows, either of the prefix or of one sequence's own, and leaves one
// part (m, l, o) per query; merge_kernel adds a query's parts.  Its waves take the
// chunk's blocks of rows in turn and never wait for each other until the end: a
// wave copies its blocks' keys and values into LDS of its own, one block ahead.
#include <algorithm>
#include <atomic>

#include "ops_common.h"

namespace ssd {
namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef unsigned u32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef unsigned u32x2 __attribute__((ext_vector_type(2)));
typedef __attribute__((address_space(3))) unsigned char lds_byte;

struct Range {  // rows of keys and values side by side
  const char *k, *v;
  int64_t row;  // bytes from row to row
};

struct PrefixAttnArgs {
  ssd_prefix_attn_desc d;
  const void *q, *kp, *vp, *ko, *vo;
  const int* own_len;
  void* out;
  float* lse;
  float2* ml;   // [query][parts] (m, l) with query = (sequence, position, head)
  float* o;     // [query][parts][head_dim]
  int p_tiles, p_chunks, p_chunk, p_blocks;  // query tiles and chunks of the prefix, its rows per chunk, its workgroups
  int o_tiles, o_chunks, o_chunk;            // of a sequence's own rows
  int parts;                                 // p_chunks + o_chunks
  float scale2;                              // scale times log2 e
};

constexpr int kWaves = 4;
constexpr float kSlack = 8.f;  // how far a score may lie above the reference before the sums are rescaled

// A block of rows in LDS: KB rows of keys, then of values, CH 16-byte chunks each.
// Chunk c of row r lies at place c ^ swizzle(r), so that the lanes of one read
// fall on different banks: 16 rows at one chunk (keys, 16 bytes a lane), or four
// rows a group of 16 lanes at 16 dims (values).
template <typename T, int D>
struct Block {
  static constexpr int KB = sizeof(T) == 2 ? 32 : 16, ROW = D * (int)sizeof(T), CH = ROW / 16;
  static constexpr int BYTES = KB * ROW, LOADS = BYTES / 1024;  // of the keys, and of the values
  static __device__ __forceinline__ int swz_k(int r) {
    return CH == 4 ? (r >> 2) & 3 : CH == 8 ? (r >> 1) & 7 : r & 15;
  }
  static __device__ __forceinline__ int swz_v(int r) {
    if (sizeof(T) == 2) return 2 * (CH == 4 ? (r >> 2) & 1 : CH == 8 ? (r >> 1) & 3 : r & 7);
    return 4 * (CH == 8 ? (r >> 2) & 1 : (r >> 2) & 3);
  }
};

// Copies rows kb .. kb + KB - 1 of a range (those from `end` on: row end - 1
// again) into the wave's LDS at dst.  By a whole wave; 2 LOADS copies in flight.
template <typename T, int D>
__device__ __forceinline__ void issue(const Range& s, int kb, int end, unsigned char* dst) {
  typedef Block<T, D> B;
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int half = 0; half < 2; ++half) {
    const char* base = half ? s.v : s.k;
#pragma unroll
    for (int i = 0; i < B::LOADS; ++i) {
      const int p = i * 64 + lane, r = p / B::CH, c = (p % B::CH) ^ (half ? B::swz_v(r) : B::swz_k(r));
      const char* src = base + (int64_t)min(kb + r, end - 1) * s.row + 16 * c;
      __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)src,
                                       (__attribute__((address_space(3))) void*)(dst + half * B::BYTES + i * 1024), 16,
                                       0, 0);
    }
  }
}

// the wave's copies but the last N are in LDS
template <int N>
__device__ __forceinline__ void copies_landed() {
  static_assert(N < 64, "the wait counts to 63");
  __builtin_amdgcn_sched_barrier(0);
  __builtin_amdgcn_s_waitcnt((N & 15) | ((N >> 4) << 14) | (7 << 4) | (15 << 8));
  asm volatile("" ::: "memory");
  __builtin_amdgcn_sched_barrier(0);
}

// Transposing LDS reads: 64 bits a lane at each address and OFF bytes above it.  As
// one block with its wait: the compiler takes such a read to depend on every
// copy into LDS in flight and would wait for them all.
template <int OFF>
__device__ __forceinline__ void read_transposed(unsigned a0, unsigned a1, u32x2 (&f0)[2], u32x2 (&f1)[2]) {
  asm volatile(
      "ds_read_b64_tr_b16 %0, %4\n"
      "ds_read_b64_tr_b16 %1, %4 offset:%6\n"
      "ds_read_b64_tr_b16 %2, %5\n"
      "ds_read_b64_tr_b16 %3, %5 offset:%6\n"
      "s_waitcnt lgkmcnt(0)"
      : "=&v"(f0[0]), "=&v"(f0[1]), "=&v"(f1[0]), "=&v"(f1[1])
      : "v"(a0), "v"(a1), "n"(OFF)
      : "memory");
}
template <int OFF>
__device__ __forceinline__ void read_transposed(unsigned a0, unsigned a1, unsigned a2, unsigned a3, u32x2 (&f0)[2],
                                                u32x2 (&f1)[2], u32x2 (&f2)[2], u32x2 (&f3)[2]) {
  asm volatile(
      "ds_read_b64_tr_b16 %0, %8\n"
      "ds_read_b64_tr_b16 %1, %8 offset:%12\n"
      "ds_read_b64_tr_b16 %2, %9\n"
      "ds_read_b64_tr_b16 %3, %9 offset:%12\n"
      "ds_read_b64_tr_b16 %4, %10\n"
      "ds_read_b64_tr_b16 %5, %10 offset:%12\n"
      "ds_read_b64_tr_b16 %6, %11\n"
      "ds_read_b64_tr_b16 %7, %11 offset:%12\n"
      "s_waitcnt lgkmcnt(0)"
      : "=&v"(f0[0]), "=&v"(f0[1]), "=&v"(f1[0]), "=&v"(f1[1]), "=&v"(f2[0]), "=&v"(f2[1]), "=&v"(f3[0]),
        "=&v"(f3[1])
      : "v"(a0), "v"(a1), "v"(a2), "v"(a3), "n"(OFF)
      : "memory");
}

// the operands and products of one type: S^T (keys x queries) and O^T (dims x queries)
template <typename T, int D, int MT>
struct Math;

template <int D, int MT>
struct Math<bf16_t, D, MT> {
  typedef Block<bf16_t, D> B;
  static constexpr int KT = 2, KK = D / 32, DT = D / 16;
  // lane l: keys 4 (l / 16) + r of each 16-key tile, query l % 16
  static __device__ __forceinline__ void scores(const unsigned char* k, const u32x4 (&q)[MT][KK], f32x4 (&s)[MT][KT]) {
    const int lane = threadIdx.x & 63, n = lane & 15, g = lane >> 4;
#pragma unroll
    for (int kt = 0; kt < KT; ++kt)
#pragma unroll
      for (int kk = 0; kk < KK; ++kk) {
        const int r = 16 * kt + n;
        const u32x4 f = *(const u32x4*)(k + r * B::ROW + 16 * ((4 * kk + g) ^ B::swz_k(r)));
#pragma unroll
        for (int mt = 0; mt < MT; ++mt)
          s[mt][kt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, f),
                                                              __builtin_bit_cast(bf16x8, q[mt][kk]),
                                                              kk ? s[mt][kt] : (f32x4){0.f, 0.f, 0.f, 0.f}, 0, 0, 0);
      }
  }
  struct P {
    u32x4 w[MT];
  };
  // the weights as the second product's operand: its lane needs the keys it holds already
  static __device__ __forceinline__ void weights(const f32x4 (&s)[MT][KT], P& p) {
#pragma unroll
    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
      for (int kt = 0; kt < KT; ++kt)
#pragma unroll
        for (int h = 0; h < 2; ++h)
          p.w[mt][2 * kt + h] = __builtin_bit_cast(
              unsigned, __builtin_convertvector((f32x2){s[mt][kt][2 * h], s[mt][kt][2 * h + 1]}, bf16x2));
  }
  // the values' operand: lane l has dim 16 dt + l % 16 of the keys its weights are of
  struct V {
    u32x2 f[DT][2];
  };
  static __device__ __forceinline__ void values(const unsigned char* v, V& x) {
    // a 16-lane group reads four rows of 16 dims and gets them transposed
    const int lane = threadIdx.x & 63, r = 4 * (lane >> 4) + ((lane & 15) >> 2);
    const unsigned at = (unsigned)(size_t)(lds_byte*)v + r * B::ROW + 16 * (((lane & 3) >> 1) ^ B::swz_v(r)) +
                        8 * (lane & 1);
    if constexpr (DT == 2) read_transposed<16 * B::ROW>(at, at ^ 32, x.f[0], x.f[1]);
    else
#pragma unroll
      for (int dt = 0; dt < DT; dt += 4)
        read_transposed<16 * B::ROW>(at ^ (32 * dt), at ^ (32 * (dt + 1)), at ^ (32 * (dt + 2)), at ^ (32 * (dt + 3)),
                                     x.f[dt], x.f[dt + 1], x.f[dt + 2], x.f[dt + 3]);
  }
  // clears infinities and NaNs; whether there were any
  static __device__ __forceinline__ bool clear(V& x) {
    bool bad = false;
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const unsigned e = h ? 0x7f800000u : 0x7f80u;
          if ((x.f[dt][i >> 1][i & 1] & e) == e) {
            x.f[dt][i >> 1][i & 1] &= h ? 0xffffu : 0xffff0000u;
            bad = true;
          }
        }
    return bad;
  }
  static __device__ __forceinline__ void add(const V& x, const P& p, f32x4 (&o)[MT][DT]) {
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) {
      const u32x4 f = {x.f[dt][0][0], x.f[dt][0][1], x.f[dt][1][0], x.f[dt][1][1]};
#pragma unroll
      for (int mt = 0; mt < MT; ++mt)
        o[mt][dt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, f),
                                                            __builtin_bit_cast(bf16x8, p.w[mt]), o[mt][dt], 0, 0, 0);
    }
  }
};

template <int D, int MT>
struct Math<float, D, MT> {
  typedef Block<float, D> B;
  static constexpr int KT = 1, KK = D / 16, DT = D / 16;
  static __device__ __forceinline__ void scores(const unsigned char* k, const u32x4 (&q)[MT][KK], f32x4 (&s)[MT][KT]) {
    const int lane = threadIdx.x & 63, n = lane & 15, g = lane >> 4;
#pragma unroll
    for (int kk = 0; kk < KK; ++kk) {
      const u32x4 f = *(const u32x4*)(k + n * B::ROW + 16 * ((4 * kk + g) ^ B::swz_k(n)));
#pragma unroll
      for (int c = 0; c < 4; ++c)
#pragma unroll
        for (int mt = 0; mt < MT; ++mt)
          s[mt][0] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(f[c]), __uint_as_float(q[mt][kk][c]),
                                                          kk || c ? s[mt][0] : (f32x4){0.f, 0.f, 0.f, 0.f}, 0, 0, 0);
    }
  }
  struct P {
    f32x4 w[MT];
  };
  static __device__ __forceinline__ void weights(const f32x4 (&s)[MT][KT], P& p) {
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) p.w[mt] = s[mt][0];
  }
  struct V {
    f32x4 f[DT];
  };
  static __device__ __forceinline__ void values(const unsigned char* v, V& x) {
    const int lane = threadIdx.x & 63, n = lane & 15, g = lane >> 4;
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int row = 4 * g + r;
        x.f[dt][r] = *(const float*)(v + row * B::ROW + 16 * ((4 * dt + (n >> 2)) ^ B::swz_v(row)) + 4 * (n & 3));
      }
  }
  static __device__ __forceinline__ bool clear(V& x) {
    bool bad = false;
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
      for (int r = 0; r < 4; ++r)
        if (!(fabsf(x.f[dt][r]) < INFINITY)) {
          x.f[dt][r] = 0.f;
          bad = true;
        }
    return bad;
  }
  static __device__ __forceinline__ void add(const V& x, const P& p, f32x4 (&o)[MT][DT]) {
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
      for (int r = 0; r < 4; ++r)
#pragma unroll
        for (int mt = 0; mt < MT; ++mt)
          o[mt][dt] = __builtin_amdgcn_mfma_f32_16x16x4f32(x.f[dt][r], p.w[mt][r], o[mt][dt], 0, 0, 0);
  }
};

// dim i of row r of a block's values
template <typename T, int D>
__device__ __forceinline__ float value_at(const unsigned char* v, int r, int i) {
  const int c = i * (int)sizeof(T) / 16;
  return op_ld((const T*)(v + r * Block<T, D>::ROW + 16 * (c ^ Block<T, D>::swz_v(r))), i % (16 / (int)sizeof(T)));
}

// The queries of a tile of MT x 16 columns from `first` on: of the prefix, all
// (sequence, position, group member) of kv head h; of own rows, sequence b's.
struct Queries {
  int h, b;     // b < 0: of every sequence
  int first, count;
  __device__ __forceinline__ void split(const ssd_prefix_attn_desc& d, int i, int& seq, int& t, int& head) const {
    const int G = d.n_head / d.n_kv_head, tg = d.n_query * G;
    seq = b < 0 ? i / tg : b;
    const int r = b < 0 ? i - seq * tg : i;
    t = r / G;
    head = h * G + (r - t * G);
  }
};

// One workgroup's work: queries against rows [k0, k1) of a range, the part left
// in slot `part`.  own: query t sees rows below len - n_query + 1 + t.
template <typename T, int D, int MT>
__device__ __forceinline__ void attend(const PrefixAttnArgs& a, const Queries& qs, const Range& range, int k0, int k1,
                                       int len, int part, unsigned char* lds) {
  typedef Block<T, D> B;
  typedef Math<T, D, MT> M;
  constexpr int KB = B::KB, KT = M::KT, KK = M::KK, DT = M::DT, STAGE = 2 * B::BYTES;
  const ssd_prefix_attn_desc& d = a.d;
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), n = lane & 15, g = lane >> 4;
  unsigned char* ring = lds + w * (2 * STAGE);
  int kb = k0 + w * KB;
  if (kb < k1) issue<T, D>(range, kb, k1, ring);
  if (kb + kWaves * KB < k1) issue<T, D>(range, kb + kWaves * KB, k1, ring + STAGE);

  u32x4 q[MT][KK];
  int lim[MT];  // rows this lane's queries see end here
#pragma unroll
  for (int mt = 0; mt < MT; ++mt) {
    int seq, t, head;
    qs.split(d, min(qs.first + 16 * mt + n, qs.count - 1), seq, t, head);
    const T* row = (const T*)a.q + (int64_t)seq * d.q_seq + (int64_t)t * d.q_row + (int64_t)head * d.q_head;
#pragma unroll
    for (int kk = 0; kk < KK; ++kk) q[mt][kk] = *((const u32x4*)row + 4 * kk + g);
    lim[mt] = qs.b < 0 ? k1 : min(k1, len - d.n_query + 1 + t);
  }
  const int all = qs.b < 0 ? k1 : min(k1, len - d.n_query + 1);  // rows below are seen by every query

  f32x4 o[MT][DT];
  float m[MT], l[MT];
#pragma unroll
  for (int mt = 0; mt < MT; ++mt) {
    m[mt] = -INFINITY;
    l[mt] = 0.f;
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) o[mt][dt] = (f32x4){0.f, 0.f, 0.f, 0.f};
  }

  int buf = 0;
  for (; kb < k1; kb += kWaves * KB, buf ^= 1) {
    if (kb + kWaves * KB < k1) copies_landed<2 * B::LOADS>();
    else copies_landed<0>();
    const unsigned char *k = ring + buf * STAGE, *v = k + B::BYTES;
    f32x4 s[MT][KT];
    M::scores(k, q, s);
    const bool masked = kb + KB > all;
#pragma unroll
    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
      for (int kt = 0; kt < KT; ++kt) {
        // (read here, in the products' own block: read past a branch, float32
        // products of two tiles were taken before they were complete)
        s[mt][kt] *= a.scale2;
        asm volatile("" : "+v"(s[mt][kt]));
      }
    if (masked) {
#pragma unroll
      for (int mt = 0; mt < MT; ++mt)
#pragma unroll
        for (int kt = 0; kt < KT; ++kt)
#pragma unroll
          for (int r = 0; r < 4; ++r)
            if (kb + 16 * kt + 4 * g + r >= lim[mt]) s[mt][kt][r] = -INFINITY;
    }
    bool above = false;
#pragma unroll
    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
      for (int kt = 0; kt < KT; ++kt)
#pragma unroll
        for (int r = 0; r < 4; ++r) above |= s[mt][kt][r] > m[mt] + kSlack;
    if (__builtin_amdgcn_ballot_w64(above)) {  // a new reference: the largest score so far
#pragma unroll
      for (int mt = 0; mt < MT; ++mt) {
        float top = m[mt];
#pragma unroll
        for (int kt = 0; kt < KT; ++kt)
#pragma unroll
          for (int r = 0; r < 4; ++r) top = fmaxf(top, s[mt][kt][r]);
        top = fmaxf(top, __shfl_xor(top, 16));
        top = fmaxf(top, __shfl_xor(top, 32));
        const float c = top == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m[mt] - top);
        m[mt] = top;
        l[mt] *= c;
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) o[mt][dt] *= c;
      }
    }
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
      const float ref = m[mt] == -INFINITY ? 0.f : m[mt];
#pragma unroll
      for (int kt = 0; kt < KT; ++kt)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          s[mt][kt][r] = __builtin_amdgcn_exp2f(s[mt][kt][r] - ref);
          l[mt] += s[mt][kt][r];
        }
    }
    typename M::P p;
    M::weights(s, p);
    typename M::V x;
    M::values(v, x);
    bool bad = false;
    if (masked) bad = M::clear(x);
    M::add(x, p, o);
    if (masked && __builtin_amdgcn_ballot_w64(bad)) {
      // weights of 0 do not silence an infinity or NaN: those values are added to
      // the queries that see their rows
      for (int r = 0; r < KB; ++r)
#pragma unroll
        for (int dt = 0; dt < DT; ++dt)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const float y = value_at<T, D>(v, r, 16 * dt + 4 * g + i);
            if (!(fabsf(y) < INFINITY)) {
#pragma unroll
              for (int mt = 0; mt < MT; ++mt)
                if (kb + r < lim[mt]) o[mt][dt][i] += y;
            }
          }
    }
    if (kb + 2 * kWaves * KB < k1) {
      // (the block's reads are over: their results went into the products above)
      __builtin_amdgcn_sched_barrier(0);
      __builtin_amdgcn_s_waitcnt(0xc07f);  // lgkmcnt(0)
      asm volatile("" ::: "memory");
      issue<T, D>(range, kb + 2 * kWaves * KB, k1, ring + buf * STAGE);
    }
  }

  // the four waves' sums, through LDS: a wave's area of the ring holds its o
  // (columns of D floats), as large as it needs with 4 query tiles
  static_assert(MT * 16 * D * 4 <= 2 * STAGE, "a wave's outputs fit its part of the ring");
  __shared__ float ref_s[kWaves][MT * 16], sum_s[kWaves][MT * 16];
#pragma unroll
  for (int mt = 0; mt < MT; ++mt) {
    l[mt] += __shfl_xor(l[mt], 16);
    l[mt] += __shfl_xor(l[mt], 32);
    if (g == 0) {
      ref_s[w][16 * mt + n] = m[mt];
      sum_s[w][16 * mt + n] = l[mt];
    }
  }
  __syncthreads();
  float* mine = (float*)ring;
#pragma unroll
  for (int mt = 0; mt < MT; ++mt) {
    float top = ref_s[0][16 * mt + n];
#pragma unroll
    for (int i = 1; i < kWaves; ++i) top = fmaxf(top, ref_s[i][16 * mt + n]);
    const float c = m[mt] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m[mt] - top);
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) *(f32x4*)(mine + (16 * mt + n) * D + 16 * dt + 4 * g) = o[mt][dt] * c;
  }
  __syncthreads();
  constexpr int Q4 = D / 4;
  for (int i = threadIdx.x; i < MT * 16 * Q4; i += 64 * kWaves) {
    const int col = i / Q4, x = i - col * Q4;
    if (qs.first + col >= qs.count) break;
    int seq, t, head;
    qs.split(d, qs.first + col, seq, t, head);
    f32x4 sum = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int j = 0; j < kWaves; ++j) sum += *(const f32x4*)(lds + j * (2 * STAGE) + (size_t)(col * D + 4 * x) * 4);
    const size_t slot = ((size_t)((size_t)seq * d.n_query + t) * d.n_head + head) * a.parts + part;
    *(f32x4*)(a.o + slot * D + 4 * x) = sum;
    if (x == 0) {
      float top = ref_s[0][col], total = 0.f;
#pragma unroll
      for (int j = 1; j < kWaves; ++j) top = fmaxf(top, ref_s[j][col]);
#pragma unroll
      for (int j = 0; j < kWaves; ++j)
        total += ref_s[j][col] == -INFINITY ? 0.f : sum_s[j][col] * __builtin_amdgcn_exp2f(ref_s[j][col] - top);
      a.ml[slot] = make_float2(top, total);
    }
  }
}

template <typename T, int D, int MP, int MO>
__global__ __launch_bounds__(64 * kWaves) void prefix_attn_kernel(PrefixAttnArgs a) {
  extern __shared__ __align__(512) unsigned char lds[];  // (a block's rows lie at multiples of their size)
  const ssd_prefix_attn_desc& d = a.d;
  const int G = d.n_head / d.n_kv_head;
  int i = blockIdx.x, k0, k1, len = 0, part;
  int64_t at, row;
  Queries qs;
  const bool shared = i < a.p_blocks;
  if (shared) {
    // (head, chunk) pairs go round the XCDs; the query tiles of one, which read
    // the same rows, are on one XCD, one after the other
    const int x = i % 8, tile = i / 8 % a.p_tiles, pair = i / (8 * a.p_tiles) * 8 + x;
    if (pair >= d.n_kv_head * a.p_chunks) return;
    const int h = pair / a.p_chunks;
    part = pair - h * a.p_chunks;
    k0 = part * a.p_chunk;
    k1 = min(k0 + a.p_chunk, d.prefix_len);
    at = (int64_t)h * d.prefix_head;
    row = d.prefix_row;
    qs = {h, -1, tile * MP * 16, d.n_seq * d.n_query * G};
  } else {
    i -= a.p_blocks;
    const int c = i % a.o_chunks, tile = i / a.o_chunks % a.o_tiles, bh = i / (a.o_chunks * a.o_tiles);
    const int b = bh / d.n_kv_head, h = bh - b * d.n_kv_head;
    len = min(a.own_len[b], d.own_rows);
    k0 = c * a.o_chunk;
    if (k0 >= len) return;
    k1 = min(k0 + a.o_chunk, len);
    part = a.p_chunks + c;
    at = (int64_t)b * d.own_seq + (int64_t)h * d.own_head;
    row = d.own_row;
    qs = {h, b, tile * MO * 16, d.n_query * G};
  }
  const Range r = {(const char*)(shared ? a.kp : a.ko) + at * (int)sizeof(T),
                   (const char*)(shared ? a.vp : a.vo) + at * (int)sizeof(T), row * (int)sizeof(T)};
  if (MP == MO || shared) attend<T, D, MP>(a, qs, r, k0, k1, len, part, lds);
  else attend<T, D, MO>(a, qs, r, k0, k1, len, part, lds);
}

// A wave per query adds its parts: lane l has dims 4 (l % (D / 4)) .. + 3 and every
// (256 / D)-th part.
template <typename T, int D>
__global__ __launch_bounds__(256) void merge_kernel(PrefixAttnArgs a, int queries) {
  constexpr int LD = D / 4, PAR = 64 / LD;
  const ssd_prefix_attn_desc& d = a.d;
  const int lane = threadIdx.x & 63, q = blockIdx.x * 4 + (threadIdx.x >> 6);
  if (q >= queries) return;
  const int h = q % d.n_head, bt = q / d.n_head, t = bt % d.n_query, b = bt / d.n_query, len = min(a.own_len[b], d.own_rows);
  const int np = len < 0 ? 0 : a.p_chunks, no = len > 0 ? (len + a.o_chunk - 1) / a.o_chunk : 0, n = np + no;
  const float2* ml = a.ml + (size_t)q * a.parts;
  const float* po = a.o + (size_t)q * a.parts * D;
  float top = -INFINITY;
  for (int i = lane; i < n; i += 64) top = fmaxf(top, ml[i < np ? i : i - np + a.p_chunks].x);
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor(top, o));
  f32x4 acc = {0.f, 0.f, 0.f, 0.f};
  float total = 0.f;
  const int x = lane % LD;
#pragma unroll 4
  for (int i = lane / LD; i < n; i += PAR) {
    const int s = i < np ? i : i - np + a.p_chunks;
    const float2 p = ml[s];
    const f32x4 v = *(const f32x4*)(po + (size_t)s * D + 4 * x);
    const float c = p.x == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(p.x - top);
    acc += c * v;
    total += c * p.y;
  }
#pragma unroll
  for (int o = 32; o >= LD; o >>= 1) {
    total += __shfl_xor(total, o);
#pragma unroll
    for (int i = 0; i < 4; ++i) acc[i] += __shfl_xor(acc[i], o);
  }
  if (lane < LD) {
    T* out = (T*)a.out + (int64_t)b * d.out_seq + (int64_t)t * d.out_row + (int64_t)h * d.out_head;
    const float inv = total == 0.f ? 0.f : 1.f / total;
#pragma unroll
    for (int i = 0; i < 4; ++i) op_st(out, 4 * x + i, acc[i] * inv);
    if (a.lse && lane == 0) a.lse[q] = total == 0.f ? -INFINITY : top * 0.6931471805599453f + logf(total);
  }
}

constexpr int kMaxRows = 1 << 30;

ssd_status check(const ssd_prefix_attn_desc* a) {
  OP_REQUIRE(a, SSD_E_INVALID_ARG, "null argument");
  OP_REQUIRE(op_dtype(a->dtype), SSD_E_INVALID_ARG, "dtype must be SSD_F32 or SSD_BF16");
  OP_REQUIRE(a->head_dim == 32 || a->head_dim == 64 || a->head_dim == 128, SSD_E_UNSUPPORTED,
             "head_dim must be 32, 64 or 128");
  OP_REQUIRE(a->n_seq >= 1 && a->n_seq <= 4096, SSD_E_INVALID_ARG, "n_seq outside [1, 4096]");
  OP_REQUIRE(a->n_query >= 1 && a->n_query <= 64, SSD_E_INVALID_ARG, "n_query outside [1, 64]");
  OP_REQUIRE(a->n_kv_head >= 1 && a->n_head >= a->n_kv_head && a->n_head <= 1024 && a->n_head % a->n_kv_head == 0,
             SSD_E_INVALID_ARG, "n_head must be a multiple of n_kv_head, at most 1024");
  OP_REQUIRE(a->prefix_len >= 0 && a->prefix_len < kMaxRows && a->own_rows >= 0 && a->own_rows < kMaxRows,
             SSD_E_INVALID_ARG, "prefix_len or own_rows outside [0, 2^30)");
  OP_REQUIRE(isfinite(a->scale), SSD_E_INVALID_ARG, "scale must be finite");
  return SSD_OK;
}

ssd_status check_strides(const ssd_prefix_attn_desc* a) {
  const int64_t s[] = {a->q_seq, a->q_row, a->q_head, a->prefix_head, a->prefix_row, a->own_seq, a->own_head,
                       a->own_row, a->out_seq, a->out_row, a->out_head};
  const int unit = 16 / op_size(a->dtype);
  for (int64_t x : s) {
    OP_REQUIRE(x >= 0, SSD_E_INVALID_ARG, "a stride is negative");
    OP_REQUIRE(x % unit == 0, SSD_E_UNSUPPORTED, "a stride is not a multiple of 16 bytes");
  }
  OP_REQUIRE((a->n_seq == 1 || a->out_seq >= a->head_dim) && (a->n_query == 1 || a->out_row >= a->head_dim) &&
                 (a->n_head == 1 || a->out_head >= a->head_dim),
             SSD_E_INVALID_ARG, "out's rows overlap");
  return SSD_OK;
}

// How a call is cut up: query tiles of 16, 32 or 64 columns, as few as hold the
// queries; chunks of the shared rows so that there are about kTarget workgroups
// (several a CU: the last to finish leave little idle), none below a block for each wave.
constexpr int kTarget = 1024;

struct Plan {
  int mp, mo;  // matrix tiles per query tile
  int p_tiles, p_chunks, p_chunk, p_blocks, o_tiles, o_chunks, o_chunk;
  int64_t blocks;
  size_t o_bytes, bytes;
};

int tile_of(int64_t columns, int most) {
  int m = 1;
  while (m < most && 16 * m < columns) m *= 2;
  return m;
}
int64_t div_up(int64_t a, int64_t b) { return (a + b - 1) / b; }

Plan plan(const ssd_prefix_attn_desc* a) {
  Plan p{};
  const int G = a->n_head / a->n_kv_head, step = kWaves * (a->dtype == SSD_F32 ? 16 : 32);
  const int64_t cols = (int64_t)a->n_seq * a->n_query * G, own_cols = (int64_t)a->n_query * G;
  p.mp = tile_of(cols, a->dtype == SSD_F32 ? 2 : 4);
  p.mo = tile_of(own_cols, 2);
  p.p_tiles = (int)div_up(cols, 16 * p.mp);
  p.o_tiles = (int)div_up(own_cols, 16 * p.mo);
  auto cut = [&](int64_t rows, int64_t sets, int& chunks, int& chunk) {
    const int64_t want = std::min(std::max<int64_t>(kTarget / sets, 1), std::max<int64_t>(div_up(rows, step), 1));
    chunk = (int)(div_up(std::max<int64_t>(div_up(rows, want), 1), step) * step);
    chunks = (int)div_up(rows, chunk);
  };
  cut(a->prefix_len, (int64_t)a->n_kv_head * p.p_tiles, p.p_chunks, p.p_chunk);
  cut(a->own_rows, (int64_t)a->n_seq * a->n_kv_head * p.o_tiles, p.o_chunks, p.o_chunk);
  p.p_blocks = (int)(div_up((int64_t)a->n_kv_head * p.p_chunks, 8) * 8 * p.p_tiles);
  p.blocks = p.p_blocks + (int64_t)a->n_seq * a->n_kv_head * p.o_tiles * p.o_chunks;
  const int64_t slots = (int64_t)a->n_seq * a->n_query * a->n_head * std::max(1, p.p_chunks + p.o_chunks);
  p.o_bytes = (size_t)slots * a->head_dim * 4;
  p.bytes = p.o_bytes + (size_t)slots * sizeof(float2);
  return p;
}

template <typename T, int D, int MP, int MO>
hipError_t launch(const PrefixAttnArgs& a, int64_t blocks, hipStream_t s) {
  constexpr int lds = kWaves * 2 * 2 * Block<T, D>::BYTES;
  // once per device: raises the kernel's limit of dynamic LDS
  static std::atomic<uint64_t> ready{0};
  int dev = 0;
  hipError_t e = hipGetDevice(&dev);
  if (e != hipSuccess) return e;
  const uint64_t bit = dev < 64 ? 1ull << dev : 0;
  if (!(ready.load(std::memory_order_acquire) & bit)) {
    e = hipFuncSetAttribute((const void*)prefix_attn_kernel<T, D, MP, MO>,
                            hipFuncAttributeMaxDynamicSharedMemorySize, lds);
    if (e != hipSuccess) return e;
    ready.fetch_or(bit, std::memory_order_release);
  }
  if (blocks > 0) prefix_attn_kernel<T, D, MP, MO><<<(unsigned)blocks, 64 * kWaves, lds, s>>>(a);
  e = hipGetLastError();
  if (e != hipSuccess) return e;
  const int queries = a.d.n_seq * a.d.n_query * a.d.n_head;
  merge_kernel<T, D><<<(queries + 3) / 4, 256, 0, s>>>(a, queries);
  return hipGetLastError();
}
template <typename T, int D>
hipError_t launch(const PrefixAttnArgs& a, const Plan& p, hipStream_t s) {
  if constexpr (sizeof(T) == 2) {
    if (p.mp == 4) return p.mo == 2 ? launch<T, D, 4, 2>(a, p.blocks, s) : launch<T, D, 4, 1>(a, p.blocks, s);
  }
  if (p.mp >= 2) return p.mo == 2 ? launch<T, D, 2, 2>(a, p.blocks, s) : launch<T, D, 2, 1>(a, p.blocks, s);
  return launch<T, D, 1, 1>(a, p.blocks, s);  // (a sequence has no more queries than all)
}
template <typename T>
hipError_t launch(const PrefixAttnArgs& a, const Plan& p, hipStream_t s) {
  switch (a.d.head_dim) {
    case 32: return launch<T, 32>(a, p, s);
    case 64: return launch<T, 64>(a, p, s);
    default: return launch<T, 128>(a, p, s);
  }
}

}  // namespace
}  // namespace ssd

using namespace ssd;

extern "C" ssd_status ssd_prefix_attn_workspace(const ssd_prefix_attn_desc* a, size_t* bytes) {
  OP_REQUIRE(bytes, SSD_E_INVALID_ARG, "null argument");
  ssd_status st = check(a);
  if (st != SSD_OK) return st;
  const Plan p = plan(a);
  OP_REQUIRE(p.blocks <= 0x7fffffff, SSD_E_CAPACITY, "too many workgroups");
  *bytes = p.bytes;
  return SSD_OK;
}

extern "C" ssd_status ssd_prefix_attn(const ssd_prefix_attn_desc* a, const void* q, const void* k_prefix,
                                      const void* v_prefix, const void* k_own, const void* v_own,
                                      const int32_t* own_len, void* out, float* lse, void* workspace,
                                      size_t workspace_bytes, void* stream) {
  size_t need = 0;
  ssd_status st = ssd_prefix_attn_workspace(a, &need);
  if (st == SSD_OK) st = check_strides(a);
  if (st != SSD_OK) return st;
  OP_REQUIRE(q && own_len && out && workspace, SSD_E_INVALID_ARG, "null argument");
  OP_REQUIRE(a->prefix_len == 0 || (k_prefix && v_prefix), SSD_E_INVALID_ARG, "null prefix");
  OP_REQUIRE(a->own_rows == 0 || (k_own && v_own), SSD_E_INVALID_ARG, "null own rows");
  const void* pointers[] = {q, k_prefix, v_prefix, k_own, v_own, out};
  for (const void* x : pointers)
    OP_REQUIRE((uintptr_t)x % 16 == 0, SSD_E_UNSUPPORTED, "a pointer is not 16-byte aligned");
  OP_REQUIRE(workspace_bytes >= need && (uintptr_t)workspace % 16 == 0, SSD_E_CAPACITY,
             "workspace below ssd_prefix_attn_workspace's bytes or not 16-byte aligned");
  const Plan p = plan(a);
  PrefixAttnArgs x{};
  x.d = *a;
  x.q = q;
  x.kp = k_prefix;
  x.vp = v_prefix;
  x.ko = k_own;
  x.vo = v_own;
  x.own_len = own_len;
  x.out = out;
  x.lse = lse;
  x.o = (float*)workspace;
  x.ml = (float2*)((char*)workspace + p.o_bytes);
  x.p_tiles = p.p_tiles;
  x.p_chunks = p.p_chunks;
  x.p_chunk = p.p_chunk;
  x.p_blocks = p.p_blocks;
  x.o_tiles = p.o_tiles;
  x.o_chunks = p.o_chunks;
  x.o_chunk = p.o_chunk;
  x.parts = p.p_chunks + p.o_chunks;
  x.scale2 = a->scale * 1.4426950408889634f;
  const hipError_t e = a->dtype == SSD_F32 ? launch<float>(x, p, (hipStream_t)stream) : launch<bf16_t>(x, p, (hipStream_t)stream);
  if (e != hipSuccess) return op_fail(SSD_E_DEVICE, hipGetErrorString(e));
  return SSD_OK;
}
