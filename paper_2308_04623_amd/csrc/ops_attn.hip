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
// part (m, l, o) per query; merge_kernel adds a query's parts.  (Where the prefix is
// short for the batch, short_attn_kernel does all for a sequence.)  Its waves take the
// chunk's blocks of rows in turn and never wait for each other until the end: a
// wave copies its blocks' keys and values into LDS of its own, one block ahead.
#include <algorithm>
#include <atomic>
#include <cstdlib>

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
  int p_cols, p_tiles, p_chunks, p_chunk, p_blocks;  // of the prefix: queries per tile, tiles, chunks, rows per chunk, workgroups
  int o_tiles, o_chunks, o_chunk;            // of a sequence's own rows
  int parts;                                 // p_chunks + o_chunks
  float scale2;                              // |scale| log2 e
};

constexpr int kWaves = 4;
constexpr float kSlack = 8.f;  // how far a score may lie above the reference before the sums are rescaled
// From references of this size on, scaled scores are rounded before the reference is taken from
// them: by one rounding (fmaf) the largest score's weight is 2^r with r the rounding of the
// reference, below 1/2 here, 2^128 for references around 2^32.
constexpr float kFar = 16777216.f;

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

// The q-th KB of a block of keys (half 0) or values (1) is copied by a wave, 16 bytes a
// lane: bytes lane_at .. of the block's row lane_row.
template <typename T, int D>
__device__ __forceinline__ int lane_row(int q) {
  return (q * 64 + (int)(threadIdx.x & 63)) / Block<T, D>::CH;
}
template <typename T, int D>
__device__ __forceinline__ int lane_at(int half, int q) {
  typedef Block<T, D> B;
  const int p = q * 64 + (int)(threadIdx.x & 63), r = p / B::CH;
  return 16 * (p % B::CH ^ (half ? B::swz_v(r) : B::swz_k(r)));
}
template <int CPOL>
__device__ __forceinline__ void copy_1k(const char* src, unsigned char* dst) {
  __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)src,
                                   (__attribute__((address_space(3))) void*)dst, 16, 0, CPOL);
}
// The whole block, rows kb .. of a matrix (those from `end` on: row end - 1 again), into
// LDS at dst; LOADS copies in flight.
template <typename T, int D, int HALF>
__device__ __forceinline__ void issue(const Range& s, int kb, int end, unsigned char* dst) {
#pragma unroll
  for (int i = 0; i < Block<T, D>::LOADS; ++i)
    copy_1k<2>((HALF ? s.v : s.k) + (int64_t)min(kb + lane_row<T, D>(i), end - 1) * s.row + lane_at<T, D>(HALF, i),
               dst + i * 1024);
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

// The same, and 2^x of eight numbers while the reads are under way.
template <int OFF>
__device__ __forceinline__ void read_transposed(unsigned a0, unsigned a1, unsigned a2, unsigned a3, u32x2 (&f0)[2],
                                                u32x2 (&f1)[2], u32x2 (&f2)[2], u32x2 (&f3)[2], f32x4 (&x)[2]) {
  float e0 = x[0][0], e1 = x[0][1], e2 = x[0][2], e3 = x[0][3], e4 = x[1][0], e5 = x[1][1], e6 = x[1][2], e7 = x[1][3];
  asm volatile(
      "ds_read_b64_tr_b16 %0, %16\n"
      "ds_read_b64_tr_b16 %1, %16 offset:%20\n"
      "ds_read_b64_tr_b16 %2, %17\n"
      "ds_read_b64_tr_b16 %3, %17 offset:%20\n"
      "ds_read_b64_tr_b16 %4, %18\n"
      "ds_read_b64_tr_b16 %5, %18 offset:%20\n"
      "ds_read_b64_tr_b16 %6, %19\n"
      "ds_read_b64_tr_b16 %7, %19 offset:%20\n"
      "v_exp_f32 %8, %8\n"
      "v_exp_f32 %9, %9\n"
      "v_exp_f32 %10, %10\n"
      "v_exp_f32 %11, %11\n"
      "v_exp_f32 %12, %12\n"
      "v_exp_f32 %13, %13\n"
      "v_exp_f32 %14, %14\n"
      "v_exp_f32 %15, %15\n"
      "s_waitcnt lgkmcnt(0)\n"
      "s_nop 0"
      : "=&v"(f0[0]), "=&v"(f0[1]), "=&v"(f1[0]), "=&v"(f1[1]), "=&v"(f2[0]), "=&v"(f2[1]), "=&v"(f3[0]),
        "=&v"(f3[1]), "+v"(e0), "+v"(e1), "+v"(e2), "+v"(e3), "+v"(e4), "+v"(e5), "+v"(e6), "+v"(e7)
      : "v"(a0), "v"(a1), "v"(a2), "v"(a3), "n"(OFF)
      : "memory");
  x[0] = (f32x4){e0, e1, e2, e3};
  x[1] = (f32x4){e4, e5, e6, e7};
}

// The N results are complete.  A vector instruction may read a matrix product's result 8
// (bfloat16) or 10 (float32) instructions' time after it and not sooner; nothing in the
// hardware holds it back, and the compiler, which puts the waits, does not count reliably
// across the end of a block (without this, scores of float32 were read one instruction after
// the last product, where a branch lay between).  So results that are read behind a
// branch are waited for here first.
template <int N>
__device__ __forceinline__ void complete(f32x4* x) {
  static_assert(N == 1 || N == 2 || N == 4 || N == 8, "one statement for all: its wait comes after every product");
  if constexpr (N == 1)
    asm volatile("s_nop 9" : "+v"(x[0]));
  else if constexpr (N == 2)
    asm volatile("s_nop 9" : "+v"(x[0]), "+v"(x[1]));
  else if constexpr (N == 4)
    asm volatile("s_nop 9" : "+v"(x[0]), "+v"(x[1]), "+v"(x[2]), "+v"(x[3]));
  else
    asm volatile("s_nop 9"
                 : "+v"(x[0]), "+v"(x[1]), "+v"(x[2]), "+v"(x[3]), "+v"(x[4]), "+v"(x[5]), "+v"(x[6]), "+v"(x[7]));
}

// 2^x of the tiles from FROM on
template <int FROM, int MT, int KT>
__device__ __forceinline__ void exp2_all(f32x4 (&s)[MT][KT]) {
#pragma unroll
  for (int mt = FROM; mt < MT; ++mt)
#pragma unroll
    for (int kt = 0; kt < KT; ++kt)
#pragma unroll
      for (int r = 0; r < 4; ++r) s[mt][kt][r] = __builtin_amdgcn_exp2f(s[mt][kt][r]);
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
    u32x4 f[KT][KK];
#pragma unroll
    for (int kt = 0; kt < KT; ++kt)
#pragma unroll
      for (int kk = 0; kk < KK; ++kk) {
        const int r = 16 * kt + n;
        f[kt][kk] = *(const u32x4*)(k + r * B::ROW + 16 * ((4 * kk + g) ^ B::swz_k(r)));
      }
    __builtin_amdgcn_sched_barrier(0);  // (all reads under way before the first product; 128 dims 339 us, 350 without)
#pragma unroll
    for (int kt = 0; kt < KT; ++kt)
#pragma unroll
      for (int kk = 0; kk < KK; ++kk)
#pragma unroll
        for (int mt = 0; mt < MT; ++mt)
          s[mt][kt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, f[kt][kk]),
                                                              __builtin_bit_cast(bf16x8, q[mt][kk]),
                                                              kk ? s[mt][kt] : (f32x4){0.f, 0.f, 0.f, 0.f}, 0, 0, 0);
  }
  struct P {
    u32x4 w[MT];
  };
  // The weights as the second product's operand: its lane needs the keys it holds already.
  // They are rounded to bfloat16, 2^-9 of themselves at most, as a product with a float32 operand
  // takes sixteen times as long; their sum takes them unrounded, for which they need not be
  // unpacked again.  (Error against 64 bits 0.0023 relative; of the output's rounding alone 0.0016.)
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
  // EXP: the weights are made of their exponents on the way
  template <bool EXP>
  static __device__ __forceinline__ void values(const unsigned char* v, V& x, f32x4 (&s)[MT][KT]) {
    // a 16-lane group reads four rows of 16 dims and gets them transposed
    const int lane = threadIdx.x & 63, r = 4 * (lane >> 4) + ((lane & 15) >> 2);
    const unsigned at = (unsigned)(size_t)(lds_byte*)v + r * B::ROW + 16 * (((lane & 3) >> 1) ^ B::swz_v(r)) +
                        8 * (lane & 1);
    if constexpr (DT == 2) {
      read_transposed<16 * B::ROW>(at, at ^ 32, x.f[0], x.f[1]);
      if (EXP) exp2_all<0>(s);
    } else {
#pragma unroll
      for (int dt = 0; dt < DT; dt += 4)
        if (EXP && dt / 4 < MT)
          read_transposed<16 * B::ROW>(at ^ (32 * dt), at ^ (32 * (dt + 1)), at ^ (32 * (dt + 2)), at ^ (32 * (dt + 3)),
                                       x.f[dt], x.f[dt + 1], x.f[dt + 2], x.f[dt + 3], s[dt / 4]);
        else
          read_transposed<16 * B::ROW>(at ^ (32 * dt), at ^ (32 * (dt + 1)), at ^ (32 * (dt + 2)), at ^ (32 * (dt + 3)),
                                       x.f[dt], x.f[dt + 1], x.f[dt + 2], x.f[dt + 3]);
      if (EXP) exp2_all<DT / 4>(s);
    }
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
  template <bool EXP>
  static __device__ __forceinline__ void values(const unsigned char* v, V& x, f32x4 (&s)[MT][KT]) {
    const int lane = threadIdx.x & 63, n = lane & 15, g = lane >> 4;
    if (EXP) exp2_all<0>(s);
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

// The queries of a tile from `first` on: of the prefix, all (sequence,
// position, group member) of kv head h; of own rows, sequence b's.
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

// MT x 16 queries of a wave and what it has of their attention.
template <typename T, int D, int MT>
struct Wave {
  typedef Block<T, D> B;
  typedef Math<T, D, MT> M;
  static constexpr int KB = B::KB, KT = M::KT, KK = M::KK, DT = M::DT;
  u32x4 q[MT][KK];
  f32x4 o[MT][DT];
  float m[MT], l[MT];
  float limit[MT];  // a scaled score above it takes the way of a new reference
  int pos[MT];  // of this lane's queries

  __device__ __forceinline__ void load(const PrefixAttnArgs& a, const Queries& qs) {
    const ssd_prefix_attn_desc& d = a.d;
    const int lane = threadIdx.x & 63, n = lane & 15, g = lane >> 4;
    // (a negative scale goes into the queries' signs: the largest score is then that of the largest product)
    const unsigned sign = d.scale < 0.f ? (sizeof(T) == 2 ? 0x80008000u : 0x80000000u) : 0u;
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
      int seq, t, head;
      qs.split(d, min(qs.first + 16 * mt + n, qs.count - 1), seq, t, head);
      pos[mt] = t;
      const T* row = (const T*)a.q + (int64_t)seq * d.q_seq + (int64_t)t * d.q_row + (int64_t)head * d.q_head;
#pragma unroll
      for (int kk = 0; kk < KK; ++kk) q[mt][kk] = *((const u32x4*)row + 4 * kk + g) ^ sign;
      m[mt] = limit[mt] = -INFINITY;
      l[mt] = 0.f;
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) o[mt][dt] = (f32x4){0.f, 0.f, 0.f, 0.f};
    }
  }

  // The first row of a block that the lane has scores of.  (Opaque: its comparisons
  // are not to be prepared in blocks that are not masked.)
  static __device__ __forceinline__ int lane_key(int kb) {
    int row = kb + 4 * (int)((threadIdx.x & 63) >> 4);
    asm volatile("" : "+v"(row));
    return row;
  }

  // The exponents of the weights of rows kb .. of a block from their raw scores.
  // masked: lane's query mt sees rows below lim[mt]; else all see all.
  __device__ __forceinline__ void exponents(f32x4 (&s)[MT][KT], int kb, bool masked, const int (&lim)[MT],
                                            float scale2) {
    if (masked) {
      const int row = lane_key(kb);
#pragma unroll
      for (int mt = 0; mt < MT; ++mt)
#pragma unroll
        for (int kt = 0; kt < KT; ++kt)
#pragma unroll
          for (int r = 0; r < 4; ++r)
            if (row + 16 * kt + r >= lim[mt]) s[mt][kt][r] = -INFINITY;
    }
    float top[MT];
    bool above = false;
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
      top[mt] = s[mt][0][0];
#pragma unroll
      for (int i = 1; i < 4 * KT; ++i) top[mt] = fmaxf(top[mt], s[mt][i / 4][i % 4]);
      above |= top[mt] * scale2 > limit[mt];
    }
    if (__builtin_amdgcn_ballot_w64(above)) {  // a new reference: the largest score so far
      bool beyond = false;
#pragma unroll
      for (int mt = 0; mt < MT; ++mt) {
        float x = top[mt] == -INFINITY ? m[mt] : fmaxf(m[mt], top[mt] * scale2);
        x = fmaxf(x, __shfl_xor(x, 16));
        x = fmaxf(x, __shfl_xor(x, 32));
        const float c = x == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m[mt] - x);
        m[mt] = x;
        limit[mt] = x + kSlack;
        complete<DT>(o[mt]);
        beyond |= x != -INFINITY && fabsf(x) >= kFar;
        l[mt] *= c;
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) o[mt][dt] *= c;
      }
      if (__builtin_amdgcn_ballot_w64(beyond)) {
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) limit[mt] = -INFINITY;  // (the next block's, too: no test of its own in the loop)
#pragma unroll
        for (int mt = 0; mt < MT; ++mt)
#pragma unroll
          for (int kt = 0; kt < KT; ++kt)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
              s[mt][kt][r] *= scale2;
              asm volatile("" : "+v"(s[mt][kt][r]));  // (rounded here: not to be made one operation with what follows)
            }
        scale2 = 1.f;
      }
    }
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
      const float ref = m[mt] == -INFINITY ? 0.f : m[mt];
#pragma unroll
      for (int kt = 0; kt < KT; ++kt)
#pragma unroll
        for (int r = 0; r < 4; ++r) s[mt][kt][r] = fmaf(s[mt][kt][r], scale2, -ref);
    }
  }

  // takes the weights into the sums
  __device__ __forceinline__ void sums(f32x4 (&s)[MT][KT], int kb, bool masked, const int (&lim)[MT],
                                       typename M::P& p) {
    if (masked) {  // (whatever came of -infinity times a scale of 0)
      const int row = lane_key(kb);
#pragma unroll
      for (int mt = 0; mt < MT; ++mt)
#pragma unroll
        for (int kt = 0; kt < KT; ++kt)
#pragma unroll
          for (int r = 0; r < 4; ++r)
            if (row + 16 * kt + r >= lim[mt]) s[mt][kt][r] = 0.f;
    }
#pragma unroll
    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
      for (int kt = 0; kt < KT; ++kt)
#pragma unroll
        for (int r = 0; r < 4; ++r) l[mt] += s[mt][kt][r];
    M::weights(s, p);
  }

  __device__ __forceinline__ void scores(const unsigned char* k, f32x4 (&s)[MT][KT]) const {
    M::scores(k, q, s);
    complete<MT * KT>(&s[0][0]);
  }

  // adds the values of a block, x read from v.  A weight of 0 does not silence
  // an infinity or NaN: in blocks that some query does not see to the end those
  // values are added to the queries that see their rows.
  __device__ __forceinline__ void add(typename M::V& x, const unsigned char* v, const typename M::P& p, int kb,
                                      bool masked, const int (&lim)[MT]) {
    bool bad = false;
    if (masked) bad = M::clear(x);
    M::add(x, p, o);
    if (masked && __builtin_amdgcn_ballot_w64(bad)) {
      const int g = (threadIdx.x & 63) >> 4;
#pragma unroll
      for (int mt = 0; mt < MT; ++mt) complete<DT>(o[mt]);
#pragma unroll 1
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
  }

  // All that a block's scores and values add.  Values under way are waited for
  // by landed(), behind the exponentials; those THERE are read while they are taken.
  template <bool THERE, typename Landed>
  __device__ __forceinline__ void take(f32x4 (&x)[MT][KT], const unsigned char* v, int kb, bool masked,
                                       const int (&lim)[MT], float scale2, Landed landed) {
    exponents(x, kb, masked, lim, scale2);
    if (!THERE) {
      exp2_all<0>(x);
      landed();
    }
    typename M::V f;
    M::template values<THERE>(v, f, x);
    typename M::P p;
    sums(x, kb, masked, lim, p);
    add(f, v, p, kb, masked, lim);
  }

  // The sums of l over the lanes of a query.  A reference of -infinity says that no row
  // was seen; NaN scores do not raise it, so a sum of theirs takes 0 and is joined as any other.
  __device__ __forceinline__ void close() {
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
      complete<DT>(o[mt]);
      l[mt] += __shfl_xor(l[mt], 16);
      l[mt] += __shfl_xor(l[mt], 32);
      if (m[mt] == -INFINITY && l[mt] != l[mt]) m[mt] = 0.f;
    }
  }
};

// a query's place among all (sequence, position, head)
__device__ __forceinline__ size_t query_of(const ssd_prefix_attn_desc& d, int seq, int t, int head) {
  return ((size_t)seq * d.n_query + t) * d.n_head + head;
}

// Four dims of a query's attention from its sums, and its log of the sum.
template <typename T>
__device__ __forceinline__ void put_query(const PrefixAttnArgs& a, int seq, int t, int head, int x, f32x4 sum, float top,
                                          float total) {
  const ssd_prefix_attn_desc& d = a.d;
  T* out = (T*)a.out + (int64_t)seq * d.out_seq + (int64_t)t * d.out_row + (int64_t)head * d.out_head;
  const float inv = total == 0.f ? 0.f : 1.f / total;
#pragma unroll
  for (int i = 0; i < 4; ++i) op_st(out, 4 * x + i, sum[i] * inv);
  if (a.lse && x == 0)
    a.lse[query_of(d, seq, t, head)] = total == 0.f ? -INFINITY : top * 0.6931471805599453f + logf(total);
}

__device__ __forceinline__ void reads_over() {
  // the wave's LDS reads so far are complete: what they read may be overwritten
  __builtin_amdgcn_sched_barrier(0);
  __builtin_amdgcn_s_waitcnt(0xc07f);  // lgkmcnt(0)
  asm volatile("" ::: "memory");
  __builtin_amdgcn_sched_barrier(0);
}

// ---- few queries: the waves of a workgroup take the blocks of rows in turn

// A wave's share of rows [k0, k1) of a range: blocks w, w + kWaves, ...  One
// block of keys and one of values are in LDS; the next keys are fetched when this
// block's scores are there, the next values when its values are in registers.
// own: query t sees rows below len - n_query + 1 + t.
template <typename T, int D, int MT>
__device__ __forceinline__ void walk(Wave<T, D, MT>& s, const Range& range, int k0, int k1, bool own, int len,
                                     int n_query, float scale2, unsigned char* lds) {
  typedef Wave<T, D, MT> W;
  typedef Block<T, D> B;
  constexpr int KB = W::KB, STEP = kWaves * KB;
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  unsigned char *k = lds + w * (2 * B::BYTES), *v = k + B::BYTES;
  int lim[MT];
#pragma unroll
  for (int mt = 0; mt < MT; ++mt) lim[mt] = own ? min(k1, len - n_query + 1 + s.pos[mt]) : k1;
  const int all = own ? min(k1, len - n_query + 1) : k1;
  int kb = k0 + w * KB;
  if (kb < k1) {
    issue<T, D, 0>(range, kb, k1, k);
    issue<T, D, 1>(range, kb, k1, v);
  }
  for (; kb < k1; kb += STEP) {
    const bool more = kb + STEP < k1;
    copies_landed<B::LOADS>();  // (the values may be under way)
    f32x4 x[MT][W::KT];
    s.scores(k, x);
    if (more) {
      reads_over();
      issue<T, D, 0>(range, kb + STEP, k1, k);
    }
    auto landed = [&] {
      if (more) copies_landed<B::LOADS>();  // (the next keys may be)
      else copies_landed<0>();
    };
    s.template take<false>(x, v, kb, kb + KB > all, lim, scale2, landed);
    if (more) {
      reads_over();
      issue<T, D, 1>(range, kb + STEP, k1, v);
    }
  }
}

// Joins the four waves' sums through LDS (a wave's blocks are over): calls
// put(column, dim / 4, four dims, reference, sum) once for each.
template <typename T, int D, int MT, typename Put>
__device__ __forceinline__ void join_waves(Wave<T, D, MT>& s, const Queries& qs, unsigned char* lds, Put put) {
  typedef Wave<T, D, MT> W;
  constexpr int AREA = 2 * Block<T, D>::BYTES, Q4 = D / 4;
  static_assert(MT * 16 * D * 4 <= AREA, "a wave's outputs fit its part of the LDS");
  __shared__ float ref_s[kWaves][MT * 16], sum_s[kWaves][MT * 16];
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, n = lane & 15, g = lane >> 4;
  s.close();
#pragma unroll
  for (int mt = 0; mt < MT; ++mt)
    if (g == 0) {
      ref_s[w][16 * mt + n] = s.m[mt];
      sum_s[w][16 * mt + n] = s.l[mt];
    }
  __syncthreads();
  float* mine = (float*)(lds + w * AREA);
#pragma unroll
  for (int mt = 0; mt < MT; ++mt) {
    float top = ref_s[0][16 * mt + n];
#pragma unroll
    for (int i = 1; i < kWaves; ++i) top = fmaxf(top, ref_s[i][16 * mt + n]);
    const float c = s.m[mt] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(s.m[mt] - top);
#pragma unroll
    for (int dt = 0; dt < W::DT; ++dt) *(f32x4*)(mine + (16 * mt + n) * D + 16 * dt + 4 * g) = s.o[mt][dt] * c;
  }
  __syncthreads();
  for (int i = threadIdx.x; i < MT * 16 * Q4; i += 64 * kWaves) {
    const int col = i / Q4, x = i - col * Q4;
    if (qs.first + col >= qs.count) break;
    f32x4 sum = {0.f, 0.f, 0.f, 0.f};
    float top = ref_s[0][col], total = 0.f;
#pragma unroll
    for (int j = 1; j < kWaves; ++j) top = fmaxf(top, ref_s[j][col]);
#pragma unroll
    for (int j = 0; j < kWaves; ++j) {
      sum += *(const f32x4*)(lds + j * AREA + (size_t)(col * D + 4 * x) * 4);
      total += ref_s[j][col] == -INFINITY ? 0.f : sum_s[j][col] * __builtin_amdgcn_exp2f(ref_s[j][col] - top);
    }
    put(col, x, sum, top, total);
  }
}

// One part: queries against rows [k0, k1) of a range.
template <typename T, int D, int MT>
__device__ __forceinline__ void part_by_rows(const PrefixAttnArgs& a, const Queries& qs, const Range& range, int k0,
                                             int k1, int len, int part, unsigned char* lds) {
  Wave<T, D, MT> s;
  s.load(a, qs);
  walk(s, range, k0, k1, qs.b >= 0, len, a.d.n_query, a.scale2, lds);
  join_waves(s, qs, lds, [&](int col, int x, f32x4 sum, float top, float total) {
    int seq, t, head;
    qs.split(a.d, qs.first + col, seq, t, head);
    const size_t slot = query_of(a.d, seq, t, head) * a.parts + part;
    *(f32x4*)(a.o + slot * D + 4 * x) = sum;
    if (x == 0) a.ml[slot] = make_float2(top, total);
  });
}

// ---- many queries: the waves take MT x 16 of them each and share the blocks

constexpr int kStages = 3;
// A stage of kStageBytes holds SUB blocks; each wave copies a quarter of it.
template <typename T, int D>
struct Stage {
  typedef Block<T, D> B;
  static constexpr int SUB = 128 / D, ROWS = SUB * B::KB, BYTES = SUB * 2 * B::BYTES, PER = BYTES / 1024 / kWaves;
  static_assert(BYTES == 16384 && PER == 4, "four copies a wave");
  typedef uint64_t u64x4 __attribute__((ext_vector_type(4)));
  u64x4 at;  // where the lane's copies of the next stage begin

  static __device__ __forceinline__ void place(int i, int& half, int& q, int& sub) {
    const int j = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) * PER + i;
    sub = j / (2 * B::LOADS);
    half = j / B::LOADS % 2;
    q = j % B::LOADS;
  }
  __device__ __forceinline__ void start(const Range& s, int kb) {
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      int half, q, sub;
      place(i, half, q, sub);
      at[i] = (uint64_t)((half ? s.v : s.k) + (int64_t)(kb + sub * B::KB + lane_row<T, D>(q)) * s.row +
                         lane_at<T, D>(half, q));
    }
  }
  // The stage of rows kb .., the next after the last one issued; rows from `end` on: row
  // end - 1 again.  (Whole stages from addresses kept: a row's product for each copy was a
  // third of the instructions around the matrix products, 303 us for 65536 rows, 350 with it.)
  __device__ __forceinline__ void issue(const Range& s, int kb, int end, unsigned char* dst) {
    dst += __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) * (PER * 1024);
    if (kb + ROWS <= end) {
      copy_1k<0>((const char*)at[0], dst);
      copy_1k<0>((const char*)at[1], dst + 1024);
      copy_1k<0>((const char*)at[2], dst + 2048);
      copy_1k<0>((const char*)at[3], dst + 3072);
    } else {
#pragma unroll
      for (int i = 0; i < PER; ++i) {
        int half, q, sub;
        place(i, half, q, sub);
        copy_1k<0>((half ? s.v : s.k) + (int64_t)min(kb + sub * B::KB + lane_row<T, D>(q), end - 1) * s.row +
                       lane_at<T, D>(half, q),
                   dst + i * 1024);
      }
    }
    at += (uint64_t)(ROWS * s.row);
  }
};

template <typename T, int D, int MT>
__device__ __forceinline__ void part_by_queries(const PrefixAttnArgs& a, Queries qs, const Range& range, int k0, int k1,
                                                int part, unsigned char* lds) {
  typedef Wave<T, D, MT> W;
  typedef Block<T, D> B;
  typedef Stage<T, D> S;
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), n = lane & 15, g = lane >> 4;
  qs.first += w * (MT * 16);
  const bool work = qs.first < qs.count;  // (a wave without queries still copies its share)
  S copies;
  copies.start(range, k0);
  copies.issue(range, k0, k1, lds);
  if (k0 + S::ROWS < k1) copies.issue(range, k0 + S::ROWS, k1, lds + S::BYTES);
  W s;
  s.load(a, qs);
  int lim[MT];
#pragma unroll
  for (int mt = 0; mt < MT; ++mt) lim[mt] = k1;
  int slot = 0;
  for (int kb = k0; kb < k1; kb += S::ROWS) {
    // this wave's copies of the stage are there; behind the barrier all waves'
    // are, and no wave still reads the stage before, whose place the next copies take
    if (kb + S::ROWS < k1) copies_landed<S::PER>();
    else copies_landed<0>();
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
    int ahead = slot + 2;
    if (ahead >= kStages) ahead -= kStages;
    if (kb + 2 * S::ROWS < k1) copies.issue(range, kb + 2 * S::ROWS, k1, lds + ahead * S::BYTES);
    if (work) {
#pragma unroll
      for (int sub = 0; sub < S::SUB; ++sub) {
        const int kr = kb + sub * B::KB;
        if (sub && kr >= k1) break;
        const unsigned char *k = lds + slot * S::BYTES + sub * (2 * B::BYTES), *v = k + B::BYTES;
        f32x4 x[MT][W::KT];
        s.scores(k, x);
        s.template take<true>(x, v, kr, kr + B::KB > k1, lim, a.scale2, [] {});
      }
      reads_over();
    }
    slot = slot + 1 == kStages ? 0 : slot + 1;
  }
  if (!work) return;
  s.close();
#pragma unroll
  for (int mt = 0; mt < MT; ++mt) {
    const int i = qs.first + 16 * mt + n;
    if (i >= qs.count) continue;
    int seq, t, head;
    qs.split(a.d, i, seq, t, head);
    const size_t at = query_of(a.d, seq, t, head) * a.parts + part;
#pragma unroll
    for (int dt = 0; dt < W::DT; ++dt) *(f32x4*)(a.o + at * D + 16 * dt + 4 * g) = s.o[mt][dt];
    if (g == 0) a.ml[at] = make_float2(s.m[mt], s.l[mt]);
  }
}

// BYQ: the prefix's workgroups share their blocks among the waves (part_by_queries).
// Few queries are bound by memory (16 sequences of 20 heads of 64 over 100,000 rows: 82
// us, 6.1 TB/s), many by the softmax's vector instructions and the matrix products, which
// follow each other with 32 queries a wave (48 x 5 queries, 32 heads on 8 of 128, over 8191
// rows: 56 us and 8 to join, 65 and 8 with up to 512 own rows a sequence; 65536 rows: 286 to 299
// us with the join, 860 to 900 TFLOP/s; 64 dims, the same vector work for half the products: 64 x 8
// queries of 20 heads over 5000 rows 36 us, 360 TFLOP/s).
template <typename T, int D, int MP, int MO, bool BYQ>
__global__ __launch_bounds__(64 * kWaves, D == 128 ? 2 : D == 64 ? 3 : 4) void prefix_attn_kernel(PrefixAttnArgs a) {
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
    qs = {h, -1, tile * a.p_cols, d.n_seq * d.n_query * G};
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
  if constexpr (BYQ)
    if (shared) return part_by_queries<T, D, MP>(a, qs, r, k0, k1, part, lds);
  if constexpr (BYQ || MP == MO) {
    part_by_rows<T, D, MO>(a, qs, r, k0, k1, len, part, lds);
  } else {
    if (shared) part_by_rows<T, D, MP>(a, qs, r, k0, k1, len, part, lds);
    else part_by_rows<T, D, MO>(a, qs, r, k0, k1, len, part, lds);
  }
}

// Prefixes that are short for the batch: a workgroup takes a tile of one
// sequence's queries over the prefix and its own rows, and writes their attention.
// One launch, no parts to write, read and join (6 sequences of 4 float32 heads of 32,
// 64 + 24 rows: 7.4 us by parts, 5.2 by this; bound by latency, two blocks a wave).
template <typename T, int D, int MO>
__global__ __launch_bounds__(64 * kWaves, D == 128 ? 2 : D == 64 ? 3 : 4) void short_attn_kernel(PrefixAttnArgs a) {
  extern __shared__ __align__(512) unsigned char lds[];
  const ssd_prefix_attn_desc& d = a.d;
  const int tile = blockIdx.x % a.o_tiles, bh = blockIdx.x / a.o_tiles, b = bh / d.n_kv_head, h = bh - b * d.n_kv_head;
  const int len = min(a.own_len[b], d.own_rows);
  const Queries qs = {h, b, tile * MO * 16, d.n_query * (d.n_head / d.n_kv_head)};
  const int64_t ap = (int64_t)h * d.prefix_head, ao = (int64_t)b * d.own_seq + (int64_t)h * d.own_head;
  constexpr int ES = sizeof(T);
  Wave<T, D, MO> s;
  s.load(a, qs);
  if (len >= 0)
    walk(s, (Range){(const char*)a.kp + ap * ES, (const char*)a.vp + ap * ES, d.prefix_row * ES}, 0, d.prefix_len, false,
         0, d.n_query, a.scale2, lds);
  reads_over();
  walk(s, (Range){(const char*)a.ko + ao * ES, (const char*)a.vo + ao * ES, d.own_row * ES}, 0, len, true, len, d.n_query,
       a.scale2, lds);
  join_waves(s, qs, lds, [&](int col, int x, f32x4 sum, float top, float total) {
    int seq, t, head;
    qs.split(d, qs.first + col, seq, t, head);
    put_query<T>(a, seq, t, head, x, sum, top, total);
  });
}

// A wave per query adds its parts: lane l has dims 4 (l % (D / 4)) .. + 3 and every
// (256 / D)-th part.  All parts' places are read, without waiting for the sequence's length to
// tell which of them were written (32 sequences over 2048 rows, both kernels: 15.3 us with the
// length first and a pass for the maximum, 14.5 so).  Bound: memory (7680 queries of 128,
// 9 parts each: 8.4 us, 4.4 TB/s) or, for few, the launch (4 us).
template <typename T, int D>
__global__ __launch_bounds__(256) void merge_kernel(PrefixAttnArgs a, int first, int queries) {
  constexpr int LD = D / 4, PAR = 64 / LD, U = 4;
  const ssd_prefix_attn_desc& d = a.d;
  const int lane = threadIdx.x & 63, q = first + blockIdx.x * 4 + (threadIdx.x >> 6);
  if (q >= queries) return;
  const int h = q % d.n_head, bt = q / d.n_head, t = bt % d.n_query, b = bt / d.n_query, len = min(a.own_len[b], d.own_rows);
  const float2* ml = a.ml + (size_t)q * a.parts;
  const float* po = a.o + (size_t)q * a.parts * D;
  const int x = lane % LD;
  f32x4 acc = {0.f, 0.f, 0.f, 0.f};
  float top = -INFINITY, total = 0.f;
  for (int i = lane / LD; i < a.parts; i += U * PAR) {
    float2 p[U];
    f32x4 v[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int s = i + u * PAR;
      p[u].x = -INFINITY;
      if (s < a.parts) {
        p[u] = ml[s];
        v[u] = *(const f32x4*)(po + (size_t)s * D + 4 * x);
      }
    }
    float m = top;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int s = i + u * PAR;
      if (s < a.p_chunks ? len < 0 : (s - a.p_chunks) * a.o_chunk >= len) p[u].x = -INFINITY;
      m = fmaxf(m, p[u].x);
    }
    const float c = top == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(top - m);
    acc *= c;
    total *= c;
    top = m;
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (p[u].x != -INFINITY) {
        const float w = __builtin_amdgcn_exp2f(p[u].x - m);
        acc += w * v[u];
        total += w * p[u].y;
      }
  }
  float all = top;
#pragma unroll
  for (int o = 32; o >= LD; o >>= 1) all = fmaxf(all, __shfl_xor(all, o));
  const float c = top == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(top - all);
  acc *= c;
  total *= c;
#pragma unroll
  for (int o = 32; o >= LD; o >>= 1) {
    total += __shfl_xor(total, o);
#pragma unroll
    for (int i = 0; i < 4; ++i) acc[i] += __shfl_xor(acc[i], o);
  }
  if (lane < LD) put_query<T>(a, b, t, h, x, acc, all, total);
}

constexpr int kMaxRows = 1 << 30;
// a grid holds fewer than 2^32 threads
constexpr int kMaxBlocks = (1 << 24) - 1;  // of 64 kWaves threads
constexpr int kMergeQueries = 1 << 25;     // of a launch

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

// whether rows of out share an element
bool out_rows_overlap(const ssd_prefix_attn_desc& a) {
  struct Dim {
    int64_t n, step;
  } d[3] = {{a.n_seq, a.out_seq}, {a.n_query, a.out_row}, {a.n_head, a.out_head}};
  for (Dim& x : d) {
    if (x.n == 1) x.step = a.head_dim;
    if (x.step < a.head_dim) return true;
  }
  std::sort(d, d + 3, [](const Dim& x, const Dim& y) { return x.step < y.step; });
  // steps that pass by all that the smaller ones reach
  int64_t reach = a.head_dim;
  bool nested = true;
  for (const Dim& x : d) {
    nested &= x.n == 1 || x.step >= reach;
    reach += (x.n - 1) * x.step;
  }
  if (nested) return false;
  // else every difference of two rows, that of the longest dimension the nearest to the others'
  std::sort(d, d + 3, [](const Dim& x, const Dim& y) { return x.n < y.n; });
  for (int64_t i = 0; i < d[0].n; ++i)
    for (int64_t j = i ? 1 - d[1].n : 0; j < d[1].n; ++j) {
      const int64_t by = i * d[0].step + j * d[1].step;
      const int64_t near = -by / d[2].step;
      for (int64_t k = std::max(near - 1, 1 - d[2].n); k <= std::min(near + 1, d[2].n - 1); ++k)
        if ((i || j || k) && std::abs(by + k * d[2].step) < a.head_dim) return true;
    }
  return false;
}

ssd_status check_strides(const ssd_prefix_attn_desc* a) {
  const int64_t s[] = {a->q_seq, a->q_row, a->q_head, a->prefix_head, a->prefix_row, a->own_seq, a->own_head,
                       a->own_row, a->out_seq, a->out_row, a->out_head};
  const int unit = 16 / op_size(a->dtype);
  for (int64_t x : s) {
    OP_REQUIRE(x >= 0, SSD_E_INVALID_ARG, "a stride is negative");
    OP_REQUIRE(x % unit == 0, SSD_E_UNSUPPORTED, "a stride is not a multiple of 16 bytes");
  }
  OP_REQUIRE(!out_rows_overlap(*a), SSD_E_INVALID_ARG, "out's rows overlap");
  return SSD_OK;
}

// whether out shares an element with an input
bool out_overlaps(const ssd_prefix_attn_desc& a, const void* q, const void* kp, const void* vp, const void* ko,
                  const void* vo, const int32_t* own_len, const void* out) {
  const int64_t es = op_size(a.dtype);
  const OpView::Dim row = {a.head_dim, es};
  auto queries = [&](const void* p, int64_t seq, int64_t pos, int64_t head) {
    return OpView{p, {{a.n_seq, seq * es}, {a.n_query, pos * es}, {a.n_head, head * es}, row}};
  };
  auto prefix = [&](const void* p) {
    return OpView{p, {{1, 0}, {a.n_kv_head, a.prefix_head * es}, {a.prefix_len, a.prefix_row * es}, row}};
  };
  auto own = [&](const void* p) {
    return OpView{p, {{a.n_seq, a.own_seq * es}, {a.n_kv_head, a.own_head * es}, {a.own_rows, a.own_row * es}, row}};
  };
  const OpView o = queries(out, a.out_seq, a.out_row, a.out_head);
  for (const OpView& in : {queries(q, a.q_seq, a.q_row, a.q_head), prefix(kp), prefix(vp), own(ko), own(vo),
                           OpView{own_len, {{1, 0}, {1, 0}, {1, 0}, {a.n_seq, 4}}}})
    if (!op_apart(o, in)) return true;
  return false;
}

// How a call is cut up.
//   Alone (short_attn_kernel): a sequence's queries take the prefix and their own rows
// in one workgroup, where the prefix is short for the number of workgroups that
// read it again: up to 2 steps of the four waves (a step: 128 rows of bfloat16, 64
// of float32), and where a tile's 32 columns are more than half used, 1 and 1 more per 16
// workgroups up to 16 steps; and where a sequence's own rows would be one chunk, or
// both are 4 steps.  Measured, split and alone (us): 1 sequence of 20 heads of 64, 256 rows
// and 64 of its own 7.2 and 5.8, 1024 rows 7.5 and 9.0; 128 sequences of it, 128
// rows 22 and 20, 512 rows 24 and 32; 8 queries, 16 heads on 4 of 128: 8
// sequences, 256 rows 12.3 and 11.9, 512 rows 12.8 and 14.1; 64 sequences, 2048 rows 38
// and 28; float32, 512 rows 49 and 33.  48 x 5 queries, 32 heads on 8 of 128:
// 2048 rows 39 and 34, 4096 rows 46 and 55.
//   Else the prefix is read once for all.  Up to 32 queries of a kv head: one
// tile, the waves split the rows.  More: tiles of 64 or 128, the waves split the
// queries.  The rows are cut so that the workgroups are one round over the CUs, and two a CU where
// there are products to overlap, in chunks longer than kOverlap rows: more, shorter chunks cost
// more parts than they even out (16 sequences over 100,000 rows: 97 us with 256
// workgroups, 100 with 512, 103 with 1024; 48 x 5 queries with grouped heads, with 256, 512
// and 1024: 65,536 rows 426, 298 and 310 us, 8,191 rows 71, 71 and 83, 4,096 rows 43, 46 and
// 57; 33 x 2, 20 heads of 64 over 3000 rows 16.5, 19.4 and 19.4; 20 x 8 float32, 32 heads on
// 8 of 128 over 3000 rows 92, 89 and 99).
constexpr int kRound = 256;
constexpr int kOverlap = 1024, kOverlapF32 = 256;  // (products of float32 take four times as long)

struct Plan {
  bool alone;  // see short_attn_kernel
  bool byq;    // see prefix_attn_kernel
  int mp, mo;  // matrix tiles per wave
  int p_cols, p_tiles, p_chunks, p_chunk, p_blocks, o_tiles, o_chunks, o_chunk;
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
  p.byq = cols > 32;
  p.mp = p.byq ? (cols > 64 ? 2 : 1) : tile_of(cols, 2);
  p.mo = tile_of(own_cols, 2);
  p.p_cols = 16 * p.mp * (p.byq ? kWaves : 1);
  p.p_tiles = (int)div_up(cols, p.p_cols);
  p.o_tiles = (int)div_up(own_cols, 16 * p.mo);
  auto cut = [&](int64_t rows, int64_t sets, int& chunks, int& chunk) {
    const bool twice = p.byq && div_up(rows, std::max<int64_t>(kRound / sets, 1)) >
                                    (a->dtype == SSD_F32 ? kOverlapF32 : kOverlap);
    const int round = twice ? 2 * kRound : kRound;
    const int64_t want = std::min(std::max<int64_t>(round / sets, 1), std::max<int64_t>(div_up(rows, step), 1));
    chunk = (int)(div_up(std::max<int64_t>(div_up(rows, want), 1), step) * step);
    chunks = (int)div_up(rows, chunk);
  };
  const int64_t own_blocks = (int64_t)a->n_seq * a->n_kv_head * p.o_tiles;
  cut(a->own_rows, own_blocks, p.o_chunks, p.o_chunk);
  const int64_t again = p.mo == 2 ? std::clamp<int64_t>(1 + own_blocks / 16, 2, 16) : 2;
  p.alone = a->prefix_len <= again * step && (p.o_chunks <= 1 || (int64_t)a->prefix_len + a->own_rows <= 4 * step);
  if (p.alone) {
    p.blocks = own_blocks;
    p.bytes = 16;  // (not used)
    return p;
  }
  cut(a->prefix_len, (int64_t)a->n_kv_head * p.p_tiles, p.p_chunks, p.p_chunk);
  p.p_blocks = (int)(div_up((int64_t)a->n_kv_head * p.p_chunks, 8) * 8 * p.p_tiles);
  p.blocks = p.p_blocks + own_blocks * p.o_chunks;
  const int64_t slots = (int64_t)a->n_seq * a->n_query * a->n_head * std::max(1, p.p_chunks + p.o_chunks);
  p.o_bytes = (size_t)slots * a->head_dim * 4;
  p.bytes = p.o_bytes + (size_t)slots * sizeof(float2);
  return p;
}

// Once per kernel and device: more than 64 KB of LDS, with the kernel's own, has
// to be asked for.
template <auto kernel>
hipError_t ask_for_lds(int bytes) {
  static std::atomic<uint64_t> ready{0};
  int dev = 0;
  hipError_t e = hipGetDevice(&dev);
  if (e != hipSuccess) return e;
  const uint64_t bit = dev < 64 ? 1ull << dev : 0;
  if (ready.load(std::memory_order_acquire) & bit) return hipSuccess;
  e = hipFuncSetAttribute((const void*)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
  if (e == hipSuccess) ready.fetch_or(bit, std::memory_order_release);
  return e;
}
template <typename T, int D, int MP, int MO, bool BYQ>
hipError_t launch(const PrefixAttnArgs& a, int64_t blocks, hipStream_t s) {
  constexpr int rows = kWaves * 2 * Block<T, D>::BYTES, queries = kStages * Stage<T, D>::BYTES;
  constexpr int lds = BYQ && queries > rows ? queries : rows;
  hipError_t e = ask_for_lds<prefix_attn_kernel<T, D, MP, MO, BYQ>>(lds);
  if (e != hipSuccess) return e;
  if (blocks > 0) prefix_attn_kernel<T, D, MP, MO, BYQ><<<(unsigned)blocks, 64 * kWaves, lds, s>>>(a);
  e = hipGetLastError();
  if (e != hipSuccess) return e;
  const int n = a.d.n_seq * a.d.n_query * a.d.n_head;
  for (int first = 0; first < n && e == hipSuccess; first += kMergeQueries) {
    merge_kernel<T, D><<<(std::min(n - first, kMergeQueries) + 3) / 4, 256, 0, s>>>(a, first, n);
    e = hipGetLastError();
  }
  return e;
}
template <typename T, int D, int MO>
hipError_t launch_short(const PrefixAttnArgs& a, int64_t blocks, hipStream_t s) {
  constexpr int lds = kWaves * 2 * Block<T, D>::BYTES;
  const hipError_t e = ask_for_lds<short_attn_kernel<T, D, MO>>(lds);
  if (e != hipSuccess) return e;
  short_attn_kernel<T, D, MO><<<(unsigned)blocks, 64 * kWaves, lds, s>>>(a);
  return hipGetLastError();
}
template <typename T, int D>
hipError_t launch(const PrefixAttnArgs& a, const Plan& p, hipStream_t s) {
  if (p.alone) return p.mo == 2 ? launch_short<T, D, 2>(a, p.blocks, s) : launch_short<T, D, 1>(a, p.blocks, s);
  if (p.byq) {
    if (p.mp == 2) return p.mo == 2 ? launch<T, D, 2, 2, true>(a, p.blocks, s) : launch<T, D, 2, 1, true>(a, p.blocks, s);
    return p.mo == 2 ? launch<T, D, 1, 2, true>(a, p.blocks, s) : launch<T, D, 1, 1, true>(a, p.blocks, s);
  }
  if (p.mp == 2) return p.mo == 2 ? launch<T, D, 2, 2, false>(a, p.blocks, s) : launch<T, D, 2, 1, false>(a, p.blocks, s);
  return launch<T, D, 1, 1, false>(a, p.blocks, s);  // (a sequence has no more queries than all)
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
  OP_REQUIRE(p.blocks <= kMaxBlocks, SSD_E_CAPACITY, "more workgroups than a grid holds");
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
  OP_REQUIRE(!out_overlaps(*a, q, k_prefix, v_prefix, k_own, v_own, own_len, out), SSD_E_INVALID_ARG,
             "out overlaps an input");
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
  x.p_cols = p.p_cols;
  x.p_tiles = p.p_tiles;
  x.p_chunks = p.p_chunks;
  x.p_chunk = p.p_chunk;
  x.p_blocks = p.p_blocks;
  x.o_tiles = p.o_tiles;
  x.o_chunks = p.o_chunks;
  x.o_chunk = p.o_chunk;
  x.parts = p.p_chunks + p.o_chunks;
  x.scale2 = fabsf(a->scale) * 1.4426950408889634f;
  const hipError_t e = a->dtype == SSD_F32 ? launch<float>(x, p, (hipStream_t)stream) : launch<bf16_t>(x, p, (hipStream_t)stream);
  if (e != hipSuccess) return op_fail(SSD_E_DEVICE, hipGetErrorString(e));
  return SSD_OK;
}
