// Attention over a paged cache in 8 bits (ssd_paged_attn of ssd_pages.h).
//
// With x_j the scaled score of row j, in units of log 2, and a set c of rows:
//   m_c >= max x_j - 8,  l_c = sum 2^(x_j - m_c),  o_c = sum 2^(x_j - m_c) v_j;
// out = sum_c 2^(m_c - M) o_c / sum_c 2^(m_c - M) l_c with M the largest m_c.
//
// A workgroup of four waves takes up to 16 NT queries of one sequence and kv head (its new rows' and the
// group's heads) and every splits-th part of the rows; a wave takes 32 rows at a time, and never
// waits for another until the end.  Codes go from memory to registers in operand order (see
// ops_pages.h), 16 bytes a lane, are made float16 there (exactly: whole numbers up to 127, or
// 4 bits), and their scales multiply scores and products:
//   x = (code_k . q) scale_k scale,   o += (code_v 2^(x - r)) 2^(r - m) scale_v,   r = max x of the 32 rows and a query.
// So a weight is rounded by what it is among its own 32 rows, which share a scale, whatever scales and weights other rows
// have, and o is float32 throughout.
// Queries are scaled by a power of two each, to the middle of float16's range, and split into
// parts of 11 bits: bfloat16's 8 bits are one, float32's 24 three.
//
// Bound, and what it measured (int8 unless said otherwise; read: 6.1 TB/s is the most this card reads at, 5.2 a copy moves at):
//   32 sequences of about 1800 rows, 20 heads of 64, one query       31 us, 145 MB: 4.7 TB/s; a short call, its loads alone 31
//   48 sequences of about 7100 rows, 32 heads on 8 of 128, 5 queries, e4m3    140 us, 712 MB: 5.1 TB/s
//   4 sequences, 8 queries over a window of 4000 rows, 20 heads of 64         16 us, 44 MB: 14 the parts, 4 the join (traced)
//   3 sequences of 200 rows, 4 heads of 32, float32                   8 us, of which a launch is 3: the chain length, table,
//                                                                     scales, codes, products, join
//   4 sequences of 4000 rows, 32 heads on 8 of 128, 64 queries        54 us: the softmax's arithmetic and the products
// With more than one query a kv head the matrix units have slots to spare (16 columns a product), so the
// vector instructions count: per item of 32 rows and 64 dims 64 turn codes into float16, whatever the
// queries' number; then comes the softmax of 8 scores a lane, its weights' two parts, and 16 operations a tile that add what
// the 32 rows add (one card, 48 x 5 queries: 152 us without either, 155 with the adding, 160 with both).
// What was measured and not kept: four queries or fewer as the rows of products, a score a
// lane (32 sequences that share one prompt 27 -> 22 us, but 35.3 -> 34.9 where the pages come from memory, float32 25.5 -> 28.6
// and four queries 92 -> 105 us); three and four items of loads ahead (36 -> 37 to 39 us).
#include <algorithm>
#include <atomic>
#include <type_traits>

#include "ops_pages.h"

namespace ssd {
namespace {

typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

constexpr int kWaves = 4;
constexpr float kFar = 4194304.f - 256.f;  // references from here on take scores that are rounded first: see weights()
// How far a score may lie above the reference (the largest so far, in units of log 2) before the sums are rescaled: weights
// up to 2^8.  So most items rescale nothing.
constexpr float kSlack = 8.f;
// float32 calls hold all weights, and with them l and o, multiplied by 2^kUp: so the lower ones of two float16 parts are not
// below what float16 holds to 11 bits.  (By the reference instead, exponents would be rounded as numbers around 15.)
constexpr float kUp = 15.f;
// Sums of 2^30 rows with weights up to 2^23 and values up to 2^128 would not be finite where their quotient is.  From finite values
// of 2^80 of rows that are seen, or scales of 2^48, on a wave's references are made larger by so much, and its weights
// smaller (their exponents are rounded as numbers around 56 then: 19 bits).
constexpr float kLift = 56.f;
constexpr unsigned kLarge = 127 + 80, kLargeScale = 127 + 48;  // (exponents, as float32 and bfloat16 hold them)

struct Args {
  ssd_paged_attn_desc d;
  const uint8_t* data;  // of the layer
  const float2* scale;
  const int *table, *length;
  int64_t table_ld;
  int n_seq, n_col, n_page, n_kv_head, page_rows;
  const char *q, *kt, *vt, *kn, *vn;
  const int64_t* anc;
  char* out;
  float* lse;
  float* o;    // [part][tile][query of the tile][head_dim]
  float2* ml;  // [part][tile][query of the tile] (m, l)
  int tiles, cols, owners;
  int parts;     // that there is room for
  int splits;    // parts of every sequence, 0: see find_part()
  int round;     // workgroups that those are cut for
  float scale2;  // scale log2 e
};

// The N results are complete.  An instruction may read a matrix product's result 8 (16-bit operands) or 10
// (float32) instructions' time after it and not sooner, and neither the hardware nor, across
// the end of a block, the compiler sees to it: results that are read behind a branch are waited
// for here first.
template <int N>
__device__ __forceinline__ void complete(f32x4* x) {
  static_assert(N == 1 || N == 2 || N == 4, "one statement for all: its wait comes after every product");
  if constexpr (N == 1)
    asm volatile("s_nop 9" : "+v"(x[0]));
  else if constexpr (N == 2)
    asm volatile("s_nop 9" : "+v"(x[0]), "+v"(x[1]));
  else
    asm volatile("s_nop 9" : "+v"(x[0]), "+v"(x[1]), "+v"(x[2]), "+v"(x[3]));
}

// eight codes as float16
template <int CODE>
__device__ __forceinline__ f16x8 codes8(unsigned lo, unsigned hi) {
  f16x2 x[4];
  if constexpr (CODE == SSD_PAGE_INT8) {
    // 0x64bb is 1024 + bb
    const f16x2 bias = {(_Float16)1152.f, (_Float16)1152.f};
    x[0] = __builtin_bit_cast(f16x2, __builtin_amdgcn_perm(0x64646464u, lo, 0x04010400u)) - bias;
    x[1] = __builtin_bit_cast(f16x2, __builtin_amdgcn_perm(0x64646464u, lo, 0x04030402u)) - bias;
    x[2] = __builtin_bit_cast(f16x2, __builtin_amdgcn_perm(0x64646464u, hi, 0x04010400u)) - bias;
    x[3] = __builtin_bit_cast(f16x2, __builtin_amdgcn_perm(0x64646464u, hi, 0x04030402u)) - bias;
  } else {
    x[0] = __builtin_bit_cast(f16x2, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, 1.f, false));
    x[1] = __builtin_bit_cast(f16x2, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, 1.f, true));
    x[2] = __builtin_bit_cast(f16x2, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, 1.f, false));
    x[3] = __builtin_bit_cast(f16x2, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, 1.f, true));
  }
  return (f16x8){x[0][0], x[0][1], x[1][0], x[1][1], x[2][0], x[2][1], x[3][0], x[3][1]};
}
__device__ __forceinline__ f32x4 product(f16x8 a, f16x8 b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ f32x4 product(bf16x8 a, bf16x8 b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ f32x4 product(float a, float b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x4f32(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ float group_max(float x) {  // over the lanes of a column, within the registers
  const u32x2 a = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  x = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
  const u32x2 b = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}
// Eight weights (1 the largest) in two float16 parts each, cut off: 20 bits from 2^-4 on, and to 2^-24.  (One part, 11 bits, moved a bfloat16 result by a step in
// one of 20 elements; the second is a product more and the time of one in 33 where queries are many: 48 x 5 queries over
// 7100 rows 155.5 -> 161 us, one query and short calls the same.  Rounded parts, 21 bits, took 164.)
__device__ __forceinline__ void halves(const f32x4 (&s)[2], f16x8& hi, f16x8& lo) {
#pragma unroll
  for (int i = 0; i < 8; i += 2) {
    const float a = s[i >> 2][i & 3], b = s[i >> 2][(i & 3) + 1];
    const f16x2 h = __builtin_bit_cast(f16x2, __builtin_amdgcn_cvt_pkrtz(a, b));
    float x, y;  // a and b less those, in one operation each
    asm("v_fma_mix_f32 %0, %1, -1.0, %2 op_sel_hi:[1,0,0]" : "=v"(x) : "v"(h), "v"(a));
    asm("v_fma_mix_f32 %0, %1, -1.0, %2 op_sel:[1,0,0] op_sel_hi:[1,0,0]" : "=v"(y) : "v"(h), "v"(b));
    const f16x2 r = __builtin_bit_cast(f16x2, __builtin_amdgcn_cvt_pkrtz(x, y));
    hi[i] = h[0];
    hi[i + 1] = h[1];
    lo[i] = r[0];
    lo[i + 1] = r[1];
  }
}
// a block's bytes of 32 rows: of keys and of values, 16 a lane each
template <int D>
struct Codes {
  u32x4 k[D / 32], v[D / 32];
  // (read once: they pass by the caches.  48 x 1 query over 7100 rows 105 us, 113 with plain loads)
  __device__ __forceinline__ void load(const uint8_t* keys, const uint8_t* values, int lane) {
#pragma unroll
    for (int i = 0; i < D / 32; ++i) k[i] = __builtin_nontemporal_load((const u32x4*)(keys + 1024 * i + 16 * lane));
#pragma unroll
    for (int i = 0; i < D / 32; ++i) v[i] = __builtin_nontemporal_load((const u32x4*)(values + 1024 * i + 16 * lane));
  }
  // bytes of step st of the product of keys 16 k .. + 15
  template <int CODE>
  __device__ __forceinline__ f16x8 keys(int k_, int st) const {
    const int i = D == 32 ? 0 : k_ * (D / 64) + (st >> 1), h = D == 32 ? k_ : st & 1;
    return codes8<CODE>(k[i][2 * h], k[i][2 * h + 1]);
  }
  // of dims 16 dt .. + 15
  template <int CODE>
  __device__ __forceinline__ f16x8 values(int dt) const {
    return codes8<CODE>(v[dt >> 1][2 * (dt & 1)], v[dt >> 1][2 * (dt & 1) + 1]);
  }
};

// the largest of eight, NaN passed over (one instruction for three: fmaxf would have each operand made quiet first)
__device__ __forceinline__ float max3(float a, float b, float c) {
  float x;
  asm("v_max3_f32 %0, %1, %2, %3" : "=v"(x) : "v"(a), "v"(b), "v"(c));
  return x;
}
__device__ __forceinline__ float largest(f32x4 a, f32x4 b) {
  return max3(max3(a[0], a[1], a[2]), max3(a[3], b[0], b[1]), max3(b[2], b[3], b[3]));
}

// What a wave knows of its call, whichever way it takes its queries.  Lane 16 g + n.
template <typename T, int D, int CODE_>
struct Base {
  typedef T Type;
  static constexpr bool F32 = sizeof(T) == 4;
  static constexpr int CODE = CODE_, DIM = D, KS = D / 32, DT = D / 16;
  static constexpr int NQ = F32 ? 3 : 1, NP = 2;  // parts of a query, of a weight
  const Args& a;
  const int lane, g, n;
  float lift;    // a reference is so far above the score that it is made of: 0 or kLift
  bool rounded;  // a reference is far from 0: see weights()

  __device__ __forceinline__ Base(const Args& args)
      : a(args), lane(threadIdx.x & 63), g(lane >> 4), n(lane & 15), lift(0.f), rounded(false) {}

  // the 8 dims from here on are what the lane has in step s of a product over dims
  __device__ __forceinline__ int dim_at(int s) const { return D == 32 ? 8 * g : 64 * (s >> 1) + 16 * g + 8 * (s & 1); }

  // A query, as it is: its loads are under way when issue() returns.  Columns behind the last query load the first of all, see
  // nothing, and have a reference that no score is above: what they hold decides nothing for the others.
  struct Query {
    u32x4 x[KS][F32 ? 2 : 1];
    int64_t anc;
    int step;  // its new row, -1: none
  };
  __device__ __forceinline__ void issue(Query& q, int b, int kv, int c) {
    const int group = a.d.n_head / a.n_kv_head, cols = a.d.n_query * group;
    const int t = group == 1 ? c : c / group;
    q.step = c < cols ? t : -1;
    const T* p = (const T*)a.q + (c < cols ? b * a.d.q_seq + t * a.d.q_row + (kv * group + c - t * group) * a.d.q_head : 0);
#pragma unroll
    for (int s = 0; s < KS; ++s)
#pragma unroll
      for (int i = 0; i < (F32 ? 2 : 1); ++i) q.x[s][i] = *(const u32x4*)(p + dim_at(s) + 4 * i);
    q.anc = a.anc ? a.anc[(int64_t)b * a.d.n_query + max(q.step, 0)] : 0;
  }
  // what it sees
  __device__ __forceinline__ void sees(const Query& q, int len, uint64_t& anc, int& seen_from) const {
    const int t = q.step;
    anc = t >= 63 ? ~0ull : (2ull << max(t, 0)) - 1;
    if (a.anc) anc = (uint64_t)q.anc & (~0ull >> (64 - a.d.n_query));
    const int depth = a.anc ? max(__popcll(anc) - 1, 0) : max(t, 0);
    seen_from = a.d.window ? len + depth - a.d.window + 1 : 0;
  }
  // its parts for products with codes, and what such a product is multiplied by
  __device__ __forceinline__ void split(const Query& q, f16x8 (&parts)[KS][NQ], float& unit) const {
    float x[KS][8], top = 0.f;
#pragma unroll
    for (int s = 0; s < KS; ++s)
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        if constexpr (F32) x[s][i] = __uint_as_float(q.x[s][i >> 2][i & 3]);
        else x[s][i] = __uint_as_float(i & 1 ? q.x[s][0][i >> 1] & 0xffff0000u : q.x[s][0][i >> 1] << 16);
        top = fmaxf(top, finite(x[s][i]) ? fabsf(x[s][i]) : 0.f);
      }
    top = group_max(top);
    // the largest finite one to [2^14, 2^15): what is smaller by up to 2^28 keeps its 11 bits
    const int e = max((int)(__float_as_uint(top) >> 23) - 127, -100);
    const float by = __uint_as_float((unsigned)(min(14 - e, 127) + 127) << 23);
    unit = fabsf(a.scale2) * __uint_as_float((unsigned)(max(e - 14, -126) + 127) << 23);
#pragma unroll
    for (int s = 0; s < KS; ++s)
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        float y = q.step < 0 ? 0.f : x[s][i] * (a.scale2 < 0.f ? -by : by);
#pragma unroll
        for (int p = 0; p < NQ; ++p) {
          parts[s][p][i] = (_Float16)y;
          y = finite(y) ? y - (float)parts[s][p][i] : 0.f;  // (infinity is one part)
        }
      }
  }

  // 32 rows in the model's type: those from x0 on of `tail` open rows, the first at place `slot` of the ring, and of
  // the new ones behind them; rows past the last are the last again.  Lane (g, n): row 16 k + n of the keys, rows
  // 16 (i / 4) + 4 g + i mod 4 of the values at dims 16 dt + n.  Loads are under way when issue_own() returns.
  struct Own {
    u32x4 k[2][KS][F32 ? 2 : 1];
    typename std::conditional<F32, float, uint16_t>::type v[DT][8];
  };
  template <bool KEYS, bool VALUES>
  __device__ __forceinline__ void issue_own(Own& rows, int b, int kv, int x0, int tail, int slot) {
    const int total = tail + a.d.n_query;
    const int64_t told = b * a.d.tail_seq + kv * a.d.tail_head, tnew = b * a.d.new_seq + kv * a.d.new_head;
    auto row = [&](const char* old, const char* add, int x) {
      x = min(x, total - 1);
      const bool open = x < tail;
      const int at = slot + x, place = open ? at - (at >= a.d.tail_rows ? a.d.tail_rows : 0) : x - tail;
      return (const T*)(open ? old : add) + (open ? told : tnew) + place * (open ? a.d.tail_row : a.d.new_row);
    };
#pragma unroll
    for (int k = 0; KEYS && k < 2; ++k) {
      const T* p = row(a.kt, a.kn, x0 + 16 * k + n);
#pragma unroll
      for (int s = 0; s < KS; ++s)
#pragma unroll
        for (int i = 0; i < (F32 ? 2 : 1); ++i) rows.k[k][s][i] = *(const u32x4*)(p + dim_at(s) + 4 * i);
    }
#pragma unroll
    for (int i = 0; VALUES && i < 8; ++i) {
      const T* p = row(a.vt, a.vn, x0 + 16 * (i >> 2) + 4 * g + (i & 3)) + n;
#pragma unroll
      for (int dt = 0; dt < DT; ++dt)
        rows.v[dt][i] = __builtin_bit_cast(typename std::conditional<F32, float, uint16_t>::type, p[16 * dt]);
    }
  }
  // products over dims of keys 16 k .. and a query
  __device__ __forceinline__ f32x4 own_scores(const Own& rows, int k, const Query& q) {
    f32x4 sum = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int s = 0; s < KS; ++s) {
      if constexpr (F32) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const float x = __uint_as_float(rows.k[k][s][i >> 2][i & 3]), y = __uint_as_float(q.x[s][i >> 2][i & 3]);
          sum = product(x, y, sum);
        }
      } else {
        const bf16x8 x = __builtin_bit_cast(bf16x8, rows.k[k][s][0]), y = __builtin_bit_cast(bf16x8, q.x[s][0]);
        sum = product(x, y, sum);
      }
    }
    return sum;
  }
  __device__ __forceinline__ bool sees_own(int x, int tail, int start, int seen_from, uint64_t anc) const {
    if (x < tail) return start + x >= seen_from || start + x < a.d.sinks;
    return x < tail + a.d.n_query && (anc >> (x - tail & 63) & 1);
  }
  static __device__ __forceinline__ bool finite(float x) { return fabsf(x) < __builtin_inff(); }
  static __device__ __forceinline__ bool finite(uint16_t x) { return (x & 0x7f80u) != 0x7f80u; }
  __device__ __forceinline__ bool all_finite(const Own& rows) const {
    bool odd = false;
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
      for (int i = 0; i < 8; ++i) odd |= !finite(rows.v[dt][i]);
    return !__builtin_amdgcn_ballot_w64(odd);
  }
  // whether |x| is 2^(from - 127) or more, and finite
  static __device__ __forceinline__ bool large(float x, unsigned from) {
    return (__float_as_uint(x) >> 23 & 255u) - from < 255u - from;
  }
  static __device__ __forceinline__ bool large(uint16_t x, unsigned from) { return (x >> 7 & 255u) - from < 255u - from; }
  // whether one of the values is so of a row that a query of the wave sees (bits: the lane's of its column's)
  __device__ __forceinline__ bool any_large(const Own& rows, unsigned bits) const {
    bool odd = false;
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
      for (int i = 0; i < 8; ++i) odd |= large(rows.v[dt][i], kLarge);
    if (!__builtin_amdgcn_ballot_w64(odd)) return false;
    odd = false;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const bool seen = __builtin_amdgcn_ballot_w64(bits >> i & 1) >> (16 * g) & 0xffff;
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) odd |= seen && large(rows.v[dt][i], kLarge);
    }
    return __builtin_amdgcn_ballot_w64(odd);
  }
  // which of a dim's values are not finite, as 1; they become 0
  __device__ __forceinline__ bf16x8 take_out(Own& rows, int dt) const {
    bf16x8 y;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const bool bad = !finite(rows.v[dt][i]);
      y[i] = (__bf16)(bad ? 1.f : 0.f);
      if (bad) rows.v[dt][i] = 0;
    }
    return y;
  }
};

// Up to 16 NT queries as the columns of products with keys and with values: lane 16 g + n has query n of every tile,
// of scores the rows 4 g + r of 16, of outputs the dims 4 g + r of 16.
template <typename T, int D, int CODE, int NT_>
struct Tiles : Base<T, D, CODE> {
  typedef Base<T, D, CODE> B;
  using typename B::Own;
  using B::a, B::g, B::n, B::lane, B::KS, B::DT, B::NQ, B::NP, B::F32;
  static constexpr int NT = NT_, COLS = 16 * NT;
  static constexpr bool EARLY = !(D == 128 && (F32 || NT == 2)) && !(F32 && D == 64 && NT == 2);  // see take_own()
  typename B::Query raw[NT];
  f16x8 q[NT][KS][NQ];
  float unit[NT];
  f32x4 o[NT][DT];
  float m[NT], l[NT];  // reference, this lane's share of the sum
  int seen_from[NT];
  uint64_t anc[NT];

  __device__ __forceinline__ Tiles(const Args& args) : B(args) {}
  __device__ __forceinline__ void issue(int b, int kv, int tile) {
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) B::issue(raw[nt], b, kv, (tile * NT + nt) * 16 + n);
  }
  __device__ __forceinline__ void begin(int len) {
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      B::sees(raw[nt], len, anc[nt], seen_from[nt]);
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) o[nt][dt] = (f32x4){0.f, 0.f, 0.f, 0.f};
      m[nt] = raw[nt].step < 0 ? INFINITY : -INFINITY;
      l[nt] = 0.f;
    }
  }
  __device__ __forceinline__ void split() {
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) B::split(raw[nt], q[nt], unit[nt]);
  }

  // s by (by >= 0) are the scores of 32 rows; what is `masked` and not seen(tile, k, r): row 16 k + 4 g + r, becomes
  // -infinity, by then 1.  top: the largest of a column.  The sums are rescaled where it is far above the reference.
  template <typename Seen>
  __device__ __forceinline__ void meet(f32x4 (&s)[NT][2], float (&by)[NT], float (&top)[NT], bool masked, Seen seen) {
    bool far = false;
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      if (masked) {
#pragma unroll
        for (int k = 0; k < 2; ++k)
#pragma unroll
          for (int r = 0; r < 4; ++r)
            s[nt][k][r] = seen(nt, k, r) ? s[nt][k][r] * by[nt] : -INFINITY;
        by[nt] = 1.f;
      }
      top[nt] = group_max(by[nt] * largest(s[nt][0], s[nt][1]));
      far |= top[nt] > m[nt] + (kSlack - this->lift);
    }
    if (__builtin_amdgcn_ballot_w64(far)) {
      bool large = false;
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        const float now = fmaxf(m[nt], top[nt] + this->lift);
        const float f = m[nt] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m[nt] - now);
        m[nt] = now;
        large |= fabsf(now) >= kFar && fabsf(now) < INFINITY;
        l[nt] *= f;
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) o[nt][dt] *= f;
      }
      if (__builtin_amdgcn_ballot_w64(large)) this->rounded = true;
    }
  }
  // s becomes 2^(s by - ref) (float32: 2^kUp times that), and sum what the lane has of its sum.  Product and difference are one operation; from
  // references of 2^22 on, where the largest score and the reference made of it would differ by the product's
  // rounding, and the weight with it, they are two.
  __device__ __forceinline__ void weights(f32x4 (&s)[NT][2], float (&by)[NT], const float (&ref)[NT], float (&sum)[NT]) {
#pragma clang fp contract(off)
    if (this->rounded) {
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
        for (int k = 0; k < 2; ++k)
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            s[nt][k][r] *= by[nt];
            asm volatile("" : "+v"(s[nt][k][r]));  // (not to be made one operation with what follows)
          }
        by[nt] = 1.f;
      }
    }
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
      for (int k = 0; k < 2; ++k)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          s[nt][k][r] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[nt][k][r], by[nt], -ref[nt]));
          if constexpr (F32) s[nt][k][r] *= 1 << (int)kUp;
        }
      sum[nt] = ((s[nt][0][0] + s[nt][0][1]) + (s[nt][0][2] + s[nt][0][3])) +
                ((s[nt][1][0] + s[nt][1][1]) + (s[nt][1][2] + s[nt][1][3]));
    }
  }

  // 32 rows of a page, the first at position `first`
  __device__ __forceinline__ void take(const Codes<D>& c, float kscale, float vscale, int first, bool masked) {
    f32x4 s[NT][2];
#pragma unroll
    for (int k = 0; k < 2; ++k) {
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) s[nt][k] = (f32x4){0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int st = 0; st < KS; ++st) {
        const f16x8 y = c.template keys<CODE>(k, st);
#pragma unroll
        for (int p = NQ - 1; p >= 0; --p)
#pragma unroll
          for (int nt = 0; nt < NT; ++nt) s[nt][k] = product(y, q[nt][st][p], s[nt][k]);
      }
    }
    complete<2 * NT>(&s[0][0]);
    if (kscale < 0.f) {
      asm volatile("");  // (a branch, not selects: stored pages have no such scale)
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) s[nt][0] = -s[nt][0], s[nt][1] = -s[nt][1];
    }
    float by[NT];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) by[nt] = fabsf(kscale) * unit[nt];
    const int sinks = a.d.sinks;
    int mine = first + 4 * g;
    if (masked) asm volatile("" : "+v"(mine));  // (not to be taken out of the condition, in eight registers)
    float top[NT], ref[NT], f[NT], sum[NT];
    meet(s, by, top, masked, [&](int nt, int k, int r) {
      return mine + 16 * k + r >= seen_from[nt] || mine + 16 * k + r < sinks;
    });
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      // (no further below the query's reference than where f is 0 all the same: `rounded` goes by that)
      const bool none = top[nt] == -INFINITY;
      ref[nt] = none ? 0.f : fmaxf(top[nt], m[nt] - 200.f);
      f[nt] = none ? 0.f : __builtin_amdgcn_exp2f(ref[nt] - m[nt]);
    }
    weights(s, by, ref, sum);
    f16x8 w[NT][NP];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      l[nt] += f[nt] * sum[nt];
      if constexpr (!F32) {
        halves(s[nt], w[nt][0], w[nt][1]);
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          float y = s[nt][i >> 2][i & 3];
#pragma unroll
          for (int p = 0; p < NP; ++p) {
            w[nt][p][i] = (_Float16)y;
            y -= (float)w[nt][p][i];
          }
        }
      }
      f[nt] = top[nt] == -INFINITY ? 0.f : f[nt] * vscale;  // rows that a query does not see count 0 whatever the scale
    }
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) {
      const f16x8 y = c.template values<CODE>(dt);
      f32x4 part[NT];
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) part[nt] = (f32x4){0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int p = NP - 1; p >= 0; --p)
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) part[nt] = product(y, w[nt][p], part[nt]);
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) o[nt][dt] += part[nt] * f[nt];
    }
  }

  // (Values come at once where the registers hold them, else when the weights are known.)
  __device__ __forceinline__ void issue_own(Own& rows, int b, int kv, int x0, int tail, int slot) {
    B::template issue_own<true, EARLY>(rows, b, kv, x0, tail, slot);
  }
  __device__ __forceinline__ void take_own(Own& rows, int b, int kv, int x0, int tail, int start, int slot) {
    f32x4 s[NT][2];
    unsigned bits[NT];  // which of the lane's 8 rows are seen
    float by[NT];
    unsigned all = 0;
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      by[nt] = a.scale2;
      bits[nt] = 0;
#pragma unroll
      for (int i = 0; i < 8; ++i)
        bits[nt] |= B::sees_own(x0 + 16 * (i >> 2) + 4 * g + (i & 3), tail, start, seen_from[nt], anc[nt]) ? 1u << i : 0u;
      if (raw[nt].step < 0) bits[nt] = 0;
      all |= bits[nt];
    }
    if (EARLY && B::any_large(rows, all)) this->lift = kLift;
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int k = 0; k < 2; ++k) s[nt][k] = B::own_scores(rows, k, raw[nt]);
    complete<2 * NT>(&s[0][0]);
    float top[NT], ref[NT], sum[NT];
    meet(s, by, top, true, [&](int nt, int k, int r) { return (bits[nt] >> (4 * k + r) & 1) != 0; });
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      ref[nt] = m[nt] == -INFINITY ? 0.f : m[nt];
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (s[nt][i >> 2][i & 3] == -INFINITY) bits[nt] &= ~(1u << i);  // (counts as one that is not seen)
    }
    weights(s, by, ref, sum);
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) l[nt] += sum[nt];
    if constexpr (!EARLY) {
      B::template issue_own<false, true>(rows, b, kv, x0, tail, slot);
      if (this->lift == 0.f && B::any_large(rows, all)) {
        this->lift = kLift;
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
          const float now = m[nt] + kLift, f = fabsf(now) < __builtin_inff() ? __builtin_amdgcn_exp2f(m[nt] - now) : 1.f;
          m[nt] = now;
          l[nt] *= f;
          s[nt][0] *= f;
          s[nt][1] *= f;
#pragma unroll
          for (int dt = 0; dt < DT; ++dt) o[nt][dt] *= f;
        }
      }
    }
    // values that are not finite are taken out of the product, and make NaN where they are seen
    if (!B::all_finite(rows)) {
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) {
        const bf16x8 y = B::take_out(rows, dt);
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
          bf16x8 z;
#pragma unroll
          for (int i = 0; i < 8; ++i) z[i] = (__bf16)(bits[nt] >> i & 1 ? 1.f : 0.f);
          f32x4 count = product(y, z, (f32x4){0.f, 0.f, 0.f, 0.f});
          complete<1>(&count);
#pragma unroll
          for (int r = 0; r < 4; ++r) o[nt][dt][r] = count[r] > 0.f ? __builtin_nanf("") : o[nt][dt][r];
        }
      }
    }
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      bf16x8 hi, lo;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float w = s[nt][i >> 2][i & 3];
        hi[i] = (__bf16)w;
        lo[i] = (__bf16)(w - (float)hi[i]);
      }
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) {
        if constexpr (F32) {
#pragma unroll
          for (int i = 0; i < 8; ++i) o[nt][dt] = product(rows.v[dt][i], s[nt][i >> 2][i & 3], o[nt][dt]);
        } else {
          bf16x8 y;
#pragma unroll
          for (int i = 0; i < 8; ++i) y[i] = __builtin_bit_cast(__bf16, rows.v[dt][i]);
          o[nt][dt] = product(y, lo, o[nt][dt]);
          o[nt][dt] = product(y, hi, o[nt][dt]);
        }
      }
    }
  }

  // the wave's references and sums to ms (COLS each, `apart` from each other), then what it adds to o
  __device__ __forceinline__ void put_sums(float* ms, int apart) {
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      float sum = l[nt];
      sum += __shfl_xor(sum, 16);
      sum += __shfl_xor(sum, 32);
      if (sum != sum && m[nt] == -INFINITY) m[nt] = 0.f;  // (-infinity says that no row is seen)
      if (g == 0) {
        ms[nt * 16 + n] = m[nt];
        ms[apart + nt * 16 + n] = sum;
      }
    }
  }
  template <typename Top>
  __device__ __forceinline__ void put_o(float* os, int width, Top top) {
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      const float f = m[nt] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m[nt] - top(nt * 16 + n));
#pragma unroll
      for (int dt = 0; dt < DT; ++dt)
        *(f32x4*)(os + (nt * 16 + n) * width + 16 * dt + 4 * g) =
            m[nt] == -INFINITY ? (f32x4){0.f, 0.f, 0.f, 0.f} : o[nt][dt] * f;
    }
  }
};

template <typename T>
__device__ __forceinline__ void put4(T* p, f32x4 x) {
  if constexpr (sizeof(T) == 4) {
    *(f32x4*)p = x;
  } else {
    u32x2 y;
#pragma unroll
    for (int i = 0; i < 2; ++i)
      y[i] = (unsigned)__builtin_bit_cast(uint16_t, (__bf16)x[2 * i]) |
             (unsigned)__builtin_bit_cast(uint16_t, (__bf16)x[2 * i + 1]) << 16;
    *(u32x2*)p = y;
  }
}
// four dims of a query's attention from its sums (m, l, o)
template <typename T>
__device__ __forceinline__ void put_query(const Args& a, int b, int t, int h, int dim, f32x4 o, float m, float l) {
  const float by = l == 0.f ? 0.f : 1.f / l;
  put4((T*)a.out + b * a.d.out_seq + t * a.d.out_row + h * a.d.out_head + dim, l == 0.f ? (f32x4){0.f, 0.f, 0.f, 0.f} : o * by);
  if (a.lse && dim == 0)
    a.lse[((int64_t)b * a.d.n_query + t) * a.d.n_head + h] =
        l == 0.f ? -INFINITY : (m + (__builtin_amdgcn_logf(l) - (sizeof(T) == 4 ? kUp : 0.f))) * 0.6931471805599453f;
}

// The cached rows that a sequence's queries can see: columns [0, sinks) and those from `from` on of its table, in all
// `count` parts of 32 rows.  (page_rows is 32 << shift.)
struct Seen {
  int sinks, from, count;
  __device__ __forceinline__ Seen(const Args& a, int len, int shift) : sinks(0), from(0) {
    const int pages = min(max(len, 0) >> (5 + shift), a.n_col);
    if (a.d.window) {
      const int rows = 32 << shift;
      sinks = min((min(a.d.sinks, pages << (5 + shift)) + rows - 1) >> (5 + shift), pages);
      from = min(max(max(len - a.d.window + 1, 0) >> (5 + shift), sinks), pages);
    }
    count = (sinks + pages - from) << shift;
  }
};

// Long sequences are cut by their own lengths: each into the nearest number of parts of an equal share of all rows
// (one at the least), parts of a head side by side, sequence by sequence.  So a batch of one long and many short
// ones fills the chip too.  (Every wave finds its part by itself: the lengths are in its lanes.)
// One sequence of 60,000 rows among 31 of about 1000, 20 heads of 64: 729 us in equal parts of the table, 55 so.
constexpr int kLeast = 24;  // 32 rows each of a part: six for each wave (16 x 1 query of 16 heads on 2 over 4000 rows 12.7 us, 13.8 with 16)
constexpr int kRound = 512;  // workgroups that sequences are cut for: two a CU (100,000 rows of one 48.2 us, 50.3 with 768)
// From this many 32 rows of a table's row on, sequences are cut by their own lengths: finding the part takes 2 us (32 sequences
// of 1500 rows of 20 heads of 64 take 30 in equal parts).  Below, equal parts, so the longest sequence sets the time: 31 of
// 1000 rows and one of 16,000 take 85 us, one of 17,000 cut by lengths 37, one of 8191 in equal parts 53.
constexpr int kLong = 512;
struct Part {
  int b, j, n;  // part j of n of sequence b,
  int at, kv;   // the at-th of all, in kv head kv
};
// sums over the lanes up to this one
__device__ __forceinline__ int scan(int x) {
  x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, false);  // 1, 2, 4, 8 lanes before, within 16
  x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false);  // the last of the 16 before, to every second 16
  x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false);  // lane 31, to the upper 32
  return x;
}
__device__ __forceinline__ int last(int x) { return __builtin_amdgcn_readlane(x, 63); }
// Part number p (SEQ: the first one of sequence p, and in kv the parts of a head); kv is n_kv_head or more where there is none.
template <bool SEQ>
__device__ __forceinline__ Part find_part(const Args& a, int p) {
  const int lane = threadIdx.x & 63, shift = a.page_rows >> 6;
  auto count = [&](int b0) { return b0 + lane < a.n_seq ? Seen(a, a.length[b0 + lane], shift).count : 0; };
  const int first = count(0);
  int sum = last(scan(first));
  for (int b0 = 64; b0 < a.n_seq; b0 += 64) sum += last(scan(count(b0)));
  const int share = max((sum * a.n_kv_head * a.tiles + a.round - 1) / a.round, kLeast);
  auto parts = [&](int b0) {
    const int n = b0 == 0 ? first : count(b0);
    return b0 + lane < a.n_seq ? max((n + (share >> 1)) / share, 1) : 0;
  };
  const int upto0 = scan(parts(0));
  int all = last(upto0);  // parts of a head
  for (int b0 = 64; b0 < a.n_seq; b0 += 64) all += last(scan(parts(b0)));
  Part x;
  x.kv = SEQ ? all : p / all;
  const int rest = SEQ ? 0 : p - x.kv * all;
  int before = 0;
  for (int b0 = 0; b0 < a.n_seq; b0 += 64) {
    const int upto = b0 == 0 ? upto0 : scan(parts(b0));
    // the lane whose sequence it is
    const unsigned long long hit = SEQ ? (p >= b0 && p < b0 + 64 ? 1ull << (p - b0) : 0ull)
                                       : __builtin_amdgcn_ballot_w64(before + upto > rest);
    if (hit) {
      const int s = __builtin_ctzll(hit), to = __builtin_amdgcn_readlane(upto, s);
      const int from = s ? __builtin_amdgcn_readlane(upto, s - 1) : 0;
      x.n = to - from;
      x.b = b0 + s;
      x.j = SEQ ? 0 : rest - before - from;
      x.at = SEQ ? before + from : p;
      return x;
    }
    before += last(upto);
  }
  x.kv = a.n_kv_head;
  return x;
}

// Items, 32 rows of pages each, go to the waves of a part of a sequence (and of its other parts) in turn: wave `me` of `all`
// has, but for the last `owners` waves, items me + k others for k < early, and then every wave each all-th one.  The last waves,
// as many as open and new rows can need, take those in place of their early items.  So which columns a wave looks at
// does not depend on the length (without a window or parts), and the table's entries are under way with it.
// What 32 rows in the model's type take, in 32 rows of pages (64 sequences of 512 rows, 20 heads of 64: 27.6 us, 31.5 with 3,
// 34.7 with 0).
constexpr int kOwnCost = 6;

// (Registers: the loads under way and the outputs.  The masks and the sign of a scale are kept out of the loop of items by
// empty statements: taken out of it by the compiler they made 200 bytes of spills, 163 us in place of 152 for heads of 128.)
template <typename W>
__global__ __launch_bounds__(64 * kWaves, W::DIM == 128 || W::COLS == 32 || W::F32 ? 2 : 3) void paged_attn_kernel(Args a) {
  typedef typename W::Type T;
  constexpr int D = W::DIM, COLS = W::COLS;
  extern __shared__ __align__(16) float lds[];
  // Blocks go round the XCDs: a part's tiles of queries run side by side on one of them, so that its pages are
  // read once into that L2, and the parts are spread evenly.
  const int xcd = blockIdx.x & 7, tile = blockIdx.x >> 3, unit = (blockIdx.z * gridDim.y + blockIdx.y) * 8 + xcd;
  int b, kv, split, splits, at;
  if (a.splits) {
    splits = a.splits;
    const int rest = unit / a.n_kv_head;
    kv = unit - rest * a.n_kv_head;
    split = splits == 1 ? 0 : rest / a.n_seq;
    b = rest - split * a.n_seq;
    if (split >= splits || b >= a.n_seq) return;
    at = (b * a.n_kv_head + kv) * splits + split;
  } else {
    const Part p = find_part<false>(a, unit);
    if (p.kv >= a.n_kv_head || p.at >= a.parts) return;
    b = __builtin_amdgcn_readfirstlane(p.b);
    kv = __builtin_amdgcn_readfirstlane(p.kv);
    split = __builtin_amdgcn_readfirstlane(p.j);
    splits = __builtin_amdgcn_readfirstlane(p.n);
    at = __builtin_amdgcn_readfirstlane(p.at);
  }
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int R0 = a.page_rows, shift = R0 >> 6, per = 1 << shift, all = splits * kWaves, me = split * kWaves + wave;
  const int owners = min(a.owners, all), others = all - owners, early = others > 0 ? kOwnCost : 0;
  const bool owner = me >= others;
  const int item0 = owner ? early * others + me : me, slow = owner ? 0 : early;
  auto item = [&](int k) { return item0 + min(k, slow) * others + max(k - slow, 0) * all; };  // the k-th of this wave
  const int* table = a.table + b * a.table_ld;
  int entry = -1;
  if (a.d.window == 0) {
    const int c = item(lane) >> shift;
    if (c < a.n_col) entry = table[c];
  }
  W w(a);
  w.issue(b, kv, tile);
  const int len = a.length[b];
  if (len < 0) {
    w.begin(0);
  } else {
    const int start = len & -R0, tail = len - start;
    const Seen look(a, len, shift);
    const int sinks = look.sinks, from = look.from, count = look.count;
    const int first_full = a.d.window ? len + a.d.n_query - a.d.window : 0;  // all queries see rows from here on
    // lane j, of item k0 + j of this wave's: its page, the page's scales, where its bytes begin and its first row's position
    int page = -1, first = 0;
    float2 sc = {0.f, 0.f};
    int64_t bytes = 0;
    auto find = [&](int k0) {
      const int i = item(k0 + lane), v = i >> shift, c = v < sinks ? v : v - sinks + from, row = 32 * (i & (per - 1));
      page = a.d.window == 0 && k0 == 0 ? entry : i < count ? table[c] : -1;
      if (i >= count || (unsigned)page >= (unsigned)a.n_page) page = -1;
      const int64_t block = (int64_t)max(page, 0) * a.n_kv_head + kv;  // (without one: page 0, for all waves the same)
      sc = a.scale[block];
      bytes = block * (2 * R0 * D) + row * D;
      first = c * R0 + row;
    };
    find(0);
    w.begin(len);
    const int owns = (tail + a.d.n_query + 31) >> 5;
    if (owner && all - 1 - me < owns) {
      const int slot = start % a.d.tail_rows;
      typename W::Own rows;
      for (int j = all - 1 - me; j < owns; j += owners) {
        w.issue_own(rows, b, kv, 32 * j, tail, slot);
        w.take_own(rows, b, kv, 32 * j, tail, start, slot);
      }
    }
    w.split();
    const int soon = slow * others, rest = count - item0;
    const int items = rest <= 0 ? 0 : rest <= soon ? (rest + others - 1) / others : slow + (rest - soon + all - 1) / all;
    for (int k0 = 0; k0 < items; k0 += 64) {
      if (k0) find(k0);
      auto fetch = [&](Codes<D>& x, int k) {
        const int j = min(k - k0, 63);
        const uint8_t* block = a.data + ((uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)bytes, j) |
                                         (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(bytes >> 32), j) << 32);
        x.load(block, block + R0 * D, lane);
      };
      auto work = [&](const Codes<D>& x, int k) {
        const int j = k - k0;
        if (__builtin_amdgcn_readlane(page, j) < 0) return;
        const float ks = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(sc.x), j));
        const float vs = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(sc.y), j));
        const int at = __builtin_amdgcn_readlane(first, j);
        w.take(x, ks, vs, at, at < first_full && at + 32 > a.d.sinks);
      };
      // Loads run ST - 1 items ahead, past the last item, too: were they under a condition, the compiler would have to
      // wait as if they had not been issued, for those of the next items with the item's own.
      constexpr int ST = 2;
      Codes<D> x[ST];
#pragma unroll
      for (int u = 0; u < ST - 1; ++u) fetch(x[u], k0 + u);
      sc.x = W::finite(sc.x) ? sc.x : __builtin_nanf("");  // (infinity times a code is infinity or NaN: all of the page is NaN)
      sc.y = W::finite(sc.y) ? sc.y : __builtin_nanf("");
      if (__builtin_amdgcn_ballot_w64(page >= 0 && W::large(sc.y, kLargeScale))) w.lift = kLift;
      const int end = min(k0 + 64, items);
      for (int k = k0; k < end; k += ST)
#pragma unroll
        for (int u = 0; u < ST; ++u) {
          fetch(x[(u + ST - 1) % ST], k + u + ST - 1);
          if (k + u < end) work(x[u], k + u);
        }
    }
  }

  // the waves' sums, joined
  constexpr int WIDTH = D + 4;          // (columns 16 bytes apart in the banks)
  float* ms = lds;                      // [wave][column] m, then l
  float* os = lds + 2 * kWaves * COLS;  // [wave][column][dim]
  w.put_sums(ms + wave * COLS, kWaves * COLS);
  __syncthreads();
  auto top_of = [&](int col) {
    float top = -INFINITY;
#pragma unroll
    for (int v = 0; v < kWaves; ++v) top = fmaxf(top, ms[v * COLS + col]);
    return top;
  };
  w.put_o(os + wave * COLS * WIDTH, WIDTH, top_of);
  __syncthreads();
  const int group = a.d.n_head / a.n_kv_head, cols = a.d.n_query * group;
  for (int x = threadIdx.x; x < COLS * (D / 4); x += 64 * kWaves) {
    const int col = x / (D / 4), dim = 4 * (x % (D / 4)), c = tile * COLS + col;
    if (c >= cols) break;
    const float top = top_of(col);
    float l = 0.f;
    f32x4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int v = 0; v < kWaves; ++v) {
      const float m = ms[v * COLS + col];
      if (m != -INFINITY) l += ms[(kWaves + v) * COLS + col] * __builtin_amdgcn_exp2f(m - top);
      o += *(const f32x4*)(os + (v * COLS + col) * WIDTH + dim);
    }
    const int t = group == 1 ? c : c / group, h = kv * group + c - t * group;
    if (splits == 1) {
      put_query<T>(a, b, t, h, dim, o, top, l);
    } else {
      const int64_t place = ((int64_t)at * a.tiles + tile) * COLS + col;
      *(f32x4*)(a.o + place * D + dim) = o;
      if (dim == 0) a.ml[place] = make_float2(top, l);
    }
  }
}

// A wave per query adds its parts, out = sum 2^(m_c - M) o_c / sum 2^(m_c - M) l_c, reading all at once; parts are added
// in their order, so results do not depend on which ended first.  Bound: latency, 4 us for 7 parts of 640 queries.
// Lane l has dims 4 (l mod (D / 4)) .. + 3 of every (256 / D)-th.
template <typename T, int D>
__global__ __launch_bounds__(256) void join_kernel(Args a) {
  constexpr int LD = D / 4, PAR = 64 / LD;
  const int lane = threadIdx.x & 63, x = lane % LD, b = blockIdx.y;
  const int query = blockIdx.x * 4 + (threadIdx.x >> 6), t = query / a.d.n_head, h = query - t * a.d.n_head;
  const int group = a.d.n_head / a.n_kv_head, kv = h / group, c = t * group + h - kv * group;
  int n = a.splits, part = (b * a.n_kv_head + kv) * n;
  if (n == 0) {
    const Part p = find_part<true>(a, b);
    n = p.n;
    part = kv * p.kv + p.at;
    if (n == 1) return;
  }
  if (t >= a.d.n_query) return;
  const int64_t step = (int64_t)a.tiles * a.cols, at = part * step + c;
  const float2* ml = a.ml + at;
  const float* po = a.o + at * D + 4 * x;
  float top = -INFINITY, l = 0.f;
  f32x4 o = {0.f, 0.f, 0.f, 0.f};
  for (int i = lane / LD; i < n; i += PAR) {
    const float2 q = ml[i * step];
    const f32x4 y = *(const f32x4*)(po + i * step * D);
    const float now = fmaxf(top, q.x);
    const float f = top == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(top - now);
    const float d = q.x == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(q.x - now);
    o = o * f + (q.x == -INFINITY ? (f32x4){0.f, 0.f, 0.f, 0.f} : y * d);
    l = l * f + (q.x == -INFINITY ? 0.f : q.y * d);
    top = now;
  }
  float all = top;
#pragma unroll
  for (int s = 32; s >= LD; s >>= 1) all = fmaxf(all, __shfl_xor(all, s));
  const float f = top == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(top - all);
  o *= f;
  l *= f;
#pragma unroll
  for (int s = 32; s >= LD; s >>= 1) {
    l += __shfl_xor(l, s);
#pragma unroll
    for (int i = 0; i < 4; ++i) o[i] += __shfl_xor(o[i], s);
  }
  if (lane < LD) put_query<T>(a, b, t, h, 4 * x, o, all, l);
}

// ---------------------------------------------------------------- host

struct Plan {
  int cols, tiles, splits, round;  // queries of a workgroup, workgroups of a sequence's and head's queries; see Args
  int64_t parts, blocks;           // parts that there can be, workgroups
  size_t o_bytes, bytes;
};
int64_t div_up(int64_t a, int64_t b) { return (a + b - 1) / b; }

Plan plan(const ssd_page_pool& p, const ssd_page_seqs& s, const ssd_paged_attn_desc& d) {
  Plan x{};
  const int64_t cols = (int64_t)d.n_query * (d.n_head / p.n_kv_head);
  x.cols = cols > 16 && !(d.dtype == SSD_F32 && p.head_dim == 128) ? 32 : 16;  // (what the registers hold)
  x.tiles = (int)div_up(cols, x.cols);
  int64_t pages = s.n_col;
  if (d.window)
    pages = std::min<int64_t>(pages, div_up(std::min<int64_t>(d.sinks, 1 << 30), p.page_rows) + d.window / p.page_rows + 2);
  const int64_t units = (int64_t)s.n_seq * p.n_kv_head * x.tiles, steps = pages * (p.page_rows / 32);
  const int64_t heads = (int64_t)s.n_seq * p.n_kv_head;
  // (numbers of 32 rows of all queries are 32-bit where the device counts them)
  if (s.n_seq > 1 && steps > kLong && units * steps < (1 << 30)) {
    x.round = kRound;
    x.parts = div_up(heads + div_up(kRound, x.tiles), 8) * 8;
  } else {
    x.splits = (int)std::max<int64_t>(1, std::min<int64_t>(kRound / units, div_up(steps, kLeast)));
    x.parts = div_up(heads * x.splits, 8) * 8;
  }
  x.blocks = x.parts * x.tiles;
  if (x.splits == 1) return x;
  x.o_bytes = (size_t)x.parts * x.tiles * x.cols * p.head_dim * 4;
  x.bytes = x.o_bytes + (size_t)x.parts * x.tiles * x.cols * sizeof(float2);
  return x;
}

template <typename W>
hipError_t launch(const Args& a, const Plan& p, hipStream_t s) {
  constexpr int lds = (2 * kWaves * W::COLS + kWaves * W::COLS * (W::DIM + 4)) * 4;
  if constexpr (lds > 65536) {  // has to be asked for, once per kernel and device
    static std::atomic<uint64_t> ready{0};
    int dev = 0;
    hipError_t e = hipGetDevice(&dev);
    if (e != hipSuccess) return e;
    const uint64_t bit = dev < 64 ? 1ull << dev : 0;
    if (!(ready.load(std::memory_order_acquire) & bit)) {
      e = hipFuncSetAttribute((const void*)paged_attn_kernel<W>, hipFuncAttributeMaxDynamicSharedMemorySize, lds);
      if (e != hipSuccess) return e;
      ready.fetch_or(bit, std::memory_order_release);
    }
  }
  const int64_t rows = 32768;  // (of a grid's dimensions, 65535 at the most)
  const dim3 grid(8 * p.tiles, (unsigned)std::min(p.parts / 8, rows), (unsigned)div_up(p.parts / 8, rows));
  paged_attn_kernel<W><<<grid, 64 * kWaves, lds, s>>>(a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || p.splits == 1) return e;
  join_kernel<typename W::Type, W::DIM><<<dim3((a.d.n_query * a.d.n_head + 3) / 4, a.n_seq), 256, 0, s>>>(a);
  return hipGetLastError();
}
template <typename T, int D, int CODE>
hipError_t launch(const Args& a, const Plan& p, hipStream_t s) {
  if constexpr (!(sizeof(T) == 4 && D == 128))
    if (p.cols == 32) return launch<Tiles<T, D, CODE, 2>>(a, p, s);
  return launch<Tiles<T, D, CODE, 1>>(a, p, s);
}
template <typename T, int D>
hipError_t launch(const Args& a, const Plan& p, int code, hipStream_t s) {
  return code == SSD_PAGE_INT8 ? launch<T, D, SSD_PAGE_INT8>(a, p, s) : launch<T, D, SSD_PAGE_E4M3>(a, p, s);
}
template <typename T>
hipError_t launch(const Args& a, const Plan& p, int d, int code, hipStream_t s) {
  return d == 32 ? launch<T, 32>(a, p, code, s) : d == 64 ? launch<T, 64>(a, p, code, s) : launch<T, 128>(a, p, code, s);
}

constexpr int64_t kMostBlocks = (1 << 24) - 1;  // a grid holds fewer than 2^32 threads

ssd_status check(const ssd_page_pool* pool, const ssd_page_seqs* seqs, const ssd_paged_attn_desc* a) {
  ssd_status st = check_pool(pool);
  if (st == SSD_OK) st = check_seqs(seqs, pool->page_rows, false);
  if (st != SSD_OK) return st;
  OP_REQUIRE(a, SSD_E_INVALID_ARG, "null argument");
  OP_REQUIRE(op_dtype(a->dtype), SSD_E_INVALID_ARG, "dtype must be SSD_F32 or SSD_BF16");
  OP_REQUIRE(a->layer >= 0 && a->layer < pool->n_layer, SSD_E_INVALID_ARG, "layer outside the pool's");
  OP_REQUIRE(a->n_query >= 1 && a->n_query <= 64, SSD_E_INVALID_ARG, "n_query outside [1, 64]");
  OP_REQUIRE(a->n_head >= pool->n_kv_head && a->n_head <= 1024 && a->n_head % pool->n_kv_head == 0, SSD_E_INVALID_ARG,
             "n_head must be a multiple of n_kv_head, at most 1024");
  OP_REQUIRE(a->tail_rows >= pool->page_rows && a->tail_rows < (1 << 30), SSD_E_INVALID_ARG,
             "tail_rows below page_rows, or 2^30");
  OP_REQUIRE(a->window >= 0 && a->sinks >= 0 && (a->window == 0 || a->window >= a->n_query), SSD_E_INVALID_ARG,
             "window or sinks is negative, or the window is shorter than n_query");
  OP_REQUIRE(isfinite(a->scale * 1.4426950408889634f), SSD_E_INVALID_ARG,
             "scale, and scale times log2 e, must be finite");
  return SSD_OK;
}

}  // namespace
}  // namespace ssd

using namespace ssd;

extern "C" ssd_status ssd_paged_attn_workspace(const ssd_page_pool* pool, const ssd_page_seqs* seqs,
                                               const ssd_paged_attn_desc* a, size_t* bytes) {
  OP_REQUIRE(bytes, SSD_E_INVALID_ARG, "null argument");
  const ssd_status st = check(pool, seqs, a);
  if (st != SSD_OK) return st;
  const Plan p = plan(*pool, *seqs, *a);
  OP_REQUIRE(p.blocks <= kMostBlocks, SSD_E_CAPACITY, "more workgroups than a grid holds");
  *bytes = p.bytes;
  return SSD_OK;
}

extern "C" ssd_status ssd_paged_attn(const ssd_page_pool* pool, const ssd_page_seqs* seqs, const ssd_paged_attn_desc* a,
                                     const void* q, const void* k_tail, const void* v_tail, const void* k_new,
                                     const void* v_new, const int64_t* anc, void* out, float* lse, void* workspace,
                                     size_t workspace_bytes, void* stream) {
  size_t need = 0;
  ssd_status st = ssd_paged_attn_workspace(pool, seqs, a, &need);
  if (st != SSD_OK) return st;
  const int G = pool->n_kv_head, D = pool->head_dim, es = op_size(a->dtype);
  const RowDim qd[4] = {{1, 0}, {seqs->n_seq, a->q_seq}, {a->n_query, a->q_row}, {a->n_head, a->q_head}};
  const RowDim od[4] = {{1, 0}, {seqs->n_seq, a->out_seq}, {a->n_query, a->out_row}, {a->n_head, a->out_head}};
  const RowDim td[4] = {{1, 0}, {seqs->n_seq, a->tail_seq}, {G, a->tail_head}, {a->tail_rows, a->tail_row}};
  const RowDim nd[4] = {{1, 0}, {seqs->n_seq, a->new_seq}, {a->n_query, a->new_row}, {G, a->new_head}};
  st = check_rows(a->dtype, qd, D, false, q, q);
  if (st == SSD_OK) st = check_rows(a->dtype, od, D, true, out, out);
  if (st == SSD_OK) st = check_rows(a->dtype, td, D, false, k_tail, v_tail);
  if (st == SSD_OK) st = check_rows(a->dtype, nd, D, false, k_new, v_new);
  if (st != SSD_OK) return st;
  OP_REQUIRE((uintptr_t)anc % 8 == 0 && (uintptr_t)lse % 4 == 0, SSD_E_INVALID_ARG, "anc or lse is not aligned");
  auto view = [&](const void* p, const RowDim(&d)[4]) {
    return OpView{p, {{d[1].n, d[1].step * es}, {d[2].n, d[2].step * es}, {d[3].n, d[3].step * es}, {D, es}}};
  };
  const OpView o = view(out, od);
  for (const OpView& in : {view(q, qd), view(k_tail, td), view(v_tail, td), view(k_new, nd), view(v_new, nd)})
    OP_REQUIRE(op_apart(o, in), SSD_E_INVALID_ARG, "out overlaps an input");
  OP_REQUIRE(workspace || need == 0, SSD_E_INVALID_ARG, "null workspace");
  OP_REQUIRE(workspace_bytes >= need && (uintptr_t)workspace % 16 == 0, SSD_E_CAPACITY,
             "workspace below ssd_paged_attn_workspace's bytes or not 16-byte aligned");
  const Plan p = plan(*pool, *seqs, *a);
  Args x{};
  x.d = *a;
  const int64_t blocks = (int64_t)a->layer * pool->n_page * G;
  x.data = (const uint8_t*)pool->data + blocks * 2 * block_bytes(*pool);
  x.scale = (const float2*)pool->scale + blocks;
  x.table = seqs->table;
  x.length = seqs->length;
  x.table_ld = seqs->table_ld;
  x.n_seq = seqs->n_seq;
  x.n_col = seqs->n_col;
  x.n_page = pool->n_page;
  x.n_kv_head = G;
  x.page_rows = pool->page_rows;
  x.q = (const char*)q;
  x.kt = (const char*)k_tail;
  x.vt = (const char*)v_tail;
  x.kn = (const char*)k_new;
  x.vn = (const char*)v_new;
  x.anc = anc;
  x.out = (char*)out;
  x.lse = lse;
  x.o = (float*)workspace;
  x.ml = (float2*)((char*)workspace + p.o_bytes);
  x.tiles = p.tiles;
  x.cols = p.cols;
  x.splits = p.splits;
  x.round = p.round;
  x.parts = (int)p.parts;
  x.owners = (pool->page_rows - 1 + a->n_query + 31) / 32;
  x.scale2 = a->scale * 1.4426950408889634f;
  const hipError_t e = a->dtype == SSD_F32 ? launch<float>(x, p, D, pool->code, (hipStream_t)stream)
                                           : launch<bf16_t>(x, p, D, pool->code, (hipStream_t)stream);
  if (e != hipSuccess) return op_fail(SSD_E_DEVICE, hipGetErrorString(e));
  return SSD_OK;
}
