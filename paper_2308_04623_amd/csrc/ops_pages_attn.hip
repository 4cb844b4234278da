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
// 4 bits), and their scales multiply scores and weights:
//   x = (code_k . q) scale_k scale,   o += code_v (2^(x - m) scale_v),
// the weights' factor scale_v relative to a power of two that the wave's result is multiplied by at the end.
// Queries are scaled by a power of two each, to the middle of float16's range, and split into
// parts of 11 bits: bfloat16's 8 bits are one, float32's 24 three.
#include <algorithm>
#include <atomic>

#include "ops_pages.h"

namespace ssd {
namespace {

typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

constexpr int kWaves = 4;
constexpr float kSlack = 8.f;  // how far a score may lie above the reference before the sums are rescaled

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
  float* o;    // [query][splits][head_dim], query = (sequence, new row, head)
  float2* ml;  // [query][splits] (m, l)
  int tiles, splits;
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
__device__ __forceinline__ float group_max(float x) {  // over the lanes of a column
  x = fmaxf(x, __shfl_xor(x, 16));
  return fmaxf(x, __shfl_xor(x, 32));
}

// a block's bytes of 32 rows: of keys and of values, 16 a lane each
template <int D>
struct Codes {
  u32x4 k[D / 32], v[D / 32];
  __device__ __forceinline__ void load(const uint8_t* keys, const uint8_t* values, int lane) {
#pragma unroll
    for (int i = 0; i < D / 32; ++i) k[i] = *(const u32x4*)(keys + 1024 * i + 16 * lane);
#pragma unroll
    for (int i = 0; i < D / 32; ++i) v[i] = *(const u32x4*)(values + 1024 * i + 16 * lane);
  }
};

// A wave's queries and results.  Lane 16 g + n has column n of every tile: of scores the rows 4 g + r
// of 16, of outputs the dims 4 g + r of 16.
template <typename T, int D, int CODE, int NT>
struct Wave {
  static constexpr bool F32 = sizeof(T) == 4;
  static constexpr int NQ = F32 ? 3 : 1, NP = F32 ? 2 : 1, KS = D / 32, DT = D / 16;
  const Args& a;
  const int lane, g, n;
  f16x8 q[NT][KS][NQ];
  float unit[NT];   // of a product of queries and codes: scale2 and the query's power of two
  f32x4 o[NT][DT];
  float m[NT], sub[NT], l[NT];  // reference, what is subtracted (0 for -infinity), this lane's share of the sum
  float vunit;                  // o is in units of this power of two
  int seen_from[NT];            // cached rows from here on, and sinks, are seen
  uint64_t anc[NT];             // new rows that are seen
  int64_t at[NT];               // the query's first element, -1: none

  __device__ __forceinline__ Wave(const Args& args)
      : a(args), lane(threadIdx.x & 63), g(lane >> 4), n(lane & 15), vunit(0.f) {}

  // the 8 dims from here on are what the lane has in step s of a product over dims
  __device__ __forceinline__ int dim_at(int s) const { return D == 32 ? 8 * g : 64 * (s >> 1) + 16 * g + 8 * (s & 1); }

  __device__ __forceinline__ void load(int b, int kv, int tile, int len) {
    const int group = a.d.n_head / a.n_kv_head, cols = a.d.n_query * group;
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      const int c = (tile * NT + nt) * 16 + n, t = c / group;
      const bool live = c < cols;
      at[nt] = live ? b * a.d.q_seq + t * a.d.q_row + (kv * group + c % group) * a.d.q_head : -1;
      float x[KS][8], top = 0.f;
#pragma unroll
      for (int s = 0; s < KS; ++s) {
        const T* p = (const T*)a.q + (live ? at[nt] : 0) + dim_at(s);
        if constexpr (F32) {
          const f32x4 u = *(const f32x4*)p, v = *(const f32x4*)(p + 4);
#pragma unroll
          for (int i = 0; i < 4; ++i) x[s][i] = u[i], x[s][4 + i] = v[i];
        } else {
          const u32x4 u = *(const u32x4*)p;
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            x[s][2 * i] = __uint_as_float(u[i] << 16);
            x[s][2 * i + 1] = __uint_as_float(u[i] & 0xffff0000u);
          }
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) top = fmaxf(top, fabsf(x[s][i]));
      }
      top = group_max(top);
      // the largest to [2^14, 2^15): what is smaller by up to 2^28 keeps its 11 bits
      const int e = top < __builtin_inff() ? max((int)(__float_as_uint(top) >> 23) - 127, -100) : 14;
      const float by = __uint_as_float((unsigned)(min(14 - e, 127) + 127) << 23);
      unit[nt] = a.scale2 * __uint_as_float((unsigned)(max(e - 14, -126) + 127) << 23);
#pragma unroll
      for (int s = 0; s < KS; ++s)
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          float y = live ? x[s][i] * by : 0.f;
#pragma unroll
          for (int p = 0; p < NQ; ++p) {
            q[nt][s][p][i] = (_Float16)y;
            y -= (float)q[nt][s][p][i];
          }
        }
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) o[nt][dt] = (f32x4){0.f, 0.f, 0.f, 0.f};
      m[nt] = -INFINITY;
      sub[nt] = l[nt] = 0.f;
      anc[nt] = t >= 63 ? ~0ull : (2ull << t) - 1;
      if (a.anc && live) anc[nt] = (uint64_t)a.anc[(int64_t)b * a.d.n_query + t] & (~0ull >> (64 - a.d.n_query));
      const int depth = a.anc ? max(__popcll(anc[nt]) - 1, 0) : t;
      seen_from[nt] = a.d.window ? len + depth - a.d.window + 1 : 0;
    }
  }

  // x = s unit, masked, in the reference's units; sums rescaled where a score is far above it
  template <typename Seen>
  __device__ __forceinline__ void weights(f32x4 (&s)[NT][2], const float (&by)[NT], bool masked, Seen seen) {
#pragma clang fp contract(off)
    bool far = false;
    float top[NT];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
      for (int k = 0; k < 2; ++k) s[nt][k] *= by[nt];
      if (masked) {
#pragma unroll
        for (int k = 0; k < 2; ++k)
#pragma unroll
          for (int r = 0; r < 4; ++r)
            if (!seen(nt, 16 * k + 4 * g + r)) s[nt][k][r] = -INFINITY;
      }
      top[nt] = fmaxf(fmaxf(fmaxf(s[nt][0][0], s[nt][0][1]), fmaxf(s[nt][0][2], s[nt][0][3])),
                      fmaxf(fmaxf(s[nt][1][0], s[nt][1][1]), fmaxf(s[nt][1][2], s[nt][1][3])));
      far |= top[nt] > m[nt] + kSlack;
    }
    if (__builtin_amdgcn_ballot_w64(far)) {
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        const float now = fmaxf(m[nt], group_max(top[nt]));
        const float by = m[nt] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m[nt] - now);
        m[nt] = now;
        sub[nt] = now == -INFINITY ? 0.f : now;
        l[nt] *= by;
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) o[nt][dt] *= by;
      }
    }
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
      for (int k = 0; k < 2; ++k)
#pragma unroll
        for (int r = 0; r < 4; ++r) s[nt][k][r] = __builtin_amdgcn_exp2f(s[nt][k][r] - sub[nt]);
      l[nt] += ((s[nt][0][0] + s[nt][0][1]) + (s[nt][0][2] + s[nt][0][3])) +
               ((s[nt][1][0] + s[nt][1][1]) + (s[nt][1][2] + s[nt][1][3]));
    }
  }

  // 32 rows of a page; first: the position of the first; rows: their number that count
  __device__ __forceinline__ void take(const Codes<D>& c, float kscale, float vscale, int first, bool masked) {
    f32x4 s[NT][2];
#pragma unroll
    for (int k = 0; k < 2; ++k)
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) s[nt][k] = (f32x4){0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int k = 0; k < 2; ++k)
#pragma unroll
      for (int st = 0; st < KS; ++st) {
        // (bytes of step st of rows 16 k ..: see the order of keys)
        const int i = D == 32 ? 0 : k * (D / 64) + (st >> 1), h = D == 32 ? k : st & 1;
        const f16x8 x = codes8<CODE>(c.k[i][2 * h], c.k[i][2 * h + 1]);
#pragma unroll
        for (int p = NQ - 1; p >= 0; --p)
#pragma unroll
          for (int nt = 0; nt < NT; ++nt) s[nt][k] = product(x, q[nt][st][p], s[nt][k]);
      }
    complete<2 * NT>(&s[0][0]);
    float by[NT];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) by[nt] = kscale * unit[nt];
    const int sinks = a.d.sinks;
    weights(s, by, masked, [&](int nt, int j) { return first + j >= seen_from[nt] || first + j < sinks; });
    // weights in units of the values' scale, and up to 2^15: float16 holds them to 2^-32 of the largest there can be
    const float size = fabsf(vscale);
    if (size > vunit * 0x1p7f && size < __builtin_inff()) {
      const unsigned up = (__float_as_uint(size) + 0x7fffffu) & 0x7f800000u;  // the next power of two
      const float now = fmaxf(fminf(__uint_as_float(up), 0x1p127f) * 0x1p-7f, 0x1p-126f);
      const float f = vunit / now;
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) o[nt][dt] *= f;
      vunit = now;
    }
    const float rel = vunit > 0.f ? vscale / vunit : vscale;
    f16x8 w[NT][NP];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        float y = s[nt][i >> 2][i & 3] * rel;
        if (masked) y = s[nt][i >> 2][i & 3] == 0.f ? 0.f : y;  // (whatever the scale)
#pragma unroll
        for (int p = 0; p < NP; ++p) {
          w[nt][p][i] = (_Float16)y;
          y -= (float)w[nt][p][i];
        }
      }
#pragma unroll
    for (int i = 0; i < D / 32; ++i)
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const f16x8 x = codes8<CODE>(c.v[i][2 * u], c.v[i][2 * u + 1]);
#pragma unroll
        for (int p = NP - 1; p >= 0; --p)
#pragma unroll
          for (int nt = 0; nt < NT; ++nt) o[nt][2 * i + u] = product(x, w[nt][p], o[nt][2 * i + u]);
      }
  }

  // 32 rows in the model's type, those from x on of `tail` open rows and the new ones behind them
  __device__ __forceinline__ void take_own(int b, int kv, int x0, int tail, int start) {
    const int total = tail + a.d.n_query;
    const int64_t told = b * a.d.tail_seq + kv * a.d.tail_head, tnew = b * a.d.new_seq + kv * a.d.new_head;
    auto row = [&](const char* old, const char* add, int x) {
      x = min(x, total - 1);
      return x < tail ? (const T*)old + told + (start + x) % a.d.tail_rows * a.d.tail_row
                      : (const T*)add + tnew + (x - tail) * a.d.new_row;
    };
    f32x4 s[NT][2];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) s[nt][0] = s[nt][1] = (f32x4){0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const T* p = row(a.kt, a.kn, x0 + 16 * k + n);
      if constexpr (F32) {
        // step i of the products has dims g (D / 4) + i
#pragma unroll
        for (int i = 0; i < D / 16; ++i) {
          const f32x4 y = *(const f32x4*)(p + g * (D / 4) + 4 * i);
#pragma unroll
          for (int nt = 0; nt < NT; ++nt) {
            const f32x4 z = *(const f32x4*)((const T*)a.q + max(at[nt], (int64_t)0) + g * (D / 4) + 4 * i);
#pragma unroll
            for (int j = 0; j < 4; ++j) s[nt][k] = product(y[j], z[j], s[nt][k]);
          }
        }
      } else {
#pragma unroll
        for (int i = 0; i < KS; ++i) {
          const bf16x8 y = __builtin_bit_cast(bf16x8, *(const u32x4*)(p + dim_at(i)));
#pragma unroll
          for (int nt = 0; nt < NT; ++nt) {
            const bf16x8 z =
                __builtin_bit_cast(bf16x8, *(const u32x4*)((const T*)a.q + max(at[nt], (int64_t)0) + dim_at(i)));
            s[nt][k] = product(y, z, s[nt][k]);
          }
        }
      }
    }
    complete<2 * NT>(&s[0][0]);
    float by[NT];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) by[nt] = a.scale2;
    const int sinks = a.d.sinks;
    unsigned bits[NT];  // which of the lane's 8 rows are seen
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      bits[nt] = 0;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int x = x0 + 16 * (i >> 2) + 4 * g + (i & 3), pos = start + x, step = x - tail;
        const bool old = x < tail && (pos >= seen_from[nt] || pos < sinks);
        const bool add = x >= tail && x < total && (anc[nt] >> (step & 63) & 1);
        bits[nt] |= (old || add) ? 1u << i : 0u;
      }
    }
    weights(s, by, true, [&](int nt, int j) { return (bits[nt] >> ((j >> 4) * 4 + (j & 3)) & 1) != 0; });
    const T* rows[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) rows[i] = row(a.vt, a.vn, x0 + 16 * (i >> 2) + 4 * g + (i & 3)) + n;
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) {
      // values that are not finite are taken out of the product, and make NaN where they are seen
      bool odd = false;
      unsigned odds = 0;
      if constexpr (F32) {
        float y[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          y[i] = rows[i][16 * dt];
          const bool bad = !(fabsf(y[i]) < __builtin_inff());
          odds |= bad ? 1u << i : 0u;
          y[i] = bad ? 0.f : y[i];
        }
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int i = 0; i < 8; ++i) o[nt][dt] = product(y[i], s[nt][i >> 2][i & 3], o[nt][dt]);
      } else {
        bf16x8 y;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          unsigned v = rows[i][16 * dt].bits;
          const bool bad = (v & 0x7f80u) == 0x7f80u;
          odds |= bad ? 1u << i : 0u;
          y[i] = __builtin_bit_cast(__bf16, (uint16_t)(bad ? 0 : v));
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
          o[nt][dt] = product(y, lo, o[nt][dt]);
          o[nt][dt] = product(y, hi, o[nt][dt]);
        }
      }
      odd = odds != 0;
      if (__builtin_amdgcn_ballot_w64(odd)) {
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
          bf16x8 y, z;
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            y[i] = (__bf16)(odds >> i & 1 ? 1.f : 0.f);
            z[i] = (__bf16)(bits[nt] >> i & 1 ? 1.f : 0.f);
          }
          f32x4 count = product(y, z, (f32x4){0.f, 0.f, 0.f, 0.f});
          complete<1>(&count);
          complete<1>(&o[nt][dt]);
#pragma unroll
          for (int r = 0; r < 4; ++r) o[nt][dt][r] = count[r] > 0.f ? __builtin_nanf("") : o[nt][dt][r];
        }
      }
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
        l == 0.f ? -INFINITY : (m + __builtin_amdgcn_logf(l)) * 0.6931471805599453f;
}

template <typename T, int D, int CODE, int NT>
__global__ __launch_bounds__(64 * kWaves, 2) void paged_attn_kernel(Args a) {
  extern __shared__ __align__(16) float lds[];
  // the sequences' workgroups of one head and part run side by side on one XCD (blocks go round
  // the XCDs): pages that they share are in its L2
  const int xcd = blockIdx.x & 7;
  int i = blockIdx.x >> 3;
  const int tile = i % a.tiles;
  i /= a.tiles;
  const int b = i % a.n_seq, hs = (i / a.n_seq) * 8 + xcd;
  if (hs >= a.n_kv_head * a.splits) return;
  const int kv = hs % a.n_kv_head, split = hs / a.n_kv_head;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int len = a.length[b], R0 = a.page_rows;

  Wave<T, D, CODE, NT> w(a);
  w.load(b, kv, tile, len);
  if (len >= 0) {
    const int pages = min(len / R0, a.n_col), start = len / R0 * R0;
    // columns [0, sinks) and [from, pages) are looked at, in parts of 32 rows
    int sinks = 0, from = 0, first_full = 0;
    if (a.d.window) {
      sinks = min((min(a.d.sinks, pages * R0) + R0 - 1) / R0, pages);
      from = min(max(max(len - a.d.window + 1, 0) / R0, sinks), pages);
      first_full = len + a.d.n_query - a.d.window;  // all queries see rows from here on
    }
    const int per = R0 / 32, count = (sinks + pages - from) * per, all = a.splits * kWaves, me = split * kWaves + wave;
    const int i0 = (int)((int64_t)count * me / all), i1 = (int)((int64_t)count * (me + 1) / all);
    const int64_t head_bytes = 2 * (int64_t)R0 * D;
    const int* table = a.table + b * a.table_ld;
    for (int p0 = i0 / per; p0 * per < i1; p0 += 64) {
      // lane j: the page of column p0 + j, and its scales
      int page = -1;
      float2 sc = {0.f, 0.f};
      {
        const int v = p0 + lane, c = v < sinks ? v : v - sinks + from;
        if (v * per < i1 && c < pages) page = table[c];
        if (page < 0 || page >= a.n_page) page = -1;
        else sc = a.scale[(int64_t)page * a.n_kv_head + kv];
      }
      const int lo = max(i0, p0 * per), hi = min(i1, (p0 + 64) * per);
      auto fetch = [&](Codes<D>& c, int i) {
        const int id = max(__builtin_amdgcn_readlane(page, i / per - p0), 0);
        const uint8_t* block = a.data + ((int64_t)id * a.n_kv_head + kv) * head_bytes + (i % per) * (32 * D);
        c.load(block, block + R0 * D, lane);
      };
      auto work = [&](const Codes<D>& c, int i) {
        const int j = i / per - p0;
        if (__builtin_amdgcn_readlane(page, j) < 0) return;
        const float ks = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(sc.x), j));
        const float vs = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(sc.y), j));
        const int v = i / per, col = v < sinks ? v : v - sinks + from, first = col * R0 + i % per * 32;
        w.take(c, ks, vs, first, first < first_full && first + 32 > a.d.sinks);
      };
      Codes<D> c0, c1;
      fetch(c0, lo);
      for (int i = lo; i < hi; i += 2) {
        if (i + 1 < hi) fetch(c1, i + 1);
        work(c0, i);
        if (i + 1 >= hi) break;
        if (i + 2 < hi) fetch(c0, i + 2);
        work(c1, i + 1);
      }
    }
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int dt = 0; dt < D / 16; ++dt) w.o[nt][dt] *= w.vunit;
    const int tail = len - start;
    for (int j = all - 1 - me; j * 32 < tail + a.d.n_query; j += all) w.take_own(b, kv, 32 * j, tail, start);
  }

  // the waves' sums, joined
  float* ms = lds;                         // [wave][column] m, then l
  float* os = lds + 2 * kWaves * 16 * NT;  // [wave][column][dim]
  constexpr int W = D + 4;                 // (columns 16 bytes apart in the banks)
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    float l = w.l[nt];
    l += __shfl_xor(l, 16);
    l += __shfl_xor(l, 32);
    if (l != l && w.m[nt] == -INFINITY) w.m[nt] = 0.f;  // (-infinity says that no row is seen)
    if (w.g == 0) {
      ms[wave * 16 * NT + nt * 16 + w.n] = w.m[nt];
      ms[(kWaves + wave) * 16 * NT + nt * 16 + w.n] = l;
    }
  }
  __syncthreads();
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    float top = -INFINITY;
#pragma unroll
    for (int v = 0; v < kWaves; ++v) top = fmaxf(top, ms[v * 16 * NT + nt * 16 + w.n]);
    const float by = w.m[nt] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(w.m[nt] - top);
#pragma unroll
    for (int dt = 0; dt < D / 16; ++dt)
      *(f32x4*)(os + (wave * 16 * NT + nt * 16 + w.n) * W + 16 * dt + 4 * w.g) =
          w.m[nt] == -INFINITY ? (f32x4){0.f, 0.f, 0.f, 0.f} : w.o[nt][dt] * by;
  }
  __syncthreads();
  const int group = a.d.n_head / a.n_kv_head, cols = a.d.n_query * group;
  for (int x = threadIdx.x; x < 16 * NT * (D / 4); x += 64 * kWaves) {
    const int col = x / (D / 4), dim = 4 * (x % (D / 4)), c = tile * NT * 16 + col;
    if (c >= cols) break;
    float top = -INFINITY, l = 0.f;
    f32x4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int v = 0; v < kWaves; ++v) top = fmaxf(top, ms[v * 16 * NT + col]);
#pragma unroll
    for (int v = 0; v < kWaves; ++v) {
      const float m = ms[v * 16 * NT + col];
      if (m != -INFINITY) l += ms[(kWaves + v) * 16 * NT + col] * __builtin_amdgcn_exp2f(m - top);
      o += *(const f32x4*)(os + (v * 16 * NT + col) * W + dim);
    }
    const int t = c / group, h = kv * group + c % group;
    if (a.splits == 1) {
      put_query<T>(a, b, t, h, dim, o, top, l);
    } else {
      const int64_t part = (((int64_t)b * a.d.n_query + t) * a.d.n_head + h) * a.splits + split;
      *(f32x4*)(a.o + part * D + dim) = o;
      if (dim == 0) a.ml[part] = make_float2(top, l);
    }
  }
}

// A wave per query adds its parts: lane l has dims 4 (l mod (D / 4)) .. + 3 of every (256 / D)-th.
template <typename T, int D>
__global__ __launch_bounds__(256) void join_kernel(Args a, int64_t queries) {
  constexpr int LD = D / 4, PAR = 64 / LD;
  const int lane = threadIdx.x & 63, x = lane % LD;
  const int64_t q = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (q >= queries) return;
  const float2* ml = a.ml + q * a.splits;
  const float* po = a.o + q * a.splits * D + 4 * x;
  float top = -INFINITY, l = 0.f;
  f32x4 o = {0.f, 0.f, 0.f, 0.f};
  for (int i = lane / LD; i < a.splits; i += PAR) {
    const float2 p = ml[i];
    const f32x4 y = *(const f32x4*)(po + (int64_t)i * D);
    const float now = fmaxf(top, p.x);
    const float c = top == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(top - now);
    const float d = p.x == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(p.x - now);
    o = o * c + (p.x == -INFINITY ? (f32x4){0.f, 0.f, 0.f, 0.f} : y * d);
    l = l * c + (p.x == -INFINITY ? 0.f : p.y * d);
    top = now;
  }
  float all = top;
#pragma unroll
  for (int s = 32; s >= LD; s >>= 1) all = fmaxf(all, __shfl_xor(all, s));
  const float c = top == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(top - all);
  o *= c;
  l *= c;
#pragma unroll
  for (int s = 32; s >= LD; s >>= 1) {
    l += __shfl_xor(l, s);
#pragma unroll
    for (int i = 0; i < 4; ++i) o[i] += __shfl_xor(o[i], s);
  }
  if (lane < LD) {
    const int h = (int)(q % a.d.n_head);
    const int64_t bt = q / a.d.n_head;
    put_query<T>(a, (int)(bt / a.d.n_query), (int)(bt % a.d.n_query), h, 4 * x, o, all, l);
  }
}

// ---------------------------------------------------------------- host

struct Plan {
  int nt, tiles, splits;
  int64_t blocks, queries;
  size_t o_bytes, bytes;
};
int64_t div_up(int64_t a, int64_t b) { return (a + b - 1) / b; }

constexpr int kRound = 1024;  // workgroups that are asked for

Plan plan(const ssd_page_pool& p, const ssd_page_seqs& s, const ssd_paged_attn_desc& d) {
  Plan x{};
  const int64_t cols = (int64_t)d.n_query * (d.n_head / p.n_kv_head);
  x.nt = cols > 16 ? 2 : 1;
  x.tiles = (int)div_up(cols, 16 * x.nt);
  int64_t pages = s.n_col;
  if (d.window)
    pages = std::min<int64_t>(pages, div_up(std::min<int64_t>(d.sinks, 1 << 30), p.page_rows) + d.window / p.page_rows + 2);
  const int64_t units = (int64_t)s.n_seq * p.n_kv_head * x.tiles, steps = pages * (p.page_rows / 32);
  x.splits = (int)std::max<int64_t>(1, std::min<int64_t>(kRound / units, div_up(steps, 4 * kWaves)));
  x.blocks = div_up((int64_t)p.n_kv_head * x.splits, 8) * 8 * s.n_seq * x.tiles;
  x.queries = (int64_t)s.n_seq * d.n_query * d.n_head;
  if (x.splits == 1) {
    x.bytes = 16;  // (not used)
    return x;
  }
  x.o_bytes = (size_t)x.queries * x.splits * p.head_dim * 4;
  x.bytes = x.o_bytes + (size_t)x.queries * x.splits * sizeof(float2);
  return x;
}

template <typename T, int D, int CODE, int NT>
hipError_t launch(const Args& a, const Plan& p, hipStream_t s) {
  constexpr int lds = (2 * kWaves * 16 * NT + kWaves * 16 * NT * (D + 4)) * 4;
  if constexpr (lds > 65536) {  // has to be asked for, once per kernel and device
    static std::atomic<uint64_t> ready{0};
    int dev = 0;
    hipError_t e = hipGetDevice(&dev);
    if (e != hipSuccess) return e;
    const uint64_t bit = dev < 64 ? 1ull << dev : 0;
    if (!(ready.load(std::memory_order_acquire) & bit)) {
      e = hipFuncSetAttribute((const void*)paged_attn_kernel<T, D, CODE, NT>,
                              hipFuncAttributeMaxDynamicSharedMemorySize, lds);
      if (e != hipSuccess) return e;
      ready.fetch_or(bit, std::memory_order_release);
    }
  }
  paged_attn_kernel<T, D, CODE, NT><<<(unsigned)p.blocks, 64 * kWaves, lds, s>>>(a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || p.splits == 1) return e;
  join_kernel<T, D><<<(unsigned)div_up(p.queries, 4), 256, 0, s>>>(a, p.queries);
  return hipGetLastError();
}
template <typename T, int D, int CODE>
hipError_t launch(const Args& a, const Plan& p, hipStream_t s) {
  return p.nt == 2 ? launch<T, D, CODE, 2>(a, p, s) : launch<T, D, CODE, 1>(a, p, s);
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
  OP_REQUIRE(isfinite(a->scale), SSD_E_INVALID_ARG, "scale must be finite");
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
  OP_REQUIRE(p.blocks <= kMostBlocks && p.queries <= 4 * kMostBlocks, SSD_E_CAPACITY, "more workgroups than a grid holds");
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
  OP_REQUIRE(workspace, SSD_E_INVALID_ARG, "null workspace");
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
  x.splits = p.splits;
  x.scale2 = a->scale * 1.4426950408889634f;
  const hipError_t e = a->dtype == SSD_F32 ? launch<float>(x, p, D, pool->code, (hipStream_t)stream)
                                           : launch<bf16_t>(x, p, D, pool->code, (hipStream_t)stream);
  if (e != hipSuccess) return op_fail(SSD_E_DEVICE, hipGetErrorString(e));
  return SSD_OK;
}
