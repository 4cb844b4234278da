// The paged cache of ssd_pages.h, but for its attention: blocks of rows into 8-bit codes and
// back, and the sequences' tables.
#include <algorithm>
#include <type_traits>

#include "ops_pages.h"

namespace ssd {
namespace {

constexpr int kThreads = 256, kWaveCount = kThreads / 64;
constexpr int kPlan = 1024, kPer = 4;  // threads of the kernels that give out pages, slots for each
static_assert(kPlan * kPer >= 4096, "a thread for every four slots");

// ---------------------------------------------------------------- codes

// 16 bytes, by the caches or past them (nontemporal).  Rows, which a call reads or writes once, go past them, whole rows at a
// time (in halves of a line they are fetched twice); codes that are made stay in them for the attention that reads them, and so do
// rows that a fork reads for several slots.  With all of it in the caches, lines that wait there for their way to memory
// stand in the way of what follows: 48 sequences of 36 layers, commit 72 us (here 51) and the read of their pages behind it 73
// (61); a prompt's rows into pages and back 210 (178); fork 39 (34); compaction 185 (172).
template <bool PAST = true>
__device__ __forceinline__ u32x4 get16(const void* p) {
  if constexpr (PAST) return __builtin_nontemporal_load((const u32x4*)p);
  else return *(const u32x4*)p;
}
__device__ __forceinline__ void put16(void* p, u32x4 x) { __builtin_nontemporal_store(x, (u32x4*)p); }

// 16 bytes of the model's type
__device__ __forceinline__ void unpack(u32x4 a, const float*, float* x) {
#pragma unroll
  for (int i = 0; i < 4; ++i) x[i] = __uint_as_float(a[i]);
}
__device__ __forceinline__ void unpack(u32x4 a, const bf16_t*, float* x) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    x[2 * i] = __uint_as_float(a[i] << 16);
    x[2 * i + 1] = __uint_as_float(a[i] & 0xffff0000u);
  }
}
__device__ __forceinline__ void store16(float* p, const float* x) {
  put16(p, __builtin_bit_cast(u32x4, (f32x4){x[0], x[1], x[2], x[3]}));
}
__device__ __forceinline__ void store16(bf16_t* p, const float* x) {
  u32x4 a;
#pragma unroll
  for (int i = 0; i < 4; ++i)
    a[i] = (unsigned)__builtin_bit_cast(uint16_t, (__bf16)x[2 * i]) |
           (unsigned)__builtin_bit_cast(uint16_t, (__bf16)x[2 * i + 1]) << 16;
  put16(p, a);
}

// Sums over the lanes up to this one, and the largest of all, within the registers.
__device__ __forceinline__ int lane_scan(int x) {
  x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, false);  // 1, 2, 4, 8 lanes before, within 16
  x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false);  // the last of the 16 before, to every second 16
  x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false);  // lane 31, to the upper 32
  return x;
}
__device__ __forceinline__ unsigned lane_max(unsigned x) {
  x = max(x, (unsigned)__builtin_amdgcn_update_dpp(0, (int)x, 0x111, 0xf, 0xf, false));
  x = max(x, (unsigned)__builtin_amdgcn_update_dpp(0, (int)x, 0x112, 0xf, 0xf, false));
  x = max(x, (unsigned)__builtin_amdgcn_update_dpp(0, (int)x, 0x114, 0xf, 0xf, false));
  x = max(x, (unsigned)__builtin_amdgcn_update_dpp(0, (int)x, 0x118, 0xf, 0xf, false));
  x = max(x, (unsigned)__builtin_amdgcn_update_dpp(0, (int)x, 0x142, 0xa, 0xf, false));
  x = max(x, (unsigned)__builtin_amdgcn_update_dpp(0, (int)x, 0x143, 0xc, 0xf, false));
  return (unsigned)__builtin_amdgcn_readlane((int)x, 63);
}

// How a block is coded (see ssd_pages.h), from the bits of its largest magnitude: as
// whole numbers those of infinities and NaN are larger than all finite ones'.
struct Coding {
  float r, scale;
  bool live;  // else: codes 0
};
template <int CODE>
__device__ __forceinline__ Coding coding(unsigned bits) {
  constexpr float top = CODE == SSD_PAGE_INT8 ? 127.f : 448.f;
  const float a = __uint_as_float(bits);
  if (bits >= 0x7f800000u) return {0.f, __uint_as_float(0x7fc00000u), false};
  if (a < 0x1p-100f) return {0.f, 0.f, false};
  return {top / a, a / top, true};
}
// Four codes, the first in the lowest byte.  (x r is rounded by itself: the clamp lies between
// it and the sum whose last bits are the nearest whole number's, ties to even.)
template <int CODE>
__device__ __forceinline__ unsigned code4(const float* x, int step, const Coding& c) {
  constexpr float top = CODE == SSD_PAGE_INT8 ? 127.f : 448.f;
  float y[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) y[i] = c.live ? fminf(fmaxf(x[i * step] * c.r, -top), top) : 0.f;
  if constexpr (CODE == SSD_PAGE_INT8) {
    unsigned u[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) u[i] = __float_as_uint(y[i] + 12583040.f);  // 1.5 2^23 + 128
    return __builtin_amdgcn_perm(u[1], u[0], 0x0c0c0400u) | __builtin_amdgcn_perm(u[3], u[2], 0x04000c0cu);
  } else {
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], 0, false);
    return (unsigned)__builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], w, true);
  }
}
template <int CODE>
__device__ __forceinline__ void values4(unsigned w, float scale, float* x, int step) {
  if constexpr (CODE == SSD_PAGE_INT8) {
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i * step] = ((float)(w >> 8 * i & 255u) - 128.f) * scale;
  } else {
    const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8(w, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8(w, true);
    x[0] = lo[0] * scale;
    x[step] = lo[1] * scale;
    x[2 * step] = hi[0] * scale;
    x[3 * step] = hi[1] * scale;
  }
}

// A wave's part of a block: 32 rows, in units of 16 bytes of a row, U elements, so that a wave's loads and stores are of whole
// rows.  Lane l has
//   keys:   units l + 64 q, q < KEYS, of the part;
//   values: for i < VALUES unit (l + 64 i) mod (D / U) of the four rows 4 ((l + 64 i) / (D / U)) .. (bfloat16 of 32 dims: 32
//           lanes do), whose codes at a dim are one 4-byte word.
// Codes get to their places, and back, through 32 D bytes of the wave's own LDS.
template <typename T, int D>
struct Part {
  static constexpr int U = 16 / sizeof(T), ROW = D / U, KEYS = ROW / 2, VALUES = (ROW + 7) / 8, BYTES = 32 * D;
  static constexpr int HELD = 4 * U * VALUES > U * KEYS ? 4 * U * VALUES : U * KEYS;  // elements of a lane
  static __device__ __forceinline__ int k_row(int lane, int q) { return (lane + 64 * q) / ROW; }
  static __device__ __forceinline__ int k_dim(int lane, int q) { return (lane + 64 * q) % ROW * U; }
  static __device__ __forceinline__ bool v_mine(int lane) { return ROW >= 8 || lane < 8 * ROW; }
  static __device__ __forceinline__ int v_row(int lane, int i) { return 4 * ((lane + 64 * i) / ROW); }
  static __device__ __forceinline__ int v_dim(int lane, int i) { return (lane + 64 * i) % ROW * U; }
  // where the codes of a row of the keys from dim d on lie, and the word of rows row .. row + 3 of the values at dim d
  static __device__ __forceinline__ int k_byte(int row, int d) {
    return D == 32 ? d / 8 * 256 + row % 16 * 16 + row / 16 * 8 + d % 8
                   : (row / 16 * (D / 64) + d / 64) * 1024 + d / 16 % 4 * 256 + row % 16 * 16 + d % 16;
  }
  static __device__ __forceinline__ int v_word(int row, int d) {
    return d / 32 * 1024 + (row / 4 % 4 * 16 + d % 16) * 16 + d / 16 % 2 * 8 + row / 16 * 4;
  }
};

// The part's elements, row r at row(r), and the bits of the largest magnitude of the lane's.
template <typename T, int D, typename Row>
__device__ __forceinline__ unsigned take_rows(bool values, int lane, Row row, float (&x)[Part<T, D>::HELD]) {
  typedef Part<T, D> P;
#pragma unroll
  for (int i = 0; i < P::HELD; ++i) x[i] = 0.f;
  if (!values) {
#pragma unroll
    for (int q = 0; q < P::KEYS; ++q) {
      const T* p = row(P::k_row(lane, q)) + P::k_dim(lane, q);
      unpack(get16(p), p, x + P::U * q);
    }
  } else {
    const int mine = P::v_mine(lane) ? lane : lane - 32;
#pragma unroll
    for (int i = 0; i < P::VALUES; ++i)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const T* p = row(P::v_row(mine, i) + r) + P::v_dim(mine, i);
        unpack(get16(p), p, x + P::U * (4 * i + r));
      }
  }
  unsigned most = 0;
#pragma unroll
  for (int i = 0; i < P::HELD; ++i) most = max(most, __float_as_uint(x[i]) & 0x7fffffffu);
  return lane_max(most);
}
// Their codes to the part at dst; lds: Part::BYTES of the wave's own.
template <typename T, int D, int CODE>
__device__ __forceinline__ void put_codes(bool values, int lane, const float (&x)[Part<T, D>::HELD], const Coding& c,
                                          uint8_t* dst, uint8_t* lds) {
  typedef Part<T, D> P;
  if (!values) {
#pragma unroll
    for (int q = 0; q < P::KEYS; ++q) {
      uint8_t* p = lds + P::k_byte(P::k_row(lane, q), P::k_dim(lane, q));
      if constexpr (P::U == 8) *(u32x2*)p = (u32x2){code4<CODE>(x + 8 * q, 1, c), code4<CODE>(x + 8 * q + 4, 1, c)};
      else *(unsigned*)p = code4<CODE>(x + 4 * q, 1, c);
    }
  } else if (P::v_mine(lane)) {
#pragma unroll
    for (int i = 0; i < P::VALUES; ++i)
#pragma unroll
      for (int j = 0; j < P::U; ++j)
        *(unsigned*)(lds + P::v_word(P::v_row(lane, i), P::v_dim(lane, i) + j)) = code4<CODE>(x + 4 * P::U * i + j, P::U, c);
  }
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
#pragma unroll
  for (int s = 0; s < P::BYTES / 1024; ++s)
    *(u32x4*)(dst + 1024 * s + 16 * lane) = *(const u32x4*)(lds + 1024 * s + 16 * lane);
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}
// The values that the part at src stands for, to row(r); the wave's lds as above.
template <typename T, int D, int CODE, typename Row>
__device__ __forceinline__ void put_values(bool values, int lane, const uint8_t* src, float scale, Row row,
                                           uint8_t* lds) {
  typedef Part<T, D> P;
#pragma unroll
  for (int s = 0; s < P::BYTES / 1024; ++s)
    *(u32x4*)(lds + 1024 * s + 16 * lane) = get16(src + 1024 * s + 16 * lane);
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
  float x[P::HELD];
  if (!values) {
#pragma unroll
    for (int q = 0; q < P::KEYS; ++q) {
      const uint8_t* p = lds + P::k_byte(P::k_row(lane, q), P::k_dim(lane, q));
#pragma unroll
      for (int w = 0; w < P::U / 4; ++w) values4<CODE>(((const unsigned*)p)[w], scale, x + P::U * q + 4 * w, 1);
      store16(row(P::k_row(lane, q)) + P::k_dim(lane, q), x + P::U * q);
    }
  } else if (P::v_mine(lane)) {
#pragma unroll
    for (int i = 0; i < P::VALUES; ++i) {
#pragma unroll
      for (int j = 0; j < P::U; ++j)
        values4<CODE>(*(const unsigned*)(lds + P::v_word(P::v_row(lane, i), P::v_dim(lane, i) + j)), scale,
                      x + 4 * P::U * i + j, P::U);
#pragma unroll
      for (int r = 0; r < 4; ++r) store16(row(P::v_row(lane, i) + r) + P::v_dim(lane, i), x + P::U * (4 * i + r));
    }
  }
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

// The waves of a workgroup take blocks, page_rows / 32 waves one.  The block's scale comes
// from all of its rows, so waves of one block meet once.
template <typename T, int D, int CODE, typename Row>
__device__ __forceinline__ void code_block(const ssd_page_pool& p, bool there, int64_t block, bool values, Row row,
                                           uint8_t (*lds)[Part<T, D>::BYTES], unsigned (&most)[kWaveCount]) {
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), waves = p.page_rows >> 5,
            part = wave % waves;
  float x[Part<T, D>::HELD];
  unsigned bits = 0;
  if (there) bits = take_rows<T, D>(values, lane, [&](int r) { return row(32 * part + r); }, x);
  if (waves > 1) {
    if (lane == 0) most[wave] = bits;
    __syncthreads();
    for (int w = 0; w < waves; ++w) bits = max(bits, most[wave - part + w]);
    __syncthreads();
  }
  if (!there) return;
  const Coding c = coding<CODE>(bits);
  put_codes<T, D, CODE>(values, lane, x, c, (uint8_t*)p.data + block * block_bytes(p) + part * Part<T, D>::BYTES,
                           lds[wave]);
  if (part == 0 && lane == 0) p.scale[block] = c.scale;
}

// ---------------------------------------------------------------- rows into pages, and back

struct BlockArgs {
  ssd_page_pool p;
  ssd_rows_desc d;
  const int* ids;
  char *k, *v;
  int first_layer;
  unsigned blocks;  // of a layer: 2 (keys, values) for each head and page
};
struct BlockAt {
  int64_t block, rows;  // the block's number in the pool (-1: none), its rows' first element
  bool values, there;
};
// blockIdx.y: the layer
__device__ __forceinline__ BlockAt block_at(const BlockArgs& a, unsigned i) {
  BlockAt x;
  x.there = i < a.blocks;
  if (!x.there) i = 0;
  const unsigned heads = 2 * a.p.n_kv_head, n = i / heads, gv = i - n * heads, l = blockIdx.y;
  x.values = gv & 1;
  const int id = a.ids[n];
  x.block = id < 0 || id >= a.p.n_page ? -1 : ((int64_t)(a.first_layer + l) * a.p.n_page + id) * heads + gv;
  x.rows = l * a.d.layer + n * a.d.seq + (gv >> 1) * a.d.head;
  return x;
}

// A wave reads 32 rows once, holds them in registers until the block's largest magnitude is known, and writes their
// bytes in the pool's order: rows are read once and no second pass is made.
//   Bound: memory.  36 layers x 63 pages x 20 heads x 32 rows of 64 bfloat16 (558 MB): 96 us, 5.8 TB/s where a large
// copy reaches 5.2.  (Block numbers in 32 bits and a layer a grid row were 117 to 124 with 64-bit divisions.)
template <typename T, int D, int CODE>
__global__ __launch_bounds__(kThreads) void store_kernel(BlockArgs a) {
  __shared__ __align__(16) uint8_t lds[kWaveCount][Part<T, D>::BYTES];
  __shared__ unsigned most[kWaveCount];
  const int waves = a.p.page_rows >> 5, units = kWaveCount / waves,
            unit = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) / waves;
  for (unsigned first = blockIdx.x * units; first < a.blocks; first += gridDim.x * units) {
    const BlockAt at = block_at(a, first + unit);
    const T* base = (const T*)(at.values ? a.v : a.k) + at.rows;
    code_block<T, D, CODE>(a.p, at.there && at.block >= 0, at.block, at.values,
                           [&](int r) { return base + r * a.d.row; }, lds, most);
  }
}
// The way back: as many bytes, 82 us of the same size (6.8 TB/s).
template <typename T, int D, int CODE>
__global__ __launch_bounds__(kThreads) void load_kernel(BlockArgs a) {
  __shared__ __align__(16) uint8_t lds[kWaveCount][Part<T, D>::BYTES];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), waves = a.p.page_rows >> 5,
            units = kWaveCount / waves, unit = wave / waves, part = wave % waves;
  for (unsigned first = blockIdx.x * units; first < a.blocks; first += gridDim.x * units) {
    const BlockAt at = block_at(a, first + unit);
    if (!at.there) continue;
    T* base = (T*)(at.values ? a.v : a.k) + at.rows;
    auto row = [&](int r) { return base + (32 * part + r) * a.d.row; };
    if (at.block < 0) {
      typedef Part<T, D> P;
      const float zero[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
      for (int q = 0; q < P::KEYS; ++q) store16(row(P::k_row(lane, q)) + P::k_dim(lane, q), zero);
    } else {
      put_values<T, D, CODE>(at.values, lane, (const uint8_t*)a.p.data + at.block * block_bytes(a.p) + part * Part<T, D>::BYTES,
                             a.p.scale[at.block], row, lds[wave]);
    }
  }
}

// ---------------------------------------------------------------- giving out pages

struct Work {  // the workspace
  int *head;            // [0]: pages that get full, [1]: pages to move, [2]: pages in use
  int4* slot;           // [n_seq] (length before, rows appended, pages that get full, whether it is served)
  int4* jobs;           // [2 n_seq] (slot, column, page, -) of those pages
  int *a, *b, *to;      // [n_page]
};
Work work_at(void* w, int n_seq, int n_page) {
  Work x;
  x.head = (int*)w;
  x.slot = (int4*)(x.head + 16);
  x.jobs = x.slot + n_seq;
  x.a = (int*)(x.jobs + 2 * n_seq);
  x.b = x.a + n_page;
  x.to = x.b + n_page;
  return x;
}
size_t work_bytes(int n_seq, int n_page) { return 64 + 48 * (size_t)n_seq + 12 * (size_t)n_page; }

// Sums over the threads before this one, and over all.  A wave's is counted to 2^26 at the most: more than there
// are pages, so what lies behind it gets none either way.
__device__ __forceinline__ int scan(int x, int* sums, int& all) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, upto = lane_scan(x);
  if (lane == 63) sums[wave] = min(upto, 1 << 26);
  __syncthreads();
  int before = 0;
  all = 0;
#pragma unroll
  for (int w = 0; w < kPlan / 64; ++w) {
    const int y = sums[w];
    before += w < wave ? y : 0;
    all += y;
  }
  __syncthreads();
  return before + upto - x;
}
// Writes the first `most` pages p in [from, to) whose refs are as asked to list, in order; how many there
// are, up to those with which the search ended.
constexpr int kLook = 8;  // refs a thread looks at
struct Refs {
  int x[kLook];
  __device__ __forceinline__ void load(const int* refs, int at, int to) {
    if (at + kLook <= to) {
      __builtin_memcpy(x, refs + at, sizeof(x));
    } else {
#pragma unroll
      for (int i = 0; i < kLook; ++i) x[i] = at + i < to ? refs[at + i] : -1;
    }
  }
};
__device__ __forceinline__ int find_pages(const Refs* first, const int* refs, int from, int to, bool in_use, int* list, int most,
                                          int* sums) {
  int found = 0;
  for (int base = from; base < to && found < most; base += kPlan * kLook) {
    const int at = base + (int)threadIdx.x * kLook;
    Refs r;
    if (first && base == from) r = *first;
    else r.load(refs, at, to);
    unsigned mask = 0;
#pragma unroll
    for (int i = 0; i < kLook; ++i)
      if (at + i < to && (r.x[i] > 0) == in_use) mask |= 1u << i;
    int all;
    int rank = found + scan(__popc(mask), sums, all);
    for (; mask; mask &= mask - 1, ++rank)
      if (rank < most) list[rank] = at + __ffs(mask) - 1;
    found += all;
  }
  return found;
}

struct PlanArgs {
  ssd_page_seqs s;
  Work w;
  int n_page, page_rows;
  const int* count;           // take
  int* got;                   // take: pages that a slot got, commit: that got full
  const int *path, *path_len; // commit
  int64_t path_ld;
  int max_path, n_new;
};

// Which slots get how many pages, and which: the lowest free ones, slots in order, so that tables do not depend on
// timing.  One workgroup: the sums over slots and pages are two scans, and a launch between workgroups would
// cost more (a launch 3 us) than the whole.
//   Bound: latency, a chain of some ten loads and meetings.  48 sequences, 1216 pages: 8.4 us (15.6 before refs, lengths
// and paths were loaded at once ahead of everything, and before scans stayed in registers); 3 sequences 3.8.  Paths take
// a turn for 16 slots: a commit of one layer takes 14 us for 512 sequences and 84 for 4096.
template <bool COMMIT>
__global__ __launch_bounds__(kPlan) void plan_kernel(PlanArgs a) {
  __shared__ int want[4096], first[4096], col0[4096], sums[kPlan / 64], jobs;
  __shared__ uint8_t rows[COMMIT ? 4096 : 1];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, n_seq = a.s.n_seq;
  // (what does not depend on anything is under way from the start)
  Refs refs;
  refs.load(a.s.refs, threadIdx.x * kLook, a.n_page);
  int len[kPer], asked[kPer];
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    const int b = threadIdx.x * kPer + i;
    len[i] = b < n_seq ? a.s.length[b] : -1;
    asked[i] = !COMMIT && b < n_seq ? a.count[b] : -1;
  }
  if (threadIdx.x == 0) jobs = 0;
  if constexpr (COMMIT) {
    // rows up to the path's first that is none, and no more than there are (a path can name one twice): a sequence then
    // grows by less than the tail has rows behind its open page, which the kernel behind this one relies on
    for (int b = wave; b < n_seq; b += kPlan / 64) {
      const int t = lane < a.max_path ? a.path[b * a.path_ld + lane] : -1, n = min(min(a.path_len[b], a.max_path), a.n_new);
      const unsigned long long bads = __ballot(lane >= n || t < 0 || t >= a.n_new);
      if (lane == 0) rows[b] = bads ? __ffsll(bads) - 1 : 64;
    }
    __syncthreads();
  }
  int need[kPer], sum = 0;
  bool can[kPer];
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    const int b = threadIdx.x * kPer + i;
    can[i] = false;
    need[i] = 0;
    if (b >= n_seq) continue;
    const int from = max(len[i], 0), col = from / a.page_rows;
    if constexpr (COMMIT) {
      const int64_t after = ((int64_t)from + rows[b]) / a.page_rows;
      can[i] = len[i] >= 0 && after <= a.s.n_col;
      need[i] = can[i] ? (int)after - col : 0;
    } else {
      can[i] = asked[i] >= 0 && from % a.page_rows == 0 && (int64_t)col + asked[i] <= a.s.n_col;
      need[i] = can[i] ? asked[i] : 0;
    }
    col0[b] = col;
    sum += min(need[i], kMaxPages + 1);  // (more than there are: as good as any number)
  }
  int all;
  int rank = scan(sum, sums, all);
  int free = 0;
  if (all > 0) {
    free = find_pages(&refs, a.s.refs, 0, a.n_page, false, a.w.a, min(all, a.n_page), sums);
    __syncthreads();
  }
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    const int b = threadIdx.x * kPer + i;
    if (b >= n_seq) continue;
    const bool ok = can[i] && (need[i] == 0 || rank + need[i] <= free);
    want[b] = ok ? need[i] : 0;
    first[b] = rank;
    rank += min(need[i], kMaxPages + 1);
    if constexpr (COMMIT) {
      const int n = ok ? rows[b] : 0;
      a.w.slot[b] = make_int4(len[i], n, ok ? need[i] : 0, ok);
      a.got[b] = ok ? need[i] : len[i] < 0 ? 0 : -1;
      if (n) a.s.length[b] = len[i] + n;
    } else {
      a.got[b] = ok ? need[i] : -1;
      if (ok) a.s.length[b] = max(len[i], 0) + need[i] * a.page_rows;
    }
  }
  __syncthreads();
  for (int b = wave; b < n_seq; b += kPlan / 64) {
    const int n = want[b];
    if (n == 0) continue;
    const int c = col0[b];
    int job = 0;
    if (COMMIT && lane == 0) job = atomicAdd(&jobs, n);  // (their order in the list changes no result)
    job = __shfl(job, 0);
    for (int j = lane; j < n; j += 64) {
      const int page = a.w.a[first[b] + j];
      a.s.table[b * a.s.table_ld + c + j] = page;
      a.s.refs[page] = 1;
      if (COMMIT) a.w.jobs[job + j] = make_int4(b, c + j, page, 0);
    }
  }
  if (COMMIT) {
    __syncthreads();
    if (threadIdx.x == 0) a.w.head[0] = jobs;
  }
}

// ---------------------------------------------------------------- commit

struct CommitArgs {
  ssd_page_pool p;
  ssd_page_seqs s;
  Work w;
  ssd_rows_desc tail, fresh;
  char *kt, *vt;
  const char *kn, *vn;
  const int* path;
  int64_t path_ld;
  int window, sinks;
  int fill;  // workgroups that fill pages
};

// the place of a row that lies less than a ring's `rows` behind its start
__device__ __forceinline__ int64_t ring(int at, int rows) { return at >= rows ? at - rows : at; }

// items 16 bytes each, of `heads` heads' `rows` rows, four a thread under way: src(head, row), dst(head, row)
// the row's first byte
template <bool PAST, typename Src, typename Dst>
__device__ __forceinline__ void copy_rows(int heads, int rows, int row_shift, bool rows_outer, Src src, Dst dst) {
  const int total = heads * rows << row_shift, inner = rows_outer ? heads : rows;  // (a row: 2^row_shift times 16 bytes)
  constexpr int U = 4;
  for (int i0 = threadIdx.x; i0 < total; i0 += U * kThreads) {
    u32x4 x[U];
    char* to[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int i = i0 + u * kThreads;
      if (i >= total) break;
      const unsigned hr = (unsigned)i >> row_shift;
      const int v = i & ((1 << row_shift) - 1), out = hr / (unsigned)inner, in = hr - out * inner;
      const int h = rows_outer ? in : out, r = rows_outer ? out : in;
      x[u] = get16<PAST>(src(h, r) + 16 * v);
      to[u] = dst(h, r) + 16 * v;
    }
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (i0 + u * kThreads < total) put16(to[u], x[u]);
  }
}

// Workgroups: first `fill` that make the pages that got full, wave by wave; then for each slot one that
// gives back what is behind the window, and for each layer and keys or values one that moves rows into the tail.
// (Rows that are moved go to other places of the tail than those of the page: from the open page's first row to the last
// new one are page_rows + new rows - 1 at the most, and tail_rows is no less, so all run side by side.)  How many pages got full is known on the device alone: the fillers share
// the blocks there are, side by side, each an equal run of them, so that most of its blocks are of one page and where
// that page's rows lie is looked up once (in the lanes, a row each).
//   Bound: memory; for few rows the launch (4.1 us for 3 sequences).  48 sequences of 36 layers and 20 heads of 64 that
// take up to 16 rows each: 50 us for 257 MB, 5.1 TB/s.  (All by the caches 72, of it the fillers alone 40, 55 while every block
// looked its page and rows up, and the moves alone 40.)
// 768, 1024 and 1536 fillers measured the same; 4 and 8 copies under way, too.
template <typename T, int D, int CODE>
__global__ __launch_bounds__(kThreads) void commit_kernel(CommitArgs a) {
  __shared__ __align__(16) uint8_t lds[kWaveCount][Part<T, D>::BYTES];
  __shared__ unsigned most[kWaveCount];
  const int R0 = a.p.page_rows, G = a.p.n_kv_head;
  if ((int)blockIdx.x < a.fill) {
    const int waves = R0 >> 5, units = kWaveCount / waves, unit = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) / waves;
    const unsigned heads = 2 * G, each = a.p.n_layer * heads;  // (of a page)
    const int64_t blocks = (int64_t)a.w.head[0] * each, turn = (int64_t)a.fill * units;
    const int64_t share = (blocks + turn - 1) / turn * units, to = min((int64_t)(blockIdx.x + 1) * share, blocks);
    const int lane = threadIdx.x & 63, part = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) % waves;
    unsigned had = ~0u;
    int b = 0, page = 0, mine = 0;  // of the job; lane r: where row 32 part + r lies, ~ its number among the new ones
    for (int64_t at = (int64_t)blockIdx.x * share; at < to; at += units) {
      int64_t i = at + unit;
      const bool there = i < to;
      if (!there) i = at;
      const unsigned which = blocks >> 32 ? (unsigned)(i / each) : (unsigned)i / each, at_page = (unsigned)(i - (int64_t)which * each);
      const unsigned l = at_page / heads, gv = at_page - l * heads, g = gv >> 1;
      if (which != had) {
        had = which;
        const int4 job = a.w.jobs[which];
        b = job.x;
        page = job.z;
        const int len = a.w.slot[b].x, pos = job.y * R0, r = 32 * part + (lane & 31);
        mine = r < len - pos ? (int)ring(pos % a.tail.rows + r, a.tail.rows) : ~a.path[b * a.path_ld + r - (len - pos)];
      }
      const bool values = gv & 1;
      const int64_t block = ((int64_t)l * a.p.n_page + page) * heads + gv;
      const T* old = (const T*)(values ? a.vt : a.kt) + l * a.tail.layer + b * a.tail.seq + g * a.tail.head;
      const T* add = (const T*)(values ? a.vn : a.kn) + l * a.fresh.layer + b * a.fresh.seq + g * a.fresh.head;
      code_block<T, D, CODE>(
          a.p, there, block, values,
          [&](int r) {
            const int x = __shfl(mine, r & 31);
            return x >= 0 ? old + x * a.tail.row : add + ~x * a.fresh.row;
          },
          lds, most);
    }
    return;
  }
  const int each = 1 + 2 * a.p.n_layer, at = (int)blockIdx.x - a.fill, b = at / each, part = at % each;
  const int4 slot = a.w.slot[b];
  if (part == 0) {
    if (a.window <= 0 || !slot.w) return;
    // pages whose rows are all at sinks or behind, and at most length - window
    const int64_t end = (int64_t)slot.x + slot.y - a.window + 1;
    const int from = (int)(((int64_t)a.sinks + R0 - 1) / R0), to = (int)min((int64_t)a.s.n_col, end > 0 ? end / R0 : 0);
    for (int c = from + threadIdx.x; c < to; c += kThreads) {
      int* entry = a.s.table + b * a.s.table_ld + c;
      const int page = *entry;
      if (page < 0) continue;
      *entry = -1;
      if (page < a.p.n_page) atomicSub(a.s.refs + page, 1);
    }
    return;
  }
  const int l = (part - 1) >> 1;
  const bool values = (part - 1) & 1;
  // rows behind the last page that got full
  const int start = max(0, (slot.x / R0 + slot.z) * R0 - slot.x), n = slot.y - start;
  if (n <= 0) return;
  char* old = (values ? a.vt : a.kt) + (l * a.tail.layer + b * a.tail.seq) * (int)sizeof(T);
  const char* add = (values ? a.vn : a.kn) + (l * a.fresh.layer + b * a.fresh.seq) * (int)sizeof(T);
  const int* path = a.path + b * a.path_ld + start;
  const int place = (slot.x + start) % a.tail.rows;
  copy_rows<true>(
      G, n, __builtin_ctz(D * sizeof(T) / 16), true,
      [&](int g, int r) { return add + (path[r] * a.fresh.row + g * a.fresh.head) * (int)sizeof(T); },
      [&](int g, int r) { return old + (ring(place + r, a.tail.rows) * a.tail.row + g * a.tail.head) * (int)sizeof(T); });
}

// ---------------------------------------------------------------- fork

struct ForkArgs {
  ssd_page_seqs s;
  ssd_rows_desc tail;
  int n_page, page_rows, n_layer, n_kv_head, row_shift;
  const int* parents;
  char *kt, *vt;
};
// blockIdx.y: the slot; blockIdx.x: 0 its table, 1 + 2 l + (keys, values) its open rows in layer l.
// A slot that is copied from stays as it is, so nothing that is read here is written here, and one launch does it.
//   Bound: memory; for few slots the launch (3.7 us).  64 slots of 36 layers and 20 heads of 64, open rows of up to 31:
// 35 us, 6.0 TB/s (210 MB; samples of one prompt read the same rows).
__global__ __launch_bounds__(kThreads) void fork_kernel(ForkArgs a) {
  const int b = blockIdx.y, s = a.parents[b];
  if (s == b) return;
  const bool kept = s >= 0 && s < a.s.n_seq && a.parents[s] == s;
  if (blockIdx.x == 0) {
    int* mine = a.s.table + b * a.s.table_ld;
    const int* its = a.s.table + s * a.s.table_ld;
    for (int c = threadIdx.x; c < a.s.n_col; c += kThreads) {
      const int old = mine[c], now = kept ? its[c] : -1;
      if (old == now) continue;
      mine[c] = now;
      if (now >= 0 && now < a.n_page) atomicAdd(a.s.refs + now, 1);
      if (old >= 0 && old < a.n_page) atomicSub(a.s.refs + old, 1);
    }
    if (threadIdx.x == 0) a.s.length[b] = kept ? a.s.length[s] : -1;
    return;
  }
  if (!kept) return;
  const int len = a.s.length[s];
  if (len <= 0) return;
  const int n = len % a.page_rows, place = (len - n) % a.tail.rows, l = (blockIdx.x - 1) >> 1, es = a.tail.dtype == SSD_F32 ? 4 : 2;
  char* base = (blockIdx.x - 1 & 1 ? a.vt : a.kt) + l * a.tail.layer * es;
  auto at = [&](int slot, int g, int r) {
    return base + (slot * a.tail.seq + g * a.tail.head + ring(place + r, a.tail.rows) * a.tail.row) * es;
  };
  copy_rows<false>(a.n_kv_head, n, a.row_shift, false, [&](int g, int r) { return (const char*)at(s, g, r); },
            [&](int g, int r) { return at(b, g, r); });
}

// ---------------------------------------------------------------- compaction

struct CompactArgs {
  ssd_page_pool p;
  ssd_page_seqs s;
  Work w;
  int* used;
};
// Which pages move where: the pages in use, counted, the free ones before and the used ones behind their number, in
// order.  Bound: latency, 5.2 us for 625 pages (8.6 with a turn of loads for every step).
__global__ __launch_bounds__(kPlan) void compact_plan_kernel(CompactArgs a) {
  __shared__ int sums[kPlan / 64];
  const int n = a.p.n_page;
  Refs refs;
  refs.load(a.s.refs, threadIdx.x * kLook, n);
  int count = 0;
#pragma unroll
  for (int i = 0; i < kLook; ++i) count += refs.x[i] > 0;
  for (int p = kPlan * kLook + threadIdx.x; p < n; p += kPlan) count += a.s.refs[p] > 0;
  int u;
  scan(count, sums, u);
  const int holes = find_pages(&refs, a.s.refs, 0, u, false, a.w.a, n, sums);
  const int movers = find_pages(nullptr, a.s.refs, u, n, true, a.w.b, n, sums);  // (as many)
  for (int p = u + threadIdx.x; p < n; p += kPlan) a.w.to[p] = p;
  __syncthreads();
  const int moves = min(holes, movers);
  for (int i = threadIdx.x; i < moves; i += kPlan) {
    const int to = a.w.a[i], from = a.w.b[i];
    a.w.to[from] = to;
    a.s.refs[to] = a.s.refs[from];
    a.s.refs[from] = 0;
  }
  if (threadIdx.x == 0) {
    a.w.head[1] = moves;
    a.w.head[2] = u;
    *a.used = u;
  }
}
// Moves pages, a piece of one layer's at a time, and names them anew.  Pages come from behind
// `used` and go before it: no piece is read and written.  16 KB a piece, 64 bytes a thread under way.
//   Bound: memory.  156 pages of 36 layers, 20 heads, 32 rows of 64 (921 MB read and written): 172 us, 5.4 TB/s.
constexpr int kPiece = 16384;
__global__ __launch_bounds__(kThreads) void compact_move_kernel(CompactArgs a) {
  const int moves = a.w.head[1], used = a.w.head[2], n = a.p.n_page, G = a.p.n_kv_head;
  const int64_t bytes = (int64_t)G * 2 * block_bytes(a.p);
  const int pieces = (int)((bytes + kPiece - 1) / kPiece);
  for (int64_t i = blockIdx.x; i < (int64_t)moves * a.p.n_layer * pieces; i += gridDim.x) {
    const int piece = (int)(i % pieces);
    const int64_t lm = i / pieces;
    const int m = (int)(lm % moves), l = (int)(lm / moves);
    const int64_t from = (int64_t)l * n + a.w.b[m], to = (int64_t)l * n + a.w.a[m];
    const int64_t at = (int64_t)piece * kPiece;
    const char* src = (const char*)a.p.data + from * bytes + at;
    char* dst = (char*)a.p.data + to * bytes + at;
    const int vec = (int)(min((int64_t)kPiece, bytes - at) / 16);
    u32x4 x[kPiece / 16 / kThreads];
#pragma unroll
    for (int u = 0; u < kPiece / 16 / kThreads; ++u)
      if ((int)threadIdx.x + u * kThreads < vec) x[u] = get16(src + 16 * (threadIdx.x + u * kThreads));
#pragma unroll
    for (int u = 0; u < kPiece / 16 / kThreads; ++u)
      if ((int)threadIdx.x + u * kThreads < vec) put16(dst + 16 * (threadIdx.x + u * kThreads), x[u]);
    if (piece == 0)
      for (int j = threadIdx.x; j < 2 * G; j += kThreads) a.p.scale[to * 2 * G + j] = a.p.scale[from * 2 * G + j];
  }
  const int64_t entries = (int64_t)a.s.n_seq * a.s.n_col;
  for (int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x; i < entries; i += (int64_t)gridDim.x * kThreads) {
    int* entry = a.s.table + i / a.s.n_col * a.s.table_ld + i % a.s.n_col;
    const int page = *entry;
    if (page >= used && page < n) *entry = a.w.to[page];
  }
}

// ---------------------------------------------------------------- host

constexpr unsigned kMostBlocks = 1 << 16;  // workgroups of kernels that take more work than that in turns

template <typename F>
void by_type(ssd_dtype t, int d, int code, F f) {
  auto with_code = [&](auto dtype, auto dim) {
    if (code == SSD_PAGE_INT8) f(dtype, dim, std::integral_constant<int, SSD_PAGE_INT8>{});
    else f(dtype, dim, std::integral_constant<int, SSD_PAGE_E4M3>{});
  };
  auto with_dim = [&](auto dtype) {
    if (d == 32) with_code(dtype, std::integral_constant<int, 32>{});
    else if (d == 64) with_code(dtype, std::integral_constant<int, 64>{});
    else with_code(dtype, std::integral_constant<int, 128>{});
  };
  if (t == SSD_F32) with_dim(float{});
  else with_dim(bf16_t{});
}

ssd_status blocks_args(const ssd_page_pool* pool, const int32_t* ids, int32_t n, int32_t first_layer, int32_t n_layer,
                       const ssd_rows_desc* d, const void* k, const void* v, bool written, BlockArgs* a) {
  ssd_status st = check_pool(pool);
  if (st != SSD_OK) return st;
  OP_REQUIRE(n >= 0 && n <= kMaxPages, SSD_E_INVALID_ARG, "n outside [0, 2^20]");
  OP_REQUIRE(first_layer >= 0 && n_layer >= 0 && (int64_t)first_layer + n_layer <= pool->n_layer, SSD_E_INVALID_ARG,
             "layers outside the pool's");
  OP_REQUIRE(d, SSD_E_INVALID_ARG, "null rows");
  a->p = *pool;
  a->d = *d;
  a->ids = ids;
  a->first_layer = first_layer;
  a->k = (char*)k;
  a->v = (char*)v;
  a->blocks = n_layer ? (unsigned)n * pool->n_kv_head * 2 : 0;  // (2^31 at the most)
  if (a->blocks == 0) return SSD_OK;
  OP_REQUIRE(ids && (uintptr_t)ids % 4 == 0, SSD_E_INVALID_ARG, "ids is null or not aligned");
  const RowDim dims[4] = {{n_layer, d->layer}, {n, d->seq}, {pool->n_kv_head, d->head}, {pool->page_rows, d->row}};
  st = check_rows(d->dtype, dims, pool->head_dim, written, k, v);
  if (st != SSD_OK) return st;
  const size_t e = rows_extent(d->dtype, dims, pool->head_dim);
  const size_t held = (size_t)pool->n_layer * pool->n_page * pool->n_kv_head * 2 * block_bytes(*pool);
  const size_t scales = (size_t)pool->n_layer * pool->n_page * pool->n_kv_head * 8;
  OP_REQUIRE(!written || !op_overlap(k, e, v, e), SSD_E_INVALID_ARG, "k and v share memory");
  for (const void* x : {k, v})
    OP_REQUIRE(!op_overlap(x, e, pool->data, held) && !op_overlap(x, e, pool->scale, scales) &&
                   (!written || !op_overlap(x, e, ids, (size_t)n * 4)),
               SSD_E_INVALID_ARG, "rows share memory with the pool or ids");
  return SSD_OK;
}

ssd_status check_work(const ssd_page_pool* pool, const ssd_page_seqs* s, const void* w, size_t bytes) {
  OP_REQUIRE(w, SSD_E_INVALID_ARG, "null workspace");
  OP_REQUIRE(bytes >= work_bytes(s->n_seq, pool->n_page) && (uintptr_t)w % 16 == 0, SSD_E_CAPACITY,
             "workspace below ssd_pages_workspace's bytes or not 16-byte aligned");
  return SSD_OK;
}

}  // namespace
}  // namespace ssd

using namespace ssd;

extern "C" ssd_status ssd_pages_store(const ssd_page_pool* pool, const int32_t* ids, int32_t n, int32_t first_layer,
                                      int32_t n_layer, const ssd_rows_desc* d, const void* k, const void* v,
                                      void* stream) {
  BlockArgs a{};
  const ssd_status st = blocks_args(pool, ids, n, first_layer, n_layer, d, k, v, false, &a);
  if (st != SSD_OK || a.blocks == 0) return st;
  by_type(d->dtype, pool->head_dim, pool->code, [&](auto t, auto dim, auto code) {
    const unsigned units = kWaveCount / (pool->page_rows / 32), want = (a.blocks + units - 1) / units;
    const dim3 grid(std::min(want, kMostBlocks), n_layer);
    store_kernel<decltype(t), dim.value, code.value>
        <<<grid, kThreads, 0, (hipStream_t)stream>>>(a);
  });
  OP_LAUNCHED();
  return SSD_OK;
}

extern "C" ssd_status ssd_pages_load(const ssd_page_pool* pool, const int32_t* ids, int32_t n, int32_t first_layer,
                                     int32_t n_layer, const ssd_rows_desc* d, void* k, void* v, void* stream) {
  BlockArgs a{};
  const ssd_status st = blocks_args(pool, ids, n, first_layer, n_layer, d, k, v, true, &a);
  if (st != SSD_OK || a.blocks == 0) return st;
  by_type(d->dtype, pool->head_dim, pool->code, [&](auto t, auto dim, auto code) {
    const unsigned units = kWaveCount / (pool->page_rows / 32), want = (a.blocks + units - 1) / units;
    const dim3 grid(std::min(want, kMostBlocks), n_layer);
    load_kernel<decltype(t), dim.value, code.value>
        <<<grid, kThreads, 0, (hipStream_t)stream>>>(a);
  });
  OP_LAUNCHED();
  return SSD_OK;
}

extern "C" ssd_status ssd_pages_workspace(const ssd_page_pool* pool, const ssd_page_seqs* seqs, size_t* bytes) {
  OP_REQUIRE(bytes, SSD_E_INVALID_ARG, "null argument");
  ssd_status st = check_pool(pool);
  if (st == SSD_OK) st = check_seqs(seqs, pool->page_rows, true);
  if (st != SSD_OK) return st;
  *bytes = work_bytes(seqs->n_seq, pool->n_page);
  return SSD_OK;
}

extern "C" ssd_status ssd_pages_take(const ssd_page_pool* pool, const ssd_page_seqs* seqs, const int32_t* count,
                                     int32_t* got, void* workspace, size_t workspace_bytes, void* stream) {
  ssd_status st = check_pool(pool);
  if (st == SSD_OK) st = check_seqs(seqs, pool->page_rows, true);
  if (st == SSD_OK) st = check_work(pool, seqs, workspace, workspace_bytes);
  if (st != SSD_OK) return st;
  OP_REQUIRE(count && got && (uintptr_t)count % 4 == 0 && (uintptr_t)got % 4 == 0, SSD_E_INVALID_ARG,
             "count or got is null or not aligned");
  PlanArgs a{};
  a.s = *seqs;
  a.w = work_at(workspace, seqs->n_seq, pool->n_page);
  a.n_page = pool->n_page;
  a.page_rows = pool->page_rows;
  a.count = count;
  a.got = got;
  plan_kernel<false><<<1, kPlan, 0, (hipStream_t)stream>>>(a);
  OP_LAUNCHED();
  return SSD_OK;
}

extern "C" ssd_status ssd_pages_commit(const ssd_page_pool* pool, const ssd_page_seqs* seqs, const ssd_rows_desc* tail,
                                       void* k_tail, void* v_tail, const ssd_rows_desc* fresh, const void* k_new,
                                       const void* v_new, const int32_t* path, int64_t path_ld, int32_t max_path,
                                       const int32_t* path_len, int32_t window, int32_t sinks, int32_t* full,
                                       void* workspace, size_t workspace_bytes, void* stream) {
  ssd_status st = check_pool(pool);
  if (st == SSD_OK) st = check_seqs(seqs, pool->page_rows, true);
  if (st == SSD_OK) st = check_work(pool, seqs, workspace, workspace_bytes);
  if (st != SSD_OK) return st;
  OP_REQUIRE(tail && fresh, SSD_E_INVALID_ARG, "null rows");
  OP_REQUIRE(tail->dtype == fresh->dtype, SSD_E_INVALID_ARG, "the tail and the new rows have two types");
  OP_REQUIRE(fresh->rows >= 1 && fresh->rows <= 64, SSD_E_INVALID_ARG, "new rows outside [1, 64]");
  OP_REQUIRE(tail->rows >= pool->page_rows + fresh->rows - 1 && tail->rows < (1 << 30), SSD_E_INVALID_ARG,
             "tail rows below page_rows + new rows - 1, or 2^30");
  OP_REQUIRE(max_path >= 0 && max_path <= 64 && (seqs->n_seq == 1 || path_ld >= max_path), SSD_E_INVALID_ARG,
             "max_path outside [0, 64], or path_ld below it");
  OP_REQUIRE(window >= 0 && sinks >= 0, SSD_E_INVALID_ARG, "window or sinks is negative");
  OP_REQUIRE((path || max_path == 0) && path_len && full && (uintptr_t)path % 4 == 0 && (uintptr_t)path_len % 4 == 0 &&
                 (uintptr_t)full % 4 == 0,
             SSD_E_INVALID_ARG, "path, path_len or full is null or not aligned");
  const RowDim td[4] = {{pool->n_layer, tail->layer}, {seqs->n_seq, tail->seq}, {pool->n_kv_head, tail->head},
                        {tail->rows, tail->row}};
  const RowDim nd[4] = {{pool->n_layer, fresh->layer}, {seqs->n_seq, fresh->seq}, {pool->n_kv_head, fresh->head},
                        {fresh->rows, fresh->row}};
  st = check_rows(tail->dtype, td, pool->head_dim, true, k_tail, v_tail);
  if (st == SSD_OK) st = check_rows(fresh->dtype, nd, pool->head_dim, false, k_new, v_new);
  if (st != SSD_OK) return st;
  const size_t te = rows_extent(tail->dtype, td, pool->head_dim), ne = rows_extent(fresh->dtype, nd, pool->head_dim);
  OP_REQUIRE(!op_overlap(k_tail, te, v_tail, te), SSD_E_INVALID_ARG, "the tail's keys and values share memory");
  for (const void* t : {(const void*)k_tail, (const void*)v_tail})
    for (const void* x : {k_new, v_new})
      OP_REQUIRE(!op_overlap(t, te, x, ne), SSD_E_INVALID_ARG, "the tail shares memory with the new rows");
  const int units = kWaveCount / (pool->page_rows / 32);
  const int fill = (int)std::min<int64_t>(((int64_t)seqs->n_seq * pool->n_layer * pool->n_kv_head * 2 + units - 1) / units, 1024);
  const int64_t blocks = fill + (int64_t)seqs->n_seq * (1 + 2 * pool->n_layer);
  OP_REQUIRE(blocks < (1 << 24), SSD_E_CAPACITY, "more workgroups than a grid holds");
  const Work w = work_at(workspace, seqs->n_seq, pool->n_page);
  PlanArgs p{};
  p.s = *seqs;
  p.w = w;
  p.n_page = pool->n_page;
  p.page_rows = pool->page_rows;
  p.got = full;
  p.path = path;
  p.path_len = path_len;
  p.path_ld = path_ld;
  p.max_path = max_path;
  p.n_new = fresh->rows;
  plan_kernel<true><<<1, kPlan, 0, (hipStream_t)stream>>>(p);
  OP_LAUNCHED();
  CommitArgs a{};
  a.p = *pool;
  a.s = *seqs;
  a.w = w;
  a.tail = *tail;
  a.fresh = *fresh;
  a.kt = (char*)k_tail;
  a.vt = (char*)v_tail;
  a.kn = (const char*)k_new;
  a.vn = (const char*)v_new;
  a.path = path;
  a.path_ld = path_ld;
  a.window = window;
  a.sinks = sinks;
  a.fill = fill;
  by_type(tail->dtype, pool->head_dim, pool->code, [&](auto t, auto dim, auto code) {
    commit_kernel<decltype(t), dim.value, code.value><<<(unsigned)blocks, kThreads, 0, (hipStream_t)stream>>>(a);
  });
  OP_LAUNCHED();
  return SSD_OK;
}

extern "C" ssd_status ssd_pages_fork(const ssd_page_seqs* seqs, int32_t n_page, int32_t page_rows,
                                     const int32_t* parents, const ssd_rows_desc* tail, int32_t n_layer,
                                     int32_t n_kv_head, int32_t head_dim, void* k_tail, void* v_tail, void* stream) {
  OP_REQUIRE(n_page >= 1 && n_page <= kMaxPages, SSD_E_INVALID_ARG, "n_page outside [1, 2^20]");
  OP_REQUIRE(page_rows == 32 || page_rows == 64 || page_rows == 128, SSD_E_UNSUPPORTED,
             "page_rows must be 32, 64 or 128");
  OP_REQUIRE(head_dim == 32 || head_dim == 64 || head_dim == 128, SSD_E_UNSUPPORTED, "head_dim must be 32, 64 or 128");
  OP_REQUIRE(n_layer >= 1 && n_layer <= 4096 && n_kv_head >= 1 && n_kv_head <= 1024, SSD_E_INVALID_ARG,
             "n_layer outside [1, 4096] or n_kv_head outside [1, 1024]");
  ssd_status st = check_seqs(seqs, page_rows, true);
  if (st != SSD_OK) return st;
  OP_REQUIRE(parents && (uintptr_t)parents % 4 == 0, SSD_E_INVALID_ARG, "parents is null or not aligned");
  OP_REQUIRE(tail, SSD_E_INVALID_ARG, "null rows");
  OP_REQUIRE(tail->rows >= page_rows && tail->rows < (1 << 30), SSD_E_INVALID_ARG, "tail rows below page_rows, or 2^30");
  const RowDim td[4] = {{n_layer, tail->layer}, {seqs->n_seq, tail->seq}, {n_kv_head, tail->head}, {tail->rows, tail->row}};
  st = check_rows(tail->dtype, td, head_dim, true, k_tail, v_tail);
  if (st != SSD_OK) return st;
  const size_t te = rows_extent(tail->dtype, td, head_dim);
  OP_REQUIRE(!op_overlap(k_tail, te, v_tail, te), SSD_E_INVALID_ARG, "the tail's keys and values share memory");
  ForkArgs a{};
  a.s = *seqs;
  a.tail = *tail;
  a.n_page = n_page;
  a.page_rows = page_rows;
  a.n_layer = n_layer;
  a.n_kv_head = n_kv_head;
  a.row_shift = __builtin_ctz(head_dim * op_size(tail->dtype) / 16);
  a.parents = parents;
  a.kt = (char*)k_tail;
  a.vt = (char*)v_tail;
  fork_kernel<<<dim3(1 + 2 * n_layer, seqs->n_seq), kThreads, 0, (hipStream_t)stream>>>(a);
  OP_LAUNCHED();
  return SSD_OK;
}

extern "C" ssd_status ssd_pages_compact(const ssd_page_pool* pool, const ssd_page_seqs* seqs, int32_t* used,
                                        void* workspace, size_t workspace_bytes, void* stream) {
  ssd_status st = check_pool(pool);
  if (st == SSD_OK) st = check_seqs(seqs, pool->page_rows, true);
  if (st == SSD_OK) st = check_work(pool, seqs, workspace, workspace_bytes);
  if (st != SSD_OK) return st;
  OP_REQUIRE(used && (uintptr_t)used % 4 == 0, SSD_E_INVALID_ARG, "used is null or not aligned");
  CompactArgs a{};
  a.p = *pool;
  a.s = *seqs;
  a.w = work_at(workspace, seqs->n_seq, pool->n_page);
  a.used = used;
  compact_plan_kernel<<<1, kPlan, 0, (hipStream_t)stream>>>(a);
  OP_LAUNCHED();
  compact_move_kernel<<<2048, kThreads, 0, (hipStream_t)stream>>>(a);
  OP_LAUNCHED();
  return SSD_OK;
}
