// Embedding rows and the table's gradient (ssd_embed, ssd_embed_grad of
// ssd_ops.h).
//
//   out[n] = s W[tok_n],   dW[v] = s sum_{n: tok_n = v} g[n].
//
// The gradient sorts the positions by token (stable, so a token's terms are added
// in a fixed order), then walks the merged sequence
//   rows of token 0, end of 0, rows of token 1, end of 1, ...
// in which a position is a row of g to read and an end a row of dW to write.  It is cut
// into equal pieces whatever the tokens' frequencies.  A cut inside the rows of a
// token with few of them is moved behind its end; the rows of a frequent token
// are cut, its pieces leave partial sums, and a second kernel adds these up.  (Few
// positions of a small table: embed_grad_few_kernel, without the sort.)
// Bound: memory (g read once, dW written once).
#include <algorithm>

#include "ops_common.h"

namespace ssd {
namespace {

typedef unsigned u32x2 __attribute__((ext_vector_type(2)));
typedef unsigned u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
// callers' rows begin at any element
typedef unsigned u32x2_a2 __attribute__((ext_vector_type(2), aligned(2)));
typedef unsigned u32x4_a2 __attribute__((ext_vector_type(4), aligned(2)));
typedef float f32x4_a4 __attribute__((ext_vector_type(4), aligned(4)));

__device__ __forceinline__ f32x4 quad(const float* p) { return *(const f32x4_a4*)p; }
__device__ __forceinline__ f32x4 quad(const bf16_t* p) {
  const u32x2 r = *(const u32x2_a2*)p;
  return (f32x4){__uint_as_float(r[0] << 16), __uint_as_float(r[0] & 0xffff0000u), __uint_as_float(r[1] << 16),
                 __uint_as_float(r[1] & 0xffff0000u)};
}
// four columns of a row from column c on; the last ones of a row where fewer are left
__device__ __forceinline__ f32x4 load4(const float* row, int c, int d) {
  if (c + 4 <= d) return quad(row + c);
  f32x4 r = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int i = 0; i < 3; ++i)
    if (c + i < d) r[i] = row[c + i];
  return r;
}
__device__ __forceinline__ f32x4 load4(const bf16_t* row, int c, int d) {
  if (c + 4 <= d) return quad(row + c);
  f32x4 r = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int i = 0; i < 3; ++i)
    if (c + i < d) r[i] = op_ld(row, c + i);
  return r;
}
// LAST: the row is not used again here and need not stay in the caches
template <bool LAST = false>
__device__ __forceinline__ void store4(float* row, int c, int d, f32x4 v) {
  if (c + 4 <= d) {
    if (LAST) __builtin_nontemporal_store(v, (f32x4_a4*)(row + c));
    else *(f32x4_a4*)(row + c) = v;
  } else {
#pragma unroll
    for (int i = 0; i < 3; ++i)
      if (c + i < d) row[c + i] = v[i];
  }
}
template <bool LAST = false>
__device__ __forceinline__ void store4(bf16_t* row, int c, int d, f32x4 v) {
  typedef __bf16 b4 __attribute__((ext_vector_type(4)));
  if (c + 4 <= d) {
    const u32x2 r = __builtin_bit_cast(u32x2, __builtin_convertvector(v, b4));
    if (LAST) __builtin_nontemporal_store(r, (u32x2_a2*)(row + c));
    else *(u32x2_a2*)(row + c) = r;
  } else {
#pragma unroll
    for (int i = 0; i < 3; ++i)
      if (c + i < d) op_st(row, c + i, v[i]);
  }
}

// ---------------------------------------------------------------- lookup

// eight columns of a row from column c on, as floats
__device__ __forceinline__ void load8(const float* row, int c, int d, f32x4 (&v)[2]) {
  v[0] = load4(row, c, d);
  v[1] = load4(row, c + 4, d);
}
__device__ __forceinline__ void load8(const bf16_t* row, int c, int d, f32x4 (&v)[2]) {
  if (c + 8 <= d) {
    const u32x4 r = *(const u32x4_a2*)(row + c);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i >> 2][i & 3] = __uint_as_float(i & 1 ? r[i >> 1] & 0xffff0000u : r[i >> 1] << 16);
  } else {
    v[0] = load4(row, c, d);
    v[1] = load4(row, c + 4, d);
  }
}
__device__ __forceinline__ void store8(float* row, int c, int d, const f32x4 (&v)[2]) {
  store4(row, c, d, v[0]);
  store4(row, c + 4, d, v[1]);
}
__device__ __forceinline__ void store8(bf16_t* row, int c, int d, const f32x4 (&v)[2]) {
  typedef __bf16 b4 __attribute__((ext_vector_type(4)));
  if (c + 8 <= d) {
    const u32x2 a = __builtin_bit_cast(u32x2, __builtin_convertvector(v[0], b4));
    const u32x2 b = __builtin_bit_cast(u32x2, __builtin_convertvector(v[1], b4));
    *(u32x4_a2*)(row + c) = (u32x4){a[0], a[1], b[0], b[1]};
  } else {
    store4(row, c, d, v[0]);
    store4(row, c + 4, d, v[1]);
  }
}

// A thread per eight columns of a row.  Bound: memory (32768 rows of 1280 float32:
// 63 us, 5.3 TB/s).
template <typename T, typename O>
__global__ __launch_bounds__(256) void embed_rows_kernel(const int* __restrict__ tokens, int64_t parts, int per,
                                                         const T* __restrict__ table, int64_t ld_table, int V, int d,
                                                         float scale, O* __restrict__ out, int64_t ld_out) {
  const int64_t q = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (q >= parts) return;
  const int64_t n = q / per;
  const int c = 8 * (int)(q - n * per), tok = tokens[n];
  f32x4 v[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
  if (tok >= 0 && tok < V) {
    load8(table + (size_t)tok * ld_table, c, d, v);
    v[0] *= scale;
    v[1] *= scale;
  }
  store8(out + (size_t)n * ld_out, c, d, v);
}

// ---------------------------------------------------------------- sort by token

// The sort leaves most of the chip's bandwidth alone, and most rows of a table are zeros
// whatever the sort finds: its launches carry workgroups that clear the table's first
// rows (see fill_bytes), and embed_grad_kernel skips those of tokens that do not occur.
struct Fill {
  void* table;
  int64_t ld;      // bytes from row to row
  int row;         // bytes of a row
  int wide;        // rows begin and end at multiples of 16 bytes, else of 4
  int first, last; // rows
  int blocks;      // workgroups
};
// by a workgroup of `threads`, number b of f.blocks
template <typename U>
__device__ __forceinline__ void clear_by(const Fill& f, int b, int threads) {
  const int per = f.row / (int)sizeof(U), rows = (f.last - f.first + f.blocks - 1) / f.blocks;
  const int r0 = f.first + b * rows, n = min(rows, f.last - r0);
  char* table = (char*)f.table + (size_t)r0 * f.ld;
  const int down = threads / per, right = threads - down * per;
  for (int r = (int)threadIdx.x / per, c = (int)threadIdx.x - r * per; r < n;) {
    __builtin_nontemporal_store(U{}, (U*)(table + (size_t)r * f.ld) + c);
    r += down;
    c += right;
    if (c >= per) {
      c -= per;
      ++r;
    }
  }
}
__device__ __forceinline__ void clear_rows(const Fill& f, int b, int threads) {
  if (f.wide) clear_by<u32x4>(f, b, threads);
  else clear_by<unsigned>(f, b, threads);
}

// a token and its position; tokens outside the vocabulary sort last, as V
struct Entry {
  int key, pos;
};

__device__ __forceinline__ int key_of(int token, int V) { return token >= 0 && token < V ? token : V; }

// Not too many positions (see by_runs): sorted runs of kRun, then every entry's place
// among all.  Within a run an entry's rank is the number of those before it, counted by
// comparing all with all: a workgroup ranks 64 positions, one per lane, and its
// waves share out the others.  (16384 positions: 6.5 and 5.0 us.)
constexpr int kRun = 2048, kRankThreads = 1024;
__global__ __launch_bounds__(kRankThreads) void rank_kernel(const int* __restrict__ tokens, int N, int V,
                                                            Entry* __restrict__ out, Fill fill) {
  constexpr int W = kRankThreads / 64;
  const int blocks = (N + 63) / 64;
  if ((int)blockIdx.x >= blocks) return clear_rows(fill, blockIdx.x - blocks, kRankThreads);
  __shared__ __align__(16) int keys[kRun];
  __shared__ int count[W][64];
  const int t = threadIdx.x, lane = t & 63, w = t >> 6;
  const int b = blockIdx.x * 64 / kRun * kRun, n = min(kRun, N - b), n4 = (n + 3) / 4;  // the run
  for (int j = t; j < 4 * n4; j += kRankThreads) keys[j] = j < n ? key_of(tokens[b + j], V) : 0x7fffffff;
  __syncthreads();
  const int i0 = blockIdx.x * 64 - b, i = i0 + lane, key = i < n ? keys[i] : 0;
  const int per = (n4 + W - 1) / W, from = min(n4, w * per), to = min(n4, from + per);
  const int first4 = min(to, max(from, i0 / 4)), last4 = max(from, min(to, i0 / 4 + 16));
  const int4* k4 = (const int4*)keys;
  int c = 0;
#pragma unroll 4
  for (int j4 = from; j4 < first4; ++j4) {  // all before this workgroup's positions
    const int4 k = k4[j4];
    c += (k.x <= key) + (k.y <= key) + (k.z <= key) + (k.w <= key);
  }
  for (int j4 = first4; j4 < last4; ++j4) {
    const int4 k = k4[j4];
    const int j = 4 * j4;
    c += (k.x < key || (k.x == key && j < i)) + (k.y < key || (k.y == key && j + 1 < i)) +
         (k.z < key || (k.z == key && j + 2 < i)) + (k.w < key || (k.w == key && j + 3 < i));
  }
#pragma unroll 4
  for (int j4 = last4; j4 < to; ++j4) {  // all after
    const int4 k = k4[j4];
    c += (k.x < key) + (k.y < key) + (k.z < key) + (k.w < key);
  }
  count[w][lane] = c;
  __syncthreads();
  if (w == 0 && i < n) {
    int r = 0;
#pragma unroll
    for (int k = 0; k < W; ++k) r += count[k][lane];
    out[b + r] = (Entry){key, b + i};
  }
}

// An entry's place: its own in its run, and in every other run the number of
// lower keys, equal ones included in the runs before.  Eight threads an entry take
// the runs in turn.  (32768 positions: 9.2 us to rank, 8.7 to place.)
__global__ __launch_bounds__(256) void merge_runs_kernel(const Entry* __restrict__ in, int N, Entry* __restrict__ out,
                                                         Fill fill) {
  const int blocks = (N + 31) / 32;
  if ((int)blockIdx.x >= blocks) return clear_rows(fill, blockIdx.x - blocks, 256);
  const int e = (blockIdx.x * 256 + threadIdx.x) >> 3, sub = threadIdx.x & 7;
  const int i = min(e, N - 1), mine = i / kRun, runs = (N + kRun - 1) / kRun;
  const Entry x = in[i];
  int place = 0;
#pragma unroll 4
  for (int r = sub; r < runs; r += 8) {
    const Entry* s = in + (size_t)r * kRun;
    const int n = min(kRun, N - r * kRun), key = r < mine ? x.key : x.key - 1;  // entries up to key come before
    int lo = 0;
#pragma unroll
    for (int step = kRun; step > 0; step >>= 1)
      if (lo + step <= n && s[lo + step - 1].key <= key) lo += step;
    place += r == mine ? i - r * kRun : lo;
  }
#pragma unroll
  for (int o = 1; o < 8; o <<= 1) place += __shfl_xor(place, o);
  if (e < N && sub == 0) out[place] = x;
}

// More positions: a stable radix sort from the lowest digit up.  At most
// kSortBlocks workgroups each own a run of positions; a pass counts every
// run's digits, and a run's entries of digit x go behind all lower digits and
// the earlier runs' x.  Every pass counts by itself: counts taken while the pass
// before places its entries are atomics that a frequent token sends to one address
// (200000 positions, one in 16 the same token: 51 us a pass, 5 and 9 by itself).
constexpr int kDigitBits = 9, kBins = 1 << kDigitBits, kSortThreads = 1024, kSortBlocks = 256;

// positions of a run: as few sub-tiles of 2 per thread as keep the runs within kSortBlocks
constexpr int kSubTile = 2 * kSortThreads;
inline int sort_run(int N) {
  const int tiles = (N + kSubTile - 1) / kSubTile;
  return kSubTile * ((tiles + kSortBlocks - 1) / kSortBlocks);
}
inline int sort_passes(int V) {  // keys 0 .. V
  int bits = 1;
  while (V >> bits) ++bits;
  return (bits + kDigitBits - 1) / kDigitBits;
}

// Whether positions are sorted by runs.  The radix sort's time is its passes', two
// launches each; the runs' grows with the square of their number.  The whole gradient by
// runs and by radix (us): 50257 x 768, two passes, 16384 positions 57 and 65, 32768
// 66 and 66, 65536 118 and 101; 300000 x 128, three, 32768 48 and 57, 50000 69 and 66;
// 500 x 128, one, 3000 27 and 24.
inline bool by_runs(int N, int V) {
  const int passes = sort_passes(V);
  return N <= (passes == 1 ? kRun : 16384 * passes);
}

// every run's digits of a pass, from the tokens (in == nullptr) or entries
__global__ __launch_bounds__(kSortThreads) void count_kernel(const int* __restrict__ tokens,
                                                             const Entry* __restrict__ in, int N, int V, int run,
                                                             int pass, int* __restrict__ counts, int blocks,
                                                             Fill fill) {
  if ((int)blockIdx.x >= blocks) return clear_rows(fill, blockIdx.x - blocks, kSortThreads);
  __shared__ int bins[kBins];
  const int t = threadIdx.x, b = blockIdx.x, shift = pass * kDigitBits;
  if (t < kBins) bins[t] = 0;
  __syncthreads();
  const int to = min((int64_t)N, (int64_t)(b + 1) * run);
  for (int j = b * run + t; j < to; j += kSortThreads)
    atomicAdd(&bins[((in ? in[j].key : key_of(tokens[j], V)) >> shift) & (kBins - 1)], 1);
  __syncthreads();
  if (t < kBins) counts[(size_t)b * kBins + t] = bins[t];
}

// one pass: from the tokens (in == nullptr) or entries, to entries (200000 positions:
// 9.4 us, bound by the latency of its steps)
__global__ __launch_bounds__(kSortThreads) void place_kernel(const int* __restrict__ tokens,
                                                             const Entry* __restrict__ in, int N, int V, int run,
                                                             int pass, const int* __restrict__ counts,
                                                             Entry* __restrict__ out, int blocks, Fill fill) {
  if ((int)blockIdx.x >= blocks) return clear_rows(fill, blockIdx.x - blocks, kSortThreads);
  constexpr int W = kSortThreads / 64;
  __shared__ int base[kBins];       // where the run's next entry of a digit goes
  __shared__ int cnt[W][kBins];     // a sub-tile's entries of a digit, by wave; then their offsets
  __shared__ int wsum[kBins / 64];
  const int t = threadIdx.x, lane = t & 63, w = t >> 6, b = blockIdx.x;
  const int shift = pass * kDigitBits;
  // base: all lower digits, then the earlier runs' entries of this one
  int total = 0, before = 0;
  if (t < kBins) {
#pragma unroll 16
    for (int k = 0; k < blocks; ++k) {
      const int c = counts[(size_t)k * kBins + t];
      before += k < b ? c : 0;
      total += c;
    }
    int s = total;  // inclusive over the wave
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const int u = __shfl_up(s, o);
      if (lane >= o) s += u;
    }
    if (lane == 63) wsum[w] = s;
    base[t] = s - total + before;
  }
  __syncthreads();
  if (t < kBins)
    for (int k = 0; k < w; ++k) base[t] += wsum[k];
  const int end = min((int64_t)N, (int64_t)(b + 1) * run);
  for (int j0 = b * run; j0 < end; j0 += kSubTile) {
    for (int k = t; k < W * kBins; k += kSortThreads) ((int*)cnt)[k] = 0;
    __syncthreads();
    // wave w has 2 x 64 consecutive positions; equal digits of a wave find each other by ballots
    Entry e[2];
    int rank[2];
#pragma unroll
    for (int r = 0; r < 2; ++r) {
      const int j = j0 + w * 128 + r * 64 + lane;
      const bool in_run = j < end;
      if (in_run) e[r] = in ? in[j] : (Entry){key_of(tokens[j], V), j};
      else e[r] = (Entry){0, 0};
      const int dg = (e[r].key >> shift) & (kBins - 1);
      unsigned long long same = __builtin_amdgcn_ballot_w64(in_run);
#pragma unroll
      for (int k = 0; k < kDigitBits; ++k) {
        const unsigned long long m = __builtin_amdgcn_ballot_w64(dg >> k & 1);
        same &= dg >> k & 1 ? m : ~m;
      }
      const int lower = __builtin_popcountll(same & ((1ull << lane) - 1));
      rank[r] = cnt[w][dg] + lower;
      __builtin_amdgcn_wave_barrier();
      if (in_run && lower == 0) cnt[w][dg] += __builtin_popcountll(same);
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      __builtin_amdgcn_wave_barrier();
    }
    __syncthreads();
    if (t < kBins) {
      int s = base[t];
      for (int k = 0; k < W; ++k) {
        const int c = cnt[k][t];
        cnt[k][t] = s;
        s += c;
      }
      base[t] = s;
    }
    __syncthreads();
#pragma unroll
    for (int r = 0; r < 2; ++r) {
      const int j = j0 + w * 128 + r * 64 + lane;
      if (j < end) {
        const int to = cnt[w][(e[r].key >> shift) & (kBins - 1)] + rank[r];
        out[to] = e[r];
      }
    }
    __syncthreads();
  }
}

// ---------------------------------------------------------------- sums of the sorted rows

struct GradArgs {
  const Entry* sorted;
  int N, V, d, items, pieces;  // items of the merged sequence per piece
  const void* grad;
  int64_t ld_grad;
  void* dtable;
  int64_t ld_table;
  float scale;
  float *head, *tail;  // [pieces][d] partial sums
  int zeroed;          // the table's rows below are zeros already
  int* open;           // [pieces]: the token whose earlier terms are in the pieces before and that ends here, or -1
};

// The first of lo .. hi - 1 for which `before` (true up to some place) is false, or
// hi; by a whole wave, which looks at 64 places at a time.  Stops with a range
// of at most `near` places that holds it (or its end).
template <typename P>
__device__ __forceinline__ void narrow(int& lo, int& hi, int near, P before) {
  const int lane = threadIdx.x & 63;
  while (hi - lo > near) {
    const int step = (hi - lo + 63) / 64, j = lo + lane * step;
    const int k = __builtin_popcountll(__builtin_amdgcn_ballot_w64(j < hi && before(j)));
    if (k == 0) {
      hi = lo;
    } else {
      const int at = lo + (k - 1) * step;
      hi = min(hi, at + step);
      lo = at + 1;
    }
  }
}

constexpr int kInFlight = 8;  // rows in flight
// Entries in LDS, from place `base` on; others are read where they are.
constexpr int kStaged = 512;
struct Staged {
  const Entry* all;
  Entry* lds;
  int base, n;
  __device__ __forceinline__ Entry at(int j) const {
    const int k = j - base;
    return (unsigned)k < (unsigned)n ? lds[k] : all[j];
  }
  // by the whole workgroup
  __device__ __forceinline__ void stage(int from, int to) {
    base = from;
    n = min(kStaged, to - from);
    __syncthreads();
    for (int k = threadIdx.x; k < n; k += blockDim.x) lds[k] = all[from + k];
    __syncthreads();
  }
};

// A cut before entry i among the rows of token v, some of which come before it: if
// v has no more than kShort rows, how many come after it; else -1.  By a whole wave.
constexpr int kShort = 32;
__device__ __forceinline__ int rows_after(const Staged& s, int N, int i, int v) {
  const int j = i - 32 + (int)(threadIdx.x & 63);
  const unsigned long long same = __builtin_amdgcn_ballot_w64(j >= 0 && j < N && s.at(j).key == v);
  const int n = __builtin_popcountll(same);
  // (with kShort rows at most and one of them before the cut, all are seen)
  const bool more = i + 32 < N && same >> 63 && s.at(i + 32).key == v;
  const bool less = i > 32 && (same & 1) && s.at(i - 33).key == v;
  return n <= kShort && !more && !less ? __builtin_popcountll(same >> 32) : -1;
}

// The table written whole: a workgroup per piece, a thread per four columns (16384
// bfloat16 rows of 1280 to 50257 of float32: 52 us, 5.8 TB/s).
// CLEARED: rows below a.zeroed are zeros already.
template <typename G, typename T, bool CLEARED>
__global__ __launch_bounds__(1024) void embed_grad_kernel(GradArgs a) {
  constexpr int U = kInFlight;
  __shared__ Entry lds[kStaged];
  Staged es = {a.sorted, lds, 0, 0};
  const int g = blockIdx.x, c = 4 * (blockIdx.y * blockDim.x + threadIdx.x), lane = threadIdx.x & 63;
  // The piece is places t0 .. t1 - 1: entry j comes at place j + key_j, after as
  // many ends as there are lower tokens.  i0, v: the entries and ends before it;
  // i1, v1: before the next.  What is looked at around them is staged at once, the
  // entries themselves included unless they are many.
  const int64_t t0 = (int64_t)g * a.items, t1 = min(t0 + a.items, (int64_t)a.N + a.V);
  int lo = 0, hi = a.N;
  narrow(lo, hi, 64, [&](int j) { return (int64_t)a.sorted[j].key + j < t0; });
  lo = __builtin_amdgcn_readfirstlane(lo);
  hi = __builtin_amdgcn_readfirstlane(hi);
  es.stage(max(0, lo - 33), (int)min((int64_t)a.N, (int64_t)hi + a.items + 34));
  auto before = [&](int from, int to, int64_t t) {  // the first of from .. to at place t or behind
    narrow(from, to, 0, [&](int j) { return (int64_t)es.at(j).key + j < t; });
    return __builtin_amdgcn_readfirstlane(from);
  };
  int i0 = before(lo, hi, t0), v = (int)(t0 - i0);
  int i1 = before(i0, (int)min((int64_t)a.N, i0 + (t1 - t0)), t1), v1 = min((int)(t1 - i1), a.V);
  auto move = [&](int& i, int& end) {
    if (i == 0 || end >= a.V || __builtin_amdgcn_readfirstlane(es.at(i - 1).key) != end) return false;
    const int n = __builtin_amdgcn_readfirstlane(rows_after(es, a.N, i, end));
    if (n < 0) return true;  // the token's rows are cut here
    i += n;
    end += 1;
    return false;
  };
  bool cont = move(i0, v);  // earlier terms of v lie in pieces before
  move(i1, v1);
  const bool col = c < a.d;
  const G* grad = (const G*)a.grad;
  T* table = (T*)a.dtable;
  int opened = -1, terms = 0;  // terms: of v in this piece
  f32x4 acc = {0.f, 0.f, 0.f, 0.f};

  auto end = [&]() {  // the end of token v
    if (cont) {
      opened = v;
      if (col) store4(a.head + (size_t)g * a.d, c, a.d, acc);
    } else if (col) {
      // (a token that does not occur: 0 whatever the scale)
      store4<true>(table + (size_t)v * a.ld_table, c, a.d, terms ? a.scale * acc : acc);
    }
    cont = false;
    terms = 0;
    acc = (f32x4){0.f, 0.f, 0.f, 0.f};
  };

  // from v, or behind it: the next token up to `to` whose row is not zeros already
  auto skip = [&](int to) {
    if (CLEARED) v = max(v, min(to, a.zeroed));
  };

  for (int j0 = i0; j0 < i1; j0 += U) {
    if (min(j0 + U, i1) > es.base + es.n) es.stage(j0, i1);
    f32x4 r[U];
    int key[U];
    // (the entries first, a lane each: one read)
    const Entry e = es.at(min(j0 + (lane & (U - 1)), i1 - 1));
#pragma unroll
    for (int u = 0; u < U; ++u) {
      key[u] = j0 + u < i1 ? __builtin_amdgcn_readlane(e.key, u) : a.V;
      const int pos = __builtin_amdgcn_readlane(e.pos, u);
      r[u] = (f32x4){0.f, 0.f, 0.f, 0.f};
      if (col && key[u] < a.V) r[u] = load4(grad + (size_t)pos * a.ld_grad, c, a.d);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (key[u] >= a.V) continue;
      if (CLEARED && !cont && terms == 0) skip(key[u]);
      for (; v < key[u]; skip(key[u])) {
        end();
        ++v;
      }
      acc += r[u];
      ++terms;
    }
  }
  if (CLEARED && !cont && terms == 0) skip(v1);
  for (; v < v1; skip(v1)) {
    end();
    ++v;
  }
  if (terms && col) store4(a.tail + (size_t)g * a.d, c, a.d, acc);
  if (blockIdx.y == 0 && threadIdx.x == 0) a.open[g] = opened;
}

// The same, added to the table: a piece is a run of entries, and the rows of the
// table that end in it are loaded with the rows of the gradient (32768 bfloat16 rows of
// 1280 to 50257 of float32: 75 us).
template <typename G, typename T>
__global__ __launch_bounds__(1024) void embed_grad_add_kernel(GradArgs a) {
  constexpr int U = kInFlight;
  __shared__ Entry lds[kStaged];
  Staged es = {a.sorted, lds, 0, 0};
  const int g = blockIdx.x, c = 4 * (blockIdx.y * blockDim.x + threadIdx.x), lane = threadIdx.x & 63;
  int i0 = (int)min((int64_t)a.N, (int64_t)g * a.items), i1 = min(a.N, i0 + a.items);
  es.stage(max(0, i0 - 33), (int)min((int64_t)a.N, (int64_t)i1 + 34));
  auto move = [&](int& i) {  // see embed_grad_kernel
    if (i == 0 || i >= a.N) return false;
    const int key = __builtin_amdgcn_readfirstlane(es.at(i).key);
    if (key >= a.V || __builtin_amdgcn_readfirstlane(es.at(i - 1).key) != key) return false;
    const int n = __builtin_amdgcn_readfirstlane(rows_after(es, a.N, i, key));
    if (n < 0) return true;
    i += n;
    return false;
  };
  bool cont = move(i0);
  move(i1);
  const bool col = c < a.d;
  const G* grad = (const G*)a.grad;
  T* table = (T*)a.dtable;
  int opened = -1, terms = 0;
  f32x4 acc = {0.f, 0.f, 0.f, 0.f};
  for (int j0 = i0; j0 < i1; j0 += U) {
    // (and the entry after: the last one's token may end with it)
    if (min(min(j0 + U, i1) + 1, a.N) > es.base + es.n) es.stage(j0, min(a.N, i1 + 1));
    f32x4 r[U], old[U];
    int key[U];
    bool ends[U];
    const int j = j0 + (lane & (2 * U - 1));
    const Entry e = j <= i1 && j < a.N ? es.at(j) : (Entry){a.V, 0};
#pragma unroll
    for (int u = 0; u < U; ++u) {
      key[u] = j0 + u < i1 ? __builtin_amdgcn_readlane(e.key, u) : a.V;
      ends[u] = key[u] != __builtin_amdgcn_readlane(e.key, u + 1);
      const int pos = __builtin_amdgcn_readlane(e.pos, u);
      r[u] = old[u] = (f32x4){0.f, 0.f, 0.f, 0.f};
      if (col && key[u] < a.V) {
        r[u] = load4(grad + (size_t)pos * a.ld_grad, c, a.d);
        if (ends[u]) old[u] = load4(table + (size_t)key[u] * a.ld_table, c, a.d);
      }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (key[u] >= a.V) continue;
      acc += r[u];
      ++terms;
      if (!ends[u]) continue;
      if (cont) {
        opened = key[u];
        if (col) store4(a.head + (size_t)g * a.d, c, a.d, acc);
      } else if (col) {
        store4(table + (size_t)key[u] * a.ld_table, c, a.d, old[u] + a.scale * acc);
      }
      cont = false;
      terms = 0;
      acc = (f32x4){0.f, 0.f, 0.f, 0.f};
    }
  }
  if (terms && col) store4(a.tail + (size_t)g * a.d, c, a.d, acc);
  if (blockIdx.y == 0 && threadIdx.x == 0) a.open[g] = opened;
}

// Adds up the partial sums of the tokens that end in a piece and began before
// it.  A workgroup looks at kJoined pieces and 4 kJoinQuads columns; the pieces of
// one token are shared out over groups of threads that cover these.  Bound by the
// chain of loads for the most frequent token (the whole gradient of 16384 tokens of
// 50257 x 1280: 70 us, with rows whole in 1024 threads 73; of 200000 368 and 373).
constexpr int kJoined = 16, kJoinThreads = 512, kJoinQuads = 64;
template <typename T, bool ACC>
__global__ __launch_bounds__(kJoinThreads) void embed_join_kernel(GradArgs a) {
  __shared__ f32x4 part[kJoinThreads];
  const int t = threadIdx.x, lane = t & 63, g0 = blockIdx.x * kJoined;
  unsigned long long open =
      __builtin_amdgcn_ballot_w64(lane < kJoined && g0 + lane < a.pieces && a.open[g0 + lane] >= 0);
  const int q0 = blockIdx.y * kJoinQuads, nq = min(kJoinQuads, (a.d + 3) / 4 - q0), groups = kJoinThreads / nq,
            k = t / nq, c = 4 * (q0 + t - k * nq);
  for (; open; open &= open - 1) {
    const int g = g0 + __builtin_ctzll(open), v = a.open[g];
    int lo = 0, hi = a.N;  // the first entry of v
    narrow(lo, hi, 0, [&](int j) { return a.sorted[j].key < v; });
    const int from = (int)((ACC ? (int64_t)lo : (int64_t)lo + v) / a.items), n = g - from;
    f32x4 acc = {0.f, 0.f, 0.f, 0.f};
    if (k < groups) {
      const int to = from + (int)((int64_t)n * (k + 1) / groups);
#pragma unroll 8
      for (int i = from + (int)((int64_t)n * k / groups); i < to; ++i)
        acc += load4(a.tail + (size_t)i * a.d, c, a.d);
    }
    __syncthreads();
    part[t] = acc;
    __syncthreads();
    if (k == 0) {
      for (int i = 1; i < groups; ++i) acc += part[i * nq + t];
      acc += load4(a.head + (size_t)g * a.d, c, a.d);
      T* row = (T*)a.dtable + (size_t)v * a.ld_table;
      f32x4 r = a.scale * acc;
      if (ACC) r += load4(row, c, a.d);
      store4(row, c, a.d, r);
    }
  }
}

// ---------------------------------------------------------------- few positions

// Up to kFew positions and a small table: a wave per row of it and 256 columns looks
// all tokens through and adds the row's positions in their order.  One launch, no sort,
// nothing to join; bound by latency (200 tokens of 512 x 128 float32: 4.2 us).
constexpr int kFew = 256;
template <typename G, typename T, bool ACC>
__global__ __launch_bounds__(256) void embed_grad_few_kernel(GradArgs a, const int* __restrict__ tokens) {
  const int lane = threadIdx.x & 63, v = __builtin_amdgcn_readfirstlane(blockIdx.x * 4 + (threadIdx.x >> 6));
  if (v >= a.V) return;
  unsigned long long here[kFew / 64], any = 0;
#pragma unroll
  for (int g = 0; g < kFew / 64; ++g) {
    const int i = 64 * g + lane;
    any |= here[g] = __builtin_amdgcn_ballot_w64(i < a.N && tokens[min(i, a.N - 1)] == v);
  }
  if (ACC && !any) return;
  // (a row's last columns: its last four, of which the new ones are written)
  const int c = 4 * ((int)blockIdx.y * 64 + lane), at = min(c, a.d - 4);
  f32x4 sum = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int g = 0; g < kFew / 64; ++g) {
    const G* rows = (const G*)a.grad + (size_t)(64 * g) * a.ld_grad + at;
    unsigned long long m = here[g];
    if (m && !(m & (m - 1))) {
      sum += quad(rows + (size_t)__builtin_ctzll(m) * a.ld_grad);
      continue;
    }
    while (m) {  // eight in flight; past the last: the last again, not added
      f32x4 x[8];
      bool more[8];
      int n = 0;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        more[j] = m != 0;
        n = m ? __builtin_ctzll(m) : n;
        m &= m - 1;  // (0 stays 0)
        x[j] = quad(rows + (size_t)n * a.ld_grad);
      }
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (more[j]) sum += x[j];
    }
  }
  T* row = (T*)a.dtable + (size_t)v * a.ld_table;
  if (any) sum *= a.scale;  // (else 0 whatever the scale)
  if (ACC) sum += quad(row + at);
  if (at == c) {
    store4<!ACC>(row, c, c + 4, sum);
  } else {
#pragma unroll
    for (int i = 1; i < 4; ++i)
      if (at + i >= c) op_st(row, at + i, sum[i]);
  }
}

// threads of four columns each: whole waves, at most 1024
int grad_threads(int d) {
  const int quads = (d + 3) / 4;
  return quads >= 1024 ? 1024 : (quads + 63) / 64 * 64;
}

// Pieces of the merged sequence: one round of workgroups over the CUs (32 waves on
// each), or more where the table's rows are most of the traffic, a piece for every
// 32 KB of them: those at work then write to one stretch of the table that moves
// along (16384 tokens to 257 MB of float32: 64 us with 1536 pieces, 53 with 4096, 48
// with 8192; to 129 MB of bfloat16: 37 with 2048, 45 with 8192).  Fewer where a
// piece would have under 4 places or the partial sums over 64 MB.
int grad_pieces(int64_t places, int64_t table_bytes, int d) {
  const int64_t round = 256 * (32 * 64 / grad_threads(d));
  const int64_t most = std::min<int64_t>(8192, std::max<int64_t>(1024, (64 << 20) / (8 * (int64_t)d)));
  const int64_t want = std::min(std::max(round, table_bytes >> 15), most);
  return (int)std::min(want, std::max<int64_t>((places + 3) / 4, 1));
}

size_t round256(size_t x) { return (x + 255) / 256 * 256; }

// Bytes of the table that a launch of the sort clears: what it has time for.  Ranks of up to
// 8192 positions leave half of the CUs idle, the radix sort's launches wait for memory;
// the ranks of more positions need the whole chip, and small tables are soon written.  The
// whole gradient, bfloat16 to float32 without and with (us): 50257 x 1280, 1000
// positions 58 and 54, 16384 71.4 and 70.6 (not taken: 58.5 and 60 to bfloat16); 50257 x 768, 3000
// positions 49 and 43; 131072 x 450, 5000 positions 92 and 82; 131072 x 280 bfloat16, 70000
// positions 79 and 74 (24 MB a launch: 75).
constexpr int64_t kFillTable = 32 << 20, kFillBlock = 64 << 10;  // least table; bytes of a workgroup
int64_t fill_bytes(int n, int V) { return by_runs(n, V) ? (n <= 8192 ? 32 << 20 : 0) : 12 << 20; }

struct Layout {
  size_t entries[2], counts, head, tail, open, bytes;
  int pieces, blocks, run, passes;
};
Layout layout(int n, int vocab, int d) {
  Layout l{};
  size_t at = 0;
  auto take = [&](size_t b) {
    const size_t o = at;
    at += round256(b);
    return o;
  };
  l.pieces = grad_pieces((int64_t)n + vocab, (int64_t)vocab * d * 4, d);  // (no fewer than a call has)
  l.entries[0] = take((size_t)n * sizeof(Entry));
  if (n > kRun) l.entries[1] = take((size_t)n * sizeof(Entry));
  if (!by_runs(n, vocab)) {
    l.run = sort_run(n);
    l.blocks = (n + l.run - 1) / l.run;
    l.passes = sort_passes(vocab);
    l.counts = take((size_t)l.blocks * kBins * 4);
  }
  l.head = take((size_t)l.pieces * d * 4);
  l.tail = take((size_t)l.pieces * d * 4);
  l.open = take((size_t)l.pieces * 4);
  l.bytes = at;
  return l;
}

// Whether embed_grad_few_kernel takes a call.  A wave per row has to be less work than
// the sort saves: tables of up to 65536 waves.  Sorted and few (us), 200 tokens of
// Zipf frequencies, float32: 512 x 128 10.5 and 4.2, 8192 x 1024 12.8 and 9.8, 50257 x 128 12.9
// and 11.8; accumulated 10.6 and 4.4, 9.6 and 6.5, but 50257 x 1280 9.7 and 19.5.  256
// times one token, the worst: 512 x 128 12 and 16.
bool few(int n, int V, int d) {
  return n > 0 && n <= kFew && d >= 4 && (int64_t)V * ((d + 255) / 256) <= 65536;
}

template <typename G, typename T, bool ACC>
void launch_grad(const GradArgs& a, const int* tokens, hipStream_t s) {
  if (few(a.N, a.V, a.d)) {
    embed_grad_few_kernel<G, T, ACC><<<dim3((a.V + 3) / 4, (a.d + 255) / 256), 256, 0, s>>>(a, tokens);
    return;
  }
  const int quads = (a.d + 3) / 4, threads = grad_threads(a.d);
  const dim3 grid(a.pieces, (quads + threads - 1) / threads);
  if (ACC) embed_grad_add_kernel<G, T><<<grid, threads, 0, s>>>(a);
  else if (a.zeroed) embed_grad_kernel<G, T, true><<<grid, threads, 0, s>>>(a);
  else embed_grad_kernel<G, T, false><<<grid, threads, 0, s>>>(a);
  embed_join_kernel<T, ACC><<<dim3((a.pieces + kJoined - 1) / kJoined, (quads + kJoinQuads - 1) / kJoinQuads),
                              kJoinThreads, 0, s>>>(a);
}
template <typename G, typename T>
void launch_grad(const GradArgs& a, bool acc, const int* tokens, hipStream_t s) {
  if (acc) launch_grad<G, T, true>(a, tokens, s);
  else launch_grad<G, T, false>(a, tokens, s);
}
template <typename G>
void launch_grad(const GradArgs& a, int table_dtype, bool acc, const int* tokens, hipStream_t s) {
  if (table_dtype == SSD_F32) launch_grad<G, float>(a, acc, tokens, s);
  else launch_grad<G, bf16_t>(a, acc, tokens, s);
}

ssd_status check(int32_t n, int32_t vocab, int32_t d) {
  OP_REQUIRE(n >= 0 && n <= 1 << 24, SSD_E_INVALID_ARG, "n outside [0, 2^24]");
  OP_REQUIRE(vocab >= 1 && vocab <= 1 << 24, SSD_E_INVALID_ARG, "vocab outside [1, 2^24]");
  OP_REQUIRE(d >= 1 && d <= 65536, SSD_E_INVALID_ARG, "d outside [1, 65536]");
  return SSD_OK;
}

template <typename T>
void launch_embed_rows(int out_dtype, const int* tokens, int n, const void* table, int64_t ld_table, int V, int d,
                       float scale, void* out, int64_t ld_out, hipStream_t s) {
  const int per = (d + 7) / 8, slice = (1 << 30) / per;  // (a grid holds fewer than 2^32 threads)
  for (int first = 0; first < n; first += slice) {
    const int rows = std::min(n - first, slice);
    const int64_t parts = (int64_t)rows * per;
    const unsigned grid = (unsigned)((parts + 255) / 256);
    char* to = (char*)out + (size_t)first * ld_out * op_size(out_dtype);
    if (out_dtype == SSD_F32)
      embed_rows_kernel<<<grid, 256, 0, s>>>(tokens + first, parts, per, (const T*)table, ld_table, V, d, scale,
                                             (float*)to, ld_out);
    else
      embed_rows_kernel<<<grid, 256, 0, s>>>(tokens + first, parts, per, (const T*)table, ld_table, V, d, scale,
                                             (bf16_t*)to, ld_out);
  }
}

}  // namespace
}  // namespace ssd

using namespace ssd;

extern "C" ssd_status ssd_embed(ssd_dtype table_dtype, ssd_dtype out_dtype, const int32_t* tokens, int32_t n,
                                const void* table, int64_t ld_table, int32_t vocab, int32_t d, float scale, void* out,
                                int64_t ld_out, void* stream) {
  OP_REQUIRE(op_dtype(table_dtype) && op_dtype(out_dtype), SSD_E_INVALID_ARG, "dtype must be SSD_F32 or SSD_BF16");
  ssd_status st = check(n, vocab, d);
  if (st != SSD_OK) return st;
  OP_REQUIRE(ld_table >= d && ld_out >= d, SSD_E_INVALID_ARG, "a row stride is below d");
  if (n == 0) return SSD_OK;
  OP_REQUIRE(tokens && table && out, SSD_E_INVALID_ARG, "null argument");
  OP_REQUIRE((uintptr_t)table % op_size(table_dtype) == 0 && (uintptr_t)out % op_size(out_dtype) == 0,
             SSD_E_INVALID_ARG, "a pointer is not aligned to its type");
  OP_REQUIRE(op_apart(op_matrix(table, vocab, ld_table, d, op_size(table_dtype)),
                      op_matrix(out, n, ld_out, d, op_size(out_dtype))),
             SSD_E_INVALID_ARG, "out overlaps the table");
  if (table_dtype == SSD_F32)
    launch_embed_rows<float>(out_dtype, tokens, n, table, ld_table, vocab, d, scale, out, ld_out, (hipStream_t)stream);
  else
    launch_embed_rows<bf16_t>(out_dtype, tokens, n, table, ld_table, vocab, d, scale, out, ld_out,
                              (hipStream_t)stream);
  OP_LAUNCHED();
  return SSD_OK;
}

extern "C" ssd_status ssd_embed_grad_workspace(int32_t n, int32_t vocab, int32_t d, size_t* bytes) {
  OP_REQUIRE(bytes, SSD_E_INVALID_ARG, "null argument");
  ssd_status st = check(n, vocab, d);
  if (st != SSD_OK) return st;
  *bytes = layout(n, vocab, d).bytes;
  return SSD_OK;
}

extern "C" ssd_status ssd_embed_grad(ssd_dtype grad_dtype, ssd_dtype table_dtype, const int32_t* tokens, int32_t n,
                                     const void* grad, int64_t ld_grad, int32_t vocab, int32_t d, float scale,
                                     int32_t accumulate, void* dtable, int64_t ld_table, void* workspace,
                                     size_t workspace_bytes, void* stream) {
  OP_REQUIRE(op_dtype(grad_dtype) && op_dtype(table_dtype), SSD_E_INVALID_ARG, "dtype must be SSD_F32 or SSD_BF16");
  size_t need = 0;
  ssd_status st = ssd_embed_grad_workspace(n, vocab, d, &need);
  if (st != SSD_OK) return st;
  OP_REQUIRE(ld_grad >= d && ld_table >= d, SSD_E_INVALID_ARG, "a row stride is below d");
  OP_REQUIRE(dtable && workspace && (n == 0 || (tokens && grad)), SSD_E_INVALID_ARG, "null argument");
  OP_REQUIRE((uintptr_t)grad % op_size(grad_dtype) == 0 && (uintptr_t)dtable % op_size(table_dtype) == 0,
             SSD_E_INVALID_ARG, "a pointer is not aligned to its type");
  OP_REQUIRE(workspace_bytes >= need && (uintptr_t)workspace % 16 == 0, SSD_E_CAPACITY,
             "workspace below ssd_embed_grad_workspace's bytes or not 16-byte aligned");
  OP_REQUIRE(op_apart(op_matrix(grad, n, ld_grad, d, op_size(grad_dtype)),
                      op_matrix(dtable, vocab, ld_table, d, op_size(table_dtype))),
             SSD_E_INVALID_ARG, "dtable overlaps grad");
  if (n == 0 && accumulate) return SSD_OK;
  const Layout l = layout(n, vocab, d);
  char* ws = (char*)workspace;
  hipStream_t s = (hipStream_t)stream;
  Entry *sorted = (Entry*)(ws + l.entries[0]), *other = (Entry*)(ws + l.entries[1]);
  int zeroed = 0;
  auto share = [&](int64_t bytes) {  // of the table for the next launch to clear
    Fill f{};
    const int es = op_size(table_dtype);
    const uintptr_t at = (uintptr_t)dtable | (uintptr_t)(ld_table * es) | (uintptr_t)(d * es);
    if (accumulate || at % 4 != 0 || (int64_t)vocab * d * es < kFillTable) return f;
    f.table = dtable;
    f.ld = ld_table * es;
    f.row = d * es;
    f.wide = at % 16 == 0;
    f.first = zeroed;
    f.last = zeroed = (int)std::min<int64_t>(vocab, zeroed + bytes / f.row);
    f.blocks = (int)std::min<int64_t>(f.last - f.first, (int64_t)(f.last - f.first) * f.row / kFillBlock + 1);
    return f;
  };
  if (!by_runs(n, vocab)) {
    int* counts = (int*)(ws + l.counts);
    for (int p = 0; p < l.passes; ++p) {
      Entry* to = (l.passes - p) & 1 ? sorted : other;  // (the last pass ends in sorted)
      const Entry* from = p == 0 ? nullptr : to == sorted ? other : sorted;
      Fill f = share(fill_bytes(n, vocab));
      count_kernel<<<l.blocks + f.blocks, kSortThreads, 0, s>>>(tokens, from, n, vocab, l.run, p, counts, l.blocks, f);
      OP_LAUNCHED();
      f = share(fill_bytes(n, vocab));
      place_kernel<<<l.blocks + f.blocks, kSortThreads, 0, s>>>(tokens, from, n, vocab, l.run, p, counts, to, l.blocks,
                                                                f);
      OP_LAUNCHED();
    }
  } else if (n > 0 && !few(n, vocab, d)) {
    const bool one = n <= kRun;
    Fill f = share(fill_bytes(n, vocab));
    rank_kernel<<<(n + 63) / 64 + f.blocks, kRankThreads, 0, s>>>(tokens, n, vocab, one ? sorted : other, f);
    OP_LAUNCHED();
    if (!one) {
      f = share(fill_bytes(n, vocab));
      merge_runs_kernel<<<(n + 31) / 32 + f.blocks, 256, 0, s>>>(other, n, sorted, f);
      OP_LAUNCHED();
    }
  }
  const int64_t places = accumulate ? (int64_t)n : (int64_t)n + vocab;
  GradArgs a{};
  a.sorted = sorted;
  a.N = n;
  a.V = vocab;
  a.d = d;
  a.pieces = grad_pieces(places, accumulate ? 0 : (int64_t)vocab * d * op_size(table_dtype), d);
  a.items = (int)((places + a.pieces - 1) / a.pieces);
  a.pieces = (int)((places + a.items - 1) / a.items);
  a.grad = grad;
  a.ld_grad = ld_grad;
  a.dtable = dtable;
  a.ld_table = ld_table;
  a.scale = scale;
  a.zeroed = zeroed;
  a.head = (float*)(ws + l.head);
  a.tail = (float*)(ws + l.tail);
  a.open = (int*)(ws + l.open);
  if (grad_dtype == SSD_F32) launch_grad<float>(a, table_dtype, accumulate != 0, tokens, s);
  else launch_grad<bf16_t>(a, table_dtype, accumulate != 0, tokens, s);
  OP_LAUNCHED();
  return SSD_OK;
}
