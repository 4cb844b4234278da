// Attention of a batch of sequences over a prefix they share and over their
// own rows (ssd_prefix_attn of ssd_ops.h).
#include "ops_common.h"

namespace ssd {
namespace {

struct PrefixAttnArgs {
  ssd_prefix_attn_desc d;
  const void *q, *kp, *vp, *ko, *vo;
  const int* own_len;
  void* out;
  float* lse;
};

// One wave per query and head: 64 keys at a time, a key's score per lane, then
// the output's dims over the lanes.
template <typename T>
__global__ __launch_bounds__(64) void prefix_attn_wave_kernel(PrefixAttnArgs a) {
  __shared__ float qs[128], ps[64];
  const ssd_prefix_attn_desc& d = a.d;
  const int lane = threadIdx.x, D = d.head_dim;
  const int h = blockIdx.x % d.n_head, bt = blockIdx.x / d.n_head, t = bt % d.n_query, b = bt / d.n_query;
  const int g = h / (d.n_head / d.n_kv_head);
  const T* q = (const T*)a.q + (int64_t)b * d.q_seq + (int64_t)t * d.q_row + (int64_t)h * d.q_head;
  T* out = (T*)a.out + (int64_t)b * d.out_seq + (int64_t)t * d.out_row + (int64_t)h * d.out_head;
  for (int i = lane; i < D; i += 64) qs[i] = op_ld(q, i) * d.scale;
  __syncthreads();
  const int n = a.own_len[b];
  const int P = n < 0 ? 0 : d.prefix_len;
  const int own = n < 0 ? 0 : max(0, min(n, d.own_rows) - d.n_query + 1 + t);
  float m = -INFINITY, l = 0.f, o0 = 0.f, o1 = 0.f;
  for (int part = 0; part < 2; ++part) {
    const T* k = part ? (const T*)a.ko + (int64_t)b * d.own_seq + (int64_t)g * d.own_head
                      : (const T*)a.kp + (int64_t)g * d.prefix_head;
    const T* v = part ? (const T*)a.vo + (int64_t)b * d.own_seq + (int64_t)g * d.own_head
                      : (const T*)a.vp + (int64_t)g * d.prefix_head;
    const int64_t row = part ? d.own_row : d.prefix_row;
    const int rows = part ? own : P;
    for (int j0 = 0; j0 < rows; j0 += 64) {
      const int j = j0 + lane;
      float x = -INFINITY;
      if (j < rows) {
        x = 0.f;
        for (int i = 0; i < D; ++i) x += qs[i] * op_ld(k + (int64_t)j * row, i);
      }
      float top = x;
      for (int o = 32; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor(top, o));
      top = fmaxf(m, top);
      const float ref = top == -INFINITY ? 0.f : top, c = __expf(m - ref), p = __expf(x - ref);
      float s = p;
      for (int o = 32; o > 0; o >>= 1) s += __shfl_xor(s, o);
      l = l * c + s;
      o0 *= c;
      o1 *= c;
      m = top;
      __syncthreads();
      ps[lane] = p;
      __syncthreads();
      for (int i = 0; i < min(64, rows - j0); ++i) {
        const T* vr = v + (int64_t)(j0 + i) * row;
        if (lane < D) o0 += ps[i] * op_ld(vr, lane);
        if (lane + 64 < D) o1 += ps[i] * op_ld(vr, lane + 64);
      }
    }
  }
  const float inv = P + own > 0 ? 1.f / l : 0.f;
  if (lane < D) op_st(out, lane, o0 * inv);
  if (lane + 64 < D) op_st(out, lane + 64, o1 * inv);
  if (a.lse && lane == 0) a.lse[blockIdx.x] = P + own > 0 ? m + logf(l) : -INFINITY;
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

}  // namespace
}  // namespace ssd

using namespace ssd;

extern "C" ssd_status ssd_prefix_attn_workspace(const ssd_prefix_attn_desc* a, size_t* bytes) {
  OP_REQUIRE(bytes, SSD_E_INVALID_ARG, "null argument");
  ssd_status st = check(a);
  if (st != SSD_OK) return st;
  *bytes = 16;
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
  const void* p[] = {q, k_prefix, v_prefix, k_own, v_own, out};
  for (const void* x : p) OP_REQUIRE((uintptr_t)x % 16 == 0, SSD_E_UNSUPPORTED, "a pointer is not 16-byte aligned");
  OP_REQUIRE(workspace_bytes >= need && (uintptr_t)workspace % 16 == 0, SSD_E_CAPACITY,
             "workspace below ssd_prefix_attn_workspace's bytes or not 16-byte aligned");
  PrefixAttnArgs args{*a, q, k_prefix, v_prefix, k_own, v_own, own_len, out, lse};
  const int rows = a->n_seq * a->n_query * a->n_head;
  if (a->dtype == SSD_F32) prefix_attn_wave_kernel<float><<<rows, 64, 0, (hipStream_t)stream>>>(args);
  else prefix_attn_wave_kernel<bf16_t><<<rows, 64, 0, (hipStream_t)stream>>>(args);
  OP_LAUNCHED();
  return SSD_OK;
}
