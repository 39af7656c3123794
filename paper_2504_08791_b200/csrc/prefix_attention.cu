// Attention of a batch whose sequences share long prefixes.
#include <cmath>
#include <cstdio>

#include "paged_device.cuh"

namespace prima {
namespace {

struct PrefixView {
  int n;
  const int32_t* seq_begin;
  const int32_t* len;
  const int32_t* table;
  int64_t table_stride;
};

struct PrefixArgs {
  PoolView pool;
  BatchView b;
  PrefixView prefix;
  int layer, n_q_heads, group;
  float scale_log2;
  const void* q;
  void* out;
  float* lse;
};

// One warp per row and query head, one position at a time.
template <typename T, typename Out, int D>
__global__ void __launch_bounds__(128) prefix_rows_kernel(const __grid_constant__ PrefixArgs a) {
  pdl_trigger();
  pdl_wait();
  const int lane = threadIdx.x & 31;
  constexpr int kE = D / 32;
  const int64_t n = static_cast<int64_t>(a.b.n_tok) * a.n_q_heads;
  for (int64_t w = (static_cast<int64_t>(blockIdx.x) * 128 + threadIdx.x) / 32; w < n; w += static_cast<int64_t>(gridDim.x) * 4) {
    const int t = static_cast<int>(w / a.n_q_heads), h = static_cast<int>(w % a.n_q_heads), head = h / a.group;
    const int s = seq_of_row(a.b, t, lane);
    if (s >= a.b.n_seq) continue;
    const int first = a.b.row_begin[s], end = a.b.row_begin[s + 1], ctx = a.b.ctx_len[s];
    if (first < 0 || t < first || end > a.b.n_tok || ctx < 0) {
      raise(a.pool.status, kBadRows);
      continue;
    }
    float q[kE], o[kE], m = -INFINITY, sum = 0.f;
    for (int e = 0; e < kE; ++e) {
      q[e] = static_cast<float>(static_cast<const T*>(a.q)[w * D + kE * lane + e]);
      o[e] = 0.f;
    }
    auto take = [&](const int32_t* table, int64_t stride, int64_t slot) {
      const int64_t row = slot_row(a.pool, table, stride, a.layer, slot);
      if (row < 0) return;
      const int64_t at = (row + (static_cast<int64_t>(head) << a.pool.page_shift)) * D + kE * lane;
      float x = 0.f;
      for (int e = 0; e < kE; ++e) x = fmaf(q[e], static_cast<float>(static_cast<const T*>(a.pool.k)[at + e]), x);
      for (int d = 16; d > 0; d >>= 1) x += __shfl_xor_sync(0xffffffffu, x, d);
      x *= a.scale_log2;
      const float top = fmaxf(m, x), f = m == -INFINITY ? 0.f : ex2(m - top), p = x == -INFINITY ? 0.f : ex2(x - top);
      m = top;
      sum = sum * f + p;
      for (int e = 0; e < kE; ++e) o[e] = o[e] * f + p * static_cast<float>(static_cast<const T*>(a.pool.v)[at + e]);
    };
    for (int p = 0; p < a.prefix.n; ++p) {
      const int b0 = a.prefix.seq_begin[p], b1 = a.prefix.seq_begin[p + 1], len = a.prefix.len[p];
      if (b0 < 0 || b1 < b0 || b1 > a.b.n_seq || len < 0) {
        raise(a.pool.status, kBadRows);
        continue;
      }
      if (s < b0 || s >= b1) continue;
      for (int j = 0; j < len; ++j) take(a.prefix.table + p * a.prefix.table_stride, a.prefix.table_stride, j);
      break;
    }
    const int32_t* table = a.b.table + s * a.b.table_stride;
    for (int64_t j = 0; j < static_cast<int64_t>(ctx) + end - first; ++j) {
      const long long i = j - ctx;
      const bool seen = i < 0 || (a.b.mask ? mask_word(reinterpret_cast<const uint32_t*>(a.b.mask + static_cast<int64_t>(t) * a.b.mask_words), 2 * a.b.mask_words, i >> 5) >> (i & 31) & 1
                                           : i <= t - first);
      if (seen) take(table, a.b.table_stride, j);
    }
    const float inv = inverse_of(sum);
    for (int e = 0; e < kE; ++e) static_cast<Out*>(a.out)[w * D + kE * lane + e] = static_cast<Out>(o[e] * inv);
    if (a.lse && lane == 0) a.lse[w] = sum == 0.f ? -INFINITY : (m + log2f(sum)) * kLn2;
  }
}

template <typename T, typename Out, int D>
cudaError_t launch_prefix(const prima_paged& pool, const PrefixArgs& a, cudaStream_t st) {
  return launch_pdl(prefix_rows_kernel<T, Out, D>, dim3(pool.sm_count * 16), dim3(128), 0, st, a);
}

}  // namespace
}  // namespace prima

using namespace prima;

extern "C" {

int64_t prima_prefix_attention_workspace(const prima_paged* p, int n_seq, int n_tok, int n_q_heads) {
  if (!p || n_seq < 1 || n_tok < 1 || n_q_heads < 1) return PRIMA_ERR_ARG;
  return 256;
}

int prima_prefix_attention(prima_paged* p, int layer, const prima_paged_batch* batch, const prima_prefix* prefix, const void* q, int n_q_heads,
                           float scale, void* out, int out_dtype, float* lse, void* workspace, int64_t workspace_bytes, void* stream) {
  const int rc = check_batch(p, batch, "prima_prefix_attention");
  if (rc != PRIMA_OK) return rc;
  auto refuse = [](const char* what) {
    char msg[160];
    snprintf(msg, sizeof msg, "prima_prefix_attention: %s", what);
    return call_fail(PRIMA_ERR_ARG, msg);
  };
  const prima_paged_config& c = p->cfg;
  if (layer < 0 || layer >= c.n_layers) return refuse("layer out of range");
  if (!prefix || prefix->n_prefix < 1 || !prefix->seq_begin || !prefix->len || !prefix->table) return refuse("a prefix with seq_begin, len and table is needed");
  if (prefix->table_stride < 1 || prefix->table_stride > 2147483647) return refuse("the prefix's table_stride is out of range");
  if (!aligned_to(prefix->seq_begin, 4) || !aligned_to(prefix->len, 4) || !aligned_to(prefix->table, 4)) return refuse("an array of the prefix is not 4-byte aligned");
  if (!q || !out) return refuse("null q or out");
  if (n_q_heads < 1 || n_q_heads % c.n_kv_heads || n_q_heads / c.n_kv_heads > 64) return refuse("n_q_heads must be a multiple of n_kv_heads, at most 64 times it");
  if (!(scale > 0.f) || std::isinf(scale)) return refuse("scale must be positive and finite");
  if (out_dtype != PRIMA_DT_F32 && out_dtype != c.dtype) return refuse("out_dtype is neither fp32 nor the cache's type");
  if (!aligned_to(q, 16) || !aligned_to(out, 16)) return refuse("q and out must be 16-byte aligned");
  if (!aligned_to(lse, 4)) return refuse("lse must be 4-byte aligned");
  if (!workspace || !aligned_to(workspace, 256) || workspace_bytes < prima_prefix_attention_workspace(p, batch->n_seq, batch->n_tok, n_q_heads))
    return refuse("workspace too small or not 256-byte aligned");
  CallDevice dev(c.device);
  if (!dev.ok) return call_fail(PRIMA_ERR_CUDA, "cudaSetDevice failed");
  PrefixArgs a;
  a.pool = view_of(*p);
  a.b = view_of(*batch);
  a.prefix = {prefix->n_prefix, prefix->seq_begin, prefix->len, prefix->table, prefix->table_stride};
  a.layer = layer;
  a.n_q_heads = n_q_heads;
  a.group = n_q_heads / c.n_kv_heads;
  a.scale_log2 = scale * kLog2e;
  a.q = q;
  a.out = out;
  a.lse = lse;
  using launcher = cudaError_t (*)(const prima_paged&, const PrefixArgs&, cudaStream_t);
  static const launcher table[2][2][2] = {{{launch_prefix<__half, float, 64>, launch_prefix<__half, float, 128>}, {launch_prefix<__half, __half, 64>, launch_prefix<__half, __half, 128>}},
                                          {{launch_prefix<__nv_bfloat16, float, 64>, launch_prefix<__nv_bfloat16, float, 128>},
                                           {launch_prefix<__nv_bfloat16, __nv_bfloat16, 64>, launch_prefix<__nv_bfloat16, __nv_bfloat16, 128>}}};
  const cudaError_t e = table[c.dtype == PRIMA_DT_BF16][out_dtype != PRIMA_DT_F32][c.head_dim == 128](*p, a, static_cast<cudaStream_t>(stream));
  return e == cudaSuccess ? PRIMA_OK : call_cuda_fail(e, "prima_prefix_attention");
}

}  // extern "C"
