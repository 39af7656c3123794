// Attention of drafted token trees over a paged cache.
#include <cmath>

#include "paged.cuh"

namespace prima {
namespace {

// One warp per (row, query head).  A lane takes one position of 32 at a time for the scores and D / 32 elements of the
// output for the second product; running maximum and sum in 32 bits.
template <typename T, typename Out, int D>
__global__ void __launch_bounds__(128) tree_simple_kernel(PoolView pool, BatchView b, int layer, const T* __restrict__ q, int n_q_heads, float scale_log2,
                                                          Out* __restrict__ out, float* __restrict__ lse) {
  const int lane = threadIdx.x & 31;
  const int64_t w = static_cast<int64_t>(blockIdx.x) * 4 + (threadIdx.x >> 5);
  const int t = static_cast<int>(w / n_q_heads), h = static_cast<int>(w % n_q_heads);
  __shared__ float s_q[4][D];
  if (t >= b.n_tok) return;
  const int s = seq_of_row(b, t, lane);
  if (s >= b.n_seq) return;
  const int first = __ldg(b.row_begin + s), end = __ldg(b.row_begin + s + 1), ctx = __ldg(b.ctx_len + s);
  if (first < 0 || t < first || end > b.n_tok || ctx < 0) {
    if (lane == 0) raise(pool.status, kBadRows);
    return;
  }
  float* my_q = s_q[threadIdx.x >> 5];
  for (int i = lane; i < D; i += 32) my_q[i] = Half2Of<T>::to_f(q[(static_cast<int64_t>(t) * n_q_heads + h) * D + i]) * scale_log2;
  __syncwarp();
  const int g = h / (n_q_heads / pool.n_kv_heads);
  const int64_t n = static_cast<int64_t>(ctx) + (end - first);
  float m = -INFINITY, sum = 0.f, acc[D / 32] = {};
  for (int64_t j0 = 0; j0 < n; j0 += 32) {
    const int64_t j = j0 + lane;
    bool seen = j < n;
    if (seen && j >= ctx) {
      const int a = static_cast<int>(j - ctx);
      seen = b.mask ? a < 64 * b.mask_words && (b.mask[static_cast<int64_t>(t) * b.mask_words + a / 64] >> (a % 64) & 1) : a <= t - first;
    }
    int64_t row = -1;
    if (seen) row = slot_row(pool, b.table + s * b.table_stride, b.table_stride, layer, j);
    if (row >= 0) row += static_cast<int64_t>(g) << pool.page_shift;
    float x = -INFINITY;
    if (row >= 0) {
      x = 0.f;
      for (int i = 0; i < D; i += 8) {
        float kk[8];
        load8(static_cast<const T*>(pool.k) + row * D + i, true, kk);
#pragma unroll
        for (int e = 0; e < 8; ++e) x += kk[e] * my_q[i + e];
      }
    }
    float top = x;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
    if (top == -INFINITY) continue;
    const float m_new = fmaxf(m, top), c = exp2f(m - m_new);
    const float p = exp2f(x - m_new);
    float ps = p;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) ps += __shfl_xor_sync(0xffffffffu, ps, o);
    sum = sum * c + ps;
    m = m_new;
#pragma unroll
    for (int e = 0; e < D / 32; ++e) acc[e] *= c;
    for (int i = 0; i < 32; ++i) {
      const int64_t r = __shfl_sync(0xffffffffu, row, i);
      const float pi = __shfl_sync(0xffffffffu, p, i);
      if (r < 0) continue;
#pragma unroll
      for (int e = 0; e < D / 32; ++e) acc[e] += pi * Half2Of<T>::to_f(static_cast<const T*>(pool.v)[r * D + 32 * e + lane]);
    }
  }
  const float inv = sum > 0.f ? 1.f / sum : 0.f;
#pragma unroll
  for (int e = 0; e < D / 32; ++e) out[(static_cast<int64_t>(t) * n_q_heads + h) * D + 32 * e + lane] = static_cast<Out>(acc[e] * inv);
  if (lse && lane == 0) lse[static_cast<int64_t>(t) * n_q_heads + h] = sum > 0.f ? (m + log2f(sum)) * 0.69314718055994531f : -INFINITY;
}

template <typename T, typename Out, int D>
cudaError_t launch_tree(const prima_paged& pool, const BatchView& b, int layer, const void* q, int n_q_heads, float scale, void* out, float* lse, cudaStream_t st) {
  const int64_t warps = static_cast<int64_t>(b.n_tok) * n_q_heads;
  tree_simple_kernel<T, Out, D><<<static_cast<unsigned>((warps + 3) / 4), 128, 0, st>>>(view_of(pool), b, layer, static_cast<const T*>(q), n_q_heads,
                                                                                     scale * 1.4426950408889634f, static_cast<Out*>(out), lse);
  return cudaGetLastError();
}

}  // namespace
}  // namespace prima

using namespace prima;

extern "C" {

int64_t prima_tree_attention_workspace(const prima_paged* p, int n_seq, int n_tok, int n_q_heads) {
  if (!p || n_seq < 1 || n_tok < 1 || n_q_heads < 1) return PRIMA_ERR_ARG;
  return 256;
}

int prima_tree_attention(prima_paged* p, int layer, const prima_paged_batch* batch, const void* q, int n_q_heads, float scale, void* out,
                         int out_dtype, float* lse, void* workspace, int64_t workspace_bytes, void* stream) {
  const int rc = check_batch(p, batch, "prima_tree_attention");
  if (rc != PRIMA_OK) return rc;
  const prima_paged_config& c = p->cfg;
  if (layer < 0 || layer >= c.n_layers) return call_fail(PRIMA_ERR_ARG, "prima_tree_attention: layer out of range");
  if (!q || !out) return call_fail(PRIMA_ERR_ARG, "prima_tree_attention: null q or out");
  if (n_q_heads < 1 || n_q_heads % c.n_kv_heads || n_q_heads / c.n_kv_heads > 64)
    return call_fail(PRIMA_ERR_ARG, "prima_tree_attention: n_q_heads must be a multiple of n_kv_heads, at most 64 times it");
  if (!(scale > 0.f) || std::isinf(scale)) return call_fail(PRIMA_ERR_ARG, "prima_tree_attention: scale must be positive and finite");
  if (out_dtype != PRIMA_DT_F32 && out_dtype != c.dtype) return call_fail(PRIMA_ERR_ARG, "prima_tree_attention: out_dtype is neither fp32 nor the cache's type");
  if ((reinterpret_cast<uintptr_t>(q) | reinterpret_cast<uintptr_t>(out)) & 15) return call_fail(PRIMA_ERR_ARG, "prima_tree_attention: q and out must be 16-byte aligned");
  if (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 255) || workspace_bytes < prima_tree_attention_workspace(p, batch->n_seq, batch->n_tok, n_q_heads))
    return call_fail(PRIMA_ERR_ARG, "prima_tree_attention: workspace too small or not 256-byte aligned");
  CallDevice dev(c.device);
  if (!dev.ok) return call_fail(PRIMA_ERR_CUDA, "cudaSetDevice failed");
  using launcher = cudaError_t (*)(const prima_paged&, const BatchView&, int, const void*, int, float, void*, float*, cudaStream_t);
  static const launcher table[2][2][2] = {{{launch_tree<__half, float, 64>, launch_tree<__half, float, 128>}, {launch_tree<__half, __half, 64>, launch_tree<__half, __half, 128>}},
                                          {{launch_tree<__nv_bfloat16, float, 64>, launch_tree<__nv_bfloat16, float, 128>},
                                           {launch_tree<__nv_bfloat16, __nv_bfloat16, 64>, launch_tree<__nv_bfloat16, __nv_bfloat16, 128>}}};
  const cudaError_t e = table[c.dtype == PRIMA_DT_BF16][out_dtype != PRIMA_DT_F32][c.head_dim == 128](*p, view_of(*batch), layer, q, n_q_heads, scale, out, lse,
                                                                                                   static_cast<cudaStream_t>(stream));
  return e == cudaSuccess ? PRIMA_OK : call_cuda_fail(e, "prima_tree_attention");
}

}  // extern "C"
