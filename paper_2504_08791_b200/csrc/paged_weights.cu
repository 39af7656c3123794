// The attention weight that cached positions receive in a step.
#include <algorithm>
#include <cmath>
#include <cstdio>

#include "paged_device.cuh"

namespace prima {
namespace {

struct WeightsArgs {
  PoolView pool;
  BatchView b;
  int layer, n_q_heads, group;
  float scale_log2, decay;
  const void* q;
  const float* lse;
  const float* weight_in;
  float* weight_out;
  int32_t* born;
  int64_t stride;
};

// One thread per position of a KV head: its key in registers, the rows one after the other.
template <typename T, int D>
__global__ void __launch_bounds__(128) weights_kernel(const __grid_constant__ WeightsArgs a, int64_t blocks) {
  pdl_trigger();
  pdl_wait();
  const int G = a.pool.n_kv_heads;
  for (int64_t w = blockIdx.x; w < blocks * G * a.b.n_seq; w += gridDim.x) {
    const int64_t block = w % blocks;
    const int head = static_cast<int>(w / blocks % G), s = static_cast<int>(w / blocks / G);
    const int first = a.b.row_begin[s], end = a.b.row_begin[s + 1], ctx = a.b.ctx_len[s];
    if (first < 0 || end < first || end > a.b.n_tok || ctx < 0) {
      raise(a.pool.status, kBadRows);
      continue;
    }
    const int64_t n = static_cast<int64_t>(ctx) + end - first, j = block * 128 + threadIdx.x;
    if (n > a.stride && end > first && block == 0) raise(a.pool.status, kBadSlot);
    if (j >= n || j >= a.stride || end == first) continue;
    const int64_t row = slot_row(a.pool, a.b.table + s * a.b.table_stride, a.b.table_stride, a.layer, j);
    float total = 0.f;
    if (row >= 0) {
      uint32_t k[D / 2];
      const uint4* src = reinterpret_cast<const uint4*>(static_cast<const T*>(a.pool.k) + (row + (static_cast<int64_t>(head) << a.pool.page_shift)) * D);
#pragma unroll
      for (int i = 0; i < D / 8; ++i) *(reinterpret_cast<uint4*>(k) + i) = __ldg(src + i);
      for (int t = first; t < end; ++t) {
        const long long i = j - ctx;
        const bool seen = i < 0 || (a.b.mask ? mask_word(reinterpret_cast<const uint32_t*>(a.b.mask + static_cast<int64_t>(t) * a.b.mask_words), 2 * a.b.mask_words, i >> 5) >> (i & 31) & 1
                                             : i <= t - first);
        if (!seen) continue;
        for (int h = 0; h < a.group; ++h) {
          const int64_t at = static_cast<int64_t>(t) * a.n_q_heads + head * a.group + h;
          const float lse = a.lse[at];
          if (lse == -INFINITY) continue;
          const uint32_t* q = reinterpret_cast<const uint32_t*>(static_cast<const T*>(a.q) + at * D);
          float x = 0.f;
#pragma unroll
          for (int d = 0; d < D / 2; ++d) {
            const float2 u = Half2Of<T>::unpack(__ldg(q + d)), v = Half2Of<T>::unpack(k[d]);
            x = fmaf(u.x, v.x, fmaf(u.y, v.y, x));
          }
          total += ex2(fmaf(x, a.scale_log2, -lse * kLog2e));
        }
      }
    }
    const int64_t at = (static_cast<int64_t>(s) * G + head) * a.stride + j;
    a.weight_out[at] = j < ctx && a.weight_in ? fmaf(a.decay, a.weight_in[at], total) : total;
    if (a.born && j >= ctx) {
      const int t = first + static_cast<int>(j - ctx);
      a.born[at] = a.b.pos ? a.b.pos[t] : static_cast<int>(j);
    }
  }
}

template <typename T, int D>
cudaError_t launch_weights(const prima_paged& pool, const WeightsArgs& a, cudaStream_t st) {
  const int64_t slots = std::min(a.stride, a.b.table_stride << pool.page_shift);
  return launch_pdl(weights_kernel<T, D>, dim3(pool.sm_count * 8), dim3(128), 0, st, a, (slots + 127) / 128);
}

}  // namespace
}  // namespace prima

using namespace prima;

extern "C" {

int prima_paged_weights(prima_paged* p, int layer, const prima_paged_batch* batch, const void* q, int n_q_heads, float scale, const float* lse,
                        const float* weight_in, float* weight_out, int32_t* born, int64_t stride, float decay, void* stream) {
  const int rc = check_batch(p, batch, "prima_paged_weights");
  if (rc != PRIMA_OK) return rc;
  auto refuse = [](const char* what) {
    char msg[160];
    snprintf(msg, sizeof msg, "prima_paged_weights: %s", what);
    return call_fail(PRIMA_ERR_ARG, msg);
  };
  const prima_paged_config& c = p->cfg;
  if (layer < 0 || layer >= c.n_layers) return refuse("layer out of range");
  if (!q || !lse || !weight_out) return refuse("null q, lse or weight_out");
  if (n_q_heads < 1 || n_q_heads % c.n_kv_heads || n_q_heads / c.n_kv_heads > 64) return refuse("n_q_heads must be a multiple of n_kv_heads, at most 64 times it");
  if (!(scale > 0.f) || std::isinf(scale)) return refuse("scale must be positive and finite");
  if (!(decay >= 0.f && decay <= 1.f)) return refuse("decay outside 0..1");
  if (stride < 1 || stride > 2147483647) return refuse("stride outside 1..2^31 - 1");
  if (!aligned_to(q, 16)) return refuse("q must be 16-byte aligned");
  if (!aligned_to(lse, 4) || !aligned_to(weight_in, 4) || !aligned_to(weight_out, 4) || !aligned_to(born, 4)) return refuse("an array is not 4-byte aligned");
  const int64_t bytes = 4 * static_cast<int64_t>(batch->n_seq) * c.n_kv_heads * stride;
  const char *in = reinterpret_cast<const char*>(weight_in), *to = reinterpret_cast<const char*>(weight_out);
  if (in && in != to && in < to + bytes && to < in + bytes) return refuse("weight_in overlaps weight_out without being it");
  CallDevice dev(c.device);
  if (!dev.ok) return call_fail(PRIMA_ERR_CUDA, "cudaSetDevice failed");
  WeightsArgs a;
  a.pool = view_of(*p);
  a.b = view_of(*batch);
  a.layer = layer;
  a.n_q_heads = n_q_heads;
  a.group = n_q_heads / c.n_kv_heads;
  a.scale_log2 = scale * kLog2e;
  a.decay = decay;
  a.q = q;
  a.lse = lse;
  a.weight_in = weight_in;
  a.weight_out = weight_out;
  a.born = born;
  a.stride = stride;
  using launcher = cudaError_t (*)(const prima_paged&, const WeightsArgs&, cudaStream_t);
  static const launcher table[2][2] = {{launch_weights<__half, 64>, launch_weights<__half, 128>}, {launch_weights<__nv_bfloat16, 64>, launch_weights<__nv_bfloat16, 128>}};
  const cudaError_t e = table[c.dtype == PRIMA_DT_BF16][c.head_dim == 128](*p, a, static_cast<cudaStream_t>(stream));
  return e == cudaSuccess ? PRIMA_OK : call_cuda_fail(e, "prima_paged_weights");
}

}  // extern "C"
