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
  int64_t stride, slots;     // slots: positions that the arrays have an entry for
};

// ---- the work ---------------------------------------------------------------------------------------------------------
// Positions are independent of one another, so nothing is joined: the blocks of kBlock positions of all (sequence, KV head)
// form one line, and every worker (a warp) takes an equal stretch of it.
struct WeightsWork {
  int seq, first, nodes, ctx, head;
  int64_t n;                 // positions that the sequence has an entry for
  int64_t block0, block1;
};
template <int kBlock>
struct WeightsCursor {
  const WeightsArgs& a;
  const int lane;
  int64_t total = 0, u = 0, u_end = 0, window = 0, before = 0, blocks = 0;
  int w0 = 0, first = 0, nodes = 0, ctx = 0;

  __device__ __forceinline__ int64_t positions(int64_t ctx_, int64_t nodes_) const { return min(ctx_ + nodes_, a.slots); }
  __device__ __forceinline__ bool read(int i) {
    const int f = __ldg(a.b.row_begin + i), e = __ldg(a.b.row_begin + i + 1), c = __ldg(a.b.ctx_len + i);
    const bool ok = f >= 0 && e >= f && e <= a.b.n_tok && c >= 0;
    first = f;
    nodes = ok ? e - f : 0;
    ctx = c;
    blocks = nodes ? (positions(c, nodes) + kBlock - 1) / kBlock * a.pool.n_kv_heads : 0;
    return ok;
  }
  __device__ void load(int64_t in_front) {
    blocks = 0;
    if (w0 + lane < a.b.n_seq) read(w0 + lane);
    int64_t x = blocks;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int64_t y = __shfl_up_sync(0xffffffffu, x, o);
      if (lane >= o) x += y;
    }
    before = in_front + x - blocks;
    window = in_front + __shfl_sync(0xffffffffu, x, 31);
  }
  __device__ WeightsCursor(const WeightsArgs& args, int lane_, int worker, int n_workers) : a(args), lane(lane_) {
    if (a.b.n_seq <= 32) {      // one window holds them all
      load(0);
      total = window;
    } else {
      for (int i = lane; i < a.b.n_seq; i += 32) {
        read(i);
        total += blocks;
      }
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) total += __shfl_xor_sync(0xffffffffu, total, o);
    }
    if (worker == 0)
      for (int i = lane; i < a.b.n_seq; i += 32) {
        if (!read(i)) raise(a.pool.status, kBadRows);
        else if (nodes && static_cast<int64_t>(ctx) + nodes > a.slots) raise(a.pool.status, kBadSlot);
      }
    const TreeShares shares = tree_shares(total, n_workers);
    u = tree_share_begin(shares, worker);
    u_end = tree_share_begin(shares, worker + 1);
    if (u < u_end) load(0);
  }
  __device__ bool next(WeightsWork* s) {
    if (u >= u_end) return false;
    unsigned hit;
    while (!(hit = __ballot_sync(0xffffffffu, u >= before && u < before + blocks))) {      // ends: u is below the total
      w0 += 32;
      load(window);
    }
    const int src = __ffs(hit) - 1;
    s->seq = w0 + src;
    s->first = __shfl_sync(0xffffffffu, first, src);
    s->nodes = __shfl_sync(0xffffffffu, nodes, src);
    s->ctx = __shfl_sync(0xffffffffu, ctx, src);
    s->n = positions(s->ctx, s->nodes);
    const int64_t at = u - __shfl_sync(0xffffffffu, before, src), per_head = (s->n + kBlock - 1) / kBlock;
    s->head = static_cast<int>(div_small(at, per_head));
    s->block0 = at - s->head * per_head;
    s->block1 = min(per_head, s->block0 + (u_end - u));
    u += s->block1 - s->block0;
    return true;
  }
};

// Whether row `node` of a sequence sees its row `i` (the position behind the context).
__device__ __forceinline__ bool sees(const WeightsArgs& a, int first, int node, int64_t i) {
  if (!a.b.mask) return i <= node;
  const uint32_t* words = reinterpret_cast<const uint32_t*>(a.b.mask + static_cast<int64_t>(first + node) * a.b.mask_words);
  return mask_word(words, 2 * a.b.mask_words, i >> 5) >> (i & 31) & 1;
}
// -lse in binary exponents; -infinity (its probabilities are 0) for a row that is none or sees nothing.
__device__ __forceinline__ float shift_of(const WeightsArgs& a, const WeightsWork& s, int64_t row) {
  if (row >= static_cast<int64_t>(s.nodes) * a.group) return -INFINITY;
  const int64_t node = row / a.group;
  const float lse = __ldg(a.lse + (s.first + node) * a.n_q_heads + s.head * a.group + (row - node * a.group));
  return lse == -INFINITY ? -INFINITY : -lse * kLog2e;
}
// What position j of the sequence has had, and where it is to be.
__device__ __forceinline__ int64_t entry_of(const WeightsArgs& a, const WeightsWork& s, int64_t j) {
  return (static_cast<int64_t>(s.seq) * a.pool.n_kv_heads + s.head) * a.stride + j;
}
__device__ __forceinline__ void put(const WeightsArgs& a, const WeightsWork& s, int64_t j, float had, float sum) {
  const int64_t at = entry_of(a, s, j);
  a.weight_out[at] = j < s.ctx && a.weight_in ? fmaf(a.decay, had, sum) : sum;
  if (a.born && j >= s.ctx) a.born[at] = a.b.pos ? __ldg(a.b.pos + s.first + (j - s.ctx)) : static_cast<int>(j);
}

// ---- few rows -----------------------------------------------------------------------------------------------------------
// Scores with the positions as rows of m16n8k16 products and the query rows as columns, S^T = K Q^T: a lane then holds
// scores of two positions, and the sum over the rows is one over its own columns and the quad.  Products do not mind in
// which order the D axis runs, as long as both operands agree: a lane takes 16 consecutive bytes of a key (and of a query)
// as its part of two products, so that keys go from memory into operands with wide loads and without shared memory.
// A warp keeps kTiles * 8 rows of queries and takes 16 positions at a time, the next 16 on their way; where a sequence has
// more rows, it reads its queries again for every 16 positions (all sums of a position before what it had is added, which
// may be larger than all of them).
constexpr int weights_ctas(int dim, int tiles) { return dim == 128 ? (tiles == 1 ? 4 : 2) : (tiles == 4 ? 3 : 4); }      // per SM: what the registers allow
template <typename T, int D, int kTiles>
__global__ void __launch_bounds__(128, weights_ctas(D, kTiles)) weights_stream_kernel(const __grid_constant__ WeightsArgs a) {
  constexpr bool kBf16 = !__is_same(T, __half);
  constexpr int kChunks = D / 32;      // 16-byte pieces of a row that a lane takes
  const int lane = threadIdx.x & 31, g = lane >> 2, t4 = lane & 3;
  pdl_trigger();
  pdl_wait();
  WeightsCursor<16> cursor(a, lane, (blockIdx.x * 128 + threadIdx.x) >> 5, gridDim.x * 4);
  WeightsWork s;
  while (cursor.next(&s)) {
    const int64_t rows = static_cast<int64_t>(s.nodes) * a.group;
    const int32_t* const table = a.b.table + s.seq * a.b.table_stride;
    const T* const keys = static_cast<const T*>(a.pool.k) + (static_cast<int64_t>(s.head) << a.pool.page_shift) * D;
    const float* const had_from = a.weight_in ? a.weight_in + entry_of(a, s, 0) : nullptr;
    uint4 q[kTiles][kChunks];
    float shift[kTiles][2];
    auto load_queries = [&](int64_t row0) {
#pragma unroll
      for (int n = 0; n < kTiles; ++n) {
        const int64_t row = row0 + 8 * n + g, node = row / a.group;
        const T* src = static_cast<const T*>(a.q) + ((s.first + node) * a.n_q_heads + s.head * a.group + (row - node * a.group)) * D;
#pragma unroll
        for (int c = 0; c < kChunks; ++c) q[n][c] = row < rows ? __ldg(reinterpret_cast<const uint4*>(src) + t4 + 4 * c) : make_uint4(0, 0, 0, 0);
#pragma unroll
        for (int e = 0; e < 2; ++e) shift[n][e] = shift_of(a, s, row0 + 8 * n + 2 * t4 + e);
      }
    };
    struct Keys {
      uint4 k[2][kChunks];
      float had;
      int bad;             // bits: position has no key
    };
    // Positions 16 block + g and + 8: pages hold at least 8 positions, so each of the two lies in one page with its
    // seven neighbours.
    auto load = [&](int64_t block, Keys& x) {
      x.bad = 0;
      x.had = 0.f;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int64_t j = block * 16 + 8 * h + g;
        int64_t row = -1;
        if (block < s.block1 && j < s.n) {
          row = find_slot(a.pool, table, a.b.table_stride, a.layer, j);
          if (row < 0) raise(a.pool.status, static_cast<int>(-row));
        }
        x.bad |= row < 0 ? 1 << h : 0;
        const uint4* src = reinterpret_cast<const uint4*>(keys + row * D);
#pragma unroll
        for (int c = 0; c < kChunks; ++c) x.k[h][c] = row >= 0 ? __ldg(src + t4 + 4 * c) : make_uint4(0, 0, 0, 0);
        if (t4 == h && had_from && block < s.block1 && j < min(s.n, static_cast<int64_t>(s.ctx))) x.had = had_from[j];
      }
    };
    const bool again = rows > 8 * kTiles;
    Keys next;
    load(s.block0, next);
    load_queries(0);
#pragma unroll 1
    for (int64_t block = s.block0; block < s.block1; ++block) {
      const Keys x = next;
      load(block + 1, next);
      float sum[2] = {0.f, 0.f};
      const bool edge = __any_sync(0xffffffffu, x.bad != 0) || block * 16 + 16 > s.ctx;
#pragma unroll 1
      for (int64_t row0 = 0; row0 < rows; row0 += 8 * kTiles) {
        if (again) load_queries(row0);
#pragma unroll
        for (int n = 0; n < kTiles; ++n) {
          float c[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int k = 0; k < kChunks; ++k) {
            const uint32_t lo[4] = {x.k[0][k].x, x.k[1][k].x, x.k[0][k].y, x.k[1][k].y}, hi[4] = {x.k[0][k].z, x.k[1][k].z, x.k[0][k].w, x.k[1][k].w};
            mma16816<kBf16>(c, lo, q[n][k].x, q[n][k].y);
            mma16816<kBf16>(c, hi, q[n][k].z, q[n][k].w);
          }
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            float p = ex2(fmaf(c[e], a.scale_log2, shift[n][e & 1]));
            if (edge) {
              const int64_t row = row0 + 8 * n + 2 * t4 + (e & 1), i = block * 16 + 8 * (e >> 1) + g - s.ctx;
              if ((x.bad >> (e >> 1) & 1) || shift[n][e & 1] == -INFINITY || (i >= 0 && !sees(a, s.first, static_cast<int>(row / a.group), i))) p = 0.f;
            }
            sum[e >> 1] += p;
          }
        }
      }
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        sum[h] += __shfl_xor_sync(0xffffffffu, sum[h], 1);
        sum[h] += __shfl_xor_sync(0xffffffffu, sum[h], 2);
      }
      if (t4 < 2) {
        const int64_t j = block * 16 + 8 * t4 + g;
        if (j < s.n) put(a, s, j, x.had, t4 ? sum[1] : sum[0]);
      }
    }
  }
}

template <typename T, int D, int kTiles>
cudaError_t launch_stream(const prima_paged& pool, const WeightsArgs& a, cudaStream_t st) {
  return launch_pdl(weights_stream_kernel<T, D, kTiles>, dim3(pool.sm_count * weights_ctas(D, kTiles)), dim3(128), 0, st, a);
}
template <typename T, int D>
cudaError_t launch_weights(const prima_paged& pool, const WeightsArgs& a, cudaStream_t st) {
  // Rows that a KV head has of a sequence on average; each variant is right for any.
  const int64_t rows = (static_cast<int64_t>(a.b.n_tok) + a.b.n_seq - 1) / a.b.n_seq * a.group;
  return (rows <= 8 ? launch_stream<T, D, 1> : rows <= 16 ? launch_stream<T, D, 2> : launch_stream<T, D, 4>)(pool, a, st);
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
  a.stride = a.slots = stride;
  using launcher = cudaError_t (*)(const prima_paged&, const WeightsArgs&, cudaStream_t);
  static const launcher table[2][2] = {{launch_weights<__half, 64>, launch_weights<__half, 128>}, {launch_weights<__nv_bfloat16, 64>, launch_weights<__nv_bfloat16, 128>}};
  const cudaError_t e = table[c.dtype == PRIMA_DT_BF16][c.head_dim == 128](*p, a, static_cast<cudaStream_t>(stream));
  return e == cudaSuccess ? PRIMA_OK : call_cuda_fail(e, "prima_paged_weights");
}

}  // extern "C"
