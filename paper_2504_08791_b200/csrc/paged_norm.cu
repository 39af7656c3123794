// Rotation and append of a step's rows with a norm of every query and key head in front.
//
//   y = gain * x / sqrt(mean x^2 + eps);  (y_a, y_b) of pair i turned by the angle p[axis i] * frequency[rank i]
//
// Rows are read and written once: bound by the copy (11,500 rows of prompts, 40 query and 8 KV heads of 128: 72 us, floor 50),
// a few rows by the latency of looking their place up (one row 4.6 us).  Tried for many rows and slower: 24 resident warps
// per SM by fewer registers 77 us, sines in shared memory 80, two or four warps a row 86 and 113.
#include <algorithm>
#include <cmath>
#include <cstdio>

#include "paged.cuh"

namespace prima {
namespace {

struct HeadNorm {
  const float* q_gain;
  const float* k_gain;
  int64_t q_gain_stride, k_gain_stride;
  float eps;
  bool wide;                   // gains may be read 16 bytes at a time
  const int32_t* positions;
  uint8_t axis[64], rank[64];
};

// As append_kernel (paged.cu): kWarps warps take one row, a lane owns the same 16 elements of every head that it takes, so
// that sines and gains stay in its registers, and a warp takes 32 / (D/16) heads at a time.  A head is multiplied by
// gain / sqrt(mean x^2 + eps) and then turned; its lanes hold it whole, so the sum of squares is one butterfly over D / 16
// lanes.  Pair i is turned by the position on its own axis, as a fraction of a turn in 64 bits.
template <typename T, typename In, int D, int kWarps, int kMode>
__global__ void __launch_bounds__(256) norm_kernel(PoolView pool, BatchView b, int layer, const In* q, const In* k, const In* v, int n_q_heads,
                                                   int64_t q_stride, int64_t k_stride, int64_t v_stride, bool wide, const double* __restrict__ freq, T* __restrict__ q_out,
                                                   const __grid_constant__ HeadNorm norm) {
  constexpr int kPairs = D / 2, kItems = D / 16, kHeads = 32 / kItems, kStep = kWarps * kHeads;
  // Elements of a head that a lane owns: 8 c .. and D/2 + 8 c .. (mode 0), or 16 c .. 16 c + 15
  constexpr int kGap = kMode == 0 ? kPairs : 8, kWide = kMode == 0 ? 8 : 16;
  __shared__ __align__(16) float2 s_cs[8][kPairs];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int t = static_cast<int>((static_cast<int64_t>(blockIdx.x) * 8 + warp) / kWarps);
  const int c = lane % kItems, G = pool.n_kv_heads, turned = n_q_heads + G, heads = turned + G;
  if (t >= b.n_tok) return;
  pdl_trigger();
  pdl_wait();
  const In* const q_row = q ? q + t * q_stride : nullptr;
  const In* const k_row = k + t * k_stride;
  const In* const v_row = v + t * v_stride;
  struct Item { Raw8<In> lo, hi; };
  // 11,500 rows of prompts: past L1 71.6 us, through it 73.7
  auto load = [&](int h, Item& x) {
    if (h >= heads || (h < n_q_heads && !q)) return;
    if (h < turned) {
      const In* src = (h < n_q_heads ? q_row + h * D : k_row + (h - n_q_heads) * D) + kWide * c;
      load8<Path::kL2>(src, wide, x.lo);
      load8<Path::kL2>(src + kGap, wide, x.hi);
    } else {
      const In* src = v_row + (h - turned) * D + 16 * c;
      load8<Path::kL2>(src, wide, x.lo);
      load8<Path::kL2>(src + 8, wide, x.hi);
    }
  };
  int h = (warp % kWarps) * kHeads + lane / kItems;
  Item x[2];
  load(h, x[0]);                       // in flight while the place is looked up
  load(h + kStep, x[1]);

  const int s = seq_of_row(b, t, lane);
  if (s >= b.n_seq) return;            // padding
  const int first = b.row_begin[s], ctx = b.ctx_len[s];
  if (t < first || first < 0 || ctx < 0) {
    if (lane == 0) raise(pool.status, kBadRows);
    return;
  }
  const int64_t slot = static_cast<int64_t>(ctx) + (t - first);
  int64_t row = lane == 0 ? slot_row(pool, b.table + s * b.table_stride, b.table_stride, layer, slot) : 0;
  for (int i = lane; i < kPairs; i += 32) {
    const int axis = norm.axis[i];
    int p = 0;                         // not turned: by an angle of 0
    if (axis != PRIMA_AXIS_NONE) p = norm.positions ? norm.positions[static_cast<int64_t>(axis) * b.n_tok + t] : b.pos ? b.pos[t] : static_cast<int>(slot);
    const double turns = p * __ldg(freq + norm.rank[i]);
    float sn, cs;
    sincospif(static_cast<float>(2.0 * (turns - rint(turns))), &sn, &cs);
    s_cs[warp][i] = make_float2(cs, sn);
  }
  row = __shfl_sync(0xffffffffu, row, 0);      // -1: a bad page or slot, nothing is appended
  __syncwarp();
  // Mode 0: cosines and sines of two pairs side by side, as the elements lie; otherwise both members of a pair are side by side.
  float2 cs[4], sn[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float2 a = s_cs[warp][8 * c + 2 * i], e = s_cs[warp][8 * c + 2 * i + 1];
    cs[i] = make_float2(a.x, e.x);
    sn[i] = make_float2(a.y, e.y);
  }

  T* const q_dst = q_out + static_cast<int64_t>(t) * n_q_heads * D;
  T* const k_dst = static_cast<T*>(pool.k) + row * D;
  T* const v_dst = static_cast<T*>(pool.v) + row * D;
  const float* gain_of = nullptr;
  Raw8<float> gain[2];
  auto pack = [](const float2 (&x)[4]) {
    return make_uint4(Half2Of<T>::pack(x[0].x, x[0].y), Half2Of<T>::pack(x[1].x, x[1].y), Half2Of<T>::pack(x[2].x, x[2].y), Half2Of<T>::pack(x[3].x, x[3].y));
  };
  auto unpack = [](const Raw8<In>& raw, float2 (&x)[4]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if constexpr (sizeof(In) == 4) x[i] = make_float2(__uint_as_float(raw.w[2 * i]), __uint_as_float(raw.w[2 * i + 1]));
      else x[i] = Half2Of<In>::unpack(raw.w[i]);
    }
  };
  // The sum of the lane's squares, where the head is normed.
  auto squares_of = [&](int h, const Item& raw) {
    if (h >= turned || !(h < n_q_heads ? norm.q_gain : norm.k_gain)) return 0.f;
    float2 lo[4], hi[4], sum = make_float2(0.f, 0.f);
    unpack(raw.lo, lo);
    unpack(raw.hi, hi);
#pragma unroll
    for (int i = 0; i < 4; ++i) sum = fma2(lo[i], lo[i], fma2(hi[i], hi[i], sum));
    return sum.x + sum.y;
  };
  auto finish = [&](int h, const Item& raw, float sum) {
    const bool is_q = h < n_q_heads;
    if (h >= heads || (is_q ? !q : row < 0)) return;
    if (h >= turned) {
      T* const dst = v_dst + (static_cast<int64_t>(h - turned) << pool.page_shift) * D + 16 * c;
      if constexpr (sizeof(In) == 2) {
        *reinterpret_cast<uint4*>(dst) = *reinterpret_cast<const uint4*>(raw.lo.w);
        *reinterpret_cast<uint4*>(dst + 8) = *reinterpret_cast<const uint4*>(raw.hi.w);
      } else {
        float2 lo[4], hi[4];
        unpack(raw.lo, lo);
        unpack(raw.hi, hi);
        *reinterpret_cast<uint4*>(dst) = pack(lo);
        *reinterpret_cast<uint4*>(dst + 8) = pack(hi);
      }
      return;
    }
    T* const dst = (is_q ? q_dst + h * D : k_dst + (static_cast<int64_t>(h - n_q_heads) << pool.page_shift) * D) + kWide * c;
    float2 lo[4], hi[4];
    unpack(raw.lo, lo);
    unpack(raw.hi, hi);
    const float* const from = is_q ? norm.q_gain : norm.k_gain;
    if (from) {
      const float* const mine = is_q ? from + h * norm.q_gain_stride : from + (h - n_q_heads) * norm.k_gain_stride;
      if (mine != gain_of) {           // the same for every head, as a rule
        load8<Path::kReadOnly>(mine + kWide * c, norm.wide, gain[0]);
        load8<Path::kReadOnly>(mine + kWide * c + kGap, norm.wide, gain[1]);
        gain_of = mine;
      }
      const float f = rsqrtf(fmaf(sum, 1.f / D, norm.eps));
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        lo[i] = mul2(lo[i], mul2(make_float2(__uint_as_float(gain[0].w[2 * i]), __uint_as_float(gain[0].w[2 * i + 1])), make_float2(f, f)));
        hi[i] = mul2(hi[i], mul2(make_float2(__uint_as_float(gain[1].w[2 * i]), __uint_as_float(gain[1].w[2 * i + 1])), make_float2(f, f)));
      }
    }
    float2 u[4], w[4];
    if constexpr (kMode == 0) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        // in the order of append_kernel: without gains the bits are the same
        u[i] = fma2(lo[i], cs[i], mul2(hi[i], make_float2(-sn[i].x, -sn[i].y)));
        w[i] = fma2(lo[i], sn[i], mul2(hi[i], cs[i]));
      }
    } else {
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        u[2 * i] = make_float2(lo[2 * i].x * cs[i].x - lo[2 * i].y * sn[i].x, lo[2 * i].x * sn[i].x + lo[2 * i].y * cs[i].x);
        u[2 * i + 1] = make_float2(lo[2 * i + 1].x * cs[i].y - lo[2 * i + 1].y * sn[i].y, lo[2 * i + 1].x * sn[i].y + lo[2 * i + 1].y * cs[i].y);
        w[2 * i] = make_float2(hi[2 * i].x * cs[2 + i].x - hi[2 * i].y * sn[2 + i].x, hi[2 * i].x * sn[2 + i].x + hi[2 * i].y * cs[2 + i].x);
        w[2 * i + 1] = make_float2(hi[2 * i + 1].x * cs[2 + i].y - hi[2 * i + 1].y * sn[2 + i].y, hi[2 * i + 1].x * sn[2 + i].y + hi[2 * i + 1].y * cs[2 + i].y);
      }
    }
    *reinterpret_cast<uint4*>(dst) = pack(u);
    *reinterpret_cast<uint4*>(dst + kGap) = pack(w);
  };
  for (int h0 = warp % kWarps * kHeads; h0 < heads; h0 += 2 * kStep, h += 2 * kStep) {
    Item y[2];
    load(h + 2 * kStep, y[0]);
    load(h + 3 * kStep, y[1]);
    float sum[2] = {squares_of(h, x[0]), squares_of(h + kStep, x[1])};
#pragma unroll
    for (int o = 1; o < kItems; o <<= 1) {
      sum[0] += __shfl_xor_sync(0xffffffffu, sum[0], o);
      sum[1] += __shfl_xor_sync(0xffffffffu, sum[1], o);
    }
    finish(h, x[0], sum[0]);
    finish(h + kStep, x[1], sum[1]);
    x[0] = y[0];
    x[1] = y[1];
  }
}

template <typename T, typename In, int D>
cudaError_t launch_norm(const prima_paged& pool, const BatchView& b, int layer, const void* q, const void* k, const void* v, int n_q_heads, int64_t qs, int64_t ks, int64_t vs,
                        void* q_out, const HeadNorm& norm, cudaStream_t st) {
  const int64_t per16 = 16 / static_cast<int64_t>(sizeof(In));
  const bool wide = (!q || (aligned_to(q, 16) && qs % per16 == 0)) && aligned_to(k, 16) && aligned_to(v, 16) && ks % per16 == 0 && vs % per16 == 0;
  // Few rows: a CTA's eight warps share one, for the shortest path; many: a warp each, which looks up least and reads gains and
  // turns once for all heads.  Eight warps against one, 32 query and 8 KV heads of 128, B200: 64 rows 5.1 and 9.3 us, 296 rows
  // 5.8 and 9.3, 592 rows 10.4 and 9.4, 2368 rows 35 and 12, 9472 rows 137 and 51.
  const bool few = b.n_tok <= 3 * pool.sm_count;
  auto kernel = pool.cfg.rope_mode == 0 ? (few ? norm_kernel<T, In, D, 8, 0> : norm_kernel<T, In, D, 1, 0>) : (few ? norm_kernel<T, In, D, 8, 1> : norm_kernel<T, In, D, 1, 1>);
  return launch_pdl(kernel, dim3(few ? b.n_tok : static_cast<unsigned>((static_cast<int64_t>(b.n_tok) + 7) / 8)), dim3(256), 0, st, view_of(pool), b, layer, static_cast<const In*>(q), static_cast<const In*>(k),
                    static_cast<const In*>(v), n_q_heads, qs, ks, vs, wide, static_cast<const double*>(pool.freq), static_cast<T*>(q_out), norm);
}

}  // namespace
}  // namespace prima

using namespace prima;

extern "C" {

int prima_paged_append_norm(prima_paged* p, int layer, const prima_paged_batch* batch, const void* q, const void* k, const void* v, int in_dtype,
                            int n_q_heads, int64_t q_stride, int64_t k_stride, int64_t v_stride, const prima_head_norm* norm, void* q_out, void* stream) {
  const int rc = check_batch(p, batch, "prima_paged_append_norm");
  if (rc != PRIMA_OK) return rc;
  if (!norm) return call_fail(PRIMA_ERR_ARG, "prima_paged_append_norm: null norm");
  const int dim = p->cfg.head_dim;
  if (!(norm->eps >= 0.f) || std::isinf(norm->eps)) return call_fail(PRIMA_ERR_ARG, "prima_paged_append_norm: eps must be finite and not negative");
  if (norm->n_axes < 1 || norm->n_axes > PRIMA_MAX_AXES) return call_fail(PRIMA_ERR_ARG, "prima_paged_append_norm: n_axes outside 1..4");
  for (int i = 0; i < dim / 2; ++i)
    if ((norm->axis[i] >= norm->n_axes && norm->axis[i] != PRIMA_AXIS_NONE) || norm->rank[i] >= dim / 2)
      return call_fail(PRIMA_ERR_ARG, "prima_paged_append_norm: an axis or rank out of range");
  if ((norm->q_gain_stride != 0 && norm->q_gain_stride < dim) || (norm->k_gain_stride != 0 && norm->k_gain_stride < dim))
    return call_fail(PRIMA_ERR_ARG, "prima_paged_append_norm: a gain's stride is neither 0 nor at least head_dim");
  if (!aligned_to(norm->q_gain, 4) || !aligned_to(norm->k_gain, 4) || !aligned_to(norm->positions, 4))
    return call_fail(PRIMA_ERR_ARG, "prima_paged_append_norm: an array is not 4-byte aligned");
  HeadNorm n;
  n.q_gain = norm->q_gain;
  n.k_gain = norm->k_gain;
  n.q_gain_stride = norm->q_gain_stride;
  n.k_gain_stride = norm->k_gain_stride;
  n.eps = norm->eps;
  n.wide = aligned_to(n.q_gain, 16) && aligned_to(n.k_gain, 16) && n.q_gain_stride % 4 == 0 && n.k_gain_stride % 4 == 0;
  n.positions = norm->positions;
  std::copy(norm->axis, norm->axis + 64, n.axis);
  std::copy(norm->rank, norm->rank + 64, n.rank);
  const int bad = check_append(p, layer, q, k, v, in_dtype, n_q_heads, q_stride, k_stride, v_stride, q_out, "prima_paged_append_norm");
  if (bad != PRIMA_OK) return bad;
  const prima_paged_config& c = p->cfg;
  CallDevice dev(c.device);
  if (!dev.ok) return call_fail(PRIMA_ERR_CUDA, "cudaSetDevice failed");
  using launcher = cudaError_t (*)(const prima_paged&, const BatchView&, int, const void*, const void*, const void*, int, int64_t, int64_t, int64_t, void*, const HeadNorm&,
                                   cudaStream_t);
  static const launcher table[2][2][2] = {
      {{launch_norm<__half, float, 64>, launch_norm<__half, float, 128>}, {launch_norm<__half, __half, 64>, launch_norm<__half, __half, 128>}},
      {{launch_norm<__nv_bfloat16, float, 64>, launch_norm<__nv_bfloat16, float, 128>},
       {launch_norm<__nv_bfloat16, __nv_bfloat16, 64>, launch_norm<__nv_bfloat16, __nv_bfloat16, 128>}}};
  const cudaError_t e = table[c.dtype == PRIMA_DT_BF16][in_dtype != PRIMA_DT_F32][c.head_dim == 128](*p, view_of(*batch), layer, q, k, v, n_q_heads, q_stride, k_stride,
                                                                                                  v_stride, q_out, n, static_cast<cudaStream_t>(stream));
  return e == cudaSuccess ? PRIMA_OK : call_cuda_fail(e, "prima_paged_append_norm");
}

}  // extern "C"
