// The paged cache: pool, rotation and append of a step's rows, accepted paths of drafted trees, reordering of beams.
//
// All three kernels move bytes and compute next to nothing; what bounds them is HBM for large steps and, for the small
// ones that decoding makes, the chain of dependent reads (row_begin -> ctx_len -> table -> entry), so each keeps that
// chain short and has everything else in flight beside it.
#include <cmath>
#include <cstdio>
#include <new>

#include "paged.cuh"

namespace prima {
namespace {

// ---- rotation and append ----------------------------------------------------------------------------------------
// Row t at position p: pair i of every query and key head is turned by 2 pi frac(p f_i), f_i = theta^(-2i/D) / (2 pi).
// p f_i is formed in 64 bits (error p f_i 2^-53 turns, below 2^-24 up to p = 2^29), its whole turns are dropped and the
// rest goes to sincospif in 32 bits.
// kWarps warps take one row, each looks its place up by itself.  A lane owns the same 8 pairs (16 elements) of every
// head that it turns, so their sines stay in registers; a warp takes 32 / (D/16) heads at a time, two items in flight.
// Four items in flight (fewer warps), or 8 and 16 rows per CTA, were slower or no faster; with the index arithmetic of a
// division per item the kernel was bound by instructions (65 us where it is 61 now).
// Prompts of 11,268 rows, 40 + 16 heads of 128, bf16, 323 MB: 61 us, 5.3 TB/s, HBM; one row 3.0 us, 278 rows of
// trees 6 us, latency.
template <typename T, typename In, int D, int kWarps>
__global__ void __launch_bounds__(256) append_kernel(PoolView pool, BatchView b, int layer, const In* q, const In* k,
                                                     const In* v, int n_q_heads, int64_t q_stride, int64_t k_stride,
                                                     int64_t v_stride, bool wide, const double* __restrict__ freq, int mode,
                                                     T* __restrict__ q_out) {
  constexpr int kPairs = D / 2, kItems = D / 16, kHeads = 32 / kItems, kStep = kWarps * kHeads;
  __shared__ __align__(16) float2 s_cs[8][kPairs];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int t = (static_cast<int>(blockIdx.x) * 8 + warp) / kWarps;
  const int c = lane % kItems, G = pool.n_kv_heads, heads = n_q_heads + 2 * G;
  if (t >= b.n_tok) return;
  pdl_trigger();
  pdl_wait();
  const In* const q_row = q ? q + t * q_stride : nullptr;
  const In* const k_row = k + t * k_stride;
  const In* const v_row = v + t * v_stride;
  struct Item { Raw8<In> lo, hi; };
  // Turned heads: elements 8 c .. and D/2 + 8 c .. (mode 0); otherwise 16 c .. 16 c + 15
  auto load = [&](int h, Item& x) {
    if (h >= heads || (h < n_q_heads && !q)) return;
    const In* src = h < n_q_heads ? q_row + h * D : h < n_q_heads + G ? k_row + (h - n_q_heads) * D : v_row + (h - n_q_heads - G) * D;
    const bool halves = mode == 0 && h < n_q_heads + G;
    load8(src + (halves ? 8 * c : 16 * c), wide, x.lo);
    load8(src + (halves ? kPairs + 8 * c : 16 * c + 8), wide, x.hi);
  };
  int h = (warp % kWarps) * kHeads + lane / kItems;
  Item x[2];
  load(h, x[0]);                       // in flight while the place is looked up
  load(h + kStep, x[1]);

  int p = b.pos ? b.pos[t] : 0;
  const int s = seq_of_row(b, t, lane);
  if (s >= b.n_seq) return;            // padding
  const int first = b.row_begin[s], ctx = b.ctx_len[s];
  if (t < first || first < 0 || ctx < 0) {
    if (lane == 0) raise(pool.status, kBadRows);
    return;
  }
  const int64_t slot = static_cast<int64_t>(ctx) + (t - first);
  if (!b.pos) p = static_cast<int>(slot);
  int64_t row = lane == 0 ? slot_row(pool, b.table + s * b.table_stride, b.table_stride, layer, slot) : 0;
  for (int i = lane; i < kPairs; i += 32) {
    const double turns = p * __ldg(freq + i);
    float sn, cs;
    sincospif(static_cast<float>(2.0 * (turns - rint(turns))), &sn, &cs);
    s_cs[warp][i] = make_float2(cs, sn);
  }
  row = __shfl_sync(0xffffffffu, row, 0);      // -1: a bad page or slot, nothing is appended
  __syncwarp();
  float2 cs[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) cs[i] = s_cs[warp][8 * c + i];

  T* const q_dst = q_out + static_cast<int64_t>(t) * n_q_heads * D;
  T* const k_dst = static_cast<T*>(pool.k) + row * D;
  T* const v_dst = static_cast<T*>(pool.v) + row * D;
  auto finish = [&](int h, const Item& raw) {
    const bool is_q = h < n_q_heads, is_v = h >= n_q_heads + G;
    if (h >= heads || (is_q ? !q : row < 0)) return;
    T* dst = is_q ? q_dst + h * D : is_v ? v_dst + (static_cast<int64_t>(h - n_q_heads - G) << pool.page_shift) * D
                                         : k_dst + (static_cast<int64_t>(h - n_q_heads) << pool.page_shift) * D;
    float lo[8], hi[8], u[8], w[8];
    to_f(raw.lo, lo);
    to_f(raw.hi, hi);
    if (is_v) {
      store8(dst + 16 * c, lo);
      store8(dst + 16 * c + 8, hi);
    } else if (mode == 0) {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        u[i] = lo[i] * cs[i].x - hi[i] * cs[i].y;
        w[i] = lo[i] * cs[i].y + hi[i] * cs[i].x;
      }
      store8(dst + 8 * c, u);
      store8(dst + kPairs + 8 * c, w);
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        u[2 * i] = lo[2 * i] * cs[i].x - lo[2 * i + 1] * cs[i].y;
        u[2 * i + 1] = lo[2 * i] * cs[i].y + lo[2 * i + 1] * cs[i].x;
        w[2 * i] = hi[2 * i] * cs[4 + i].x - hi[2 * i + 1] * cs[4 + i].y;
        w[2 * i + 1] = hi[2 * i] * cs[4 + i].y + hi[2 * i + 1] * cs[4 + i].x;
      }
      store8(dst + 16 * c, u);
      store8(dst + 16 * c + 8, w);
    }
  };
  for (; h < heads; h += 2 * kStep) {
    Item y[2];
    load(h + 2 * kStep, y[0]);
    load(h + 3 * kStep, y[1]);
    finish(h, x[0]);
    finish(h + kStep, x[1]);
    x[0] = y[0];
    x[1] = y[1];
  }
}

// ---- accepted paths ---------------------------------------------------------------------------------------------
// Rows path[0..n-1] of a sequence's step move to rows 0..n-1, in every layer.  blockIdx.x = the sequence; its CTAs look
// the rows' places up once and share the columns: a column is 16 bytes of one head of keys or values of one layer, and
// a thread moves it for all rows, in ascending order.  path ascends, so path[j] >= j: what is read for row j is
// overwritten at the earliest for row path[j], and a batch that is read whole before any of it is written keeps that.  An
// entry that is not above the one before it is reported and stays where it is.
// Bound by scattered reads of 256 bytes in flight: 32 paths of 1 to 12 rows, 80 layers, 83 MB: 13.6 us (part of it from
// L2; 17 when other data went through it); one path of 4 rows, 32 layers: 2.9 us.
constexpr int kPathBatch = 8, kPathBlock = 256;
template <int D>
__global__ void __launch_bounds__(256) accept_kernel(PoolView pool, BatchView b, const int32_t* path, const int32_t* path_len,
                                                     int path_stride) {
  constexpr int kPieces = D / 8;                  // 16-byte pieces of a row
  __shared__ int2 s_move[kPathBlock];             // page and row in the page, packed: from, to; from < 0: stays
  __shared__ int2 s_in[kPathBlock];
  pdl_trigger();
  pdl_wait();
  const int s = blockIdx.x, G = pool.n_kv_heads;
  const int first = b.row_begin[s], end = b.row_begin[s + 1], ctx = b.ctx_len[s], n = path_len[s];
  if (first < 0 || end < first || end > b.n_tok || ctx < 0 || n < 0 || n > path_stride) {
    if (threadIdx.x == 0) raise(pool.status, n < 0 || n > path_stride ? kBadPath : kBadRows);
    return;
  }
  const int32_t* table = b.table + s * b.table_stride;
  const int in_page = (1 << pool.page_shift) - 1;
  const int64_t columns = static_cast<int64_t>(pool.n_layers) * 2 * G * kPieces;
  for (int j0 = 0; j0 < n; j0 += kPathBlock) {
    const int m = min(n - j0, kPathBlock);
    __syncthreads();
    if (static_cast<int>(threadIdx.x) < m) {
      const int j = j0 + threadIdx.x, a = path[static_cast<int64_t>(s) * path_stride + j];
      int2 pages = make_int2(-1, 0), rows = make_int2(0, 0);
      if (a < 0 || a >= end - first || (j > 0 && a <= path[static_cast<int64_t>(s) * path_stride + j - 1])) {
        raise(pool.status, kBadPath);
      } else if (a != j) {
        const int64_t from = static_cast<int64_t>(ctx) + a, to = static_cast<int64_t>(ctx) + j;
        if (slot_row(pool, table, b.table_stride, 0, from) >= 0 && slot_row(pool, table, b.table_stride, 0, to) >= 0) {
          pages = make_int2(table[from >> pool.page_shift], table[to >> pool.page_shift]);
          rows = make_int2(static_cast<int>(from) & in_page, static_cast<int>(to) & in_page);
        }
      }
      s_move[threadIdx.x] = pages;
      s_in[threadIdx.x] = rows;
    }
    __syncthreads();
    for (int64_t c = static_cast<int64_t>(blockIdx.y) * 256 + threadIdx.x; c < columns; c += static_cast<int64_t>(gridDim.y) * 256) {
      const int piece = static_cast<int>(c % kPieces), w = static_cast<int>(c / kPieces), g = w % G, lv = w / G;      // lv: layer and keys or values
      uint4* const base = static_cast<uint4*>(lv & 1 ? pool.v : pool.k) + piece;
      const int64_t layer = static_cast<int64_t>(lv >> 1) * pool.n_pages;
      auto at = [&](int page, int row) { return ((((layer + page) * G + g) << pool.page_shift) + row) * kPieces; };
      for (int j = 0; j < m; j += kPathBatch) {
        uint4 x[kPathBatch];
#pragma unroll
        for (int i = 0; i < kPathBatch; ++i)
          if (j + i < m && s_move[j + i].x >= 0) x[i] = __ldcg(base + at(s_move[j + i].x, s_in[j + i].x));
#pragma unroll
        for (int i = 0; i < kPathBatch; ++i)
          if (j + i < m && s_move[j + i].x >= 0) base[at(s_move[j + i].y, s_in[j + i].y)] = x[i];
      }
    }
  }
}

// ---- reordering of beams ----------------------------------------------------------------------------------------
// blockIdx.x = new row; the first CTA of a row writes its table and length.  When an earlier row of the request has the
// same parent, the row's CTAs copy the entries of the last page in all layers; those of one head are consecutive,
// (length % page_size) * head_dim * 2 bytes.  128 rows, 16 layers, 8 KV heads: 9.7 us, bound by the reads that a warp has
// in flight; with index arithmetic per 16 bytes it took 20.
template <int D>
__global__ void __launch_bounds__(256) reorder_kernel(PoolView pool, int n_beams, int keep, const int32_t* table_in, int64_t stride,
                                                      const int32_t* length_in, const int32_t* parent,
                                                      const int32_t* fresh, int32_t* __restrict__ table_out, int32_t* __restrict__ length_out) {
  pdl_trigger();
  pdl_wait();
  const int r = blockIdx.x, req = r / keep, j = r - req * keep;
  const int lane = threadIdx.x & 31;
  const int G = pool.n_kv_heads;
  int p = parent[r];
  const int f = fresh[r];
  bool shared_parent = false;
  for (int i = lane; i < j; i += 32) shared_parent |= parent[r - j + i] == p;
  shared_parent = __any_sync(0xffffffffu, shared_parent);
  if (!shared_parent && blockIdx.y > 0) return;
  const bool bad = p < 0 || p >= n_beams;
  if (bad) p = 0;
  const int64_t src = static_cast<int64_t>(req) * n_beams + p;
  const int len = length_in[src];
  const int64_t pages = (static_cast<int64_t>(max(len, 0)) + (1 << pool.page_shift) - 1) >> pool.page_shift;
  const int tail = len & ((1 << pool.page_shift) - 1);
  const bool bad_len = len < 0 || pages > stride;
  const bool empty = bad || bad_len;      // continues nothing: it must not share another row's partly filled page
  const int last = !empty && pages > 0 ? table_in[src * stride + pages - 1] : 0;
  const bool copies = shared_parent && tail != 0 && !empty;
  const bool bad_page = copies && (static_cast<unsigned>(last) >= static_cast<unsigned>(pool.n_pages) || static_cast<unsigned>(f) >= static_cast<unsigned>(pool.n_pages));
  if (blockIdx.y == 0) {
    if (threadIdx.x == 0) {
      if (bad) raise(pool.status, kBadPath);
      if (!bad && bad_len) raise(pool.status, kBadRows);
      if (bad_page) raise(pool.status, kBadPage);
      length_out[r] = empty ? 0 : len;
    }
    for (int64_t i = threadIdx.x; i < stride; i += blockDim.x)
      table_out[r * stride + i] = empty || i >= pages ? -1 : copies && i == pages - 1 ? f : table_in[src * stride + i];
  }
  if (!copies || bad_page) return;
  // A warp takes one head of keys or values of one layer at a time (index arithmetic per 16 bytes would bound the kernel).
  const int n = tail * (D / 8);      // 16-byte pieces
  const int64_t page_step = (static_cast<int64_t>(G) << pool.page_shift) * (D / 8);
  for (int w = blockIdx.y * 8 + (threadIdx.x >> 5); w < pool.n_layers * 2 * G; w += gridDim.y * 8) {
    const int lv = w / G, g = w - lv * G;
    uint4* const base = static_cast<uint4*>(lv & 1 ? pool.v : pool.k) + (lv >> 1) * page_step * pool.n_pages + ((static_cast<int64_t>(g) << pool.page_shift) * (D / 8));
    const uint4* const from = base + page_step * last;
    uint4* const to = base + page_step * f;
    for (int i = lane; i < n; i += 128) {
      uint4 x[4];
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (i + 32 * j < n) x[j] = __ldcg(from + i + 32 * j);
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (i + 32 * j < n) to[i + 32 * j] = x[j];
    }
  }
}

// Takes the reported bits out of the status word: a kernel on another stream may have raised others since it was read.
__global__ void clear_bits_kernel(int* status, int bits) { atomicAnd(status, ~bits); }

bool aligned16(const void* p) { return aligned_to(p, 16); }

template <typename T, typename In, int D>
cudaError_t launch_append(const prima_paged& pool, const BatchView& b, int layer, const void* q, const void* k, const void* v, int n_q_heads,
                          int64_t qs, int64_t ks, int64_t vs, void* q_out, cudaStream_t st) {
  const int64_t per16 = 16 / static_cast<int64_t>(sizeof(In));
  const bool wide = (!q || (aligned16(q) && qs % per16 == 0)) && aligned16(k) && aligned16(v) && ks % per16 == 0 && vs % per16 == 0;
  // Few rows: a CTA's eight warps share one, for the shortest path; many: a warp each, which looks up least.  40 + 16
  // heads of 128, 64 rows 3.3 and 7.8 us, 1200 rows 9.5 and 10.2, 2400 rows 16.9 and 16.5, 9600 rows 66 and 56.
  const bool few = b.n_tok <= 16 * pool.sm_count;
  auto kernel = few ? append_kernel<T, In, D, 8> : append_kernel<T, In, D, 1>;
  return launch_pdl(kernel, dim3(few ? b.n_tok : (b.n_tok + 7) / 8), dim3(256), 0, st, view_of(pool), b, layer, static_cast<const In*>(q), static_cast<const In*>(k),
                    static_cast<const In*>(v), n_q_heads, qs, ks, vs, wide, static_cast<const double*>(pool.freq), pool.cfg.rope_mode, static_cast<T*>(q_out));
}

}  // namespace

int check_batch(const prima_paged* pool, const prima_paged_batch* b, const char* who) {
  char msg[160];
  const char* bad = nullptr;
  if (!pool || !b) bad = "null pool or batch";
  else if (b->n_seq < 1 || b->n_tok < 1) bad = "n_seq and n_tok must be positive";
  else if (!b->row_begin || !b->ctx_len || !b->table || b->table_stride < 1) bad = "row_begin, ctx_len and table are needed";
  else if (b->table_stride > 2147483647) bad = "table_stride reaches 2^31";
  else if (b->mask && (b->mask_words < 1 || b->mask_words > 16)) bad = "mask_words outside 1..16";
  else if (!aligned_to(b->row_begin, 4) || !aligned_to(b->ctx_len, 4) || !aligned_to(b->table, 4) || !aligned_to(b->pos, 4) || !aligned_to(b->mask, 8))
    bad = "an array is not aligned to its elements";
  if (!bad) return PRIMA_OK;
  snprintf(msg, sizeof msg, "%s: %s", who, bad);
  return call_fail(PRIMA_ERR_ARG, msg);
}

int check_append(const prima_paged* pool, int layer, const void* q, const void* k, const void* v, int in_dtype, int n_q_heads, int64_t q_stride, int64_t k_stride,
                 int64_t v_stride, const void* q_out, const char* who) {
  const prima_paged_config& c = pool->cfg;
  const size_t size = in_dtype == PRIMA_DT_F32 ? 4 : 2;
  const int64_t need_q = static_cast<int64_t>(n_q_heads) * c.head_dim, need_kv = static_cast<int64_t>(c.n_kv_heads) * c.head_dim;
  char msg[160];
  const char* bad = nullptr;
  if (layer < 0 || layer >= c.n_layers) bad = "layer out of range";
  else if (!k || !v || (q != nullptr) != (q_out != nullptr)) bad = "null k or v, or only one of q and q_out";
  else if (in_dtype != PRIMA_DT_F32 && in_dtype != c.dtype) bad = "in_dtype is neither fp32 nor the cache's type";
  else if (q ? n_q_heads < 1 || n_q_heads > (1 << 16) : n_q_heads != 0) bad = "n_q_heads";
  else if (!aligned_to(q, size) || !aligned_to(k, size) || !aligned_to(v, size)) bad = "q, k or v is not aligned to its elements";
  else if (!aligned_to(q_out, 16)) bad = "q_out must be 16-byte aligned";
  else if ((q && q_stride < need_q) || k_stride < need_kv || v_stride < need_kv) bad = "a stride is shorter than a row";
  if (!bad) return PRIMA_OK;
  snprintf(msg, sizeof msg, "%s: %s", who, bad);
  return call_fail(PRIMA_ERR_ARG, msg);
}

}  // namespace prima

using namespace prima;

extern "C" {

int prima_paged_create(const prima_paged_config* cfg, void* dev_k, void* dev_v, prima_paged** out) {
  if (out) *out = nullptr;
  if (!cfg || !out || !dev_k || !dev_v) return call_fail(PRIMA_ERR_ARG, "prima_paged_create: null argument");
  const prima_paged_config& c = *cfg;
  if (c.n_layers < 1 || c.n_pages < 1 || c.page_size < 8 || c.page_size > 32768 || (c.page_size & (c.page_size - 1)) || c.n_kv_heads < 1 ||
      c.n_kv_heads > 1024 || (c.head_dim != 64 && c.head_dim != 128) || (c.dtype != PRIMA_DT_F16 && c.dtype != PRIMA_DT_BF16) ||
      !(c.rope_theta > 0.f) || std::isinf(c.rope_theta) || (c.rope_mode != 0 && c.rope_mode != 1) || c.device < 0)
    return call_fail(PRIMA_ERR_ARG, "prima_paged_create: inconsistent shape");
  if (static_cast<double>(c.n_layers) * c.n_pages * c.n_kv_heads * c.page_size >= 2147483648.0)
    return call_fail(PRIMA_ERR_ARG, "prima_paged_create: layers * pages * heads * page_size must stay below 2^31");
  if (!aligned16(dev_k) || !aligned16(dev_v)) return call_fail(PRIMA_ERR_ARG, "prima_paged_create: the arrays must be 16-byte aligned");
  int n_dev = 0;
  cudaError_t e = cudaGetDeviceCount(&n_dev);
  if (e != cudaSuccess) return call_cuda_fail(e, "cudaGetDeviceCount");
  if (c.device >= n_dev) return call_fail(PRIMA_ERR_ARG, "prima_paged_create: no such device");
  CallDevice dev(c.device);
  if (!dev.ok) return call_fail(PRIMA_ERR_CUDA, "cudaSetDevice failed");
  prima_paged* p = new (std::nothrow) prima_paged();
  if (!p) return call_fail(PRIMA_ERR_NOMEM, "out of host memory");
  p->cfg = c;
  p->k = dev_k;
  p->v = dev_v;
  while ((1 << p->page_shift) < c.page_size) ++p->page_shift;
  double freq[64];
  for (int i = 0; i < c.head_dim / 2; ++i)
    freq[i] = std::pow(static_cast<double>(c.rope_theta), -2.0 * i / c.head_dim) / 6.283185307179586476925286766559;
  e = cudaDeviceGetAttribute(&p->sm_count, cudaDevAttrMultiProcessorCount, c.device);
  if (e == cudaSuccess) e = cudaMalloc(reinterpret_cast<void**>(&p->freq), sizeof freq);
  if (e == cudaSuccess) e = cudaMemcpy(p->freq, freq, sizeof(double) * c.head_dim / 2, cudaMemcpyHostToDevice);
  if (e == cudaSuccess) e = cudaMalloc(reinterpret_cast<void**>(&p->status), sizeof(int));
  if (e == cudaSuccess) e = cudaMemset(p->status, 0, sizeof(int));
  if (e == cudaSuccess) e = make_tree_maps(p);
  if (e == cudaSuccess) e = cudaDeviceSynchronize();
  if (e != cudaSuccess) {
    prima_paged_destroy(p);
    return call_cuda_fail(e, "prima_paged_create");
  }
  *out = p;
  return PRIMA_OK;
}

int prima_paged_destroy(prima_paged* p) {
  if (!p) return PRIMA_OK;
  CallDevice dev(p->cfg.device);
  cudaDeviceSynchronize();
  cudaFree(p->freq);
  cudaFree(p->status);
  free_tree_maps(p);
  delete p;
  return PRIMA_OK;
}

int prima_paged_sync(prima_paged* p, void* stream) {
  if (!p) return call_fail(PRIMA_ERR_ARG, "prima_paged_sync: null pool");
  CallDevice dev(p->cfg.device);
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  int status = 0;
  cudaError_t e = cudaMemcpyAsync(&status, p->status, sizeof(int), cudaMemcpyDeviceToHost, st);
  if (e == cudaSuccess) e = cudaStreamSynchronize(st);
  if (e == cudaSuccess && status) {
    clear_bits_kernel<<<1, 1, 0, st>>>(p->status, status);
    e = cudaGetLastError();
    if (e == cudaSuccess) e = cudaStreamSynchronize(st);
  }
  if (e != cudaSuccess) return call_cuda_fail(e, "prima_paged_sync");
  if (!status) return PRIMA_OK;
  char msg[200];
  snprintf(msg, sizeof msg, "entries were skipped:%s%s%s%s%s", status & kBadPage ? " a page id outside the pool;" : "",
           status & kBadSlot ? " a slot beyond the page table;" : "", status & kBadRows ? " bad row_begin or length;" : "",
           status & kBadPath ? " a path entry or parent out of range;" : "", status & kGaveUp ? " a bounded wait inside a kernel gave up;" : "");
  return call_fail(PRIMA_ERR_DEVICE, msg);
}

int prima_paged_append(prima_paged* p, int layer, const prima_paged_batch* batch, const void* q, const void* k, const void* v, int in_dtype,
                       int n_q_heads, int64_t q_stride, int64_t k_stride, int64_t v_stride, void* q_out, void* stream) {
  const int rc = check_batch(p, batch, "prima_paged_append");
  if (rc != PRIMA_OK) return rc;
  const int bad = check_append(p, layer, q, k, v, in_dtype, n_q_heads, q_stride, k_stride, v_stride, q_out, "prima_paged_append");
  if (bad != PRIMA_OK) return bad;
  const prima_paged_config& c = p->cfg;
  CallDevice dev(c.device);
  if (!dev.ok) return call_fail(PRIMA_ERR_CUDA, "cudaSetDevice failed");
  const BatchView b = view_of(*batch);
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  using launcher = cudaError_t (*)(const prima_paged&, const BatchView&, int, const void*, const void*, const void*, int, int64_t, int64_t, int64_t, void*, cudaStream_t);
  static const launcher table[2][2][2] = {
      {{launch_append<__half, float, 64>, launch_append<__half, float, 128>}, {launch_append<__half, __half, 64>, launch_append<__half, __half, 128>}},
      {{launch_append<__nv_bfloat16, float, 64>, launch_append<__nv_bfloat16, float, 128>},
       {launch_append<__nv_bfloat16, __nv_bfloat16, 64>, launch_append<__nv_bfloat16, __nv_bfloat16, 128>}}};
  const cudaError_t e = table[c.dtype == PRIMA_DT_BF16][in_dtype != PRIMA_DT_F32][c.head_dim == 128](*p, b, layer, q, k, v, n_q_heads, q_stride, k_stride,
                                                                                                  v_stride, q_out, st);
  return e == cudaSuccess ? PRIMA_OK : call_cuda_fail(e, "prima_paged_append");
}

int prima_paged_accept(prima_paged* p, const prima_paged_batch* batch, const int32_t* path, const int32_t* path_len, int path_stride, void* stream) {
  const int rc = check_batch(p, batch, "prima_paged_accept");
  if (rc != PRIMA_OK) return rc;
  if (!path || !path_len || path_stride < 1) return call_fail(PRIMA_ERR_ARG, "prima_paged_accept: path, path_len and a positive path_stride are needed");
  if (!aligned_to(path, 4) || !aligned_to(path_len, 4)) return call_fail(PRIMA_ERR_ARG, "prima_paged_accept: path or path_len is not 4-byte aligned");
  CallDevice dev(p->cfg.device);
  if (!dev.ok) return call_fail(PRIMA_ERR_CUDA, "cudaSetDevice failed");
  // CTAs of a sequence: as many as its columns fill, and as keep every SM busy with all sequences together
  const int64_t columns = static_cast<int64_t>(p->cfg.n_layers) * 2 * p->cfg.n_kv_heads * (p->cfg.head_dim / 8);
  const int64_t share = std::max<int64_t>(1, (8 * static_cast<int64_t>(p->sm_count) + batch->n_seq - 1) / batch->n_seq);
  const dim3 grid(static_cast<unsigned>(batch->n_seq), static_cast<unsigned>(std::min<int64_t>({(columns + 255) / 256, share, 65535})));
  auto kernel = p->cfg.head_dim == 128 ? accept_kernel<128> : accept_kernel<64>;
  const cudaError_t e = launch_pdl(kernel, grid, dim3(256), 0, static_cast<cudaStream_t>(stream), view_of(*p), view_of(*batch), path, path_len, path_stride);
  return e == cudaSuccess ? PRIMA_OK : call_cuda_fail(e, "prima_paged_accept");
}

int prima_paged_reorder(prima_paged* p, int n_req, int n_beams, int keep, const int32_t* table_in, int64_t table_stride, const int32_t* length_in,
                        const int32_t* parent, const int32_t* fresh, int32_t* table_out, int32_t* length_out, void* stream) {
  if (!p || !table_in || !length_in || !parent || !fresh || !table_out || !length_out)
    return call_fail(PRIMA_ERR_ARG, "prima_paged_reorder: null argument");
  if (n_req < 1 || n_beams < 1 || keep < 1 || n_beams > 65536 || keep > 65536 || table_stride < 1 || table_stride > 2147483647 ||
      static_cast<int64_t>(n_req) * std::max(n_beams, keep) > 2147483647)
    return call_fail(PRIMA_ERR_ARG, "prima_paged_reorder: bad size");
  for (const int32_t* x : {table_in, length_in, parent, fresh, static_cast<const int32_t*>(table_out), static_cast<const int32_t*>(length_out)})
    if (!aligned_to(x, 4)) return call_fail(PRIMA_ERR_ARG, "prima_paged_reorder: an array is not 4-byte aligned");
  const int64_t rows_in = static_cast<int64_t>(n_req) * n_beams, rows_out = static_cast<int64_t>(n_req) * keep;
  auto overlap = [](const int32_t* a, int64_t na, const int32_t* b, int64_t nb) { return a < b + nb && b < a + na; };
  if (overlap(table_in, rows_in * table_stride, table_out, rows_out * table_stride) || overlap(length_in, rows_in, length_out, rows_out))
    return call_fail(PRIMA_ERR_ARG, "prima_paged_reorder: the new tables overlap the old ones");
  CallDevice dev(p->cfg.device);
  if (!dev.ok) return call_fail(PRIMA_ERR_CUDA, "cudaSetDevice failed");
  // CTAs of a row: enough that a few rows which copy a page fill the GPU, as far as there are heads for their warps
  const int64_t heads = static_cast<int64_t>(p->cfg.n_layers) * 2 * p->cfg.n_kv_heads;
  if (heads > 2147483647) return call_fail(PRIMA_ERR_ARG, "prima_paged_reorder: layers * KV heads too large");
  const int64_t share = std::max<int64_t>(1, (16 * static_cast<int64_t>(p->sm_count) + rows_out - 1) / rows_out);
  const dim3 grid(static_cast<unsigned>(rows_out), static_cast<unsigned>(std::min<int64_t>({(heads + 7) / 8, share, 65535})));
  auto kernel = p->cfg.head_dim == 128 ? reorder_kernel<128> : reorder_kernel<64>;
  const cudaError_t e = launch_pdl(kernel, grid, dim3(256), 0, static_cast<cudaStream_t>(stream), view_of(*p), n_beams, keep, table_in, table_stride, length_in, parent,
                                   fresh, table_out, length_out);
  return e == cudaSuccess ? PRIMA_OK : call_cuda_fail(e, "prima_paged_reorder");
}

}  // extern "C"
