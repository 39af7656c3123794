// Eviction from the paged cache: of a sequence's entries, those of largest weight stay and come together in front.
//
// Every (layer, sequence, KV head) chooses for itself, so a batch has hundreds of independent choices.  One kernel makes
// them, a CTA each, moves weights and positions and lists the rows of the cache that move; a second one moves keys and values
// with the whole GPU, however few the choices are.  Moving only what lies behind slot m, into the free slots in front of it,
// costs m (n - m) / n entries of n where a compaction in order would move nearly all m.
//
// The choice is bound by latency (six prompts of up to 16,001 entries in ten layers: 34 us of 90, the longest sequence
// decides), the moves by the copy (55 us at 5.3 TB/s; floor of both 58).  One request: 23 us, floor 10.
#include <algorithm>
#include <cstdio>

#include "paged_device.cuh"

namespace prima {
namespace {

constexpr int kThreads = 512, kWarps = kThreads / 32, kPer = 4, kTile = kThreads * kPer;
constexpr int kBins = 2048;                           // of a digit: 11, 11 and 10 bits
constexpr int kListed = 2048;                         // keys with the border's first digit that are set apart
constexpr int kFlight = 8;                            // loads of a thread in flight
constexpr int kRanked = 64;                           // sequences that are taken by length
// Keys that a CTA keeps in shared memory; those behind are made from the arrays again in every pass.  Two CTAs share an SM.
constexpr int kCached = 16384;

struct EvictArgs {
  PoolView pool;
  int n_seq;
  const int32_t* table;
  int64_t table_stride;
  const int32_t* length;
  const float* weight;
  const int32_t* born;
  int64_t stride;
  const int32_t* keep;
  int first;
  const int32_t* recent_from;
  float* weight_out;
  int32_t* born_out;
  int32_t* length_out;
  int32_t* counts;      // [items]
  int32_t* lists;       // [items][2 * half]: free slots in front, chosen ones behind; then their rows in the cache
  int64_t half;
  int cached;
};

// What the numbers of a sequence say; n < 0: they are bad.
struct Sizes {
  int n, m;
};
__device__ __forceinline__ Sizes sizes_of(const EvictArgs& a, int seq, int* length) {
  const int n = a.length[seq], keep = a.keep[seq];
  *length = n;
  if (n < 0 || keep < 0 || n > a.stride || n > (a.table_stride << a.pool.page_shift)) return {-1, 0};
  return {n, min(n, keep)};
}

// Larger is kept.  Whole numbers in the order of the weights: NaN below all, -0 equal to 0, protected entries above all.
__device__ __forceinline__ uint32_t key_of(float w, bool is_protected) {
  if (is_protected) return 0xffffffffu;
  if (w != w) return 0u;
  const uint32_t u = __float_as_uint(w + 0.f);
  return u >> 31 ? ~u : u | 0x80000000u;
}

// Inclusive sums over the threads of the CTA; `total` is the sum of all.  One barrier: two scans that follow one another use
// the two halves of s_warp in turns.
__device__ __forceinline__ uint32_t block_scan(uint32_t x, uint32_t (*s_warp)[kWarps], uint32_t& turn, uint32_t* total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const uint32_t y = __shfl_up_sync(0xffffffffu, x, o);
    if (lane >= o) x += y;
  }
  uint32_t* const sums = s_warp[turn++ & 1];
  if (lane == 31) sums[warp] = x;
  __syncthreads();
  uint32_t before = 0, all = 0;
#pragma unroll
  for (int i = 0; i < kWarps; ++i) {
    const uint32_t y = sums[i];
    before += i < warp ? y : 0u;
    all += y;
  }
  *total = all;
  return x + before;
}

// The same for kPer counts of every warp, those of place i behind all of place i - 1; `front`: what is in front of this warp's.
__device__ __forceinline__ void tile_scan(const uint32_t (&count)[kPer], uint32_t (&front)[kPer], uint32_t (*s_tile)[kPer * kWarps], uint32_t& turn, uint32_t* total) {
  static_assert(kPer * kWarps == 64, "two counts a lane");
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  uint32_t* const counts = s_tile[turn++ & 1];
#pragma unroll
  for (int i = 0; i < kPer; ++i)
    if (lane == i) counts[i * kWarps + warp] = count[i];
  __syncthreads();
  const uint2 mine = *reinterpret_cast<const uint2*>(counts + 2 * lane);
  uint32_t x = mine.x + mine.y;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const uint32_t y = __shfl_up_sync(0xffffffffu, x, o);
    if (lane >= o) x += y;
  }
  *total = __shfl_sync(0xffffffffu, x, 31);
  const uint32_t second = x - mine.y, first = second - mine.x;
#pragma unroll
  for (int i = 0; i < kPer; ++i) front[i] = __shfl_sync(0xffffffffu, warp & 1 ? second : first, (i * kWarps + warp) >> 1);
}

// The m-th largest key by its digits, from the top: a histogram of the digit among the keys that agree with those found so
// far, and the bin in which the count from above reaches what is still wanted.
// Bound by latency: the passes over the keys of a CTA and their barriers.
__global__ void __launch_bounds__(kThreads) evict_choose_kernel(const __grid_constant__ EvictArgs a) {
  extern __shared__ __align__(16) uint32_t s_key[];
  __shared__ uint32_t s_hist[2][kBins];
  __shared__ uint32_t s_list[kListed];
  __shared__ uint32_t s_warp[2][kWarps];
  __shared__ __align__(8) uint32_t s_tile[2][kPer * kWarps];
  __shared__ uint32_t s_found[3], s_listed;      // bin, keys above it, keys in it
  uint32_t turn = 0;
  __shared__ int s_seq;
  const int per_seq = gridDim.x / a.n_seq, layer = blockIdx.x % per_seq / a.pool.n_kv_heads, head = blockIdx.x % a.pool.n_kv_heads, tid = threadIdx.x, lane = tid & 31;
  int seq = blockIdx.x / per_seq;
  pdl_trigger();
  pdl_wait();
  // All choices of the longest sequence first, and so on: the GPU ends with short ones.  A thread ranks one sequence, in every
  // choice, which many sequences do not pay back: six of up to 16,001 entries in ten layers 90 us, 101 by layers, two in 16
  // layers 20 and 24, 64 in four 192 and 194, 500 in one 367 and 191.
  if (a.n_seq > 1 && a.n_seq <= kRanked) {
    int* const lengths = reinterpret_cast<int*>(s_hist[0]);
    const int mine = tid < a.n_seq ? a.length[tid] : 0;
    if (tid < a.n_seq) lengths[tid] = mine;
    __syncthreads();
    if (tid < a.n_seq) {
      int rank = 0;
      for (int i = 0; i < a.n_seq; ++i) rank += lengths[i] > mine || (lengths[i] == mine && i < tid);
      if (rank == seq) s_seq = tid;
    }
    __syncthreads();
    seq = s_seq;
  }
  const int64_t item = (static_cast<int64_t>(layer) * a.n_seq + seq) * a.pool.n_kv_heads + head;
  int length;
  const Sizes z = sizes_of(a, seq, &length);
  const int n = z.n, m = z.m;
  if (n < 0 && tid == 0 && layer == 0 && head == 0) raise(a.pool.status, length < 0 || a.keep[seq] < 0 ? kBadRows : kBadSlot);
  const int64_t at = item * a.stride;
  const float* const weight = a.weight + at;
  const int32_t* const born = a.born + at;
  const bool apart = a.weight_out != a.weight;
  if (n <= m || m == 0) {      // all stay, none, or bad numbers
    if (tid == 0) a.counts[item] = 0;
    if (apart)
      for (int j = tid; j < m; j += kThreads) {
        a.weight_out[at + j] = weight[j];
        a.born_out[at + j] = born[j];
      }
    return;
  }
  const bool some_recent = a.recent_from != nullptr;
  const int recent_from = some_recent ? a.recent_from[seq] : 0;
  auto make = [&](float w, int b) { return key_of(w, b < a.first || (some_recent && b >= recent_from)); };
  const int cached = min(n, a.cached);
  for (int i = tid; i < kBins; i += kThreads) s_hist[0][i] = s_hist[1][i] = 0;
  if (tid == 0) s_listed = 0;
  __syncthreads();
  // Keys, and the histogram of their first digit
  for (int j0 = tid; j0 < n; j0 += kThreads * kFlight) {
    float w[kFlight];
    int b[kFlight];
#pragma unroll
    for (int i = 0; i < kFlight; ++i) {
      const int j = j0 + i * kThreads;
      w[i] = j < n ? weight[j] : 0.f;
      b[i] = j < n ? born[j] : 0;
    }
#pragma unroll
    for (int i = 0; i < kFlight; ++i) {
      const int j = j0 + i * kThreads;
      if (j >= n) continue;
      const uint32_t k = make(w[i], b[i]);
      if (j < cached) s_key[j] = k;
      if (apart && j < m) {      // as if all of them stayed; what moves there overwrites them
        a.weight_out[at + j] = w[i];
        a.born_out[at + j] = b[i];
      }
      atomicAdd(&s_hist[0][k >> 21], 1u);
    }
  }
  __syncthreads();
  auto key = [&](int j) { return j < cached ? s_key[j] : make(weight[j], born[j]); };

  uint32_t prefix = 0, above = 0;      // digits found; keys that are larger
  auto find = [&](const uint32_t* hist, int bits) {
    // thread t has the `per` bins below bins - t * per
    constexpr int kMost = kBins / kThreads;
    const int per = (1 << bits) / kThreads, low = (1 << bits) - (tid + 1) * per;
    uint32_t v[kMost], mine = 0, total;
#pragma unroll
    for (int i = 0; i < kMost; ++i) {
      v[i] = i < per ? hist[low + i] : 0;
      mine += v[i];
    }
    const uint32_t upto = block_scan(mine, s_warp, turn, &total), wanted = m - above;
    if (upto >= wanted && upto - mine < wanted) {      // one thread
      uint32_t sum = upto - mine;
      bool found = false;
#pragma unroll
      for (int i = kMost - 1; i >= 0; --i) {
        if (i >= per || found) continue;
        if (sum + v[i] >= wanted) {
          s_found[0] = low + i;
          s_found[1] = sum;
          s_found[2] = v[i];
          found = true;
        }
        sum += v[i];
      }
    }
    __syncthreads();
    prefix = prefix << bits | s_found[0];
    above += s_found[1];
  };
  find(s_hist[0], 11);
  // The keys with this first digit, few as a rule, are set apart in any order: only their numbers count.
  const bool listed = s_found[2] <= kListed;
  const int n_listed = listed ? static_cast<int>(s_found[2]) : n;
  if (listed) {
    for (int j = 4 * tid; j < n; j += 4 * kThreads) {
      uint32_t k[4];
      if (j + 4 <= cached) {
        *reinterpret_cast<uint4*>(k) = *reinterpret_cast<const uint4*>(s_key + j);
      } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) k[i] = j + i < n ? key(j + i) : ~prefix << 21;
      }
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (k[i] >> 21 == prefix) s_list[atomicAdd(&s_listed, 1u)] = k[i];
    }
  }
  for (int i = tid; i < kBins; i += kThreads) s_hist[0][i] = 0;      // all have found the first digit; for the third
  __syncthreads();
#pragma unroll
  for (int d = 1; d < 3; ++d) {
    const int shift = d == 1 ? 10 : 0, done = d == 1 ? 21 : 10;
    uint32_t* const hist = s_hist[d & 1];
    for (int j = tid; j < n_listed; j += kThreads) {
      const uint32_t k = listed ? s_list[j] : key(j);
      if (k >> done == prefix) atomicAdd(&hist[(k >> shift) & (d == 1 ? 2047 : 1023)], 1u);
    }
    __syncthreads();
    find(hist, d == 1 ? 11 : 10);
  }
  // Of the keys equal to the border, the first `wanted` stay; nearly always those are all.
  const uint32_t border = prefix, wanted = m - above;
  const bool some_equal = s_found[2] != wanted;

  // What is out of place, in the order of the slots: the free slots in front, then as many chosen ones behind.
  int32_t* const list = a.lists + 2 * a.half * item;
  uint32_t equal_before = 0, listed_before = 0;
  const uint32_t below = (1u << lane) - 1u;
  for (int j0 = 0; j0 < n; j0 += kTile) {
    // Slot j0 + i * kThreads + tid: a warp's slots are consecutive, so that ranks are counts of bits and the list is written
    // side by side.
    uint32_t k[kPer], moves[kPer], count[kPer], front[kPer], total;
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      const int j = j0 + i * kThreads + tid;
      k[i] = j < n ? key(j) : 0u;
      moves[i] = __ballot_sync(0xffffffffu, j < n && (k[i] > border || (k[i] == border && !some_equal)) != (j < m));
    }
    if (some_equal) {
      uint32_t equal[kPer];
#pragma unroll
      for (int i = 0; i < kPer; ++i) {
        equal[i] = __ballot_sync(0xffffffffu, j0 + i * kThreads + tid < n && k[i] == border);
        count[i] = __popc(equal[i]);
      }
      tile_scan(count, front, s_tile, turn, &total);
#pragma unroll
      for (int i = 0; i < kPer; ++i)      // one that stays after all
        moves[i] ^= __ballot_sync(0xffffffffu, (equal[i] >> lane & 1) && equal_before + front[i] + __popc(equal[i] & below) < wanted);
      equal_before += total;
    }
#pragma unroll
    for (int i = 0; i < kPer; ++i) count[i] = __popc(moves[i]);
    tile_scan(count, front, s_tile, turn, &total);
#pragma unroll
    for (int i = 0; i < kPer; ++i)
      if (moves[i] >> lane & 1) list[listed_before + front[i] + __popc(moves[i] & below)] = j0 + i * kThreads + tid;
    listed_before += total;
  }
  __syncthreads();
  // Weights and positions move here (all that read the free slots' are done), and the list becomes rows of the cache.
  const int n_moves = static_cast<int>(listed_before / 2);
  const int32_t* const table = a.table + seq * a.table_stride;
  if (tid == 0) a.counts[item] = n_moves;
#pragma unroll 4
  for (int i = tid; i < n_moves; i += kThreads) {
    const int hole = list[i], mover = list[n_moves + i];
    const float w = weight[mover];
    const int b = born[mover];
    const int64_t to = slot_row(a.pool, table, a.table_stride, layer, hole), from = slot_row(a.pool, table, a.table_stride, layer, mover);
    const bool good = to >= 0 && from >= 0;      // a row is below 2^31 (prima_paged_create); otherwise nothing of the entry moves
    if (good) {
      a.weight_out[at + hole] = w;
      a.born_out[at + hole] = b;
    }
    list[i] = good ? static_cast<int>(to) + (head << a.pool.page_shift) : -1;
    list[n_moves + i] = good ? static_cast<int>(from) + (head << a.pool.page_shift) : -1;
  }
}

// blockIdx.x = (layer, sequence, KV head); its warps share the moves.  A warp takes the key and the value of 32 / (D / 4)
// entries at a time, 16 bytes a lane, kFlight times in flight, while the rows of the next ones are read.
template <int D>
__global__ void __launch_bounds__(256) evict_move_kernel(const __grid_constant__ EvictArgs a) {
  constexpr int kPieces = D / 8, kEntries = 16 / kPieces;
  const int item = blockIdx.x, head = item % a.pool.n_kv_heads, seq = item / a.pool.n_kv_heads % a.n_seq;
  const int lane = threadIdx.x & 31, warp = blockIdx.y * 8 + (threadIdx.x >> 5), n_warps = gridDim.y * 8;
  pdl_trigger();
  pdl_wait();
  if (item < a.n_seq * a.pool.n_kv_heads && head == 0 && blockIdx.y == 0 && threadIdx.x == 0) {      // the choices have read `length`
    int length;
    const Sizes z = sizes_of(a, seq, &length);
    a.length_out[seq] = z.n < 0 ? length : z.m;
  }
  // Ordinary loads: the choices wrote counts and lists while this grid may have been resident, and lists share lines.
  const int count = a.counts[item];
  const int32_t* const to = a.lists + 2 * a.half * item;
  const int32_t* const from = to + count;
  const int entry = lane / (2 * kPieces), piece = lane % kPieces, is_v = lane / kPieces & 1;
  uint4* const base = static_cast<uint4*>(is_v ? a.pool.v : a.pool.k) + piece;
  int row_to[kFlight], row_from[kFlight];
  auto rows = [&](int i0) {
#pragma unroll
    for (int f = 0; f < kFlight; ++f) {
      const int i = i0 + f * kEntries + entry;
      row_to[f] = i < count ? to[i] : -1;
      row_from[f] = i < count ? from[i] : -1;
    }
  };
  int i0 = warp * kEntries * kFlight;
  rows(i0);
  for (; i0 < count; i0 += n_warps * kEntries * kFlight) {
    uint4 x[kFlight];
    int dst[kFlight];
#pragma unroll
    for (int f = 0; f < kFlight; ++f) {
      dst[f] = row_to[f];
      if (dst[f] >= 0) x[f] = __ldcs(base + static_cast<int64_t>(row_from[f]) * kPieces);
    }
    rows(i0 + n_warps * kEntries * kFlight);
#pragma unroll
    for (int f = 0; f < kFlight; ++f)
      if (dst[f] >= 0) base[static_cast<int64_t>(dst[f]) * kPieces] = x[f];
  }
}

int64_t padded(int64_t n) { return (n + 255) / 256 * 256; }

}  // namespace
}  // namespace prima

using namespace prima;

extern "C" {

int64_t prima_paged_evict_workspace(const prima_paged* p, int n_seq, int64_t stride) {
  if (!p || n_seq < 1 || stride < 1 || stride > (1 << 30)) return PRIMA_ERR_ARG;
  const int64_t items = static_cast<int64_t>(p->cfg.n_layers) * n_seq * p->cfg.n_kv_heads;
  if (items > 2147483647) return PRIMA_ERR_ARG;
  return padded(items * 4) + padded(items * 2 * ((stride + 1) / 2) * 4);
}

int prima_paged_evict(prima_paged* p, int n_seq, const int32_t* table, int64_t table_stride, const int32_t* length, const float* weight,
                      const int32_t* born, int64_t stride, const int32_t* keep, int first, const int32_t* recent_from, float* weight_out,
                      int32_t* born_out, int32_t* length_out, void* workspace, int64_t workspace_bytes, void* stream) {
  auto refuse = [](const char* what) {
    char msg[160];
    snprintf(msg, sizeof msg, "prima_paged_evict: %s", what);
    return call_fail(PRIMA_ERR_ARG, msg);
  };
  if (!p || !table || !length || !weight || !born || !keep || !weight_out || !born_out || !length_out) return refuse("null argument");
  if (n_seq < 1 || table_stride < 1 || table_stride > 2147483647 || stride < 1 || stride > (1 << 30)) return refuse("bad size");
  for (const void* x : {static_cast<const void*>(table), static_cast<const void*>(length), static_cast<const void*>(weight), static_cast<const void*>(born),
                        static_cast<const void*>(keep), static_cast<const void*>(recent_from), static_cast<const void*>(weight_out),
                        static_cast<const void*>(born_out), static_cast<const void*>(length_out)})
    if (!aligned_to(x, 4)) return refuse("an array is not 4-byte aligned");
  const int64_t items = static_cast<int64_t>(p->cfg.n_layers) * n_seq * p->cfg.n_kv_heads;
  if (items > 2147483647) return refuse("layers * sequences * KV heads reach 2^31");
  // Entries that move are read by one CTA and written by another: either the arrays are the same, entry for entry, or apart.
  const bool same = weight == weight_out;
  if (same != (born == born_out)) return refuse("weight_out is weight, but born_out is not born, or the other way round");
  auto overlap = [&](const void* x, const void* y, int64_t n) {
    const char *a = static_cast<const char*>(x), *b = static_cast<const char*>(y);
    return a < b + 4 * n && b < a + 4 * n;
  };
  if (!same && (overlap(weight, weight_out, items * stride) || overlap(born, born_out, items * stride))) return refuse("the new arrays overlap the old ones");
  if (length != length_out && overlap(length, length_out, n_seq)) return refuse("length_out overlaps length");
  if (!workspace || !aligned_to(workspace, 256) || workspace_bytes < prima_paged_evict_workspace(p, n_seq, stride))
    return refuse("workspace too small or not 256-byte aligned");
  CallDevice dev(p->cfg.device);
  if (!dev.ok) return call_fail(PRIMA_ERR_CUDA, "cudaSetDevice failed");
  EvictArgs a;
  a.pool = view_of(*p);
  a.n_seq = n_seq;
  a.table = table;
  a.table_stride = table_stride;
  a.length = length;
  a.weight = weight;
  a.born = born;
  a.stride = stride;
  a.keep = keep;
  a.first = first;
  a.recent_from = recent_from;
  a.weight_out = weight_out;
  a.born_out = born_out;
  a.length_out = length_out;
  a.counts = static_cast<int32_t*>(workspace);
  a.lists = reinterpret_cast<int32_t*>(static_cast<char*>(workspace) + padded(items * 4));
  a.half = (stride + 1) / 2;
  a.cached = static_cast<int>(std::min<int64_t>(stride, kCached));
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  static bool done[kMaxDevices] = {};
  cudaError_t e = allow_smem(evict_choose_kernel, kCached * sizeof(uint32_t), done);
  if (e == cudaSuccess) e = launch_pdl(evict_choose_kernel, dim3(static_cast<unsigned>(items)), dim3(kThreads), a.cached * sizeof(uint32_t), st, a);
  // CTAs of a choice's moves: enough that a few choices fill the GPU
  const int64_t share = std::max<int64_t>(1, (16 * static_cast<int64_t>(p->sm_count) + items - 1) / items);
  const int64_t most = (a.half + 63) / 64;
  const dim3 grid(static_cast<unsigned>(items), static_cast<unsigned>(std::min<int64_t>({share, most, 65535})));
  if (e == cudaSuccess) e = launch_pdl(p->cfg.head_dim == 128 ? evict_move_kernel<128> : evict_move_kernel<64>, grid, dim3(256), 0, st, a);
  return e == cudaSuccess ? PRIMA_OK : call_cuda_fail(e, "prima_paged_evict");
}

}  // extern "C"
