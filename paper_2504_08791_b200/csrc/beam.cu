// Beam selection: the best continuations of a request's beams over the vocabulary.
//
//   score(b, w) = cum[b] + (x[b][w] - m_b - log sum_v exp(x[b][v] - m_b)),   m_b = max_v x[b][v]
//
// The logits are read once.  A CTA holds slices of one row in registers, one after the other, and leaves their
// maximum, their sum of exponentials and their `keep` best logits; a second kernel joins the slices of a request.  Within a row the order of
// the scores is the order of the logits, so the slices can be cut down before the row's sum is known.
// Which of two near candidates of DIFFERENT beams is ahead depends on the last bits of the two sums, so all that is added
// behind a thread's own 8 or 32 words is added in 64 bits.  The exponentials of a slice (of its words and of the
// differences between its maxima) are 32-bit ones, 2^-22 each; in 64 bits they would cost about as much as all else (some
// 40 operations a word, not measured).  Every sum has a fixed order that follows the index in the row, not the address:
// equal rows get equal bits, and their candidates tie exactly (the lower index wins).
// Rows that cannot contribute (finished beams, cum = -infinity) are not read.
#include <cfloat>
#include <cstdio>

#include "paged.cuh"

namespace prima {
namespace {

constexpr int kThreads = 256;
constexpr int kMaxKeep = 64;

struct Best { float x; int32_t w; };                   // a logit and its word; x = -infinity: none
struct SliceStat { double sum; float top; int32_t unused; };

template <typename T> __device__ __forceinline__ float as_float(T x);
template <> __device__ __forceinline__ float as_float<float>(float x) { return x; }
template <> __device__ __forceinline__ float as_float<__half>(__half x) { return __half2float(x); }
template <> __device__ __forceinline__ float as_float<__nv_bfloat16>(__nv_bfloat16 x) { return __bfloat162float(x); }

// NaN and -infinity: no candidate; +infinity: the largest finite value.
__device__ __forceinline__ float usable(float x) { return fminf(fmaxf(x, -INFINITY), FLT_MAX); }
__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// A bound that at least `keep` of the threads' values reach (-infinity if fewer are above it): the keep-th largest of
// the maxima of groups of threads.  The groups are the smallest number, 8 .. 64, that holds keep; of thousands of
// values a few dozen reach the bound, at the cost of a few shuffles.  A group is every 8th .. 64th thread, so that a short
// last slice, or one beam's candidates, still reach every group: with a group that has nothing the bound is -infinity and
// everything is ranked against everything (512 words of a slice: 17 us).  s_group: kThreads values, s_max: 64.
template <typename V>
__device__ __forceinline__ V block_bound(V mine, int keep, V* s_group, V* s_max, V* s_bound) {
  const int n_groups = keep <= 8 ? 8 : keep <= 16 ? 16 : keep <= 32 ? 32 : 64, per = min(n_groups, 32);      // per: values of a warp
  const V lowest = static_cast<V>(-INFINITY);
  const int tid = threadIdx.x, lane = tid & 31;
  for (int o = 16; o >= per; o >>= 1) {
    const V other = __shfl_xor_sync(0xffffffffu, mine, o);
    mine = other > mine ? other : mine;
  }
  if (lane < per) s_group[(tid >> 5) * per + lane] = mine;
  if (tid == 0) *s_bound = lowest;
  __syncthreads();
  if (tid < n_groups) {
    V v = lowest;
    for (int j = tid; j < kThreads / 32 * per; j += n_groups) v = s_group[j] > v ? s_group[j] : v;
    s_max[tid] = v;
  }
  __syncthreads();
  if (tid < n_groups) {
    const V v = s_max[tid];
    int rank = 0;
    for (int j = 0; j < n_groups; ++j) rank += s_max[j] > v || (s_max[j] == v && j < tid);
    if (rank == keep - 1) *s_bound = v;
  }
  __syncthreads();
  return *s_bound;
}

// What is ahead: the higher value, of equal ones the lower index.
template <typename V>
__device__ __forceinline__ bool ahead(V x, int i, V y, int j) { return x > y || (x == y && i < j); }

// The best of the CTA's (value, index) pairs, for every thread.
template <typename V>
__device__ __forceinline__ void block_best(V& x, int& i, V* s_x, int* s_i) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    const V y = __shfl_xor_sync(0xffffffffu, x, o);
    const int j = __shfl_xor_sync(0xffffffffu, i, o);
    if (ahead(y, j, x, i)) {
      x = y;
      i = j;
    }
  }
  __syncthreads();
  if ((threadIdx.x & 31) == 0) {
    s_x[threadIdx.x >> 5] = x;
    s_i[threadIdx.x >> 5] = i;
  }
  __syncthreads();
  for (int w = 0; w < kThreads / 32; ++w)
    if (ahead(s_x[w], s_i[w], x, i)) {
      x = s_x[w];
      i = s_i[w];
    }
}

// Logits of a CTA that reach the bound.  With keep = 64 the bound is the least of 64 groups' maxima: of 8192 words with no
// order in them more than n reach it in a share of at most 64 (1 - n / 8192)^128 of the CTAs (of 2048 words, 64 (1 - n / 2048)^32).
// For 512 that is 1.7 % (0.6 %), which a call of hundreds of CTAs nearly always meets, and one that runs over searches its
// words once per place: 16 requests of 8 beams of 152,064 words, keep = 64, took 1340 us (keep = 63: 87).  For 1024, 2e-6.
constexpr int kSliceFound = 1024;

// Two 32-bit operations in one instruction.
__device__ __forceinline__ float2 add2(float2 x, float2 y) {
  unsigned long long d;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(*reinterpret_cast<unsigned long long*>(&x)), "l"(*reinterpret_cast<unsigned long long*>(&y)));
  return *reinterpret_cast<float2*>(&d);
}
__device__ __forceinline__ float2 mul2(float2 x, float2 y) {
  unsigned long long d;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(*reinterpret_cast<unsigned long long*>(&x)), "l"(*reinterpret_cast<unsigned long long*>(&y)));
  return *reinterpret_cast<float2*>(&d);
}

// E logits per thread: a slice of kThreads * E words of one row.  A CTA takes `per_split` consecutive slices of a row
// and leaves a maximum, a sum and the `keep` best logits.  Every thread sums its own words against its own running
// maximum.  After the first slice, whose best make the bound that later logits have to reach, the warps go on without
// barriers, the next logits in flight.  Not bound by HBM: 7.6 instructions per logit (reading, maximum, difference,
// exponential, sum, comparison with the bound) and the latency of the beginning and the end of a CTA; 128 rows of 152,064
// fp32 logits, of which 64 MB are read: about 20 us, 3.2 TB/s (27.5 us with the joining kernel).
template <typename T, int E>
__global__ void __launch_bounds__(kThreads, 3) beam_slice_kernel(const T* __restrict__ logits, int64_t row_stride, int vocab, const float* __restrict__ cum,
                                                              const uint8_t* __restrict__ finished, int keep, int n_slices, int per_split, bool wide,
                                                              SliceStat* __restrict__ stat, Best* __restrict__ best) {
  constexpr int kVec = 16 / sizeof(T);
  constexpr float kLog2e = 1.4426950408889634f;
  __shared__ float s_group[kThreads], s_max[64], s_bound, s_x[kSliceFound], s_top[kThreads / 32];
  __shared__ int s_w[kSliceFound], s_n;
  __shared__ double s_sum[kThreads / 32];
  __shared__ Best s_keep[kMaxKeep];
  pdl_trigger();
  pdl_wait();
  const int row = blockIdx.y, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const float c = __ldg(cum + row);
  if ((finished && finished[row]) || !(c > -INFINITY)) return;
  const T* x0 = logits + row * row_stride;
  const int slice0 = blockIdx.x * per_split, slice1 = min(slice0 + per_split, n_slices);
  // element i of a thread is word slice * kThreads * E + (i / kVec) * kThreads * kVec + tid * kVec + i % kVec
  auto word = [&](int slice, int i) { return slice * kThreads * E + (i / kVec) * kThreads * kVec + tid * kVec + i % kVec; };
  auto load = [&](int slice, uint4 (&u)[E / kVec]) {
    const T* const p = x0 + word(slice, 0);
    if (wide && (slice + 1) * kThreads * E <= vocab) {
#pragma unroll
      for (int i = 0; i < E / kVec; ++i) u[i] = __ldcs(reinterpret_cast<const uint4*>(p) + i * kThreads);
      return;
    }
    const T none = static_cast<T>(-INFINITY);
#pragma unroll
    for (int i = 0; i < E / kVec; ++i)
#pragma unroll
      for (int j = 0; j < kVec; ++j) reinterpret_cast<T*>(u + i)[j] = word(slice, i * kVec + j) < vocab ? p[i * kThreads * kVec + j] : none;
  };
  uint4 next[E / kVec];
  load(slice0, next);
  if (tid == 0) s_n = 0;
  const int period = max(1, 512 / (4 * keep));      // slices between two cuts of the list
  float bound = -INFINITY;
  float ref = -INFINITY;       // the sum is of exp(x - ref)
  double sum = 0;
  bool overflow = false;
  for (int slice = slice0; slice < slice1; ++slice) {
    float x[E];
#pragma unroll
    for (int i = 0; i < E; ++i) x[i] = as_float<T>(reinterpret_cast<const T*>(next)[i]);
    if (slice + 1 < slice1) load(slice + 1, next);
    constexpr int kChunk = E / 4;
    float tops[4];             // of four stretches of the thread's words; a NaN loses every comparison
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      tops[j] = -INFINITY;
#pragma unroll
      for (int i = 0; i < kChunk; ++i) tops[j] = fmaxf(tops[j], x[j * kChunk + i]);
    }
    const float top = fminf(fmaxf(fmaxf(tops[0], tops[1]), fmaxf(tops[2], tops[3])), FLT_MAX);
    if (slice == slice0) bound = block_bound(top, keep, s_group, s_max, &s_bound);
    if (top > -INFINITY) {
      if (top > ref) {
        sum *= ex2((ref - top) * kLog2e);
        ref = top;
      }
      // The difference first (exact for the large terms), then one ex2 (relative error 2^-22).
      float2 part[2] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
#pragma unroll
      for (int i = 0; i < E; i += 2) {
        const float2 d = mul2(add2(make_float2(x[i], x[i + 1]), make_float2(-ref, -ref)), make_float2(kLog2e, kLog2e));
        part[i >> 1 & 1] = add2(part[i >> 1 & 1], make_float2(ex2(d.x), ex2(d.y)));
      }
      float total = (part[0].x + part[0].y) + (part[1].x + part[1].y);
      if (!(total <= FLT_MAX)) {      // a NaN or an infinity among them: once more, word by word
        total = 0.f;
#pragma unroll 1
        for (int i = 0; i < E; ++i) {
          const int w = word(slice, i);
          if (w < vocab) total += ex2((usable(as_float<T>(x0[w])) - ref) * kLog2e);
        }
      }
      sum += total;
      if (top >= bound) {
#pragma unroll
        for (int j = 0; j < 4; ++j)
          if (tops[j] >= bound) {
#pragma unroll
            for (int i = j * kChunk; i < (j + 1) * kChunk; ++i)
              if (x[i] >= bound && x[i] > -INFINITY) {
                const int at = atomicAdd(&s_n, 1);
                if (at < kSliceFound) {
                  s_x[at] = fminf(x[i], FLT_MAX);
                  s_w[at] = word(slice, i);
                }
              }
          }
      }
    }
    // Cut the list down to the best: after the first slice, at the end, and in between before it can run over (as it
    // still may where the logits rise from slice to slice).
    if ((slice - slice0) % period == 0 || slice + 1 == slice1) {
      __syncthreads();
      overflow |= s_n > kSliceFound;
      const int n = min(s_n, kSliceFound), kept = min(n, keep);
      for (int i = tid; i < n; i += kThreads) {
        int rank = 0;
        for (int j = 0; j < n; ++j) rank += ahead(s_x[j], s_w[j], s_x[i], s_w[i]);
        if (rank < keep) s_keep[rank] = {s_x[i], s_w[i]};
      }
      __syncthreads();
      if (tid < kept) {
        s_x[tid] = s_keep[tid].x;
        s_w[tid] = s_keep[tid].w;
      }
      if (tid == 0) s_n = kept;
      if (kept == keep) bound = fmaxf(bound, s_keep[keep - 1].x);
      __syncthreads();
    }
  }
  // The CTA's maximum and sum
  float top = ref;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
  if (lane == 0) s_top[warp] = top;
  __syncthreads();
  for (int w = 0; w < kThreads / 32; ++w) top = fmaxf(top, s_top[w]);
  sum *= ref == -INFINITY ? 0.f : ex2((ref - top) * kLog2e);
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
  if (lane == 0) s_sum[warp] = sum;
  __syncthreads();
  const int64_t out = static_cast<int64_t>(row) * gridDim.x + blockIdx.x;
  if (tid == 0) {
    double total = 0;
    for (int w = 0; w < kThreads / 32; ++w) total += s_sum[w];
    stat[out] = {total, top, 0};
  }
  Best* mine = best + out * keep;
  if (!overflow) {
    for (int i = tid; i < keep; i += kThreads) mine[i] = i < s_n ? Best{s_x[i], s_w[i]} : Best{-INFINITY, 0};
    return;
  }
  // More logits reach the bound than the list holds, equal ones or ones that rise from slice to slice: one after the
  // other, from memory.
  float last = INFINITY;
  int last_w = -1;
  for (int place = 0; place < keep; ++place) {
    float bx = -INFINITY;
    int bw = 0x7fffffff;
    for (int w = slice0 * kThreads * E + tid; w < min(slice1 * kThreads * E, vocab); w += kThreads) {
      const float y = usable(as_float<T>(x0[w]));
      if (y > -INFINITY && ahead(last, last_w, y, w) && ahead(y, w, bx, bw)) {
        bx = y;
        bw = w;
      }
    }
    block_best(bx, bw, s_x, s_w);
    if (tid == 0) mine[place] = {bx, bw};
    last = bx;
    last_w = bw;
  }
}

// One CTA per request joins the slices of its beams: 5 to 9 us, latency of its reads, of the sums in 64 bits and of the
// barriers.
constexpr int kFound = 1024;
__global__ void __launch_bounds__(kThreads) beam_join_kernel(int n_beams, int vocab, const float* __restrict__ cum, const uint8_t* __restrict__ finished,
                                                             int end_token, int keep, int n_splits, const SliceStat* __restrict__ stat,
                                                             const Best* __restrict__ best, float* __restrict__ score, int32_t* __restrict__ parent,
                                                             int32_t* __restrict__ token) {
  // of every beam: what its logits are measured from, log of the sum; a beam without candidates: +infinity, 0;
  // a finished one: NaN (its only candidate is the end token)
  __shared__ double s_top[kMaxKeep], s_log[kMaxKeep], s_cum[kMaxKeep];
  __shared__ double s_group[kThreads], s_max[64], s_bound, s_score[kFound], s_bx[kThreads / 32];
  __shared__ int s_at[kFound], s_n, s_bi[kThreads / 32];
  pdl_trigger();
  pdl_wait();
  const int req = blockIdx.x, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int row0 = req * n_beams, per_beam = n_splits * keep;
  for (int b = warp; b < n_beams; b += kThreads / 32) {
    const float c = __ldg(cum + row0 + b);
    const bool done = finished && finished[row0 + b];
    double top = INFINITY, sum = 1;
    if (done && c > -INFINITY) {
      top = NAN;
    } else if (c > -INFINITY) {
      const SliceStat* st = stat + static_cast<int64_t>(row0 + b) * n_splits;
      float m = -INFINITY;
      for (int i = lane; i < n_splits; i += 32) m = fmaxf(m, __ldcg(&st[i].top));
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
      sum = 0;
      for (int i = lane; i < n_splits; i += 32) {
        const float t = __ldcg(&st[i].top);
        if (t > -INFINITY) sum += __ldcg(&st[i].sum) * exp(static_cast<double>(t) - static_cast<double>(m));
      }
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
      if (m > -INFINITY) top = m;
    }
    if (lane == 0) {
      s_top[b] = top;
      s_log[b] = log(sum);
      s_cum[b] = c;
    }
  }
  if (tid == 0) s_n = 0;
  __syncthreads();

  // Calls f(score, index) for the thread's candidates.  They are dealt out one by one, of a beam first the best of every
  // slice, so that every group of threads whose maximum counts for the bound has some of the best, even if one beam holds
  // them all.
  const unsigned n_all = static_cast<unsigned>(n_beams) * per_beam;
  const Best* list = best + static_cast<int64_t>(row0) * per_beam;
  auto each = [&](auto f) {
#pragma unroll 4
    for (unsigned i = tid; i < n_all; i += kThreads) {
      const unsigned b = i / per_beam, r = i - b * per_beam, place = r / n_splits, split = r - place * n_splits;
      const double top = s_top[b];
      if (top < INFINITY) {
        const float2 e = __ldcg(reinterpret_cast<const float2*>(list + (b * n_splits + split) * keep + place));
        if (e.x > -INFINITY) f(s_cum[b] + ((static_cast<double>(e.x) - top) - s_log[b]), static_cast<int>(b) * vocab + __float_as_int(e.y));
      } else if (top != top && r == 0) {
        f(s_cum[b], static_cast<int>(b) * vocab + end_token);
      }
    }
  };
  double my = -INFINITY;
  each([&](double sc, int) { my = sc > my ? sc : my; });
  const double bound = block_bound(my, keep, s_group, s_max, &s_bound);
  if (my >= bound)
    each([&](double sc, int at) {
      if (sc >= bound) {
        const int place = atomicAdd(&s_n, 1);
        if (place < kFound) {
          s_score[place] = sc;
          s_at[place] = at;
        }
      }
    });
  __syncthreads();
  const int found = s_n;
  float* o_score = score + static_cast<int64_t>(req) * keep;
  int32_t* o_parent = parent + static_cast<int64_t>(req) * keep;
  int32_t* o_token = token + static_cast<int64_t>(req) * keep;
  auto put = [&](int place, double sc, int at) {
    const bool none = sc == -INFINITY;
    o_score[place] = static_cast<float>(sc);
    o_parent[place] = none ? 0 : at / vocab;
    o_token[place] = none ? -1 : at % vocab;
  };
  for (int i = found + tid; i < keep; i += kThreads) put(i, -INFINITY, 0);
  if (found <= kFound) {
    for (int i = tid; i < found; i += kThreads) {
      const double sc = s_score[i];
      const int at = s_at[i];
      int rank = 0;
#pragma unroll 8
      for (int j = 0; j < found; ++j) rank += ahead(s_score[j], s_at[j], sc, at);
      if (rank < keep) put(rank, sc, at);
    }
    return;
  }
  // More candidates near the bound than fit (thousands of equal scores): one after the other.
  double last = INFINITY;
  int last_at = -1;
  for (int place = 0; place < keep; ++place) {
    double bs = -INFINITY;
    int ba = 0x7fffffff;
    each([&](double sc, int at) {
      if (ahead(last, last_at, sc, at) && ahead(sc, at, bs, ba)) {
        bs = sc;
        ba = at;
      }
    });
    block_best(bs, ba, s_bx, s_bi);
    if (tid == 0) put(place, bs, ba);
    last = bs;
    last_at = ba;
  }
}

// How a row is cut.  Words per thread: 8 where all slices then fit the GPU at a time, for the latency of small calls (four
// rows of 32,000 logits: 7.7 us, with 32 words 9.0; of 64,000: 8.8 and 9.1), else 32 (eight rows of 152,064: 14.1 us, with 8
// words 17.8; 24 rows of it: 15.8 and 27).  A row's slices are dealt to as many CTAs as fit the GPU at a time.
struct Cut {
  int words, n_slices, n_splits, per_split;
};
Cut cut_of(int64_t rows, int vocab) {
  constexpr int kSms = 148;
  Cut c;
  c.words = rows * ((vocab + 8 * kThreads - 1) / (8 * kThreads)) <= 3 * kSms ? 8 : 32;
  c.n_slices = (vocab + c.words * kThreads - 1) / (c.words * kThreads);
  const int64_t splits = std::min<int64_t>(c.n_slices, std::max<int64_t>(1, 3 * kSms / rows));
  c.per_split = static_cast<int>((c.n_slices + splits - 1) / splits);
  c.n_splits = (c.n_slices + c.per_split - 1) / c.per_split;
  return c;
}

template <typename T>
cudaError_t launch_select(const void* logits, int n_req, int n_beams, int vocab, int64_t row_stride, const float* cum, const uint8_t* finished,
                          int end_token, int keep, float* score, int32_t* parent, int32_t* token, void* workspace, cudaStream_t st) {
  const int64_t rows = static_cast<int64_t>(n_req) * n_beams;
  const Cut cut = cut_of(rows, vocab);
  SliceStat* stat = static_cast<SliceStat*>(workspace);
  Best* best = reinterpret_cast<Best*>(stat + rows * cut.n_splits);
  const bool wide = (reinterpret_cast<uintptr_t>(logits) & 15) == 0 && row_stride % (16 / static_cast<int64_t>(sizeof(T))) == 0;
  const dim3 grid(static_cast<unsigned>(cut.n_splits), static_cast<unsigned>(rows));
  auto kernel = cut.words == 32 ? beam_slice_kernel<T, 32> : beam_slice_kernel<T, 8>;
  cudaError_t err = launch_pdl(kernel, grid, dim3(kThreads), 0, st, static_cast<const T*>(logits), row_stride, vocab, cum, finished, keep,
                               cut.n_slices, cut.per_split, wide, stat, best);
  if (err != cudaSuccess) return err;
  return launch_pdl(beam_join_kernel, dim3(static_cast<unsigned>(n_req)), dim3(kThreads), 0, st, n_beams, vocab, cum, finished, end_token, keep, cut.n_splits,
                    static_cast<const SliceStat*>(stat), static_cast<const Best*>(best), score, parent, token);
}

const char* select_error(int n_req, int n_beams, int vocab, int keep) {
  if (n_req < 1 || vocab < 1) return "n_req and vocab must be positive";
  if (n_beams < 1 || n_beams > kMaxKeep || keep < 1 || keep > kMaxKeep) return "n_beams and keep are 1..64";
  if (vocab > 2147483647 - 8191) return "vocab is above 2^31 - 8192";      // words are numbered in 32 bits to the end of the last slice
  if (static_cast<int64_t>(n_beams) * vocab > 2147483647) return "n_beams * vocab reaches 2^31";
  if (static_cast<int64_t>(n_req) * n_beams > 65535) return "more than 65535 beams";
  return nullptr;
}

}  // namespace
}  // namespace prima

using namespace prima;

extern "C" {

int64_t prima_beam_select_workspace(int n_req, int n_beams, int vocab, int keep) {
  if (select_error(n_req, n_beams, vocab, keep)) return PRIMA_ERR_ARG;
  const int64_t rows = static_cast<int64_t>(n_req) * n_beams;
  const Cut cut = cut_of(rows, vocab);
  return rows * cut.n_splits * (static_cast<int64_t>(sizeof(SliceStat)) + static_cast<int64_t>(keep) * static_cast<int64_t>(sizeof(Best)));
}

int prima_beam_select(const void* logits, int dtype, int n_req, int n_beams, int vocab, int64_t row_stride, const float* cum,
                      const uint8_t* finished, int end_token, int keep, float* score, int32_t* parent, int32_t* token, void* workspace,
                      int64_t workspace_bytes, void* stream) {
  if (const char* bad = select_error(n_req, n_beams, vocab, keep)) {
    char msg[120];
    snprintf(msg, sizeof msg, "prima_beam_select: %s", bad);
    return call_fail(PRIMA_ERR_ARG, msg);
  }
  if (!logits || !cum || !score || !parent || !token || !workspace) return call_fail(PRIMA_ERR_ARG, "prima_beam_select: null argument");
  if (dtype != PRIMA_DT_F32 && dtype != PRIMA_DT_F16 && dtype != PRIMA_DT_BF16) return call_fail(PRIMA_ERR_ARG, "prima_beam_select: unknown dtype");
  if (!aligned_to(logits, dtype == PRIMA_DT_F32 ? 4 : 2) || !aligned_to(cum, 4) || !aligned_to(score, 4) || !aligned_to(parent, 4) || !aligned_to(token, 4))
    return call_fail(PRIMA_ERR_ARG, "prima_beam_select: an array is not aligned to its elements");
  if (row_stride < vocab) return call_fail(PRIMA_ERR_ARG, "prima_beam_select: row_stride is shorter than a row");
  if (finished && (end_token < 0 || end_token >= vocab)) return call_fail(PRIMA_ERR_ARG, "prima_beam_select: end_token outside the vocabulary");
  if ((reinterpret_cast<uintptr_t>(workspace) & 255) || workspace_bytes < prima_beam_select_workspace(n_req, n_beams, vocab, keep))
    return call_fail(PRIMA_ERR_ARG, "prima_beam_select: workspace too small or not 256-byte aligned");
  auto run = dtype == PRIMA_DT_F32 ? launch_select<float> : dtype == PRIMA_DT_F16 ? launch_select<__half> : launch_select<__nv_bfloat16>;
  const cudaError_t e = run(logits, n_req, n_beams, vocab, row_stride, cum, finished, end_token, keep, score, parent, token, workspace,
                            static_cast<cudaStream_t>(stream));
  return e == cudaSuccess ? PRIMA_OK : call_cuda_fail(e, "prima_beam_select");
}

}  // extern "C"
