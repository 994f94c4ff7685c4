// token_logprobs.cu -- log probabilities of given tokens, the entropy of their
// distributions and the likeliest alternatives (hpd_token_logprobs).
//
//   d_v = (x_v - max x) scale,  Z = sum exp(d_v) = 1 + R   (R without one largest term)
//   logprob = d_token - log(1 + R),  entropy = log(1 + R) - sum exp(d_v) d_v / Z
// Both terms of the entropy are positive, and log(1 + R) keeps the digits of a small
// R: nothing cancels where a token is nearly sure.
//
// A row is read once, 16 bytes a load, by a CTA of 256 threads or, of few rows, by a cluster
// of up to eight.  Every thread has sums in 32 bits against a base of its own, the largest of
// its first pieces with a value above -inf, moved only by a value 2^kWindow above it: no branch
// depends on where a row's maxima stand.  All values are in the sums; where that leaves the rest of a row too few
// digits beside its largest value (a rest below kSure), the thread that has that one sums its
// values once more without it, and the others lose nothing.
// Top values: every thread knows its own maximum.  The top-th largest maximum of 64 groups
// of threads is a lower bound of the last of the top values, which only few threads (some
// 1.5 times `top`) reach: their pieces are read again, from L2, by the whole CTA, and what
// reaches the bound (a few more than `top`) is ranked, each against all.  Many equal values,
// or an order that follows a thread's share, give too many: then the value that the last of
// them has is found by halving the range of its bits, a pass over the share each.
//
// What bounds it, and what it measured on a GB300 (in a graph):
//   6,144 rows of 32,000 in bf16, sums alone: 68.4 us, 5.7 TB/s, 85 % of a copy's rate; with
//     8 alternatives 92.0: six barriers and two dependent reads of L2 a row, during which the
//     SM's other four CTAs stream; with 32 alternatives 114.
//   160 rows of 100,003 in fp32: 15.1 us; with 20 alternatives 21.2, of which 6 are those.
//   64 rows of 32,000: 4.1 us, with 8 alternatives 6.0; one row of 151,936 4.3, with 20 9.9:
//     latency: loads, join, bound, second reads, ranks, and the lists of a cluster's CTAs.
// A warp a row, each value against a running maximum: 1,263 us for the 6,144 rows.  Rereading by the warps that have the hot threads (eight of them in one warp,
// one after the other) and ranks by a scan of the cluster's lists: 160 rows 27.4, one 13.8.
#include <cooperative_groups.h>

#include <atomic>

#include "common.cuh"

namespace cg = cooperative_groups;

namespace hpd {
namespace {

constexpr int kThreads = 256, kWarps = kThreads / 32;
constexpr int kUnroll = 4;      // 16-byte loads of a thread on their way at once
constexpr int kCtasPerSm = 5;
constexpr int kMaxCluster = 8;  // CTAs of a row
constexpr int kTop = 32;
// A sum of weights beside the largest one's 1 below which that is left out of them: 2^-24 of
// it is 2^-22 of the rest here.
constexpr float kSure = 0.25f;
constexpr int kGroups = 64;      // of threads, whose maxima bound the top values from below
constexpr int kCandidates = 1024;
constexpr int kLogpSms = 152;

struct LogpArgs {
  const void *logits;
  long long row_stride;
  const int32_t *tokens;
  float *logprob, *entropy;
  int32_t *top_tokens;
  float *top_logprobs;
  int V, top;
  float scale, scale_log2;
};

__device__ __forceinline__ float inf() { return __int_as_float(0x7f800000); }
__device__ __forceinline__ float nan() { return __int_as_float(0x7fffffff); }

// A place in a row's order: larger values first, lower indices first among equal ones.
struct Place {
  float x;
  int i;
};
__device__ __forceinline__ bool before(const Place &a, const Place &b) { return a.x > b.x || (a.x == b.x && a.i < b.i); }

// The order of values as whole numbers (-0 is +0).
__device__ __forceinline__ uint32_t key_of(float x) {
  const uint32_t u = __float_as_uint(x + 0.f);
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}

__device__ __forceinline__ float value_of(uint32_t key) {
  return __uint_as_float(key & 0x80000000u ? key & 0x7fffffffu : ~key);
}

// 16 bytes of a row, and their largest value (NaN only if there is nothing else).
template <class T>
struct Vec;
template <>
struct Vec<__nv_bfloat16> {
  static constexpr int kN = 8;
  static __device__ __forceinline__ void unpack(const uint4 &v, float *x) {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[2 * i] = __uint_as_float(w[i] << 16);
      x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
  }
  static __device__ __forceinline__ uint32_t max2(uint32_t a, uint32_t b) {
    asm("max.bf16x2 %0, %0, %1;" : "+r"(a) : "r"(b));
    return a;
  }
  static __device__ __forceinline__ uint32_t fold(const uint4 &v) { return max2(max2(v.x, v.y), max2(v.z, v.w)); }
  static __device__ __forceinline__ float of_fold(uint32_t w) {
    return fmaxf(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u));
  }
  static __device__ __forceinline__ float largest(const uint4 &v) { return of_fold(fold(v)); }
  static __device__ __forceinline__ float largest4(const uint4 *v) {
    return of_fold(max2(max2(fold(v[0]), fold(v[1])), max2(fold(v[2]), fold(v[3]))));
  }
};
template <>
struct Vec<float> {
  static constexpr int kN = 4;
  static __device__ __forceinline__ void unpack(const uint4 &v, float *x) {
    x[0] = __uint_as_float(v.x);
    x[1] = __uint_as_float(v.y);
    x[2] = __uint_as_float(v.z);
    x[3] = __uint_as_float(v.w);
  }
  static __device__ __forceinline__ float largest(const uint4 &v) {
    return fmaxf(fmaxf(__uint_as_float(v.x), __uint_as_float(v.y)), fmaxf(__uint_as_float(v.z), __uint_as_float(v.w)));
  }
  static __device__ __forceinline__ float largest4(const uint4 *v) {
    return fmaxf(fmaxf(largest(v[0]), largest(v[1])), fmaxf(largest(v[2]), largest(v[3])));
  }
};

// Of some values: the largest; with d = (x - m) scale log2(e) the sums of 2^d, but for one
// of the largest values (whose 2^d is 1), and of 2^d d.  NaN among them is in `rest`.
struct Sums {
  float m, rest, mean;
};
// log2: a limit kWindow above a base may be twice that above it once rounded (a step of the
// values may be as much), and sums of 2^30 terms have to fit all the same; 2^kNothing is 0.
constexpr float kWindow = 45.f, kNothing = -300.f;

__device__ __forceinline__ float max_nan(float a, float b) {
  asm("max.NaN.f32 %0, %0, %1;" : "+f"(a) : "f"(b));
  return a;
}

// A thread's values.  Sums are taken against a base, the largest of the first piece that has a
// value above -inf, which moves only when a value passes it by 2^kWindow: no branch depends on
// where a row's maxima stand (one at every new maximum had two in three of the pieces in both of
// its sides).  Until then there is nothing to sum: a base of 0, say, would lose all of a row
// that begins with -inf and whose other values are e^-88 and less.  All values are in the sums; of a row whose other values have little weight
// beside the largest, whoever has that sums once more without it.
template <class T>
struct Running {
  float m;            // the largest value; -inf: none yet
  float base, limit;  // and what moves it (-inf: there is none yet; NaN: bf16, and no floor below it is a number)
  uint32_t floor2;    // bf16: what is below has 2^d = 0
  float2 sum, mean;   // of 2^d and 2^d d, d against the base

  __device__ __forceinline__ void set_base(float b, float c) {
    base = b;
    limit = b + kWindow / c;
    if (sizeof(T) == 2) {
      // (2^-6 of the base: the floor stays that far below it once rounded)
      const float f = b - fmaxf(-kNothing / c, fabsf(b) * 0x1p-6f);
      floor2 = pack_bf16x2(f, f);
      if (b < -1e37f) limit = nan();
    }
  }
  __device__ __forceinline__ void start(float c) {
    m = -inf();
    sum = mean = make_float2(0.f, 0.f);
    set_base(0.f, c);
    limit = -inf();
  }
  __device__ __forceinline__ void add2(float2 x, bool floored, float c) {
    float2 d = __fmul2_rn(__fadd2_rn(x, make_float2(-base, -base)), make_float2(c, c));
    // (0 times minus infinity is kept out)
    if (!floored) d = make_float2(max_nan(d.x, kNothing), max_nan(d.y, kNothing));
    const float2 e = make_float2(fast_exp2(d.x), fast_exp2(d.y));
    sum = __fadd2_rn(sum, e);
    mean = __ffma2_rn(e, d, mean);
  }
  template <bool kFloored>
  __device__ __forceinline__ void add(const uint4 &v, float c) {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
    if constexpr (sizeof(T) == 4) {
      add2(make_float2(__uint_as_float(w[0]), __uint_as_float(w[1])), false, c);
      add2(make_float2(__uint_as_float(w[2]), __uint_as_float(w[3])), false, c);
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        uint32_t u = w[i];
        if (kFloored) asm("max.NaN.bf16x2 %0, %0, %1;" : "+r"(u) : "r"(floor2));
        // (a product and not a shift: another pipe)
        add2(make_float2(__uint_as_float(u * 65536u), __uint_as_float(u & 0xffff0000u)), kFloored, c);
      }
    }
  }
  // N pieces, the largest of whose values is given.
  template <int N>
  __device__ __forceinline__ void take(const uint4 *v, float largest, float c) {
    m = fmaxf(m, largest);
    if (!(largest <= limit)) {
      if (limit == -inf() || largest > base + kWindow / c) raise(largest, c);
      if (limit != limit) {
#pragma unroll
        for (int i = 0; i < N; ++i) add<false>(v[i], c);
        return;
      }
    }
#pragma unroll
    for (int i = 0; i < N; ++i) add<true>(v[i], c);
  }
  __device__ __forceinline__ void raise(float to, float c) {
    const float d = fminf(fmaxf((base - to) * c, kNothing), 0.f), w = fast_exp2(d);
    // (w is 0 where nothing is left; sums that are NaN stay NaN; of a first base they are 0, or NaN)
    mean = make_float2(w * fmaf(d, sum.x, mean.x), w * fmaf(d, sum.y, mean.y));
    sum = make_float2(w * sum.x, w * sum.y);
    set_base(to, c);
  }
  // The sums against the thread's own largest value, that one among them.
  __device__ __forceinline__ Sums result(float c) const {
    Sums s{m, sum.x + sum.y, mean.x + mean.y};
    if (m == -inf()) return s;
    const float d = fmaxf((base - m) * c, kNothing), w = fast_exp2(d);
    s.mean = w * fmaf(d, s.rest, s.mean);
    s.rest *= w;
    return s;
  }
};

// Of two parts, each without one of its largest values.
__device__ __forceinline__ Sums join(Sums a, Sums b, float c) {
  if (b.m > a.m) {
    const Sums t = a;
    a = b;
    b = t;
  }
  if (b.m > -inf()) {
    const float d = (b.m - a.m) * c, w = fast_exp2(d), z = 1.f + b.rest;
    a.rest += w * z;
    if (w != 0.f) a.mean += w * fmaf(d, z, b.mean);
  } else {
    a.rest += b.rest;
  }
  return a;
}
// Of the parts of n lanes (a power of two), each with its largest value in `rest`.
__device__ __forceinline__ Sums join_lanes(Sums s, int n, float c) {
  float m = s.m;
#pragma unroll
  for (int o = 1; o < n; o <<= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
  const float d = s.m == m ? 0.f : fmaxf((s.m - m) * c, kNothing), w = fast_exp2(d);
  s.mean = w * fmaf(d, s.rest, s.mean);
  s.rest *= w;
  s.m = m;
#pragma unroll
  for (int o = 1; o < n; o <<= 1) {
    s.rest += __shfl_xor_sync(0xffffffffu, s.rest, o);
    s.mean += __shfl_xor_sync(0xffffffffu, s.mean, o);
  }
  return s;
}

struct LogpShared {
  Sums warp[kWarps];
  float2 again[kWarps];
  uint32_t __align__(16) group[kGroups];  // keys of the groups' maxima, made different by the groups' numbers
  uint32_t least;  // a lower bound of the last of the top values, as a key
  int found;       // candidates, some perhaps beyond their room
  int count;       // of a scan
  int hots;        // threads whose largest value reaches the bound, and which
  uint8_t hot[kThreads];
  int per_warp[kWarps];
  Place candidate[kCandidates];
  Place best[kTop];
  // of the CTAs of a row, in the first one
  Sums part[kMaxCluster];
  Place list[kMaxCluster][kTop];
};

// A CTA's share of a row: single values up to an aligned address (the first CTA's) and
// behind the last whole 16 bytes (the last one's), and the 16-byte pieces between.
template <class T>
struct Share {
  const T *row;
  int head, tail0, tail;  // values before the pieces; first and number of those behind
  int v0, v1;             // pieces
  __device__ __forceinline__ uint4 piece(int v) const { return reinterpret_cast<const uint4 *>(row + head)[v]; }
  __device__ __forceinline__ int index(int v) const { return head + v * Vec<T>::kN; }
};

// f(value, index) of every value of the share, a piece a thread.
template <class T, class F>
__device__ __forceinline__ void for_values(const Share<T> &s, F f) {
  const int tid = threadIdx.x;
  if (tid < s.head && s.v0 == 0) f(static_cast<float>(s.row[tid]), tid);
  if (tid < s.tail) f(static_cast<float>(s.row[s.tail0 + tid]), s.tail0 + tid);
#pragma unroll 1
  for (int v = s.v0 + tid; v < s.v1; v += kThreads) {
    float x[Vec<T>::kN];
    Vec<T>::unpack(s.piece(v), x);
#pragma unroll
    for (int i = 0; i < Vec<T>::kN; ++i) f(x[i], s.index(v) + i);
  }
}

__device__ __forceinline__ void propose(LogpShared &sh, float x, int i) {
  const int at = atomicAdd(&sh.found, 1);
  if (at < kCandidates) sh.candidate[at] = Place{x, i};
}

// The first values of the share that equal x, in the order of their indices, `need` of
// them at most, become candidates.
template <class T>
__device__ __noinline__ void propose_equal(LogpShared &sh, const Share<T> &s, float x, int need) {
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int begin = s.v0 == 0 ? 0 : s.index(s.v0), end = s.tail ? s.tail0 + s.tail : s.index(s.v1);
  for (int i0 = begin; i0 < end && need > 0; i0 += kThreads) {
    const int i = i0 + tid;
    const bool here = i < end && static_cast<float>(s.row[i]) == x;
    const unsigned all = __ballot_sync(0xffffffffu, here);
    if (lane == 0) sh.per_warp[warp] = __popc(all);
    __syncthreads();
    int at = __popc(all & ((1u << lane) - 1u)), total = 0;
    for (int w = 0; w < kWarps; ++w) {
      at += w < warp ? sh.per_warp[w] : 0;
      total += sh.per_warp[w];
    }
    if (here && at < need) propose(sh, x, i);
    need -= total;
    __syncthreads();
  }
}

// Too many values reach the bound (ties, or an order that a thread's share of the row
// follows): the last of the top values by halving the range of keys, a pass over the
// share each time, then those above it and the first of its equals.
template <class T>
__device__ __noinline__ void select_by_halves(LogpShared &sh, const Share<T> &s, int top) {
  uint32_t lo = sh.least, hi = 0xffffffffu;
  while (lo < hi) {
    const uint32_t mid = lo + (hi - lo) / 2 + 1;
    __syncthreads();
    if (threadIdx.x == 0) sh.count = 0;
    __syncthreads();
    int n = 0;
    for_values(s, [&](float x, int) { n += x == x && key_of(x) >= mid; });
    n = __reduce_add_sync(0xffffffffu, n);
    if ((threadIdx.x & 31) == 0) atomicAdd(&sh.count, n);
    __syncthreads();
    if (sh.count >= top) lo = mid; else hi = mid - 1;
  }
  __syncthreads();
  if (threadIdx.x == 0) sh.found = 0;
  __syncthreads();
  for_values(s, [&](float x, int i) {
    if (x == x && key_of(x) > lo) propose(sh, x, i);
  });
  __syncthreads();
  const int need = top - sh.found;
  propose_equal(sh, s, value_of(lo), need);
}

__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.aligned;" ::: "memory"); }

// A row has a cluster of `ctas` CTAs, each with its share of the row, read once:
//  - sums against each thread's own maximum, joined over the CTA;
//  - top values: every thread's maximum is known, so that of 64 groups of threads; the
//    top-th largest of those bounds the top values from below.  Only threads whose maximum
//    reaches the bound (some 1.5 times `top` of them) look at their values again, in L2, a
//    warp at each, and what reaches it is ranked against one another.
// The first CTA joins the others' sums and lists, which come through distributed shared
// memory.
template <class T, bool kAlternatives>
__global__ void __launch_bounds__(kThreads, kCtasPerSm) token_logprobs_kernel(const LogpArgs a, int ctas) {
  using V = Vec<T>;
  __shared__ LogpShared sh;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int rank = ctas > 1 ? static_cast<int>(blockIdx.x % ctas) : 0;
  const size_t r = ctas > 1 ? blockIdx.x / ctas : blockIdx.x;
  const float c = a.scale_log2;
  if (ctas > 1) cluster_arrive();
  pdl_wait();
  pdl_trigger();
  Share<T> s;
  s.row = static_cast<const T *>(a.logits) + static_cast<long long>(r) * a.row_stride;
  s.head = min(a.V, static_cast<int>((16u - (reinterpret_cast<uintptr_t>(s.row) & 15u)) & 15u) / static_cast<int>(sizeof(T)));
  const int pieces = (a.V - s.head) / V::kN;
  s.v0 = static_cast<int>(static_cast<long long>(pieces) * rank / ctas);
  s.v1 = static_cast<int>(static_cast<long long>(pieces) * (rank + 1) / ctas);
  s.tail0 = s.head + pieces * V::kN;
  s.tail = rank == ctas - 1 ? a.V - s.tail0 : 0;
  float x_token = 0.f;
  int token = -1;
  if (rank == 0 && tid == 0) {
    token = a.tokens[r];
    if (token >= 0 && token < a.V) x_token = static_cast<float>(s.row[token]);
  }

  Running<T> run;
  // a single value, as a piece with nothing else
  auto single = [&](int i) {
    uint4 w;
    if constexpr (sizeof(T) == 2)
      w = make_uint4(0xff800000u | *reinterpret_cast<const uint16_t *>(s.row + i), 0xff80ff80u, 0xff80ff80u, 0xff80ff80u);
    else
      w = make_uint4(__float_as_uint(s.row[i]), 0xff800000u, 0xff800000u, 0xff800000u);
    run.template take<1>(&w, V::largest(w), c);
  };
  run.start(c);
  int v = s.v0 + tid;
#pragma unroll 1
  for (; v + (kUnroll - 1) * kThreads < s.v1; v += kUnroll * kThreads) {
    uint4 w[kUnroll];
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) w[u] = s.piece(v + u * kThreads);
    run.template take<kUnroll>(w, V::largest4(w), c);
  }
#pragma unroll 1
  for (; v < s.v1; v += kThreads) {
    const uint4 w = s.piece(v);
    run.template take<1>(&w, V::largest(w), c);
  }
  if (tid < s.head && rank == 0) single(tid);
  if (tid < s.tail) single(s.tail0 + tid);
  if constexpr (kAlternatives) {
    float g = run.m;
#pragma unroll
    for (int o = 1; o < kThreads / kGroups; o <<= 1) g = fmaxf(g, __shfl_xor_sync(0xffffffffu, g, o));
    if (lane % (kThreads / kGroups) == 0) {
      const int k = tid / (kThreads / kGroups);
      sh.group[k] = (key_of(g) & ~static_cast<uint32_t>(kGroups - 1)) | k;
    }
    if (tid == 0) sh.found = sh.hots = 0;
  }
  const Sums own = run.result(c);
  Sums all = join_lanes(own, 32, c);
  if (lane == 0) sh.warp[warp] = all;
  __syncthreads();
  all = join_lanes(sh.warp[lane % kWarps], kWarps, c);
  all.rest -= 1.f;
  // f(value) of the share's values that thread t of this warp has, by all of its lanes
  auto again = [&](int t, auto f) {
    if (lane == 0 && t < s.head && rank == 0) f(static_cast<float>(s.row[t]));
    if (lane == 31 && t < s.tail) f(static_cast<float>(s.row[s.tail0 + t]));
#pragma unroll 1
    for (int v = s.v0 + t + lane * kThreads; v < s.v1; v += 32 * kThreads) {
      const uint4 w = s.piece(v);
      float x[V::kN];
      V::unpack(w, x);
#pragma unroll
      for (int i = 0; i < V::kN; ++i) f(x[i]);
    }
  };
  if (all.rest < kSure) {  // (as for all of the CTA) the largest value leaves its sum too few digits
    const float m = all.m;
    float2 part = make_float2(0.f, 0.f);
    if (own.m > -inf() && own.m < m) {
      const float d = (own.m - m) * c, w = fast_exp2(d);
      part = make_float2(w * own.rest, w == 0.f ? 0.f : w * fmaf(d, own.rest, own.mean));
    }
    const unsigned has = __ballot_sync(0xffffffffu, own.m == m);  // one thread of the CTA
    if (has)
      again(warp * 32 + __ffs(has) - 1, [&](float x) {
        const float d = fmaxf((x - m) * c, kNothing), e = x == m ? 0.f : fast_exp2(d);
        part.x += e;
        part.y = fmaf(e, d, part.y);
      });
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
      part.x += __shfl_xor_sync(0xffffffffu, part.x, o);
      part.y += __shfl_xor_sync(0xffffffffu, part.y, o);
    }
    if (lane == 0) sh.again[warp] = part;
    __syncthreads();
    all.rest = all.mean = 0.f;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) {
      all.rest += sh.again[w].x;
      all.mean += sh.again[w].y;
    }
  }

  if constexpr (kAlternatives) {
    const int top = a.top;
    if (tid < top) sh.best[tid] = Place{nan(), -1};
    {  // the top-th largest of the groups' maxima, a group's place by four threads
      constexpr int kPer = kThreads / kGroups;
      const uint32_t key = sh.group[tid / kPer];
      int ahead = 0;
#pragma unroll
      for (int j = 0; j < kGroups / kPer; j += 4) {
        const uint4 k = *reinterpret_cast<const uint4 *>(sh.group + tid % kPer * (kGroups / kPer) + j);
        ahead += (k.x > key) + (k.y > key) + (k.z > key) + (k.w > key);
      }
#pragma unroll
      for (int o = 1; o < kPer; o <<= 1) ahead += __shfl_xor_sync(0xffffffffu, ahead, o);
      if (tid % kPer == 0 && ahead == top - 1) sh.least = key & ~static_cast<uint32_t>(kGroups - 1);
    }
    __syncthreads();
    // (else fewer than `top` groups have a value above -inf: those are looked for)
    const bool any = sh.least >= key_of(-3.4028235e38f);
    const float least = any ? value_of(sh.least) : -inf();
    auto reaches = [&](float x) { return any ? x >= least : x > least; };
    auto look = [&](float x, int i) {
      if (reaches(x)) propose(sh, x, i);
    };
    // threads whose largest value reaches the bound: their pieces, by all threads
    if (reaches(run.m)) {
      sh.hot[atomicAdd(&sh.hots, 1)] = static_cast<uint8_t>(tid);
      if (tid < s.head && rank == 0) look(static_cast<float>(s.row[tid]), tid);
      if (tid < s.tail) look(static_cast<float>(s.row[s.tail0 + tid]), s.tail0 + tid);
    }
    __syncthreads();
    const int each = (s.v1 - s.v0 + kThreads - 1) / kThreads, work = sh.hots * each;
#pragma unroll 1
    for (int i0 = tid; i0 - tid < work; i0 += kUnroll * kThreads) {
      uint4 w[kUnroll];
      int v[kUnroll];
#pragma unroll
      for (int u = 0; u < kUnroll; ++u) {
        const int i = i0 + u * kThreads, t = i / each;
        v[u] = i < work ? s.v0 + sh.hot[t] + (i - t * each) * kThreads : s.v1;
        if (v[u] < s.v1) w[u] = s.piece(v[u]);
      }
#pragma unroll
      for (int u = 0; u < kUnroll; ++u) {
        if (v[u] >= s.v1 || V::largest(w[u]) < least) continue;
        float x[V::kN];
        V::unpack(w[u], x);
#pragma unroll
        for (int e = 0; e < V::kN; ++e) look(x[e], s.index(v[u]) + e);
      }
    }
    __syncthreads();
    if (sh.found > kCandidates || (!any && sh.found < top)) {
      if (sh.found > kCandidates) select_by_halves(sh, s, top);
      else propose_equal(sh, s, -inf(), top - sh.found);
      __syncthreads();
    }
    const int found = min(sh.found, kCandidates);
    if (found <= kThreads / 4) {  // a candidate's place by four threads
      const Place p = sh.candidate[min(tid / 4, max(found - 1, 0))];
      int ahead = 0;
      for (int j = tid % 4; j < found; j += 4) ahead += before(sh.candidate[j], p);
      ahead += __shfl_xor_sync(0xffffffffu, ahead, 1);
      ahead += __shfl_xor_sync(0xffffffffu, ahead, 2);
      if (tid % 4 == 0 && tid / 4 < found && ahead < top) sh.best[ahead] = p;
    } else {
      for (int k = tid; k < found; k += kThreads) {
        const Place p = sh.candidate[k];
        int ahead = 0;
        for (int j = 0; j < found; ++j) ahead += before(sh.candidate[j], p);
        if (ahead < top) sh.best[ahead] = p;
      }
    }
    __syncthreads();
  }

  if (ctas > 1) {
    cg::cluster_group cluster = cg::this_cluster();
    cluster_wait();  // (the first CTA runs: its shared memory may be written)
    LogpShared *first = cluster.map_shared_rank(&sh, 0);
    if (tid == 0) first->part[rank] = all;
    if (kAlternatives && tid < a.top) first->list[rank][tid] = sh.best[tid];
    cluster.sync();
    if (rank != 0) return;
  }
  if (ctas > 1) {
    all = sh.part[0];
#pragma unroll 1
    for (int w = 1; w < ctas; ++w) all = join(all, sh.part[w], c);
  }
  if (!(fabsf(all.m) < inf())) all.rest = nan();
  const float log_z = log1pf(all.rest);
  // (by halves, which are exact: a difference of two logits may be out of range)
  auto logprob = [&](float x) {
    return all.rest == all.rest ? (0.5f * x - 0.5f * all.m) * (2.f * a.scale) - log_z : nan();
  };
  if (tid == 0) {
    a.logprob[r] = logprob(token >= 0 && token < a.V ? x_token : -inf());
    if (a.entropy) a.entropy[r] = log_z - all.mean * kLn2 / (1.f + all.rest);
  }
  if constexpr (kAlternatives) {
    const int top = a.top;
    auto put = [&](int k, const Place &p) {
      a.top_tokens[r * top + k] = p.i;
      a.top_logprobs[r * top + k] = p.i >= 0 ? logprob(p.x) : nan();
    };
    if (ctas == 1) {
      if (tid < top) put(tid, sh.best[tid]);
      return;
    }
    if (tid < top) sh.best[tid] = Place{nan(), -1};
    __syncthreads();
    if (tid < ctas * top) {
      const Place p = sh.list[tid / top][tid % top];
      int ahead = 0;
#pragma unroll 4
      for (int w = 0; w < ctas; ++w) {  // how many of each list, which are in order, come before
        int at = 0;
#pragma unroll
        for (int half = kTop / 2; half > 0; half /= 2)
          if (at + half <= top && before(sh.list[w][at + half - 1], p)) at += half;
        if (at < top && before(sh.list[w][at], p)) ++at;
        ahead += at;
      }
      if (p.i >= 0 && ahead < top) sh.best[ahead] = p;
    }
    __syncthreads();
    if (tid < top) put(tid, sh.best[tid]);
  }
}

template <class T, bool kAlternatives>
cudaError_t launch_logprobs(const LogpArgs &k, int R, cudaStream_t s) {
  // CTAs of a row: as many as keep the GPU's SMs busy, none with less than 32 KB, or 64 where the
  // cluster has lists to join, which costs some 1 us a doubling.  One, two, four and eight CTAs, 64
  // rows in bf16 (us, in a graph):
  //                                    32,000               32,768               65,536               100,003
  //   sums alone             4.1  4.1  4.1  5.7   3.9  3.5  3.4  5.5   5.7  4.4  4.0  6.0   8.1  5.7  5.0   7.2
  //   with 8 alternatives    5.9  7.2  8.5 12.0   5.8  6.6  8.0 11.9   7.8  7.5  8.3 12.6  10.2  9.0  9.2  13.7
  // (One row: 65,536 with 8 7.2, 7.1, 7.4 and 9.2; 100,003 in fp32 11.8, 9.3, 8.3 and 9.5, alone 10.0,
  // 6.5, 4.7 and 4.1.)
  constexpr long long kLeastBytes = kAlternatives ? 65536 : 32768;
  int ctas = 1;
  while (ctas < kMaxCluster && static_cast<long long>(R) * ctas * 2 <= 4 * kLogpSms &&
         static_cast<long long>(k.V) * static_cast<int>(sizeof(T)) >= 2 * ctas * kLeastBytes)
    ctas *= 2;
  static std::atomic<uint64_t> done{0};
  // (five CTAs an SM need a quarter of its 228 KB shared; the rest is for the loads)
  cudaError_t e = prefer_l1(token_logprobs_kernel<T, kAlternatives>, done, 28);
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(static_cast<unsigned>(R) * static_cast<unsigned>(ctas));
  cfg.blockDim = dim3(kThreads);
  cfg.stream = s;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = static_cast<unsigned>(ctas);
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = ctas > 1 ? 2 : 1;
  return cudaLaunchKernelEx(&cfg, token_logprobs_kernel<T, kAlternatives>, k, ctas);
}

}  // namespace
}  // namespace hpd

extern "C" hpd_status hpd_token_logprobs(const hpd_token_logprobs_args *a, hpd_stream_t stream) {
  using namespace hpd;
  // (of the logits' own range, the scale leaves neither differences nor the floor of the sums without a number)
  if (!a || a->R < 0 || a->V < 1 || a->top < 0 || a->top > a->V || a->row_stride < 0 ||
      !(a->scale == 0.f || (a->scale >= 0x1p-120f && a->scale <= 0x1p120f)) || (a->fp32 != 0 && a->fp32 != 1))
    return HPD_ERR_INVALID_ARG;
  if (a->top > 32 || a->V > 1 << 30) return HPD_ERR_UNSUPPORTED;
  if (a->R > 1 && a->row_stride != 0 && a->row_stride < a->V) return HPD_ERR_INVALID_ARG;
  if (a->R == 0) return HPD_OK;
  if (!a->logits || !a->tokens || !a->logprob || (a->top > 0 && (!a->top_tokens || !a->top_logprobs)))
    return HPD_ERR_INVALID_ARG;
  if ((reinterpret_cast<uintptr_t>(a->logits) & (a->fp32 ? 3u : 1u)) != 0) return HPD_ERR_INVALID_ARG;
  for (const void *p : {static_cast<const void *>(a->tokens), static_cast<const void *>(a->logprob),
                        static_cast<const void *>(a->entropy), static_cast<const void *>(a->top_tokens),
                        static_cast<const void *>(a->top_logprobs)})
    if ((reinterpret_cast<uintptr_t>(p) & 3u) != 0) return HPD_ERR_INVALID_ARG;
  LogpArgs k{};
  k.logits = a->logits;
  k.row_stride = a->row_stride ? a->row_stride : a->V;
  k.tokens = a->tokens;
  k.logprob = a->logprob;
  k.entropy = a->entropy;
  k.top_tokens = a->top_tokens;
  k.top_logprobs = a->top_logprobs;
  k.V = a->V;
  k.top = a->top;
  k.scale = a->scale != 0.f ? a->scale : 1.f;
  cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  k.scale_log2 = k.scale * kLog2e;
  const cudaError_t e = a->fp32 ? (k.top ? launch_logprobs<float, true>(k, a->R, s) : launch_logprobs<float, false>(k, a->R, s))
                        : k.top ? launch_logprobs<__nv_bfloat16, true>(k, a->R, s)
                                : launch_logprobs<__nv_bfloat16, false>(k, a->R, s);
  return e == cudaSuccess ? HPD_OK : record_cuda_error(e);
}
