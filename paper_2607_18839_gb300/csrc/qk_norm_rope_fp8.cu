// qk_norm_rope_fp8.cu -- RMS norms and rotation of queries and keys, and the write of
// keys and values to the paged cache as 8-bit codes with a scale for each page and
// head (hpd_qk_norm_rope_fp8).
//
// Norms and rotation as in qk_norm_rope.cu, whose kernel has the queries.  Keys and
// values: the rows of one page ("run", n of them from offset o) belong to one warp
// for each head, which holds them in registers, 32 bits a value:
//   a = max |x| / 448;  o = 0: s = max(a, 2^-100);  o > 0: s = s_old 2^k, least k >= 0
//   with a <= s;  code = e4m3(x / s), and the codes of rows below o times 2^-k
// Doublings of a scale leave a code's bits but for its exponent as they are, so that
// nothing is rounded twice until it falls below e4m3's normal numbers.
// Norm, rotation and quotient are in 32 bits; the code is a key's only rounding (the quotient
// is a product with 1 / s, 2^-23 of it off at most, which can decide a tie).
//
// One launch; a warp has items, one after the other: rows of queries, and of keys and values
// the runs that begin in some rows, head by head.  A page's scale has to be known before its
// first code is written: a run is in its warp's registers in between (of 16 rows of 128 values
// 64 of its 128), and its rows come with one wait.
// What bounds it, and what it measured on a GB300 (in a graph):
//   32,749 rows of 16 + 2 + 2 heads of 128: 73.5 us, 4.6 TB/s, 68 % of a copy's rate (the
//     bf16 form of the queries, keys and values 60.6).  Queries alone are at the memory; the
//     8,188 runs have the rest, some 7 us each for a warp, 16 warps an SM: slots, rows and
//     scale, the table's rows, maximum, codes, one after the other.
//   3,292 rows of 32 + 8 + 8 heads: 22.4 us, 3.4 TB/s: the same in one wave.
//   256 tokens of 256 sequences, 32 + 8 + 8 heads: 7.2 us, latency: 4,096 runs of a row, some
//     of which have to halve the codes before theirs.  16 tokens, 8 + 2 + 2 heads of 64: 2.5.
// The table's rows a round ahead: 872 bytes of spills, 74.5 and 25.8 us; with the turned keys
// in shared memory instead of registers 75.0 and 23.5.
#include "fp8.cuh"
#include "qk_norm_rope.cuh"

namespace hpd {
namespace {

struct Fp8Args {
  RopeArgs rope;     // what rows, positions, slots and norms are; H_kv = 0: its items are the queries'
  uint8_t *k_cache, *v_cache;
  float *k_scale, *v_scale;
  int H_kv;
  int kv_ctas;       // CTAs of keys and values, the first ones; 0: all have both
  int chunk;         // rows whose runs are an item's: those that begin there
  int items;
  FastDiv div_parts;  // by 2 H_kv
};

// Least k >= 0 with a <= s 2^k (a finite, s a normal number).
__device__ __forceinline__ int doublings(float a, float s) {
  if (!(a > s)) return 0;
  const uint32_t x = __float_as_uint(a), y = __float_as_uint(s);
  return static_cast<int>(x >> 23) - static_cast<int>(y >> 23) + ((x & 0x7fffffu) > (y & 0x7fffffu));
}

// A page's scale grows 2^k times: its rows below `off`, D codes each, times 2^-k.
template <int D>
__device__ __noinline__ void shrink_rows(uint8_t *base, size_t stride, int off, int k) {
  constexpr int kLanes = D / 16, kRows = 32 / kLanes;
  const int lane = threadIdx.x & 31;
  const float shrink = k > 40 ? 0.f : __uint_as_float(static_cast<uint32_t>(127 - k) << 23);
  for (int i = lane / kLanes; i < off; i += kRows) {
    uint4 *const p = reinterpret_cast<uint4 *>(base + i * stride + 16 * (lane % kLanes));
    uint4 v = *p;
    uint32_t *const w = reinterpret_cast<uint32_t *>(&v);
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      float2 lo, hi;
      of_codes4(w[c], lo, hi);
      w[c] = to_codes4(lo.x * shrink, lo.y * shrink, hi.x * shrink, hi.y * shrink);
    }
    *p = v;
  }
}

// A run: n rows from row t and cache row `slot` on; part: head of K, or H_kv + head of V.
struct Run {
  int t, n, slot, part;
};

// How a warp holds a run: a row has kLanes lanes, each with 8 values of its lower half and 8
// of its upper, a round kRows rows.
template <int D>
struct Hold {
  static constexpr int kLanes = D / 16, kRows = 32 / kLanes, kRounds = kPage / kRows;
  uint4 w[kRounds][2];  // as they come
  int at[kRounds];      // positions on the axis of the lane's first frequency
  float had;            // the page's scale so far
};

template <int D>
__device__ __forceinline__ void load_run(const Fp8Args &f, const Run &r, Hold<D> &x) {
  using H = Hold<D>;
  const RopeArgs &a = f.rope;
  const int lane = threadIdx.x & 31, sub = lane % H::kLanes, row0 = lane / H::kLanes;
  const bool is_k = r.part < f.H_kv;
  const int h = is_k ? r.part : r.part - f.H_kv;
  const __nv_bfloat16 *src = (is_k ? a.k + r.t * a.k_stride : a.v + r.t * a.v_stride) + h * D + 8 * sub;
  const long long stride = is_k ? a.k_stride : a.v_stride;
  const int32_t *const pos = a.pos + static_cast<long long>(a.axis[sub >> 1] >> (16 * (sub & 1)) & 3u) * a.T + r.t;
  x.had = 0.f;
  if (r.slot % kPage > 0) x.had = (is_k ? f.k_scale : f.v_scale)[static_cast<size_t>(r.slot / kPage) * f.H_kv + h];
#pragma unroll
  for (int u = 0; u < H::kRounds; ++u) {
    const int i = u * H::kRows + row0;
    x.w[u][0] = x.w[u][1] = make_uint4(0u, 0u, 0u, 0u);
    x.at[u] = 0;
    if (i < r.n) {
      x.w[u][0] = *reinterpret_cast<const uint4 *>(src + i * stride);
      x.w[u][1] = *reinterpret_cast<const uint4 *>(src + i * stride + D / 2);
      if (is_k) x.at[u] = pos[i];
    }
  }
}

// Round u of a run of keys, normed and rotated.
template <int D>
__device__ __forceinline__ void turn_round(const Fp8Args &f, const Run &r, const Hold<D> &in, const uint4 *kw, int u,
                                           float2 *x) {
  using H = Hold<D>;
  const RopeArgs &a = f.rope;
  const int lane = threadIdx.x & 31, sub = lane % H::kLanes, i = u * H::kRows + lane / H::kLanes;
  unpack8(in.w[u][0], x);
  unpack8(in.w[u][1], x + 4);
  if (u * H::kRows >= r.n) return;
  float2 s2 = make_float2(0.f, 0.f);
#pragma unroll
  for (int c = 0; c < 8; ++c) s2 = __ffma2_rn(x[c], x[c], s2);
  float ss = s2.x + s2.y;
#pragma unroll
  for (int o = 1; o < H::kLanes; o <<= 1) ss += __shfl_xor_sync(0xffffffffu, ss, o);
  if (i >= r.n) return;
  const float norm = rsqrtf(ss * (1.0f / D) + a.eps);
  const float2 r2 = make_float2(norm, norm);
  if (a.k_weight) {
    float2 wx[8];
    unpack8(kw[0], wx);
    unpack8(kw[1], wx + 4);
#pragma unroll
    for (int c = 0; c < 8; ++c) x[c] = __fmul2_rn(x[c], wx[c]);
  }
  const uint32_t axes = a.axis[sub >> 1] >> (16 * (sub & 1)) & 0xffffu;
  const bool one_axis = axes == (axes & 3u) * 0x5555u;  // all eight of this lane's frequencies
  auto row = [&](int p) {  // this lane's frequencies at a position
    if (static_cast<unsigned>(p) >= static_cast<unsigned>(a.max_pos)) {
      flag_error(a.err, HPD_DEVERR_POSITION);
      p = min(max(p, 0), a.max_pos - 1);
    }
    return a.rope + (static_cast<long long>(p) * (D / 2) + 8 * sub) * 2;
  };
  float4 cs[4];  // of two frequencies each
  if (one_axis) {
    const float4 *const mine = reinterpret_cast<const float4 *>(row(in.at[u]));
#pragma unroll
    for (int c = 0; c < 4; ++c) cs[c] = mine[c];
  } else {
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      const int32_t *const at = a.pos + r.t + i;
      const float2 c0 = *reinterpret_cast<const float2 *>(
          row(at[static_cast<long long>(axes >> (4 * c) & 3u) * a.T]) + 4 * c);
      const float2 c1 = *reinterpret_cast<const float2 *>(
          row(at[static_cast<long long>(axes >> (4 * c + 2) & 3u) * a.T]) + 4 * c + 2);
      cs[c] = make_float4(c0.x, c0.y, c1.x, c1.y);
    }
  }
#pragma unroll
  for (int c = 0; c < 4; ++c) {
    const float2 cos = make_float2(cs[c].x, cs[c].z), sin = make_float2(cs[c].y, cs[c].w);
    const float2 xn = __fmul2_rn(x[c], r2), yn = __fmul2_rn(x[c + 4], r2), ys = __fmul2_rn(yn, sin);
    x[c] = __ffma2_rn(xn, cos, make_float2(-ys.x, -ys.y));
    x[c + 4] = __ffma2_rn(yn, cos, __fmul2_rn(xn, sin));
  }
}

__device__ __forceinline__ unsigned max2(unsigned a, unsigned b) {
  asm("max.u16x2 %0, %0, %1;" : "+r"(a) : "r"(b));
  return a;
}
__device__ __forceinline__ float max_nan(float a, float b) {
  asm("max.NaN.f32 %0, %0, %1;" : "+f"(a) : "f"(b));
  return a;
}

// The scale of a run whose largest magnitude is `most`, in its place, with the rows before
// it brought to it; returns its reciprocal.
template <int D>
__device__ __forceinline__ float settle_scale(const Fp8Args &f, const Run &r, float most, float had) {
  const bool is_k = r.part < f.H_kv;
  const int h = is_k ? r.part : r.part - f.H_kv, off = r.slot % kPage;
  const size_t page = static_cast<size_t>(r.slot / kPage);
  const float need = __fdiv_rn(most, kCodeMax);
  float s = fmaxf(need, kLeastScale);
  if (off > 0) {
    s = had;
    if (!(s >= kLeastScale && s <= kMostScale)) {
      if ((threadIdx.x & 31) == 0) flag_error(f.rope.err, HPD_DEVERR_SCALE);
      s = kLeastScale;
    }
    const int k = doublings(need, s);
    if (k > 0) {
      // (one after the other: 2^k alone may be out of range)
      s *= __uint_as_float(static_cast<uint32_t>(min(k, 127) + 127) << 23);
      s *= __uint_as_float(static_cast<uint32_t>(max(k - 127, 0) + 127) << 23);
      shrink_rows<D>((is_k ? f.k_cache : f.v_cache) + (page * kPage * f.H_kv + h) * D, static_cast<size_t>(f.H_kv) * D,
                     off, k);
    }
  }
  if ((threadIdx.x & 31) == 0) (is_k ? f.k_scale : f.v_scale)[page * f.H_kv + h] = s;
  return __fdiv_rn(1.f, s);
}

// 16 values of a row as codes; wild: some may not be finite (e4m3 has no infinities: they
// would become 448).
template <int D>
__device__ __forceinline__ void put_codes(uint8_t *dst, const float2 *x, float inv, bool wild) {
  const float INF = __int_as_float(0x7f800000), nan = __int_as_float(0x7fffffff);
  float2 y[8];
#pragma unroll
  for (int c = 0; c < 8; ++c) y[c] = __fmul2_rn(x[c], make_float2(inv, inv));
  if (wild) {
#pragma unroll
    for (int c = 0; c < 8; ++c)
      y[c] = make_float2(fabsf(x[c].x) < INF ? y[c].x : nan, fabsf(x[c].y) < INF ? y[c].y : nan);
  }
  *reinterpret_cast<uint2 *>(dst) =
      make_uint2(to_codes4(y[0].x, y[0].y, y[1].x, y[1].y), to_codes4(y[2].x, y[2].y, y[3].x, y[3].y));
  *reinterpret_cast<uint2 *>(dst + D / 2) =
      make_uint2(to_codes4(y[4].x, y[4].y, y[5].x, y[5].y), to_codes4(y[6].x, y[6].y, y[7].x, y[7].y));
}
// Largest of the finite magnitudes among values that are not all finite.
__device__ __forceinline__ float largest_finite(float most, const float2 *x) {
  const float INF = __int_as_float(0x7f800000);
#pragma unroll
  for (int c = 0; c < 8; ++c) {
    if (fabsf(x[c].x) < INF) most = fmaxf(most, fabsf(x[c].x));
    if (fabsf(x[c].y) < INF) most = fmaxf(most, fabsf(x[c].y));
  }
  return most;
}

// Keys and values, by warp `first` of `step`: runs that begin in an item's rows, item by
// item.
template <int D>
__device__ __forceinline__ void put_runs(const Fp8Args &f, int first, int step) {
  using H = Hold<D>;
  const RopeArgs &a = f.rope;
  const int lane = threadIdx.x & 31;
  // A lane's row is the item's first one - 1 + lane: a run that begins in the item ends there.
  const int parts = 2 * f.H_kv;
  auto fetch = [&](int item) {
    const int i = f.div_parts(item) * f.chunk - 1 + lane;
    return item < f.items && i >= 0 && i < a.T ? a.slot[i] : -1;
  };
  int item = first - step, slot = -1, next = fetch(first);
  unsigned heads = 0, goes_on = 0;
  auto advance = [&](Run &r) {
    while (!heads) {
      item += step;
      if (item >= f.items) return false;
      slot = next;
      next = fetch(item + step);
      const int prev = __shfl_up_sync(0xffffffffu, slot, 1), after = __shfl_down_sync(0xffffffffu, slot, 1);
      const bool here = lane >= 1 && lane <= f.chunk && slot >= 0;
      if (here && slot >= a.num_slots) flag_error(a.err, HPD_DEVERR_PAGE_ID);
      heads = __ballot_sync(0xffffffffu, here && slot < a.num_slots && (slot % kPage == 0 || prev != slot - 1));
      goes_on = __ballot_sync(0xffffffffu, lane < 31 && (slot + 1) % kPage != 0 && after == slot + 1);
    }
    const int l = __ffs(heads) - 1;
    heads &= heads - 1;
    const int q = f.div_parts(item);
    r = Run{q * f.chunk - 1 + l, __ffs(~(goes_on >> l)), __shfl_sync(0xffffffffu, slot, l), item - q * parts};
    return true;
  };
  const int sub = lane % H::kLanes, row0 = lane / H::kLanes;
  const float INF = __int_as_float(0x7f800000);
  // (magnitudes are in the order of their bits, NaN and infinity the largest)
  auto of_warp = [](float m) { return __uint_as_float(__reduce_max_sync(0xffffffffu, __float_as_uint(m))); };
  uint4 kw[2];  // the keys' weights of this lane's values
  kw[0] = kw[1] = make_uint4(0u, 0u, 0u, 0u);
  if (a.k_weight) {
    kw[0] = *reinterpret_cast<const uint4 *>(a.k_weight + 8 * sub);
    kw[1] = *reinterpret_cast<const uint4 *>(a.k_weight + D / 2 + 8 * sub);
  }
  Run r;
  while (advance(r)) {
    Hold<D> in;
    load_run(f, r, in);
    const bool is_k = r.part < f.H_kv;
    const size_t stride = static_cast<size_t>(f.H_kv) * D;
    uint8_t *const dst = (is_k ? f.k_cache : f.v_cache) + static_cast<size_t>(r.slot) * stride +
                         (is_k ? r.part : r.part - f.H_kv) * D + 8 * sub;
    if (is_k) {
      float2 x[H::kRounds][8];
      float most = 0.f;
#pragma unroll
      for (int u = 0; u < H::kRounds; ++u) {
        turn_round<D>(f, r, in, kw, u, x[u]);
#pragma unroll
        for (int c = 0; c < 8; ++c) most = max_nan(max_nan(most, fabsf(x[u][c].x)), fabsf(x[u][c].y));
      }
      most = of_warp(fabsf(most));
      const bool wild = !(most < INF);
      if (wild) {
        most = 0.f;
#pragma unroll
        for (int u = 0; u < H::kRounds; ++u) most = largest_finite(most, x[u]);
        most = of_warp(most);
      }
      const float inv = settle_scale<D>(f, r, most, in.had);
#pragma unroll
      for (int u = 0; u < H::kRounds; ++u)
        if (u * H::kRows + row0 < r.n) put_codes<D>(dst + (u * H::kRows + row0) * stride, x[u], inv, wild);
    } else {
      const auto &w = in.w;
      unsigned m2 = 0u;  // of two values at once, as their bits
#pragma unroll
      for (int u = 0; u < H::kRounds; ++u)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const uint4 v = w[u][e];
          m2 = max2(max2(m2, max2(v.x & 0x7fff7fffu, v.y & 0x7fff7fffu)), max2(v.z & 0x7fff7fffu, v.w & 0x7fff7fffu));
        }
      float most = of_warp(__uint_as_float(max(m2 << 16, m2 & 0xffff0000u)));
      const bool wild = !(most < INF);
      if (wild) {
        most = 0.f;
#pragma unroll
        for (int u = 0; u < H::kRounds; ++u) {
          float2 x[8];
          unpack8(w[u][0], x);
          unpack8(w[u][1], x + 4);
          most = largest_finite(most, x);
        }
        most = of_warp(most);
      }
      const float inv = settle_scale<D>(f, r, most, in.had);
#pragma unroll
      for (int u = 0; u < H::kRounds; ++u)
        if (u * H::kRows + row0 < r.n) {
          float2 x[8];
          unpack8(w[u][0], x);
          unpack8(w[u][1], x + 4);
          put_codes<D>(dst + (u * H::kRows + row0) * stride, x, inv, wild);
        }
    }
  }
}

// Calls that fill no more than the GPU once have warps for the queries and others for keys
// and values (16 tokens 2.5 us; 3.6 if each warp has both); in larger ones every warp has a share of both, one after the other (32,749
// rows of 16 / 2 heads of 128: 76 us; every second CTA in the other order 78 to 81; CTAs of
// their own for keys and values, as many as took least time, 88: a run takes its warp some
// 7 us, of which its loads are few).
template <int D>
__global__ void __launch_bounds__(32 * kRopeWarps, kRopeCtas) qk_norm_rope_fp8_kernel(const Fp8Args f) {
  pdl_wait();
  pdl_trigger();
  const int warp = threadIdx.x >> 5, b = blockIdx.x, all = gridDim.x * kRopeWarps;
  if (f.kv_ctas > 0) {
    if (b < f.kv_ctas) put_runs<D>(f, b * kRopeWarps + warp, f.kv_ctas * kRopeWarps);
    else norm_rope_rows<D>(f.rope, (b - f.kv_ctas) * kRopeWarps + warp, all - f.kv_ctas * kRopeWarps);
    return;
  }
  norm_rope_rows<D>(f.rope, b * kRopeWarps + warp, all);
  put_runs<D>(f, b * kRopeWarps + warp, all);
}

template <int D>
cudaError_t launch_fp8(Fp8Args &f, cudaStream_t s) {
  constexpr int kMost = kRopeSms * kRopeCtas;
  const long long T = f.rope.T, parts = 2LL * f.H_kv;
  // Items of as many rows as leave one to each warp of the GPU (a row each: 32,749 rows 317
  // us instead of 74, 3,292 rows of 32 + 8 + 8 heads 32 instead of 22).
  f.chunk = 1;
  while (f.chunk < kPage && T * parts >= 2LL * f.chunk * kMost * kRopeWarps) f.chunk *= 2;
  const long long items = (T + f.chunk - 1) / f.chunk * parts, q_items = plan_items(f.rope, D);
  if (items >= 1LL << 30 || q_items >= 1LL << 30) return cudaErrorInvalidValue;
  f.items = static_cast<int>(items);
  auto ctas = [](long long n) { return (n + kRopeWarps - 1) / kRopeWarps; };
  const long long kv = ctas(items), q = ctas(q_items);
  f.kv_ctas = kv + q <= kMost ? static_cast<int>(kv) : 0;
  f.div_parts.set(static_cast<int>(parts));
  return launch_kernel(true, qk_norm_rope_fp8_kernel<D>, dim3(static_cast<unsigned>(std::min<long long>(kv + q, kMost))), dim3(32 * kRopeWarps), 0, s, f);
}

}  // namespace
}  // namespace hpd

extern "C" hpd_status hpd_qk_norm_rope_fp8(const hpd_qk_norm_rope_fp8_args *f, hpd_stream_t stream) {
  using namespace hpd;
  const hpd_qk_norm_rope_args *a = f ? &f->rope : nullptr;
  const hpd_status st = check_norm_rope(a);
  if (st != HPD_OK) return st;
  if (!f->k_scale || !f->v_scale || a->num_slots % kPage != 0) return HPD_ERR_INVALID_ARG;
  if (((reinterpret_cast<uintptr_t>(f->k_scale) | reinterpret_cast<uintptr_t>(f->v_scale)) & 3u) != 0)
    return HPD_ERR_INVALID_ARG;
  if (a->T == 0) return HPD_OK;
  Fp8Args k{};
  k.rope = rope_args(a);
  k.rope.H_kv = 0;
  k.k_cache = static_cast<uint8_t *>(a->k_cache);
  k.v_cache = static_cast<uint8_t *>(a->v_cache);
  k.k_scale = f->k_scale;
  k.v_scale = f->v_scale;
  k.H_kv = a->H_kv;
  cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  const cudaError_t e = a->D == 64 ? launch_fp8<64>(k, s) : launch_fp8<128>(k, s);
  return e == cudaSuccess ? HPD_OK : record_cuda_error(e);
}
