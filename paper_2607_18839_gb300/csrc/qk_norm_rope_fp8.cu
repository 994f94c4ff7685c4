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
#include "fp8.cuh"
#include "qk_norm_rope.cuh"

namespace hpd {
namespace {

struct Fp8Args {
  RopeArgs rope;     // what rows, positions, slots and norms are; H_kv = 0: its items are the queries'
  uint8_t *k_cache, *v_cache;
  float *k_scale, *v_scale;
  int H_kv;
  int kv_ctas;       // CTAs of keys and values among all
  int chunk;         // rows whose runs are an item's: those that begin there
  int items;
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

// The run of n rows from row t and cache row `slot` on, of head h of K or V.
template <int D, bool kIsK>
__device__ __forceinline__ void put_run(const Fp8Args &f, int t, int n, int slot, int h) {
  const RopeArgs &a = f.rope;
  constexpr int kLanes = D / 16, kRows = 32 / kLanes;  // lanes of a row, rows of a round
  constexpr int kRounds = kPage / kRows;
  const int lane = threadIdx.x & 31, sub = lane % kLanes, row0 = lane / kLanes;
  const float INF = __int_as_float(0x7f800000);
  const int off = slot % kPage, page = slot / kPage;
  float *const at_scale = (kIsK ? f.k_scale : f.v_scale) + static_cast<size_t>(page) * f.H_kv + h;
  uint8_t *const base = (kIsK ? f.k_cache : f.v_cache) + (static_cast<size_t>(page) * kPage * f.H_kv + h) * D;
  const size_t stride = static_cast<size_t>(f.H_kv) * D;
  float had = 0.f;
  if (off > 0) had = *at_scale;
  // (every load on its way before the first use)
  uint4 w[kRounds][2];
  int at[kRounds];
  const uint32_t axes = a.axis[sub >> 1] >> (16 * (sub & 1)) & 0xffffu;
  const bool one_axis = axes == (axes & 3u) * 0x5555u;
  const int32_t *const pos = a.pos + static_cast<long long>(axes & 3u) * a.T + t;
#pragma unroll
  for (int u = 0; u < kRounds; ++u) {
    const int i = u * kRows + row0;
    w[u][0] = w[u][1] = make_uint4(0u, 0u, 0u, 0u);
    at[u] = 0;
    if (i < n) {
      const __nv_bfloat16 *src = (kIsK ? a.k + (t + i) * a.k_stride : a.v + (t + i) * a.v_stride) + h * D + 8 * sub;
      w[u][0] = *reinterpret_cast<const uint4 *>(src);
      w[u][1] = *reinterpret_cast<const uint4 *>(src + D / 2);
      if (kIsK) at[u] = pos[i];
    }
  }
  float2 x[kRounds][8];  // 8 values of a row's lower half, 8 of its upper
  float most = 0.f;
  bool odd = false;
#pragma unroll
  for (int u = 0; u < kRounds; ++u) {
    const int i = u * kRows + row0;
    unpack8(w[u][0], x[u]);
    unpack8(w[u][1], x[u] + 4);
    if (kIsK && u * kRows < n) {
      float2 s2 = make_float2(0.f, 0.f);
#pragma unroll
      for (int c = 0; c < 8; ++c) s2 = __ffma2_rn(x[u][c], x[u][c], s2);
      float ss = s2.x + s2.y;
#pragma unroll
      for (int o = 1; o < kLanes; o <<= 1) ss += __shfl_xor_sync(0xffffffffu, ss, o);
      if (i < n) {
        const float r = rsqrtf(ss * (1.0f / D) + a.eps);
        const float2 r2 = make_float2(r, r);
        if (a.k_weight) {
          float2 wx[8];
          unpack8(*reinterpret_cast<const uint4 *>(a.k_weight + 8 * sub), wx);
          unpack8(*reinterpret_cast<const uint4 *>(a.k_weight + D / 2 + 8 * sub), wx + 4);
#pragma unroll
          for (int c = 0; c < 8; ++c) x[u][c] = __fmul2_rn(x[u][c], wx[c]);
        }
        auto row = [&](int p) {  // this lane's frequencies at a position
          if (static_cast<unsigned>(p) >= static_cast<unsigned>(a.max_pos)) {
            flag_error(a.err, HPD_DEVERR_POSITION);
            p = min(max(p, 0), a.max_pos - 1);
          }
          return a.rope + (static_cast<long long>(p) * (D / 2) + 8 * sub) * 2;
        };
        const float *const mine = row(at[u]);
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          float4 cs;  // of two frequencies
          if (one_axis) {
            cs = *reinterpret_cast<const float4 *>(mine + 4 * c);
          } else {
            const float2 c0 = *reinterpret_cast<const float2 *>(
                row(a.pos[static_cast<long long>(axes >> (4 * c) & 3u) * a.T + t + i]) + 4 * c);
            const float2 c1 = *reinterpret_cast<const float2 *>(
                row(a.pos[static_cast<long long>(axes >> (4 * c + 2) & 3u) * a.T + t + i]) + 4 * c + 2);
            cs = make_float4(c0.x, c0.y, c1.x, c1.y);
          }
          const float2 cos = make_float2(cs.x, cs.z), sin = make_float2(cs.y, cs.w);
          const float2 xn = __fmul2_rn(x[u][c], r2), yn = __fmul2_rn(x[u][c + 4], r2), ys = __fmul2_rn(yn, sin);
          x[u][c] = __ffma2_rn(xn, cos, make_float2(-ys.x, -ys.y));
          x[u][c + 4] = __ffma2_rn(yn, cos, __fmul2_rn(xn, sin));
        }
      }
    }
#pragma unroll
    for (int c = 0; c < 8; ++c) {
      const float p = fabsf(x[u][c].x), q = fabsf(x[u][c].y);
      odd |= !(p < INF) || !(q < INF);
      most = fmaxf(most, fmaxf(p < INF ? p : 0.f, q < INF ? q : 0.f));
    }
  }
  // (magnitudes are in the order of their bits)
  most = __uint_as_float(__reduce_max_sync(0xffffffffu, __float_as_uint(most)));
  const float need = __fdiv_rn(most, kCodeMax);
  float s = fmaxf(need, kLeastScale);
  if (off > 0) {
    s = had;
    if (!(s >= kLeastScale && s <= kMostScale)) {
      if (lane == 0) flag_error(a.err, HPD_DEVERR_SCALE);
      s = kLeastScale;
    }
    const int k = doublings(need, s);
    if (k > 0) {
      s *= __uint_as_float(static_cast<uint32_t>(min(k, 127) + 127) << 23) *
           __uint_as_float(static_cast<uint32_t>(max(k - 127, 0) + 127) << 23);
      shrink_rows<D>(base, stride, off, k);
    }
  }
  if (lane == 0) *at_scale = s;
  const float inv = __fdiv_rn(1.f, s);
  const float2 inv2 = make_float2(inv, inv);
  const float nan = __int_as_float(0x7fffffff);
#pragma unroll
  for (int u = 0; u < kRounds; ++u) {
    const int i = u * kRows + row0;
    if (i >= n) break;
    float2 y[8];
#pragma unroll
    for (int c = 0; c < 8; ++c) y[c] = __fmul2_rn(x[u][c], inv2);
    if (odd) {  // (e4m3 has no infinities: they would become 448)
#pragma unroll
      for (int c = 0; c < 8; ++c)
        y[c] = make_float2(fabsf(x[u][c].x) < INF ? y[c].x : nan, fabsf(x[u][c].y) < INF ? y[c].y : nan);
    }
    uint8_t *const dst = base + (off + i) * stride + 8 * sub;
    *reinterpret_cast<uint2 *>(dst) =
        make_uint2(to_codes4(y[0].x, y[0].y, y[1].x, y[1].y), to_codes4(y[2].x, y[2].y, y[3].x, y[3].y));
    *reinterpret_cast<uint2 *>(dst + D / 2) =
        make_uint2(to_codes4(y[4].x, y[4].y, y[5].x, y[5].y), to_codes4(y[6].x, y[6].y, y[7].x, y[7].y));
  }
}

// CTAs of queries (norm_rope_rows) and of keys and values side by side.
template <int D>
__global__ void __launch_bounds__(32 * kRopeWarps, kRopeCtas) qk_norm_rope_fp8_kernel(const Fp8Args f) {
  const RopeArgs &a = f.rope;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int b = blockIdx.x, all = gridDim.x;
  // (spread evenly: which one this is among those of keys and values, if it is one)
  const int mine = static_cast<int>(static_cast<long long>(b) * f.kv_ctas / all);
  const bool kv = static_cast<int>(static_cast<long long>(b + 1) * f.kv_ctas / all) > mine;
  pdl_wait();
  pdl_trigger();
  if (!kv) {
    norm_rope_rows<D>(a, (b - mine) * kRopeWarps + warp, (all - f.kv_ctas) * kRopeWarps);
    return;
  }
  const int parts = 2 * f.H_kv, step = f.kv_ctas * kRopeWarps;
  // a lane's row is the item's first one - 1 + lane: a run that begins in the item ends there
  auto fetch = [&](int item) {
    const int i = item / parts * f.chunk - 1 + lane;
    return item < f.items && i >= 0 && i < a.T ? a.slot[i] : -1;
  };
  int item = mine * kRopeWarps + warp, next = fetch(item);
  for (; item < f.items; item += step) {
    const int slot = next, part = item % parts, first = item / parts * f.chunk - 1;
    next = fetch(item + step);
    const int prev = __shfl_up_sync(0xffffffffu, slot, 1), after = __shfl_down_sync(0xffffffffu, slot, 1);
    const bool here = lane >= 1 && lane <= f.chunk && slot >= 0;
    if (here && slot >= a.num_slots) flag_error(a.err, HPD_DEVERR_PAGE_ID);
    unsigned heads = __ballot_sync(0xffffffffu, here && slot < a.num_slots && (slot % kPage == 0 || prev != slot - 1));
    const unsigned goes_on = __ballot_sync(0xffffffffu, lane < 31 && (slot + 1) % kPage != 0 && after == slot + 1);
    while (heads) {
      const int l = __ffs(heads) - 1;
      heads &= heads - 1;
      const int n = __ffs(~(goes_on >> l)), s = __shfl_sync(0xffffffffu, slot, l);
      if (part < f.H_kv) put_run<D, true>(f, first + l, n, s, part);
      else put_run<D, false>(f, first + l, n, s, part - f.H_kv);
    }
  }
}

template <int D>
cudaError_t launch_fp8(Fp8Args &f, cudaStream_t s) {
  constexpr int kMost = kRopeSms * kRopeCtas;
  const long long T = f.rope.T, parts = 2LL * f.H_kv;
  // Items of as many rows as leave one to each warp of the GPU.
  f.chunk = 1;
  while (f.chunk < kPage && T * parts >= 2LL * f.chunk * kMost * kRopeWarps) f.chunk *= 2;
  const long long items = (T + f.chunk - 1) / f.chunk * parts, q_items = plan_items(f.rope, D);
  if (items >= 1LL << 30 || q_items >= 1LL << 30) return cudaErrorInvalidValue;
  f.items = static_cast<int>(items);
  auto ctas = [](long long n) { return (n + kRopeWarps - 1) / kRopeWarps; };
  long long kv = ctas(items), q = ctas(q_items);
  if (kv + q > kMost) {
    // Shares by the bytes of each, a run's counted kRunCost times.
    constexpr double kRunCost = 1.5;
    const double of_kv = kRunCost * 3 * parts, of_q = 4.0 * f.rope.H_q;
    kv = std::min(kv, std::max(1LL, static_cast<long long>(kMost * of_kv / (of_kv + of_q) + 0.5)));
    q = std::min(q, kMost - kv);
    kv = std::min(ctas(items), kMost - q);
  }
  f.kv_ctas = static_cast<int>(kv);
  return launch_kernel(true, qk_norm_rope_fp8_kernel<D>, dim3(static_cast<unsigned>(kv + q)), dim3(32 * kRopeWarps), 0, s, f);
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
