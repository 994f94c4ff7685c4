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

namespace hpd {
namespace {

constexpr int kWarps = 4;

struct PutArgs {
  const __nv_bfloat16 *k, *v;
  long long k_stride, v_stride;
  const __nv_bfloat16 *k_weight;
  const float *rope;
  const int32_t *pos, *slot;
  uint8_t *k_cache, *v_cache;
  float *k_scale, *v_scale;
  uint32_t *err;
  long long num_slots;
  float eps;
  int T, H_kv, max_pos;
  uint32_t axis[4];  // 2 bits a frequency, 8 frequencies (a lane's) in 16
};

// Least k >= 0 with a <= s 2^k (a finite, s a normal number).
__device__ __forceinline__ int doublings(float a, float s) {
  if (!(a > s)) return 0;
  const uint32_t x = __float_as_uint(a), y = __float_as_uint(s);
  return static_cast<int>(x >> 23) - static_cast<int>(y >> 23) + ((x & 0x7fffffu) > (y & 0x7fffffu));
}

template <int D>
__global__ void __launch_bounds__(32 * kWarps) put_codes_kernel(const PutArgs a) {
  constexpr int kLanes = D / 16, kRows = 32 / kLanes;  // lanes of a row, rows of a round
  constexpr int kRounds = kPage / kRows;
  const int lane = threadIdx.x & 31, sub = lane % kLanes, row0 = lane / kLanes;
  const float INF = __int_as_float(0x7f800000);
  pdl_wait();
  pdl_trigger();
  const long long item = static_cast<long long>(blockIdx.x) * kWarps + (threadIdx.x >> 5);
  const int t = static_cast<int>(item / (2 * a.H_kv)), part = static_cast<int>(item % (2 * a.H_kv));
  if (t >= a.T) return;
  const bool is_k = part < a.H_kv;
  const int h = is_k ? part : part - a.H_kv;
  const int slot = a.slot[t];
  if (slot < 0) return;
  if (slot >= a.num_slots) {
    if (lane == 0) flag_error(a.err, HPD_DEVERR_PAGE_ID);
    return;
  }
  const int off = slot % kPage, page = slot / kPage;
  if (t > 0 && off > 0 && a.slot[t - 1] == slot - 1) return;  // another row's run
  const bool next = lane < kPage - off && t + lane < a.T && a.slot[min(t + lane, a.T - 1)] == slot + lane;
  const int n = __ffs(~__ballot_sync(0xffffffffu, next)) - 1;

  float x[kRounds][16], most = 0.f;  // 8 values of a row's lower half, 8 of its upper
  bool odd = false;
  const uint32_t axes = a.axis[sub >> 1] >> (16 * (sub & 1)) & 0xffffu;
#pragma unroll
  for (int u = 0; u < kRounds; ++u) {
    const int i = u * kRows + row0;
    if (u * kRows >= n) break;
    const bool have = i < n;
    uint4 w[2] = {make_uint4(0u, 0u, 0u, 0u), make_uint4(0u, 0u, 0u, 0u)};
    if (have) {
      const __nv_bfloat16 *src = (is_k ? a.k + (t + i) * a.k_stride : a.v + (t + i) * a.v_stride) + h * D + 8 * sub;
      w[0] = *reinterpret_cast<const uint4 *>(src);
      w[1] = *reinterpret_cast<const uint4 *>(src + D / 2);
    }
    auto unpack = [](const uint4 &v, float *y) {
      const uint32_t p[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        y[2 * c] = __uint_as_float(p[c] << 16);
        y[2 * c + 1] = __uint_as_float(p[c] & 0xffff0000u);
      }
    };
    unpack(w[0], x[u]);
    unpack(w[1], x[u] + 8);
    if (is_k) {
      float ss = 0.f;
#pragma unroll
      for (int c = 0; c < 16; ++c) ss = fmaf(x[u][c], x[u][c], ss);
#pragma unroll
      for (int o = 1; o < kLanes; o <<= 1) ss += __shfl_xor_sync(0xffffffffu, ss, o);
      const float r = rsqrtf(ss * (1.0f / D) + a.eps);
      if (have) {
        float wx[16];
#pragma unroll
        for (int c = 0; c < 16; ++c) wx[c] = 1.f;
        if (a.k_weight) {
          unpack(*reinterpret_cast<const uint4 *>(a.k_weight + 8 * sub), wx);
          unpack(*reinterpret_cast<const uint4 *>(a.k_weight + D / 2 + 8 * sub), wx + 8);
        }
#pragma unroll
        for (int c = 0; c < 8; ++c) {
          int at = a.pos[static_cast<long long>(axes >> (2 * c) & 3u) * a.T + t + i];
          if (static_cast<unsigned>(at) >= static_cast<unsigned>(a.max_pos)) {
            flag_error(a.err, HPD_DEVERR_POSITION);
            at = min(max(at, 0), a.max_pos - 1);
          }
          const float2 cs = *reinterpret_cast<const float2 *>(a.rope + (static_cast<long long>(at) * (D / 2) + 8 * sub + c) * 2);
          const float lo = x[u][c] * wx[c] * r, hi = x[u][c + 8] * wx[c + 8] * r;
          x[u][c] = fmaf(lo, cs.x, -hi * cs.y);
          x[u][c + 8] = fmaf(hi, cs.x, lo * cs.y);
        }
      }
    }
#pragma unroll
    for (int c = 0; c < 16; ++c) {
      const float m = fabsf(x[u][c]);
      odd |= !(m < INF);
      most = fmaxf(most, m < INF ? m : 0.f);
    }
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, o));
  const float need = __fdiv_rn(most, kCodeMax);

  float *const at_scale = (is_k ? a.k_scale : a.v_scale) + static_cast<size_t>(page) * a.H_kv + h;
  uint8_t *const base = (is_k ? a.k_cache : a.v_cache) + (static_cast<size_t>(page) * kPage * a.H_kv + h) * D;
  const size_t stride = static_cast<size_t>(a.H_kv) * D;
  float s = fmaxf(need, kLeastScale);
  if (off > 0) {
    s = *at_scale;
    __syncwarp();  // (read by all before one writes)
    if (!(s >= kLeastScale && s <= kMostScale)) {
      if (lane == 0) flag_error(a.err, HPD_DEVERR_SCALE);
      s = kLeastScale;
    }
    const int k = doublings(need, s);
    if (k > 0) {
      s *= __uint_as_float(static_cast<uint32_t>(min(k, 127) + 127) << 23) *
           __uint_as_float(static_cast<uint32_t>(max(k - 127, 0) + 127) << 23);
      const float shrink = k > 40 ? 0.f : __uint_as_float(static_cast<uint32_t>(127 - k) << 23);
      for (int i = row0; i < off; i += kRows) {
        uint4 *const p = reinterpret_cast<uint4 *>(base + i * stride + 16 * sub);
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
  }
  if (lane == 0) *at_scale = s;
  const float inv = __fdiv_rn(1.f, s);
  const float nan = __int_as_float(0x7fffffff);
#pragma unroll
  for (int u = 0; u < kRounds; ++u) {
    const int i = u * kRows + row0;
    if (i >= n) break;
    float y[16];
#pragma unroll
    for (int c = 0; c < 16; ++c) y[c] = x[u][c] * inv;
    if (odd) {  // (e4m3 has no infinities: they would become 448)
#pragma unroll
      for (int c = 0; c < 16; ++c) y[c] = fabsf(x[u][c]) < INF ? y[c] : nan;
    }
    uint8_t *const dst = base + (off + i) * stride + 8 * sub;
    *reinterpret_cast<uint2 *>(dst) = make_uint2(to_codes4(y[0], y[1], y[2], y[3]), to_codes4(y[4], y[5], y[6], y[7]));
    *reinterpret_cast<uint2 *>(dst + D / 2) =
        make_uint2(to_codes4(y[8], y[9], y[10], y[11]), to_codes4(y[12], y[13], y[14], y[15]));
  }
}

template <int D>
cudaError_t launch_put(const PutArgs &k, cudaStream_t s) {
  const long long items = 2LL * k.T * k.H_kv, ctas = (items + kWarps - 1) / kWarps;
  if (ctas >= 1LL << 31) return cudaErrorInvalidValue;
  return launch_kernel(true, put_codes_kernel<D>, dim3(static_cast<unsigned>(ctas)), dim3(32 * kWarps), 0, s, k);
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
  PutArgs k{};
  k.k = static_cast<const __nv_bfloat16 *>(a->k);
  k.v = static_cast<const __nv_bfloat16 *>(a->v);
  k.k_stride = a->k_stride;
  k.v_stride = a->v_stride;
  k.k_weight = static_cast<const __nv_bfloat16 *>(a->k_weight);
  k.rope = a->rope;
  k.pos = a->pos;
  k.slot = a->slot;
  k.k_cache = static_cast<uint8_t *>(a->k_cache);
  k.v_cache = static_cast<uint8_t *>(a->v_cache);
  k.k_scale = f->k_scale;
  k.v_scale = f->v_scale;
  k.err = static_cast<uint32_t *>(a->workspace);
  k.num_slots = a->num_slots;
  k.eps = a->eps;
  k.T = a->T;
  k.H_kv = a->H_kv;
  k.max_pos = a->max_pos;
  for (int i = 0; i < a->D / 2; ++i) k.axis[i >> 4] |= static_cast<uint32_t>(a->axis[i]) << (2 * (i & 15));
  cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  cudaError_t e = launch_norm_rope(a, true, s);
  if (e == cudaSuccess) e = a->D == 64 ? launch_put<64>(k, s) : launch_put<128>(k, s);
  return e == cudaSuccess ? HPD_OK : record_cuda_error(e);
}
