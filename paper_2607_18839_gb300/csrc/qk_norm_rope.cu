// qk_norm_rope.cu -- RMS norms of queries and keys for each head, their rotation
// by position and the write of keys and values to the paged cache, in one pass
// (hpd_qk_norm_rope).
//
//   x'_i = x_i * rsqrt(mean_j x_j^2 + eps) * w_i
//   y_i  = x'_i cos a_i - x'_{i+D/2} sin a_i,   y_{i+D/2} = x'_{i+D/2} cos a_i + x'_i sin a_i
//   a_i  the angle of frequency i at the row's position on axis(i)   (0 <= i < D/2)
//
// Values are read once and written once; sums, norm and rotation are in 32 bits
// with one rounding to bf16 at the end.  D / 16 lanes hold a head: lane l values
// 8l .. 8l + 7 of its lower and of its upper half, so that every rotated pair is in one
// lane, all accesses are 16 bytes and a warp has 512 / D heads at once.  A warp
// takes one row and kUnroll rounds of heads, whose loads are all issued before
// the first is used; cosines and sines are read once for them.
// What bounds it: HBM, reading and writing T (H_q + 2 H_kv) D values.
#include "common.cuh"

namespace hpd {
namespace {

constexpr int kRopeWarps = 4;

struct RopeArgs {
  const __nv_bfloat16 *q, *k, *v;
  long long q_stride, k_stride, v_stride;
  const __nv_bfloat16 *q_weight, *k_weight;
  const float *rope;
  const int32_t *pos, *slot;
  __nv_bfloat16 *q_out, *k_cache, *v_cache;
  uint32_t *err;
  long long num_slots, items;
  float eps;
  int T, H_q, H_kv, max_pos, groups;
  int n_axes;
  uint32_t axis[4];  // 2 bits a frequency, 8 frequencies (a lane's) in 16
};

__device__ __forceinline__ void unpack8(const uint4 &v, float *x) {
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    x[2 * i] = __uint_as_float(w[i] << 16);
    x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
  }
}
__device__ __forceinline__ uint4 pack8(const float *x) {
  return make_uint4(pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]), pack_bf16x2(x[4], x[5]),
                    pack_bf16x2(x[6], x[7]));
}

template <int D, int kUnroll>
__global__ void __launch_bounds__(32 * kRopeWarps) qk_norm_rope_kernel(const RopeArgs a) {
  constexpr int kLanes = D / 16;           // lanes of a head
  constexpr int kHeads = 32 / kLanes;      // heads of a warp at once
  const int lane = threadIdx.x & 31, sub = lane % kLanes;
  const long long item = static_cast<long long>(blockIdx.x) * kRopeWarps + (threadIdx.x >> 5);
  pdl_wait();     // rows, positions, slots and the caches as the kernel before leaves them
  pdl_trigger();
  if (item >= a.items) return;
  const int t = a.groups == 1 ? static_cast<int>(item) : static_cast<int>(item / a.groups);
  const int h0 = static_cast<int>(item - static_cast<long long>(t) * a.groups) * (kHeads * kUnroll) + lane / kLanes;
  const int n_heads = a.H_q + 2 * a.H_kv;
  uint4 lo[kUnroll], hi[kUnroll];
#pragma unroll
  for (int u = 0; u < kUnroll; ++u) {
    const int h = h0 + u * kHeads;
    lo[u] = hi[u] = make_uint4(0u, 0u, 0u, 0u);
    if (h >= n_heads) continue;
    const __nv_bfloat16 *src = h < a.H_q            ? a.q + t * a.q_stride + h * D
                               : h < a.H_q + a.H_kv ? a.k + t * a.k_stride + (h - a.H_q) * D
                                                    : a.v + t * a.v_stride + (h - a.H_q - a.H_kv) * D;
    lo[u] = *reinterpret_cast<const uint4 *>(src + 8 * sub);
    hi[u] = *reinterpret_cast<const uint4 *>(src + D / 2 + 8 * sub);
  }
  const int slot = a.slot[t];
  float cs[16];  // cos, sin of this lane's 8 frequencies
  int p[4] = {0, 0, 0, 0};
  if (h0 - lane / kLanes < a.H_q + a.H_kv) {
    for (int i = 0; i < 4; ++i) {
      if (i >= a.n_axes) break;
      p[i] = a.pos[static_cast<long long>(i) * a.T + t];
      if (static_cast<unsigned>(p[i]) >= static_cast<unsigned>(a.max_pos)) {
        if (lane == 0) atomicOr(a.err, HPD_DEVERR_POSITION);
        p[i] = min(max(p[i], 0), a.max_pos - 1);
      }
    }
    const uint32_t axes = a.axis[sub >> 1] >> (16 * (sub & 1)) & 0xffffu;
    auto row = [&](uint32_t i) {  // this lane's frequencies at the position on axis i
      const int at = i == 0 ? p[0] : i == 1 ? p[1] : i == 2 ? p[2] : p[3];
      return a.rope + (static_cast<long long>(at) * (D / 2) + 8 * sub) * 2;
    };
    if (axes == (axes & 3u) * 0x5555u) {  // all eight on one axis
      const float4 *r = reinterpret_cast<const float4 *>(row(axes & 3u));
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float4 c = r[i];
        cs[4 * i] = c.x;
        cs[4 * i + 1] = c.y;
        cs[4 * i + 2] = c.z;
        cs[4 * i + 3] = c.w;
      }
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float2 c = reinterpret_cast<const float2 *>(row(axes >> (2 * i) & 3u))[i];
        cs[2 * i] = c.x;
        cs[2 * i + 1] = c.y;
      }
    }
  }
  const bool write_kv = slot >= 0 && slot < a.num_slots;
  if (slot >= a.num_slots && lane == 0) atomicOr(a.err, HPD_DEVERR_PAGE_ID);
#pragma unroll
  for (int u = 0; u < kUnroll; ++u) {
    const int h = h0 + u * kHeads;
    const bool is_q = h < a.H_q, is_k = !is_q && h < a.H_q + a.H_kv;
    float x[8], y[8], ss = 0.f;
    unpack8(lo[u], x);
    unpack8(hi[u], y);
    if (is_q || is_k) {
#pragma unroll
      for (int i = 0; i < 8; ++i) ss = fmaf(x[i], x[i], fmaf(y[i], y[i], ss));
    }
#pragma unroll
    for (int o = 1; o < kLanes; o <<= 1) ss += __shfl_xor_sync(0xffffffffu, ss, o);
    if (h >= n_heads) continue;
    __nv_bfloat16 *dst;
    if (is_q || is_k) {
      const float r = rsqrtf(ss * (1.0f / D) + a.eps);
      const __nv_bfloat16 *w = is_q ? a.q_weight : a.k_weight;
      float wx[8], wy[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) wx[i] = wy[i] = 1.f;
      if (w) {
        unpack8(*reinterpret_cast<const uint4 *>(w + 8 * sub), wx);
        unpack8(*reinterpret_cast<const uint4 *>(w + D / 2 + 8 * sub), wy);
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float c = cs[2 * i], s = cs[2 * i + 1];
        const float xn = x[i] * r * wx[i], yn = y[i] * r * wy[i];
        x[i] = fmaf(xn, c, -yn * s);
        y[i] = fmaf(yn, c, xn * s);
      }
      dst = is_q ? a.q_out + (static_cast<long long>(t) * a.H_q + h) * D
                 : a.k_cache + (static_cast<long long>(slot) * a.H_kv + (h - a.H_q)) * D;
      lo[u] = pack8(x);
      hi[u] = pack8(y);
    } else {
      dst = a.v_cache + (static_cast<long long>(slot) * a.H_kv + (h - a.H_q - a.H_kv)) * D;
    }
    if (is_q || write_kv) {
      *reinterpret_cast<uint4 *>(dst + 8 * sub) = lo[u];
      *reinterpret_cast<uint4 *>(dst + D / 2 + 8 * sub) = hi[u];
    }
  }
}

template <int D, int kUnroll>
cudaError_t launch_rope(RopeArgs &a, cudaStream_t s) {
  constexpr int per = 512 / D * kUnroll;  // heads of an item
  a.groups = (a.H_q + 2 * a.H_kv + per - 1) / per;
  a.items = static_cast<long long>(a.T) * a.groups;
  const long long ctas = (a.items + kRopeWarps - 1) / kRopeWarps;
  if (ctas > INT32_MAX) return cudaErrorInvalidConfiguration;
  return launch_kernel(true, qk_norm_rope_kernel<D, kUnroll>, dim3(static_cast<unsigned>(ctas)),
                       dim3(32 * kRopeWarps), 0, s, a);
}

}  // namespace
}  // namespace hpd

extern "C" hpd_status hpd_qk_norm_rope(const hpd_qk_norm_rope_args *a, hpd_stream_t stream) {
  using namespace hpd;
  if (!a || a->T < 0 || a->H_q < 1 || a->H_kv < 1 || a->n_axes < 1 || a->n_axes > 4 || a->max_pos < 1 ||
      a->num_slots < 1 || !(a->eps >= 0.f) || a->eps > 3.4e38f)
    return HPD_ERR_INVALID_ARG;
  if (a->D != 64 && a->D != 128) return HPD_ERR_UNSUPPORTED;
  if (static_cast<long long>(a->H_q) + 2LL * a->H_kv > (1 << 20)) return HPD_ERR_UNSUPPORTED;
  if (!a->q || !a->k || !a->v || !a->rope || !a->pos || !a->slot || !a->q_out || !a->k_cache || !a->v_cache)
    return HPD_ERR_INVALID_ARG;
  if (!a->workspace || (reinterpret_cast<uintptr_t>(a->workspace) & 255u) != 0) return HPD_ERR_WORKSPACE;
  for (const void *p : {a->q, a->k, a->v, a->q_weight, a->k_weight, static_cast<const void *>(a->rope),
                        static_cast<const void *>(a->q_out), static_cast<const void *>(a->k_cache),
                        static_cast<const void *>(a->v_cache)})
    if ((reinterpret_cast<uintptr_t>(p) & 15u) != 0) return HPD_ERR_INVALID_ARG;
  if (((reinterpret_cast<uintptr_t>(a->pos) | reinterpret_cast<uintptr_t>(a->slot)) & 3u) != 0)
    return HPD_ERR_INVALID_ARG;
  if (a->q_stride % 8 != 0 || a->k_stride % 8 != 0 || a->v_stride % 8 != 0) return HPD_ERR_INVALID_ARG;
  for (int i = 0; i < a->D / 2; ++i)
    if (a->axis[i] >= a->n_axes) return HPD_ERR_INVALID_ARG;
  if (a->T == 0) return HPD_OK;
  RopeArgs k{};
  k.q = static_cast<const __nv_bfloat16 *>(a->q);
  k.k = static_cast<const __nv_bfloat16 *>(a->k);
  k.v = static_cast<const __nv_bfloat16 *>(a->v);
  k.q_stride = a->q_stride;
  k.k_stride = a->k_stride;
  k.v_stride = a->v_stride;
  k.q_weight = static_cast<const __nv_bfloat16 *>(a->q_weight);
  k.k_weight = static_cast<const __nv_bfloat16 *>(a->k_weight);
  k.rope = a->rope;
  k.pos = a->pos;
  k.slot = a->slot;
  k.q_out = static_cast<__nv_bfloat16 *>(a->q_out);
  k.k_cache = static_cast<__nv_bfloat16 *>(a->k_cache);
  k.v_cache = static_cast<__nv_bfloat16 *>(a->v_cache);
  k.err = static_cast<uint32_t *>(a->workspace);
  k.num_slots = a->num_slots;
  k.eps = a->eps;
  k.T = a->T;
  k.H_q = a->H_q;
  k.H_kv = a->H_kv;
  k.max_pos = a->max_pos;
  k.n_axes = a->n_axes;
  for (int i = 0; i < a->D / 2; ++i) k.axis[i >> 4] |= static_cast<uint32_t>(a->axis[i]) << (2 * (i & 15));
  cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  const cudaError_t e = a->D == 64 ? launch_rope<64, 2>(k, s) : launch_rope<128, 4>(k, s);
  return e == cudaSuccess ? HPD_OK : record_cuda_error(e);
}
