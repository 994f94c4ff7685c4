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
// lane, all accesses are 16 bytes and a warp has 512 / D heads (a round) at once.
// A warp takes items of up to kUnroll rounds of a row in turn and issues all loads
// of an item at once; the next item's positions and slot are on their way
// meanwhile.
// What bounds it: HBM, reading and writing T (H_q + 2 H_kv) D values.  32,749 rows
// of 16 + 2 + 2 heads of 128 take 60.6 us, 5.8 TB/s and 86% of a copy's rate; 3,201 of
// 32 + 8 + 8 heads take 17.2 (11.9 at that rate, and a launch; 13.4 where call after call
// has the same rows, which L2 then holds).  In us, those two (17.1 that day): a
// CTA for every four items instead of CTAs that stay 75.0, 17.9; kUnroll 3 67.9,
// 18.4; 4 68.8, 16.7; 6 61.9, 18.1; five CTAs an SM (96 registers) 64.9, 18.6.  One
// value an instruction, whole rows loaded four rounds ahead: 82.3, 25.6 (288
// instructions a round, which bounded it).
#include <algorithm>

#include "common.cuh"

namespace hpd {
namespace {

constexpr int kRopeWarps = 4;
constexpr int kUnroll = 5;
constexpr int kRopeSms = 152, kRopeCtas = 4;  // CTAs of an SM

struct RopeArgs {
  const __nv_bfloat16 *q, *k, *v;
  long long q_stride, k_stride, v_stride;
  const __nv_bfloat16 *q_weight, *k_weight;
  const float *rope;
  const int32_t *pos, *slot;
  __nv_bfloat16 *q_out, *k_cache, *v_cache;
  uint32_t *err;
  long long num_slots;
  float eps;
  int T, H_q, H_kv, max_pos;
  int rounds, seg;      // rounds of a row, of an item (at most)
  int segs;             // items of a row
  uint32_t axis[4];  // 2 bits a frequency, 8 frequencies (a lane's) in 16
};

// Eight values as four pairs, and back: the arithmetic is two values an
// instruction.
__device__ __forceinline__ void unpack8(const uint4 &v, float2 *x) {
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int i = 0; i < 4; ++i)
    x[i] = make_float2(__uint_as_float(w[i] << 16), __uint_as_float(w[i] & 0xffff0000u));
}
__device__ __forceinline__ uint4 pack8(const float2 *x) {
  return make_uint4(pack_bf16x2(x[0].x, x[0].y), pack_bf16x2(x[1].x, x[1].y), pack_bf16x2(x[2].x, x[2].y),
                    pack_bf16x2(x[3].x, x[3].y));
}

template <int D>
__global__ void __launch_bounds__(32 * kRopeWarps, kRopeCtas) qk_norm_rope_kernel(const RopeArgs a) {
  constexpr int kLanes = D / 16;           // lanes of a head
  constexpr int kHeads = 32 / kLanes;      // heads of a round
  const int lane = threadIdx.x & 31, sub = lane % kLanes;
  const int step = static_cast<int>(gridDim.x) * kRopeWarps;
  const int n_rot = a.H_q + a.H_kv, n_heads = n_rot + a.H_kv;
  const uint32_t axes = a.axis[sub >> 1] >> (16 * (sub & 1)) & 0xffffu;
  pdl_wait();     // rows, positions, slots and the caches as the kernel before leaves them
  pdl_trigger();
  int t = blockIdx.x * kRopeWarps + (threadIdx.x >> 5), part = 0;  // row and part of it: item t * segs + part
  if (a.segs > 1) {
    part = t % a.segs;
    t /= a.segs;
  }
  const int step_t = step / a.segs, step_part = step - step_t * a.segs;
  const bool one_axis = axes == (axes & 3u) * 0x5555u;  // all eight of this lane's frequencies
  const int32_t *pos = a.pos + static_cast<long long>(axes & 3u) * a.T;
  int p_next = 0, slot_next = 0;
  auto fetch_place = [&] {
    if (t >= a.T) return;
    p_next = pos[t];
    slot_next = a.slot[t];
  };
  fetch_place();
  while (t < a.T) {
    int slot = slot_next;
    const int p = p_next, r0 = part * a.seg, n = min(a.seg, a.rounds - r0), h0 = r0 * kHeads + lane / kLanes;
    // (base pointers less the heads before theirs, at this lane's columns)
    const __nv_bfloat16 *q_in = a.q + t * a.q_stride + 8 * sub;
    const __nv_bfloat16 *k_in = a.k + t * a.k_stride + 8 * sub - a.H_q * D;
    const __nv_bfloat16 *v_in = a.v + t * a.v_stride + 8 * sub - n_rot * D;
    uint4 lo[kUnroll], hi[kUnroll];
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      const int h = h0 + u * kHeads;
      lo[u] = hi[u] = make_uint4(0u, 0u, 0u, 0u);
      if (u < n && h < n_heads) {
        const uint4 *src = reinterpret_cast<const uint4 *>((h < a.H_q ? q_in : h < n_rot ? k_in : v_in) + h * D);
        lo[u] = src[0];
        hi[u] = src[D / 16];
      }
    }
    const int t_now = t;
    t += step_t;
    part += step_part;
    if (part >= a.segs) {
      part -= a.segs;
      ++t;
    }
    float2 cos[4], sin[4];  // of this lane's 8 frequencies
    if (r0 * kHeads < n_rot) {
      auto row = [&](int at) {  // this lane's frequencies at a position
        if (static_cast<unsigned>(at) >= static_cast<unsigned>(a.max_pos)) {
          atomicOr(a.err, HPD_DEVERR_POSITION);
          at = min(max(at, 0), a.max_pos - 1);
        }
        return a.rope + (static_cast<long long>(at) * (D / 2) + 8 * sub) * 2;
      };
      if (one_axis) {
        const float4 *r = reinterpret_cast<const float4 *>(row(p));
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float4 c = r[i];
          cos[i] = make_float2(c.x, c.z);
          sin[i] = make_float2(c.y, c.w);
        }
      } else {  // (few lanes: the positions are not ahead)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int32_t *at = a.pos + t_now;
          const float *c0 = row(at[static_cast<long long>(axes >> (4 * i) & 3u) * a.T]) + 4 * i;
          const float *c1 = row(at[static_cast<long long>(axes >> (4 * i + 2) & 3u) * a.T]) + 4 * i + 2;
          cos[i] = make_float2(c0[0], c1[0]);
          sin[i] = make_float2(c0[1], c1[1]);
        }
      }
    }
    fetch_place();
    if (slot >= a.num_slots) {
      if (lane == 0) atomicOr(a.err, HPD_DEVERR_PAGE_ID);
      slot = -1;
    }
    __nv_bfloat16 *q_out = a.q_out + static_cast<long long>(t_now) * a.H_q * D + 8 * sub;
    const long long row = static_cast<long long>(slot) * a.H_kv * D + 8 * sub;
    __nv_bfloat16 *k_out = a.k_cache + row - a.H_q * D, *v_out = a.v_cache + row - n_rot * D;
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      if (u >= n) break;
      const int h = h0 + u * kHeads;
      const bool is_q = h < a.H_q;
      if ((r0 + u) * kHeads < n_rot) {
        float2 x[4], y[4], s2 = make_float2(0.f, 0.f);
        unpack8(lo[u], x);
        unpack8(hi[u], y);
#pragma unroll
        for (int i = 0; i < 4; ++i) s2 = __ffma2_rn(x[i], x[i], __ffma2_rn(y[i], y[i], s2));
        float ss = s2.x + s2.y;
#pragma unroll
        for (int o = 1; o < kLanes; o <<= 1) ss += __shfl_xor_sync(0xffffffffu, ss, o);
        if (h < n_rot) {
          const float r = rsqrtf(ss * (1.0f / D) + a.eps);
          const float2 r2 = make_float2(r, r);
          const uint4 *w = reinterpret_cast<const uint4 *>((is_q ? a.q_weight : a.k_weight) + 8 * sub);
          if (is_q ? a.q_weight : a.k_weight) {
            float2 wx[4], wy[4];
            unpack8(w[0], wx);
            unpack8(w[D / 16], wy);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              x[i] = __fmul2_rn(x[i], wx[i]);
              y[i] = __fmul2_rn(y[i], wy[i]);
            }
          }
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const float2 xn = __fmul2_rn(x[i], r2), yn = __fmul2_rn(y[i], r2);
            const float2 ys = __fmul2_rn(yn, sin[i]);
            x[i] = __ffma2_rn(xn, cos[i], make_float2(-ys.x, -ys.y));
            y[i] = __ffma2_rn(yn, cos[i], __fmul2_rn(xn, sin[i]));
          }
          lo[u] = pack8(x);
          hi[u] = pack8(y);
        }
      }
      if (h < n_heads && (is_q || slot >= 0)) {
        uint4 *dst = reinterpret_cast<uint4 *>((is_q ? q_out : h < n_rot ? k_out : v_out) + h * D);
        dst[0] = lo[u];
        dst[D / 16] = hi[u];
      }
    }
  }
}

// Items of as many rounds as there are, up to kUnroll, where whole rows fill the
// GPU with warps, else of fewer.
template <int D>
cudaError_t launch_rope(RopeArgs &a, cudaStream_t s) {
  constexpr int heads = 512 / D, warps = kRopeSms * 16;
  a.rounds = (a.H_q + 2 * a.H_kv + heads - 1) / heads;
  const int least = std::max(1, std::min(a.rounds, warps / a.T));  // parts of a row that fill the GPU
  const int segs = std::max(least, (a.rounds + kUnroll - 1) / kUnroll);
  a.seg = (a.rounds + segs - 1) / segs;
  a.segs = (a.rounds + a.seg - 1) / a.seg;
  const long long items = static_cast<long long>(a.T) * a.segs;
  const int ctas =
      static_cast<int>(std::min<long long>((items + kRopeWarps - 1) / kRopeWarps, kRopeSms * kRopeCtas));
  return launch_kernel(true, qk_norm_rope_kernel<D>, dim3(ctas), dim3(32 * kRopeWarps), 0, s, a);
}

}  // namespace

hpd_status check_norm_rope(const hpd_qk_norm_rope_args *a) {
  if (!a || a->T < 0 || a->H_q < 1 || a->H_kv < 1 || a->n_axes < 1 || a->n_axes > 4 || a->max_pos < 1 ||
      a->num_slots < 1 || !(a->eps >= 0.f) || a->eps > 3.4e38f)
    return HPD_ERR_INVALID_ARG;
  if (a->D != 64 && a->D != 128) return HPD_ERR_UNSUPPORTED;
  if (static_cast<long long>(a->H_q) + 2LL * a->H_kv > (1 << 20)) return HPD_ERR_UNSUPPORTED;
  if (!a->rope || !a->k_cache || !a->v_cache) return HPD_ERR_INVALID_ARG;
  if (a->T > 0 && (!a->q || !a->k || !a->v || !a->pos || !a->slot || !a->q_out)) return HPD_ERR_INVALID_ARG;
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
  return HPD_OK;
}

cudaError_t launch_norm_rope(const hpd_qk_norm_rope_args *a, bool queries_only, cudaStream_t s) {
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
  k.H_kv = queries_only ? 0 : a->H_kv;
  k.max_pos = a->max_pos;
  for (int i = 0; i < a->D / 2; ++i) k.axis[i >> 4] |= static_cast<uint32_t>(a->axis[i]) << (2 * (i & 15));
  return a->D == 64 ? launch_rope<64>(k, s) : launch_rope<128>(k, s);
}

}  // namespace hpd

extern "C" hpd_status hpd_qk_norm_rope(const hpd_qk_norm_rope_args *a, hpd_stream_t stream) {
  using namespace hpd;
  const hpd_status st = check_norm_rope(a);
  if (st != HPD_OK || a->T == 0) return st;
  const cudaError_t e = launch_norm_rope(a, false, reinterpret_cast<cudaStream_t>(stream));
  return e == cudaSuccess ? HPD_OK : record_cuda_error(e);
}
