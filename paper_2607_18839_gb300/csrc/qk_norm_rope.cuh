// qk_norm_rope.cuh -- rows of queries, keys and values normed, rotated and written as they
// are: the body of hpd_qk_norm_rope's kernel (qk_norm_rope.cu says what bounds it), and
// what hpd_qk_norm_rope_fp8's has for its queries.
#pragma once

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

// Rows of a call, by warp `warp` of `step`.
template <int D>
__device__ __forceinline__ void norm_rope_rows(const RopeArgs &a, int warp, int step) {
  constexpr int kLanes = D / 16;           // lanes of a head
  constexpr int kHeads = 32 / kLanes;      // heads of a round
  const int lane = threadIdx.x & 31, sub = lane % kLanes;
  const int n_rot = a.H_q + a.H_kv, n_heads = n_rot + a.H_kv;
  const uint32_t axes = a.axis[sub >> 1] >> (16 * (sub & 1)) & 0xffffu;
  int t = warp, part = 0;  // row and part of it: item t * segs + part
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

// ------------------------------------------------------------------ host --

// Items of as many rounds as there are, up to kUnroll, where whole rows fill the
// GPU with warps, else of fewer.  Returns their number.
inline long long plan_items(RopeArgs &a, int D) {
  const int heads = 512 / D, warps = kRopeSms * 16;
  a.rounds = (a.H_q + 2 * a.H_kv + heads - 1) / heads;
  const int least = std::max(1, std::min(a.rounds, warps / a.T));  // parts of a row that fill the GPU
  const int segs = std::max(least, (a.rounds + kUnroll - 1) / kUnroll);
  a.seg = (a.rounds + segs - 1) / segs;
  a.segs = (a.rounds + a.seg - 1) / a.seg;
  return static_cast<long long>(a.T) * a.segs;
}

inline RopeArgs rope_args(const hpd_qk_norm_rope_args *a) {
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
  for (int i = 0; i < a->D / 2; ++i) k.axis[i >> 4] |= static_cast<uint32_t>(a->axis[i]) << (2 * (i & 15));
  return k;
}

}  // namespace
}  // namespace hpd
