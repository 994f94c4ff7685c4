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
#include "qk_norm_rope.cuh"

namespace hpd {
namespace {

template <int D>
__global__ void __launch_bounds__(32 * kRopeWarps, kRopeCtas) qk_norm_rope_kernel(const RopeArgs a) {
  pdl_wait();     // rows, positions, slots and the caches as the kernel before leaves them
  pdl_trigger();
  norm_rope_rows<D>(a, blockIdx.x * kRopeWarps + (threadIdx.x >> 5), static_cast<int>(gridDim.x) * kRopeWarps);
}

template <int D>
cudaError_t launch_rope(RopeArgs &a, cudaStream_t s) {
  const long long items = plan_items(a, D);
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

cudaError_t launch_norm_rope(const hpd_qk_norm_rope_args *a, cudaStream_t s) {
  RopeArgs k = rope_args(a);
  return a->D == 64 ? launch_rope<64>(k, s) : launch_rope<128>(k, s);
}

}  // namespace hpd

extern "C" hpd_status hpd_qk_norm_rope(const hpd_qk_norm_rope_args *a, hpd_stream_t stream) {
  using namespace hpd;
  const hpd_status st = check_norm_rope(a);
  if (st != HPD_OK || a->T == 0) return st;
  const cudaError_t e = launch_norm_rope(a, reinterpret_cast<cudaStream_t>(stream));
  return e == cudaSuccess ? HPD_OK : record_cuda_error(e);
}
