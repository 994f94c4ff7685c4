// chunk_attn.cu -- attention of a chunk of new tokens over the paged cache
// (hpd_chunk_attn): one warp to a row and head, 32 keys at a time with a running
// maximum and sum.
#include <algorithm>
#include <cmath>

#include "common.cuh"

namespace hpd {
namespace {

struct ChunkArgs {
  const __nv_bfloat16 *q;
  long long q_stride;
  const int32_t *chunk_cu, *seq_len, *full_len;
  const __nv_bfloat16 *k_cache, *v_cache;
  const int32_t *page_table;
  int S, T, H_q, H_kv, G, num_pages, max_pages;
  float scale_log2;
  __nv_bfloat16 *out;
  float *lse;
  uint32_t *err;
};

constexpr int kWarps = 4;

template <int D>
__global__ void __launch_bounds__(32 * kWarps) chunk_attn_simple_kernel(const ChunkArgs a) {
  __shared__ float s_q[kWarps][D];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const long long item = static_cast<long long>(blockIdx.x) * kWarps + warp;
  pdl_wait();
  pdl_trigger();
  if (item >= static_cast<long long>(a.T) * a.H_q) return;
  const int t = static_cast<int>(item / a.H_q), h = static_cast<int>(item % a.H_q), g = h / a.G;
  // the row's sequence (offsets clamped into 0 .. T)
  int s = -1, c0 = 0, c1 = 0;
  for (int i = 0; i < a.S && s < 0; ++i) {
    c0 = min(max(a.chunk_cu[i], 0), a.T);
    c1 = min(max(a.chunk_cu[i + 1], 0), a.T);
    if (c1 < c0 || c0 != a.chunk_cu[i] || c1 != a.chunk_cu[i + 1]) flag_error(a.err, HPD_DEVERR_BRANCH_CU);
    if (t >= c0 && t < c1) s = i;
  }
  if (s < 0) return;
  int L = a.seq_len[s];
  if (L < 0 || L > a.max_pages * kPage) {
    flag_error(a.err, HPD_DEVERR_BRANCH_LEN);
    L = min(max(L, 0), a.max_pages * kPage);
  }
  int lim = L - (c1 - c0) + (t - c0) + 1;
  if (a.full_len) lim = max(lim, a.full_len[s]);
  lim = min(lim, L);
  for (int c = lane; c < D; c += 32)
    s_q[warp][c] = __bfloat162float(a.q[t * a.q_stride + h * D + c]);
  __syncwarp();
  const float NEG_INF = -__int_as_float(0x7f800000);
  float m = NEG_INF, l = 0.f, o[D / 32];
  for (int c = 0; c < D / 32; ++c) o[c] = 0.f;
  for (int j0 = 0; j0 < lim; j0 += 32) {
    const int j = j0 + lane;
    int pg = 0;
    float x = NEG_INF;
    if (j < lim) {
      pg = a.page_table[static_cast<size_t>(s) * a.max_pages + j / kPage];
      if (pg < 0 || pg >= a.num_pages) {
        flag_error(a.err, HPD_DEVERR_PAGE_ID);
        pg = 0;
      }
      const __nv_bfloat16 *k = a.k_cache + ((static_cast<size_t>(pg) * kPage + j % kPage) * a.H_kv + g) * D;
      x = 0.f;
      for (int c = 0; c < D; ++c) x = fmaf(s_q[warp][c], __bfloat162float(k[c]), x);
      x *= a.scale_log2;
    }
    float mx = x;
    for (int w = 16; w > 0; w >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, w));
    const float m_new = fmaxf(m, mx), base = m_new == NEG_INF ? 0.f : m_new;
    const float alpha = exp2f(m - base), p = exp2f(x - base);
    m = m_new;
    float sum = p;
    for (int w = 16; w > 0; w >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, w);
    l = l * alpha + sum;
    for (int c = 0; c < D / 32; ++c) o[c] *= alpha;
    for (int i = 0; i < min(32, lim - j0); ++i) {
      const float pi = __shfl_sync(0xffffffffu, p, i);
      const int pgi = __shfl_sync(0xffffffffu, pg, i);
      const __nv_bfloat16 *v =
          a.v_cache + ((static_cast<size_t>(pgi) * kPage + (j0 + i) % kPage) * a.H_kv + g) * D;
      for (int c = 0; c < D / 32; ++c) o[c] = fmaf(pi, __bfloat162float(v[c * 32 + lane]), o[c]);
    }
  }
  const float inv = l > 0.f ? 1.f / l : l;
  for (int c = 0; c < D / 32; ++c) a.out[item * D + c * 32 + lane] = __float2bfloat16(o[c] * inv);
  if (lane == 0 && a.lse) a.lse[item] = l > 0.f || l != l ? (m + log2f(l)) * kLn2 : NEG_INF;
}

hpd_status check_scalars(const hpd_chunk_attn_args *a) {
  if (!a) return HPD_ERR_INVALID_ARG;
  if (a->S < 1 || a->T < 1 || a->H_q < 1 || a->H_kv < 1 || a->num_pages < 1 || a->max_pages < 1 ||
      a->max_seq_len < 0 || a->q_stride < 0 || a->q_stride % 8 != 0)
    return HPD_ERR_INVALID_ARG;
  if (a->H_q % a->H_kv != 0 || !std::isfinite(a->scale)) return HPD_ERR_INVALID_ARG;
  if (a->H_q / a->H_kv > 16 || (a->D != 64 && a->D != 128)) return HPD_ERR_UNSUPPORTED;
  if (a->q_stride != 0 && a->q_stride < static_cast<int64_t>(a->H_q) * a->D) return HPD_ERR_INVALID_ARG;
  if (static_cast<long long>(a->max_pages) * kPage >= (1LL << 30)) return HPD_ERR_UNSUPPORTED;
  return HPD_OK;
}

}  // namespace
}  // namespace hpd

extern "C" {

size_t hpd_chunk_attn_workspace_size(const hpd_chunk_attn_args *a) {
  return hpd::check_scalars(a) == HPD_OK ? 256 : 0;
}

hpd_status hpd_chunk_attn(const hpd_chunk_attn_args *a, hpd_stream_t stream) {
  using namespace hpd;
  const hpd_status st = check_scalars(a);
  if (st != HPD_OK) return st;
  if (!a->q || !a->chunk_cu || !a->seq_len || !a->k_cache || !a->v_cache || !a->page_table || !a->out)
    return HPD_ERR_INVALID_ARG;
  for (const void *p : {a->q, a->k_cache, a->v_cache, static_cast<const void *>(a->out)})
    if ((reinterpret_cast<uintptr_t>(p) & 15u) != 0) return HPD_ERR_INVALID_ARG;
  for (const void *p : {static_cast<const void *>(a->chunk_cu), static_cast<const void *>(a->seq_len),
                        static_cast<const void *>(a->full_len), static_cast<const void *>(a->page_table),
                        static_cast<const void *>(a->lse)})
    if ((reinterpret_cast<uintptr_t>(p) & 3u) != 0) return HPD_ERR_INVALID_ARG;
  if (!a->workspace || (reinterpret_cast<uintptr_t>(a->workspace) & 255u) != 0 ||
      a->workspace_bytes < hpd_chunk_attn_workspace_size(a))
    return HPD_ERR_WORKSPACE;
  ChunkArgs k{};
  k.q = static_cast<const __nv_bfloat16 *>(a->q);
  k.q_stride = a->q_stride ? a->q_stride : static_cast<long long>(a->H_q) * a->D;
  k.chunk_cu = a->chunk_cu;
  k.seq_len = a->seq_len;
  k.full_len = a->full_len;
  k.k_cache = static_cast<const __nv_bfloat16 *>(a->k_cache);
  k.v_cache = static_cast<const __nv_bfloat16 *>(a->v_cache);
  k.page_table = a->page_table;
  k.S = a->S;
  k.T = a->T;
  k.H_q = a->H_q;
  k.H_kv = a->H_kv;
  k.G = a->H_q / a->H_kv;
  k.num_pages = a->num_pages;
  k.max_pages = a->max_pages;
  k.scale_log2 = (a->scale != 0.f ? a->scale : 1.0f / std::sqrt(static_cast<float>(a->D))) * kLog2e;
  k.out = static_cast<__nv_bfloat16 *>(a->out);
  k.lse = a->lse;
  k.err = static_cast<uint32_t *>(a->workspace);
  const long long ctas = (static_cast<long long>(a->T) * a->H_q + kWarps - 1) / kWarps;
  if (ctas > INT32_MAX) return HPD_ERR_UNSUPPORTED;
  cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  const dim3 grid(static_cast<unsigned>(ctas)), block(32 * kWarps);
  const cudaError_t e = a->D == 64 ? launch_kernel(true, chunk_attn_simple_kernel<64>, grid, block, 0, s, k)
                                   : launch_kernel(true, chunk_attn_simple_kernel<128>, grid, block, 0, s, k);
  return e == cudaSuccess ? HPD_OK : record_cuda_error(e);
}

}  // extern "C"
