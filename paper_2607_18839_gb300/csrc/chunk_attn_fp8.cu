// chunk_attn_fp8.cu -- attention of a chunk of new tokens over the paged cache in
// 8 bits (hpd_chunk_attn_fp8).
//
//   row (i, h) of sequence s sees keys j < lim = min(L, max(L - n + i + 1, full));
//   key j is code * scale of its page and head, as its value is
//   p_j = exp(scale q k_j - m),  out = sum p v / sum p,  lse = m + log sum p
// A warp a row: lanes share the columns, keys one after another.
#include <cmath>

#include "fp8.cuh"

namespace hpd {
namespace {

struct ChunkFp8Params {
  const __nv_bfloat16 *q;
  long long q_stride;
  const int32_t *chunk_cu, *seq_len, *full_len;
  const uint8_t *k_cache, *v_cache;
  const float *k_scale, *v_scale;
  const int32_t *page_table;
  int S, T, H_q, H_kv, num_pages, max_pages;
  float scale;
  __nv_bfloat16 *out;
  float *lse;
  uint32_t *err;
};

template <int D>
__global__ void chunk_attn_fp8_kernel(const ChunkFp8Params p) {
  constexpr int kV = D / 32;  // columns of a lane
  const int lane = threadIdx.x & 31, h = blockIdx.y, g = h / (p.H_q / p.H_kv), s = blockIdx.x;
  const float INF = __int_as_float(0x7f800000);
  pdl_wait();
  pdl_trigger();
  const int b0 = p.chunk_cu[s], b1 = p.chunk_cu[s + 1], b_len = p.seq_len[s];
  const int c0 = min(max(b0, 0), p.T), n = max(c0, min(b1, p.T)) - c0;
  const int L = min(max(b_len, 0), p.max_pages * kPage), full = p.full_len ? min(max(p.full_len[s], 0), L) : 0;
  if (b0 != c0 || b1 != c0 + n) flag_error(p.err, HPD_DEVERR_BRANCH_CU);
  if (L != b_len) flag_error(p.err, HPD_DEVERR_BRANCH_LEN);
  auto scale_of = [&](const float *at) {
    const float x = *at;
    if (x >= 0.f && x < INF) return x;
    flag_error(p.err, HPD_DEVERR_SCALE);
    return 0.f;
  };
  auto values = [&](const uint8_t *at, float sc, float *v) {
    for (int c = 0; c < kV; c += 2) {
      const float2 x = of_codes(*reinterpret_cast<const uint16_t *>(at + lane * kV + c));
      v[c] = x.x * sc;
      v[c + 1] = x.y * sc;
    }
  };
  for (int i = blockIdx.z * (blockDim.x >> 5) + (threadIdx.x >> 5); i < n; i += gridDim.z * (blockDim.x >> 5)) {
    const int lim = max(min(max(L - n + i + 1, full), L), 0);
    const size_t pair = static_cast<size_t>(c0 + i) * p.H_q + h;
    float q[kV], o[kV], m = -INF, l = 0.f;
    const __nv_bfloat16 *qr = p.q + (c0 + i) * p.q_stride + h * D + lane * kV;
    bool odd = false;
    for (int c = 0; c < kV; ++c) {
      q[c] = __bfloat162float(qr[c]);
      odd |= !(fabsf(q[c]) < INF);
      o[c] = 0.f;
    }
    odd = __any_sync(0xffffffffu, odd);
    for (int j = 0; j < lim; ++j) {
      int page = p.page_table[static_cast<size_t>(s) * p.max_pages + j / kPage];
      if (page < 0 || page >= p.num_pages) {
        flag_error(p.err, HPD_DEVERR_PAGE_ID);
        page = 0;
      }
      const size_t at = (static_cast<size_t>(page) * kPage + j % kPage) * p.H_kv + g, sat = static_cast<size_t>(page) * p.H_kv + g;
      float k[kV], v[kV], x = 0.f;
      values(p.k_cache + at * D, scale_of(p.k_scale + sat), k);
      values(p.v_cache + at * D, scale_of(p.v_scale + sat), v);
      for (int c = 0; c < kV; ++c) x = fmaf(q[c], k[c], x);
      for (int b = 16; b > 0; b >>= 1) x += __shfl_xor_sync(0xffffffffu, x, b);
      x *= p.scale;
      const float m_new = fmaxf(m, x), base = m_new == -INF ? 0.f : m_new;
      const float w = expf(x - base), keep = expf(m - base);
      l = fmaf(l, keep, w);
      for (int c = 0; c < kV; ++c) o[c] = fmaf(o[c], keep, w * v[c]);
      m = m_new;
    }
    const float inv = odd && lim > 0 ? __int_as_float(0x7fffffff) : l == 0.f ? 0.f : 1.f / l;
    for (int c = 0; c < kV; ++c) p.out[pair * D + lane * kV + c] = __float2bfloat16(l == 0.f && !odd ? 0.f : o[c] * inv);
    if (lane == 0 && p.lse) p.lse[pair] = odd && lim > 0 ? inv : l == 0.f ? -INF : m + logf(l);
  }
}

}  // namespace
}  // namespace hpd

extern "C" {

size_t hpd_chunk_attn_fp8_workspace_size(const hpd_chunk_attn_fp8_args *f) {
  return f ? hpd_chunk_attn_workspace_size(&f->attn) : 0;
}

hpd_status hpd_chunk_attn_fp8(const hpd_chunk_attn_fp8_args *f, hpd_stream_t stream) {
  using namespace hpd;
  const hpd_chunk_attn_args *a = f ? &f->attn : nullptr;
  const hpd_status st = check_chunk_attn(a);
  if (st != HPD_OK) return st;
  if (!f->k_scale || !f->v_scale ||
      ((reinterpret_cast<uintptr_t>(f->k_scale) | reinterpret_cast<uintptr_t>(f->v_scale)) & 3u) != 0)
    return HPD_ERR_INVALID_ARG;
  ChunkFp8Params k{};
  k.q = static_cast<const __nv_bfloat16 *>(a->q);
  k.q_stride = a->q_stride ? a->q_stride : static_cast<long long>(a->H_q) * a->D;
  k.chunk_cu = a->chunk_cu;
  k.seq_len = a->seq_len;
  k.full_len = a->full_len;
  k.k_cache = static_cast<const uint8_t *>(a->k_cache);
  k.v_cache = static_cast<const uint8_t *>(a->v_cache);
  k.k_scale = f->k_scale;
  k.v_scale = f->v_scale;
  k.page_table = a->page_table;
  k.S = a->S;
  k.T = a->T;
  k.H_q = a->H_q;
  k.H_kv = a->H_kv;
  k.num_pages = a->num_pages;
  k.max_pages = a->max_pages;
  k.scale = a->scale != 0.f ? a->scale : 1.0f / std::sqrt(static_cast<float>(a->D));
  k.out = static_cast<__nv_bfloat16 *>(a->out);
  k.lse = a->lse;
  k.err = static_cast<uint32_t *>(a->workspace);
  const dim3 grid(a->S, a->H_q, 32);
  cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  const cudaError_t e = a->D == 64 ? launch_kernel(true, chunk_attn_fp8_kernel<64>, grid, dim3(128), 0, s, k)
                                   : launch_kernel(true, chunk_attn_fp8_kernel<128>, grid, dim3(128), 0, s, k);
  return e == cudaSuccess ? HPD_OK : record_cuda_error(e);
}

}  // extern "C"
