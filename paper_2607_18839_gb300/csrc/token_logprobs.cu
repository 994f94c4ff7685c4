// token_logprobs.cu -- log probabilities of given tokens, the entropy of their
// distributions and the likeliest alternatives (hpd_token_logprobs).
//
//   d_v = (x_v - max x) scale,  Z = sum exp(d_v) = 1 + R   (R without one largest term)
//   logprob = d_token - log(1 + R),  entropy = log(1 + R) - sum exp(d_v) d_v / Z
// Both terms of the entropy are positive, and log(1 + R) keeps the digits of a small
// R: nothing cancels where a token is nearly sure.
#include <cmath>

#include "common.cuh"

namespace hpd {
namespace {

constexpr int kThreads = 512, kWarps = kThreads / 32;

struct LogpArgs {
  const void *logits;
  long long row_stride;
  const int32_t *tokens;
  float *logprob, *entropy;
  int32_t *top_tokens;
  float *top_logprobs;
  int V, top;
  float scale;
};

// A place in a row's order: larger values first, lower indices first among equal ones.
// (NaN is in none: its value is never asked for.)
struct Place {
  float x;
  int i;
};
__device__ __forceinline__ bool before(const Place &a, const Place &b) { return a.x > b.x || (a.x == b.x && a.i < b.i); }

template <class T>
__device__ __forceinline__ float value(const T *row, int i) {
  return static_cast<float>(row[i]);
}

// One CTA a row: the row is read for the maximum, for the sums, and once for each
// alternative.
template <class T>
__global__ void __launch_bounds__(kThreads) token_logprobs_kernel(const LogpArgs a) {
  __shared__ Place s_place[kWarps];
  __shared__ float s_sum[2][kWarps];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const float INF = __int_as_float(0x7f800000), nan = __int_as_float(0x7fffffff);
  pdl_wait();
  pdl_trigger();
  const size_t r = blockIdx.x;
  const T *row = static_cast<const T *>(a.logits) + static_cast<long long>(r) * a.row_stride;
  // the first place behind `last`
  auto next_of = [&](Place last) {
    Place best{-INF, a.V};
    for (int i = tid; i < a.V; i += kThreads) {
      const Place p{value(row, i), i};
      if (p.x == p.x && before(last, p) && before(p, best)) best = p;
    }
    for (int o = 16; o > 0; o >>= 1) {
      const Place p{__shfl_xor_sync(0xffffffffu, best.x, o), __shfl_xor_sync(0xffffffffu, best.i, o)};
      if (before(p, best)) best = p;
    }
    __syncthreads();
    if (lane == 0) s_place[warp] = best;
    __syncthreads();
    for (int w = 0; w < kWarps; ++w)
      if (before(s_place[w], best)) best = s_place[w];
    return best;
  };
  const Place first = next_of(Place{INF, -1});
  const float m = first.x;
  float rest = 0.f, mean = 0.f;
  for (int i = tid; i < a.V; i += kThreads) {
    const float d = (value(row, i) - m) * a.scale, e = expf(d);
    if (i != first.i) rest += e;
    if (e > 0.f) mean = fmaf(e, d, mean);
  }
  for (int o = 16; o > 0; o >>= 1) {
    rest += __shfl_xor_sync(0xffffffffu, rest, o);
    mean += __shfl_xor_sync(0xffffffffu, mean, o);
  }
  if (lane == 0) {
    s_sum[0][warp] = rest;
    s_sum[1][warp] = mean;
  }
  __syncthreads();
  rest = mean = 0.f;
  for (int w = 0; w < kWarps; ++w) {
    rest += s_sum[0][w];
    mean += s_sum[1][w];
  }
  if (first.i == a.V || !(fabsf(m) < INF)) rest = nan;
  const float log_z = log1pf(rest);
  if (tid == 0) {
    const int t = a.tokens[r];
    const float x = t >= 0 && t < a.V ? value(row, t) : -INF;
    a.logprob[r] = rest == rest ? (x - m) * a.scale - log_z : nan;
    if (a.entropy) a.entropy[r] = log_z - mean / (1.f + rest);
  }
  Place p = first;
  for (int k = 0; k < a.top; ++k) {
    if (tid == 0) {
      a.top_tokens[r * a.top + k] = p.i < a.V ? p.i : -1;
      a.top_logprobs[r * a.top + k] = p.i < a.V && rest == rest ? (p.x - m) * a.scale - log_z : nan;
    }
    if (p.i < a.V && k + 1 < a.top) p = next_of(p);
  }
}

}  // namespace
}  // namespace hpd

extern "C" hpd_status hpd_token_logprobs(const hpd_token_logprobs_args *a, hpd_stream_t stream) {
  using namespace hpd;
  if (!a || a->R < 0 || a->V < 1 || a->top < 0 || a->top > a->V || a->row_stride < 0 || !std::isfinite(a->scale) ||
      a->scale < 0.f || (a->fp32 != 0 && a->fp32 != 1))
    return HPD_ERR_INVALID_ARG;
  if (a->top > 32) return HPD_ERR_UNSUPPORTED;
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
  const cudaError_t e =
      a->fp32 ? launch_kernel(true, token_logprobs_kernel<float>, dim3(a->R), dim3(kThreads), 0, s, k)
              : launch_kernel(true, token_logprobs_kernel<__nv_bfloat16>, dim3(a->R), dim3(kThreads), 0, s, k);
  return e == cudaSuccess ? HPD_OK : record_cuda_error(e);
}
