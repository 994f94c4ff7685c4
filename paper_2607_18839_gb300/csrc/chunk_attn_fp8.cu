// chunk_attn_fp8.cu -- attention of a chunk of new tokens over the paged cache in
// 8 bits (hpd_chunk_attn_fp8).
//
//   k_j = code * ks[page][head],  v_j likewise;  everything else as in chunk_attn.cuh,
// whose kernel this is with kFp8.  What differs:
//   S: the tensor cores take the codes of K as they are, and Q in two e4m3 parts of one
//      power of two for each row (bf16 has eight significant bits, e4m3 four: the second
//      part holds what the first leaves, but for values below 2^-9 of the row's largest,
//      which keep 2^-17 of that).  8-bit products run twice as fast, so the two take as
//      long as one of bf16, and K is never widened.  Scales go to the scores, 16 at a time.
//   P V: V is widened to bf16, which holds every code, by four warps that load it; V's
//      scale goes to the weights before their rounding.
#include "chunk_attn.cuh"

extern "C" {

size_t hpd_chunk_attn_fp8_workspace_size(const hpd_chunk_attn_fp8_args *f) {
  return f ? hpd_chunk_attn_workspace_size(&f->attn) : 0;
}

hpd_status hpd_chunk_attn_fp8(const hpd_chunk_attn_fp8_args *f, hpd_stream_t stream) {
  using namespace hpd;
  const hpd_status st = check_chunk_attn(f ? &f->attn : nullptr);
  if (st != HPD_OK) return st;
  if (!f->k_scale || !f->v_scale ||
      ((reinterpret_cast<uintptr_t>(f->k_scale) | reinterpret_cast<uintptr_t>(f->v_scale)) & 3u) != 0)
    return HPD_ERR_INVALID_ARG;
  return run_chunk_attn<true>(&f->attn, f->k_scale, f->v_scale, stream);
}

}  // extern "C"
