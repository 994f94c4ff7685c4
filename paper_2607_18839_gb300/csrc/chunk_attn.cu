// chunk_attn.cu -- attention of a chunk of new tokens over a paged cache in bf16
// (hpd_chunk_attn); the kernel is in chunk_attn.cuh.
#include "chunk_attn.cuh"

namespace hpd {

hpd_status check_chunk_attn(const hpd_chunk_attn_args *a) {
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
  if (!a->workspace || (reinterpret_cast<uintptr_t>(a->workspace) & (kAlign - 1)) != 0 ||
      a->workspace_bytes < make_plan(a).bytes)
    return HPD_ERR_WORKSPACE;
  return HPD_OK;
}

}  // namespace hpd

extern "C" {

size_t hpd_chunk_attn_workspace_size(const hpd_chunk_attn_args *a) {
  return hpd::check_scalars(a) == HPD_OK ? hpd::make_plan(a).bytes : 0;
}

hpd_status hpd_chunk_attn(const hpd_chunk_attn_args *a, hpd_stream_t stream) {
  const hpd_status st = hpd::check_chunk_attn(a);
  return st != HPD_OK ? st : hpd::run_chunk_attn<false>(a, nullptr, nullptr, stream);
}

}  // extern "C"
