// chunk_slots.cu -- pages and slots of a step's new tokens, from the lengths of
// its sequences (hpd_chunk_slots).
//
//   held_s = ceil(L_s / 16), need_s = ceil((L_s + n_s) / 16)
//   cu_s   = sum of n before s;  pg_s = sum of (need - held) before s
//   page p of s, held_s <= p < need_s:  free_pages[top - total + pg_s + p - held_s]
//   token t of s: pos = L_s + t - cu_s, slot = 16 * page(pos / 16) + pos % 16
//
// One launch.  Every CTA scans all lengths (both sums at once) into shared
// memory, which is cheaper than a second launch that would wait for the first;
// then it takes a share of the tokens, four to a thread, whose sequence a binary
// search of cu finds.  The first token of a page that is new enters it in the
// table.  The last CTA to have read the lengths writes the new ones and the
// stack's top, so that both may be updated in place.
// What bounds it: the chain of lengths, scan, page id and store.  4 sequences with 46
// new tokens take 4.2 us, 512 with 63,260 take 5.8; their bytes would take 0.08 at a
// copy's rate.  (With every CTA waiting for the answer of the count before its tokens,
// fences in a call of one CTA among them: 4.7 and 6.2.)
#include <algorithm>

#include "common.cuh"

namespace hpd {
namespace {

constexpr int kSlotThreads = 512;
constexpr int kSlotTokens = 4;  // tokens of a thread: one 16-byte store
constexpr int kMaxSeqs = 16384;

struct SlotArgs {
  const int32_t *new_len, *seq_len;
  int32_t *page_table;
  const int32_t *free_pages, *free_top;
  int32_t *seq_len_out, *free_top_out, *chunk_cu, *slot, *pos;
  uint32_t *err;
  int *ticket;
  int S, max_pages, num_pages, max_tokens;
};

// Sums that stop at 2^31 - 1 (associative, as no term is negative): a total that
// large is refused whatever it would have been.
__device__ __forceinline__ int add_sat(int a, int b) {
  return static_cast<int>(min(static_cast<uint32_t>(a) + static_cast<uint32_t>(b), 0x7fffffffu));
}

__device__ __forceinline__ int2 scan_step(int2 v, int o, int lane) {
  const int x = __shfl_up_sync(0xffffffffu, v.x, o), y = __shfl_up_sync(0xffffffffu, v.y, o);
  return lane >= o ? make_int2(add_sat(v.x, x), add_sat(v.y, y)) : v;
}

__global__ void __launch_bounds__(kSlotThreads) chunk_slots_kernel(const SlotArgs a) {
  extern __shared__ int s_dyn[];
  int *s_cu = s_dyn;              // [S + 1] tokens before a sequence
  int *s_pg = s_cu + a.S + 1;     // [S + 1] new pages before a sequence
  int *s_len = s_pg + a.S + 1;    // [S] tokens it had
  __shared__ int2 s_warp[kSlotThreads / 32];
  __shared__ int s_bad, s_last, s_top;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  if (tid == 0) s_bad = s_cu[0] = s_pg[0] = 0;
  pdl_wait();     // the lengths, tables and the stack as the kernel before leaves them
  pdl_trigger();  // the next kernel may launch; it waits for this one
  if (tid == kSlotThreads - 1) s_top = *a.free_top;  // on its way with the lengths
  int2 base = make_int2(0, 0);
  for (int s0 = 0; s0 < a.S; s0 += kSlotThreads) {
    const int s = s0 + tid;
    int2 v = make_int2(0, 0);
    bool bad = false;
    if (s < a.S) {
      const int n = a.new_len[s], L = a.seq_len[s];
      const int cap = a.max_pages * kPage;
      bad = n < 0 || L < 0 || L > cap || n > cap - L;
      if (!bad) v = make_int2(n, ceil_div_i(L + n, kPage) - ceil_div_i(L, kPage));
      s_len[s] = L;
    }
    int2 incl = v;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) incl = scan_step(incl, o, lane);
    if (lane == 31) s_warp[warp] = incl;
    if (__syncthreads_or(bad) && tid == 0) s_bad = 1;
    if (warp == 0) {
      int2 w = lane < kSlotThreads / 32 ? s_warp[lane] : make_int2(0, 0);
#pragma unroll
      for (int o = 1; o < kSlotThreads / 32; o <<= 1) w = scan_step(w, o, lane);
      if (lane < kSlotThreads / 32) s_warp[lane] = w;
    }
    __syncthreads();
    if (warp > 0) incl = make_int2(add_sat(incl.x, s_warp[warp - 1].x), add_sat(incl.y, s_warp[warp - 1].y));
    incl = make_int2(add_sat(incl.x, base.x), add_sat(incl.y, base.y));
    if (s < a.S) {
      s_cu[s + 1] = incl.x;
      s_pg[s + 1] = incl.y;
    }
    const int2 all = s_warp[kSlotThreads / 32 - 1];
    base = make_int2(add_sat(base.x, all.x), add_sat(base.y, all.y));
    __syncthreads();  // s_warp is reused
  }
  // This CTA has read all lengths and the top into shared memory: who is the last to
  // say so writes the new ones, once the answer is here.
  int before = 0;
  if (gridDim.x > 1 && tid == 0) {
    __threadfence();
    before = atomicAdd(a.ticket, 1);
  }
  const int total = base.x, pages = base.y, top = s_top;
  const uint32_t why = s_bad                                                          ? HPD_DEVERR_BRANCH_LEN
                       : total > a.max_tokens                                         ? HPD_DEVERR_CHUNK_CAP
                       : top < 0 || top > a.num_pages || pages > top                  ? HPD_DEVERR_POOL
                                                                                      : 0u;
  auto write_lengths = [&] {
    for (int s = tid; s < a.S; s += kSlotThreads)
      a.seq_len_out[s] = why ? s_len[s] : s_len[s] + (s_cu[s + 1] - s_cu[s]);
    if (tid == 0) {
      *a.free_top_out = why ? top : top - pages;
      if (why) atomicOr(a.err, why);
    }
  };
  if (gridDim.x == 1) write_lengths();
  if (blockIdx.x == 0)
    for (int s = tid; s <= a.S; s += kSlotThreads) a.chunk_cu[s] = why ? 0 : s_cu[s];
  const int end = why ? 0 : total, first = top - pages;
  const bool vec = ((reinterpret_cast<uintptr_t>(a.slot) | reinterpret_cast<uintptr_t>(a.pos)) & 15u) == 0;
  const long long step = static_cast<long long>(gridDim.x) * kSlotThreads * kSlotTokens;
  for (long long t0 = (static_cast<long long>(blockIdx.x) * kSlotThreads + tid) * kSlotTokens;
       t0 < a.max_tokens; t0 += step) {
    int slot[kSlotTokens], pos[kSlotTokens];
    int s = 0;
    if (t0 < end) {  // the last sequence that starts at or before t0
      int hi = a.S;
      while (hi - s > 1) {
        const int mid = (s + hi) >> 1;
        if (s_cu[mid] <= t0) s = mid; else hi = mid;
      }
    }
#pragma unroll
    for (int i = 0; i < kSlotTokens; ++i) {
      const int t = static_cast<int>(t0) + i;
      slot[i] = -1;
      pos[i] = 0;
      if (t >= end) continue;
      while (s_cu[s + 1] <= t) ++s;  // (t < s_cu[S], and empty sequences are passed over)
      const int L = s_len[s], p = L + (t - s_cu[s]);
      const int held = ceil_div_i(L, kPage), page = p / kPage;
      int32_t *entry = a.page_table + static_cast<size_t>(s) * a.max_pages + page;
      int id;
      if (page < held) {
        id = *entry;
      } else {
        id = a.free_pages[first + s_pg[s] + (page - held)];
        if (p % kPage == 0) *entry = id;
      }
      pos[i] = p;
      if (id >= 0 && id < a.num_pages) slot[i] = id * kPage + p % kPage;
      else atomicOr(a.err, HPD_DEVERR_PAGE_ID);
    }
    if (vec && t0 + kSlotTokens <= a.max_tokens) {
      *reinterpret_cast<int4 *>(a.slot + t0) = make_int4(slot[0], slot[1], slot[2], slot[3]);
      if (a.pos) *reinterpret_cast<int4 *>(a.pos + t0) = make_int4(pos[0], pos[1], pos[2], pos[3]);
    } else {
#pragma unroll
      for (int i = 0; i < kSlotTokens; ++i)
        if (t0 + i < a.max_tokens) {
          a.slot[t0 + i] = slot[i];
          if (a.pos) a.pos[t0 + i] = pos[i];
        }
    }
  }
  if (gridDim.x > 1) {
    if (tid == 0) {
      s_last = before == static_cast<int>(gridDim.x) - 1;
      if (s_last) {
        *a.ticket = 0;
        __threadfence();
      }
    }
    __syncthreads();
    if (s_last) write_lengths();
  }
}

}  // namespace
}  // namespace hpd

extern "C" hpd_status hpd_chunk_slots(const hpd_chunk_slots_args *a, hpd_stream_t stream) {
  using namespace hpd;
  if (!a || !a->new_len || !a->seq_len || !a->page_table || !a->free_pages || !a->free_top ||
      !a->seq_len_out || !a->free_top_out || !a->chunk_cu || !a->slot)
    return HPD_ERR_INVALID_ARG;
  if (!a->workspace || (reinterpret_cast<uintptr_t>(a->workspace) & 255u) != 0) return HPD_ERR_WORKSPACE;
  if (a->S < 1 || a->max_pages < 1 || a->num_pages < 1 || a->max_tokens < 1) return HPD_ERR_INVALID_ARG;
  if (a->S > kMaxSeqs || a->max_pages > INT32_MAX / kPage || a->num_pages > INT32_MAX / kPage)
    return HPD_ERR_UNSUPPORTED;
  for (const void *p : {static_cast<const void *>(a->new_len), static_cast<const void *>(a->seq_len),
                        static_cast<const void *>(a->page_table), static_cast<const void *>(a->free_pages),
                        static_cast<const void *>(a->free_top), static_cast<const void *>(a->seq_len_out),
                        static_cast<const void *>(a->free_top_out), static_cast<const void *>(a->chunk_cu),
                        static_cast<const void *>(a->slot), static_cast<const void *>(a->pos)})
    if ((reinterpret_cast<uintptr_t>(p) & 3u) != 0) return HPD_ERR_INVALID_ARG;
  const size_t smem = (3 * static_cast<size_t>(a->S) + 2) * sizeof(int);
  if (smem > 47 * 1024) {  // (the default of 48 KB holds the kernel's own 144 bytes too)
    const cudaError_t e = cudaFuncSetAttribute(chunk_slots_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                               (3 * kMaxSeqs + 2) * static_cast<int>(sizeof(int)));
    if (e != cudaSuccess) return record_cuda_error(e);
  }
  SlotArgs k{a->new_len, a->seq_len, a->page_table, a->free_pages, a->free_top, a->seq_len_out, a->free_top_out,
             a->chunk_cu, a->slot, a->pos, static_cast<uint32_t *>(a->workspace),
             static_cast<int *>(a->workspace) + 1, a->S, a->max_pages, a->num_pages, a->max_tokens};
  constexpr long long per_cta = kSlotThreads * kSlotTokens;
  const int grid = static_cast<int>(std::min<long long>((a->max_tokens + per_cta - 1) / per_cta, 152));
  const cudaError_t e = launch_kernel(true, chunk_slots_kernel, dim3(grid), dim3(kSlotThreads), smem,
                                      reinterpret_cast<cudaStream_t>(stream), k);
  return e == cudaSuccess ? HPD_OK : record_cuda_error(e);
}
