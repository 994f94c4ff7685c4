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
//   P V: V is widened to f16, which holds every code, and a weight goes to the tensor cores
//      as f16 too, times its value's scale over v_ref (the largest of the unit's first block,
//      a power of two), with its row's base, so weighted, from 2^3 to 2^4: 2^12 times that fits,
//      and the least that f16 keeps loses 2^-28 of it at most, whatever the scales are: the row's
//      products add up to it at least.  2^-11 of a weight is what the rounding costs otherwise, an
//      eighth of bf16's.  A unit whose O is not finite (a weight or a scale above f16's range) is
//      run again against true maxima with V and weights in bf16, which has the range, and so is one
//      with scales below 2^-14 of v_ref in a block that all rows see, or of a row's base.
//      Where all rows see all of a block, v_ref is the unit's, and the scale's log2 is an addend
//      of the weights' exponents: one product a weight less, and one for 16 keys more in the
//      sums, which are of the weights alone.
//   Roles beside those of chunk_attn.cuh: warps 2, 3 load V's codes; warp 7 has the pages'
//      scales in shared memory a few blocks ahead; warps 20 to 23 part the queries, which go
//      to TMEM as the tensor cores' A, and widen V's codes from one ring of shared memory into
//      another.  24 warps, 80 registers a thread.
//   Tiles of 32 rows and fewer (a token or a few of a sequence) have their rows four times
//      among the 128: each copy has one page of each half of a block, a quarter of the
//      exponentials, and the output warps add the copies' O and sums.
//   Order: where there is more than a unit an SM, the longest sequences' units come first.
//
// What bounds it, and what it measured on a GB300 (calls one after another; bf16 cache in
// brackets):
//   64 sequences of a token, 32 / 8 heads of 128, contexts of 100 to 8,191: 121 to 127 us [206],
//     5.1 TB/s of 6.7: HBM, behind some 5 us until the first scores and 5 of tail.  19 of
//     8,191: 60.6 us.
//   2,048 tokens behind 14,336, 32 / 8 heads of 128: 308 us [295], 1.67 PFLOP/s, 334 to 341
//     after seconds of it, the power limit [337 to 349]; a block 0.76 us, whose MMAs have 0.65: the issue
//     slots, of which a quarter of an SM's two softmax warps have most.
//   24 ragged chunks of up to 300, half of them a token, 40 / 8: 120 to 123 us [97 to 110 of
//     other lengths]: units' changes (a unit's queries are in parts some 3,000 cycles after its
//     slot is free) and blocks, of which the single tokens' have five rows.
//   One token behind 255, 8 / 2 heads of 64: 8.4 us [8.3], latency.
// These are of normal scores with a standard deviation of 1.  A unit that is run again takes three
// passes, two of which have its blocks one by one through the masked path.  Sharper scores (us; other
// contexts of the 64 tokens, with a deviation of 1 101 [175]):
//   deviation               2          2.5          3          4          5
//   64 tokens          101 [175]    101 [176]   198 [176]  318 [175]  342 [175]
//   long chunk         528 [295]    772 [295]  1,002 [294] 1,141 [293] 1,141 [293]
// Rows four times, and once: 64 sequences of a token 123 us and 132, 24 of 16 / 2 heads 18.4
// and 19.9, 19 of 8,191 with heads of 64 48.0 and 51.3; at 32 rows (19 times 32 tokens) 66.7
// and 66.8.  Longest first, and in order: 123 and 139, 124 and 129.
// Conversions are what V costs.  The long chunk: to bf16 by the warps that load it, three
// instructions a pair, 606 us; to f16 by warps of their own 393; halves of registers as
// operands of the conversions 328; queries parted by four lanes a row, which read it once,
// instead of one 317; scales as addends of the exponents 308 (320 without in that run; the
// ragged chunks 120 and 129, 19 times 32 tokens with heads of 64 52.7 and 54.8).
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
