// chunk_attn.cuh -- attention of a chunk of new tokens over the paged cache on
// 5th-generation tensor cores: the kernel of hpd_chunk_attn (a bf16 cache) and, with
// kFp8, of hpd_chunk_attn_fp8 (e4m3 codes; what differs is said in chunk_attn_fp8.cu).
//
//   row (i, h) of sequence s, h = g G + e:  keys j < lim_i,
//     lim_i = min(L, max(L - n + i + 1, full))
//   S = scale Q K^T over them, P = exp(S - max), out = P V / sum P,
//   lse = max + log sum P
//
// The rows that read KV head g are stacked, token by token, into tiles of 128
// (row r of a tile: token r / G, head g G + r % G; with a G that does not divide
// 128 its last rows are unused), and a tile walks the 128-key blocks, 8 pages
// each, up to the last key that one of its rows sees.
//
// Work units: (tile, KV head, split of the tile's blocks).  One CTA per SM
// takes units from an atomic counter; its roles run apart, so that little drains
// between units:
//   warp 6      scheduler: finds the next unit in the step's lengths and puts
//               its metadata into one of three slots
//   warps 0..3  TMA producers, two of K (and each unit's Q tile ahead of it), two
//               of V: three-stage rings, 128-byte swizzle.  A warp has four pages
//               of each block, one box where they are consecutive in the pool, else
//               four: a box takes its warp some 130 cycles to issue, the tensor map
//               unit 68, so that two warps with eight boxes bounded the kernel.
//   warp 4      Q tile into TMEM (tcgen05.cp), S = Q K^T into one of two buffers
//   warp 5      O += P V, P read from TMEM where S was
//   warps 8..15 softmax: two warpgroups, each with half of a block's keys; a
//               thread owns one row
//   warps 16..19 output: O of a finished unit, a row a thread, while the softmax
//               warps are at the next unit
// A row's base is its maximum over keys 0-31 and 64-95 of the unit's first block
// (a row that sees any key of the unit sees key 0 of that): the scores that P does
// not replace, so that both threads of the row read them and neither waits for the
// other.  Exponentials are taken against that base throughout, which is exact to
// the same relative error as a running maximum as long as nothing overflows: a
// unit in which a weight would exceed 2^64, or O is not finite, is
// run again with its rows' true maxima, which a pass over S alone finds first.
// Which units are is a matter of their own scores and values alone, so that a
// call's bits do not depend on which CTA took which unit.  O is never rescaled.
// P is rounded to bf16, as the tensor cores take it (2^-8 of each weight at most, in
// either direction: the output is off by 0.0023 of its size, where weights of 32 bits
// leave 0.0017, the rounding of the output); its sum is of the values before, in 32
// bits, like scores and O.  A second bf16 part of P, as the branch attention has for
// head ratios that do not divide 128 (whose calls had one before), would take P V
// twice: half as much again of the MMAs that bound long chunks.  P goes to
// the tensor cores in two parts: while the exponentials of the second 32 keys of a
// half are taken, P V of the first 32 runs.
//
// Rows that see no key are written by the scheduler.  Cache rows past a
// sequence's end may hold anything: pages past it are not loaded (their box lies
// outside the map and reads zeros), scores behind it are masked, and the rows of V
// behind it in its last page are zeroed in shared memory (a weight of zero would
// not keep out what is not finite).
// A value that is not finite in a row that some of a tile's rows see and others do
// not would reach the others as 0 times it: when a unit is run again, such values are
// taken out of the blocks (two at most) that some of its rows see part of, and added to
// the rows that see them.
// All waits are bounded, as in the branch attention kernel.
//
// What bounds it, and what it measured on a GB300 (calls one after another):
//   2,048 tokens behind 14,336, 32 / 8 heads of 128: 337-349 us, 1.48-1.53 PFLOP/s;
//     the power limit.  At the full clock 286 us, 1.80 PFLOP/s, with the tensor pipe
//     at work 87 % of the time.
//   64 sequences that bring a token, contexts to 8,191, 32 / 8 heads of 128: 203-207
//     us, 6.1 TB/s of 6.8: HBM.
//   1,152 tokens of one page, 16 / 2 heads of 128: 15.3 us, of which the blocks have
//     6: 3.4 us pass until the first scores (lengths, page ids, Q and K one after the
//     other, through code that runs for the first time), 3.5 from the last P V to
//     the end (O, its stores, the exit).
//   A unit's change takes some 2 us and a block 0.63 with heads of 128 (0.53 of it MMAs);
//     0.7 and 0.54 with heads of 64, where no pipe is full: a look at a barrier
//     takes a warp 150 to 200 cycles while the others work, and each role makes
//     two or three a block.
// 640 threads leave 96 registers each.  What does not fit (32 bytes of spill stores, 60
// of loads with heads of 128; 24 and 44 with 64) is not in the blocks' loops: 246 local
// loads an SM in a call of some 400 blocks an SM.  (With kFp8, 80 registers each: 108 bytes
// of stores and 136 of loads, 116 and 156 with heads of 64; 541 local loads an SM in the same call.)
// Halves of a block for the two softmax warpgroups, and not alternate blocks: those
// took 0.67 us a block with heads of 128 and 0.52 with heads of 64 (three buffers of
// scores, five stages).
#pragma once

#include <algorithm>
#include <atomic>
#include <cmath>
#include <type_traits>

#include "fp8.cuh"
#include "tc_common.cuh"

namespace hpd {
namespace {

using namespace sm100;
using tc::kBlk;
using tc::kRows;

constexpr uint32_t kTmemCols = 512;
constexpr int kPagesPerBlock = kBlk / kPage, kPagesEach = kPagesPerBlock / 2;  // of a producer
constexpr int kSoftmaxWarp = 8, kSoftmaxWarps = 8;
constexpr int kOutputWarp = kSoftmaxWarp + kSoftmaxWarps, kOutputWarps = 4;
constexpr int kProducers = 4;  // warps 0, 1: K; 2, 3: V
constexpr int kQkWarp = 4, kPvWarp = 5, kSchedWarp = 6;
constexpr int kScaleWarp = 7;  // 8-bit cache: the pages' scales
constexpr int kWideWarp = kOutputWarp + kOutputWarps, kWideWarps = 4;  // 8-bit cache: Q parts, V to f16
template <bool kFp8>
constexpr int kThreads = 32 * (kWideWarp + (kFp8 ? kWideWarps : 0));
// What a pass over a unit does: exponentials against the first block's maxima;
// nothing but the rows' maxima; exponentials against those.
enum Pass { kFirst, kMaxima, kAgain };
constexpr int kMetaSlots = 3, kLastUnits = 16;
// of a metadata slot: producers, two MMA issuers, softmax and output warps
template <bool kFp8>
constexpr uint32_t kMetaConsumers = kProducers + 2 + kSoftmaxWarps + kOutputWarps + (kFp8 ? 1 + kWideWarps : 0);
template <bool kFp8>
struct Rings {
  static constexpr int kStages = 3, kVStages = 3;  // of K and V
};
template <>
struct Rings<true> {
  static constexpr int kStages = 4, kVStages = 2;  // of K's codes, and of V as f16
  static constexpr int kCodeStages = 4;            // of V's codes
  static_assert(kCodeStages == kStages, "their barriers are made together");
};
constexpr int kMaxStages = 4;
constexpr int kScaleBlocks = 8;  // blocks whose scales are held
constexpr int kCopies = 4;       // of the rows of a tile of a quarter of its 128 at most
// 8-bit cache, a first pass, whose weights times their values' scales are f16: log2 of what the
// row's base has at least (2^12 times that fits; less is off by 2^-11 of it or by 2^-28 of the
// base's), and how many powers of two scales may be below the unit's where these are addends of
// the exponents (further away they would take digits from them).
constexpr float kFirstLog2 = 3.f, kFarLog2 = 14.f;
constexpr int kGroup = 256;      // sequences whose lengths the scheduler holds at once
constexpr int kMaxSplits = 32;
constexpr int kTailWaves = 4;    // most waves of the units of split tiles
constexpr int kNoUnit = (1 << 30) - 1;  // every unit's number is below
constexpr uint64_t kBlockLimitNs = 10000;  // of a unit's time: a block takes some 0.7 us

// A unit of a tile whose blocks are split: what the merge needs to know.
struct __align__(16) SlotInfo {
  int tok0, nrows, g, split, nsplit, pad[3];
};
static_assert(sizeof(SlotInfo) == 32, "read 16 bytes at a time");

struct ChunkParams {
  const __nv_bfloat16 *q;
  long long q_stride;
  const int32_t *chunk_cu, *seq_len, *full_len;
  const void *k_cache, *v_cache;     // bf16, or e4m3 codes
  const float *k_scale, *v_scale;    // of codes
  const int32_t *page_table;
  int S, T, H_q, H_kv, G, num_pages, max_pages;
  float scale_log2;
  __nv_bfloat16 *out;
  float *lse;
  uint32_t *err;
  int *unit_ctr;   // [2] next unit and finished CTAs, zero between calls
  int units;       // most units of whole tiles
  int slots;       // most units of split tiles; 0: no tile is split
  float *o_part;   // [slots][128][D]
  float *l_part;   // [slots][128]
  SlotInfo *slot;  // [slots]
  int *n_slots;    // units of split tiles
  FastDiv div_G, div_Hkv, div_tile;  // div_tile: tokens of a tile
};

// Metadata of one unit, written by the scheduler warp, read 16 bytes at a time.
struct __align__(16) UnitMeta {
  int valid;     // 0: no units left
  int n_blocks, blk_lo;
  int pass;
  int nrows;     // stacked rows
  int lim0;      // keys that the tile's first token sees by its place (a token more each)
  int full, L;   // keys that every token sees; tokens of the sequence
  int seq, g;
  int tok0;      // first row (of T) of the tile
  int pages;     // pages up to the last key that the tile sees
  int split, nsplit;
  int slot;      // where a split tile's unit leaves its result
  int copies;    // of the tile's rows among the 128: 1, or kCopies (8-bit cache, few rows)
};
__device__ __forceinline__ UnitMeta read_meta(const UnitMeta &m) {
  UnitMeta r;
#pragma unroll
  for (int i = 0; i < 4; ++i) reinterpret_cast<int4 *>(&r)[i] = reinterpret_cast<const int4 *>(&m)[i];
  return r;
}

template <int D, bool kFp8>
struct Layout {
  using R = Rings<kFp8>;
  static constexpr int kChunks = D / 64;                // 64-column (128-byte) boxes
  static constexpr uint32_t kChunkBytes = kRows * 128;  // 128 rows x 128 bytes
  static constexpr uint32_t kTileBytes = kChunks * kChunkBytes;
  // a block's pages: 8-key groups of kChunks x 1024 bytes
  static constexpr uint32_t kGroupBytes = kChunks * 1024, kPageBytes = 2 * kGroupBytes;
  static constexpr uint32_t kCodeBytes = kRows * D;              // a block's codes
  static constexpr uint32_t kKBytes = kFp8 ? kCodeBytes : kTileBytes;
  static constexpr uint32_t kK = 0;
  static constexpr uint32_t kV = kK + R::kStages * kKBytes;
  static constexpr uint32_t kCodes = kV + R::kVStages * kTileBytes;  // codes of V
  static constexpr int kCodeStages = kFp8 ? Rings<true>::kCodeStages : 0;
  static constexpr uint32_t kStage = kCodes + kCodeStages * kCodeBytes;  // 128 bytes of each output row
  static constexpr uint32_t kBytes = kStage + kRows * 128;
  static constexpr uint32_t kDynSmem = kBytes + 1024;   // slack to align to 1024
  // TMEM columns: S of block buffer i, O, Q rows of unit slot u
  static constexpr uint32_t kColO = 256;
  static __device__ __forceinline__ uint32_t col_s(int i) { return i ? 128u : 0u; }
  static __device__ __forceinline__ uint32_t col_q(int u) { return u ? 448u : 384u; }
};

struct __align__(16) Shared {
  uint64_t meta_full[kMetaSlots], meta_empty[kMetaSlots];
  uint64_t taken;  // the K producer has begun a unit
  uint64_t k_full[kMaxStages], v_full[kMaxStages], k_empty[kMaxStages], v_empty[kMaxStages];
  // per S buffer: scores written; P written, by part; P V issued
  uint64_t s_full[2], p_full[2][2], s_free[2];
  uint64_t sums[kMetaSlots];  // of the unit in the slot (softmax may be units ahead of its output)
  uint64_t o_full, o_empty;
  uint64_t mma_done[2];
  uint32_t tmem_base;
  int abort;
  // of the last units: a row's base; its sums (pass over maxima: maxima) by half
  float xbase[kMetaSlots][kRows], xsum[kMetaSlots][2][kRows];
  int max_seq[4][2];  // [quadrant][half]: units whose maxima are published
  unsigned redo;            // units (by number in this CTA, modulo kLastUnits) to run once more
  int units_done;           // output warps that looked at a unit's output
  uint32_t sieved[kMetaSlots][128];  // what sieve_block found in the unit of the slot, by column
  int sieved_seq;                    // units of which that is complete
  int unit_id[kLastUnits];  // the last units issued
  UnitMeta meta[kMetaSlots];
  // 8-bit cache: codes of V landed and widened; Q parts written and done with; a row's
  // factor of its parts; scales of a block's pages, of K and then of V, log2 of V's over the
  // largest of the unit's first block, and that over V's
  uint64_t code_full[kMaxStages], code_empty[kMaxStages], q_full[2], q_free[2];
  uint64_t copied;  // the output warps are done with a piece of the copies' sums
  float q_scale[kMetaSlots][kRows], v_ref[kMetaSlots][kRows];  // (v_ref: what O is in units of)
  float __align__(16) scales[kScaleBlocks][4 * kPagesPerBlock];
  // the scheduler's group of sequences: units before each, first rows, rows, lengths,
  // keys that all their rows see, tiles left whole, splits of the others
  uint8_t g_order[kGroup];  // (8-bit cache) sequences in the order of their units
  int g_units[kGroup], g_cu[kGroup], g_n[kGroup], g_len[kGroup], g_full[kGroup], g_whole[kGroup], g_split[kGroup];
};

__device__ __forceinline__ void set_abort(Shared &sh, uint32_t *err) {
  atomicExch(&sh.abort, 1);
  flag_error(err, HPD_DEVERR_TIMEOUT);
}
__device__ __forceinline__ bool aborted(const Shared &sh) {
  return *reinterpret_cast<const volatile int *>(&sh.abort) != 0;
}
__device__ __forceinline__ void publish_seq(int *flag, int seq) {
  __syncwarp();
  if ((threadIdx.x & 31) == 0)
    asm volatile("st.release.cta.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(flag)), "r"(seq)
                 : "memory");
}
__device__ __forceinline__ int load_seq(const int *flag) {
  int v;
  asm volatile("ld.acquire.cta.shared::cta.b32 %0, [%1];" : "=r"(v) : "r"(smem_u32(flag)) : "memory");
  return v;
}
__device__ __noinline__ bool await_seq_slow(const int *flag, int seq, const int *abort) {
  const uint64_t t0 = globaltimer();
  for (uint32_t i = 1; load_seq(flag) < seq; ++i)
    if ((i & 63u) == 0 &&
        (*reinterpret_cast<const volatile int *>(abort) || globaltimer() - t0 > kWaitLimitNs))
      return false;
  return true;
}
__device__ __forceinline__ bool await_seq(const int *flag, int seq, const Shared &sh) {
  return load_seq(flag) >= seq || await_seq_slow(flag, seq, &sh.abort);
}

// Wait until n output warps have looked at their units; false when the time is up
// or a wait elsewhere gave up.
__device__ __noinline__ bool await_outputs(Shared &sh, int n, uint64_t limit_ns, uint32_t *err) {
  const uint64_t t0 = globaltimer();
  for (uint32_t i = 1; load_seq(&sh.units_done) < n; ++i) {
    if ((i & 63u) != 0) continue;
    if (aborted(sh)) return false;
    if (globaltimer() - t0 > limit_ns) {
      set_abort(sh, err);
      return false;
    }
  }
  return true;
}

// Natural log of 2^m * l with one rounding at the result's size.
__device__ __forceinline__ float lse_of(float m, float l) {
  const int e = static_cast<int>(__float_as_uint(l) >> 23) - 127;
  const float f = __uint_as_float((__float_as_uint(l) & 0x007fffffu) | 0x3f800000u);
  return fmaf(static_cast<float>(e), kLn2, fmaf(m, kLn2, __log2f(f) * kLn2));
}

// Largest score of 32 columns at s_addr and of 32 at s_addr + apart; hi: visible
// columns, the second 32 starting at `apart`.  (Out of line, one loop: code off the
// inner loops exists once and keeps its loops, as the CTA is bound by fetching it.)
__device__ __noinline__ float row_max(uint32_t s_addr, int apart, bool plain, int hi, float sl2) {
  const float NEG_INF = -__int_as_float(0x7f800000);
  const bool raw = sl2 > 0.f;
  float mx[4] = {NEG_INF, NEG_INF, NEG_INF, NEG_INF};
#pragma unroll 1
  for (int part = 0; part < 2; ++part) {
    uint32_t v[32];
    tmem_ld32(s_addr, v);
    tmem_ld_wait32(v);
    if (!plain) tc::mask32(v, 0, hi, !raw, sl2);
#pragma unroll
    for (int c = 0; c < 32; c += 8)
#pragma unroll
      for (int a = 0; a < 4; ++a)
        mx[a] = tc::fmax3(mx[a], __uint_as_float(v[c + 2 * a]), __uint_as_float(v[c + 2 * a + 1]));
    s_addr += apart;
    hi -= apart;
  }
  return fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3])) * (raw ? sl2 : 1.f);
}

// 16 consecutive 32-bit TMEM columns of this thread's lane, and the wait for them.
__device__ __forceinline__ void tmem_ld16(uint32_t taddr, uint32_t *r) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 "
      "{%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
        "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
      : "r"(taddr));
}
__device__ __forceinline__ void tmem_ld_wait16(uint32_t *r) {
  asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
  asm volatile(""
               : "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]), "+r"(r[6]), "+r"(r[7]),
                 "+r"(r[8]), "+r"(r[9]), "+r"(r[10]), "+r"(r[11]), "+r"(r[12]), "+r"(r[13]), "+r"(r[14]),
                 "+r"(r[15])::"memory");
}

// A row's half block: P = exp2(scaled score - base) as bf16 pairs, and its sum.  P of
// the half's keys 32-63 goes to the first 16 columns of their scores, then P of keys
// 0-31 to the next 16: publish(part) once it is on its way.  (The scores of keys 0-31
// stay until the next Q K^T.)  Returns false when a score lies above the window of
// the base.  Here every row of the warp sees every key and the scale is positive (its
// order is then the raw scores').
template <class Publish>
__device__ __forceinline__ bool softmax_plain(uint32_t s_addr, float sl2, float m_run, float2 *l4, Publish publish) {
  const float NEG_INF = -__int_as_float(0x7f800000);
  float mx4[4] = {NEG_INF, NEG_INF, NEG_INF, NEG_INF};
  const float base = m_run == NEG_INF ? 0.f : m_run;
  // 16 scores at a time, the next 16 on their way
  uint32_t v[2][16], pk[16];
  const float2 mul2 = make_float2(sl2, sl2), nbase2 = make_float2(-base, -base);
  tmem_ld16(s_addr + 32, v[0]);
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    uint32_t *const x = v[q & 1];
    tmem_ld_wait16(x);
    if (q < 3) tmem_ld16(s_addr + (q == 0 ? 48 : q == 1 ? 0 : 16), v[(q & 1) ^ 1]);
#pragma unroll
    for (int c = 0; c < 16; c += 2) {
      const float2 a = make_float2(__uint_as_float(x[c]), __uint_as_float(x[c + 1]));
      const float2 arg = __ffma2_rn(a, mul2, nbase2);
      const float2 e = make_float2(fast_exp2(arg.x), fast_exp2(arg.y));
      l4[(c >> 1) & 3] = __fadd2_rn(l4[(c >> 1) & 3], e);
      pk[(q & 1) * 8 + c / 2] = pack_bf16x2(e.x, e.y);
      mx4[(c >> 1) & 3] = tc::fmax3(mx4[(c >> 1) & 3], a.x, a.y);
    }
    if (q & 1) {
      tmem_st16(s_addr + 32 + (q >> 1) * 16, pk);
      publish(q >> 1);
    }
  }
  return fmaxf(fmaxf(mx4[0], mx4[1]), fmaxf(mx4[2], mx4[3])) * sl2 <= base + tc::kWindowLog2;
}
// The same where rows see some of the keys, or the scale is not positive.  hi: visible
// columns of the half.
template <class Publish>
__device__ __forceinline__ bool softmax_masked(uint32_t s_addr, int hi, float sl2, float m_run, float2 *l4,
                                               Publish publish) {
  const float NEG_INF = -__int_as_float(0x7f800000);
  const bool raw = sl2 > 0.f;
  const float mul = raw ? sl2 : 1.f, base = m_run == NEG_INF ? 0.f : m_run;
  float mx4[4] = {NEG_INF, NEG_INF, NEG_INF, NEG_INF};
#pragma unroll 1
  for (int part = 0; part < 2; ++part) {
    uint32_t v[32];
    tmem_ld32(s_addr + 32 - 32 * part, v);
    tmem_ld_wait32(v);
    tc::mask32(v, 0, hi - 32 + 32 * part, !raw, sl2);
    tc::exp32<true, false>(s_addr + 32 + 16 * part, v, mul, base, l4, mx4);
    publish(part);
  }
  return fmaxf(fmaxf(mx4[0], mx4[1]), fmaxf(mx4[2], mx4[3])) * mul <= base + tc::kWindowLog2;
}

// Values that are not finite in a block of V that some of the tile's rows do not see all
// of: they are taken out of shared memory, as 0 times them would reach those rows too,
// and `first` keeps, for every column, the first key with NaN, +inf and -inf (10 bits
// each, keys counted from key0 = 0 at the first such block; kNoKey: none).  A lane has
// D / 32 columns, in `first` too.  v0: the block in shared memory.
constexpr uint32_t kNoKey = 1023u;
template <int D>
__device__ __noinline__ void sieve_block(uint32_t v0, int key0, uint32_t *first) {
  using L = Layout<D, false>;  // (V is in bf16 here, whatever the cache)
  constexpr int kCols = D / 32;
  const int c = (threadIdx.x & 31) * kCols;
  uint32_t seen[kCols];
#pragma unroll
  for (int i = 0; i < kCols; ++i) seen[i] = first[c + i];
#pragma unroll 1
  for (int r = 0; r < kBlk; ++r) {
    const uint32_t at = v0 + (r >> 3) * L::kGroupBytes + (c / 64) * 1024 + (r & 7) * 128 +
                        (((c % 64 / 8) ^ (r & 7)) << 4) + c % 8 * 2;
    uint32_t w[kCols / 2];
    bool any = false;
#pragma unroll
    for (int i = 0; i < kCols / 2; ++i) {
      asm volatile("ld.shared.b32 %0, [%1];" : "=r"(w[i]) : "r"(at + 4 * i) : "memory");
      any |= (w[i] & 0x7f80u) == 0x7f80u || (w[i] & 0x7f800000u) == 0x7f800000u;
    }
    if (!any) continue;
#pragma unroll
    for (int i = 0; i < kCols; ++i) {
      const uint32_t x = w[i / 2] >> (16 * (i & 1)) & 0xffffu;
      if ((x & 0x7f80u) != 0x7f80u) continue;
      const int shift = x & 0x7fu ? 0 : x & 0x8000u ? 20 : 10;
      if ((seen[i] >> shift & kNoKey) == kNoKey)
        seen[i] = (seen[i] & ~(kNoKey << shift)) | static_cast<uint32_t>(key0 + r) << shift;
      w[i / 2] &= ~(0xffffu << (16 * (i & 1)));
    }
#pragma unroll
    for (int i = 0; i < kCols / 2; ++i) asm volatile("st.shared.b32 [%0], %1;" ::"r"(at + 4 * i), "r"(w[i]) : "memory");
  }
#pragma unroll
  for (int i = 0; i < kCols; ++i) first[c + i] = seen[i];
}
// A row's sums with those values of its first `keys` keys (counted as above) added, in o_f,
// or in o_b if o_f is null.  Their weights are positive: what they are does not matter.
template <int D>
__device__ __noinline__ void add_sieved(const uint32_t *first, int keys, float *o_f, __nv_bfloat16 *o_b) {
#pragma unroll 1
  for (int c = 0; c < D; ++c) {
    const uint32_t f = first[c];
    if (f == ((kNoKey << 20) | (kNoKey << 10) | kNoKey)) continue;
    auto sees = [&](int shift) { return static_cast<int>(f >> shift & kNoKey) < keys; };
    const float inf = __int_as_float(0x7f800000);
    float add = sees(0) ? __int_as_float(0x7fffffff) : 0.f;
    if (sees(10)) add += inf;
    if (sees(20)) add -= inf;
    if (add == 0.f) continue;
    if (o_f) o_f[c] += add;
    else o_b[c] = __float2bfloat16(__bfloat162float(o_b[c]) + add);
  }
}

// The same pieces over an 8-bit cache.  A raw score is that of the query's parts with
// codes: what it is scaled by is row_mul (the softmax scale and the parts' factor) times
// the key's scale, one for the 16 keys of a page.  A weight goes to the tensor cores
// times its value's scale over the row's v_ref, rounded once; its sum is of the weight
// alone.  In a first pass that is to f16, 2^-11 of it and as V's codes widen with one
// instruction for two.  The base is lowered by as many powers of two as the scale of its own page
// is below v_ref: the products add up to 2^kFirstLog2 at least, so that what those below f16's
// normal numbers lose, 2^-25 each, is 2^-28 of the sum at most, however small the scales are.
// (Without, a row whose weight is all on pages of 2^-13 of v_ref was off by a sixth.)  What f16
// cannot hold is run again with bf16: a product that is too large becomes infinite, which the
// reader of O finds.  ks, vs: scales of the first of the pages.
//
// A row's largest score of 32 columns at s_addr and of 32 at s_addr + apart, and the scale of
// V of its page (of none: the first one's).  sc: scales of K of the first of the pages, V's behind.
__device__ __noinline__ float2 row_max_fp8(uint32_t s_addr, int apart, bool plain, int hi, float row_mul,
                                           const float *sc) {
  const float NEG_INF = -__int_as_float(0x7f800000);
  float2 best = make_float2(NEG_INF, sc[kPagesPerBlock]);
#pragma unroll 1
  for (int part = 0; part < 2; ++part) {
    uint32_t v[32];
    tmem_ld32(s_addr, v);
    tmem_ld_wait32(v);
#pragma unroll
    for (int c = 0; c < 32; ++c) v[c] = __float_as_uint(__uint_as_float(v[c]) * (row_mul * sc[c / kPage]));
    if (!plain) tc::mask32(v, 0, hi, false, 1.f);
#pragma unroll
    for (int i = 0; i < 32 / kPage; ++i) {
      float mx[2] = {NEG_INF, NEG_INF};
#pragma unroll
      for (int c = i * kPage; c < (i + 1) * kPage; c += 4)
#pragma unroll
        for (int a = 0; a < 2; ++a)
          mx[a] = tc::fmax3(mx[a], __uint_as_float(v[c + 2 * a]), __uint_as_float(v[c + 2 * a + 1]));
      const float m = fmaxf(mx[0], mx[1]);
      if (m > best.x) best = make_float2(m, sc[kPagesPerBlock + i]);
    }
    s_addr += apart;
    hi -= apart;
    sc += apart / kPage;
  }
  return best;
}
// Largest scale of V among a block's pages that have one of its first `keys` keys.
__device__ __forceinline__ float largest_scale(const float *vs, int keys) {
  float m = 0.f;
#pragma unroll
  for (int i = 0; i < kPagesPerBlock; ++i) m = i * kPage < keys ? fmaxf(m, vs[i]) : m;
  return m;
}
// The power of two at or below it (from 2^-100 to 2^126, which has a reciprocal), and that over one.
__device__ __forceinline__ float ref_of(float scale) {
  return __uint_as_float(min(max(__float_as_uint(scale), 27u << 23), 253u << 23) & 0x7f800000u);
}
__device__ __forceinline__ float over_ref(float ref) { return __uint_as_float((254u << 23) - __float_as_uint(ref)); }
// Where every row of the warp sees every key, so that v_ref is the unit's: a weight times its
// value's scale is an exponential with that scale's log2 among its addends, and what the sum
// is of has it taken out once for 16 keys.  lv, iv: log2 and reciprocals of the scales over
// v_ref, of the first of the pages (a scale of 0, whose weights count all the same, does not fit).
template <class Publish>
__device__ __forceinline__ bool softmax_plain_fp8(uint32_t s_addr, float row_mul, const float *ks, const float *lv,
                                                  const float *iv, float base, float2 *l4, Publish publish) {
  uint32_t v[2][16], pk[16];
  tmem_ld16(s_addr + 32, v[0]);
  const float4 k4 = *reinterpret_cast<const float4 *>(ks), v4 = *reinterpret_cast<const float4 *>(lv),
               i4 = *reinterpret_cast<const float4 *>(iv);
  const float kq[4] = {k4.z, k4.w, k4.x, k4.y}, vq[4] = {v4.z, v4.w, v4.x, v4.y}, iq[4] = {i4.z, i4.w, i4.x, i4.y};
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    uint32_t *const x = v[q & 1];
    tmem_ld_wait16(x);
    if (q < 3) tmem_ld16(s_addr + (q == 0 ? 48 : q == 1 ? 0 : 16), v[(q & 1) ^ 1]);
    const float mul = row_mul * kq[q], add = vq[q] - base;
    const float2 mul2 = make_float2(mul, mul), add2 = make_float2(add, add), inv2 = make_float2(iq[q], iq[q]);
    float2 sum[2];
#pragma unroll
    for (int c = 0; c < 16; c += 2) {
      const float2 arg = __ffma2_rn(make_float2(__uint_as_float(x[c]), __uint_as_float(x[c + 1])), mul2, add2);
      const float2 w = make_float2(fast_exp2(arg.x), fast_exp2(arg.y));
      sum[(c >> 1) & 1] = c < 4 ? w : __fadd2_rn(sum[(c >> 1) & 1], w);
      pk[(q & 1) * 8 + c / 2] = pack_f16x2(w.x, w.y);
    }
#pragma unroll
    for (int i = 0; i < 2; ++i) l4[(q & 1) * 2 + i] = __ffma2_rn(sum[i], inv2, l4[(q & 1) * 2 + i]);
    if (q & 1) {
      tmem_st16(s_addr + 32 + (q >> 1) * 16, pk);
      publish(q >> 1);
    }
  }
  return fminf(fminf(v4.x, v4.y), fminf(v4.z, v4.w)) >= -kFarLog2;
}
template <bool kBf16, class Publish>
__device__ __forceinline__ void softmax_masked_fp8(uint32_t s_addr, int hi, float row_mul, float val_mul,
                                                   const float *ks, const float *vs, float base, float2 *l4,
                                                   Publish publish) {
#pragma unroll 1
  for (int part = 0; part < 2; ++part) {
    uint32_t v[32], pk[16];
    tmem_ld32(s_addr + 32 - 32 * part, v);
    tmem_ld_wait32(v);
    const int p0 = 2 - 2 * part;
    const float mul[2] = {row_mul * ks[p0], row_mul * ks[p0 + 1]}, val[2] = {val_mul * vs[p0], val_mul * vs[p0 + 1]};
#pragma unroll
    for (int c = 0; c < 32; ++c) v[c] = __float_as_uint(fmaf(__uint_as_float(v[c]), mul[c / kPage], -base));
    tc::mask32(v, 0, hi - 32 + 32 * part, false, 1.f);
#pragma unroll
    for (int c = 0; c < 32; c += 2) {
      const float2 e = make_float2(fast_exp2(__uint_as_float(v[c])), fast_exp2(__uint_as_float(v[c + 1])));
      l4[(c >> 1) & 3] = __fadd2_rn(l4[(c >> 1) & 3], e);
      // (a key that the row does not see may have a page whose scale is any multiple of v_ref)
      const float2 w = make_float2(e.x == 0.f ? 0.f : e.x * val[c / kPage], e.y == 0.f ? 0.f : e.y * val[c / kPage]);
      pk[c / 2] = kBf16 ? pack_bf16x2(w.x, w.y) : pack_f16x2(w.x, w.y);
    }
    tmem_st16(s_addr + 32 + 16 * part, pk);
    publish(part);
  }
}

// The same of a row that the tile has kCopies times: a copy takes one of the half's pages
// and leaves weights of 0 for the others.  (A thread's 64 columns bound the blocks of tiles
// of few rows, where most softmax threads had no row.)
template <class Publish>
__device__ __forceinline__ void softmax_share_fp8(uint32_t s_addr, int copy, int hi, float row_mul, float val_mul,
                                                  const float *ks, const float *vs, float base, float2 *l4,
                                                  Publish publish) {
  static_assert(kCopies * kPage == kBlk / 2, "a page each");
  const float NEG_INF = -__int_as_float(0x7f800000);
  uint32_t v[16], pk[8];
  tmem_ld16(s_addr + copy * kPage, v);
  const float mul = row_mul * ks[copy], val = val_mul * vs[copy];
  const int seen = hi - copy * kPage;
  const float2 mul2 = make_float2(mul, mul), nbase2 = make_float2(-base, -base);
  tmem_ld_wait16(v);
#pragma unroll
  for (int c = 0; c < kPage; c += 2) {
    const float2 arg = __ffma2_rn(make_float2(__uint_as_float(v[c]), __uint_as_float(v[c + 1])), mul2, nbase2);
    const float2 e = make_float2(fast_exp2(c < seen ? arg.x : NEG_INF), fast_exp2(c + 1 < seen ? arg.y : NEG_INF));
    l4[(c >> 1) & 3] = __fadd2_rn(l4[(c >> 1) & 3], e);
    // (a key that the row does not see may have a page whose scale is any multiple of v_ref)
    pk[c / 2] = pack_f16x2(e.x == 0.f ? 0.f : e.x * val, e.y == 0.f ? 0.f : e.y * val);
  }
#pragma unroll
  for (int i = 0; i < kCopies; ++i) {  // pages 2, 3, 0, 1
    if ((i ^ 2) == copy) {
      tmem_st8(s_addr + 32 + 8 * i, pk);
    } else {
      const uint32_t zero[8] = {0u, 0u, 0u, 0u, 0u, 0u, 0u, 0u};
      tmem_st8(s_addr + 32 + 8 * i, zero);
    }
  }
  publish();
}

// Rows row0 to row0 + rows - 1 (32 at most) of a tile's queries in two e4m3 parts, one
// behind the other, in TMEM at q_addr: q 2^t = q1 + q2 with the row's largest value from 2^7
// to 2^8.  q1 has four of bf16's eight bits, and what is left of them fits into q2, but for
// values below 2^-9 of the largest, which keep 2^-17 of that.  factor: 2^-t of each row; NaN
// for one with a value that is not finite.  Four lanes have a row, eight of each 32 columns
// a lane, so that it is loaded once, in pieces of 64 bytes.
template <int D>
__device__ __forceinline__ void part_rows(const __nv_bfloat16 *q, long long q_stride, int G, FastDiv div_G, int row0,
                                          int rows, uint32_t q_addr, float *factor) {
  const int lane = threadIdx.x & 31;
#pragma unroll(D == 64 ? 2 : 1)  // (with 128 columns the 80 registers hold 16 rows' pieces)
  for (int r0 = lane >> 2; r0 - (lane >> 2) < rows; r0 += 16, q_addr += 16u << 16) {
    uint4 x[2][D / 32];  // of rows r0 and r0 + 8
    float up[2];
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const int row = row0 + r0 + 8 * e, t = div_G(row);
      const uint4 *const src = reinterpret_cast<const uint4 *>(q + t * q_stride + (row - t * G) * D) + (lane & 3);
#pragma unroll
      for (int g = 0; g < D / 32; ++g) x[e][g] = r0 + 8 * e < rows ? src[4 * g] : make_uint4(0u, 0u, 0u, 0u);
    }
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      unsigned most = 0u;
#pragma unroll
      for (int g = 0; g < D / 32; ++g)
        most = __vmaxu2(__vmaxu2(most, __vmaxu2(x[e][g].x & 0x7fff7fffu, x[e][g].y & 0x7fff7fffu)),
                        __vmaxu2(x[e][g].z & 0x7fff7fffu, x[e][g].w & 0x7fff7fffu));
      most = __vmaxu2(most, __shfl_xor_sync(0xffffffffu, most, 1));
      most = __vmaxu2(most, __shfl_xor_sync(0xffffffffu, most, 2));
      most = max(most & 0xffffu, most >> 16);
      const int t = min(134 - static_cast<int>(most >> 7), 126);
      up[e] = __uint_as_float(static_cast<uint32_t>(127 + t) << 23);
      if ((lane & 3) == 0 && r0 + 8 * e < rows)
        factor[r0 + 8 * e] =
            most >= 0x7f80u ? __int_as_float(0x7fffffff) : __uint_as_float(static_cast<uint32_t>(127 - t) << 23);
    }
#pragma unroll
    for (int g = 0; g < D / 32; ++g) {
      uint32_t c1[4], c2[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int e = i >> 1;
        const uint32_t a = i & 1 ? x[e][g].z : x[e][g].x, b = i & 1 ? x[e][g].w : x[e][g].y;
        const float q0 = __uint_as_float(a << 16) * up[e], q1 = __uint_as_float(a & 0xffff0000u) * up[e];
        const float q2 = __uint_as_float(b << 16) * up[e], q3 = __uint_as_float(b & 0xffff0000u) * up[e];
        c1[i] = to_codes4(q0, q1, q2, q3);
        float2 f, h;
        of_codes4(c1[i], f, h);
        c2[i] = to_codes4(q0 - f.x, q1 - f.y, q2 - h.x, q3 - h.y);
      }
      tmem_st_rows(q_addr + 8 * g, c1);
      tmem_st_rows(q_addr + D / 4 + 8 * g, c2);
    }
  }
  tmem_st_wait();
}

// 32 keys' codes at `from` as bf16 at `to`, both as the blocks hold them (of a unit that is
// run again; out of line, as what is not in the blocks' loops is).
template <int D>
__device__ __noinline__ void widen_again(uint32_t from, uint32_t to) {
  using L = Layout<D, true>;
  const int lane = threadIdx.x & 31, r = lane & 7, c0 = lane >> 3;
#pragma unroll 1
  for (int i = 0; i < D / 16; ++i) {
    const int group = D == 128 ? i >> 1 : i, h = D == 128 ? i & 1 : 0;
    uint32_t x[4], y[8];
    asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];"
                 : "=r"(x[0]), "=r"(x[1]), "=r"(x[2]), "=r"(x[3])
                 : "r"(from + (group * 8 + r) * D + ((D == 128 ? (c0 + 4 * h) ^ r : c0 ^ (r >> 1 & 3)) << 4)));
#pragma unroll
    for (int n = 0; n < 4; ++n) f16_of_codes(x[n], y[2 * n], y[2 * n + 1]);
#pragma unroll
    for (int n = 0; n < 8; ++n) y[n] = bf16_of_f16(y[n]);
#pragma unroll
    for (int n = 0; n < 2; ++n)
      asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(to + group * L::kGroupBytes + h * 1024 + r * 128 +
                                                                   (((c0 * 2 + n) ^ r) << 4)),
                   "r"(y[4 * n]), "r"(y[4 * n + 1]), "r"(y[4 * n + 2]), "r"(y[4 * n + 3])
                   : "memory");
  }
}

template <int D, bool kFp8>
__global__ void __launch_bounds__(kThreads<kFp8>, 1)
    chunk_attn_kernel(const __grid_constant__ CUtensorMap tm_k, const __grid_constant__ CUtensorMap tm_k4,
                      const __grid_constant__ CUtensorMap tm_v, const __grid_constant__ CUtensorMap tm_v4,
                      const __grid_constant__ CUtensorMap tm_q, const ChunkParams p) {
  using L = Layout<D, kFp8>;
  constexpr int kStages = Rings<kFp8>::kStages, kVStages = Rings<kFp8>::kVStages;
  extern __shared__ uint8_t smem_raw[];
  __shared__ Shared sh;
  const uint32_t sbase = (smem_u32(smem_raw) + 1023u) & ~1023u;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int G = p.G;
  const int TT = kRows / G;  // tokens of a tile
  const float NEG_INF = -__int_as_float(0x7f800000);
  auto bar = [](uint64_t &b) { return smem_u32(&b); };
  auto wait_bar = [&](uint64_t &b, int parity) {
    // (one look by the whole warp, then a branch that is the warp's: a branch lane by
    // lane had 2 to 6 % of the kernel's time)
    return __all_sync(0xffffffffu, mbar_try_wait(bar(b), parity)) ||
           __all_sync(0xffffffffu, mbar_wait_slow(bar(b), parity, &sh.abort, kWaitLimitNs));
  };

  if (tid == 0) {
    sh.abort = 0;
    sh.redo = 0u;
    sh.units_done = 0;
    sh.sieved_seq = 0;
  }
  if constexpr (!kFp8) {
    if (tid == 0) {
      for (int s = 0; s < kStages; ++s) {
        mbar_init(bar(sh.k_full[s]), 2);
        mbar_init(bar(sh.v_full[s]), 2);
        mbar_init(bar(sh.k_empty[s]), 1);
        mbar_init(bar(sh.v_empty[s]), 1);
      }
      for (int s = 0; s < kMetaSlots; ++s) {
        mbar_init(bar(sh.meta_full[s]), 1);
        mbar_init(bar(sh.meta_empty[s]), kMetaConsumers<kFp8>);
        mbar_init(bar(sh.sums[s]), kSoftmaxWarps);
      }
      for (int s = 0; s < 2; ++s) {
        mbar_init(bar(sh.s_full[s]), 1);
        mbar_init(bar(sh.p_full[s][0]), kSoftmaxWarps);
        mbar_init(bar(sh.p_full[s][1]), kSoftmaxWarps);
        mbar_init(bar(sh.s_free[s]), 1);
      }
      mbar_init(bar(sh.taken), 1);
      mbar_init(bar(sh.o_full), 1);
      mbar_init(bar(sh.o_empty), kOutputWarps);
      mbar_init(bar(sh.mma_done[0]), 1);
      mbar_init(bar(sh.mma_done[1]), 1);
      fence_mbar_init();
    }
  } else if (tid < 32) {  // (a lane each: there are twice as many)
    const int s = tid;
    if (s < kStages) {
      mbar_init(bar(sh.k_full[s]), 3);
      mbar_init(bar(sh.k_empty[s]), 1);
      mbar_init(bar(sh.code_full[s]), 2);
      mbar_init(bar(sh.code_empty[s]), kWideWarps);
    }
    if (s < kVStages) {
      mbar_init(bar(sh.v_full[s]), kWideWarps);
      mbar_init(bar(sh.v_empty[s]), 1);
    }
    if (s < kMetaSlots) {
      mbar_init(bar(sh.meta_full[s]), 1);
      mbar_init(bar(sh.meta_empty[s]), kMetaConsumers<kFp8>);
      mbar_init(bar(sh.sums[s]), kSoftmaxWarps);
    }
    if (s < 2) {
      mbar_init(bar(sh.s_full[s]), 1);
      mbar_init(bar(sh.p_full[s][0]), kSoftmaxWarps);
      mbar_init(bar(sh.p_full[s][1]), kSoftmaxWarps);
      mbar_init(bar(sh.s_free[s]), 1);
      mbar_init(bar(sh.q_full[s]), kWideWarps);
      mbar_init(bar(sh.q_free[s]), 1);
      mbar_init(bar(sh.mma_done[s]), 1);
    }
    if (s == 0) {
      mbar_init(bar(sh.taken), 1);
      mbar_init(bar(sh.o_full), 1);
      mbar_init(bar(sh.o_empty), kOutputWarps);
      mbar_init(bar(sh.copied), kOutputWarps);
    }
    fence_mbar_init();
  }
  if (tid < 8) (&sh.max_seq[0][0])[tid] = 0;
  if (warp == kQkWarp) {
    tmem_alloc(smem_u32(&sh.tmem_base), kTmemCols);
    tmem_relinquish();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = sh.tmem_base;
  // (each role waits for the kernels before where it starts, with its first code fetched)

  if (warp == kSchedWarp) {
    // ------------------------------------------------------- scheduler --
    // Units are numbered sequence by sequence, in each its tiles from the last
    // (longest) to the first, in each its splits and then its KV heads.
    int g0 = -kGroup, before = 0, group_units = 0;  // the group held, units before it and of it
    int first_slot = kNoUnit;                       // the first unit of the tiles that may be split
    // What a lane loads of a sequence, from the start on its way for its first one.
    int a0 = 0, a1 = 0, len = 0, full = 0;
    auto fetch = [&](int i) {
      if (i >= p.S) return;
      a0 = p.chunk_cu[i];
      a1 = p.chunk_cu[i + 1];
      len = p.seq_len[i];
      if (p.full_len) full = p.full_len[i];
    };
    pdl_wait();     // queries, cache, tables and lengths as the kernels before leave them
    pdl_trigger();  // the merge of the splits may launch; it waits for this grid
    int fetched = 0;  // group whose first lengths are on their way
    fetch(lane);
    bool sorted = false;
    auto seq_at = [&](int i) { return kFp8 && sorted ? sh.g_order[i] : i; };
    // A group of no more than 64 sequences, kPer to a lane (lane + 32 u of them): what
    // load_group does, in registers (the first unit of 64 is known 4 us earlier, of 24 two).
    auto load_few = [&](auto per_lane) {
      constexpr int kPer = decltype(per_lane)::value;
      const int count = p.S, grid = static_cast<int>(gridDim.x);
      g0 = before = 0;
      int n[kPer], blocks[kPer];  // tiles; blocks of one
#pragma unroll
      for (int u = 0; u < kPer; ++u) {
        const int i = lane + 32 * u;
        if (u > 0) fetch(i);
        const int c0 = min(max(a0, 0), p.T), c1 = max(c0, min(a1, p.T)), Ls = min(max(len, 0), p.max_pages * kPage);
        if (i < count) {
          if (a0 != c0 || a1 != c1) flag_error(p.err, HPD_DEVERR_BRANCH_CU);
          if (Ls != len) flag_error(p.err, HPD_DEVERR_BRANCH_LEN);
          sh.g_cu[i] = c0;
          sh.g_n[i] = c1 - c0;
          sh.g_len[i] = Ls;
          sh.g_full[i] = min(max(full, 0), Ls);
        }
        n[u] = i < count ? p.div_tile(c1 - c0 + TT - 1) : 0;
        blocks[u] = ceil_div_i(Ls, kBlk);
      }
      auto sum_of = [&](auto f) {
        unsigned x = f(0);
        if (kPer > 1) x += f(kPer - 1);
        return __reduce_add_sync(0xffffffffu, x);
      };
      const unsigned most_tiles = sum_of([&](int u) { return static_cast<unsigned>(n[u]); });
      // (offsets out of order can make more tiles than there are rows for)
      const bool in_order = static_cast<long long>(most_tiles) * p.H_kv <= p.units;
      const int all = in_order ? static_cast<int>(most_tiles) * p.H_kv : kNoUnit;
      sorted = in_order && all > grid;
      if (sorted) {  // the longest first: a bitonic sort of lengths in blocks, with the sequences' numbers
        unsigned key[kPer];
#pragma unroll
        for (int u = 0; u < kPer; ++u)
          key[u] = lane + 32 * u < count ? static_cast<unsigned>(blocks[u] + 1) << 6 | (63 - lane - 32 * u) : 0u;
#pragma unroll 1
        for (int size = 2; size <= 32 * kPer; size *= 2)
#pragma unroll 1
          for (int apart = size / 2; apart > 0; apart /= 2) {
            if (kPer > 1 && apart == 32) {
              const unsigned a = key[0], b = key[kPer - 1];
              key[0] = max(a, b);
              key[kPer - 1] = min(a, b);
              continue;
            }
#pragma unroll
            for (int u = 0; u < kPer; ++u) {
              const unsigned other = __shfl_xor_sync(0xffffffffu, key[u], apart);
              const bool larger = !(lane & apart) == !((lane + 32 * u) & size);
              key[u] = larger ? max(key[u], other) : min(key[u], other);
            }
          }
        __syncwarp();
#pragma unroll
        for (int u = 0; u < kPer; ++u) {
          n[u] = blocks[u] = 0;
          if (lane + 32 * u < count) {
            const int seq = 63 - static_cast<int>(key[u] & 63u);
            sh.g_order[lane + 32 * u] = static_cast<uint8_t>(seq);
            n[u] = p.div_tile(sh.g_n[seq] + TT - 1);
            blocks[u] = static_cast<int>(key[u] >> 6) - 1;
          }
        }
      }
      auto scan = [&](const int *x, int *prior) {  // sums of those before (that stop at kNoUnit); of all
        int sum = 0;
#pragma unroll
        for (int u = 0; u < kPer; ++u) {
          int incl = x[u];
#pragma unroll
          for (int o = 1; o < 32; o <<= 1) {
            const int v = __shfl_up_sync(0xffffffffu, incl, o);
            if (lane >= o) incl = min(incl + v, kNoUnit);
          }
          const int v = __shfl_up_sync(0xffffffffu, incl, 1);
          prior[u] = min(sum + (lane ? v : 0), kNoUnit);
          sum = min(sum + __shfl_sync(0xffffffffu, incl, 31), kNoUnit);
        }
        return sum;
      };
      const bool may_split = p.slots > 0 && in_order;
      int whole = kNoUnit, w[kPer], splits[kPer], first[kPer], units[kPer];
#pragma unroll
      for (int u = 0; u < kPer; ++u) {
        w[u] = n[u];
        splits[u] = 1;
      }
      if (may_split) {
        whole = p.div_Hkv(all / grid * grid);
        scan(n, first);
#pragma unroll
        for (int u = 0; u < kPer; ++u) w[u] = max(min(whole - first[u], n[u]), 0);
        const float left = static_cast<float>(
            sum_of([&](int u) { return min(static_cast<unsigned>(n[u] - w[u]) * static_cast<unsigned>(blocks[u]), 1u << 25); }));
        const float rest = static_cast<float>(all - whole * p.H_kv), total = left * p.H_kv;
        const float mean = rest > 0.f ? __fdividef(total, rest) : 0.f;
        const int waves = (lane & (kTailWaves - 1)) + 1;  // a lane tries one
        const int share = max(2, static_cast<int>(ceilf(__fdividef(total, grid * waves))));
        const float f = fmaxf(floorf(__fdividef(mean, share)), 1.f);
        const float cost = ceilf(__fdividef(rest * f, grid)) * (ceilf(__fdividef(mean, f)) + 3.5f);
        const unsigned least = __reduce_min_sync(0xffffffffu, __float_as_uint(cost));
        const int per = __shfl_sync(0xffffffffu, share, __ffs(__ballot_sync(0xffffffffu, __float_as_uint(cost) == least)) - 1);
#pragma unroll
        for (int u = 0; u < kPer; ++u)
          if (n[u] > w[u]) splits[u] = min(max(blocks[u] / per, 1), kMaxSplits);
      }
#pragma unroll
      for (int u = 0; u < kPer; ++u) units[u] = min((w[u] + (n[u] - w[u]) * splits[u]) * p.H_kv, kNoUnit);
      int sum = scan(units, first);
      if (may_split && sum - whole * p.H_kv > p.slots) {  // more than there is room for: nothing is split
#pragma unroll
        for (int u = 0; u < kPer; ++u) {
          splits[u] = 1;
          units[u] = n[u] * p.H_kv;
        }
        sum = scan(units, first);
      }
#pragma unroll
      for (int u = 0; u < kPer; ++u)
        if (lane + 32 * u < count) {
          sh.g_units[lane + 32 * u] = first[u];
          sh.g_split[lane + 32 * u] = splits[u];
          sh.g_whole[lane + 32 * u] = w[u];
        }
      first_slot = may_split ? whole * p.H_kv : kNoUnit;
      if (p.slots > 0 && blockIdx.x == 0 && lane == 0) *p.n_slots = max(sum - first_slot, 0);
      group_units = sum;
      __syncwarp();
    };
    auto load_group = [&](int s0, int units_before) {
      g0 = s0;
      before = units_before;
      const int count = min(kGroup, p.S - s0);
      if constexpr (kFp8) {
        if (p.S <= 64) {
          if (p.S <= 32) load_few(std::integral_constant<int, 1>{});
          else load_few(std::integral_constant<int, 2>{});
          return;
        }
      }
      // (loops left as loops, a step's loads ahead: code that runs once is bound by
      // fetching it)
      if (fetched != s0) fetch(s0 + lane);
      fetched = -1;
#pragma unroll 1
      for (int i = lane; i - lane < count; i += 32) {
        const int b0 = a0, b1 = a1, b_len = len, b_full = full;
        if (i + 32 < count) fetch(s0 + i + 32);
        if (i >= count) continue;
        const int c0 = min(max(b0, 0), p.T), c1 = max(c0, min(b1, p.T)), Ls = min(max(b_len, 0), p.max_pages * kPage);
        if (b0 != c0 || b1 != c1) flag_error(p.err, HPD_DEVERR_BRANCH_CU);
        if (Ls != b_len) flag_error(p.err, HPD_DEVERR_BRANCH_LEN);
        sh.g_cu[i] = c0;
        sh.g_n[i] = c1 - c0;
        sh.g_len[i] = Ls;
        sh.g_full[i] = min(max(b_full, 0), Ls);
      }
      if constexpr (kFp8) {
        // Longest sequences first, by eighths of the longest, where there is more than a unit
        // an SM: a long one begun late has the others wait.
        sorted = p.units - p.slots > static_cast<int>(gridDim.x);
        if (sorted) {
          __syncwarp();
          int most = 0;
#pragma unroll 1
          for (int i = lane; i < count; i += 32) most = max(most, sh.g_len[i]);
          const float eighths = 8.f / (__reduce_max_sync(0xffffffffu, most) + 1);
          int placed = 0;
#pragma unroll 1
          for (int c = 7; c >= 0; --c) {
#pragma unroll 1
            for (int i = lane; i - lane < count; i += 32) {
              const bool here = i < count && min(static_cast<int>(sh.g_len[i] * eighths), 7) == c;
              const unsigned all = __ballot_sync(0xffffffffu, here);
              if (here) sh.g_order[placed + __popc(all & ((1u << lane) - 1u))] = static_cast<uint8_t>(i);
              placed += __popc(all);
            }
          }
          __syncwarp();
        }
      }
      // (sums that stop at kNoUnit, which offsets out of order could pass)
      auto add = [](int a, int b) { return min(a + b, kNoUnit); };
      // exclusive prefix of x over the lanes, from base, which it adds their sum to
      auto scan = [&](int x, int &base) {
        int incl = x;
#pragma unroll 1
        for (int o = 1; o < 32; o <<= 1) {
          const int v = __shfl_up_sync(0xffffffffu, incl, o);
          if (lane >= o) incl = add(incl, v);
        }
        const int prior = __shfl_up_sync(0xffffffffu, incl, 1), r = add(base, lane ? prior : 0);
        base = add(base, __shfl_sync(0xffffffffu, incl, 31));
        return r;
      };
      auto tiles_of = [&](int i) { return i < count ? p.div_tile(sh.g_n[seq_at(i)] + TT - 1) : 0; };
      int whole = kNoUnit, per = 1 << 30;  // tiles left whole; blocks of a split of the others
      int tiles = 0;
      if (p.slots > 0) {
#pragma unroll 1
        for (int i = lane; i - lane < count; i += 32) {
          const int prior = scan(tiles_of(i), tiles);
          if (i < count) sh.g_whole[i] = prior;
        }
      }
      // (offsets out of order can make more tiles than there are rows for)
      const bool may_split = p.slots > 0 && static_cast<long long>(tiles) * p.H_kv <= p.units;
      // of a sequence with n tiles, those that stay whole
      auto whole_of = [&](int i, int n) { return may_split ? max(min(whole - sh.g_whole[i], n), 0) : n; };
      if (may_split) {
        // (one group) The tiles of full waves stay whole; what is left over after them
        // is split, into as many even waves as take the least time: a unit's start and
        // end are worth some 3.5 blocks.
        whole = p.div_Hkv(tiles * p.H_kv / static_cast<int>(gridDim.x) * static_cast<int>(gridDim.x));
        float blocks = 0.f;  // of the others, all heads
#pragma unroll 1
        for (int i = lane; i < count; i += 32) {
          const int n = tiles_of(i);
          blocks += static_cast<float>(n - whole_of(i, n)) * ceil_div_i(sh.g_len[seq_at(i)], kBlk) * p.H_kv;
        }
        __syncwarp();
#pragma unroll 1
        for (int o = 16; o > 0; o >>= 1) blocks += __shfl_xor_sync(0xffffffffu, blocks, o);
        const float units = static_cast<float>(tiles - whole) * p.H_kv, mean = units > 0.f ? blocks / units : 0.f;
        const int waves = (lane & (kTailWaves - 1)) + 1;  // a lane tries one
        const int share = max(2, static_cast<int>(ceilf(blocks / (gridDim.x * waves))));
        const float f = fmaxf(floorf(mean / share), 1.f);
        const float cost = ceilf(units * f / gridDim.x) * (ceilf(mean / f) + 3.5f);
        // (costs are positive: their order is their bits')
        const unsigned least = __reduce_min_sync(0xffffffffu, __float_as_uint(cost));
        per = __shfl_sync(0xffffffffu, share, __ffs(__ballot_sync(0xffffffffu, __float_as_uint(cost) == least)) - 1);
      }
      int units = 0;
#pragma unroll 1
      for (int pass = 0; pass < 2; ++pass) {
        units = 0;
#pragma unroll 1
        for (int i = lane; i - lane < count; i += 32) {
          const int n = tiles_of(i), w = i < count ? whole_of(i, n) : 0;
          const int f = n > w ? min(max(ceil_div_i(sh.g_len[seq_at(i)], kBlk) / per, 1), kMaxSplits) : 1;
          const int first = scan(min((w + (n - w) * f) * p.H_kv, kNoUnit), units);
          if (i < count) {
            sh.g_units[i] = first;
            sh.g_split[i] = f;
          }
        }
        if (!may_split || units - whole * p.H_kv <= p.slots) break;
        per = 1 << 30;  // more than there is room for: nothing is split
      }
#pragma unroll 1
      for (int i = lane; i < count; i += 32) sh.g_whole[i] = whole_of(i, tiles_of(i));
      __syncwarp();
      const int base = units;
      first_slot = may_split ? whole * p.H_kv : kNoUnit;
      if (p.slots > 0 && blockIdx.x == 0 && lane == 0) *p.n_slots = max(units - first_slot, 0);
      group_units = base;
      __syncwarp();
    };
    unsigned redo = 0;  // units to run again
    int again = -1;     // the unit whose maxima the last pass took
    int outputs = 0;    // passes that write a unit's output
    bool asked = false;
    int nb_last = 0, nb_before = 0;
    auto take_redo = [&] {
      unsigned r = 0;
      if (lane == 0 && *static_cast<volatile unsigned *>(&sh.redo)) r = atomicExch(&sh.redo, 0u);
      return __shfl_sync(0xffffffffu, r, 0);
    };
    // The unit's place in the group held (moved there); false: no such unit.
    auto locate = [&](int u) {
      if (u < before) {
        g0 = -kGroup;
        before = group_units = 0;
      }
      while (u - before >= group_units) {
        if (g0 + kGroup >= p.S) return false;
        load_group(g0 + kGroup, min(before + group_units, kNoUnit));
      }
      return u < kNoUnit;
    };
    for (int k = 0;; ++k) {
      const int slot = k % kMetaSlots;
      // a unit is taken when the K producer begins the one before: no earlier, as
      // another CTA may come to it sooner
      if ((k >= kMetaSlots && !wait_bar(sh.meta_empty[slot], (k / kMetaSlots - 1) & 1)) ||
          (k >= 1 && !wait_bar(sh.taken, (k - 1) & 1))) {
        if (lane == 0) set_abort(sh, p.err);
        break;
      }
      UnitMeta &M = sh.meta[slot];
      bool have = false;
      for (;;) {
        int u = again, pass = kAgain;
        if (!redo) redo = take_redo();
        if (again >= 0) {
          again = -1;
        } else if (redo) {
          u = again = sh.unit_id[__ffs(redo) - 1];
          pass = kMaxima;
          redo &= redo - 1;
        } else {
          pass = kFirst;
          u = blockIdx.x;  // the first one asked for; then whatever is next
          if (asked) {
            if (lane == 0) u = gridDim.x + atomicAdd(p.unit_ctr, 1);
            u = __shfl_sync(0xffffffffu, u, 0);
          }
          asked = true;
          if (__any_sync(0xffffffffu, aborted(sh))) break;
        }
        if (!locate(u)) {
          // none left, once the units still running (the last two) need not be run
          // again; who gives up here sets the abort word and the error
          const uint64_t limit = kWaitLimitNs + (static_cast<uint64_t>(nb_last) + nb_before) * kBlockLimitNs;
          if (!__all_sync(0xffffffffu, await_outputs(sh, kOutputWarps * outputs, limit, p.err))) break;
          redo = take_redo();
          if (!redo) break;
          continue;
        }
        int lo = 0, hi = min(kGroup, p.S - g0);  // the last sequence that starts at or before the unit
        while (hi - lo > 1) {
          const int mid = (lo + hi) >> 1;
          if (sh.g_units[mid] <= u - before) lo = mid; else hi = mid;
        }
        const int seq = seq_at(lo);
        const int c0 = sh.g_cu[seq], n = sh.g_n[seq], len = sh.g_len[seq], full = sh.g_full[seq];
        const int w = sh.g_whole[lo], f = sh.g_split[lo];
        const int idx = u - before - sh.g_units[lo], us = p.div_Hkv(idx), g = idx - us * p.H_kv;
        const int nsplit = us < w ? 1 : f, ut = us < w || f == 1 ? us : w + (us - w) / f;
        const int split = nsplit == 1 ? 0 : (us - w) - (ut - w) * f;
        const int tile = p.div_tile(n + TT - 1) - 1 - ut;
        const int i0 = tile * TT, ntok = min(TT, n - i0), nrows = ntok * G;
        const int lim0 = len - n + i0 + 1;
        const int kmax = min(max(max(lim0 + ntok - 1, full), 0), len);
        const int N = ceil_div_i(kmax, kBlk);
        // (N below 2^23, at most 32 splits)
        const int blk_lo = nsplit > 1 ? split * N / nsplit : 0, blk_hi = nsplit > 1 ? (split + 1) * N / nsplit : N;
        const int slot_id = u - first_slot;  // of the units of tiles that may be split
        if (slot_id >= 0 && lane == 0) p.slot[slot_id] = SlotInfo{c0 + i0, nrows, g, split, nsplit, {0, 0, 0}};
        if (blk_hi <= blk_lo) {
          // no key: zero output, or an empty partial
#pragma unroll 1
          for (int r = lane; r < nrows; r += 32) {
            const int rt = p.div_G(r);
            const size_t pair = static_cast<size_t>(c0 + i0 + rt) * p.H_q + g * G + r - rt * G;
            if (nsplit == 1) {
              uint4 *o = reinterpret_cast<uint4 *>(p.out + pair * D);
#pragma unroll 1
              for (int c = 0; c < D / 8; ++c) o[c] = make_uint4(0u, 0u, 0u, 0u);
              if (p.lse) p.lse[pair] = NEG_INF;
            } else {
              p.l_part[static_cast<size_t>(slot_id) * kRows + r] = NEG_INF;
            }
          }
          continue;
        }
        if (lane == 0) {
          M.valid = 1;
          M.g = g;
          M.split = split;
          M.nsplit = nsplit;
          M.slot = slot_id;
          M.seq = g0 + seq;
          M.tok0 = c0 + i0;
          M.nrows = nrows;
          M.lim0 = lim0;
          M.full = full;
          M.L = len;
          M.pages = ceil_div_i(kmax, kPage);
          M.blk_lo = blk_lo;
          M.n_blocks = blk_hi - blk_lo;
          M.pass = pass;
          M.copies = kFp8 && pass == kFirst && nrows <= kRows / kCopies ? kCopies : 1;
          sh.unit_id[k & (kLastUnits - 1)] = u;
        }
        nb_before = nb_last;
        nb_last = blk_hi - blk_lo;
        outputs += pass != kMaxima;
        have = true;
        break;
      }
      if (lane == 0) {  // (the arrival releases this lane's writes)
        if (!have) M.valid = 0;
        mbar_arrive(bar(sh.meta_full[slot]));
      }
      if (!have) break;
    }
  } else if (warp < kProducers) {
    // ------------------------------------------------------- producers --
    const bool is_k = warp < 2;
    const int half = warp & 1;
    if (lane == 0) {
      if (!kFp8) prefetch_tmap(&tm_q);
      prefetch_tmap(is_k ? &tm_k : &tm_v);
      prefetch_tmap(is_k ? &tm_k4 : &tm_v4);
    }
    __syncwarp();
    pdl_wait();
    uint64_t *const full = is_k ? sh.k_full : kFp8 ? sh.code_full : sh.v_full;
    uint64_t *const empty = is_k ? sh.k_empty : kFp8 ? sh.code_empty : sh.v_empty;
    const CUtensorMap *const page_map = is_k ? &tm_k : &tm_v, *const run_map = is_k ? &tm_k4 : &tm_v4;
    const uint32_t ring = sbase + (is_k ? L::kK : kFp8 ? L::kCodes : L::kV), mine = half * (L::kKBytes / 2);
    int issued = 0;  // ring entries
    bool ok = true;
    for (int k = 0; ok; ++k) {
      const int slot = k % kMetaSlots;
      if (!(ok = wait_bar(sh.meta_full[slot], (k / kMetaSlots) & 1))) break;
      const UnitMeta M = read_meta(sh.meta[slot]);
      __syncwarp();
      if (!M.valid) break;
      if (lane == 0) {
        mbar_arrive(bar(sh.meta_empty[slot]));
        if (warp == 0) mbar_arrive(bar(sh.taken));
      }
      if (!is_k && M.pass == kMaxima) continue;
      const int32_t *const row = p.page_table + static_cast<size_t>(M.seq) * p.max_pages;
      // Ids of this warp's pages of eight blocks at once, looked up eight blocks
      // ahead of their use (a look-up a block, one ahead, had the producers wait for
      // it: some 700 cycles a block); pages past the last one that the tile sees lie
      // outside the map, whose boxes read zeros.
      constexpr int kIdBlocks = 32 / kPagesEach;
      const int page0 = M.blk_lo * kPagesPerBlock + (lane / kPagesEach) * kPagesPerBlock + half * kPagesEach +
                        lane % kPagesEach;
      int ids = p.num_pages, ids_next = p.num_pages;
      auto look_up = [&](int j) {
        const int i = page0 + j * kPagesPerBlock;
        ids_next = p.num_pages;
        // (a coherent load: the kernel before may write the table while this one starts)
        if (i < M.pages) ids_next = row[i];
      };
      look_up(0);
#pragma unroll 1
      for (int j = is_k && !kFp8 ? -1 : 0; j < M.n_blocks; ++j) {
        const int e = issued, s = e % kStages;
        if (e >= kStages && !(ok = wait_bar(empty[s], ((e / kStages) - 1) & 1))) break;
        ++issued;
        const uint32_t dst = ring + s * L::kKBytes, b = bar(full[s]);
        if (!kFp8 && j < 0) {  // the unit's Q tile, 64 columns a warp
          if (half < L::kChunks) {
            mbar_arrive_expect_tx_elect(b, TT * G * 128);
            tma_load_3d_elect(dst + half * L::kChunkBytes, &tm_q, b, half * 64, M.g * G, M.tok0);
          } else if (lane == 0) {
            mbar_arrive(b);
          }
          __syncwarp();
          continue;
        }
        if (j % kIdBlocks == 0) {
          ids = ids_next;
          if (page0 + j * kPagesPerBlock < M.pages && static_cast<unsigned>(ids) >= static_cast<unsigned>(p.num_pages)) {
            flag_error(p.err, HPD_DEVERR_PAGE_ID);
            ids = 0;
          }
          look_up(j + kIdBlocks);
          __syncwarp();
        }
        const int pg = __shfl_sync(0xffffffffu, ids, (j % kIdBlocks) * kPagesEach + (lane & (kPagesEach - 1)));
        mbar_arrive_expect_tx_elect(b, L::kKBytes / 2);
        const int right = __shfl_down_sync(0xffffffffu, pg, 1);
        const unsigned run = __ballot_sync(0xffffffffu, lane < kPagesEach - 1 && right == pg + 1);
        const bool one = p.num_pages >= kPagesEach && (run & 7u) == 7u;
        if (lane < (one ? 1 : kPagesEach)) {
          if constexpr (kFp8)
            tma_load_3d(dst + mine + lane * (kPage * D), one ? run_map : page_map, b, 0, M.g, kPage * pg);
          else
            tma_load_5d(dst + mine + lane * L::kPageBytes, one ? run_map : page_map, b, 0, 0, 0, 2 * pg, M.g);
        }
        __syncwarp();
      }
    }
    if (!ok && lane == 0) set_abort(sh, p.err);
    // no exit while a copy into this CTA's shared memory is in flight
    for (int e = max(0, issued - kStages); e < issued; ++e)
      mbar_wait(bar(full[e % kStages]), (e / kStages) & 1);
  } else if (kFp8 && warp == kScaleWarp) {
    if constexpr (kFp8) {
      // ---------------------------------------------------------- scales --
      // A lane has a page of four blocks at once: its id is looked up eight blocks ahead
      // of their use, its scales four.
      pdl_wait();
      const float INF = __int_as_float(0x7f800000);
      constexpr int kAtOnce = 32 / kPagesPerBlock;
      int e = 0;  // blocks in all
      bool ok = true;
      for (int k = 0; ok; ++k) {
        const int slot = k % kMetaSlots;
        if (!(ok = wait_bar(sh.meta_full[slot], (k / kMetaSlots) & 1))) break;
        const UnitMeta M = read_meta(sh.meta[slot]);
        __syncwarp();
        if (!M.valid) break;
        if (lane == 0) mbar_arrive(bar(sh.meta_empty[slot]));
        const int32_t *const row = p.page_table + static_cast<size_t>(M.seq) * p.max_pages;
        int at = M.blk_lo * kPagesPerBlock + lane;  // the page whose id is looked up next
        auto look_up = [&] {  // (one of no block: any page's scales, as 0)
          const int id = at < M.pages ? row[at] : 0;
          at += 32;
          return id;
        };
        float ks = 0.f, vs = 0.f;
        auto fetch = [&](int id, int of) {
          ks = vs = 0.f;
          if (of >= M.pages) return;
          const size_t i = static_cast<size_t>(static_cast<unsigned>(id) < static_cast<unsigned>(p.num_pages) ? id : 0) * p.H_kv + M.g;
          ks = p.k_scale[i];
          vs = p.v_scale[i];
        };
        const int first = look_up();
        int id = look_up();
        fetch(first, at - 64);
        float ref = 1.f;  // what V's scales are taken over
#pragma unroll 1
        for (int j = 0; j < M.n_blocks; j += kAtOnce) {
          float k1 = ks, v1 = vs;
          if (j + kAtOnce < M.n_blocks) {
            fetch(id, at - 32);
            id = look_up();
          }
          if (!(k1 >= 0.f && k1 < INF && v1 >= 0.f && v1 < INF)) {
            flag_error(p.err, HPD_DEVERR_SCALE);
            if (!(k1 >= 0.f && k1 < INF)) k1 = 0.f;
            if (!(v1 >= 0.f && v1 < INF)) v1 = 0.f;
          }
          __syncwarp();
          if (j == 0) ref = ref_of(__uint_as_float(__reduce_max_sync(0xffffffffu, lane < kPagesPerBlock ? __float_as_uint(v1) : 0u)));
          const float over = v1 * over_ref(ref), lv = log2f(over), iv = __fdiv_rn(1.f, over);
#pragma unroll 1
          for (int i = 0; i < min(kAtOnce, M.n_blocks - j); ++i, ++e) {
            if (e >= kStages && !(ok = wait_bar(sh.k_empty[e % kStages], ((e / kStages) - 1) & 1))) break;
            if (lane / kPagesPerBlock == i) {
              sh.scales[e % kScaleBlocks][lane % kPagesPerBlock] = k1;
              sh.scales[e % kScaleBlocks][kPagesPerBlock + lane % kPagesPerBlock] = v1;
              sh.scales[e % kScaleBlocks][2 * kPagesPerBlock + lane % kPagesPerBlock] = lv;
              sh.scales[e % kScaleBlocks][3 * kPagesPerBlock + lane % kPagesPerBlock] = iv;
            }
            __syncwarp();
            if (lane == 0) mbar_arrive(bar(sh.k_full[e % kStages]));
          }
          if (!ok) break;
        }
      }
      if (!ok && lane == 0) set_abort(sh, p.err);
    }
  } else if (warp == kQkWarp) {
    // ---------------------------------------------------- Q K^T issuer --
    // The MMA warps run their loops with warp-uniform values; one elected lane
    // issues each group of MMAs and its commits.
    constexpr uint32_t idesc_qk = idesc_bf16_f32(kRows, kBlk, false);
    constexpr uint32_t idesc_codes = idesc_e4m3_f32(kRows, kBlk);
    const uint64_t dq0 = smem_desc_sw128(sbase + L::kK, 16, 1024);
    const uint64_t dk0 = !kFp8      ? smem_desc_sw128(sbase + L::kK, 16, L::kGroupBytes)
                         : D == 128 ? smem_desc_sw128(sbase + L::kK, 16, 1024)
                                    : smem_desc_sw64(sbase + L::kK, 16, 512);
    const bool issuer = elect_one();
    pdl_wait();
    uint32_t sk = 0, pk = 0;  // K ring: stage, phase
    int jg = 0;               // blocks issued
    bool ok = true;
    for (int k = 0; ok; ++k) {
      const int slot = k % kMetaSlots;
      if (!(ok = wait_bar(sh.meta_full[slot], (k / kMetaSlots) & 1))) break;
      const bool valid = sh.meta[slot].valid != 0;
      const int nb = sh.meta[slot].n_blocks;
      __syncwarp();
      if (!valid) break;
      if (lane == 0) mbar_arrive(bar(sh.meta_empty[slot]));
      const uint32_t q_col = tmem + L::col_q(k & 1);
      // entry -1 of the unit: its Q, copied into TMEM (in order with the MMAs: unit
      // k - 2's Q K^T are done with the slot)
      if (kFp8 && !(ok = wait_bar(sh.q_full[k & 1], (k >> 1) & 1))) break;
      for (int j = kFp8 ? 0 : -1; j < nb; ++j) {
        if (!(ok = wait_bar(sh.k_full[sk], pk))) break;
        // the S buffer is free for what is issued behind P V of the block before last
        if (j >= 0 && jg >= 2 && !(ok = wait_bar(sh.s_free[jg & 1], ((jg >> 1) - 1) & 1))) break;
        tc_fence_after();
        if (issuer) {
          const uint32_t off = (sk * L::kKBytes) >> 4;
          if constexpr (kFp8) {
            const uint32_t col = tmem + L::col_s(jg & 1);
#pragma unroll
            for (int kk = 0; kk < D / 16; ++kk)  // the first parts' 32 columns a time, then the second's
              mma_ts_codes_one(col, q_col + kk * 8, dk0 + off + kk % (D / 32) * 2, idesc_codes, kk > 0);
            mma_commit_one(bar(sh.s_full[jg & 1]));
            if (j == nb - 1) mma_commit_one(bar(sh.q_free[k & 1]));
          } else if (j < 0) {
#pragma unroll
            for (int kk = 0; kk < D / 16; ++kk)
              tmem_cp_128x256b(q_col + kk * 8, dq0 + off + (((kk >> 2) * L::kChunkBytes + (kk & 3) * 32) >> 4));
          } else {
            const uint32_t col = tmem + L::col_s(jg & 1);
#pragma unroll
            for (int kk = 0; kk < D / 16; ++kk)
              mma_ts_one(col, q_col + kk * 8, dk0 + off + (((kk >> 2) * 1024 + (kk & 3) * 32) >> 4), idesc_qk, kk > 0);
            mma_commit_one(bar(sh.s_full[jg & 1]));
          }
          mma_commit_one(bar(sh.k_empty[sk]));
        }
        __syncwarp();
        if (++sk == kStages) {
          sk = 0;
          pk ^= 1u;
        }
        jg += j >= 0;
      }
    }
    if (!ok && lane == 0) set_abort(sh, p.err);
  } else if (warp == kPvWarp) {
    // ------------------------------------------------------ P V issuer --
    constexpr uint32_t idesc_bf16 = idesc_bf16_f32(kRows, D, true), idesc_f16 = idesc_f16_f32(kRows, D, true);
    const uint64_t dv0 = smem_desc_sw128(sbase + L::kV, 1024, L::kGroupBytes);
    const bool issuer = elect_one();
    pdl_wait();
    uint32_t sv = 0, pv = 0;  // V ring: stage, phase
    int jg = 0;               // blocks issued
    int outputs = 0;          // units whose O was made
    bool ok = true;
    for (int k = 0; ok; ++k) {
      const int slot = k % kMetaSlots;
      if (!(ok = wait_bar(sh.meta_full[slot], (k / kMetaSlots) & 1))) break;
      const bool valid = sh.meta[slot].valid != 0;
      const int pass = sh.meta[slot].pass;
      const uint32_t idesc_pv = kFp8 && pass != kAgain ? idesc_f16 : idesc_bf16;
      const int nb = sh.meta[slot].n_blocks, len = sh.meta[slot].L;
      // the block with rows behind the sequence's end in its last page
      const int j_tail = len % kPage ? len / kBlk - sh.meta[slot].blk_lo : -1;
      // the first block that not every row of the tile sees all of (its first token sees
      // least, the last one at most 127 keys more: two blocks at most), in a unit that is
      // run again
      int j_sieve = nb;
      if (pass == kAgain)
        j_sieve = max(max(min(max(sh.meta[slot].lim0, sh.meta[slot].full), len), 0) / kBlk - sh.meta[slot].blk_lo, 0);
      __syncwarp();
      if (!valid) break;
      if (lane == 0) mbar_arrive(bar(sh.meta_empty[slot]));
      if (pass == kAgain) {
        for (int c = lane; c < D; c += 32) sh.sieved[slot][c] = (kNoKey << 20) | (kNoKey << 10) | kNoKey;
        __syncwarp();
      }
      if (pass == kMaxima) {  // nothing to multiply: the scores are only read
        for (int j = 0; j < nb; ++j, ++jg) {
          if (!(ok = wait_bar(sh.p_full[jg & 1][0], (jg >> 1) & 1) && wait_bar(sh.p_full[jg & 1][1], (jg >> 1) & 1)))
            break;
          tc_fence_after();
          tc_fence_before();
          if (issuer) mbar_arrive(bar(sh.s_free[jg & 1]));
          __syncwarp();
        }
        continue;
      }
      for (int j = 0; j < nb; ++j) {
        if (!(ok = wait_bar(sh.v_full[sv], pv))) break;
        // O last held the output before, which must have been read
        if (j == 0 && outputs >= 1 && !(ok = wait_bar(sh.o_empty, (outputs - 1) & 1))) break;
        if (j == j_tail) {
          const uint32_t v0 = sbase + L::kV + sv * L::kTileBytes;
          for (int i = (len % kBlk) * (L::kChunks * 8) + lane; i < (len % kBlk / kPage + 1) * kPage * (L::kChunks * 8);
               i += 32) {
            const int r = i / (L::kChunks * 8), c = i % (L::kChunks * 8);
            asm volatile("st.shared.v4.b32 [%0], {%1, %1, %1, %1};" ::"r"(v0 + (r >> 3) * L::kGroupBytes +
                                                                         (c >> 3) * 1024 + (r & 7) * 128 + (c & 7) * 16),
                         "r"(0)
                         : "memory");
          }
          asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
          __syncwarp();
        }
        if (j >= j_sieve) {
          sieve_block<D>(sbase + L::kV + sv * L::kTileBytes, (j - j_sieve) * kBlk, sh.sieved[slot]);
          asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
          __syncwarp();
        }
        // O (+)= P V: 16 keys per MMA, P in the S buffer: of half h, keys 32-63 at
        // column 64 h + 32, then keys 0-31 at column 64 h + 48
        const uint64_t vd = dv0 + ((sv * L::kTileBytes) >> 4);
        const uint32_t col = tmem + L::col_s(jg & 1);
#pragma unroll
        for (int part = 0; part < 2; ++part) {
          if (!(ok = wait_bar(sh.p_full[jg & 1][part], (jg >> 1) & 1))) break;
          tc_fence_after();
          if (issuer) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const int kk = (i >> 1) * 4 + (1 - part) * 2 + (i & 1);  // 16 keys of the block
              mma_ts_one(tmem + L::kColO, col + (i >> 1) * 64 + 32 + part * 16 + (i & 1) * 8,
                         vd + kk * ((2 * L::kGroupBytes) >> 4), idesc_pv, (j > 0 || part > 0 || i > 0) ? 1u : 0u);
            }
          }
          __syncwarp();
        }
        if (!ok) break;
        if (issuer) {
          // (Q K^T of the next block but one, into this S buffer, may be issued: MMAs
          // run in the order of issue)
          tc_fence_before();
          mbar_arrive(bar(sh.s_free[jg & 1]));
          mma_commit_one(bar(sh.v_empty[sv]));
          if (j == nb - 1) mma_commit_one(bar(sh.o_full));
        }
        __syncwarp();
        if (++sv == kVStages) {
          sv = 0;
          pv ^= 1u;
        }
        ++jg;
      }
      ++outputs;
      if (pass == kAgain) publish_seq(&sh.sieved_seq, k + 1);
    }
    if (!ok && lane == 0) set_abort(sh, p.err);
  } else if (kFp8 && warp >= kWideWarp) {
    if constexpr (kFp8) {
      // -------------------------------------------- Q parts, V to f16 --
      const int quad = warp & 3;  // its 32 rows of a tile, its 32 keys of a block
      constexpr int kCodeStages = Rings<true>::kCodeStages;
      pdl_wait();
      int e = 0;                // blocks widened
      uint32_t sv = 0, pv = 1;  // V ring: stage, phase of its being free
      bool ok = true;
      for (int k = 0; ok; ++k) {
        const int slot = k % kMetaSlots;
        if (!(ok = wait_bar(sh.meta_full[slot], (k / kMetaSlots) & 1))) break;
        const UnitMeta M = read_meta(sh.meta[slot]);
        __syncwarp();
        if (!M.valid) break;
        if (lane == 0) mbar_arrive(bar(sh.meta_empty[slot]));
        if (k >= 2 && !(ok = wait_bar(sh.q_free[k & 1], ((k >> 1) - 1) & 1))) break;
        tc_fence_after();
        const int row0 = M.copies > 1 ? 0 : quad * 32;
        part_rows<D>(p.q + M.tok0 * p.q_stride + M.g * G * D, p.q_stride, G, p.div_G, row0, min(M.nrows - row0, 32),
                     tmem + (static_cast<uint32_t>(quad * 32) << 16) + L::col_q(k & 1), &sh.q_scale[slot][quad * 32]);
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(bar(sh.q_full[k & 1]));
        if (M.pass == kMaxima) continue;
#pragma unroll 1
        for (int j = 0; j < M.n_blocks; ++j, ++e) {
          const int st = e % kCodeStages;
          if (!(ok = wait_bar(sh.code_full[st], (e / kCodeStages) & 1))) break;
          const uint32_t from = sbase + L::kCodes + st * L::kCodeBytes + quad * 32 * D;
          // a lane has a row of each 8 keys and 16 columns of each 64: reads and writes of
          // eight lanes are of eight rows, whose swizzles differ
          const int r = lane & 7, c0 = lane >> 3;
          // (the next keys' codes are read before these are written: a block's codes at once
          // would hold 32 registers)
          constexpr int kPieces = D / 64;
          uint32_t x[kPieces][4];
          const uint32_t src = from + r * D + ((D == 128 ? c0 ^ r : c0 ^ (r >> 1 & 3)) << 4);
          auto read = [&](int group) {
#pragma unroll
            for (int h = 0; h < kPieces; ++h)
              asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];"
                           : "=r"(x[h][0]), "=r"(x[h][1]), "=r"(x[h][2]), "=r"(x[h][3])
                           : "r"((src ^ h << 6) + group * 8 * D));
          };
          read(0);
          if (!(ok = wait_bar(sh.v_empty[sv], pv))) break;
          if (M.pass == kAgain) {
            widen_again<D>(from, sbase + L::kV + sv * L::kTileBytes + quad * 4 * L::kGroupBytes);
          } else {
            const uint32_t to = sbase + L::kV + sv * L::kTileBytes + quad * 4 * L::kGroupBytes + r * 128;
            const uint32_t to0 = to + ((c0 * 2 ^ r) << 4), to1 = to + (((c0 * 2 + 1) ^ r) << 4);
#pragma unroll
            for (int group = 0; group < 4; ++group) {
              uint32_t y[kPieces][8];
#pragma unroll
              for (int h = 0; h < kPieces; ++h)
#pragma unroll
                for (int n = 0; n < 4; ++n) f16_of_codes(x[h][n], y[h][2 * n], y[h][2 * n + 1]);
              if (group < 3) read(group + 1);
#pragma unroll
              for (int h = 0; h < kPieces; ++h)
#pragma unroll
                for (int n = 0; n < 2; ++n)
                  asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"((n ? to1 : to0) + group * L::kGroupBytes + h * 1024),
                               "r"(y[h][4 * n]), "r"(y[h][4 * n + 1]), "r"(y[h][4 * n + 2]), "r"(y[h][4 * n + 3])
                               : "memory");
            }
          }
          asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
          __syncwarp();
          if (lane == 0) {
            mbar_arrive(bar(sh.v_full[sv]));
            mbar_arrive(bar(sh.code_empty[st]));
          }
          if (++sv == kVStages) {
            sv = 0;
            pv ^= 1u;
          }
        }
      }
      if (!ok && lane == 0) set_abort(sh, p.err);
    }
  } else if (warp >= kOutputWarp) {
    // ---------------------------------------------------------- output --
    const int quad = warp & 3;          // TMEM lane quadrant this warp may access
    const int r_in = quad * 32 + lane;  // row within the tile
    const uint32_t o_addr = tmem + (static_cast<uint32_t>(quad * 32) << 16) + L::kColO;
    const uint32_t stage = sbase + L::kStage + quad * 32 * 128;  // of this warp's rows
    constexpr int kOnce = kFp8 ? 16 : 32;  // columns of O at once (there are 80 registers, or 96)
    pdl_wait();
    const int rt = p.div_G(r_in);
    int outputs = 0;
    unsigned copied = 0;  // phases of the barrier of that name
    bool ok = true;
    for (int k = 0; ok; ++k) {
      const int slot = k % kMetaSlots;
      if (!(ok = wait_bar(sh.meta_full[slot], (k / kMetaSlots) & 1))) break;
      const UnitMeta &M = sh.meta[slot];
      if (!M.valid) break;
      if (!(ok = wait_bar(sh.sums[slot], (k / kMetaSlots) & 1))) break;
      const int pass = M.pass, nrows = M.nrows, nsplit = M.nsplit;
      if constexpr (kFp8) {
        if (M.copies > 1) {
          // A row's sums are those of its copies together.  O goes through shared memory, as
          // many columns at once as the copies' rows have room for.
          // (rows are 32 apart, a warp has a copy of each)
          const int width = nrows <= 8 ? 128 : nrows <= 16 ? 64 : 32;
          const int tok0 = M.tok0, head0 = M.g * G;
          const size_t part_row = static_cast<size_t>(M.slot) * kRows;
          const uint32_t base = sbase + L::kStage;
          auto sum_of_row = [&](int row) {
            float l = 0.f;
            for (int c = 0; c < kRows; c += 32) l += sh.xsum[slot][0][row + c] + sh.xsum[slot][1][row + c];
            return l;
          };
          bool odd = false;
          if (r_in < nrows) {
            const float l = sum_of_row(r_in), lse = l == 0.f ? NEG_INF : l > 0.f ? lse_of(sh.xbase[slot][r_in], l) : l;
            if (nsplit > 1) p.l_part[part_row + r_in] = lse;
            else if (p.lse) p.lse[(tok0 + rt) * p.H_q + head0 + r_in - rt * G] = lse;
            odd = l != l;
            // (what O's sums are to be multiplied by, in the base's place)
            sh.xbase[slot][r_in] = l == 0.f ? 0.f : __fdividef(sh.v_ref[slot][r_in], l);
          }
          // (the unit before may have rows on their way through the same memory)
          __syncwarp();
          if (lane == 0) mbar_arrive(bar(sh.copied));
          if (!(ok = wait_bar(sh.copied, copied & 1) && wait_bar(sh.o_full, outputs & 1))) break;
          ++copied;
          ++outputs;
          tc_fence_after();
#pragma unroll 1
          for (int col = 0; col < D && ok; col += width) {
            const int w = min(width, D - col);
#pragma unroll 1
            for (int c = 0; c < w; c += 32) {
              uint32_t o[32];
              tmem_ld32(o_addr + col + c, o);
              tmem_ld_wait32(o);
              if (lane < nrows) {
#pragma unroll
                for (int e = 0; e < 8; ++e)
                  asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(base + ((quad * nrows + lane) * width + c) * 4 +
                                                                               ((e ^ lane) & 7) * 16),
                               "r"(o[4 * e]), "r"(o[4 * e + 1]), "r"(o[4 * e + 2]), "r"(o[4 * e + 3])
                               : "memory");
              }
            }
            if (col + width >= D) tc_fence_before();
            __syncwarp();
            if (lane == 0) {
              if (col + width >= D) mbar_arrive(bar(sh.o_empty));
              mbar_arrive(bar(sh.copied));
            }
            if (!(ok = wait_bar(sh.copied, copied & 1))) break;
            ++copied;
            for (int i = r_in; i < nrows * (w / 4); i += kRows) {
              const int row = i / (w / 4), c = i % (w / 4);  // four columns
              float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 1
              for (int n = 0; n < kCopies; ++n) {
                float4 x;
                asm volatile("ld.shared.v4.f32 {%0, %1, %2, %3}, [%4];"
                             : "=f"(x.x), "=f"(x.y), "=f"(x.z), "=f"(x.w)
                             : "r"(base + ((n * nrows + row) * width + (c & ~7) * 4) * 4 + (((c ^ row) & 7) << 4))
                             : "memory");
                v.x += x.x;
                v.y += x.y;
                v.z += x.z;
                v.w += x.w;
              }
              const float inv = sh.xbase[slot][row];
              odd |= !(v.x * 0.f == 0.f && v.y * 0.f == 0.f && v.z * 0.f == 0.f && v.w * 0.f == 0.f);
              v = make_float4(v.x * inv, v.y * inv, v.z * inv, v.w * inv);
              if (nsplit > 1) {
                *reinterpret_cast<float4 *>(p.o_part + (part_row + row) * D + col + 4 * c) = v;
              } else {
                const int t = p.div_G(row);
                *reinterpret_cast<uint2 *>(p.out + (static_cast<size_t>(tok0 + t) * p.H_q + head0 + row - t * G) * D + col + 4 * c) =
                    make_uint2(pack_bf16x2(v.x, v.y), pack_bf16x2(v.z, v.w));
              }
            }
            __syncwarp();
            if (col + width >= D) break;
            if (lane == 0) mbar_arrive(bar(sh.copied));
            if (!(ok = wait_bar(sh.copied, copied & 1))) break;
            ++copied;
          }
          if (!ok) break;
          const bool redo = __any_sync(0xffffffffu, odd);
          if (lane == 0) {
            if (redo) {
              atomicOr(&sh.redo, 1u << (k & (kLastUnits - 1)));
              __threadfence_block();
            }
            mbar_arrive(bar(sh.meta_empty[slot]));
            asm volatile("red.relaxed.cta.shared::cta.add.u32 [%0], 1;" ::"r"(smem_u32(&sh.units_done)) : "memory");
          }
          // (the next unit's sums may come here once all have read these)
          if (lane == 0) mbar_arrive(bar(sh.copied));
          if (!(ok = wait_bar(sh.copied, copied & 1))) break;
          ++copied;
          continue;
        }
      }
      const bool idle = quad * 32 >= nrows, valid = r_in < nrows;
      const int pair = (M.tok0 + rt) * p.H_q + M.g * G + r_in - rt * G;  // row and head
      const size_t part_row = static_cast<size_t>(M.slot) * kRows + r_in;
      float *const part = nsplit > 1 ? p.o_part + part_row * D : nullptr;
      float inv = 0.f;
      bool odd = false;
      if (valid && pass != kMaxima) {
        const float l = sh.xsum[slot][0][r_in] + sh.xsum[slot][1][r_in];
        const float lse = l == 0.f ? NEG_INF : l > 0.f ? lse_of(sh.xbase[slot][r_in], l) : l;
        if (part) p.l_part[part_row] = lse;
        else if (p.lse) p.lse[pair] = lse;
        inv = l == 0.f ? 0.f : __fdividef(kFp8 ? sh.v_ref[slot][r_in] : 1.f, l);  // (a sum that is NaN stays one; others are below 2^126)
        odd = l != l;
      }
      __syncwarp();
      // (what was sieved from a unit that was run again is still to be read)
      if (lane == 0 && pass != kAgain) mbar_arrive(bar(sh.meta_empty[slot]));
      if (pass == kMaxima) continue;
      if (!(ok = wait_bar(sh.o_full, outputs & 1))) break;
      ++outputs;
      tc_fence_after();
      float2 finite = make_float2(0.f, 0.f);  // NaN once an infinity or NaN is added
      // 64 columns at a time, through shared memory, so that a store instruction
      // writes whole 128-byte lines of four rows instead of a sector of 32; O is
      // read ahead of the stores, as the next unit's P V waits for that
#pragma unroll 1
      for (int half = 0; half <= D / 64; ++half) {
        uint32_t keep[32];
        if (half < D / 64) {
#pragma unroll
          for (int c = 0; c < 64; c += kOnce) {
            uint32_t o[kOnce];
            if (!idle) {
              if constexpr (kFp8) {
                tmem_ld16(o_addr + half * 64 + c, o);
                tmem_ld_wait16(o);
              } else {
                tmem_ld32(o_addr + half * 64 + c, o);
                tmem_ld_wait32(o);
              }
            }
            if (half == D / 64 - 1 && c == 64 - kOnce) {  // O may be overwritten once every warp has read it
              tc_fence_before();
              __syncwarp();
              if (lane == 0) mbar_arrive(bar(sh.o_empty));
            }
            if (idle) continue;
#pragma unroll
            for (int e = 0; e < kOnce; e += 2) {
              const float2 v = make_float2(__uint_as_float(o[e]), __uint_as_float(o[e + 1]));
              finite = __ffma2_rn(v, make_float2(0.f, 0.f), finite);
              const float2 x = __fmul2_rn(v, make_float2(inv, inv));
              o[e] = __float_as_uint(x.x);
              o[e + 1] = __float_as_uint(x.y);
              keep[(c + e) / 2] = pack_bf16x2(x.x, x.y);
            }
            if (part && valid) {
#pragma unroll
              for (int e = 0; e < kOnce; e += 8) st_global_v8(part + half * 64 + c + e, o + e);
            }
          }
        }
        if (half == D / 64 - 1) {
          // O has been looked at: the scheduler may go on, or end, beside the stores
          const bool wild = valid && !(finite.x == 0.f && finite.y == 0.f);  // an output that is not finite
          const bool redo = __any_sync(0xffffffffu, pass == kFirst && (odd || wild));
          if (lane == 0) {
            // (released only where there is something to release: it waits for the stores)
            if (redo) {
              atomicOr(&sh.redo, 1u << (k & (kLastUnits - 1)));
              __threadfence_block();
            }
            asm volatile("red.relaxed.cta.shared::cta.add.u32 [%0], 1;" ::"r"(smem_u32(&sh.units_done)) : "memory");
          }
        }
        if (idle || part) continue;
        if (half > 0) {  // the columns before these
#pragma unroll 1
          for (int i = 0; i < 32; i += 8) {
            uint32_t w[2][4];
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              const int r = (lane >> 3) + i + 4 * e;
              asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];"
                           : "=r"(w[e][0]), "=r"(w[e][1]), "=r"(w[e][2]), "=r"(w[e][3])
                           : "r"(stage + r * 128 + (((lane ^ r) & 7) << 4)));
            }
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              const int r = (lane >> 3) + i + 4 * e, at = __shfl_sync(0xffffffffu, pair, r);
              if (quad * 32 + r < nrows)
                *reinterpret_cast<uint4 *>(p.out + static_cast<size_t>(at) * D + half * 64 - 64 + (lane & 7) * 8) =
                    make_uint4(w[e][0], w[e][1], w[e][2], w[e][3]);
            }
          }
          __syncwarp();
        }
        if (half < D / 64) {
#pragma unroll
          for (int e = 0; e < 8; ++e)
            asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(stage + lane * 128 + (((lane ^ e) & 7) << 4)),
                         "r"(keep[4 * e]), "r"(keep[4 * e + 1]), "r"(keep[4 * e + 2]), "r"(keep[4 * e + 3])
                         : "memory");
          __syncwarp();
        }
      }
      if (pass != kAgain) continue;
      // values that are not finite in the blocks that some rows see part of
      if (!(ok = __all_sync(0xffffffffu, await_seq(&sh.sieved_seq, k + 1, sh)))) break;
      const int lim = min(max(M.lim0 + rt, M.full), M.L);
      const int sieve0 = max(max(min(max(M.lim0, M.full), M.L), 0) / kBlk, M.blk_lo) * kBlk;
      __syncwarp();  // (rows of out were stored by other lanes)
      if (valid && inv > 0.f)
        add_sieved<D>(sh.sieved[slot], lim - sieve0, part, p.out + static_cast<size_t>(pair) * D);
      __syncwarp();
      if (lane == 0) mbar_arrive(bar(sh.meta_empty[slot]));
    }
    if (!ok && lane == 0) set_abort(sh, p.err);
  } else if (warp >= kSoftmaxWarp) {
    // --------------------------------------------------------- softmax --
    const int h = (warp - kSoftmaxWarp) >> 2;  // half of a block's keys
    const int quad = warp & 3;                 // TMEM lane quadrant this warp may access
    const int r_in = quad * 32 + lane;         // row within the tile
    const uint32_t t_lane = tmem + (static_cast<uint32_t>(quad * 32) << 16);
    const int rt = p.div_G(r_in);
    const float sl2 = p.scale_log2;
    pdl_wait();
    int jg = 0;            // blocks in all
    float given = NEG_INF;  // the row's maximum, which a pass over the maxima found
    bool ok = true;
    for (int k = 0; ok; ++k) {
      const int slot = k % kMetaSlots;
      if (!(ok = wait_bar(sh.meta_full[slot], (k / kMetaSlots) & 1))) break;
      const UnitMeta M = read_meta(sh.meta[slot]);
      __syncwarp();
      if (!M.valid) break;
      if (!kFp8 && lane == 0) mbar_arrive(bar(sh.meta_empty[slot]));
      const int nb = M.n_blocks, blk_lo = M.blk_lo, pass = M.pass;
      const int r = kFp8 && M.copies > 1 ? lane : r_in;
      const bool idle = r - lane >= M.nrows;
      // (rows that are no query count as seeing everything, so that their warp
      // needs no masks for them; their results are not stored)
      const int lim = r < M.nrows ? min(max(M.lim0 + (kFp8 ? p.div_G(r) : rt), M.full), M.L) : 1 << 30;
      // blocks of the unit that every row of the warp sees all of
      const int n_plain = kFp8 || sl2 > 0.f ? min(max(__reduce_min_sync(0xffffffffu, lim), 0) / kBlk - blk_lo, nb) : 0;
      auto await_s = [&] {
        if (!wait_bar(sh.s_full[jg & 1], (jg >> 1) & 1)) return false;
        tc_fence_after();
        return true;
      };
      auto publish = [&](int part) {
        tmem_st_wait();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(bar(sh.p_full[jg & 1][part]));
      };
      float row_mul = sl2, val_mul = 1.f, v_ref = 1.f;
      if constexpr (kFp8) {  // (the factor of the row's parts is there with its first scores)
        if (!idle) {
          if (!(ok = await_s())) break;
          row_mul *= sh.q_scale[slot][r_in];
          __syncwarp();
        }
        if (lane == 0) mbar_arrive(bar(sh.meta_empty[slot]));
      }
      auto publish_both = [&] {
        tmem_st_wait();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) {
          mbar_arrive(bar(sh.p_full[jg & 1][0]));
          mbar_arrive(bar(sh.p_full[jg & 1][1]));
        }
      };
      if (idle) {  // (whatever is there instead of P reaches only rows that are not stored)
        for (int j = 0; j < nb; ++j, ++jg) {
          if (!(ok = await_s())) break;
          publish(0);
          publish(1);
        }
        if (lane == 0) mbar_arrive(bar(sh.sums[slot]));
        continue;
      }
      float m_run = given, mx_run = NEG_INF;
      float2 l4[4];         // the row's sum so far, in parts
      bool inside = true;   // the scores stay in the window of their base
#pragma unroll
      for (int i = 0; i < 4; ++i) l4[i] = make_float2(0.f, 0.f);
      int j = 0;
      if (pass == kMaxima) {
        for (; j < nb; ++j, ++jg) {
          if (!(kFp8 && j == 0) && !(ok = await_s())) break;
          const int hi = min(lim - (blk_lo + j) * kBlk, kBlk) - h * 64;
          const uint32_t at = t_lane + L::col_s(jg & 1) + h * 64;
          if constexpr (kFp8) {
            const float *const sc = sh.scales[jg % kScaleBlocks];
            mx_run = fmaxf(mx_run, row_max_fp8(at, 32, j < n_plain, hi, row_mul, sc + 4 * h).x);
          } else {
            mx_run = fmaxf(mx_run, row_max(at, 32, j < n_plain, hi, sl2));
          }
          publish(0);
          publish(1);
        }
      } else {
        if (!kFp8 && !(ok = await_s())) break;
        if (pass == kFirst) {
          const uint32_t at = t_lane + L::col_s(jg & 1);
          const int hi = min(lim - blk_lo * kBlk, kBlk);
          if constexpr (kFp8) {
            const float *const sc = sh.scales[jg % kScaleBlocks];
            const float2 first = row_max_fp8(at, 64, n_plain > 0, hi, row_mul, sc);
            v_ref = ref_of(largest_scale(sc + kPagesPerBlock, hi));
            const int below =  // powers of two
                static_cast<int>(__float_as_uint(v_ref) - __float_as_uint(ref_of(first.y))) >> 23;
            m_run = first.x - (kFirstLog2 + below);
            inside = below <= kFarLog2;
          } else {
            m_run = row_max(at, 64, n_plain > 0, hi, sl2);
          }
        }
        if constexpr (kFp8) {
          val_mul = over_ref(v_ref);
          if (h == 0) sh.v_ref[slot][r_in] = v_ref;
        }
        // (scores of -inf alone give no base to a row that sees the unit's keys)
        inside &= pass != kFirst || m_run > NEG_INF || lim <= blk_lo * kBlk;
        if constexpr (kFp8) {
          for (; M.copies > 1 && j < nb; ++j, ++jg) {
            if (j > 0 && !(ok = await_s())) break;
            const float *const sc = sh.scales[jg % kScaleBlocks] + 4 * h;
            softmax_share_fp8(t_lane + L::col_s(jg & 1) + h * 64, quad, min(lim - (blk_lo + j) * kBlk, kBlk) - h * 64,
                              row_mul, val_mul, sc, sc + kPagesPerBlock, m_run == NEG_INF ? 0.f : m_run, l4, publish_both);
          }
          if (!ok) break;
        }
        // blocks that every row of the warp sees all of: nothing to decide
        for (; j < (kFp8 && pass == kAgain ? 0 : n_plain); ++j, ++jg) {
          if (j > 0 && !(ok = await_s())) break;
          const uint32_t at = t_lane + L::col_s(jg & 1) + h * 64;
          const float *const sc = sh.scales[jg % kScaleBlocks] + 4 * h;
          if constexpr (kFp8)
            inside &= softmax_plain_fp8(at, row_mul, sc, sc + 2 * kPagesPerBlock, sc + 3 * kPagesPerBlock,
                                        m_run == NEG_INF ? 0.f : m_run, l4, publish);
          else
            inside &= softmax_plain(at, sl2, m_run, l4, publish);
        }
        if (!ok) break;
        for (; j < nb; ++j, ++jg) {
          if (j > 0 && !(ok = await_s())) break;
          const int hi = min(lim - (blk_lo + j) * kBlk, kBlk) - h * 64;
          const uint32_t at = t_lane + L::col_s(jg & 1) + h * 64;
          const float *const sc = sh.scales[jg % kScaleBlocks] + 4 * h;
          if constexpr (kFp8)
            pass == kAgain ? softmax_masked_fp8<true>(at, hi, row_mul, 1.f, sc, sc + kPagesPerBlock,
                                                      m_run == NEG_INF ? 0.f : m_run, l4, publish)
                           : softmax_masked_fp8<false>(at, hi, row_mul, val_mul, sc, sc + kPagesPerBlock,
                                                       m_run == NEG_INF ? 0.f : m_run, l4, publish);
          else
            inside &= softmax_masked(at, hi, sl2, m_run, l4, publish);
        }
      }
      if (!ok) break;
      // (weights of pages whose scales are next to nothing may be beyond any product: the two halves'
      // sum, and v_ref over it, have to be numbers)
      if constexpr (kFp8) inside &= pass != kFirst || tc::sum_of(l4) <= fminf(over_ref(val_mul), 0x1p-26f) * 0x1p125f;
      sh.xsum[slot][h][r_in] = pass == kMaxima ? mx_run : inside ? tc::sum_of(l4) : __int_as_float(0x7fffffff);
      if (h == 0) sh.xbase[slot][r_in] = m_run;
      __syncwarp();
      if (lane == 0) mbar_arrive(bar(sh.sums[slot]));
      if (pass == kMaxima) {
        publish_seq(&sh.max_seq[quad][h], k + 1);
        if (!(ok = __all_sync(0xffffffffu, await_seq(&sh.max_seq[quad][h ^ 1], k + 1, sh)))) break;
        given = fmaxf(sh.xsum[slot][0][r_in], sh.xsum[slot][1][r_in]);
      }
    }
    if (!ok && lane == 0) set_abort(sh, p.err);
  }

  // ------------------------------------------------------------ teardown --
  if (warp == kQkWarp || warp == kPvWarp) {
    uint64_t &done = sh.mma_done[warp == kQkWarp ? 0 : 1];
    mma_commit(bar(done));
    mbar_wait(bar(done), 0);
  }
  tc_fence_before();
  __syncthreads();
  if (warp == kQkWarp) {
    tc_fence_after();
    tmem_dealloc(tmem, kTmemCols);
  }
  // the last CTA to finish resets the unit counters for the next call
  if (tid == 0) {
    __threadfence();
    if (atomicAdd(p.unit_ctr + 1, 1) == static_cast<int>(gridDim.x) - 1) {
      atomicExch(p.unit_ctr, 0);
      atomicExch(p.unit_ctr + 1, 0);
    }
  }
}

// Joins the splits of a tile, a CTA for every split, each with its share of the rows,
// a warp a row:
//   lse = log sum_s exp(lse_s),  out = sum_s exp(lse_s - lse) out_s
// What bounds it: the launch and three loads one after the other (the tile, then its
// sums and results together) where rows are few; else reading the results from L2.
// With it, one token behind 3,999 (16 / 2 heads of 128) takes 12.6 us, some 1 us more than
// without; 700 behind 2,300 with 40 / 8 heads 38.6, without 32.2.
constexpr int kMergeWarps = 16;
constexpr int kMergeAhead = 8;  // splits whose results are on their way at once
template <int D>
__global__ void __launch_bounds__(32 * kMergeWarps) chunk_merge_kernel(const ChunkParams p) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  pdl_wait();
  pdl_trigger();
  int n_slots, tok0, nrows, g, split, n;  // (both loads before the first decision)
  asm volatile("ld.global.b32 %0, [%1];" : "=r"(n_slots) : "l"(p.n_slots));
  asm volatile("ld.global.v4.b32 {%0, %1, %2, %3}, [%4];"
               : "=r"(tok0), "=r"(nrows), "=r"(g), "=r"(split)
               : "l"(&p.slot[blockIdx.x]));
  asm volatile("ld.global.b32 %0, [%1];" : "=r"(n) : "l"(&p.slot[blockIdx.x].nsplit));
  if (static_cast<int>(blockIdx.x) >= n_slots || n <= 1) return;
  const size_t slot0 = blockIdx.x - split * p.H_kv;  // of split 0; the next are H_kv on
  const float NEG_INF = -__int_as_float(0x7f800000);
  constexpr int kV = D / 32;  // values of a lane
  const size_t stride = static_cast<size_t>(p.H_kv) * kRows * D;
  const int lo = split * nrows / n, hi = (split + 1) * nrows / n;
  for (int r = lo + warp; r < hi; r += kMergeWarps) {
    const float *src = p.o_part + (slot0 * kRows + r) * D + lane * kV;
    const float l = lane < n ? p.l_part[(slot0 + static_cast<size_t>(lane) * p.H_kv) * kRows + r] : NEG_INF;
    float v[kMergeAhead][kV];
    auto load = [&](int s0) {
#pragma unroll
      for (int i = 0; i < kMergeAhead; ++i)
        if (s0 + i < n) {
          if constexpr (kV == 4)
            *reinterpret_cast<float4 *>(v[i]) = *reinterpret_cast<const float4 *>(src + (s0 + i) * stride);
          else
            *reinterpret_cast<float2 *>(v[i]) = *reinterpret_cast<const float2 *>(src + (s0 + i) * stride);
        }
    };
    load(0);
    float m = l;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
    const float base = m == NEG_INF ? 0.f : m;
    const float w = exp2f((l - base) * kLog2e);
    float sum = w;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    const float inv = sum == 0.f ? 0.f : 1.f / sum;
    const float w_or = l == NEG_INF ? -1.f : w;  // (an empty partial is not written; another's weight may be 0)
    float acc[kV];
#pragma unroll
    for (int c = 0; c < kV; ++c) acc[c] = 0.f;
#pragma unroll 1
    for (int s0 = 0; s0 < n; s0 += kMergeAhead) {
      if (s0 > 0) load(s0);
#pragma unroll
      for (int i = 0; i < kMergeAhead; ++i) {
        const float ws = __shfl_sync(0xffffffffu, w_or, s0 + i);
#pragma unroll
        for (int c = 0; c < kV; ++c) acc[c] = ws < 0.f ? acc[c] : fmaf(ws, v[i][c], acc[c]);
      }
    }
    const int rt = p.div_G(r);
    const size_t pair = static_cast<size_t>(tok0 + rt) * p.H_q + g * p.G + r - rt * p.G;
    uint32_t *dst = reinterpret_cast<uint32_t *>(p.out + pair * D) + lane * (kV / 2);
#pragma unroll
    for (int c = 0; c < kV; c += 2) dst[c / 2] = pack_bf16x2(acc[c] * inv, acc[c + 1] * inv);
    if (lane == 0 && p.lse) p.lse[pair] = sum == 0.f ? NEG_INF : m + logf(sum);
  }
}

// ------------------------------------------------------------------ host --

hpd_status check_scalars(const hpd_chunk_attn_args *a) {
  if (!a) return HPD_ERR_INVALID_ARG;
  if (a->S < 1 || a->T < 1 || a->H_q < 1 || a->H_kv < 1 || a->num_pages < 1 || a->max_pages < 1 ||
      a->max_seq_len < 0 || a->q_stride < 0 || a->q_stride % 8 != 0)
    return HPD_ERR_INVALID_ARG;
  if (a->H_q % a->H_kv != 0 || !std::isfinite(a->scale)) return HPD_ERR_INVALID_ARG;
  if (a->H_q / a->H_kv > 16 || (a->D != 64 && a->D != 128)) return HPD_ERR_UNSUPPORTED;
  if (a->q_stride != 0 && a->q_stride < static_cast<int64_t>(a->H_q) * a->D) return HPD_ERR_INVALID_ARG;
  if (static_cast<long long>(a->max_pages) * kPage >= (1LL << 30)) return HPD_ERR_UNSUPPORTED;
  if (static_cast<long long>(a->num_pages) * kPage >= (1LL << 31)) return HPD_ERR_UNSUPPORTED;
  // units (at most a row and head each, kMaxSplits times) stay below kNoUnit
  if (static_cast<long long>(a->T) * a->H_q >= (1LL << 30) / kMaxSplits) return HPD_ERR_UNSUPPORTED;
  return HPD_OK;
}

constexpr int kPlanSms = 152;  // SMs the split plan assumes (GB300)
constexpr size_t kAlign = 256;
size_t align_up(size_t x) { return (x + kAlign - 1) / kAlign * kAlign; }

struct ChunkPlan {
  int slots;        // units of split tiles; 0: none is split
  long long units;  // upper bound
  size_t off_opart, off_lpart, off_slot, bytes;
};

// Tiles may be split where the call's units leave SMs idle in their last (or only)
// wave.  Only host scalars enter (the kernel then splits by the true lengths): the
// time of units of the longest sequences, in blocks, whole against split after the
// full waves, a unit's start and end counted as 3.5 blocks, the merge as 10.  (us,
// split and whole, 16 / 2 heads of 128: one token behind 1,799 12.0 and 16.2, behind 2,499
// 12.5 and 18.9, 16 behind 8,984 16.1 and 47.7; 2,048 behind 14,336 with 32 / 8 heads 295
// and 310, in bursts of 40 calls; 500 behind 2,000 with 16 / 4 heads of 64 21.6 and 19.0,
// which stays whole.  The other way: 700 behind 2,300 with 40 / 8 heads is split, and
// 38.6 and 36.1.)
// A bound far above the lengths costs short calls time: they are split, or have a merge
// launched that finds nothing.  With a bound of 8,192 and with the exact one: one token
// behind 255 11.2 and 9.5, 640 of one page 15.4 and 12.0, 1,300 23.6 and 18.7, 300 behind
// 1,200 17.8 and 15.7, 500 alone with 16 / 4 heads of 64 17.0 and 9.7.
ChunkPlan make_plan(const hpd_chunk_attn_args *a) {
  ChunkPlan pl{};
  const int G = a->H_q / a->H_kv, TT = kRows / G;
  const long long seqs = std::min(a->S, a->T);
  const long long units = std::max<long long>(seqs, (a->T + TT - 1) / TT) * a->H_kv;
  const int cap = a->max_pages * kPage;
  const int longest = a->max_seq_len > 0 ? std::min(a->max_seq_len, cap) : cap;
  const int N = std::max(1, (longest + kBlk - 1) / kBlk);
  const long long left = units % kPlanSms;
  const double full = static_cast<double>(units / kPlanSms) * (N + 3.5), none = full + (left ? N + 3.5 : 0.0);
  double split = none;
  for (int waves = 1; waves <= kTailWaves && left; ++waves) {
    const long long share = std::max<long long>(2, (left * N + kPlanSms * waves - 1) / (kPlanSms * waves));
    const long long f = std::min<long long>(std::max<long long>(N / share, 1), kMaxSplits);
    split = std::min(split, full + 10 + ((left * f + kPlanSms - 1) / kPlanSms) * ((N + f - 1) / f + 3.5));
  }
  // Room for split tiles wherever some number of rows up to T could have them (of four
  // blocks at least), so that a workspace serves every call of no more rows.  At most
  // an SM's share of blocks a unit, and the units that are no longer than it.
  const int room = a->S <= kGroup && N >= 4 ? (kTailWaves + 1) * kPlanSms + 2 * a->H_kv : 0;
  const long long tiles_max = (a->T + seqs * (TT - 1)) / TT;
  if (split < 0.97 * none)
    pl.slots = static_cast<int>(std::min<long long>(room, tiles_max * a->H_kv * std::min(kMaxSplits, N)));
  pl.units = tiles_max * a->H_kv + pl.slots;
  pl.off_opart = kAlign;
  pl.off_lpart = align_up(pl.off_opart + static_cast<size_t>(room) * kRows * a->D * sizeof(float));
  pl.off_slot = align_up(pl.off_lpart + static_cast<size_t>(room) * kRows * sizeof(float));
  pl.bytes = align_up(pl.off_slot + static_cast<size_t>(room) * sizeof(SlotInfo));
  return pl;
}

cudaError_t make_q_map(CUtensorMap *map, const ChunkParams &p, int D) {
  auto fn = tc::encode_fn();
  if (!fn) return cudaErrorNotSupported;
  const cuuint64_t dims[3] = {static_cast<cuuint64_t>(D), static_cast<cuuint64_t>(p.H_q),
                              static_cast<cuuint64_t>(p.T)};
  const cuuint64_t strides[2] = {static_cast<cuuint64_t>(D) * 2, static_cast<cuuint64_t>(p.q_stride) * 2};
  const cuuint32_t box[3] = {64, static_cast<cuuint32_t>(p.G), static_cast<cuuint32_t>(kRows / p.G)};
  const cuuint32_t es[3] = {1, 1, 1};
  const CUresult r = fn(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<__nv_bfloat16 *>(p.q), dims, strides,
                        box, es, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
                        CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  return r == CUDA_SUCCESS ? cudaSuccess : cudaErrorInvalidValue;
}

// Codes of the paged cache: a box is the rows of some consecutive pages of one KV head,
// D bytes each, swizzled as wide as a row is.
inline cudaError_t make_code_map(CUtensorMap *map, const void *base, int D, int H_kv, int num_pages, int box_pages) {
  auto fn = tc::encode_fn();
  if (!fn) return cudaErrorNotSupported;
  const cuuint64_t dims[3] = {static_cast<cuuint64_t>(D), static_cast<cuuint64_t>(H_kv),
                              static_cast<cuuint64_t>(num_pages) * kPage};
  const cuuint64_t strides[2] = {static_cast<cuuint64_t>(D), static_cast<cuuint64_t>(H_kv) * D};
  const cuuint32_t box[3] = {static_cast<cuuint32_t>(D), 1, static_cast<cuuint32_t>(box_pages * kPage)};
  const cuuint32_t es[3] = {1, 1, 1};
  const CUresult r = fn(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 3, const_cast<void *>(base), dims, strides, box, es,
                        CU_TENSOR_MAP_INTERLEAVE_NONE, D == 128 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B,
                        CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  return r == CUDA_SUCCESS ? cudaSuccess : cudaErrorInvalidValue;
}

template <int D, bool kFp8>
cudaError_t launch(const ChunkParams &p, long long units, cudaStream_t s) {
  using L = Layout<D, kFp8>;
  static_assert(L::kDynSmem + sizeof(Shared) <= 227 * 1024, "shared memory");
  CUtensorMap tk, tk4, tv, tv4, tq;
  const int run = std::min(kPagesEach, p.num_pages);  // box never longer than the pool
  cudaError_t e;
  if constexpr (kFp8) {
    e = make_code_map(&tk, p.k_cache, D, p.H_kv, p.num_pages, 1);
    if (e == cudaSuccess) e = make_code_map(&tk4, p.k_cache, D, p.H_kv, p.num_pages, run);
    if (e == cudaSuccess) e = make_code_map(&tv, p.v_cache, D, p.H_kv, p.num_pages, 1);
    if (e == cudaSuccess) e = make_code_map(&tv4, p.v_cache, D, p.H_kv, p.num_pages, run);
    tq = tk;  // (not used)
  } else {
    e = make_q_map(&tq, p, D);
    if (e == cudaSuccess) e = tc::make_page_map(&tk, p.k_cache, D, p.H_kv, p.num_pages);
    if (e == cudaSuccess) e = tc::make_page_map(&tv, p.v_cache, D, p.H_kv, p.num_pages);
    if (e == cudaSuccess) e = tc::make_page_map(&tv4, p.v_cache, D, p.H_kv, p.num_pages, run);
    if (e == cudaSuccess) e = tc::make_page_map(&tk4, p.k_cache, D, p.H_kv, p.num_pages, run);
  }
  int dev = 0;
  if (e == cudaSuccess) e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  static std::atomic<uint64_t> configured{0};
  static std::atomic<int> sms[64];
  const uint64_t bit = 1ull << (dev & 63);
  if (!(configured.load(std::memory_order_acquire) & bit)) {
    int n = 0;
    e = cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev);
    if (e == cudaSuccess)
      e = cudaFuncSetAttribute(chunk_attn_kernel<D, kFp8>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                               static_cast<int>(L::kDynSmem));
    if (e != cudaSuccess) return e;
    sms[dev & 63].store(n);
    configured.fetch_or(bit, std::memory_order_acq_rel);
  }
  const unsigned grid = static_cast<unsigned>(std::min<long long>(units, sms[dev & 63].load()));
  e = launch_kernel(true, chunk_attn_kernel<D, kFp8>, dim3(grid), dim3(kThreads<kFp8>), L::kDynSmem, s, tk, tk4,
                    tv, tv4, tq, p);
  if (e != cudaSuccess || p.slots == 0) return e;
  return launch_kernel(true, chunk_merge_kernel<D>, dim3(p.slots), dim3(32 * kMergeWarps), 0, s, p);
}

// The call with these (checked) arguments; scales: of an 8-bit cache.
template <bool kFp8>
hpd_status run_chunk_attn(const hpd_chunk_attn_args *a, const float *k_scale, const float *v_scale,
                          hpd_stream_t stream) {
  const ChunkPlan pl = make_plan(a);
  uint8_t *ws = static_cast<uint8_t *>(a->workspace);
  ChunkParams k{};
  k.q = static_cast<const __nv_bfloat16 *>(a->q);
  k.q_stride = a->q_stride ? a->q_stride : static_cast<long long>(a->H_q) * a->D;
  k.chunk_cu = a->chunk_cu;
  k.seq_len = a->seq_len;
  k.full_len = a->full_len;
  k.k_cache = a->k_cache;
  k.v_cache = a->v_cache;
  k.k_scale = k_scale;
  k.v_scale = v_scale;
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
  k.err = reinterpret_cast<uint32_t *>(ws);
  k.unit_ctr = reinterpret_cast<int *>(ws + 8);
  k.units = static_cast<int>(pl.units);
  k.slots = pl.slots;
  k.o_part = reinterpret_cast<float *>(ws + pl.off_opart);
  k.l_part = reinterpret_cast<float *>(ws + pl.off_lpart);
  k.slot = reinterpret_cast<SlotInfo *>(ws + pl.off_slot);
  k.n_slots = reinterpret_cast<int *>(ws + 16);
  k.div_G.set(k.G);
  k.div_Hkv.set(k.H_kv);
  k.div_tile.set(kRows / k.G);
  cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  const cudaError_t e = a->D == 64 ? launch<64, kFp8>(k, pl.units, s) : launch<128, kFp8>(k, pl.units, s);
  return e == cudaSuccess ? HPD_OK : record_cuda_error(e);
}

}  // namespace
}  // namespace hpd
