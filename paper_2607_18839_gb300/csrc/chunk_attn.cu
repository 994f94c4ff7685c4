// chunk_attn.cu -- attention of a chunk of new tokens over the paged cache
// (hpd_chunk_attn) on 5th-generation tensor cores.
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
// loads an SM in a call of some 400 blocks an SM.
// Halves of a block for the two softmax warpgroups, and not alternate blocks: those
// took 0.67 us a block with heads of 128 and 0.52 with heads of 64 (three buffers of
// scores, five stages).
#include <algorithm>
#include <atomic>
#include <cmath>

#include "tc_common.cuh"

namespace hpd {
namespace {

using namespace sm100;
using tc::kBlk;
using tc::kRows;

constexpr uint32_t kTmemCols = 512;
constexpr int kPagesPerBlock = kBlk / kPage, kPagesEach = kPagesPerBlock / 2;  // of a producer
constexpr int kProducers = 4;  // warps 0, 1: K; 2, 3: V
constexpr int kQkWarp = 4, kPvWarp = 5, kSchedWarp = 6;
constexpr int kSoftmaxWarp = 8, kSoftmaxWarps = 8;
constexpr int kOutputWarp = kSoftmaxWarp + kSoftmaxWarps, kOutputWarps = 4;
constexpr int kThreads = 32 * (kOutputWarp + kOutputWarps);
// What a pass over a unit does: exponentials against the first block's maxima;
// nothing but the rows' maxima; exponentials against those.
enum Pass { kFirst, kMaxima, kAgain };
constexpr int kMetaSlots = 3;
// of a metadata slot: producers, two MMA issuers, softmax and output warps
constexpr uint32_t kMetaConsumers = kProducers + 2 + kSoftmaxWarps + kOutputWarps;
constexpr int kStages = 3;
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
  const __nv_bfloat16 *k_cache, *v_cache;
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
  int pad;
};
__device__ __forceinline__ UnitMeta read_meta(const UnitMeta &m) {
  UnitMeta r;
#pragma unroll
  for (int i = 0; i < 4; ++i) reinterpret_cast<int4 *>(&r)[i] = reinterpret_cast<const int4 *>(&m)[i];
  return r;
}

template <int D>
struct Layout {
  static constexpr int kChunks = D / 64;                // 64-column (128-byte) boxes
  static constexpr uint32_t kChunkBytes = kRows * 128;  // 128 rows x 128 bytes
  static constexpr uint32_t kTileBytes = kChunks * kChunkBytes;
  // a block's pages: 8-key groups of kChunks x 1024 bytes
  static constexpr uint32_t kGroupBytes = kChunks * 1024, kPageBytes = 2 * kGroupBytes;
  static constexpr uint32_t kK = 0;
  static constexpr uint32_t kV = kK + kStages * kTileBytes;
  static constexpr uint32_t kStage = kV + kStages * kTileBytes;  // 128 bytes of each output row
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
  uint64_t k_full[kStages], v_full[kStages], k_empty[kStages], v_empty[kStages];
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
  unsigned redo;            // units (by number in this CTA, modulo 32) to run once more
  int units_done;           // output warps that looked at a unit's output
  uint32_t sieved[kMetaSlots][128];  // what sieve_block found in the unit of the slot, by column
  int sieved_seq;                    // units of which that is complete
  int unit_id[32];          // the last units issued
  UnitMeta meta[kMetaSlots];
  // the scheduler's group of sequences: units before each, first rows, rows, lengths,
  // keys that all their rows see, tiles left whole, splits of the others
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
  using L = Layout<D>;
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

template <int D>
__global__ void __launch_bounds__(kThreads, 1)
    chunk_attn_kernel(const __grid_constant__ CUtensorMap tm_k, const __grid_constant__ CUtensorMap tm_k4,
                      const __grid_constant__ CUtensorMap tm_v, const __grid_constant__ CUtensorMap tm_v4,
                      const __grid_constant__ CUtensorMap tm_q, const ChunkParams p) {
  using L = Layout<D>;
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
    for (int s = 0; s < kStages; ++s) {
      mbar_init(bar(sh.k_full[s]), 2);
      mbar_init(bar(sh.v_full[s]), 2);
      mbar_init(bar(sh.k_empty[s]), 1);
      mbar_init(bar(sh.v_empty[s]), 1);
    }
    for (int s = 0; s < kMetaSlots; ++s) {
      mbar_init(bar(sh.meta_full[s]), 1);
      mbar_init(bar(sh.meta_empty[s]), kMetaConsumers);
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
    auto load_group = [&](int s0, int units_before) {
      g0 = s0;
      before = units_before;
      const int count = min(kGroup, p.S - s0);
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
      auto tiles_of = [&](int i) { return i < count ? p.div_tile(sh.g_n[i] + TT - 1) : 0; };
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
          blocks += static_cast<float>(n - whole_of(i, n)) * ceil_div_i(sh.g_len[i], kBlk) * p.H_kv;
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
          const int f = n > w ? min(max(ceil_div_i(sh.g_len[i], kBlk) / per, 1), kMaxSplits) : 1;
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
        const int c0 = sh.g_cu[lo], n = sh.g_n[lo], len = sh.g_len[lo], full = sh.g_full[lo];
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
          M.seq = g0 + lo;
          M.tok0 = c0 + i0;
          M.nrows = nrows;
          M.lim0 = lim0;
          M.full = full;
          M.L = len;
          M.pages = ceil_div_i(kmax, kPage);
          M.blk_lo = blk_lo;
          M.n_blocks = blk_hi - blk_lo;
          M.pass = pass;
          sh.unit_id[k & 31] = u;
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
      prefetch_tmap(&tm_q);
      prefetch_tmap(is_k ? &tm_k : &tm_v);
      prefetch_tmap(is_k ? &tm_k4 : &tm_v4);
    }
    __syncwarp();
    pdl_wait();
    uint64_t *const full = is_k ? sh.k_full : sh.v_full, *const empty = is_k ? sh.k_empty : sh.v_empty;
    const CUtensorMap *const page_map = is_k ? &tm_k : &tm_v, *const run_map = is_k ? &tm_k4 : &tm_v4;
    const uint32_t ring = sbase + (is_k ? L::kK : L::kV), mine = half * (L::kTileBytes / 2);
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
      for (int j = is_k ? -1 : 0; j < M.n_blocks; ++j) {
        const int e = issued, s = e % kStages;
        if (e >= kStages && !(ok = wait_bar(empty[s], ((e / kStages) - 1) & 1))) break;
        ++issued;
        const uint32_t dst = ring + s * L::kTileBytes, b = bar(full[s]);
        if (j < 0) {  // the unit's Q tile, 64 columns a warp
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
        mbar_arrive_expect_tx_elect(b, L::kTileBytes / 2);
        const int right = __shfl_down_sync(0xffffffffu, pg, 1);
        const unsigned run = __ballot_sync(0xffffffffu, lane < kPagesEach - 1 && right == pg + 1);
        const bool one = p.num_pages >= kPagesEach && (run & 7u) == 7u;
        if (lane < (one ? 1 : kPagesEach))
          tma_load_5d(dst + mine + lane * L::kPageBytes, one ? run_map : page_map, b, 0, 0, 0, 2 * pg, M.g);
        __syncwarp();
      }
    }
    if (!ok && lane == 0) set_abort(sh, p.err);
    // no exit while a copy into this CTA's shared memory is in flight
    for (int e = max(0, issued - kStages); e < issued; ++e)
      mbar_wait(bar(full[e % kStages]), (e / kStages) & 1);
  } else if (warp == kQkWarp) {
    // ---------------------------------------------------- Q K^T issuer --
    // The MMA warps run their loops with warp-uniform values; one elected lane
    // issues each group of MMAs and its commits.
    constexpr uint32_t idesc_qk = idesc_bf16_f32(kRows, kBlk, false);
    const uint64_t dq0 = smem_desc_sw128(sbase + L::kK, 16, 1024);
    const uint64_t dk0 = smem_desc_sw128(sbase + L::kK, 16, L::kGroupBytes);
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
      for (int j = -1; j < nb; ++j) {
        if (!(ok = wait_bar(sh.k_full[sk], pk))) break;
        // the S buffer is free for what is issued behind P V of the block before last
        if (j >= 0 && jg >= 2 && !(ok = wait_bar(sh.s_free[jg & 1], ((jg >> 1) - 1) & 1))) break;
        tc_fence_after();
        if (issuer) {
          const uint32_t off = (sk * L::kTileBytes) >> 4;
          if (j < 0) {
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
    constexpr uint32_t idesc_pv = idesc_bf16_f32(kRows, D, true);
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
        if (++sv == kStages) {
          sv = 0;
          pv ^= 1u;
        }
        ++jg;
      }
      ++outputs;
      if (pass == kAgain) publish_seq(&sh.sieved_seq, k + 1);
    }
    if (!ok && lane == 0) set_abort(sh, p.err);
  } else if (warp >= kOutputWarp) {
    // ---------------------------------------------------------- output --
    const int quad = warp & 3;          // TMEM lane quadrant this warp may access
    const int r_in = quad * 32 + lane;  // row within the tile
    const uint32_t o_addr = tmem + (static_cast<uint32_t>(quad * 32) << 16) + L::kColO;
    const uint32_t stage = sbase + L::kStage + quad * 32 * 128;  // of this warp's rows
    pdl_wait();
    const int rt = p.div_G(r_in);
    int outputs = 0;
    bool ok = true;
    for (int k = 0; ok; ++k) {
      const int slot = k % kMetaSlots;
      if (!(ok = wait_bar(sh.meta_full[slot], (k / kMetaSlots) & 1))) break;
      const UnitMeta &M = sh.meta[slot];
      if (!M.valid) break;
      if (!(ok = wait_bar(sh.sums[slot], (k / kMetaSlots) & 1))) break;
      const int pass = M.pass, nrows = M.nrows, nsplit = M.nsplit;
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
        inv = l == 0.f ? 0.f : __fdividef(1.f, l);  // (a sum that is NaN stays one; others are below 2^126)
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
          for (int c = 0; c < 64; c += 32) {
            uint32_t o[32];
            if (!idle) {
              tmem_ld32(o_addr + half * 64 + c, o);
              tmem_ld_wait32(o);
            }
            if (half == D / 64 - 1 && c == 32) {  // O may be overwritten once every warp has read it
              tc_fence_before();
              __syncwarp();
              if (lane == 0) mbar_arrive(bar(sh.o_empty));
            }
            if (idle) continue;
#pragma unroll
            for (int e = 0; e < 32; e += 2) {
              const float2 v = make_float2(__uint_as_float(o[e]), __uint_as_float(o[e + 1]));
              finite = __ffma2_rn(v, make_float2(0.f, 0.f), finite);
              const float2 x = __fmul2_rn(v, make_float2(inv, inv));
              o[e] = __float_as_uint(x.x);
              o[e + 1] = __float_as_uint(x.y);
              keep[(c + e) / 2] = pack_bf16x2(x.x, x.y);
            }
            if (part && valid) {
#pragma unroll
              for (int e = 0; e < 32; e += 8) st_global_v8(part + half * 64 + c + e, o + e);
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
              atomicOr(&sh.redo, 1u << (k & 31));
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
      if (lane == 0) mbar_arrive(bar(sh.meta_empty[slot]));
      const int nb = M.n_blocks, blk_lo = M.blk_lo, pass = M.pass;
      const bool idle = quad * 32 >= M.nrows;
      // (rows that are no query count as seeing everything, so that their warp
      // needs no masks for them; their results are not stored)
      const int lim = r_in < M.nrows ? min(max(M.lim0 + rt, M.full), M.L) : 1 << 30;
      // blocks of the unit that every row of the warp sees all of
      const int n_plain = sl2 > 0.f ? min(max(__reduce_min_sync(0xffffffffu, lim), 0) / kBlk - blk_lo, nb) : 0;
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
          if (!(ok = await_s())) break;
          const int hi = min(lim - (blk_lo + j) * kBlk, kBlk) - h * 64;
          mx_run = fmaxf(mx_run, row_max(t_lane + L::col_s(jg & 1) + h * 64, 32, j < n_plain, hi, sl2));
          publish(0);
          publish(1);
        }
      } else {
        if (!(ok = await_s())) break;
        if (pass == kFirst)
          m_run = row_max(t_lane + L::col_s(jg & 1), 64, n_plain > 0, min(lim - blk_lo * kBlk, kBlk), sl2);
        // (scores of -inf alone give no base to a row that sees the unit's keys)
        inside = pass != kFirst || m_run > NEG_INF || lim <= blk_lo * kBlk;
        // blocks that every row of the warp sees all of: nothing to decide
        for (; j < n_plain; ++j, ++jg) {
          if (j > 0 && !(ok = await_s())) break;
          inside &= softmax_plain(t_lane + L::col_s(jg & 1) + h * 64, sl2, m_run, l4, publish);
        }
        if (!ok) break;
        for (; j < nb; ++j, ++jg) {
          if (j > 0 && !(ok = await_s())) break;
          const int hi = min(lim - (blk_lo + j) * kBlk, kBlk) - h * 64;
          inside &= softmax_masked(t_lane + L::col_s(jg & 1) + h * 64, hi, sl2, m_run, l4, publish);
        }
      }
      if (!ok) break;
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

template <int D>
cudaError_t launch(const ChunkParams &p, long long units, cudaStream_t s) {
  using L = Layout<D>;
  static_assert(L::kDynSmem + sizeof(Shared) <= 227 * 1024, "shared memory");
  CUtensorMap tk, tk4, tv, tv4, tq;
  const int run = std::min(kPagesEach, p.num_pages);  // box never longer than the pool
  cudaError_t e = make_q_map(&tq, p, D);
  if (e == cudaSuccess) e = tc::make_page_map(&tk, p.k_cache, D, p.H_kv, p.num_pages);
  if (e == cudaSuccess) e = tc::make_page_map(&tv, p.v_cache, D, p.H_kv, p.num_pages);
  if (e == cudaSuccess) e = tc::make_page_map(&tv4, p.v_cache, D, p.H_kv, p.num_pages, run);
  if (e == cudaSuccess) e = tc::make_page_map(&tk4, p.k_cache, D, p.H_kv, p.num_pages, run);
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
      e = cudaFuncSetAttribute(chunk_attn_kernel<D>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                               static_cast<int>(L::kDynSmem));
    if (e != cudaSuccess) return e;
    sms[dev & 63].store(n);
    configured.fetch_or(bit, std::memory_order_acq_rel);
  }
  const unsigned grid = static_cast<unsigned>(std::min<long long>(units, sms[dev & 63].load()));
  e = launch_kernel(true, chunk_attn_kernel<D>, dim3(grid), dim3(kThreads), L::kDynSmem, s, tk, tk4, tv, tv4, tq, p);
  if (e != cudaSuccess || p.slots == 0) return e;
  return launch_kernel(true, chunk_merge_kernel<D>, dim3(p.slots), dim3(32 * kMergeWarps), 0, s, p);
}

}  // namespace
}  // namespace hpd

extern "C" {

size_t hpd_chunk_attn_workspace_size(const hpd_chunk_attn_args *a) {
  return hpd::check_scalars(a) == HPD_OK ? hpd::make_plan(a).bytes : 0;
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
  const ChunkPlan pl = make_plan(a);
  if (!a->workspace || (reinterpret_cast<uintptr_t>(a->workspace) & (kAlign - 1)) != 0 ||
      a->workspace_bytes < pl.bytes)
    return HPD_ERR_WORKSPACE;
  uint8_t *ws = static_cast<uint8_t *>(a->workspace);
  ChunkParams k{};
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
  const cudaError_t e = a->D == 64 ? launch<64>(k, pl.units, s) : launch<128>(k, pl.units, s);
  return e == cudaSuccess ? HPD_OK : record_cuda_error(e);
}

}  // extern "C"
