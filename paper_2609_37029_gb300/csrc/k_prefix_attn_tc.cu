// Shared-prefix attention on the tcgen05 tensor cores: bf16, head dim 64 or 128
// (mathematics: k_prefix_attn.cu, work distribution: prefix_sched.cuh).
//
// A persistent CTA per SM works through its segments.  Two "streams" keep two
// score tiles of 128 rows x 128 keys in flight, so that the tensor cores
// multiply for one while the other takes exponentials.  A segment with two row
// tiles gives each stream one, both over every key block; a segment with one
// (few rows: decoding) gives both streams the same rows and alternate key
// blocks, and stream 0 adds the two up at the end.
//
//   warps 0-3, 4-7  streams 0 and 1: thread = row; scores from TMEM, running
//                   maximum and sum, weights rounded to bf16 back to TMEM over
//                   the scores, at the end the sums to the workspace
//   warp 11         plans: what the CTA's segments are, a few ahead of the others
//   warp 8          loads: query tiles, then key and value blocks, page by page
//                   (TMA, 128-byte swizzle), into a ring of tiles
//   warps 9, 10     products of streams 0 and 1: S = Q K^T (both from shared
//                   memory) and O += P V (P from TMEM, V MN-major from shared
//                   memory), one lane issuing
//
// A product of 128 x 128 x 16 takes 64 cycles, the tensor cores queue a handful,
// and a commit waits in line behind them, so every wait of an issuing warp shows
// unless another warp's products run meanwhile: hence a warp for each stream.
// They take turns -- P V of a block and the scores of the next -- because left
// alone the streams drift into step, and then multiply at the same time and take
// exponentials at the same time (32 requests over 128K, when this was chosen: one
// warp for both 0.88 ms, two without turns 1.08, with them 0.87).  P V starts when
// half of the weights are there, for a stream is bound by its chain: scores, their
// maximum, exponentials, P V, the next scores.
//
// Measured: 32 requests of 9 to 17 rows over 128K 757 to 826 us in all (1.46 to 1.33
// PFLOP/s: the clock falls in long runs), 16 of 17 over 32K 133 to 136 us (1.1
// PFLOP/s), 16 of one over 32K 45 us (3.3 TB/s, of which 26 us at 5.7 TB/s; the rest
// is finding the work, the first loads and the join); 4 prompt chunks of 232 to 591
// rows over 2K to 7K tokens in pages of 16 133 us (0.75 PFLOP/s).  In the long ones a
// block of two tiles takes 1.46 us, some 2800 cycles: 2048 of products, and as many
// of shared memory, which the scores (both operands from there) read at its full
// rate while the next keys and values are written.
//
// A stream's order is S(0) PV(0) S(1) PV(1) ...: S(j + 1) overwrites the weights
// that PV(j) reads, and the products of one thread complete in order.  TMEM:
// scores of stream t at columns 128 t, sums at 256 + 128 t.
//
// Over a cache in 4 bits (kQ4; format: q4.cuh) four more warps, 12 to 15, come
// between the loads and the ring: warp 8 copies a tile's codes and scales into one of
// a few places behind it, and the four write its 128 keys as bf16 where TMA would
// have put them, as eighths (three steps a pair; as they are, in four, 156 and 46.5 us
// below): some 700 cycles a tile next to the softmax (75 values a lane and 1000 cycles of
// the products), half of it the integer and 16-bit pipes' own.  16 requests of 17 rows
// over 32K 152 to 161 us (0.94 PFLOP/s); with the unpacking left out 141 where it took
// 153, and what the rest over bf16's 133 is, no run has shown.  16 of one row over 32K
// 41 us; when it took 45, 10 were until the first scores, 21 for 14 blocks, 4 for the
// segment's sums, 10 for the join, and 41 in all with the unpacking left out: the
// softmax's chain bounds the blocks more than the unpacking does.  A tile's way through
// its place, load, unpacking and back, is a chain too: steps in the loading loop show
// (one copy of its code for keys and values instead of five 42.3 -> 41.1 us).
// Tried and dropped: codes straight from memory into registers (the prefetched ones
// hold too few bytes in flight, 512 us), the next tile's words fetched early (spills, or
// nothing gained), places given back before the words are unpacked (nothing), the next
// blocks fetched into L2 (172 and 48), softmax warps without rows standing aside (nothing).
//
// The maximum is raised (and the sums rescaled) only when it would grow by more
// than 2^8, as attention kernels in the literature do: weights stay below 2^8 and
// the sums, in fp32, lose nothing.
#include <algorithm>
#include <type_traits>

#include "barrier_wait.cuh"
#include "prefix_sched.cuh"
#include "q4.cuh"

namespace lsp {
namespace {

constexpr int kRows = kPrefixTcRows, kKeys = kPrefixTcKeys, kTiles = kPrefixTcTiles;
constexpr int kLoadWarp = 8, kMmaWarp = 9, kUnpackWarp = 12;    // the second products' warp and the plan's come between
constexpr int kUnpackWarps = 4;
constexpr size_t kMostSmem = 227 * 1024;         // of a CTA
template <bool kQ4>
constexpr int kThreads = 32 * (kQ4 ? kUnpackWarp + kUnpackWarps : kUnpackWarp);
constexpr int kAhead = 4;                        // segments planned ahead
constexpr int kFirstKeys = 64;                   // keys whose weights are handed over before the rest's (when chosen 0.75 ms over 128K; 32: 0.79, 96: 0.81)
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kRaise = 8.0f;                   // log2 of the most a weight may exceed 1

template <int HD>
struct TcShape {
  static constexpr int kHalves = HD / 64;                    // 128-byte column blocks of a row
  static constexpr uint32_t kHalf = 128 * 128;               // bytes of a column block of a tile
  static constexpr uint32_t kTile = kHalves * kHalf;
  static constexpr int kStages = HD == 128 ? 4 : 8;
  static constexpr uint32_t kRing = kTiles * kTile;          // offset of the ring behind the query tiles
  static constexpr uint32_t kMisc = kRing + kStages * kTile;
};

struct TcMisc {
  uint64_t full[8], empty[8], q_full[2], q_empty[2], s_full[2], p_first[2], p_full[2], o_full[2], o_free[2], turn[2];
  uint64_t seg_full[kAhead], seg_empty[kAhead], lone_full[2], drain;
  uint32_t tmem;
  int abort;
  struct Planned {
    PrefixSeg g;
    int more;
  } planned[kAhead];
  PrefixSched sched;
  float2 lone_ml[2][kRows];                      // stream 1's maximum and sum of segments with one row tile, by turns
  uint64_t packed_full[4], packed_empty[4];      // kQ4: tiles in 4 bits
  int packed_keys[4];                            // keys of one, + kLone where one stream alone takes it; -1: no more tiles
  uint64_t landed;                               // kQ4: a tile that load_packed_role looks through
  int lost;                                      // and whether one of them was changed
};

constexpr int kLone = 256;
// A tile of a cache in 4 bits: codes, then scales.
template <int HD>
struct Packed {
  static constexpr int kCodes = kKeys * HD / 2, kBytes = kCodes + kKeys * HD / 16;
};

// Shared memory: query tiles and ring, TcMisc, places in the line and sequences of the batch, packed tiles.
__host__ __device__ constexpr size_t tc_seqs(int n) { return ((size_t)n * (sizeof(PrefixSeq) + sizeof(int64_t)) + sizeof(int64_t) + 127) & ~(size_t)127; }
template <int HD>
constexpr size_t tc_smem(int n, int packed) {
  return TcShape<HD>::kMisc + ((sizeof(TcMisc) + 127) & ~(size_t)127) + tc_seqs(n) + (size_t)packed * Packed<HD>::kBytes + 1024;
}

__device__ __forceinline__ void tma_load_3d(uint32_t dst, const void* map, uint32_t bar, int x, int y, int z) {
  asm volatile(
      "cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];" ::"r"(dst),
      "l"(reinterpret_cast<uint64_t>(map)), "r"(bar), "r"(x), "r"(y), "r"(z)
      : "memory");
}
__device__ __forceinline__ void tma_load_4d(uint32_t dst, const void* map, uint32_t bar, int x, int y, int z, int w) {
  asm volatile(
      "cp.async.bulk.tensor.4d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5, %6}], [%2];" ::"r"(
          dst),
      "l"(reinterpret_cast<uint64_t>(map)), "r"(bar), "r"(x), "r"(y), "r"(z), "r"(w)
      : "memory");
}

// Shared-memory matrix descriptors of 128-byte swizzled tiles (8-row groups 1024
// bytes apart).  Only the start address differs between the products of a CTA:
// the low word is formed per product (address / 16, plus the offset between
// 64-element blocks of an MN-major operand), the high word is a constant.
constexpr uint32_t kDescHi = (1024u >> 4) | (1u << 14) | (2u << 29);   // group stride, version, 128-byte swizzle
__device__ __forceinline__ uint32_t desc_lo(uint32_t saddr, uint32_t lbo) { return ((saddr & 0x3FFFFu) >> 4) | ((lbo >> 4) << 16); }

// D[tmem] (+)= A[smem] B[smem] and A[tmem] B[smem], bf16 (A in TMEM: two per 32-bit column).
__device__ __forceinline__ void mma_ss(uint32_t d, uint32_t a_lo, uint32_t b_lo, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n .reg .pred p;\n .reg .b64 x, y;\n setp.ne.b32 p, %4, 0;\n mov.b64 x, {%1, %5};\n mov.b64 y, {%2, %5};\n"
      " tcgen05.mma.cta_group::1.kind::f16 [%0], x, y, %3, p;\n}" ::"r"(d),
      "r"(a_lo), "r"(b_lo), "r"(idesc), "r"(accumulate), "r"(kDescHi)
      : "memory");
}
__device__ __forceinline__ void mma_ts(uint32_t d, uint32_t a_tmem, uint32_t b_lo, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n .reg .pred p;\n .reg .b64 y;\n setp.ne.b32 p, %4, 0;\n mov.b64 y, {%2, %5};\n"
      " tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], y, %3, p;\n}" ::"r"(d),
      "r"(a_tmem), "r"(b_lo), "r"(idesc), "r"(accumulate), "r"(kDescHi)
      : "memory");
}

// kind::f16: bf16 A and B, fp32 D, M = 128, N = n; B K-major or MN-major.
__device__ constexpr uint32_t idesc_bf16(int n, bool b_mn) {
  return (1u << 4) | (1u << 7) | (1u << 10) | (b_mn ? (1u << 16) : 0u) | ((uint32_t)(n >> 3) << 17) | ((uint32_t)(kRows >> 4) << 24);
}

#define LSP_R4(v, i) "=r"(v[i]), "=r"(v[i + 1]), "=r"(v[i + 2]), "=r"(v[i + 3])
#define LSP_R16(v, i) LSP_R4(v, i), LSP_R4(v, i + 4), LSP_R4(v, i + 8), LSP_R4(v, i + 12)
#define LSP_T4(v, i) "+r"(v[i]), "+r"(v[i + 1]), "+r"(v[i + 2]), "+r"(v[i + 3])
#define LSP_T16(v, i) LSP_T4(v, i), LSP_T4(v, i + 4), LSP_T4(v, i + 8), LSP_T4(v, i + 12)
#define LSP_I4(v, i) "r"(v[i]), "r"(v[i + 1]), "r"(v[i + 2]), "r"(v[i + 3])
#define LSP_I16(v, i) LSP_I4(v, i), LSP_I4(v, i + 4), LSP_I4(v, i + 8), LSP_I4(v, i + 12)

// 32 lanes x 64 consecutive columns (one row per thread): the values may be used
// after tmem_wait_ld64 of the same registers, which ties them to the wait.
__device__ __forceinline__ void tmem_ld64(uint32_t taddr, uint32_t* r) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x64.b32 {"
      "%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31,"
      "%32,%33,%34,%35,%36,%37,%38,%39,%40,%41,%42,%43,%44,%45,%46,%47,%48,%49,%50,%51,%52,%53,%54,%55,%56,%57,%58,%59,%60,%61,%62,%63"
      "}, [%64];"
      : LSP_R16(r, 0), LSP_R16(r, 16), LSP_R16(r, 32), LSP_R16(r, 48)
      : "r"(taddr)
      : "memory");
}
__device__ __forceinline__ void tmem_wait_ld64(uint32_t* r) {
  asm volatile("tcgen05.wait::ld.sync.aligned;" : LSP_T16(r, 0), LSP_T16(r, 16), LSP_T16(r, 32), LSP_T16(r, 48)::"memory");
}

// 32 lanes x 32 consecutive columns; complete after tmem_wait_st.
__device__ __forceinline__ void tmem_st32(uint32_t taddr, const uint32_t* v) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], {"
      "%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31,%32};" ::"r"(taddr),
      LSP_I16(v, 0), LSP_I16(v, 16)
      : "memory");
}
__device__ __forceinline__ void tmem_st16(uint32_t taddr, const uint32_t* v) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};" ::"r"(taddr),
      LSP_I16(v, 0)
      : "memory");
}
__device__ __forceinline__ void tmem_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

__device__ __forceinline__ float ex2a(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// Maximum of 64 scores of a row (four chains); edge: those from `left` on become -inf.
__device__ __forceinline__ float row_max64(uint32_t* r, int left, bool edge) {
  if (edge) {
#pragma unroll
    for (int c = 0; c < 64; ++c)
      if (c >= left) r[c] = 0xff800000u;
  }
  float b[4];
#pragma unroll
  for (int k = 0; k < 4; ++k) b[k] = fmaxf(__uint_as_float(r[k]), __uint_as_float(r[k + 4]));
#pragma unroll
  for (int c = 8; c < 64; c += 8)
#pragma unroll
    for (int k = 0; k < 4; ++k) b[k] = fmaxf(fmaxf(b[k], __uint_as_float(r[c + k])), __uint_as_float(r[c + k + 4]));
  return fmaxf(fmaxf(b[0], b[1]), fmaxf(b[2], b[3]));
}

// How a segment's key blocks fall to the streams.
struct Jobs {
  bool lone;          // one row tile: the streams take alternate blocks
  int count;          // jobs of both streams
};
__device__ __forceinline__ Jobs seg_jobs(const PrefixAttnParams& p, const PrefixSeg& g) {
  const int blocks = g.kb1 - g.kb0;
  const bool lone = g.tokens <= p.tok_tile;
  return {lone, lone ? blocks : 2 * blocks};
}
__device__ __forceinline__ int stream_jobs(const Jobs& j, int stream) { return (j.count + 1 - stream) >> 1; }
// Places in the ring, from the segment's first tile on: keys and values of its
// block i.  Two row tiles: K0 V0 K1 V1 ...; one: K0 K1 V0 K2 V1 K3 ..., the order
// in which two streams of alternate blocks come to them.
__device__ __forceinline__ uint32_t key_tile(const Jobs& j, int i) { return j.lone ? (i > 0 ? 2 * i - 1 : 0) : 2 * i; }
__device__ __forceinline__ uint32_t value_tile(const Jobs& j, int i) { return j.lone ? i + min(i + 2, j.count) : 2 * i + 1; }

// The plan of the CTA's segments, handed on through shared memory: finding the
// next one takes some 500 cycles, which nobody should spend between two segments.
template <class W>
__device__ __forceinline__ void plan_role(const PrefixAttnParams& p, TcMisc* m, const int64_t* line_base, const PrefixSeq* info) {
  const int lane = threadIdx.x & 31;
  PrefixSegs<W> segs(p, m->sched, line_base, info, blockIdx.x);
  PrefixSeg g;
  uint32_t k = 0;
  auto publish = [&](bool more) {
    if (!tc_wait(smem_u32(&m->seg_empty[k % kAhead]), ((k / kAhead) & 1) ^ 1, &m->abort, p.err)) return false;
    if (lane == 0) {
      if (more) m->planned[k % kAhead].g = g;
      m->planned[k % kAhead].more = more;
      mbar_arrive(smem_u32(&m->seg_full[k % kAhead]));
    }
    __syncwarp();
    ++k;
    return true;
  };
  while (segs.next_shared(g))
    if (!publish(true)) return;
  while (segs.next_own(g))
    if (!publish(true)) return;
  publish(false);
}
// One reader of the plan: every warp of the other roles.
struct SegReader {
  TcMisc* m;
  unsigned* err;
  uint32_t k = 0;
  __device__ __forceinline__ bool next(PrefixSeg& g) {
    const uint32_t at = k % kAhead;
    if (!tc_wait(smem_u32(&m->seg_full[at]), (k / kAhead) & 1, &m->abort, err)) return false;
    const bool more = m->planned[at].more;
    if (more) g = m->planned[at].g;
    __syncwarp();
    if ((threadIdx.x & 31) == 0) mbar_arrive(smem_u32(&m->seg_empty[at]));
    ++k;
    return more;
  }
};

// The query tiles of a segment.
template <int HD>
__device__ __forceinline__ bool load_queries(const PrefixAttnParams& p, const CUtensorMap* mq, uint32_t sm, TcMisc* m,
                                             const PrefixSeg& g, const Jobs& jobs, uint32_t& nq) {
  using Sh = TcShape<HD>;
  const int tiles = jobs.lone ? 1 : 2;
  for (int t = 0; t < tiles; ++t, ++nq) {
    const uint32_t slot = nq & 1, bar = smem_u32(&m->q_full[slot]);
    if (!tc_wait(smem_u32(&m->q_empty[slot]), ((nq >> 1) & 1) ^ 1, &m->abort, p.err)) return false;
    if ((threadIdx.x & 31) == 0) {
      mbar_expect_tx(bar, (uint32_t)(Sh::kHalves * p.tok_tile * p.rep * 128));
      for (int h = 0; h < Sh::kHalves; ++h)
        tma_load_3d(sm + slot * Sh::kTile + h * Sh::kHalf, mq, bar, 64 * h, g.head * p.rep, g.t0 + t * p.tok_tile);
    }
  }
  return true;
}

template <int HD>
__device__ __forceinline__ void load_role(const PrefixAttnParams& p, const CUtensorMap* mq, const CUtensorMap* mk,
                                          const CUtensorMap* mv, uint32_t sm, TcMisc* m, SegReader segs) {
  using Sh = TcShape<HD>;
  const int lane = threadIdx.x & 31;
  const int box = min(p.page, kKeys), boxes = kKeys / box;
  const int page_bits = 31 - __clz(p.page);      // (a power of two)
  uint32_t fill = 0, nq = 0;
  PrefixSeg g;
  while (segs.next(g)) {
    const Jobs jobs = seg_jobs(p, g);
    if (!load_queries<HD>(p, mq, sm, m, g, jobs, nq)) return;
    // lane l loads page l of a block; a page past the keys or outside the pool reads as zeros
    auto entry = [&](int kb) {
      const int pos = g.k0 + kb * kKeys + lane * box;
      int pg = p.pages;
      if (lane < boxes && kb < g.kb1 && pos < g.k_end) {
        pg = __ldg(g.tab + (pos >> page_bits));
        if (pg < 0 || pg >= p.pages) {
          set_err(p.err, LSP_DEV_BAD_SEQ);
          pg = p.pages;
        }
      }
      return pg;
    };
    auto load = [&](const CUtensorMap* map, int kb, int pg) {
      const uint32_t st = fill % Sh::kStages, bar = smem_u32(&m->full[st]);
      if (!tc_wait(smem_u32(&m->empty[st]), ((fill / Sh::kStages) & 1) ^ 1, &m->abort, p.err)) return false;
      if (lane == 0) mbar_expect_tx(bar, Sh::kTile);
      __syncwarp();
      if (lane < boxes) {
        const uint32_t dst = sm + Sh::kRing + st * Sh::kTile + (uint32_t)(lane * box) * 128u;
        const int slot = (g.k0 + kb * kKeys + lane * box) & (p.page - 1);
        for (int h = 0; h < Sh::kHalves; ++h) tma_load_4d(dst + h * Sh::kHalf, map, bar, 64 * h, slot, g.head, pg);
      }
      ++fill;
      return true;
    };
    // first uses: keys lead values by one job (two streams' worth where both take every block)
    const int lead = jobs.lone ? 2 : 1;
    int e0 = entry(g.kb0), e1 = entry(g.kb0 + 1);
    const int blocks = g.kb1 - g.kb0;
    if (!load(mk, g.kb0, e0)) return;
    if (lead == 2 && blocks > 1 && !load(mk, g.kb0 + 1, e1)) return;
    for (int i = 0; i < blocks; ++i) {
      const int e2 = entry(g.kb0 + i + 2);
      if (!load(mv, g.kb0 + i, e0)) return;
      if (i + lead < blocks && !load(mk, g.kb0 + i + lead, lead == 2 ? e2 : e1)) return;
      e0 = e1;
      e1 = e2;
    }
  }
}

// A value that is NaN must not enter the sums of rows that do not see it (0 x NaN): in tiles of which rows see a part, its
// scale becomes 0 here, and spoil_rows makes the sums of the rows that see it NaN.  Scales [from, to) of the tile.
__device__ __forceinline__ void leave_out(uint16_t* scales, int from, int to, int* lost) {
#pragma unroll 1
  for (int x = max(from, 0) + (threadIdx.x & 31); x < to; x += 32)
    if ((scales[x] & 0x7F80) == 0x7F80) {
      scales[x] = 0;
      *lost = 1;
    }
  fence_proxy_async_smem();
  __syncwarp();
}

// Codes and scales of the tiles, in the order of the ring's places, and the query tiles.  Tiles of values that not every
// row sees all of, one or two of a sequence, are waited for and looked through here (16 requests of 17 rows over 32K
// 152 us; code for that in the unpacking or the softmax warps slowed every tile: 158 to 188).
template <int HD>
__device__ __forceinline__ void load_packed_role(const PrefixAttnParams& p, const CUtensorMap* mq, uint32_t sm, uint8_t* packed,
                                                 int count, TcMisc* m, SegReader segs) {
  using Pk = Packed<HD>;
  const int lane = threadIdx.x & 31;
  const int run = min(p.page, kKeys), runs = kKeys / run, page_bits = 31 - __clz(p.page);
  const uint32_t codes = run * (HD / 2), scales = run * (HD / 16);
  const int block_codes = p.page * (HD / 2);
  uint32_t nq = 0, looked = 0;
  Place place = {0, 1};                          // (the first uses wait for nobody)
  PrefixSeg g;
  while (segs.next(g)) {
    const Jobs jobs = seg_jobs(p, g);
    if (!load_queries<HD>(p, mq, sm, m, g, jobs, nq)) return;
    // lane l loads run l of a block
    auto entry = [&](int kb) {
      const int pos = g.k0 + kb * kKeys + lane * run;
      return lane < runs && kb < g.kb1 && pos < g.k_end ? g.tab[pos >> page_bits] : -1;
    };
    auto load = [&](const char* pool, int kb, int pg, bool values) {
      const uint32_t at = place.stage;
      const int first = g.k0 + kb * kKeys, keys = min(g.k_end - first, kKeys), seen = g.see0 - first;
      const bool look = values && seen < keys;
      const uint32_t bar = smem_u32(look ? &m->landed : &m->packed_full[at]);
      const int pos = first + lane * run;
      const bool mine = lane < runs && pos < g.k_end, held = mine && pg >= 0 && pg < p.pages;
      if (!tc_wait(smem_u32(&m->packed_empty[at]), place.phase, &m->abort, p.err)) return false;
      uint8_t* to = packed + at * Pk::kBytes;
      if (mine && !held) {                       // a page of no pool: scales of 0
        set_err(p.err, LSP_DEV_BAD_SEQ);
        for (uint32_t i = 0; i < scales; i += 16) *reinterpret_cast<uint4*>(to + Pk::kCodes + lane * scales + i) = make_uint4(0, 0, 0, 0);
        fence_proxy_async_smem();
      }
      const int n = __popc(__ballot_sync(0xffffffffu, held));
      __syncwarp();
      if (lane == 0) {
        m->packed_keys[at] = keys + (jobs.lone ? kLone : 0);
        mbar_expect_tx(bar, n * (codes + scales));
      }
      __syncwarp();
      if (held) {
        const int slot = pos & (p.page - 1);
        const char* block = pool + (int64_t)pg * p.s_page + (int64_t)g.head * p.s_head;
        bulk_load(smem_u32(to) + lane * codes, block + slot * (HD / 2), codes, bar);
        bulk_load(smem_u32(to) + Pk::kCodes + lane * scales, block + block_codes + slot * (HD / 16), scales, bar);
      }
      if (look) {
        if (!tc_wait(bar, looked++ & 1, &m->abort, p.err)) return false;
        leave_out(reinterpret_cast<uint16_t*>(to + Pk::kCodes), seen * (HD / 32), keys * (HD / 32), &m->lost);
        if (lane == 0) mbar_arrive(smem_u32(&m->packed_full[at]));
      }
      place.next(count);
      return true;
    };
    // first uses: keys lead values by one job (two streams' worth where both take every block)
    const int lead = jobs.lone ? 2 : 1, blocks = g.kb1 - g.kb0;
    int e0 = entry(g.kb0), e1 = entry(g.kb0 + 1), e2 = entry(g.kb0 + 2);         // pages of the blocks from v on
    for (int k = 0, v = 0; v < blocks;) {
      const bool values = k >= blocks || k >= v + lead;
      if (!load(values ? p.v : p.k, g.kb0 + (values ? v : k), values || k == v ? e0 : k == v + 1 ? e1 : e2, values)) return;
      if (values) {
        ++v;
        e0 = e1;
        e1 = e2;
        e2 = entry(g.kb0 + v + 2);
      } else {
        ++k;
      }
    }
  }
  const uint32_t at = place.stage;
  if (!tc_wait(smem_u32(&m->packed_empty[at]), place.phase, &m->abort, p.err)) return;
  if (lane == 0) {
    m->packed_keys[at] = -1;
    mbar_arrive(smem_u32(&m->packed_full[at]));
  }
  __syncwarp();
}

// Tiles from 4 bits to bf16, eighths of the values, 32 keys of each to a warp.  A lane takes two words of codes, 16 dims, at a time: a
// warp's words lie side by side, and eight lanes store to eight different columns of 16 bytes (lanes of the second
// half of a row's dims begin with their second word).
template <int HD>
__device__ __forceinline__ void unpack_role(const PrefixAttnParams& p, int warp, uint8_t* smp, const uint8_t* packed, int count,
                                            TcMisc* m) {
  using Sh = TcShape<HD>;
  using Pk = Packed<HD>;
  constexpr int kPairs = HD / 16, kKeysOf = 32 / kPairs, kSteps = 32 / kKeysOf;  // pairs of words of a key; keys of a step
  const int lane = threadIdx.x & 31, pair = lane & (kPairs - 1), first = 32 * warp + lane / kPairs;
  const bool second = pair >= 4;                 // of the row's halves of 64 dims
  const uint32_t base = smem_u32(packed) + first * (HD / 2) + pair * 8, scale_base = smem_u32(packed) + Pk::kCodes + first * (HD / 16) + (pair >> 1) * 2;
  const uint32_t to = smem_u32(smp) + Sh::kRing + (second ? Sh::kHalf : 0u) + first * 128;
  const int column = (2 * pair & 7) | (second ? 1 : 0);
  const Q4Eighths consts;
  Place place = {0, 0}, ring = {0, 1};
  for (;; place.next(count), ring.next(Sh::kStages)) {
    const uint32_t at = place.stage, st = ring.stage;
    if (!tc_wait(smem_u32(&m->packed_full[at]), place.phase, &m->abort, p.err)) return;
    const int word = m->packed_keys[at], keys = word & (kLone - 1);
    if (word < 0) return;
    uint32_t w[kSteps][2], s[kSteps];
#pragma unroll
    for (int i = 0; i < kSteps; ++i) {
      ld_shared2(base + at * Pk::kBytes + i * kKeysOf * (HD / 2), w[i][0], w[i][1]);
      s[i] = ld_shared_u16(scale_base + at * Pk::kBytes + i * kKeysOf * (HD / 16));
    }
    if (keys < kKeys) {                          // slots of a page past the last key hold anything
#pragma unroll
      for (int i = 0; i < kSteps; ++i)
        if (first + i * kKeysOf >= keys) s[i] = 0;
    }
    if (!tc_wait(smem_u32(&m->empty[st]), ring.phase, &m->abort, p.err)) return;
#pragma unroll
    for (int i = 0; i < kSteps; ++i) {
      const uint32_t scale = s[i] * 0x10001u, row = to + st * Sh::kTile + i * kKeysOf * 128;
      const int key = first + i * kKeysOf;
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        uint32_t x[4];
        q4_eighths(consts, second ? w[i][1 - e] : w[i][e], scale, x);
        st_shared4(row + (((column ^ e ^ key) & 7) << 4), x[0], x[1], x[2], x[3]);
      }
    }
    fence_proxy_async_smem();
    __syncwarp();
    if (lane == 0) {
      if (warp == 0 && word >= kLone) mbar_arrive(smem_u32(&m->empty[st]));      // (for the stream without use for it)
      mbar_arrive(smem_u32(&m->full[st]));
      mbar_arrive(smem_u32(&m->packed_empty[at]));
    }
  }
}

__device__ __forceinline__ bool elect_one() {
  uint32_t e;
  asm volatile("{\n .reg .pred p;\n elect.sync _|p, 0xffffffff;\n selp.u32 %0, 1, 0, p;\n}" : "=r"(e));
  return e != 0;
}
__device__ __forceinline__ int uniform(int x) { return __shfl_sync(0xffffffffu, x, 0); }

// The products of stream t.  The whole warp runs this, in step, and one lane
// issues, so that operands stay in uniform registers (from a single thread's own
// branch a product took 2.7 times as long).  Both streams come to every tile of
// the ring and every query tile in order, and each arrives at it once: when its
// products are done with the tile, or at once where it has no use for it.  So
// neither is ever more than a phase from the other.  (kQ4: where the streams take
// alternate blocks, what a tile's stream alone comes to, the unpacking warps have
// arrived for the other: the ring does not wait for a stream that is busy elsewhere.)
template <int HD, bool kQ4>
__device__ __forceinline__ void mma_role(const PrefixAttnParams& p, int t, uint32_t sm, uint32_t tmem, TcMisc* m,
                                         SegReader segs) {
  using Sh = TcShape<HD>;
  constexpr uint32_t kIdescS = idesc_bf16(kKeys, false), kIdescO = idesc_bf16(HD, true), kTileDesc = Sh::kTile >> 4;
  const uint32_t qd = desc_lo(sm, 16), kd = desc_lo(sm + Sh::kRing, 16), vd = desc_lo(sm + Sh::kRing, Sh::kHalf);
  const uint32_t full = smem_u32(m->full), empty = smem_u32(m->empty), q_full = smem_u32(m->q_full), q_empty = smem_u32(m->q_empty);
  const uint32_t s_full = smem_u32(&m->s_full[t]), p_first = smem_u32(&m->p_first[t]), p_full = smem_u32(&m->p_full[t]);
  const uint32_t o_full = smem_u32(&m->o_full[t]), o_free = smem_u32(&m->o_free[t]);
  const uint32_t ds = tmem + 128u * t, od = ds + 256u;
  uint32_t turns = 0;
  const uint32_t turn = smem_u32(m->turn);
  uint32_t tiles = 0, seen = 0, nq = 0, pp = 0, po = 1;   // ring and query tiles, places passed; phases
  auto wait = [&](uint32_t bar, uint32_t parity) { return tc_wait(bar, parity, &m->abort, p.err); };
  auto landed = [&](uint32_t tile) { return wait(full + 8 * (tile & (Sh::kStages - 1)), (tile / Sh::kStages) & 1); };
  auto pass = [&](uint32_t upto) {               // the other stream's tiles
    if (kQ4) seen = upto;
    for (; seen < upto; ++seen) {
      if (!landed(seen)) return false;
      if (elect_one()) mbar_arrive(empty + 8 * (seen & (Sh::kStages - 1)));
      __syncwarp();
    }
    return true;
  };
  PrefixSeg g;
  while (uniform(segs.next(g))) {
    Jobs jobs = seg_jobs(p, g);
    jobs.lone = uniform(jobs.lone) != 0;
    jobs.count = uniform(jobs.count);
    const int mine = stream_jobs(jobs, t), tiles_q = jobs.lone ? 1 : 2;
    const uint32_t slot = (nq + (jobs.lone ? 0 : t)) & 1;
    for (int x = 0; x < tiles_q; ++x, ++nq) {
      if (!wait(q_full + 8 * (nq & 1), (nq >> 1) & 1)) return;
      if (mine == 0 || (nq & 1) != slot) {
        if (elect_one()) mbar_arrive(q_empty + 8 * (nq & 1));
        __syncwarp();
      }
    }
    uint32_t kst = 0;
    auto keys = [&](int n) {                     // the stream's n-th key tile is there
      const uint32_t kt = tiles + key_tile(jobs, jobs.lone ? 2 * n + t : n);
      kst = kt & (Sh::kStages - 1);
      if (!pass(kt) || !landed(kt)) return false;
      seen = kt + 1;
      return true;
    };
    auto scores = [&]() {
      const uint32_t a = qd + slot * kTileDesc, b = kd + kst * kTileDesc;
#pragma unroll
      for (int s = 0; s < HD / 16; ++s) {
        const uint32_t at = ((uint32_t)(s >> 2) * Sh::kHalf + (uint32_t)(s & 3) * 32u) >> 4;
        mma_ss(ds, a + at, b + at, kIdescS, s > 0 ? 1u : 0u);
      }
    };
    if (mine > 0) {
      if (!keys(0)) return;
      tc_fence_after();
      if (elect_one()) {
        scores();
        umma_commit(s_full);
        umma_commit(empty + 8 * kst);
        if (mine == 1) umma_commit(q_empty + 8 * slot);
      }
      __syncwarp();
    }
    // Turns of P V and the next scores, the two streams' in alternation: what a
    // turn waits for is waited for during the other stream's.
    for (int n = 0; n < (jobs.count + 1) >> 1; ++n, ++turns) {
      const bool on = n + 1 < mine;
      uint32_t vst = 0;
      if (n < mine) {
        const uint32_t vt = tiles + value_tile(jobs, jobs.lone ? 2 * n + t : n);
        vst = vt & (Sh::kStages - 1);
        if (!pass(vt) || !landed(vt)) return;
        seen = vt + 1;
        if (on && !keys(n + 1)) return;
        if (n == 0) {                            // the sums of the segment before are read
          if (!wait(o_free, po)) return;
          po ^= 1;
        }
      }
      if (!wait(turn + 8 * t, (turns & 1) ^ (t == 0 ? 1u : 0u))) return;
      if (n < mine && !wait(p_first, pp)) return;
      tc_fence_after();
      const uint32_t b = vd + vst * kTileDesc;
      if (n < mine) {
        if (elect_one()) {
#pragma unroll
          for (int s = 0; s < kFirstKeys / 16; ++s) mma_ts(od, ds + 8u * s, b + 128u * s, kIdescO, s > 0 || n > 0 ? 1u : 0u);
        }
        __syncwarp();
        if (!wait(p_full, pp)) return;
        pp ^= 1;
        tc_fence_after();
      }
      if (elect_one()) {
        if (n < mine) {
#pragma unroll
          for (int s = kFirstKeys / 16; s < kKeys / 16; ++s) mma_ts(od, ds + 8u * s, b + 128u * s, kIdescO, 1u);
          if (on) scores();
        }
        mbar_arrive(turn + 8 * (t ^ 1));
        if (n < mine) {
          if (on) {
            umma_commit(s_full);
            umma_commit(empty + 8 * kst);
            if (n + 2 == mine) umma_commit(q_empty + 8 * slot);
          } else {
            umma_commit(o_full);
          }
          umma_commit(empty + 8 * vst);
        }
      }
      __syncwarp();
    }
    tiles += 2 * (jobs.lone ? jobs.count : jobs.count >> 1);
    if (!pass(tiles)) return;
  }
}

// The sums of stream t's rows that see a value that leave_out left out become NaN, in its dims: behind all segments, which
// are gone through again.  (Not inlined: 16 requests of 17 rows over 32K 153 us with it between the loops, 152 without.)
template <int HD>
__device__ __noinline__ void spoil_rows(const PrefixAttnParams& p, int t, int row, const PrefixSched& sched, const int64_t* line_base,
                                           const PrefixSeq* info) {
  const float nan = __uint_as_float(0x7FC00000u);
  const int tok = row / p.rep;
  PrefixSegs<TcQ4Work> segs(p, sched, line_base, info, blockIdx.x);
  PrefixSeg g;
  while (segs.next_shared(g)) {}                 // (every row sees all of their keys)
  while (segs.next_own(g)) {
    const bool lone = seg_jobs(p, g).lone;
    const int i = (lone ? 0 : t * p.tok_tile) + tok;
    const bool mine = tok < p.tok_tile && i < g.tokens && (t == 0 || !lone);
    const int64_t at = g.part + (!lone && t ? p.tok_tile * p.rep : 0) + row;
    const int begin = max(g.k0 + g.kb0 * kKeys, g.see0), end = min(g.k0 + g.kb1 * kKeys, g.k_end);
#pragma unroll 1
    for (int group = 0; group < HD / 32; ++group) {
      int first = INT_MAX;
      for (int pos = begin + (threadIdx.x & 31); pos < end; pos += 32) {
        const int pg = g.tab[pos / p.page];
        if (pg < 0 || pg >= p.pages) continue;
        const char* block = p.v + (int64_t)pg * p.s_page + (int64_t)g.head * p.s_head + p.page * (HD / 2);
        const uint16_t s = reinterpret_cast<const uint16_t*>(block)[(pos % p.page) * (HD / 32) + group];
        if ((s & 0x7F80) == 0x7F80) first = min(first, pos);
      }
      first = __reduce_min_sync(0xffffffffu, first);
      if (mine && first < g.see0 + i)
        for (int c = 8 * group; c < 8 * group + 8; ++c) *part_chunk<HD>(p.part_o, at, c) = make_float4(nan, nan, nan, nan);
    }
  }
}

template <int HD, bool kQ4>
__device__ __forceinline__ void softmax_role(const PrefixAttnParams& p, int t, uint8_t* smp, uint32_t tmem, TcMisc* m,
                                             SegReader segs) {
  const int lane = threadIdx.x & 31, quad = (threadIdx.x >> 5) & 3, row = quad * 32 + lane;
  const uint32_t ts = tmem + ((uint32_t)(quad * 32) << 16) + 128u * t, to = ts + 256u;
  const int tok = row / p.rep;
  constexpr float kUnit = kQ4 ? 8.0f : 1.0f;     // (unpacked tiles hold eighths)
  const float sl = kUnit * p.scale * kLog2e;
  uint32_t ns = 0, no = 0, no1 = 0;              // jobs; segments of this stream, of stream 1 (as stream 0 sees them)
  uint32_t lones = 0, tiles = 0;                 // segments that both streams add up; ring tiles of the segments before
  PrefixSeg g;
  while (segs.next(g)) {
    const Jobs jobs = seg_jobs(p, g);
    const int mine = stream_jobs(jobs, t), i = (jobs.lone ? 0 : t * p.tok_tile) + tok;
    const bool valid = tok < p.tok_tile && i < g.tokens;
    const int lim = valid ? min(g.see0 + i, g.k_end) - g.k0 : kKeys * g.kb1;   // keys this row sees, from k0 on
    float mx = -INFINITY, sum = 0.f;             // maximum of the raw scores, sum of the weights
    for (int n = 0; n < mine; ++n) {
      const int kb = g.kb0 + (jobs.lone ? 2 * n + t : n), left = lim - kb * kKeys;
      if (!tc_wait(smem_u32(&m->s_full[t]), ns & 1, &m->abort, p.err)) return;
      ++ns;
      tc_fence_after();
      uint32_t r[128];
      tmem_ld64(ts, r);
      tmem_wait_ld64(r);
      tmem_ld64(ts + 64, r + 64);                // lands while the first half's maximum is taken
      const bool edge = !__all_sync(0xffffffffu, left >= kKeys);
      float b = row_max64(r, left, edge);
      tmem_wait_ld64(r + 64);
      b = fmaxf(b, row_max64(r + 64, left - 64, edge));
      if (n == 0) {
        mx = b;
      } else {
        const bool raise = valid && ((b - mx) * sl > kRaise || (mx == -INFINITY && b > -INFINITY));
        if (__any_sync(0xffffffffu, raise)) {
          // PV of the job before is complete: its product was issued before this score's
          const float keep = !raise || mx == -INFINITY ? 1.f : ex2a((mx - b) * sl);
#pragma unroll 1
          for (int c = 0; c < HD; c += 32) {
            float o[32];
            tmem_ld32(to + c, o);
            uint32_t w[32];
#pragma unroll
            for (int e = 0; e < 32; ++e) w[e] = __float_as_uint(o[e] * keep);
            tmem_st32(to + c, w);
          }
          sum *= keep;
          if (raise) mx = b;
        }
      }
      if (!kQ4 && (jobs.lone || t == 0)) {       // (unpacked tiles have zeros there)
        // slots of a page past the last key hold anything: their weights are 0, and 0 x V must be 0
        // (where both streams use the tile, stream 1's turn comes after stream 0's)
        const int keys = g.k_end - g.k0 - kb * kKeys;
        if (keys < kKeys) {
          const int upto = min(kKeys, (keys + p.page - 1) / p.page * p.page);
          const uint32_t at = tiles + value_tile(jobs, kb - g.kb0), st = at & (TcShape<HD>::kStages - 1);
          // (the ring is past this place's use before: the products have come to this block's keys)
          if (!tc_wait(smem_u32(&m->full[st]), (at / TcShape<HD>::kStages) & 1, &m->abort, p.err)) return;
          uint8_t* v = smp + TcShape<HD>::kRing + st * TcShape<HD>::kTile;
          for (int c = keys * 8 + row; c < upto * 8; c += kRows)
            for (int h = 0; h < TcShape<HD>::kHalves; ++h)
              *reinterpret_cast<uint4*>(v + h * TcShape<HD>::kHalf + c * 16) = make_uint4(0, 0, 0, 0);
          fence_proxy_async_smem();
        }
      }
      const float base = mx == -INFINITY ? 0.f : -mx * sl;
      const float2 sl2 = make_float2(sl, sl), base2 = make_float2(base, base);
      float2 acc[4];
#pragma unroll
      for (int c = 0; c < 4; ++c) acc[c] = make_float2(0.f, 0.f);
#pragma unroll
      for (int h = 0; h < 4; ++h) {
        uint32_t w[16];
#pragma unroll
        for (int c = 0; c < 32; c += 2) {
          const float2 x = fma2(make_float2(__uint_as_float(r[32 * h + c]), __uint_as_float(r[32 * h + c + 1])), sl2, base2);
          const float2 e = make_float2(ex2a(x.x), ex2a(x.y));
          acc[(c >> 1) & 3] = add2(acc[(c >> 1) & 3], e);
          w[c >> 1] = pack_bf16(e.x, e.y);
        }
        // (for the product with V the weights are rounded to the storage type, 2^-9 of each; their sum is not.
        // The other operand is bf16, and an output's own rounding outweighs it: off by 0.0017 of 64 bits in all, 0.0016
        // with fp32 weights, over 32K)
        tmem_st16(ts + 16 * h, w);
        if (32 * (h + 1) == kFirstKeys) {
          tmem_wait_st();
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(smem_u32(&m->p_first[t]));
        }
      }
      acc[0] = add2(add2(acc[0], acc[1]), add2(acc[2], acc[3]));
      sum += acc[0].x + acc[0].y;
      tmem_wait_st();
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(smem_u32(&m->p_full[t]));
    }
    tiles += 2 * (g.kb1 - g.kb0);
    const bool pair = jobs.lone && jobs.count > 1;         // stream 1's part of the same rows is added here
    if (pair) {
      if (t == 1) {
        m->lone_ml[lones & 1][row] = make_float2(mx, sum);
        __syncwarp();
        if (lane == 0) mbar_arrive(smem_u32(&m->lone_full[lones & 1]));
        ++lones;                                 // (at most one segment ahead of stream 0: it frees the sums)
        ++no;
        continue;
      }
    } else if (mine == 0) {
      continue;
    }
    if (!tc_wait(smem_u32(&m->o_full[t]), no & 1, &m->abort, p.err)) return;
    ++no;
    float w0 = 1.f, w1 = 0.f;
    if (t == 0 && jobs.count > 1) {              // (two row tiles: stream 1 waits for its own)
      if (pair) {
        // lone_full first: stream 1 has then waited for its sums of a segment with two row tiles, which stream 0
        // does not, so that o_full[1] is at most one phase behind and its parity tells this segment's from the last
        if (!tc_wait(smem_u32(&m->lone_full[lones & 1]), (lones >> 1) & 1, &m->abort, p.err)) return;
        if (!tc_wait(smem_u32(&m->o_full[1]), no1 & 1, &m->abort, p.err)) return;
        const float2 other = m->lone_ml[lones & 1][row];
        ++lones;
        const float top = fmaxf(mx, other.x);
        w0 = mx == -INFINITY ? 0.f : ex2a((mx - top) * sl);
        w1 = other.x == -INFINITY ? 0.f : ex2a((other.x - top) * sl);
        mx = top;
        sum = sum * w0 + other.y * w1;
        w0 *= kUnit;
        w1 *= kUnit;
      }
      ++no1;
    }
    tc_fence_after();
    const int64_t at = g.part + (!jobs.lone && t ? p.tok_tile * p.rep : 0) + row;
#pragma unroll 1
    for (int c = 0; c < HD; c += 32) {
      float o[32];
      tmem_ld32(to + c, o);
      if (pair) {
        float x[32];
        tmem_ld32(to + 128 + c, x);
#pragma unroll
        for (int e = 0; e < 32; ++e) o[e] = o[e] * w0 + x[e] * w1;
      } else if (kQ4) {
#pragma unroll
        for (int e = 0; e < 32; ++e) o[e] *= kUnit;
      }
      if (c + 32 == HD) {                        // the sums are in registers: the next segment may start
        tc_fence_before();
        __syncwarp();
        if (lane == 0) {
          mbar_arrive(smem_u32(&m->o_free[t]));
          if (pair) mbar_arrive(smem_u32(&m->o_free[1]));
        }
      }
      if (valid) {
#pragma unroll
        for (int e = 0; e < 32; e += 4)
          *part_chunk<HD>(p.part_o, at, (c + e) / 4) = make_float4(o[e], o[e + 1], o[e + 2], o[e + 3]);
      }
    }
    if (valid) p.part_ml[at] = make_float2(mx == -INFINITY ? mx : mx * sl, sum);
  }
}

template <int HD, bool kQ4>
__global__ void __launch_bounds__(kThreads<kQ4>, 1)
    prefix_attn_tc_kernel(const __grid_constant__ CUtensorMap mq, const __grid_constant__ CUtensorMap mk,
                          const __grid_constant__ CUtensorMap mv, const PrefixAttnParams p, int count) {
  using Work = std::conditional_t<kQ4, TcQ4Work, TcWork>;
  extern __shared__ uint8_t tc_raw[];
  uint8_t* smp = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(tc_raw) + 1023) & ~static_cast<uintptr_t>(1023));
  TcMisc* m = reinterpret_cast<TcMisc*>(smp + TcShape<HD>::kMisc);
  PrefixSeq* info = reinterpret_cast<PrefixSeq*>(smp + TcShape<HD>::kMisc + ((sizeof(TcMisc) + 127) & ~(size_t)127));
  int64_t* line_base = reinterpret_cast<int64_t*>(info + p.n);
  uint8_t* packed = reinterpret_cast<uint8_t*>(info) + tc_seqs(p.n);
  const uint32_t sm = smem_u32(smp);
  const int warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31, cta = blockIdx.x;
  if (threadIdx.x == kLoadWarp * 32) {
    for (int i = 0; i < 8; ++i) {
      mbar_init(smem_u32(&m->full[i]), kQ4 ? kUnpackWarps : 1);
      mbar_init(smem_u32(&m->empty[i]), 2);
    }
    for (int i = 0; i < kAhead; ++i) {
      mbar_init(smem_u32(&m->seg_full[i]), 1);
      mbar_init(smem_u32(&m->seg_empty[i]), 11);
    }
    for (int i = 0; i < 4; ++i) {
      mbar_init(smem_u32(&m->packed_full[i]), 1);
      mbar_init(smem_u32(&m->packed_empty[i]), kUnpackWarps);
    }
    for (int i = 0; i < 2; ++i) mbar_init(smem_u32(&m->lone_full[i]), 4);
    mbar_init(smem_u32(&m->drain), 2);
    mbar_init(smem_u32(&m->landed), 1);
    for (int i = 0; i < 2; ++i) {
      mbar_init(smem_u32(&m->turn[i]), 1);
      mbar_init(smem_u32(&m->q_full[i]), 1);
      mbar_init(smem_u32(&m->q_empty[i]), 2);
      mbar_init(smem_u32(&m->s_full[i]), 1);
      mbar_init(smem_u32(&m->p_first[i]), 4);
      mbar_init(smem_u32(&m->p_full[i]), 4);
      mbar_init(smem_u32(&m->o_full[i]), 1);
      mbar_init(smem_u32(&m->o_free[i]), 4);
    }
    m->abort = 0;
    m->lost = 0;
    fence_barrier_init();
    tma_prefetch_desc(&mq);
    if (!kQ4) {
      tma_prefetch_desc(&mk);
      tma_prefetch_desc(&mv);
    }
  }
  if (warp == kMmaWarp) tmem_alloc(smem_u32(&m->tmem), 512);
  griddep_wait();
  griddep_launch();
  if (warp == 0) {
    const PrefixSched sc = build_sched<Work>(p, line_base, info, cta == 0);
    if (lane == 0) m->sched = sc;
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = m->tmem;
  const SegReader segs{m, p.err};
  // registers: 384 threads x 168 at launch = 256 x 200 (softmax) + 128 x 96 and some left over;
  // with the unpacking warps 512 x 128 = 256 x 184 + 256 x 72
  if (warp >= kLoadWarp) {
    if constexpr (kQ4)
      asm volatile("setmaxnreg.dec.sync.aligned.u32 72;");
    else
      asm volatile("setmaxnreg.dec.sync.aligned.u32 96;");
    if (warp == kLoadWarp) {
      if constexpr (kQ4)
        load_packed_role<HD>(p, &mq, sm, packed, count, m, segs);
      else
        load_role<HD>(p, &mq, &mk, &mv, sm, m, segs);
    } else if (kQ4 && warp >= kUnpackWarp)
      unpack_role<HD>(p, warp - kUnpackWarp, smp, packed, count, m);
    else if (warp < kMmaWarp + 2)
      mma_role<HD, kQ4>(p, warp - kMmaWarp, sm, tmem, m, segs);
    else
      plan_role<Work>(p, m, line_base, info);
  } else {
    if constexpr (kQ4)
      asm volatile("setmaxnreg.inc.sync.aligned.u32 184;");
    else
      asm volatile("setmaxnreg.inc.sync.aligned.u32 200;");
    softmax_role<HD, kQ4>(p, warp >> 2, smp, tmem, m, segs);
    if (kQ4 && __any_sync(0xffffffffu, *reinterpret_cast<volatile int*>(&m->lost))) spoil_rows<HD>(p, warp >> 2, threadIdx.x & 127, m->sched, line_base, info);
  }
  tc_fence_before();
  __syncthreads();
  // Every load has been waited for by its product, unless a wait gave up: then
  // loads may still be landing, and the CTA stays for them (bounded).
  if (m->abort && threadIdx.x == 0) {
    const uint64_t t0 = global_ns();
    while (global_ns() - t0 < 1000000ull) {}
  }
  if (warp == kMmaWarp || warp == kMmaWarp + 1) {
    if (elect_one()) umma_commit(smem_u32(&m->drain));
    __syncwarp();
    if (warp == kMmaWarp) {
      if (lane == 0) mbar_wait(smem_u32(&m->drain), 0, p.err);
      __syncwarp();
      tc_fence_after();
      tmem_dealloc(tmem, 512);
    }
  }
  __syncthreads();
}

// The most sequences that leave room for so many packed tiles.
template <int HD>
constexpr int most_seqs(int packed) {
  int n = kPrefixMaxSeqs;
  while (n > 0 && tc_smem<HD>(n, packed) > kMostSmem) --n;
  return n;
}

template <int HD, bool kQ4>
int launch(const PrefixAttnParams& p, cudaStream_t s) {
  static bool set[8] = {};
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess) return LSP_ERR_CUDA;
  if (dev >= 8 || !set[dev]) {
    if (cudaFuncSetAttribute(prefix_attn_tc_kernel<HD, kQ4>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kMostSmem) != cudaSuccess)
      return LSP_ERR_CUDA;
    if (dev < 8) set[dev] = true;
  }
  constexpr int four = most_seqs<HD>(4), three = most_seqs<HD>(3);
  const int packed = !kQ4 ? 0 : p.n <= four ? 4 : p.n <= three ? 3 : 2;
  CUtensorMap mq = {}, mk = {}, mv = {};
  int rc;
  {
    const uint64_t dims[3] = {HD, (uint64_t)p.nq, (uint64_t)p.total}, st[2] = {HD * 2, (uint64_t)p.q_stride * 2};
    const uint32_t box[3] = {64, (uint32_t)p.rep, (uint32_t)p.tok_tile};
    if ((rc = tmap_bf16_sw128(&mq, p.q, 3, dims, st, box)) != LSP_OK) return rc;
  }
  if constexpr (!kQ4) {
    const uint64_t dims[4] = {HD, (uint64_t)p.page, (uint64_t)p.nkv, (uint64_t)p.pages};
    const uint64_t st[3] = {(uint64_t)p.s_slot * 2, (uint64_t)p.s_head * 2, (uint64_t)p.s_page * 2};
    const uint32_t box[4] = {64, (uint32_t)std::min(p.page, kKeys), 1, 1};
    if ((rc = tmap_bf16_sw128(&mk, p.k, 4, dims, st, box)) != LSP_OK || (rc = tmap_bf16_sw128(&mv, p.v, 4, dims, st, box)) != LSP_OK)
      return rc;
  }
  return launch_pdl(prefix_attn_tc_kernel<HD, kQ4>, dim3(p.grid), dim3(kThreads<kQ4>), tc_smem<HD>(p.n, packed), s, mq, mk, mv, p,
                    packed) == cudaSuccess
             ? LSP_OK
             : LSP_ERR_CUDA;
}

}  // namespace

int prefix_tc_q4_seqs(int d) {
  constexpr int wide = most_seqs<128>(2), narrow = most_seqs<64>(2);
  return d == 128 ? wide : narrow;
}

int launch_prefix_attn_tc(const PrefixAttnParams& p, cudaStream_t s) {
  if (p.q4) return p.d == 128 ? launch<128, true>(p, s) : launch<64, true>(p, s);
  return p.d == 128 ? launch<128, false>(p, s) : launch<64, false>(p, s);
}

}  // namespace lsp
