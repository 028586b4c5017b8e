// Shared-prefix attention over a cache held in 4 bits, for rows of bf16 or f32
// (mathematics: k_prefix_attn.cu, work distribution: prefix_sched.cuh, format:
// q4.cuh).
//
// The keys and values go from their packed form in shared memory straight into the
// registers of the products, which are taken transposed so that 16 keys (or dims)
// fill a product's 16 rows and 8 query rows its columns:
//   S^T [keys][rows] = K Q^T     A: K, 16 keys x 16 dims    B: Q^T
//   O^T [dims][rows] = V^T P^T   A: V^T, 16 dims x 16 keys  B: P^T
// (mma m16n8k16, bf16 in, fp32 sums).  In both, what a lane has to bring to A is a
// few whole words of codes, because the contracted index may run in any order:
//   K  lane (r, t) brings the dims [t HD/4, (t + 1) HD/4) of keys r and r + 8;
//   V  the dims [r HD/8, (r + 1) HD/8) of keys 2t, 2t + 1, 2t + 8 and 2t + 9, the
//      words of two keys joined half by half, so that a pair is one dim of two keys.
// Scores become P^T by a transposition of 8 x 8 in registers (movmatrix).
//
// f32 rows: q and the weights are each a sum of three bf16 numbers (3 x 8 bits = the
// 24 of fp32), and every product is three; keys and values are bf16 exactly.
//
// A CTA has eight warps that multiply and one that finds the CTA's segments and
// loads their key blocks (bulk copies of each page's codes and scales into a ring).
// A segment has up to 64 rows; a warp takes 8 of them and, of each key block, every
// (8 / row groups)-th slice of 16 keys.  At its end the warps of the same rows add
// up through shared memory.
//
// Few rows (decoding) leave the values to be unpacked as the work: 3.75 instructions
// for a pair of them (shift, mask and magic number, minus 136, times the scale), half
// of those on the half-rate integer pipe, and one product for 256, beside 0.56 bytes
// of memory a value.  Measured (bf16, 32 heads on 8 of 128): 32 requests of one row
// over 500 to 16000 tokens of their own 95 us in all for 354 MB (3.7 TB/s).  Without
// any work on the blocks that is 76 us: 57 at 6.2 TB/s, 6 until the first block is there
// (lengths, schedule, first segment, page, block: a chain of loads), 12 for the last
// segments' sums and the join.  The other 20 are the multiplying warps': some 430
// instructions for 16 keys, 0.65 of the issue slots and half of the integer pipe.
// Tried and dropped: a fourth stage (nothing), stages given back ahead of the second
// product (100: spills), scores in two chains of products (nothing), eighths in three
// steps a pair (101 for values or both, 98 for keys; they pay in k_prefix_attn_tc.cu), one CTA an SM with twice the registers
// (123), four row tiles a warp for 9 to 64 rows (16 requests of one row over 32K: 90
// us, with one tile 89: products of 8 columns are as slow as unpacking), shifts as
// products in the other pipe (108 to 122).  Rows past 16 an item go to the tensor cores'
// own memory (k_prefix_attn_tc.cu), which takes a block's time whatever its rows.
#include <algorithm>

#include "barrier_wait.cuh"
#include "prefix_sched.cuh"
#include "q4.cuh"

namespace lsp {
namespace {

constexpr int kKeys = kPrefixQ4Keys, kSlice = 16, kSlices = kKeys / kSlice;
constexpr int kWarps = 8, kThreads = 32 * (kWarps + 1);
constexpr int kAhead = 4;                        // segments planned ahead
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kRaise = 8.0f;                   // log2 of the most a weight may exceed 1

template <typename T>
constexpr int kPieces = sizeof(T) == 2 ? 1 : 3;  // bf16 numbers that make up a row's element
template <typename T, int HD>
constexpr int kPerSm = sizeof(T) == 2 ? 2 : 1;   // CTAs of an SM (f32 rows take the registers of two)

template <int HD>
struct Stage {
  static constexpr int kCodes = kKeys * HD / 2, kScales = kKeys * HD / 16;     // bytes of keys or values
  static constexpr int kBytes = 2 * (kCodes + kScales);
  static constexpr int kCount = HD == 128 ? 3 : 6;
  // of a stage: keys' codes, values' codes, keys' scales, values' scales
};

template <int HD>
struct Smem {
  alignas(128) uint8_t ring[Stage<HD>::kCount][Stage<HD>::kBytes];
  float merge[kWarps][8][HD + 4];                // a warp's sums, padded
  float2 merge_ml[kWarps][8];
  uint64_t full[Stage<HD>::kCount], empty[Stage<HD>::kCount], seg_full[kAhead], seg_empty[kAhead], meet;
  struct Planned {
    PrefixSeg g;
    int more;
  } planned[kAhead];
  PrefixSched sched;
  int abort;
};
// behind it: PrefixSeq info[n], int64_t line_base[n + 1]
template <int HD>
size_t smem_bytes(int n) { return sizeof(Smem<HD>) + (size_t)n * (sizeof(PrefixSeq) + sizeof(int64_t)) + sizeof(int64_t) + 128; }

__device__ __forceinline__ float ex2a(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ uint32_t transpose8(uint32_t x) {     // of an 8 x 8 matrix of 16-bit elements
  uint32_t y;
  asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
  return y;
}
// Key of a slice at row m of its tile: neighbours and every other row in different halves of 128 bytes
// (rows of 64 bytes: reads of keys then meet no bank twice, reads of values two at most).
__device__ __forceinline__ int key_at(int m) { return m ^ ((m >> 1) & 1); }

// A value that is the same in all of a warp, as one that the compiler knows to be.
__device__ __forceinline__ int uniform(int x) { return __shfl_sync(0xffffffffu, x, 0); }

// Pairs of x, y as kPieces bf16 numbers each, of falling size.
template <int P>
__device__ __forceinline__ void split_pair(float x, float y, uint32_t* out) {
#pragma unroll
  for (int i = 0; i < P; ++i) {
    out[i] = pack_bf16(x, y);
    if (i + 1 < P) {
      x -= __uint_as_float(out[i] << 16);
      y -= __uint_as_float(out[i] & 0xFFFF0000u);
    }
  }
}

// The warp that plans and loads.
template <int HD>
__device__ __forceinline__ void load_role(const PrefixAttnParams& p, Smem<HD>& sm, const int64_t* line_base, const PrefixSeq* info) {
  using St = Stage<HD>;
  const int lane = threadIdx.x & 31;
  const int run = min(p.page, kKeys), runs = kKeys / run, page_bits = 31 - __clz(p.page);
  const uint32_t codes = run * (HD / 2), scales = run * (HD / 16);
  const int block_codes = p.page * (HD / 2);
  PrefixSegs<Q4Work> segs(p, sm.sched, line_base, info, blockIdx.x);
  PrefixSeg g;
  uint32_t k = 0;
  Place ring = {0, 1};                           // (the first uses wait for nobody)
  bool more, shared = true;
  do {
    more = shared && segs.next_shared(g);
    if (!more) {
      shared = false;
      more = segs.next_own(g);
    }
    if (!tc_wait(smem_u32(&sm.seg_empty[k % kAhead]), ((k / kAhead) & 1) ^ 1, &sm.abort, p.err)) return;
    if (lane == 0) {
      if (more) sm.planned[k % kAhead].g = g;
      sm.planned[k % kAhead].more = more;
      mbar_arrive(smem_u32(&sm.seg_full[k % kAhead]));
    }
    __syncwarp();
    ++k;
    if (!more) break;
    // lane l loads run l of a block
    auto entry = [&](int kb) {
      const int pos = g.k0 + kb * kKeys + lane * run;
      return lane < runs && kb < g.kb1 && pos < g.k_end ? g.tab[pos >> page_bits] : -1;
    };
    int pg = entry(g.kb0);
    for (int kb = g.kb0; kb < g.kb1; ++kb, ring.next(St::kCount)) {
      const int next = entry(kb + 1);
      const int pos = g.k0 + kb * kKeys + lane * run;
      const bool mine = lane < runs && pos < g.k_end, held = mine && pg >= 0 && pg < p.pages;
      const uint32_t bar = smem_u32(&sm.full[ring.stage]);
      if (!tc_wait(smem_u32(&sm.empty[ring.stage]), ring.phase, &sm.abort, p.err)) return;
      uint8_t* at = sm.ring[ring.stage];
      if (mine && !held) {                       // a page of no pool: scales of 0
        set_err(p.err, LSP_DEV_BAD_SEQ);
        for (uint32_t i = 0; i < scales; i += 16) {
          *reinterpret_cast<uint4*>(at + 2 * St::kCodes + lane * scales + i) = make_uint4(0, 0, 0, 0);
          *reinterpret_cast<uint4*>(at + 2 * St::kCodes + St::kScales + lane * scales + i) = make_uint4(0, 0, 0, 0);
        }
        fence_proxy_async_smem();
      }
      const int n = __popc(__ballot_sync(0xffffffffu, held));
      __syncwarp();
      if (lane == 0) mbar_expect_tx(bar, n * 2 * (codes + scales));
      __syncwarp();
      if (held) {
        const int slot = pos & (p.page - 1);
        const int64_t block = (int64_t)pg * p.s_page + (int64_t)g.head * p.s_head;
        const uint32_t dst = smem_u32(at);
        bulk_load(dst + lane * codes, p.k + block + slot * (HD / 2), codes, bar);
        bulk_load(dst + 2 * St::kCodes + lane * scales, p.k + block + block_codes + slot * (HD / 16), scales, bar);
        bulk_load(dst + St::kCodes + lane * codes, p.v + block + slot * (HD / 2), codes, bar);
        bulk_load(dst + 2 * St::kCodes + St::kScales + lane * scales, p.v + block + block_codes + slot * (HD / 16), scales, bar);
      }
      __syncwarp();
      pg = next;
    }
  } while (more);
}

// A warp's part of the products of a segment.
template <typename T, int HD>
__device__ __forceinline__ bool multiply(const PrefixAttnParams& p, Smem<HD>& sm, const PrefixSeg& g, int rg, int kg, int kgs,
                                         Place& ring, float (&o)[HD / 16][4], float2& m_out, float2& l_out) {
  using St = Stage<HD>;
  constexpr int P = kPieces<T>, kQ = HD / 8;     // registers of a row's quarter, of one piece
  constexpr int kWordsK = HD / 32, kWordsV = HD / 64;
  const int lane = threadIdx.x & 31, r = lane >> 2, t = lane & 3;
  const int rows = g.tokens * p.rep;
  const bool live = 8 * rg < rows;
  uint32_t q[P][kQ];
  {
    const int row = 8 * rg + r, tok = row / p.rep;
    const T* from = static_cast<const T*>(p.q) + (int64_t)(g.t0 + tok) * p.q_stride + (int64_t)(g.head * p.rep + row - tok * p.rep) * HD + t * (HD / 4);
#pragma unroll
    for (int i = 0; i < kQ; i += 4) {
      uint32_t x[4] = {0, 0, 0, 0};
      if constexpr (P == 1) {
        if (row < rows) {
          const uint4 y = *reinterpret_cast<const uint4*>(from + 2 * i);
          x[0] = y.x; x[1] = y.y; x[2] = y.z; x[3] = y.w;
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) q[0][i + e] = x[e];
      } else {
#pragma unroll
        for (int e = 0; e < 4; e += 2) {
          float4 y = make_float4(0.f, 0.f, 0.f, 0.f);
          if (row < rows) y = *reinterpret_cast<const float4*>(from + 2 * (i + e));
          uint32_t a[P], b[P];
          split_pair<P>(y.x, y.y, a);
          split_pair<P>(y.z, y.w, b);
#pragma unroll
          for (int k = 0; k < P; ++k) q[k][i + e] = a[k], q[k][i + e + 1] = b[k];
        }
      }
    }
  }
  const float sl = p.scale * kLog2e;
  // keys that rows 2t, 2t + 1 and the warp's first row see (rows past the last: all, and nobody reads them)
  int lim[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int row = 8 * rg + 2 * t + i;
    lim[i] = row < rows ? min(g.see0 + row / p.rep, g.k_end) : INT_MAX;
  }
  const int least = min(g.see0 + 8 * rg / p.rep, g.k_end);
  // maximum of the base-2 scores, the raw score from which on it is raised, sum of the weights
  float m[2] = {-INFINITY, -INFINITY}, reach[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f};
#pragma unroll
  for (int i = 0; i < HD / 16; ++i)
#pragma unroll
    for (int e = 0; e < 4; ++e) o[i][e] = 0.f;
  // where the lane's words and scales lie in a stage: of keys r and r + 8, of values 2t (2t + 8) and 2t + 1 (2t + 9)
  const int ka = key_at(r), kv[2] = {key_at(2 * t), key_at(2 * t + 1)};
  const int k_at = ka * (HD / 2) + t * (HD / 8), ks_at = 2 * St::kCodes + ka * (HD / 16) + (HD == 128 ? t : t >> 1) * 2;
  int v_at[2], vs_at[2];
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    v_at[j] = St::kCodes + kv[j] * (HD / 2) + r * (HD / 16);
    vs_at[j] = 2 * St::kCodes + St::kScales + kv[j] * (HD / 16) + (HD == 128 ? r >> 1 : r >> 2) * 2;
  }
  const uint32_t ring_at = smem_u32(sm.ring), full_at = smem_u32(sm.full), empty_at = smem_u32(sm.empty);
  const uint32_t zero = (uint32_t)p.n >> 31;
  uint32_t read = 0;
  const Q4Consts consts;
  // 16 keys, the first of them key `key` of the sequence, from `codes` and `scales` on; edge: some row does not see some key
  auto slice = [&](uint32_t codes, uint32_t scales, int key, auto edge) {
    constexpr bool kEdge = decltype(edge)::value;
    float s[4] = {0.f, 0.f, 0.f, 0.f};
    {
      uint32_t wa[kWordsK], wb[kWordsK];
      if constexpr (HD == 128) {
        const uint4 x = ld_shared4(codes + k_at), y = ld_shared4(codes + k_at + 8 * (HD / 2));
        wa[0] = x.x; wa[1] = x.y; wa[2] = x.z; wa[3] = x.w;
        wb[0] = y.x; wb[1] = y.y; wb[2] = y.z; wb[3] = y.w;
      } else {
        ld_shared2(codes + k_at, wa[0], wa[1]);
        ld_shared2(codes + k_at + 8 * (HD / 2), wb[0], wb[1]);
      }
      const uint32_t sa = ld_shared_u16(scales + ks_at) * 0x10001u, sb = ld_shared_u16(scales + ks_at + 8 * (HD / 16)) * 0x10001u;
#pragma unroll
      for (int i = 0; i < kWordsK; ++i)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const uint32_t x[4] = {q4_pair(consts, wa[i] >> (8 * h), sa), q4_pair(consts, wb[i] >> (8 * h), sb),
                                 q4_pair(consts, wa[i] >> (8 * h + 4), sa), q4_pair(consts, wb[i] >> (8 * h + 4), sb)};
#pragma unroll
          for (int k = 0; k < P; ++k) mma_bf16(s, x, q[k][4 * i + 2 * h], q[k][4 * i + 2 * h + 1]);
        }
    }
    uint32_t vw[4][kWordsV], sv[4];              // (read while the scores are on their way)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const uint32_t a = codes + v_at[j & 1] + (j >> 1) * 8 * (HD / 2);
      if constexpr (HD == 128)
        ld_shared2(a, vw[j][0], vw[j][1]);
      else
        vw[j][0] = ld_shared(a);
      sv[j] = ld_shared_u16(scales + vs_at[j & 1] + (j >> 1) * 8 * (HD / 16));
      // slots of a page past the last key hold anything: their weights are 0, and 0 x V must be 0
      if (kEdge && key + kv[j & 1] + (j >> 1) * 8 >= g.k_end) sv[j] = 0;
    }
    if (kEdge) {
      // A value that is NaN must not enter the sums of rows that do not see it (0 x NaN): it is left out, and the
      // lane's dims of the rows that see it become NaN.  (Eighths of the others cannot be infinite.)
      bool lost = false;
#pragma unroll
      for (int j = 0; j < 4; ++j) lost |= (sv[j] & 0x7F80u) == 0x7F80u;
      if (__any_sync(0xffffffffu, lost)) {
        uint32_t hit = 0;                        // keys of the slice, of the lane's group of dims
#pragma unroll
        for (int j = 0; j < 4; ++j)
          if ((sv[j] & 0x7F80u) == 0x7F80u) hit |= 1u << (kv[j & 1] + (j >> 1) * 8), sv[j] = 0;
        hit |= __shfl_xor_sync(0xffffffffu, hit, 1);
        hit |= __shfl_xor_sync(0xffffffffu, hit, 2);
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const int seen = lim[i] - key;
          if (seen <= 0 || !(hit & (seen < 16 ? (1u << seen) - 1 : 0xFFFFu))) continue;
#pragma unroll
          for (int d = 0; d < HD / 16; ++d) o[d][i] = o[d][i + 2] = __uint_as_float(0x7FC00000u);
        }
      }
    }
    // rows 2t, 2t + 1 (s[0], s[1]) of key ka, and (s[2], s[3]) of key ka + 8
    if (kEdge) {
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (key + ka + (e & 2) * 4 >= lim[e & 1]) s[e] = -INFINITY;
    }
    // (in raw scores: m is the running maximum, and a row is raised where a score exceeds it by kRaise in base 2)
    const bool raise = fmaxf(s[0], s[2]) > reach[0] || fmaxf(s[1], s[3]) > reach[1];
    if (__any_sync(0xffffffffu, raise)) {
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        float top = fmaxf(s[i], s[i + 2]);
#pragma unroll
        for (int w = 4; w < 32; w <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, w));
        if (!(top > reach[i])) continue;
        top *= sl;
        const float keep = ex2a(m[i] - top);     // (0 for the first)
        m[i] = top;
        reach[i] = (top + kRaise) / sl;
        l[i] *= keep;
#pragma unroll
        for (int d = 0; d < HD / 16; ++d) o[d][i] *= keep, o[d][i + 2] *= keep;
      }
    }
    uint32_t b0[P], b1[P];
    {
      float w[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        w[e] = ex2a(fmaf(s[e], sl, kEdge && m[e & 1] == -INFINITY ? 0.f : -m[e & 1]));
        l[e & 1] += w[e];
        if (kEdge) w[e] *= 8.0f;                 // (for the values' eighths)
      }
      // (bf16: the weights of the product are rounded to 2^-9 of each, their sum is not: the other operand is bf16,
      // and the rounding of the output outweighs it)
      split_pair<P>(w[0], w[1], b0);
      split_pair<P>(w[2], w[3], b1);
#pragma unroll
      for (int k = 0; k < P; ++k) b0[k] = transpose8(b0[k]), b1[k] = transpose8(b1[k]);
    }
    uint32_t sa = sv[0] | sv[1] << 16, sb = sv[2] | sv[3] << 16;
    if (kEdge) {
      sa = bf2_bits(__hmul2(bits_bf2(sa), bits_bf2(0x3E003E00u)));           // (exact: scales are multiples of 2^-130)
      sb = bf2_bits(__hmul2(bits_bf2(sb), bits_bf2(0x3E003E00u)));
    }
    read = sa ^ sb ^ vw[0][0] ^ vw[1][0] ^ vw[2][0] ^ vw[3][0];      // (the keys' words the votes above have needed)
#pragma unroll
    for (int i = 0; i < kWordsV; ++i) {
      const uint32_t lo_a = __byte_perm(vw[0][i], vw[1][i], 0x5410), hi_a = __byte_perm(vw[0][i], vw[1][i], 0x7632);
      const uint32_t lo_b = __byte_perm(vw[2][i], vw[3][i], 0x5410), hi_b = __byte_perm(vw[2][i], vw[3][i], 0x7632);
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const uint32_t x[4] = {q4_pair(consts, lo_a >> (4 * k), sa), q4_pair(consts, hi_a >> (4 * k), sa),
                               q4_pair(consts, lo_b >> (4 * k), sb), q4_pair(consts, hi_b >> (4 * k), sb)};
#pragma unroll
        for (int c = 0; c < P; ++c) mma_bf16(o[4 * i + k], x, b0[c], b1[c]);
      }
    }
  };
  for (int kb = g.kb0; kb < g.kb1; ++kb) {
    if (!tc_wait(full_at + 8 * ring.stage, ring.phase, &sm.abort, p.err)) return false;
    if (live) {
      const uint32_t at = ring_at + ring.stage * St::kBytes;
      const int key0 = g.k0 + kb * kKeys;
      if (key0 + kKeys > least) {
        for (int i = kg; i < kSlices; i += kgs) slice(at + i * kSlice * (HD / 2), at + i * kSlice * (HD / 16), key0 + i * kSlice, BoolTag<true>());
      } else {
        for (int i = kg; i < kSlices; i += kgs) slice(at + i * kSlice * (HD / 2), at + i * kSlice * (HD / 16), key0 + i * kSlice, BoolTag<false>());
      }
    }
    arrive_after_reads(empty_at + 8 * ring.stage, read, zero);
    ring.next(St::kCount);
  }
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int w = 4; w < 32; w <<= 1) l[i] += __shfl_xor_sync(0xffffffffu, l[i], w);
  m_out = make_float2(part_max(make_float2(m[0], l[0])), part_max(make_float2(m[1], l[1])));
  l_out = make_float2(l[0], l[1]);
  return true;
}

template <typename T, int HD>
__device__ __forceinline__ void multiply_role(const PrefixAttnParams& p, Smem<HD>& sm) {
  const int lane = threadIdx.x & 31, warp = uniform(threadIdx.x >> 5), r = lane >> 2, t = lane & 3;
  Place ring = {0, 0};
  uint32_t met = 0;
  // the multiplying warps wait for each other (within the limit of every wait: one of them may have given up)
  auto meet = [&]() {
    __syncwarp();
    if (lane == 0) mbar_arrive(smem_u32(&sm.meet));
    return tc_wait(smem_u32(&sm.meet), met++ & 1, &sm.abort, p.err);
  };
  for (uint32_t k = 0;; ++k) {
    const uint32_t at = k % kAhead;
    if (!tc_wait(smem_u32(&sm.seg_full[at]), (k / kAhead) & 1, &sm.abort, p.err)) break;
    const bool more = uniform(sm.planned[at].more) != 0;
    PrefixSeg g;
    if (more) {
      g = sm.planned[at].g;
      g.head = uniform(g.head), g.t0 = uniform(g.t0), g.tokens = uniform(g.tokens);
      g.k0 = uniform(g.k0), g.kb0 = uniform(g.kb0), g.kb1 = uniform(g.kb1), g.k_end = uniform(g.k_end), g.see0 = uniform(g.see0);
    }
    __syncwarp();
    if (lane == 0) mbar_arrive(smem_u32(&sm.seg_empty[at]));
    if (!more) break;
    const int rows = g.tokens * p.rep;
    const int rgs = rows <= 8 ? 1 : rows <= 16 ? 2 : rows <= 32 ? 4 : 8, kgs = kWarps / rgs;
    const int rg = warp & (rgs - 1), kg = warp / rgs;
    float o[HD / 16][4];
    float2 m, l;
    if (!multiply<T, HD>(p, sm, g, rg, kg, kgs, ring, o, m, l)) break;
    if (r == 0) {
      sm.merge_ml[warp][2 * t] = make_float2(m.x, l.x);
      sm.merge_ml[warp][2 * t + 1] = make_float2(m.y, l.y);
    }
    if (!meet()) break;
    // a warp's sums, at the weight of its maximum among the warps of its rows: lane (r, t) has dims [r HD/8, (r + 1) HD/8)
    // of rows 2t and 2t + 1
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int row = 2 * t + i;
      const float mine = i ? m.y : m.x;
      float top = mine;
      for (int j = 0; j < kgs; ++j) top = max_nan(top, sm.merge_ml[j * rgs + rg][row].x);
      const float f = mine == -INFINITY ? 0.f : ex2a(mine - top);
#pragma unroll
      for (int d0 = 0; d0 < HD / 32; ++d0) {
        const int d = HD == 128 ? d0 ^ (r & 1) : d0;       // (dims 4 d of the lane's; the order keeps lanes off each other's banks)
        float4 x;
        if (d == d0)
          x = make_float4(o[2 * d0][i], o[2 * d0][i + 2], o[2 * d0 + 1][i], o[2 * d0 + 1][i + 2]);
        else
          x = make_float4(o[2 * (d0 ^ 1)][i], o[2 * (d0 ^ 1)][i + 2], o[2 * (d0 ^ 1) + 1][i], o[2 * (d0 ^ 1) + 1][i + 2]);
        x.x *= f; x.y *= f; x.z *= f; x.w *= f;
        *reinterpret_cast<float4*>(&sm.merge[warp][row][r * (HD / 8) + 4 * d]) = x;
      }
    }
    if (!meet()) break;
    // four rows' chunks lie side by side in the workspace: threads go through them in that order
    for (int i = threadIdx.x; i < rgs * 8 * (HD / 4); i += 32 * kWarps) {
      const int row = (i & 3) | (i / HD) << 2, c = (i >> 2) & (HD / 4 - 1);
      if (row >= rows) continue;
      float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
      for (int j = 0; j < kgs; ++j) {
        const float4 y = *reinterpret_cast<const float4*>(&sm.merge[j * rgs + (row >> 3)][row & 7][4 * c]);
        x.x += y.x; x.y += y.y; x.z += y.z; x.w += y.w;
      }
      *part_chunk<HD>(p.part_o, g.part + row, c) = x;
      if (c == 0) {
        float top = -INFINITY, sum = 0.f;
        for (int j = 0; j < kgs; ++j) top = max_nan(top, sm.merge_ml[j * rgs + (row >> 3)][row & 7].x);
        for (int j = 0; j < kgs; ++j) {
          const float2 y = sm.merge_ml[j * rgs + (row >> 3)][row & 7];
          if (y.x != -INFINITY) sum += y.y * ex2a(y.x - top);
        }
        p.part_ml[g.part + row] = make_float2(top, sum);
      }
    }
    if (!meet()) break;                          // the sums are read
  }
}

template <typename T, int HD>
__global__ void __launch_bounds__(kThreads, kPerSm<T, HD>) prefix_attn_q4_kernel(const PrefixAttnParams p) {
  extern __shared__ uint8_t q4_raw[];
  Smem<HD>& sm = *reinterpret_cast<Smem<HD>*>((reinterpret_cast<uintptr_t>(q4_raw) + 127) & ~static_cast<uintptr_t>(127));
  PrefixSeq* info = reinterpret_cast<PrefixSeq*>(&sm + 1);
  int64_t* line_base = reinterpret_cast<int64_t*>(info + p.n);
  const int warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
  if (threadIdx.x == 0) {
    for (int i = 0; i < Stage<HD>::kCount; ++i) {
      mbar_init(smem_u32(&sm.full[i]), 1);
      mbar_init(smem_u32(&sm.empty[i]), kWarps);
    }
    for (int i = 0; i < kAhead; ++i) {
      mbar_init(smem_u32(&sm.seg_full[i]), 1);
      mbar_init(smem_u32(&sm.seg_empty[i]), kWarps);
    }
    mbar_init(smem_u32(&sm.meet), kWarps);
    sm.abort = 0;
    fence_barrier_init();
  }
  griddep_wait();
  griddep_launch();
  if (warp == kWarps) {
    const PrefixSched s = build_sched<Q4Work>(p, line_base, info, blockIdx.x == 0);
    if (lane == 0) sm.sched = s;
  }
  __syncthreads();
  if (warp == kWarps)
    load_role<HD>(p, sm, line_base, info);
  else
    multiply_role<T, HD>(p, sm);
  __syncthreads();
  // Every load has been waited for, unless a wait gave up: then loads may still be landing, and the CTA stays for
  // them (bounded).
  if (*reinterpret_cast<volatile int*>(&sm.abort) && threadIdx.x == 0) {
    const uint64_t t0 = global_ns();
    while (global_ns() - t0 < 1000000ull) {}
  }
  __syncthreads();
}

template <typename T, int HD>
int launch(const PrefixAttnParams& p, cudaStream_t s) {
  static bool set[8] = {};
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess) return LSP_ERR_CUDA;
  if (dev >= 8 || !set[dev]) {
    if (cudaFuncSetAttribute(prefix_attn_q4_kernel<T, HD>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                             (int)smem_bytes<HD>(kPrefixMaxSeqs)) != cudaSuccess)
      return LSP_ERR_CUDA;
    if (dev < 8) set[dev] = true;
  }
  return launch_pdl(prefix_attn_q4_kernel<T, HD>, dim3(p.grid), dim3(kThreads), smem_bytes<HD>(p.n), s, p) == cudaSuccess
             ? LSP_OK
             : LSP_ERR_CUDA;
}

}  // namespace

int prefix_q4_per_sm(int dtype, int d) {
  if (dtype == LSP_DTYPE_BF16) return d == 128 ? kPerSm<bf16, 128> : kPerSm<bf16, 64>;
  return d == 128 ? kPerSm<float, 128> : kPerSm<float, 64>;
}

int launch_prefix_attn_q4(const PrefixAttnParams& p, int dtype, cudaStream_t s) {
  if (dtype == LSP_DTYPE_BF16) return p.d == 128 ? launch<bf16, 128>(p, s) : launch<bf16, 64>(p, s);
  return p.d == 128 ? launch<float, 128>(p, s) : launch<float, 64>(p, s);
}

}  // namespace lsp
