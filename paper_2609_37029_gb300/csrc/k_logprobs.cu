// Log probabilities of given tokens, entropies and the likeliest alternatives of
// rows of logits (contract: include/lsp.h).
//
// With t_v = (z_v - m) log2(e) / T and e_v = 2^t_v, m the row's largest logit:
//   S = sum e_v,  A = sum e_v t_v
//   logprob = (z_token - m) / T - ln S,  entropy = ln 2 (log2 S - A / S)
// One pass: every thread keeps (m, S, A) of its elements and moves them to a higher
// m as 2^t times (S, A + S t).
//
// The k largest, from the same pass: a thread has a stripe of the row (every 256th
// piece of 16 bytes), whose largest logit and its first place it knows at the end.
// Each of the k largest elements is in one of the k stripes whose first are the
// largest -- an element in any other stripe has k elements before it -- so those
// stripes alone are read again (k of 256, mostly from L2), and what comes at or
// before the k-th stripe's first goes to a list, some more than k elements as a
// rule, which is ranked by counting.  Places decide between equal logits all the
// way.  Should the list overflow (a row made for it: thousands of large elements in
// few stripes), the elements are taken one at a time instead, k passes over L2.
//
// A row is split over a cluster of CTAs, whose first joins the parts out of the
// others' shared memory: no workspace, no second launch.
//
// Bound by memory.
#include <algorithm>

#include <cooperative_groups.h>

#include "common.cuh"
#include "lsp_internal.h"

namespace lsp {
namespace {

namespace cg = cooperative_groups;

constexpr int kThreads = 256, kWarps = kThreads / 32;
constexpr int kMaxCluster = 8;
constexpr int kAhead = 4;                        // 16-byte pieces a thread has in flight
constexpr int kList = 1024;                      // candidates of a CTA
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLeast = -150.0f;                // 2^t is 0 from here on
constexpr float kLowest = -3.402823466e38f;

struct Smem {
  unsigned long long list[kList];
  unsigned long long sorted[kLogprobsMaxK];      // of the CTA: key and place, 0: none
  unsigned long long all[kMaxCluster * kLogprobsMaxK];
  uint32_t stripe[kThreads];
  float red[kWarps];
  float2 red2[kWarps];
  unsigned long long best[kWarps];
  uint32_t least[kWarps];
  int count, stripes;
  float m, s, a;
};

__device__ __forceinline__ float ex2a(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ float max_nan(float a, float b) {     // NaN if either is
  float y;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(y) : "f"(a), "f"(b));
  return y;
}

// Whole numbers that order as the logits do (-0 as 0; NaN below all); 0 stands for no element.
__device__ __forceinline__ uint32_t key_of(float x) {
  if (x != x) return 1u;
  const uint32_t u = __float_as_uint(x + 0.0f);
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float of_key(uint32_t k) { return __uint_as_float(k & 0x80000000u ? k & 0x7FFFFFFFu : ~k); }
// Key and place in one: the larger, and of equal ones the first, is the larger.
__device__ __forceinline__ unsigned long long entry(uint32_t key, uint32_t at) { return (unsigned long long)key << 32 | ~at; }

template <typename T>
struct Vec {
  static constexpr int kElems = 16 / (int)sizeof(T);
  __device__ static __forceinline__ void unpack(const uint4& v, float* x) {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if constexpr (sizeof(T) == 2) {
        x[2 * i] = __uint_as_float(w[i] << 16);
        x[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
      } else {
        x[i] = __uint_as_float(w[i]);
      }
    }
  }
  // the largest and the smallest, NaN aside
  __device__ static __forceinline__ void range(const uint4& v, const float* x, float* top, float* low) {
    if constexpr (sizeof(T) == 2) {
      const __nv_bfloat162* p = reinterpret_cast<const __nv_bfloat162*>(&v);
      const __nv_bfloat162 a = __hmax2(__hmax2(p[0], p[1]), __hmax2(p[2], p[3])), b = __hmin2(__hmin2(p[0], p[1]), __hmin2(p[2], p[3]));
      *top = fmaxf(__low2float(a), __high2float(a));
      *low = fminf(__low2float(b), __high2float(b));
    } else {
      *top = fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3]));
      *low = fminf(fminf(x[0], x[1]), fminf(x[2], x[3]));
    }
  }
};

// A CTA's part of a row, in places: the row's elements before its first 16-byte
// boundary (place tid < head), the part's pieces (places kThreads + i), and the
// elements behind the last piece (from place `tail_at` on).  Places rise with the index.
template <typename T>
struct Part {
  const T* z;
  int head, body, first, pieces, tail, tail_at;  // body: index of the row's first piece; first: of the part's, in pieces
  __device__ __forceinline__ uint4 piece(uint32_t place) const {
    return __ldcg(reinterpret_cast<const uint4*>(z + body) + (first + (int)(place - kThreads)));
  }
  __device__ __forceinline__ int index(uint32_t place) const {   // of a place's first element
    if (place < kThreads) return (int)place;
    if (place < (uint32_t)tail_at) return body + (first + (int)(place - kThreads)) * Vec<T>::kElems;
    return tail_index + (int)(place - tail_at);
  }
  int tail_index;
};

struct Scale {
  float c, inv;         // log2(e) / T, its reciprocal
  float large;          // logits up to here leave every t finite
};

// Of a thread's elements: the largest logit and its place, and the sums relative to `m`.
struct Stats {
  float m, best;
  float2 s, a;          // of every other element, to be added
  uint32_t place;
};

// (a0, a1) + b, a b, a + b and a b + c: two fp32 operations an instruction
__device__ __forceinline__ float2 add2s(float a0, float a1, float b) {
  float2 d;
  asm("{\n .reg .b64 x, y;\n mov.b64 x, {%2, %3};\n mov.b64 y, {%4, %4};\n add.rn.f32x2 x, x, y;\n mov.b64 {%0, %1}, x;\n}"
      : "=f"(d.x), "=f"(d.y)
      : "f"(a0), "f"(a1), "f"(b));
  return d;
}
__device__ __forceinline__ float2 mul2s(float2 a, float b) {
  float2 d;
  asm("{\n .reg .b64 x, y;\n mov.b64 x, {%2, %3};\n mov.b64 y, {%4, %4};\n mul.rn.f32x2 x, x, y;\n mov.b64 {%0, %1}, x;\n}"
      : "=f"(d.x), "=f"(d.y)
      : "f"(a.x), "f"(a.y), "f"(b));
  return d;
}
__device__ __forceinline__ float2 add2(float2 a, float2 b) {
  float2 d;
  asm("{\n .reg .b64 x, y;\n mov.b64 x, {%2, %3};\n mov.b64 y, {%4, %5};\n add.rn.f32x2 x, x, y;\n mov.b64 {%0, %1}, x;\n}"
      : "=f"(d.x), "=f"(d.y)
      : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
  return d;
}
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
  float2 d;
  asm("{\n .reg .b64 x, y, z;\n mov.b64 x, {%2, %3};\n mov.b64 y, {%4, %5};\n mov.b64 z, {%6, %7};\n"
      " fma.rn.f32x2 x, x, y, z;\n mov.b64 {%0, %1}, x;\n}"
      : "=f"(d.x), "=f"(d.y)
      : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y), "f"(c.x), "f"(c.y));
  return d;
}

// Elements x, of which top and low are the largest and the smallest (NaN aside).  As
// long as logits stay within +-large, every t is finite, and e t = 0 where e = 0.
// What is below (-inf, a banned token) is raised to where e is 0 already; a row of
// larger numbers takes its steps one by one with t limited.
template <int N>
__device__ __forceinline__ void add_elems(Stats& st, float* x, float top, float low, const Scale& k) {
  if (top > st.m) {
    const float t = max_nan((st.m - top) * k.c, kLeast), r = ex2a(t);
    st.a = make_float2(r * (st.a.x + st.s.x * t), r * (st.a.y + st.s.y * t));
    st.s = make_float2(r * st.s.x, r * st.s.y);
    st.m = top;
  }
  if (!(low > -k.large) || fabsf(st.m) > k.large) {
    if (fabsf(st.m) > k.large) {
#pragma unroll 1
      for (int i = 0; i < N; ++i) {
        float y = x[0];                          // (no indexed registers)
#pragma unroll
        for (int e = 1; e < N; ++e) y = e == i ? x[e] : y;
        const float t = max_nan((y - st.m) * k.c, kLeast), e = ex2a(t);
        st.s.x += e;
        st.a.x = fmaf(e, t, st.a.x);
      }
      return;
    }
    // (200 / c below m; where m's last place is more than that, some of those below)
    const float least = st.m - fmaxf(200.0f * k.inv, fabsf(st.m) * 0x1p-20f);
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] = max_nan(x[i], least);
  }
#pragma unroll
  for (int i = 0; i < N; i += 2) {
    const float2 t = mul2s(add2s(x[i], x[i + 1], -st.m), k.c), e = make_float2(ex2a(t.x), ex2a(t.y));
    st.s = add2(st.s, e);
    st.a = fma2(e, t, st.a);
  }
}

__device__ __forceinline__ void add_one(Stats& st, float x, uint32_t place, const Scale& k) {
  if (x > st.best) st.best = x, st.place = place;
  float pair[2] = {x, -INFINITY};
  add_elems<2>(st, pair, x, -INFINITY, k);
}

__device__ __forceinline__ unsigned long long block_max(unsigned long long v, Smem& sm) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v = max(v, __shfl_xor_sync(0xffffffffu, v, o));
  __syncthreads();
  if (lane == 0) sm.best[warp] = v;
  __syncthreads();
  v = sm.best[lane & (kWarps - 1)];
#pragma unroll
  for (int o = kWarps / 2; o > 0; o >>= 1) v = max(v, __shfl_xor_sync(0xffffffffu, v, o));
  return v;
}

// sm.sorted = the k largest elements of the part (0 where it has fewer).
template <typename T>
__device__ __forceinline__ void part_top(const Part<T>& part, const Stats& st, int k, Smem& sm) {
  constexpr int VE = Vec<T>::kElems;
  const int tid = threadIdx.x;
  const int rounds = (part.pieces + kThreads - 1) / kThreads;    // pieces of a stripe
  const bool some = tid < part.head || tid < part.pieces || tid < part.tail;
  const uint32_t key = some ? key_of(st.best) : 0u;
  if (tid == 0) sm.count = sm.stripes = 0;
  if (tid < k) sm.sorted[tid] = 0;
  // the largest `cut` that k stripes reach, bit by bit; among equal ones, the place that makes them k
  uint32_t cut = 0, last = 0xFFFFFFFFu;
  int reach = kThreads;
  for (uint32_t bit = 1u << 31; bit; bit >>= 1) {
    const int n = __syncthreads_count(key >= (cut | bit));
    if (n >= k) {
      cut |= bit;
      reach = n;
      if (n == k) break;
    }
  }
  if (reach == k) {                              // the least of theirs
    const uint32_t least = __reduce_min_sync(0xffffffffu, key >= cut ? key : 0xFFFFFFFFu);
    if ((tid & 31) == 0) sm.least[tid >> 5] = least;
    __syncthreads();
    cut = __reduce_min_sync(0xffffffffu, sm.least[tid & (kWarps - 1)]);
  } else if (cut > 0) {
    uint32_t below = 0;                          // places < below leave less than k stripes
    for (uint32_t bit = 1u << 31; bit; bit >>= 1) {
      const uint32_t x = below | bit;
      if (__syncthreads_count(key > cut || (key == cut && st.place < x)) < k) below = x;
    }
    last = below;
  }
  auto in = [&](uint32_t e_key, uint32_t place) { return e_key > cut || (e_key == cut && place <= last); };
  if (some && in(key, st.place)) sm.stripe[atomicAdd(&sm.stripes, 1)] = tid;
  __syncthreads();
  const int per = rounds + 2;                    // places of a stripe
  auto put = [&](float x, uint32_t place, int index) {
    const uint32_t e = key_of(x);
    if (!in(e, place)) return;
    const int at = atomicAdd(&sm.count, 1);
    if (at < kList) sm.list[at] = entry(e, (uint32_t)index);
  };
  for (int i = tid; i < sm.stripes * per; i += kThreads) {
    const int stripe = (int)sm.stripe[i / per], j = i % per;
    if (j == 0) {
      if (stripe < part.head) put(to_f(part.z[stripe]), stripe, stripe);
    } else if (j <= rounds) {
      const uint32_t place = (uint32_t)j * kThreads + stripe;
      if ((j - 1) * kThreads + stripe >= part.pieces) continue;
      float x[VE];
      Vec<T>::unpack(part.piece(place), x);
#pragma unroll
      for (int e = 0; e < VE; ++e) put(x[e], place, part.index(place) + e);
    } else if (stripe < part.tail) {
      put(to_f(part.z[part.tail_index + stripe]), part.tail_at + stripe, part.tail_index + stripe);
    }
  }
  __syncthreads();
  const int n = sm.count;
  if (n <= kList) {
    for (int i = tid; i < n; i += kThreads) {
      const unsigned long long mine = sm.list[i];
      int rank = 0;
      for (int j = 0; j < n; ++j) rank += sm.list[j] > mine;
      if (rank < k) sm.sorted[rank] = mine;
    }
    __syncthreads();
    return;
  }
  unsigned long long before = ~0ull;
  for (int r = 0; r < k; ++r) {
    unsigned long long best = 0;
    auto see = [&](float x, int index) {
      const unsigned long long e = entry(key_of(x), (uint32_t)index);
      if (e < before && e > best) best = e;
    };
    if (tid < part.head) see(to_f(part.z[tid]), tid);
    for (int i = tid; i < part.pieces; i += kThreads) {
      float x[VE];
      Vec<T>::unpack(part.piece(kThreads + i), x);
#pragma unroll
      for (int e = 0; e < VE; ++e) see(x[e], part.index(kThreads + i) + e);
    }
    if (tid < part.tail) see(to_f(part.z[part.tail_index + tid]), part.tail_index + tid);
    best = block_max(best, sm);
    if (tid == 0) sm.sorted[r] = best;
    before = best;
    if (best == 0) break;
  }
  __syncthreads();
}

template <typename T>
__global__ void __launch_bounds__(kThreads, 4) logprobs_kernel(const LogprobsParams p, int cluster) {
  constexpr int VE = Vec<T>::kElems;
  __shared__ Smem sm;
  griddep_wait();
  griddep_launch();
  cg::cluster_group group = cg::this_cluster();
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int row = blockIdx.x / cluster, rank = blockIdx.x - row * cluster;
  const int token = p.tokens[row];
  if (token < 0 || token >= p.V) {               // (every CTA of the cluster)
    if (rank > 0) return;
    if (tid < p.k) {
      if (p.top) p.top[(int64_t)row * p.k + tid] = -1;
      if (p.top_logprob) p.top_logprob[(int64_t)row * p.k + tid] = -INFINITY;
    }
    if (tid == 0) {
      p.logprob[row] = -INFINITY;
      if (p.entropy) p.entropy[row] = 0.f;
      if (token != -1) set_err(p.err, LSP_DEV_BAD_TOKEN);
    }
    return;
  }
  const float c = kLog2e / p.temperature;
  const Scale scale = {c, p.temperature * 0.69314718055994531f, 1e38f / fmaxf(c, 1.0f)};
  Part<T> part;
  part.z = static_cast<const T*>(p.z) + (int64_t)row * p.ld;
  const int off = (int)((16 - (reinterpret_cast<uintptr_t>(part.z) & 15)) & 15) / (int)sizeof(T);
  part.body = min(off, p.V);
  const int pieces = (p.V - part.body) / VE, per = (pieces + cluster - 1) / cluster;
  part.first = min(rank * per, pieces);
  part.pieces = min(per, pieces - part.first);
  part.head = rank == 0 ? part.body : 0;
  part.tail_index = part.body + pieces * VE;
  part.tail = rank == cluster - 1 ? p.V - part.tail_index : 0;
  part.tail_at = ((part.pieces + kThreads - 1) / kThreads + 1) * kThreads;
  Stats st = {kLowest, -INFINITY, {0.f, 0.f}, {0.f, 0.f}, 0u};
  // (a thread's first place, for stripes of -inf alone)
  st.place = tid < part.head ? tid : tid < part.pieces ? kThreads + tid : part.tail_at + tid;
  if (tid < part.head) {
    add_one(st, to_f(part.z[tid]), tid, scale);
  }
  for (int i0 = tid; i0 < part.pieces; i0 += kThreads * kAhead) {
    uint4 v[kAhead];
#pragma unroll
    for (int q = 0; q < kAhead; ++q)
      if (i0 + q * kThreads < part.pieces) v[q] = part.piece(kThreads + i0 + q * kThreads);
#pragma unroll
    for (int q = 0; q < kAhead; ++q) {
      if (i0 + q * kThreads >= part.pieces) break;
      float x[VE], top, low;
      Vec<T>::unpack(v[q], x);
      Vec<T>::range(v[q], x, &top, &low);
      if (top > st.best) st.best = top, st.place = kThreads + i0 + q * kThreads;
      add_elems<VE>(st, x, top, low, scale);
    }
  }
  if (tid < part.tail) {
    add_one(st, to_f(part.z[part.tail_index + tid]), part.tail_at + tid, scale);
  }
  // the CTA's sums
  const float wm = warp_max(st.m);
  if (lane == 0) sm.red[warp] = wm;
  __syncthreads();
  float m = sm.red[lane & (kWarps - 1)];
#pragma unroll
  for (int o = kWarps / 2; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
  {
    const float t = max_nan((st.m - m) * c, kLeast), r = ex2a(t);
    const float s = warp_sum(r * (st.s.x + st.s.y)), a = warp_sum(r * (st.a.x + st.a.y + (st.s.x + st.s.y) * t));
    if (lane == 0) sm.red2[warp] = make_float2(s, a);
  }
  __syncthreads();
  if (tid == 0) {
    float s = 0.f, a = 0.f;
    for (int w = 0; w < kWarps; ++w) s += sm.red2[w].x, a += sm.red2[w].y;
    sm.m = m; sm.s = s; sm.a = a;
  }
  if (p.k > 0) part_top<T>(part, st, p.k, sm);
  if (cluster > 1) group.sync(); else __syncthreads();
  if (rank == 0) {
    float top = kLowest;
    for (int r = 0; r < cluster; ++r) top = fmaxf(top, *group.map_shared_rank(&sm.m, r));
    float s = 0.f, a = 0.f;
    for (int r = 0; r < cluster; ++r) {
      const float rs = *group.map_shared_rank(&sm.s, r), t = max_nan((*group.map_shared_rank(&sm.m, r) - top) * c, kLeast), x = ex2a(t);
      s += x * rs;
      a += x * (*group.map_shared_rank(&sm.a, r) + rs * t);
    }
    const bool none = !(s > 0.f) || !isfinite(top);      // no distribution
    const float nan = __uint_as_float(0x7FC00000u), ln_s = logf(s);
    if (tid == 0) {
      p.logprob[row] = none ? nan : (to_f(part.z[token]) - top) / p.temperature - ln_s;
      if (p.entropy) p.entropy[row] = none ? nan : fmaxf(ln_s - a / s * 0.69314718055994531f, 0.f);
    }
    if (p.k > 0) {
      const int n = cluster * p.k;
      for (int i = tid; i < n; i += kThreads) sm.all[i] = group.map_shared_rank(sm.sorted, i / p.k)[i % p.k];
      __syncthreads();
      for (int i = tid; i < n; i += kThreads) {
        const unsigned long long mine = sm.all[i];
        int at = 0;
        if (cluster > 1) {
          for (int j = 0; j < n; ++j) at += sm.all[j] > mine;
        } else {
          at = i;
        }
        if (at >= p.k || mine == 0) continue;    // (k <= V: k elements there are)
        const int64_t to = (int64_t)row * p.k + at;
        if (p.top) p.top[to] = none ? -1 : (int)~(uint32_t)mine;
        if (p.top_logprob) p.top_logprob[to] = none ? nan : (of_key((uint32_t)(mine >> 32)) - top) / p.temperature - ln_s;
      }
    }
  }
  if (cluster > 1) group.sync();                 // the first CTA has read the others' parts
}

// CTAs of a row: enough that they fill the GPU twice over, while each has two rounds of loads.
int choose_cluster(int rows, int V, int es, int num_sms) {
  const int64_t pieces = (int64_t)V * es / 16;
  int n = 1;
  while (n < kMaxCluster && (int64_t)rows * n < 12 * num_sms && pieces > (int64_t)kThreads * n) n *= 2;
  return n;
}

}  // namespace

int launch_logprobs(const LogprobsParams& p, int dtype, int num_sms, cudaStream_t s) {
  const int cluster = choose_cluster(p.rows, p.V, dtype == LSP_DTYPE_BF16 ? 2 : 4, num_sms);
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(p.rows * cluster));
  cfg.blockDim = dim3(kThreads);
  cfg.stream = s;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = cluster;
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  const cudaError_t e = dtype == LSP_DTYPE_BF16 ? cudaLaunchKernelEx(&cfg, logprobs_kernel<bf16>, p, cluster)
                                                : cudaLaunchKernelEx(&cfg, logprobs_kernel<float>, p, cluster);
  return e == cudaSuccess ? LSP_OK : LSP_ERR_CUDA;
}

}  // namespace lsp
