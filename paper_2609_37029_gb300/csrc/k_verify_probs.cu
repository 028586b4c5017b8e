// Acceptance of drafted tokens from given probabilities and random numbers
// (Sec. 2.1, Eq. acceptance, Eq. residual): y_i is accepted iff
// u_i q_i(y_i) < p_i(y_i); the next token is argmax_v w_v / e_v with
// w = [p - q]_+ at the first rejected position, w = p after the last accepted
// one.  With e_v ~ Exp(1) independent, argmax w_v / e_v falls on v with
// probability w_v / sum w (the smallest of exponentials of rates w_v), so no
// row is ever normalised and every score is one fp32 subtraction and one
// correctly rounded division: the decision does not depend on how the
// vocabulary is split.
//
// One launch, one cluster of CTAs per request.  Every CTA makes the few
// acceptance tests itself (lane i of warp 0 tests candidate i), scans its slice
// of the one row that decides (p, q, e), and the CTAs exchange their best
// (score, index) through distributed shared memory.  No workspace, no atomics.
//
// 4 requests of 32001 entries take 5.6 us: launch, and the chain token -> p, q ->
// row -> exchange.  16 of 151936 entries: 10.6 us for 29 MB, 64 with 16-bit
// probabilities and drafts without a distribution: 17.4 us for 58 MB (3.4 TB/s);
// the rounds of loads of a slice bound it, two CTAs of 512 threads on an SM.
#include <cooperative_groups.h>

#include <algorithm>
#include <climits>
#include <utility>

#include "common.cuh"
#include "lsp_internal.h"

namespace lsp {
namespace {

namespace cg = cooperative_groups;

constexpr int kVpThreads = 512;
constexpr int kVpMaxCluster = 8;                 // CTAs per request at most (16 requests: 10.6 us with 8, 15.9 with 16)
constexpr unsigned kAll = 0xffffffffu;

__device__ __forceinline__ bool better(float v, int i, float bv, int bi) { return v > bv || (v == bv && i < bi); }

// VEC consecutive values as they lie in memory (one load), and as fp32
template <typename T, int VEC>
struct Vals {
  static constexpr int kRegs = sizeof(T) * VEC < 4 ? 1 : (int)sizeof(T) * VEC / 4;
  uint32_t w[kRegs];
  __device__ __forceinline__ void load(const T* p) {
    if constexpr (VEC == 1) {
      w[0] = sizeof(T) == 4 ? __ldg(reinterpret_cast<const uint32_t*>(p)) : (uint32_t)__ldg(reinterpret_cast<const uint16_t*>(p));
    } else if constexpr (sizeof(T) == 4) {
      const uint4 v = __ldg(reinterpret_cast<const uint4*>(p));
      w[0] = v.x; w[1] = v.y; w[2] = v.z; w[3] = v.w;
    } else {
      const uint2 v = __ldg(reinterpret_cast<const uint2*>(p));
      w[0] = v.x; w[1] = v.y;
    }
  }
  __device__ __forceinline__ void zero() {
#pragma unroll
    for (int k = 0; k < kRegs; ++k) w[k] = 0;
  }
  __device__ __forceinline__ float get(int j) const {
    if constexpr (sizeof(T) == 4) return __uint_as_float(w[j]);
    return __uint_as_float(j & 1 ? w[j >> 1] & 0xffff0000u : w[j >> 1] << 16);
  }
};

__device__ __noinline__ float quotient(float w, float e) { return __fdiv_rn(w, e); }

// kQ: subtract the row q, or drop the one token `skip` (a point mass; -1: none).
// Few entries can still win once some have been seen, and a correctly rounded
// division takes longer than all the rest: an entry is only divided if w >= e
// times the warp's best so far, less 2^-19 of it for the roundings (and always
// where the best or the product is tiny or no number).
template <typename T, int VEC, bool kQ>
__device__ __forceinline__ void scan_row(const T* p, const T* q, const float* e, int skip, int g0, int g1, float& bv, int& bi) {
  // loads in flight: what some 32 registers hold
  constexpr int kBatch = VEC == 1 ? 8 : 32 / ((kQ ? 2 : 1) * Vals<T, VEC>::kRegs + VEC);
  float bound = -1.f;
  for (int first = g0; first < g1; first += kBatch * kVpThreads) {     // the same count for the whole CTA
    const int base = first + threadIdx.x;
    Vals<T, VEC> a[kBatch], b[kBatch];
    Vals<float, VEC> x[kBatch];
#pragma unroll
    for (int k = 0; k < kBatch; ++k) {
      const int g = base + k * kVpThreads;
      a[k].zero();
      if (kQ) b[k].zero();
      x[k].zero();
      if (g < g1) {
        a[k].load(p + (size_t)g * VEC);
        if (kQ) b[k].load(q + (size_t)g * VEC);
        x[k].load(e + (size_t)g * VEC);
      }
    }
#pragma unroll
    for (int k = 0; k < kBatch; ++k) {
      const int v0 = (base + k * kVpThreads) * VEC;
      bool any = false;
      float w[VEC];
#pragma unroll
      for (int j = 0; j < VEC; ++j) {
        w[j] = kQ ? a[k].get(j) - b[k].get(j) : a[k].get(j);
        if (!kQ && v0 + j == skip) w[j] = 0.f;
        const float least = bound * x[k].get(j);
        any |= w[j] > 0.f && (!(w[j] < least) || !(least > 1e-36f));
      }
      if (any) {
#pragma unroll
        for (int j = 0; j < VEC; ++j)
          if (w[j] > 0.f) {
            const float sc = quotient(w[j], x[k].get(j));
            // indices rise within a thread: a strict > keeps the lowest on ties
            if (sc > bv) { bv = sc; bi = v0 + j; }
          }
      }
    }
    float top = bv;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(kAll, top, o));
    bound = top > 1e-30f ? top * (1.f - 1.9073486328125e-06f) : -1.f;
  }
}

// Best of the cluster; every CTA gets it.  s_val, s_idx: a slot for each of its CTAs.
__device__ __forceinline__ void cluster_best(cg::cluster_group cl, float& v, int& i, float* s_val, int* s_idx, float* w_val,
                                             int* w_idx) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    const float ov = __shfl_xor_sync(kAll, v, o);
    const int oi = __shfl_xor_sync(kAll, i, o);
    if (better(ov, oi, v, i)) { v = ov; i = oi; }
  }
  if (lane == 0) { w_val[warp] = v; w_idx[warp] = i; }
  __syncthreads();
  if (warp == 0) {
    v = lane < kVpThreads / 32 ? w_val[lane] : -1.f;
    i = lane < kVpThreads / 32 ? w_idx[lane] : INT_MAX;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
      const float ov = __shfl_xor_sync(kAll, v, o);
      const int oi = __shfl_xor_sync(kAll, i, o);
      if (better(ov, oi, v, i)) { v = ov; i = oi; }
    }
    const int me = (int)cl.block_rank();
    if (lane < (int)cl.num_blocks()) {
      cl.map_shared_rank(s_val, lane)[me] = v;
      cl.map_shared_rank(s_idx, lane)[me] = i;
    }
  }
  cl.sync();
  v = s_val[0];
  i = s_idx[0];
  for (int k = 1; k < (int)cl.num_blocks(); ++k)
    if (better(s_val[k], s_idx[k], v, i)) { v = s_val[k]; i = s_idx[k]; }
}

template <typename T, int VEC>
__global__ void __launch_bounds__(kVpThreads, 2) verify_probs_kernel(const VerifyProbsParams p) {
  __shared__ float s_val[2][kVpMaxCluster], w_val[32];
  __shared__ int s_idx[2][kVpMaxCluster], w_idx[32];
  __shared__ int s_r;
  cg::cluster_group cl = cg::this_cluster();
  cg::cluster_group::arrival_token started = cl.barrier_arrive();
  griddep_wait();
  griddep_launch();
  const int parts = (int)cl.num_blocks(), b = blockIdx.x / parts, ch = (int)cl.block_rank(), B = p.B, V = p.V;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const T* pt = static_cast<const T*>(p.pt) + (int64_t)b * (B + 1) * p.ld_t;
  const T* pq = p.pq ? static_cast<const T*>(p.pq) + (int64_t)b * B * p.ld_q : nullptr;
  const int32_t* y = p.y + (size_t)b * B;
  int n = B;
  if (p.n) {
    n = p.n[b];
    if (n < 0 || n > B) {
      if (threadIdx.x == 0) set_err(p.err, LSP_DEV_BAD_DELTA);
      n = n < 0 ? 0 : B;
    }
  }
  const float* e = p.e + (size_t)b * V;
  const int ng = V / VEC;                        // VEC > 1 only where V % VEC == 0
  const int g0 = (int)((int64_t)ch * ng / parts), g1 = (int)((int64_t)(ch + 1) * ng / parts);
  if (warp == 0) {
    int r = n;
    for (int i0 = 0; i0 < n; i0 += 32) {
      const int i = i0 + lane;
      bool rej = false;
      if (i < n) {
        const int t = y[i];
        if (t < 0 || t >= V) {
          set_err(p.err, LSP_DEV_BAD_TOKEN);
          rej = true;
        } else {
          const float py = to_f(pt[(int64_t)i * p.ld_t + t]);
          const float qy = pq ? to_f(pq[(int64_t)i * p.ld_q + t]) : 1.f;
          rej = !(__fmul_rn(p.u[(size_t)b * B + i], qy) < py);
        }
      }
      const unsigned m = __ballot_sync(kAll, rej);
      if (m) { r = i0 + __ffs(m) - 1; break; }
    }
    if (lane == 0) s_r = r;
  }
  __syncthreads();
  const int r = s_r;
  const T* row = pt + (int64_t)r * p.ld_t;
  float bv = -1.f;
  int bi = INT_MAX;
  if (r < n && pq)
    scan_row<T, VEC, true>(row, pq + (int64_t)r * p.ld_q, e, -1, g0, g1, bv, bi);
  else
    scan_row<T, VEC, false>(row, nullptr, e, r < n ? y[r] : -1, g0, g1, bv, bi);
  cl.barrier_wait(std::move(started));           // every CTA of the cluster runs: its slots can be written
  cluster_best(cl, bv, bi, s_val[0], s_idx[0], w_val, w_idx);
  if (bi == INT_MAX && r < n) {                  // nothing left of p: draw from p itself
    bv = -1.f;
    scan_row<T, VEC, false>(row, nullptr, e, -1, g0, g1, bv, bi);
    cluster_best(cl, bv, bi, s_val[1], s_idx[1], w_val, w_idx);
  }
  if (ch != 0) return;
  const int tok = bi == INT_MAX ? -1 : bi;
  if (threadIdx.x == 0) {
    p.accepted[b] = r;
    p.next_token[b] = tok;
  }
  if (p.out_tokens)
    for (int i = threadIdx.x; i <= B; i += kVpThreads)
      p.out_tokens[(size_t)b * (B + 1) + i] = i < r ? y[i] : (i == r ? tok : -1);
}

template <typename T, int VEC>
cudaError_t launch(const VerifyProbsParams& p, int parts, cudaStream_t s) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(p.C * parts);
  cfg.blockDim = dim3(kVpThreads);
  cfg.stream = s;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = parts;
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  return cudaLaunchKernelEx(&cfg, verify_probs_kernel<T, VEC>, p);
}

}  // namespace

int launch_verify_probs(const VerifyProbsParams& p, int dtype, int num_sms, cudaStream_t s) {
  const int es = dtype == LSP_DTYPE_BF16 ? 2 : 4;
  // four values a load where every row starts on a load's boundary (64 requests of 16-bit
  // probabilities: 17.4 us, one value a load 21.6)
  const uintptr_t at = reinterpret_cast<uintptr_t>(p.pt) | reinterpret_cast<uintptr_t>(p.pq);
  const bool vec = p.V % 4 == 0 && p.ld_t % 4 == 0 && (!p.pq || p.ld_q % 4 == 0) && at % (4 * es) == 0 &&
                   reinterpret_cast<uintptr_t>(p.e) % 16 == 0;
  // as many CTAs a request as are resident at once, two on an SM (64 requests: 17.4 us with 4, 23 with 8)
  int parts = kVpMaxCluster;
  while (parts > 1 && (int64_t)p.C * parts > 2 * num_sms) parts /= 2;
  cudaError_t e;
  if (dtype == LSP_DTYPE_BF16)
    e = vec ? launch<bf16, 4>(p, parts, s) : launch<bf16, 1>(p, parts, s);
  else
    e = vec ? launch<float, 4>(p, parts, s) : launch<float, 1>(p, parts, s);
  return e == cudaSuccess ? LSP_OK : LSP_ERR_CUDA;
}

}  // namespace lsp
