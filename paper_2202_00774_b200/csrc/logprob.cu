// Log probabilities of given tokens, with entropy and top alternatives, and their gradient: the head of a language model, sm_100a.
//
// With z the logits of a row over its `classes` tokens, p = softmax(z) and lse = log sum exp z:
//   logprob = z_t - lse,  entropy H = - sum_j p_j log p_j,
//   d z_j = g (1[j = t] - p_j) - h p_j (log p_j + H)          for gradients g of logprob and h of H.
// d z is the dL/dO of the layer that made the logits - the first one of the backward chain -, so the gradient kernel is a producer like
// those below a ReLU: it writes dL/dO and its compressed pruned copy in one pass.
#include <float.h>

#include "elements.cuh"
#include "ptx.cuh"
#include "sdgp_internal.cuh"

namespace sdgp {
namespace {

constexpr int kThreads = 256;
constexpr int kWarps = kThreads / 32;
constexpr float kLog2e = 1.4426950408889634f;
// Below this difference of two logits the exponential is zero in fp32. Differences are cut off there, so that a masked logit
// (-infinity, or the type's lowest value) gives the product 0 * (a number), never 0 * infinity.
constexpr float kFarBelow = -1.0e4f;

// ------------------------------------------------------------------------------------------------ statistics of a row
//
// One pass over the logits with a running maximum m: s = sum exp(z - m), t = sum exp(z - m) (z - m). Then lse = m + log s and
// H = log s - t / s. All in fp32.
struct Stats {
  float m, s, t;
};

__device__ __forceinline__ float finite_reference(float m) { return fmaxf(m, -FLT_MAX); }

// Statistics a and b of two parts of a row.
__device__ __forceinline__ Stats join(const Stats& a, const Stats& b) {
  const float m = fmaxf(a.m, b.m), ref = finite_reference(m);
  const float da = max_nan(a.m - ref, kFarBelow), db = max_nan(b.m - ref, kFarBelow);
  const float fa = exp2_approx(da * kLog2e), fb = exp2_approx(db * kLog2e);
  return {m, a.s * fa + b.s * fb, fa * (a.t + a.s * da) + fb * (b.t + b.s * db)};
}

// ---- the k <= 32 largest logits ----
//
// A warp keeps its 32 largest so far in descending order, one in each lane, as keys that order by value and, among equal values, by the
// lower index first; 0 is the key of no element.
using Key = unsigned long long;

__device__ __forceinline__ Key make_key(float x, uint32_t index) {
  const uint32_t b = __float_as_uint(x + 0.0f);  // (-0 equals +0)
  return ((Key)(b ^ ((uint32_t)((int32_t)b >> 31) | 0x80000000u)) << 32) | (uint32_t)~index;
}
__device__ __forceinline__ float key_value(Key k) {
  const uint32_t o = (uint32_t)(k >> 32);
  return __uint_as_float((o & 0x80000000u) ? o ^ 0x80000000u : ~o);
}

__device__ __forceinline__ Key larger(Key a, Key b) { return a > b ? a : b; }
__device__ __forceinline__ Key smaller(Key a, Key b) { return a > b ? b : a; }

// Sorts a bitonic sequence of 32 keys (one a lane) in descending order.
__device__ __forceinline__ Key sort_bitonic(Key k, int lane) {
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) {
    const Key o = __shfl_xor_sync(0xFFFFFFFFu, k, d);
    k = (lane & d) ? smaller(k, o) : larger(k, o);
  }
  return k;
}
__device__ __forceinline__ Key sort32(Key k, int lane) {
#pragma unroll
  for (int size = 2; size <= 32; size <<= 1) {
#pragma unroll
    for (int d = size >> 1; d > 0; d >>= 1) {
      const Key o = __shfl_xor_sync(0xFFFFFFFFu, k, d);
      const bool up = (lane & size) != 0 && size < 32;  // this part in ascending order
      k = (((lane & d) != 0) != up) ? smaller(k, o) : larger(k, o);
    }
  }
  return k;
}
// The 32 largest of two descending lists.
__device__ __forceinline__ Key merge_lists(Key a, Key b, int lane) {
  return sort_bitonic(larger(a, __shfl_sync(0xFFFFFFFFu, b, 31 - lane)), lane);
}
// One more key (the same in all lanes) into a descending list.
__device__ __forceinline__ Key insert(Key list, Key k, int lane) {
  const int place = __popc(__ballot_sync(0xFFFFFFFFu, list > k));
  const Key up = __shfl_up_sync(0xFFFFFFFFu, list, 1);
  return lane < place ? list : lane == place ? k : up;
}

struct LogprobParams {
  const void* logits;  // [rows, K]
  const int64_t* targets;
  int64_t K;
  int classes;
  int top;
  float *logprob, *entropy, *lse, *top_logprob;  // entropy, lse, top_logprob, top_token: optional
  int64_t* top_token;
};

constexpr int kUnroll = 4;  // vectors of eight elements a thread has in flight

// A cluster of CTAs (one where there are rows enough for all multiprocessors) reads a row in slices; its first CTA joins what the others found
// through distributed shared memory.
template <int DT, bool TOP>
__global__ void __launch_bounds__(kThreads)
logprob_kernel(const LogprobParams p) {
  using E = Element<DT>;
  __shared__ Stats stats[kWarps];
  __shared__ Key lists[TOP ? kWarps : 1][32];
  ptx::wait_for_previous_grid();
  ptx::launch_dependents();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const uint32_t parts = ptx::cluster_nctarank(), part = ptx::cluster_ctarank();
  const int64_t row = blockIdx.x / parts;
  const uint8_t* base = (const uint8_t*)p.logits + row * p.K * E::kBytes;
  // elements up to the row's first 16-byte boundary, whole vectors of eight, the rest
  const int head = min(p.classes, (int)((16u - ((uint32_t)(uintptr_t)base & 15u)) & 15u) / E::kBytes);
  const int nvec = (p.classes - head) / 8;
  const int tail0 = head + nvec * 8;
  const void* body = base + (int64_t)head * E::kBytes;

  Stats st = {-INFINITY, 0.0f, 0.0f};
  Key list = 0;
  float floor_value = 0.0f;  // the k-th largest so far; nothing at or below it enters (what is read later has a higher index)
  bool full = false;

  const int stride = (int)parts * kThreads;
  for (int v0 = (int)part * kThreads + warp * 32; v0 < nvec; v0 += stride * kUnroll) {
    typename E::Raw raw[kUnroll];
    int live = 0;
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      const int v = v0 + lane + u * stride;
      if (v < nvec) {
        raw[u] = E::load8(body, (int64_t)v * 8);
        live = u + 1;
      }
    }
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      float x[8];
      E::widen(raw[u], x);
      const bool on = u < live;
      float most = -INFINITY;
#pragma unroll
      for (int e = 0; e < 8; ++e) most = fmaxf(most, x[e]);
      if (on) {
        const float m = fmaxf(st.m, most), ref = finite_reference(m);
        const float ds = max_nan(st.m - ref, kFarBelow), f = exp2_approx(ds * kLog2e);
        st.t = f * (st.t + st.s * ds);
        st.s *= f;
        st.m = m;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float d = max_nan(x[e] - ref, kFarBelow), w = exp2_approx(d * kLog2e);
          st.s += w;
          st.t = fmaf(w, d, st.t);
        }
      }
      if (TOP) {
        if (!__any_sync(0xFFFFFFFFu, on && (!full || most > floor_value))) continue;
        const uint32_t i0 = (uint32_t)(head + (v0 + lane + u * stride) * 8);
        uint32_t mask = 0;
        if (!full) {
          // the largest of each lane start the list
          Key best = 0;
#pragma unroll
          for (int e = 0; e < 8; ++e)
            if (on && x[e] == x[e]) best = larger(best, make_key(x[e], i0 + e));
          list = merge_lists(list, sort32(best, lane), lane);
          const Key kth = __shfl_sync(0xFFFFFFFFu, list, p.top - 1);
          full = kth != 0;
          if (full) floor_value = key_value(kth);
          // (an element equal to the k-th may have a lower index here: the comparison of keys decides)
#pragma unroll
          for (int e = 0; e < 8; ++e)
            if (on && x[e] == x[e] && (!full || x[e] >= floor_value) && make_key(x[e], i0 + e) != best) mask |= 1u << e;
        } else {
#pragma unroll
          for (int e = 0; e < 8; ++e)
            if (on && x[e] > floor_value) mask |= 1u << e;
        }
        Key kth = __shfl_sync(0xFFFFFFFFu, list, p.top - 1);
        for (;;) {
          const uint32_t lanes = __ballot_sync(0xFFFFFFFFu, mask != 0);
          if (lanes == 0) break;
          const int src = __ffs(lanes) - 1;
          Key k = 0;
          if (lane == src) {
            const int e = __ffs(mask) - 1;
            mask &= mask - 1;
            k = make_key(E::load(base, i0 + e), i0 + e);
          }
          k = __shfl_sync(0xFFFFFFFFu, k, src);
          if (k > kth) {
            list = insert(list, k, lane);
            kth = __shfl_sync(0xFFFFFFFFu, list, p.top - 1);
          }
        }
        full = kth != 0;
        if (full) floor_value = key_value(kth);
      }
    }
  }

  // elements before and behind the vectors: one a lane of the first CTA's last warp
  if (part == 0 && warp == kWarps - 1) {
    const int i = lane < head ? lane : tail0 + (lane - head);
    const bool live = i < p.classes;
    const float x = live ? E::load(base, i) : 0.0f;
    if (live) st = join(st, {fmaxf(x, -INFINITY), x == -INFINITY ? 0.0f : x - x + 1.0f, 0.0f});  // (x - x: NaN for NaN and +infinity)
    if (TOP) list = merge_lists(list, sort32(live && x == x ? make_key(x, (uint32_t)i) : 0, lane), lane);
  }

  // lanes, warps, CTAs
#pragma unroll
  for (int d = 16; d > 0; d >>= 1)
    st = join(st, {__shfl_xor_sync(0xFFFFFFFFu, st.m, d), __shfl_xor_sync(0xFFFFFFFFu, st.s, d), __shfl_xor_sync(0xFFFFFFFFu, st.t, d)});
  if (lane == 0) stats[warp] = st;
  if (TOP) lists[warp][lane] = list;
  __syncthreads();
  if (TOP) {
#pragma unroll
    for (int d = kWarps / 2; d > 0; d >>= 1) {
      if (warp < d) {
        list = merge_lists(list, lists[warp + d][lane], lane);
        lists[warp][lane] = list;
      }
      __syncthreads();
    }
  }
  if (warp == 0) {
    st = lane < kWarps ? stats[lane] : Stats{-INFINITY, 0.0f, 0.0f};
#pragma unroll
    for (int d = kWarps / 2; d > 0; d >>= 1)
      st = join(st, {__shfl_xor_sync(0xFFFFFFFFu, st.m, d), __shfl_xor_sync(0xFFFFFFFFu, st.s, d), __shfl_xor_sync(0xFFFFFFFFu, st.t, d)});
    if (lane == 0) stats[0] = st;
  }
  if (parts > 1) {
    ptx::cluster_sync();
    if (part == 0) {
      if (warp == 0) {
        st = {-INFINITY, 0.0f, 0.0f};
        if (lane < (int)parts) {
          const uint32_t at = ptx::map_to_cta(&stats[0], (uint32_t)lane);
          st = {ptx::ld_cluster_f32(at), ptx::ld_cluster_f32(at + 4), ptx::ld_cluster_f32(at + 8)};
        }
#pragma unroll
        for (int d = 16; d > 0; d >>= 1)
          st = join(st, {__shfl_xor_sync(0xFFFFFFFFu, st.m, d), __shfl_xor_sync(0xFFFFFFFFu, st.s, d), __shfl_xor_sync(0xFFFFFFFFu, st.t, d)});
      }
      if (TOP) {
        // (a cluster has at most as many CTAs as a CTA has warps)
        list = warp < (int)parts ? ptx::ld_cluster_u64(ptx::map_to_cta(&lists[0][lane], (uint32_t)warp)) : 0;
        __syncthreads();  // the first CTA's own list has been read
        lists[warp][lane] = list;
        __syncthreads();
#pragma unroll
        for (int d = kWarps / 2; d > 0; d >>= 1) {
          if (warp < d) {
            list = merge_lists(list, lists[warp + d][lane], lane);
            lists[warp][lane] = list;
          }
          __syncthreads();
        }
      }
    }
    ptx::cluster_sync();  // the others' shared memory has been read
  }
  if (part != 0 || warp != 0) return;
  st = {__shfl_sync(0xFFFFFFFFu, st.m, 0), __shfl_sync(0xFFFFFFFFu, st.s, 0), __shfl_sync(0xFFFFFFFFu, st.t, 0)};
  const bool empty = st.m == -INFINITY && st.s == 0.0f;  // nothing but -infinity
  const float log_s = logf(st.s);
  const float lse = empty ? -INFINITY : st.m + log_s;
  if (lane == 0) {
    const int64_t t = p.targets[row];
    float lp = 0.0f;
    if (t >= p.classes) lp = NAN;
    else if (t >= 0) lp = empty ? -INFINITY : (E::load(base, t) - st.m) - log_s;
    p.logprob[row] = lp;
    if (p.lse) p.lse[row] = lse;
    if (p.entropy) p.entropy[row] = empty ? 0.0f : log_s - st.t / st.s;
  }
  if (TOP && lane < p.top) {
    if (p.top_token) p.top_token[row * p.top + lane] = list ? (int64_t)(uint32_t)~(uint32_t)list : -1;
    if (p.top_logprob) p.top_logprob[row * p.top + lane] = !list ? NAN : empty ? -INFINITY : (key_value(list) - st.m) - log_s;
  }
}

// ------------------------------------------------------------------------------------------------ gradient

struct GradParams {
  const void* logits;  // [rows, K]
  const int64_t* targets;
  const float *lse, *entropy, *d_logprob, *d_entropy;  // d_logprob, or d_entropy (then entropy too): optional
  int64_t rows, K, classes;
  uint32_t seed_lo, seed_hi;
  void* grad;  // optional
  uint4* values;
  uint16_t* meta;
};

// What a row's elements have in common: d z = -p (c + h log p), and `hot` at the target's column.
struct RowTerms {
  float lse, c, h, hot;
  int64_t target;  // -1: none
  bool empty;
};
__device__ __forceinline__ RowTerms row_terms(const GradParams& p, int64_t row) {
  RowTerms r;
  r.lse = p.lse[row];
  r.target = p.targets[row];
  r.empty = r.lse == -INFINITY;
  float g = p.d_logprob ? p.d_logprob[row] : 0.0f;
  if (r.target < 0) g = 0.0f;
  if (r.target >= p.classes) g = NAN;
  r.h = p.d_entropy ? p.d_entropy[row] : 0.0f;
  r.c = p.d_entropy ? fmaf(r.h, p.entropy[row], g) : g;
  r.hot = g;
  return r;
}
__device__ __forceinline__ float grad_of(const RowTerms& r, float x) {
  const float logp = max_nan(x - r.lse, kFarBelow);
  return -exp2_approx(logp * kLog2e) * fmaf(r.h, logp, r.c);
}

// Two vectors of eight a thread, all rows as one sequence of elements; they end inside a row wherever K is no multiple of 16.
// N == 0: nothing is pruned.
template <int DT, int M, int N, int SCHEME>
__global__ void __launch_bounds__(kThreads)
logprob_grad_kernel(const GradParams p) {
  using E = Element<DT>;
  ptx::wait_for_previous_grid();
  ptx::launch_dependents();
  const int64_t total = p.rows * p.K, pair = (int64_t)blockIdx.x * kThreads + threadIdx.x, i0 = pair * 16;
  const bool on = i0 < total;
  if (M == 32 ? !__any_sync(0xFFFFFFFFu, on) : !on) return;
  float x[2][8];
  typename E::Raw raw[2];
  if (!on) {
    raw[0].a = raw[0].b = raw[1].a = raw[1].b = make_uint4(0u, 0u, 0u, 0u);
  } else {
    const bool fits32 = total <= 0xFFFFFFFFll;
    int64_t row = fits32 ? (int64_t)((uint32_t)i0 / (uint32_t)p.K) : i0 / p.K;
    int64_t col = i0 - row * p.K;
    RowTerms r = row_terms(p, row);
    if (col + 16 <= p.K) {
      raw[0] = E::load8(p.logits, i0);
      raw[1] = E::load8(p.logits, i0 + 8);
      const bool whole = col + 16 <= p.classes;
      const int64_t hot = r.target - col;
#pragma unroll
      for (int v = 0; v < 2; ++v) {
        E::widen(raw[v], x[v]);
#pragma unroll
        for (int e = 0; e < 8; ++e) x[v][e] = grad_of(r, x[v][e]);
      }
      if ((uint64_t)hot < 16u && r.target < p.classes) {
#pragma unroll
        for (int k = 0; k < 16; ++k)
          if (k == hot) x[k >> 3][k & 7] += r.hot;
      }
      if (!whole || r.empty) {
#pragma unroll
        for (int k = 0; k < 16; ++k)
          if (r.empty || col + k >= p.classes) x[k >> 3][k & 7] = 0.0f;
      }
      raw[0] = E::narrow(x[0]);
      raw[1] = E::narrow(x[1]);
      if (p.grad) {
        E::store8(p.grad, i0, raw[0]);
        E::store8(p.grad, i0 + 8, raw[1]);
      }
    } else {  // a row ends here (only where K is no multiple of 16: nothing is pruned there)
      const int left = (int)min((int64_t)16, total - i0);
      if (left == 16) {
        raw[0] = E::load8(p.logits, i0);
        raw[1] = E::load8(p.logits, i0 + 8);
        E::widen(raw[0], x[0]);
        E::widen(raw[1], x[1]);
      } else {
#pragma unroll
        for (int k = 0; k < 16; ++k) x[k >> 3][k & 7] = k < left ? E::load(p.logits, i0 + k) : 0.0f;
      }
#pragma unroll
      for (int k = 0; k < 16; ++k) {
        if (col == p.K && k < left) {
          col = 0;
          r = row_terms(p, ++row);
        }
        float g = 0.0f;
        if (col < p.classes && !r.empty) {
          g = grad_of(r, x[k >> 3][k & 7]);
          if (col == r.target) g += r.hot;
        }
        x[k >> 3][k & 7] = g;
        ++col;
      }
      if (left == 16) {
        E::store8(p.grad, i0, E::narrow(x[0]));
        E::store8(p.grad, i0 + 8, E::narrow(x[1]));
      } else {
#pragma unroll
        for (int k = 0; k < 16; ++k)
          if (k < left) E::store(p.grad, i0 + k, x[k >> 3][k & 7]);
      }
      return;
    }
  }
  if constexpr (N > 0) {
    uint4 out;
    uint32_t pa, pb;
    KeepFlags ka, kb;
    compress_pair<M, N, SCHEME, E::kF16>(raw[0].a, raw[1].a, 2 * pair, p.seed_lo, p.seed_hi, M == 32 ? (int)(threadIdx.x & 1) : 0,
                                         0xFFFFFFFFu, out, pa, pb, ka, kb);
    if (!on) return;
    if (p.values) p.values[pair] = out;
    if (p.meta) p.meta[pair] = (uint16_t)prmt(pa, pb, 0x0073);
  }
}

template <typename... Params>
cudaError_t launch(void (*kernel)(Params...), int64_t blocks, int cluster, cudaStream_t stream, const Params&... args) {
  if (blocks > 0x7FFFFFFF) return cudaErrorInvalidValue;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)blocks);
  cfg.blockDim = dim3(kThreads);
  cfg.stream = stream;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = (unsigned)cluster;
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  return cudaLaunchKernelEx(&cfg, kernel, args...);
}

template <int DT>
cudaError_t launch_logprob_typed(const LogprobParams& p, int64_t rows, cudaStream_t stream) {
  // CTAs that share a row: as many as it has work for, while there are too few rows to fill the multiprocessors
  int cluster = 1;
  while (cluster < kWarps && rows * cluster < 2 * (int64_t)sm_count() && p.classes > cluster * kThreads * 8) cluster *= 2;
  return p.top > 0 ? launch(logprob_kernel<DT, true>, rows * cluster, cluster, stream, p)
                   : launch(logprob_kernel<DT, false>, rows * cluster, cluster, stream, p);
}

template <int DT, int M, int N>
cudaError_t launch_grad_scheme(const GradParams& p, int scheme, int64_t blocks, cudaStream_t stream) {
  if (scheme == SDGP_RANDOM) return launch(logprob_grad_kernel<DT, M, N, SDGP_RANDOM>, blocks, 1, stream, p);
  if (scheme == SDGP_MAGNITUDE) return launch(logprob_grad_kernel<DT, M, N, SDGP_MAGNITUDE>, blocks, 1, stream, p);
  return launch(logprob_grad_kernel<DT, M, N, SDGP_RESCALED_MAGNITUDE>, blocks, 1, stream, p);
}

template <int DT>
cudaError_t launch_grad_typed(const GradParams& p, int n, int m, int scheme, cudaStream_t stream) {
  const int64_t blocks = (p.rows * p.K + 16 * kThreads - 1) / (16 * kThreads);
  if (!p.values && !p.meta) return launch(logprob_grad_kernel<DT, 4, 0, 0>, blocks, 1, stream, p);
  if constexpr (DT != SDGP_FP32) {
    switch (m * 4 + n) {
      case 17: return launch_grad_scheme<DT, 4, 1>(p, scheme, blocks, stream);
      case 18: return launch_grad_scheme<DT, 4, 2>(p, scheme, blocks, stream);
      case 33: return launch_grad_scheme<DT, 8, 1>(p, scheme, blocks, stream);
      case 34: return launch_grad_scheme<DT, 8, 2>(p, scheme, blocks, stream);
      case 65: return launch_grad_scheme<DT, 16, 1>(p, scheme, blocks, stream);
      case 66: return launch_grad_scheme<DT, 16, 2>(p, scheme, blocks, stream);
      case 129: return launch_grad_scheme<DT, 32, 1>(p, scheme, blocks, stream);
      case 130: return launch_grad_scheme<DT, 32, 2>(p, scheme, blocks, stream);
    }
  }
  return cudaErrorInvalidValue;
}

}  // namespace

cudaError_t launch_token_logprob(const void* logits, const int64_t* targets, int64_t rows, int64_t K, int64_t classes, int dtype, int top,
                                 float* logprob, float* entropy, float* lse, float* top_logprob, int64_t* top_token,
                                 cudaStream_t stream) {
  const LogprobParams p = {logits, targets, K, (int)classes, top, logprob, entropy, lse, top_logprob, top_token};
  if (dtype == SDGP_BF16) return launch_logprob_typed<SDGP_BF16>(p, rows, stream);
  if (dtype == SDGP_FP16) return launch_logprob_typed<SDGP_FP16>(p, rows, stream);
  return launch_logprob_typed<SDGP_FP32>(p, rows, stream);
}

cudaError_t launch_token_logprob_backward(const void* logits, const int64_t* targets, const float* lse, const float* entropy,
                                          const float* d_logprob, const float* d_entropy, int64_t rows, int64_t K, int64_t classes, int n,
                                          int m, int scheme, uint64_t seed, int dtype, void* grad, void* values, void* meta,
                                          cudaStream_t stream) {
  const GradParams p = {logits, targets, lse, entropy, d_logprob, d_entropy, rows, K, classes, (uint32_t)seed, (uint32_t)(seed >> 32),
                        grad, (uint4*)values, (uint16_t*)meta};
  if (dtype == SDGP_BF16) return launch_grad_typed<SDGP_BF16>(p, n, m, scheme, stream);
  if (dtype == SDGP_FP16) return launch_grad_typed<SDGP_FP16>(p, n, m, scheme, stream);
  return launch_grad_typed<SDGP_FP32>(p, n, m, scheme, stream);
}

}  // namespace sdgp
