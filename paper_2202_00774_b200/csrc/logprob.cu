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
// Keys order by value and, among equal values, by the lower index first; 0 is the key of no element. A CTA collects keys that reach a
// bound below which k others are known to lie: to begin with, a value that k threads' largest elements reach; later, the k-th largest key
// collected. With random logits 20 of 131072 leave some dozens of keys to be sorted. (Lists kept sorted in each warp's registers, an insertion
// at a time, took 26 us for one row of 131072 bf16 logits on a cluster of eight CTAs; it takes 8.8 us so, 2.5 without the alternatives.)
using Key = unsigned long long;

__device__ __forceinline__ uint32_t ordered(float x) {
  const uint32_t b = __float_as_uint(x + 0.0f);  // (-0 equals +0)
  return b ^ ((uint32_t)((int32_t)b >> 31) | 0x80000000u);
}
__device__ __forceinline__ Key make_key(float x, uint32_t index) { return ((Key)ordered(x) << 32) | (uint32_t)~index; }
__device__ __forceinline__ float key_value(Key k) {
  const uint32_t o = (uint32_t)(k >> 32);
  return __uint_as_float((o & 0x80000000u) ? o ^ 0x80000000u : ~o);
}

constexpr int kMostKeys = 512;      // that a CTA collects
constexpr int kSortAbove = 48;      // as many are sorted out: a higher bound lets fewer of what follows in

struct Candidates {
  Key keys[kMostKeys];
  Key best[32];
  uint32_t bound[96], least;  // of find_bound, at most 64 + 15 and four
  int count;
};

// Where a row takes a CTA several rounds, a meeting in each of them and the keys of lower bounds cost as much as the sums do (top 20 of
// 4096 x 131072 bf16: 324 us, and 180 without). There only the largest element of each thread's part of some rounds is kept; the threads'
// largest give the bound once the row has been read, and the few parts that reach it are read again: 208 us; 256 rows 31.7 -> 19.7 us. A
// row of one round has its elements still in registers (on a cluster 10.3 us, 11.9 so), and a warp's own rows need no meeting.
enum Top { kNone, kAlong, kBehind };  // alternatives: none, found as the row is read or behind it
constexpr int kMostHits = 128;
template <int NT>
struct Parts {
  static constexpr int kEach = NT > 256 ? 16 : 32;  // parts of a thread
  float most[kEach * NT];
  uint32_t hits[kMostHits];
  int count;
};

// The `top` largest of the first n keys to c.best in descending order (fewer: zeros behind them). Keys of elements all
// differ, so a key's place is the number of larger ones. All threads of the CTA; ends with a barrier.
template <int NT>
__device__ __forceinline__ void sort_out(Candidates& c, int n, int top) {
  if (threadIdx.x < 32) c.best[threadIdx.x] = 0;
  __syncthreads();
  for (int i = threadIdx.x; i < n; i += NT) {
    const Key k = c.keys[i];
    int place = 0;
    int j = 0;
    for (; j + 2 <= n; j += 2) {
      const ulonglong2 o = *(const ulonglong2*)&c.keys[j];
      place += (o.x > k) + (o.y > k);
    }
    if (j < n) place += c.keys[j] > k;
    if (place < top) c.best[place] = k;
  }
  __syncthreads();
}

struct LogprobParams {
  const void* logits;  // [rows, K]
  const int64_t* targets;
  int64_t rows, K;
  int classes;
  int top;
  float *logprob, *entropy, *lse, *top_logprob;  // entropy, lse, top_logprob, top_token: optional
  int64_t* top_token;
};

constexpr int kUnroll = 4;  // vectors of eight elements a thread has in flight
constexpr int kMostParts = 8;

// A cluster of CTAs (one where there are rows enough for all multiprocessors) reads a row in slices; its first CTA joins what the others found
// through distributed shared memory.
template <int DT, int TOP, int NT>  // TOP: a Top
__device__ __forceinline__ void logprob_row(const LogprobParams& p, int64_t row, Stats* stats, Candidates& c, Parts<NT>* seen) {
  using E = Element<DT>;
  constexpr int kWarps = NT / 32;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const uint32_t parts = NT == 32 ? 1u : ptx::cluster_nctarank(), part = NT == 32 ? 0u : ptx::cluster_ctarank();
  const uint8_t* base = (const uint8_t*)p.logits + row * p.K * E::kBytes;
  // elements up to the row's first 16-byte boundary, whole vectors of eight, the rest
  const int head = min(p.classes, (int)((16u - ((uint32_t)(uintptr_t)base & 15u)) & 15u) / E::kBytes);
  const int nvec = (p.classes - head) / 8;
  const int tail0 = head + nvec * 8;
  const void* body = base + (int64_t)head * E::kBytes;

  float m = -INFINITY;
  float2 s = {0.0f, 0.0f}, t = {0.0f, 0.0f};  // sums of even and of odd elements
  Key bound = 0;
  int held = 0;  // keys of the rounds before
  if (TOP && threadIdx.x == 0) {
    c.count = 0;
    if (TOP == kBehind) seen->count = 0;
  }

  // the CTA's slice, a round of it at a time (the same number of rounds in all its warps: the candidates meet at barriers)
  const int stride = (int)parts * NT, first = (int)part * NT;
  const int rounds = nvec > first ? (nvec - first + stride * kUnroll - 1) / (stride * kUnroll) : 0;
  typename E::Raw raw[kUnroll];
  float x[kUnroll][8], top_of[kUnroll], most;
  auto load_round = [&](int v0) {
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) raw[u] = v0 + u * stride < nvec ? E::load8(body, (int64_t)(v0 + u * stride) * 8) : E::lowest8();
    most = -INFINITY;
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      E::widen(raw[u], x[u]);
      top_of[u] = E::largest(raw[u], x[u]);
      most = fmaxf(most, top_of[u]);
    }
  };
  // A value that at least `top` elements reach. Few warps: ceil(top / warps) lanes of each reach the least of their bounds. Many: the least of
  // all would let several times as many keys in, so it is the top-th of the largest elements of about 2 top lanes, for two rounds of compares
  // and a barrier (131072 bf16 on a cluster of CTAs of 16 warps: 10.3 -> 9.1 us; 16384 x 4000 fp32, CTAs of four: 100 us, 107 with the latter).
  auto find_bound = [&](float largest) {
    constexpr bool kRanked = kWarps >= 8;
    const int with = min(kWarps, (nvec - first + 31) / 32), each = kRanked ? min(32, (2 * p.top + with - 1) / with) : (p.top + with - 1) / with;
    uint32_t mine = first + (int)threadIdx.x < nvec ? ordered(largest) : 0u, reached = 0u;
    for (int i = 0; i < each; ++i) {
      reached = __reduce_max_sync(0xFFFFFFFFu, mine);
      if (lane == __ffs(__ballot_sync(0xFFFFFFFFu, mine == reached)) - 1) mine = 0u;
      if (kRanked && lane == 0 && warp < with) c.bound[warp * each + i] = reached;
    }
    if constexpr (kRanked) {
      const int n = with * each;
      if (threadIdx.x < 4) c.bound[n + threadIdx.x] = 0u;
      __syncthreads();
      if ((int)threadIdx.x < n) {
        const uint32_t v = c.bound[threadIdx.x];
        int above = 0, reach = 0;
        for (int j = 0; j < n; j += 4) {
          const uint4 o = *(const uint4*)&c.bound[j];
          above += (o.x > v) + (o.y > v) + (o.z > v) + (o.w > v);
          reach += (o.x >= v) + (o.y >= v) + (o.z >= v) + (o.w >= v);
        }
        if (above < p.top && p.top <= reach) c.least = v;  // (equal ones write the same)
      }
      __syncthreads();
      reached = c.least;
    } else {
      if (lane == 0) c.bound[warp] = reached;
      __syncthreads();
      reached = 0xFFFFFFFFu;
      for (int w = 0; w < with; ++w) reached = min(reached, c.bound[w]);
    }
    bound = (Key)reached << 32;
  };
  auto add_keys = [&](const float (&v)[8], int vec) {  // of a vector of eight
    const float least = bound ? key_value(bound) : -INFINITY;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      if (v[e] >= least) {
        const Key k = make_key(v[e], (uint32_t)(head + vec * 8 + e));
        if (k >= bound) {
          const int at = atomicAdd(&c.count, 1);
          if (at < kMostKeys) c.keys[at] = k;
        }
      }
    }
  };
  // the keys of a round, by all threads
  auto meet = [&](int v0) {
    for (;;) {
      const float least = bound ? key_value(bound) : -INFINITY;
      bool added = false;
      if (most >= least) {
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) {
          if (!(top_of[u] >= least)) continue;
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            if (x[u][e] >= least && v0 + u * stride < nvec) {
              const Key k = make_key(x[u][e], (uint32_t)(head + (v0 + u * stride) * 8 + e));
              if (k >= bound) {
                const int at = atomicAdd(&c.count, 1);
                if (at < kMostKeys) c.keys[at] = k;
                added = true;
              }
            }
          }
        }
      }
      if (!__syncthreads_or(added)) break;
      const int n = c.count;
      __syncthreads();
      if (n <= kSortAbove) {
        held = n;
        break;
      }
      sort_out<NT>(c, min(n, kMostKeys), p.top);
      bound = c.best[p.top - 1];
      // all of them seen: the best stay. More than there is room for: this round again, from what was there before it, with the higher bound
      // (at least kMostKeys - 32 elements lie below that, so a round ends)
      const bool again = n > kMostKeys;
      if (!again && threadIdx.x < p.top) c.keys[threadIdx.x] = c.best[threadIdx.x];
      if (!again) held = p.top;
      if (threadIdx.x == 0) c.count = held;
      __syncthreads();
      if (!again) break;
    }
  };

  float part_most = -INFINITY;
  int part_rounds = 0, parts_seen = 0;
  const int rounds_each = (rounds + Parts<NT>::kEach - 1) / Parts<NT>::kEach;
  for (int round = 0; round < rounds; ++round) {
    const int v0 = first + round * stride * kUnroll + (int)threadIdx.x;
    load_round(v0);
    {
      const float old = m;
      m = fmaxf(m, most);
      const float ref = finite_reference(m), ds = max_nan(old - ref, kFarBelow), f = exp2_approx(ds * kLog2e);
      const float2 f2 = {f, f}, ds2 = {ds, ds}, minus_ref = {-ref, -ref}, log2e = {kLog2e, kLog2e};
      t = mul2(f2, fma2(s, ds2, t));
      s = mul2(s, f2);
#pragma unroll
      for (int u = 0; u < kUnroll; ++u) {
#pragma unroll
        for (int e = 0; e < 8; e += 2) {
          float2 d = add2({x[u][e], x[u][e + 1]}, minus_ref);
          d = {max_nan(d.x, kFarBelow), max_nan(d.y, kFarBelow)};
          float2 w = mul2(d, log2e);
          w = {exp2_approx(w.x), exp2_approx(w.y)};
          s = add2(s, w);
          t = fma2(w, d, t);
        }
      }
    }
    if constexpr (TOP == kAlong) {
      if (round == 0) find_bound(most);
      meet(v0);
    }
    if constexpr (TOP == kBehind) {
      part_most = fmaxf(part_most, most);
      if (++part_rounds == rounds_each || round + 1 == rounds) {
        seen->most[parts_seen++ * NT + threadIdx.x] = part_most;
        part_most = -INFINITY;
        part_rounds = 0;
      }
    }
  }
  if constexpr (TOP == kBehind) {
    if (rounds > 0) {
      find_bound(m);
      const float least = bound ? key_value(bound) : -INFINITY;
      for (int i = 0; i < parts_seen; ++i) {
        if (seen->most[i * NT + threadIdx.x] >= least) {
          const int at = atomicAdd(&seen->count, 1);
          if (at < kMostHits) seen->hits[at] = (uint32_t)(i * NT + (int)threadIdx.x);
        }
      }
      __syncthreads();
      const int hits = seen->count;
      if (hits <= kMostHits) {
        const int vectors = rounds_each * kUnroll;  // of a part
        for (int i = threadIdx.x; i < hits * vectors; i += NT) {
          const int hit = (int)seen->hits[i / vectors], of = i % vectors;
          const int64_t vec = first + ((int64_t)(hit / NT) * vectors + of) * stride + hit % NT;
          if (vec >= nvec) continue;
          float v[8];
          E::widen(E::load8(body, vec * 8), v);
          add_keys(v, (int)vec);
        }
        __syncthreads();
      }
      held = c.count;
      if (hits > kMostHits || held > kMostKeys - 32) {  // equal elements: round by round, so that the lowest indexes stay
        __syncthreads();
        if (threadIdx.x == 0) c.count = 0;
        held = 0;
        __syncthreads();
        for (int round = 0; round < rounds; ++round) {
          const int v0 = first + round * stride * kUnroll + (int)threadIdx.x;
          load_round(v0);
          meet(v0);
        }
      }
    }
  }

  Stats st = {m, s.x + s.y, t.x + t.y};
  // elements before and behind the vectors: one a lane of the first CTA's last warp
  if (TOP) __syncthreads();  // (c.count is set)
  if (part == 0 && warp == kWarps - 1) {
    const int i = lane < head ? lane : tail0 + (lane - head);
    const bool live = i < p.classes;
    const float z = live ? E::load(base, i) : 0.0f;
    if (live) st = join(st, {fmaxf(z, -INFINITY), z == -INFINITY ? 0.0f : z - z + 1.0f, 0.0f});  // (z - z: NaN for NaN and +infinity)
    // (at most 14 more than kSortAbove)
    if (TOP && live && z == z && make_key(z, (uint32_t)i) >= bound) c.keys[atomicAdd(&c.count, 1)] = make_key(z, (uint32_t)i);
  }

  // lanes, warps, CTAs
#pragma unroll
  for (int d = 16; d > 0; d >>= 1)
    st = join(st, {__shfl_xor_sync(0xFFFFFFFFu, st.m, d), __shfl_xor_sync(0xFFFFFFFFu, st.s, d), __shfl_xor_sync(0xFFFFFFFFu, st.t, d)});
  if constexpr (NT > 32) {
    if (lane == 0) stats[warp] = st;
    __syncthreads();
    if (TOP || warp == 0) {  // (with alternatives every warp needs them)
      st = stats[lane % kWarps];
#pragma unroll
      for (int d = kWarps / 2; d > 0; d >>= 1)
        st = join(st, {__shfl_xor_sync(0xFFFFFFFFu, st.m, d), __shfl_xor_sync(0xFFFFFFFFu, st.s, d), __shfl_xor_sync(0xFFFFFFFFu, st.t, d)});
    }
  } else if (TOP) {
    __syncthreads();
  }
  if (TOP) sort_out<NT>(c, c.count, p.top);
  if (NT > 32 && parts > 1) {
    if (TOP) __syncthreads();  // all warps have read stats
    if (threadIdx.x == 0) stats[0] = st;
    ptx::cluster_sync();
    if (part == 0) {
      st = {-INFINITY, 0.0f, 0.0f};
      if (lane < (int)parts) {
        const uint32_t at = ptx::map_to_cta(&stats[0], (uint32_t)lane);
        st = {ptx::ld_cluster_f32(at), ptx::ld_cluster_f32(at + 4), ptx::ld_cluster_f32(at + 8)};
      }
#pragma unroll
      for (int d = kMostParts / 2; d > 0; d >>= 1)
        st = join(st, {__shfl_xor_sync(0xFFFFFFFFu, st.m, d), __shfl_xor_sync(0xFFFFFFFFu, st.s, d), __shfl_xor_sync(0xFFFFFFFFu, st.t, d)});
      if (TOP) {
        for (int i = threadIdx.x; i < (int)parts * p.top; i += NT)
          c.keys[i] = ptx::ld_cluster_u64(ptx::map_to_cta(&c.best[i % p.top], (uint32_t)(i / p.top)));
        __syncthreads();
      }
    }
    ptx::cluster_sync();  // the others' shared memory has been read
    if (part != 0) return;
    if (TOP) sort_out<NT>(c, (int)parts * p.top, p.top);
  }
  st = {__shfl_sync(0xFFFFFFFFu, st.m, 0), __shfl_sync(0xFFFFFFFFu, st.s, 0), __shfl_sync(0xFFFFFFFFu, st.t, 0)};
  if (warp != 0) return;
  const bool empty = st.m == -INFINITY && st.s == 0.0f;  // nothing but -infinity
  const float log_s = logf(st.s);
  if (lane == 0) {
    const int64_t target = p.targets[row];
    float lp = 0.0f;
    if (target >= p.classes) lp = NAN;
    else if (target >= 0) lp = empty ? -INFINITY : (E::load(base, target) - st.m) - log_s;
    p.logprob[row] = lp;
    if (p.lse) p.lse[row] = empty ? -INFINITY : st.m + log_s;
    if (p.entropy) p.entropy[row] = empty ? 0.0f : log_s - st.t / st.s;
  }
  if (TOP && lane < p.top) {
    const Key k = c.best[lane];
    if (p.top_token) p.top_token[row * p.top + lane] = k ? (int64_t)(uint32_t)~(uint32_t)k : -1;
    if (p.top_logprob) p.top_logprob[row * p.top + lane] = !k ? NAN : empty ? -INFINITY : (key_value(k) - st.m) - log_s;
  }
}

template <int DT, int TOP, int NT>
__global__ void __launch_bounds__(NT, NT == 32 ? 24 : 1024 / NT)
logprob_kernel(const LogprobParams p) {
  __shared__ Stats stats[NT / 32];
  __shared__ __align__(16) Candidates found;
  constexpr bool kParts = TOP == kBehind;
  __shared__ __align__(16) uint8_t parts_room[kParts ? sizeof(Parts<NT>) : 16];
  Parts<NT>* seen = kParts ? (Parts<NT>*)parts_room : nullptr;
  ptx::wait_for_previous_grid();
  ptx::launch_dependents();
  if constexpr (NT == 32) {  // (as many CTAs as fit; one for each row, 16384 short rows took 18 us to be dealt out)
    for (int64_t row = blockIdx.x; row < p.rows; row += gridDim.x) {
      logprob_row<DT, TOP, NT>(p, row, stats, found, seen);
      __syncwarp();
    }
  } else {
    logprob_row<DT, TOP, NT>(p, blockIdx.x / ptx::cluster_nctarank(), stats, found, seen);
  }
}

// ------------------------------------------------------------------------------------------------ gradient

struct GradParams {
  const void* logits;  // [rows, K]
  const int64_t* targets;
  const float *lse, *entropy, *d_logprob, *d_entropy;  // d_logprob, or d_entropy (then entropy too): optional
  int64_t rows, K, classes;
  uint32_t seed_lo, seed_hi;
  bool aligned32;  // logits and grad start on 32-byte boundaries
  void* grad;  // optional
  uint4* values;
  uint16_t* meta;
};

// What a row's elements have in common: d z = -p (c + h log p), and `hot` at the target's column.
struct RowTerms {
  float lse, c, h, hot;
  int64_t target;
  bool empty;
};
template <bool ENTROPY>
__device__ __forceinline__ RowTerms row_terms(const GradParams& p, int64_t row) {
  RowTerms r;
  r.lse = p.lse[row];
  r.target = p.targets[row];
  r.empty = r.lse == -INFINITY;
  float g = p.d_logprob ? p.d_logprob[row] : 0.0f;
  if (r.target < 0) g = 0.0f;
  if (r.target >= p.classes) g = NAN;
  r.h = ENTROPY ? p.d_entropy[row] : 0.0f;
  r.c = ENTROPY ? fmaf(r.h, p.entropy[row], g) : g;
  r.hot = g;
  return r;
}
template <bool ENTROPY>
__device__ __forceinline__ float2 grad_of(const RowTerms& r, float2 x) {
  float2 logp = add2(x, {-r.lse, -r.lse});
  if (ENTROPY) logp = {max_nan(logp.x, kFarBelow), max_nan(logp.y, kFarBelow)};  // (0 times a number, not 0 times infinity)
  const float2 d = mul2(logp, {kLog2e, kLog2e}), w = {exp2_approx(d.x), exp2_approx(d.y)};
  return mul2(w, ENTROPY ? fma2({-r.h, -r.h}, logp, {-r.c, -r.c}) : float2{-r.c, -r.c});
}

constexpr int kGradThreads = 256;
constexpr int kGradUnits = 2;  // pairs of vectors of a thread

// Sixteen elements, two vectors, in memory order.
template <int DT>
__device__ __forceinline__ void load_unit(const void* src, int64_t i, bool aligned32, typename Element<DT>::Raw (&r)[2]) {
  const uint8_t* q = (const uint8_t*)src + i * Element<DT>::kBytes;
  auto load32 = [&](const uint8_t* at, uint4& a, uint4& b) {
    if (aligned32) {
      asm volatile("ld.global.L1::no_allocate.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                   : "=r"(a.x), "=r"(a.y), "=r"(a.z), "=r"(a.w), "=r"(b.x), "=r"(b.y), "=r"(b.z), "=r"(b.w)
                   : "l"(at)
                   : "memory");
    } else {
      a = *(const uint4*)at;
      b = *(const uint4*)(at + 16);
    }
  };
  if constexpr (Element<DT>::k32) {
    load32(q, r[0].a, r[0].b);
    load32(q + 32, r[1].a, r[1].b);
  } else {
    load32(q, r[0].a, r[1].a);
  }
}
template <int DT>
__device__ __forceinline__ void store_unit(void* dst, int64_t i, bool aligned32, const typename Element<DT>::Raw (&r)[2]) {
  uint8_t* q = (uint8_t*)dst + i * Element<DT>::kBytes;
  auto store32 = [&](uint8_t* at, const uint4& a, const uint4& b) {
    if (aligned32) {
      const uint32_t w[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
      ptx::st_global_256(at, w);
    } else {
      *(uint4*)at = a;
      *(uint4*)(at + 16) = b;
    }
  };
  if constexpr (Element<DT>::k32) {
    store32(q, r[0].a, r[0].b);
    store32(q + 32, r[1].a, r[1].b);
  } else {
    store32(q, r[0].a, r[1].a);
  }
}

// Units of two vectors, all rows as one sequence of elements; a unit lies inside a row wherever K is a multiple of 16. N == 0: nothing
// is pruned. ENTROPY: d_entropy is there. For rows that are short, or of no multiple of 16 elements.
template <int DT, int M, int N, int SCHEME, bool ENTROPY>
__global__ void __launch_bounds__(kGradThreads)
logprob_grad_kernel(const GradParams p) {
  using E = Element<DT>;
  ptx::wait_for_previous_grid();
  ptx::launch_dependents();
  const int64_t total = p.rows * p.K, unit0 = (int64_t)blockIdx.x * (kGradThreads * kGradUnits) + threadIdx.x;
  const bool fits32 = total <= 0xFFFFFFFFll;
  typename E::Raw raw[kGradUnits][2];
  RowTerms terms[kGradUnits];
  int64_t col[kGradUnits];
#pragma unroll
  for (int u = 0; u < kGradUnits; ++u) {
    const int64_t i0 = (unit0 + u * kGradThreads) * 16;
    raw[u][0].a = raw[u][0].b = raw[u][1].a = raw[u][1].b = make_uint4(0u, 0u, 0u, 0u);
    col[u] = 0;
    if (i0 < total) {
      const int64_t row = fits32 ? (int64_t)((uint32_t)i0 / (uint32_t)p.K) : i0 / p.K;
      col[u] = i0 - row * p.K;
      if (i0 + 16 <= total) load_unit<DT>(p.logits, i0, p.aligned32, raw[u]);
      terms[u] = row_terms<ENTROPY>(p, row);
    }
  }
#pragma unroll
  for (int u = 0; u < kGradUnits; ++u) {
    const int64_t unit = unit0 + u * kGradThreads, i0 = unit * 16;
    const bool on = i0 < total;
    if (M == 32 ? !__any_sync(0xFFFFFFFFu, on) : !on) continue;
    float x[2][8];
    E::widen(raw[u][0], x[0]);
    E::widen(raw[u][1], x[1]);
    RowTerms& r = terms[u];
    if (on && col[u] + 16 <= p.K) {
#pragma unroll
      for (int k = 0; k < 16; k += 2) {
        const float2 g = grad_of<ENTROPY>(r, {x[k >> 3][k & 7], x[k >> 3][(k & 7) + 1]});
        x[k >> 3][k & 7] = g.x;
        x[k >> 3][(k & 7) + 1] = g.y;
      }
      const int64_t hot = r.target - col[u];
      if ((uint64_t)hot < 16u && r.target < p.classes) {
#pragma unroll
        for (int k = 0; k < 16; ++k)
          if (k == hot) x[k >> 3][k & 7] += r.hot;
      }
      if (col[u] + 16 > p.classes || r.empty) {
#pragma unroll
        for (int k = 0; k < 16; ++k)
          if (r.empty || col[u] + k >= p.classes) x[k >> 3][k & 7] = 0.0f;
      }
      raw[u][0] = E::narrow(x[0]);
      raw[u][1] = E::narrow(x[1]);
      if (p.grad) store_unit<DT>(p.grad, i0, p.aligned32, raw[u]);
    } else if (on) {  // a row ends here (only where K is no multiple of 16: nothing is pruned there)
      const int left = (int)min((int64_t)16, total - i0);
      if (left < 16) {
#pragma unroll
        for (int k = 0; k < 16; ++k) x[k >> 3][k & 7] = k < left ? E::load(p.logits, i0 + k) : 0.0f;
      }
      int64_t row = (i0 - col[u]) / p.K, at = col[u];
#pragma unroll
      for (int k = 0; k < 16; ++k) {
        if (at == p.K && k < left) {
          at = 0;
          r = row_terms<ENTROPY>(p, ++row);
        }
        float g = 0.0f;
        if (at < p.classes && !r.empty) {
          g = grad_of<ENTROPY>(r, {x[k >> 3][k & 7], 0.0f}).x;
          if (at == r.target) g += r.hot;
        }
        x[k >> 3][k & 7] = g;
        ++at;
      }
      raw[u][0] = E::narrow(x[0]);
      raw[u][1] = E::narrow(x[1]);
      if (left == 16) {
        store_unit<DT>(p.grad, i0, p.aligned32, raw[u]);
      } else {
#pragma unroll
        for (int k = 0; k < 16; ++k)
          if (k < left) E::store(p.grad, i0 + k, x[k >> 3][k & 7]);
      }
      continue;
    }
    if constexpr (N > 0) {
      uint4 out;
      uint32_t pa, pb;
      KeepFlags ka, kb;
      compress_pair<M, N, SCHEME, E::kF16>(raw[u][0].a, raw[u][1].a, 2 * unit, p.seed_lo, p.seed_hi, M == 32 ? (int)(threadIdx.x & 1) : 0,
                                           0xFFFFFFFFu, out, pa, pb, ka, kb);
      if (!on) continue;
      if (p.values) p.values[unit] = out;
      if (p.meta) p.meta[unit] = (uint16_t)prmt(pa, pb, 0x0073);
    }
  }
}

// The same where rows are long and K is a multiple of 16: a CTA takes a stretch of one row, so what the row's elements share is the same for all
// its threads and no thread has to find its row. (4096 x 131072 bf16: 15 instructions an element in the kernel above, 423 us.)
constexpr int kStretchUnits = 4;
constexpr int kStretch = 16 * kGradThreads * kStretchUnits;
template <int DT, int M, int N, int SCHEME, bool ENTROPY>
__global__ void __launch_bounds__(kGradThreads)
logprob_grad_stretch_kernel(const GradParams p, int stretches) {
  using E = Element<DT>;
  ptx::wait_for_previous_grid();
  ptx::launch_dependents();
  const int64_t row = blockIdx.x / (unsigned)stretches;
  // (unsigned: the last stretch of a row may end past 2^31)
  const uint32_t col0 = (blockIdx.x - (uint32_t)row * (uint32_t)stretches) * kStretch + threadIdx.x * 16;
  const uint32_t K = (uint32_t)p.K, classes = (uint32_t)p.classes;
  const int64_t base = row * p.K;
  typename E::Raw raw[kStretchUnits][2];
#pragma unroll
  for (int u = 0; u < kStretchUnits; ++u) {
    const uint32_t col = col0 + u * 16 * kGradThreads;
    raw[u][0].a = raw[u][0].b = raw[u][1].a = raw[u][1].b = make_uint4(0u, 0u, 0u, 0u);
    if (col < K) load_unit<DT>(p.logits, base + col, p.aligned32, raw[u]);
  }
  const RowTerms r = row_terms<ENTROPY>(p, row);
  const int64_t hot0 = r.target < p.classes ? r.target : -1;
#pragma unroll
  for (int u = 0; u < kStretchUnits; ++u) {
    const uint32_t col = col0 + u * 16 * kGradThreads;
    const bool on = col < K;
    if (M == 32 ? !__any_sync(0xFFFFFFFFu, on) : !on) continue;
    float x[2][8];
#pragma unroll
    for (int v = 0; v < 2; ++v) {
      E::widen(raw[u][v], x[v]);
#pragma unroll
      for (int e = 0; e < 8; e += 2) {
        const float2 g = grad_of<ENTROPY>(r, {x[v][e], x[v][e + 1]});
        x[v][e] = g.x;
        x[v][e + 1] = g.y;
      }
    }
    const int64_t hot = hot0 - (int64_t)col;
    if ((uint64_t)hot < 16u) {
#pragma unroll
      for (int k = 0; k < 16; ++k)
        if (k == hot) x[k >> 3][k & 7] += r.hot;
    }
    if (r.empty || col + 16 > classes) {
#pragma unroll
      for (int k = 0; k < 16; ++k)
        if (r.empty || col + k >= classes) x[k >> 3][k & 7] = 0.0f;
    }
    raw[u][0] = E::narrow(x[0]);
    raw[u][1] = E::narrow(x[1]);
    if (on && p.grad) store_unit<DT>(p.grad, base + col, p.aligned32, raw[u]);
    if constexpr (N > 0) {
      const int64_t unit = (base + col) >> 4;
      uint4 out;
      uint32_t pa, pb;
      KeepFlags ka, kb;
      compress_pair<M, N, SCHEME, E::kF16>(raw[u][0].a, raw[u][1].a, 2 * unit, p.seed_lo, p.seed_hi, M == 32 ? (int)(threadIdx.x & 1) : 0,
                                           0xFFFFFFFFu, out, pa, pb, ka, kb);
      if (!on) continue;
      if (p.values) p.values[unit] = out;
      if (p.meta) p.meta[unit] = (uint16_t)prmt(pa, pb, 0x0073);
    }
  }
}

template <typename... Params>
cudaError_t launch(void (*kernel)(Params...), int64_t blocks, int threads, int cluster, cudaStream_t stream, const Params&... args) {
  if (blocks > 0x7FFFFFFF) return cudaErrorInvalidValue;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)blocks);
  cfg.blockDim = dim3((unsigned)threads);
  cfg.stream = stream;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = (unsigned)cluster;
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = cluster > 1 ? 2 : 1;
  return cudaLaunchKernelEx(&cfg, kernel, args...);
}

constexpr int kWarpRow = 2048;  // tokens up to which a row is one warp's

template <int DT, int NT>
cudaError_t launch_logprob_rows(const LogprobParams& p, int64_t rows, int cluster, cudaStream_t stream) {
  if (p.top == 0) return launch(logprob_kernel<DT, kNone, NT>, rows * cluster, NT, cluster, stream, p);
  if constexpr (NT == 32) {
    return launch(logprob_kernel<DT, kAlong, NT>, rows * cluster, NT, cluster, stream, p);
  } else {
    if constexpr (NT == 512) {
      if (p.classes <= cluster * NT * kUnroll * 8) return launch(logprob_kernel<DT, kAlong, NT>, rows * cluster, NT, cluster, stream, p);
    }
    return launch(logprob_kernel<DT, kBehind, NT>, rows * cluster, NT, cluster, stream, p);
  }
}

template <int DT>
cudaError_t launch_logprob_typed(const LogprobParams& p, int64_t rows, cudaStream_t stream) {
  if (p.classes <= kWarpRow) {
    const int64_t fit = 24 * (int64_t)sm_count();
    return launch_logprob_rows<DT, 32>(p, rows < fit ? rows : fit, 1, stream);
  }
  // CTAs of 512 threads that share a row: as many as it has work for, while there are too few rows to fill the multiprocessors. With rows
  // enough, CTAs of 128 threads, eight to a multiprocessor: as one's sums meet, the others read (16384 x 4096 fp32: 45 us, 84 with 256
  // threads).
  int cluster = 1;
  while (cluster < kMostParts && rows * cluster < (int64_t)sm_count() && p.classes > cluster * 512 * 8) cluster *= 2;
  if (rows <= 2 * (int64_t)sm_count()) return launch_logprob_rows<DT, 512>(p, rows, cluster, stream);
  if (rows <= 8 * (int64_t)sm_count()) return launch_logprob_rows<DT, 256>(p, rows, 1, stream);
  return launch_logprob_rows<DT, 128>(p, rows, 1, stream);
}

template <int DT, int M, int N, int SCHEME>
cudaError_t launch_grad_form(const GradParams& p, int64_t blocks, cudaStream_t stream) {
  // rows of at least half a stretch (a last stretch's idle threads end at once)
  if (p.K % 16 == 0 && 2 * p.K >= kStretch) {
    const int stretches = (int)((p.K + kStretch - 1) / kStretch);
    return p.d_entropy ? launch(logprob_grad_stretch_kernel<DT, M, N, SCHEME, true>, p.rows * stretches, kGradThreads, 1, stream, p, stretches)
                       : launch(logprob_grad_stretch_kernel<DT, M, N, SCHEME, false>, p.rows * stretches, kGradThreads, 1, stream, p, stretches);
  }
  return p.d_entropy ? launch(logprob_grad_kernel<DT, M, N, SCHEME, true>, blocks, kGradThreads, 1, stream, p)
                     : launch(logprob_grad_kernel<DT, M, N, SCHEME, false>, blocks, kGradThreads, 1, stream, p);
}

template <int DT, int M, int N>
cudaError_t launch_grad_scheme(const GradParams& p, int scheme, int64_t blocks, cudaStream_t stream) {
  if (scheme == SDGP_RANDOM) return launch_grad_form<DT, M, N, SDGP_RANDOM>(p, blocks, stream);
  if (scheme == SDGP_MAGNITUDE) return launch_grad_form<DT, M, N, SDGP_MAGNITUDE>(p, blocks, stream);
  return launch_grad_form<DT, M, N, SDGP_RESCALED_MAGNITUDE>(p, blocks, stream);
}

template <int DT>
cudaError_t launch_grad_typed(const GradParams& p, int n, int m, int scheme, cudaStream_t stream) {
  constexpr int64_t per_block = 16 * kGradThreads * kGradUnits;
  const int64_t blocks = (p.rows * p.K + per_block - 1) / per_block;
  if (!p.values && !p.meta) return launch_grad_form<DT, 4, 0, 0>(p, blocks, stream);
  if constexpr (DT != SDGP_FP32) {
#define SDGP_FORM(M, N) \
  if (m == M && n == N) return launch_grad_scheme<DT, M, N>(p, scheme, blocks, stream);
    SDGP_FORM(4, 1) SDGP_FORM(4, 2) SDGP_FORM(8, 1) SDGP_FORM(8, 2) SDGP_FORM(16, 1) SDGP_FORM(16, 2) SDGP_FORM(32, 1) SDGP_FORM(32, 2)
#undef SDGP_FORM
  }
  return cudaErrorInvalidValue;
}

}  // namespace

cudaError_t launch_token_logprob(const void* logits, const int64_t* targets, int64_t rows, int64_t K, int64_t classes, int dtype, int top,
                                 float* logprob, float* entropy, float* lse, float* top_logprob, int64_t* top_token,
                                 cudaStream_t stream) {
  const LogprobParams p = {logits, targets, rows, K, (int)classes, top, logprob, entropy, lse, top_logprob, top_token};
  if (dtype == SDGP_BF16) return launch_logprob_typed<SDGP_BF16>(p, rows, stream);
  if (dtype == SDGP_FP16) return launch_logprob_typed<SDGP_FP16>(p, rows, stream);
  return launch_logprob_typed<SDGP_FP32>(p, rows, stream);
}

cudaError_t launch_token_logprob_backward(const void* logits, const int64_t* targets, const float* lse, const float* entropy,
                                          const float* d_logprob, const float* d_entropy, int64_t rows, int64_t K, int64_t classes, int n,
                                          int m, int scheme, uint64_t seed, int dtype, void* grad, void* values, void* meta,
                                          cudaStream_t stream) {
  const GradParams p = {logits, targets, lse, entropy, d_logprob, d_entropy, rows, K, classes, (uint32_t)seed, (uint32_t)(seed >> 32),
                        (((uintptr_t)logits | (uintptr_t)grad) & 31u) == 0, grad, (uint4*)values, (uint16_t*)meta};
  if (dtype == SDGP_BF16) return launch_grad_typed<SDGP_BF16>(p, n, m, scheme, stream);
  if (dtype == SDGP_FP16) return launch_grad_typed<SDGP_FP16>(p, n, m, scheme, stream);
  return launch_grad_typed<SDGP_FP32>(p, n, m, scheme, stream);
}

}  // namespace sdgp
