// The boundary between two blocks of a residual network of linear layers (a transformer's), and its gradient, sm_100a:
//   n = b rstd(b) w_post      the norm behind a block whose last layer gave b (w_post absent: n = b)
//   o = alpha r + g n         residual scale and gate
//   y = o rstd(o) w_pre       the norm before the next block (w_pre absent: no y),      rstd(v) = 1 / sqrt(mean(v^2) + eps)
// Backward, from gradients d_o and d_y, with u = o rstd(o), v = b rstd(b) (v = b without w_post) and means over a row:
//   d = d_o + rstd(o) (w_pre d_y - u mean(w_pre d_y u)),   d_r = alpha d,   d_w_pre = sum over rows of d_y u
//   d_b = rstd(b) (q - v mean(q v)),  q = d g w_post,      d_g = sum of d v w_post,  d_w_post = sum of d g v
// d_b is the dL/dO of the block's last layer: like the producers below a ReLU the kernel writes it and its compressed pruned copy in one
// pass.
//
// Both passes are bound by memory: 4 (backward 6) tensors are read or written once, rows stay in registers between the sums and their use.
// TPR threads own a row, eight columns each, and go through rows at a fixed stride, so that sums over rows stay in registers as well.
// A thread copies its own vectors of the next rows to shared memory asynchronously (nobody else reads them: no barrier), a row's sums
// need one exchange between its warps.
//
// Rows of a width that is no multiple of eight start at any of eight places in a 16-byte vector. Ownership goes by the vectors of memory, not by
// columns; the rows that one group of threads takes start at the same place (the strides are multiples of the period at which places
// return), so a thread keeps its columns.
#include "dgrad_common.cuh"
#include "elements.cuh"

namespace sdgp {
namespace {

constexpr int kMaxWarpsPerRow = 32;

__device__ __forceinline__ void cp_async16(uint32_t dst, const void* src, uint32_t bytes) {  // the rest of the 16 bytes is zeroed
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
}
__device__ __forceinline__ void cp_async_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void cp_async_wait() {
  asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}

// Threads of a CTA, and stages of the copies that are under way, for rows of TPR threads and A input tensors.
template <int TPR>
constexpr int kCtaThreads = TPR > 256 ? TPR : 256;
template <int DT, int TPR, int VECTORS, int LEAST>
struct Ring {  // VECTORS: of a thread and row, in all tensors; LEAST: stages that a kernel cannot do without
  static constexpr int kChunk = kCtaThreads<TPR> * 16;               // 16 bytes of each thread side by side
  static constexpr int kVec = kChunk * (Element<DT>::kBytes / 2);    // a vector: one chunk, or two of fp32
  static constexpr int kStage = VECTORS * kVec;
  // of a multiprocessor's 227 KB: forward (LEAST 1) up to 1024 threads share it, backward 512
  static constexpr int kRoom = (TPR > 512 ? 200 : LEAST == 1 ? (TPR > 256 ? 110 : 55) : TPR > 256 ? 200 : 110) * 1024;
  static constexpr int kFit = kRoom / kStage;
  static constexpr int kStages = kFit > 4 ? 4 : kFit < LEAST ? LEAST : kFit;
  static constexpr int kBytes = kStage * kStages;
};

// A thread's part of a row: eight elements of memory from element `first` of the row (negative in the row's first vector if the row does
// not start on a vector), of which [lo, hi) are the row's.
struct Part {
  int first, lo, hi;
  bool full;
};
__device__ __forceinline__ Part part_of(int64_t row, int C, int t) {
  const int a = (int)((uint64_t)row * (uint64_t)C & 7u);
  Part p;
  p.first = t * 8 - a;
  p.lo = t == 0 ? a : 0;
  p.hi = max(0, min(8, C - p.first));
  p.full = p.lo == 0 && p.hi == 8;
  return p;
}

// A thread's vector of a row to its place in a stage. fp32 vectors are two chunks: where rows are whole vectors, a warp copies its 32 vectors
// together, 512 contiguous bytes an instruction (each its own 16 of every 32 bytes took twice the requests), so a warp has to meet
// (__syncwarp) between the copies' arrival and their use, and between the use and the next copies.
template <int DT, int CHUNK>
__device__ __forceinline__ void copy_part(uint32_t dst, const void* src, int64_t row_at, const Part& p, int C) {
  using E = Element<DT>;
  if constexpr (E::k32) {
    if (C % 8 == 0) {
      const int lane = threadIdx.x & 31, half = lane & 1;
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        const int other = 16 * k + (lane >> 1), at = p.first + (other - lane) * 8 + half * 4;  // that lane's vector
        cp_async16(dst + (other - lane) * 16 + half * CHUNK, (const float*)src + row_at + (at < C ? at : 0), at < C ? 16u : 0u);
      }
      return;
    }
  }
  const uint8_t* q = (const uint8_t*)src + (row_at + p.first) * E::kBytes;
  const int bytes = p.hi * E::kBytes;
  cp_async16(dst, q, (uint32_t)min(16, bytes));
  if (E::k32) cp_async16(dst + CHUNK, bytes > 16 ? q + 16 : q, (uint32_t)max(0, bytes - 16));
}
template <int DT, int CHUNK>
__device__ __forceinline__ void read_part(const uint8_t* at, float (&x)[8]) {
  using E = Element<DT>;
  typename E::Raw r;
  r.a = *(const uint4*)at;
  r.b = E::k32 ? *(const uint4*)(at + CHUNK) : make_uint4(0u, 0u, 0u, 0u);
  E::widen(r, x);
}
// The end of the row before, copied along with a row's first vector, becomes zeros, in COUNT tensors (what lies behind the row was never
// copied and is zero). Once a row and not where the vectors are read, which is twice, a branch each.
template <int DT, int CHUNK, int COUNT>
__device__ __forceinline__ void clear_before(uint8_t* at, int vector_bytes, const Part& p) {
  using E = Element<DT>;
  if (p.lo == 0) return;
#pragma unroll 1
  for (int v = 0; v < COUNT; ++v) {
    for (int e = 0; e < p.lo; ++e) {
      uint8_t* to = at + v * vector_bytes;
      if (E::k32) *(float*)(to + (e >= 4 ? CHUNK : 0) + (e & 3) * 4) = 0.0f;
      else *(uint16_t*)(to + e * 2) = 0;
    }
  }
}
template <int DT, bool ALIGNED = false>
__device__ __forceinline__ void write_part(void* dst, int64_t row_at, const Part& p, const typename Element<DT>::Raw& r) {
  using E = Element<DT>;
  const int64_t at = row_at + p.first;
  if (p.full) {
    E::store8(dst, at, r);
  } else if (!ALIGNED) {
    const uint32_t w[8] = {r.a.x, r.a.y, r.a.z, r.a.w, r.b.x, r.b.y, r.b.z, r.b.w};
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      if (e >= p.lo && e < p.hi) {
        if (E::k32) ((uint32_t*)dst)[at + e] = w[e];
        else ((uint16_t*)dst)[at + e] = (uint16_t)(w[e / 2] >> (e % 2 * 16));
      }
    }
  }
}
// The thread's elements of a vector of C elements, as they are in memory; ones where there is no vector.
template <int DT>
__device__ __forceinline__ typename Element<DT>::Raw column_part(const void* src, int64_t offset, const Part& p) {
  using E = Element<DT>;
  if (src && p.full && ((offset + p.first) & 7) == 0) return E::load8(src, offset + p.first);
  float x[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) x[e] = !src ? 1.0f : e >= p.lo && e < p.hi ? E::load(src, offset + p.first + e) : 0.0f;
  return E::narrow(x);
}
__device__ __forceinline__ void write_columns(float* dst, const Part& p, const float (&x)[8]) {
  if (p.full && ((uintptr_t)(dst + p.first) & 15u) == 0) {
    *(float4*)(dst + p.first) = make_float4(x[0], x[1], x[2], x[3]);
    *(float4*)(dst + p.first + 4) = make_float4(x[4], x[5], x[6], x[7]);
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (e >= p.lo && e < p.hi) dst[p.first + e] = x[e];
  }
}

// Sums over the TPR threads of a row, in two halves with a barrier of those threads between them (rows of one warp need none).
template <int TPR>
__device__ __forceinline__ void put_sum(float s, float* b) {
  s = warp_sum(s);
  if ((threadIdx.x & 31) == 0) b[(threadIdx.x % TPR) >> 5] = s;
}
template <int W>
__device__ __forceinline__ float sum_lanes(float s) {  // over W neighbouring lanes
#pragma unroll
  for (int d = W / 2; d > 0; d >>= 1) s += __shfl_xor_sync(0xFFFFFFFFu, s, d);
  return s;
}
// At once. `turn` alternates between two buffers, so one barrier a call is enough.
template <int TPR, int N>
__device__ __forceinline__ void row_sums(float (&s)[N], float* buffer, int slot, int& turn) {
  if constexpr (TPR == 32) {
#pragma unroll
    for (int i = 0; i < N; ++i) s[i] = warp_sum(s[i]);
  } else {
    constexpr int W = TPR / 32;
    float* b = buffer + (turn * (kCtaThreads<TPR> / TPR) + slot) * W * N;
#pragma unroll
    for (int i = 0; i < N; ++i) put_sum<TPR>(s[i], b + i * W);
    ptx::named_bar_sync(1 + slot, TPR);
#pragma unroll
    for (int i = 0; i < N; ++i) s[i] = sum_lanes<W>(b[i * W + (threadIdx.x & 31) % W]);
    turn ^= 1;
  }
}

// ------------------------------------------------------------------------------------------------ forward

struct NormParams {
  const void *branch, *residual;  // [rows, C]
  const void *post_weight, *gate, *pre_weight;  // [C], [groups, C], [C]; each optional
  void *out, *y;
  float *post_rstd, *pre_rstd;
  int64_t rows, rows_per_group;
  int C, groups;
  float alpha, eps;
};

// A thread owns NV vectors, TPR apart.
template <int DT, int TPR, int NV>
__global__ void __launch_bounds__(kCtaThreads<TPR>, TPR > 512 ? 1 : 1024 / kCtaThreads<TPR>)
norm_kernel(const NormParams p) {
  using E = Element<DT>;
  using R = Ring<DT, TPR, 2 * NV, 1>;
  constexpr int SLOTS = kCtaThreads<TPR> / TPR;
  extern __shared__ __align__(16) uint8_t ring[];
  __shared__ float buffer[2 * SLOTS * kMaxWarpsPerRow];
  ptx::wait_for_previous_grid();
  ptx::launch_dependents();
  const int slot = threadIdx.x / TPR, t = threadIdx.x % TPR;
  const int64_t first = (int64_t)blockIdx.x * SLOTS + slot, stride = (int64_t)gridDim.x * SLOTS;
  if (first >= p.rows) return;  // (a slot's threads share no barrier with the others)
  Part part[NV];
#pragma unroll
  for (int j = 0; j < NV; ++j) part[j] = part_of(first, p.C, t + j * TPR);
  uint8_t* mine = ring + threadIdx.x * 16;
  const uint32_t mine_u32 = ptx::smem_u32(mine);
  auto fetch = [&](int64_t row, int stage) {
    if (row < p.rows) {
#pragma unroll
      for (int j = 0; j < NV; ++j) {
        copy_part<DT, R::kChunk>(mine_u32 + stage * R::kStage + 2 * j * R::kVec, p.branch, row * p.C, part[j], p.C);
        copy_part<DT, R::kChunk>(mine_u32 + stage * R::kStage + (2 * j + 1) * R::kVec, p.residual, row * p.C, part[j], p.C);
      }
    }
    cp_async_commit();
  };
#pragma unroll
  for (int s = 0; s < R::kStages; ++s) fetch(first + s * stride, s);
  typename E::Raw w_post[NV], w_pre[NV], gate[NV];
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    w_post[j] = column_part<DT>(p.post_weight, 0, part[j]);
    w_pre[j] = column_part<DT>(p.pre_weight, 0, part[j]);
    gate[j] = column_part<DT>(p.gate, 0, part[j]);
  }
  const float inv_c = 1.0f / (float)p.C;
  int stage = 0, turn = 0;
  for (int64_t row = first; row < p.rows; row += stride) {
    if (p.groups > 1) {
      const int64_t at = row / p.rows_per_group * p.C;
#pragma unroll
      for (int j = 0; j < NV; ++j) gate[j] = column_part<DT>(p.gate, at, part[j]);
    }
    cp_async_wait<R::kStages - 1>();
    if (E::k32) __syncwarp();
    clear_before<DT, R::kChunk, 2>(mine + stage * R::kStage, R::kVec, part[0]);
    float o[NV][8], rstd = 1.0f;  // the branch, then its sum with the residual
    float s[1] = {0.0f};
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      read_part<DT, R::kChunk>(mine + stage * R::kStage + 2 * j * R::kVec, o[j]);
#pragma unroll
      for (int e = 0; e < 8; ++e) s[0] = fmaf(o[j][e], o[j][e], s[0]);
    }
    if (p.post_weight) {
      row_sums<TPR>(s, buffer, slot, turn);
      rstd = rsqrtf(fmaf(s[0], inv_c, p.eps));
      if (t == 0 && p.post_rstd) p.post_rstd[row] = rstd;
    }
    s[0] = 0.0f;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      float r[8], w[8], g[8];
      read_part<DT, R::kChunk>(mine + stage * R::kStage + (2 * j + 1) * R::kVec, r);
      E::widen(w_post[j], w);
      E::widen(gate[j], g);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float n = p.post_weight ? o[j][e] * rstd * w[e] : o[j][e];
        o[j][e] = fmaf(g[e], n, p.alpha * r[e]);
        s[0] = fmaf(o[j][e], o[j][e], s[0]);
      }
      write_part<DT>(p.out, row * p.C, part[j], E::narrow(o[j]));
    }
    if (p.pre_weight) {  // (of the sums before their rounding to 16 bits)
      row_sums<TPR>(s, buffer, slot, turn);
      rstd = rsqrtf(fmaf(s[0], inv_c, p.eps));
      if (t == 0 && p.pre_rstd) p.pre_rstd[row] = rstd;
#pragma unroll
      for (int j = 0; j < NV; ++j) {
        float w[8];
        E::widen(w_pre[j], w);
#pragma unroll
        for (int e = 0; e < 8; ++e) o[j][e] = o[j][e] * rstd * w[e];
        write_part<DT>(p.y, row * p.C, part[j], E::narrow(o[j]));
      }
    }
    if (E::k32) __syncwarp();
    fetch(row + R::kStages * stride, stage);
    if (++stage == R::kStages) stage = 0;
  }
  cp_async_wait<0>();
}

// ------------------------------------------------------------------------------------------------ backward

struct NormGradParams {
  const void *branch, *out, *d_out, *d_y;       // [rows, C]; d_out and d_y (then out as well) optional
  const void *post_weight, *gate, *pre_weight;  // as in the forward pass; pre_weight only with d_y
  const float *post_rstd, *pre_rstd;
  void *d_residual, *d_branch;                  // [rows, C]; each optional
  uint2* values;                                // compressed pruned copy of d_branch; each optional
  uint8_t* meta;
  float* d_gate;                                // [groups, C]; optional
  // Sums over a slot's rows of d_y u and of d g v, [slots, pitch], and over a unit's rows of d v, [groups, gate_rows, pitch]; null where they
  // are not needed (post_sums: only with GATES; else the sums of d v give d_w_post too). A row of sums is laid out as its rows are in their
  // vectors: column c at c + (place of the first row in its vector), so that threads write whole vectors.
  float *pre_sums, *post_sums, *unit_sums;
  int64_t rows, rows_per_group;
  int C, pitch, splits, units, gate_rows;  // gate_rows: units of a gate that have rows
  float alpha;
  int n, m, scheme;
  uint32_t seed_lo, seed_hi;
};

// The pruning function as a call of its own: 24 forms, inlined into none of the kernels that use it (some 100 of their instructions per eight
// elements: 16384 x 4096 bf16 with the 2:4 copy take 270 us, 148 without it, 136 by their bytes).
template <bool F16>
__device__ __noinline__ uint4 prune_any(uint4 w, int64_t v, uint32_t seed_lo, uint32_t seed_hi, int n, int m, int scheme, int part) {
  uint2 out = make_uint2(0u, 0u);
  uint32_t pos = 0u;
  KeepFlags k;
#define SDGP_FORM(M, N)                                                                                                         \
  if (m == M && n == N) {                                                                                                       \
    const int l = part % (M <= 8 ? 1 : M / 8); /* the vector's place in a group that spans lanes */                             \
    if (scheme == SDGP_RANDOM) compress_vector<M, N, SDGP_RANDOM, F16>(w, v, seed_lo, seed_hi, l, 0xFFFFFFFFu, out, pos, k);    \
    else if (scheme == SDGP_MAGNITUDE) compress_vector<M, N, SDGP_MAGNITUDE, F16>(w, v, seed_lo, seed_hi, l, 0xFFFFFFFFu, out, pos, k); \
    else compress_vector<M, N, SDGP_RESCALED_MAGNITUDE, F16>(w, v, seed_lo, seed_hi, l, 0xFFFFFFFFu, out, pos, k);              \
  }
  SDGP_FORM(4, 1) SDGP_FORM(4, 2) SDGP_FORM(8, 1) SDGP_FORM(8, 2) SDGP_FORM(16, 1) SDGP_FORM(16, 2) SDGP_FORM(32, 1) SDGP_FORM(32, 2)
#undef SDGP_FORM
  return make_uint4(out.x, out.y, pos >> 24, 0u);
}

// Rows are dealt out in units: rows of one gate, at a stride of `splits`. A slot takes units at the stride of all slots (without GATES: one
// unit).
struct Walk {
  int64_t row, at;  // at = row * C
  int left;         // rows of the unit from this one on; 0: no row
  int unit, group;
};
template <bool GATES>
__device__ __forceinline__ void start_unit(Walk& w, const NormGradParams& p, int ids) {  // the first row of w.unit, or of the next unit that has one
  w.left = 0;
  for (; w.unit < p.units; w.unit += ids) {
    w.group = w.unit / p.splits;
    const int first = w.unit - w.group * p.splits;
    w.left = (int)((p.rows_per_group - first + p.splits - 1) / p.splits);
    w.row = (int64_t)w.group * p.rows_per_group + first;
    w.at = w.row * p.C;
    if (w.left > 0 || !GATES) return;
  }
}
template <bool GATES>
__device__ __forceinline__ void advance(Walk& w, const NormGradParams& p, int ids, int64_t step) {
  if (w.left == 0) return;
  w.row += p.splits;
  w.at += step;
  if (--w.left == 0 && GATES) {
    w.unit += ids;
    start_unit<GATES>(w, p, ids);
  }
}

__device__ __forceinline__ float2 pair_of(const float (&x)[8], int i) { return {x[2 * i], x[2 * i + 1]}; }
__device__ __forceinline__ float2 both(float x) { return {x, x}; }

__device__ __forceinline__ void write_sums(float* dst, const float2 (&x)[4]) {
  *(float4*)dst = make_float4(x[0].x, x[0].y, x[1].x, x[1].y);
  *(float4*)(dst + 4) = make_float4(x[2].x, x[2].y, x[3].x, x[3].y);
}

// Three sums of a warp in six exchanges instead of fifteen: the first two of them halve what a lane carries. Lanes 0-7 end with the
// first, 16-23 with the second, 8-15 and 24-31 with the third.
__device__ __forceinline__ float warp_sums3(float a, float b, float c) {
  const int lane = threadIdx.x & 31;
  const bool high = lane & 16, third = lane & 8;
  const float ab = (high ? b : a) + __shfl_xor_sync(0xFFFFFFFFu, high ? a : b, 16);
  c += __shfl_xor_sync(0xFFFFFFFFu, c, 16);
  float s = (third ? c : ab) + __shfl_xor_sync(0xFFFFFFFFu, third ? ab : c, 8);
#pragma unroll
  for (int d = 4; d > 0; d >>= 1) s += __shfl_xor_sync(0xFFFFFFFFu, s, d);
  return s;
}

// The two means of the formulas hang on each other: mean(q d v) needs d, which needs mean(w_pre d_y u). Written out,
//   sum q d v = sum q v (d_o + rstd w_pre d_y) - rstd mean(w_pre d_y u) sum q v u,
// so one exchange of three sums does. They are taken a row ahead: between two barriers a group of threads sums its next row and writes the
// outputs of the present one, reading its inputs from shared memory a second time instead of keeping them. (With the sums of a row, a
// barrier and its outputs in turn: 279 us for 16384 x 4096 bf16.)
//
// GATES: a slot's rows have more than one gate, so gates go along with the rows. Else q = g w_post stays in registers, and a thread has
// room for NV = 2 vectors, TPR threads apart: half the exchanges, addresses and barriers an element.
// CL: CTAs that share rows too wide for one. Each sends its warps' sums to all, into one of four places in turn, and an mbarrier of each
// place counts them. A warp sends row i + 4's sums, into the place of row i, after it has read those of row i + 2. All warps have sent those by
// then, and each did so after it had read row i's: no place is written before everyone has read it, and no sums are counted on the phase of an
// earlier row. (Three places are too few: the sender of row i + 3 has read row i + 1, whose sums a warp sends before it reads row i's.)
// (With a barrier of the cluster a row, which waits for the outputs of all rows before: 313 us for 4096 x 8192 fp32, 222 now.)
constexpr unsigned kSumsError = 0x100u;  // in the error word: sums that did not come
template <int DT, int TPR, int NV, int CL, bool GATES, bool ALIGNED, bool PRUNE>
__global__ void __launch_bounds__(kCtaThreads<TPR>, TPR > 256 ? 1 : 2)
norm_grad_kernel(const NormGradParams p) {
  using E = Element<DT>;
  using R = Ring<DT, TPR, 4 * NV, 2>;
  constexpr int SLOTS = kCtaThreads<TPR> / TPR, S = R::kStages, W = TPR / 32, WC = W * CL;  // WC: warps of a row
  constexpr int PLACES = CL > 1 ? 4 : 2;
  constexpr uint32_t kSumBytes = 3 * WC * sizeof(float);
  static_assert(CL == 1 || SLOTS == 1, "");
  extern __shared__ __align__(16) uint8_t ring[];
  __shared__ float buffer[PLACES * 3 * SLOTS * WC];
  __shared__ uint64_t arrived[PLACES];  // CL > 1
  ptx::wait_for_previous_grid();
  ptx::launch_dependents();
  const int slot = threadIdx.x / TPR, t = threadIdx.x % TPR, lane = threadIdx.x & 31;
  const int rank = CL > 1 ? (int)ptx::cluster_ctarank() : 0, v0 = rank * TPR * NV + t;  // v0: the thread's first vector of a row
  const int id = (int)blockIdx.x / CL * SLOTS + slot, ids = (int)gridDim.x / CL * SLOTS;
  const int64_t step = (int64_t)p.splits * p.C;
  Walk here;
  here.unit = id;
  start_unit<GATES>(here, p, ids);
  if (here.left <= 0) {
    // no row at all: the sums of this slot are zero
    const float2 zero[4] = {};
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int at = (v0 + j * TPR) * 8;
      if (at < p.pitch && p.pre_sums) write_sums(p.pre_sums + (int64_t)id * p.pitch + at, zero);
      if (at < p.pitch && p.post_sums) write_sums(p.post_sums + (int64_t)id * p.pitch + at, zero);
    }
    return;
  }
  Part part[NV];
#pragma unroll
  for (int j = 0; j < NV; ++j) part[j] = part_of(here.row, p.C, v0 + j * TPR);
  uint8_t* mine = ring + threadIdx.x * 16;
  const uint32_t mine_u32 = ptx::smem_u32(mine);
  auto fetch = [&](const Walk& w, int stage) {
    if (w.left > 0) {
#pragma unroll
      for (int j = 0; j < NV; ++j) {
        const uint32_t at = mine_u32 + stage * R::kStage + j * 4 * R::kVec;
        copy_part<DT, R::kChunk>(at, p.branch, w.at, part[j], p.C);
        if (p.d_out) copy_part<DT, R::kChunk>(at + R::kVec, p.d_out, w.at, part[j], p.C);
        if (p.d_y) {
          copy_part<DT, R::kChunk>(at + 2 * R::kVec, p.out, w.at, part[j], p.C);
          copy_part<DT, R::kChunk>(at + 3 * R::kVec, p.d_y, w.at, part[j], p.C);
        }
      }
    }
    cp_async_commit();
  };
  // what belongs to a row beside its elements, loaded a row before it is summed
  struct Beside {
    float rstd_b, rstd;
    typename E::Raw gate;  // GATES only
  };
  auto load_beside = [&](const Walk& w, int known_group, Beside& b) {
    if (w.left <= 0) return;
    b.rstd_b = p.post_weight ? p.post_rstd[w.row] : 1.0f;
    b.rstd = p.d_y ? p.pre_rstd[w.row] : 0.0f;
    if (GATES && w.group != known_group) b.gate = column_part<DT>(p.gate, (int64_t)w.group * p.C, part[0]);
  };
  typename E::Raw w_post[NV], raw_gate[NV], raw_pre[NV];
  float q_kept[NV][8], w_kept[NV][8];
  auto factors = [&](const Beside& beside, int j, float (&q)[8]) {  // q = g w_post
    if constexpr (GATES) {
      float w[8];
      E::widen(beside.gate, q);
      E::widen(w_post[j], w);
#pragma unroll
      for (int e = 0; e < 8; ++e) q[e] *= w[e];
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) q[e] = q_kept[j][e];
    }
  };
  auto meet = [&]() {
    if (CL == 1 && TPR > 32) ptx::named_bar_sync(1 + slot, TPR);
  };
  if constexpr (CL > 1) {
    if (threadIdx.x == 0) {
#pragma unroll
      for (int i = 0; i < PLACES; ++i) {
        ptx::mbar_init(&arrived[i], 1);
        ptx::mbar_arrive_expect_tx(&arrived[i], kSumBytes);
      }
      ptx::fence_mbar_init();
    }
    __syncthreads();
    ptx::cluster_sync();  // the others run: their shared memory may be written
  }
  const float inv_c = 1.0f / (float)p.C;
  auto sum_row = [&](const Beside& beside, int stage, int turn) -> float {
    float2 s0 = both(0.0f), s1 = both(0.0f), s2 = both(0.0f);
    if (!ALIGNED) clear_before<DT, R::kChunk, 4>(mine + stage * R::kStage, R::kVec, part[0]);
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const uint8_t* at = mine + stage * R::kStage + j * 4 * R::kVec;
      float b[8], q[8], d[8];
      read_part<DT, R::kChunk>(at, b);
      factors(beside, j, q);
      float o[8], y[8];
      read_part<DT, R::kChunk>(at + R::kVec, d);
      read_part<DT, R::kChunk>(at + 2 * R::kVec, o);
      read_part<DT, R::kChunk>(at + 3 * R::kVec, y);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float2 wd = mul2(pair_of(y, i), pair_of(w_kept[j], i)), qb = mul2(pair_of(q, i), pair_of(b, i));
        s0 = fma2(wd, pair_of(o, i), s0);
        s1 = fma2(qb, fma2(both(beside.rstd), wd, pair_of(d, i)), s1);
        s2 = fma2(qb, pair_of(o, i), s2);
      }
    }
    const float s = warp_sums3(beside.rstd * (s0.x + s0.y), beside.rstd_b * (s1.x + s1.y), beside.rstd_b * beside.rstd * (s2.x + s2.y));
    if (TPR > 32 && (lane & 7) == 0 && lane != 24) {
      float* to = &buffer[(turn * SLOTS + slot) * WC * 3 + (lane == 0 ? 0 : lane == 16 ? WC : 2 * WC) + rank * W + (t >> 5)];
      if constexpr (CL == 1) {
        *to = s;
      } else {
#pragma unroll
        for (int c = 0; c < CL; ++c) ptx::st_cluster_async_f32(ptx::map_to_cta(to, (uint32_t)c), s, ptx::map_to_cta(&arrived[turn], (uint32_t)c));
      }
    }
    return s;
  };

  // tensors that are absent are zeros
  for (int v = 0; v < 4 * NV * S; ++v) {
    if (v % 4 == 0 || (v % 4 == 1 ? p.d_out : p.d_y) != nullptr) continue;
    *(uint4*)(mine + v * R::kVec) = make_uint4(0u, 0u, 0u, 0u);
    if (E::k32) *(uint4*)(mine + v * R::kVec + R::kChunk) = make_uint4(0u, 0u, 0u, 0u);
  }
  Walk next = here;
  advance<GATES>(next, p, ids, step);
  Walk after = next, ahead = here;
  advance<GATES>(after, p, ids, step);
#pragma unroll
  for (int s = 0; s < S; ++s) {
    fetch(ahead, s);
    advance<GATES>(ahead, p, ids, step);
  }
  // (all loads are under way before the first of them is waited for)
  Beside beside = {}, beside_next = {}, beside_after = {};
  load_beside(here, -1, beside);
  beside_next.gate = beside.gate;
  load_beside(next, here.group, beside_next);
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    w_post[j] = column_part<DT>(p.post_weight, 0, part[j]);
    raw_pre[j] = column_part<DT>(p.pre_weight, 0, part[j]);
    if (!GATES) raw_gate[j] = column_part<DT>(p.gate, p.gate ? (int64_t)here.group * p.C : 0, part[j]);
  }
  beside_after = beside_next;
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    E::widen(raw_pre[j], w_kept[j]);
    if constexpr (!GATES) {
      float w[8];
      E::widen(raw_gate[j], q_kept[j]);
      E::widen(w_post[j], w);
#pragma unroll
      for (int e = 0; e < 8; ++e) q_kept[j][e] *= w[e];
    }
  }
  cp_async_wait<S - 1>();
  if (E::k32) __syncwarp();
  float own = sum_row(beside, 0, 0), own_next = own;
  meet();

  float2 pre_sum[NV][4] = {}, post_sum[NV][4] = {}, gate_sum[NV][4] = {};
  int stage = 0, turn = 0;
  uint32_t parity = 0;
  while (here.left > 0) {
    const int stage_next = stage + 1 == S ? 0 : stage + 1, turn_next = turn + 1 == PLACES ? 0 : turn + 1;
    load_beside(after, next.group, beside_after);
    if (next.left > 0) {
      cp_async_wait<S - 2>();
      if (E::k32) __syncwarp();
      own_next = sum_row(beside_next, stage_next, turn_next);
    }
    if constexpr (CL > 1) {
      ptx::mbar_wait(&arrived[turn], parity, &g_device_error, kSumsError);  // (one that gives up carries on to the end)
      __syncwarp();
      if (t == 0) ptx::mbar_arrive_expect_tx(&arrived[turn], kSumBytes);
    }
    float s0, s1, s2;
    if constexpr (TPR > 32) {
      constexpr int L = WC < 32 ? WC : 32;
      const float* from = buffer + (turn * SLOTS + slot) * WC * 3 + lane % L;
      s0 = from[0], s1 = from[WC], s2 = from[2 * WC];
      if constexpr (WC > 32) {
        s0 += from[32];
        s1 += from[WC + 32];
        s2 += from[2 * WC + 32];
      }
      s0 = sum_lanes<L>(s0);
      s1 = sum_lanes<L>(s1);
      s2 = sum_lanes<L>(s2);
    } else {
      s0 = __shfl_sync(0xFFFFFFFFu, own, 0);
      s1 = __shfl_sync(0xFFFFFFFFu, own, 16);
      s2 = __shfl_sync(0xFFFFFFFFu, own, 8);
    }
    const float k = beside.rstd * (s0 * inv_c), mean = (s1 - k * s2) * inv_c;
    const bool unit_ends = here.left == 1;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const uint8_t* at = mine + stage * R::kStage + j * 4 * R::kVec;
      float b[8], q[8], d[8], out[8];
      read_part<DT, R::kChunk>(at, b);
      float o[8], y[8];
      read_part<DT, R::kChunk>(at + R::kVec, d);
      read_part<DT, R::kChunk>(at + 2 * R::kVec, o);
      read_part<DT, R::kChunk>(at + 3 * R::kVec, y);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float2 dy = pair_of(y, i), u = mul2(pair_of(o, i), both(beside.rstd));
        pre_sum[j][i] = fma2(dy, u, pre_sum[j][i]);
        const float2 x = fma2(both(-k), u, fma2(both(beside.rstd), mul2(dy, pair_of(w_kept[j], i)), pair_of(d, i)));
        d[2 * i] = x.x;
        d[2 * i + 1] = x.y;
      }
      if (p.d_residual) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float2 x = mul2(both(p.alpha), pair_of(d, i));
          out[2 * i] = x.x;
          out[2 * i + 1] = x.y;
        }
        write_part<DT, ALIGNED>(p.d_residual, here.at, part[j], E::narrow(out));
      }
      factors(beside, j, q);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float2 x = pair_of(d, i), v = mul2(pair_of(b, i), both(beside.rstd_b));
        gate_sum[j][i] = fma2(x, v, gate_sum[j][i]);
        float2 y = mul2(pair_of(q, i), x);
        if (p.post_weight) y = mul2(fma2(v, both(-mean), y), both(beside.rstd_b));
        out[2 * i] = y.x;
        out[2 * i + 1] = y.y;
      }
      const typename E::Raw packed = E::narrow(out);
      if (p.d_branch) write_part<DT, ALIGNED>(p.d_branch, here.at, part[j], packed);
      if constexpr (PRUNE) {  // (rows of whole groups of 16: every part is full or empty, and a group's lanes alike)
        const int64_t vec = (here.at >> 3) + v0 + j * TPR;
        const uint4 c = prune_any<E::kF16>(packed.a, vec, p.seed_lo, p.seed_hi, p.n, p.m, p.scheme, t & 3);
        if (part[j].full) {
          if (p.values) p.values[vec] = make_uint2(c.x, c.y);
          if (p.meta) p.meta[vec] = (uint8_t)c.z;
        }
      }
      if (unit_ends) {  // sum of d v over the unit's rows: times g for d_w_post, times w_post for d_g
        const bool some = part[j].hi > 0;
        if (p.unit_sums && some)
          write_sums(p.unit_sums + ((int64_t)here.group * p.gate_rows + (here.unit - here.group * p.splits)) * p.pitch + (v0 + j * TPR) * 8, gate_sum[j]);
        if constexpr (GATES) {
          float g[8], w[8];
          E::widen(beside.gate, g);
          E::widen(w_post[j], w);
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            post_sum[j][i] = fma2(pair_of(g, i), gate_sum[j][i], post_sum[j][i]);
            out[2 * i] = w[2 * i] * gate_sum[j][i].x;
            out[2 * i + 1] = w[2 * i + 1] * gate_sum[j][i].y;
            gate_sum[j][i] = both(0.0f);
          }
          if (!p.unit_sums && p.d_gate) write_columns(p.d_gate + (int64_t)here.group * p.C, part[j], out);
        }
      }
    }
    if (E::k32) __syncwarp();
    fetch(ahead, stage);
    advance<GATES>(ahead, p, ids, step);
    here = next;
    next = after;
    advance<GATES>(after, p, ids, step);
    beside = beside_next;
    beside_next = beside_after;
    own = own_next;
    stage = stage_next;
    if (CL > 1 && turn_next == 0) parity ^= 1u;
    turn = turn_next;
    meet();
  }
  cp_async_wait<0>();
  if (CL > 1) ptx::cluster_sync();  // no CTA ends while another may send to it
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    if (part[j].hi <= 0) continue;
    const int64_t at = (int64_t)id * p.pitch + (v0 + j * TPR) * 8;
    if (p.pre_sums) write_sums(p.pre_sums + at, pre_sum[j]);
    if (GATES && p.post_sums) write_sums(p.post_sums + at, post_sum[j]);
  }
}

// Sums of those sums, in a fixed order. A CTA takes 32 columns: with its lines of threads either one line of sums of the slots each
// (job 0: d_pre_weight; job 1, with GATES: d_post_weight) or, job 2, groups and their units: d_gate = w_post sum d v of each group and, without
// GATES, d_post_weight = sum over groups of g sum d v.
struct SumParams {
  const float *pre_sums, *post_sums, *unit_sums;
  const void *gate, *post_weight;
  float *d_pre_weight, *d_post_weight, *d_gate;
  int64_t rows_per_group, groups;
  int C, pitch, slots, splits, gate_rows;
  bool shifted;  // lines of sums start at the place of their first row in its vector
  int jobs;
  uint32_t order;  // of the jobs, four bits each (an array, indexed, is copied to local memory: 2 us)
};
constexpr int kSumLines = 32;  // of threads of a CTA, at most

__device__ __forceinline__ float sum_lines(float (*part)[33], float s, int from, int n) {  // over lines [from, from + n), in order
  part[threadIdx.y][threadIdx.x] = s;
  __syncthreads();
  s = 0.0f;
  for (int i = from; i < from + n; ++i) s += part[i][threadIdx.x];
  __syncthreads();
  return s;
}

// Sum of lines i = first, first + stride, ... below n, eight loads at a time (one after another they took 12 us for 296 lines).
template <class Line>
__device__ __forceinline__ float sum_of_lines(int first, int stride, int n, Line line) {
  float s = 0.0f;
  for (int i = first; i < n; i += 8 * stride) {
    float v[8];
#pragma unroll
    for (int u = 0; u < 8; ++u) v[u] = i + u * stride < n ? *line(i + u * stride) : 0.0f;
#pragma unroll
    for (int u = 0; u < 8; ++u) s += v[u];
  }
  return s;
}

template <int DT, int LINES>
__global__ void __launch_bounds__(32 * LINES) norm_sums_kernel(const SumParams p) {
  using E = Element<DT>;
  __shared__ float part[LINES][33];
  ptx::wait_for_previous_grid();
  ptx::launch_dependents();
  const int job = (int)(p.order >> 4 * (blockIdx.x % (uint32_t)p.jobs) & 15u), c = (int)(blockIdx.x / p.jobs) * 32 + threadIdx.x, line = threadIdx.y;
  const bool on = c < p.C;
  auto place = [&](int64_t row) { return (int)((uint64_t)row * (uint64_t)p.C & 7u); };  // of a line of sums whose first row this is
  if (job < 2) {
    const float* src = job == 0 ? p.pre_sums : p.post_sums;
    float s = 0.0f;
    if (on && !p.shifted) s = sum_of_lines(line, LINES, p.slots, [&](int i) { return src + (int64_t)i * p.pitch + c; });
    else if (on)
      s = sum_of_lines(line, LINES, p.slots, [&](int i) {
        const int group = i / p.splits;
        return src + (int64_t)i * p.pitch + place((int64_t)group * p.rows_per_group + (i - group * p.splits)) + c;
      });
    s = sum_lines(part, s, 0, LINES);
    if (on && line == 0) (job == 0 ? p.d_pre_weight : p.d_post_weight)[c] = s;
    return;
  }
  auto sum_of_group = [&](int64_t g, int first, int stride) {
    return sum_of_lines(first, stride, p.gate_rows, [&](int i) {
      return p.unit_sums + (g * p.gate_rows + i) * p.pitch + (p.shifted ? place(g * p.rows_per_group + i) : 0) + c;
    });
  };
  // as many groups at a time as there are lines, or several lines for each group
  int at_once = 1;
  while (at_once < LINES && at_once < p.groups) at_once *= 2;
  const int each = LINES / at_once, mine = line / each;
  const float w = on && p.post_weight ? E::load(p.post_weight, c) : 1.0f;
  float post = 0.0f;
  for (int64_t g = mine; g - mine < p.groups; g += at_once) {
    const bool here = on && g < p.groups;
    const float gate = here && p.gate ? E::load(p.gate, g * p.C + c) : 1.0f;
    float s = here ? sum_of_group(g, line % each, each) : 0.0f;
    if (each > 1) s = sum_lines(part, s, mine * each, each);
    if (here && line % each == 0) {
      if (p.d_gate) p.d_gate[g * p.C + c] = w * s;
      post = fmaf(gate, s, post);
    }
  }
  if (p.d_post_weight && !p.post_sums) {
    post = sum_lines(part, post, 0, LINES);
    if (on && line == 0) p.d_post_weight[c] = post;
  }
}

// ------------------------------------------------------------------------------------------------ rows wider than a CTA's registers
//
// One CTA a row, all vectors of it in turn; what a second pass needs again comes from the caches. The sums over rows are kept in the
// slot's row of the workspace, each element by the thread that owns it.
constexpr int kWideThreads = 1024;

template <int DT>
__device__ __forceinline__ void load_part(const void* src, int64_t row, int C, const Part& p, float (&x)[8]) {
  using E = Element<DT>;
  const int64_t at = row * C + p.first;
  if (src && p.full) {
    E::widen(E::load8(src, at), x);
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = src && e >= p.lo && e < p.hi ? E::load(src, at + e) : 0.0f;
  }
}
template <int DT>
__device__ __forceinline__ void load_columns(const void* src, int64_t offset, const Part& p, float (&x)[8]) {
  Element<DT>::widen(column_part<DT>(src, offset, p), x);
}
__device__ __forceinline__ void add_sums(float* dst, const Part& p, const float (&x)[8], bool start) {
#pragma unroll
  for (int e = 0; e < 8; ++e)
    if (e >= p.lo && e < p.hi) dst[p.first + e] = start ? x[e] : dst[p.first + e] + x[e];
}

template <int DT>
__global__ void __launch_bounds__(kWideThreads, 1) norm_wide_kernel(const NormParams p) {
  using E = Element<DT>;
  __shared__ float buffer[2 * kMaxWarpsPerRow];
  ptx::wait_for_previous_grid();
  ptx::launch_dependents();
  const float inv_c = 1.0f / (float)p.C;
  const int vectors = (p.C + 14) / 8, t = threadIdx.x;  // (at any place of the row's start)
  int turn = 0;
  for (int64_t row = blockIdx.x; row < p.rows; row += gridDim.x) {
    const int64_t gate_at = p.groups > 1 ? row / p.rows_per_group * p.C : 0;
    float rstd_b = 1.0f;
    if (p.post_weight) {
      float s[1] = {0.0f};
      for (int j = t; j < vectors; j += kWideThreads) {
        float b[8];
        load_part<DT>(p.branch, row, p.C, part_of(row, p.C, j), b);
#pragma unroll
        for (int e = 0; e < 8; ++e) s[0] = fmaf(b[e], b[e], s[0]);
      }
      row_sums<kWideThreads>(s, buffer, 0, turn);
      rstd_b = rsqrtf(fmaf(s[0], inv_c, p.eps));
      if (t == 0 && p.post_rstd) p.post_rstd[row] = rstd_b;
    }
    // (the output may lie in the place of an input: its sums are taken before anything is written, and formed again to be)
    auto sums_of = [&](const Part& part, float (&o)[8]) {
      float b[8], w[8], g[8];
      load_part<DT>(p.branch, row, p.C, part, b);
      load_part<DT>(p.residual, row, p.C, part, o);
      load_columns<DT>(p.gate, gate_at, part, g);
      load_columns<DT>(p.post_weight, 0, part, w);
#pragma unroll
      for (int e = 0; e < 8; ++e) o[e] = fmaf(g[e], p.post_weight ? b[e] * rstd_b * w[e] : b[e], p.alpha * o[e]);
    };
    float rstd = 1.0f;
    if (p.pre_weight) {
      float s[1] = {0.0f};
      for (int j = t; j < vectors; j += kWideThreads) {
        float o[8];
        sums_of(part_of(row, p.C, j), o);
#pragma unroll
        for (int e = 0; e < 8; ++e) s[0] = fmaf(o[e], o[e], s[0]);
      }
      row_sums<kWideThreads>(s, buffer, 0, turn);
      rstd = rsqrtf(fmaf(s[0], inv_c, p.eps));
      if (t == 0 && p.pre_rstd) p.pre_rstd[row] = rstd;
    }
    for (int j = t; j < vectors; j += kWideThreads) {
      const Part part = part_of(row, p.C, j);
      float o[8], w[8];
      sums_of(part, o);
      write_part<DT>(p.out, row * p.C, part, E::narrow(o));
      if (p.pre_weight) {
        load_columns<DT>(p.pre_weight, 0, part, w);
#pragma unroll
        for (int e = 0; e < 8; ++e) o[e] = o[e] * rstd * w[e];
        write_part<DT>(p.y, row * p.C, part, E::narrow(o));
      }
    }
  }
}

template <int DT, bool PRUNE>
__global__ void __launch_bounds__(kWideThreads, 1) norm_grad_wide_kernel(const NormGradParams p) {
  using E = Element<DT>;
  __shared__ float buffer[2 * 3 * kMaxWarpsPerRow];
  ptx::wait_for_previous_grid();
  ptx::launch_dependents();
  const float inv_c = 1.0f / (float)p.C;
  const int vectors = (p.C + 14) / 8, rounds = (vectors + kWideThreads - 1) / kWideThreads, t = threadIdx.x;
  int turn = 0;
  bool first_row = true;
  for (int unit = blockIdx.x; unit < p.units; unit += gridDim.x) {
    const int group = unit / p.splits;
    for (int64_t i = unit % p.splits; i < p.rows_per_group; i += p.splits) {
      const int64_t row = group * p.rows_per_group + i;
      const bool first_of_unit = i < p.splits;
      const float rstd_b = p.post_weight ? p.post_rstd[row] : 1.0f, rstd = p.d_y ? p.pre_rstd[row] : 0.0f;
      // v, u, q and d_o + rstd w_pre d_y of one vector, as in norm_grad_kernel
      auto load_terms = [&](const Part& part, float (&v)[8], float (&u)[8], float (&q)[8], float (&d)[8], float (&wd)[8]) {
        float w[8];
        load_part<DT>(p.branch, row, p.C, part, v);
        load_part<DT>(p.d_out, row, p.C, part, d);
        load_columns<DT>(p.gate, (int64_t)group * p.C, part, q);
        load_columns<DT>(p.post_weight, 0, part, w);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          v[e] *= rstd_b;
          q[e] *= w[e];
          u[e] = wd[e] = 0.0f;
        }
        if (p.d_y) {
          load_part<DT>(p.out, row, p.C, part, u);
          load_part<DT>(p.d_y, row, p.C, part, wd);
          load_columns<DT>(p.pre_weight, 0, part, w);
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            u[e] *= rstd;
            wd[e] *= w[e];
            d[e] = fmaf(rstd, wd[e], d[e]);
          }
        }
      };
      float s[3] = {0.0f, 0.0f, 0.0f};
      for (int j = t; j < vectors; j += kWideThreads) {
        const Part part = part_of(row, p.C, j);
        float v[8], u[8], q[8], d[8], wd[8];
        load_terms(part, v, u, q, d, wd);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          s[0] = fmaf(wd[e], u[e], s[0]);
          s[1] = fmaf(q[e] * v[e], d[e], s[1]);
          s[2] = fmaf(q[e] * v[e], u[e], s[2]);
        }
      }
      row_sums<kWideThreads>(s, buffer, 0, turn);
      const float k = rstd * (s[0] * inv_c), mean = (s[1] - k * s[2]) * inv_c;
      for (int round = 0; round < rounds; ++round) {
        const int j = t + round * kWideThreads;
        const Part part = part_of(row, p.C, j);
        float v[8], u[8], q[8], d[8], x[8], w[8];
        load_terms(part, v, u, q, d, x);
        if (p.pre_sums) {
          load_part<DT>(p.d_y, row, p.C, part, x);
#pragma unroll
          for (int e = 0; e < 8; ++e) x[e] *= u[e];
          add_sums(p.pre_sums + (int64_t)blockIdx.x * p.pitch, part, x, first_row);
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          d[e] = fmaf(-k, u[e], d[e]);
          x[e] = p.alpha * d[e];
        }
        if (p.d_residual) write_part<DT>(p.d_residual, row * p.C, part, E::narrow(x));
        if (p.post_sums) {
          load_columns<DT>(p.gate, (int64_t)group * p.C, part, w);
#pragma unroll
          for (int e = 0; e < 8; ++e) x[e] = d[e] * v[e] * w[e];
          add_sums(p.post_sums + (int64_t)blockIdx.x * p.pitch, part, x, first_row);
        }
        if (p.unit_sums || p.d_gate) {
          load_columns<DT>(p.unit_sums ? nullptr : p.post_weight, 0, part, w);
#pragma unroll
          for (int e = 0; e < 8; ++e) x[e] = d[e] * v[e] * w[e];
          add_sums(p.unit_sums ? p.unit_sums + ((int64_t)group * p.gate_rows + unit % p.splits) * p.pitch : p.d_gate + (int64_t)group * p.C, part,
                   x, first_of_unit);
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = p.post_weight ? rstd_b * fmaf(q[e], d[e], -v[e] * mean) : q[e] * d[e];
        const typename E::Raw packed = E::narrow(x);
        if (p.d_branch) write_part<DT>(p.d_branch, row * p.C, part, packed);
        if constexpr (PRUNE) {
          const int64_t vec = row * (p.C / 8) + j;
          const uint4 c = prune_any<E::kF16>(packed.a, vec, p.seed_lo, p.seed_hi, p.n, p.m, p.scheme, j & 3);
          if (part.full) {
            if (p.values) p.values[vec] = make_uint2(c.x, c.y);
            if (p.meta) p.meta[vec] = (uint8_t)c.z;
          }
        }
      }
      first_row = false;
    }
  }
  if (first_row) {
    const float zero[8] = {};
    for (int j = t; j < vectors; j += kWideThreads) {
      const Part none = part_of(0, p.C, j);
      if (p.pre_sums) add_sums(p.pre_sums + (int64_t)blockIdx.x * p.pitch, none, zero, true);
      if (p.post_sums) add_sums(p.post_sums + (int64_t)blockIdx.x * p.pitch, none, zero, true);
    }
  }
}

// ------------------------------------------------------------------------------------------------ host

int gcd8(int c) { return c % 8 == 0 ? 8 : c % 4 == 0 ? 4 : c % 2 == 0 ? 2 : 1; }

// Threads of a row of `vectors` vectors each: the smallest power of two from 32 to `most` that holds it at any place that it may start
// at; 0: the wide kernels.
int threads_of_row(int64_t C, int vectors, int most) {
  for (int t = 32; t <= most; t *= 2)
    if (C + 8 - gcd8((int)(C % 8)) <= 8 * vectors * t) return t;
  return 0;
}

struct Plan {
  int tpr, vectors, cluster, slots_per_cta, ctas, period, splits, units, gate_rows;  // ctas: clusters of them where cluster > 1
  bool gates;  // a slot's rows may have several gates: the kernel that carries them along
  int ids() const { return ctas * slots_per_cta; }
  bool carries() const { return gates || tpr == 0; }  // d_post_weight needs sums of its own
  bool by_units() const { return !carries() || splits > 1; }
  size_t lines(int64_t groups) const {  // of sums in the workspace
    return (size_t)ids() * (carries() ? 2 : 1) + (by_units() ? (size_t)groups * gate_rows : 0);
  }
};
int64_t pitch_of(int64_t C) { return (C + 7 + 7) / 8 * 8; }  // (a row may start at the last place of its first vector)

// How rows are dealt to slots (groups of threads). All rows of a slot start at the same place of a vector: they are multiples of the period
// apart.
Plan plan_slots(int64_t rows, int64_t C, int tpr, int ctas_per_sm) {
  Plan p = {};
  p.tpr = tpr;
  p.vectors = p.cluster = 1;
  p.slots_per_cta = tpr == 0 || tpr >= 256 ? 1 : 256 / tpr;
  p.period = 8 / gcd8((int)(C % 8));
  const int64_t most = (int64_t)sm_count() * ctas_per_sm, wanted = (rows + p.slots_per_cta - 1) / p.slots_per_cta;
  p.ctas = (int)(wanted < most ? wanted : most);
  return p;
}

// Forward: rows at the stride of all slots.
Plan forward_plan(int64_t rows, int64_t C) {
  int tpr = threads_of_row(C, 1, 1024), vectors = 1;
  if (tpr == 0) tpr = threads_of_row(C, vectors = 2, 1024);
  Plan p = plan_slots(rows, C, tpr, tpr == 0 ? 2 : tpr > 512 ? 1 : tpr > 256 ? 2 : 4);
  p.vectors = vectors;
  if (p.ids() < rows && p.period > p.slots_per_cta) p.ctas -= p.ctas % (p.period / p.slots_per_cta);
  return p;
}

// Backward: rows in units of one gate.
Plan deal_units(Plan p, int64_t rows, int64_t groups) {
  const int64_t per_group = rows / groups;
  int64_t ctas = p.ctas;
  const int64_t ids = ctas * p.slots_per_cta;
  int64_t splits = ids / groups;
  splits -= splits % p.period;
  if (splits < p.period) splits = per_group == 1 || p.period == 1 ? 1 : p.period;
  if (splits >= per_group) splits = (per_group + p.period - 1) / p.period * p.period;
  if (per_group == 1) splits = 1;
  p.splits = (int)splits;
  p.units = (int)(groups * splits);
  p.gate_rows = (int)(splits < per_group ? splits : per_group);
  if (p.units > ids) {
    // a slot takes several units: the first rows of two of them are ids / splits groups apart, or (splits == 1) ids groups
    const int64_t multiple = splits == 1 ? p.period : (int64_t)p.period * splits;
    const int64_t need = multiple > p.slots_per_cta ? multiple / p.slots_per_cta : 1;
    ctas = ctas < need ? need : ctas - ctas % need;
  } else {
    ctas = (p.units + p.slots_per_cta - 1) / p.slots_per_cta;
  }
  p.ctas = (int)ctas;
  p.gates = p.units > p.ids();
  return p;
}

Plan backward_plan(int64_t rows, int64_t C, int64_t groups, bool fp32) {
  // one gate a slot: two vectors a thread (fp32: shared memory holds the stages of one)
  const int vectors = fp32 ? 1 : 2;
  int tpr = 0, cluster = 1;
  for (; tpr == 0 && cluster <= 4; cluster *= 2) tpr = threads_of_row(C, vectors * cluster, 512);
  cluster /= 2;
  if (tpr != 0) {
    Plan p = plan_slots(rows, C, tpr, tpr > 256 ? 1 : 2);
    // (clusters of four: not every multiprocessor finds three neighbours)
    const int fit = cluster == 4 ? sm_count() / 4 * 7 / 8 : sm_count() / 2;
    if (cluster > 1 && p.ctas > fit) p.ctas = fit;
    p = deal_units(p, rows, groups);
    p.vectors = vectors;
    p.cluster = cluster;
    if (!p.gates) return p;
  }
  tpr = threads_of_row(C, 1, fp32 ? 512 : 1024);
  Plan p = deal_units(plan_slots(rows, C, tpr, tpr == 0 || tpr > 256 ? 1 : 2), rows, groups);
  p.gates = tpr != 0;
  return p;
}

template <auto Kernel, typename... Args>
cudaError_t launch(int64_t ctas, dim3 block, int smem, int cluster, cudaStream_t stream, const Args&... args) {
  static bool done[kMaxDevices] = {};  // (what a kernel asks for is always the same)
  const int dev = current_device();
  if (dev < 0) return cudaErrorInvalidDevice;
  if (smem > 0 && !done[dev]) {
    const cudaError_t e = cudaFuncSetAttribute(Kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
    if (e != cudaSuccess) return e;
    done[dev] = true;
  }
  if (ctas > 0x7FFFFFFF) return cudaErrorInvalidValue;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)ctas);
  cfg.blockDim = block;
  cfg.dynamicSmemBytes = (size_t)smem;
  cfg.stream = stream;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = (unsigned)cluster;
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = cluster > 1 ? 2 : 1;
  return cudaLaunchKernelEx(&cfg, Kernel, args...);
}

template <int DT>
cudaError_t launch_forward(const NormParams& p, const Plan& plan, cudaStream_t stream) {
  switch (plan.tpr * plan.vectors) {
#define SDGP_ROW(T, NV) \
  case T * NV: return launch<norm_kernel<DT, T, NV>>(plan.ctas, dim3(kCtaThreads<T>), Ring<DT, T, 2 * NV, 1>::kBytes, 1, stream, p);
    SDGP_ROW(32, 1) SDGP_ROW(64, 1) SDGP_ROW(128, 1) SDGP_ROW(256, 1) SDGP_ROW(512, 1) SDGP_ROW(1024, 1) SDGP_ROW(1024, 2)
#undef SDGP_ROW
  }
  return launch<norm_wide_kernel<DT>>(plan.ctas, dim3(kWideThreads), 0, 1, stream, p);
}

template <int DT, bool ALIGNED, bool PRUNE>
cudaError_t launch_backward_form(const NormGradParams& p, const Plan& plan, cudaStream_t stream) {
#define SDGP_ROW(T, NV, CL, GATES)                                                                                                \
  case T * CL:                                                                                                                     \
    return launch<norm_grad_kernel<DT, T, NV, CL, GATES, ALIGNED, PRUNE>>((int64_t)plan.ctas * CL, dim3(kCtaThreads<T>),            \
                                                                          Ring<DT, T, 4 * NV, 2>::kBytes, CL, stream, p);
  if (!plan.gates) {
    constexpr int NV = DT == SDGP_FP32 ? 1 : 2;
    if (plan.vectors == NV) {
      switch (plan.tpr * plan.cluster) {
        SDGP_ROW(32, NV, 1, false) SDGP_ROW(64, NV, 1, false) SDGP_ROW(128, NV, 1, false) SDGP_ROW(256, NV, 1, false) SDGP_ROW(512, NV, 1, false)
        SDGP_ROW(512, NV, 2, false) SDGP_ROW(512, NV, 4, false)
      }
    }
  } else {
    switch (plan.tpr) {
      SDGP_ROW(32, 1, 1, true) SDGP_ROW(64, 1, 1, true) SDGP_ROW(128, 1, 1, true) SDGP_ROW(256, 1, 1, true) SDGP_ROW(512, 1, 1, true)
    }
    if constexpr (DT != SDGP_FP32) {
      switch (plan.tpr) { SDGP_ROW(1024, 1, 1, true) }
    }
  }
#undef SDGP_ROW
  return launch<norm_grad_wide_kernel<DT, PRUNE>>(plan.ctas, dim3(kWideThreads), 0, 1, stream, p);
}

template <int DT>
cudaError_t launch_backward(const NormGradParams& p, const Plan& plan, cudaStream_t stream) {
  if (plan.period != 1) return launch_backward_form<DT, false, false>(p, plan, stream);
  if constexpr (DT != SDGP_FP32) {
    if (p.values || p.meta) return launch_backward_form<DT, true, true>(p, plan, stream);
  }
  return launch_backward_form<DT, true, false>(p, plan, stream);
}

template <int DT>
cudaError_t launch_sums(const SumParams& p, int64_t ctas, int lines, cudaStream_t stream) {
  if (lines == 8) return launch<norm_sums_kernel<DT, 8>>(ctas, dim3(32, 8), 0, 1, stream, p);
  if (lines == 16) return launch<norm_sums_kernel<DT, 16>>(ctas, dim3(32, 16), 0, 1, stream, p);
  return launch<norm_sums_kernel<DT, kSumLines>>(ctas, dim3(32, kSumLines), 0, 1, stream, p);
}

}  // namespace

cudaError_t take_error_norm(unsigned int* word) { return take_error_word(word); }

cudaError_t launch_residual_norm(const void* branch, const void* residual, const void* post_weight, const void* gate, const void* pre_weight,
                                 int64_t rows, int64_t C, int64_t groups, float alpha, float eps, int dtype, void* out, void* y,
                                 float* post_rstd, float* pre_rstd, cudaStream_t stream) {
  const NormParams p = {branch, residual, post_weight, gate, pre_weight, out, y, post_rstd, pre_rstd, rows, rows / groups, (int)C, (int)groups,
                        alpha, eps};
  const Plan plan = forward_plan(rows, C);
  if (dtype == SDGP_BF16) return launch_forward<SDGP_BF16>(p, plan, stream);
  if (dtype == SDGP_FP16) return launch_forward<SDGP_FP16>(p, plan, stream);
  return launch_forward<SDGP_FP32>(p, plan, stream);
}

size_t residual_norm_backward_floats(int64_t rows, int64_t C, int64_t groups) {
  size_t most = 0;
  for (const int64_t g : {groups, (int64_t)1}) {  // (1: a call without gates)
    for (const bool fp32 : {false, true}) {
      const size_t lines = backward_plan(rows, C, g, fp32).lines(g);
      if (lines > most) most = lines;
    }
  }
  return most * pitch_of(C);
}

cudaError_t launch_residual_norm_backward(const void* branch, const void* out, const void* d_out, const void* d_y, const void* post_weight,
                                          const void* gate, const void* pre_weight, const float* post_rstd, const float* pre_rstd,
                                          int64_t rows, int64_t C, int64_t groups, float alpha, int n, int m, int scheme, uint64_t seed,
                                          int dtype, void* d_residual, void* d_branch, float* d_gate, float* d_post_weight,
                                          float* d_pre_weight, void* values, void* meta, float* workspace, cudaStream_t stream) {
  if (!gate) groups = 1;
  const Plan plan = backward_plan(rows, C, groups, dtype == SDGP_FP32);
  const int64_t pitch = pitch_of(C), slot_floats = plan.ids() * pitch;
  float* pre_sums = d_pre_weight ? workspace : nullptr;
  float* post_sums = d_post_weight && plan.carries() ? workspace + slot_floats : nullptr;
  float* unit_sums = plan.by_units() && (d_gate || (d_post_weight && !plan.carries())) ? workspace + slot_floats * (plan.carries() ? 2 : 1) : nullptr;
  const NormGradParams p = {branch, out, d_out, d_y, post_weight, gate, pre_weight, post_rstd, pre_rstd, d_residual, d_branch,
                            (uint2*)values, (uint8_t*)meta, d_gate, pre_sums, post_sums, unit_sums, rows, rows / groups, (int)C, (int)pitch,
                            plan.splits, plan.units, plan.gate_rows, alpha, n, m, scheme, (uint32_t)seed, (uint32_t)(seed >> 32)};
  const cudaError_t e = dtype == SDGP_BF16   ? launch_backward<SDGP_BF16>(p, plan, stream)
                        : dtype == SDGP_FP16 ? launch_backward<SDGP_FP16>(p, plan, stream)
                                             : launch_backward<SDGP_FP32>(p, plan, stream);
  if (e != cudaSuccess || (!pre_sums && !post_sums && !unit_sums)) return e;
  SumParams q = {pre_sums, post_sums, unit_sums, gate, post_weight, d_pre_weight, d_post_weight, d_gate, rows / groups, groups, (int)C,
                 (int)pitch, plan.ids(), plan.splits, plan.gate_rows, plan.tpr != 0 && plan.period != 1, 0, 0u};
  const bool present[3] = {pre_sums != nullptr, post_sums != nullptr, unit_sums != nullptr};
  for (uint32_t job = 0; job < 3; ++job)
    if (present[job]) q.order |= job << 4 * q.jobs++;
  // As many lines of threads as let the CTAs of two jobs run at once (16384 columns: 31 us with 32 lines everywhere). Not by the jobs that there
  // are: which sums are asked for changes none of them.
  const int64_t columns = (C + 31) / 32, ctas = q.jobs * columns;
  int lines = kSumLines;
  while (lines > 8 && 2 * columns * 32 * lines > (int64_t)sm_count() * 2048) lines /= 2;
  return dtype == SDGP_BF16   ? launch_sums<SDGP_BF16>(q, ctas, lines, stream)
         : dtype == SDGP_FP16 ? launch_sums<SDGP_FP16>(q, ctas, lines, stream)
                              : launch_sums<SDGP_FP32>(q, ctas, lines, stream);
}

}  // namespace sdgp
