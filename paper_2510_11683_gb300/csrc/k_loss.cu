// Losses on token log-probabilities, with their gradients: the clipped policy loss
// with a KL term and the preference loss on paired log ratios (include/bgpo_train.h
// has the formulas).
//
// Both are elementwise over [rows, T] arrays apart from two sums over a row (its token
// count n and its sum of log ratios) and the loss itself. A row (a pair of rows) is the
// work of one team: a warp up to 256 tokens, a block of up to 512 threads up to 4,096, a
// cluster of up to 8 such blocks beyond. Each thread of a team holds 8 tokens in
// registers while the team's sums go through shuffles, shared memory and the cluster's
// shared memory, then writes their gradients: every input is read once. (A row of more than
// 32,768 tokens is read twice by one cluster, both times with loads that ask L2 to let go of
// their lines first: 64 rows of 40,000, half of the tokens counting, 24 us; 4 of 10^6 without
// a mask 55.) Where a loss needs no sum over a row its chunks of 256 tokens are dealt to
// warps. The mean over all tokens of a masked batch needs their count first, which a kernel
// of its own takes from the mask. Blocks leave their shares of the loss; the last to finish
// adds them up in block order.
//
// The mask comes first: values of tokens that do not count are never used, and not loaded
// but beside ones that do. Arrays that run along memory move in vectors of eight tokens.
//
// Sums are fp32 in trees of a bounded depth (a thread's eight, a warp, a block, a cluster, the
// blocks); chains whose length grows with the batch or the row carry what their roundings
// leave out.
//
// What bounds them: HBM where a batch outgrows L2 (policy loss with KL, 4096 x 4096 tokens
// without a mask: 44 us for 268 MB, 6.1 TB/s; with ragged rows and the mean by rows, 59% of
// the tokens counting: 43 us for 202 MB, a team's barrier and the longest row of a round
// beside it), the chain mask - values - sums - gradient and a few rounds of teams below
// (preference loss, 1024 pairs of 2,047: 16 us for 40 MB; policy loss, 512 x 1023 with the mean
// over tokens: 8.6 for both kernels, from L2), and for smaller ones the host: 8 to 12 us in the
// call, and as much again in a caller's transposed views of Monte Carlo samples.
#include <math.h>

#include "bgpo_device.cuh"
#include "bgpo_train.h"
#include "train_internal.h"

namespace bgpo {

namespace {

constexpr int kE = 8;                    // tokens of a thread
constexpr int kChunk = 32 * kE;          // tokens of a warp
constexpr int kWarpTeams = 8;            // warps of a block of warp teams
constexpr int kMaxThreads = 512;
constexpr int kMaxCluster = 8;
constexpr int32_t kStatusNonfinite = 5;  // BGPO_ERR_NONFINITE

__device__ __forceinline__ int32_t warp_sum_i(int32_t v) {
  return (int32_t)__reduce_add_sync(0xffffffffu, (unsigned)v);
}

// (for what is read once; when it came, 44.4 -> 42.0 us at 4096 x 4096 with ragged rows)
__device__ __forceinline__ void load8(const float* p, float (&v)[kE]) {
  asm volatile("ld.global.L1::no_allocate.L2::evict_first.v8.f32 "
               "{%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
               : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3]), "=f"(v[4]), "=f"(v[5]),
                 "=f"(v[6]), "=f"(v[7])
               : "l"(p)
               : "memory");
}
__device__ __forceinline__ void store8(float* p, const float (&v)[kE]) {
  asm volatile("st.global.v8.f32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p), "f"(v[0]),
               "f"(v[1]), "f"(v[2]), "f"(v[3]), "f"(v[4]), "f"(v[5]), "f"(v[6]), "f"(v[7])
               : "memory");
}

// ---- tokens of a thread -------------------------------------------------------------

// How a thread's eight tokens of a chunk lie:
//   kEights   eight neighbours, on 32 bytes in every array (8 in a mask), one load or store
//             of 32 bytes an array; rows begin and end with an eight
//   kShifted  the same, but rows may start and end between boundaries (in all arrays
//             alike), so that a row's first and last eight may reach past its ends
//   kSingle   eight single tokens, a team's width apart, at any strides
// The first two ask that the arrays have one row stride, so that one offset serves them all.
// 1024 pairs of 2,047 took 30 us in single tokens, 21 in vectors.
enum Mode : int { kSingle = 0, kEights = 1, kShifted = 2 };

// Tokens of one thread in a chunk of a row (T <= 2^30).
template <int MODE>
struct Span {
  int64_t off;     // kEights, kShifted: of the first token in every array
  uint32_t row;    // kSingle
  int32_t col, step, T;
  __device__ __forceinline__ Span() {}
  // stride: of the arrays' rows; phase: elements by which the arrays start past a boundary
  __device__ __forceinline__ Span(uint32_t row_, uint32_t chunk0, int threads, int tid, int32_t T_,
                                  int64_t stride, int phase)
      : row(row_), step(threads), T(T_) {
    if (MODE == kSingle) {
      col = (int32_t)chunk0 + tid;
    } else {
      const int64_t begin = (int64_t)row_ * stride;
      col = (int32_t)chunk0 + 8 * tid;
      if (MODE == kShifted) col -= (int)((uint32_t)begin + (uint32_t)phase & 7u);
      off = begin + col;
    }
  }
  __device__ __forceinline__ bool whole() const {   // all of the eight lies in the row
    return MODE == kEights ? col < T : col >= 0 && col + kE <= T;
  }
  __device__ __forceinline__ bool has(int k) const {
    if (MODE == kSingle) return col + k * step < T;
    return MODE != kEights && col + k >= 0 && col + k < T;   // (where it is not whole)
  }
};

// The mask at a thread's tokens, as loaded; bits() waits for it. Bit k: token k counts.
template <int MODE>
struct Mask {
  uint32_t q[MODE == kSingle ? kE : 2];
  __device__ __forceinline__ void load(const View<const uint8_t>& m, const Span<MODE>& c) {
    if (MODE == kSingle) {
      const uint8_t* p = m.p + c.row * m.row + c.col * m.col;
      const int64_t step = c.step * m.col;
#pragma unroll
      for (int k = 0; k < kE; ++k) q[k] = !c.has(k) ? 0u : m.p ? p[k * step] : 1u;
    } else if (c.whole()) {
      q[0] = q[1] = 0x01010101u;
      if (m.p) {
        const uint2 w = *reinterpret_cast<const uint2*>(m.p + c.off);
        q[0] = w.x;
        q[1] = w.y;
      }
    } else {
      q[0] = q[1] = 0;
#pragma unroll
      for (int k = 0; k < kE; ++k)
        if (c.has(k) && (!m.p || m.p[c.off + k])) q[k / 4] |= 1u << (8 * (k % 4));
    }
  }
  __device__ __forceinline__ uint32_t bits() const {
    uint32_t b = 0;
    if (MODE == kSingle) {
#pragma unroll
      for (int k = 0; k < kE; ++k) b |= q[k] ? 1u << k : 0u;
    } else {
#pragma unroll
      for (int g = 0; g < 2; ++g) {
        // bit 7 of each byte: the byte is not zero; gathered into four bits
        const uint32_t nz = (q[g] | ((q[g] & 0x7f7f7f7fu) + 0x7f7f7f7fu)) & 0x80808080u;
        b |= ((nz * 0x00204081u) >> 28) << (4 * g);
      }
    }
    return b;
  }
};

template <int MODE>
__device__ __forceinline__ uint32_t load_mask(const View<const uint8_t>& m, const Span<MODE>& c) {
  Mask<MODE> q;
  q.load(m, c);
  return q.bits();
}

// Values of the tokens in `bits`; others are left or overwritten as it comes.
template <int MODE>
__device__ __forceinline__ void load_floats(const View<const float>& a, const Span<MODE>& c,
                                            uint32_t bits, float (&v)[kE]) {
  if (MODE == kSingle) {
    const float* p = a.p + c.row * a.row + c.col * a.col;
    const int64_t step = c.step * a.col;
#pragma unroll
    for (int k = 0; k < kE; ++k)
      if ((bits >> k) & 1u) v[k] = p[k * step];
  } else if (bits) {
    const float* p = a.p + c.off;
    if (c.whole()) {
      load8(p, v);
    } else {
#pragma unroll
      for (int k = 0; k < kE; ++k)
        if ((bits >> k) & 1u) v[k] = p[k];
    }
  }
}

template <int MODE>
__device__ __forceinline__ void store_floats(const View<float>& a, const Span<MODE>& c,
                                             const float (&v)[kE]) {
  if (MODE == kSingle) {
    float* p = a.p + c.row * a.row + c.col * a.col;
    const int64_t step = c.step * a.col;
#pragma unroll
    for (int k = 0; k < kE; ++k)
      if (c.has(k)) p[k * step] = v[k];
  } else {
    float* p = a.p + c.off;
    if (c.whole()) {
      store8(p, v);
    } else {
#pragma unroll
      for (int k = 0; k < kE; ++k)
        if (c.has(k)) p[k] = v[k];
    }
  }
}

// Who works on a row: kNone where no sum over it is needed (its chunks go to warps as they
// come), else a team: a warp, a block, a cluster of blocks (each a part of the row), or a
// cluster of which a thread takes more tokens of the row than its registers hold.
enum TeamKind : int { kNone = 0, kWarp = 1, kBlock = 2, kCluster = 3, kMany = 4 };

// Most threads of a block, and blocks of that size that an SM holds by the registers they
// may take: 85 a thread for warps on their own (24 an SM; at 64, spills made 4096 x 4096
// tokens without a mask take 52 us instead of 43), 64 in blocks (one block of 512 threads
// and 128 registers instead of two: 45 us instead of 41 at 4096 x 4096 ragged), 128 for
// single tokens, whose addresses take more. What still spills, in bytes a thread: policy
// kernels of blocks and clusters 28 to 44, of single tokens 36; preference kernels of blocks
// up to 12, of single tokens 268.
constexpr int most_threads(int team) { return team >= kBlock ? kMaxThreads : 32 * kWarpTeams; }
constexpr int blocks_per_sm(int mode, int team) {
  return team >= kBlock ? (mode == kSingle ? 1 : 2) : (mode == kSingle ? 2 : 3);
}

// ---- sums ------------------------------------------------------------------------------

// A team's sums of M counts and (with_s) values at once, the same in all its threads. Every
// warp adds the block's up alike (a tree), blocks of a cluster in their order. The buffers
// alternate from call to call: one barrier a call keeps them apart.
template <int M>
struct TeamSums {
  struct Shared {
    int32_t n[2][M][kMaxThreads / 32];
    float s[2][M][kMaxThreads / 32];
    int32_t cn[2][M];
    float cs[2][M];
  };
  Shared* sh;
  int turn;
  uint32_t blocks;   // of the cluster
  __device__ __forceinline__ TeamSums(Shared* p, uint32_t cluster)
      : sh(p), turn(0), blocks(cluster) {}
  template <int TEAM>
  __device__ __forceinline__ void sum(int32_t (&n)[M], float (&s)[M], bool with_s) {
#pragma unroll
    for (int i = 0; i < M; ++i) {
      n[i] = warp_sum_i(n[i]);
      if (with_s) s[i] = warp_sum(s[i]);
    }
    if (TEAM < kBlock) return;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
    turn ^= 1;
    if (lane == 0) {
#pragma unroll
      for (int i = 0; i < M; ++i) {
        sh->n[turn][i][warp] = n[i];
        if (with_s) sh->s[turn][i][warp] = s[i];
      }
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < M; ++i) {
      n[i] = warp_sum_i(lane < warps ? sh->n[turn][i][lane] : 0);
      if (with_s) s[i] = warp_sum(lane < warps ? sh->s[turn][i][lane] : 0.f);
    }
    if (TEAM < kCluster) return;
    if (threadIdx.x == 0) {
#pragma unroll
      for (int i = 0; i < M; ++i) {
        sh->cn[turn][i] = n[i];
        sh->cs[turn][i] = with_s ? s[i] : 0.f;
      }
    }
    __syncwarp();
    cluster_sync();
#pragma unroll
    for (int i = 0; i < M; ++i) {
      n[i] = 0;
      s[i] = 0.f;
      for (uint32_t r = 0; r < blocks; ++r) {
        int32_t qn;
        float qs;
        asm volatile("ld.shared::cluster.s32 %0, [%1];"
                     : "=r"(qn) : "r"(map_to_cta(smem_addr(&sh->cn[turn][i]), r)) : "memory");
        asm volatile("ld.shared::cluster.f32 %0, [%1];"
                     : "=f"(qs) : "r"(map_to_cta(smem_addr(&sh->cs[turn][i]), r)) : "memory");
        n[i] += qn;
        s[i] += qs;
      }
    }
  }
};

// Adds up the threads' values of all blocks: four floats and three counts each. True in
// thread 0 of the last block to leave its own, which then has the totals, added in block
// order. (The fence and the ticket cost about 2 us, so a grid of one block skips them.)
__device__ __forceinline__ void warp_totals(LossTotals& t) {
#pragma unroll
  for (int i = 0; i < 4; ++i) t.f[i] = warp_sum(t.f[i]);
#pragma unroll
  for (int i = 0; i < 3; ++i)
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) t.c[i] += __shfl_xor_sync(0xffffffffu, t.c[i], o);
}

__device__ __forceinline__ void block_totals(LossTotals& t, LossTotals (&s)[kMaxThreads / 32]) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
  warp_totals(t);
  if (lane == 0) s[warp] = t;
  __syncthreads();
  if (warp != 0) return;
  if (lane < warps) {
    t = s[lane];
  } else {
    t = LossTotals{};
  }
  warp_totals(t);
}

__device__ __forceinline__ bool grid_totals(const TrainWs& w, LossTotals& t) {
  __shared__ LossTotals s_t[kMaxThreads / 32];
  __shared__ bool s_last;
  block_totals(t, s_t);
  if (gridDim.x == 1) return threadIdx.x == 0;
  if (threadIdx.x == 0) {
    w.sums[blockIdx.x] = t;
    __threadfence();
    s_last = atomicInc(w.ticket, gridDim.x - 1) == gridDim.x - 1;
    __threadfence();
  }
  __syncthreads();
  if (!s_last) return false;
  t = LossTotals{};
  Sum2 sum[4] = {};
  for (int b = threadIdx.x; b < (int)gridDim.x; b += blockDim.x) {
    const float4 f = __ldcg(reinterpret_cast<const float4*>(w.sums[b].f));
    sum[0].add(f.x); sum[1].add(f.y); sum[2].add(f.z); sum[3].add(f.w);
#pragma unroll
    for (int i = 0; i < 3; ++i) t.c[i] += __ldcg(&w.sums[b].c[i]);
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) t.f[i] = sum[i].value();
  block_totals(t, s_t);
  return threadIdx.x == 0;
}

// ---- tokens that count, over the whole mask ----------------------------------------------

template <int MODE>
__global__ void __launch_bounds__(32 * kWarpTeams)
    k_count_tokens(int32_t N, int32_t T, uint32_t per_row, int phase, View<const uint8_t> mask,
                   TrainWs w) {
  pdl_begin();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const uint32_t units = (uint32_t)N * per_row;
  uint32_t n = 0;
  for (uint32_t u = blockIdx.x * kWarpTeams + warp; u < units; u += gridDim.x * kWarpTeams) {
    const uint32_t row = u / per_row;
    n += __popc(load_mask<MODE>(
        mask, Span<MODE>(row, (u - row * per_row) * kChunk, 32, lane, T, mask.row, phase)));
  }
  __shared__ unsigned long long s_n[kWarpTeams];
  n = __reduce_add_sync(0xffffffffu, n);
  if (lane == 0) s_n[warp] = n;
  __syncthreads();
  if (threadIdx.x == 0) {
    unsigned long long t = 0;
    for (int i = 0; i < kWarpTeams; ++i) t += s_n[i];
    w.totals[blockIdx.x] = t;
  }
}

// ---- clipped policy loss with a KL term ---------------------------------------------------

// e^k - 1 - k for |k| <= 1. It is k^2 / 2 for small k, where the difference would keep few
// of its bits (none below k = 2e-4): the series of e^k, whose first left-out term is below
// 1.2 x 2^-24 of it (most at k = -1).
__device__ __forceinline__ float exp_rest(float k) {
  float p = fmaf(k, 1.f / 3628800.f, 1.f / 362880.f);
  p = fmaf(k, p, 1.f / 40320.f);
  p = fmaf(k, p, 1.f / 5040.f);
  p = fmaf(k, p, 1.f / 720.f);
  p = fmaf(k, p, 1.f / 120.f);
  p = fmaf(k, p, 1.f / 24.f);
  p = fmaf(k, p, 1.f / 6.f);
  p = fmaf(k, p, 0.5f);
  return k * k * p;
}

// Two fp32 values in one 64-bit register: one instruction works on both.
struct Two {
  uint64_t r;
  __device__ __forceinline__ Two(float a, float b) {
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
  }
  __device__ __forceinline__ void get(float& a, float& b) const {
    asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(r));
  }
};
__device__ __forceinline__ Two fma2(Two a, Two b, Two c) {
  asm("fma.rn.f32x2 %0, %1, %2, %0;" : "+l"(c.r) : "l"(a.r), "l"(b.r));
  return c;
}
__device__ __forceinline__ Two mul2(Two a, Two b) {
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(a.r) : "l"(a.r), "l"(b.r));
  return a;
}
__device__ __forceinline__ Two add2(Two a, Two b) {
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(a.r) : "l"(a.r), "l"(b.r));
  return a;
}

__device__ __forceinline__ Two sub2(Two a, Two b) {
  asm("sub.rn.f32x2 %0, %1, %2;" : "=l"(a.r) : "l"(a.r), "l"(b.r));
  return a;
}

// exp_rest of two values.
__device__ __forceinline__ Two exp_rest2(Two k) {
  Two p = fma2(k, Two(1.f / 3628800.f, 1.f / 3628800.f), Two(1.f / 362880.f, 1.f / 362880.f));
  p = fma2(k, p, Two(1.f / 40320.f, 1.f / 40320.f));
  p = fma2(k, p, Two(1.f / 5040.f, 1.f / 5040.f));
  p = fma2(k, p, Two(1.f / 720.f, 1.f / 720.f));
  p = fma2(k, p, Two(1.f / 120.f, 1.f / 120.f));
  p = fma2(k, p, Two(1.f / 24.f, 1.f / 24.f));
  p = fma2(k, p, Two(1.f / 6.f, 1.f / 6.f));
  p = fma2(k, p, Two(0.5f, 0.5f));
  return mul2(mul2(k, k), p);
}

// A thread's sums over all its units. They carry what their roundings leave out: a chain of
// plain additions grows with the batch (2 x 10^4 equal ones: 1.6e-4 off).
// Blocks, whose 64 registers a thread are full, keep them in shared memory (32 bytes of spills
// a thread instead of 112 for rows in vectors).
enum PolicySum : int { kPg = 0, kKl = 1, kRat = 2 };
template <bool BLOCK>
struct PolicySums {
  Sum2 q[BLOCK ? 1 : 3];
  Sum2* slot;    // of this thread: sum i is slot[i * blockDim.x]
  uint32_t low = 0, high = 0, tok = 0;
  __device__ __forceinline__ explicit PolicySums(Sum2* slots) : slot(slots + threadIdx.x) {
#pragma unroll
    for (int i = 0; i < 3; ++i) at(i) = {};
  }
  __device__ __forceinline__ Sum2& at(int i) {
    return BLOCK ? slot[i * blockDim.x] : q[BLOCK ? 0 : i];
  }
  __device__ __forceinline__ void add(PolicySum i, float x) { at(i).add(x); }
  __device__ __forceinline__ float value(PolicySum i) { return at(i).value(); }
};

// An advantage as its magnitude and a sign s: with x = s r, a token's term is -|A| min(x,
// bound) and is clipped where x > bound. (bound: 1 + clip_high for A > 0, -(1 - clip_low) for
// A < 0; infinite for A = 0 and NaN.)
struct Side {
  float mag, s, bound;
  __device__ __forceinline__ Side(const PolicyArgs& a, float A)
      : mag(fabsf(A)), s(A < 0.f ? -1.f : 1.f),
        bound(A > 0.f ? a.hi : A < 0.f ? -a.lo : INFINITY) {}
};

// Instructions come next after HBM (120 a token took 94 us at 4096 x 4096, 67 took 48, 40 took
// 39; the sums' remainders and the mask in them made it 45 and 41): what is the same for all tokens is asked once a unit, a warp whose tokens all count
// tests none of them, and two values go through one instruction where they can. A token that
// does not count has log ratios 0: its ratio is 1, inside every clipping range, and is dropped
// before the sums (adding it and taking a count of them out again would leave an absolute
// error, which small ratios behind a scattered mask vanish in).
template <int MODE>
struct PolicyChunk {
  uint32_t bits;
  bool live, full;                // one token, every token of the warp counts
  float d[kE], kr[kE], adv[kE];   // log ratios to the old policy and of the reference
  // Starts the loads of the tokens that count in `b`.
  __device__ __forceinline__ void load(const PolicyArgs& a, const Span<MODE>& c, uint32_t b) {
    bits = b;
    live = __any_sync(0xffffffffu, b != 0);
    full = __all_sync(0xffffffffu, b == 0xffu);
    if (!live) return;
    load_floats<MODE>(a.lp, c, bits, lp);
    load_floats<MODE>(a.old, c, bits, d);
    if (a.ref.p) load_floats<MODE>(a.ref, c, bits, kr);
    if (a.token_adv) load_floats<MODE>(a.adv, c, bits, adv);
  }
  __device__ __forceinline__ void ratios(const PolicyArgs& a) {
    if (!live) return;
#pragma unroll
    for (int k = 0; k < kE; k += 2)
      sub2(Two(lp[k], lp[k + 1]), Two(d[k], d[k + 1])).get(d[k], d[k + 1]);
    if (a.ref.p) {
#pragma unroll
      for (int k = 0; k < kE; k += 2)
        sub2(Two(kr[k], kr[k + 1]), Two(lp[k], lp[k + 1])).get(kr[k], kr[k + 1]);
    }
    if (full) return;
    // (an eight brings the neighbours of its tokens too, and may not have been loaded)
#pragma unroll
    for (int k = 0; k < kE; ++k) {
      const bool m = (bits >> k) & 1u;
      d[k] = m ? d[k] : 0.f;
      kr[k] = m ? kr[k] : 0.f;
      adv[k] = m ? adv[k] : 0.f;
    }
  }
  __device__ __forceinline__ float log_ratios() const {   // their sum
    float s = 0.f;
    if (live) {
#pragma unroll
      for (int k = 0; k < kE; ++k) s += d[k];
    }
    return s;
  }
  // Gradients of the chunk's tokens, and what they add to the sums. w: weight of a token;
  // A_row, r_row: the row's advantage and ratio where they are one a row.
  template <bool BLOCK>
  __device__ __forceinline__ void finish(const PolicyArgs& a, const Span<MODE>& c, float w,
                                         float A_row, float r_row, PolicySums<BLOCK>& t) {
    float g[kE];
#pragma unroll
    for (int k = 0; k < kE; ++k) g[k] = 0.f;
    if (live) {
      const uint32_t n = __popc(bits);
      t.tok += n;
      if (a.token_adv) {
        float pg = 0.f, rat = 0.f;
#pragma unroll
        for (int k = 0; k < kE; ++k) {
          const Side sd(a, adv[k]);         // magnitude 0 where the token does not count
          const float r = expf(d[k]), x = sd.s * r;
          const bool clipped = x > sd.bound;
          pg = fmaf(sd.mag, clipped ? sd.bound : x, pg);
          t.low += clipped && sd.s < 0.f ? 1u : 0u;
          t.high += clipped && sd.s > 0.f ? 1u : 0u;
          g[k] = clipped ? 0.f : -(sd.mag * w) * x;
          rat += (bits >> k) & 1u ? r : 0.f;
        }
        t.add(kPg, -w * pg);
        t.add(kRat, rat);
      } else {
        const Side sd(a, A_row);
        const float mw = sd.mag * w;
        uint32_t clips = 0;
        float pg, rat;
        if (a.sequence) {
          const float x = sd.s * r_row;
          const bool clipped = x > sd.bound;
          pg = (float)n * (clipped ? sd.bound : x);
          rat = (float)n * x;
          clips = clipped ? n : 0u;
          const float gx = clipped ? 0.f : -mw * x;
#pragma unroll
          for (int k = 0; k < kE; ++k) g[k] = gx;
        } else {
          Two sp(0.f, 0.f), sr(0.f, 0.f);
#pragma unroll
          for (int k = 0; k < kE; k += 2) {
            const Two x2 = mul2(Two(sd.s, sd.s), Two(expf(d[k]), expf(d[k + 1])));
            float x[2];
            x2.get(x[0], x[1]);
            const bool c0 = x[0] > sd.bound, c1 = x[1] > sd.bound;
            clips += c0 ? 1u : 0u;
            clips += c1 ? 1u : 0u;
            x[0] = (bits >> k) & 1u ? x[0] : 0.f;
            x[1] = (bits >> (k + 1)) & 1u ? x[1] : 0.f;
            sr = add2(sr, Two(x[0], x[1]));
            sp = add2(sp, Two(c0 ? sd.bound : x[0], c1 ? sd.bound : x[1]));
            mul2(Two(-mw, -mw), Two(c0 ? 0.f : x[0], c1 ? 0.f : x[1])).get(g[k], g[k + 1]);
          }
          float odd;
          sp.get(pg, odd);
          pg += odd;
          sr.get(rat, odd);
          rat += odd;
        }
        // (a lane without tokens adds nothing, whatever its row's values are)
        if (n > 0) {
          t.add(kPg, -mw * pg);
          t.add(kRat, sd.s * rat);
        }
        t.low += sd.s < 0.f ? clips : 0u;
        t.high += sd.s < 0.f ? 0u : clips;
      }
      if (a.ref.p) {
        float kl = 0.f, far = 0.f;
#pragma unroll
        for (int k = 0; k < kE; ++k) far = fmaxf(far, fabsf(kr[k]));
        if (far <= 1.f) {
          Two sum(0.f, 0.f);
#pragma unroll
          for (int k = 0; k < kE; k += 2) {
            const Two x(kr[k], kr[k + 1]), q = exp_rest2(x);
            sum = add2(sum, q);
            add2(x, q).get(kr[k], kr[k + 1]);   // e^k - 1
          }
          float odd;
          sum.get(kl, odd);
          kl += odd;
        } else {
#pragma unroll
          for (int k = 0; k < kE; ++k) {
            const float x = kr[k], e1 = expf(x) - 1.f;
            const bool near = fabsf(x) <= 1.f;
            const float q = near ? exp_rest(x) : e1 - x;
            kl += q;
            kr[k] = near ? x + q : e1;
          }
        }
        t.add(kKl, w * kl);
        if (a.beta != 0.f) {
          const float bw = -a.beta * w;
#pragma unroll
          for (int k = 0; k < kE; k += 2)
            fma2(Two(bw, bw), Two(kr[k], kr[k + 1]), Two(g[k], g[k + 1])).get(g[k], g[k + 1]);
        }
      }
      if (!full) {
#pragma unroll
        for (int k = 0; k < kE; ++k) g[k] = (bits >> k) & 1u ? g[k] : 0.f;
      }
    }
    if (a.d.p) store_floats<MODE>(a.d, c, g);
  }

 private:
  float lp[kE];                   // (until ratios())
};

template <int MODE, int TEAM>
__global__ void __launch_bounds__(most_threads(TEAM), blocks_per_sm(MODE, TEAM))
    k_policy(const __grid_constant__ PolicyArgs a) {
  pdl_begin();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  float w = a.scale;
  if (a.norm == BGPO_NORM_TOKENS) {
    unsigned long long c = 0;
    if (a.mask.p) {
      __shared__ unsigned long long s_c[kMaxThreads / 32];
      for (int i = threadIdx.x; i < a.count_blocks; i += blockDim.x) c += a.w.totals[i];
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) c += __shfl_xor_sync(0xffffffffu, c, o);
      if (lane == 0) s_c[warp] = c;
      __syncthreads();
      c = 0;
      for (int i = 0; i < (int)(blockDim.x >> 5); ++i) c += s_c[i];
    } else {
      c = (unsigned long long)a.N * (unsigned long long)a.T;
    }
    w = a.scale / (float)(c > 0 ? c : 1);
  } else if (a.norm == BGPO_NORM_ROWS) {
    w = a.scale / ((float)a.N * (float)a.T);   // without a mask
  }
  constexpr bool BLOCK = TEAM >= kBlock, sums_rows = TEAM != kNone;
  extern __shared__ Sum2 s_sums[];   // (blocks: 3 a thread)
  PolicySums<BLOCK> t(s_sums);
  PolicyChunk<MODE> x;
  __shared__ typename TeamSums<1>::Shared s_team;
  const uint32_t cl = TEAM >= kCluster ? a.cluster : 1;
  const uint32_t rank = TEAM >= kCluster ? cluster_ctarank() : 0;
  const int threads = BLOCK ? blockDim.x : 32, tid = BLOCK ? threadIdx.x : lane;
  const uint32_t chunk0 = rank * (uint32_t)threads * kE;
  TeamSums<1> sums(&s_team, cl);
  const uint32_t per_row = sums_rows ? 1 : a.chunks;
  const uint32_t units = (uint32_t)a.N * per_row;
  uint32_t u = BLOCK ? blockIdx.x / cl : blockIdx.x * kWarpTeams + warp;
  const uint32_t step = BLOCK ? gridDim.x / cl : gridDim.x * kWarpTeams;
  if (TEAM != kMany) {
    // the next unit's mask and advantage are on their way while this one is worked on, and a
    // row's count is known before its floats are there (72 -> 50 us at 4096 x 4096 when these
    // came; asking L2 for the next unit's floats as well, or staging them in shared memory,
    // made it slower)
    Mask<MODE> q;
    Span<MODE> c;
    float A_row = 0.f;
    // row and chunk of the unit to begin, and what a step adds to them
    uint32_t row = sums_rows ? u : u / per_row, part = sums_rows ? 0u : u - row * per_row;
    const uint32_t rows = sums_rows ? step : step / per_row;
    const uint32_t parts = sums_rows ? 0u : step - rows * per_row;
    const auto begin = [&]() {
      c = Span<MODE>(row, chunk0 + part * kChunk, threads, tid, a.T, a.lp.row, a.phase);
      q.load(a.mask, c);
      if (!a.token_adv) A_row = a.adv.p[row * a.adv.row];
      row += rows;
      part += parts;
      if (part >= per_row) {
        part -= per_row;
        ++row;
      }
    };
    if (u < units) begin();
    for (; u < units; u += step) {
      x.load(a, c, q.bits());
      const Span<MODE> this_c = c;
      const float A = A_row;
      if (u + step < units) begin();
      float wr = w, r_row = 0.f;
      if (sums_rows) {
        int32_t n[1] = {__popc(x.bits)};
        float s[1] = {0.f};
        if (a.sequence) {
          x.ratios(a);
          s[0] = x.log_ratios();
        }
        sums.template sum<TEAM>(n, s, a.sequence);
        const float nf = (float)max(n[0], 1);
        if (a.norm == BGPO_NORM_ROWS) wr = a.scale / ((float)a.N * nf);
        if (a.sequence) r_row = expf(s[0] / nf);
      }
      if (!a.sequence) x.ratios(a);
      x.finish(a, this_c, wr, A, r_row, t);
    }
  } else {
    const uint32_t stride = cl * (uint32_t)threads * kE;
    for (; u < units; u += step) {
      const float A_row = a.token_adv ? 0.f : a.adv.p[u * a.adv.row];
      int32_t n[1] = {0};
      Sum2 row = {};
      uint32_t c0 = chunk0;
      do {
        const Span<MODE> c(u, c0, threads, tid, a.T, a.lp.row, a.phase);
        x.load(a, c, load_mask<MODE>(a.mask, c));
        x.ratios(a);
        n[0] += __popc(x.bits);
        if (a.sequence) row.add(x.log_ratios());
        c0 += stride;
      } while (c0 < (uint32_t)a.T + 7);
      float s[1] = {row.value()};
      sums.template sum<TEAM>(n, s, a.sequence);
      const float nf = (float)max(n[0], 1);
      const float wr = a.norm == BGPO_NORM_ROWS ? a.scale / ((float)a.N * nf) : w;
      const float r_row = a.sequence ? expf(s[0] / nf) : 0.f;
      c0 = chunk0;
      do {
        const Span<MODE> c(u, c0, threads, tid, a.T, a.lp.row, a.phase);
        x.load(a, c, load_mask<MODE>(a.mask, c));
        x.ratios(a);
        x.finish(a, c, wr, A_row, r_row, t);
        c0 += stride;
      } while (c0 < (uint32_t)a.T + 7);
    }
  }
  if (TEAM >= kCluster) {   // until no block reads this one's shared memory
    __syncwarp();
    cluster_sync();
  }
  LossTotals all = {{t.value(kPg), t.value(kKl), t.value(kRat), 0.f}, {t.low, t.high, t.tok}};
  if (!grid_totals(a.w, all)) return;
  const float n = (float)max(all.c[2], 1ull);
  const float loss = a.beta != 0.f ? all.f[0] + a.beta * all.f[1] : all.f[0];
  a.out[0] = loss;
  a.out[1] = all.f[0];
  a.out[2] = all.f[1];
  a.out[3] = (float)all.c[0] / n;
  a.out[4] = (float)all.c[1] / n;
  a.out[5] = all.f[2] / n;
  if (!isfinite(loss)) set_device_error(a.w.err, kStatusNonfinite, KID_POLICY_LOSS * 16);
}

// ---- preference loss on paired log ratios ----------------------------------------------------

struct Pair {
  float h, dh, loss;   // margin, loss'(h), loss(h)
};

__device__ __forceinline__ Pair pair_of(const PrefArgs& a, float sc, float sr) {
  Pair p;
  p.h = a.beta * (sc - sr) - a.margin;
  if (a.kind == BGPO_PREF_SIGMOID) {
    // -log s(h) = max(-h, 0) + log(1 + e^-|h|), s(h) = 1 / (1 + e^-h)
    const float l = log1pf(expf(-fabsf(p.h)));   // NaN for a NaN
    p.loss = a.eps < 1.f ? (1.f - a.eps) * (fmaxf(-p.h, 0.f) + l) : 0.f;
    if (a.eps > 0.f) p.loss += a.eps * (fmaxf(p.h, 0.f) + l);
    p.dh = a.eps / (1.f + expf(-p.h)) - (1.f - a.eps) / (1.f + expf(p.h));
  } else if (a.kind == BGPO_PREF_HINGE) {
    p.loss = p.h >= 1.f ? 0.f : 1.f - p.h;
    p.dh = p.h >= 1.f ? 0.f : p.h < 1.f ? -1.f : p.h;   // NaN for a NaN
  } else {
    const float x = (p.h - 0.5f) / a.beta;
    p.loss = x * x;
    p.dh = 2.f * x / a.beta;
  }
  return p;
}

template <int MODE, int TEAM>   // kWarp to kMany
__global__ void __launch_bounds__(most_threads(TEAM), blocks_per_sm(MODE, TEAM))
    k_preference(const __grid_constant__ PrefArgs a) {
  pdl_begin();
  constexpr bool BLOCK = TEAM >= kBlock, ONCE = TEAM != kMany;
  __shared__ typename TeamSums<2>::Shared s_team;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const uint32_t cl = TEAM >= kCluster ? a.cluster : 1;
  const uint32_t rank = TEAM >= kCluster ? cluster_ctarank() : 0;
  const int threads = BLOCK ? blockDim.x : 32, tid = BLOCK ? threadIdx.x : lane;
  const uint32_t team = BLOCK ? blockIdx.x / cl : blockIdx.x * kWarpTeams + warp;
  const uint32_t teams = BLOCK ? gridDim.x / cl : gridDim.x * kWarpTeams;
  const uint32_t chunk0 = rank * (uint32_t)threads * kE, stride = cl * (uint32_t)threads * kE;
  const float unit = a.beta * (a.scale / (float)a.K);
  TeamSums<2> sums(&s_team, cl);
  // over the team's pairs, as PolicySums; the team's first thread's
  __shared__ Sum2 s_pairs[BLOCK ? 1 : kWarpTeams][4];
  Sum2* const f = s_pairs[BLOCK ? 0 : warp];
  if (tid == 0) {
#pragma unroll
    for (int i = 0; i < 4; ++i) f[i] = {};
  }
  uint32_t right = 0;
  const auto span_of = [&](uint32_t k, int i, uint32_t c0) {
    const PrefSide& sd = a.side[i];
    return Span<MODE>(k, c0, threads, tid, sd.T, sd.lp.row, sd.phase);
  };
  // the next pair's masks are on their way while this one is worked on
  Mask<MODE> q[2];
#pragma unroll
  for (int i = 0; i < 2; ++i)
    if (ONCE && team < (uint32_t)a.K)
      q[i].load(a.side[i].mask, span_of(team, i, chunk0));
  for (uint32_t k = team; k < (uint32_t)a.K; k += teams) {
    uint32_t bits[2];
    int32_t n[2] = {0, 0};
    float s[2] = {0.f, 0.f};
    if (ONCE) {
      float x[2][kE], y[2][kE];
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const PrefSide& sd = a.side[i];
        const Span<MODE> c = span_of(k, i, chunk0);
        bits[i] = q[i].bits();
        n[i] = __popc(bits[i]);
        load_floats<MODE>(sd.lp, c, bits[i], x[i]);
        if (sd.ref.p) load_floats<MODE>(sd.ref, c, bits[i], y[i]);
      }
#pragma unroll
      for (int i = 0; i < 2; ++i)
        if (k + teams < (uint32_t)a.K)
          q[i].load(a.side[i].mask, span_of(k + teams, i, chunk0));
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        if (a.side[i].ref.p) {
#pragma unroll
          for (int j = 0; j < kE; ++j) x[i][j] -= y[i][j];
        }
#pragma unroll
        for (int j = 0; j < kE; ++j)   // (an eight brings the neighbours of its tokens too)
          s[i] += (bits[i] >> j) & 1u ? x[i][j] : 0.f;
      }
    } else {
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const PrefSide& sd = a.side[i];
        uint32_t c0 = chunk0;
        Sum2 row = {};
        do {
          const Span<MODE> c = span_of(k, i, c0);
          bits[i] = load_mask<MODE>(sd.mask, c);
          n[i] += __popc(bits[i]);
          float x[kE], y[kE];
          load_floats<MODE>(sd.lp, c, bits[i], x);
          if (sd.ref.p) {
            load_floats<MODE>(sd.ref, c, bits[i], y);
#pragma unroll
            for (int j = 0; j < kE; ++j) x[j] -= y[j];
          }
          float part = 0.f;
#pragma unroll
          for (int j = 0; j < kE; ++j) part += (bits[i] >> j) & 1u ? x[j] : 0.f;
          row.add(part);
          c0 += stride;
        } while (c0 < (uint32_t)sd.T + 7);
        s[i] = row.value();
      }
    }
    sums.template sum<TEAM>(n, s, true);
    const float div[2] = {a.average ? (float)max(n[0], 1) : 1.f,
                          a.average ? (float)max(n[1], 1) : 1.f};
    const float sc = s[0] / div[0], sr = s[1] / div[1];
    const Pair p = pair_of(a, sc, sr);
    if (tid == 0 && rank == 0) {
      if (a.margins) a.margins[k] = p.h;
      f[0].add(p.loss);
      f[1].add(p.h);
      f[2].add(sc);
      f[3].add(sr);
      right += p.h > 0.f ? 1 : 0;
    }
    if (!a.side[0].d.p) continue;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const PrefSide& sd = a.side[i];
      const float g = (i ? -p.dh : p.dh) * unit / div[i];
      uint32_t c0 = chunk0;
      do {
        const Span<MODE> c = span_of(k, i, c0);
        if (!ONCE) bits[i] = load_mask<MODE>(sd.mask, c);
        float v[kE];
#pragma unroll
        for (int j = 0; j < kE; ++j) v[j] = (bits[i] >> j) & 1u ? g : 0.f;
        store_floats<MODE>(sd.d, c, v);
        c0 += stride;
      } while (!ONCE && c0 < (uint32_t)sd.T + 7);
    }
  }
  if (TEAM >= kCluster) {   // until no block reads this one's shared memory
    __syncwarp();
    cluster_sync();
  }
  LossTotals t = {};
  if (tid == 0) t = {{f[0].value(), f[1].value(), f[2].value(), f[3].value()}, {right, 0, 0}};
  if (!grid_totals(a.w, t)) return;
  const float K = (float)a.K;
  const float loss = a.scale * (t.f[0] / K);
  a.out[0] = loss;
  a.out[1] = (float)t.c[0] / K;
  a.out[2] = t.f[1] / K;
  a.out[3] = a.beta * (t.f[2] / K);
  a.out[4] = a.beta * (t.f[3] / K);
  if (!isfinite(loss)) set_device_error(a.w.err, kStatusNonfinite, KID_PREFERENCE_LOSS * 16);
}

// ---- launches ----------------------------------------------------------------------------

// The team of rows of T tokens: threads (32: a warp) and blocks of the cluster.
struct Team {
  TeamKind kind;
  int threads, cluster;
};

Team team_of(int64_t T) {
  if (T <= kChunk) return {kWarp, 32, 1};
  int cluster = 1;
  while (cluster < kMaxCluster && (int64_t)cluster * kMaxThreads * kE < T) cluster *= 2;
  const int64_t threads = round_up(ceil_div(T, cluster * kE), 32);
  if (threads > kMaxThreads) return {kMany, kMaxThreads, cluster};
  return {cluster > 1 ? kCluster : kBlock, (int)threads, cluster};
}

// Threads that an SM holds.
int resident(Mode m, TeamKind t) { return blocks_per_sm(m, t) * most_threads(t); }

// Blocks of a launch: as many as there is work for, at most what the device holds at once
// with `resident` threads an SM: later units then find their masks loaded. (Twice as many
// blocks, when tried: 17 us instead of 14 at 1024 pairs x 2,047.)
unsigned loss_blocks(int64_t blocks, int threads, int cluster, int resident, int num_sms) {
  int64_t most = (int64_t)num_sms * (resident / threads);
  if (most > kTrainMaxBlocks) most = kTrainMaxBlocks;
  most -= most % cluster;
  return (unsigned)(blocks < 1 ? 1 : blocks < most ? blocks : most);
}

template <class Args>
cudaError_t launch_team(void (*kernel)(Args), unsigned grid, unsigned threads, int cluster,
                        size_t shared, cudaStream_t s, const Args& a) {
  cudaLaunchAttribute attr[2] = {};
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = (unsigned)cluster;
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(grid, 1, 1);
  cfg.blockDim = dim3(threads, 1, 1);
  cfg.dynamicSmemBytes = shared;
  cfg.stream = s;
  cfg.attrs = attr;
  cfg.numAttrs = cluster > 1 ? 2 : 1;
  cudaLaunchKernelEx(&cfg, kernel, a);
  return cudaGetLastError();
}

// Elements by which an array starts past a boundary of eight.
template <class T>
int phase_of(const View<T>& v) {
  return (int)(reinterpret_cast<uintptr_t>(v.p) / sizeof(T) % 8);
}

// Whether an array moves in eights together with `like`: columns side by side, the same row
// stride and the same start past a boundary (an absent array does).
template <class T>
bool in_eights(const View<T>& v, const View<const float>& like, int64_t rows) {
  return !v.p || (v.col == 1 && (rows == 1 || v.row == like.row) && phase_of(v) == phase_of(like));
}

Mode mode_of(bool eights, int phase, int64_t row_stride, int64_t rows, int64_t T) {
  if (!eights) return kSingle;
  return phase == 0 && T % 8 == 0 && (rows == 1 || row_stride % 8 == 0) ? kEights : kShifted;
}

}  // namespace

// Columns that a team has to cover for rows of T tokens: they may start up to 7 past a
// boundary.
static int64_t covered(Mode m, int64_t T) { return m == kShifted ? T + 7 : T; }

// The kernel of a mode and a kind of team.
template <int MODE>
static auto policy_kernel(TeamKind t) {
  return t == kNone ? k_policy<MODE, kNone>
       : t == kWarp ? k_policy<MODE, kWarp>
       : t == kBlock ? k_policy<MODE, kBlock>
       : t == kCluster ? k_policy<MODE, kCluster> : k_policy<MODE, kMany>;
}
template <int MODE>
static auto preference_kernel(TeamKind t) {
  return t == kWarp ? k_preference<MODE, kWarp>
       : t == kBlock ? k_preference<MODE, kBlock>
       : t == kCluster ? k_preference<MODE, kCluster> : k_preference<MODE, kMany>;
}

cudaError_t launch_count_tokens(int32_t N, int32_t T, const View<const uint8_t>& mask,
                                const TrainWs& w, int num_sms, int* blocks, cudaStream_t s) {
  const int phase = phase_of(mask);
  const Mode m = mode_of(mask.col == 1, phase, mask.row, N, T);
  const uint32_t per_row = (uint32_t)ceil_div(covered(m, T), kChunk);
  *blocks = (int)loss_blocks(ceil_div((int64_t)N * per_row, kWarpTeams), 32 * kWarpTeams, 1,
                             2048, num_sms);
  return launch_dependent(m == kEights    ? k_count_tokens<kEights>
                          : m == kShifted ? k_count_tokens<kShifted>
                                          : k_count_tokens<kSingle>,
                          (unsigned)*blocks, 32 * kWarpTeams, 0, s, N, T, per_row, phase, mask, w);
}

cudaError_t launch_policy_loss(const PolicyArgs& args, int num_sms, cudaStream_t s) {
  PolicyArgs a = args;
  const bool eights = in_eights(a.lp, a.lp, a.N) && in_eights(a.old, a.lp, a.N) &&
                      in_eights(a.ref, a.lp, a.N) && in_eights(a.mask, a.lp, a.N) &&
                      in_eights(a.d, a.lp, a.N) &&
                      (!a.token_adv || in_eights(a.adv, a.lp, a.N));
  a.phase = phase_of(a.lp);
  const Mode m = mode_of(eights, a.phase, a.lp.row, a.N, a.T);
  const int64_t cols = covered(m, a.T);
  const Team t = a.row_sums ? team_of(cols) : Team{kNone, 32, 1};
  a.cluster = (uint32_t)t.cluster;
  a.chunks = (uint32_t)ceil_div(cols, kChunk);
  const bool block = t.kind >= kBlock;
  const int threads = block ? t.threads : 32 * kWarpTeams;
  const int64_t warps = a.row_sums ? a.N : (int64_t)a.N * a.chunks;
  const unsigned grid = loss_blocks(block ? (int64_t)a.N * t.cluster : ceil_div(warps, kWarpTeams),
                                    threads, t.cluster, resident(m, t.kind), num_sms);
  return launch_team(m == kEights    ? policy_kernel<kEights>(t.kind)
                     : m == kShifted ? policy_kernel<kShifted>(t.kind)
                                     : policy_kernel<kSingle>(t.kind),
                     grid, (unsigned)threads, t.cluster, block ? 3 * sizeof(Sum2) * threads : 0, s,
                     a);
}

cudaError_t launch_preference_loss(const PrefArgs& args, int num_sms, cudaStream_t s) {
  PrefArgs a = args;
  Mode m = kEights;       // of the side that asks for more
  for (PrefSide& sd : a.side) {
    const bool eights = in_eights(sd.lp, sd.lp, a.K) && in_eights(sd.ref, sd.lp, a.K) &&
                        in_eights(sd.mask, sd.lp, a.K) && in_eights(sd.d, sd.lp, a.K);
    sd.phase = phase_of(sd.lp);
    const Mode mine = mode_of(eights, sd.phase, sd.lp.row, a.K, sd.T);
    if (m != kSingle && mine != kEights) m = mine;
  }
  const int64_t cols = covered(m, a.side[0].T > a.side[1].T ? a.side[0].T : a.side[1].T);
  const Team t = team_of(cols);
  a.cluster = (uint32_t)t.cluster;
  const bool block = t.kind >= kBlock;
  const int threads = block ? t.threads : 32 * kWarpTeams;
  const unsigned grid = loss_blocks(block ? (int64_t)a.K * t.cluster : ceil_div(a.K, kWarpTeams),
                                    threads, t.cluster, resident(m, t.kind), num_sms);
  return launch_team(m == kEights    ? preference_kernel<kEights>(t.kind)
                     : m == kShifted ? preference_kernel<kShifted>(t.kind)
                                     : preference_kernel<kSingle>(t.kind),
                     grid, (unsigned)threads, t.cluster, 0, s, a);
}

}  // namespace bgpo
