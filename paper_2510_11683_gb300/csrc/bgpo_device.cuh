// Device helpers for sm_103a: mbarriers with bounded waits, TMA tensor loads,
// tcgen05 (TMEM allocation, MMA, commit, loads), shared-memory matrix
// descriptors and the device error word.
#pragma once

#include <cuda.h>           // CUtensorMap (type only; no driver symbol is linked)
#include <cuda_runtime.h>
#include <cuda_bf16.h>
#include <stdint.h>

#include "bgpo_plan.h"

namespace bgpo {

// A bounded wait gives up after this many nanoseconds of %globaltimer. The
// longest legitimate wait in these kernels is one tile's main loop (well under
// 10 ms at the largest supported sizes).
constexpr uint64_t kWaitTimeoutNs = 2000000000ull;
// ... or after this many polls, whichever comes first.
constexpr uint32_t kWaitMaxPolls = 1u << 30;

// Records the first device-side failure of a workspace: status and where.
__device__ __forceinline__ void set_device_error(int32_t* err, int32_t status, int32_t where) {
  if (atomicCAS(&err[ERR_STATUS], 0, status) == 0) atomicExch(&err[ERR_WHERE], where);
}

// Bounds checks of the checked build (compiled with -DBGPO_CHECKED): a check
// that fails records BGPO_ERR_BOUNDS (9) and `where` in the workspace error word
// and evaluates to false, so that the caller skips the guarded access. The
// normal build does not evaluate the condition.
#ifdef BGPO_CHECKED
#define BGPO_IN_BOUNDS(err, cond, where) \
  ((cond) ? true : (::bgpo::set_device_error((err), 9, (where)), false))
#else
#define BGPO_IN_BOUNDS(err, cond, where) true
#endif

__device__ __forceinline__ uint32_t smem_addr(const void* p) {
  return static_cast<uint32_t>(__cvta_generic_to_shared(p));
}

__device__ __forceinline__ uint64_t globaltimer_ns() {
  uint64_t t;
  asm volatile("mov.u64 %0, %%globaltimer;" : "=l"(t));
  return t;
}

// ---- mbarrier -----------------------------------------------------------------

__device__ __forceinline__ void mbar_init(uint32_t bar, uint32_t count) {
  asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count) : "memory");
}

__device__ __forceinline__ void fence_barrier_init() {
  asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
}

__device__ __forceinline__ void mbar_arrive(uint32_t bar) {
  asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory");
}

__device__ __forceinline__ void mbar_arrive_expect_tx(uint32_t bar, uint32_t bytes) {
  asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes)
               : "memory");
}

// One try_wait: the hardware suspends the thread until the phase completes or, at
// most, for about kWaitHintNs. Without a hint a wait is a loop of short tries, and
// the GEMMs' waiting warps (each epilogue warp for a tile's main loop) spent issue
// slots and, at the power cap, clock on it: 7B head 45.51 -> 44.88 ms a sample,
// forwards of 1,124 and 983 rows on the 4096 x 126464 head 1445 -> 1414 us, a
// sample on a 2048 x 32000 one 261.5 -> 258.6 us; a hint of 1 us within 0.3%.
constexpr uint32_t kWaitHintNs = 20000;

__device__ __forceinline__ bool mbar_try_wait(uint32_t bar, uint32_t parity) {
  uint32_t done;
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2, %3;\n\t"
      "selp.u32 %0, 1, 0, p;\n\t}"
      : "=r"(done)
      : "r"(bar), "r"(parity), "r"(kWaitHintNs)
      : "memory");
  return done != 0;
}

// Waits until the phase with parity `parity` of barrier `bar` has completed.
// Returns false (without waiting further) when *abort becomes non-zero or the
// wait runs out of time (timeout_ns) or polls.
__device__ __forceinline__ bool mbar_wait_timeout(uint32_t bar, uint32_t parity,
                                                  volatile int* abort, uint64_t timeout_ns) {
  if (mbar_try_wait(bar, parity)) return true;
  const uint64_t t0 = globaltimer_ns();
  for (uint32_t poll = 1; poll < kWaitMaxPolls; ++poll) {
    if (mbar_try_wait(bar, parity)) return true;
    if (*abort) return false;
    if ((poll & 7u) == 0 && globaltimer_ns() - t0 > timeout_ns) return false;
  }
  return false;
}

__device__ __forceinline__ bool mbar_wait(uint32_t bar, uint32_t parity, volatile int* abort) {
  return mbar_wait_timeout(bar, parity, abort, kWaitTimeoutNs);
}

// 2^x by the special-function unit's approximation (PTX ex2.approx.ftz.f32:
// relative error within 2^-22, subnormal inputs and results flushed to zero).
// The arguments here are logits minus their row's log-sum-exp or running
// maximum, so a flushed result is below 2^-126 of the row's largest term.
__device__ __forceinline__ float ex2_ftz(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// ---- TMA -----------------------------------------------------------------------

__device__ __forceinline__ void tma_prefetch_map(const CUtensorMap* map) {
  asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(map)) : "memory");
}

// ---- TMA tensor stores / reductions (shared -> global, bulk-group completion) ----

// Makes this thread's generic-proxy shared-memory writes visible to the async
// proxy (TMA) before another thread issues a bulk copy that reads them.
__device__ __forceinline__ void fence_proxy_async_shared() {
  asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
}

__device__ __forceinline__ void tma_store_2d(const CUtensorMap* map, uint32_t src, int32_t c0,
                                             int32_t c1) {
  asm volatile(
      "cp.async.bulk.tensor.2d.global.shared::cta.bulk_group [%0, {%2, %3}], [%1];" ::"l"(
          reinterpret_cast<uint64_t>(map)),
      "r"(src), "r"(c0), "r"(c1)
      : "memory");
}

// global[tile] += shared[tile], element type from the tensor map (f32 here).
__device__ __forceinline__ void tma_reduce_add_2d(const CUtensorMap* map, uint32_t src, int32_t c0,
                                                  int32_t c1) {
  asm volatile(
      "cp.reduce.async.bulk.tensor.2d.global.shared::cta.add.bulk_group [%0, {%2, %3}], [%1];" ::"l"(
          reinterpret_cast<uint64_t>(map)),
      "r"(src), "r"(c0), "r"(c1)
      : "memory");
}

// Asks L2 to fetch `bytes` (a multiple of 16) from a 16-byte aligned global address.
__device__ __forceinline__ void bulk_prefetch_l2(const void* src, uint32_t bytes) {
  asm volatile("cp.async.bulk.prefetch.L2.global [%0], %1;" ::"l"(src), "r"(bytes) : "memory");
}

__device__ __forceinline__ void bulk_commit_group() {
  asm volatile("cp.async.bulk.commit_group;" ::: "memory");
}

// Waits until at most N committed bulk groups still read their shared source.
template <int N>
__device__ __forceinline__ void bulk_wait_group_read() {
  asm volatile("cp.async.bulk.wait_group.read %0;" ::"n"(N) : "memory");
}

// Waits until at most N committed bulk groups are still in flight at all.
template <int N>
__device__ __forceinline__ void bulk_wait_group() {
  asm volatile("cp.async.bulk.wait_group %0;" ::"n"(N) : "memory");
}

// ---- tcgen05 ----------------------------------------------------------------------

__device__ __forceinline__ void tc_fence_before() {
  asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
}

__device__ __forceinline__ void tc_fence_after() {
  asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
}

// 32 lanes x 32 consecutive 32-bit columns: thread t of the warp gets lane
// (taddr.lane + t), columns taddr.col .. taddr.col + 31.
__device__ __forceinline__ void tmem_ld_32x32b_x32(uint32_t taddr, uint32_t (&v)[32]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
      "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
      "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
      : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]),
        "=r"(v[7]), "=r"(v[8]), "=r"(v[9]), "=r"(v[10]), "=r"(v[11]), "=r"(v[12]), "=r"(v[13]),
        "=r"(v[14]), "=r"(v[15]), "=r"(v[16]), "=r"(v[17]), "=r"(v[18]), "=r"(v[19]),
        "=r"(v[20]), "=r"(v[21]), "=r"(v[22]), "=r"(v[23]), "=r"(v[24]), "=r"(v[25]),
        "=r"(v[26]), "=r"(v[27]), "=r"(v[28]), "=r"(v[29]), "=r"(v[30]), "=r"(v[31])
      : "r"(taddr));
}

__device__ __forceinline__ void tmem_ld_wait() {
  asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
}

// The same wait, with `v` (the destination of an earlier tcgen05.ld) as its
// operands, so that the compiler cannot move a use of v above it while other
// work runs between the load and the wait.
__device__ __forceinline__ void tmem_ld_wait_regs(uint32_t (&v)[32]) {
  asm volatile("tcgen05.wait::ld.sync.aligned;"
               : "+r"(v[0]), "+r"(v[1]), "+r"(v[2]), "+r"(v[3]), "+r"(v[4]), "+r"(v[5]),
                 "+r"(v[6]), "+r"(v[7]), "+r"(v[8]), "+r"(v[9]), "+r"(v[10]), "+r"(v[11]),
                 "+r"(v[12]), "+r"(v[13]), "+r"(v[14]), "+r"(v[15]), "+r"(v[16]), "+r"(v[17]),
                 "+r"(v[18]), "+r"(v[19]), "+r"(v[20]), "+r"(v[21]), "+r"(v[22]), "+r"(v[23]),
                 "+r"(v[24]), "+r"(v[25]), "+r"(v[26]), "+r"(v[27]), "+r"(v[28]), "+r"(v[29]),
                 "+r"(v[30]), "+r"(v[31])
               :
               : "memory");
}

// Shared-memory matrix descriptor for a tile stored with the 128-byte swizzle
// (rows of 128 bytes, 8-row / 1024-byte swizzle atoms, 1024-byte aligned base).
//   bits  0-13 start address >> 4
//   bits 16-29 leading-dimension byte offset >> 4
//   bits 32-45 stride-dimension byte offset >> 4
//   bits 46-48 fixed 0b001
//   bits 49-51 base offset (0: atoms start on 1024-byte boundaries)
//   bits 61-63 layout: 2 = 128-byte swizzle
// K-major operand: rows are M/N, 64 K-elements per row; SBO = 1024 (next 8 rows),
//   LBO unused (1); the K step of one MMA adds 32 bytes to the start address.
// MN-major operand: rows are K, 64 M/N-elements per row; LBO = byte distance
//   between 64-element M/N chunks, SBO = 1024 (next 8 K rows); the K step of one
//   MMA adds 16 rows = 2048 bytes.
__device__ __forceinline__ uint64_t smem_desc_sw128(uint32_t saddr, uint32_t lbo, uint32_t sbo) {
  uint64_t d = 0;
  d |= (uint64_t)((saddr & 0x3FFFFu) >> 4);
  d |= (uint64_t)((lbo >> 4) & 0x3FFFu) << 16;
  d |= (uint64_t)((sbo >> 4) & 0x3FFFu) << 32;
  d |= (uint64_t)1 << 46;
  d |= (uint64_t)2 << 61;
  return d;
}

// Instruction descriptor of tcgen05.mma kind::f16 with bf16 A/B and fp32 D.
//   bits 4-5 D type (1 = f32), 7-9 A type (1 = bf16), 10-12 B type (1 = bf16),
//   bit 15 A major (0 = K, 1 = MN), bit 16 B major, bits 17-22 N >> 3,
//   bits 24-28 M >> 4.
__host__ __device__ constexpr uint32_t idesc_bf16_f32(int m, int n, bool a_mn, bool b_mn) {
  return (1u << 4) | (1u << 7) | (1u << 10) | ((a_mn ? 1u : 0u) << 15) |
         ((b_mn ? 1u : 0u) << 16) | ((uint32_t)(n >> 3) << 17) | ((uint32_t)(m >> 4) << 24);
}

// ---- CTA pairs (2-CTA clusters) ------------------------------------------------------

__device__ __forceinline__ uint32_t cluster_ctarank() {
  uint32_t r;
  asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return r;
}

// Shared::cluster address of the same shared-memory location in CTA `rank`.
__device__ __forceinline__ uint32_t map_to_cta(uint32_t saddr, uint32_t rank) {
  uint32_t out;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(out) : "r"(saddr), "r"(rank));
  return out;
}

// Every thread of both CTAs arrives, then waits for all of them.
__device__ __forceinline__ void cluster_sync() {
  asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" :::
                   "memory");
}

// Arrive on an mbarrier given by a shared::cluster address (possibly the peer's).
__device__ __forceinline__ void mbar_arrive_cluster(uint32_t cbar) {
  asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(cbar)
               : "memory");
}

// TMA load into this CTA's shared memory that signals an mbarrier which may
// live in the peer CTA of the pair (shared::cluster address).
__device__ __forceinline__ void tma_load_2d_pair(uint32_t dst, const CUtensorMap* map,
                                                 uint32_t cbar, int32_t c0, int32_t c1) {
  asm volatile(
      "cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes"
      " [%0], [%1, {%3, %4}], [%2];" ::"r"(dst),
      "l"(reinterpret_cast<uint64_t>(map)), "r"(cbar), "r"(c0), "r"(c1)
      : "memory");
}

// TMEM of a CTA pair: executed by one warp in each of the two CTAs.
__device__ __forceinline__ void tmem_alloc_pair(uint32_t dst_smem, uint32_t ncols) {
  asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(dst_smem),
               "r"(ncols)
               : "memory");
}

__device__ __forceinline__ void tmem_relinquish_pair() {
  asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
}

__device__ __forceinline__ void tmem_dealloc_pair(uint32_t taddr, uint32_t ncols) {
  asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(taddr), "r"(ncols)
               : "memory");
}

// D[tmem of both CTAs] (+)= A[smem of both CTAs] * B[smem of both CTAs]^T, issued
// by the even CTA of the pair; M = 256 rows (128 per CTA), B columns split
// 128 / 128 between the CTAs.
__device__ __forceinline__ void umma_bf16_pair(uint32_t d_tmem, uint64_t a_desc, uint64_t b_desc,
                                               uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d_tmem),
      "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(accumulate)
      : "memory");
}

// Arrives once on the mbarrier at shared offset `bar` in every CTA of `cta_mask`
// when all tcgen05 operations issued so far by this thread have completed.
__device__ __forceinline__ void umma_commit_pair(uint32_t bar, uint16_t cta_mask) {
  asm volatile(
      "tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64"
      " [%0], %1;" ::"r"(bar),
      "h"(cta_mask)
      : "memory");
}

// ---- dependent launches --------------------------------------------------------------

// Every kernel of the path is launched with programmatic stream serialization
// (launch_dependent): its blocks may start while the kernel before it in the
// stream still runs. pdl_wait() returns once that kernel has completed and its
// writes are visible; nothing before it touches global memory other than the
// kernel's own parameters. Each kernel waits in every block, so a kernel that
// has completed implies that all kernels before it have.
__device__ __forceinline__ void pdl_launch_dependents() {
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
}

__device__ __forceinline__ void pdl_wait() { asm volatile("griddepcontrol.wait;" ::: "memory"); }

// The head of a kernel without a prologue of its own. `early`: the next kernel may
// start at once; otherwise when this one has ended.
__device__ __forceinline__ void pdl_begin(bool early = true) {
  if (early) pdl_launch_dependents();
  pdl_wait();
}

// dx_plan with one candidate per lane (whole warps call it).
__device__ __forceinline__ DxPlan dx_plan_warp(const Geometry& g, int32_t M, int num_pairs) {
  static_assert(2 * kMaxSplits == 32, "one candidate per lane");
  if (M <= 0) return DxPlan{kDxWide, 1};
  const DxPlan usual = dx_plan_usual(g, M, num_pairs);
  const DxPlan c = dx_candidate((int)(threadIdx.x & 31));
  // costs are positive: their bits order as they do
  const uint32_t cost = dx_allowed(g, M, usual, c)
                            ? __float_as_uint(dx_cost(g, M, num_pairs, c.wide, c.splits))
                            : 0xffffffffu;
  const uint32_t least = __reduce_min_sync(0xffffffffu, cost);
  const int who = __ffs(__ballot_sync(0xffffffffu, cost == least)) - 1;
  return dx_plan_of(g, M, num_pairs, usual, dx_candidate(who), __uint_as_float(least));
}

// ---- misc -----------------------------------------------------------------------

__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}

// A running sum and what its roundings have left out (Knuth's two-sum; single roundings, so
// that no product of the caller's is fused into it).
struct alignas(8) Sum2 {
  float s, c;
  __device__ __forceinline__ void add(float x) {
    const float t = __fadd_rn(s, x), xs = __fsub_rn(t, s);
    c += __fsub_rn(s, __fsub_rn(t, xs)) + __fsub_rn(x, xs);
    s = t;
  }
  __device__ __forceinline__ void add(const Sum2& o) {
    add(o.s);
    c += o.c;
  }
  // Over the lanes of a warp, the same in all of them.
  __device__ __forceinline__ void over_warp() {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
      Sum2 q;
      q.s = __shfl_xor_sync(0xffffffffu, s, o);
      q.c = __shfl_xor_sync(0xffffffffu, c, o);
      add(q);
    }
  }
  // (an infinite or NaN sum has a NaN remainder)
  __device__ __forceinline__ float value() const { return isfinite(s) ? s + c : s; }
};

}  // namespace bgpo
