// Global norm of many gradients, and the gradients scaled to a largest norm
// (include/bgpo_train.h has the formulas).
//
// Both stream every tensor once; HBM bounds them, and for many small tensors the walk
// over the list. The list travels in the kernel's parameters (up to 32 KB of them), so a
// call needs no table in device memory and nothing of it outlives the call; a longer list
// takes several launches. Work is cut into units of 8,192 elements of one tensor, which
// persistent blocks take in turn; a unit's tensor is found by bisection in the list's
// running unit counts. Units start on 32-byte boundaries of the source, so that a tensor at
// any address moves in vectors of eight elements but for its two ends (when the output lies
// as far past a boundary as the source). The clipping takes the units from the last to the
// first: L2 then still holds what the norm read last.
#include <cuda_fp16.h>
#include <math.h>

#include "bgpo_device.cuh"
#include "bgpo_train.h"
#include "train_internal.h"

namespace bgpo {

namespace {

constexpr int kThreads = 256;
constexpr int kWarps = kThreads / 32;
constexpr int32_t kStatusNonfinite = 5;  // BGPO_ERR_NONFINITE

__device__ __forceinline__ void unpack(const uint4& q, float (&v)[8], __nv_bfloat16) {
  const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    v[2 * i] = __uint_as_float(w[i] << 16);
    v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
  }
}
__device__ __forceinline__ void unpack(const uint4& q, float (&v)[8], __half) {
  const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&w[i]));
    v[2 * i] = f.x;
    v[2 * i + 1] = f.y;
  }
}

// Eight elements at an address aligned to their size, in one load.
template <class T>
struct Vec8 {
  uint4 q;
  __device__ __forceinline__ void load(const T* p) { q = __ldcg(reinterpret_cast<const uint4*>(p)); }
  __device__ __forceinline__ void get(float (&v)[8]) const { unpack(q, v, T{}); }
};
// 32 bytes a lane: two loads of 16 that share their 32-byte sectors ask L2 for each twice
template <>
struct Vec8<float> {
  float f[8];
  __device__ __forceinline__ void load(const float* p) {
    asm volatile("ld.global.v8.f32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                 : "=f"(f[0]), "=f"(f[1]), "=f"(f[2]), "=f"(f[3]), "=f"(f[4]), "=f"(f[5]),
                   "=f"(f[6]), "=f"(f[7])
                 : "l"(p)
                 : "memory");
  }
  __device__ __forceinline__ void get(float (&v)[8]) const {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = f[i];
  }
};

__device__ __forceinline__ float to_float(float x) { return x; }
__device__ __forceinline__ float to_float(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ float to_float(__half x) { return __half2float(x); }

__device__ __forceinline__ void put(float* p, float x) { *p = x; }
__device__ __forceinline__ void put(__nv_bfloat16* p, float x) { *p = __float2bfloat16_rn(x); }
__device__ __forceinline__ void put(__half* p, float x) { *p = __float2half_rn(x); }

__device__ __forceinline__ void put8(float* p, const float (&v)[8]) {
  asm volatile("st.global.v8.f32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p), "f"(v[0]),
               "f"(v[1]), "f"(v[2]), "f"(v[3]), "f"(v[4]), "f"(v[5]), "f"(v[6]), "f"(v[7])
               : "memory");
}
__device__ __forceinline__ void put8(__nv_bfloat16* p, const float (&v)[8]) {
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const __nv_bfloat162 h = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
    w[i] = *reinterpret_cast<const uint32_t*>(&h);
  }
  *reinterpret_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
}
__device__ __forceinline__ void put8(__half* p, const float (&v)[8]) {
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const __half2 h = __floats2half2_rn(v[2 * i], v[2 * i + 1]);
    w[i] = *reinterpret_cast<const uint32_t*>(&h);
  }
  *reinterpret_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
}

// The tensor that unit u belongs to.
template <int CAP>
__device__ __forceinline__ int tensor_of(const GradList<CAP>& l, uint32_t u) {
  int lo = 0, hi = l.count;          // begin[lo] <= u < begin[hi]
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (l.t[mid].begin <= u) lo = mid; else hi = mid;
  }
  return lo;
}

// First element of unit u of a tensor (below 0 for the first unit of a shifted one).
__device__ __forceinline__ int64_t unit_begin(const GradTensor& t, uint32_t u) {
  return (int64_t)(u - t.begin) * kGradUnit - t.shift;
}

// Sum of squares of this thread's elements of a unit that starts at element e0.
template <class T>
__device__ __forceinline__ float unit_squares(const GradTensor& t, int64_t e0) {
  const T* p = static_cast<const T*>(t.src);
  const int64_t i0 = e0 + 8 * threadIdx.x;
  if (e0 >= 0 && e0 + kGradUnit <= t.n) {   // block-uniform: a whole unit
    Vec8<T> q[kGradVecs];
#pragma unroll
    for (int k = 0; k < kGradVecs; ++k) q[k].load(p + i0 + k * 8 * kThreads);
    float s[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int k = 0; k < kGradVecs; ++k) {
      float v[8];
      q[k].get(v);
#pragma unroll
      for (int j = 0; j < 8; ++j) s[j] = fmaf(v[j], v[j], s[j]);
    }
    return ((s[0] + s[1]) + (s[2] + s[3])) + ((s[4] + s[5]) + (s[6] + s[7]));
  }
  // the ends of a tensor: neighbouring lanes take neighbouring elements, eight loads in flight
  float acc = 0.f;
  for (int64_t i = e0 + threadIdx.x; i < e0 + kGradUnit && i < t.n; i += 8 * kThreads) {
    float v[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int64_t x = i + j * kThreads;
      v[j] = x >= 0 && x < t.n ? to_float(p[x]) : 0.f;
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) acc = fmaf(v[j], v[j], acc);
  }
  return acc;
}

template <int CAP>
__global__ void __launch_bounds__(kThreads, 4)
    k_grad_norm(const __grid_constant__ GradList<CAP> l, GradNormArgs a) {
  pdl_begin();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  Sum2 mine = {};
  for (uint32_t u = blockIdx.x; u < l.units; u += gridDim.x) {
    const GradTensor& t = l.t[tensor_of(l, u)];
    const int64_t e0 = unit_begin(t, u);
    if (t.type == BGPO_F32) mine.add(unit_squares<float>(t, e0));
    else if (t.type == BGPO_BF16) mine.add(unit_squares<__nv_bfloat16>(t, e0));
    else mine.add(unit_squares<__half>(t, e0));
  }
  __shared__ Sum2 s_warp[kWarps];
  __shared__ bool s_last;
  mine.over_warp();
  if (lane == 0) s_warp[warp] = mine;
  __syncthreads();
  if (threadIdx.x == 0) {
    for (int i = 1; i < kWarps; ++i) mine.add(s_warp[i]);
    a.w.squares[1 + blockIdx.x] = make_float2(mine.s, mine.c);
    __threadfence();
    s_last = atomicInc(a.w.ticket, gridDim.x - 1) == gridDim.x - 1;
    __threadfence();
  }
  __syncthreads();
  if (!s_last) return;
  mine = {};
  for (int b = threadIdx.x; b < (int)gridDim.x; b += kThreads) {
    const float2 q = __ldcg(&a.w.squares[1 + b]);
    mine.add(Sum2{q.x, q.y});
  }
  mine.over_warp();
  if (lane == 0) s_warp[warp] = mine;
  __syncthreads();
  if (threadIdx.x != 0) return;
  for (int i = 1; i < kWarps; ++i) mine.add(s_warp[i]);
  if (!a.first) {                    // the launches before this one, of the same call
    const float2 q = a.w.squares[0];
    mine.add(Sum2{q.x, q.y});
  }
  a.w.squares[0] = make_float2(mine.s, mine.c);
  if (a.last) {
    const float norm = sqrtf(mine.value());
    *a.norm = norm;
    if (!isfinite(norm)) set_device_error(a.w.err, kStatusNonfinite, KID_GRAD_NORM * 16);
  }
}

template <class T, class O>
__device__ __forceinline__ void unit_scale(const GradTensor& t, int64_t e0, float f) {
  const T* p = static_cast<const T*>(t.src);
  O* o = static_cast<O*>(t.dst);
  const int64_t i0 = e0 + 8 * threadIdx.x;
  if (e0 >= 0 && e0 + kGradUnit <= t.n && (t.flags & kGradVector)) {   // block-uniform
    Vec8<T> q[kGradVecs];
#pragma unroll
    for (int k = 0; k < kGradVecs; ++k) q[k].load(p + i0 + k * 8 * kThreads);
#pragma unroll
    for (int k = 0; k < kGradVecs; ++k) {
      float v[8];
      q[k].get(v);
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] = f == 1.f ? v[j] : v[j] * f;   // 1 x keeps a NaN's bits
      put8(o + i0 + k * 8 * kThreads, v);
    }
    return;
  }
  // the ends of a tensor, and outputs that lie otherwise: neighbouring lanes take
  // neighbouring elements, eight loads in flight
  for (int64_t i = e0 + threadIdx.x; i < e0 + kGradUnit && i < t.n; i += 8 * kThreads) {
    float v[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int64_t x = i + j * kThreads;
      v[j] = x >= 0 && x < t.n ? to_float(p[x]) : 0.f;
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int64_t x = i + j * kThreads;
      if (x >= 0 && x < t.n) put(o + x, f == 1.f ? v[j] : v[j] * f);
    }
  }
}

template <class T>
__device__ __forceinline__ void unit_scale_to(const GradTensor& t, int64_t e0, float f) {
  if (t.out_type == BGPO_F32) unit_scale<T, float>(t, e0, f);
  else if (t.out_type == BGPO_BF16) unit_scale<T, __nv_bfloat16>(t, e0, f);
  else unit_scale<T, __half>(t, e0, f);
}

template <int CAP>
__global__ void __launch_bounds__(kThreads, 4)
    k_grad_clip(const __grid_constant__ GradList<CAP> l, GradClipArgs a) {
  pdl_begin();
  const float norm = *a.norm;
  const float f = isfinite(norm) ? fminf(1.f, a.max_norm / (norm + 1e-6f)) : 1.f;
  if (a.err && !isfinite(norm) && blockIdx.x == 0 && threadIdx.x == 0)
    set_device_error(a.err, kStatusNonfinite, KID_GRAD_CLIP * 16);
  for (uint32_t i = blockIdx.x; i < l.units; i += gridDim.x) {
    const uint32_t u = l.units - 1 - i;
    const GradTensor& t = l.t[tensor_of(l, u)];
    if (f == 1.f && (t.flags & kGradInPlace)) continue;   // 1 x is x
    const int64_t e0 = unit_begin(t, u);
    if (t.type == BGPO_F32) unit_scale_to<float>(t, e0, f);
    else if (t.type == BGPO_BF16) unit_scale_to<__nv_bfloat16>(t, e0, f);
    else unit_scale_to<__half>(t, e0, f);
  }
}

// Twice as many blocks as the device holds at once (64 registers a thread): 759 us for the
// norm and the clipping of 2.1 GB of fp32 into bf16, 820 with as many as it holds.
int grad_blocks(uint32_t units, int num_sms) {
  const int64_t most = 8 * (int64_t)num_sms < kTrainMaxBlocks ? 8 * (int64_t)num_sms
                                                              : (int64_t)kTrainMaxBlocks;
  return (int)(units < 1 ? 1 : units < most ? units : most);
}

template <int CAP>
void copy_list(const GradList<kGradMany>& from, GradList<CAP>* to) {
  to->count = from.count;
  to->units = from.units;
  for (int i = 0; i < from.count; ++i) to->t[i] = from.t[i];
}

}  // namespace

cudaError_t launch_grad_norm(const GradList<kGradMany>& l, const GradNormArgs& a, int num_sms,
                             cudaStream_t s) {
  const unsigned grid = (unsigned)grad_blocks(l.units, num_sms);
  if (l.count > kGradFew) return launch_dependent(k_grad_norm<kGradMany>, grid, kThreads, 0, s, l, a);
  GradList<kGradFew> few;
  copy_list(l, &few);
  return launch_dependent(k_grad_norm<kGradFew>, grid, kThreads, 0, s, few, a);
}

cudaError_t launch_grad_clip(const GradList<kGradMany>& l, const GradClipArgs& a, int num_sms,
                             cudaStream_t s) {
  const unsigned grid = (unsigned)grad_blocks(l.units, num_sms);
  if (l.count > kGradFew) return launch_dependent(k_grad_clip<kGradMany>, grid, kThreads, 0, s, l, a);
  GradList<kGradFew> few;
  copy_list(l, &few);
  return launch_dependent(k_grad_clip<kGradFew>, grid, kThreads, 0, s, few, a);
}

}  // namespace bgpo
