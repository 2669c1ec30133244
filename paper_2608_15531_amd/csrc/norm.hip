// The norm after a block, its gate, the residual sum and the norm before the next
// block (fq_gated_residual_norm): one pass over the rows.
//
//     u = x rsqrt(mean(x^2) + eps) w_post,  r = a residual + g u,
//     h = r rsqrt(mean(r^2) + eps) w_pre
//
// A row stays in the registers of the threads that share it (8 columns a thread at a
// time) from its one read to its one write, so both means cost no second pass.  The
// kernel is bound by memory: 13 operations against 10 bytes and more an element.  8191
// rows of 8192, bf16 x and gate, fp32 residual: 196 us, 4.8 TB/s (a copy of 1 GiB: 5.1);
// 4 rows of 4096: 3.2 us, a chain of loads, two sums over the workgroup and stores.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "device.hpp"
#include "lanes.hpp"
#include "layer.hpp"

namespace fqk {

namespace {

// Eight elements with the alignment of one: the hardware takes 16-byte loads and
// stores at any address, so rows of odd length need no path of their own but for
// their last vector.
struct __attribute__((packed, aligned(2))) Bf16x8 { uint32_t w[4]; };
struct __attribute__((packed, aligned(4))) F32x8 { float f[8]; };

struct NormArgs {
  const void* x;
  const void* residual;
  const uint16_t* post;
  const uint16_t* gate;
  const uint16_t* pre;
  void* out;
  uint16_t* h;
  int64_t x_stride, residual_stride, gate_stride, out_stride, h_stride;
  int rows, cols;
  float eps, scale;
};

__device__ __forceinline__ void load8(const uint16_t* p, int n, float v[8]) {
  if (n >= 8) {
    const Bf16x8 q = *reinterpret_cast<const Bf16x8*>(p);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      v[2 * i] = __builtin_bit_cast(float, q.w[i] << 16);
      v[2 * i + 1] = __builtin_bit_cast(float, q.w[i] & 0xFFFF0000u);
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = i < n ? bf16_bits_to_f32(p[i]) : 0.f;
  }
}

__device__ __forceinline__ void load8(const float* p, int n, float v[8]) {
  if (n >= 8) {
    const F32x8 q = *reinterpret_cast<const F32x8*>(p);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = q.f[i];
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = i < n ? p[i] : 0.f;
  }
}

__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
  typedef __bf16 b2 __attribute__((__vector_size__(4)));
  const b2 r = {static_cast<__bf16>(lo), static_cast<__bf16>(hi)};
  return __builtin_bit_cast(uint32_t, r);
}

__device__ __forceinline__ void store8(uint16_t* p, int n, const float v[8]) {
  if (n >= 8) {
    Bf16x8 q;
#pragma unroll
    for (int i = 0; i < 4; ++i) q.w[i] = pack_bf16(v[2 * i], v[2 * i + 1]);
    *reinterpret_cast<Bf16x8*>(p) = q;
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i < n) p[i] = uint16_t(pack_bf16(v[i], 0.f));
  }
}

__device__ __forceinline__ void store8(float* p, int n, const float v[8]) {
  if (n >= 8) {
    F32x8 q;
#pragma unroll
    for (int i = 0; i < 8; ++i) q.f[i] = v[i];
    *reinterpret_cast<F32x8*>(p) = q;
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i < n) p[i] = v[i];
  }
}

// Sum over the TPR threads of a row (the same in all of them).  `part` has one
// float per wave; a second sum of the same row uses another one.
template <int TPR>
__device__ __forceinline__ float row_sum(float v, float* part) {
  v = over_lanes<64>(v, Add{});
  if constexpr (TPR > 64) {
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = v;
    __syncthreads();
    v = 0.f;
#pragma unroll
    for (int w = 0; w < TPR / 64; ++w) v += part[w];
  }
  return v;
}

// TPR threads a row, NV vectors of 8 columns a thread; blockDim = max(TPR, 256), so
// rows of up to 1024 columns go four to a workgroup.
template <class XT, class RT, int TPR, int NV>
__global__ void __launch_bounds__(TPR < 256 ? 256 : TPR) norm_kernel(NormArgs a) {
  __shared__ float part[2][16];
  const int row = TPR < 256 ? int(blockIdx.x * (256 / TPR) + threadIdx.x / TPR) : int(blockIdx.x);
  if (TPR == 64 && row >= a.rows) return;   // whole waves, and no barrier below with TPR == 64
  const int t = threadIdx.x % TPR;
  float x[NV][8];
  const XT* xr = static_cast<const XT*>(a.x) + row * a.x_stride;
#pragma unroll
  for (int v = 0; v < NV; ++v) {
    const int c = (v * TPR + t) * 8;
    load8(xr + c, a.cols - c, x[v]);
  }
  float res[NV][8];
  if (a.residual) {
    const RT* rr = static_cast<const RT*>(a.residual) + row * a.residual_stride;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const int c = (v * TPR + t) * 8;
      load8(rr + c, a.cols - c, res[v]);
    }
  }
  const float inv_n = 1.f / float(a.cols);
  if (a.post) {
    float s = 0.f;
#pragma unroll
    for (int v = 0; v < NV; ++v)
#pragma unroll
      for (int i = 0; i < 8; ++i) s = fmaf(x[v][i], x[v][i], s);
    const float f = 1.f / sqrtf(row_sum<TPR>(s, part[0]) * inv_n + a.eps);
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const int c = (v * TPR + t) * 8;
      float w[8];
      load8(a.post + c, a.cols - c, w);
#pragma unroll
      for (int i = 0; i < 8; ++i) x[v][i] = x[v][i] * f * w[i];
    }
  }
  if (a.gate) {
    const uint16_t* gr = a.gate + row * a.gate_stride;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const int c = (v * TPR + t) * 8;
      float w[8];
      load8(gr + c, a.cols - c, w);
#pragma unroll
      for (int i = 0; i < 8; ++i) x[v][i] *= w[i];
    }
  }
  if (a.residual) {
#pragma unroll
    for (int v = 0; v < NV; ++v)
#pragma unroll
      for (int i = 0; i < 8; ++i) x[v][i] = fmaf(a.scale, res[v][i], x[v][i]);
  }
  if (a.out) {
    RT* orow = static_cast<RT*>(a.out) + row * a.out_stride;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const int c = (v * TPR + t) * 8;
      store8(orow + c, a.cols - c, x[v]);
    }
  }
  if (a.h) {
    float s = 0.f;
#pragma unroll
    for (int v = 0; v < NV; ++v)
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if ((v * TPR + t) * 8 + i < a.cols) s = fmaf(x[v][i], x[v][i], s);
    const float f = 1.f / sqrtf(row_sum<TPR>(s, part[1]) * inv_n + a.eps);
    uint16_t* hr = a.h + row * a.h_stride;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const int c = (v * TPR + t) * 8;
      float w[8];
      load8(a.pre + c, a.cols - c, w);
#pragma unroll
      for (int i = 0; i < 8; ++i) w[i] = x[v][i] * f * w[i];
      store8(hr + c, a.cols - c, w);
    }
  }
}

// Rows of one launch, of up to 1024 threads each: HIP takes fewer than 2^32 threads in one
// dimension of a grid.
constexpr int kMostRows = 1 << 21;

template <class T>
T* from_row(T* p, int64_t row, int64_t stride) { return p ? p + row * stride : p; }

template <class XT, class RT>
NormArgs part_of(const NormArgs& all, int64_t row) {
  NormArgs a = all;
  a.x = from_row(static_cast<const XT*>(all.x), row, all.x_stride);
  a.residual = from_row(static_cast<const RT*>(all.residual), row, all.residual_stride);
  a.gate = from_row(all.gate, row, all.gate_stride);
  a.out = from_row(static_cast<RT*>(all.out), row, all.out_stride);
  a.h = from_row(all.h, row, all.h_stride);
  a.rows = int(std::min<int64_t>(all.rows - row, kMostRows));
  return a;
}

template <class XT, class RT>
int launch_part(const NormArgs& a, hipStream_t s) {
  const dim3 grid(a.rows), four((unsigned(a.rows) + 3) / 4);
  if (a.cols <= 512) hipLaunchKernelGGL((norm_kernel<XT, RT, 64, 1>), four, dim3(256), 0, s, a);
  else if (a.cols <= 1024) hipLaunchKernelGGL((norm_kernel<XT, RT, 64, 2>), four, dim3(256), 0, s, a);
  else if (a.cols <= 2048) hipLaunchKernelGGL((norm_kernel<XT, RT, 256, 1>), grid, dim3(256), 0, s, a);
  else if (a.cols <= 4096) hipLaunchKernelGGL((norm_kernel<XT, RT, 256, 2>), grid, dim3(256), 0, s, a);
  else if (a.cols <= 8192) hipLaunchKernelGGL((norm_kernel<XT, RT, 256, 4>), grid, dim3(256), 0, s, a);
  else if (a.cols <= 16384) hipLaunchKernelGGL((norm_kernel<XT, RT, 1024, 2>), grid, dim3(1024), 0, s, a);
  else hipLaunchKernelGGL((norm_kernel<XT, RT, 1024, 4>), grid, dim3(1024), 0, s, a);
  return int(hipGetLastError());
}

template <class XT, class RT>
int launch_typed(const NormArgs& a, hipStream_t s) {
  int e = 0;
  for (int64_t row = 0; row < a.rows && e == 0; row += kMostRows) e = launch_part<XT, RT>(part_of<XT, RT>(a, row), s);
  return e;
}

}  // namespace

}  // namespace fqk

namespace fqi {

int launch_norm(const fq_norm& n, const void* x, const void* residual, const uint16_t* post_weight,
                const uint16_t* gate, const uint16_t* pre_weight, void* residual_out, uint16_t* h,
                void* stream) {
  fqk::NormArgs a{x, residual, post_weight, gate, pre_weight, residual_out, h,
                  n.x_stride, n.residual_stride, n.gate_stride, n.residual_out_stride, n.h_stride,
                  int(n.rows), n.cols, n.eps, n.residual_scale};
  hipStream_t s = static_cast<hipStream_t>(stream);
  const bool xf = n.x_dtype == FQ_Y_F32, rf = n.residual_dtype == FQ_Y_F32;
  if (xf && rf) return fqk::launch_typed<float, float>(a, s);
  if (xf) return fqk::launch_typed<float, uint16_t>(a, s);
  if (rf) return fqk::launch_typed<uint16_t, float>(a, s);
  return fqk::launch_typed<uint16_t, uint16_t>(a, s);
}

}  // namespace fqi
