// The paged KV cache: rows quantised as they are written, and read back.
//
// A row's range needs all of its channels and nothing else, so D / 8 lanes hold one
// row, 16 bytes of bf16 each, and agree on its range without LDS.  A workgroup takes
// consecutive tokens of one head: in a page these rows follow one another, so the
// stores of a workgroup fill whole cache lines, while each row's read is 128 or 256
// contiguous bytes wherever it lies.  Both kernels are bound by memory.
#include <hip/hip_runtime.h>

#include "device.hpp"
#include "layer.hpp"

namespace fqk {

namespace {

struct CacheArgs {
  char* rows[2];           // K, V
  uint32_t* meta[2];
  int64_t page_stride, head_stride, token_stride, meta_page_stride, meta_head_stride;
  int64_t n_slots;
  uint32_t page_size;
};

struct Place {
  int64_t page;
  uint32_t off;
};

__device__ __forceinline__ Place place_of(int64_t slot, const CacheArgs& a) {
  // slots of a cache of up to 2^31 pages fit 47 bits; the 32-bit division serves all but
  // the largest caches
  Place p;
  if (slot >> 32) {
    p.page = slot / int64_t(a.page_size);
  } else {
    p.page = uint32_t(slot) / a.page_size;
  }
  p.off = uint32_t(slot - p.page * int64_t(a.page_size));
  return p;
}

__device__ __forceinline__ uint32_t pack2(float lo, float hi) {
  typedef __bf16 b2 __attribute__((__vector_size__(4)));
  const b2 r = {static_cast<__bf16>(lo), static_cast<__bf16>(hi)};
  return __builtin_bit_cast(uint32_t, r);
}

template <int KIND>
constexpr float kTop = KIND == FQ_KV_INT8 ? 255.f : 15.f;

// The scale of a row: the smallest bf16 not below span / top (the next 16 bits up of
// a value that is not negative).  The quotient is the correctly rounded one: with a
// product by 1 / top, spans that are a multiple of a bf16 would get the next step.
template <int KIND>
__device__ __forceinline__ float scale_of(float span) {
  if (!(span > 0.f)) return 1.f;
  const float q = __fdiv_rn(span, kTop<KIND>);
  return __builtin_bit_cast(float, (__builtin_bit_cast(uint32_t, q) + 0xFFFFu) & 0xFFFF0000u);
}

template <int KIND, int D>
__global__ void __launch_bounds__(256)
kv_write_kernel(CacheArgs a, const uint16_t* K, const uint16_t* V, int64_t k_token, int64_t k_head,
                int64_t v_token, int64_t v_head, const int64_t* slots, int n_tokens) {
  constexpr int LPR = D / 8;   // lanes a row
  const int t = int(blockIdx.x) * (256 / LPR) + int(threadIdx.x) / LPR;
  const int i = int(threadIdx.x) % LPR;
  const int head = int(blockIdx.y);
  const int which = int(blockIdx.z);   // 0: K, 1: V
  const bool in = t < n_tokens;
  const int64_t slot = in ? slots[t] : -1;
  const bool store = uint64_t(slot) < uint64_t(a.n_slots);
  const uint16_t* src = (which ? V + head * v_head : K + head * k_head) + (which ? v_token : k_token) * int64_t(t);
  uint4 w{0, 0, 0, 0};
  if (store) w = reinterpret_cast<const uint4*>(src)[i];
  const Place p = place_of(store ? slot : 0, a);
  char* dst = a.rows[which] + p.page * a.page_stride + head * a.head_stride + int64_t(p.off) * a.token_stride;
  if constexpr (KIND == FQ_KV_BF16) {
    if (store) reinterpret_cast<uint4*>(dst)[i] = w;
    return;
  } else {
    float x[8];
    const uint32_t ws[4] = {w.x, w.y, w.z, w.w};
    float hi = 0.f, lo = 0.f;
    bool odd = false;   // an infinity or a NaN
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      x[2 * j] = __builtin_bit_cast(float, ws[j] << 16);
      x[2 * j + 1] = __builtin_bit_cast(float, ws[j] & 0xFFFF0000u);
      odd |= (ws[j] & 0x7F80u) == 0x7F80u || (ws[j] & 0x7F800000u) == 0x7F800000u;
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      hi = fmaxf(hi, x[j]);
      lo = fminf(lo, x[j]);
    }
    if (odd) hi = __builtin_inff();
#pragma unroll
    for (int m = 1; m < LPR; m <<= 1) {
      hi = fmaxf(hi, __shfl_xor(hi, m));
      lo = fminf(lo, __shfl_xor(lo, m));
    }
    const float span = hi - lo;
    const bool bad = !(span <= 3.4028234663852886e38f);
    const float s = scale_of<KIND>(bad ? 0.f : span);
    const float z = fminf(fmaxf(rintf(__fdiv_rn(-lo, s)), 0.f), kTop<KIND>);
    uint32_t c[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float q = fminf(fmaxf(rintf(__fdiv_rn(x[j], s)) + z, 0.f), kTop<KIND>);
      c[j] = bad ? 0u : uint32_t(q);
    }
    if (!store) return;
    if constexpr (KIND == FQ_KV_INT8) {
      uint2 o;
      o.x = c[0] | c[1] << 8 | c[2] << 16 | c[3] << 24;
      o.y = c[4] | c[5] << 8 | c[6] << 16 | c[7] << 24;
      reinterpret_cast<uint2*>(dst)[i] = o;
    } else {
      uint32_t o = 0;
#pragma unroll
      for (int j = 0; j < 8; ++j) o |= c[j] << (4 * j);
      reinterpret_cast<uint32_t*>(dst)[i] = o;
    }
    if (i == 0) {
      const uint32_t zb = bad ? 0u : __builtin_bit_cast(uint32_t, z) & 0xFFFF0000u;
      const uint32_t sb = bad ? 0x7FC0u : __builtin_bit_cast(uint32_t, s) >> 16;
      a.meta[which][p.page * a.meta_page_stride + head * a.meta_head_stride + p.off] = sb | zb;
    }
  }
}

template <int KIND, int D, bool F32>
__global__ void __launch_bounds__(256)
kv_read_kernel(CacheArgs a, const int64_t* slots, int n_tokens, void* K, void* V) {
  constexpr int LPR = D / 8;
  const int t = int(blockIdx.x) * (256 / LPR) + int(threadIdx.x) / LPR;
  const int i = int(threadIdx.x) % LPR;
  const int head = int(blockIdx.y);
  const int which = int(blockIdx.z);
  if (t >= n_tokens) return;
  const int64_t slot = slots[t];
  const bool in = uint64_t(slot) < uint64_t(a.n_slots);
  const Place p = place_of(in ? slot : 0, a);
  const char* src = a.rows[which] + p.page * a.page_stride + head * a.head_stride + int64_t(p.off) * a.token_stride;
  float x[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
  if (in) {
    if constexpr (KIND == FQ_KV_BF16) {
      const uint4 w = reinterpret_cast<const uint4*>(src)[i];
      const uint32_t ws[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        x[2 * j] = __builtin_bit_cast(float, ws[j] << 16);
        x[2 * j + 1] = __builtin_bit_cast(float, ws[j] & 0xFFFF0000u);
      }
    } else {
      const uint32_t m = a.meta[which][p.page * a.meta_page_stride + head * a.meta_head_stride + p.off];
      const float s = __builtin_bit_cast(float, m << 16), z = __builtin_bit_cast(float, m & 0xFFFF0000u);
      if constexpr (KIND == FQ_KV_INT8) {
        const uint2 w = reinterpret_cast<const uint2*>(src)[i];
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] = s * (float(((j < 4 ? w.x : w.y) >> (8 * (j & 3))) & 255u) - z);
      } else {
        const uint32_t w = reinterpret_cast<const uint32_t*>(src)[i];
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] = s * (float((w >> (4 * j)) & 15u) - z);
      }
    }
  }
  const int64_t at = (int64_t(t) * gridDim.y + head) * D + i * 8;
  if constexpr (F32) {
    float* o = static_cast<float*>(which ? V : K) + at;
    reinterpret_cast<float4*>(o)[0] = float4{x[0], x[1], x[2], x[3]};
    reinterpret_cast<float4*>(o)[1] = float4{x[4], x[5], x[6], x[7]};
  } else {
    uint16_t* o = static_cast<uint16_t*>(which ? V : K) + at;
    *reinterpret_cast<uint4*>(o) = uint4{pack2(x[0], x[1]), pack2(x[2], x[3]), pack2(x[4], x[5]), pack2(x[6], x[7])};
  }
}

CacheArgs cache_args(const fq_kv_cache& c) {
  return CacheArgs{{static_cast<char*>(c.k), static_cast<char*>(c.v)},
                   {static_cast<uint32_t*>(c.k_meta), static_cast<uint32_t*>(c.v_meta)},
                   c.page_stride, c.head_stride, c.token_stride, c.meta_page_stride, c.meta_head_stride,
                   c.n_pages * c.page_size, uint32_t(c.page_size)};
}

// f(integral_constant KIND, integral_constant D) for the cache's kind and head size.
template <class F>
void by_kind(const fq_kv_cache& c, F&& f) {
  auto with = [&](auto kind) {
    if (c.head_dim == 64) f(kind, std::integral_constant<int, 64>{});
    else f(kind, std::integral_constant<int, 128>{});
  };
  if (c.kind == FQ_KV_BF16) with(std::integral_constant<int, FQ_KV_BF16>{});
  else if (c.kind == FQ_KV_INT8) with(std::integral_constant<int, FQ_KV_INT8>{});
  else with(std::integral_constant<int, FQ_KV_INT4>{});
}

dim3 token_grid(const fq_kv_cache& c, int64_t n_tokens) {
  const int per = 256 / (c.head_dim / 8);
  return dim3(unsigned((n_tokens + per - 1) / per), unsigned(c.n_kv_heads), 2);
}

}  // namespace

}  // namespace fqk

namespace fqi {

int launch_kv_write(const fq_kv_cache& c, const uint16_t* K, const uint16_t* V,
                    int64_t k_token_stride, int64_t k_head_stride, int64_t v_token_stride,
                    int64_t v_head_stride, const int64_t* slots, int64_t n_tokens, void* stream) {
  const fqk::CacheArgs a = fqk::cache_args(c);
  fqk::by_kind(c, [&](auto kind, auto dim) {
    hipLaunchKernelGGL((fqk::kv_write_kernel<kind.value, dim.value>), fqk::token_grid(c, n_tokens), dim3(256), 0,
                       static_cast<hipStream_t>(stream), a, K, V, k_token_stride, k_head_stride, v_token_stride,
                       v_head_stride, slots, int(n_tokens));
  });
  return int(hipGetLastError());
}

int launch_kv_read(const fq_kv_cache& c, const int64_t* slots, int64_t n_tokens, void* K, void* V,
                   bool f32, void* stream) {
  const fqk::CacheArgs a = fqk::cache_args(c);
  fqk::by_kind(c, [&](auto kind, auto dim) {
    if (f32)
      hipLaunchKernelGGL((fqk::kv_read_kernel<kind.value, dim.value, true>), fqk::token_grid(c, n_tokens), dim3(256),
                         0, static_cast<hipStream_t>(stream), a, slots, int(n_tokens), K, V);
    else
      hipLaunchKernelGGL((fqk::kv_read_kernel<kind.value, dim.value, false>), fqk::token_grid(c, n_tokens), dim3(256),
                         0, static_cast<hipStream_t>(stream), a, slots, int(n_tokens), K, V);
  });
  return int(hipGetLastError());
}

}  // namespace fqi
