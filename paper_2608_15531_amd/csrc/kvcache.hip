// The paged KV cache: rows quantised as they are written, and read back.
//
// A row's range needs all of its channels and nothing else, so D / 8 lanes hold one
// row, 16 bytes of bf16 each, and agree on its range without LDS.  A thread takes K and V
// of a token and head, both loads first.  A workgroup takes consecutive tokens of one head:
// in a page these rows follow one another, so their stores fill whole cache lines.
//
// Memory bounds both kernels (a copy of 1 GiB: 5.1 TB/s), and with codes the arithmetic of
// the write stands next to it.  4096 tokens of 8 heads x 128, bf16, written: 5.8 us, 5.8
// TB/s; 12001 tokens at 4 bits: written in 13.7 us, 4.5 TB/s (18 with general divisions and
// conversions), read back in 12, 5.2 TB/s; 30007 tokens at 8 bits read as fp32: 49 us, 6.3
// TB/s.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "device.hpp"
#include "lanes.hpp"
#include "layer.hpp"
#include "quotient.hpp"

namespace fqk {

using fqi::inverse;
using fqi::quotient;

namespace {

struct CacheArgs {
  char* rows[2];           // K, V
  uint32_t* meta[2];
  int64_t page_stride, head_stride, token_stride, meta_page_stride, meta_head_stride;
  int64_t n_slots;
  uint32_t page_size;
  uint32_t page_magic, page_shift;   // of the division by the page's 16-token blocks
};

struct Place {
  uint32_t page, off;
};

// Page and token of a slot below n_slots (up to 2^47).  A slot of 32 bits has a block b of
// 28, and with P <= 2^l blocks a page and m = ceil(2^(28 + l) / P) the page is
// b m >> (28 + l): m is less than 1 too large, which adds less than 2^-l <= 1 / P.
__device__ __forceinline__ Place place_of(int64_t slot, const CacheArgs& a) {
  Place p;
  if (slot >> 32) p.page = uint32_t(slot / int64_t(a.page_size));
  else p.page = uint32_t(uint64_t(uint32_t(slot) >> 4) * a.page_magic >> a.page_shift);
  p.off = uint32_t(slot) - p.page * a.page_size;
  return p;
}

__device__ __forceinline__ uint32_t pack2(float lo, float hi) {
  typedef __bf16 b2 __attribute__((__vector_size__(4)));
  const b2 r = {static_cast<__bf16>(lo), static_cast<__bf16>(hi)};
  return __builtin_bit_cast(uint32_t, r);
}

template <int KIND>
constexpr float kTop = KIND == FQ_KV_INT8 ? 255.f : 15.f;

// Maximum and minimum that a NaN passes through.
struct MaxNan {
  __device__ __forceinline__ float operator()(float a, float b) const { return __builtin_elementwise_maximum(a, b); }
};
struct MinNan {
  __device__ __forceinline__ float operator()(float a, float b) const { return __builtin_elementwise_minimum(a, b); }
};

// The next bf16 up of a value that is not negative, unless it is one.
__device__ __forceinline__ float bf16_up(float v) {
  return __builtin_bit_cast(float, (__builtin_bit_cast(uint32_t, v) + 0xFFFFu) & 0xFFFF0000u);
}

// Quantises a row's 8 channels of this lane and stores them.  The scale is the smallest
// bf16 not below span / top, and every quotient is the correctly rounded one: with
// products by rounded inverses, spans that are a multiple of a bf16 would get the next
// scale, and ties the next code.  Rows of ordinary size take quotient(), about a third of
// the operations of the general division, which rows of zeros, of extreme sizes and of
// infinities or NaN take.
//
// To whole numbers by sums with 1.5 2^23, where floats are 1 apart: the code is then the
// low bits of the float.
template <int KIND, int D>
__device__ __forceinline__ void store_row(char* dst, uint32_t* meta, uint4 w, int i, bool store) {
  if constexpr (KIND == FQ_KV_BF16) {
    if (store) reinterpret_cast<uint4*>(dst)[i] = w;
  } else {
    constexpr int LPR = D / 8;
    constexpr float top = kTop<KIND>, whole = 0x1.8p23f;
    float x[8];
    const uint32_t ws[4] = {w.x, w.y, w.z, w.w};
    float hi = 0.f, lo = 0.f;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      x[2 * j] = __builtin_bit_cast(float, ws[j] << 16);
      x[2 * j + 1] = __builtin_bit_cast(float, ws[j] & 0xFFFF0000u);
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      hi = MaxNan{}(hi, x[j]);
      lo = MinNan{}(lo, x[j]);
    }
    hi = over_lanes<LPR>(hi, MaxNan{});
    lo = over_lanes<LPR>(lo, MinNan{});
    const float span = hi - lo;
    float s, zq;
    uint32_t sb;
    if (span > 0x1p-90f && span < 0x1p90f) {
      s = bf16_up(quotient(span, top, 1.f / top));
      const float r = inverse(s, __builtin_amdgcn_rcpf(s));
      zq = quotient(-lo, s, r);
#pragma unroll
      for (int j = 0; j < 8; ++j) x[j] = quotient(x[j], s, r);
      sb = __builtin_bit_cast(uint32_t, s) >> 16;
    } else {
      const bool bad = !(span <= 3.4028234663852886e38f);   // an infinity or NaN, or a span beyond fp32
      s = span > 0.f && !bad ? bf16_up(__fdiv_rn(span, top)) : 1.f;
      zq = bad ? 0.f : __fdiv_rn(-lo, s);
#pragma unroll
      for (int j = 0; j < 8; ++j) x[j] = bad ? 0.f : __fdiv_rn(x[j], s);
      sb = bad ? 0x7FC0u : __builtin_bit_cast(uint32_t, s) >> 16;
    }
    const float z = __builtin_amdgcn_fmed3f(zq + whole, whole, whole + top) - whole;
    uint32_t c[8];
#pragma unroll
    for (int j = 0; j < 8; ++j)
      c[j] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_fmed3f(x[j] + whole + z, whole, whole + top));
    if (!store) return;
    // the codes are the low bits; the bits above the low 16 are those of 1.5 2^23
    const auto bytes = [](uint32_t a, uint32_t b, uint32_t e, uint32_t f) {
      return __builtin_amdgcn_perm(__builtin_amdgcn_perm(f, e, 0x0C0C0400u), __builtin_amdgcn_perm(b, a, 0x0C0C0400u),
                                   0x05040100u);
    };
    if constexpr (KIND == FQ_KV_INT8) {
      reinterpret_cast<uint2*>(dst)[i] = uint2{bytes(c[0], c[1], c[2], c[3]), bytes(c[4], c[5], c[6], c[7])};
    } else {
      reinterpret_cast<uint32_t*>(dst)[i] =
          bytes(c[0] | c[1] << 4, c[2] | c[3] << 4, c[4] | c[5] << 4, c[6] | c[7] << 4);
    }
    if (i == 0) *meta = sb | (__builtin_bit_cast(uint32_t, z) & 0xFFFF0000u);
  }
}

template <int KIND, int D>
__global__ void __launch_bounds__(256)
kv_write_kernel(CacheArgs a, const uint16_t* K, const uint16_t* V, int64_t k_token, int64_t k_head,
                int64_t v_token, int64_t v_head, const int64_t* slots, int n_tokens) {
  constexpr int LPR = D / 8, PER = 256 / LPR;   // lanes a row, rows of a workgroup
  const int i = int(threadIdx.x) % LPR;
  const int head = int(blockIdx.y);
  const int t = int(blockIdx.x) * PER + int(threadIdx.x) / LPR;
  if (t >= n_tokens) return;   // whole rows: the lanes of a row have the same token
  const int64_t slot = slots[t];
  const uint4 k = reinterpret_cast<const uint4*>(K + head * k_head + k_token * int64_t(t))[i];
  const uint4 v = reinterpret_cast<const uint4*>(V + head * v_head + v_token * int64_t(t))[i];
  const bool store = uint64_t(slot) < uint64_t(a.n_slots);
  const Place p = place_of(store ? slot : 0, a);
  const int64_t at = p.page * a.page_stride + head * a.head_stride + int64_t(p.off) * a.token_stride;
  const int64_t word = p.page * a.meta_page_stride + head * a.meta_head_stride + p.off;
  store_row<KIND, D>(a.rows[0] + at, a.meta[0] + word, k, i, store);
  store_row<KIND, D>(a.rows[1] + at, a.meta[1] + word, v, i, store);
}

// N channels from channel c of a row on, as numbers.
template <int KIND, int N>
__device__ __forceinline__ void load_channels(const char* row, int c, uint32_t meta, float (&x)[N]) {
  if constexpr (KIND == FQ_KV_BF16) {
#pragma unroll
    for (int j = 0; j < N / 4; ++j) {
      const uint2 w = reinterpret_cast<const uint2*>(row + 2 * c)[j];
      x[4 * j] = __builtin_bit_cast(float, w.x << 16);
      x[4 * j + 1] = __builtin_bit_cast(float, w.x & 0xFFFF0000u);
      x[4 * j + 2] = __builtin_bit_cast(float, w.y << 16);
      x[4 * j + 3] = __builtin_bit_cast(float, w.y & 0xFFFF0000u);
    }
  } else {
    const float s = __builtin_bit_cast(float, meta << 16), z = __builtin_bit_cast(float, meta & 0xFFFF0000u);
    if constexpr (KIND == FQ_KV_INT8) {
#pragma unroll
      for (int j = 0; j < N / 4; ++j) {
        const uint32_t w = reinterpret_cast<const uint32_t*>(row + c)[j];
#pragma unroll
        for (int e = 0; e < 4; ++e) x[4 * j + e] = s * (float((w >> (8 * e)) & 255u) - z);
      }
    } else {
      uint32_t w;
      if constexpr (N == 8) w = *reinterpret_cast<const uint32_t*>(row + c / 2);
      else w = *reinterpret_cast<const uint16_t*>(row + c / 2);
#pragma unroll
      for (int e = 0; e < N; ++e) x[e] = s * (float((w >> (4 * e)) & 15u) - z);
    }
  }
}

// A 16-byte store; STREAM: past the caches, for outputs that do not fit them.
template <bool STREAM, class T, class V>
__device__ __forceinline__ void put(T* p, V v) {
  if constexpr (STREAM) __builtin_nontemporal_store(v, reinterpret_cast<V*>(p));
  else *reinterpret_cast<V*>(p) = v;
}

// A lane's channels: 8 in a row for bf16 out; for fp32 4 in each half of the row, so that
// a store of 16 bytes a lane is contiguous over the lanes.
template <int KIND, int D, bool F32, bool STREAM>
__global__ void __launch_bounds__(256)
kv_read_kernel(CacheArgs a, const int64_t* slots, int n_tokens, void* K, void* V) {
  constexpr int LPR = D / 8, PER = 256 / LPR;
  const int i = int(threadIdx.x) % LPR;
  const int head = int(blockIdx.y);
  const int t = int(blockIdx.x) * PER + int(threadIdx.x) / LPR;
  if (t >= n_tokens) return;
  const int64_t slot = slots[t];
  const bool in = uint64_t(slot) < uint64_t(a.n_slots);
  const Place p = place_of(in ? slot : 0, a);
  const int64_t at = p.page * a.page_stride + head * a.head_stride + int64_t(p.off) * a.token_stride;
  const int64_t word = p.page * a.meta_page_stride + head * a.meta_head_stride + p.off;
  float x[2][8];
#pragma unroll
  for (int v = 0; v < 2; ++v) {
    if (!in) {
#pragma unroll
      for (int j = 0; j < 8; ++j) x[v][j] = 0.f;
      continue;
    }
    const uint32_t meta = KIND == FQ_KV_BF16 ? 0u : a.meta[v][word];
    if constexpr (F32) {
      float lo[4], hi[4];
      load_channels<KIND, 4>(a.rows[v] + at, 4 * i, meta, lo);
      load_channels<KIND, 4>(a.rows[v] + at, D / 2 + 4 * i, meta, hi);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        x[v][j] = lo[j];
        x[v][4 + j] = hi[j];
      }
    } else {
      load_channels<KIND, 8>(a.rows[v] + at, 8 * i, meta, x[v]);
    }
  }
  const int64_t to = (int64_t(t) * gridDim.y + head) * D;
#pragma unroll
  for (int v = 0; v < 2; ++v) {
    const float* y = x[v];
    if constexpr (F32) {
      float* o = static_cast<float*>(v ? V : K) + to;
      put<STREAM>(o + 4 * i, f32x4_t{y[0], y[1], y[2], y[3]});
      put<STREAM>(o + D / 2 + 4 * i, f32x4_t{y[4], y[5], y[6], y[7]});
    } else {
      uint16_t* o = static_cast<uint16_t*>(v ? V : K) + to;
      put<STREAM>(o + 8 * i, u32x4_t{pack2(y[0], y[1]), pack2(y[2], y[3]), pack2(y[4], y[5]), pack2(y[6], y[7])});
    }
  }
}

CacheArgs cache_args(const fq_kv_cache& c) {
  const uint32_t blocks = uint32_t(c.page_size) / 16;
  uint32_t l = 0;
  while ((1u << l) < blocks) ++l;
  return CacheArgs{{static_cast<char*>(c.k), static_cast<char*>(c.v)},
                   {static_cast<uint32_t*>(c.k_meta), static_cast<uint32_t*>(c.v_meta)},
                   c.page_stride, c.head_stride, c.token_stride, c.meta_page_stride, c.meta_head_stride,
                   c.n_pages * c.page_size, uint32_t(c.page_size),
                   uint32_t(((uint64_t(1) << (28 + l)) + blocks - 1) / blocks), 28 + l};
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

dim3 token_grid(const fq_kv_cache& c, int n_tokens) {
  const int per = 256 / (c.head_dim / 8);
  return dim3(unsigned((n_tokens + per - 1) / per), unsigned(c.n_kv_heads));
}

// Tokens of one launch, of 16 threads and a head each at most: HIP takes fewer than 2^32
// threads in one dimension of a grid.
constexpr int64_t kMostTokens = int64_t(1) << 24;

// f(first token, tokens) for each launch, while it returns 0.
template <class F>
int in_parts(int64_t n_tokens, F&& f) {
  int e = 0;
  for (int64_t t = 0; t < n_tokens && e == 0; t += kMostTokens) e = f(t, int(std::min(n_tokens - t, kMostTokens)));
  return e;
}

}  // namespace

}  // namespace fqk

namespace fqi {

namespace {
// Outputs larger than this go past the caches.
constexpr int64_t kStreamBytes = int64_t(32) << 20;
}  // namespace

int launch_kv_write(const fq_kv_cache& c, const uint16_t* K, const uint16_t* V,
                    int64_t k_token_stride, int64_t k_head_stride, int64_t v_token_stride,
                    int64_t v_head_stride, const int64_t* slots, int64_t n_tokens, void* stream) {
  const fqk::CacheArgs a = fqk::cache_args(c);
  return fqk::in_parts(n_tokens, [&](int64_t t, int n) {
    fqk::by_kind(c, [&](auto kind, auto dim) {
      hipLaunchKernelGGL((fqk::kv_write_kernel<kind.value, dim.value>), fqk::token_grid(c, n), dim3(256), 0,
                         static_cast<hipStream_t>(stream), a, K + t * k_token_stride, V + t * v_token_stride,
                         k_token_stride, k_head_stride, v_token_stride, v_head_stride, slots + t, n);
    });
    return int(hipGetLastError());
  });
}

int launch_kv_read(const fq_kv_cache& c, const int64_t* slots, int64_t n_tokens, void* K, void* V,
                   bool f32, void* stream) {
  const fqk::CacheArgs a = fqk::cache_args(c);
  const int64_t token_bytes = int64_t(c.n_kv_heads) * c.head_dim * (f32 ? 4 : 2);
  const bool past = 2 * n_tokens * token_bytes > kStreamBytes;
  return fqk::in_parts(n_tokens, [&](int64_t t, int n) {
    fqk::by_kind(c, [&](auto kind, auto dim) {
      auto go = [&](auto wide, auto streamed) {
        hipLaunchKernelGGL((fqk::kv_read_kernel<kind.value, dim.value, wide.value, streamed.value>),
                           fqk::token_grid(c, n), dim3(256), 0, static_cast<hipStream_t>(stream), a, slots + t, n,
                           static_cast<void*>(static_cast<char*>(K) + t * token_bytes),
                           static_cast<void*>(static_cast<char*>(V) + t * token_bytes));
      };
      if (f32 && past) go(std::true_type{}, std::true_type{});
      else if (f32) go(std::true_type{}, std::false_type{});
      else if (past) go(std::false_type{}, std::true_type{});
      else go(std::false_type{}, std::false_type{});
    });
    return int(hipGetLastError());
  });
}

}  // namespace fqi
