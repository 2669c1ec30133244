// The paged KV cache: rows quantised as they are written, and read back.
//
// A row's range needs all of its channels and nothing else, so D / 8 lanes hold one
// row, 16 bytes of bf16 each, and agree on its range without LDS.  A thread takes K and V
// of kTokens tokens of one head, all loads first: the chain slot, row, store is latency,
// and several rows a thread hide it.  A workgroup takes consecutive tokens of one head: in
// a page these rows follow one another, so their stores fill whole cache lines.  Both
// kernels are bound by memory.
#include <hip/hip_runtime.h>

#include "device.hpp"
#include "lanes.hpp"
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

constexpr int kTokens = 1;   // a thread

// Quantises a row's 8 channels of this lane and stores them.  The quotients x / s are the
// correctly rounded ones: of numbers of 8 bits they round to the same integer as the exact
// quotients do, ties among them.  With r = 1 / s rounded correctly, y = x r and the exact
// remainder e = x - y s, fma(e, r, y) is the rounded quotient (Markstein) as long as r and
// e s are far from the ends of the range.
template <int KIND, int D>
__device__ __forceinline__ void store_row(char* dst, uint32_t* meta, uint4 w, int i, bool store) {
  if constexpr (KIND == FQ_KV_BF16) {
    if (store) reinterpret_cast<uint4*>(dst)[i] = w;
  } else {
    constexpr int LPR = D / 8;
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
    hi = over_lanes<LPR>(hi, Max{});
    lo = over_lanes<LPR>(lo, Min{});
    const float span = hi - lo;
    const bool bad = !(span <= 3.4028234663852886e38f);
    const float s = scale_of<KIND>(bad ? 0.f : span);
    const float z = fminf(fmaxf(rintf(__fdiv_rn(-lo, s)), 0.f), kTop<KIND>);
    uint32_t c[8];
    const bool middle = s > 0x1p-100f && s < 0x1p100f;
    const float r = __fdiv_rn(1.f, s);
    if (middle) {
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float y = x[j] * r;
        x[j] = fmaf(fmaf(-y, s, x[j]), r, y);
      }
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) x[j] = __fdiv_rn(x[j], s);
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) c[j] = uint32_t(fminf(fmaxf(rintf(x[j]) + z, 0.f), kTop<KIND>));
    if (bad) {
#pragma unroll
      for (int j = 0; j < 8; ++j) c[j] = 0u;
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
      *meta = sb | zb;
    }
  }
}

template <int KIND, int D>
__global__ void __launch_bounds__(256)
kv_write_kernel(CacheArgs a, const uint16_t* K, const uint16_t* V, int64_t k_token, int64_t k_head,
                int64_t v_token, int64_t v_head, const int64_t* slots, int n_tokens) {
  constexpr int LPR = D / 8, PER = 256 / LPR;   // lanes a row, rows of a workgroup at a time
  const int i = int(threadIdx.x) % LPR;
  const int head = int(blockIdx.y);
  const int t0 = int(blockIdx.x) * (PER * kTokens) + int(threadIdx.x) / LPR;
  int64_t slot[kTokens];
  uint4 k[kTokens], v[kTokens];
#pragma unroll
  for (int u = 0; u < kTokens; ++u) {
    const int t = t0 + u * PER;
    const bool in = t < n_tokens;
    slot[u] = in ? slots[t] : -1;
    k[u] = v[u] = uint4{0, 0, 0, 0};
    if (in) {
      k[u] = reinterpret_cast<const uint4*>(K + head * k_head + k_token * int64_t(t))[i];
      v[u] = reinterpret_cast<const uint4*>(V + head * v_head + v_token * int64_t(t))[i];
    }
  }
#pragma unroll
  for (int u = 0; u < kTokens; ++u) {
    const bool store = uint64_t(slot[u]) < uint64_t(a.n_slots);
    const Place p = place_of(store ? slot[u] : 0, a);
    const int64_t at = p.page * a.page_stride + head * a.head_stride + int64_t(p.off) * a.token_stride;
    const int64_t word = p.page * a.meta_page_stride + head * a.meta_head_stride + p.off;
    store_row<KIND, D>(a.rows[0] + at, a.meta[0] + word, k[u], i, store);
    store_row<KIND, D>(a.rows[1] + at, a.meta[1] + word, v[u], i, store);
  }
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
  const int t0 = int(blockIdx.x) * (PER * kTokens) + int(threadIdx.x) / LPR;
  float x[kTokens][2][8];
#pragma unroll
  for (int u = 0; u < kTokens; ++u) {
    const int t = t0 + u * PER;
    const int64_t slot = t < n_tokens ? slots[t] : -1;
    const bool in = uint64_t(slot) < uint64_t(a.n_slots);
    const Place p = place_of(in ? slot : 0, a);
    const int64_t at = p.page * a.page_stride + head * a.head_stride + int64_t(p.off) * a.token_stride;
    const int64_t word = p.page * a.meta_page_stride + head * a.meta_head_stride + p.off;
#pragma unroll
    for (int v = 0; v < 2; ++v) {
      if (!in) {
#pragma unroll
        for (int j = 0; j < 8; ++j) x[u][v][j] = 0.f;
        continue;
      }
      const uint32_t meta = KIND == FQ_KV_BF16 ? 0u : a.meta[v][word];
      if constexpr (F32) {
        float lo[4], hi[4];
        load_channels<KIND, 4>(a.rows[v] + at, 4 * i, meta, lo);
        load_channels<KIND, 4>(a.rows[v] + at, D / 2 + 4 * i, meta, hi);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          x[u][v][j] = lo[j];
          x[u][v][4 + j] = hi[j];
        }
      } else {
        load_channels<KIND, 8>(a.rows[v] + at, 8 * i, meta, x[u][v]);
      }
    }
  }
#pragma unroll
  for (int u = 0; u < kTokens; ++u) {
    const int t = t0 + u * PER;
    if (t >= n_tokens) return;
    const int64_t at = (int64_t(t) * gridDim.y + head) * D;
#pragma unroll
    for (int v = 0; v < 2; ++v) {
      const float* y = x[u][v];
      if constexpr (F32) {
        float* o = static_cast<float*>(v ? V : K) + at;
        put<STREAM>(o + 4 * i, f32x4_t{y[0], y[1], y[2], y[3]});
        put<STREAM>(o + D / 2 + 4 * i, f32x4_t{y[4], y[5], y[6], y[7]});
      } else {
        uint16_t* o = static_cast<uint16_t*>(v ? V : K) + at;
        put<STREAM>(o + 8 * i, u32x4_t{pack2(y[0], y[1]), pack2(y[2], y[3]), pack2(y[4], y[5]), pack2(y[6], y[7])});
      }
    }
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
  const int per = 256 / (c.head_dim / 8) * kTokens;
  return dim3(unsigned((n_tokens + per - 1) / per), unsigned(c.n_kv_heads));
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
  const bool past = 2 * n_tokens * c.n_kv_heads * c.head_dim * (f32 ? 4 : 2) > kStreamBytes;
  fqk::by_kind(c, [&](auto kind, auto dim) {
    auto go = [&](auto wide, auto streamed) {
      hipLaunchKernelGGL((fqk::kv_read_kernel<kind.value, dim.value, wide.value, streamed.value>),
                         fqk::token_grid(c, n_tokens), dim3(256), 0, static_cast<hipStream_t>(stream), a, slots,
                         int(n_tokens), K, V);
    };
    if (f32 && past) go(std::true_type{}, std::true_type{});
    else if (f32) go(std::true_type{}, std::false_type{});
    else if (past) go(std::false_type{}, std::true_type{});
    else go(std::false_type{}, std::false_type{});
  });
  return int(hipGetLastError());
}

}  // namespace fqi
