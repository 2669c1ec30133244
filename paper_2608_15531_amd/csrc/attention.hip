// Attention of new tokens over a paged KV cache (fq_paged_attention).
//
// Rows.  The query heads that share a KV head see the same keys, so a "row" is one
// (token, query head) of a sequence and a KV head, and the G = n_heads / n_kv_heads
// heads of a token are G neighbouring rows.  A workgroup takes a block of 16 rows of
// one (sequence, KV head) and one range of the keys; its four waves take tiles of 32
// keys in turn and join their results at the end.
//
// Products.  Both run on v_mfma_f32_16x16x32_bf16, as S^T = K Q^T and O^T = V^T P^T, so
// that a lane holds everything of its row (lane & 15): with S^T as the result its 8
// scores of a tile belong to the keys 4 q .. 4 q + 3 and 16 + 4 q .. (q = lane >> 4),
// and those are, packed to bf16, just the 8 k-slots that the lane feeds to the second
// product.  Running maximum, sum, rescaling and output scale need no exchange but the
// maximum over the four lanes of a row.  The order of the k-slots is free as long as
// both operands agree: K rows come from memory 16 bytes a lane, and V, of which an
// operand needs 8 keys of one channel, is read as 8 keys x 8 channels a lane and put
// together by byte permutes, two keys to a register.  Nothing goes through LDS.
//
// Quantised caches.  A code c becomes a bf16 exactly (4 bits: 16 + c by one and-or, the
// smallest offset that takes no more; 8 bits: through fp32), and the affine map is applied
// to the sums:
//     q . k = s_k (sum q c - z_k sum q),   sum p v = sum p' c - sum p' z_v,
//     p' = bf16(p s_v).
// The offset's own sums cancel in fp32: with 128 + c, a bf16's last bits, the log-sum over
// three keys was off by 5e-7 of itself, with 16 + c by what it is off in bf16.
//
// The weights (times s_v) of the second product are bf16, as its operand: in fp32 each would
// take two.  They move a row by up to 2^-8 sum w |v|; statistics and sums are fp32.
//
// Memory bounds it: 64 sequences of 100 to 8190 keys at 8 bits take 130 us, 4.3 TB/s, and
// 16 of 24000 to 32767 at 4 bits, 64 heads, 101 us, 4.9 TB/s (a copy: 5.1).  One token over
// 1000 keys takes 8 us, which is latency.  16 rows and no LDS keep four waves a SIMD under
// way; loads for the next tile in further registers cost a third of them, and 107 became
// 120 us for the 16 sequences.
#include <algorithm>

#include "attention.hpp"

namespace fqk {

namespace {

// Maximum and sum over the four lanes of a row (lanes l, l ^ 16, l ^ 32, l ^ 48).
__device__ __forceinline__ float row_max(float v) { return across32(across16(v, Max{}), Max{}); }
__device__ __forceinline__ float row_add(float v) { return across32(across16(v, Add{}), Add{}); }

// Channels of the lane's 8 k-slots in product step `st` of S^T: the first of them.
// They follow from the 16 (or 8) bytes of a K row that a lane loads at once.
template <int KIND, int D>
__device__ __forceinline__ int q_channel(int st, int q) {
  if constexpr (KIND == FQ_KV_BF16) return st * 32 + q * 8;
  else if constexpr (KIND == FQ_KV_INT8) return (st >> 1) * 64 + q * 16 + (st & 1) * 8;
  else return q * (D / 4) + st * 8;
}

// Codes i and 4 + i of a word of eight as the bf16 pair 16 + c.
constexpr uint32_t kSixteens = 0x41804180u;
__device__ __forceinline__ uint32_t codes_plus_16(uint32_t w, int i) {
  return and_or(i == 0 ? w << 3 : w >> (4 * i - 3), 0x00780078u, kSixteens);
}

// One K row's share of a lane: the codes or bf16 of all its k-slots.
template <int KIND, int D>
struct KRow {
  static constexpr int W = KIND == FQ_KV_BF16 ? D / 8 : KIND == FQ_KV_INT8 ? D / 16 : D / 32;
  uint32_t w[W];
  __device__ __forceinline__ void load(const char* row, int q) {
    if constexpr (W >= 4) {
#pragma unroll
      for (int i = 0; i < W / 4; ++i) {
        const uint4 x = *reinterpret_cast<const uint4*>(row + i * 64 + q * 16);
        w[4 * i] = x.x;
        w[4 * i + 1] = x.y;
        w[4 * i + 2] = x.z;
        w[4 * i + 3] = x.w;
      }
    } else {
      const uint2 x = *reinterpret_cast<const uint2*>(row + q * 8);
      w[0] = x.x;
      w[1] = x.y;
    }
  }
  __device__ __forceinline__ bf16x8_t operand(int st) const {
    u32x4_t r;
    if constexpr (KIND == FQ_KV_BF16) {
      r = u32x4_t{w[4 * st], w[4 * st + 1], w[4 * st + 2], w[4 * st + 3]};
    } else if constexpr (KIND == FQ_KV_INT8) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint32_t c = w[2 * st + i / 2] >> (16 * (i & 1));
        r[i] = __builtin_amdgcn_perm(__builtin_bit_cast(uint32_t, float((c >> 8) & 255u)),
                                     __builtin_bit_cast(uint32_t, float(c & 255u)), 0x07060302u);
      }
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) r[i] = codes_plus_16(w[st], i);
    }
    return __builtin_bit_cast(bf16x8_t, r);
  }
};

// Eight V rows' share of a lane: D / 16 channels from (lane & 15) * D / 16 on.
template <int KIND, int D>
struct VRows {
  static constexpr int C = D / 16;   // channels a lane = 16-channel blocks of O^T
  static constexpr int BYTES = KIND == FQ_KV_BF16 ? 2 * C : KIND == FQ_KV_INT8 ? C : C / 2;
  static constexpr int W = (BYTES + 3) / 4;
  uint32_t w[8][W];
  __device__ __forceinline__ void load(int j, const char* row, int c16) {
    const char* p = row + c16 * BYTES;
    if constexpr (BYTES == 16) {
      const uint4 x = *reinterpret_cast<const uint4*>(p);
      w[j][0] = x.x;
      w[j][1] = x.y;
      w[j][2] = x.z;
      w[j][3] = x.w;
    } else if constexpr (BYTES == 8) {
      const uint2 x = *reinterpret_cast<const uint2*>(p);
      w[j][0] = x.x;
      w[j][1] = x.y;
    } else if constexpr (BYTES == 4) {
      w[j][0] = *reinterpret_cast<const uint32_t*>(p);
    } else {
      w[j][0] = *reinterpret_cast<const uint16_t*>(p);
    }
  }
  // The A operand of channel block c: two keys to a register.
  __device__ __forceinline__ bf16x8_t operand(int c) const {
    u32x4_t r;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t* a = w[2 * i];
      const uint32_t* b = w[2 * i + 1];
      if constexpr (KIND == FQ_KV_BF16) {
        r[i] = __builtin_amdgcn_perm(b[c / 2], a[c / 2], (c & 1) ? 0x07060302u : 0x05040100u);
      } else if constexpr (KIND == FQ_KV_INT8) {
        const uint32_t x = (a[c / 4] >> (8 * (c & 3))) & 255u, y = (b[c / 4] >> (8 * (c & 3))) & 255u;
        r[i] = __builtin_amdgcn_perm(__builtin_bit_cast(uint32_t, float(y)), __builtin_bit_cast(uint32_t, float(x)),
                                     0x07060302u);
      } else {
        const uint32_t t = __builtin_amdgcn_perm(b[0], a[0], c < 4 ? 0x05040100u : 0x07060302u);
        r[i] = codes_plus_16(t, c & 3);
      }
    }
    return __builtin_bit_cast(bf16x8_t, r);
  }
};

constexpr int kWaves = 4;

constexpr int kMaxSplit = 128;   // ranges

// LDS: the waves' sums [kWaves][16][D + 4], then their maxima and row sums; for the join of
// the ranges their maxima and row sums [2][16][kMaxSplit] and 16 rows of sums instead.
template <int D>
constexpr size_t kAttnLds = std::max((size_t(kWaves) * 16 * (D + 4) + 2 * kWaves * 16) * 4,
                                     (size_t(2) * 16 * kMaxSplit + 16 * D) * 4);

template <int KIND, int D>
__global__ void __launch_bounds__(64 * kWaves, 4) attn_rows_kernel(AttnArgs a) {
  constexpr int STEPS = D / 32, CB = D / 16;
  extern __shared__ __attribute__((aligned(16))) float lds[];
  __shared__ uint32_t last_flag;
  float* l_acc = lds;
  float* l_max = lds + kWaves * 16 * (D + 4);
  float* l_sum = l_max + kWaves * 16;
  const int tid = int(threadIdx.x), lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int r16 = lane & 15, q = lane >> 4;

  Item it;
  if (!it.set<16, kKvTile>(a)) return;
  Row mine;
  mine.set(a, it, r16);
  // softmax in powers of two of |scale|; a negative scale changes the sign of q, 0 makes it 0
  const uint32_t q_sign = a.scale_log2 < 0.f ? 0x80008000u : 0u;
  const float c2 = a.scale_log2 == 0.f ? 1.f : fabsf(a.scale_log2);
  const float grow = grow_of(c2);
  const bool use_q = mine.in && a.scale_log2 != 0.f;
  const uint16_t* qp = a.Q + (it.t0 + mine.token) * a.q_token + mine.head * a.q_head;
  bf16x8_t qv[STEPS];
  float q_sum = 0.f;
#pragma unroll
  for (int st = 0; st < STEPS; ++st) {
    uint4 w{0, 0, 0, 0};
    if (use_q) w = *reinterpret_cast<const uint4*>(qp + q_channel<KIND, D>(st, q));
    w = uint4{w.x ^ q_sign, w.y ^ q_sign, w.z ^ q_sign, w.w ^ q_sign};
    if constexpr (KIND != FQ_KV_BF16) {
      const uint32_t ws[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
      for (int i = 0; i < 4; ++i)
        q_sum += bf16_bits_to_f32(ws[i]) + __builtin_bit_cast(float, ws[i] & 0xFFFF0000u);
    }
    if constexpr (KIND == FQ_KV_INT4) w = permute_chunk(w);
    qv[st] = __builtin_bit_cast(bf16x8_t, w);
  }
  if constexpr (KIND != FQ_KV_BF16) q_sum = row_add(q_sum);
  // the offset of the codes is taken off where the products of K start from
  const float from = KIND == FQ_KV_INT4 ? -16.f * q_sum : 0.f;
  const f32x4_t d0{from, from, from, from};

  f32x4_t acc[CB];
#pragma unroll
  for (int c = 0; c < CB; ++c) acc[c] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  float m = kNegInf, l = 0.f, corr = 0.f;
  bool odd = false;   // V had infinities or NaN in a tile that is not seen whole

  const int32_t* table = a.table + it.seq * a.table_stride;
  const char* kh = a.k + it.head * a.head_stride;
  const char* vh = a.v + it.head * a.head_stride;
  const uint32_t* kmh = KIND == FQ_KV_BF16 ? nullptr : a.k_meta + it.head * a.meta_head_stride;
  const uint32_t* vmh = KIND == FQ_KV_BF16 ? nullptr : a.v_meta + it.head * a.meta_head_stride;

  for (int i = it.i_lo + wave; i < it.i_hi; i += kWaves) {
    const int key0 = it.tr.tile(i) * kKvTile;
    KRow<KIND, D> kr[2];
    VRows<KIND, D> vr;
    uint4 km[2], vm[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      // a block past the last key is masked: any page in range will do
      const int key = key0 + h * kKvBlock;
      const BlockPlace at = block_place(a, table, key < it.kv_seen ? key : key0);
      const char* kb = kh + at.page * a.page_stride + at.token * int64_t(a.token_stride);
      const char* vb = vh + at.page * a.page_stride + at.token * int64_t(a.token_stride);
      kr[h].load(kb + uint32_t(r16) * a.token_stride, q);
#pragma unroll
      for (int j = 0; j < 4; ++j) vr.load(4 * h + j, vb + uint32_t(4 * q + j) * a.token_stride, r16);
      if constexpr (KIND != FQ_KV_BF16) {
        km[h] = *reinterpret_cast<const uint4*>(kmh + at.page * a.meta_page_stride + at.token + 4 * q);
        vm[h] = *reinterpret_cast<const uint4*>(vmh + at.page * a.meta_page_stride + at.token + 4 * q);
      }
    }
    // scores
    float s[8];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      f32x4_t d = d0;
#pragma unroll
      for (int st = 0; st < STEPS; ++st) d = mfma16(kr[h].operand(st), qv[st], d);
      const uint32_t kmw[4] = {km[h].x, km[h].y, km[h].z, km[h].w};
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        if constexpr (KIND == FQ_KV_BF16) s[4 * h + j] = d[j];
        else s[4 * h + j] = fmaf(-__builtin_bit_cast(float, kmw[j] & 0xFFFF0000u), q_sum, d[j]) * bf16_bits_to_f32(kmw[j]);
      }
    }
    // the mask, where the tile is not seen whole by every row; a key that is not seen counts
    // nothing, whatever its scale and zero-point
    const bool whole = it.whole<kKvTile>(a, key0);
    uint32_t vmw[8] = {vm[0].x, vm[0].y, vm[0].z, vm[0].w, vm[1].x, vm[1].y, vm[1].z, vm[1].w};
    if (!whole) {
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const bool see = mine.sees(a, key0 + (j >> 2) * kKvBlock + 4 * q + (j & 3));
        s[j] = see ? s[j] : kNegInf;
        if constexpr (KIND != FQ_KV_BF16) vmw[j] = see ? vmw[j] : 0u;
      }
    }
    float top = s[0];
#pragma unroll
    for (int j = 1; j < 8; ++j) top = fmaxf(top, s[j]);
    top = row_max(top);
    // the sums move to a new maximum only when some row's has grown by more than 2^8: until
    // then its weights are up to 2^8, which fp32 sums and bf16 weights hold as well
    if (__any(top > m + grow)) {
      const float m_new = fmaxf(m, top);
      const float shrink = __builtin_amdgcn_exp2f((m - (m_new == kNegInf ? 0.f : m_new)) * c2);
      m = m_new;
      l *= shrink;
      corr *= shrink;
#pragma unroll
      for (int c = 0; c < CB; ++c) acc[c] *= shrink;
    }
    const float base = m == kNegInf ? 0.f : -m * c2;
    float p[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      p[j] = __builtin_amdgcn_exp2f(fmaf(s[j], c2, base));
      l += p[j];
      if constexpr (KIND != FQ_KV_BF16) p[j] *= bf16_bits_to_f32(vmw[j]);
    }
    u32x4_t pw;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      pw[e] = pk_bf16(p[2 * e], p[2 * e + 1]);
      if constexpr (KIND != FQ_KV_BF16) {
        const uint32_t w = pw[e];
        corr = dot2_bf16(w, __builtin_amdgcn_perm(vmw[2 * e + 1], vmw[2 * e], 0x07060302u), corr);
        if constexpr (KIND == FQ_KV_INT4) corr = dot2_bf16(w, kSixteens, corr);   // the offset
      }
    }
    if constexpr (KIND == FQ_KV_BF16) {
      if (!whole) {
        bool any = false;
#pragma unroll
        for (int j = 0; j < 8; ++j)
#pragma unroll
          for (int w = 0; w < VRows<KIND, D>::W; ++w) {
            any |= nonfinite_pair(vr.w[j][w]);
            vr.w[j][w] = finite_pair(vr.w[j][w]);
          }
        odd |= __any(any);
      }
    }
    const bf16x8_t pb = __builtin_bit_cast(bf16x8_t, pw);
#pragma unroll
    for (int c = 0; c < CB; ++c) acc[c] = mfma16(vr.operand(c), pb, acc[c]);
  }
  if constexpr (KIND == FQ_KV_BF16) {
    if (odd) {
      walk_partial_tiles<kKvTile>(a, it, table, vh, it.i_lo + wave, kWaves, [&](int key, const uint16_t* v) {
        if (!mine.in || !mine.sees(a, key)) return;
#pragma unroll
        for (int c = 0; c < CB; ++c)
#pragma unroll
          for (int i = 0; i < 4; ++i) acc[c][i] += if_nonfinite(v[(4 * q + i) * CB + c]);
      });
    }
  }

  // join the waves: lane (r16, q) has channels (4 q + i) CB + c of row r16
  m *= c2;
  l = row_add(l);
  if constexpr (KIND != FQ_KV_BF16) corr = row_add(corr);
  {
    float* dst = l_acc + (wave * 16 + r16) * (D + 4) + 4 * q * CB;
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int c = 0; c < CB; c += 4)
        *reinterpret_cast<f32x4_t*>(dst + i * CB + c) =
            f32x4_t{acc[c][i] - corr, acc[c + 1][i] - corr, acc[c + 2][i] - corr, acc[c + 3][i] - corr};
    if (q == 0) {
      l_max[wave * 16 + r16] = m;
      l_sum[wave * 16 + r16] = l;
    }
  }
  __syncthreads();
  // thread (row, channels ch .. ch + CB - 1)
  const int row = tid >> 4, ch = (tid & 15) * CB;
  float o[CB], mx = kNegInf, sum = 0.f;
#pragma unroll
  for (int c = 0; c < CB; ++c) o[c] = 0.f;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) mx = fmaxf(mx, l_max[w * 16 + row]);
  const float base = mx == kNegInf ? 0.f : mx;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) {
    // (a NaN maximum cannot be: fmaxf drops it; the sum then is NaN)
    const float f = __builtin_amdgcn_exp2f(l_max[w * 16 + row] - base);
    sum = fmaf(f, l_sum[w * 16 + row], sum);
    const float* src = l_acc + (w * 16 + row) * (D + 4) + ch;
#pragma unroll
    for (int c = 0; c < CB; ++c) o[c] = fmaf(f, src[c], o[c]);
  }

  if (it.n_parts > 1) {
    // partial sums: [item][range][row][D] floats, then [item][range][row][2]
    const int64_t item = it.number;
    const uint32_t part_words = uint32_t(a.part_rows) * (D + 4);
    float* base_p = a.partials + item * a.split * part_words;
    const __amdgpu_buffer_rsrc_t prs = make_rsrc(base_p, uint32_t(a.split) * part_words * 4u);
    if (row < it.rows) {
      const uint32_t at = (uint32_t(it.part) * part_words + uint32_t(row) * (D + 4)) * 4u;
#pragma unroll
      for (int c = 0; c < CB; c += 4)
        __builtin_amdgcn_raw_buffer_store_b128(
            __builtin_bit_cast(u32x4_t, f32x4_t{o[c], o[c + 1], o[c + 2], o[c + 3]}), prs, int(at + (ch + c) * 4u), 0, kSc1);
      if ((tid & 15) == 0)
        __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4_t, f32x4_t{mx, sum, 0.f, 0.f}), prs,
                                               int(at + D * 4u), 0, kSc1);
    }
    __builtin_amdgcn_s_waitcnt(0);   // this thread's partial stores have completed
    __syncthreads();
    if (tid == 0) {
      const uint32_t old = __hip_atomic_fetch_add(a.counters + item, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      last_flag = old == uint32_t(it.n_parts - 1);
    }
    __syncthreads();
    if (!last_flag) return;
    if (tid == 0) __hip_atomic_store(a.counters + item, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    // The last to arrive adds the ranges.  A trip to memory costs more than a range's sums
    // are worth, so few trips: the 16-thread groups that have no row of their own share the
    // ranges with those that do, all maxima are read at once and the sums eight at a time.
    // Every sum has a fixed order.
    const int p2 = it.rows <= 1 ? 1 : it.rows <= 2 ? 2 : it.rows <= 4 ? 4 : it.rows <= 8 ? 8 : 16;
    const int groups = 16 / p2, g = (tid >> 4) / p2, grow = (tid >> 4) % p2, i16 = tid & 15;
    const uint32_t row_at = uint32_t(min(grow, it.rows - 1)) * (D + 4) * 4u;
    float* weight = lds + grow * kMaxSplit;
    float* sums = lds + (16 + grow) * kMaxSplit;
    float* shared_o = lds + 2 * 16 * kMaxSplit;   // [groups][p2][D]
    {
      f32x4_t ms[kMaxSplit / 16];
#pragma unroll
      for (int j = 0; j < kMaxSplit / 16; ++j) {
        const int s2 = (j * groups + g) * 16 + i16;
        if (j * groups * 16 < it.n_parts)
          ms[j] = __builtin_bit_cast(f32x4_t, __builtin_amdgcn_raw_buffer_load_b128(
              prs, int(uint32_t(min(s2, it.n_parts - 1)) * part_words * 4u + row_at + D * 4u), 0, kSc1));
      }
#pragma unroll
      for (int j = 0; j < kMaxSplit / 16; ++j) {
        const int s2 = (j * groups + g) * 16 + i16;
        if (s2 < it.n_parts) {
          weight[s2] = ms[j][0];
          sums[s2] = ms[j][1];
        }
      }
    }
    __syncthreads();
    float top = kNegInf;
    for (int s2 = i16; s2 < it.n_parts; s2 += 16) top = fmaxf(top, weight[s2]);
    mx = over_lanes<16>(top, Max{});
    const float b2 = mx == kNegInf ? 0.f : mx;
    sum = 0.f;
    for (int s2 = i16; s2 < it.n_parts; s2 += 16) sum = fmaf(__builtin_amdgcn_exp2f(weight[s2] - b2), sums[s2], sum);
    sum = over_lanes<16>(sum, Add{});
#pragma unroll
    for (int c = 0; c < CB; ++c) o[c] = 0.f;
    for (int s0 = g; s0 < it.n_parts; s0 += 8 * groups) {
      u32x4_t v[8][CB / 4];
#pragma unroll
      for (int j = 0; j < 8; ++j)
#pragma unroll
        for (int c = 0; c < CB / 4; ++c)   // in range; surplus loads unused
          v[j][c] = __builtin_amdgcn_raw_buffer_load_b128(
              prs, int(uint32_t(min(s0 + j * groups, it.n_parts - 1)) * part_words * 4u + row_at + (ch + 4 * c) * 4u), 0, kSc1);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        if (s0 + j * groups >= it.n_parts) break;
        const float f = __builtin_amdgcn_exp2f(weight[s0 + j * groups] - b2);
#pragma unroll
        for (int c = 0; c < CB / 4; ++c) {
          const f32x4_t x = __builtin_bit_cast(f32x4_t, v[j][c]);
#pragma unroll
          for (int e = 0; e < 4; ++e) o[4 * c + e] = fmaf(f, x[e], o[4 * c + e]);
        }
      }
    }
    if (groups > 1) {
#pragma unroll
      for (int c = 0; c < CB; c += 4)
        *reinterpret_cast<f32x4_t*>(shared_o + (g * p2 + grow) * D + ch + c) = f32x4_t{o[c], o[c + 1], o[c + 2], o[c + 3]};
      __syncthreads();
      if (g > 0 || grow >= it.rows) return;
      for (int g2 = 1; g2 < groups; ++g2)
#pragma unroll
        for (int c = 0; c < CB; ++c) o[c] += shared_o[(g2 * p2 + grow) * D + ch + c];
    }
  }
  if (row >= it.rows) return;
  Row dst;
  dst.set(a, it, row);
  const float inv = sum == 0.f ? 0.f : 1.f / sum;
  uint16_t* op = a.O + (it.t0 + dst.token) * a.o_token + dst.head * a.o_head + ch;
  uint32_t w[CB / 2];
#pragma unroll
  for (int c = 0; c < CB; c += 2)
    w[c / 2] = sum == 0.f ? 0u : pk_bf16(o[c] * inv, o[c + 1] * inv);
  if constexpr (CB == 8) *reinterpret_cast<uint4*>(op) = uint4{w[0], w[1], w[2], w[3]};
  else *reinterpret_cast<uint2*>(op) = uint2{w[0], w[1]};
  if (a.lse && (tid & 15) == 0)
    a.lse[(it.t0 + dst.token) * a.n_heads + dst.head] = sum == 0.f ? kNegInf : (mx + __log2f(sum)) * 0.69314718055994530942f;
}

}  // namespace

}  // namespace fqk

namespace fqi {

namespace {

// The kernel for few rows splits the keys until there are two workgroups to a CU, into
// ranges of 128 keys (a tile a wave) at least.  Beyond that it makes eight ranges of the
// longest sequence, of 768 to 4096 keys, which evens out sequences of different lengths.
constexpr int kTargetWorkgroups = 512;
constexpr int kMinSplitTiles = 4;
constexpr int kEvenRanges = 8, kEvenMinTiles = 24, kEvenMaxTiles = 128;
// The kernel for few rows reads the keys once for each block of 16 rows, the one for many
// once for 128, at a longer start and with a second kernel for the join.  By measurement
// (us, few / many), with what the blocks of 16 rows read in all: 40 tokens of 4 heads a
// group over 540 keys, bf16, 22 MB: 10 / 18; 16 over 8000, bf16, 131 MB: 25 / 23; 300 over
// 600, bf16, 184 MB: 19 / 27; 10 over 2000, 16 sequences, 8 bits, 204 MB: 38 / 44; 16 over
// 4000, 8 sequences, 8 bits, 271 MB: 46 / 46; 20 over 2000, 8 sequences, bf16, 331 MB: 35 / 27.
constexpr int64_t kFewRowsBytes = int64_t(224) << 20;
// The kernel for many rows has two workgroups to a CU; it splits the keys where that makes
// rounds * (tiles of a range + kRangeCost) + bytes of the partial sums / kTileBytes smaller:
// a range's start and its part in the join are worth so many tiles, and in a tile's time, 2.3
// us, that many bytes are written and read again.
// (Up to 2048 ranges: with more of them, not all of the longest sequence's length, the rounds
// say little.  With 4096 20 to 900 tokens of 8 sequences over 500 to 8000 keys went from 534 to
// 673 us, but 2000, 10 and 100 over 0, 8000 and 20000, 4 bits, 64 heads, from 693 to 508.)
constexpr int kTileSlots = 512;
constexpr int kRangeCost = 4;
constexpr int kRoundsRanges = 2048;
constexpr int64_t kTileBytes = int64_t(5) << 20;
// Of several sequences one may be much longer than the others, and its ranges then are what
// takes long: they have 10240 keys at most.  (us, without / with: 2000, 10 and 100 tokens over
// 0, 8000 and 20000 keys, 4 bits, 64 heads: 979 / 693; 5 to 300 of 6 sequences over 500 to
// 30000, 8 bits: 693 both; but equal ones are split too, 4 times 1024 over 16000, 8 bits: 1579
// / 1637.  With 4096 keys the first took 509, but 20 to 900 tokens of 8 sequences over 500 to
// 8000 564 instead of 534, and the second 764.)
constexpr int64_t kEvenTiles = 160;
// Partial results are bounded: 4096 ranges of 128 rows are 277 MB, 8192 of 16 rows 69.
constexpr int64_t kMostTileRanges = 4096, kMostRanges = 8192;
// Workgroups of 256 threads in one dimension of a grid: HIP takes fewer than 2^32 threads.
constexpr int64_t kMostGrid = (int64_t(1) << 24) - 1;

// Keys are numbered below 2^28, so a wider window sees the same ones; positions before the
// first key less the window stay in 32 bits.
constexpr int kWidestWindow = 1 << 30;

int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

}  // namespace

bool plan_attention(const fq_attention& a, const fq_kv_cache& c, AttnPlan* pl) {
  const int64_t group = a.n_heads / c.n_kv_heads;
  const int64_t rows = a.max_q * group;
  const int64_t key_bytes = c.kind == FQ_KV_BF16 ? 4 * c.head_dim : c.kind == FQ_KV_INT8 ? 2 * c.head_dim + 8
                                                                                        : c.head_dim + 8;
  const int64_t seen_keys = a.window > 0 ? std::min<int64_t>(a.max_kv, int64_t(a.window) + a.sinks + a.max_q) : a.max_kv;
  const bool few = rows <= 32 || ceil_div(rows, 16) * a.n_seqs * c.n_kv_heads <= kFewRowsBytes / (seen_keys * key_bytes);
  pl->kernel = few ? FQ_ATTN_ROWS : FQ_ATTN_TILES;
  pl->rows = pl->kernel == FQ_ATTN_TILES ? kTilesRows : 16;
  pl->tile = pl->kernel == FQ_ATTN_TILES ? kTilesKeys : kKvTile;
  const int64_t row_blocks = ceil_div(rows, pl->rows);
  if (row_blocks > (1 << 24) || a.n_seqs > 65535) return false;
  pl->row_blocks = int(row_blocks);
  const int64_t grid = row_blocks * c.n_kv_heads * a.n_seqs;
  // Of those, the ones that can hold rows: in the kernel for many rows sequences of very
  // different lengths are common.  (The one for few keeps a counter for each by its place in
  // the grid, which no content of cu_q can make two blocks share.)
  int64_t blocks = row_blocks * a.n_seqs;
  pl->dense_blocks = 0;
  if (pl->kernel == FQ_ATTN_TILES && a.total_q / pl->rows < blocks) {
    const int64_t dense = dense_blocks(a.total_q, group, pl->rows, a.n_seqs);
    if (dense < blocks) {
      blocks = dense;
      pl->dense_blocks = 1;
    }
  }
  const int64_t items = blocks * c.n_kv_heads;
  // tiles that a block of rows can see at most: those of the first keys, and a window of
  // every token of the block, at any place
  int64_t tiles = ceil_div(a.max_kv, pl->tile);
  if (a.window > 0)
    tiles = std::min<int64_t>(tiles, ceil_div(a.window + ceil_div(pl->rows, group), pl->tile) + 2 +
                                         ceil_div(a.sinks, pl->tile));
  int64_t split = 1;
  // every item has a counter, and the ranges and their join a grid
  const int64_t most_split = kMostGrid / std::max<int64_t>(row_blocks * c.n_kv_heads, 1);
  if (items <= kMaxStrips && most_split >= fqk::kJoinBlocks) {
    if (pl->kernel == FQ_ATTN_TILES) {
      const int64_t range_bytes = std::min<int64_t>(pl->rows, rows) * (c.head_dim + 4) * 4;
      const auto cost = [&](int64_t n) {
        return ceil_div(items * n, kTileSlots) * (ceil_div(tiles, n) + kRangeCost) +
               (n > 1 ? items * n * range_bytes / kTileBytes : 0);
      };
      if (a.n_seqs > 1) split = std::max<int64_t>(1, std::min(ceil_div(tiles, kEvenTiles), kMostTileRanges / items));
      for (int64_t n = split + 1; n <= std::min<int64_t>(tiles / 2, 64) && items * n <= kRoundsRanges; ++n)
        if (cost(n) < cost(split)) split = n;
    } else {
      if (items < kTargetWorkgroups)
        split = std::max<int64_t>(1, std::min(ceil_div(kTargetWorkgroups, items), tiles / kMinSplitTiles));
      split = std::min<int64_t>(
          std::max(split, ceil_div(tiles, std::clamp<int64_t>(tiles / kEvenRanges, kEvenMinTiles, kEvenMaxTiles))),
          std::min<int64_t>(fqk::kMaxSplit, std::max<int64_t>(1, kMostRanges / items)));
    }
    split = std::min(split, most_split);
  }
  pl->split_tiles = int(ceil_div(tiles, split));
  pl->split = int(ceil_div(tiles, pl->split_tiles));
  if (pl->split * row_blocks * c.n_kv_heads > kMostGrid) return false;
  pl->workgroups = grid * pl->split;
  if (pl->workgroups > INT32_MAX) return false;
  if (pl->kernel == FQ_ATTN_TILES) pl->lds_bytes = fqk::attn_tiles_lds(c.head_dim);
  else pl->lds_bytes = c.head_dim == 64 ? fqk::kAttnLds<64> : fqk::kAttnLds<128>;
  pl->part_rows = int(std::min<int64_t>(pl->rows, rows));
  pl->partial_bytes = pl->split > 1 ? size_t(items) * pl->split * pl->part_rows * (c.head_dim + 4) * 4 : 0;
  pl->ws_bytes = kCounterRegion + pl->partial_bytes;
  return true;
}

int launch_attention(const AttnPlan& pl, const fq_attention& a, const fq_kv_cache& c,
                     const uint16_t* Q, const int32_t* cu_q, const int32_t* kv_lens,
                     const int32_t* table, uint16_t* O, float* lse, void* workspace,
                     void* stream) {
  const int group = a.n_heads / c.n_kv_heads;
  fqk::AttnArgs g{};
  g.Q = Q;
  g.k = static_cast<const char*>(c.k);
  g.v = static_cast<const char*>(c.v);
  g.k_meta = static_cast<const uint32_t*>(c.k_meta);
  g.v_meta = static_cast<const uint32_t*>(c.v_meta);
  g.cu_q = cu_q;
  g.kv_lens = kv_lens;
  g.table = table;
  g.O = O;
  g.lse = lse;
  g.counters = static_cast<uint32_t*>(workspace);
  g.partials = reinterpret_cast<float*>(static_cast<char*>(workspace) + kCounterRegion);
  g.page_stride = c.page_stride;
  g.head_stride = c.head_stride;
  g.meta_page_stride = c.meta_page_stride;
  g.meta_head_stride = c.meta_head_stride;
  g.table_stride = a.table_stride;
  g.q_token = a.q_token_stride;
  g.q_head = a.q_head_stride;
  g.o_token = a.o_token_stride;
  g.o_head = a.o_head_stride;
  g.total_q = a.total_q;
  g.token_stride = uint32_t(c.token_stride);
  g.page_blocks = uint32_t(c.page_size / kKvBlock);
  g.page_magic = ((uint64_t(1) << 36) + g.page_blocks - 1) / g.page_blocks;
  g.n_pages = uint32_t(c.n_pages);
  g.group = group;
  g.n_heads = a.n_heads;
  g.n_kv_heads = c.n_kv_heads;
  g.max_q = a.max_q;
  g.max_kv = a.max_kv;
  g.window = std::min(a.window, kWidestWindow);
  g.sinks = a.sinks;
  g.row_blocks = pl.row_blocks;
  g.split = pl.split;
  g.split_tiles = pl.split_tiles;
  g.part_rows = pl.part_rows;
  g.dense_blocks = pl.dense_blocks;
  g.scale_log2 = a.scale * kLog2e;
  const dim3 grid(unsigned(int64_t(pl.row_blocks) * pl.split * c.n_kv_heads), unsigned(a.n_seqs));
  const hipStream_t s = static_cast<hipStream_t>(stream);
  if (pl.kernel == FQ_ATTN_TILES) return fqk::launch_attn_tiles(g, c.kind, c.head_dim, grid, s);
  auto go = [&](auto kind) {
    if (c.head_dim == 64)
      hipLaunchKernelGGL((fqk::attn_rows_kernel<kind.value, 64>), grid, dim3(64 * fqk::kWaves), pl.lds_bytes, s, g);
    else
      hipLaunchKernelGGL((fqk::attn_rows_kernel<kind.value, 128>), grid, dim3(64 * fqk::kWaves), pl.lds_bytes, s, g);
  };
  if (c.kind == FQ_KV_BF16) go(std::integral_constant<int, FQ_KV_BF16>{});
  else if (c.kind == FQ_KV_INT8) go(std::integral_constant<int, FQ_KV_INT8>{});
  else go(std::integral_constant<int, FQ_KV_INT4>{});
  return int(hipGetLastError());
}

}  // namespace fqi
