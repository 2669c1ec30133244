// Attention over a paged cache for many rows of a sequence (prompts and their chunks):
// the keys go through LDS once for 128 rows.
//
// A workgroup has 128 rows of one (sequence, KV head), 32 a wave, and walks over tiles of
// 64 keys.  Products are v_mfma_f32_32x32x16_bf16 as S^T = K Q^T and O^T = V^T P^T: lane l
// holds 32 of the 64 scores of row l & 31 of its wave, in the order in which the second
// product takes them as weights, so only the row's maximum crosses lanes (l and l ^ 32).
//
// LDS has a tile of K and one of V as they lie in the cache, rows of channels in bf16; the
// 16-byte chunks of a row are permuted by the row's number, so that the operand reads
// spread over the banks: K's take the same chunk of 32 rows, V's, of which an operand needs
// 8 keys of one channel, are transposing reads (ds_read_b64_tr_b16: 4 rows x 16 channels
// by 16 lanes).  bf16 rows go from memory straight to LDS, without a register.  Two tiles:
// the next one is under way during a tile's products.
//
// Quantised caches: the codes become bf16 on the way into LDS, exactly, and the affine map is
// applied to the sums in fp32, as in the kernel for few rows, so that any zero-point counts
// as it is (c - z of one above 255 or not whole does not fit a bf16):
//     q . k = s_k (sum q c - z_k sum q),   sum p v = sum p' c - sum p' z_v,   p' = bf16(p s_v).
// z_k sum q is one more product a 32 keys, with sum q as three bf16 that together are the
// fp32 number (700 tokens over 2700 keys, 8 bits: 92 us; as 32 multiply-adds 95; 88 with
// c - z formed in LDS, which holds whole z up to 255 only).
//
// The weights of the second product are bf16, as its operand (in fp32 each would take two and
// the product twice as long); they are what a row's error is beyond its own rounding, up to
// 2^-8 sum w |v|.  Statistics and sums are fp32.
//
// 2048 tokens over 8192 keys, 32 heads on 8, D = 128, bf16: 264 to 274 us, 880 to 912
// TFLOP/s (a product of 8192^3, both operands along k: 1630).  The matrix cores are busy 39 %
// of the time: a wave's tile takes 32 products, about 1000 cycles, and about 200 vector
// instructions, 32 of them exponentials at a quarter of the rate, about 1200 more, and by
// these numbers the one hardly runs beside the other.  One barrier a tile keeps the waves of
// a workgroup in the same phase, nothing holds the two workgroups of a CU in opposite ones,
// and 256 registers leave no room to compute one tile's scores beside another's softmax
// (374 us, with spills).  256 rows a workgroup: 300 us.
#include "attention.hpp"

namespace fqk {

namespace {

typedef float f32x16_t __attribute__((__vector_size__(16 * sizeof(float))));

constexpr int kTile = fqi::kTilesKeys;     // keys
constexpr int kRows = fqi::kTilesRows;
constexpr int kTileWaves = 4;
static_assert(kTile == 64 && kRows == 32 * kTileWaves, "layout of the tiles");

__device__ __forceinline__ f32x16_t mfma32(bf16x8_t a, bf16x8_t b, f32x16_t c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
}

// Maximum and sum over lanes l and l ^ 32.
__device__ __forceinline__ float pair_max(float v) { return across32(v, Max{}); }
__device__ __forceinline__ float pair_add(float v) { return across32(v, Add{}); }

__device__ __forceinline__ float upper_bf16(float v) {
  return __builtin_bit_cast(float, __builtin_bit_cast(uint32_t, v) & 0xFFFF0000u);
}

// Two f32 whose upper halves are exact bf16, as a pair.
__device__ __forceinline__ uint32_t pack_exact(float lo, float hi) {
  return __builtin_amdgcn_perm(__builtin_bit_cast(uint32_t, hi), __builtin_bit_cast(uint32_t, lo), 0x07060302u);
}

template <int D>
struct TileLds {
  static constexpr int K = kTile * D * 2, V = K;
  static constexpr int kv = K + V;
  static constexpr int meta = kTile * 4;            // of K, then of V: bf16 s | bf16 z << 16
  static constexpr int one = kv + 2 * meta;
  static constexpr int bytes = 2 * one;
};

// The permutation of a row's chunks (8 channels): chunk c of row r lies at place
// c ^ swizzle(r).  Sixteen rows in a row differ in it (128 channels; with 64, rows that
// start in the same half of the banks), and of 4 rows' neighbouring 4 chunks each none
// share a place.
template <int D>
__device__ __forceinline__ int swizzle(int r) {
  return D == 128 ? ((r & 3) << 2 | ((r >> 2) & 3)) : ((r & 2) << 1 | ((r >> 2) & 3));
}

// A thread's share of a tile: the same pieces of K and V.
template <int KIND, int D>
struct Share {
  static constexpr int RB = KIND == FQ_KV_BF16 ? 2 * D : KIND == FQ_KV_INT8 ? D : D / 2;   // bytes a row
  static constexpr int PB = RB / 4 < 16 ? RB / 4 : 16;   // bytes a load
  static constexpr int NP = RB / 4 / PB;                 // loads
  static constexpr int PPR = RB / PB;                    // loads a row
  uint32_t w[2][NP][KIND == FQ_KV_BF16 ? 1 : PB / 4];    // K, V on their way (codes only)
  uint32_t meta[2][NP];

  // The pages of the 16-key blocks that this wave's loads fall into.
  struct Places {
    BlockPlace at[NP];
  };
  __device__ static __forceinline__ Places places(const AttnArgs& a, const int32_t* table, int key0, int kv_seen,
                                                  int wave) {
    Places p;
    if (a.page_blocks % (kTile / kKvBlock) == 0) {   // one look-up where pages hold whole tiles
      const BlockPlace first = block_place(a, table, key0);
#pragma unroll
      for (int i = 0; i < NP; ++i)
        p.at[i] = BlockPlace{first.page, first.token + uint32_t((i * 256 + wave * 64) / PPR / kKvBlock * kKvBlock)};
      return p;
    }
#pragma unroll
    for (int i = 0; i < NP; ++i) {
      const int key = key0 + (i * 256 + wave * 64) / PPR / kKvBlock * kKvBlock;
      p.at[i] = block_place(a, table, key < kv_seen ? key : key0);   // past the last key: masked, any page will do
    }
    return p;
  }

  // Starts the loads; with bf16 into `lds`, which nothing reads any more.
  __device__ __forceinline__ void load(const AttnArgs& a, const char* kh, const char* vh, const uint32_t* kmh,
                                       const uint32_t* vmh, const Places& p, int tid, int wave, uint32_t lds) {
#pragma unroll
    for (int i = 0; i < NP; ++i) {
      const uint32_t idx = i * 256 + tid, row = idx / PPR, r = row % kKvBlock, piece = idx % PPR;
      const int64_t block = p.at[i].page * a.page_stride + p.at[i].token * int64_t(a.token_stride);
      if constexpr (KIND == FQ_KV_BF16) {
        // lane n of the wave fills 16 bytes at n * 16 from the wave's place on: the chunk
        // that belongs there
        const uint32_t off = r * a.token_stride + (piece ^ uint32_t(swizzle<D>(row))) * 16;
        const uint32_t to = lds + (i * 256 + wave * 64) * 16;
        to_lds(kh + block + off, to);
        to_lds(vh + block + off, to + TileLds<D>::K);
      } else {
        const uint32_t off = r * a.token_stride + piece * PB;
        get(kh + block + off, w[0][i]);
        get(vh + block + off, w[1][i]);
        const int64_t word = p.at[i].page * a.meta_page_stride + p.at[i].token + r;
        meta[0][i] = kmh[word];
        meta[1][i] = vmh[word];
      }
    }
  }

  // 16 bytes a lane from memory to LDS bytes lds + 16 lane.  (In assembly: the compiler
  // would wait for it before any LDS read, of the other tile too.)
  __device__ static __forceinline__ void to_lds(const char* p, uint32_t lds) {
    asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, off"
                 :: "v"(p), "s"(__builtin_amdgcn_readfirstlane(lds)) : "memory", "m0");
  }

  template <int W>
  __device__ static __forceinline__ void get(const char* p, uint32_t (&x)[W]) {
    if constexpr (W == 4) {
      const uint4 v = *reinterpret_cast<const uint4*>(p);
      x[0] = v.x;
      x[1] = v.y;
      x[2] = v.z;
      x[3] = v.w;
    } else {
      const uint2 v = *reinterpret_cast<const uint2*>(p);
      x[0] = v.x;
      x[1] = v.y;
    }
  }

  // code j of words x
  template <int W>
  __device__ static __forceinline__ float value(const uint32_t (&x)[W], int j) {
    if constexpr (KIND == FQ_KV_INT8) return float((x[j / 4] >> (8 * (j & 3))) & 255u);
    else return float((x[j / 8] >> (4 * (j & 7))) & 15u);
  }

  // Codes into a tile as bf16.
  __device__ __forceinline__ void store(char* lds, int tid) const {
    if constexpr (KIND != FQ_KV_BF16) {
      constexpr int CH = PB * (KIND == FQ_KV_INT8 ? 1 : 2) / 8;   // chunks a load
#pragma unroll
      for (int i = 0; i < NP; ++i) {
        const int idx = i * 256 + tid, row = idx / PPR, piece = idx % PPR;
#pragma unroll
        for (int v = 0; v < 2; ++v) {
#pragma unroll
          for (int c = 0; c < CH; ++c) {
            uint32_t o[4];
#pragma unroll
            for (int e = 0; e < 4; ++e)
              o[e] = pack_exact(value(w[v][i], 8 * c + 2 * e), value(w[v][i], 8 * c + 2 * e + 1));
            *reinterpret_cast<uint4*>(lds + v * TileLds<D>::K + row * 2 * D + ((piece * CH + c) ^ swizzle<D>(row)) * 16) =
                uint4{o[0], o[1], o[2], o[3]};
          }
        }
        if (piece == 0) {
          *reinterpret_cast<uint32_t*>(lds + TileLds<D>::kv + 4 * row) = meta[0][i];
          *reinterpret_cast<uint32_t*>(lds + TileLds<D>::kv + TileLds<D>::meta + 4 * row) = meta[1][i];
        }
      }
    }
  }
};

__device__ __forceinline__ bf16x8_t lds_read16(uint32_t lds, int offset) {
  typedef __attribute__((address_space(3))) const u32x4_t lds_u32x4;
  return __builtin_bit_cast(bf16x8_t, *reinterpret_cast<lds_u32x4*>(uintptr_t(lds + offset)));
}

typedef short s16x4_t __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) s16x4_t lds_s16x4;

// Four keys of one channel a lane, from the 8 bytes of four rows by sixteen channels that
// the lanes of a group of sixteen point to.
__device__ __forceinline__ uint2 read_transposed(uint32_t lds) {
  return __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16(reinterpret_cast<lds_s16x4*>(uintptr_t(lds))));
}

// The order of a stretch of N products: each one's R operand reads are AHEAD products
// earlier, PRE vector operations come before the first and V after each.  (The compiler
// alone puts each read right before its product, and the wave then waits for LDS.)
template <int N, int R, int AHEAD, int PRE, int V>
__device__ __forceinline__ void order_products() {
  constexpr int kMfma = 0x8, kDsRead = 0x100, kValu = 0x2, kTrans = 0x400;
  __builtin_amdgcn_sched_group_barrier(kDsRead, R * AHEAD, 0);
  if constexpr (PRE > 0) __builtin_amdgcn_sched_group_barrier(kValu | kTrans, PRE, 0);
#pragma unroll
  for (int i = 0; i < N; ++i) {
    __builtin_amdgcn_sched_group_barrier(kMfma, 1, 0);
    if (i + AHEAD < N) __builtin_amdgcn_sched_group_barrier(kDsRead, R, 0);
    if constexpr (V > 0) __builtin_amdgcn_sched_group_barrier(kValu | kTrans, V, 0);
  }
}

template <int KIND, int D>
__global__ void __launch_bounds__(64 * kTileWaves, 2) attn_tiles_kernel(AttnArgs a) {
  constexpr int STEPS = D / 16, DB = D / 32;
  extern __shared__ __attribute__((aligned(1024))) char tile_lds[];
  __shared__ uint32_t odd_flag;
  const int tid = int(threadIdx.x), lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int r32 = lane & 31, h = lane >> 5;

  Item it;
  if (!it.set<kRows, kTile>(a)) return;
  Row mine;
  mine.set(a, it, wave * 32 + r32);
  // what the rows of this wave see, for leaving tiles out and for the mask
  const int w_lo = min(wave * 32, it.rows - 1), w_hi = min(wave * 32 + 31, it.rows - 1);
  const int wt_lo = it.p0 + int((it.row0 + w_lo) / uint32_t(a.group)), wt_hi = it.p0 + int((it.row0 + w_hi) / uint32_t(a.group));
  const int wp_lo = min(wt_lo, it.kv_seen - 1);
  const int wp_hi = wave * 32 < it.rows ? min(wt_hi, it.kv_seen - 1) : -1;

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
    if (use_q) w = *reinterpret_cast<const uint4*>(qp + st * 16 + h * 8);
    const u32x4_t ws{w.x ^ q_sign, w.y ^ q_sign, w.z ^ q_sign, w.w ^ q_sign};
    if constexpr (KIND != FQ_KV_BF16) {
#pragma unroll
      for (int i = 0; i < 4; ++i)
        q_sum += bf16_bits_to_f32(ws[i]) + __builtin_bit_cast(float, ws[i] & 0xFFFF0000u);
    }
    qv[st] = __builtin_bit_cast(bf16x8_t, ws);
  }
  // - sum q as three bf16, 8 bits each, against z, z, z
  bf16x8_t zq;
  if constexpr (KIND != FQ_KV_BF16) {
    const float all = -pair_add(q_sum), hi = upper_bf16(all), mid = upper_bf16(all - hi), lo = all - hi - mid;
    zq = __builtin_bit_cast(bf16x8_t, u32x4_t{pack_exact(hi, mid), pack_exact(lo, 0.f), 0u, 0u});
  }
  f32x16_t acc[DB];
#pragma unroll
  for (int c = 0; c < DB; ++c)
#pragma unroll
    for (int i = 0; i < 16; ++i) acc[c][i] = 0.f;
  // m in units of q.k, of this lane's row; l and the sum of p' z_v of this lane's keys
  float m = kNegInf, l = 0.f, corr = 0.f;

  const int32_t* table = a.table + it.seq * a.table_stride;
  const char* kh = a.k + it.head * a.head_stride;
  const char* vh = a.v + it.head * a.head_stride;
  const uint32_t* kmh = KIND == FQ_KV_BF16 ? nullptr : a.k_meta + it.head * a.meta_head_stride;
  const uint32_t* vmh = KIND == FQ_KV_BF16 ? nullptr : a.v_meta + it.head * a.meta_head_stride;
  using S = Share<KIND, D>;
  S share;
  typename S::Places places;
  const uint32_t lds0 = lds_address(tile_lds);
  if (it.i_lo < it.i_hi) {
    places = S::places(a, table, it.tr.tile(it.i_lo) * kTile, it.kv_seen, wave);
    share.load(a, kh, vh, kmh, vmh, places, tid, wave, lds0);
    if (it.i_lo + 1 < it.i_hi) places = S::places(a, table, it.tr.tile(it.i_lo + 1) * kTile, it.kv_seen, wave);
    share.store(tile_lds, tid);
  }
  if (KIND == FQ_KV_BF16 && tid == 0) odd_flag = 0u;
  wait_vmcnt<0>();
  __syncthreads();

  // this lane's places in a tile: of K, chunk 2 st + h of row r32; of V, rows 4 h + r (and 8
  // more), channels 16 g + 4 x of each 32, as the transposing read takes them
  uint32_t k_at[STEPS], v_at[DB][2];
#pragma unroll
  for (int st = 0; st < STEPS; ++st) k_at[st] = lds0 + r32 * 2 * D + ((2 * st + h) ^ swizzle<D>(r32)) * 16;
  const int vr = (lane & 15) >> 2, vx = lane & 3, vg = (lane >> 4) & 1;
#pragma unroll
  for (int c = 0; c < DB; ++c)
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const int row = 8 * e + 4 * h + vr;
      v_at[c][e] = lds0 + TileLds<D>::K + row * 2 * D + ((4 * c + 2 * vg + vx / 2) ^ swizzle<D>(row)) * 16 + (vx & 1) * 8;
    }

  for (int i = it.i_lo; i < it.i_hi; ++i) {
    const int key0 = it.tr.tile(i) * kTile;
    const int buf = (i - it.i_lo) & 1;
    const uint32_t at = buf * TileLds<D>::one;
    char* lds = tile_lds + at;
    const bool more = i + 1 < it.i_hi;
    if (more) {
      share.load(a, kh, vh, kmh, vmh, places, tid, wave, lds0 + (buf ^ 1) * TileLds<D>::one);
      if (i + 2 < it.i_hi) places = S::places(a, table, it.tr.tile(i + 2) * kTile, it.kv_seen, wave);
    }
    if constexpr (KIND == FQ_KV_BF16) {
      if (!it.whole<kTile>(a, key0)) {
        // what is not finite in V is left out and noted
        bool any = false;
#pragma unroll
        for (int j = 0; j < S::NP; ++j) {
          uint4* p = reinterpret_cast<uint4*>(lds + TileLds<D>::K) + j * 256 + tid;
          const uint4 w = *p;
          if (nonfinite_pair(w.x) || nonfinite_pair(w.y) || nonfinite_pair(w.z) || nonfinite_pair(w.w)) {
            *p = uint4{finite_pair(w.x), finite_pair(w.y), finite_pair(w.z), finite_pair(w.w)};
            any = true;
          }
        }
        if (any) odd_flag = 1u;
        __syncthreads();
      }
    }
    // a wave leaves out tiles that none of its rows sees
    const bool skip = key0 > wp_hi || (a.window > 0 && key0 + kTile <= wt_lo - a.window + 1 && key0 >= a.sinks);
    if (!skip) {
      f32x16_t s[2];
#pragma unroll
      for (int kb = 0; kb < 2; ++kb)
#pragma unroll
        for (int j = 0; j < 16; ++j) s[kb][j] = 0.f;
      if constexpr (KIND != FQ_KV_BF16) {
#pragma unroll
        for (int kb = 0; kb < 2; ++kb) {
          const uint32_t w = *reinterpret_cast<const uint32_t*>(lds + TileLds<D>::kv + 4 * (kb * 32 + r32));
          const uint32_t z = h ? 0u : w >> 16;   // the other half of the operand's 16 places is 0
          s[kb] = mfma32(__builtin_bit_cast(bf16x8_t, u32x4_t{z | z << 16, z, 0u, 0u}), zq, s[kb]);
        }
      }
#pragma unroll
      for (int kb = 0; kb < 2; ++kb)
#pragma unroll
        for (int st = 0; st < STEPS; ++st)
          s[kb] = mfma32(lds_read16(k_at[st] + at, kb * 32 * 2 * D), qv[st], s[kb]);
      order_products<2 * STEPS, 1, 4, 0, 0>();
      if constexpr (KIND != FQ_KV_BF16) {
#pragma unroll
        for (int kb = 0; kb < 2; ++kb)
#pragma unroll
          for (int g = 0; g < 4; ++g) {
            const uint4 w = *reinterpret_cast<const uint4*>(lds + TileLds<D>::kv + 4 * (kb * 32 + 8 * g + 4 * h));
            const uint32_t ws[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
            for (int e = 0; e < 4; ++e)
              s[kb][4 * g + e] *= bf16_bits_to_f32(ws[e]);
          }
      }
      const bool whole = key0 + kTile - 1 <= wp_lo &&
                         (a.window == 0 || key0 > wt_hi - a.window || key0 + kTile <= a.sinks);
      uint32_t seen = ~0u;   // bit 16 kb + j
      if (!whole) {
        // bounds of the keys' constant places in the tile, so that the comparisons take
        // constants and no register for each key
        const int from = key0 + 4 * h, last = mine.pos - from, window = max(mine.win_lo, -(1 << 30)) - from,
                  sinks = a.sinks - from;
        seen = 0u;
#pragma unroll
        for (int kb = 0; kb < 2; ++kb)
#pragma unroll
          for (int j = 0; j < 16; ++j) {
            const int c = kb * 32 + 8 * (j / 4) + j % 4;
            const bool see = c <= last && (c >= window || c < sinks);
            s[kb][j] = see ? s[kb][j] : kNegInf;
            seen |= see ? 1u << (16 * kb + j) : 0u;
          }
      }
      float top = s[0][0];
#pragma unroll
      for (int kb = 0; kb < 2; ++kb)
#pragma unroll
        for (int j = 0; j < 16; ++j) top = fmaxf(top, s[kb][j]);
      top = pair_max(top);
      // the sums move to a new maximum only when some row's has grown by more than 2^8: until
      // then its weights are up to 2^8, which fp32 sums and bf16 weights hold as well
      if (__any(top > m + grow)) {
        const float m_new = fmaxf(m, top);
        const float shrink = __builtin_amdgcn_exp2f((m - (m_new == kNegInf ? 0.f : m_new)) * c2);
        m = m_new;
        l *= shrink;
        if constexpr (KIND != FQ_KV_BF16) corr *= shrink;
#pragma unroll
        for (int c = 0; c < DB; ++c) acc[c] *= shrink;
      }
      const float base = m == kNegInf ? 0.f : -m * c2;
#pragma unroll
      for (int st = 0; st < 4; ++st) {
        const int kb = st / 2;
        float p[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          p[e] = __builtin_amdgcn_exp2f(fmaf(s[kb][8 * (st & 1) + e], c2, base));
          l += p[e];
        }
        uint32_t vmw[8];
        if constexpr (KIND != FQ_KV_BF16) {
#pragma unroll
          for (int g = 0; g < 2; ++g) {
            const uint4 w = *reinterpret_cast<const uint4*>(lds + TileLds<D>::kv + TileLds<D>::meta +
                                                            4 * (st * 16 + 8 * g + 4 * h));
            const uint32_t ws[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              // a key that is not seen counts nothing, whatever its scale and zero-point
              vmw[4 * g + e] = whole || ((seen >> (st * 8 + 4 * g + e)) & 1u) ? ws[e] : 0u;
              p[4 * g + e] *= bf16_bits_to_f32(vmw[4 * g + e]);
            }
          }
        }
        const u32x4_t pw{pk_bf16(p[0], p[1]), pk_bf16(p[2], p[3]), pk_bf16(p[4], p[5]), pk_bf16(p[6], p[7])};
        const bf16x8_t pb = __builtin_bit_cast(bf16x8_t, pw);
        if constexpr (KIND != FQ_KV_BF16) {
#pragma unroll
          for (int e = 0; e < 4; ++e)
            corr = dot2_bf16(pw[e], __builtin_amdgcn_perm(vmw[2 * e + 1], vmw[2 * e], 0x07060302u), corr);
        }
#pragma unroll
        for (int c = 0; c < DB; ++c) {
          const uint2 lo = read_transposed(v_at[c][0] + at + st * 16 * 2 * D);
          const uint2 hi = read_transposed(v_at[c][1] + at + st * 16 * 2 * D);
          acc[c] = mfma32(__builtin_bit_cast(bf16x8_t, u32x4_t{lo.x, lo.y, hi.x, hi.y}), pb, acc[c]);
        }
      }
      // (with codes there are twice as many vector operations, which this order holds back:
      // 700 tokens over 2700 keys, 8 bits, 97 us with it)
      if constexpr (KIND == FQ_KV_BF16) order_products<4 * DB, 2, 4, 28, 7>();
    }
    if (more) {
      share.store(tile_lds + (buf ^ 1) * TileLds<D>::one, tid);
      wait_vmcnt<0>();
      __syncthreads();
    }
  }

  if constexpr (KIND == FQ_KV_BF16) {
    __syncthreads();
    if (__builtin_amdgcn_readfirstlane(odd_flag)) {
      walk_partial_tiles<kTile>(a, it, table, vh, it.i_lo, 1, [&](int key, const uint16_t* v) {
        if (!mine.in || !mine.sees(a, key)) return;
#pragma unroll
        for (int c = 0; c < DB; ++c)
#pragma unroll
          for (int i = 0; i < 16; ++i) acc[c][i] += if_nonfinite(v[32 * c + 8 * (i / 4) + 4 * h + i % 4]);
      });
    }
  }
  // lane (r32, h) has channels 32 c + 8 (i / 4) + 4 h + i % 4 of its row
  l = pair_add(l);
  if constexpr (KIND != FQ_KV_BF16) {
    corr = pair_add(corr);
#pragma unroll
    for (int c = 0; c < DB; ++c) acc[c] -= corr;
  }
  if (it.n_parts > 1) {
    // partial sums for join_kernel: [item][range][row][D + 4] floats, the last four: m c2, l
    const int64_t item = it.number;
    if (!mine.in) return;
    float* to = a.partials + ((item * a.split + it.part) * a.part_rows + wave * 32 + r32) * (D + 4);
#pragma unroll
    for (int c = 0; c < DB; ++c)
#pragma unroll
      for (int g = 0; g < 4; ++g)
        *reinterpret_cast<f32x4_t*>(to + 32 * c + 8 * g + 4 * h) =
            f32x4_t{acc[c][4 * g], acc[c][4 * g + 1], acc[c][4 * g + 2], acc[c][4 * g + 3]};
    if (h == 0) *reinterpret_cast<f32x4_t*>(to + D) = f32x4_t{m * c2, l, 0.f, 0.f};
    return;
  }
  m *= c2;
  if (!mine.in) return;
  // (with a maximum beyond fp32 every weight came out as 0 as well: such a row is NaN)
  const bool none = l == 0.f && m == kNegInf;
  const float inv = 1.f / l;
  uint16_t* op = a.O + (it.t0 + mine.token) * a.o_token + mine.head * a.o_head;
#pragma unroll
  for (int c = 0; c < DB; ++c)
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      uint2 w{0, 0};
      if (!none)
        w = uint2{pk_bf16(acc[c][4 * g] * inv, acc[c][4 * g + 1] * inv), pk_bf16(acc[c][4 * g + 2] * inv, acc[c][4 * g + 3] * inv)};
      *reinterpret_cast<uint2*>(op + 32 * c + 8 * g + 4 * h) = w;
    }
  if (a.lse && h == 0)
    a.lse[(it.t0 + mine.token) * a.n_heads + mine.head] = none ? kNegInf : (m + __log2f(l)) * 0.69314718055994530942f;
}

// Joins the ranges of rows whose keys were split, in their order: D / 8 threads a row,
// eight channels each.  (By the last workgroup of a block, as the kernel for few rows does,
// the 128 rows of 32 ranges took 130 us of one CU.)
template <int D>
__global__ void __launch_bounds__(256) join_kernel(AttnArgs a) {
  constexpr int T = D / 8, PER = 256 / T;   // threads a row, rows of a workgroup
  constexpr int kBlocks = kRows / PER;      // workgroups of a block of rows
  static_assert(kBlocks <= kJoinBlocks, "the plan bounds the grid");
  Item it;
  const int x = int(blockIdx.x) / kBlocks, first = int(blockIdx.x) % kBlocks * PER;
  const int head = x % a.n_kv_heads, rb = x / a.n_kv_heads;
  if (!it.set_rows<kRows, kTile>(a, int(blockIdx.y), rb, head)) return;
  const int n = it.parts(a);
  const int r = first + int(threadIdx.x) / T, ch = int(threadIdx.x) % T * 8;
  if (n <= 1 || r >= it.rows) return;
  const int64_t item = it.number;
  const int64_t step = int64_t(a.part_rows) * (D + 4);
  const float* from = a.partials + item * a.split * step + int64_t(r) * (D + 4);
  constexpr int U = 8;   // ranges read at a time
  float m = kNegInf;
  for (int p0 = 0; p0 < n; p0 += U) {
    float t[U];
#pragma unroll
    for (int u = 0; u < U; ++u) t[u] = from[min(p0 + u, n - 1) * step + D];
#pragma unroll
    for (int u = 0; u < U; ++u) m = fmaxf(m, t[u]);
  }
  const float base = m == kNegInf ? 0.f : m;
  float l = 0.f, o[8];
#pragma unroll
  for (int c = 0; c < 8; ++c) o[c] = 0.f;
  for (int p0 = 0; p0 < n; p0 += U) {
    f32x4_t v[U][2];
    float2 ml[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {   // in range; surplus loads unused
      const float* q = from + min(p0 + u, n - 1) * step;
      v[u][0] = *reinterpret_cast<const f32x4_t*>(q + ch);
      v[u][1] = *reinterpret_cast<const f32x4_t*>(q + ch + 4);
      ml[u] = *reinterpret_cast<const float2*>(q + D);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const float f = p0 + u < n ? __builtin_amdgcn_exp2f(ml[u].x - base) : 0.f;
      l = fmaf(f, ml[u].y, l);
      if (p0 + u < n) {
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          o[c] = fmaf(f, v[u][0][c], o[c]);
          o[4 + c] = fmaf(f, v[u][1][c], o[4 + c]);
        }
      }
    }
  }
  Row dst;
  dst.set(a, it, r);
  const float inv = l == 0.f ? 0.f : 1.f / l;
  uint32_t w[4];
#pragma unroll
  for (int c = 0; c < 4; ++c) w[c] = l == 0.f ? 0u : pk_bf16(o[2 * c] * inv, o[2 * c + 1] * inv);
  *reinterpret_cast<uint4*>(a.O + (it.t0 + dst.token) * a.o_token + dst.head * a.o_head + ch) = uint4{w[0], w[1], w[2], w[3]};
  if (a.lse && ch == 0)
    a.lse[(it.t0 + dst.token) * a.n_heads + dst.head] = l == 0.f ? kNegInf : (m + __log2f(l)) * 0.69314718055994530942f;
}

template <int KIND, int D>
int launch_one(const AttnArgs& g, dim3 grid, hipStream_t s) {
  hipLaunchKernelGGL((attn_tiles_kernel<KIND, D>), grid, dim3(64 * kTileWaves), TileLds<D>::bytes, s, g);
  if (g.split > 1)
    hipLaunchKernelGGL((join_kernel<D>), dim3(grid.x / unsigned(g.split) * (kRows / (256 / (D / 8))), grid.y), dim3(256),
                       0, s, g);
  return int(hipGetLastError());
}

}  // namespace

size_t attn_tiles_lds(int head_dim) { return head_dim == 64 ? TileLds<64>::bytes : TileLds<128>::bytes; }

int launch_attn_tiles(const AttnArgs& g, int kind, int head_dim, dim3 grid, hipStream_t s) {
  if (head_dim == 64) {
    if (kind == FQ_KV_BF16) return launch_one<FQ_KV_BF16, 64>(g, grid, s);
    if (kind == FQ_KV_INT8) return launch_one<FQ_KV_INT8, 64>(g, grid, s);
    return launch_one<FQ_KV_INT4, 64>(g, grid, s);
  }
  if (kind == FQ_KV_BF16) return launch_one<FQ_KV_BF16, 128>(g, grid, s);
  if (kind == FQ_KV_INT8) return launch_one<FQ_KV_INT8, 128>(g, grid, s);
  return launch_one<FQ_KV_INT4, 128>(g, grid, s);
}

}  // namespace fqk
