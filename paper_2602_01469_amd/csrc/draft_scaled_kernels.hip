// The inference-side drafting step (Sec. 2 of the paper) on a paged cache that is held in 8 bits with a power-of-two scale for
// each page and KV head, or in 4 bits with one for each token, KV head and 32 features: the K new rows of each request see its
// cached keys and the new keys of their own chain.
//
// With k = 2^ek a and v = 2^ev b for the codes a, b, S = scale Q K^T, P = 2^(S log2(e) - m), O = P V / sum P.  A code
// has four significant bits or fewer, so that with its scale it is a bf16 number (zero where that would not be a normal one,
// infinite from 2^128 on): codes are widened to bf16, scale and all, by one instruction for two of them, between LDS and the
// matrix instruction.  (The matrix instruction for 8-bit types, with queries split into two numbers of them, would need no widening
// of keys, but its sums are not fp32 sums: 64 products of normal data came out 4e-5 of the largest sum off.)
// The cache is read once, 2 Hkv D bytes a token, and bounds a large call on 8 bits.  In 4 bits a token has 17/16 Hkv D bytes, and no unit
// alone bounds a large call (below).  A small one is a chain of memory round trips.
#include "attn_kernels.h"
#include "attn_util.h"
#include "cache_kernels.h"

#include <climits>
#include <type_traits>

namespace peagle {

namespace {

template <CacheType T>
constexpr bool kFour = T == CacheType::kE2M1;  // two codes a byte

// Eight codes, times `scale` (a power of two), as a matrix operand.
template <CacheType T>
__device__ __forceinline__ bf16x8 widen8(uint32_t a, uint32_t b, float scale) {
  u32x4 u;
  auto two = [&](uint32_t w, auto high) {
    constexpr bool H = decltype(high)::value;
    const bf16x2 x = T == CacheType::kE5M2 ? __builtin_amdgcn_cvt_scalef32_pk_bf16_bf8(w, scale, H) : __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale, H);
    return __builtin_bit_cast(uint32_t, x);
  };
  u[0] = two(a, std::false_type{});
  u[1] = two(a, std::true_type{});
  u[2] = two(b, std::false_type{});
  u[3] = two(b, std::true_type{});
  return __builtin_bit_cast(bf16x8, u);
}
// Eight codes of 4 bits.  (Of the scale the instruction takes the exponent alone; 255 makes NaN of every code.)
__device__ __forceinline__ bf16x8 widen4(uint32_t w, float scale) {
  u32x4 u;
  u[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 0));
  u[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 1));
  u[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 2));
  u[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 3));
  return __builtin_bit_cast(bf16x8, u);
}

// LDS image of 32 tokens of a page, row (token) by row of D bytes: the 16-byte chunk c of row r stands at c ^ swz8(r), so that both
// reads below touch sixteen different 16-byte places modulo 256 bytes at a time:
//   keys    lane <-> row, 16 rows, the same chunk
//   values  rows {0..3, 8..11} or {4..7, 12..15} of a group of sixteen, two neighbouring chunks
// D = 64 (four rows per 256 bytes): bits 2 and 3 of the row.  D = 128 (two rows): bits 1..3, in the order that puts rows 0, 2, 8
// and 10 into different pairs of chunks.
template <int D>
__device__ __forceinline__ int swz8(int row) {
  const int r = row >> 1;
  return D == 64 ? (row >> 2) & 3 : (r & 4) | ((r & 1) << 1) | ((r >> 1) & 1);
}
// The same of rows of D / 2 bytes, codes of 4 bits, of which 16 lanes read the same chunk of 16 rows (eight, at D = 128 four, per
// 256 bytes).
template <int D>
__device__ __forceinline__ int swz4(int row) {
  return D == 64 ? (row >> 3) & 1 : (row >> 2) & 3;
}
template <int D, CacheType T>
__device__ __forceinline__ int swz_codes(int row) {
  return kFour<T> ? swz4<D>(row) : swz8<D>(row);
}

// Which eight features step i of the product with the keys takes in lanes of half g: those that follow each other in a 16-byte read
// of the keys' codes, two steps' with codes of 8 bits, four steps' with codes of 4 bits (which so have one scale).  SHARED: the keys
// are read as bf16.
template <CacheType T, bool SHARED = false>
__device__ __forceinline__ int q_chunk(int i, int g) {
  return SHARED ? 2 * i + g : kFour<T> ? 8 * (i / 4) + 4 * g + i % 4 : 4 * (i / 2) + 2 * g + i % 2;
}

// State of RB blocks of 32 query rows: lane <-> row, registers <-> features 32 db + 8 (i / 4) + 4 g + i % 4.
template <int D, int RB>
struct Rows {
  bf16x8 q[RB][D / 16];  // eight features of each step, see q_chunk()
  f32x16 o[RB][D / 32];
  float m[RB];           // reference of the exponents (log2)
  float l[RB], w[RB];    // sums over this lane's keys of the probabilities: as they are, and as they weigh the values
};

// Scores of 32 keys (registers <-> keys 8 (i / 4) + 4 g + i % 4) to probabilities, as operands of the product with the values.
// A probability is rounded to bf16 to weigh its value, by up to 2^-9 of itself wherever it stands, so that the reference need not be
// near the row's largest score.  It must not be far below it: it moves where a lane's sum of probabilities is above `limit` (also at
// the first keys, which meet the start value), and no maximum is taken otherwise.  The output is divided by the sum of the rounded
// probabilities, which makes a row of one heavy key exact; the LSE takes the sum of the unrounded ones.
// The limit keeps what is summed for the values inside fp32: with scales up to 2^40 a value is below 2^56, and weights of 2^41 a
// block of 32 keys, up to 2^25 of them, leave their sum below 2^122.  Larger values are weighed by 1 at most, as by a running maximum.
constexpr float kFarLimit = 0x1p40f, kNearLimit = 1.0f;
constexpr int kFarScale = 127 + 40;  // largest code of a page's values that goes with kFarLimit
template <int D, int RB>
__device__ __forceinline__ void soft(Rows<D, RB>& r, int rb, const f32x16& s, float c, float limit, bf16x8 (&pb)[2]) {
  f32x16 x;
  auto weigh = [&] {
    float sum[4];
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      x[i] = exp2_fast(__builtin_fmaf(s[i], c, -r.m[rb]));
      sum[i % 4] = i < 4 ? x[i] : sum[i % 4] + x[i];
    }
    return (sum[0] + sum[1]) + (sum[2] + sum[3]);
  };
  float sum = weigh();
  if (__builtin_amdgcn_ballot_w64(sum > limit) != 0) {
    const float mx = max_halves(max16(s)) * c;
    const bool need = max_halves(sum) > limit && mx > r.m[rb];
    const float m_new = need ? mx : r.m[rb], alpha = exp2_fast(r.m[rb] - m_new);
    r.m[rb] = m_new;
    r.l[rb] *= alpha;
    r.w[rb] *= alpha;
#pragma unroll
    for (int db = 0; db < D / 32; ++db)
#pragma unroll
      for (int i = 0; i < 16; ++i) r.o[rb][db][i] *= alpha;
    sum = weigh();
  }
  r.l[rb] += sum;
  pb[0] = pack8_sum(x, 0, r.w[rb]);
  pb[1] = pack8_sum(x, 1, r.w[rb]);
}

// The bytes of a word whose bits, from the lowest on, are set in `keep` (four of them).
__device__ __forceinline__ uint32_t bytes_of(uint32_t keep) { return ((keep & 0xfu) * 0x00204081u & 0x01010101u) * 0xffu; }

// 32 keys, staged with their values, of which the first n count.  The others are masked, and their codes of values made zero: a
// probability of zero times an infinity, which E5M2 holds and any code becomes beyond bf16, would be NaN.
template <int D, CacheType T, int RB>
__device__ __forceinline__ void cached_keys(Rows<D, RB>& r, const char* k_at, const char* v_at, const int (&k_off)[D / 32],
                                            const int (&v_off)[D / 32], float ks, float vs, float limit, int n, int g,
                                            float c) {
  // All LDS reads first: one at a time in front of its use, as the compiler places them otherwise, each would be waited for.
  typedef __attribute__((ext_vector_type(2))) int i32x2;
  u32x4 kw[D / 32];
  i32x2 vw[2][D / 32];
#pragma unroll
  for (int i = 0; i < D / 32; ++i) kw[i] = *reinterpret_cast<const u32x4*>(k_at + k_off[i]);
#pragma unroll
  for (int t = 0; t < 2; ++t)
#pragma unroll
    for (int db = 0; db < D / 32; ++db)
      vw[t][db] = __builtin_amdgcn_ds_read_tr8_b64_v2i32(PEAGLE_LDS_PTR(i32x2, v_at + v_off[db] + t * 16 * D));
  __builtin_amdgcn_sched_barrier(0);
  // (A wave at its products goes before one at its softmax, which then has the vector units while the products run: 48 requests of
  // 500 to 8191 tokens with 128 rows of 128 features 92.9 -> 87.9 us, 56 rows of 64 features 0 to 3 %.)
  __builtin_amdgcn_s_setprio(1);
  f32x16 s[RB];
#pragma unroll
  for (int rb = 0; rb < RB; ++rb) s[rb] = zero16();
#pragma unroll
  for (int i = 0; i < D / 32; ++i) {
    const bf16x8 a0 = widen8<T>(kw[i][0], kw[i][1], ks), a1 = widen8<T>(kw[i][2], kw[i][3], ks);
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
      s[rb] = mfma32(a0, r.q[rb][2 * i], s[rb]);
      s[rb] = mfma32(a1, r.q[rb][2 * i + 1], s[rb]);
    }
  }
  __builtin_amdgcn_s_setprio(0);
  if (n < 32) {
    const uint32_t bits = ((1u << n) - 1) >> (4 * g);
#pragma unroll
    for (int rb = 0; rb < RB; ++rb)
#pragma unroll
      for (int i = 0; i < 16; ++i) s[rb][i] = mask_sel(s[rb][i], bits, 8 * (i / 4) + (i % 4));
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int db = 0; db < D / 32; ++db)
#pragma unroll
        for (int w = 0; w < 2; ++w) vw[t][db][w] &= (int)bytes_of(bits >> (16 * t + 8 * w));
  }
  bf16x8 pb[RB][2];
#pragma unroll
  for (int rb = 0; rb < RB; ++rb) soft(r, rb, s[rb], c, limit, pb[rb]);
  __builtin_amdgcn_s_setprio(1);
#pragma unroll
  for (int t = 0; t < 2; ++t)
#pragma unroll
    for (int db = 0; db < D / 32; ++db) {
      const bf16x8 a = widen8<T>((uint32_t)vw[t][db][0], (uint32_t)vw[t][db][1], vs);
#pragma unroll
      for (int rb = 0; rb < RB; ++rb) r.o[rb][db] = mfma32(a, pb[rb][t], r.o[rb][db]);
    }
  __builtin_amdgcn_s_setprio(0);
}

// The same of codes of 4 bits.  Two neighbouring keys' values have scales of their own, so that the codes of one feature cannot be
// widened as the product takes them, two keys at a time.  They are widened as they stand instead - lane <-> key, 32 features and
// one scale, as the keys - and written to this wave's part of LDS as a tile of bf16 rows, which is read transposed as new keys' values
// are.
template <int D>
struct Off4 {
  int codes[D / 64], scale[D / 64];      // of a lane's 16-byte chunk j, features 32 (2 j + g) .. + 32 of key lane % 32, and its scale
  int v_codes[D / 64], v_scale[D / 64];  // of its chunk of value_key()
  int out[D / 64][4];                    // of that one's eight features w in the tile
  TrOff<D> tr;
};
// The key whose values a lane widens, of 32: eight lanes that follow each other write to eight different 16-byte places modulo 128
// bytes of the tile (in the lanes' own order two of them share each place, which takes twice as long).
template <int D>
__device__ __forceinline__ int value_key(int ln) {
  const int i = ln & 7, h = (ln >> 3) & 1;
  return (ln & 16) | (D == 64 ? 2 * i + h : ((i >> 1) << 2) | (h << 1) | (i & 1));
}
template <int D, int RB>
__device__ __forceinline__ void cached_keys4(Rows<D, RB>& r, const char* k_at, const char* v_at, const char* ks_at, const char* vs_at, char* tile,
                                             const Off4<D>& off, int n, int ln, int g, float c) {
  u32x4 kw[D / 64], vw[D / 64];
  uint32_t ks[D / 64], vs[D / 64];
#pragma unroll
  for (int j = 0; j < D / 64; ++j) {
    kw[j] = *reinterpret_cast<const u32x4*>(k_at + off.codes[j]);
    ks[j] = *reinterpret_cast<const uint8_t*>(ks_at + off.scale[j]);
  }
#pragma unroll
  for (int j = 0; j < D / 64; ++j) {
    vw[j] = *reinterpret_cast<const u32x4*>(v_at + off.v_codes[j]);
    vs[j] = *reinterpret_cast<const uint8_t*>(vs_at + off.v_scale[j]);
  }
  __builtin_amdgcn_sched_barrier(0);
  if (n < 32) {  // (whatever stands behind the last key: zeros)
#pragma unroll
    for (int j = 0; j < D / 64; ++j) {
      vs[j] = value_key<D>(ln) < n ? vs[j] : 127u;
#pragma unroll
      for (int w = 0; w < 4; ++w) vw[j][w] = value_key<D>(ln) < n ? vw[j][w] : 0u;
    }
  }
  bool large = false;
#pragma unroll
  for (int j = 0; j < D / 64; ++j) large |= vs[j] > (uint32_t)kFarScale && vs[j] != 255u;  // (NaN changes no bit of other features)
  const float limit = __builtin_amdgcn_ballot_w64(large) != 0 ? kNearLimit : kFarLimit;
  __builtin_amdgcn_s_setprio(1);
  f32x16 s[RB];
#pragma unroll
  for (int rb = 0; rb < RB; ++rb) s[rb] = zero16();
#pragma unroll
  for (int j = 0; j < D / 64; ++j)
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      const uint32_t word = kw[j][w];
      const bf16x8 a = widen4(word, __builtin_bit_cast(float, ks[j] << 23));
#pragma unroll
      for (int rb = 0; rb < RB; ++rb) s[rb] = mfma32(a, r.q[rb][4 * j + w], s[rb]);
    }
  __builtin_amdgcn_s_setprio(0);
#pragma unroll
  for (int j = 0; j < D / 64; ++j)
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      const uint32_t word = vw[j][w];
      *reinterpret_cast<bf16x8*>(tile + off.out[j][w]) = widen4(word, __builtin_bit_cast(float, vs[j] << 23));
    }
  asm volatile("" : : : "memory");  // (the tile is this wave's, whose LDS accesses take place in their order)
  if (n < 32) {
    const uint32_t bits = ((1u << n) - 1) >> (4 * g);
#pragma unroll
    for (int rb = 0; rb < RB; ++rb)
#pragma unroll
      for (int i = 0; i < 16; ++i) s[rb][i] = mask_sel(s[rb][i], bits, 8 * (i / 4) + (i % 4));
  }
  bf16x8 pb[RB][2];
#pragma unroll
  for (int rb = 0; rb < RB; ++rb) soft(r, rb, s[rb], c, limit, pb[rb]);
  __builtin_amdgcn_s_setprio(1);
#pragma unroll
  for (int t = 0; t < 2; ++t)
#pragma unroll
    for (int db = 0; db < D / 32; ++db) {
      const bf16x8 a = frag_tr<D>(tile, off.tr, 16 * t, db);
#pragma unroll
      for (int rb = 0; rb < RB; ++rb) r.o[rb][db] = mfma32(a, pb[rb][t], r.o[rb][db]);
    }
  __builtin_amdgcn_s_setprio(0);
  asm volatile("" : : : "memory");
}

// 32 keys in stages, for a wave that has two at work: while the vector unit turns the scores of one into probabilities, the matrix
// unit multiplies the next one's keys.  (64 requests of 512 to 8192 tokens, 56 rows of 64 features: 68 us for a step, 73 with cached_keys4();
// 48 of 500 to 8191, 128 rows of 128 features, 92 and 101.)
template <int D>
struct Keys4 {
  u32x4 k[D / 64], v[D / 64];
  uint32_t ks[D / 64], vs[D / 64];
};
template <int D>
__device__ __forceinline__ void load4(Keys4<D>& x, const char* k_at, const char* v_at, const char* ks_at, const char* vs_at, const Off4<D>& off) {
#pragma unroll
  for (int j = 0; j < D / 64; ++j) {
    x.k[j] = *reinterpret_cast<const u32x4*>(k_at + off.codes[j]);
    x.ks[j] = *reinterpret_cast<const uint8_t*>(ks_at + off.scale[j]);
  }
#pragma unroll
  for (int j = 0; j < D / 64; ++j) {
    x.v[j] = *reinterpret_cast<const u32x4*>(v_at + off.v_codes[j]);
    x.vs[j] = *reinterpret_cast<const uint8_t*>(vs_at + off.v_scale[j]);
  }
}
template <int D>
__device__ __forceinline__ bf16x8 key_features(const Keys4<D>& x, int i) {  // of step i of the product with the queries
  const uint32_t word = x.k[i / 4][i % 4];
  return widen4(word, __builtin_bit_cast(float, x.ks[i / 4] << 23));
}
template <int D, int RB>
__device__ __forceinline__ void scores4(const Keys4<D>& x, const Rows<D, RB>& r, f32x16 (&s)[RB]) {
#pragma unroll
  for (int i = 0; i < D / 16; ++i) {
    const bf16x8 a = key_features(x, i);
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) s[rb] = mfma32(a, r.q[rb][i], i == 0 ? zero16() : s[rb]);
  }
}
// The values to the tile, zeros from key n on.  Returns the limit that goes with their scales.
template <int D>
__device__ __forceinline__ float values4(Keys4<D>& x, char* tile, const Off4<D>& off, int n, int ln) {
  if (n < 32) {
#pragma unroll
    for (int j = 0; j < D / 64; ++j) {
      x.vs[j] = value_key<D>(ln) < n ? x.vs[j] : 127u;
#pragma unroll
      for (int w = 0; w < 4; ++w) x.v[j][w] = value_key<D>(ln) < n ? x.v[j][w] : 0u;
    }
  }
  bool large = false;
#pragma unroll
  for (int j = 0; j < D / 64; ++j) {
    large |= x.vs[j] > (uint32_t)kFarScale && x.vs[j] != 255u;  // (NaN changes no bit of other features)
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      const uint32_t word = x.v[j][w];
      *reinterpret_cast<bf16x8*>(tile + off.out[j][w]) = widen4(word, __builtin_bit_cast(float, x.vs[j] << 23));
      __builtin_amdgcn_sched_barrier(0);
    }
  }
  return __builtin_amdgcn_ballot_w64(large) != 0 ? kNearLimit : kFarLimit;
}
// One turn: what the scores s of n keys weigh in the output, their values being in the tile; the next keys' scores.  Every matrix
// instruction is followed by its share of the vector instructions, and by a fence so that this order stays.  With two blocks of rows
// the second one's product with the values waits for the next turn (`Held4`), so that fewer registers hold what is in between.
template <int D>
struct Held4 {
  bf16x8 v[2][D / 32], p[2];
};
template <int D, int RB>
__device__ __forceinline__ void take4(Rows<D, RB>& r, f32x16 (&s)[RB], f32x16 (&s_next)[RB], const Keys4<D>& next, Held4<D>& held, const char* tile,
                                      const Off4<D>& off, int n, float limit, int g, float c) {
  static_assert(RB <= 2, "");
  constexpr int kSteps = D / 16, kFrags = D / 32;
  auto load_values = [&](int t) {
#pragma unroll
    for (int db = 0; db < kFrags; ++db) held.v[t][db] = frag_tr<D>(tile, off.tr, 16 * t, db);
  };
  if (n < 32) {
    const uint32_t bits = n <= 0 ? 0u : ((1u << n) - 1) >> (4 * g);
#pragma unroll
    for (int rb = 0; rb < RB; ++rb)
#pragma unroll
      for (int i = 0; i < 16; ++i) s[rb][i] = mask_sel(s[rb][i], bits, 8 * (i / 4) + (i % 4));
  }
  f32x16 x;
  float sum[4];
  auto weigh = [&](int rb, int from, int to) {
#pragma unroll
    for (int i = from; i < to; ++i) {
      x[i] = exp2_fast(__builtin_fmaf(s[rb][i], c, -r.m[rb]));
      sum[i % 4] = i < 4 ? x[i] : sum[i % 4] + x[i];
    }
  };
  auto check = [&](int rb) {
    float total = (sum[0] + sum[1]) + (sum[2] + sum[3]);
    if (__builtin_expect(__builtin_amdgcn_ballot_w64(total > limit) != 0, 0)) {
      const float mx = max_halves(max16(s[rb])) * c;
      const bool need = max_halves(total) > limit && mx > r.m[rb];
      const float m_new = need ? mx : r.m[rb], alpha = exp2_fast(r.m[rb] - m_new);
      r.m[rb] = m_new;
      r.l[rb] *= alpha;
      r.w[rb] *= alpha;
#pragma unroll
      for (int db = 0; db < D / 32; ++db)
#pragma unroll
        for (int i = 0; i < 16; ++i) r.o[rb][db][i] *= alpha;
      weigh(rb, 0, 16);
      total = (sum[0] + sum[1]) + (sum[2] + sum[3]);
    }
    r.l[rb] += total;
    held.p[0] = pack8_sum(x, 0, r.w[rb]);
    held.p[1] = pack8_sum(x, 1, r.w[rb]);
  };
  auto weigh_value = [&](int rb, int k) { r.o[rb][k % kFrags] = mfma32(held.v[k / kFrags][k % kFrags], held.p[k / kFrags], r.o[rb][k % kFrags]); };
  if constexpr (RB == 2) {
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int k = 0; k < 2 * kFrags; ++k) {
      weigh_value(1, k);
      weigh(0, 16 * k / (2 * kFrags), 16 * (k + 1) / (2 * kFrags));
      __builtin_amdgcn_sched_barrier(0);
    }
    check(0);
    load_values(0);
    load_values(1);
  }
  constexpr int kNext = RB * kSteps, kMatrix = kNext + (RB == 2 ? 2 * kFrags : 0);
  __builtin_amdgcn_sched_barrier(0);
  bf16x8 a = key_features(next, 0);
#pragma unroll
  for (int k = 0; k < kMatrix; ++k) {
    if (k < kNext) s_next[k % RB] = mfma32(a, r.q[k % RB][k / RB], k < RB ? zero16() : s_next[k % RB]);
    else weigh_value(0, k - kNext);
    weigh(RB - 1, 16 * k / kMatrix, 16 * (k + 1) / kMatrix);
    if (k % RB == RB - 1 && k + 1 < kNext) a = key_features(next, (k + 1) / RB);
    __builtin_amdgcn_sched_barrier(0);
  }
  if (RB == 1) load_values(0);
  check(RB - 1);
  __builtin_amdgcn_sched_barrier(0);
  if constexpr (RB == 1) {
    load_values(1);
#pragma unroll
    for (int k = 0; k < 2 * kFrags; ++k) weigh_value(0, k);
    __builtin_amdgcn_sched_barrier(0);
  }
}

// Four waves with different rows: each widens a quarter of 32 keys, and all of them read them as bf16 rows of two tiles of keys and
// two of values, one of each being written while the other is read.  Codes come from memory straight to registers, two turns before
// they are widened.  (128 rows of 128 features: 84 us for a step of 48 requests of 500 to 8191 tokens, 92 where each wave widens all
// keys.  Two waves that widen half of them each gain nothing.)
struct Raw4 {  // a lane's share: sixteen features of one key, and their scale
  u32x2 w;
  uint32_t scale;
};
struct Share4 {
  int key, codes, scale;  // which key of 32; offsets of its codes and its scale
  int out;                // place of its first eight features in a tile
  __device__ __forceinline__ Share4(int part, int lane) {
    constexpr int D = 128;
    const int i = lane & 7, block = (lane >> 3) & 3, half = lane >> 5;
    // (eight lanes that follow each other write to eight places modulo 128 bytes, as in value_key())
    key = (part >> 1) * 16 + (((i >> 1) << 2) | ((part & 1) << 1) | (i & 1));
    codes = key * (D / 2) + block * 16 + half * 8;
    scale = key * (D / 32) + block;
    out = tile_off<D>(key, 4 * block + 2 * half);
  }
};
// (as global memory: a load that might be from LDS would be waited for with the LDS reads)
template <class V>
__device__ __forceinline__ V load_global(const uint8_t* base, uint32_t off) {
  typedef const __attribute__((address_space(1))) uint8_t bytes;
  return *(const __attribute__((address_space(1))) V*)((bytes*)base + off);
}
__device__ __forceinline__ void load_share(Raw4& x, const uint8_t* codes, const uint8_t* scales, const Share4& mine) {
  x.w = load_global<u32x2>(codes, (uint32_t)mine.codes);
  x.scale = load_global<uint8_t>(scales, (uint32_t)mine.scale);
}
__device__ __forceinline__ void put_share(const Raw4& x, char* tile, const Share4& mine, int i) {  // its eight features i
  const uint32_t word = x.w[i];
  *reinterpret_cast<bf16x8*>(tile + (mine.out ^ (i << 4))) = widen4(word, __builtin_bit_cast(float, x.scale << 23));
}
__device__ __forceinline__ void keep_first(Raw4& x, const Share4& mine, int n) {  // zeros from key n on
  if (n < 32) {
    x.scale = mine.key < n ? x.scale : 127u;
#pragma unroll
    for (int i = 0; i < 2; ++i) x.w[i] = mine.key < n ? x.w[i] : 0u;
  }
}
__device__ __forceinline__ bool far_scale(const Raw4& x) {
  return __builtin_amdgcn_ballot_w64(x.scale > (uint32_t)kFarScale && x.scale != 255u) != 0;
}
// LDS of a workgroup whose waves share: all that it has written is there, and what it has read need not be any more.
__device__ __forceinline__ void meet() {
  asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" : : : "memory");
}

// Sixteen of the request's new keys (bf16, staged in a slot: K rows of 2 D bytes, V behind them, in the layout of the bf16 tiles),
// the first of them key k0; the row of depth d sees keys 0..d.  A masked key weighs zero, and zero times an infinity or NaN is
// NaN: such values are taken out of the product and added to the rows that see them, from v_new (key 0 of the KV head, the next
// one `stride` elements on).
constexpr int kNewKeys = 16;
template <int D, CacheType T, int RB, bool SHARED>
__device__ __forceinline__ void new_keys(Rows<D, RB>& r, const char* k_at, const char* v_at, int k0, int K, const __bf16* v_new, uint32_t stride,
                                         const int (&depth)[RB], float c) {
  const int lane = lane_id(), g = lane >> 5, row = lane % kNewKeys;
  bf16x8 ka[D / 16], va[D / 32];
  const TrOff<D> to = tr_offsets<D>(lane);
#pragma unroll
  for (int i = 0; i < D / 16; ++i) ka[i] = *reinterpret_cast<const bf16x8*>(k_at + tile_off<D>(row, q_chunk<T, SHARED>(i, g)));
#pragma unroll
  for (int db = 0; db < D / 32; ++db) va[db] = frag_tr<D>(v_at, to, 0, db);
  __builtin_amdgcn_sched_barrier(0);
  f32x16 s[RB];
#pragma unroll
  for (int rb = 0; rb < RB; ++rb) s[rb] = zero16();
#pragma unroll
  for (int i = 0; i < D / 16; ++i)
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) s[rb] = mfma32(ka[i], r.q[rb][i], s[rb]);
  bf16x8 pb[RB][2];
#pragma unroll
  for (int rb = 0; rb < RB; ++rb) {
    const int sees = depth[rb] + 1 - k0, n = sees < kNewKeys ? sees : kNewKeys;
    const uint32_t bits = (n <= 0 ? 0u : (1u << n) - 1) >> (4 * g);
#pragma unroll
    for (int i = 0; i < 16; ++i) s[rb][i] = mask_sel(s[rb][i], bits, 8 * (i / 4) + (i % 4));
    soft(r, rb, s[rb], c, kNearLimit, pb[rb]);
  }
  bool odd = false;
#pragma unroll
  for (int db = 0; db < D / 32; ++db) {
    u32x4 a = __builtin_bit_cast(u32x4, va[db]);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const uint32_t w = a[j];
      const bool lo = (w & 0x7f80u) == 0x7f80u, hi = (w & 0x7f800000u) == 0x7f800000u;
      odd |= lo | hi;
      a[j] = w & ((lo ? 0u : 0xffffu) | (hi ? 0u : 0xffff0000u));
    }
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) r.o[rb][db] = mfma32(__builtin_bit_cast(bf16x8, a), pb[rb][0], r.o[rb][db]);
  }
  if (__builtin_expect(__builtin_amdgcn_ballot_w64(odd) != 0, 0)) {
    for (int e = k0; e < K && e < k0 + kNewKeys; ++e) {
      const uint32_t v = (uint32_t)e * stride + 4 * g;
#pragma unroll
      for (int db = 0; db < D / 32; ++db)
#pragma unroll
        for (int i4 = 0; i4 < 4; ++i4) {
          __builtin_amdgcn_sched_barrier(0);  // (seldom here: few registers rather than many loads on their way)
          const u32x2 w = *reinterpret_cast<const u32x2*>(v_new + v + (db * 32 + 8 * i4));
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const uint32_t x = j % 2 ? w[j / 2] & 0xffff0000u : w[j / 2] << 16;
            const float add = (x & 0x7f800000u) == 0x7f800000u ? __builtin_bit_cast(float, x) : 0.f;
#pragma unroll
            for (int rb = 0; rb < RB; ++rb) r.o[rb][db][4 * i4 + j] += depth[rb] >= e ? add : 0.f;
          }
        }
    }
  }
}

// Sum of x over the lanes up to and including this one.
__device__ __forceinline__ int scan_lanes(int x) {
  x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, true);   // within rows of 16 lanes: from 1, 2, 4, 8 lanes below
  x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, true);
  x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, true);
  x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, true);
  x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false);  // the last lane of rows 0 and 2 to rows 1 and 3
  x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false);  // lane 31 to rows 2 and 3
  return x;
}

// Cached tokens of a request, clamped to what its table can describe.
__device__ __forceinline__ int clamp_len(int n, int max_pages) {
  return n < 0 ? 0 : n > max_pages * kKeysPerTile ? max_pages * kKeysPerTile : n;
}
__device__ __forceinline__ int pages_of(int n) { return (n + kKeysPerTile - 1) / kKeysPerTile; }

// Every workgroup of a KV head takes the same share of all requests' work, counted in pages: workgroup w the units [w share,
// (w + 1) share) of the requests one after the other.  A request is `lead` units that stand for what its start costs a workgroup
// that has another request's pages before it, its pages, and one unit for the new keys.
struct Share {
  int share, c, skip;   // units a workgroup; its first request, and the units of that which stand before its own
  int lens, lens_from;  // ctx_len of request lens_from + lane, of some requests from the first on
  bool any;
};
__device__ __forceinline__ Share share_of(const int32_t* ctx_len, int C, int max_pages, int w, int n_wgs, int least, int lead, int lane) {
  const int per = (C + 63) / 64;
  Share s;
  s.lens = 0;
  s.lens_from = 0;
  int mine = 0;
  for (int i = 0; i < per; ++i) {
    const int c = lane * per + i;
    if (c < C) s.lens = ctx_len[c];
    mine += c < C ? pages_of(clamp_len(s.lens, max_pages)) + lead + 1 : 0;
  }
  int end = scan_lanes(mine);
  const int total = __builtin_amdgcn_readlane(end, 63);
  s.share = (total + n_wgs - 1) / n_wgs;
  s.share = s.share < least ? least : s.share;
  const int64_t at64 = (int64_t)w * s.share;
  s.any = at64 < total;
  const int at = s.any ? (int)at64 : 0;
  int l = __builtin_ctzll(__builtin_amdgcn_ballot_w64(end > at));
  int before = __builtin_amdgcn_readlane(end - mine, l);
  s.c = l * per;
  if (per > 1) {
    const int c = s.c + lane;
    s.lens_from = s.c;
    s.lens = c < C ? ctx_len[c] : 0;
    mine = lane < per && c < C ? pages_of(clamp_len(s.lens, max_pages)) + lead + 1 : 0;
    end = before + scan_lanes(mine);
    l = __builtin_ctzll(__builtin_amdgcn_ballot_w64(end > at));
    before = __builtin_amdgcn_readlane(end - mine, l);
    s.c += l;
  }
  s.skip = at - before;
  return s;
}

template <int N, int PER>
__device__ __forceinline__ void wait_slots(int pending) {  // until at most `pending` (<= N) slots' copies are on their way
  if constexpr (N == 0) {
    wait_outstanding<0>();
  } else {
    if (pending >= N) wait_outstanding<N * PER>();
    else wait_slots<N - 1, PER>(pending);
  }
}

// A value that the compiler keeps in scalar registers rather than loading it again: a kernel's parameters, all loaded at its start
// (each first use of a line of them waits for memory), and none in the loops.
template <class T>
__device__ __forceinline__ T held(T x) {
  asm volatile("" : "+s"(x));
  return x;
}
template <class T>
__device__ __forceinline__ T* held(T* x) {  // (as a pointer to global memory, which an opaque pointer is not known to be)
  __attribute__((address_space(1))) T* g = (__attribute__((address_space(1))) T*)x;
  asm volatile("" : "+s"(g));
  return (T*)g;
}

// A stream's share of LDS: a ring of slots of kTokens tokens each and, with codes of 4 bits, a tile for each of its waves.  Codes of
// 4 bits take one of three loops:
//   kShared  128 rows of 128 features, four waves: put_share()
//   kPiped   two waves a SIMD, whose registers hold two sets of scores: take4(); not at D = 128 with a wave a stream, for which slots
//            of a whole page, as its two turns need them, would not fit
//   else     cached_keys4(), where four waves a SIMD overlap each other's turns and where a stream is short (LONG: see the launch)
// Two slots are enough for a page's turns: three and four gained nothing on either batch above.
template <int D, CacheType T, int RB, int PARTS, int WAVES, bool LONG>
struct Ring {
  static constexpr bool kSmall = D == 64 && RB == 1 && !(kFour<T> && LONG);  // four waves a SIMD, otherwise two
  static constexpr int kRow = kFour<T> ? D / 2 : D;                 // bytes of a token's codes
  static constexpr int kSpace = (kSmall ? 8192 : 16384) * PARTS;    // codes of 8 bits: 128 KiB a CU
  static constexpr bool kShared = kFour<T> && D == 128 && PARTS == 4;  // waves with different rows widen each key once between them
  static constexpr bool kPiped = kFour<T> && !kSmall && !kShared && !(D == 128 && PARTS == 1);
  static constexpr int kTokens = kFour<T> ? (PARTS == 1 && !kPiped ? 32 : 64) : kSpace >= 4 * 64 * D ? 64 : 32;
  static constexpr int kHalf = kTokens * kRow, kSlot = 2 * kHalf + (kFour<T> ? (kTokens * D / 32 > 128 ? 512 : 256) : 0);  // bytes of a slot's keys; in all, with scales
  static constexpr int kDepth = !kFour<T> ? kSpace / kSlot : D == 64 && RB == 2 ? 2 * PARTS : 2;  // slots
  static constexpr int kDataCopies = 2 * kHalf / 1024 / PARTS;      // of a slot, by each of its waves
  static constexpr int kCopies = kDataCopies + (!kFour<T> ? 0 : kTokens * D / 32 > 128 && PARTS == 1 ? 2 : 1);
  static constexpr int kTile = kFour<T> ? 64 * D : 0;               // 32 keys' values as bf16
  static constexpr int kMerge = PARTS * RB * 32 * D * 4;            // what the merge of the streams puts here
  static constexpr int kUsed = kShared ? 4 * kTile : kDepth * kSlot + PARTS * kTile;
  static constexpr int kBytes = kUsed > kMerge ? kUsed : kMerge;
};

// Workgroup = (share of the work, KV head).  A wave holds RB blocks of 32 of the K x Hq/Hkv query rows that share the KV head (row =
// depth * group + head); PARTS waves with different rows make a stream, and the streams take a request's pages in turn.  A stream
// has a ring of slots in LDS (a page each where the ring holds two, otherwise 32 tokens), filled by its waves some slots ahead of their
// use.  With one wave a stream (up to 32 rows, at D = 64 up to 64) a wave waits for its own copies only and the loop has no barrier;
// more rows share what a stream copies, which costs a barrier a slot.  At the end of a request's pages the streams' sums are merged
// through LDS, and leave the results where the request is one workgroup's, otherwise a partial record.
// Bound: memory (64 requests of 8192 tokens: 102 us on MI355X with 24 rows of 128 features, 5.3 TB/s), with 56 rows of 64 features
// vector issue beside it (121 us, 4.4 TB/s: 204 instructions a slot of 32 keys and 64 rows - a quarter of it exponentials - keep the vector
// units busy for 64 % of a wave's time, the 16 matrix instructions theirs for 34 %).
// In 4 bits the bytes are half of that and the instructions as many, and no unit alone bounds a batch.  64 requests of 512 to 8192 tokens,
// 56 rows of 64 features: 67 us a step (2.3 TB/s), without any copies 10 % less; 48 of 500 to 8191, 128 rows of 128 features: 83 us (1.5 TB/s).  Of
// the launch's cycles the vector units are busy for 60 and 46 %, the matrix units for 28 and 34 %; its waves are there for 86 and 96 % (starts,
// unequal ends), and wait for memory, LDS or a barrier 28 and 30 % of that, for issue 24 and 30 %; LDS conflicts are none.
template <int D, CacheType T, int RB, int PARTS, int WAVES, bool LONG = false>
__global__ __launch_bounds__(WAVES * 64, (Ring<D, T, RB, PARTS, WAVES, LONG>::kSmall ? 4 : 2)) void draft_scaled_kernel(ScaledDecodeParams sp) {
  constexpr int kWaves = WAVES, kStreams = kWaves / PARTS;
  using R = Ring<D, T, RB, PARTS, WAVES, LONG>;
  constexpr int kTokens = R::kTokens, kHalf = R::kHalf, kSlot = R::kSlot, kDepth = R::kDepth, kRow = R::kRow;
  constexpr int kPerPage = kKeysPerTile / kTokens;                            // slots of a page
  constexpr int kCopies = R::kCopies;                                         // of a slot, by each of a stream's waves
  constexpr int kAhead = PARTS == 1 ? kDepth : kDepth - 1;                    // slots on their way or in use
  __shared__ __attribute__((aligned(16))) char ring[kStreams][R::kBytes];     // slots and, with codes of 4 bits, the waves' tiles
  __shared__ f32x4 stats[kWaves][RB * 32];  // of each wave's rows: reference, the two sums
  __shared__ int far[kStreams][2][PARTS];   // a wave's share of the values in either tile has large scales
  __shared__ int wave_bad[kWaves];

  DecodeParams p = sp.d;
  p.q_new = held(p.q_new);
  p.k_new = held(p.k_new);
  p.v_new = held(p.v_new);
  p.block_table = held(p.block_table);
  p.ctx_len = held(p.ctx_len);
  p.o = held(p.o);
  p.lse = held(p.lse);
  p.status = held(p.status);
  p.part_o = held(p.part_o);
  p.part_ml = held(p.part_ml);
  p.C = held(p.C);
  p.K = held(p.K);
  p.Hq = held(p.Hq);
  p.Hkv = held(p.Hkv);
  p.n_pages = held(p.n_pages);
  p.max_pages = held(p.max_pages);
  p.rows_pad = held(p.rows_pad);
  p.group = held(p.group);
  p.group_reciprocal = held(p.group_reciprocal);
  p.c_log2 = held(p.c_log2);
  const uint8_t *k_pages = held(sp.k_pages), *v_pages = held(sp.v_pages), *k_scale = held(sp.k_scale), *v_scale = held(sp.v_scale);
  int2* pieces = held(sp.pieces);
  const int shares = held(sp.shares), least_share = held(sp.least_share), lead = held(sp.lead);

  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, g = lane >> 5, ln = lane & 31;
  const int kvh = blockIdx.y, part = wave % PARTS, stream = wave / PARTS, n_groups = gridDim.x;
  const int n_rows = p.K * p.group;

  Share s{0, (int)blockIdx.x, 0, 0, -64, true};
  int left = INT_MAX;
  if (shares > 0) {
    s = share_of(p.ctx_len, p.C, p.max_pages, blockIdx.x, shares, least_share, lead, lane);
    if (!s.any) return;
    left = s.share;
  }
  int c = s.c, skip = s.skip;

  int k_off[D / 32], v_off[D / 32];
  Off4<D> off4;
  char* const tile = &ring[stream][R::kShared ? 0 : kDepth * kSlot] + part * R::kTile;
  if constexpr (kFour<T>) {
    off4.tr = tr_offsets<D>(lane);
#pragma unroll
    for (int j = 0; j < D / 64; ++j) {
      const int vl = value_key<D>(ln);
      off4.codes[j] = ln * kRow + (((2 * j + g) ^ swz4<D>(ln)) << 4);
      off4.scale[j] = ln * (D / 32) + 2 * j + g;
      off4.v_codes[j] = vl * kRow + (((2 * j + g) ^ swz4<D>(vl)) << 4);
      off4.v_scale[j] = vl * (D / 32) + 2 * j + g;
#pragma unroll
      for (int w = 0; w < 4; ++w) off4.out[j][w] = tile_off<D>(vl, 4 * (2 * j + g) + w);
    }
  } else {
    const int i = lane & 15, row = 4 * g + (i >> 1 & 3) + (i >> 3) * 8;
#pragma unroll
    for (int j = 0; j < D / 32; ++j) {
      k_off[j] = ln * D + (((2 * j + g) ^ swz8<D>(ln)) << 4);
      v_off[j] = row * D + (((2 * j + (lane >> 4 & 1)) ^ swz8<D>(row)) << 4) + (i & 1) * 8;
    }
  }
  // Copies: lane l of the 1 KiB block b of a slot's half owns LDS bytes [1024 b + 16 l, + 16) and fetches the chunk that lives there.
  constexpr int kLanes = kRow / 16;  // of a row
  uint32_t voff[2];
#pragma unroll
  for (int b = 0; b < 2; ++b)
    voff[b] = (uint32_t)((lane / kLanes) * kRow + ((lane % kLanes ^ swz_codes<D, T>(b * (64 / kLanes) + lane / kLanes)) << 4));
  const uint32_t ring_at = lds_scalar_addr(&ring[stream][0]);
  // This wave's copies of a slot: f(values rather than keys?, block of 1 KiB).
  auto each_copy = [&](auto f) {
    constexpr int n = R::kDataCopies;
    if constexpr (PARTS == 1) {
#pragma unroll
      for (int b = 0; b < n / 2; ++b) f(false, b);
#pragma unroll
      for (int b = 0; b < n / 2; ++b) f(true, b);
    } else {
      const int b0 = part % (PARTS / 2) * n;
#pragma unroll
      for (int b = 0; b < n; ++b) f(part >= PARTS / 2, b0 + b);
    }
  };
  // Scales of a slot with codes of 4 bits, a word a lane: those of K and behind them those of V by one copy where they are 64 words or
  // fewer (every wave of a stream makes it, the same), otherwise by two, of which the waves that copy K make one.
  constexpr int kScaleWords = kTokens * (D / 32) / 4;
  const uint8_t* scale_at = nullptr;
  if constexpr (kFour<T>) scale_at = (kScaleWords <= 32 && lane / kScaleWords % 2 != 0 ? v_scale : k_scale) + lane % kScaleWords * 4;
  auto copy_scales = [&](size_t at, uint32_t dst) {
    if constexpr (kScaleWords <= 32) {
      dma4_untracked(scale_at + at, dst + 2 * kHalf);
    } else {
      const uint32_t off = (uint32_t)lane_id() * 4;
      if (PARTS == 1 || part < PARTS / 2) dma4_untracked(uniform_ptr(k_scale + at), off, dst + 2 * kHalf);
      if (PARTS == 1 || part >= PARTS / 2) dma4_untracked(uniform_ptr(v_scale + at), off, dst + 2 * kHalf + 4 * kScaleWords);
    }
  };

  for (int segment = 0;;) {
    int n_ctx;
    if ((unsigned)(c - s.lens_from) < 64u) n_ctx = __builtin_amdgcn_readlane(s.lens, c - s.lens_from);
    else n_ctx = __builtin_amdgcn_readfirstlane(p.ctx_len[c + (lane_id() & 0)]);  // (by a vector load: no scalar one in a loop)
    bool bad = n_ctx < 0 || n_ctx > p.max_pages * kKeysPerTile;
    n_ctx = clamp_len(n_ctx, p.max_pages);
    const int n_pg = pages_of(n_ctx), units = lead + n_pg + 1;
    const int n_units = units - skip < left ? units - skip : left, to = skip + n_units;
    if (to <= lead) return;  // (the share ends before the request's pages)
    const int p0 = skip > lead ? skip - lead : 0, p1 = to - lead < n_pg ? to - lead : n_pg;
    const bool has_start = skip <= lead, has_new = to == units, whole = has_start && has_new;

    Rows<D, RB> r;
    int depth[RB];
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
#pragma unroll
      for (int db = 0; db < D / 32; ++db) r.o[rb][db] = zero16();
      r.m[rb] = -3.402823466e38f;  // (any score is above it, and it less any score is no NaN)
      r.l[rb] = r.w[rb] = 0.f;
    }
    auto load_queries = [&] {
      const int l = lane_id();
#pragma unroll
      for (int rb = 0; rb < RB; ++rb) {
        const int row = (part * RB + rb) * 32 + (l & 31);
        depth[rb] = row < n_rows ? small_quotient(row, p.group_reciprocal) : 0;
        const int head = kvh * p.group + (row < n_rows ? row - depth[rb] * p.group : 0);
        const __bf16* q = p.q_new + (((size_t)c * p.K + depth[rb]) * p.Hq + head) * D + 8 * q_chunk<T, R::kShared>(0, 1) * (l >> 5);
#pragma unroll
        for (int i = 0; i < D / 16; ++i) r.q[rb][i] = as_frag(ld16(q + 8 * q_chunk<T, R::kShared>(i, 0)));
      }
    };

    // The last stream has the new keys first: in its first slots or, with codes of 4 bits, in its waves' tiles.
    const int n_new = has_new ? (p.K + kNewKeys - 1) / kNewKeys : 0, my_new = stream == kStreams - 1 ? n_new : 0;
    const size_t new_at = ((size_t)c * p.K * p.Hkv + kvh) * D;
    const __bf16* k_new = uniform_ptr(p.k_new + new_at);
    const __bf16* v_new = uniform_ptr(p.v_new + new_at);
    const int n_pages_0 = (p1 - p0 + kStreams - 1) / kStreams;  // pages of stream 0, the most
    const int n_mine = p1 - p0 > stream ? (p1 - p0 - stream + kStreams - 1) / kStreams : 0;

    // This stream's pages, 64 at a time, one a lane: page, keys present (0: page id outside the pool), scales.  With them their
    // copies are begun: slots [0, q0) hold new keys, n_q slots in all.
    int page, keys, kcode, vcode, q0, n_q, issued;
    auto copy = [&](int q) {
      const uint32_t dst = ring_at + (uint32_t)q % kDepth * kSlot;
      if (!kFour<T> && q < q0) {
        const int l = lane_id();
        each_copy([&](bool half, int b) {
          const int row = b * (512 / D) + l / (D / 8), key = q * kNewKeys + row;
          const uint32_t off = (uint32_t)(key < p.K ? key : p.K - 1) * (uint32_t)(p.Hkv * D * 2) + ((l % (D / 8) ^ swz<D>(row)) << 4);
          dma16_untracked(half ? v_new : k_new, off, dst + (half ? kHalf : 0) + b * 1024);
        });
        return;
      }
      const int j = (q - q0) / kPerPage, sub = (q - q0) % kPerPage;
      const size_t page_head = (size_t)(uint32_t)__builtin_amdgcn_readlane(page, j) * p.Hkv + kvh;
      const size_t at = page_head * (kKeysPerTile * kRow) + sub * kHalf;
      if constexpr (kFour<T>) copy_scales((page_head * kKeysPerTile + sub * kTokens) * (D / 32), dst);
      const int present = __builtin_amdgcn_readlane(keys, j) - sub * kTokens;
      if (present >= kTokens) {
        each_copy([&](bool half, int b) {
          dma16_untracked(uniform_ptr((half ? v_pages : k_pages) + at) + b * 1024, voff[b & 1], dst + (half ? kHalf : 0) + b * 1024);
        });
      } else {  // rows behind the last token are read as that token, and masked
        const int last = present > 0 ? present - 1 : 0, l = lane_id();
        each_copy([&](bool half, int b) {
          const int row = b * (64 / kLanes) + l / kLanes;
          const uint32_t off = (uint32_t)((row < last ? row : last) * kRow + ((l % kLanes ^ swz_codes<D, T>(row)) << 4));
          dma16_untracked(uniform_ptr((half ? v_pages : k_pages) + at), off, dst + (half ? kHalf : 0) + b * 1024);
        });
      }
    };
    auto take_pages = [&](int first, int n_before) {
      const int pi = p0 + stream + kStreams * (first + lane_id());
      const bool there = pi < p1;
      page = there ? p.block_table[(size_t)c * p.max_pages + pi] : 0;
      if (first == 0) {  // (what the lookup of the pages takes, the queries take too)
        __builtin_amdgcn_sched_barrier(0);
        load_queries();
      }
      const bool fine = page >= 0 && page < p.n_pages;
      bad |= !fine;
      page = fine ? page : 0;
      const int keys_here = n_ctx - pi * kKeysPerTile;
      keys = !there || !fine ? 0 : keys_here < kKeysPerTile ? keys_here : kKeysPerTile;
      kcode = vcode = 0;
      if (!kFour<T> && there) {
        kcode = k_scale[(size_t)page * p.Hkv + kvh];
        vcode = v_scale[(size_t)page * p.Hkv + kvh];
      }
      const int n_here = n_mine - first < 64 ? n_mine - first : 64;
      q0 = kFour<T> ? 0 : n_before;
      n_q = R::kShared ? 0 : q0 + (n_here > 0 ? n_here * kPerPage : 0);  // (none where waves load their shares)
      // (one slot's copies with the loads: behind more, the wait for the loads would be one for the slots that are due later)
      issued = 0;
      if (n_q > 0) copy(issued++);
      __builtin_amdgcn_s_waitcnt(0x0F70);  // (the compiler's own loads: none is waited for in the loop, behind its copies)
      for (; issued < kAhead && issued < n_q; ++issued) copy(issued);
    };
    // A slot's turn: what it holds has landed; with several waves a stream, everyone is done with the slot before it, which is
    // filled again.
    auto begin = [&](int q) {
      if constexpr (R::kPiped) {  // (fewer than kAhead - 1 slots behind this one are only its last ones)
        if (issued - 1 - q >= kAhead - 1) wait_outstanding<(kAhead - 1) * kCopies>();
        else wait_outstanding<0>();
      } else {
        wait_slots<kAhead - 1, kCopies>(issued - 1 - q);
      }
      if (PARTS > 1) {
        __syncthreads();
        if (issued < n_q) copy(issued++);
      }
    };
    auto end = [&] {
      if (PARTS > 1) return;
      asm volatile("s_waitcnt lgkmcnt(0)" : : : "memory");  // the slot's last reads have left it
      if (issued < n_q) copy(issued++);
    };

    const uint32_t tile_at = ring_at + (uint32_t)((R::kShared ? 0 : kDepth * kSlot) + part * R::kTile);
    auto copy_new = [&](int i) {  // sixteen new keys to this wave's tile, K rows of 2 D bytes, V behind them
      const int l = lane_id();
#pragma unroll
      for (int b = 0; b < D / 16; ++b) {
        const int row = b % (D / 32) * (512 / D) + l / (D / 8), key = i * kNewKeys + row;
        const uint32_t off = (uint32_t)(key < p.K ? key : p.K - 1) * (uint32_t)(p.Hkv * D * 2) + ((l % (D / 8) ^ swz<D>(row)) << 4);
        dma16_untracked(b >= D / 32 ? v_new : k_new, off, tile_at + b * 1024);
      }
    };
    if (kFour<T> && my_new > 0) copy_new(0);
    take_pages(0, my_new);
    int q = 0;
    if constexpr (kFour<T>) {
      for (int i = 0; i < my_new; ++i) {
        if (i == 0) {
          wait_slots<kAhead, kCopies>(issued);
        } else {
          asm volatile("s_waitcnt lgkmcnt(0)" : : : "memory");  // the tile's last reads have left it
          copy_new(i);
          wait_outstanding<0>();
        }
        new_keys<D, T, RB, R::kShared>(r, tile, tile + kNewKeys * 2 * D, i * kNewKeys, p.K, v_new, (uint32_t)(p.Hkv * D), depth, p.c_log2);
      }
      asm volatile("" : : : "memory");
    }
    // (where streams meet at barriers, the others wait for the new keys' turns)
    for (int i = 0; !kFour<T> && i < (PARTS > 1 ? n_new : my_new); ++i) {
      if (my_new > 0) begin(q);
      else if (PARTS > 1) __syncthreads();
      if (my_new > 0) {
        const char* at = &ring[stream][(uint32_t)q % kDepth * kSlot];
        new_keys<D, T, RB, false>(r, at, at + kHalf, q * kNewKeys, p.K, v_new, (uint32_t)(p.Hkv * D), depth, p.c_log2);
        end();
        ++q;
      }
    }
    for (int first = 0;;) {
      if constexpr (R::kShared) {
        const int n = n_pages_0 - first < 64 ? n_pages_0 - first : 64;
        const Share4 mine(part, lane_id());
        const NatOff<D> nat = nat_offsets<D>(lane_id());
        char* const tiles = &ring[stream][0];
        auto k_tile = [&](int b) { return tiles + b * R::kTile; };
        auto v_tile = [&](int b) { return tiles + (2 + b) * R::kTile; };
        auto load = [&](Raw4& x, int u, const uint8_t* pages, const uint8_t* scales) {  // of 32 keys u
          u = u < 2 * n ? u : u % 2;  // (always a load, so that what is under way can be counted)
          const size_t page_head = (size_t)(uint32_t)__builtin_amdgcn_readlane(page, u / 2) * p.Hkv + kvh;
          load_share(x, uniform_ptr(pages + page_head * (64 * kRow) + u % 2 * (32 * kRow)),
                     uniform_ptr(scales + page_head * (2 * D) + u % 2 * D), mine);
        };
        auto keys_of = [&](int u) { return __builtin_amdgcn_readlane(keys, u / 2) - u % 2 * 32; };
        auto put = [&](const Raw4& x, char* to) {
#pragma unroll
          for (int i = 0; i < 2; ++i) put_share(x, to, mine, i);
        };
        auto put_values = [&](Raw4& x, int u, int b) {
          keep_first(x, mine, keys_of(u));
          const int large = far_scale(x);
          put(x, v_tile(b));
          if (lane == 0) far[stream][b][part] = large;
        };
        if (n > 0) {
          Raw4 kr[2], vr[2];
          load(kr[0], 0, k_pages, k_scale);
          load(vr[0], 0, v_pages, v_scale);
          load(kr[1], 1, k_pages, k_scale);
          load(vr[1], 1, v_pages, v_scale);
          meet();  // (new keys, and what was here before, have been read)
          put(kr[0], k_tile(0));
          put_values(vr[0], 0, 0);
          put(kr[1], k_tile(1));
          load(kr[0], 2, k_pages, k_scale);
          load(kr[1], 3, k_pages, k_scale);
          load(vr[0], 2, v_pages, v_scale);
          meet();
          f32x16 sa, sb;
#pragma unroll
          for (int i = 0; i < D / 16; ++i) sa = mfma32(frag_nat<D>(k_tile(0), nat, 0, i), r.q[0][i], i == 0 ? zero16() : sa);
          // One turn: keys u weigh the output, the scores of keys u + 1 are formed, keys u + 2 and the values of keys u + 1 widened.
          // What is behind the last keys is what has been before, and counts nowhere.
          auto turn = [&](auto b_, int u, f32x16& s, f32x16& s_next) {
            constexpr int b = decltype(b_)::value, kSteps = D / 16, kFrags = D / 32;
            meet();
            int any_far = 0;
#pragma unroll
            for (int i = 0; i < PARTS; ++i) any_far |= far[stream][b][i];
            bf16x8 kf[2], vf[2][kFrags];
            kf[0] = frag_nat<D>(k_tile(1 - b), nat, 0, 0);
            kf[1] = frag_nat<D>(k_tile(1 - b), nat, 0, 1);
            const int n_keys = keys_of(u);
            if (n_keys < 32) {
              const uint32_t bits = n_keys <= 0 ? 0u : ((1u << n_keys) - 1) >> (4 * g);
#pragma unroll
              for (int i = 0; i < 16; ++i) s[i] = mask_sel(s[i], bits, 8 * (i / 4) + (i % 4));
            }
            float x[16], sum[4];
            auto weigh = [&](int from, int to) {
#pragma unroll
              for (int i = from; i < to; ++i) {
                const float e = exp2_fast(__builtin_fmaf(s[i], p.c_log2, -r.m[0]));
                asm volatile("" : : "v"(e));  // (here, not where it is used: the compiler gathers what it may behind the fences)
                x[i] = e;
                sum[i % 4] = i < 4 ? e : sum[i % 4] + e;
              }
            };
            __builtin_amdgcn_s_setprio(1);  // (1 % here)
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int i = 0; i < kSteps; ++i) {
              s_next = mfma32(kf[i % 2], r.q[0][i], i == 0 ? zero16() : s_next);
              if (i + 2 < kSteps) kf[i % 2] = frag_nat<D>(k_tile(1 - b), nat, 0, i + 2);
              weigh(2 * i, 2 * i + 2);
              if (i % (kSteps / 2) == 0) put_share(kr[b], k_tile(b), mine, i / (kSteps / 2));
              __builtin_amdgcn_sched_barrier(0);
            }
#pragma unroll
            for (int db = 0; db < kFrags; ++db) vf[0][db] = frag_tr<D>(v_tile(b), off4.tr, 0, db);
            __builtin_amdgcn_s_setprio(0);
            load(kr[b], u + 4, k_pages, k_scale);
            const float limit = __builtin_amdgcn_ballot_w64(any_far != 0) != 0 ? kNearLimit : kFarLimit;
            float total = (sum[0] + sum[1]) + (sum[2] + sum[3]);
            if (__builtin_expect(__builtin_amdgcn_ballot_w64(total > limit) != 0, 0)) {
              const float mx = max_halves(max16(s)) * p.c_log2;
              const bool need = max_halves(total) > limit && mx > r.m[0];
              const float m_new = need ? mx : r.m[0], alpha = exp2_fast(r.m[0] - m_new);
              r.m[0] = m_new;
              r.l[0] *= alpha;
              r.w[0] *= alpha;
#pragma unroll
              for (int db = 0; db < kFrags; ++db)
#pragma unroll
                for (int i = 0; i < 16; ++i) r.o[0][db][i] *= alpha;
              weigh(0, 16);
              total = (sum[0] + sum[1]) + (sum[2] + sum[3]);
            }
            r.l[0] += total;
            bf16x8 pb[2];
#pragma unroll
            for (int t = 0; t < 2; ++t) {
              u32x4 w;
#pragma unroll
              for (int i = 0; i < 4; ++i) {
                w[i] = pack_bf16(x[8 * t + 2 * i], x[8 * t + 2 * i + 1]);
                r.w[0] = add_pair_bf16(w[i], r.w[0]);
              }
              pb[t] = __builtin_bit_cast(bf16x8, w);
            }
            keep_first(vr[1 - b], mine, keys_of(u + 1));
            const int large = far_scale(vr[1 - b]);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int db = 0; db < kFrags; ++db) vf[1][db] = frag_tr<D>(v_tile(b), off4.tr, 16, db);
#pragma unroll
            for (int k = 0; k < 2 * kFrags; ++k) {
              r.o[0][k % kFrags] = mfma32(vf[k / kFrags][k % kFrags], pb[k / kFrags], r.o[0][k % kFrags]);
              if (k % kFrags == 0) put_share(vr[1 - b], v_tile(1 - b), mine, k / kFrags);
              __builtin_amdgcn_sched_barrier(0);
            }
            if (lane == 0) far[stream][1 - b][part] = large;
            load(vr[1 - b], u + 3, v_pages, v_scale);
          };
          for (int u = 0; u < 2 * n; u += 2) {
            turn(std::integral_constant<int, 0>(), u, sa, sb);
            turn(std::integral_constant<int, 1>(), u + 1, sb, sa);
          }
        }
        meet();  // (the tiles' last reads have left them)
        first += 64;
        if (first >= n_pages_0) break;
        take_pages(first, 0);
        continue;
      }
      if constexpr (R::kPiped) {
        // A slot is a page, a page two turns.  Its second half is read when the first one's turn begins, and its slot filled again
        // when that has arrived.
        static_assert(kTokens == 64, "");
        const int n = PARTS > 1 ? (n_pages_0 - first < 64 ? n_pages_0 - first : 64) : n_q;
        Keys4<D> x;
        auto load = [&](int j, int half) {
          const char* slot = &ring[stream][(uint32_t)j % kDepth * kSlot];
          const char* scales = slot + 2 * kHalf + half * D;
          load4(x, slot + half * 32 * kRow, slot + kHalf + half * 32 * kRow, scales, scales + 4 * kScaleWords, off4);
        };
        f32x16 sa[RB], sb[RB];
        Held4<D> held{};
        float limit_a = kFarLimit, limit_b = kFarLimit;
        if (n > 0) {
          int keys_here = __builtin_amdgcn_readlane(keys, 0);
          begin(0);
          load(0, 0);
          scores4(x, r, sa);
          limit_a = values4(x, tile, off4, keys_here, ln);
          load(0, 1);
          // (the last turn's next keys are such as have been before, and count nowhere)
          for (int j = 0; j < n; ++j) {
            take4<D, RB>(r, sa, sb, x, held, tile, off4, keys_here, limit_a, g, p.c_log2);
            limit_b = values4(x, tile, off4, keys_here - 32, ln);
            end();
            const int keys_next = __builtin_amdgcn_readlane(keys, j + 1);
            if (j + 1 < n) {
              begin(j + 1);
              load(j + 1, 0);
            }
            take4<D, RB>(r, sb, sa, x, held, tile, off4, keys_here - 32, limit_b, g, p.c_log2);
            limit_a = values4(x, tile, off4, keys_next, ln);
            if (j + 1 < n) load(j + 1, 1);
            keys_here = keys_next;
          }
          if (RB == 2) {
#pragma unroll
            for (int k = 0; k < D / 16; ++k) r.o[RB - 1][k % (D / 32)] = mfma32(held.v[k / (D / 32)][k % (D / 32)], held.p[k / (D / 32)], r.o[RB - 1][k % (D / 32)]);
          }
        }
        if (PARTS > 1) __syncthreads();  // (the slots' last reads have left them)
        first += 64;
        if (first >= n_pages_0) break;
        take_pages(first, 0);
        q = 0;
        continue;
      }
      const int rounds = PARTS > 1 ? (n_pages_0 - first < 64 ? n_pages_0 - first : 64) * 2 : (n_q - q0) * (kTokens / 32);
      for (int i = 0; i < rounds; ++i) {
        const bool starts = kTokens == 32 || i % 2 == 0, ends = kTokens == 32 || i % 2 != 0;  // a slot's turn
        if (starts) begin(q);
        const int j = i / 2, n = __builtin_amdgcn_readlane(keys, j) - i % 2 * 32;  // (0 behind this stream's pages)
        const char* slot = &ring[stream][(uint32_t)q % kDepth * kSlot];
        const int half = kTokens == 32 ? 0 : i % 2;
        const char* at = slot + half * 32 * kRow;
        if constexpr (kFour<T>) {
          const char* scales = slot + 2 * kHalf + half * D;
          if (n > 0) cached_keys4<D, RB>(r, at, at + kHalf, scales, scales + 4 * kScaleWords, tile, off4, n, ln, g, p.c_log2);
        } else {
          const float ks = __builtin_bit_cast(float, __builtin_amdgcn_readlane(kcode, j) << 23);
          const int v_code = __builtin_amdgcn_readlane(vcode, j);
          const float vs = __builtin_bit_cast(float, v_code << 23), limit = v_code > kFarScale ? kNearLimit : kFarLimit;
          if (n > 0) cached_keys<D, T, RB>(r, at, at + kHalf, k_off, v_off, ks, vs, limit, n, g, p.c_log2);
        }
        if (ends) {
          end();
          ++q;
        }
      }
      if (PARTS > 1) __syncthreads();  // (the slots' last reads have left them)
      first += 64;
      if (first >= n_pages_0) break;
      take_pages(first, 0);
      q = 0;
    }

    // Merge of the streams' waves with the same rows.  Each leaves its references and sums, learns the common ones, leaves its O
    // against those (in its part of the rings, 16 bytes of features by 16 bytes, the rows of feature group d4 in the order row ^ d4),
    // and the threads add them up in order.
    const int l = lane_id();
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
      const float a = sum_halves(r.l[rb]), b = sum_halves(r.w[rb]);
      if (l < 32) stats[wave][rb * 32 + l] = f32x4{r.m[rb], a, b, 0.f};
    }
    if (l == 0) wave_bad[wave] = 0;
    if (__builtin_amdgcn_ballot_w64(bad) != 0 && l == 0) wave_bad[wave] = 1;
    __syncthreads();
    int any_bad = 0;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) any_bad |= wave_bad[w];
    const size_t rec = ((size_t)kvh * n_groups + blockIdx.x) * 2 + (segment > 0 ? 1 : 0);
    constexpr int kRegion = RB * 32 * D / 4;
    static_assert(kWaves * kRegion * 16 <= (int)sizeof(ring), "the rows' O must fit a wave's part of the rings");
    f32x4* regions = reinterpret_cast<f32x4*>(&ring[0][0]);
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
      const int at = rb * 32 + (l & 31), row = part * RB * 32 + at;
      float M = r.m[rb], L = 0.f, W = 0.f;
#pragma unroll
      for (int i = 0; i < kStreams; ++i) M = __builtin_fmaxf(M, stats[i * PARTS + part][at][0]);
#pragma unroll
      for (int i = 0; i < kStreams; ++i) {
        const f32x4 x = stats[i * PARTS + part][at];
        const float f = exp2_fast(x[0] - M);
        L = __builtin_fmaf(x[1], f, L);
        W = __builtin_fmaf(x[2], f, W);
      }
      if (stream == 0 && l < 32) {
        if (whole) {
          if (row < n_rows) {
            const int dep = small_quotient(row, p.group_reciprocal), head = kvh * p.group + (row - dep * p.group);
            p.lse[((size_t)c * p.Hq + head) * p.K + dep] = (M + __builtin_log2f(L)) * kLn2;
          }
        } else if (row < p.rows_pad) {
          reinterpret_cast<f32x4*>(p.part_ml)[rec * p.rows_pad + row] = f32x4{M, L, W, any_bad ? 1.f : 0.f};
        }
      }
      const float turn = exp2_fast(r.m[rb] - M) * (whole ? 1.0f / W : 1.0f);
#pragma unroll
      for (int db = 0; db < D / 32; ++db)
#pragma unroll
        for (int i4 = 0; i4 < 4; ++i4) {
          const int d4 = db * 8 + 2 * i4 + (l >> 5);
          const f32x16& o = r.o[rb][db];
          regions[wave * kRegion + (rb * (D / 4) + d4) * 32 + ((l ^ d4) & 31)] =
              f32x4{o[4 * i4] * turn, o[4 * i4 + 1] * turn, o[4 * i4 + 2] * turn, o[4 * i4 + 3] * turn};
        }
    }
    __syncthreads();
    constexpr int kItems = 32 * RB * PARTS * (D / 4) / (kWaves * 64);
#pragma unroll 4
    for (int k = 0; k < kItems; ++k) {
      const int item = (k * kWaves + wave) * 64 + l;
      const int d4 = item % (D / 4), row = item / (D / 4), at = row % (RB * 32), h = row / (RB * 32);
      f32x4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int i = 0; i < kStreams; ++i) o += regions[(i * PARTS + h) * kRegion + (at / 32 * (D / 4) + d4) * 32 + ((at ^ d4) & 31)];
      if (whole) {
        if (row < n_rows) {
          const int dep = small_quotient(row, p.group_reciprocal), head = kvh * p.group + (row - dep * p.group);
          u32x2 out;
          out[0] = pack_bf16(o[0], o[1]);
          out[1] = pack_bf16(o[2], o[3]);
          *reinterpret_cast<u32x2*>(p.o + (((size_t)c * p.K + dep) * p.Hq + head) * D + d4 * 4) = out;
        }
      } else if (row < p.rows_pad) {
        *reinterpret_cast<f32x4*>(p.part_o + (rec * p.rows_pad + row) * D + d4 * 4) = o;
      }
    }
    if (tid == 0 && kvh == 0) {
      if (whole && p.status) p.status[c] = any_bad;
      // where the request's records stand: the first, and how many workgroups leave one
      if (s.share > 0 && has_start) pieces[c] = make_int2((int)blockIdx.x * 2 + (segment > 0 ? 1 : 0), 1 + (units - to + s.share - 1) / s.share);
    }
    ++segment;
    left -= n_units;
    skip = 0;
    if (shares == 0 || ++c >= p.C || left <= 0) return;
    __syncthreads();  // the merge's reads have left the rings
  }
}

// Merges a request's partial records: M = max m_s, each sum and O the sum of the records' times 2^(m_s - M).  A row's threads - D / 4
// for its features, LANES of them for the records in turn - look at EACH records at a time, whose loads are issued before the
// first is used.  With more LANES than a wave has for a row, four waves take it and are merged through LDS.
template <int D, int LANES>
constexpr int kMergeRows = 256 / (D / 4 * LANES);  // of a workgroup
template <int D, int LANES, int EACH>
__global__ __launch_bounds__(256) void draft_scaled_combine_kernel(ScaledDecodeParams sp) {
  constexpr int kWaveLanes = D / 4 * LANES > 64 ? 256 / D : LANES;  // of a row in one wave
  static_assert(kWaveLanes == LANES || kMergeRows<D, LANES> == 1, "");
  const DecodeParams& p = sp.d;
  const int d4 = threadIdx.x % (D / 4), sl = threadIdx.x / (D / 4) % LANES;
  const int kvh = blockIdx.y, c = blockIdx.z, n_rows = p.K * p.group;
  const int2 piece = sp.pieces[c];
  const int n = piece.y;
  if (n <= 1) return;  // (its workgroup has left the results)
  const int row = (int)blockIdx.x * kMergeRows<D, LANES> + (int)threadIdx.x / (D / 4 * LANES);
  if (row >= n_rows) return;
  // record 0 may be its workgroup's second, the others are their workgroups' first
  const size_t rec0 = (size_t)kvh * sp.shares * 2;
  auto record = [&](int s) { return rec0 + (s == 0 ? piece.x : (piece.x / 2 + s) * 2); };
  float M = -3.402823466e38f, L = 0.f, W = 0.f;
  f32x4 acc = {0.f, 0.f, 0.f, 0.f};
  int bad = 0;
  for (int s0 = 0; s0 < n; s0 += LANES * EACH) {
    f32x4 ml[EACH], ov[EACH];
#pragma unroll
    for (int j = 0; j < EACH; ++j) {
      if (s0 + j * LANES >= n) continue;
      const int s = s0 + j * LANES + sl;  // (past the last it is read again)
      const size_t at = record(s < n ? s : n - 1) * p.rows_pad + row;
      ml[j] = reinterpret_cast<const f32x4*>(p.part_ml)[at];
      ov[j] = *reinterpret_cast<const f32x4*>(p.part_o + at * D + d4 * 4);
    }
    float m_new = M;
#pragma unroll
    for (int j = 0; j < EACH; ++j)
      if (s0 + j * LANES < n) m_new = __builtin_fmaxf(m_new, ml[j][0]);
    const float turn = exp2_fast(M - m_new);
    M = m_new;
    L *= turn;
    W *= turn;
    acc *= turn;
#pragma unroll
    for (int j = 0; j < EACH; ++j) {
      if (s0 + j * LANES + sl < n) {  // (not by a weight of zero: a record may hold infinities)
        const float w = exp2_fast(ml[j][0] - M);
        L = __builtin_fmaf(ml[j][1], w, L);
        W = __builtin_fmaf(ml[j][2], w, W);
        acc += ov[j] * w;
        bad |= ml[j][3] != 0.f;
      }
    }
  }
#pragma unroll
  for (int x = D / 4; x < D / 4 * kWaveLanes; x <<= 1) {
    const float m_other = __shfl_xor(M, x), m_new = __builtin_fmaxf(M, m_other);
    const float a = exp2_fast(M - m_new), b = exp2_fast(m_other - m_new);
    M = m_new;
    L = L * a + __shfl_xor(L, x) * b;
    W = W * a + __shfl_xor(W, x) * b;
#pragma unroll
    for (int j = 0; j < 4; ++j) acc[j] = acc[j] * a + __shfl_xor(acc[j], x) * b;
    bad |= __shfl_xor(bad, x);
  }
  if constexpr (kWaveLanes < LANES) {
    __shared__ f32x4 sums[256 / 64], parts[256 / 64][D / 4];
    const int wave = threadIdx.x >> 6;
    if (sl % kWaveLanes == 0) {
      parts[wave][d4] = acc;
      if (d4 == 0) sums[wave] = f32x4{M, L, W, bad ? 1.f : 0.f};
    }
    __syncthreads();
    if (sl != 0) return;
#pragma unroll
    for (int i = 1; i < 256 / 64; ++i) {
      const f32x4 x = sums[i], o = parts[i][d4];
      const float m_new = __builtin_fmaxf(M, x[0]), a = exp2_fast(M - m_new), b = exp2_fast(x[0] - m_new);
      M = m_new;
      L = L * a + x[1] * b;
      W = W * a + x[2] * b;
#pragma unroll
      for (int j = 0; j < 4; ++j) acc[j] = acc[j] * a + o[j] * b;
      bad |= x[3] != 0.f;
    }
  }
  if (sl != 0) return;
  if (p.status && row == 0 && kvh == 0 && d4 == 0) p.status[c] = bad;
  const float inv = 1.0f / W;
  const int depth = small_quotient(row, p.group_reciprocal), head = kvh * p.group + (row - depth * p.group);
  u32x2 out;
  out[0] = pack_bf16(acc[0] * inv, acc[1] * inv);
  out[1] = pack_bf16(acc[2] * inv, acc[3] * inv);
  *reinterpret_cast<u32x2*>(p.o + (((size_t)c * p.K + depth) * p.Hq + head) * D + d4 * 4) = out;
  if (d4 == 0) p.lse[((size_t)c * p.Hq + head) * p.K + depth] = (M + __builtin_log2f(L)) * kLn2;
}

constexpr int kCus = 256;  // compute units of the device

}  // namespace

// How the work of a KV head is shared, from the sizes that the host knows; times as microseconds a step on MI355X, D 64, 8 heads
// of keys, 7 or 8 rows a position unless noted.
//   lead   the start of a request's part (table, queries, merge) takes as long as some 8 pages: with 4 or 16 4 requests of 2048 to
//          4096 take 16.6 or 15.3 instead of 14.7, 48 of 500 to 8191 (D 128, 128 rows) 95.8 or 96.3 instead of 91.  (On 4 bits, where a page
//          takes less, 12 would be better by up to 5 % for nine of twelve sizes, and worse by 1, 1 and 6 % for three.)
//   least  two pages a stream, so that each wave has copies under way while it works.
//   By request, without the second launch: where one request's pages are too few to divide (at most two a stream), and where
//          eight a stream or fewer meet half the CUs' worth of workgroups: 14.8 against 21.1 for 16 requests of 1000 tokens, 22.0
//          against 33.0 for 32 of 1000 to 2000; sixteen a stream would help some (51.7 against 57.5 for 64 of 300 to 4000) and
//          cost others (33.5 against 28.5 for 16 of 2500 to 4000).  With fewer workgroups the pages are divided (D 128, 4 requests
//          of 768 tokens: 14.1 against 15.8).
//   shares a workgroup on each CU while each would have fewer than 12 units with two a CU, as the starts and the records weigh
//          more than the reads in flight: 16.1 against 18.8 for 4 requests of 2048 to 4096, 21.9 against 25.9 for 2 of 10800 to
//          20000 (D 128), 17.5 against 20.3 for one of 20000.  Above that D 64 takes two a CU: 89.7 against 95.6 for 64 of 512 to
//          8192.
//   waves  D 128 takes one workgroup of eight waves a CU there instead, which leaves half the records: 48 of 500 to 8191 (128
//          rows) 91 against 95, 64 of 8192 (24 rows) 102 against 116.  (D 64: 84 against 80, by request too, as its starts find no other
//          workgroup to work meanwhile.)  By request likewise where a CU gets one workgroup anyway: 40 of 300 to 2000 with 24 rows 16.7
//          against 18.7, with 128 rows 27.5 against 26.9; with several for each CU two side by side are better: 100 of 100 to 1000
//          with 128 rows 27.9 against 33.9.
//   C > 1024   by request, as every workgroup would look through all lengths: 120 against 132 for 2000 of 500 to 3000 with one KV head, no
//          difference with several.  A long request among short ones pays for it: 135 against 57 for one of 20000 among 1500 of 100 to 1000.
// The rule sees the table's width; lengths are on the device.  In a table wider than they need, shares and their merge are taken where
// a workgroup for each request would be faster: with 320 columns 17.7 instead of 12.5 for 16 of 1000, 26.3 instead of 18.8 for 32 of
// 1000 to 2000, 17.7 instead of 13.6 for 4 of 2048 to 4096 (two workgroups a CU instead of one); nothing for 64 of 512 to 8192.  (4 bits:
// 18.8 instead of 13.6, 26.4 instead of 20.2, 18.1 instead of 14.8, nothing.)
ShareRule draft_scaled_rule(int C, int Hkv, int max_pages, int blocks, int D) {
  ShareRule r;
  r.waves = D == 64 && blocks == 1 ? 8 : 4;
  // Streams that these waves make: a block of rows, at D = 64 two, is a wave's.
  int streams = r.waves / (D == 64 ? (blocks + 1) / 2 : blocks == 3 ? 4 : blocks);
  r.least = 2 * streams;
  r.lead = 8;
  r.shares = 0;
  const int64_t most = (int64_t)C * (max_pages + r.lead + 1);  // units of a KV head
  if (C > 1024 || max_pages <= 2 * streams || most > 1 << 30) return r;
  if (max_pages <= 8 * streams && (int64_t)C * Hkv >= kCus / 2) {
    if (D == 128 && (int64_t)C * Hkv <= kCus) r.waves = 8;
    return r;
  }
  const bool large = most * Hkv >= 12 * 2 * kCus;
  if (D == 128 && large) {
    r.waves = 8;
    r.least *= 2;
  }
  const int64_t wgs = large && D == 64 ? 2 * kCus : kCus;
  const int64_t slots = (wgs + Hkv - 1) / Hkv, useful = (most + r.least - 1) / r.least;
  r.shares = (int)(slots < useful ? slots : useful);
  return r;
}

hipError_t launch_draft_scaled(const ScaledDecodeParams& pin, int D, CacheType cache, hipStream_t stream) {
  ScaledDecodeParams p = pin;
  p.d.group = p.d.Hq / p.d.Hkv;
  p.d.group_reciprocal = small_reciprocal(p.d.group);
  const int blocks = p.d.rows_pad / 32;
  const ShareRule rule = draft_scaled_rule(p.d.C, p.d.Hkv, p.d.max_pages, blocks, D);
  p.shares = rule.shares;
  p.least_share = rule.least;
  p.lead = rule.lead;
  const dim3 grid((unsigned)(p.shares > 0 ? p.shares : p.d.C), (unsigned)p.d.Hkv);
  // With a workgroup a CU at most, two blocks of rows at D = 64 are two waves' rather than one's: what a wave does for a slot is
  // the time then (15.0 against 15.9 us for 4 requests of 2048 to 4096 tokens).  With more, widening each value once counts (91
  // against 94 us for 64 of 512 to 8192).  With codes of 4 bits such a workgroup takes the turns that overlap where it has a whole request
  // (20.4 us, otherwise 21.5, for 30 of 1000 to 2000 tokens), and not where it has a page or two a stream (15.0, otherwise 14.5, for 4 of
  // 2048 to 4096).
  const bool alone = (int64_t)grid.x * grid.y <= kCus;
  auto go = [&](auto type) {
    constexpr CacheType T = decltype(type)::value;
    constexpr bool four = T == CacheType::kE2M1;
    auto run = [&](auto kernel, int waves) { hipLaunchKernelGGL(kernel, grid, dim3((unsigned)waves * 64), 0, stream, p); };
    if (D == 64) {
      if (blocks == 1) run(draft_scaled_kernel<64, T, 1, 1, 8>, 8);
      else if (blocks == 2 && alone && four && p.shares == 0) run(draft_scaled_kernel<64, T, 1, 2, 8, four>, 8);
      else if (blocks == 2 && alone) run(draft_scaled_kernel<64, T, 1, 2, 8>, 8);
      else if (blocks == 2) run(draft_scaled_kernel<64, T, 2, 1, 4>, 4);
      else run(draft_scaled_kernel<64, T, 2, 2, 4>, 4);
    } else if (rule.waves == 4) {
      if (blocks == 1) run(draft_scaled_kernel<128, T, 1, 1, 4>, 4);
      else if (blocks == 2) run(draft_scaled_kernel<128, T, 1, 2, 4>, 4);
      else run(draft_scaled_kernel<128, T, 1, 4, 4>, 4);
    } else {
      if (blocks == 1) run(draft_scaled_kernel<128, T, 1, 1, 8>, 8);
      else if (blocks == 2) run(draft_scaled_kernel<128, T, 1, 2, 8>, 8);
      else run(draft_scaled_kernel<128, T, 1, 4, 8>, 8);
    }
  };
  switch (cache) {
    case CacheType::kE4M3: go(std::integral_constant<CacheType, CacheType::kE4M3>()); break;
    case CacheType::kE5M2: go(std::integral_constant<CacheType, CacheType::kE5M2>()); break;
    case CacheType::kE2M1: go(std::integral_constant<CacheType, CacheType::kE2M1>()); break;
  }
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || p.shares == 0) return e;
  auto merge = [&](auto kernel, int rows) {
    const dim3 grid((unsigned)((p.d.K * p.d.group + rows - 1) / rows), (unsigned)p.d.Hkv, (unsigned)p.d.C);
    hipLaunchKernelGGL(kernel, grid, dim3(256), 0, stream, p);
  };
  // One thread for all of a row's records and four features where a request has a few records (64 requests of 512 to 8192 tokens, two or
  // three each: the step 79.8 us, 83.2 with four), otherwise four (D 64; two at D 128), or each would wait for more reads one after the
  // other (4 requests, nine each: 14.6, 15.1 with one).
  // Four waves for a row, where the table leaves room for 32 records and more a request, which a wave would read in two rounds and more (codes
  // of 4 bits; with 8 a row's sums keep the order, and so the last bits, that they have had).  Lengths, and with them how many records there
  // are, only the device knows: with two or three in tables of 320 columns either merge takes as long (eight steps of 12 to 15 us, 0.15 apart
  // at most).  With the tables' width full:
  // D 128, one of 12000 tokens 16.6 us, otherwise 19.9 (99 records, one KV head) and 15.7, 17.5 (50, four heads), 2 of 10800 to 20000
  // 19.1, 20.3 (32, four heads); 4 of 9000 to 12000 17.3, 17.8 (32, two heads); D 64, 4 of 2000 to 9000 15.8, 16.2 (64, one head).  With
  // fewer the waves' own merge costs more: 6 of 9000 to 12000 (D 64, 21 records, two heads) 15.5, otherwise 15.3, 4 of 2048 to 4096 15.5, 14.4.
  const bool few = p.shares <= 4 * p.d.C, many = cache == CacheType::kE2M1 && p.shares >= 32 * p.d.C;
  if (many && D == 64) merge(draft_scaled_combine_kernel<64, 16, 4>, kMergeRows<64, 16>);
  else if (many) merge(draft_scaled_combine_kernel<128, 8, 8>, kMergeRows<128, 8>);
  else if (D == 64) few ? merge(draft_scaled_combine_kernel<64, 1, 4>, kMergeRows<64, 1>) : merge(draft_scaled_combine_kernel<64, 4, 8>, kMergeRows<64, 4>);
  else few ? merge(draft_scaled_combine_kernel<128, 1, 4>, kMergeRows<128, 1>) : merge(draft_scaled_combine_kernel<128, 2, 16>, kMergeRows<128, 2>);
  return hipGetLastError();
}

}  // namespace peagle
