// The inference-side drafting step (Sec. 2 of the paper) on a paged cache that is held in 8 bits with a power-of-two scale for
// each page and KV head: the K new rows of each request see its cached keys and the new keys of their own chain.
//
// With k = 2^ek a and v = 2^ev b for the codes a, b of a page, S = scale Q K^T, P = 2^(S log2(e) - m), O = P V / sum P.  The
// type's values have four significant bits or three, so that a code times its page's scale is a bf16 number: codes are widened to
// bf16 with the scale in one instruction for two of them, between LDS and the matrix instruction, exactly.
// The cache is read once, 2 Hkv D bytes a token, and bounds a large call; a small one is a chain of memory round trips.
#include "attn_kernels.h"
#include "attn_util.h"

#include <type_traits>

namespace peagle {

namespace {

constexpr int kWaves = 4, kSlotBytes = 8192;  // a slot of a wave's ring: 4 KiB of K, 4 KiB of V

// Eight codes, times `scale` (a power of two), as a matrix operand.
template <bool E5M2>
__device__ __forceinline__ bf16x8 widen8(uint32_t a, uint32_t b, float scale) {
  u32x4 u;
  auto two = [&](uint32_t w, auto high) {
    constexpr bool H = decltype(high)::value;
    const bf16x2 x = E5M2 ? __builtin_amdgcn_cvt_scalef32_pk_bf16_bf8(w, scale, H) : __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale, H);
    return __builtin_bit_cast(uint32_t, x);
  };
  u[0] = two(a, std::false_type{});
  u[1] = two(a, std::true_type{});
  u[2] = two(b, std::false_type{});
  u[3] = two(b, std::true_type{});
  return __builtin_bit_cast(bf16x8, u);
}

// LDS image of 4 KiB of a page, row (token) by row of D bytes: the 16-byte chunk c of row r stands at c ^ swz8(r), so that both
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

// State of RB blocks of 32 query rows: lane <-> row, registers <-> features 32 db + 8 (i / 4) + 4 g + i % 4.
template <int D, int RB>
struct Rows {
  bf16x8 q[RB][D / 16];  // features 32 i + 16 g + 8 j .. + 8 of step 2 i + j
  f32x16 o[RB][D / 32];
  float m[RB], l[RB];    // reference of the exponents (log2), sum over this lane's keys
};

// Scores of 32 keys (registers <-> keys 8 (i / 4) + 4 g + i % 4) to probabilities, as operands of the product with the values.
// The reference is the running maximum.  The row sum takes the probabilities unrounded.
template <int D, int RB>
__device__ __forceinline__ void soft(Rows<D, RB>& r, int rb, f32x16& s, float c, bf16x8 (&pb)[2]) {
  const float mx = max_halves(max16(s)) * c;
  const bool need = mx > r.m[rb];
  if (__builtin_amdgcn_ballot_w64(need) != 0) {
    const float m_new = need ? mx : r.m[rb], alpha = exp2_fast(r.m[rb] - m_new);
    r.m[rb] = m_new;
    r.l[rb] *= alpha;
#pragma unroll
    for (int db = 0; db < D / 32; ++db)
#pragma unroll
      for (int i = 0; i < 16; ++i) r.o[rb][db][i] *= alpha;
  }
  const float neg_m = -r.m[rb];
  float sum[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    s[i] = exp2_fast(__builtin_fmaf(s[i], c, neg_m));
    sum[i % 4] += s[i];
  }
  r.l[rb] += (sum[0] + sum[1]) + (sum[2] + sum[3]);
  pb[0] = pack8(s, 0);
  pb[1] = pack8(s, 1);
}

// Keys of a slot, `visible` of its first keys (the others are masked; their values are finite).
template <int D, bool E5M2, int RB>
__device__ __forceinline__ void cached_keys(Rows<D, RB>& r, const char* slot, const int (&k_off)[D / 32], const int (&v_off)[D / 32],
                                            float ks, float vs, int visible, int g, float c) {
#pragma unroll
  for (int kb = 0; kb < 4096 / D / 32; ++kb) {
    const int n = visible - kb * 32;
    if (n <= 0) break;
    bf16x8 pb[RB][2];
    f32x16 s[RB];
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) s[rb] = zero16();
#pragma unroll
    for (int i = 0; i < D / 32; ++i) {
      const u32x4 w = *reinterpret_cast<const u32x4*>(slot + k_off[i] + kb * 32 * D);
      const bf16x8 a0 = widen8<E5M2>(w[0], w[1], ks), a1 = widen8<E5M2>(w[2], w[3], ks);
#pragma unroll
      for (int rb = 0; rb < RB; ++rb) {
        s[rb] = mfma32(a0, r.q[rb][2 * i], s[rb]);
        s[rb] = mfma32(a1, r.q[rb][2 * i + 1], s[rb]);
      }
    }
    if (n < 32) {
      const uint32_t bits = ((1u << n) - 1) >> (4 * g);
#pragma unroll
      for (int rb = 0; rb < RB; ++rb)
#pragma unroll
        for (int i = 0; i < 16; ++i) s[rb][i] = mask_sel(s[rb][i], bits, 8 * (i / 4) + (i % 4));
    }
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) soft(r, rb, s[rb], c, pb[rb]);
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int db = 0; db < D / 32; ++db) {
        typedef __attribute__((ext_vector_type(2))) int i32x2;
        const i32x2 w = __builtin_amdgcn_ds_read_tr8_b64_v2i32(PEAGLE_LDS_PTR(i32x2, slot + 4096 + v_off[db] + (kb * 2 + t) * 16 * D));
        const bf16x8 a = widen8<E5M2>((uint32_t)w[0], (uint32_t)w[1], vs);
#pragma unroll
        for (int rb = 0; rb < RB; ++rb) r.o[rb][db] = mfma32(a, pb[rb][t], r.o[rb][db]);
      }
  }
}

// The request's K new keys (bf16), straight from memory; the row of depth d sees keys 0..d.  k_new, v_new: key 0 of the KV head,
// the next one `stride` elements on.  A masked key weighs zero, and zero times an infinity or NaN is NaN: such values are taken
// out of the product and added to the rows that see them.
template <int D, int RB>
__device__ __forceinline__ void new_keys(Rows<D, RB>& r, const __bf16* k_new, const __bf16* v_new, uint32_t stride, int K,
                                         const int (&depth)[RB], float c) {
  const int lane = lane_id(), g = lane >> 5, ln = lane & 31;
  for (int k0 = 0; k0 < K; k0 += 32) {
    const uint32_t row = (uint32_t)(k0 + ln < K ? k0 + ln : K - 1) * stride + 16 * g;
    bf16x8 pb[RB][2];
    f32x16 s[RB];
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) s[rb] = zero16();
#pragma unroll
    for (int i = 0; i < D / 16; ++i) {
      const bf16x8 a = as_frag(ld16(k_new + row + ((i / 2) * 32 + (i % 2) * 8)));
#pragma unroll
      for (int rb = 0; rb < RB; ++rb) s[rb] = mfma32(a, r.q[rb][i], s[rb]);
    }
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
      const int n = depth[rb] + 1 - k0;
      const uint32_t bits = (n >= 32 ? 0xffffffffu : n <= 0 ? 0u : (1u << n) - 1) >> (4 * g);
#pragma unroll
      for (int i = 0; i < 16; ++i) s[rb][i] = mask_sel(s[rb][i], bits, 8 * (i / 4) + (i % 4));
      soft(r, rb, s[rb], c, pb[rb]);
    }
    bool odd = false;
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      if (k0 + 16 * t >= K) break;
#pragma unroll
      for (int db = 0; db < D / 32; ++db) {
        u32x4 a;
#pragma unroll
        for (int j = 0; j < 8; j += 2) {
          uint32_t pair = 0;
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            const int at = k0 + 16 * t + 4 * g + (j < 4 ? 0 : 4) + j + h;
            const uint32_t from = (uint32_t)(at < K ? at : K - 1) * stride + ln;
            const uint32_t x = *reinterpret_cast<const uint16_t*>(v_new + from + db * 32);
            const bool fine = (x & 0x7f80u) != 0x7f80u;
            odd |= !fine;
            pair |= (fine ? x : 0u) << (16 * h);
          }
          a[j / 2] = pair;
        }
        const bf16x8 frag = __builtin_bit_cast(bf16x8, a);
#pragma unroll
        for (int rb = 0; rb < RB; ++rb) r.o[rb][db] = mfma32(frag, pb[rb][t], r.o[rb][db]);
      }
    }
    if (__builtin_amdgcn_ballot_w64(odd) != 0) {
      for (int e = k0; e < K && e < k0 + 32; ++e) {
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
}

// Workgroup = (piece of a context, KV head, request), four waves.  A wave holds RB blocks of 32 of the K x Hq/Hkv query rows that
// share the KV head (row = depth * group + head) and takes every n-th page of the piece by itself: it copies pages to a ring of
// its own in LDS, two slots, and computes on one while the other is on its way, so that the loop has no barrier and a wave waits
// for its own copies only.  The four waves hold the same rows (one block at D = 128, where two leave too few registers, one or two
// at D = 64); more rows are shared out over two or all of them.  At the end the sums of waves with the same rows are merged
// through LDS.  Eight waves a CU (two workgroups) have up to 128 KiB on their way.
template <int D, bool E5M2, int RB>
__global__ __launch_bounds__(kWaves * 64, 2) void draft_scaled_kernel(ScaledDecodeParams sp) {
  constexpr int kSubKeys = 4096 / D, kSubs = kKeysPerTile / kSubKeys;  // keys of a slot; slots of a page
  const DecodeParams& p = sp.d;
  __shared__ __attribute__((aligned(16))) char ring[kWaves][2][kSlotBytes];
  __shared__ float stats[kWaves][RB * 32][2];  // of each wave's rows: reference, sum
  __shared__ int wave_bad[kWaves];

  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, g = lane >> 5, ln = lane & 31;
  const int split = blockIdx.x, kvh = blockIdx.y, c = blockIdx.z;
  const int share = p.rows_pad > 64 * RB ? 2 : p.rows_pad > 32 * RB ? 1 : 0;  // log2 of the waves that share the rows out
  const int part = wave & ((1 << share) - 1), stream = wave >> share, n_streams = kWaves >> share;
  const int n_rows = p.K * p.group;

  int n_ctx = p.ctx_len[c];
  bool bad = n_ctx < 0 || n_ctx > p.max_pages * kKeysPerTile;
  n_ctx = n_ctx < 0 ? 0 : (n_ctx > p.max_pages * kKeysPerTile ? p.max_pages * kKeysPerTile : n_ctx);
  const int n_pg = (n_ctx + kKeysPerTile - 1) / kKeysPerTile;
  int up = n_pg + p.n_splits - 1;
  const int per = split_by(up, p.by_splits);
  const int p0 = split * per < n_pg ? split * per : n_pg;
  const int p1 = p0 + per < n_pg ? p0 + per : n_pg;
  const int n_mine = p1 - p0 > stream ? (p1 - p0 - stream + n_streams - 1) / n_streams : 0;  // pages of this wave

  Rows<D, RB> r;
  int depth[RB];
#pragma unroll
  for (int rb = 0; rb < RB; ++rb) {
    const int row = (part * RB + rb) * 32 + ln;
    depth[rb] = row < n_rows ? small_quotient(row, p.group_reciprocal) : 0;
    const int head = kvh * p.group + (row < n_rows ? row - depth[rb] * p.group : 0);
    const __bf16* q = p.q_new + (((size_t)c * p.K + depth[rb]) * p.Hq + head) * D + 16 * g;
#pragma unroll
    for (int i = 0; i < D / 16; ++i) r.q[rb][i] = as_frag(ld16(q + (i / 2) * 32 + (i % 2) * 8));
#pragma unroll
    for (int db = 0; db < D / 32; ++db) r.o[rb][db] = zero16();
    r.m[rb] = -3.402823466e38f;  // (any score is above it, and it less any score is no NaN)
    r.l[rb] = 0.f;
  }

  int k_off[D / 32], v_off[D / 32];
  {
    const int i = lane & 15, row = 4 * g + (i >> 1 & 3) + (i >> 3) * 8;
#pragma unroll
    for (int j = 0; j < D / 32; ++j) {
      k_off[j] = ln * D + (((2 * j + g) ^ swz8<D>(ln)) << 4);
      v_off[j] = row * D + (((2 * j + (lane >> 4 & 1)) ^ swz8<D>(row)) << 4) + (i & 1) * 8;
    }
  }
  // Copies: lane l of the 1 KiB block b of a slot's half owns LDS bytes [1024 b + 16 l, + 16) and fetches the chunk that lives there.
  constexpr int kLanes = D / 16;  // of a row
  uint32_t voff[2];
#pragma unroll
  for (int b = 0; b < 2; ++b)
    voff[b] = (uint32_t)((lane / kLanes) * D + ((lane % kLanes ^ swz8<D>(b * (64 / kLanes) + lane / kLanes)) << 4));
  const uint32_t ring_at = lds_scalar_addr(&ring[wave][0][0]);

  for (int first = 0; first == 0 || first < n_mine; first += 64) {
    // This wave's next pages, one a lane: page, keys present (0: page id outside the pool), scales.
    const int pi = p0 + stream + n_streams * (first + lane);
    const bool there = pi < p1;
    int page = there ? p.block_table[(size_t)c * p.max_pages + pi] : 0;
    const bool fine = page >= 0 && page < p.n_pages;
    bad |= !fine;
    page = fine ? page : 0;
    const int keys_here = n_ctx - pi * kKeysPerTile;
    int keys = !there || !fine ? 0 : keys_here < kKeysPerTile ? keys_here : kKeysPerTile;
    int kcode = 0, vcode = 0;
    if (there) {
      kcode = sp.k_scale[(size_t)page * p.Hkv + kvh];
      vcode = sp.v_scale[(size_t)page * p.Hkv + kvh];
    }
    const int n_here = n_mine - first < 64 ? n_mine - first : 64;
    const int n_sub = n_here > 0 ? n_here * kSubs : 0;

    auto copy = [&](int s) {
      const int j = s / kSubs, sub = s % kSubs;
      const size_t at = ((size_t)(uint32_t)__builtin_amdgcn_readlane(page, j) * p.Hkv + kvh) * (kKeysPerTile * D) + sub * 4096;
      const uint8_t* kp = uniform_ptr(sp.k_pages + at);
      const uint8_t* vp = uniform_ptr(sp.v_pages + at);
      const uint32_t dst = ring_at + (uint32_t)(s & 1) * kSlotBytes;
      const int present = __builtin_amdgcn_readlane(keys, j) - sub * kSubKeys;
      if (present >= kSubKeys) {
#pragma unroll
        for (int b = 0; b < 4; ++b) dma16_untracked(kp + b * 1024, voff[b & 1], dst + b * 1024);
#pragma unroll
        for (int b = 0; b < 4; ++b) dma16_untracked(vp + b * 1024, voff[b & 1], dst + 4096 + b * 1024);
      } else {  // rows behind the last token are read as that token: they are masked, and zero times its values adds nothing
        const int last = present > 0 ? present - 1 : 0, l = lane_id();
#pragma unroll
        for (int b = 0; b < 4; ++b) {
          const int row = b * (64 / kLanes) + l / kLanes;
          const uint32_t off = (uint32_t)((row < last ? row : last) * D + ((l % kLanes ^ swz8<D>(row)) << 4));
          dma16_untracked(kp, off, dst + b * 1024);
          dma16_untracked(vp, off, dst + 4096 + b * 1024);
        }
      }
    };
    asm volatile("s_waitcnt lgkmcnt(0)" : : : "memory");  // (after 64 pages: the slots' last reads have left them)
    if (n_sub > 0) copy(0);
    if (n_sub > 1) copy(1);
    if (first == 0 && split == 0 && stream == (p1 - p0) % n_streams) {
      const size_t at = ((size_t)c * p.K * p.Hkv + kvh) * D;
      new_keys<D, RB>(r, uniform_ptr(p.k_new + at), uniform_ptr(p.v_new + at), (uint32_t)(p.Hkv * D), p.K, depth, p.c_log2);
    }
    __builtin_amdgcn_s_waitcnt(0x0F70);  // (the compiler's own loads: none is waited for in the loop, behind its copies)
    for (int s = 0; s < n_sub; ++s) {
      if (s + 1 < n_sub) wait_outstanding<8>();
      else wait_outstanding<0>();
      const int j = s / kSubs, visible = __builtin_amdgcn_readlane(keys, j) - s % kSubs * kSubKeys;
      const float ks = __builtin_bit_cast(float, __builtin_amdgcn_readlane(kcode, j) << 23);
      const float vs = __builtin_bit_cast(float, __builtin_amdgcn_readlane(vcode, j) << 23);
      cached_keys<D, E5M2, RB>(r, ring[wave][s & 1], k_off, v_off, ks, vs, visible, g, p.c_log2);
      if (s + 2 < n_sub) {
        asm volatile("s_waitcnt lgkmcnt(0)" : : : "memory");  // the slot's last reads have left it
        copy(s + 2);
      }
    }
  }

  // Merge of the waves that hold the same rows: each leaves reference, sum and O (32 rows at a time, in its ring, 16 bytes of
  // features by 16 bytes, the rows of feature group d4 in the order row ^ d4), and the threads add them up in order.
  bad = __builtin_amdgcn_ballot_w64(bad) != 0;
#pragma unroll
  for (int rb = 0; rb < RB; ++rb) {
    const float l = sum_halves(r.l[rb]);
    if (g == 0) {
      stats[wave][rb * 32 + ln][0] = r.m[rb];
      stats[wave][rb * 32 + ln][1] = l;
    }
  }
  if (lane == 0) wave_bad[wave] = bad;
  f32x4* mine = reinterpret_cast<f32x4*>(&ring[wave][0][0]);
  const int l = lane_id();
  static_assert(32 * D * 4 <= 2 * kSlotBytes, "32 rows of O must fit a wave's ring");
  const size_t rec = ((size_t)c * p.Hkv + kvh) * p.n_splits + split;
#pragma unroll
  for (int rb = 0; rb < RB; ++rb) {
    if (rb > 0) __syncthreads();
#pragma unroll
    for (int db = 0; db < D / 32; ++db)
#pragma unroll
      for (int i4 = 0; i4 < 4; ++i4) {
        const int d4 = db * 8 + 2 * i4 + (l >> 5);
        mine[d4 * 32 + ((l ^ d4) & 31)] = f32x4{r.o[rb][db][4 * i4], r.o[rb][db][4 * i4 + 1], r.o[rb][db][4 * i4 + 2], r.o[rb][db][4 * i4 + 3]};
      }
    __syncthreads();
    const bool any_bad = (wave_bad[0] | wave_bad[1] | wave_bad[2] | wave_bad[3]) != 0;
    for (int item = wave * 64 + l; item < (32 << share) * (D / 4); item += kWaves * 64) {
      const int d4 = item % (D / 4), in_block = item / (D / 4) % 32, h = item / (32 * (D / 4));
      const int row = (h * RB + rb) * 32 + in_block;
      float M = stats[h][rb * 32 + in_block][0];
      for (int s = 1; s < n_streams; ++s) M = __builtin_fmaxf(M, stats[(s << share) + h][rb * 32 + in_block][0]);
      float L = 0.f;
      f32x4 o = {0.f, 0.f, 0.f, 0.f};
      for (int s = 0; s < n_streams; ++s) {
        const int w = (s << share) + h;
        const float f = exp2_fast(stats[w][rb * 32 + in_block][0] - M);
        L = __builtin_fmaf(stats[w][rb * 32 + in_block][1], f, L);
        o += reinterpret_cast<const f32x4*>(&ring[w][0][0])[d4 * 32 + (in_block ^ (d4 & 31))] * f;
      }
      if (p.n_splits == 1) {
        if (row < n_rows) {
          const int dep = small_quotient(row, p.group_reciprocal), head = kvh * p.group + (row - dep * p.group);
          const float inv = 1.0f / L;
          u32x2 out;
          out[0] = pack_bf16(o[0] * inv, o[1] * inv);
          out[1] = pack_bf16(o[2] * inv, o[3] * inv);
          *reinterpret_cast<u32x2*>(p.o + (((size_t)c * p.K + dep) * p.Hq + head) * D + d4 * 4) = out;
          if (d4 == 0) p.lse[((size_t)c * p.Hq + head) * p.K + dep] = (M + __builtin_log2f(L)) * kLn2;
        }
      } else if (row < p.rows_pad) {
        *reinterpret_cast<f32x4*>(p.part_o + (rec * p.rows_pad + row) * D + d4 * 4) = o;
        if (d4 == 0) {
          float* ml = p.part_ml + rec * 3 * p.rows_pad + row;
          ml[0] = M;
          ml[p.rows_pad] = L;
          ml[2 * p.rows_pad] = any_bad ? 1.f : 0.f;
        }
      }
    }
    if (rb == 0 && p.n_splits == 1 && p.status && kvh == 0 && tid == 0) p.status[c] = any_bad;
  }
}

constexpr int kCus = 256;  // compute units of the device

}  // namespace

// Pieces of a request: two workgroups per CU in all where each wave still has a page of its own.
int draft_scaled_pieces(int64_t wgs_per_piece, int max_pages, int) {
  const int64_t want = (2 * kCus + wgs_per_piece - 1) / wgs_per_piece, most = (max_pages + kWaves - 1) / kWaves;
  const int64_t n = want < most ? want : most;
  return (int)(n < 1 ? 1 : n > 32 ? 32 : n);
}

hipError_t launch_draft_scaled(const ScaledDecodeParams& pin, int D, bool e5m2, hipStream_t stream) {
  ScaledDecodeParams p = pin;
  p.d.group = p.d.Hq / p.d.Hkv;
  p.d.group_reciprocal = small_reciprocal(p.d.group);
  p.d.by_splits = make_divisor(p.d.n_splits);
  const dim3 grid((unsigned)p.d.n_splits, (unsigned)p.d.Hkv, (unsigned)p.d.C);
  auto run = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, dim3(kWaves * 64), 0, stream, p); };
  if (D == 128) e5m2 ? run(draft_scaled_kernel<128, true, 1>) : run(draft_scaled_kernel<128, false, 1>);
  else if (p.d.rows_pad == 32) e5m2 ? run(draft_scaled_kernel<64, true, 1>) : run(draft_scaled_kernel<64, false, 1>);
  else e5m2 ? run(draft_scaled_kernel<64, true, 2>) : run(draft_scaled_kernel<64, false, 2>);
  const hipError_t e = hipGetLastError();
  return e != hipSuccess || p.d.n_splits == 1 ? e : launch_draft_combine(p.d, D, stream);
}

}  // namespace peagle
