// The inference-side drafting step (Sec. 2 of the paper) on a paged cache that is held in 8 bits with a power-of-two scale for
// each page and KV head: the K new rows of each request see its cached keys and the new keys of their own chain.
//
// With k = 2^ek a and v = 2^ev b for the codes a, b of a page, S = scale Q K^T, P = 2^(S log2(e) - m), O = P V / sum P.  A code
// has four significant bits or three, so that with its page's scale it is a bf16 number (zero where that would not be a normal one,
// infinite from 2^128 on): codes are widened to bf16, scale and all, by one instruction for two of them, between LDS and the
// matrix instruction.  (The matrix instruction for 8-bit types, with queries split into two numbers of them, would need no widening
// of keys, but its sums are not fp32 sums: 64 products of normal data came out 4e-5 of the largest sum off.)
// The cache is read once, 2 Hkv D bytes a token, and bounds a large call; a small one is a chain of memory round trips.
#include "attn_kernels.h"
#include "attn_util.h"
#include "cache_kernels.h"

#include <climits>
#include <type_traits>

namespace peagle {

namespace {

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

// State of RB blocks of 32 query rows: lane <-> row, registers <-> features 32 db + 8 (i / 4) + 4 g + i % 4.
template <int D, int RB>
struct Rows {
  bf16x8 q[RB][D / 16];  // features 32 i + 16 g + 8 j .. + 8 of step 2 i + j
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
template <int D, bool E5M2, int RB>
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
    const bf16x8 a0 = widen8<E5M2>(kw[i][0], kw[i][1], ks), a1 = widen8<E5M2>(kw[i][2], kw[i][3], ks);
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
      const bf16x8 a = widen8<E5M2>((uint32_t)vw[t][db][0], (uint32_t)vw[t][db][1], vs);
#pragma unroll
      for (int rb = 0; rb < RB; ++rb) r.o[rb][db] = mfma32(a, pb[rb][t], r.o[rb][db]);
    }
  __builtin_amdgcn_s_setprio(0);
}

// Sixteen of the request's new keys (bf16, staged in a slot: K rows of 2 D bytes, V behind them, in the layout of the bf16 tiles),
// the first of them key k0; the row of depth d sees keys 0..d.  A masked key weighs zero, and zero times an infinity or NaN is
// NaN: such values are taken out of the product and added to the rows that see them, from v_new (key 0 of the KV head, the next
// one `stride` elements on).
constexpr int kNewKeys = 16;
template <int D, int RB>
__device__ __forceinline__ void new_keys(Rows<D, RB>& r, const char* k_at, const char* v_at, int k0, int K, const __bf16* v_new, uint32_t stride,
                                         const int (&depth)[RB], float c) {
  const int lane = lane_id(), g = lane >> 5, row = lane % kNewKeys;
  bf16x8 ka[D / 16], va[D / 32];
  const TrOff<D> to = tr_offsets<D>(lane);
#pragma unroll
  for (int i = 0; i < D / 16; ++i) ka[i] = *reinterpret_cast<const bf16x8*>(k_at + tile_off<D>(row, 4 * (i / 2) + 2 * g + i % 2));
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

// Workgroup = (share of the work, KV head).  A wave holds RB blocks of 32 of the K x Hq/Hkv query rows that share the KV head (row =
// depth * group + head); PARTS waves with different rows make a stream, and the streams take a request's pages in turn.  A stream
// has a ring of slots in LDS (a page each where the ring holds two, otherwise 32 tokens), filled by its waves some slots ahead of their
// use.  With one wave a stream (up to 32 rows, at D = 64 up to 64) a wave waits for its own copies only and the loop has no barrier;
// more rows share what a stream copies, which costs a barrier a slot.  At the end of a request's pages the streams' sums are merged
// through LDS, and leave the results where the request is one workgroup's, otherwise a partial record.
// Bound: memory (64 requests of 8192 tokens: 102 us on MI355X with 24 rows of 128 features, 5.3 TB/s), with 56 rows of 64 features
// vector issue beside it (121 us, 4.4 TB/s: 204 instructions a slot of 32 keys and 64 rows - a quarter of it exponentials - keep the vector
// units busy for 64 % of a wave's time, the 16 matrix instructions theirs for 34 %).
template <int D, bool E5M2, int RB, int PARTS, int WAVES>
__global__ __launch_bounds__(WAVES * 64, D == 64 && RB == 1 ? 4 : 2) void draft_scaled_kernel(ScaledDecodeParams sp) {
  constexpr int kWaves = WAVES, kStreams = kWaves / PARTS;
  constexpr int kRing = (D == 64 && RB == 1 ? 8192 : 16384) * kWaves / kStreams;  // bytes of a stream's ring: 128 KiB a CU
  constexpr int kTokens = kRing >= 4 * 64 * D ? 64 : 32, kHalf = kTokens * D, kSlot = 2 * kHalf;  // a slot: bytes of its keys, in all
  constexpr int kPerPage = kKeysPerTile / kTokens, kDepth = kRing / kSlot;                        // slots of a page, of a ring
  constexpr int kCopies = kSlot / 1024 / PARTS;                               // of a slot, by each of a stream's waves
  constexpr int kAhead = PARTS == 1 ? kDepth : kDepth - 1;                    // slots on their way or in use
  __shared__ __attribute__((aligned(16))) char ring[kStreams][kDepth][kSlot];
  __shared__ f32x4 stats[kWaves][RB * 32];  // of each wave's rows: reference, the two sums
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
  const uint32_t ring_at = lds_scalar_addr(&ring[stream][0][0]);
  // This wave's copies of a slot: f(values rather than keys?, block of 1 KiB).
  auto each_copy = [&](auto f) {
    if constexpr (PARTS == 1) {
#pragma unroll
      for (int b = 0; b < kCopies / 2; ++b) f(false, b);
#pragma unroll
      for (int b = 0; b < kCopies / 2; ++b) f(true, b);
    } else {
      const int b0 = part % (PARTS / 2) * kCopies;
#pragma unroll
      for (int b = 0; b < kCopies; ++b) f(part >= PARTS / 2, b0 + b);
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
        const __bf16* q = p.q_new + (((size_t)c * p.K + depth[rb]) * p.Hq + head) * D + 16 * (l >> 5);
#pragma unroll
        for (int i = 0; i < D / 16; ++i) r.q[rb][i] = as_frag(ld16(q + (i / 2) * 32 + (i % 2) * 8));
      }
    };

    // The last stream's slots hold the new keys first.
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
      const uint32_t dst = ring_at + (uint32_t)(q & (kDepth - 1)) * kSlot;
      if (q < q0) {
        const int l = lane_id();
        each_copy([&](bool half, int b) {
          const int row = b * (512 / D) + l / (D / 8), key = q * kNewKeys + row;
          const uint32_t off = (uint32_t)(key < p.K ? key : p.K - 1) * (uint32_t)(p.Hkv * D * 2) + ((l % (D / 8) ^ swz<D>(row)) << 4);
          dma16_untracked(half ? v_new : k_new, off, dst + (half ? kHalf : 0) + b * 1024);
        });
        return;
      }
      const int j = (q - q0) / kPerPage, sub = (q - q0) % kPerPage;
      const size_t at = ((size_t)(uint32_t)__builtin_amdgcn_readlane(page, j) * p.Hkv + kvh) * (kKeysPerTile * D) + sub * kHalf;
      const int present = __builtin_amdgcn_readlane(keys, j) - sub * kTokens;
      if (present >= kTokens) {
        each_copy([&](bool half, int b) {
          dma16_untracked(uniform_ptr((half ? v_pages : k_pages) + at) + b * 1024, voff[b & 1], dst + (half ? kHalf : 0) + b * 1024);
        });
      } else {  // rows behind the last token are read as that token, and masked
        const int last = present > 0 ? present - 1 : 0, l = lane_id();
        each_copy([&](bool half, int b) {
          const int row = b * (64 / kLanes) + l / kLanes;
          const uint32_t off = (uint32_t)((row < last ? row : last) * D + ((l % kLanes ^ swz8<D>(row)) << 4));
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
      if (there) {
        kcode = k_scale[(size_t)page * p.Hkv + kvh];
        vcode = v_scale[(size_t)page * p.Hkv + kvh];
      }
      const int n_here = n_mine - first < 64 ? n_mine - first : 64;
      q0 = n_before;
      n_q = q0 + (n_here > 0 ? n_here * kPerPage : 0);
      // (one slot's copies with the loads: behind more, the wait for the loads would be one for the slots that are due later)
      issued = 0;
      if (n_q > 0) copy(issued++);
      __builtin_amdgcn_s_waitcnt(0x0F70);  // (the compiler's own loads: none is waited for in the loop, behind its copies)
      for (; issued < kAhead && issued < n_q; ++issued) copy(issued);
    };
    // A slot's turn: what it holds has landed; with several waves a stream, everyone is done with the slot before it, which is
    // filled again.
    auto begin = [&](int q) {
      wait_slots<kAhead - 1, kCopies>(issued - 1 - q);
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

    take_pages(0, my_new);
    int q = 0;
    // (where streams meet at barriers, the others wait for the new keys' turns)
    for (int i = 0; i < (PARTS > 1 ? n_new : my_new); ++i) {
      if (my_new > 0) begin(q);
      else if (PARTS > 1) __syncthreads();
      if (my_new > 0) {
        const char* at = ring[stream][q & (kDepth - 1)];
        new_keys<D, RB>(r, at, at + kHalf, q * kNewKeys, p.K, v_new, (uint32_t)(p.Hkv * D), depth, p.c_log2);
        end();
        ++q;
      }
    }
    for (int first = 0;;) {
      const int rounds = PARTS > 1 ? (n_pages_0 - first < 64 ? n_pages_0 - first : 64) * 2 : (n_q - q0) * (kTokens / 32);
      for (int i = 0; i < rounds; ++i) {
        const bool starts = kTokens == 32 || i % 2 == 0, ends = kTokens == 32 || i % 2 != 0;  // a slot's turn
        if (starts) begin(q);
        const int j = i / 2, n = __builtin_amdgcn_readlane(keys, j) - i % 2 * 32;  // (0 behind this stream's pages)
        const float ks = __builtin_bit_cast(float, __builtin_amdgcn_readlane(kcode, j) << 23);
        const int v_code = __builtin_amdgcn_readlane(vcode, j);
        const float vs = __builtin_bit_cast(float, v_code << 23), limit = v_code > kFarScale ? kNearLimit : kFarLimit;
        const char* at = ring[stream][q & (kDepth - 1)] + (kTokens == 32 ? 0 : i % 2 * 32 * D);
        if (n > 0) cached_keys<D, E5M2, RB>(r, at, at + kHalf, k_off, v_off, ks, vs, limit, n, g, p.c_log2);
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
    f32x4* regions = reinterpret_cast<f32x4*>(&ring[0][0][0]);
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
// first is used.
template <int D, int LANES>
constexpr int kMergeRows = 256 / (D / 4 * LANES);  // of a workgroup
template <int D, int LANES, int EACH>
__global__ __launch_bounds__(256) void draft_scaled_combine_kernel(ScaledDecodeParams sp) {
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
  for (int x = D / 4; x < D / 4 * LANES; x <<= 1) {
    const float m_other = __shfl_xor(M, x), m_new = __builtin_fmaxf(M, m_other);
    const float a = exp2_fast(M - m_new), b = exp2_fast(m_other - m_new);
    M = m_new;
    L = L * a + __shfl_xor(L, x) * b;
    W = W * a + __shfl_xor(W, x) * b;
#pragma unroll
    for (int j = 0; j < 4; ++j) acc[j] = acc[j] * a + __shfl_xor(acc[j], x) * b;
    bad |= __shfl_xor(bad, x);
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
//          4096 take 16.6 or 15.3 instead of 14.7, 48 of 500 to 8191 (D 128, 128 rows) 95.8 or 96.3 instead of 91.
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
// 1000 to 2000, 17.7 instead of 13.6 for 4 of 2048 to 4096 (two workgroups a CU instead of one); nothing for 64 of 512 to 8192.
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

hipError_t launch_draft_scaled(const ScaledDecodeParams& pin, int D, bool e5m2, hipStream_t stream) {
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
  // against 94 us for 64 of 512 to 8192).
  const bool alone = (int64_t)grid.x * grid.y <= kCus;
  auto go = [&](auto type) {
    constexpr bool T = decltype(type)::value;
    auto run = [&](auto kernel, int waves) { hipLaunchKernelGGL(kernel, grid, dim3((unsigned)waves * 64), 0, stream, p); };
    if (D == 64) {
      if (blocks == 1) run(draft_scaled_kernel<64, T, 1, 1, 8>, 8);
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
  e5m2 ? go(std::true_type{}) : go(std::false_type{});
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || p.shares == 0) return e;
  auto merge = [&](auto kernel, int rows) {
    const dim3 grid((unsigned)((p.d.K * p.d.group + rows - 1) / rows), (unsigned)p.d.Hkv, (unsigned)p.d.C);
    hipLaunchKernelGGL(kernel, grid, dim3(256), 0, stream, p);
  };
  // One thread for all of a row's records and four features where a request has a few records (64 requests of 512 to 8192 tokens, two or
  // three each: the step 79.8 us, 83.2 with four), otherwise four (D 64; two at D 128), or each would wait for more reads one after the
  // other (4 requests, nine each: 14.6, 15.1 with one).
  const bool few = p.shares <= 4 * p.d.C;
  if (D == 64) few ? merge(draft_scaled_combine_kernel<64, 1, 4>, kMergeRows<64, 1>) : merge(draft_scaled_combine_kernel<64, 4, 8>, kMergeRows<64, 4>);
  else few ? merge(draft_scaled_combine_kernel<128, 1, 4>, kMergeRows<128, 1>) : merge(draft_scaled_combine_kernel<128, 2, 16>, kMergeRows<128, 2>);
  return hipGetLastError();
}

}  // namespace peagle
