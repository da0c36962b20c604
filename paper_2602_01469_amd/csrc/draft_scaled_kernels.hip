// The inference-side drafting step (Sec. 2 of the paper) on a paged cache that is held in 8 bits with a power-of-two scale for
// each page and KV head: the K new rows of each request see its cached keys and the new keys of their own chain.
//
// With k = 2^ek a and v = 2^ev b for the codes a, b of a page, S = scale Q K^T, P = 2^(S log2(e) - m), O = P V / sum P.  The
// type's values have four significant bits or three, so that a code times its page's scale is a bf16 number: codes are widened to
// bf16 with the scale in one instruction for two of them, between LDS and the matrix instruction, exactly.
// The cache is read once, 2 Hkv D bytes a token, and bounds a large call; a small one is a chain of memory round trips.
#include "attn_kernels.h"
#include "attn_util.h"

#include <climits>
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

// A block of the request's new keys (bf16, staged in a slot: K rows of 2 D bytes, V behind them, in the layout of the bf16 tiles),
// the first of them key k0; the row of depth d sees keys 0..d.  A masked key weighs zero, and zero times an infinity or NaN is
// NaN: such values are taken out of the product and added to the rows that see them, from v_new (key 0 of the KV head, the next
// one `stride` elements on).
template <int D, int RB>
__device__ __forceinline__ void new_keys(Rows<D, RB>& r, const char* slot, int k0, int K, const __bf16* v_new, uint32_t stride,
                                         const int (&depth)[RB], float c) {
  constexpr int kKeys = 2048 / D;  // of a slot
  const int lane = lane_id(), g = lane >> 5, ln = lane & 31, row = ln % kKeys;
  f32x16 s[RB];
#pragma unroll
  for (int rb = 0; rb < RB; ++rb) s[rb] = zero16();
#pragma unroll
  for (int i = 0; i < D / 16; ++i) {
    const bf16x8 a = *reinterpret_cast<const bf16x8*>(slot + tile_off<D>(row, 4 * (i / 2) + 2 * g + i % 2));
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) s[rb] = mfma32(a, r.q[rb][i], s[rb]);
  }
  bf16x8 pb[RB][2];
#pragma unroll
  for (int rb = 0; rb < RB; ++rb) {
    const int sees = depth[rb] + 1 - k0, n = sees < kKeys ? sees : kKeys;
    const uint32_t bits = (n >= 32 ? 0xffffffffu : n <= 0 ? 0u : (1u << n) - 1) >> (4 * g);
#pragma unroll
    for (int i = 0; i < 16; ++i) s[rb][i] = mask_sel(s[rb][i], bits, 8 * (i / 4) + (i % 4));
    soft(r, rb, s[rb], c, pb[rb]);
  }
  bool odd = false;
  const TrOff<D> to = tr_offsets<D>(lane);
#pragma unroll
  for (int t = 0; t < kKeys / 16; ++t)
#pragma unroll
    for (int db = 0; db < D / 32; ++db) {
      u32x4 a = __builtin_bit_cast(u32x4, frag_tr<D>(slot + 4096, to, t * 16, db));
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const uint32_t w = a[j];
        const bool lo = (w & 0x7f80u) == 0x7f80u, hi = (w & 0x7f800000u) == 0x7f800000u;
        odd |= lo | hi;
        a[j] = w & ((lo ? 0u : 0xffffu) | (hi ? 0u : 0xffff0000u));
      }
#pragma unroll
      for (int rb = 0; rb < RB; ++rb) r.o[rb][db] = mfma32(__builtin_bit_cast(bf16x8, a), pb[rb][t], r.o[rb][db]);
    }
  if (__builtin_amdgcn_ballot_w64(odd) != 0) {
    for (int e = k0; e < K && e < k0 + kKeys; ++e) {
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
__device__ __forceinline__ int scan_lanes(int x, int lane) {
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const int y = __shfl_up(x, d);
    x += lane >= d ? y : 0;
  }
  return x;
}

// Cached tokens of a request, clamped to what its table can describe.
__device__ __forceinline__ int clamp_len(int n, int max_pages) {
  return n < 0 ? 0 : n > max_pages * kKeysPerTile ? max_pages * kKeysPerTile : n;
}
__device__ __forceinline__ int pages_of(int n) { return (n + kKeysPerTile - 1) / kKeysPerTile; }

// Every workgroup of a KV head takes the same share of all requests' work, counted in pages with one more for a request's new
// keys: workgroup w the units [w share, (w + 1) share) of the requests one after the other.
struct Share {
  int share, c, skip;  // units a workgroup; its first request, and the units of that which others take
  bool any;
};
__device__ __forceinline__ Share share_of(const int32_t* ctx_len, int C, int max_pages, int w, int n_wgs, int least, int lane) {
  const int per = (C + 63) / 64;
  int mine = 0;
  for (int i = 0; i < per; ++i) {
    const int c = lane * per + i;
    mine += c < C ? pages_of(clamp_len(ctx_len[c], max_pages)) + 1 : 0;
  }
  int end = scan_lanes(mine, lane);
  const int total = __builtin_amdgcn_readlane(end, 63);
  Share s;
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
    mine = lane < per && c < C ? pages_of(clamp_len(ctx_len[c], max_pages)) + 1 : 0;
    end = before + scan_lanes(mine, lane);
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

// Workgroup = (share of the work, KV head), four waves.  A wave holds RB blocks of 32 of the K x Hq/Hkv query rows that share the
// KV head (row = depth * group + head); PARTS waves with different rows make a stream, and the streams take a request's pages in
// turn.  A stream has a ring of slots in LDS, filled by its waves some slots ahead of their use.  With one wave a stream (up to 32
// rows, at D = 64 up to 64) a wave waits for its own copies only and the loop has no barrier; more rows share what a stream copies,
// which costs a barrier a slot.  At the end of a request's pages the streams' sums are merged through LDS, and leave the results
// where the request is one workgroup's, otherwise a partial record.
template <int D, bool E5M2, int RB, int PARTS>
__global__ __launch_bounds__(kWaves * 64, 2) void draft_scaled_kernel(ScaledDecodeParams sp) {
  constexpr int kSubKeys = 4096 / D, kSubs = kKeysPerTile / kSubKeys;  // keys of a slot; slots of a page
  constexpr int kNewKeys = 2048 / D;                                   // new keys of a slot
  constexpr int kStreams = kWaves / PARTS, kDepth = 2 * PARTS, kPer = 8 / PARTS;  // slots of a ring; copies a wave issues for one
  constexpr int kAhead = PARTS == 1 ? kDepth : kDepth - 1;             // slots on their way or in use
  const DecodeParams& p = sp.d;
  __shared__ __attribute__((aligned(16))) char ring[kStreams][kDepth][kSlotBytes];
  __shared__ float stats[kWaves][RB * 32][2];  // of each wave's rows: reference, sum
  __shared__ int wave_bad[kWaves];

  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, g = lane >> 5, ln = lane & 31;
  const int kvh = blockIdx.y, part = wave % PARTS, stream = wave / PARTS;
  const int n_rows = p.K * p.group;

  int c = blockIdx.x, skip = 0, left = INT_MAX, share = 0;
  if (sp.shares > 0) {
    const Share s = share_of(p.ctx_len, p.C, p.max_pages, blockIdx.x, sp.shares, sp.least_share, lane);
    if (!s.any) return;
    c = s.c;
    skip = s.skip;
    left = share = s.share;
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
  const uint32_t ring_at = lds_scalar_addr(&ring[stream][0][0]);
  // This wave's copies of a slot: f(which half, block of 1 KiB).
  auto each_copy = [&](auto f) {
    if constexpr (PARTS == 1) {
#pragma unroll
      for (int b = 0; b < 4; ++b) f(false, b);
#pragma unroll
      for (int b = 0; b < 4; ++b) f(true, b);
    } else {
      const int b0 = part % (PARTS / 2) * kPer;
#pragma unroll
      for (int b = 0; b < kPer; ++b) f(part >= PARTS / 2, b0 + b);
    }
  };

  for (int segment = 0;; ++segment) {
    int n_ctx = p.ctx_len[c];
    bool bad = n_ctx < 0 || n_ctx > p.max_pages * kKeysPerTile;
    n_ctx = clamp_len(n_ctx, p.max_pages);
    const int n_pg = pages_of(n_ctx), units = n_pg + 1;
    const int n_units = units - skip < left ? units - skip : left;
    const int p0 = skip, p1 = skip + n_units < n_pg ? skip + n_units : n_pg;
    const bool has_new = skip + n_units == units, whole = n_units == units;

    Rows<D, RB> r;
    int depth[RB];
    const int lane_here = lane_id();
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
      const int row = (part * RB + rb) * 32 + (lane_here & 31);
      depth[rb] = row < n_rows ? small_quotient(row, p.group_reciprocal) : 0;
      const int head = kvh * p.group + (row < n_rows ? row - depth[rb] * p.group : 0);
      const __bf16* q = p.q_new + (((size_t)c * p.K + depth[rb]) * p.Hq + head) * D + 16 * (lane_here >> 5);
#pragma unroll
      for (int i = 0; i < D / 16; ++i) r.q[rb][i] = as_frag(ld16(q + (i / 2) * 32 + (i % 2) * 8));
#pragma unroll
      for (int db = 0; db < D / 32; ++db) r.o[rb][db] = zero16();
      r.m[rb] = -3.402823466e38f;  // (any score is above it, and it less any score is no NaN)
      r.l[rb] = 0.f;
    }

    // The last stream's slots hold the new keys first.
    const int n_new = has_new ? (p.K + kNewKeys - 1) / kNewKeys : 0, my_new = stream == kStreams - 1 ? n_new : 0;
    const size_t new_at = ((size_t)c * p.K * p.Hkv + kvh) * D;
    const __bf16* k_new = uniform_ptr(p.k_new + new_at);
    const __bf16* v_new = uniform_ptr(p.v_new + new_at);
    const int n_pages_0 = (p1 - p0 + kStreams - 1) / kStreams;  // pages of stream 0, the most
    const int n_mine = p1 - p0 > stream ? (p1 - p0 - stream + kStreams - 1) / kStreams : 0;

    for (int first = 0; first == 0 || first < n_pages_0; first += 64) {
      // This stream's next pages, one a lane: page, keys present (0: page id outside the pool), scales.
      const int pi = p0 + stream + kStreams * (first + lane_id());
      const bool there = pi < p1;
      int page = there ? p.block_table[(size_t)c * p.max_pages + pi] : 0;
      const bool fine = page >= 0 && page < p.n_pages;
      bad |= !fine;
      page = fine ? page : 0;
      const int keys_here = n_ctx - pi * kKeysPerTile;
      const int keys = !there || !fine ? 0 : keys_here < kKeysPerTile ? keys_here : kKeysPerTile;
      int kcode = 0, vcode = 0;
      if (there) {
        kcode = sp.k_scale[(size_t)page * p.Hkv + kvh];
        vcode = sp.v_scale[(size_t)page * p.Hkv + kvh];
      }
      const int n_here = n_mine - first < 64 ? n_mine - first : 64;
      const int q0 = first == 0 ? my_new : 0, n_q = q0 + (n_here > 0 ? n_here * kSubs : 0);  // slots: new keys', all

      auto copy = [&](int q) {
        const uint32_t dst = ring_at + (uint32_t)(q % kDepth) * kSlotBytes;
        if (q < q0) {
          const int l = lane_id();
          each_copy([&](bool half, int b) {
            const int row = b * (512 / D) + l / (D / 8), key = q * kNewKeys + row;
            const uint32_t off = (uint32_t)(key < p.K ? key : p.K - 1) * (uint32_t)(p.Hkv * D * 2) + ((l % (D / 8) ^ swz<D>(row)) << 4);
            dma16_untracked(half ? v_new : k_new, off, dst + (half ? 4096 : 0) + b * 1024);
          });
          return;
        }
        const int j = (q - q0) / kSubs, sub = (q - q0) % kSubs;
        const size_t at = ((size_t)(uint32_t)__builtin_amdgcn_readlane(page, j) * p.Hkv + kvh) * (kKeysPerTile * D) + sub * 4096;
        const int present = __builtin_amdgcn_readlane(keys, j) - sub * kSubKeys;
        if (present >= kSubKeys) {
          each_copy([&](bool half, int b) {
            dma16_untracked(uniform_ptr((half ? sp.v_pages : sp.k_pages) + at) + b * 1024, voff[b & 1], dst + (half ? 4096 : 0) + b * 1024);
          });
        } else {  // rows behind the last token are read as that token: they are masked, and zero times its values adds nothing
          const int last = present > 0 ? present - 1 : 0, l = lane_id();
          each_copy([&](bool half, int b) {
            const int row = b * (64 / kLanes) + l / kLanes;
            const uint32_t off = (uint32_t)((row < last ? row : last) * D + ((l % kLanes ^ swz8<D>(row)) << 4));
            dma16_untracked(uniform_ptr((half ? sp.v_pages : sp.k_pages) + at), off, dst + (half ? 4096 : 0) + b * 1024);
          });
        }
      };
      int issued = 0;
      for (; issued < kAhead && issued < n_q; ++issued) copy(issued);
      __builtin_amdgcn_s_waitcnt(0x0F70);  // (the compiler's own loads: none is waited for in the loop, behind its copies)
      // A slot's turn: what it holds has landed; with several waves a stream, everyone is done with the slot before it, which is
      // filled again.
      auto begin = [&](int q) {
        if (q < n_q) wait_slots<kAhead - 1, kPer>(issued - 1 - q);
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
      int q = 0;
      if (first == 0) {
        // (where streams meet at barriers, the others wait for the new keys' turns)
        for (int i = 0; i < (PARTS > 1 ? n_new : my_new); ++i) {
          if (my_new == 0) {
            if (PARTS > 1) __syncthreads();
            continue;
          }
          begin(q);
          new_keys<D, RB>(r, ring[stream][q % kDepth], q * kNewKeys, p.K, v_new, (uint32_t)(p.Hkv * D), depth, p.c_log2);
          end();
          ++q;
        }
      }
      const int rounds = PARTS > 1 ? (n_pages_0 - first < 64 ? n_pages_0 - first : 64) * kSubs : n_q - q0;
      for (int i = 0; i < rounds; ++i, ++q) {
        begin(q);
        if (q < n_q) {
          const int j = i / kSubs, visible = __builtin_amdgcn_readlane(keys, j) - i % kSubs * kSubKeys;
          const float ks = __builtin_bit_cast(float, __builtin_amdgcn_readlane(kcode, j) << 23);
          const float vs = __builtin_bit_cast(float, __builtin_amdgcn_readlane(vcode, j) << 23);
          cached_keys<D, E5M2, RB>(r, ring[stream][q % kDepth], k_off, v_off, ks, vs, visible, g, p.c_log2);
        }
        end();
      }
      if (PARTS > 1) __syncthreads();  // (the slots' last reads have left them)
    }

    // Merge of the waves that hold the same rows: each leaves reference, sum and O (32 rows at a time, in its part of the rings, 16
    // bytes of features by 16 bytes, the rows of feature group d4 in the order row ^ d4), and the threads add them up in order.
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
    constexpr int kRegion = 2 * kSlotBytes / 16;
    static_assert(32 * D / 4 <= kRegion, "32 rows of O must fit a wave's part of the rings");
    f32x4* regions = reinterpret_cast<f32x4*>(&ring[0][0][0]);
    const int l = lane_id();
    const size_t rec = ((size_t)kvh * gridDim.x + blockIdx.x) * 2 + (segment > 0 ? 1 : 0);
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
      if (rb > 0) __syncthreads();
#pragma unroll
      for (int db = 0; db < D / 32; ++db)
#pragma unroll
        for (int i4 = 0; i4 < 4; ++i4) {
          const int d4 = db * 8 + 2 * i4 + (l >> 5);
          regions[wave * kRegion + d4 * 32 + ((l ^ d4) & 31)] =
              f32x4{r.o[rb][db][4 * i4], r.o[rb][db][4 * i4 + 1], r.o[rb][db][4 * i4 + 2], r.o[rb][db][4 * i4 + 3]};
        }
      __syncthreads();
      const bool any_bad = (wave_bad[0] | wave_bad[1] | wave_bad[2] | wave_bad[3]) != 0;
      for (int item = wave * 64 + l; item < 32 * PARTS * (D / 4); item += kWaves * 64) {
        const int d4 = item % (D / 4), in_block = item / (D / 4) % 32, h = item / (32 * (D / 4));
        const int row = (h * RB + rb) * 32 + in_block;
        float M = stats[h][rb * 32 + in_block][0];
#pragma unroll
        for (int s = 1; s < kStreams; ++s) M = __builtin_fmaxf(M, stats[s * PARTS + h][rb * 32 + in_block][0]);
        float L = 0.f;
        f32x4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int s = 0; s < kStreams; ++s) {
          const int w = s * PARTS + h;
          const float f = exp2_fast(stats[w][rb * 32 + in_block][0] - M);
          L = __builtin_fmaf(stats[w][rb * 32 + in_block][1], f, L);
          o += regions[w * kRegion + d4 * 32 + (in_block ^ (d4 & 31))] * f;
        }
        if (whole) {
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
      if (rb == 0 && tid == 0 && kvh == 0) {
        if (whole && p.status) p.status[c] = any_bad;
        // where the request's records stand: the first, and how many workgroups leave one
        if (share > 0 && skip == 0) sp.pieces[c] = make_int2((int)blockIdx.x * 2 + (segment > 0 ? 1 : 0), 1 + (units - n_units + share - 1) / share);
      }
    }
    left -= n_units;
    skip = 0;
    if (sp.shares == 0 || ++c >= p.C || left <= 0) return;
    __syncthreads();  // the merge's reads have left the rings
  }
}

// Merges a request's partial records: M = max m_s, L = sum l_s 2^(m_s - M), O = sum O_s 2^(m_s - M) / L.  kLanes threads per (row,
// 4 features) take the records in turn, kEach at a time, whose loads are issued before the first is used.
template <int D>
__global__ __launch_bounds__(256) void draft_scaled_combine_kernel(ScaledDecodeParams sp) {
  constexpr int kLanes = 256 / D, kEach = 4;
  const DecodeParams& p = sp.d;
  const int lane = threadIdx.x & 63, d4 = lane % (D / 4), sl = lane / (D / 4);
  const int kvh = blockIdx.y, c = blockIdx.z, n_rows = p.K * p.group;
  const int2 piece = sp.pieces[c];
  const int n = piece.y;
  if (n <= 1) return;  // (its workgroup has left the results)
  const int row = (int)blockIdx.x * 4 + (int)(threadIdx.x >> 6);
  if (row >= n_rows) return;
  // record 0 may be its workgroup's second, the others are their workgroups' first
  const size_t rec0 = (size_t)kvh * sp.shares * 2;
  auto record = [&](int s) { return rec0 + (s == 0 ? piece.x : (piece.x / 2 + s) * 2); };
  float M = -3.402823466e38f, L = 0.f;
  f32x4 acc = {0.f, 0.f, 0.f, 0.f};
  bool bad = false;
  for (int s0 = 0; s0 < n; s0 += kLanes * kEach) {
    float mv[kEach], lv[kEach], fv[kEach];
    f32x4 ov[kEach];
#pragma unroll
    for (int j = 0; j < kEach; ++j) {  // (records past the last are read as the last and weigh nothing)
      const int s = s0 + j * kLanes + sl;
      const size_t rec = record(s < n ? s : n - 1);
      const float* ml = p.part_ml + rec * 3 * p.rows_pad + row;
      mv[j] = ml[0];
      lv[j] = ml[p.rows_pad];
      fv[j] = ml[2 * p.rows_pad];
      ov[j] = *reinterpret_cast<const f32x4*>(p.part_o + (rec * p.rows_pad + row) * D + d4 * 4);
    }
    float m_new = M;
#pragma unroll
    for (int j = 0; j < kEach; ++j) m_new = __builtin_fmaxf(m_new, mv[j]);
    const float turn = exp2_fast(M - m_new);
    M = m_new;
    L *= turn;
    acc *= turn;
#pragma unroll
    for (int j = 0; j < kEach; ++j) {
      const float w = s0 + j * kLanes + sl < n ? exp2_fast(mv[j] - M) : 0.f;
      L = __builtin_fmaf(lv[j], w, L);
      acc += ov[j] * w;
      bad |= fv[j] != 0.f;
    }
  }
#pragma unroll
  for (int x = D / 4; x < 64; x <<= 1) {
    const float m_other = __shfl_xor(M, x), l_other = __shfl_xor(L, x), m_new = __builtin_fmaxf(M, m_other);
    const float a = exp2_fast(M - m_new), b = exp2_fast(m_other - m_new);
    M = m_new;
    L = L * a + l_other * b;
#pragma unroll
    for (int j = 0; j < 4; ++j) acc[j] = acc[j] * a + __shfl_xor(acc[j], x) * b;
  }
  if (p.status && row == 0 && kvh == 0) {
    const bool any = __builtin_amdgcn_ballot_w64(bad) != 0;
    if (lane == 0) p.status[c] = any;
  }
  if (sl != 0) return;
  const float inv = 1.0f / L;
  const int depth = small_quotient(row, p.group_reciprocal), head = kvh * p.group + (row - depth * p.group);
  u32x2 out;
  out[0] = pack_bf16(acc[0] * inv, acc[1] * inv);
  out[1] = pack_bf16(acc[2] * inv, acc[3] * inv);
  *reinterpret_cast<u32x2*>(p.o + (((size_t)c * p.K + depth) * p.Hq + head) * D + d4 * 4) = out;
  if (d4 == 0) p.lse[((size_t)c * p.Hq + head) * p.K + depth] = (M + __builtin_log2f(L)) * kLn2;
}

constexpr int kCus = 256;  // compute units of the device
constexpr int kLeastShare = 8;  // pages

}  // namespace

// Workgroups that share the work of a KV head, 0: a workgroup for each request.
int draft_scaled_shares(int C, int Hkv, int max_pages) {
  if (C > 1024 || max_pages < kLeastShare || (int64_t)C * (max_pages + 1) > INT_MAX) return 0;
  const int64_t slots = (2 * kCus + Hkv - 1) / Hkv, most = ((int64_t)C * (max_pages + 1) + kLeastShare - 1) / kLeastShare;
  return (int)(slots < most ? slots : most);
}

hipError_t launch_draft_scaled(const ScaledDecodeParams& pin, int D, bool e5m2, hipStream_t stream) {
  ScaledDecodeParams p = pin;
  p.d.group = p.d.Hq / p.d.Hkv;
  p.d.group_reciprocal = small_reciprocal(p.d.group);
  p.least_share = kLeastShare;
  const dim3 grid((unsigned)(p.shares > 0 ? p.shares : p.d.C), (unsigned)p.d.Hkv);
  auto run = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, dim3(kWaves * 64), 0, stream, p); };
  auto go = [&](auto type) {
    constexpr bool T = decltype(type)::value;
    const int blocks = p.d.rows_pad / 32;
    if (D == 64) {
      if (blocks == 1) run(draft_scaled_kernel<64, T, 1, 1>);
      else if (blocks == 2) run(draft_scaled_kernel<64, T, 2, 1>);
      else run(draft_scaled_kernel<64, T, 2, 2>);
    } else {
      if (blocks == 1) run(draft_scaled_kernel<128, T, 1, 1>);
      else if (blocks == 2) run(draft_scaled_kernel<128, T, 1, 2>);
      else run(draft_scaled_kernel<128, T, 1, 4>);
    }
  };
  e5m2 ? go(std::true_type{}) : go(std::false_type{});
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || p.shares == 0) return e;
  const dim3 rows((unsigned)((p.d.K * p.d.group + 3) / 4), (unsigned)p.d.Hkv, (unsigned)p.d.C);
  if (D == 64) hipLaunchKernelGGL(draft_scaled_combine_kernel<64>, rows, dim3(256), 0, stream, p);
  else hipLaunchKernelGGL(draft_scaled_combine_kernel<128>, rows, dim3(256), 0, stream, p);
  return hipGetLastError();
}

}  // namespace peagle
