// The paged cache of the drafting step between the steps: block tables and slot maps from request lengths, and new tokens'
// keys and values stored in 8 bits with one power-of-two scale for each page and KV head.
#include "cache_kernels.h"
#include "mfma_util.h"

#include <type_traits>

namespace peagle {

namespace {

// x of the lane that the DPP control `CTRL` names, 0 where there is none or the row mask leaves the lane out.
template <int CTRL, int ROWS, bool BOUND>
__device__ __forceinline__ int64_t from_lane(int64_t x) {
  const uint32_t lo = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, CTRL, ROWS, 0xf, BOUND);
  const int hi = __builtin_amdgcn_update_dpp(0, (int)(x >> 32), CTRL, ROWS, 0xf, BOUND);
  return ((int64_t)hi << 32) | lo;
}
// Sum of x over the lanes of a row of 16, or of the wave, up to and including this one.
__device__ __forceinline__ int64_t row_scan(int64_t x) {
  x += from_lane<0x111, 0xf, true>(x);  // from 1, 2, 4, 8 lanes below
  x += from_lane<0x112, 0xf, true>(x);
  x += from_lane<0x114, 0xf, true>(x);
  x += from_lane<0x118, 0xf, true>(x);
  return x;
}
__device__ __forceinline__ int64_t wave_scan(int64_t x) {
  x = row_scan(x);
  x += from_lane<0x142, 0xa, false>(x);  // the last lane of rows 0 and 2 to rows 1 and 3
  x += from_lane<0x143, 0xc, false>(x);  // lane 31 to rows 2 and 3
  return x;
}
__device__ __forceinline__ int64_t lane_of(int64_t x, int lane) {
  return ((int64_t)__builtin_amdgcn_readlane((int)(x >> 32), lane) << 32) | (uint32_t)__builtin_amdgcn_readlane((int)x, lane);
}

// N sums over the threads before this one, and over all of them in `total`.  sums: N entries for each of up to 16 waves; the
// caller's barriers keep one call's use of them apart from the next's.
template <int N>
__device__ __forceinline__ void block_scan(const int64_t (&x)[N], int64_t (*sums)[16], int64_t (&before)[N], int64_t (&total)[N]) {
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), waves = blockDim.x >> 6;
  int64_t up_to[N];
#pragma unroll
  for (int k = 0; k < N; ++k) {
    up_to[k] = wave_scan(x[k]);
    if (lane == 63) sums[k][wave] = up_to[k];
  }
  __syncthreads();
#pragma unroll
  for (int k = 0; k < N; ++k) {
    const int64_t through = row_scan((lane & 15) < waves ? sums[k][lane & 15] : 0);
    total[k] = lane_of(through, 15);
    before[k] = up_to[k] - x[k] + (wave > 0 ? lane_of(through, wave - 1) : 0);
  }
}

__device__ __forceinline__ int pages_of(int64_t tokens) { return (int)((tokens + kKeysPerTile - 1) / kKeysPerTile); }

// Largest i < n with list[i] <= x, for some x at a time (each is a chain of reads); list ascends and list[0] <= x.
constexpr int kPlanEach = 4;
template <class T, int N>
__device__ __forceinline__ void last_not_above(const T* list, int n, const T (&x)[N], int (&at)[N]) {
#pragma unroll
  for (int e = 0; e < N; ++e) at[e] = 0;
  while (n > 1) {
    const int half = n >> 1;
#pragma unroll
    for (int e = 0; e < N; ++e) at[e] += list[at[e] + half] <= x[e] ? half : 0;
    n -= half;
  }
}

constexpr int kPlanThreads = 1024;  // requests that the plan kernel takes at a time

// A request as the call finds it.
struct PlanRequest {
  int ctx, held, want;  // cached tokens; pages held, and to be held if it is served
  int64_t rows;         // of the new tokens' arrays
  bool ok;              // lengths in range
};
__device__ __forceinline__ PlanRequest plan_request(const PlanParams& p, int c) {
  PlanRequest r{0, 0, 0, 0, false};
  if (c >= p.C) return r;
  const int fresh = p.new_len[c];
  r.ctx = p.ctx_len[c];
  r.held = p.held[c];
  r.rows = fresh > 0 ? fresh : 0;
  const int64_t len = (int64_t)r.ctx + fresh;
  r.ok = r.ctx >= 0 && fresh >= 0 && len <= (int64_t)p.max_pages * kKeysPerTile && r.held >= pages_of(r.ctx) && r.held <= p.max_pages;
  r.want = r.ok ? pages_of(len) : r.held;
  return r;
}

// Slots of the new tokens [first, last) by this workgroup's threads, some at a time, as each is a chain of reads.  starts[i]: row
// of the first new token of request i * stride, n_starts of them; total: rows in all.
__device__ __forceinline__ void write_slots(const PlanParams& p, const PlanRecord* records, const int* starts, int n_starts, int stride,
                                            int total, int first, int last) {
  constexpr int kEach = kPlanEach;
  for (int t0 = first + (int)threadIdx.x; t0 < last; t0 += kEach * (int)blockDim.x) {
    int x[kEach], at[kEach];
#pragma unroll
    for (int e = 0; e < kEach; ++e) x[e] = t0 + e * (int)blockDim.x;
    last_not_above(starts, n_starts, x, at);
    int page[kEach], pos[kEach];
    int32_t* entry[kEach];  // of the table, for a token that enters its page there
#pragma unroll
    for (int e = 0; e < kEach; ++e) {
      const int t = x[e];
      page[e] = -1;
      entry[e] = nullptr;
      if (t >= total || t >= last) continue;
      int c = at[e] * stride;
      if (stride > 1) {
        int more[1];
        last_not_above(p.token_start + c, min(stride, p.C - c), {t}, more);
        c += more[0];
      }
      const PlanRecord r = records[c];
      if (r.held < 0) continue;
      pos[e] = r.ctx + (t - r.start);
      const int b = pos[e] / kKeysPerTile;
      int32_t* place = p.block_table + (size_t)c * p.max_pages + b;
      if (b >= r.held && pos[e] % kKeysPerTile == 0) entry[e] = place;
      page[e] = *(b < r.held ? place : p.free_pages + (r.take - (b - r.held)));
    }
#pragma unroll
    for (int e = 0; e < kEach; ++e) {
      const int t = x[e];
      if (entry[e]) *entry[e] = page[e];
      if (t < last) p.slots[t] = page[e] >= 0 && page[e] < p.n_pages ? (int64_t)page[e] * kKeysPerTile + pos[e] % kKeysPerTile : -1;
    }
  }
}

// One workgroup: sums over the requests, in order, of new tokens, of pages that are given back and of pages that are lacking;
// the pages given back go on the list.  The slots follow here where they are few, otherwise in plan_slots_kernel.
// A call's time is memory round trips one after the other - lengths, tables or list, slots -, not bandwidth.
__global__ __launch_bounds__(kPlanThreads) void plan_kernel(PlanParams p, bool with_slots) {
  __shared__ int64_t sums[4][kPlanThreads / 64];
  __shared__ int64_t given_before[kPlanThreads];  // pages that the requests before each of a round's give back
  __shared__ int given_from[kPlanThreads];        // ... and the first block that it gives back
  __shared__ int starts[kPlanThreads];
  __shared__ PlanRecord records[kPlanThreads];
  const int tid = threadIdx.x, lane = tid & 63, n_threads = blockDim.x;
  const int rounds = (p.C + n_threads - 1) / n_threads;

  // What is given back is put on the list in reverse, so that its first page ends up on top: places depend on the total.
  int64_t given = 0;
  if (rounds > 1) {
    int64_t rows = 0, before[1], total[1];
    for (int r = 0; r < rounds; ++r) {
      const PlanRequest q = plan_request(p, r * n_threads + tid);
      block_scan<1>({q.rows}, sums, before, total);
      const bool fits = q.ok && rows + before[0] + q.rows <= p.max_tokens;
      rows += total[0];
      block_scan<1>({fits && q.held > q.want ? q.held - q.want : 0}, sums + 1, before, total);
      given += total[0];
      __syncthreads();
    }
  }
  int count = *p.free_count;
  count = count < 0 ? 0 : count > p.n_pages ? p.n_pages : count;

  int64_t rows = 0, gave = 0, lacked = 0;  // sums over the rounds before
  int64_t there = 0, taken = 0;
  for (int r = 0; r < rounds; ++r) {
    const int c = r * n_threads + tid;
    PlanRequest q = plan_request(p, c);
    int64_t before[1], total[1];
    block_scan<1>({q.rows}, sums, before, total);
    const int64_t row0 = rows + before[0];
    q.ok = q.ok && row0 + q.rows <= p.max_tokens;
    if (!q.ok) q.want = q.held;
    const int gives = q.held > q.want ? q.held - q.want : 0, lacks = q.want > q.held ? q.want - q.held : 0;
    int64_t pages_before[2], pages[2];
    block_scan<2>({gives, lacks}, sums + 1, pages_before, pages);
    const int64_t need0 = lacked + pages_before[1], given_here = pages[0];
    if (rounds == 1) given = given_here;
    there = count + given < p.n_pages ? count + given : p.n_pages;
    const bool served = q.ok && (lacks == 0 || need0 + lacks <= there);
    given_before[tid] = pages_before[0];
    given_from[tid] = q.want;
    const int start = row0 < p.max_tokens ? (int)row0 : p.max_tokens;
    const PlanRecord record{served ? q.held : -1, (int)(there - 1 - need0), q.ctx, start};
    starts[tid] = start;
    records[tid] = record;
    if (c < p.C) {
      p.token_start[c] = start;
      p.status[c] = !q.ok ? 1 : served ? 0 : 2;
      p.seq_len[c] = q.ctx + (served ? (int)q.rows : 0);
      p.held_out[c] = served ? q.want : q.held;
      if (!with_slots) p.records[c] = record;
    }
    // (requests are served in order: the last that lacks pages and gets them has taken what all before it have, and its own)
    const uint64_t takers = __builtin_amdgcn_ballot_w64(served && lacks > 0);
    if (lane == (takers ? 63 - __builtin_clzll(takers) : 0)) sums[3][tid >> 6] = takers ? need0 + lacks : 0;
    rows += total[0];
    lacked += pages[1];
    __syncthreads();
    for (int64_t k0 = tid; k0 < given_here; k0 += kPlanEach * n_threads) {
      int64_t k[kPlanEach];
      int of[kPlanEach];
#pragma unroll
      for (int e = 0; e < kPlanEach; ++e) k[e] = k0 + e * n_threads;
      last_not_above(given_before, min(n_threads, p.C - r * n_threads), k, of);
#pragma unroll
      for (int e = 0; e < kPlanEach; ++e) {
        const int64_t at = count + given - 1 - (gave + k[e]);
        if (k[e] < given_here && at < p.n_pages)
          p.free_pages[at] = p.block_table[(size_t)(r * n_threads + of[e]) * p.max_pages + given_from[of[e]] + (int)(k[e] - given_before[of[e]])];
      }
    }
    gave += given_here;
    if (tid == 0)
      for (int w = 0; w < n_threads / 64; ++w) taken = sums[3][w] > taken ? sums[3][w] : taken;
    if (r + 1 < rounds || given_here > 0) __syncthreads();  // (before the arrays' next use, and of the pages given back)
  }
  const int total = rows < p.max_tokens ? (int)rows : p.max_tokens;
  if (tid == 0) {
    p.token_start[p.C] = total;
    *p.free_count_out = (int)(there - taken);
  }
  if (with_slots) write_slots(p, records, starts, p.C, 1, total, 0, p.max_tokens);
}

constexpr int kSlotsPerGroup = 1024;
__global__ __launch_bounds__(256) void plan_slots_kernel(PlanParams p, int stride) {
  __shared__ int starts[kPlanThreads];
  const int n = (p.C + stride - 1) / stride;
  for (int i = threadIdx.x; i < n; i += 256) starts[i] = p.token_start[i * stride];
  __syncthreads();
  const int first = blockIdx.x * kSlotsPerGroup, last = min(first + kSlotsPerGroup, p.max_tokens);
  write_slots(p, p.records, starts, n, stride, p.token_start[p.C], first, last);
}

// ------------------------------------------------------------------------------------------------------------ append

// Two values as two codes of the cache's type, rounded to nearest, ties to even (|x| at most the largest value, or not finite:
// the type's NaN or infinity).
template <bool E5M2>
__device__ __forceinline__ uint32_t narrow2(float a, float b, uint32_t old, bool high) {
  if (E5M2) return high ? __builtin_amdgcn_cvt_pk_bf8_f32(a, b, (int)old, true) : __builtin_amdgcn_cvt_pk_bf8_f32(a, b, (int)old, false);
  return high ? __builtin_amdgcn_cvt_pk_fp8_f32(a, b, (int)old, true) : __builtin_amdgcn_cvt_pk_fp8_f32(a, b, (int)old, false);
}
template <bool E5M2>
__device__ __forceinline__ uint32_t narrow4(float a, float b, float c, float d) {
  return narrow2<E5M2>(c, d, narrow2<E5M2>(a, b, 0, false), true);
}
// Four codes times f.
template <bool E5M2>
__device__ __forceinline__ uint32_t turn4(uint32_t w, float f) {
  float x[4];
  if (E5M2) {
    x[0] = __builtin_amdgcn_cvt_f32_bf8((int)w, 0);
    x[1] = __builtin_amdgcn_cvt_f32_bf8((int)w, 1);
    x[2] = __builtin_amdgcn_cvt_f32_bf8((int)w, 2);
    x[3] = __builtin_amdgcn_cvt_f32_bf8((int)w, 3);
  } else {
    x[0] = __builtin_amdgcn_cvt_f32_fp8((int)w, 0);
    x[1] = __builtin_amdgcn_cvt_f32_fp8((int)w, 1);
    x[2] = __builtin_amdgcn_cvt_f32_fp8((int)w, 2);
    x[3] = __builtin_amdgcn_cvt_f32_fp8((int)w, 3);
  }
  return narrow4<E5M2>(x[0] * f, x[1] * f, x[2] * f, x[3] * f);
}

__device__ __forceinline__ float low_bf16(uint32_t w) { return __builtin_bit_cast(float, w << 16); }
__device__ __forceinline__ float high_bf16(uint32_t w) { return __builtin_bit_cast(float, w & 0xffff0000u); }
// 2^(code - 127), code in [1, 254]
__device__ __forceinline__ float power_of(int code) { return __builtin_bit_cast(float, (uint32_t)code << 23); }

// Code of the smallest scale that holds `amax`, given as the bits of a non-negative finite bf16: the largest value of either
// type is 1.75 times a power of two, so the exponent tells, plus one where the fraction is above 0.75.
template <bool E5M2>
__device__ __forceinline__ int scale_code(uint32_t amax) {
  const int code = (int)(amax >> 7) - (E5M2 ? 15 : 8) + ((amax & 0x7fu) > 0x60u ? 1 : 0);
  return code < 127 + kMinScaleExponent ? 127 + kMinScaleExponent : code;
}

// Tokens of one run - consecutive slots of one page - of one KV head, K or V.  A wave looks for the runs that begin among
// per_wave consecutive tokens (most tokens begin none; the slots of the 64 behind its first are all it needs) and stores each: all
// its rows are loaded before the first is waited for, their largest value gives the scale, and what the page holds before the run
// is turned to the new scale if that is larger.  Every value is read and written once, so bandwidth bounds a large call (16 prompts
// of 203 to 16001 tokens, 4 heads of 128: 399 MB in 84 us on MI355X, 4.8 TB/s, the rate of a large copy), a launch and memory round
// trips (slots; rows and the old scale) a small one (256 requests' 1 to 8 tokens: 5.1 us; 11.8 where every page's scale grows).  The waves of a workgroup take chunks
// that follow each other, so that the workgroups of a prompt, whose runs begin 64 tokens apart, are equally busy: with the heads
// there instead, a prompt of 3891 tokens took 9.8 us rather than 5.8, as most XCDs had none.
constexpr int kAppendWaves = 4;
template <int D, bool E5M2>
__global__ __launch_bounds__(kAppendWaves * 64) void cache_append_kernel(AppendParams p) {
  constexpr int kLanes = D / 8, kRows = 64 / kLanes;  // lanes of a row, rows a load
  constexpr int kLoads = kKeysPerTile / kRows;        // of a whole page
  const int lane = threadIdx.x & 63;
  const int which = (int)blockIdx.x;  // K of head 0, 1, ..., V of head 0, ...
  const bool is_v = which >= p.Hkv;
  const int head = is_v ? which - p.Hkv : which;
  const __bf16* src = (is_v ? p.v_new : p.k_new) + (size_t)head * D + (lane % kLanes) * 8;
  const int64_t stride = is_v ? p.v_stride : p.k_stride;
  uint8_t* pages = is_v ? p.v_pages : p.k_pages;
  uint8_t* scales = is_v ? p.v_scale : p.k_scale;
  const int row0 = lane / kLanes;

  const int64_t chunk = ((int64_t)blockIdx.z * gridDim.y + blockIdx.y) * kAppendWaves + __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
  if (chunk * p.per_wave >= p.n_tokens) return;
  const int t0 = (int)(chunk * p.per_wave);
  const int64_t limit = (int64_t)p.n_pages * kKeysPerTile;
  const int t_mine = t0 + lane;
  const int64_t slot = t_mine < p.n_tokens ? p.slots[t_mine] : -1;
  const int64_t next = t_mine + 64 < p.n_tokens ? p.slots[t_mine + 64] : -1;  // (a run may reach behind the first 64)
  const int64_t before = t_mine > 0 && t_mine <= p.n_tokens ? p.slots[t_mine - 1] : -1;
  const bool stored = slot >= 0 && slot < limit;
  const bool begins = stored && lane < p.per_wave && !(before >= 0 && slot == before + 1 && slot % kKeysPerTile != 0);
  uint64_t runs = __builtin_amdgcn_ballot_w64(begins);
  while (runs != 0) {
    const int first = __builtin_ctzll(runs);
    runs &= runs - 1;
    const int t = t0 + first;
    const int64_t s = ((int64_t)__builtin_amdgcn_readlane((int)(slot >> 32), first) << 32) |
                      (uint32_t)__builtin_amdgcn_readlane((int)slot, first);
    const int off = (int)(s % kKeysPerTile);
    const size_t page_head = (size_t)(s / kKeysPerTile) * p.Hkv + head;
    uint8_t* page = pages + page_head * (kKeysPerTile * D);
    const int old_code = scales[page_head];
    // slots less their lanes' numbers are alike within a run
    const uint64_t in_run = __builtin_amdgcn_ballot_w64(stored && slot - lane == s - first) >> first;
    const uint64_t in_next = __builtin_amdgcn_ballot_w64(next >= 0 && next - lane == s + 64 - first);
    const uint64_t same = in_run | (first > 0 ? in_next << (64 - first) : 0);
    const uint64_t on_page = ~0ull >> off;  // (a run ends with its page)
    const uint64_t apart = ~(same & on_page);
    const int n = apart == 0 ? 64 : __builtin_ctzll(apart);

    int code = 0;
    auto store_run = [&](auto loads) {  // a run of at most loads x kRows rows
      constexpr int kRun = decltype(loads)::value;
      u32x4 x[kRun];
#pragma unroll
      for (int i = 0; i < kRun; ++i) {
        const int row = i * kRows + row0;
        x[i] = u32x4{0u, 0u, 0u, 0u};
        if (row < n) x[i] = *reinterpret_cast<const u32x4*>(src + (int64_t)(t + row) * stride);
      }
      uint32_t amax = 0;  // bits of |x|: they order as the values do
#pragma unroll
      for (int i = 0; i < kRun; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const uint32_t w = x[i][j], lo = w & 0x7fffu, hi = (w >> 16) & 0x7fffu;
          amax = max(amax, lo < 0x7f80u ? lo : 0u);  // (infinities and NaN take no part)
          amax = max(amax, hi < 0x7f80u ? hi : 0u);
        }
#pragma unroll
      for (int d = 1; d < 64; d <<= 1) amax = max(amax, (uint32_t)__shfl_xor((int)amax, d));
      amax = (uint32_t)__builtin_amdgcn_readfirstlane((int)amax);
      const int fresh_code = scale_code<E5M2>(amax);
      code = off == 0 || fresh_code > old_code ? fresh_code : old_code;
      if (code != old_code && lane == 0) scales[page_head] = (uint8_t)code;
      const float f = code < 254 ? power_of(254 - code) : 0.f;  // 2^-(code - 127); no append leaves a larger code
#pragma unroll
      for (int i = 0; i < kRun; ++i) {
        const int row = i * kRows + row0;
        if (row >= n) continue;
        u32x2 w;
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const uint32_t a = x[i][2 * j], b = x[i][2 * j + 1];
          w[j] = narrow4<E5M2>(low_bf16(a) * f, high_bf16(a) * f, low_bf16(b) * f, high_bf16(b) * f);
        }
        *reinterpret_cast<u32x2*>(page + (off + row) * D + (lane % kLanes) * 8) = w;
      }
    };
    // (the few tokens of a decoding step without the instructions of a whole page)
    if (n <= 2 * kRows) store_run(std::integral_constant<int, 2>());
    else store_run(std::integral_constant<int, kLoads>());
    if (off > 0 && code > old_code) {
      const int by = code - old_code;
      const float turn = power_of(by > 126 ? 1 : 127 - by);
      u32x2* old = reinterpret_cast<u32x2*>(page + row0 * D + (lane % kLanes) * 8);
      u32x2 w[kLoads];
#pragma unroll
      for (int i = 0; i < kLoads; ++i)
        if (i * kRows + row0 < off) w[i] = old[i * kRows * D / 8];
#pragma unroll
      for (int i = 0; i < kLoads; ++i)
        if (i * kRows + row0 < off) old[i * kRows * D / 8] = u32x2{turn4<E5M2>(w[i][0], turn), turn4<E5M2>(w[i][1], turn)};
    }
  }
}

// ------------------------------------------------------------------------------------- rows to 4 bits, and rows back

// Eight features of a token a lane: D / 8 lanes a token's KV head, 64 / (D / 8) tokens a wave and step, kRowSteps steps a wave.  All
// loads of a wave are issued before the first is used.  (Two steps: with four 130 k tokens of 4 heads of 128 features are stored
// in 67.8 us instead of 64.9, with one as fast but read back in 90.9 instead of 79.5.)
constexpr int kRowSteps = 2, kRowWaves = 4;
template <int D>
struct RowLane {
  static constexpr int kLanes = D / 8, kTokens = 64 / kLanes;
  const bool is_v;
  const int head, lane, chunk;  // chunk: which eight features
  int64_t first;                // token of step 0
  __device__ __forceinline__ explicit RowLane(const RowsParams& p)
      : is_v((int)blockIdx.x >= p.Hkv), head(is_v ? (int)blockIdx.x - p.Hkv : (int)blockIdx.x), lane(threadIdx.x & 63), chunk(lane % kLanes) {
    const int64_t wave = ((int64_t)blockIdx.z * gridDim.y + blockIdx.y) * kRowWaves + (threadIdx.x >> 6);
    first = wave * (kRowSteps * kTokens) + lane / kLanes;
  }
};

// A block of 32 features of one token and KV head: the smallest scale 2^e that brings its largest value to 6 or below, the code of
// each value times 2^-e.  Both come from integers and one instruction for two values: of the bits of |x| the largest tells the
// exponent (6 is 1.5 times a power of two, so one more where the fraction is above 0.5).
// Bound: memory.  STREAM: the rows are read past the caches.
template <int D, bool STREAM>
__global__ __launch_bounds__(kRowWaves * 64) void cache_append_blocks_kernel(RowsParams p) {
  using L = RowLane<D>;
  const L at(p);
  const __bf16* rows = (at.is_v ? p.v_rows : p.k_rows) + (size_t)at.head * D + at.chunk * 8;
  const int64_t stride = at.is_v ? p.v_stride : p.k_stride, limit = (int64_t)p.n_pages * kKeysPerTile;
  uint8_t* pages = at.is_v ? p.v_pages : p.k_pages;
  uint8_t* scales = at.is_v ? p.v_scale : p.k_scale;
  int64_t slot[kRowSteps];
  u32x4 x[kRowSteps];
#pragma unroll
  for (int i = 0; i < kRowSteps; ++i) {
    const int64_t t = at.first + i * L::kTokens;
    slot[i] = -1;
    x[i] = u32x4{0u, 0u, 0u, 0u};
    if (t < p.n_tokens) {
      slot[i] = p.slots[t];
      const u32x4* row = reinterpret_cast<const u32x4*>(rows + t * stride);
      x[i] = STREAM ? __builtin_nontemporal_load(row) : *row;
    }
  }
#pragma unroll
  for (int i = 0; i < kRowSteps; ++i) {
    uint32_t amax = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const uint32_t w = x[i][j];
      amax = max(amax, max(w & 0x7fffu, (w >> 16) & 0x7fffu));
    }
    amax = max(amax, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)amax, 0xb1, 0xf, 0xf, true));  // the other lane of each pair,
    amax = max(amax, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)amax, 0x4e, 0xf, 0xf, true));  // the other pair of each four
    int code = (int)((amax + 0x3fu) >> 7) - 2;
    code = code < 127 + kMinScaleExponent ? 127 + kMinScaleExponent : code;
    const float scale = power_of(code);
    uint32_t codes = 0;
    auto two = [&](uint32_t w) { return __builtin_bit_cast(bf16x2, w); };
    codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(codes, two(x[i][0]), scale, 0);
    codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(codes, two(x[i][1]), scale, 1);
    codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(codes, two(x[i][2]), scale, 2);
    codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(codes, two(x[i][3]), scale, 3);
    if (amax >= 0x7f80u) {  // an infinity or NaN: 4 bits have neither, the scale has NaN
      code = 255;
      codes = 0;
    }
    // a token's scale codes to its first lane
    code |= __builtin_amdgcn_update_dpp(0, code, 0x104, 0xf, 0xf, true) << 8;  // from 4 lanes above
    if (D == 128) code |= __builtin_amdgcn_update_dpp(0, code, 0x108, 0xf, 0xf, true) << 16;
    if (slot[i] < 0 || slot[i] >= limit) continue;
    const size_t place = ((size_t)(slot[i] / kKeysPerTile) * p.Hkv + at.head) * kKeysPerTile + (size_t)(slot[i] % kKeysPerTile);
    reinterpret_cast<uint32_t*>(pages)[place * (D / 8) + at.chunk] = codes;
    if (at.chunk == 0) {
      if (D == 64) reinterpret_cast<uint16_t*>(scales)[place] = (uint16_t)code;
      else reinterpret_cast<uint32_t*>(scales)[place] = (uint32_t)code;
    }
  }
}

// PAST: the rows leave past the caches (see the launch).
template <int D, CacheType T, bool PAST>
__global__ __launch_bounds__(kRowWaves * 64) void cache_read_kernel(RowsParams p) {
  using L = RowLane<D>;
  constexpr bool kFour = T == CacheType::kE2M1;
  const L at(p);
  __bf16* rows = (at.is_v ? p.v_rows : p.k_rows) + (size_t)at.head * D + at.chunk * 8;
  const int64_t stride = at.is_v ? p.v_stride : p.k_stride, limit = (int64_t)p.n_pages * kKeysPerTile;
  const uint8_t* pages = at.is_v ? p.v_pages : p.k_pages;
  const uint8_t* scales = at.is_v ? p.v_scale : p.k_scale;
  u32x2 w[kRowSteps];
  int code[kRowSteps];
  int64_t slot[kRowSteps];
#pragma unroll
  for (int i = 0; i < kRowSteps; ++i) {
    const int64_t t = at.first + i * L::kTokens;
    slot[i] = t < p.n_tokens ? p.slots[t] : -1;
  }
#pragma unroll
  for (int i = 0; i < kRowSteps; ++i) {
    w[i] = u32x2{0u, 0u};  // (zero, whatever the scale but NaN)
    code[i] = 127;
    if (slot[i] < 0 || slot[i] >= limit) continue;
    const size_t page_head = (size_t)(slot[i] / kKeysPerTile) * p.Hkv + at.head;
    const size_t place = page_head * kKeysPerTile + (size_t)(slot[i] % kKeysPerTile);
    if (kFour) {
      w[i][0] = reinterpret_cast<const uint32_t*>(pages)[place * (D / 8) + at.chunk];
      code[i] = scales[place * (D / 32) + at.chunk / 4];
    } else {
      w[i] = reinterpret_cast<const u32x2*>(pages)[place * (D / 8) + at.chunk];
      code[i] = scales[page_head];
    }
  }
#pragma unroll
  for (int i = 0; i < kRowSteps; ++i) {
    const int64_t t = at.first + i * L::kTokens;
    if (t >= p.n_tokens) continue;
    const float scale = __builtin_bit_cast(float, (uint32_t)code[i] << 23);
    const uint32_t a = w[i][0], b = w[i][1];
    u32x4 out;
    auto put = [&](int j, bf16x2 v) { out[j] = __builtin_bit_cast(uint32_t, v); };
    if (T == CacheType::kE2M1) {
      put(0, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(a, scale, 0));
      put(1, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(a, scale, 1));
      put(2, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(a, scale, 2));
      put(3, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(a, scale, 3));
    } else if (T == CacheType::kE5M2) {
      put(0, __builtin_amdgcn_cvt_scalef32_pk_bf16_bf8(a, scale, false));
      put(1, __builtin_amdgcn_cvt_scalef32_pk_bf16_bf8(a, scale, true));
      put(2, __builtin_amdgcn_cvt_scalef32_pk_bf16_bf8(b, scale, false));
      put(3, __builtin_amdgcn_cvt_scalef32_pk_bf16_bf8(b, scale, true));
    } else {
      put(0, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, scale, false));
      put(1, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, scale, true));
      put(2, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, scale, false));
      put(3, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, scale, true));
    }
    u32x4* row = reinterpret_cast<u32x4*>(rows + t * stride);
    if (PAST) __builtin_nontemporal_store(out, row);
    else *row = out;
  }
}

dim3 rows_grid(const RowsParams& p, int D) {
  const int64_t span = (int64_t)kRowWaves * kRowSteps * (64 / (D / 8)), spans = (p.n_tokens + span - 1) / span;
  const unsigned y = (unsigned)(spans < 32768 ? spans : 32768);
  return dim3((unsigned)(2 * p.Hkv), y, (unsigned)((spans + y - 1) / y));
}

}  // namespace

// Bytes of K and V rows that one kernel leaves in the last cache for the next.
constexpr int64_t kKeptRows = 72ll << 20;

hipError_t launch_cache_append_blocks(const RowsParams& p, int D, hipStream_t stream) {
  auto run = [&](auto kernel) { hipLaunchKernelGGL(kernel, rows_grid(p, D), dim3(kRowWaves * 64), 0, stream, p); };
  // Rows that the last cache (256 MiB) holds from the kernel that has written them are read from it, others past it.  That kernel (a
  // copy) and the append, D 64, past the cache and otherwise: 41 MB 24.2 and 24.0 us, 58 MB 31.5 and 31.1, 72 MB 37.5 and 37.2, 78 MB 39.9 and
  // 41.5, 90 MB 45.3 and 52.6, 110 MB 60.0 and 74.0, 128 MB 72.2 and 80.9, 266 MB 161 and 168; D 128 alike.  (Rows that nothing has written since the
  // cache took them are faster from it up to 110 MB, 25.9 against 30.2.)
  const bool large = (int64_t)p.n_tokens * p.Hkv * D * 4 > kKeptRows;
  if (D == 64) large ? run(cache_append_blocks_kernel<64, true>) : run(cache_append_blocks_kernel<64, false>);
  else large ? run(cache_append_blocks_kernel<128, true>) : run(cache_append_blocks_kernel<128, false>);
  return hipGetLastError();
}

// What is read is for a kernel that comes next: rows that the last cache (256 MiB) can hold for it stay there, others leave past it.
// Read and a copy of the rows, 8 heads of 64 features, 4 bits: 28 MB of rows 18.3 us (20.4 from codes that no cache holds), past the
// caches 20.7 (23.7), though the read by itself takes 7.8 instead of 6.1; 61 MB 32.7, past 37.5; 75 MB 45.1 and 45.3; 95 MB 65.3,
// past 63.3; 134 MB 94.5, past 91.0; 285 MB 195, past 188, and the read by itself 84 instead of 53.  (What only reads the rows gains
// from keeping them at each of these sizes: 5 to 8 % of both up to 134 MB, 2 % at 285.)
hipError_t launch_cache_read(const RowsParams& p, int D, CacheType cache, hipStream_t stream) {
  auto run = [&](auto kernel) { hipLaunchKernelGGL(kernel, rows_grid(p, D), dim3(kRowWaves * 64), 0, stream, p); };
  const bool past = (int64_t)p.n_tokens * p.Hkv * D * 4 > kKeptRows;
  auto go = [&](auto type) {
    constexpr CacheType T = decltype(type)::value;
    if (D == 64) past ? run(cache_read_kernel<64, T, true>) : run(cache_read_kernel<64, T, false>);
    else past ? run(cache_read_kernel<128, T, true>) : run(cache_read_kernel<128, T, false>);
  };
  switch (cache) {
    case CacheType::kE4M3: go(std::integral_constant<CacheType, CacheType::kE4M3>()); break;
    case CacheType::kE5M2: go(std::integral_constant<CacheType, CacheType::kE5M2>()); break;
    case CacheType::kE2M1: go(std::integral_constant<CacheType, CacheType::kE2M1>()); break;
  }
  return hipGetLastError();
}

hipError_t launch_cache_plan(const PlanParams& p, hipStream_t stream) {
  const bool one = p.C <= kPlanThreads && p.max_tokens <= 4096;
  // (a thread for each request, or for kPlanEach slots: 256 requests and 2048 slots take 6.4 us, with a thread a slot 7.4)
  const int per_thread = (p.max_tokens + kPlanEach - 1) / kPlanEach, most = one && per_thread > p.C ? per_thread : p.C;
  const int threads = most >= kPlanThreads ? kPlanThreads : (most + 63) / 64 * 64;
  hipLaunchKernelGGL(plan_kernel, dim3(1), dim3((unsigned)threads), 0, stream, p, one);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || one) return e;
  const int stride = (p.C + kPlanThreads - 1) / kPlanThreads;
  hipLaunchKernelGGL(plan_slots_kernel, dim3((unsigned)((p.max_tokens + kSlotsPerGroup - 1) / kSlotsPerGroup)), dim3(256), 0, stream, p,
                     stride);
  return hipGetLastError();
}

hipError_t launch_cache_append(const AppendParams& pin, int D, bool e5m2, hipStream_t stream) {
  AppendParams p = pin;
  // Some 4096 waves, whose chunks hold a run or less: 256 requests' new tokens take 5.1 us, 6.1 with 2048 waves, 8.1 with 1024, and
  // a prompt of 3891 tokens 5.5, 7.0 with 8192 and 11 with 65536, most of which find nothing.
  p.per_wave = 1;
  while (p.per_wave < 64 && (int64_t)p.n_tokens * 2 * p.Hkv > 4096 * (int64_t)p.per_wave) p.per_wave *= 2;
  const int64_t span = (int64_t)kAppendWaves * p.per_wave, spans = (p.n_tokens + span - 1) / span;
  const unsigned y = (unsigned)(spans < 32768 ? spans : 32768);
  const dim3 grid((unsigned)(2 * p.Hkv), y, (unsigned)((spans + y - 1) / y));
  auto run = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, dim3(kAppendWaves * 64), 0, stream, p); };
  if (D == 64) e5m2 ? run(cache_append_kernel<64, true>) : run(cache_append_kernel<64, false>);
  else e5m2 ? run(cache_append_kernel<128, true>) : run(cache_append_kernel<128, false>);
  return hipGetLastError();
}

}  // namespace peagle
