// The paged cache of the drafting step between the steps: block tables and slot maps from request lengths, and new tokens'
// keys and values stored in 8 bits with one power-of-two scale for each page and KV head.
#include "cache_kernels.h"
#include "mfma_util.h"

namespace peagle {

namespace {

// Sum of x over the lanes up to and including this one.
__device__ __forceinline__ int64_t wave_scan(int64_t x, int lane) {
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const int64_t y = __shfl_up(x, d);
    x += lane >= d ? y : 0;
  }
  return x;
}

// Sum of x over the threads before this one, and over all of them in `total`.  sums: an entry for each wave; the caller's
// barriers keep one call's use of it apart from the next's.
__device__ __forceinline__ int64_t block_scan(int64_t x, int64_t* sums, int64_t& total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, waves = blockDim.x >> 6;
  const int64_t up_to = wave_scan(x, lane);
  if (lane == 63) sums[wave] = up_to;
  __syncthreads();
  int64_t before = 0;
  total = 0;
  for (int w = 0; w < waves; ++w) {
    before += w < wave ? sums[w] : 0;
    total += sums[w];
  }
  return before + up_to - x;
}

__device__ __forceinline__ int pages_of(int64_t tokens) { return (int)((tokens + kKeysPerTile - 1) / kKeysPerTile); }

// Largest i < n with list[i] <= x; list ascends and list[0] <= x.
template <class T>
__device__ __forceinline__ int last_not_above(const T* list, int n, T x) {
  int lo = 0;
  while (n > 1) {
    const int half = n >> 1;
    lo += list[lo + half] <= x ? half : 0;
    n -= half;
  }
  return lo;
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

// Slots of the new tokens [first, last) by this workgroup's threads.  starts[i]: row of the first new token of request
// i * stride, n_starts of them; total: rows in all.
__device__ __forceinline__ void write_slots(const PlanParams& p, const int* starts, int n_starts, int stride, int total, int first,
                                            int last) {
  for (int t = first + (int)threadIdx.x; t < last; t += (int)blockDim.x) {
    int64_t slot = -1;
    if (t < total) {
      int c = last_not_above(starts, n_starts, t) * stride;
      if (stride > 1) c += last_not_above(p.token_start + c, min(stride, p.C - c), t);
      const PlanRecord r = p.records[c];
      if (r.held >= 0) {
        const int pos = r.ctx + (t - r.start), b = pos / kKeysPerTile;
        int32_t* entry = p.block_table + (size_t)c * p.max_pages + b;
        int page;
        if (b < r.held) {
          page = *entry;
        } else {  // a page from the list; the token that begins the block enters it in the table
          page = p.free_pages[r.take - (b - r.held)];
          if (pos % kKeysPerTile == 0) *entry = page;
        }
        if (page >= 0 && page < p.n_pages) slot = (int64_t)page * kKeysPerTile + pos % kKeysPerTile;
      }
    }
    p.slots[t] = slot;
  }
}

// One workgroup: sums over the requests, in order, of new tokens, of pages that are given back and of pages that are lacking;
// the pages given back go on the list.  The slots follow here where they are few, otherwise in plan_slots_kernel.
// A call's time is memory round trips one after the other - lengths, tables or list, slots -, not bandwidth.
__global__ __launch_bounds__(kPlanThreads) void plan_kernel(PlanParams p, bool with_slots) {
  __shared__ int64_t sums[3][kPlanThreads / 64];
  __shared__ int64_t given_before[kPlanThreads];  // pages that the requests before each of a round's give back
  __shared__ int given_from[kPlanThreads];        // ... and the first block that it gives back
  __shared__ int starts[kPlanThreads];
  const int tid = threadIdx.x, n_threads = blockDim.x;
  const int rounds = (p.C + n_threads - 1) / n_threads;

  // What is given back is put on the list in reverse, so that its first page ends up on top: places depend on the total.
  int64_t given = 0;
  if (rounds > 1) {
    int64_t rows = 0, total;
    for (int r = 0; r < rounds; ++r) {
      const PlanRequest q = plan_request(p, r * n_threads + tid);
      const int64_t before = rows + block_scan(q.rows, sums[0], total);
      rows += total;
      block_scan(q.ok && before + q.rows <= p.max_tokens ? (q.held > q.want ? q.held - q.want : 0) : 0, sums[1], total);
      given += total;
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
    int64_t rows_here, given_here, lacking_here;
    const int64_t row0 = rows + block_scan(q.rows, sums[0], rows_here);
    q.ok = q.ok && row0 + q.rows <= p.max_tokens;
    if (!q.ok) q.want = q.held;
    const int gives = q.held > q.want ? q.held - q.want : 0, lacks = q.want > q.held ? q.want - q.held : 0;
    const int64_t gives_before = block_scan(gives, sums[1], given_here), need0 = lacked + block_scan(lacks, sums[2], lacking_here);
    if (rounds == 1) given = given_here;
    there = count + given < p.n_pages ? count + given : p.n_pages;
    const bool served = q.ok && (lacks == 0 || need0 + lacks <= there);
    given_before[tid] = gives_before;
    given_from[tid] = q.want;
    const int start = row0 < p.max_tokens ? (int)row0 : p.max_tokens;
    starts[tid] = start;
    if (c < p.C) {
      p.token_start[c] = start;
      p.status[c] = !q.ok ? 1 : served ? 0 : 2;
      p.seq_len[c] = q.ctx + (served ? (int)q.rows : 0);
      p.held_out[c] = served ? q.want : q.held;
      p.records[c] = PlanRecord{served ? q.held : -1, (int)(there - 1 - need0), q.ctx, start};
    }
    // (requests are served in order: those that lack pages and get them come before all that do not)
    const int64_t mine = served ? need0 + lacks : 0;
    rows += rows_here;
    lacked += lacking_here;
    __syncthreads();
    for (int64_t k = tid; k < given_here; k += n_threads) {
      const int i = last_not_above<int64_t>(given_before, n_threads, k);
      const int64_t at = count + given - 1 - (gave + k);
      if (at < p.n_pages)
        p.free_pages[at] = p.block_table[(size_t)(r * n_threads + i) * p.max_pages + given_from[i] + (int)(k - given_before[i])];
    }
    gave += given_here;
    int64_t best = lacks > 0 ? mine : 0;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
      const int64_t y = __shfl_xor(best, d);
      best = y > best ? y : best;
    }
    if ((tid & 63) == 0) sums[0][tid >> 6] = best;
    __syncthreads();
    for (int w = 0; w < n_threads / 64; ++w) taken = sums[0][w] > taken ? sums[0][w] : taken;
    __syncthreads();
  }
  const int total = rows < p.max_tokens ? (int)rows : p.max_tokens;
  if (tid == 0) {
    p.token_start[p.C] = total;
    *p.free_count_out = (int)(there - taken);
  }
  if (with_slots) write_slots(p, starts, p.C, 1, total, 0, p.max_tokens);
}

constexpr int kSlotsPerGroup = 1024;
__global__ __launch_bounds__(256) void plan_slots_kernel(PlanParams p, int stride) {
  __shared__ int starts[kPlanThreads];
  const int n = (p.C + stride - 1) / stride;
  for (int i = threadIdx.x; i < n; i += 256) starts[i] = p.token_start[i * stride];
  __syncthreads();
  const int first = blockIdx.x * kSlotsPerGroup, last = min(first + kSlotsPerGroup, p.max_tokens);
  write_slots(p, starts, n, stride, p.token_start[p.C], first, last);
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
// per_wave consecutive tokens (most tokens begin none) and stores each: all its rows are loaded before the first is waited for,
// their largest value gives the scale, and what the page holds before the run is turned to the new scale if that is larger.
// Every value is read and written once, so bandwidth bounds a large call, memory round trips (slots; rows and the old scale) a
// small one.
template <int D, bool E5M2>
__global__ __launch_bounds__(256) void cache_append_kernel(AppendParams p) {
  constexpr int kLanes = D / 8, kRows = 64 / kLanes;  // lanes of a row, rows a load
  constexpr int kLoads = kKeysPerTile / kRows;        // of a whole page
  const int lane = threadIdx.x & 63;
  const int which = __builtin_amdgcn_readfirstlane((int)(blockIdx.y * 4 + (threadIdx.x >> 6)));  // K of head 0, 1, ..., V of head 0, ...
  if (which >= 2 * p.Hkv) return;
  const bool is_v = which >= p.Hkv;
  const int head = is_v ? which - p.Hkv : which;
  const __bf16* src = (is_v ? p.v_new : p.k_new) + (size_t)head * D + (lane % kLanes) * 8;
  const int64_t stride = is_v ? p.v_stride : p.k_stride;
  uint8_t* pages = is_v ? p.v_pages : p.k_pages;
  uint8_t* scales = is_v ? p.v_scale : p.k_scale;
  const int row0 = lane / kLanes;

  const int t0 = (int)blockIdx.x * p.per_wave;
  const int64_t limit = (int64_t)p.n_pages * kKeysPerTile;
  const int t_mine = t0 + lane;
  const int64_t slot = t_mine < p.n_tokens ? p.slots[t_mine] : -1;
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
    const bool follows = off + lane < kKeysPerTile && t + lane < p.n_tokens && p.slots[t + lane] == s + lane;
    const uint64_t apart = ~__builtin_amdgcn_ballot_w64(follows);
    const int n = apart == 0 ? 64 : __builtin_ctzll(apart);

    u32x4 x[kLoads];
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const int row = i * kRows + row0;
      x[i] = u32x4{0u, 0u, 0u, 0u};
      if (row < n) x[i] = *reinterpret_cast<const u32x4*>(src + (int64_t)(t + row) * stride);
    }
    uint32_t amax = 0;  // bits of |x|: they order as the values do
#pragma unroll
    for (int i = 0; i < kLoads; ++i)
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
    const int code = off == 0 || fresh_code > old_code ? fresh_code : old_code;
    if (code != old_code && lane == 0) scales[page_head] = (uint8_t)code;

    const float f = code < 254 ? power_of(254 - code) : 0.f;  // 2^-(code - 127); no append leaves a larger code
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
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
    if (off > 0 && code > old_code) {
      const int by = code - old_code;
      const float turn = power_of(by > 126 ? 1 : 127 - by);
      for (int row = row0; row < off; row += kRows) {
        u32x2* at = reinterpret_cast<u32x2*>(page + row * D + (lane % kLanes) * 8);
        u32x2 w = *at;
        w[0] = turn4<E5M2>(w[0], turn);
        w[1] = turn4<E5M2>(w[1], turn);
        *at = w;
      }
    }
  }
}

}  // namespace

hipError_t launch_cache_plan(const PlanParams& p, hipStream_t stream) {
  const bool one = p.C <= kPlanThreads && p.max_tokens <= 4096;
  const int most = one && p.max_tokens > p.C ? p.max_tokens : p.C;
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
  p.per_wave = 1;
  while (p.per_wave < 64 && (int64_t)p.n_tokens * 2 * p.Hkv > 4096 * (int64_t)p.per_wave) p.per_wave *= 2;
  const dim3 grid((unsigned)((p.n_tokens + p.per_wave - 1) / p.per_wave), (unsigned)((2 * p.Hkv + 3) / 4));
  auto run = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, dim3(256), 0, stream, p); };
  if (D == 64) e5m2 ? run(cache_append_kernel<64, true>) : run(cache_append_kernel<64, false>);
  else e5m2 ? run(cache_append_kernel<128, true>) : run(cache_append_kernel<128, false>);
  return hipGetLastError();
}

}  // namespace peagle
