// Kernel parameter blocks and host launchers of the serving operators around the paged cache.
#pragma once

#include <hip/hip_runtime.h>

#include "attn_kernels.h"
#include "tilemap.h"

namespace peagle {

constexpr int kMinScaleExponent = -100;  // of a page's scale, see peagle_cache_append_scaled()

// What the slots of a request's new tokens are made of, left by the plan kernel for the kernel that writes them.
struct PlanRecord {
  int32_t held;   // pages that the request held before the call; -1: its tokens get no slot
  int32_t take;   // list index of the page of block `held`; the blocks that follow take the entries below it
  int32_t ctx;    // cached tokens
  int32_t start;  // row of its first new token
};

struct PlanParams {
  const int32_t* ctx_len;     // [C]
  const int32_t* new_len;     // [C]
  const int32_t* held;        // [C]
  int32_t* held_out;          // [C], may be `held`
  int32_t* free_pages;        // [n_pages]
  const int32_t* free_count;  // [1]
  int32_t* free_count_out;    // [1], may be `free_count`
  int32_t* block_table;       // [C, max_pages]
  int32_t* token_start;       // [C + 1]
  int64_t* slots;             // [max_tokens]
  int32_t* seq_len;           // [C]
  int32_t* status;            // [C]
  PlanRecord* records;        // workspace [C]
  int C, max_pages, n_pages, max_tokens;
};
hipError_t launch_cache_plan(const PlanParams& p, hipStream_t stream);

struct AppendParams {
  const __bf16* k_new;    // [n_tokens] rows of Hkv x D, k_stride elements apart
  const __bf16* v_new;
  const int64_t* slots;   // [n_tokens]
  uint8_t* k_pages;       // [n_pages, Hkv, 64, D]
  uint8_t* v_pages;
  uint8_t* k_scale;       // [n_pages, Hkv]
  uint8_t* v_scale;
  int64_t k_stride, v_stride;
  int n_tokens, Hkv, n_pages;
  int per_wave;           // filled by the launcher: tokens whose runs a wave looks for, a power of two up to 64
};
hipError_t launch_cache_append(const AppendParams& p, int D, bool e5m2, hipStream_t stream);

// Tokens' rows and their places in a cache: stored in 4 bits, or read back from any type.
struct RowsParams {
  const int64_t* slots;  // [n_tokens]
  __bf16* k_rows;        // [n_tokens] rows of Hkv x D, k_stride elements apart; not written by the append
  __bf16* v_rows;
  uint8_t* k_pages;      // [n_pages, Hkv, 64, D] or, with codes of 4 bits, [n_pages, Hkv, 64, D / 2]; not written by the read
  uint8_t* v_pages;
  uint8_t* k_scale;      // [n_pages, Hkv] or [n_pages, Hkv, 64, D / 32]
  uint8_t* v_scale;
  int64_t k_stride, v_stride;
  int n_tokens, Hkv, n_pages;
};
hipError_t launch_cache_append_blocks(const RowsParams& p, int D, hipStream_t stream);
hipError_t launch_cache_read(const RowsParams& p, int D, CacheType cache, hipStream_t stream);

}  // namespace peagle
