// Declarations shared by the operators around a small cache: the 4-bit cache and attention with a sliding window.
#pragma once

#include "common.h"

// Attention of short query blocks (Tq <= 16) over a 4-bit cache, or over a bf16 cache with a window (attn_cache.hip).
// `a` holds what the shared combine kernel reads: shapes, units, partials, outputs and the block's own tokens.
struct CacheAttnArgs {
  AttnArgs a;                        // k, v and the strides in elements: bf16 caches; indices NULL: all tokens
  const uint8_t *codes, *scales;     // 4-bit cache; strides in bytes
  int64_t code_b, code_h, code_n, code_page;
  int64_t scale_b, scale_h, scale_n, scale_page;
  int32_t tq_inv;                    // r / Tq = r * tq_inv >> 16 for r < 64
  int32_t window, sinks;             // bf16 cache: see sts_window_attn
  int32_t behind;                    // bf16 cache: 1 = the block's own tokens are not in the cache (k_new)
};

struct PackedRowsArgs {
  uint16_t *k, *v;                   // [B,T,Hkv,d]
  const int32_t *pos, *lens;
  uint8_t *codes, *scales;
  int64_t code_b, code_h, code_n, code_page;
  int64_t scale_b, scale_h, scale_n, scale_page;
  const int32_t *block_table;
  int32_t table_stride, num_pages, page_shift, N;
  int32_t B, T, Hkv, d;
};

// n / d for 0 <= n < 2^31 as a product (Granlund and Montgomery, "Division by invariant integers using multiplication"): with 2^l
// >= d > 2^(l-1) and mul = floor(2^(31+l) / d) + 1, n * mul >> 31 + l is exact. A division takes a wave some forty instructions.
struct Divisor {
  uint32_t mul, shift;
  __host__ __device__ __forceinline__ int of(int n) const { return (int)(((uint64_t)(uint32_t)n * mul) >> shift); }
};
inline Divisor divide_by(int d) {
  uint32_t l = 0;
  while ((1ll << l) < d) ++l;
  return {(uint32_t)(((uint64_t)1 << (31 + l)) / (uint64_t)d + 1), 31 + l};
}

// Attention with a window over many query rows (attn_window.hip)
struct WindowArgs {
  const uint16_t *q, *k, *v;
  int64_t stride_b, stride_h, stride_n, stride_page;     // elements
  const int32_t *seq_lens, *block_table;
  int32_t B, Tq, Hq, Hkv, G, N, window, sinks;
  int32_t page_shift, table_stride, num_pages;
  float scale, scale_log2;
  int32_t num_splits;                // workgroups per block of rows, each with a part of its keys
  int32_t blocks;                    // blocks of STS_WINDOW_ROWS rows of a KV head
  Divisor by_splits, by_blocks, by_heads, by_group;
  float *part_o, *part_ml;           // [units][num_splits][STS_WINDOW_ROWS][d], [..][2]
  void *out;
  float *lse_out;
  int32_t out_dtype;
};
constexpr int STS_WINDOW_ROWS = 128, STS_WINDOW_KEYS = 64;      // query rows of a block, keys of a tile

hipError_t launch_packed_store(const PackedRowsArgs &a, hipStream_t s);
hipError_t launch_packed_load(const PackedRowsArgs &a, hipStream_t s);
// far: rows at offsets of more than 32 bits, or pages
hipError_t launch_cache_attn(const CacheAttnArgs &a, int d, int nq, bool four_bit, bool far, hipStream_t s);
hipError_t launch_window_prompt(const WindowArgs &a, int d, hipStream_t s);
hipError_t launch_window_combine(const WindowArgs &a, int d, hipStream_t s);
