// Declarations shared by the layers over packed batches: attention over whole prompts and linear attention with decays.
#pragma once

#include "cache.h"
#include "common.h"

// Sequences whose rows lie one after the other: those of b are starts[b] .. starts[b + 1] - 1, or `each` of them where starts is NULL.
struct PackedSeqs {
  const int32_t *starts;
  int32_t B, T, each;
};

// The rows of sequence b are cut into pieces of `per` (times a factor: rows of several heads). Piece i of sequence b has the number
// first(b) + i with first(b) = floor(begin(b) / per) + b: no two sequences' pieces get the same number, there are floor(T / per) + B numbers,
// and nothing has to be added up over the sequences before b. Numbers that no piece has are left out.
inline int64_t piece_numbers(int64_t rows, int64_t per, int64_t B) { return rows / per + B; }

struct PackedPiece {
  int b;            // -1: no piece has this number
  int begin, len;   // the sequence's first row and its length
  int index;        // which piece of it
};

// the rows of sequence b: the first, and how many; always within [0, T)
__device__ __forceinline__ void seq_rows(const PackedSeqs &s, int b, int &begin, int &len) {
  begin = s.starts ? min(max(s.starts[b], 0), s.T) : b * s.each;
  len = s.starts ? max(min(max(s.starts[b + 1], 0), s.T) - begin, 0) : s.each;
}

// Which piece has the number: 64 sequences are looked at at once, so that up to 64 (4096) sequences take one (two) loads. Starts that are out
// of order or out of range name wrong pieces, but none outside [0, T).
template <class First>
__device__ __forceinline__ PackedPiece find_piece(const PackedSeqs &s, int number, First first) {
  const int lane = threadIdx.x & 63;
  int lo = 0, n = s.B, begin = 0, end = 0;
  do {
    const int step = (n + 63) >> 6, at = lo + min(lane * step, n - 1);
    begin = s.starts ? min(max(s.starts[at], 0), s.T) : at * s.each;
    end = s.starts ? min(max(s.starts[at + 1], 0), s.T) : begin + s.each;
    const uint64_t before = __builtin_amdgcn_ballot_w64(lane * step < n && first(begin) + at <= number);
    if (before == 0) return {-1, 0, 0, 0};
    const int k = 63 - __builtin_clzll(before);
    begin = __builtin_amdgcn_readlane(begin, k);
    end = __builtin_amdgcn_readlane(end, k);
    lo += k * step;
    n = min(step, n - k * step);
  } while (n > 1);
  return {lo, begin, max(end - begin, 0), number - (first(begin) + lo)};
}

// attention over whole prompts (attn_prompt.hip)
struct PromptArgs {
  const uint16_t *q, *k, *v;
  int64_t q_stride_n, q_stride_h, kv_stride_n, kv_stride_h;     // elements
  PackedSeqs seqs;
  int32_t Hq, Hkv, G;
  int32_t numbers;                  // of blocks of a KV head (piece_numbers)
  float scale, scale_log2;
  Divisor by_numbers, by_group;
  void *out;                        // [T,Hq,d]
  float *lse_out;                   // [Hq,T]
  int32_t out_dtype;
};
constexpr int STS_PROMPT_ROWS = 128;      // query rows of a block: positions times the heads of a group

hipError_t launch_prompt_attn(const PromptArgs &a, int d, hipStream_t s);

// linear attention with decays (linear.hip)
struct LinearArgs {
  const uint16_t *q, *k, *v;                                    // q and out NULL: states only
  int64_t q_stride_n, q_stride_h, kv_stride_n, kv_stride_h;     // elements
  const float *decay;                                           // [Hkv], or [T,Hkv]
  int32_t decay_rows;
  PackedSeqs seqs;
  const int32_t *lens;
  int32_t max_len;                   // rows of a sequence behind it are left out
  int32_t Hq, Hkv, G;
  float scale;
  const float *state;                // NULL: zeros
  float *state_out;                  // NULL: not kept
  const int32_t *slots, *slots_out;  // NULL: slot b
  int64_t state_stride, state_out_stride;
  int32_t num_slots, num_slots_out;
  void *out;
  int32_t out_dtype;
  // Chunked form: rows of a segment (a multiple of STS_LINEAR_CHUNK), of which each workgroup has one; numbers of segments (piece_numbers); what each segment
  // adds to the state and the logarithm of its decay, later the states before the segments
  int32_t segment, numbers;
  int32_t heads;                     // of a group that a workgroup of the results has, 1 or 2
  Divisor by_segment, by_heads, by_group, by_turns;
  float *part;                       // [numbers][Hkv][d][d], or NULL: nothing is handed on
  double *part_log;                  // [numbers][Hkv]
};
constexpr int STS_LINEAR_CHUNK = 32, STS_LINEAR_STEP = 16;      // rows of a chunk; rows of a sequence that the recurrent form takes at most

hipError_t launch_linear_step(const LinearArgs &a, int d, hipStream_t s);
hipError_t launch_linear_sums(const LinearArgs &a, int d, hipStream_t s);
hipError_t launch_linear_carry(const LinearArgs &a, int d, hipStream_t s);
hipError_t launch_linear_chunks(const LinearArgs &a, int d, hipStream_t s);
