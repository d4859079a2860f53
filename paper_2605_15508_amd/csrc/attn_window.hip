// Attention with a sliding window and sinks over many query rows: a prompt, or a chunk of one (gfx950).
//
// A workgroup of four waves has 128 query rows of one KV head: row r of the head's Tq * G rows is query r / G of the
// group's head r % G, so that the heads of a group share every K and V tile and a block spans 128 / G positions: with a
// window of W it looks at W + 128 / G keys and the sinks, one list of keys. A wave has 32 rows; tiles are 64 keys, K and V
// in LDS, two of each, the next tile on its way there while one is worked on.
//
// Transposed as in the split kernels, on v_mfma_f32_32x32x16_bf16: S^T = K Q^T gives lane (h, c) = (lane / 32, lane % 32) the
// scores of query c with keys 8 j + 4 h + i (j = 0..3, i = 0..3) of each 32, two j of which are what it supplies as the B operand of
// O^T += V^T P^T for 16 keys: P stays in its lane, and V's operand takes the keys in that order. It comes from V's rows in
// LDS by the transposing read (four lanes have 16 channels of a key, lane i gets channel i of four keys).
// LDS chunks of 16 bytes are permuted within a row so that neither K's reads (16 rows, one chunk each) nor V's (4 rows, 64
// bytes each) meet in a bank.
//
// What bounds it: matrix and vector instructions of two waves on a SIMD (three at head size 64) that wait for each other at a barrier
// per tile. 8192 rows, all causal: 555 us, 990 TFLOP/s, where this card's 8192^3 product reaches 1270. Window 1024: 171 to 180 us, 720 to
// 757 (17 tiles a block, the first wait for which and the masked ends do not shrink with the window; vector instructions take 51% of the
// cycles, matrix instructions 39%, and a wave waits for 28% of its time). 1999 rows behind 33001 tokens, window 4096: 148 us, 907
// (49%, 44%, 30%). Head size 64 (two prompts of up to 4000 rows, window 512): 47 to 58 us, by their lengths: vector instructions,
// 61% of the cycles and 17 for every matrix instruction (25%), an eighth of them exponentials; ten tiles a block, and a wave waits
// for 34% of its time.
#include <float.h>

#include "attn_util.h"
#include "cache.h"

namespace {

constexpr int WAVES = 4, ROWS = STS_WINDOW_ROWS, TK = STS_WINDOW_KEYS;
static_assert(ROWS == 32 * WAVES && TK == 64, "");

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) s16x4 *lds_s16x4;

// where chunk c of row r lies in its row
template <int D> __device__ __forceinline__ int k_chunk(int r, int c) { return D == 128 ? c ^ (r & 15) : c ^ ((r >> 1) & 7); }
template <int D> __device__ __forceinline__ int v_chunk(int r, int c) { return D == 128 ? c ^ ((r & 3) << 2) : c ^ ((r & 2) << 1); }

// bits 0 .. n - 1, none for n <= 0
__device__ __forceinline__ uint64_t first_keys(int n) { return n <= 0 ? 0 : n >= 64 ? ~0ull : (1ull << n) - 1; }

// PAGES: 0 none; 1 with rows at up to 2^32 units of 16 bytes in the pool; 2 further away
template <int D, int PAGES>
// (head size 64: registers for three workgroups on a compute unit: 4000 rows, pages of one token 65 us, with two 71)
__global__ void __launch_bounds__(64 * WAVES, D == 64 && PAGES < 2 ? 3 : 2) window_prompt_kernel(const WindowArgs A) {
  constexpr int KS = D / 16;             // contraction steps of S
  constexpr int DT = D / 32;             // 32-channel tiles of O
  constexpr int CH = D / 8;              // 16-byte chunks of a row
  constexpr int NL = TK * CH / (64 * WAVES);       // chunks of K (and of V) per thread and tile
  constexpr int RL = 64 / CH;                      // rows that a wave's load covers
  // (four arrays, not two of two: so the compiler can tell the loads that fill one from the reads of another)
  __shared__ __attribute__((aligned(16))) u32x4 lds_k0[TK * CH], lds_k1[TK * CH], lds_v0[TK * CH], lds_v1[TK * CH];
  __shared__ __attribute__((aligned(16))) uint32_t lds_odd[2][WAVES];

  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const int h = lane >> 5, col = lane & 31;
  // what the first loads need of the arguments, asked for together: waits for scalar loads cannot tell them apart
  asm volatile("" ::"s"(A.q), "s"(A.k), "s"(A.v), "s"(A.stride_b), "s"(A.stride_h), "s"(A.stride_n), "s"(A.seq_lens), "s"(A.block_table), "s"(A.Tq), "s"(A.Hq), "s"(A.Hkv),
               "s"(A.G), "s"(A.N), "s"(A.window), "s"(A.sinks), "s"(A.scale), "s"(A.scale_log2), "s"(A.num_splits), "s"(A.blocks), "s"(A.by_splits.mul),
               "s"(A.by_splits.shift), "s"(A.by_blocks.mul), "s"(A.by_blocks.shift), "s"(A.by_heads.mul), "s"(A.by_heads.shift), "s"(A.by_group.mul),
               "s"(A.by_group.shift));
  // Blocks of one KV head next to each other on one die (workgroup i runs on die i % 8), the later positions, which may have
  // more keys, first.
  const int total = gridDim.x, x = blockIdx.x % STS_XCDS;
  const int j = x * (total / STS_XCDS) + min(x, total % STS_XCDS) + blockIdx.x / STS_XCDS;
  const int unit = A.by_splits.of(j), split = j - unit * A.num_splits;
  const int head_unit = A.by_blocks.of(unit), blk = A.blocks - 1 - (unit - head_unit * A.blocks);
  const int bt = A.by_heads.of(head_unit), g = head_unit - bt * A.Hkv;

  const int L = A.seq_lens ? min(max(A.seq_lens[bt], 0), A.N) : A.N;
  const int p_first = L - A.Tq;                                   // position of query 0
  const int rows = A.Tq * A.G, row_0 = blk * ROWS, row_w = row_0 + wave * 32;
  const bool ok = row_w + col < rows;
  const int r = min(row_w + col, rows - 1);
  const int qi = A.by_group.of(r), head = g * A.G + r - qi * A.G;
  const int p = p_first + qi;                                     // this lane's query
  const int b_lo = p_first + A.by_group.of(row_0), b_hi = p_first + A.by_group.of(min(row_0 + ROWS - 1, rows - 1));          // the workgroup's
  const int w_lo = p_first + A.by_group.of(min(row_w, rows - 1)), w_hi = p_first + A.by_group.of(min(row_w + 31, rows - 1)); // the wave's

  // The keys that some query of the block sees, one after the other: those of `firsts` sinks before lo, then lo .. end - 1. Place v
  // holds key v, or v + skipped from `firsts` on.
  const int end = max(min(b_hi + 1, L), 0);
  const int lo = (int)min(max((int64_t)b_lo - A.window + 1, (int64_t)0), (int64_t)end);
  const int firsts = min(A.sinks, lo), skipped = lo - firsts;
  const int places = end - skipped, all_tiles = (places + TK - 1) / TK;
  // (few blocks: several workgroups to each, with a part of its tiles)
  const int per_split = (all_tiles + A.num_splits - 1) / A.num_splits, begin = split * per_split, tiles = min(begin + per_split, all_tiles);
  // the key at a tile's first place, if that is none of the sinks
  auto first_of = [&](int t) { return t * TK + skipped; };

  // ---- Q, as the B operand: channels 16 s + 8 h .. of query col. The scale's sign goes to Q.
  const uint32_t q_keep = A.scale == 0.f ? 0u : 0xffffffffu, q_flip = A.scale < 0.f ? 0x80008000u : 0u;
  const float sl2 = A.scale == 0.f ? 1.f : fabsf(A.scale_log2);
  bf16x8 Q[KS];
  {
    const uint16_t *qp = A.q + (((size_t)bt * A.Tq + qi) * A.Hq + head) * D + 8 * h;
#pragma unroll
    for (int s = 0; s < KS; ++s) Q[s] = __builtin_bit_cast(bf16x8, (*reinterpret_cast<const u32x4 *>(qp + 16 * s) & q_keep) ^ q_flip);
  }

  // ---- loads, straight to LDS: load m of a wave fills the 1 KB of rows (wave NL + m) RL .., lane by lane, so the permutation of a
  // row's chunks is in what a lane asks for. Rows that no query of the block sees are read from ones that some query does: their weight
  // is 0, but 0 times what lies there may be NaN.
  const int row0 = wave * NL * RL + lane / CH, slot0 = lane % CH;
  const int64_t row_bytes = A.stride_n * 2, page_bytes = A.stride_page * 2, head_off = ((PAGES ? 0 : bt * A.stride_b) + g * A.stride_h) * 2;
  const unsigned char *kbase = reinterpret_cast<const unsigned char *>(A.k) + head_off, *vbase = reinterpret_cast<const unsigned char *>(A.v) + head_off;
  const int32_t *table = PAGES ? A.block_table + (size_t)bt * A.table_stride : nullptr;
  auto row_of = [&](int v) {           // (past the last place: the last key)
    v = min(v, places - 1);
    return v < firsts ? v : v + skipped;
  };
  typedef __attribute__((address_space(3))) unsigned char *lds_ptr;
  // where a lane's chunks of a tile lie, counted from its first row
  uint32_t k_off[NL], v_off[NL];
#pragma unroll
  for (int m = 0; m < NL; ++m) {
    const int row = row0 + RL * m;
    k_off[m] = (uint32_t)row * (uint32_t)row_bytes + 16 * k_chunk<D>(row, slot0);
    v_off[m] = (uint32_t)row * (uint32_t)row_bytes + 16 * v_chunk<D>(row, slot0);
  }
  // Pages: lane i looks up the page of row i % 16 of its wave's sixteen and tells the lanes that ask for the rows where they lie, a tile
  // before they do (looked up when asked for, with offsets in 64 bits: 33001 tokens in pages of 16, 181 us; so 167; without pages 151).
  struct Where {
    uint32_t row[PAGES == 1 ? NL : 1];
  };
  const uint32_t page_mask = (1u << A.page_shift) - 1;
  auto my_row = [&](int t) { return row_of(min(t, tiles - 1) * TK + wave * (NL * RL) + lane % (NL * RL)); };
  auto page_of = [&](int t) { return PAGES ? min(max(table[my_row(t) >> A.page_shift], 0), A.num_pages - 1) : 0; };
  auto where = [&](int t, int page) {
    Where at;
    if constexpr (PAGES == 1) {
      const uint32_t mine = (uint32_t)page * (uint32_t)(A.stride_page / 8) + ((uint32_t)my_row(t) & page_mask) * (uint32_t)(A.stride_n / 8);
#pragma unroll
      for (int m = 0; m < NL; ++m) at.row[m] = (uint32_t)__shfl((int)mine, lane / CH + RL * m, 64);
    } else {
      at.row[0] = (uint32_t)page;
    }
    return at;
  };
  static_assert(NL * RL == 16, "");
  // K's or V's tile t (past the last: the last again, which nobody reads)
  auto load = [&](int t, const unsigned char *from, u32x4 *to, bool is_v, const Where &at) {
    const int v0 = min(t, tiles - 1) * TK, n0 = v0 + skipped;
    u32x4 *const mine = to + wave * NL * 64;
    auto chunk = [&](int m) { return is_v ? v_chunk<D>(row0 + RL * m, slot0) : k_chunk<D>(row0 + RL * m, slot0); };
    if (!PAGES && v0 >= firsts && v0 + TK <= places) {
      const __amdgpu_buffer_rsrc_t rows = __builtin_amdgcn_make_buffer_rsrc(const_cast<unsigned char *>(from + n0 * row_bytes), 0, 0xffffffff, 0x00027000);
#pragma unroll
      for (int m = 0; m < NL; ++m) __builtin_amdgcn_raw_ptr_buffer_load_lds(rows, (lds_ptr)(mine + 64 * m), 16, (int)(is_v ? v_off[m] : k_off[m]), 0, 0, 0);
    } else {
      // (sinks, the cache's end, pages: any row at any distance)
      typedef const __attribute__((address_space(1))) unsigned char *global_ptr;
#pragma unroll
      for (int m = 0; m < NL; ++m) {
        uint64_t off;            // (none of the factors is negative)
        if constexpr (PAGES == 1) {
          off = (uint64_t)(at.row[m] + chunk(m)) << 4;
        } else if constexpr (PAGES == 2) {
          const uint32_t page = (uint32_t)__shfl((int)at.row[0], lane / CH + RL * m, 64);
          off = (uint64_t)page * (uint64_t)page_bytes + ((uint32_t)row_of(v0 + row0 + RL * m) & page_mask) * (uint32_t)row_bytes + 16 * chunk(m);
        } else {
          off = (uint64_t)(uint32_t)row_of(v0 + row0 + RL * m) * (uint64_t)row_bytes + 16 * chunk(m);
        }
        __builtin_amdgcn_global_load_lds((global_ptr)(from + off), (lds_ptr)(mine + 64 * m), 16, 0, 0);
      }
    }
  };
  // does every query of the wave see all keys of tile t?
  auto masked = [&](int t) {
    const int n0 = first_of(t);
    return !(n0 + TK - 1 <= w_lo && (n0 + TK <= A.sinks || w_hi - max(n0, lo) < A.window));
  };

  float m_run = -INFINITY, l_run = 0.f;
  f32x16 acc[DT];
#pragma unroll
  for (int dt = 0; dt < DT; ++dt)
#pragma unroll
    for (int i = 0; i < 16; ++i) acc[dt][i] = 0.f;

  // Where the lane reads: K's chunk 2 s + h of row 32 kt + col, and V's operand for channels 32 dt .. and keys 16 s .., two transposed
  // reads of keys 16 s + 4 h + 0..3 and 8 further on. Both are one address with a few bits flipped by s or dt, plus a constant.
  typedef const __attribute__((address_space(3))) u32x4 *lds_u32x4;
  const int k_lane = col * CH * 16 + 16 * k_chunk<D>(col, h);
  const int t_row = 4 * h + ((lane & 15) >> 2), t_col = (lane & 16) + 4 * (lane & 3);       // within 16 keys, 32 channels
  const int v_lane = (t_row * CH + v_chunk<D>(t_row, t_col >> 3)) * 16 + (t_col & 7) * 2;
  auto v_operand = [&](const u32x4 *v, int at, int dt, int s) {
    u32x4 w;
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const u32x2 v2 = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4)((lds_ptr)v + (at ^ (64 * dt)) + (16 * s + 8 * e) * CH * 16)));
      w[2 * e] = v2[0];
      w[2 * e + 1] = v2[1];
    }
    return w;
  };

  // which keys of tile t the lane's query sees, a bit each: the sinks, then those up to it, without those between the sinks and its
  // window
  auto seen_keys = [&](int t) {
    const int n0 = first_of(t);
    return first_keys(firsts - t * TK) |
           (first_keys(p + 1 - n0) & (first_keys(A.sinks - n0) | ~first_keys((int)max((int64_t)p - A.window + 1, (int64_t)0) - n0)));
  };
  // S of one tile
  auto product = [&](const u32x4 *k, f32x16 (&S)[2]) {
    int k_at = k_lane;
    asm("" : "+v"(k_at));                        // (what comes of it is made anew in every tile, not kept in registers)
    const f32x16 zero = {};
#pragma unroll
    for (int s = 0; s < KS; ++s)
#pragma unroll
      for (int kt = 0; kt < 2; ++kt) {
        const bf16x8 Ka = __builtin_bit_cast(bf16x8, *(lds_u32x4)((lds_ptr)k + (k_at ^ (32 * s)) + 32 * kt * CH * 16));
        S[kt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(Ka, Q[s], s ? S[kt] : zero, 0, 0, 0);
      }
  };
  // keys that the query does not see score -inf
  auto hide = [&](int t, f32x16 (&S)[2]) {
    const uint64_t seen = seen_keys(t) >> (4 * h);
#pragma unroll
    for (int kt = 0; kt < 2; ++kt) {
      const int word = (int)(uint32_t)(seen >> (32 * kt));
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const uint32_t keep = (uint32_t)__builtin_amdgcn_sbfe(word, (i & 3) + 8 * (i >> 2), 1);
        const float x = S[kt][i];
        S[kt][i] = __builtin_bit_cast(float, (__builtin_bit_cast(uint32_t, x) & keep) | (0xff800000u & ~keep));
      }
    }
  };
  auto highest = [&](const f32x16 (&S)[2]) {
    float m[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) m[j] = top(S[0][j], S[1][j]);
#pragma unroll
    for (int i = 4; i < 16; ++i) m[i & 3] = top(m[i & 3], top(S[0][i], S[1][i]));
    return sl2 * top(top(m[0], m[1]), top(m[2], m[3]));
  };
  // the running maximum takes in a tile's; both halves of the wave hold half of a query's scores
  auto raise = [&](float mine) {
    if (__builtin_amdgcn_ballot_w64(mine > m_run) != 0) {
      const uint32_t w = __builtin_bit_cast(uint32_t, mine);
      const auto q = __builtin_amdgcn_permlane32_swap(w, w, false, false);
      const uint32_t q0 = q[0], q1 = q[1];
      const float m_new = fmaxf(m_run, top(__builtin_bit_cast(float, q0), __builtin_bit_cast(float, q1)));
      const float alpha = m_new == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m_run - m_new);
      l_run *= alpha;
      m_run = m_new;
#pragma unroll
      for (int dt = 0; dt < DT; ++dt)
#pragma unroll
        for (int i = 0; i < 16; ++i) acc[dt][i] *= alpha;
    }
  };
  // exp(S - m), as the B operands of the second product (bf16, half a step, 2^-8 of each), and their sum in fp32
  auto weights = [&](const f32x16 (&S)[2], u32x4 (&P)[4]) {
    const float m_ref = m_run == -INFINITY ? 0.f : m_run;
    float sum[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int s = 0; s < 4; ++s)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float p0 = __builtin_amdgcn_exp2f(__builtin_fmaf(S[s >> 1][8 * (s & 1) + 2 * e], sl2, -m_ref));
        const float p1 = __builtin_amdgcn_exp2f(__builtin_fmaf(S[s >> 1][8 * (s & 1) + 2 * e + 1], sl2, -m_ref));
        sum[e] += p0 + p1;
        P[s][e] = __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{p0, p1}), bf16x2));
      }
    return (sum[0] + sum[1]) + (sum[2] + sum[3]);
  };
  // A tile that not every query of the block sees whole: has it a value that is no number, or infinite? Each wave looks through the rows
  // that it asked for, in slot `at`; the answer is there after the next barrier.
  auto partly_seen = [&](int t) {
    const int n0 = first_of(t);
    return !(n0 + TK - 1 <= b_lo && (n0 + TK <= A.sinks || b_hi - max(n0, lo) < A.window));
  };
  auto look_through = [&](const u32x4 *v, int at) {
    float z[4] = {0.f, 0.f, 0.f, 0.f};            // sums of 0 times the values: 0, or no number
    const bf16x2 none = {(__bf16)0.f, (__bf16)0.f};
#pragma unroll
    for (int m = 0; m < NL; ++m) {
      const u32x4 w = *(lds_u32x4)((lds_ptr)v + 16 * (lane + 64 * (wave * NL + m)));
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const uint32_t x = w[e];
        z[e] = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, x), none, z[e], false);
      }
    }
    const float all = (z[0] + z[1]) + (z[2] + z[3]);
    const bool mine = __builtin_amdgcn_ballot_w64(all != 0.f) != 0;       // (true for what is no number)
    if (lane == 0) lds_odd[at][wave] = mine;
  };
  auto odd_values = [&](int at) {
    asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
    uint32_t any = 0;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) any |= lds_odd[at][w];
    return __builtin_amdgcn_readfirstlane((int)any) != 0;
  };

  // ---- The next tile's scores are worked out while this one's weights are: matrix and vector instructions of one wave, which do
  // not wait for each other. K is a tile ahead of V.
  // What was asked for has come, and what was read is in registers: the tiles change hands.
  auto arrived = [] { asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory"); };
  bool later = false;              // tiles left for the end: see below
  if (begin < tiles) {
    f32x16 S[2];
    const int page0 = page_of(begin), page1 = page_of(begin + 1), page2 = page_of(begin + 2);
    Where at_v = where(begin, page0);
    load(begin, kbase, lds_k0, false, at_v);
    load(begin, vbase, lds_v0, true, at_v);
    at_v = where(begin + 1, page1);
    load(begin + 1, kbase, lds_k1, false, at_v);
    Where at_k = where(begin + 2, page2);
    arrived();
    product(lds_k0, S);
    if (masked(begin)) hide(begin, S);
    raise(highest(S));
    auto step = [&](int t, const u32x4 *k_next, u32x4 *k_free, const u32x4 *v, u32x4 *v_free) {
      arrived();
      load(t + 2, kbase, k_free, false, at_k);
      load(t + 1, vbase, v_free, true, at_v);
      at_v = at_k;
      at_k = where(t + 3, page_of(t + 3));
      bool odd = false;
      if (partly_seen(t)) {
        look_through(v, t & 1);
        odd = odd_values(t & 1);
      }
      f32x16 N[2];
      u32x4 P[4];
      product(k_next, N);
      const float sum = weights(S, P);
      if (!odd) {
        l_run += sum;
        int v_at = v_lane;
        asm("" : "+v"(v_at));
#pragma unroll
        for (int s = 0; s < 4; ++s)
#pragma unroll
          for (int dt = 0; dt < DT; ++dt)
            acc[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, v_operand(v, v_at, dt, s)), __builtin_bit_cast(bf16x8, P[s]), acc[dt], 0, 0, 0);
      }
      later |= odd;
      if (t + 1 < tiles) {
        if (masked(t + 1)) hide(t + 1, N);
        raise(highest(N));
      }
#pragma unroll
      for (int kt = 0; kt < 2; ++kt) S[kt] = N[kt];
    };
    for (int t = begin;; t += 2) {
      step(t, lds_k1, lds_k0, lds_v0, lds_v1);
      if (t + 1 >= tiles) break;
      step(t + 1, lds_k0, lds_k1, lds_v1, lds_v0);
      if (t + 2 >= tiles) break;
    }
    __builtin_amdgcn_s_waitcnt(0x0f70);              // all that was asked for has come
    // What is infinite or no number must not reach queries that do not see it, and 0 times it is not 0: such tiles come last, key
    // by key, and a key's row is taken in only where it is seen.
    if (__syncthreads_or(later)) {
      for (int t = begin; t < tiles; ++t) {
        arrived();
        const Where at = where(t, page_of(t));
        load(t, kbase, lds_k0, false, at);
        load(t, vbase, lds_v0, true, at);
        arrived();
        if (!partly_seen(t)) continue;
        look_through(lds_v0, 0);
        if (!odd_values(0)) continue;
        u32x4 P[4];
        product(lds_k0, S);
        hide(t, S);
        l_run += weights(S, P);
        const uint64_t seen = seen_keys(t);
#pragma unroll
        for (int s = 0; s < 4; ++s)
          for (int key = 0; key < 16; ++key) {
            u32x4 own;       // element e of the lane's eight: key 4 h + e % 4 + 8 (e / 4)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const int k0 = 4 * h + 2 * (e & 1) + 8 * (e >> 1);
              own[e] = (key == k0 ? 0xffffu : 0u) | (key == k0 + 1 ? 0xffff0000u : 0u);
            }
            const bool see = (seen >> (16 * s + key)) & 1u;
#pragma unroll
            for (int dt = 0; dt < DT; ++dt) {
              const f32x16 zero = {};
              const f32x16 z = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, v_operand(lds_v0, v_lane, dt, s) & own),
                                                                       __builtin_bit_cast(bf16x8, P[s] & own), zero, 0, 0, 0);
#pragma unroll
              for (int i = 0; i < 16; ++i) acc[dt][i] += see ? z[i] : 0.f;
              __builtin_amdgcn_sched_barrier(0);         // (one product's registers at a time)
            }
          }
      }
    }
  }

  // ---- out
  {
    const uint32_t w = __builtin_bit_cast(uint32_t, l_run);
    const auto q = __builtin_amdgcn_permlane32_swap(w, w, false, false);
    const uint32_t q0 = q[0], q1 = q[1];
    l_run = __builtin_bit_cast(float, q0) + __builtin_bit_cast(float, q1);
  }
  if (A.num_splits > 1) {            // a partial: the sums as they are, and what they are relative to
    const size_t part = (size_t)unit * A.num_splits + split, row = part * ROWS + wave * 32 + col;
    float *o = A.part_o + row * D + 4 * h;
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
      for (int e = 0; e < 4; ++e)
        *reinterpret_cast<f32x4 *>(o + 32 * dt + 8 * e) = f32x4{acc[dt][4 * e], acc[dt][4 * e + 1], acc[dt][4 * e + 2], acc[dt][4 * e + 3]};
    // (scores that are no numbers raise no maximum: without one the part would be taken for an empty one)
    if (h == 0) *reinterpret_cast<f32x2 *>(A.part_ml + row * 2) = f32x2{l_run != l_run ? top(m_run, -FLT_MAX) : m_run, l_run};
    return;
  }
  if (!ok) return;
  const float inv = l_run == 0.f ? 0.f : 1.f / l_run;
  const size_t at = (((size_t)bt * A.Tq + qi) * A.Hq + head) * D + 4 * h;
#pragma unroll
  for (int dt = 0; dt < DT; ++dt)
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const f32x4 o = {acc[dt][4 * e] * inv, acc[dt][4 * e + 1] * inv, acc[dt][4 * e + 2] * inv, acc[dt][4 * e + 3] * inv};
      if (A.out_dtype == STS_F32) {
        *reinterpret_cast<f32x4 *>(static_cast<float *>(A.out) + at + 32 * dt + 8 * e) = o;
      } else {
        const u32x2 w = {__builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{o[0], o[1]}), bf16x2)),
                         __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{o[2], o[3]}), bf16x2))};
        *reinterpret_cast<u32x2 *>(static_cast<uint16_t *>(A.out) + at + 32 * dt + 8 * e) = w;
      }
    }
  if (A.lse_out && h == 0)
    A.lse_out[((size_t)bt * A.Hq + head) * A.Tq + qi] = l_run > 0.f ? (m_run + __builtin_amdgcn_logf(l_run)) * 0.69314718055994530942f : -INFINITY;
}

// The parts of a block's rows put together, in order: D / 4 threads a row, four channels each.
template <int D>
__global__ void __launch_bounds__(256) window_combine_kernel(const WindowArgs A) {
  constexpr int LANES = D / 4, AT_ONCE = 4;
  const int nb = (int)(((int64_t)A.Tq * A.G + ROWS - 1) / ROWS);
  const int64_t row_id = (int64_t)blockIdx.x * (256 / LANES) + threadIdx.x / LANES;        // unit * ROWS + row of the block
  const int64_t unit = row_id / ROWS;
  const int row = (int)(row_id - unit * ROWS), chan = 4 * (threadIdx.x % LANES);
  const int blk = nb - 1 - (int)(unit % nb), g = (int)(unit / nb % A.Hkv), bt = (int)(unit / nb / A.Hkv);
  const int64_t r = (int64_t)blk * ROWS + row;
  if (bt >= A.B || r >= (int64_t)A.Tq * A.G) return;
  const int S = A.num_splits;
  float m = -INFINITY, l = 0.f;
  f32x4 o = {0.f, 0.f, 0.f, 0.f};
  for (int s0 = 0; s0 < S; s0 += AT_ONCE) {
    f32x2 ml[AT_ONCE];
    f32x4 x[AT_ONCE];
#pragma unroll
    for (int j = 0; j < AT_ONCE; ++j) {
      const size_t at = ((size_t)unit * S + min(s0 + j, S - 1)) * ROWS + row;
      ml[j] = *reinterpret_cast<const f32x2 *>(A.part_ml + at * 2);
      x[j] = *reinterpret_cast<const f32x4 *>(A.part_o + at * D + chan);
    }
#pragma unroll
    for (int j = 0; j < AT_ONCE; ++j) {
      if (s0 + j >= S || ml[j][0] == -INFINITY) continue;
      const float m_new = fmaxf(m, ml[j][0]);
      const float fo = __builtin_amdgcn_exp2f(m - m_new), fn = __builtin_amdgcn_exp2f(ml[j][0] - m_new);
      l = l * fo + ml[j][1] * fn;
      o = o * fo + x[j] * fn;
      m = m_new;
    }
  }
  const int qi = (int)(r / A.G), head = g * A.G + (int)(r - (int64_t)qi * A.G);
  o *= l == 0.f ? 0.f : 1.f / l;
  const size_t at = (((size_t)bt * A.Tq + qi) * A.Hq + head) * D + chan;
  if (A.out_dtype == STS_F32) {
    *reinterpret_cast<f32x4 *>(static_cast<float *>(A.out) + at) = o;
  } else {
    const u32x2 w = {__builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{o[0], o[1]}), bf16x2)),
                     __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{o[2], o[3]}), bf16x2))};
    *reinterpret_cast<u32x2 *>(static_cast<uint16_t *>(A.out) + at) = w;
  }
  if (A.lse_out && chan == 0)
    A.lse_out[((size_t)bt * A.Hq + head) * A.Tq + qi] = l > 0.f ? (m + __builtin_amdgcn_logf(l)) * 0.69314718055994530942f : -INFINITY;
}

}  // namespace

hipError_t launch_window_prompt(const WindowArgs &a, int d, hipStream_t s) {
  const dim3 grid((unsigned)(((int64_t)a.Tq * a.G + ROWS - 1) / ROWS * a.Hkv * a.B * a.num_splits)), block(64 * WAVES);
  // a pool whose rows lie within 64 GB: their offsets fit 32 bits in units of 16 bytes
  const int pages = !a.block_table ? 0 : (a.num_pages + 1.0) * (double)a.stride_page + 32.0 * (double)a.stride_n < 8.0 * 4294967296.0 ? 1 : 2;
  if (d == 128) {
    if (pages == 2) STS_LAUNCH((window_prompt_kernel<128, 2>), grid, block, 0, s, a);
    else if (pages) STS_LAUNCH((window_prompt_kernel<128, 1>), grid, block, 0, s, a);
    else STS_LAUNCH((window_prompt_kernel<128, 0>), grid, block, 0, s, a);
  } else {
    if (pages == 2) STS_LAUNCH((window_prompt_kernel<64, 2>), grid, block, 0, s, a);
    else if (pages) STS_LAUNCH((window_prompt_kernel<64, 1>), grid, block, 0, s, a);
    else STS_LAUNCH((window_prompt_kernel<64, 0>), grid, block, 0, s, a);
  }
  return sts_take_launch_status();
}

hipError_t launch_window_combine(const WindowArgs &a, int d, hipStream_t s) {
  const int64_t rows = ((int64_t)a.Tq * a.G + ROWS - 1) / ROWS * ROWS * a.Hkv * a.B;
  const dim3 grid((unsigned)(rows / (256 / (d / 4)))), block(256);
  if (d == 128) STS_LAUNCH(window_combine_kernel<128>, grid, block, 0, s, a);
  else STS_LAUNCH(window_combine_kernel<64>, grid, block, 0, s, a);
  return sts_take_launch_status();
}
