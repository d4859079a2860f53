// Causal attention over whole prompts whose rows are packed one after the other (gfx950).
//
// A workgroup of four waves has 128 query rows of one sequence and KV head: row r of the sequence's L * G rows is position r / G of
// the group's head r % G, so that the heads of a group share every K and V tile and a block spans 128 / G positions. It looks at the keys 0
// .. of the sequence up to its last position, 64 at a time; K and V go to LDS, two tiles of each, the next on its way there while one is
// worked on.
//
// Transposed, on v_mfma_f32_32x32x16_bf16: S^T = K Q^T gives lane (h, c) = (lane / 32, lane % 32) the scores of query c with keys 8 j + 4 h + i
// (j = 0..3, i = 0..3) of each 32, two j of which are what it supplies as the B operand of O^T += V^T P^T for 16 keys: P stays in its lane,
// and V's operand takes the keys in that order, out of V's rows in LDS by the transposing read.
//
// What bounds it: the two products, and beside them at head size 128 the power that the card has: 8192 rows, 32 heads in groups of 4, take 490 us,
// 1.1 PFLOP/s of what rows see (a plain product of the library reaches 1.2 to 1.4), with matrix instructions 67% of the cycles and vector
// instructions 60% at a clock of 1.7 GHz that the load leaves (alone on its compute unit a block takes 0.87 us for a tile, of which the products are 0.43). At
// head size 64 every exponential stands beside half the products: sixteen prompts of 100 to 4000 rows, 205 us, 0.8 PFLOP/s, vector instructions 82%.
// Two workgroups on a compute unit (three at head size 64), since one wave's softmax is another's product. 128 rows of a block, not more, as the tiles that its
// rows see in part cost as much as whole ones; 64 keys of a tile are what two tiles of K and V each leave of LDS.
#include <float.h>

#include "attn_util.h"
#include "layers.h"

namespace {

constexpr int WAVES = 4, ROWS = STS_PROMPT_ROWS, TK = 64;
static_assert(ROWS == 32 * WAVES, "");

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) s16x4 *lds_s16x4;
typedef __attribute__((address_space(3))) unsigned char *lds_ptr;
typedef const __attribute__((address_space(3))) u32x4 *lds_u32x4;

// Where 16-byte chunk c of row r lies in its row: K's reads (16 rows, one chunk each) and V's (4 rows, 64 bytes each) meet in no bank.
template <int D> __device__ __forceinline__ int k_chunk(int r, int c) { return D == 128 ? c ^ (r & 15) : c ^ ((r >> 1) & 7); }
template <int D> __device__ __forceinline__ int v_chunk(int r, int c) { return D == 128 ? c ^ ((r & 3) << 2) : c ^ ((r & 2) << 1); }

// bits 0 .. n - 1, none for n <= 0
__device__ __forceinline__ uint64_t first_keys(int n) { return n <= 0 ? 0 : n >= 64 ? ~0ull : (1ull << n) - 1; }

// sum over the wave (DPP: within rows of 16, then along the rows)
__device__ __forceinline__ int wave_sum(int x) {
  auto add = [&](auto ctrl, auto rows) { x += __builtin_amdgcn_update_dpp(0, x, decltype(ctrl)::value, decltype(rows)::value, 0xf, true); };
  add(std::integral_constant<int, 0x111>(), std::integral_constant<int, 0xf>());      // row_shr:1
  add(std::integral_constant<int, 0x112>(), std::integral_constant<int, 0xf>());
  add(std::integral_constant<int, 0x114>(), std::integral_constant<int, 0xf>());
  add(std::integral_constant<int, 0x118>(), std::integral_constant<int, 0xf>());
  add(std::integral_constant<int, 0x142>(), std::integral_constant<int, 0xa>());      // row_bcast:15
  add(std::integral_constant<int, 0x143>(), std::integral_constant<int, 0xc>());      // row_bcast:31
  return __builtin_amdgcn_readlane(x, 63);
}

// The block of rank `rank` where those furthest along their sequences, which see the most keys, come first: of up to 64 sequences, one to a lane. (Batches of
// more go by the blocks' numbers, the last sequence first: with that many the order is worth nothing. 64 sequences of 33 to 300 rows, 32 heads of 128 in groups of
// four, 53 us so and 50 by numbers, of 33 to 1000 rows 152 and 148.) A
// block's place in its sequence is the least i with no more than `rank` blocks behind it.
__device__ __forceinline__ PackedPiece block_of_rank(const PackedSeqs &s, int G, int rank) {
  const int lane = threadIdx.x & 63, b = min(lane, s.B - 1);
  const int begin = min(max(s.starts[b], 0), s.T), len = max(min(max(s.starts[b + 1], 0), s.T) - begin, 0);
  const int blocks = lane < s.B ? (int)(((int64_t)len * G + ROWS - 1) / ROWS) : 0;
  int lo = 0, hi = 0, behind = 0;
  if (s.B == 1) {
    lo = __builtin_amdgcn_readlane(blocks, 0) - 1 - rank;
    behind = rank;
  } else {
    if (rank >= wave_sum(blocks)) return {-1, 0, 0, 0};
    while (__builtin_amdgcn_ballot_w64(blocks > hi) != 0) hi = 2 * hi + 1;      // (the longest sequence's blocks, up to a power of two: 2^24 at most)
    while (lo < hi) {
      const int mid = (lo + hi) >> 1, n = wave_sum(max(blocks - mid - 1, 0));
      if (n <= rank) hi = mid;
      else lo = mid + 1;
    }
    behind = wave_sum(max(blocks - lo - 1, 0));
  }
  const uint64_t there = __builtin_amdgcn_ballot_w64(blocks > lo);
  const int nth = __builtin_amdgcn_mbcnt_hi((uint32_t)(there >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)there, 0));
  const uint64_t mine = __builtin_amdgcn_ballot_w64(blocks > lo && nth == rank - behind);
  if (lo < 0 || mine == 0) return {-1, 0, 0, 0};
  const int k = __builtin_ctzll(mine);
  return {k, __builtin_amdgcn_readlane(begin, k), __builtin_amdgcn_readlane(len, k), lo};
}

template <int D>
__global__ void __launch_bounds__(64 * WAVES, D == 64 ? 3 : 2) prompt_attn_kernel(const PromptArgs A) {
  constexpr int KS = D / 16;             // contraction steps of S
  constexpr int DT = D / 32;             // 32-channel tiles of O
  constexpr int CH = D / 8;              // 16-byte chunks of a row
  constexpr int NL = TK * CH / (64 * WAVES);       // chunks of K (and of V) per thread and tile
  constexpr int RL = 64 / CH;                      // rows that a wave's load covers
  __shared__ __attribute__((aligned(16))) u32x4 lds_k0[TK * CH], lds_k1[TK * CH], lds_v0[TK * CH], lds_v1[TK * CH];
  __shared__ __attribute__((aligned(16))) uint32_t lds_odd[2][WAVES];

  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const int h = lane >> 5, col = lane & 31;
  // Blocks of one KV head next to each other on one die (workgroup i runs on die i % 8), those with more keys first.
  const int total = gridDim.x, x = blockIdx.x % STS_XCDS;
  const int j = x * (total / STS_XCDS) + min(x, total % STS_XCDS) + blockIdx.x / STS_XCDS;
  const int g = A.by_numbers.of(j), rank = j - g * A.numbers;
  const PackedPiece piece = A.seqs.B <= 64 ? block_of_rank(A.seqs, A.G, rank)
                                           : find_piece(A.seqs, A.numbers - 1 - rank, [&](int begin) { return (int)((int64_t)begin * A.G / ROWS); });
  const int L = piece.len, rows = L * A.G, row_0 = piece.index * ROWS;
  if (piece.b < 0 || row_0 >= rows) return;

  const int row_w = row_0 + wave * 32;
  const bool ok = row_w + col < rows;
  const int r = min(row_w + col, rows - 1);
  const int p = A.by_group.of(r), head = g * A.G + r - p * A.G;          // this lane's query
  const int b_lo = A.by_group.of(row_0), b_hi = A.by_group.of(min(row_0 + ROWS - 1, rows - 1));      // the workgroup's positions
  const int w_lo = A.by_group.of(min(row_w, rows - 1));                                              // the wave's first
  const int places = b_hi + 1, tiles = (places + TK - 1) / TK;           // keys that some query of the block sees

  // ---- Q, as the B operand: channels 16 s + 8 h .. of query col. The scale's sign goes to Q.
  const uint32_t q_keep = A.scale == 0.f ? 0u : 0xffffffffu, q_flip = A.scale < 0.f ? 0x80008000u : 0u;
  const float sl2 = A.scale == 0.f ? 1.f : fabsf(A.scale_log2);
  bf16x8 Q[KS];
  {
    const uint16_t *qp = A.q + (piece.begin + (int64_t)p) * A.q_stride_n + head * A.q_stride_h + 8 * h;
#pragma unroll
    for (int s = 0; s < KS; ++s) Q[s] = __builtin_bit_cast(bf16x8, (*reinterpret_cast<const u32x4 *>(qp + 16 * s) & q_keep) ^ q_flip);
  }

  // ---- loads, straight to LDS: load m of a wave fills the 1 KB of rows (wave NL + m) RL .., lane by lane, so the permutation of a
  // row's chunks is in what a lane asks for. Rows that no query of the block sees lie behind the end that the loads are told and come as zeros.
  const int row0 = wave * NL * RL + lane / CH, slot0 = lane % CH;
  const int64_t row_bytes = A.kv_stride_n * 2, from = (piece.begin * A.kv_stride_n + g * A.kv_stride_h) * 2;
  const unsigned char *kbase = reinterpret_cast<const unsigned char *>(A.k) + from, *vbase = reinterpret_cast<const unsigned char *>(A.v) + from;
  uint32_t k_off[NL], v_off[NL];
#pragma unroll
  for (int m = 0; m < NL; ++m) {
    const int row = row0 + RL * m;
    k_off[m] = (uint32_t)row * (uint32_t)row_bytes + 16 * k_chunk<D>(row, slot0);
    v_off[m] = (uint32_t)row * (uint32_t)row_bytes + 16 * v_chunk<D>(row, slot0);
  }
  // the wave's load m of K's or V's tile t (past the last: nothing but zeros)
  auto load_part = [&](int t, const unsigned char *base, u32x4 *to, bool is_v, int m) {
    const int n = __builtin_amdgcn_readfirstlane(min(places - t * TK, TK)), end = n > 0 ? (n - 1) * (int)row_bytes + 2 * D : 0;
    const __amdgpu_buffer_rsrc_t at = __builtin_amdgcn_make_buffer_rsrc(const_cast<unsigned char *>(base + (int64_t)t * TK * row_bytes), 0, end, 0x00027000);
    __builtin_amdgcn_raw_ptr_buffer_load_lds(at, (lds_ptr)(to + (wave * NL + m) * 64), 16, (int)(is_v ? v_off[m] : k_off[m]), 0, 0, 0);
  };
  auto load = [&](int t, const unsigned char *base, u32x4 *to, bool is_v) {
#pragma unroll
    for (int m = 0; m < NL; ++m) load_part(t, base, to, is_v, m);
  };

  float m_run = -INFINITY, l_run = 0.f;
  f32x16 acc[DT];
#pragma unroll
  for (int dt = 0; dt < DT; ++dt)
#pragma unroll
    for (int i = 0; i < 16; ++i) acc[dt][i] = 0.f;

  // Where the lane reads: K's chunk 2 s + h of row 32 kt + col, and V's operand for channels 32 dt .. and keys 16 s .., two transposed
  // reads of keys 16 s + 4 h + 0..3 and 8 further on. Both are one address with a few bits flipped by s or dt, plus a constant.
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
  // keys behind the query score -inf
  auto hide = [&](int t, f32x16 (&S)[2]) {
    const uint64_t seen = first_keys(p + 1 - t * TK) >> (4 * h);
#pragma unroll
    for (int kt = 0; kt < 2; ++kt) {
      const int word = (int)(uint32_t)(seen >> (32 * kt));
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const uint32_t keep = (uint32_t)__builtin_amdgcn_sbfe(word, (i & 3) + 8 * (i >> 2), 1);
        const float s = S[kt][i];
        S[kt][i] = __builtin_bit_cast(float, (__builtin_bit_cast(uint32_t, s) & keep) | (0xff800000u & ~keep));
      }
    }
  };
  auto highest = [&](const f32x16 (&S)[2]) {
    float m[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) m[i] = top(S[0][i], S[1][i]);
#pragma unroll
    for (int i = 4; i < 16; ++i) m[i & 3] = top(m[i & 3], top(S[0][i], S[1][i]));
    return sl2 * top(top(m[0], m[1]), top(m[2], m[3]));
  };
  // The running maximum takes in a tile's; both halves of the wave hold half of a query's scores. It may lag behind by a factor of 2^8, which weights and
  // sums have room for: so the sums are multiplied anew in the first tiles only, not wherever one of 32 queries finds a larger score.
  auto raise = [&](float mine) {
    if (__builtin_amdgcn_ballot_w64(mine > m_run + 8.f) != 0) {
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
  auto partly_seen = [&](int t) { return t * TK + TK - 1 > b_lo; };
  auto look_through = [&](const u32x4 *v, int at) {
    float z[4] = {0.f, 0.f, 0.f, 0.f};            // sums of 0 times the values: 0, or no number
    const bf16x2 none = {(__bf16)0.f, (__bf16)0.f};
#pragma unroll
    for (int m = 0; m < NL; ++m) {
      const u32x4 w = *(lds_u32x4)((lds_ptr)v + 16 * (lane + 64 * (wave * NL + m)));
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const uint32_t two = w[e];
        z[e] = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, two), none, z[e], false);
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
  // does a query of the wave not see all keys of tile t?
  auto masked = [&](int t) { return t * TK + TK - 1 > w_lo; };

  // ---- The next tile's scores are worked out while this one's weights are: matrix and vector instructions of one wave, which do
  // not wait for each other. K is a tile ahead of V.
  // What was asked for has come, and what was read is in registers: the tiles change hands.
  auto arrived = [] { asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory"); };
  bool later = false;              // tiles left for the end: see below
  {
    f32x16 S[2];
    load(0, kbase, lds_k0, false);
    asm volatile("" ::: "memory");               // (the others are asked for behind K's first tile, which is waited for alone)
    load(0, vbase, lds_v0, true);
    load(1, kbase, lds_k1, false);
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(2 * NL) : "memory");
    product(lds_k0, S);
    if (masked(0)) hide(0, S);
    raise(highest(S));
    // The order of instructions is given, step by step (the compiler asks for each operand right before it needs it): matrix instructions beside a part
    // of the weights, operands asked for two steps ahead. `edge`: a tile that not every query of the block sees whole, or such a next one.
    auto step = [&](auto edge, int t, const u32x4 *k_next, u32x4 *k_free, const u32x4 *v, u32x4 *v_free) {
      constexpr bool EDGE = decltype(edge)::value;
      arrived();
      int k_at = k_lane, v_at = v_lane;
      asm("" : "+v"(k_at), "+v"(v_at));
      constexpr int PART = 16 / KS;          // pairs of weights beside the two matrix instructions of a step
      const f32x16 zero = {};
      f32x16 N[2];
      u32x4 P[4], V[2][DT];
      bf16x8 K[3][2];
      auto read_k = [&](int s) {
#pragma unroll
        for (int kt = 0; kt < 2; ++kt) K[s % 3][kt] = __builtin_bit_cast(bf16x8, *(lds_u32x4)((lds_ptr)k_next + (k_at ^ (32 * s)) + 32 * kt * CH * 16));
      };
      auto read_v = [&](int s) {
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) V[s % 2][dt] = v_operand(v, v_at, dt, s);
      };
      bool odd = false;
      if (EDGE && partly_seen(t)) {
        look_through(v, t & 1);
        odd = odd_values(t & 1);
      }
      const float m_ref = m_run == -INFINITY ? 0.f : m_run;
      float sum[4] = {0.f, 0.f, 0.f, 0.f};
      auto weigh = [&](int pair) {
        const int at = 2 * (pair & 7);
        const float p0 = __builtin_amdgcn_exp2f(__builtin_fmaf(S[pair >> 3][at], sl2, -m_ref));
        const float p1 = __builtin_amdgcn_exp2f(__builtin_fmaf(S[pair >> 3][at + 1], sl2, -m_ref));
        sum[pair & 3] += p0 + p1;
        P[pair >> 2][pair & 3] = __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{p0, p1}), bf16x2));
      };
      // The last tile has no next one, and often no query sees its second half: eight prompts of 33 to 2049 rows 71.7 us without a look at that, 67.9 with.
      // (At head size 64 the branches take more registers than three workgroups on a compute unit leave.)
      const bool last = EDGE && D == 128 && t + 1 >= tiles;
      if (last) {
        read_v(0);
        read_v(1);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int pair = 0; pair < 16; ++pair) weigh(pair);
      } else {
        read_k(0);
        read_k(1);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int s = 0; s < KS; ++s) {
          if (s < NL) {                        // (all at once they would hold up the wave: 8192 rows 527 us, 516 so)
            load_part(t + 2, kbase, k_free, false, s);
            load_part(t + 1, vbase, v_free, true, s);
          }
          if (s + 2 < KS) read_k(s + 2);
          else if (s + 2 == KS) read_v(0);
          else read_v(1);
#pragma unroll
          for (int kt = 0; kt < 2; ++kt) N[kt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(K[s % 3][kt], Q[s], s ? N[kt] : zero, 0, 0, 0);
#pragma unroll
          for (int i = 0; i < PART; ++i) weigh(s * PART + i);
          __builtin_amdgcn_sched_barrier(0);
        }
      }
      if (!EDGE || !odd) {
        l_run += (sum[0] + sum[1]) + (sum[2] + sum[3]);
        float most[4];
#pragma unroll
        for (int s = 0; s < 4; ++s) {
          if (last && s == 2 && places - t * TK <= TK / 2) break;
#pragma unroll
          for (int dt = 0; dt < DT; ++dt) acc[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, V[s % 2][dt]), __builtin_bit_cast(bf16x8, P[s]), acc[dt], 0, 0, 0);
          if (s + 2 < 4) read_v(s + 2);
          if (!EDGE) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const float two = top(N[0][4 * s + i], N[1][4 * s + i]);
              most[i] = s ? top(most[i], two) : two;
            }
          }
          __builtin_amdgcn_sched_barrier(0);
        }
        if (!EDGE) raise(sl2 * top(top(most[0], most[1]), top(most[2], most[3])));
      }
      if (EDGE) {
        later |= odd;
        if (t + 1 < tiles) {
          if (masked(t + 1)) hide(t + 1, N);
          raise(highest(N));
        }
      }
#pragma unroll
      for (int kt = 0; kt < 2; ++kt) S[kt] = N[kt];
    };
    const int seen_whole = __builtin_amdgcn_readfirstlane((b_lo + 1) / TK);
    int t = 0;
    for (; t + 2 < seen_whole; t += 2) {
      step(std::false_type(), t, lds_k1, lds_k0, lds_v0, lds_v1);
      step(std::false_type(), t + 1, lds_k0, lds_k1, lds_v1, lds_v0);
    }
    for (;; t += 2) {
      step(std::true_type(), t, lds_k1, lds_k0, lds_v0, lds_v1);
      if (t + 1 >= tiles) break;
      step(std::true_type(), t + 1, lds_k0, lds_k1, lds_v1, lds_v0);
      if (t + 2 >= tiles) break;
    }
    __builtin_amdgcn_s_waitcnt(0x0f70);              // all that was asked for has come
    // What is infinite or no number must not reach queries that do not see it, and 0 times it is not 0: such tiles come last, key
    // by key, and a key's row is taken in only where it is seen.
    if (__syncthreads_or(later)) {
      for (int t = 0; t < tiles; ++t) {
        if (!partly_seen(t)) continue;
        arrived();
        load(t, kbase, lds_k0, false);
        load(t, vbase, lds_v0, true);
        arrived();
        look_through(lds_v0, 0);
        if (!odd_values(0)) continue;
        u32x4 P[4];
        product(lds_k0, S);
        hide(t, S);
        l_run += weights(S, P);
        const uint64_t seen = first_keys(p + 1 - t * TK);
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
      __syncthreads();             // (nobody reads the tiles any more)
    }
  }

  // ---- out
  {
    const uint32_t w = __builtin_bit_cast(uint32_t, l_run);
    const auto q = __builtin_amdgcn_permlane32_swap(w, w, false, false);
    const uint32_t q0 = q[0], q1 = q[1];
    l_run = __builtin_bit_cast(float, q0) + __builtin_bit_cast(float, q1);
  }
  // The wave's rows go through LDS (16 bytes at a time, at other places in every row, so that neither way meets in a bank), to be written as they lie in memory:
  // lane by lane they would leave in pieces of 8 or 16 bytes.
  const float inv = l_run == 0.f ? 0.f : 1.f / l_run;
  const size_t row = (size_t)piece.begin + p;
  const lds_ptr mine = (lds_ptr)(wave == 0 ? lds_k0 : wave == 1 ? lds_k1 : wave == 2 ? lds_v0 : lds_v1);
  auto write_out = [&](auto wide) {
    constexpr bool F32 = decltype(wide)::value;
    constexpr int PIECES = D * (F32 ? 4 : 2) / 16, AT_ONCE = 64 / PIECES;       // of a row; rows that a store covers
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
      for (int j = 0; j < (F32 ? 4 : 2); ++j) {
        u32x4 w;
        int at;
        if constexpr (F32) {
#pragma unroll
          for (int i = 0; i < 4; ++i) w[i] = __builtin_bit_cast(uint32_t, acc[dt][4 * j + i] * inv);
          at = 8 * dt + 2 * j + h;
        } else {
          // (channels 16 j + 4 h .. and 8 further on: the halves of the wave exchange some, so that each has eight side by side)
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            const uint32_t lo = __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{acc[dt][8 * j + 2 * i] * inv, acc[dt][8 * j + 2 * i + 1] * inv}), bf16x2));
            const uint32_t hi = __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{acc[dt][8 * j + 4 + 2 * i] * inv, acc[dt][8 * j + 5 + 2 * i] * inv}), bf16x2));
            const auto q = __builtin_amdgcn_permlane32_swap(lo, hi, false, false);
            w[i] = q[0];
            w[2 + i] = q[1];
          }
          at = 4 * dt + 2 * j + h;
        }
        *(__attribute__((address_space(3))) u32x4 *)(mine + 16 * (col * PIECES + (at ^ (col & (PIECES - 1))))) = w;
      }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");             // (of this wave alone)
    const int piece_at = lane % PIECES;
#pragma unroll
    for (int i = 0; i < 32 / AT_ONCE; ++i) {
      const int at = i * AT_ONCE + lane / PIECES, r = row_w + at;
      const u32x4 w = *(lds_u32x4)(mine + 16 * (at * PIECES + (piece_at ^ (at & (PIECES - 1)))));
      const int pos = A.by_group.of(min(r, rows - 1));
      if (r < rows) *reinterpret_cast<u32x4 *>(static_cast<unsigned char *>(A.out) + (((size_t)piece.begin + pos) * A.Hq + g * A.G + r - pos * A.G) * (D * (F32 ? 4 : 2)) + 16 * piece_at) = w;
    }
  };
  if (A.out_dtype == STS_F32) write_out(std::true_type());
  else write_out(std::false_type());
  if (!ok) return;
  // (a row whose sum is no number has the logarithm -inf, as everywhere in the library)
  if (A.lse_out && h == 0) A.lse_out[(size_t)head * A.seqs.T + row] = l_run > 0.f ? (m_run + __builtin_amdgcn_logf(l_run)) * 0.69314718055994530942f : -INFINITY;
}

}  // namespace

hipError_t launch_prompt_attn(const PromptArgs &a, int d, hipStream_t s) {
  const dim3 grid((unsigned)((int64_t)a.numbers * a.Hkv)), block(64 * WAVES);
  if (d == 128) STS_LAUNCH(prompt_attn_kernel<128>, grid, block, 0, s, a);
  else STS_LAUNCH(prompt_attn_kernel<64>, grid, block, 0, s, a);
  return sts_take_launch_status();
}
