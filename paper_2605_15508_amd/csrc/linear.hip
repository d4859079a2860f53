// Linear attention with a decay for each head (gfx950): per KV head a state S of d x d numbers in fp32, and
//     S_i = exp(g_i) S_(i-1) + k_i v_i^T,    out_i = scale q_i^T S_i.
//
// The recurrent form (few rows of a sequence) does just that. A workgroup has 32 columns of a state, a thread 4 of them in d / 32 rows; the state
// is read once, stays in registers for all rows and is written once. What bounds it: memory, 8 bytes for every number of the state.
//
// The chunked form (prompts) takes 32 rows at a time. With c_i the sum of g over the chunk's rows up to i,
//     out_i = scale (exp(c_i) q_i^T S + sum_(j <= i) exp(c_i - c_j) (q_i . k_j) v_j),    S' = exp(c_32) S + sum_j exp(c_32 - c_j) k_j v_j^T.
// A wave has 32 columns of the state (and of out) in the accumulators of v_mfma_f32_32x32x16_bf16 and works out the chunk's 32 x 32
// products q . k by itself, so that these pass from accumulator to operand in their lane, as the state does: nothing goes through LDS but
// rows of Q, K and V. Long sequences are cut into segments: one kernel sums up what each segment adds to the state, one
// adds these up along the sequence, and a third starts every segment from the state before it.
// What bounds it without groups: memory. 8192 rows with 32 heads of 128 take 118 us: sums 35 (170 MB, 4.8 TB/s), adding up 14 (64 MB), results 60
// (300 MB, 5.0 TB/s), and what lies between three launches; 131 us where no input is left in the cache behind the L2s from the pass before (sums 43, results 61 to 72).
// With groups of heads, of which a workgroup of the results has two that share a state, matrix and vector instructions, which hardly overlap: six prompts of 77
// to 6001 rows, 32 heads in groups of four, 89 us, of which the results 61 (with a head for each workgroup 103 and 75).
#include "attn_util.h"
#include "layers.h"

namespace {

constexpr int C = STS_LINEAR_CHUNK;
constexpr float LOG2E = 1.44269504088896340736f;
constexpr double LOG2E_64 = 1.44269504088896340736;
constexpr float WEAKEST = -30.f;          // the logarithm (of base 2) of a chunk's decays from which on its pairs of rows get weights of their own
static_assert(C == 32, "");

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) s16x4 *lds_s16x4;
typedef __attribute__((address_space(3))) unsigned char *lds_ptr;
typedef const __attribute__((address_space(3))) u32x4 *lds_u32x4;
typedef __attribute__((address_space(3))) float *lds_f32;

// 2^x in 64 bits (to some 1e-14), for x <= 1000: the series of exp on [-ln(2) / 2, ln(2) / 2]
__device__ __forceinline__ double exp2_64(double x) {
  const double n = __builtin_rint(x), r = (x - n) * 0.69314718055994530942;
  double p = 1.0 / 39916800.0;
  p = __builtin_fma(p, r, 1.0 / 3628800.0);
  p = __builtin_fma(p, r, 1.0 / 362880.0);
  p = __builtin_fma(p, r, 1.0 / 40320.0);
  p = __builtin_fma(p, r, 1.0 / 5040.0);
  p = __builtin_fma(p, r, 1.0 / 720.0);
  p = __builtin_fma(p, r, 1.0 / 120.0);
  p = __builtin_fma(p, r, 1.0 / 24.0);
  p = __builtin_fma(p, r, 1.0 / 6.0);
  p = __builtin_fma(p, r, 0.5);
  p = __builtin_fma(p, r, 1.0);
  p = __builtin_fma(p, r, 1.0);
  return x < -1000.0 ? 0.0 : __builtin_ldexp(p, (int)n);
}

// the same in 32 bits, of a sum that is kept in 64
__device__ __forceinline__ float exp2_32(double x) {
  const float y = (float)x, rest = (float)(x - (double)y);
  return __builtin_amdgcn_exp2f(y) * (1.f + 0.6931471806f * rest);
}

// where the state of sequence b begins, or NULL: there is none (a slot outside the pool stands for none)
__device__ __forceinline__ const float *state_in(const LinearArgs &A, int b) {
  if (!A.state) return nullptr;
  const int slot = A.slots ? A.slots[b] : b;
  return slot < 0 || slot >= A.num_slots ? nullptr : A.state + slot * A.state_stride;
}
__device__ __forceinline__ float *state_out(const LinearArgs &A, int b) {
  if (!A.state_out) return nullptr;
  const int slot = A.slots_out ? A.slots_out[b] : b;
  return slot < 0 || slot >= A.num_slots_out ? nullptr : A.state_out + slot * A.state_out_stride;
}
// the rows of a sequence that count
__device__ __forceinline__ int rows_of(const LinearArgs &A, int b, int len) { return min(A.lens ? min(max(A.lens[b], 0), len) : len, A.max_len); }

__device__ __forceinline__ float of_bf16(uint32_t bits) { return __builtin_bit_cast(float, bits << 16); }

// ---------------------------------------------------------------------------------------------- recurrent form
template <int N> struct Words { uint32_t w[N]; };

// A workgroup has 32 columns of a state, a thread four of them in D / 32 rows. All that it reads is asked for at once; the state stays in registers
// and is written once. AT_ONCE rows of 4 / AT_ONCE heads each are a step: four results, whose sums over the state's rows are made together.
//
// With one row memory bounds it: 64 sequences with 32 heads of 128 take 53 us for the 268 MB of their states, 5.1 TB/s. More rows add vector instructions, 140
// for a step of the wave: without other waves on its SIMD 0.5 us (0.2 us for each of four rows at once, 0.5 for one after the other).
// The matrix instruction for fp32 (4x4x1, k v^T and q^T S both) was as slow: 13.1 us for 16 rows of a sequence with groups of four heads, 11.7 here.
template <int D, int AT_ONCE>
__global__ void __launch_bounds__(256) linear_step_kernel(const LinearArgs A) {
  constexpr int RK = D / 32;              // rows of the state per thread
  constexpr int SLICES = D / 32, MAX = STS_LINEAR_STEP, HEADS = 4 / AT_ONCE;
  constexpr int QUERIES = 64, CHUNKS = D / 8, ASKS = QUERIES * CHUNKS / 256;
  static_assert(QUERIES >= STS_MAX_GROUP && MAX * CHUNKS <= 256, "");
  __shared__ __attribute__((aligned(16))) uint16_t lds_k[MAX + 3][D], lds_v[MAX + 3][32], lds_q[QUERIES + 3][D];      // (a step may look at what no row has)
  __shared__ float lds_f[MAX + 3];
  __shared__ __attribute__((aligned(16))) float lds_o[2][4][4][32];

  const int tid = threadIdx.x, wave = tid >> 6;
  const int unit = blockIdx.x / SLICES, slice = blockIdx.x % SLICES;
  const int b = A.by_heads.of(unit), g = unit - b * A.Hkv;
  int begin, len;
  seq_rows(A.seqs, b, begin, len);
  const int n = min(rows_of(A, b, len), MAX);
  const int col = 32 * slice + 4 * (tid & 7), row = RK * (tid >> 3);
  f32x4 S[RK];
  const float *from = state_in(A, b);
  const size_t head_at = (size_t)g * D * D;
#pragma unroll
  for (int r = 0; r < RK; ++r) S[r] = f32x4{0.f, 0.f, 0.f, 0.f};
  if (from) {
#pragma unroll
    for (int r = 0; r < RK; ++r) S[r] = *reinterpret_cast<const f32x4 *>(from + head_at + (row + r) * D + col);
  }
  // Queries of as many rows as there is room for. They, the rows of K and V and the decays are all asked for before any is waited for.
  const int rows = QUERIES / A.G;        // (a multiple of AT_ONCE where that is not 1)
  u32x4 q[ASKS];
  auto ask = [&](int t0) {
    const int count = min(rows, n - t0) * A.G * CHUNKS;
#pragma unroll
    for (int i = 0; i < ASKS; ++i) {
      const int at = tid + 256 * i, r = A.by_group.of(at / CHUNKS), h = at / CHUNKS - r * A.G;
      if (at < count) q[i] = *reinterpret_cast<const u32x4 *>(A.q + (begin + t0 + (int64_t)r) * A.q_stride_n + (g * A.G + h) * A.q_stride_h + 8 * (at % CHUNKS));
    }
  };
  auto put = [&](int t0) {
    const int count = min(rows, n - t0) * A.G * CHUNKS;
#pragma unroll
    for (int i = 0; i < ASKS; ++i)
      if (tid + 256 * i < count) *reinterpret_cast<u32x4 *>(&lds_q[0][8 * (tid + 256 * i)]) = q[i];
    __syncthreads();
  };
  if (n > 0) {
    const int tk = tid / CHUNKS, tv = tid / 4;
    const u32x4 k = *reinterpret_cast<const u32x4 *>(A.k + (begin + (int64_t)min(tk, n - 1)) * A.kv_stride_n + g * A.kv_stride_h + 8 * (tid % CHUNKS));
    const u32x4 v = *reinterpret_cast<const u32x4 *>(A.v + (begin + (int64_t)min(tv, n - 1)) * A.kv_stride_n + g * A.kv_stride_h + 32 * slice + 8 * (tid % 4));
    const float decay = A.decay[A.decay_rows ? (begin + (size_t)min(tid, n - 1)) * A.Hkv + g : g];
    if (A.out) ask(0);
    if (tk < n) *reinterpret_cast<u32x4 *>(&lds_k[tk][8 * (tid % CHUNKS)]) = k;
    if (tv < n) *reinterpret_cast<u32x4 *>(&lds_v[tv][8 * (tid % 4)]) = v;
    if (tid < n) lds_f[tid] = (float)exp2_64((double)decay * LOG2E_64);
    if (A.out) put(0);
    else __syncthreads();
  }

  struct Row { Words<RK / 2> k; u32x2 v; float f; };
  auto row_of = [&](int t) { return Row{*reinterpret_cast<const Words<RK / 2> *>(&lds_k[t][row]), *reinterpret_cast<const u32x2 *>(&lds_v[t][4 * (tid & 7)]), lds_f[t]}; };
  auto half = [](const auto &w, int i) { return of_bf16(i % 2 ? w[i / 2] >> 16 : w[i / 2] & 0xffffu); };
  auto take_in = [&](const Row &x) {
    const uint32_t v0 = x.v[0], v1 = x.v[1];
    const f32x4 v = {of_bf16(v0 & 0xffffu), of_bf16(v0 >> 16), of_bf16(v1 & 0xffffu), of_bf16(v1 >> 16)};
#pragma unroll
    for (int r = 0; r < RK; ++r) S[r] = S[r] * x.f + v * half(x.k.w, r);
  };
  if (!A.out) {
#pragma unroll 4
    for (int t = 0; t < n; ++t) take_in(row_of(t));
  }
  const int u = tid >> 5, c = tid & 31;             // the result of a step that the thread brings
  const size_t own_out = ((size_t)(begin + u / HEADS) * A.Hq + g * A.G + u % HEADS) * D + 32 * slice + c;
  for (int t = 0, r0 = 0, parity = 0; A.out && t < n; t += AT_ONCE) {
    if (t - r0 >= rows) {
      r0 = t;            // (all that is in LDS was read before the last barrier)
      ask(t);
      put(t);
    }
    Row own[AT_ONCE];
#pragma unroll
    for (int i = 0; i < AT_ONCE; ++i) own[i] = row_of(t + i);
    for (int h0 = 0; h0 < A.G; h0 += HEADS) {
      Words<RK / 2> w[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) w[i] = *reinterpret_cast<const Words<RK / 2> *>(&lds_q[(t - r0) * A.G + h0 + i][row]);
      f32x4 o[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if (i % HEADS == 0 && h0 == 0 && t + i / HEADS < n) take_in(own[i / HEADS]);
        o[i] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int r = 0; r < RK; ++r) o[i] += S[r] * half(w[i].w, r);
      }
      // The wave's eight groups of rows are added up: first the halves, of which each goes on with two of the four, then the rows of 16 lanes, with one
      // each, then the lanes that are 8 apart.
      f32x4 x;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        float y[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const float lo = o[i][e], hi = o[i + 2][e];
          const auto p = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(uint32_t, lo), __builtin_bit_cast(uint32_t, hi), false, false);
          const uint32_t p0 = p[0], p1 = p[1];
          y[i] = __builtin_bit_cast(float, p0) + __builtin_bit_cast(float, p1);
        }
        const auto p = __builtin_amdgcn_permlane16_swap(__builtin_bit_cast(uint32_t, y[0]), __builtin_bit_cast(uint32_t, y[1]), false, false);
        const uint32_t p0 = p[0], p1 = p[1];
        const float z = __builtin_bit_cast(float, p0) + __builtin_bit_cast(float, p1);
        x[e] = z + __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, z), 0x128, 0xf, 0xf, true));       // row_ror:8
      }
      if (!(tid & 8)) *reinterpret_cast<f32x4 *>(&lds_o[parity][(tid >> 5 & 1) * 2 + (tid >> 4 & 1)][wave][4 * (tid & 7)]) = x;
      __syncthreads();
      if (u < 4 && t + u / HEADS < n && h0 + u % HEADS < A.G) {
        const float o = A.scale * ((lds_o[parity][u][0][c] + lds_o[parity][u][1][c]) + (lds_o[parity][u][2][c] + lds_o[parity][u][3][c]));
        const size_t to = own_out + ((size_t)t * A.Hq + h0) * D;
        if (A.out_dtype == STS_F32) static_cast<float *>(A.out)[to] = o;
        else static_cast<__bf16 *>(A.out)[to] = (__bf16)o;
      }
      parity ^= 1;         // (the next results go elsewhere; those after them come behind the next barrier)
    }
  }
  float *to = state_out(A, b);
  if (!to) return;
#pragma unroll
  for (int r = 0; r < RK; ++r) *reinterpret_cast<f32x4 *>(to + head_at + (row + r) * D + col) = S[r];
}

// ------------------------------------------------------------------------------------------------ chunked form
// Where 16-byte chunk c of row r lies in its row: neither reads of one chunk of 16 rows nor transposing reads of 64 bytes of 4 rows meet in a
// bank.
template <int D> __device__ __forceinline__ int place(int r, int c) {
  return D == 128 ? c ^ ((r & 3) << 2 | (r >> 2 & 3)) : c ^ ((r >> 1 & 1) << 2 | (r >> 2 & 3));
}

// Sums over a half's 32 lanes, of which both halves hold the same: up to the lane's own, or behind it. Within rows of 16 lanes by shifts, from row to row
// by a scalar.
template <int FIRST>
__device__ __forceinline__ float scan16(float x) {
  auto add = [&](auto ctrl) { x += __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), decltype(ctrl)::value, 0xf, 0xf, true)); };
  add(std::integral_constant<int, FIRST>());
  add(std::integral_constant<int, FIRST + 1>());
  add(std::integral_constant<int, FIRST + 3>());
  add(std::integral_constant<int, FIRST + 7>());
  return x;
}
__device__ __forceinline__ float lane_of(float x, int lane) { return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, x), lane)); }
__device__ __forceinline__ float sum_up_to(float x) {
  x = scan16<0x111>(x);                                    // row_shr
  return threadIdx.x & 16 ? x + lane_of(x, 15) : x;
}
__device__ __forceinline__ float sum_behind(float x) {
  const float next = __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), 0x101, 0xf, 0xf, true));      // row_shl:1
  const float y = scan16<0x101>((threadIdx.x & 31) == 15 ? lane_of(x, 16) : next);
  return threadIdx.x & 16 ? y : y + lane_of(y, 16);
}

// the same in 64 bits over `places` lanes, up to the one before
__device__ __forceinline__ double lane_of(double x, int lane) {
  const u32x2 w = __builtin_bit_cast(u32x2, x);
  const uint32_t w0 = w[0], w1 = w[1];
  return __builtin_bit_cast(double, u32x2{(uint32_t)__builtin_amdgcn_readlane((int)w0, lane), (uint32_t)__builtin_amdgcn_readlane((int)w1, lane)});
}
template <int PLACES>
__device__ __forceinline__ double sums_before(double x) {
  auto lower = [&](auto ctrl) {
    const u32x2 w = __builtin_bit_cast(u32x2, x);
    const uint32_t w0 = w[0], w1 = w[1];
    return __builtin_bit_cast(double, u32x2{(uint32_t)__builtin_amdgcn_update_dpp(0, (int)w0, decltype(ctrl)::value, 0xf, 0xf, true), (uint32_t)__builtin_amdgcn_update_dpp(0, (int)w1, decltype(ctrl)::value, 0xf, 0xf, true)});
  };
  x += lower(std::integral_constant<int, 0x111>());        // row_shr
  x += lower(std::integral_constant<int, 0x112>());
  x += lower(std::integral_constant<int, 0x114>());
  x += lower(std::integral_constant<int, 0x118>());
  const double y = lower(std::integral_constant<int, 0x111>());
  return PLACES == 32 && threadIdx.x & 16 ? y + lane_of(x, 15) : y;
}

// A segment's numbers lie as the waves hold them: element 4 e .. of tile m, four side by side, lane by lane, wave by wave. Place 4 q .. is this number of
// the state and the three below it:
template <int D> __device__ __forceinline__ int state_place(int q) {
  constexpr int NW = D / 32;
  const int lane = q & 63, wave = (q >> 6) % NW, e = (q >> 6) / NW % 4, m = (q >> 6) / NW / 4;
  return (32 * m + 16 * (e >> 1) + 8 * (lane >> 5) + 4 * (e & 1)) * D + 32 * wave + (lane & 31);
}

// Two workgroups of four waves on a compute unit (head size 64: four of two waves), three chunks in LDS for each: one that is worked on, one that has come, one under
// way; two of them where the queries of two heads come with each. A chunk of 32 rows takes 24 matrix instructions of a wave at head size 128 for the state, whose terms
// are split in three, 18 for each head, and some 160 vector instructions for either.
//
// OUT: results, from the state before the segment; else what the segment adds to the state (or, of a sequence with one segment, its
// state)
template <int D, bool OUT, int HEADS>
__global__ void __launch_bounds__(2 * D, 2) linear_chunk_kernel(const LinearArgs A) {
  constexpr int NW = D / 32;             // waves, each with 32 columns of the state
  constexpr int KS = D / 16, MT = D / 32, CH = D / 8;
  constexpr int NL = C * CH / (64 * NW), RL = 64 / CH;      // loads of a wave for 32 rows, rows that each covers
  // (What LDS has left at two and four workgroups. Each time takes 2 us: 8192 rows, 17 chunks a segment, 123 us with 15 at once, 119 with 18.)
  constexpr int BLOCK = D == 128 ? 18 : HEADS == 2 ? 16 : 9, MINE = (BLOCK + NW - 1) / NW;   // chunks whose decays are worked out at once, those of a wave
  constexpr int PLACES = BLOCK >= 16 ? 32 : 16;              // lanes that have one of them, or none
  // Three chunks of K, V and Q, and a block's decays: for each row its sum c, its weight as a key, its factor as a query, and for each chunk what
  // concerns all rows. Arrays of their own, so that the compiler can tell the loads that fill one from the reads of another; it would have reads of an array
  // that no load fills wait for all loads, so that one load of no bytes goes to the decays', too.
  constexpr int TILE = C * CH, AT_V = TILE, AT_Q = 2 * TILE, ALL = (OUT ? 2 + HEADS : 2) * TILE, DEPTH = HEADS == 2 ? 2 : 3;
  constexpr int LOADS = (OUT ? 2 + HEADS : 2) * NL, STORES = OUT ? 2 * HEADS : 0;      // of a wave and chunk
  constexpr int AT_KEY = MINE * NW * C * 4, AT_QUERY = 2 * AT_KEY, AT_CHUNK = 3 * AT_KEY;
  __shared__ __attribute__((aligned(16))) u32x4 lds_0[ALL], lds_1[ALL], lds_2[DEPTH == 3 ? ALL : 1], lds_d[AT_CHUNK / 16 + PLACES];

  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const int h = lane >> 5, col = lane & 31;
  // Neighbouring units on different dies (workgroup i runs on die i % 8), which evens out the numbers that no segment has; the heads of a group (each
  // with a state of its own, which is the same) on one die, one after the other: they read the same K and V.
  const int turns = blockIdx.x / STS_XCDS, eight = OUT ? A.by_turns.of(turns) : turns, hd = OUT ? turns * HEADS - eight * A.G : 0;
  const int unit = eight * STS_XCDS + blockIdx.x % STS_XCDS;
  if (unit >= A.numbers * A.Hkv) return;
  const int number = A.by_heads.of(unit), g = unit - number * A.Hkv, head = g * A.G + hd;
  const PackedPiece piece = find_piece(A.seqs, number, [&](int begin) { return A.by_segment.of(begin); });
  if (piece.b < 0) return;
  const int len = rows_of(A, piece.b, piece.len), first = piece.index * A.segment;
  const int segments = max((len + A.segment - 1) / A.segment, 1);
  if (first >= max(len, 1)) return;
  // (the last segment's state is brought by the results' kernel)
  if (!OUT && A.out && piece.index >= segments - 1) return;
  // (the same for all lanes, which the compiler does not see)
  const int rows = __builtin_amdgcn_readfirstlane(min(A.segment, len - first)), begin = __builtin_amdgcn_readfirstlane(piece.begin + first), chunks = (rows + C - 1) / C;
  const bool last = first + rows >= len;

  // ---- loads, straight to LDS. Rows behind the last lie behind the end that the loads are told and come as zeros; so do whole chunks (the number of
  // loads is always the same).
  const int row0 = wave * NL * RL + lane / CH, slot0 = lane % CH;
  uint32_t kv_off[NL], q_off[NL];
#pragma unroll
  for (int m = 0; m < NL; ++m) {
    const int row = row0 + RL * m;
    kv_off[m] = (uint32_t)row * (uint32_t)(A.kv_stride_n * 2) + 16 * place<D>(row, slot0);
    q_off[m] = (uint32_t)row * (uint32_t)(A.q_stride_n * 2) + 16 * place<D>(row, slot0);
  }
  auto load_rows = [&](int chunk, const uint16_t *base, int64_t stride, const uint32_t (&off)[NL], u32x4 *to) {
    const int n = __builtin_amdgcn_readfirstlane(min(rows - chunk * C, C)), end = n > 0 ? (n - 1) * (int)(stride * 2) + 2 * D : 0;
    const __amdgpu_buffer_rsrc_t at = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint16_t *>(base + (int64_t)chunk * C * stride), 0, end, 0x00027000);
#pragma unroll
    for (int m = 0; m < NL; ++m) __builtin_amdgcn_raw_ptr_buffer_load_lds(at, (lds_ptr)(to + (wave * NL + m) * 64), 16, (int)off[m], 0, 0, 0);
  };
  const uint16_t *k = A.k + begin * A.kv_stride_n + g * A.kv_stride_h, *v = A.v + begin * A.kv_stride_n + g * A.kv_stride_h;
  const uint16_t *q = A.q + begin * A.q_stride_n + head * A.q_stride_h;
  auto load = [&](int chunk, u32x4 *to) {
    load_rows(chunk, k, A.kv_stride_n, kv_off, to);
    load_rows(chunk, v, A.kv_stride_n, kv_off, to + AT_V);
    if constexpr (OUT) {
#pragma unroll
      for (int hh = 0; hh < HEADS; ++hh) load_rows(chunk, q + hh * A.q_stride_h, A.q_stride_n, q_off, to + AT_Q + hh * TILE);
    }
    asm volatile("" ::: "memory");       // (a chunk's stores come behind these loads: see `turn`)
  };
  // (a wave's part of a block's decays: row `col` of every NW-th chunk; of a sequence without rows that of a row next to it, which nothing comes of)
  float gates[MINE];
  auto load_gates = [&](int base) {
#pragma unroll
    for (int i = 0; i < MINE; ++i) gates[i] = A.decay[A.decay_rows ? (size_t)max(begin + min((base + wave + i * NW) * C + col, rows - 1), 0) * A.Hkv + g : g];
  };
  // (the load of no bytes: it writes zeros all the same, whenever it ends, so that it goes where no chunk has anything)
  static_assert(16 * (PLACES - MINE * NW) >= 64, "");
  if (lane < 16)
    __builtin_amdgcn_raw_ptr_buffer_load_lds(__builtin_amdgcn_make_buffer_rsrc(const_cast<uint16_t *>(A.k), 0, 0, 0x00027000), (lds_ptr)lds_d + AT_CHUNK + 16 * MINE * NW, 4, 0, 0, 0, 0);
  load_gates(0);
  load(0, lds_0);

  // ---- the state: lane (h, col) has column 32 wave + col, in element 4 j + i of tile m the row 32 m + 16 (j / 2) + 8 h + 4 (j % 2) + i
  f32x16 S[MT];
  const size_t part = (size_t)number * A.Hkv + g, part_at = part * D * D;
  // (Workgroups of one group start from a copy of a sequence's state: the one that writes the state behind its rows may be done before another begins.)
  const bool carried = A.part && (segments > 1 || (OUT && A.G > HEADS));
  const float *from = carried ? (OUT ? A.part + part_at : nullptr) : state_in(A, piece.b);
  if (!carried && from) from += (size_t)g * D * D;
  const int s_at = 8 * h * D + 32 * wave + col, p_at = 256 * wave + 4 * lane;
  if (from && carried) {
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const f32x4 x = *reinterpret_cast<const f32x4 *>(from + p_at + (4 * m + e) * NW * 256);
#pragma unroll
        for (int i = 0; i < 4; ++i) S[m][4 * e + i] = x[i];
      }
  } else if (from) {
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
      for (int e = 0; e < 16; ++e) S[m][e] = from[s_at + (32 * m + 16 * (e >> 3) + (e & 7)) * D];
  } else {
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
      for (int e = 0; e < 16; ++e) S[m][e] = 0.f;
  }

  // ---- reads: chunk 2 s + h of row col; by the transposing read rows 16 s + 4 h + 0..3 and 8 further on of 32 channels. For K the middle two
  // of each 16 channels' fours change places: then the state's rows lie in a lane's accumulators in the order of an operand.
  const int r_lane = col * CH * 16 + 16 * place<D>(col, h);
  const int t_row = 4 * h + ((lane & 15) >> 2), t_four = lane & 3;
  auto first_of = [&](int chan) { return (t_row * CH + place<D>(t_row, chan >> 3)) * 16 + (chan & 7) * 2; };
  const int v_lane = first_of(32 * wave + (lane & 16) + 4 * t_four), k_lane = first_of((lane & 16) + 4 * ((t_four & 1) << 1 | t_four >> 1));
  // (8 rows further on bit 1 of a chunk's place changes, 32 channels further on bit 2)
  auto transposed = [&](const u32x4 *tile, int at, int m, int s) {
    u32x4 w;
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const u32x2 two = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4)((lds_ptr)tile + (at ^ (64 * m) ^ (32 * e)) + (16 * s + 8 * e) * CH * 16)));
      w[2 * e] = two[0];
      w[2 * e + 1] = two[1];
    }
    return __builtin_bit_cast(bf16x8, w);
  };
  // The chunk has come: behind its loads lie the next chunk's and the last chunk's stores at least (memory operations end in their order). And
  // what was read is in registers.
  auto turn = [] { asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(DEPTH == 3 ? LOADS + STORES : STORES) : "memory"); };
  auto all_waves = [] { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); };

  // ---- Decays, in powers of two: c_i the sum over the chunk's rows up to i. With u_i = exp(c_i - c_32)
  //     out_i = scale u_i (q_i . (exp(c_32) S) + sum exp(c_32 - c_j) (q_i . k_j) v_j),
  // so that each key has one weight, which the state takes too. Not where a chunk's decays make up less than 2^-30, a row's doubles the state or a decay is
  // no number: in such a chunk (`apart`) each pair's weight is worked out, which takes the results' kernel a quarter to a third longer (8192 rows with 32
  // heads 119 us in all without such chunks, 134 with none but such; another six prompts in groups of four heads 103 and 125). Sums in a chunk that is not
  // apart are smaller than the results by up to u F, 2^46; with 2^-60 in place of 2^-30, 2^76, results of values of 1e-20 were lost among fp32's smallest
  // numbers. Where the scale is beyond 2^48, its product with u F could leave fp32's range (u F is up to 2^78 where decays are above 0): every chunk is apart.
  // The state is held as S / F with 1 <= F < 2^16: F is the decays' product so far but for a power of 2^16, by which the state is multiplied
  // where F would leave that range (exactly), and a key's weight is divided by F. F's logarithm `low` is a sum in 64 bits: no factor's rounding adds up
  // over a long sequence.
  // A chunk has the power of two, apart (1) or not (0), the logarithm of F before it, and 1 where a row doubles the state.
  double all = 0.0, low = 0.0;
  const float weakest = __builtin_fabsf(A.scale) < 0x1p48f ? WEAKEST : INFINITY;
  const lds_ptr decays = (lds_ptr)lds_d;
  auto number_of = [&](int at) { return *(lds_f32)(decays + at); };
  auto work_out = [&](int base) {
    auto power = [](float decay) { return decay * LOG2E < -150.f ? -150.f : decay * LOG2E; };      // (2^-150 is 0 in fp32; an infinite sum would have no differences)
    float c[MINE], after[MINE];
#pragma unroll
    for (int i = 0; i < MINE; ++i) {
      const int chunk = wave + i * NW;
      const float own = (base + chunk) * C + col < rows ? power(gates[i]) : 0.f;
      c[i] = sum_up_to(own);
      after[i] = sum_behind(own);
      *(lds_f32)(decays + chunk * C * 4 + 4 * col) = c[i];
      *(lds_f32)(decays + AT_CHUNK + 16 * chunk + 12) = __builtin_amdgcn_ballot_w64(own > 1.f) ? 1.f : 0.f;
    }
    if (HEADS == 1) load_gates(base + BLOCK);
    all_waves();
    // (no branches but those that all lanes take alike: the loop around would get ways through it that there are not, and the compiler's waits with them)
    int mine = lane & (PLACES - 1);        // the lane's chunk
    asm("" : "+v"(mine));                   // (what comes of it is made anew, not kept in registers)
    const float end = number_of((min(mine, BLOCK - 1) * C + 31) * 4), grows = number_of(AT_CHUNK + 16 * mine + 12);
    const double sum = sums_before<PLACES>(mine < BLOCK ? end : 0.0), before = low + sum, behind = before + end;      // (0 behind the last chunk)
    const double total = lane_of(sum, BLOCK - 1) + lane_of(end, BLOCK - 1);
    low += total;
    all += total;
    auto whole = [](double x) { return __builtin_floor(x * 0.0625) * 16.0; };
    const double low_before = before - whole(before), low_behind = behind - whole(behind);
    const float F = exp2_32(low_behind), F_inv = exp2_32(-low_behind), step = __builtin_amdgcn_exp2f((float)(whole(behind) - whole(before)));
    low = lane_of(low - whole(low), 0);        // (the same in all lanes, and so in scalar registers)
    *(__attribute__((address_space(3))) f32x4 *)(decays + AT_CHUNK + 16 * mine) = f32x4{step, end >= weakest && grows == 0.f ? 0.f : 1.f, (float)low_before, grows};
#pragma unroll
    for (int i = 0; i < MINE; ++i) {
      const int chunk = wave + i * NW, row = (base + chunk) * C, at = chunk * C * 4;
      auto of_chunk = [&](float x) { return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, x), min(chunk, BLOCK - 1))); };
      const float factor = of_chunk(F), inverse = of_chunk(F_inv), c_end = of_chunk(end);
      *(lds_f32)(decays + AT_KEY + at + 4 * col) = row + col < rows ? __builtin_amdgcn_exp2f(after[i]) * inverse : 0.f;
      *(lds_f32)(decays + AT_QUERY + at + 4 * col) = A.scale * (c_end >= weakest && of_chunk(grows) == 0.f ? factor * __builtin_amdgcn_exp2f(c[i] - c_end) : 1.f);
    }
    all_waves();
  };
  auto multiply = [&](float f) {
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
      for (int e = 0; e < 16; ++e) S[m][e] *= f;
  };

  auto body = [&](int chunk, int in_block, u32x4 *lds, u32x4 *free) {
    turn();
    load(chunk + DEPTH - 1, free);         // (before the reads: behind them the compiler would wait for the next chunk's)
    // (what comes of these is made anew in every chunk, not kept in registers)
    int r_at = r_lane, v_at = v_lane, k_at = k_lane;
    asm("" : "+v"(r_at), "+v"(v_at), "+v"(k_at));
    // what is read is asked for first
    const lds_ptr mine = decays + in_block * C * 4;
    const f32x4 four = *(const __attribute__((address_space(3))) f32x4 *)(decays + AT_CHUNK + 16 * in_block);
    bf16x8 K[KS], Q[KS], T[2 * MT], V[2];
#pragma unroll
    for (int s = 0; s < 2; ++s) V[s] = transposed(lds + AT_V, v_at, 0, s);
    float left[16];                // weights of keys 8 j + 4 h + i
#pragma unroll
    for (int e = 0; e < 16; ++e) left[e] = *(lds_f32)(mine + AT_KEY + 4 * (8 * (e >> 2) + 4 * h + (e & 3)));
    const float own_factor = OUT ? *(lds_f32)(mine + AT_QUERY + 4 * col) : 0.f;
    auto read_rows = [&](int hh) {
#pragma unroll
      for (int s = 0; s < KS; ++s) {
        K[s] = __builtin_bit_cast(bf16x8, *(lds_u32x4)((lds_ptr)lds + (r_at ^ (32 * s))));
        Q[s] = __builtin_bit_cast(bf16x8, *(lds_u32x4)((lds_ptr)(lds + AT_Q + hh * TILE) + (r_at ^ (32 * s))));
      }
    };
    if constexpr (OUT) read_rows(0);
    __builtin_amdgcn_sched_barrier(0);
    if (chunk >= chunks) return;
    const float f0 = four[0], f1 = four[1];        // (a cast of a vector's element would be one of its first)
    const float f = __builtin_bit_cast(float, __builtin_amdgcn_readfirstlane(__builtin_bit_cast(int, f0)));
    if (f != 1.f && f1 == 0.f) multiply(f);
    const bool apart = __builtin_amdgcn_readfirstlane(__builtin_bit_cast(int, f1)) != 0;

    // ---- X^T = K Q^T: row q . k of keys 8 j + 4 h + i and query col; O^T = S^T Q^T. The state enters the product as bf16 (half a step, 2^-8 of
    // each number; the state itself stays as it is). The order of instructions is given (the compiler's own waits for every operand by itself): matrix
    // instructions alternate with what makes operands of the state and of V.
    bf16x8 W[3][2];
#pragma unroll
    for (int hh = 0; hh < HEADS; ++hh) {
      const bool to_state = hh == HEADS - 1;
      if (hh > 0) {
        read_rows(hh);
        __builtin_amdgcn_sched_barrier(0);
      }
      f32x16 X = {}, O = {};
      if constexpr (OUT) {
#pragma unroll
        for (int s = 0; s < KS; ++s) {
          X = __builtin_amdgcn_mfma_f32_32x32x16_bf16(K[s], Q[s], X, 0, 0, 0);
          u32x4 w;
#pragma unroll
          for (int e = 0; e < 4; ++e) w[e] = __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{S[s / 2][8 * (s % 2) + 2 * e], S[s / 2][8 * (s % 2) + 2 * e + 1]}), bf16x2));
          O = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, w), Q[s], O, 0, 0, 0);
        }
      }
      // V with its weights as the sum of three bf16 numbers, which hold an fp32's bits: the products enter the state as exactly as in fp32
      if (to_state)
#pragma unroll
      for (int s = 0; s < 2; ++s) {
        const u32x4 two = __builtin_bit_cast(u32x4, V[s]);
        u32x4 w[3];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          f32x2 x = {left[8 * s + 2 * e] * __builtin_bit_cast(float, two[e] << 16), left[8 * s + 2 * e + 1] * __builtin_bit_cast(float, two[e] & 0xffff0000u)};
#pragma unroll
          for (int i = 0; i < 3; ++i) {
            const uint32_t top2 = __builtin_bit_cast(uint32_t, __builtin_convertvector(x, bf16x2));
            w[i][e] = top2;
            x[0] -= __builtin_bit_cast(float, top2 << 16);
            x[1] -= __builtin_bit_cast(float, top2 & 0xffff0000u);
          }
        }
#pragma unroll
        for (int i = 0; i < 3; ++i) W[i][s] = __builtin_bit_cast(bf16x8, w[i]);
      }
      if (to_state)
#pragma unroll
      for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int s = 0; s < 2; ++s) T[2 * m + s] = transposed(lds, k_at, m, s);
      bool odd = false;
      if constexpr (OUT) {
        // Has the chunk a value that is infinite or no number? Rows before it do not see it, but 0 times it is not 0.
        float z = 0.f;
        const bf16x2 none = {(__bf16)0.f, (__bf16)0.f};
#pragma unroll
        for (int s = 0; s < 2; ++s)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const uint32_t two = __builtin_bit_cast(u32x4, V[s])[e];
            z = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, two), none, z, false);
          }
        odd = __builtin_amdgcn_ballot_w64(z != 0.f) != 0;
#pragma unroll
        for (int i = 0; i < 2 * KS; ++i) {
          __builtin_amdgcn_sched_group_barrier(0x8, 1, 0);
          __builtin_amdgcn_sched_group_barrier(0x2, 160 / (2 * KS), 0);
          __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
        }
        __builtin_amdgcn_sched_barrier(0);
      }
      // Where decays are strong, q . S may leave fp32's range though what they leave of it does not: then it is made from S 2^-32.
      float unscale = 1.f;
      if (apart) {
        if constexpr (OUT) {
          float z[2] = {0.f, 0.f};             // 0 times the products: 0, or no number
#pragma unroll
          for (int e = 0; e < 16; ++e) z[e % 2] = __builtin_fmaf(O[e], 0.f, z[e % 2]);
          if (__builtin_amdgcn_ballot_w64(z[0] + z[1] != 0.f) != 0) {
            unscale = 0x1p32f;
            int at = r_lane;
            asm("" : "+v"(at));
#pragma unroll
            for (int s = 0; s < KS; ++s) {
              u32x4 w;
#pragma unroll
              for (int e = 0; e < 4; ++e) w[e] = __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{S[s / 2][8 * (s % 2) + 2 * e] * 0x1p-32f, S[s / 2][8 * (s % 2) + 2 * e + 1] * 0x1p-32f}), bf16x2));
              const f32x16 zero = {};
              O = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, w), __builtin_bit_cast(bf16x8, *(lds_u32x4)((lds_ptr)(lds + AT_Q + hh * TILE) + (at ^ (32 * s)))), s ? O : zero, 0, 0, 0);
              __builtin_amdgcn_sched_barrier(0);         // (one operand's registers at a time)
            }
          }
        }
        if (to_state) multiply(f);
      }

      // ---- The state, and the weights of the chunk's rows, as bf16 (half a step, 2^-8 of each): none for keys behind the query, whatever their
      // product is. (Worked out without a look at `apart` and `odd`, and once more where one of them holds.)
      f32x16 R = O;
      auto weights = [&](const f32x16 &x, bf16x8 (&P)[2]) {
#pragma unroll
        for (int s = 0; s < 2; ++s) {
          u32x4 w;
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            f32x2 y;
#pragma unroll
            for (int i = 0; i < 2; ++i) {
              const int at = 8 * s + 2 * e + i, key = 8 * (at >> 2) + 4 * h + (at & 3);
              y[i] = key <= col ? x[at] : 0.f;
            }
            w[e] = __builtin_bit_cast(uint32_t, __builtin_convertvector(y, bf16x2));
          }
          P[s] = __builtin_bit_cast(bf16x8, w);
        }
      };
      if constexpr (OUT) {
        f32x16 x;
#pragma unroll
        for (int e = 0; e < 16; ++e) x[e] = X[e] * left[e];
        bf16x8 P[2];
        weights(x, P);
#pragma unroll
        for (int s = 0; s < 2; ++s) R = __builtin_amdgcn_mfma_f32_32x32x16_bf16(V[s], P[s], R, 0, 0, 0);
      }
      if (to_state)
#pragma unroll
      for (int s = 0; s < 2; ++s)
#pragma unroll
        for (int i = 2; i >= 0; --i)
#pragma unroll
          for (int m = 0; m < MT; ++m) S[m] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(T[2 * m + s], W[i][s], S[m], 0, 0, 0);
      if constexpr (OUT) {
#pragma unroll
        for (int i = 0; i < 6 * MT; ++i) {
          __builtin_amdgcn_sched_group_barrier(0x8, 1, 1);
          __builtin_amdgcn_sched_group_barrier(0x2, 48 / (4 * MT), 1);
        }
        __builtin_amdgcn_sched_barrier(0);
        if (apart || odd) {
          const float c = *(lds_f32)(mine + 4 * col), own = apart ? exp2_32((double)four[2] + c) * unscale : 1.f;
#pragma unroll
          for (int e = 0; e < 16; ++e) {
            const float pair = __builtin_amdgcn_exp2f(c - *(lds_f32)(mine + 4 * (8 * (e >> 2) + 4 * h + (e & 3))));
            R[e] = O[e] * own;
            X[e] *= apart ? pair : left[e];
          }
          bf16x8 P[2];
          weights(X, P);
#pragma unroll
          for (int s = 0; s < 2; ++s) {
            if (!odd) R = __builtin_amdgcn_mfma_f32_32x32x16_bf16(V[s], P[s], R, 0, 0, 0);
            for (int key = 0; key < (odd ? 16 : 0); ++key) {      // key by key, and a row is taken in only where it is seen
              u32x4 own_key;       // element e of the lane's eight: key 4 h + e % 4 + 8 (e / 4)
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                const int k0 = 4 * h + 2 * (e & 1) + 8 * (e >> 1);
                own_key[e] = (key == k0 ? 0xffffu : 0u) | (key == k0 + 1 ? 0xffff0000u : 0u);
              }
              const f32x16 zero = {};
              const f32x16 x = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, __builtin_bit_cast(u32x4, V[s]) & own_key),
                                                                       __builtin_bit_cast(bf16x8, __builtin_bit_cast(u32x4, P[s]) & own_key), zero, 0, 0, 0);
#pragma unroll
              for (int e = 0; e < 16; ++e) R[e] += 16 * s + key <= col ? x[e] : 0.f;
            }
          }
        }
      }
      if constexpr (OUT) {
        // Two stores or more, which `turn` counts. The lane has channels 8 j + 4 h + i; as bf16 the halves of the wave exchange some, so that each
        // has eight channels side by side.
#pragma unroll
        for (int e = 0; e < 16; ++e) R[e] *= own_factor;
        // (rows behind the last are behind the end that the stores are told)
        const int n = __builtin_amdgcn_readfirstlane(min(rows - chunk * C, C)), bytes = A.out_dtype == STS_F32 ? 4 : 2, pitch = A.Hq * D * bytes;
        const __amdgpu_buffer_rsrc_t to = __builtin_amdgcn_make_buffer_rsrc(static_cast<unsigned char *>(A.out) + (((int64_t)begin + chunk * C) * A.Hq + head + hh) * D * bytes, 0,
                                                                            (n - 1) * pitch + D * bytes, 0x00027000);
        const int at = col * pitch + 32 * wave * bytes;
        if (A.out_dtype == STS_F32) {
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const f32x4 o = {R[4 * j], R[4 * j + 1], R[4 * j + 2], R[4 * j + 3]};
            __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, o), to, at + 32 * j + 16 * h, 0, 0);
          }
        } else {
          u32x4 w[2];
#pragma unroll
          for (int j = 0; j < 2; ++j) {
#pragma unroll
            for (int i = 0; i < 2; ++i) {
              const uint32_t x = __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{R[8 * j + 2 * i], R[8 * j + 2 * i + 1]}), bf16x2));
              const uint32_t y = __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{R[8 * j + 4 + 2 * i], R[8 * j + 5 + 2 * i]}), bf16x2));
              const auto swapped = __builtin_amdgcn_permlane32_swap(x, y, false, false);
              w[j][i] = swapped[0];
              w[j][2 + i] = swapped[1];
            }
          }
          // At head size 64 the rows of 16 lanes do so, too: a store writes the wave's 64 bytes of 16 rows, not 32 of 32 (sixteen prompts 109.4 us without, 104.1
          // with; at head size 128, where more waves share a row, it makes no difference: 8192 rows 119 us without, 121 with, six prompts 90 and 89).
#pragma unroll
          for (int i = 0; D == 64 && i < 4; ++i) {
            const uint32_t x = w[0][i], y = w[1][i];
            const auto swapped = __builtin_amdgcn_permlane16_swap(x, y, false, false);
            w[0][i] = swapped[0];
            w[1][i] = swapped[1];
          }
#pragma unroll
          for (int j = 0; j < 2; ++j) __builtin_amdgcn_raw_buffer_store_b128(w[j], to, D == 64 ? (16 * j + (col & 15)) * pitch + 32 * wave * bytes + 2 * (col & 16) + 16 * h : at + 32 * j + 16 * h, 0, 0);
        }
      }
    }
  };
  work_out(0);
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");              // (no stores come behind the first loads)
  if (DEPTH == 3) load(1, lds_1);
  // (three chunks at a time, present or not: with more ways out of the loop than one the compiler would see ways back into it that there are not, and
  // wait for the loads of a chunk to come)
  for (int base = 0;;) {
    int i = 0;
    do {
      body(base + i, i, lds_0, DEPTH == 3 ? lds_2 : lds_1);
      body(base + i + 1, i + 1, lds_1, lds_0);
      if (DEPTH == 3) body(base + i + 2, i + 2, lds_2, lds_1);
      i += DEPTH;
    } while (i < BLOCK && base + i < chunks);
    base += BLOCK;
    if (base >= chunks) break;
    if (HEADS == 2) load_gates(base);      // (only now: it has no registers for them meanwhile, and rarely more than one block)
    all_waves();                           // (nobody reads the last block's decays any more)
    work_out(base);
  }
  multiply(exp2_32(low));

  if (!OUT && carried) {
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
      for (int e = 0; e < 4; ++e)
        *reinterpret_cast<f32x4 *>(A.part + part_at + p_at + (4 * m + e) * NW * 256) = f32x4{S[m][4 * e], S[m][4 * e + 1], S[m][4 * e + 2], S[m][4 * e + 3]};
    if (threadIdx.x == 0) A.part_log[part] = all;
    return;
  }
  if (!last || hd != 0) return;
  float *to = state_out(A, piece.b);
  if (!to) return;
  to += (size_t)g * D * D;
  const int again = __builtin_amdgcn_mbcnt_hi(~0u, __builtin_amdgcn_mbcnt_lo(~0u, 0u)), s_end = 8 * (again >> 5) * D + 32 * wave + (again & 31);      // (s_at, not kept in a register)
#pragma unroll
  for (int m = 0; m < MT; ++m)
#pragma unroll
    for (int e = 0; e < 16; ++e) to[s_end + (32 * m + 16 * (e >> 3) + (e & 7)) * D] = S[m][e];
}

// Along each sequence of several segments: the state before every segment takes the place of what the segment adds. A thread has four numbers, and asks for
// those of eight segments at once. Memory bounds it: 15 segments of 32 heads, 64 MB, 14 us (4.6 TB/s).
template <int D>
__global__ void __launch_bounds__(256) linear_carry_kernel(const LinearArgs A) {
  constexpr int PER = D * D / 1024;      // workgroups for a state
  const int unit = blockIdx.x / PER, q = (blockIdx.x % PER) * 256 + threadIdx.x, at = 4 * q, place = state_place<D>(q);
  const int b = A.by_heads.of(unit), g = unit - b * A.Hkv;
  int begin, len;
  seq_rows(A.seqs, b, begin, len);
  len = rows_of(A, b, len);
  // (what the sums' kernel leaves: the segments before the last, or all of a sequence with several of them where there are no results)
  const int segments = max((len + A.segment - 1) / A.segment, 1);
  if (segments < 2 && !(A.out && A.G > A.heads)) return;
  const int sums = A.out ? segments - 1 : segments;
  const float *from = state_in(A, b);
  f32x4 S = {0.f, 0.f, 0.f, 0.f};
  if (from) {
#pragma unroll
    for (int i = 0; i < 4; ++i) S[i] = from[(size_t)g * D * D + place + i * D];
  }
  const size_t first = ((size_t)A.by_segment.of(begin) + b) * A.Hkv + g;
  constexpr int AT_ONCE = 8;
  for (int i0 = 0; i0 < segments; i0 += AT_ONCE) {
    f32x4 own[AT_ONCE];
    float f[AT_ONCE];
#pragma unroll
    for (int i = 0; i < AT_ONCE; ++i) {
      const size_t part = first + (size_t)min(i0 + i, max(sums - 1, 0)) * A.Hkv;
      own[i] = i0 + i < sums ? *reinterpret_cast<const f32x4 *>(A.part + part * D * D + at) : f32x4{0.f, 0.f, 0.f, 0.f};
      f[i] = i0 + i < sums ? (float)exp2_64(A.part_log[part]) : 1.f;
    }
#pragma unroll
    for (int i = 0; i < AT_ONCE; ++i) {
      if (A.out && i0 + i < segments) *reinterpret_cast<f32x4 *>(A.part + (first + (size_t)(i0 + i) * A.Hkv) * D * D + at) = S;
      S = S * f[i] + own[i];
    }
  }
  if (A.out) return;
  float *to = state_out(A, b);
  if (!to) return;
#pragma unroll
  for (int i = 0; i < 4; ++i) to[(size_t)g * D * D + place + i * D] = S[i];
}

}  // namespace

hipError_t launch_linear_step(const LinearArgs &a, int d, hipStream_t s) {
  const dim3 grid((unsigned)((int64_t)a.seqs.B * a.Hkv * (d / 32))), block(256);
  // Several rows at once where a group has fewer than four heads: 16 rows of 64 sequences without groups take 89 us, row by row 137. One row takes more
  // registers then for nothing (54.5 us for those 53).
  const int at_once = a.max_len == 1 || a.G > 2 ? 1 : a.G == 2 ? 2 : 4;
  auto launch = [&](auto dim) {
    constexpr int D = decltype(dim)::value;
    if (at_once == 4) STS_LAUNCH((linear_step_kernel<D, 4>), grid, block, 0, s, a);
    else if (at_once == 2) STS_LAUNCH((linear_step_kernel<D, 2>), grid, block, 0, s, a);
    else STS_LAUNCH((linear_step_kernel<D, 1>), grid, block, 0, s, a);
  };
  if (d == 128) launch(std::integral_constant<int, 128>());
  else launch(std::integral_constant<int, 64>());
  return sts_take_launch_status();
}

template <int D, bool OUT, int HEADS>
static hipError_t launch_chunks(const LinearArgs &a, hipStream_t s) {
  const dim3 grid((unsigned)(((int64_t)a.numbers * a.Hkv + STS_XCDS - 1) / STS_XCDS * STS_XCDS * (OUT ? a.G / HEADS : 1))), block(2 * D);
  STS_LAUNCH((linear_chunk_kernel<D, OUT, HEADS>), grid, block, 0, s, a);
  return sts_take_launch_status();
}
hipError_t launch_linear_sums(const LinearArgs &a, int d, hipStream_t s) { return d == 128 ? launch_chunks<128, false, 1>(a, s) : launch_chunks<64, false, 1>(a, s); }
hipError_t launch_linear_chunks(const LinearArgs &a, int d, hipStream_t s) {
  if (a.heads == 2) return d == 128 ? launch_chunks<128, true, 2>(a, s) : launch_chunks<64, true, 2>(a, s);
  return d == 128 ? launch_chunks<128, true, 1>(a, s) : launch_chunks<64, true, 1>(a, s);
}

hipError_t launch_linear_carry(const LinearArgs &a, int d, hipStream_t s) {
  const dim3 grid((unsigned)((int64_t)a.seqs.B * a.Hkv * (d * d / 1024))), block(256);
  if (d == 128) STS_LAUNCH(linear_carry_kernel<128>, grid, block, 0, s, a);
  else STS_LAUNCH(linear_carry_kernel<64>, grid, block, 0, s, a);
  return sts_take_launch_status();
}
