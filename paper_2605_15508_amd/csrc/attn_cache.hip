// Split attention of short query blocks (up to 16 rows) over a cache of one of two forms (gfx950): held in 4 bits
// (sts_packed_attn: all tokens, or index lists), or bf16 with a sliding window and sinks (sts_window_attn).
//
// Units, splits and partials are those of the bf16 kernels (attn.hip), whose combine kernel merges the splits and appends
// the block's own tokens. A workgroup that has a unit whole appends them itself (64 sequences of 1500 tokens, 5 rows: 34 us, with the
// combine kernel 56). One workgroup of four waves per (batch, unit, split); waves take alternating tiles of 32 keys and keep an online
// softmax of their own, with maximum, sum and accumulators in fp32.
//
// Tiles in the transposed orientation, S^T = K Q^T and O^T += V^T P^T on v_mfma_f32_16x16x32_bf16, lane (a, b) =
// (lane / 16, lane % 16). Which key a row of K's operand holds is free, so row 4a + i of half h is the tile's key
// a + 4i + 16h. Then
//   - lane (a, b) ends up with the scores of keys a + 4m, m = 0..7, of query b, which is what it has to supply as the B
//     operand of the second product: P stays in its lane;
//   - V's rows for it are a + 4m, so that the four lane groups load four neighbouring rows at a time;
//   - K's operand is loaded as it is used, a lane's share of one key's row: no LDS, no exchange. Of a row of 4-bit codes
//     lane a has the a-th quarter, 16 bytes at head size 128 and one scale; of a bf16 row every fourth chunk of 16 bytes.
// S over 4-bit codes: v_mfma_scale_f32_16x16x128_f8f6f4 takes K's codes and scales as they lie in memory, a lane 32 channels of a key
// and their scale. Q, the other operand, is the sum of two e4m3 numbers, high and low, with a scale per 32 channels: four
// significant bits each hold the eight of a bf16 exactly for values of at least 2^-9 of their group's largest, and others to 2^-17
// of that largest (to 2^-136 where the scale is at its smallest).
// At head size 64 both halves go into one instruction, K's row taken twice.
// V's codes become bf16 pairs in the chip's conversion, scale included, exactly. The pairs are two channels of one key and have to
// become two keys of one channel: two byte permutes per pair of registers, as for bf16.
// Scales: a lane loads the word of one token of the tile, K's in the lower half of the wave, V's in the upper, and
// the lanes pick up those of their rows from LDS, one tile ahead of their use: bytes for K, the conversion's floats for V.
//
// What bounds it. 4 bits, 20 query rows on a KV head (128K tokens, batch 4): 571 MB in 107 us, 5.3 TB/s, vector instructions 65%
// and matrix instructions 31% of the time: converting V takes as many as the softmax does. 16 rows and fewer: memory (one row 4.2
// TB/s); 64 rows on a KV head are two units, each of which converts V (123 MB in 55 us; units of 64 rows do not fit the registers).
// Lists: rows of 136 bytes are a line of codes and a piece of one of scales (121 MB in 29 us). The bf16 window: memory (16
// sequences, window 4096: 269 MB in 45 us, 6.0 TB/s). Few keys: the chain length -> page -> row -> product -> merge, 6 to 9 us, and
// 3.5 to 5 of the combine kernel.
// Three tiles of 4 bits are on the way in each wave, of bf16 two at head size 64 and one at 128: so two workgroups fit a compute
// unit, one where there are few (with two tiles on the way one fits: 40 sequences of 5 rows, window 600 53 us, so 43; 16 of one
// row, window 4096 the same).
#include <float.h>

#include "attn_util.h"
#include "cache.h"

namespace {

// a lane's share of a row: K's quarter and V's D / 16 channels
template <int D, bool FOUR> struct Share;
template <> struct Share<128, true> { typedef u32x4 k; typedef uint32_t v; };
template <> struct Share<64, true> { typedef u32x4 k; typedef uint16_t v; };
template <> struct Share<128, false> { typedef u32x4 k; typedef u32x4 v; };
template <> struct Share<64, false> { typedef u32x4 k; typedef u32x2 v; };

// bits 0 .. n - 1 of a word, none for n <= 0
__device__ __forceinline__ uint32_t first_keys(int n) { return n <= 0 ? 0u : n >= 32 ? ~0u : (1u << n) - 1; }

template <int D, bool FOUR> constexpr int tiles_ahead() { return FOUR ? 3 : D == 128 ? 1 : 2; }

typedef int i32x8 __attribute__((ext_vector_type(8)));

// The larger magnitude of both halves of 8 words of bf16 pairs
__device__ __forceinline__ uint32_t largest(const uint32_t (&w)[8]) {
  typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
  u16x2 m = {0, 0};
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const uint32_t x = w[i] & 0x7fff7fffu;
    m = __builtin_elementwise_max(m, __builtin_bit_cast(u16x2, x));
  }
  const uint32_t lo = m[0], hi = m[1];
  return max(lo, hi);
}

// 16 bf16 values as e4m3 numbers hi + lo, each times 2^(s - 127); s puts a group's largest value, of magnitude bits m, at 2^7 ..
// 2^8 (255 for one that is no number, or infinite: the products are NaN then)
__device__ __forceinline__ uint32_t q_scale(uint32_t m) { return m >= 0x7f80u ? 255u : (uint32_t)max((int)(m >> 7) - 7, 1); }
__device__ __forceinline__ void q_halves(const uint32_t (&w)[8], uint32_t s, u32x4 &hi, u32x4 &lo) {
  typedef short s16x2 __attribute__((ext_vector_type(2)));
  const float f = __builtin_bit_cast(float, s << 23);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    s16x2 h = {0, 0}, l = {0, 0};
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const uint32_t x = w[2 * i + e];
      h = e ? __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(h, __builtin_bit_cast(bf16x2, x), f, true)
            : __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(h, __builtin_bit_cast(bf16x2, x), f, false);
      const f32x2 back = e ? __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(__builtin_bit_cast(uint32_t, h), f, true)
                           : __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(__builtin_bit_cast(uint32_t, h), f, false);
      const float r0 = __builtin_bit_cast(float, x << 16) - back[0], r1 = __builtin_bit_cast(float, x & 0xffff0000u) - back[1];
      l = e ? __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(l, r0, r1, f, true) : __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(l, r0, r1, f, false);
    }
    hi[i] = __builtin_bit_cast(uint32_t, h);
    lo[i] = __builtin_bit_cast(uint32_t, l);
  }
}

__device__ __forceinline__ f32x4 scaled_product(u32x4 codes, uint32_t k_scale, u32x4 q0, u32x4 q1, uint32_t q_scale, f32x4 c) {
  const i32x8 A = {(int)codes[0], (int)codes[1], (int)codes[2], (int)codes[3], 0, 0, 0, 0};
  const i32x8 B = {(int)q0[0], (int)q0[1], (int)q0[2], (int)q0[3], (int)q1[0], (int)q1[1], (int)q1[2], (int)q1[3]};
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(A, B, c, 4 /* e2m1 */, 0 /* e4m3 */, 0, (int)k_scale, 0, (int)q_scale);
}

__device__ __forceinline__ uint32_t pair_of(uint32_t codes, float scale, int byte) {
  switch (byte) {
    case 0: return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 0));
    case 1: return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 1));
    case 2: return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 2));
    default: return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 3));
  }
}

// FOUR: a 4-bit cache without a window, else a bf16 cache with one. GATHER: the rows come from a list or a page
// table, at offsets of 64 bits (FAR) or 32.
template <int D, int NQ, bool FOUR, bool GATHER, bool FAR>
__global__ void __launch_bounds__(64 * STS_WG_WAVES, 2) cache_attn_kernel(const CacheAttnArgs C) {
  typedef typename Share<D, FOUR>::k k_t;
  typedef typename Share<D, FOUR>::v v_t;
  typedef typename std::conditional<FAR, uint64_t, uint32_t>::type off_t;
  constexpr int W = STS_WG_WAVES, TK = STS_TILE_KEYS, PF = tiles_ahead<D, FOUR>();
  constexpr int NT = D / 16, KK = D / 32;
  constexpr int KL = FOUR ? 1 : KK;              // loads of K per lane and half tile
  constexpr int QR = FOUR ? D / 32 : KK;         // quads of registers of Q per lane and query tile: bf16, or halves in e4m3
  constexpr int OPITCH = D + 4;
  constexpr bool WIN = !FOUR;
  constexpr bool QLDS = NQ >= 2;
  __shared__ __attribute__((aligned(16))) float lds_o[W * 16 * OPITCH];
  __shared__ float lds_ml[W][NQ * 16][2];
  __shared__ __attribute__((aligned(16))) u32x4 lds_q[NQ * QR * 64];
  __shared__ uint32_t lds_qs[NQ][2][64];
  __shared__ __attribute__((aligned(16))) off_t lds_off[GATHER ? W : 1][2][TK];                // by (slot % 4) * 8 + slot / 4
  __shared__ __attribute__((aligned(16))) uint32_t lds_sc[FOUR ? W : 1][2][2][D / 32][TK];     // [tile parity][K, V][group], slots as above

  const AttnArgs &A = C.a;
  // what the first loads need of the arguments, asked for together: waits for scalar loads cannot tell them apart
  uint32_t unit = A.units.unit[blockIdx.y];
  asm volatile("" ::"s"(unit), "s"(A.q), "s"(A.indices), "s"(A.counts), "s"(A.seq_lens), "s"(A.idx_stride_b), "s"(A.cnt_stride_b), "s"(A.Tq), "s"(A.Hq),
               "s"(A.G), "s"(A.N), "s"(A.kmax), "s"(A.num_splits), "s"(A.z_rounds), "s"(A.page), "s"(A.page_shift), "s"(A.block_table), "s"(A.scale),
               "s"(A.scale_log2), "s"(C.tq_inv));
  if (FOUR) asm volatile("" ::"s"(C.codes), "s"(C.scales), "s"(C.code_b), "s"(C.code_h), "s"(C.code_n), "s"(C.scale_b), "s"(C.scale_h), "s"(C.scale_n));
  else asm volatile("" ::"s"(A.k), "s"(A.v), "s"(A.stride_b), "s"(A.stride_h), "s"(A.stride_n), "s"(C.window), "s"(C.sinks), "s"(C.behind));
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const int a = lane >> 4, b = lane & 15;
  const int S = A.num_splits, U = A.num_units;
  int split = blockIdx.x, bt = blockIdx.z;
  const int u = blockIdx.y;
  if (A.z_rounds > 1) {                 // more batch elements than a grid's last dimension holds
    bt += split / S * STS_GRID_Z;
    split %= S;
    if (bt >= A.B) return;
  }
  const int g = unit & 0xff;
  const uint32_t mask = (unit >> 8) & 0xffff;
  const int nheads = (unit >> 24) & 0x1f;
  const int rows_valid = nheads * A.Tq;
  const int head0 = g * A.G + __builtin_ctz(mask);
  const int psh = A.page_shift, pmask = A.page - 1;
  const bool list = GATHER && A.indices != nullptr, paged = GATHER && A.block_table != nullptr;

  // ---- the keys of this unit: positions 0 .. c - 1 of its list (or of the cache), and which tiles of 32 are looked at
  const int32_t *len_src = list ? (A.counts ? A.counts + (int64_t)bt * A.cnt_stride_b + head0 : nullptr) : (A.seq_lens ? A.seq_lens + bt : nullptr);
  const int n_max = list ? A.kmax : A.N;
  const int c = (len_src ? min(max(*len_src, 0), n_max) : n_max) << (list ? psh : 0);
  const int tiles_end = (c + TK - 1) / TK;
  // a window: tiles of sinks, then those from row 0's first key in the window on
  const int p0 = WIN ? (C.behind ? c : c - A.Tq) : 0;
  const int lo = WIN ? max(0, (int)max((int64_t)p0 - C.window + 1, (int64_t)0)) : 0;
  const int sink_tiles = WIN ? min((min(C.sinks, c) + TK - 1) / TK, lo / TK) : 0;
  const int skipped = WIN ? lo / TK - sink_tiles : 0;
  const int tiles = max(tiles_end - skipped, 0);
  const int tps = (tiles + S - 1) / S;
  const int t_begin = split * tps, t_end = min(t_begin + tps, tiles);
  const int nv = t_end - t_begin > wave ? (t_end - t_begin - wave + W - 1) / W : 0;       // tiles of this wave
  auto tile_of = [&](int v) { return min(t_begin + wave + v * W, t_end - 1); };           // past the last, the last again
  auto first_of = [&](int t) { return (WIN && t >= sink_tiles ? t + skipped : t) * TK; };   // position of a tile's first key

  // ---- query rows of this lane: row nq * 16 + b. A negative scale turns the signs of Q, a scale of 0 clears it.
  const uint32_t q_keep = A.scale == 0.f ? 0u : 0xffffffffu, q_flip = A.scale < 0.f ? 0x80008000u : 0u;
  const float sl2 = A.scale == 0.f ? 1.f : fabsf(A.scale_log2);
  u32x4 Q[QLDS ? 1 : NQ][QLDS ? 1 : QR];
  uint32_t qs[NQ];
  int q_tq[NQ];
  auto row_of_lane = [&](int nq, bool &ok, int &hsel) {
    const int r = nq * 16 + b;
    ok = r < rows_valid;
    hsel = ok ? (r * C.tq_inv) >> 16 : 0;              // r / Tq
    q_tq[nq] = ok ? r - hsel * A.Tq : 0;
  };
  auto take_q = [&] {
    // The work is divided among the waves, which find the operands in LDS.
    constexpr int PARTS = FOUR ? D / 64 : 1;
#pragma unroll
    for (int nq = 0; nq < NQ; ++nq) {
      bool ok;
      int hsel;
      row_of_lane(nq, ok, hsel);
#pragma unroll
      for (int j = 0; j < PARTS; ++j) {
        if (wave != (nq * PARTS + j) % W) continue;
        const uint16_t *qp = A.q + (((size_t)bt * A.Tq + q_tq[nq]) * A.Hq + g * A.G + nth_member(mask, hsel)) * D;
        auto get = [&](int chan) { return (*reinterpret_cast<const u32x4 *>(qp + chan) & (ok ? q_keep : 0u)) ^ q_flip; };
        if constexpr (FOUR) {
          // Channels 16 a .. of the first 64 (j = 0) or of the rest: the first or the second half of the operand. A group of 32 channels
          // is in two neighbouring lane groups.
          const u32x4 w0 = get(64 * j + 16 * a), w1 = get(64 * j + 16 * a + 8);
          const uint32_t w[8] = {w0[0], w0[1], w0[2], w0[3], w1[0], w1[1], w1[2], w1[3]};
          uint32_t m = largest(w);
          m = max(m, (uint32_t)__shfl_xor((int)m, 16, 64));
          const uint32_t s = q_scale(m);
          u32x4 hi, lo;
          q_halves(w, s, hi, lo);
          lds_q[(nq * QR + (D == 128 ? j : 0)) * 64 + lane] = hi;
          lds_q[(nq * QR + (D == 128 ? 2 + j : 1)) * 64 + lane] = lo;
          lds_qs[nq][j][lane] = s;
        } else {
#pragma unroll
          for (int kk = 0; kk < KK; ++kk) lds_q[(nq * QR + kk) * 64 + lane] = get(8 * (a + 4 * kk));
        }
      }
    }
    __syncthreads();
    // (the scale of a group goes to the lane group that has K's share of it)
    if (FOUR)
#pragma unroll
      for (int nq = 0; nq < NQ; ++nq) qs[nq] = lds_qs[nq][D == 128 ? a >> 1 : 0][(a & 1) * 32 + b];
    if (!QLDS)
#pragma unroll
      for (int i = 0; i < QR; ++i) Q[0][QLDS ? 0 : i] = lds_q[i * 64 + lane];
  };

  float m_run[NQ], l_run[NQ];
  f32x4 acc[NQ][NT];
#pragma unroll
  for (int nq = 0; nq < NQ; ++nq) {
    m_run[nq] = -INFINITY;
    l_run[nq] = 0.f;
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) acc[nq][nt] = f32x4{0.f, 0.f, 0.f, 0.f};
  }

  // ---- loads
  struct Tile {
    k_t k[2][KL];
    v_t v[8];
    uint32_t sc;
  };
  const int64_t row_bytes = FOUR ? C.code_n : A.stride_n * 2, page_bytes = FOUR ? C.code_page : A.stride_page * 2;
  const int64_t head_off = FOUR ? (paged ? 0 : bt * C.code_b) + g * C.code_h : ((paged ? 0 : bt * A.stride_b) + g * A.stride_h) * 2;
  const unsigned char *kuni = (FOUR ? C.codes : reinterpret_cast<const unsigned char *>(A.k)) + head_off;
  const unsigned char *vuni = (FOUR ? C.codes + D / 2 : reinterpret_cast<const unsigned char *>(A.v)) + head_off;
  const unsigned char *suni = FOUR ? C.scales + (paged ? 0 : bt * C.scale_b) + g * C.scale_h : nullptr;
  constexpr int VCH = FOUR ? D / 32 : D / 8;      // bytes of a lane's chunk of V
  const int k_chunk = FOUR && D == 64 ? (a & 1) * 16 : a * 16;
  const int slot = lane & 31, slot_at = (slot & 3) * 8 + (slot >> 2);
  const int k_slot = (b >> 2) + 4 * (b & 3), k_at = (b >> 2) * 8 + (b & 3);
  const uint32_t half = FOUR && D == 128 ? (lane >> 5) * 4 : 0;            // K's or V's word of a token's scales

  auto load_k = [&](const unsigned char *base, off_t off, k_t (&k)[KL]) {
#pragma unroll
    for (int j = 0; j < KL; ++j) k[j] = *reinterpret_cast<const k_t *>(base + (off + (off_t)(64 * j)));
  };
  // (V of a bf16 cache past the caches, where K's halves of a line meet: 16 sequences, window 4096, 55.4 us without, 49.3 so)
  auto load_v = [&](const unsigned char *base, off_t off) {
    const v_t *src = reinterpret_cast<const v_t *>(base + off);
    return FOUR ? *src : __builtin_nontemporal_load(src);
  };

  // contiguous: offsets of the lane's rows in a tile, which a tile's end and gap move to rows that are attended to (their weight is 0,
  // but 0 times what lies there may be NaN)
  uint32_t k_off[2], v_off[8];
  if (!GATHER) {
#pragma unroll
    for (int h = 0; h < 2; ++h) k_off[h] = (uint32_t)((k_slot + 16 * h) * (int)row_bytes + k_chunk);
#pragma unroll
    for (int m = 0; m < 8; ++m) v_off[m] = (uint32_t)((a + 4 * m) * (int)row_bytes + b * VCH);
  }
  auto seen_row = [&](int n) { return WIN && n >= C.sinks && n < lo ? lo : n; };
  auto issue_near = [&](int t, Tile &R) {
    const int n0 = first_of(t);
    // (the scales first: they are waited for a tile before the rest)
    if (FOUR) R.sc = *reinterpret_cast<const uint32_t *>(suni + n0 * C.scale_n + (min(slot, c - 1 - n0) * (int)C.scale_n + (int)half));
    const unsigned char *kb = kuni + n0 * row_bytes, *vb = vuni + n0 * row_bytes;
    if (WIN && n0 < lo) {               // tiles of sinks, and the one that the window begins in
#pragma unroll
      for (int h = 0; h < 2; ++h) load_k(kuni + min(seen_row(n0 + k_slot + 16 * h), c - 1) * row_bytes, (off_t)k_chunk, R.k[h]);
#pragma unroll
      for (int m = 0; m < 8; ++m) R.v[m] = load_v(vuni + min(seen_row(n0 + a + 4 * m), c - 1) * row_bytes, (off_t)(b * VCH));
    } else {
      const uint32_t last = (uint32_t)(min(c - 1 - n0, TK - 1) * (int)row_bytes), last_k = last + k_chunk, last_v = last + b * VCH;
#pragma unroll
      for (int h = 0; h < 2; ++h) load_k(kb, (off_t)min(k_off[h], last_k), R.k[h]);
#pragma unroll
      for (int m = 0; m < 8; ++m) R.v[m] = load_v(vb, (off_t)min(v_off[m], last_v));
    }
  };

  // gather: list entry (or block) -> page -> offset, each a step of its own
  const int32_t *idx_row = list ? A.indices + (size_t)bt * A.idx_stride_b + (size_t)head0 * A.kmax : nullptr;
  const int32_t *table_row = paged ? A.block_table + (size_t)bt * A.table_stride : nullptr;
  const int nb_max = (A.N + A.page - 1) >> psh;
  auto fetch = [&](int t) -> int {      // entry of this lane's slot of tile t
    const int pos = min(seen_row(first_of(t) + slot), c - 1) >> psh;
    return list ? idx_row[pos] : pos;
  };
  auto block_of = [&](int entry) { return min(max(entry, 0), nb_max - 1); };
  auto look_up = [&](int blk) { return paged ? table_row[blk] : blk; };
  off_t scale_off = 0;
  auto place = [&](int blk, int page, int t, int par, uint32_t &tile_mask) {
    const int pos = first_of(t) + slot, in_page = min(seen_row(pos), c - 1) & pmask, tok = (blk << psh) + in_page;
    // (of a block that the cache's end cuts, the rows behind it read the cache's last row, which is in the block)
    const int over = max(tok - (A.N - 1), 0), at = paged ? in_page - over : tok - over;
    if (!WIN) tile_mask = (uint32_t)__ballot(pos < c && over == 0);
    const int64_t pg = paged ? (int64_t)min(max(page, 0), A.num_pages - 1) : 0;
    lds_off[GATHER ? wave : 0][par][slot_at] = (off_t)((FAR ? pg * page_bytes : 0) + at * row_bytes);
    if (FOUR) scale_off = (off_t)((FAR ? pg * C.scale_page : 0) + at * C.scale_n) + (off_t)half;
  };
  auto issue_far = [&](int par, Tile &R) {
    off_t ko[2], vo[8];
    if (FOUR) R.sc = *reinterpret_cast<const uint32_t *>(suni + scale_off);
#pragma unroll
    for (int h = 0; h < 2; ++h) ko[h] = lds_off[GATHER ? wave : 0][par][k_at + 4 * h];
#pragma unroll
    for (int m = 0; m < 8; ++m) vo[m] = lds_off[GATHER ? wave : 0][par][a * 8 + m];
#pragma unroll
    for (int h = 0; h < 2; ++h) load_k(kuni, ko[h] + (off_t)k_chunk, R.k[h]);
#pragma unroll
    for (int m = 0; m < 8; ++m) R.v[m] = load_v(vuni, vo[m] + (off_t)(b * VCH));
  };

  // ---- scales of one tile: own token's word -> LDS -> the two of K's rows and the eight of V's
  uint32_t ks[2], vs[8];
  auto put_scales = [&](uint32_t w, int par) {
    if constexpr (FOUR) {
      const int kv = D == 128 ? lane >> 5 : 0, up = kv ? 23 : 0;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const uint32_t s = (w >> (8 * j)) & 255u;
        if (D == 128) lds_sc[wave][par][kv][j & (D / 32 - 1)][slot_at] = s << up;
        else lds_sc[wave][par][j >> 1][j & 1][slot_at] = j >= 2 ? s << 23 : s;
      }
    }
  };
  auto get_scales = [&](int par) {
    if constexpr (FOUR) {
#pragma unroll
      for (int h = 0; h < 2; ++h) ks[h] = lds_sc[wave][par][0][a & (D / 32 - 1)][k_at + 4 * h];
#pragma unroll
      for (int m = 0; m < 8; ++m) vs[m] = lds_sc[wave][par][1][b * (D / 32) / 16][a * 8 + m];
    }
  };

  // ---- one tile
  // S^T = K Q^T
  // (Q's first quads are read from LDS while the tile before is worked on)
  u32x4 q_next[2];
  auto next_q = [&] {
    if (FOUR && QLDS) {
      q_next[0] = lds_q[lane];
      q_next[1] = lds_q[64 + lane];
    }
  };
  auto scores = [&](const Tile &R, f32x4 (&St)[NQ][2]) {
    const f32x4 zero = {0.f, 0.f, 0.f, 0.f};
    auto q_at = [&](int nq, int i) { return QLDS ? lds_q[(nq * QR + i) * 64 + lane] : Q[QLDS ? 0 : nq][QLDS ? 0 : i]; };
    if constexpr (FOUR) {
#pragma unroll
      for (int j = 0; j < NQ; ++j) {
        const u32x4 q0 = QLDS && j == 0 ? q_next[0] : q_at(j, 0), q1 = QLDS && j == 0 ? q_next[1] : q_at(j, 1);
        const uint32_t s = qs[j];
        f32x4 x[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) x[h] = scaled_product(R.k[h][0], ks[h], q0, q1, s, zero);
        if constexpr (D == 128) {
          const u32x4 l0 = q_at(j, 2), l1 = q_at(j, 3);
#pragma unroll
          for (int h = 0; h < 2; ++h) St[j][h] = scaled_product(R.k[h][0], ks[h], l0, l1, s, x[h]);
          // The instruction takes eight passes: a result in registers that are partly an operand's would be wrong, and the compiler
          // sees to that for larger results only. So all operands are in use until the results are there.
          asm volatile("" ::"v"(St[j][0]), "v"(St[j][1]), "v"(x[0]), "v"(x[1]), "v"(q0), "v"(q1), "v"(l0), "v"(l1), "v"(R.k[0][0]), "v"(R.k[1][0]),
                       "v"(ks[0]), "v"(ks[1]), "v"(s));
        } else {
          St[j][0] = x[0];
          St[j][1] = x[1];
          asm volatile("" ::"v"(x[0]), "v"(x[1]), "v"(q0), "v"(q1), "v"(R.k[0][0]), "v"(R.k[1][0]), "v"(ks[0]), "v"(ks[1]), "v"(s));
        }
      }
    } else {
#pragma unroll
      for (int kk = 0; kk < KK; ++kk)
#pragma unroll
        for (int j = 0; j < NQ; ++j) {
          const u32x4 Qb = q_at(j, kk);
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            const u32x4 Ka = R.k[h][FOUR ? 0 : kk];
            St[j][h] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, Ka), __builtin_bit_cast(bf16x8, Qb), kk ? St[j][h] : zero, 0, 0, 0);
          }
        }
    }
  };
  // a window: which of the keys from n0 on query row q_tq[nq] sees: those up to it, without those between the sinks and its window
  auto seen_keys = [&](int n0, int nq) {
    const int p = p0 + q_tq[nq];
    return first_keys(min(p + 1, c) - n0) & (first_keys(C.sinks - n0) | ~first_keys((int)max((int64_t)p - C.window + 1, (int64_t)0) - n0));
  };
  // ... and whether some row does not see some of them
  auto partly_seen = [&](int n0) {
    return !(n0 + TK <= c && n0 + TK - 1 <= p0 && (n0 + TK <= C.sinks || p0 + A.Tq - 1 - n0 < C.window));
  };
  // keys that a row does not see score -inf
  auto hide = [&](int n0, uint32_t tile_mask, f32x4 (&St)[NQ][2]) {
#pragma unroll
    for (int j = 0; j < NQ; ++j) {
      const int mine = (int)((WIN ? seen_keys(n0, j) : tile_mask) >> a);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const uint32_t keep = (uint32_t)__builtin_amdgcn_sbfe(mine, 4 * i, 1);
        const float x = St[j][i >> 2][i & 3];
        St[j][i >> 2][i & 3] = __builtin_bit_cast(float, (__builtin_bit_cast(uint32_t, x) & keep) | (0xff800000u & ~keep));
      }
    }
  };
  // the weights exp(S - m) as the B operand of the second product: bf16 (half a step, 2^-8 of each); their sums in fp32
  auto weights = [&](const f32x4 (&St)[NQ][2], u32x4 (&P)[NQ]) {
#pragma unroll
    for (int j = 0; j < NQ; ++j) {
      const float m_ref = WIN && m_run[j] == -INFINITY ? 0.f : m_run[j];
      float p[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) p[i] = __builtin_amdgcn_exp2f(__builtin_fmaf(St[j][i >> 2][i & 3], sl2, -m_ref));
      l_run[j] += ((p[0] + p[1]) + (p[2] + p[3])) + ((p[4] + p[5]) + (p[6] + p[7]));
#pragma unroll
      for (int i = 0; i < 4; ++i) P[j][i] = __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{p[2 * i], p[2 * i + 1]}), bf16x2));
    }
  };
  // pair j of channels of the lane's 8 keys, and of those the keys of channel 2 j (hi: 2 j + 1) as pairs
  auto v_pairs = [&](const Tile &R, int j, uint32_t (&w)[8]) {
#pragma unroll
    for (int m = 0; m < 8; ++m) {
      if constexpr (FOUR) w[m] = pair_of(R.v[m], __builtin_bit_cast(float, vs[m]), j);
      else w[m] = R.v[m][j];
    }
  };
  auto v_keys = [&](const uint32_t (&w)[8], bool hi) {
    u32x4 x;
#pragma unroll
    for (int j = 0; j < 4; ++j) x[j] = __builtin_amdgcn_perm(w[2 * j + 1], w[2 * j], hi ? 0x07060302u : 0x05040100u);
    return x;
  };
  // values of the tile that are no numbers, or infinite: 0 times them is not 0
  auto odd_values = [&](const Tile &R) {
    float z = 0.f;
    if constexpr (!FOUR) {
      const bf16x2 none = {(__bf16)0.f, (__bf16)0.f};
#pragma unroll
      for (int m = 0; m < 8; ++m)
#pragma unroll
        for (int j = 0; j < NT / 2; ++j) {
          const uint32_t x = R.v[m][j];
          z = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, x), none, z, false);
        }
    }
    return __builtin_amdgcn_ballot_w64(z != 0.f) != 0;
  };
  bool later = false;              // tiles left for the end: see below
  auto consume = [&](const Tile &R, int t, uint32_t tile_mask) {
    const int n0 = first_of(t);
    f32x4 St[NQ][2];
    scores(R, St);
    // (V's conversions do not move up here, where their results would take the registers of the tiles on the way)
    if (FOUR && NQ >= 2) __builtin_amdgcn_sched_barrier(0);
    bool odd = false;
    if (WIN ? partly_seen(n0) : tile_mask != 0xffffffffu) {
      hide(n0, tile_mask, St);
      if (WIN) odd = odd_values(R);
    }
    // Most tiles of a long list raise no row's maximum: it is put together from the four lanes of a row only where one of them does.
    float mine[NQ];
    bool grown = false;
#pragma unroll
    for (int j = 0; j < NQ; ++j) {
      const f32x4 s0 = St[j][0], s1 = St[j][1];
      mine[j] = sl2 * top(top(top(s0[0], s0[1]), top(s0[2], s0[3])), top(top(s1[0], s1[1]), top(s1[2], s1[3])));
      grown |= mine[j] > m_run[j];
    }
    if (__builtin_amdgcn_ballot_w64(grown) != 0) {
#pragma unroll
      for (int j = 0; j < NQ; ++j) {
        const float m_new = larger(m_run[j], max_over_groups(mine[j]));
        const float alpha = m_new == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m_run[j] - m_new);
        l_run[j] *= alpha;
        m_run[j] = m_new;
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) acc[j][nt] *= alpha;
      }
    }
    later |= odd;
    if (!odd) {
      u32x4 P[NQ];
      weights(St, P);
#pragma unroll
      for (int j = 0; j < NT / 2; ++j) {
        uint32_t w[8];
        v_pairs(R, j, w);
#pragma unroll
        for (int hi = 0; hi < 2; ++hi) {
          const bf16x8 Va = __builtin_bit_cast(bf16x8, v_keys(w, hi));
#pragma unroll
          for (int nq = 0; nq < NQ; ++nq)
            acc[nq][2 * j + hi] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(Va, __builtin_bit_cast(bf16x8, P[nq]), acc[nq][2 * j + hi], 0, 0, 0);
        }
      }
    }
  };

  // ---- main loop: PF tiles on the way, each asked for again when it has been used. One exit, and code of its own for what is left
  // over, so that the loop's head knows which loads are in flight. Q comes while the first tiles are on their way.
  // GATHER: a list entry is fetched 3 PF tiles ahead of its use, its page looked up 2 PF ahead, the offset placed PF + 1 ahead.
  Tile R[PF];
  uint32_t seen[PF], next_seen = 0;
  int entry[PF], blk[PF], page[PF];
  if (nv > 0) {
    if constexpr (!GATHER) {
#pragma unroll
      for (int j = 0; j < PF; ++j) issue_near(tile_of(j), R[j]);
    } else {
      int e0[PF + 1], pg0[PF + 1];
#pragma unroll
      for (int j = 0; j <= PF; ++j) e0[j] = fetch(tile_of(j));
#pragma unroll
      for (int j = 0; j < PF; ++j) blk[(j + 1) % PF] = fetch(tile_of(PF + 1 + j));
#pragma unroll
      for (int j = 0; j < PF; ++j) entry[(j + 1) % PF] = fetch(tile_of(2 * PF + 1 + j));
#pragma unroll
      for (int j = 0; j <= PF; ++j) e0[j] = block_of(e0[j]), pg0[j] = look_up(e0[j]);
#pragma unroll
      for (int j = 0; j < PF; ++j) blk[j] = block_of(blk[j]), page[j] = look_up(blk[j]);
#pragma unroll
      for (int j = 0; j <= PF; ++j) {
        place(e0[j], pg0[j], tile_of(j), j & 1, next_seen);
        if (j < PF) {
          issue_far(j & 1, R[j]);
          seen[j] = next_seen;
        }
      }
    }
    __builtin_amdgcn_sched_barrier(0);
  }
  take_q();
  if (nv > 0) {
    put_scales(R[0].sc, 0);
    get_scales(0);
    next_q();
    auto step = [&](int v, int j, bool more) {
      const int t = tile_of(v), n = (j + 1) % PF, left = c - first_of(t);
      put_scales(R[n].sc, (v + 1) & 1);
      consume(R[j], t, GATHER ? seen[j] : left >= TK ? 0xffffffffu : (1u << left) - 1u);
      get_scales((v + 1) & 1);
      next_q();
      if (more) {
        if constexpr (!GATHER) {
          issue_near(tile_of(v + PF), R[j]);
        } else {
          issue_far((v + PF) & 1, R[j]);
          seen[j] = next_seen;
          __builtin_amdgcn_sched_barrier(0);
          place(blk[n], page[n], tile_of(v + PF + 1), (v + PF + 1) & 1, next_seen);
          blk[n] = block_of(entry[n]);
          page[n] = look_up(blk[n]);
          entry[n] = fetch(tile_of(v + 3 * PF + 1));
        }
      }
      __builtin_amdgcn_sched_barrier(0);
    };
    int v = 0;
    for (; v + PF <= nv; v += PF) {
#pragma unroll
      for (int j = 0; j < PF; ++j) step(v + j, j, true);
    }
#pragma unroll
    for (int j = 0; j < PF - 1; ++j)
      if (v + j < nv) step(v + j, j, false);
    if constexpr (WIN) {
      // What is infinite or no number must not reach the rows that do not see it: such tiles come last, key by key, and a key's
      // row of V is taken in only where it is seen.
      if (later) {
        for (v = 0; v < nv; ++v) {
          const int t = tile_of(v), n0 = first_of(t);
          if (!partly_seen(n0)) continue;
          if constexpr (GATHER) {
            const int e = block_of(fetch(t));
            place(e, look_up(e), t, 0, next_seen);
            issue_far(0, R[0]);
          } else {
            issue_near(t, R[0]);
          }
          if (!odd_values(R[0])) continue;
          f32x4 St[NQ][2];
          u32x4 P[NQ];
          scores(R[0], St);
          hide(n0, 0u, St);
          weights(St, P);
          for (int key = 0; key < TK; ++key) {
            u32x4 own;
#pragma unroll
            for (int i = 0; i < 4; ++i) own[i] = (a + 8 * i == key ? 0xffffu : 0u) | (a + 8 * i + 4 == key ? 0xffff0000u : 0u);
#pragma unroll
            for (int nq = 0; nq < NQ; ++nq) {
              const bool see = (seen_keys(n0, nq) >> key) & 1u;
#pragma unroll
              for (int nt = 0; nt < NT; ++nt) {
                uint32_t w[8];
                v_pairs(R[0], nt >> 1, w);
                const f32x4 zero = {0.f, 0.f, 0.f, 0.f};
                const f32x4 x = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, v_keys(w, nt & 1) & own),
                                                                        __builtin_bit_cast(bf16x8, P[nq] & own), zero, 0, 0, 0);
#pragma unroll
                for (int r = 0; r < 4; ++r) acc[nq][nt][r] += see ? x[r] : 0.f;
              }
            }
          }
        }
      }
    }
  }

  // ---- the waves are merged, the workgroup's partial is written (or the result, where nothing is left to be merged)
#pragma unroll
  for (int nq = 0; nq < NQ; ++nq) {
    float l = l_run[nq];
    l += __shfl_xor(l, 16, 64);
    l += __shfl_xor(l, 32, 64);
    if (a == 0) {
      // (scores that are no numbers raise no maximum: without one the part would be taken for an empty one)
      lds_ml[wave][nq * 16 + b][0] = l != l ? top(m_run[nq], -FLT_MAX) : m_run[nq];
      lds_ml[wave][nq * 16 + b][1] = l;
    }
  }
  __syncthreads();
  const size_t part = ((size_t)bt * U + u) * S + split;
  float *po = A.part_o + part * (size_t)(NQ * 16 * D), *pml = A.part_ml + part * (size_t)(NQ * 16 * 2);
#pragma unroll
  for (int nq = 0; nq < NQ; ++nq) {
    auto top_of = [&](int r) {
      float m = -INFINITY;
#pragma unroll
      for (int w = 0; w < W; ++w) m = fmaxf(m, lds_ml[w][r][0]);
      return m;
    };
    const float m_all = top_of(nq * 16 + b);
    const float f = m_run[nq] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m_run[nq] - m_all);
    float *orow = lds_o + (wave * 16 + b) * OPITCH;
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
      for (int v4 = 0; v4 < NT / 4; ++v4) {
        f32x4 o;
#pragma unroll
        for (int e = 0; e < 4; ++e) o[e] = acc[nq][4 * v4 + e][r] * f;
        *reinterpret_cast<f32x4 *>(orow + NT * (4 * a + r) + 4 * v4) = o;
      }
    __syncthreads();
    constexpr int SEGF = D / 16, OWN = 4;
    typedef typename std::conditional<D == 128, u32x4, u32x2>::type seg_t;
    auto widen = [](const uint16_t *from, float (&to)[SEGF]) {
      const seg_t w = *reinterpret_cast<const seg_t *>(from);
#pragma unroll
      for (int e = 0; e < SEGF; ++e) to[e] = __builtin_bit_cast(float, e & 1 ? w[e >> 1] & 0xffff0000u : w[e >> 1] << 16);
    };
    const int row = threadIdx.x >> 4, seg = threadIdx.x & 15, r = nq * 16 + row;
    float sum[SEGF];
#pragma unroll
    for (int e = 0; e < SEGF; ++e) sum[e] = 0.f;
#pragma unroll
    for (int w = 0; w < W; ++w)
#pragma unroll
      for (int e = 0; e < SEGF; e += 4) {
        const f32x4 x = *reinterpret_cast<const f32x4 *>(lds_o + (w * 16 + row) * OPITCH + seg * SEGF + e);
#pragma unroll
        for (int i = 0; i < 4; ++i) sum[e + i] += x[i];
      }
    const float m = top_of(r);
    float L = 0.f;
#pragma unroll
    for (int w = 0; w < W; ++w) {
      const float mw = lds_ml[w][r][0];
      L += mw == -INFINITY ? 0.f : lds_ml[w][r][1] * __builtin_amdgcn_exp2f(mw - m);
    }
    if (!A.direct) {
#pragma unroll
      for (int e = 0; e < SEGF; e += 4) *reinterpret_cast<f32x4 *>(po + (size_t)r * D + seg * SEGF + e) = f32x4{sum[e], sum[e + 1], sum[e + 2], sum[e + 3]};
      if (seg == 0) *reinterpret_cast<f32x2 *>(pml + r * 2) = f32x2{m, L};
    } else if (r < rows_valid) {
      const int hsel = (r * C.tq_inv) >> 16, tq = r - hsel * A.Tq, head = g * A.G + nth_member(mask, hsel);
      const size_t at = (((size_t)bt * A.Tq + tq) * A.Hq + head) * D + seg * SEGF;
      float m_all = m;
      if (A.k_new) {
        // The block's own tokens 0 .. tq (all of them, if not causal), in order, each like one more part; the 16 threads of a row have
        // D / 16 channels each.
        const int mine = A.causal ? tq + 1 : A.Tq;
        float q[SEGF], k[SEGF], v[SEGF];
        widen(A.q + at, q);
        for (int j0 = 0; j0 < A.Tq; j0 += OWN) {
          seg_t kw[OWN], vw[OWN];
#pragma unroll
          for (int j = 0; j < OWN; ++j) {
            const size_t from = (((size_t)bt * A.Tq + min(j0 + j, A.Tq - 1)) * A.Hkv + g) * D + seg * SEGF;
            kw[j] = *reinterpret_cast<const seg_t *>(A.k_new + from);
            vw[j] = *reinterpret_cast<const seg_t *>(A.v_new + from);
          }
#pragma unroll
          for (int j = 0; j < OWN; ++j) {
            widen(reinterpret_cast<const uint16_t *>(&kw[j]), k);
            widen(reinterpret_cast<const uint16_t *>(&vw[j]), v);
            float dot = 0.f;
#pragma unroll
            for (int e = 0; e < SEGF; ++e) dot += q[e] * k[e];
            const float s = row_sum16(dot) * A.scale_log2;
            merge_part(m_all, L, sum, j0 + j < mine ? s : -INFINITY, 1.f, v);
          }
        }
      }
      const float inv = L == 0.f ? 0.f : 1.f / L;
#pragma unroll
      for (int e = 0; e < SEGF; e += 4) {
        const f32x4 x = f32x4{sum[e], sum[e + 1], sum[e + 2], sum[e + 3]} * inv;
        if (A.out_dtype == STS_F32) {
          *reinterpret_cast<f32x4 *>(static_cast<float *>(A.out) + at + e) = x;
        } else {
          const u32x2 w = {__builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{x[0], x[1]}), bf16x2)),
                           __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{x[2], x[3]}), bf16x2))};
          *reinterpret_cast<u32x2 *>(static_cast<uint16_t *>(A.out) + at + e) = w;
        }
      }
      if (A.lse_out && seg == 0)
        A.lse_out[((size_t)bt * A.Hq + head) * A.Tq + tq] = L > 0.f ? (m_all + __builtin_amdgcn_logf(L)) * 0.69314718055994530942f : -INFINITY;
    }
    __syncthreads();
  }
}

template <int D, int NQ>
hipError_t launch(const CacheAttnArgs &a, bool four_bit, bool far, hipStream_t s) {
  const unsigned z = a.a.B < STS_GRID_Z ? a.a.B : STS_GRID_Z;
  const dim3 grid((unsigned)(a.a.num_splits * a.a.z_rounds), a.a.num_units, z), block(64 * STS_WG_WAVES);
  const bool gather = a.a.indices || a.a.block_table;
  if (four_bit) {
    if (far) STS_LAUNCH((cache_attn_kernel<D, NQ, true, true, true>), grid, block, 0, s, a);
    else if (gather) STS_LAUNCH((cache_attn_kernel<D, NQ, true, true, false>), grid, block, 0, s, a);
    else STS_LAUNCH((cache_attn_kernel<D, NQ, true, false, false>), grid, block, 0, s, a);
  } else {
    if (far) STS_LAUNCH((cache_attn_kernel<D, NQ, false, true, true>), grid, block, 0, s, a);
    else STS_LAUNCH((cache_attn_kernel<D, NQ, false, false, false>), grid, block, 0, s, a);
  }
  return sts_take_launch_status();
}

}  // namespace

hipError_t launch_cache_attn(const CacheAttnArgs &a, int d, int nq, bool four_bit, bool far, hipStream_t s) {
  if ((size_t)a.a.B * a.a.num_units * a.a.num_splits == 0) return hipSuccess;
  if (nq > 2) return hipErrorInvalidValue;
  if (d == 128) return nq == 1 ? launch<128, 1>(a, four_bit, far, s) : launch<128, 2>(a, four_bit, far, s);
  return nq == 1 ? launch<64, 1>(a, four_bit, far, s) : launch<64, 2>(a, four_bit, far, s);
}
