// The 4-bit cache: rows of K and V in, and the values that it holds for them out (gfx950).
//
// A group of 32 channels takes s = floor(log2(max|x|)) - 2 + 127, one more where max|x| > 1.75 * 2^floor(log2(max|x|)); in the
// bits of a bf16 magnitude m (exponent e, 7 bits of fraction f) that is ((m + 31) >> 7) - 2: f > 96 carries into the exponent. The
// codes are what the chip's own conversion gives for x * 2^(127 - s): the nearest of 0, 0.5, 1, 1.5, 2, 3, 4, 6, ties to the even
// code, at most 6. With max|x| <= 7 * 2^(s - 127) the limit is the nearest code, too. Nothing here rounds but that conversion.
//
// What bounds both: memory. A lane holds 8 channels, 16 bytes of bf16 and 4 of codes, so that a wave's accesses are whole rows; K's
// and V's row are under way together. 100003 tokens of 8 KV heads out of the cache: 518 MB in 100 us, 5.2 TB/s read and written,
// where a copy of 512 MB reaches 5.3; 2 x 8191 rows into a pool of pages 16.5 us. A step's few rows take a launch, 3 us.
#include "cache.h"

namespace {

constexpr int THREADS = 256;

// the place of position n of batch element b and KV head h: byte offsets of its codes and its scales
__device__ __forceinline__ void place_of(const PackedRowsArgs &A, int b, int h, int n, int64_t &code, int64_t &scale) {
  if (A.block_table) {
    const int page = min(max(A.block_table[(size_t)b * A.table_stride + (n >> A.page_shift)], 0), A.num_pages - 1);
    const int slot = n & ((1 << A.page_shift) - 1);
    code = page * A.code_page + h * A.code_h + slot * A.code_n;
    scale = page * A.scale_page + h * A.scale_h + slot * A.scale_n;
  } else {
    code = b * A.code_b + h * A.code_h + n * A.code_n;
    scale = b * A.scale_b + h * A.scale_h + n * A.scale_n;
  }
}

__device__ __forceinline__ uint32_t max16(uint32_t x, uint32_t y) {        // of both halves
  typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
  return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2, x), __builtin_bit_cast(u16x2, y)));
}

template <int CTRL>
__device__ __forceinline__ uint32_t dpp(uint32_t x) {
  return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, CTRL, 0xf, 0xf, false);
}

// 8 channels -> 8 codes; s: the group's scale byte. The four lanes of a quad hold a group.
__device__ __forceinline__ uint32_t to_codes(u32x4 x, uint32_t &s) {
  uint32_t m = max16(max16(x[0] & 0x7fff7fffu, x[1] & 0x7fff7fffu), max16(x[2] & 0x7fff7fffu, x[3] & 0x7fff7fffu));
  m = max16(m, dpp<0xb1>(m));        // lane ^ 1
  m = max16(m, dpp<0x4e>(m));        // lane ^ 2
  m = max(m & 0xffffu, m >> 16);
  const bool bad = m >= 0x7f80u;     // an infinity or a NaN
  s = bad ? 255u : (uint32_t)min(max((int)((m + 31) >> 7) - 2, 2), 252);
  const float f = __builtin_bit_cast(float, s << 23);
  const uint32_t x0 = x[0], x1 = x[1], x2 = x[2], x3 = x[3];      // (a cast of a vector's element would be one of its first)
  uint32_t c = 0;
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2, x0), f, 0);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2, x1), f, 1);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2, x2), f, 2);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2, x3), f, 3);
  return bad ? 0u : c;
}

// the scale bytes of a row's D / 32 quads, in the row's first lane
template <int D>
__device__ __forceinline__ uint32_t row_scales(uint32_t s) {
  uint32_t w = s | dpp<0x104>(s) << 8;                                      // row_shl: lane + 4
  if (D == 128) w |= dpp<0x108>(s) << 16 | dpp<0x10c>(s) << 24;
  return w;
}

// grid (rows of T * Hkv, B); a row of D channels is D / 8 lanes
template <int D>
__global__ void __launch_bounds__(THREADS) packed_store_kernel(const PackedRowsArgs A) {
  constexpr int LANES = D / 8;
  const int b = blockIdx.y, row = blockIdx.x * (THREADS / LANES) + threadIdx.x / LANES, lane = threadIdx.x % LANES;
  const int t = row / A.Hkv, h = row - t * A.Hkv;
  const int n = (int)((uint32_t)(A.pos ? A.pos[b] : 0) + (uint32_t)t);          // (past the largest int: negative)
  const bool live = t < (A.lens ? min(A.lens[b], A.T) : A.T) && n >= 0 && n < A.N;
  // (a quad's lanes all hold the same row; lanes of rows that are not stored take part in the exchange with zeros)
  u32x4 k = {0, 0, 0, 0}, v = {0, 0, 0, 0};
  if (live) {
    const size_t at = ((size_t)b * A.T * A.Hkv + row) * D + lane * 8;
    k = *reinterpret_cast<const u32x4 *>(A.k + at);
    v = *reinterpret_cast<const u32x4 *>(A.v + at);
  }
  uint32_t ks, vs;
  const uint32_t kc = to_codes(k, ks), vc = to_codes(v, vs);
  ks = row_scales<D>(ks);
  vs = row_scales<D>(vs);
  if (!live) return;
  int64_t code, scale;
  place_of(A, b, h, n, code, scale);
  uint32_t *c = reinterpret_cast<uint32_t *>(A.codes + code);
  c[lane] = kc;
  c[LANES + lane] = vc;
  if (lane == 0) {
    if (D == 128) *reinterpret_cast<u32x2 *>(A.scales + scale) = u32x2{ks, vs};
    else *reinterpret_cast<uint32_t *>(A.scales + scale) = ks | vs << 16;
  }
}

template <int D>
__global__ void __launch_bounds__(THREADS) packed_load_kernel(const PackedRowsArgs A) {
  constexpr int LANES = D / 8;
  const int b = blockIdx.y, row = blockIdx.x * (THREADS / LANES) + threadIdx.x / LANES, lane = threadIdx.x % LANES;
  const int t = row / A.Hkv, h = row - t * A.Hkv;
  if (t >= (A.lens ? min(A.lens[b], A.T) : A.T)) return;
  const int n = (int)((uint32_t)(A.pos ? A.pos[b] : 0) + (uint32_t)t);          // (past the largest int: negative)
  u32x4 k = {0, 0, 0, 0}, v = {0, 0, 0, 0};
  if (n >= 0 && n < A.N) {
    int64_t code, scale;
    place_of(A, b, h, n, code, scale);
    const uint32_t *c = reinterpret_cast<const uint32_t *>(A.codes + code);
    const uint8_t *s = A.scales + scale;
    const uint32_t kc = c[lane], vc = c[LANES + lane];
    const float ks = __builtin_bit_cast(float, (uint32_t)s[lane / 4] << 23), vs = __builtin_bit_cast(float, (uint32_t)s[D / 32 + lane / 4] << 23);
    k[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(kc, ks, 0));
    k[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(kc, ks, 1));
    k[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(kc, ks, 2));
    k[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(kc, ks, 3));
    v[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(vc, vs, 0));
    v[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(vc, vs, 1));
    v[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(vc, vs, 2));
    v[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(vc, vs, 3));
  }
  const size_t at = ((size_t)b * A.T * A.Hkv + row) * D + lane * 8;
  *reinterpret_cast<u32x4 *>(A.k + at) = k;
  *reinterpret_cast<u32x4 *>(A.v + at) = v;
}

inline dim3 grid_of(const PackedRowsArgs &a, int d) {
  const int rows = THREADS / (d / 8);
  return dim3((unsigned)(((int64_t)a.T * a.Hkv + rows - 1) / rows), (unsigned)a.B);
}

}  // namespace

hipError_t launch_packed_store(const PackedRowsArgs &a, hipStream_t s) {
  if (a.d == 128) STS_LAUNCH(packed_store_kernel<128>, grid_of(a, 128), dim3(THREADS), 0, s, a);
  else STS_LAUNCH(packed_store_kernel<64>, grid_of(a, 64), dim3(THREADS), 0, s, a);
  return sts_take_launch_status();
}

hipError_t launch_packed_load(const PackedRowsArgs &a, hipStream_t s) {
  if (a.d == 128) STS_LAUNCH(packed_load_kernel<128>, grid_of(a, 128), dim3(THREADS), 0, s, a);
  else STS_LAUNCH(packed_load_kernel<64>, grid_of(a, 64), dim3(THREADS), 0, s, a);
  return sts_take_launch_status();
}
