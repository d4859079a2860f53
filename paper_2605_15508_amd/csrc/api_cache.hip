// Host side of the operators around a small cache: sts_packed_store, sts_packed_load, sts_packed_attn, sts_window_attn. Argument
// checks, launch plans, workspaces.
#include <math.h>
#include <string.h>

#include "cache.h"

namespace {

inline size_t align256(size_t x) { return (x + 255) & ~(size_t)255; }
inline bool aligned(const void *p, size_t to) { return reinterpret_cast<uintptr_t>(p) % to == 0; }
inline int page_of(int page_size) { return page_size <= 1 ? 1 : page_size; }
inline bool page_ok(int page) { return page == 1 || page == 2 || page == 4 || page == 8 || page == 16 || page == 32; }
inline int shift_of(int page) {
  int s = 0;
  while ((1 << s) < page) ++s;
  return s;
}

sts_status validate_cache(const sts_packed_cache &c, int d) {
  if (d != 64 && d != 128) return STS_EUNSUPPORTED;
  if (c.N < 0) return STS_EINVAL;
  if (c.N > 0x7fffffff - 65536) return STS_EUNSUPPORTED;
  const int page = page_of(c.page_size), sw = d / 16;
  if (!page_ok(page)) return STS_EUNSUPPORTED;
  if (c.code_stride_n < d || c.scale_stride_n < sw || c.code_stride_b < 0 || c.code_stride_h < 0 || c.scale_stride_b < 0 || c.scale_stride_h < 0)
    return STS_EUNSUPPORTED;
  if (c.code_stride_n % 16 || c.code_stride_h % 16 || c.code_stride_b % 16 || c.scale_stride_n % sw || c.scale_stride_h % sw || c.scale_stride_b % sw)
    return STS_EUNSUPPORTED;
  // (a tile's row offsets are 32-bit)
  if (c.code_stride_n > (int64_t)1 << 26 || c.scale_stride_n > (int64_t)1 << 26) return STS_EUNSUPPORTED;
  if (!aligned(c.codes, 16) || !aligned(c.scales, sw)) return STS_EUNSUPPORTED;
  if (c.block_table) {
    if (c.num_pages < 1 || c.code_stride_page < 1 || c.scale_stride_page < 1) return STS_EINVAL;
    if (c.code_stride_page % 16 || c.scale_stride_page % sw) return STS_EUNSUPPORTED;
    if ((int64_t)c.table_stride * page < c.N) return STS_EINVAL;
  }
  return STS_OK;
}

sts_status rows_call(const sts_packed_rows_params *p, bool store, hipStream_t s) {
  if (!p || p->B < 0 || p->T < 0 || p->Hkv < 1) return STS_EINVAL;
  const sts_status v = validate_cache(p->cache, p->d);
  if (v != STS_OK) return v;
  // (a grid's dimension holds 2^32 threads, of which a row takes up to 16)
  if (p->B > 65535 || (int64_t)p->T * p->Hkv > (1 << 28) - 65536) return STS_EUNSUPPORTED;
  if (p->B == 0 || p->T == 0) return STS_OK;
  if (store && p->cache.N == 0) return STS_OK;       // no place for any row
  if (!p->k || !p->v || (p->cache.N > 0 && (!p->cache.codes || !p->cache.scales))) return STS_EINVAL;
  if (!aligned(p->k, 16) || !aligned(p->v, 16)) return STS_EUNSUPPORTED;
  PackedRowsArgs a;
  memset(&a, 0, sizeof(a));
  a.k = static_cast<uint16_t *>(p->k);
  a.v = static_cast<uint16_t *>(p->v);
  a.pos = p->pos;
  a.lens = p->lens;
  a.codes = p->cache.codes;
  a.scales = p->cache.scales;
  a.code_b = p->cache.code_stride_b; a.code_h = p->cache.code_stride_h; a.code_n = p->cache.code_stride_n; a.code_page = p->cache.code_stride_page;
  a.scale_b = p->cache.scale_stride_b; a.scale_h = p->cache.scale_stride_h; a.scale_n = p->cache.scale_stride_n; a.scale_page = p->cache.scale_stride_page;
  a.block_table = p->cache.block_table;
  a.table_stride = p->cache.table_stride;
  a.num_pages = p->cache.num_pages;
  a.page_shift = shift_of(page_of(p->cache.page_size));
  a.N = p->cache.N;
  a.B = p->B; a.T = p->T; a.Hkv = p->Hkv; a.d = p->d;
  const hipError_t rc = sts_run_kernel(store ? STS_K_PACKED_STORE : STS_K_PACKED_LOAD, s,
                                       [&] { return store ? launch_packed_store(a, s) : launch_packed_load(a, s); });
  return rc == hipSuccess ? STS_OK : STS_EHIP;
}

struct CachePlan {
  int nq, num_units, num_splits;
  size_t part_o_bytes, part_ml_bytes;
  AttnUnitTable units;
  size_t total() const {
    const size_t n = part_o_bytes + part_ml_bytes;
    return n ? n : 256;
  }
};

// Units of a short block and how many parts their tiles are cut into, `tiles` of them at most per unit: so many that `resident`
// workgroups run at once, with two tiles for each of their four waves at least, or one (one_each) as long as every workgroup has a
// compute unit of its own. Lists of up to 16 tiles stay whole, as for the bf16 cache: a second launch takes as long as they do. Not
// so with own tokens (tail) and two tiles of query rows, which a whole unit's workgroup takes in one after the other, as long as
// there are few units (500 tokens of 4 bits, 5 rows, one sequence: 11.1 us in parts, 12.4 whole; 64 heads of 16 rows, 4 sequences:
// 20.3 and 18.1).
sts_status plan_splits(int B, int Tq, int Hq, int Hkv, int d, int most_rows, const int32_t *head_map, bool whole_groups, int64_t tiles, int row_bytes,
                       bool one_each, bool tail, int64_t (*resident)(int d), CachePlan &pl) {
  int max_heads = most_rows / Tq;
  if (max_heads < 1) max_heads = 1;
  if (max_heads > STS_MAX_GROUP) max_heads = STS_MAX_GROUP;
  int rows = 0;
  const int nu = sts_group_units(Hq, Hkv, Tq, max_heads, head_map, whole_groups, pl.units, rows);
  if (nu < 0) return STS_EUNSUPPORTED;
  pl.num_units = nu;
  pl.nq = rows <= 16 ? 1 : 2;
  const int64_t total = (int64_t)B * nu;
  auto parts_of = [&](int64_t workgroups, int wave_tiles) {
    const int64_t most = (tiles + wave_tiles * STS_WG_WAVES - 1) / (wave_tiles * STS_WG_WAVES), S = total > 0 ? workgroups / total : 1;
    return S < most ? S : most;
  };
  const bool whole = tiles <= 16 && !(tail && pl.nq == 2 && 4 * total <= sts_cu_count());
  int64_t S = whole ? 1 : parts_of(resident(d), 2);
  if (one_each && !whole) {
    const int64_t more = parts_of(sts_cu_count(), 1);
    if (more > S) S = more;
  }
  if (S < 1) S = 1;
  // Between one and two units for each compute unit some would have two to work on and most one. Parts even that out, where a unit is a
  // megabyte of the cache or more: 33 sequences, window 4096 138 us whole, 118 in parts; 16000 tokens of 4 bits 146 and 124; 4000
  // of them 42 and 43.
  const int64_t cus = sts_cu_count();
  if (total > cus && total < 2 * cus && tiles * STS_TILE_KEYS * row_bytes >= 1 << 20) {
    int64_t rounds = 2;                    // with S parts; the shortest is that of the least rounds / S
    for (int64_t s = 2; s <= 4; ++s) {
      const int64_t r = (total * s + cus - 1) / cus;
      if (r * S < rounds * s) rounds = r, S = s;
    }
  }
  if (S > 256) S = 256;
  pl.num_splits = (int)S;
  const size_t parts = (size_t)total * (size_t)S;
  if (parts > 0x7fffffffull) return STS_EUNSUPPORTED;
  pl.part_o_bytes = align256(parts * (size_t)pl.nq * 16 * d * sizeof(float));
  pl.part_ml_bytes = align256(parts * (size_t)pl.nq * 16 * 2 * sizeof(float));
  return STS_OK;
}

// what sts_packed_attn and sts_window_attn have in common
sts_status validate_heads(int B, int Tq, int Hq, int Hkv, int d, int out_dtype, float scale, const void *k_new, const void *v_new) {
  if (B < 0 || Tq < 1 || Hq < 1 || Hkv < 1 || Hq % Hkv != 0) return STS_EINVAL;
  if (d != 64 && d != 128) return STS_EUNSUPPORTED;
  if (Hq > STS_MAX_HEADS || Hq / Hkv > STS_MAX_GROUP) return STS_EUNSUPPORTED;
  if (out_dtype != STS_BF16 && out_dtype != STS_F32) return STS_EINVAL;
  if (!isfinite(scale * 1.44269504088896340736f)) return STS_EINVAL;         // (of which the kernels take the product with log2(e))
  if ((k_new == nullptr) != (v_new == nullptr)) return STS_EINVAL;
  if (!aligned(k_new, 16) || !aligned(v_new, 16)) return STS_EUNSUPPORTED;
  return STS_OK;
}

int64_t packed_resident(int) { return (int64_t)sts_cu_count() * 2; }

sts_status plan_packed(const sts_packed_attn_params *p, CachePlan &pl) {
  if (!p) return STS_EINVAL;
  sts_status v = validate_heads(p->B, p->Tq, p->Hq, p->Hkv, p->d, p->out_dtype, p->scale, p->k_new, p->v_new);
  if (v != STS_OK) return v;
  if (p->Tq > 16) return STS_EUNSUPPORTED;
  v = validate_cache(p->cache, p->d);
  if (v != STS_OK) return v;
  const int page = page_of(p->cache.page_size);
  const bool lists = p->indices != nullptr;
  if (lists) {
    if (p->kmax < 0 || p->seq_lens) return STS_EINVAL;
    if ((int64_t)p->kmax * page > 0x7fffffffll - 65536) return STS_EUNSUPPORTED;
    if (p->kmax > 0 && p->cache.N == 0) return STS_EINVAL;
    if (p->idx_stride_b < 0 || p->cnt_stride_b < 0) return STS_EINVAL;
    if (p->idx_stride_b && p->idx_stride_b < (int64_t)p->Hq * p->kmax) return STS_EINVAL;
    if (p->cnt_stride_b && p->cnt_stride_b < p->Hq) return STS_EINVAL;
    if (p->head_map)
      for (int t = 0; t < p->Hq; ++t)
        if (p->head_map[t] < 0) return STS_EINVAL;
  } else if (p->counts || p->head_map || p->kmax != 0) {
    return STS_EINVAL;
  }
  const int64_t len = lists ? (int64_t)p->kmax * page : p->cache.N;
  return plan_splits(p->B, p->Tq, p->Hq, p->Hkv, p->d, 32, p->head_map, !lists, (len + STS_TILE_KEYS - 1) / STS_TILE_KEYS, p->d + p->d / 16, false, p->k_new != nullptr,
                     packed_resident, pl);
}

int64_t window_resident(int d) { return (int64_t)sts_cu_count() * (d == 128 ? 1 : 2); }

sts_status plan_window(const sts_window_params *p, CachePlan &pl, bool &prompt) {
  if (!p) return STS_EINVAL;
  const sts_status v = validate_heads(p->B, p->Tq, p->Hq, p->Hkv, p->d, p->out_dtype, p->scale, p->k_new, p->v_new);
  if (v != STS_OK) return v;
  if (p->N < 0 || p->window < 1 || p->sinks < 0) return STS_EINVAL;
  if (p->N > 0x7fffffff - 65536 || p->Tq > 0x7fffffff - 65536) return STS_EUNSUPPORTED;
  if (p->k_new && (p->Tq > 16 || p->window < p->Tq)) return STS_EUNSUPPORTED;
  if (p->kv_stride_n < p->d || p->kv_stride_n % 8 || p->kv_stride_h % 8 || p->kv_stride_b % 8 || p->kv_stride_h < 0 || p->kv_stride_b < 0) return STS_EUNSUPPORTED;
  if (p->kv_stride_n > (int64_t)1 << 25) return STS_EUNSUPPORTED;
  const int page = page_of(p->page_size);
  if (!page_ok(page)) return STS_EUNSUPPORTED;
  if (p->block_table) {
    if (p->num_pages < 1 || p->kv_stride_page < 1) return STS_EINVAL;
    if (p->kv_stride_page % 8) return STS_EUNSUPPORTED;
    if ((int64_t)p->table_stride * page < p->N) return STS_EINVAL;
  }
  // Which kernel: by the number of query rows. 16 rows in units of up to 32 rows of a KV head, and 17 in blocks of 128, over 8 KV heads, window
  // 4096 of 32768 tokens: 1, 2, 4, 8 query heads each and one sequence 13.2 and 19.6 us, 15.3 and 20.6, 15.8 and 20.8, 18.8 and 22.4; 16
  // sequences 47 and 64, 50 and 64, 80 and 67, 159 and 99. (With 64 rows and more on a KV head, where several units read the same
  // window, the second would be ahead in large batches.)
  prompt = p->Tq > 16;
  memset(&pl, 0, sizeof(pl));
  if (prompt) {
    // Blocks of rows; where they leave compute units without work, several workgroups share a block's keys, four tiles each at least.
    const int G = p->Hq / p->Hkv;
    const int64_t blocks = ((int64_t)p->Tq * G + STS_WINDOW_ROWS - 1) / STS_WINDOW_ROWS * p->Hkv * p->B;
    if ((int64_t)p->Tq * G > 0x7fffffffll - 65536 || blocks >= 1 << 24) return STS_EUNSUPPORTED;      // (256 threads each: see above)
    const int64_t span = (int64_t)p->sinks + p->window + STS_WINDOW_ROWS / G + 1, keys = span < p->N ? span : p->N;
    const int64_t tiles = (keys + STS_WINDOW_KEYS - 1) / STS_WINDOW_KEYS;
    int64_t S = blocks > 0 ? 2 * sts_cu_count() / blocks : 1;
    if (S > tiles / 4) S = tiles / 4;
    if (S > 64) S = 64;
    if (S < 1) S = 1;
    pl.num_splits = (int)S;
    if (S > 1) {
      pl.part_o_bytes = align256((size_t)(blocks * S) * STS_WINDOW_ROWS * p->d * sizeof(float));
      pl.part_ml_bytes = align256((size_t)(blocks * S) * STS_WINDOW_ROWS * 2 * sizeof(float));
    }
    return STS_OK;
  }
  // no more tiles than the cache has, than the sinks and the window span (one more where the window begins inside a tile).
  // One for a wave: 5 rows, window 1024, pages 13.2 us, with two 15.3 (over 4 bits 4096 tokens 9.2 us, with two 8.6).
  const int64_t all = ((int64_t)p->N + STS_TILE_KEYS - 1) / STS_TILE_KEYS;
  const int64_t some = ((int64_t)p->sinks + STS_TILE_KEYS - 1) / STS_TILE_KEYS + ((int64_t)p->window + p->Tq + STS_TILE_KEYS - 1) / STS_TILE_KEYS + 1;
  return plan_splits(p->B, p->Tq, p->Hq, p->Hkv, p->d, 32, nullptr, true, all < some ? all : some, 4 * p->d, true, p->k_new != nullptr, window_resident, pl);
}

sts_status launch_short(CacheAttnArgs &c, const CachePlan &pl, int d, bool four_bit, bool far, int kind, void *ws, size_t ws_bytes, hipStream_t s) {
  if (!ws || ws_bytes < pl.part_o_bytes + pl.part_ml_bytes || !aligned(ws, 256)) return STS_EWORKSPACE;
  AttnArgs &a = c.a;
  c.tq_inv = 65536 / a.Tq + 1;
  a.num_units = pl.num_units;
  a.num_splits = pl.num_splits;
  a.z_rounds = (a.B + STS_GRID_Z - 1) / STS_GRID_Z;
  a.units = pl.units;
  a.scale_log2 = a.scale * 1.44269504088896340736f;
  a.part_o = static_cast<float *>(ws);
  a.part_ml = reinterpret_cast<float *>(static_cast<unsigned char *>(ws) + pl.part_o_bytes);
  a.direct = pl.num_splits == 1;
  hipError_t rc = sts_run_kernel(kind, s, [&] { return launch_cache_attn(c, d, pl.nq, four_bit, far, s); });
  if (rc == hipSuccess && !a.direct) rc = sts_run_kernel(STS_K_ATTN_COMBINE, s, [&] { return launch_attn_combine(a, d, pl.nq, s); });
  return rc == hipSuccess ? STS_OK : STS_EHIP;
}

}  // namespace

extern "C" {

sts_status sts_packed_store(const sts_packed_rows_params *p, void *stream) { return rows_call(p, true, static_cast<hipStream_t>(stream)); }
sts_status sts_packed_load(const sts_packed_rows_params *p, void *stream) { return rows_call(p, false, static_cast<hipStream_t>(stream)); }

size_t sts_packed_attn_workspace_bytes(const sts_packed_attn_params *p) {
  CachePlan pl;
  return plan_packed(p, pl) == STS_OK ? pl.total() : 0;
}

sts_status sts_packed_attn(const sts_packed_attn_params *p, void *stream) {
  CachePlan pl;
  const sts_status v = plan_packed(p, pl);
  if (v != STS_OK) return v;
  if (p->B == 0) return STS_OK;
  if (!p->q || !p->out) return STS_EINVAL;
  if (p->cache.N > 0 && (!p->cache.codes || !p->cache.scales)) return STS_EINVAL;
  if (!aligned(p->q, 16) || !aligned(p->out, 16)) return STS_EUNSUPPORTED;
  CacheAttnArgs c;
  memset(&c, 0, sizeof(c));
  AttnArgs &a = c.a;
  const bool lists = p->indices != nullptr;
  a.q = static_cast<const uint16_t *>(p->q);
  a.indices = p->indices;
  a.counts = p->counts;
  a.seq_lens = p->seq_lens;
  a.idx_stride_b = p->idx_stride_b ? p->idx_stride_b : (int64_t)p->Hq * p->kmax;
  a.cnt_stride_b = p->cnt_stride_b ? p->cnt_stride_b : p->Hq;
  a.B = p->B; a.Tq = p->Tq; a.Hq = p->Hq; a.Hkv = p->Hkv; a.G = p->Hq / p->Hkv; a.N = p->cache.N; a.kmax = p->kmax;
  a.page = page_of(p->cache.page_size);
  a.page_shift = shift_of(a.page);
  a.block_table = p->cache.block_table;
  a.table_stride = p->cache.table_stride;
  a.num_pages = p->cache.num_pages;
  a.k_new = static_cast<const uint16_t *>(p->k_new);
  a.v_new = static_cast<const uint16_t *>(p->v_new);
  a.causal = p->causal;
  a.scale = p->scale;
  a.out = p->out;
  a.lse_out = p->lse_out;
  a.out_dtype = p->out_dtype;
  c.codes = p->cache.codes;
  c.scales = p->cache.scales;
  c.code_b = p->cache.code_stride_b; c.code_h = p->cache.code_stride_h; c.code_n = p->cache.code_stride_n; c.code_page = p->cache.code_stride_page;
  c.scale_b = p->cache.scale_stride_b; c.scale_h = p->cache.scale_stride_h; c.scale_n = p->cache.scale_stride_n; c.scale_page = p->cache.scale_stride_page;
  // 32-bit offsets into one head's rows, the chunk's own included
  const int64_t widest = c.code_n > c.scale_n ? c.code_n : c.scale_n;
  const bool far = p->cache.block_table || (lists && (int64_t)p->cache.N * widest > 0xffffffffll);
  return launch_short(c, pl, p->d, true, far, STS_K_PACKED_ATTN, p->workspace, p->workspace_bytes, static_cast<hipStream_t>(stream));
}

size_t sts_window_attn_workspace_bytes(const sts_window_params *p) {
  CachePlan pl;
  bool prompt;
  return plan_window(p, pl, prompt) == STS_OK ? pl.total() : 0;
}

sts_status sts_window_attn(const sts_window_params *p, void *stream) {
  CachePlan pl;
  bool prompt;
  const sts_status v = plan_window(p, pl, prompt);
  if (v != STS_OK) return v;
  if (p->B == 0) return STS_OK;
  if (!p->q || !p->out || (p->N > 0 && (!p->k || !p->v))) return STS_EINVAL;
  if (!aligned(p->q, 16) || !aligned(p->out, 16) || !aligned(p->k, 16) || !aligned(p->v, 16)) return STS_EUNSUPPORTED;
  const int page = page_of(p->page_size);
  hipStream_t s = static_cast<hipStream_t>(stream);
  if (prompt) {
    WindowArgs w;
    memset(&w, 0, sizeof(w));
    w.q = static_cast<const uint16_t *>(p->q);
    w.k = static_cast<const uint16_t *>(p->k);
    w.v = static_cast<const uint16_t *>(p->v);
    w.stride_b = p->kv_stride_b; w.stride_h = p->kv_stride_h; w.stride_n = p->kv_stride_n; w.stride_page = p->kv_stride_page;
    w.seq_lens = p->seq_lens;
    w.block_table = p->block_table;
    w.B = p->B; w.Tq = p->Tq; w.Hq = p->Hq; w.Hkv = p->Hkv; w.G = p->Hq / p->Hkv; w.N = p->N;
    w.window = p->window; w.sinks = p->sinks;
    w.page_shift = shift_of(page);
    w.table_stride = p->table_stride;
    w.num_pages = p->num_pages;
    w.scale = p->scale;
    w.scale_log2 = p->scale * 1.44269504088896340736f;
    w.out = p->out;
    w.lse_out = p->lse_out;
    w.out_dtype = p->out_dtype;
    w.num_splits = pl.num_splits;
    w.blocks = (int32_t)(((int64_t)w.Tq * w.G + STS_WINDOW_ROWS - 1) / STS_WINDOW_ROWS);
    w.by_splits = divide_by(w.num_splits);
    w.by_blocks = divide_by(w.blocks);
    w.by_heads = divide_by(w.Hkv);
    w.by_group = divide_by(w.G);
    if (pl.num_splits > 1) {
      if (!p->workspace || p->workspace_bytes < pl.part_o_bytes + pl.part_ml_bytes || !aligned(p->workspace, 256)) return STS_EWORKSPACE;
      w.part_o = static_cast<float *>(p->workspace);
      w.part_ml = reinterpret_cast<float *>(static_cast<unsigned char *>(p->workspace) + pl.part_o_bytes);
    }
    hipError_t rc = sts_run_kernel(STS_K_WINDOW, s, [&] { return launch_window_prompt(w, p->d, s); });
    if (rc == hipSuccess && pl.num_splits > 1) rc = sts_run_kernel(STS_K_ATTN_COMBINE, s, [&] { return launch_window_combine(w, p->d, s); });
    return rc == hipSuccess ? STS_OK : STS_EHIP;
  }
  CacheAttnArgs c;
  memset(&c, 0, sizeof(c));
  AttnArgs &a = c.a;
  a.q = static_cast<const uint16_t *>(p->q);
  a.k = static_cast<const uint16_t *>(p->k);
  a.v = static_cast<const uint16_t *>(p->v);
  a.stride_b = p->kv_stride_b; a.stride_h = p->kv_stride_h; a.stride_n = p->kv_stride_n; a.stride_page = p->kv_stride_page;
  a.seq_lens = p->seq_lens;
  a.B = p->B; a.Tq = p->Tq; a.Hq = p->Hq; a.Hkv = p->Hkv; a.G = p->Hq / p->Hkv; a.N = p->N;
  a.page = page;
  a.page_shift = shift_of(page);
  a.block_table = p->block_table;
  a.table_stride = p->table_stride;
  a.num_pages = p->num_pages;
  a.k_new = static_cast<const uint16_t *>(p->k_new);
  a.v_new = static_cast<const uint16_t *>(p->v_new);
  a.causal = 1;
  a.scale = p->scale;
  a.out = p->out;
  a.lse_out = p->lse_out;
  a.out_dtype = p->out_dtype;
  c.window = p->window;
  c.sinks = p->sinks;
  c.behind = p->k_new ? 1 : 0;
  return launch_short(c, pl, p->d, false, p->block_table != nullptr, STS_K_WINDOW, p->workspace, p->workspace_bytes, s);
}

}  // extern "C"
