// Host-side sanitizer driver for the operators around a small cache (test infrastructure, not part of libsts.so): linked with their host
// file only. The kernel launchers are stubs that check their launch arguments and touch no device memory.
#include <math.h>
#include <stdio.h>
#include <stdlib.h>
#include <string.h>

#include <vector>

#include "cache.h"

static long g_launches = 0, g_combines = 0;
static const unsigned char *g_ws_lo = nullptr, *g_ws_hi = nullptr;

static void fail(const char *what) {
  fprintf(stderr, "host check failed: %s\n", what);
  exit(3);
}
static void in_ws(const void *p, size_t bytes, const char *what) {
  const unsigned char *c = static_cast<const unsigned char *>(p);
  if (c < g_ws_lo || c + bytes > g_ws_hi) fail(what);
}

hipError_t sts_run_launch(int kind, hipStream_t, hipError_t (*launch)(void *), void *with) {
  if (kind < 0 || kind >= STS_K_COUNT_) fail("kernel kind");
  return launch(with);
}
int sts_cu_count() { return 256; }

hipError_t launch_packed_store(const PackedRowsArgs &a, hipStream_t) {
  ++g_launches;
  if (a.N < 1 || a.B < 1 || a.T < 1 || (1 << a.page_shift) > 32) fail("store: args");
  return hipSuccess;
}
hipError_t launch_packed_load(const PackedRowsArgs &a, hipStream_t) {
  ++g_launches;
  if (a.B < 1 || a.T < 1 || (1 << a.page_shift) > 32) fail("load: args");
  return hipSuccess;
}
static void check_parts(const AttnArgs &a, int d, int nq) {
  if (a.num_splits < 1 || a.num_splits > 256 || a.num_units < 1 || a.num_units > STS_MAX_HEADS) fail("split: grid");
  if (a.direct != (a.num_splits == 1)) fail("split: where results go");
  const size_t parts = (size_t)a.B * a.num_units * a.num_splits;
  in_ws(a.part_o, parts * nq * 16 * d * 4, "split: part_o");
  in_ws(a.part_ml, parts * nq * 16 * 2 * 4, "split: part_ml");
}
hipError_t launch_cache_attn(const CacheAttnArgs &c, int d, int nq, bool four_bit, bool far, hipStream_t) {
  ++g_launches;
  const AttnArgs &a = c.a;
  if ((d != 64 && d != 128) || (nq != 1 && nq != 2)) fail("split: d / nq");
  if (a.block_table && !far) fail("split: pages with short offsets");
  if (!four_bit && (c.window < 1 || c.sinks < 0 || a.indices)) fail("window: args");
  for (int r = 0; r < 32; ++r)
    if (r * c.tq_inv >> 16 != r / a.Tq) fail("split: division by Tq");
  std::vector<int> heads(a.Hq, 0);
  for (int u = 0; u < a.num_units; ++u) {
    const uint32_t unit = a.units.unit[u];
    const int g = unit & 0xff, n = (unit >> 24) & 0x1f;
    const uint32_t mask = (unit >> 8) & 0xffff;
    if (g >= a.Hkv || n < 1 || n * a.Tq > nq * 16 || __builtin_popcount(mask) != n || mask >> a.G) fail("split: unit table");
    for (int i = 0; i < a.G; ++i) heads[g * a.G + i] += mask >> i & 1;
  }
  for (int n : heads)
    if (n != 1) fail("split: a head in no unit, or in two");
  check_parts(a, d, nq);
  return hipSuccess;
}
hipError_t launch_attn_combine(const AttnArgs &a, int d, int nq, hipStream_t) {
  ++g_combines;
  if (a.direct) fail("combine after a direct launch");
  check_parts(a, d, nq);
  return hipSuccess;
}
static void check_window(const WindowArgs &a, int d) {
  if (a.blocks != (a.Tq * (int64_t)a.G + STS_WINDOW_ROWS - 1) / STS_WINDOW_ROWS || a.by_blocks.of(a.blocks) != 1 || a.by_heads.of(a.Hkv) != 1) fail("window: divisors");
  if (a.num_splits < 1 || a.num_splits > 64 || a.Tq <= 16 || a.window < 1 || a.sinks < 0) fail("window: args");
  if (a.num_splits > 1) {
    const size_t blocks = ((size_t)a.Tq * a.G + STS_WINDOW_ROWS - 1) / STS_WINDOW_ROWS * a.Hkv * a.B, rows = blocks * a.num_splits * STS_WINDOW_ROWS;
    in_ws(a.part_o, rows * d * 4, "window: part_o");
    in_ws(a.part_ml, rows * 2 * 4, "window: part_ml");
  }
}
hipError_t launch_window_prompt(const WindowArgs &a, int d, hipStream_t) { ++g_launches; check_window(a, d); return hipSuccess; }
hipError_t launch_window_combine(const WindowArgs &a, int d, hipStream_t) {
  ++g_combines;
  if (a.num_splits < 2) fail("window: combine of one part");
  check_window(a, d);
  return hipSuccess;
}

static unsigned char *const fake = reinterpret_cast<unsigned char *>(uintptr_t(1) << 40);
static unsigned char *const ws = reinterpret_cast<unsigned char *>(uintptr_t(2) << 40);

// the call with the workspace that it asks for, and with one byte less
template <class P, class Q, class F>
static bool with_workspace(P &p, Q query, F call, bool always) {
  const size_t need = query(&p);
  p.workspace = ws;
  p.workspace_bytes = need;
  g_ws_lo = ws;
  g_ws_hi = ws + need;
  const sts_status rc = call(&p, nullptr);
  if ((need > 0) != (rc == STS_OK)) fail("the size query and the call disagree");
  if (rc == STS_OK && p.B > 0 && need > 256 && always) {
    const long before = g_launches;
    p.workspace_bytes = need - 257;
    if (call(&p, nullptr) != STS_EWORKSPACE) fail("short workspace accepted");
    if (g_launches != before) fail("kernels enqueued before a refusal");
  }
  return rc == STS_OK;
}

// the divisions by multiplication: small divisors and next to powers of two, dividends next to multiples and at the ends
static void check_divisors() {
  auto one = [](int64_t d) {
    if (d < 1 || d > 0x7fffffff) return;
    const Divisor by = divide_by((int)d);
    const int64_t most = 0x7fffffff / d * d;
    for (int64_t n : {(int64_t)0, (int64_t)1, d - 1, d, d + 1, 2 * d - 1, 2 * d, 977 * d - 1, 977 * d, most - 1, most, (int64_t)0x7fffffff})
      if (n >= 0 && n <= 0x7fffffff && by.of((int)n) != n / d) fail("division by multiplication");
  };
  for (int d = 1; d <= 100000; ++d) one(d);
  for (int s = 0; s <= 31; ++s)
    for (int64_t k = -3; k <= 3; ++k) one((1ll << s) + k);
}

int main() {
  long calls = 0, accepted = 0;
  check_divisors();
  const int Bs[] = {0, 1, 4, 33, 70000}, Tqs[] = {1, 3, 5, 8, 16, 17, 300, 8192}, Ns[] = {0, 1, 31, 4096, 131072, 0x7fffffff - 65536};
  for (int B : Bs) for (int Tq : Tqs) for (int N : Ns) for (int d : {64, 128})
    for (int Hkv : {1, 2, 8, 16}) for (int G : {1, 3, 4, 8, 16}) {
      const int Hq = Hkv * G;
      if (Hq > 256) continue;
      for (int page : {0, 8})
        for (int extra = 0; extra < 2; ++extra) {
          for (int lists = 0; lists < 3; ++lists) {
            sts_packed_attn_params p;
            memset(&p, 0, sizeof(p));
            p.B = B; p.Tq = Tq; p.Hq = Hq; p.Hkv = Hkv; p.d = d;
            p.cache.codes = fake; p.cache.scales = fake;
            p.cache.code_stride_n = d; p.cache.code_stride_h = (int64_t)N * d; p.cache.code_stride_b = (int64_t)Hkv * N * d;
            p.cache.scale_stride_n = d / 16; p.cache.scale_stride_h = (int64_t)N * d / 16; p.cache.scale_stride_b = (int64_t)Hkv * N * d / 16;
            p.cache.N = N; p.cache.page_size = page;
            if (page && extra) {
              p.cache.block_table = reinterpret_cast<const int32_t *>(fake);
              p.cache.table_stride = (int32_t)(((int64_t)N + page - 1) / page); p.cache.num_pages = 5;
              p.cache.code_stride_page = page * d; p.cache.scale_stride_page = page * d / 16;
            }
            std::vector<int32_t> hm(Hq);
            for (int t = 0; t < Hq; ++t) hm[t] = lists == 1 ? t : t / 2;
            if (lists && N) {
              p.indices = reinterpret_cast<const int32_t *>(fake);
              p.kmax = N / 10 + 1;
              if (lists == 2) p.head_map = hm.data();
            }
            p.scale = 0.1f;
            p.q = fake; p.out = fake;
            if (extra) { p.k_new = fake; p.v_new = fake; p.causal = 1; }
            accepted += with_workspace(p, sts_packed_attn_workspace_bytes, sts_packed_attn, true);
            ++calls;
          }
          for (int window : {1, 100, 4096, 0x7fffffff})
            for (int sinks : {0, 5, 0x7fffffff}) {
              sts_window_params p;
              memset(&p, 0, sizeof(p));
              p.B = B; p.Tq = Tq; p.Hq = Hq; p.Hkv = Hkv; p.d = d; p.N = N; p.page_size = page;
              p.kv_stride_n = d; p.kv_stride_h = (int64_t)N * d; p.kv_stride_b = (int64_t)Hkv * N * d;
              p.q = fake; p.k = fake; p.v = fake; p.out = fake;
              p.window = window; p.sinks = sinks;
              p.scale = -0.1f;
              if (extra && Tq <= 16) { p.k_new = fake; p.v_new = fake; }
              accepted += with_workspace(p, sts_window_attn_workspace_bytes, sts_window_attn, true);
              ++calls;
            }
        }
    }
  for (int B : Bs) for (int T : {0, 1, 5, 100000, 0x7fffffff}) for (int N : Ns) for (int d : {64, 96, 128}) for (int page : {0, 1, 3, 32}) {
    sts_packed_rows_params p;
    memset(&p, 0, sizeof(p));
    p.B = B; p.T = T; p.Hkv = 8; p.d = d; p.k = fake; p.v = fake;
    p.cache.codes = fake; p.cache.scales = fake; p.cache.N = N; p.cache.page_size = page;
    p.cache.code_stride_n = d; p.cache.scale_stride_n = d / 16;
    const long before = g_launches;
    const bool good = d != 96 && page != 3 && B <= 65535 && T != 0x7fffffff;
    const bool stored = sts_packed_store(&p, nullptr) == STS_OK, loaded = sts_packed_load(&p, nullptr) == STS_OK;
    if (stored != good || loaded != good) fail("rows: wrong verdict");
    if (g_launches - before != (good && B && T ? (N ? 2 : 1) : 0)) fail("rows: launches");
    accepted += good;
    calls += 2;
  }
  if (accepted == 0 || g_launches == 0 || g_combines == 0) fail("nothing was accepted: the driver checks nothing");
  printf("host checks done: %ld calls, %ld accepted, %ld stub launches, %ld combines\n", calls, accepted, g_launches, g_combines);
  return 0;
}
