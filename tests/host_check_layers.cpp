// Host-side sanitizer driver for the layers over packed batches (test infrastructure, not part of libsts.so): linked with their host file
// only. The kernel launchers are stubs that check their launch arguments and touch no device memory.
#include <stdio.h>
#include <stdlib.h>
#include <string.h>

#include "layers.h"

static long g_prompts = 0, g_steps = 0, g_sums = 0, g_carries = 0, g_chunks = 0;
static const unsigned char *g_ws_lo = nullptr, *g_ws_hi = nullptr;
static int g_d = 0;

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

static void check_divisor(const Divisor &by, int d, const char *what) {
  for (int64_t n : {(int64_t)0, (int64_t)1, (int64_t)d - 1, (int64_t)d, (int64_t)0x7fffffff / d * d - 1, (int64_t)0x7fffffff})
    if (n >= 0 && by.of((int)n) != n / d) fail(what);
}
hipError_t launch_prompt_attn(const PromptArgs &a, int d, hipStream_t) {
  ++g_prompts;
  if (d != g_d || a.G * a.Hkv != a.Hq || a.seqs.each || !a.seqs.starts) fail("prompt: args");
  if (a.numbers != (int64_t)a.seqs.T * a.G / STS_PROMPT_ROWS + a.seqs.B || (int64_t)a.numbers * a.Hkv >= 1 << 24) fail("prompt: grid");
  if ((int64_t)a.seqs.T * a.G + STS_PROMPT_ROWS > 0x7fffffff || 63 * a.kv_stride_n * 2 + 2 * d > 0x7fffffff) fail("prompt: rows or offsets beyond 32 bits");
  check_divisor(a.by_numbers, a.numbers, "prompt: by_numbers");
  check_divisor(a.by_group, a.G, "prompt: by_group");
  return hipSuccess;
}
static void check_linear(const LinearArgs &a, int d) {
  if (d != g_d || a.G * a.Hkv != a.Hq || (a.q == nullptr) != (a.out == nullptr)) fail("linear: args");
  if (!a.seqs.starts && (int64_t)a.seqs.each * a.seqs.B != a.seqs.T) fail("linear: rows of a sequence");
  if (a.max_len < 0 || a.max_len > a.seqs.T) fail("linear: max_len");
  if (a.state && (a.num_slots < (a.slots ? 0 : a.seqs.B) || a.state_stride < (int64_t)a.Hkv * d * d)) fail("linear: pool");
  check_divisor(a.by_heads, a.Hkv, "linear: by_heads");
  check_divisor(a.by_group, a.G, "linear: by_group");
}
static void check_chunks(const LinearArgs &a, int d) {
  check_linear(a, d);
  if (a.max_len <= STS_LINEAR_STEP) fail("chunks: few rows");
  if (a.segment < STS_LINEAR_CHUNK || a.segment % STS_LINEAR_CHUNK || a.numbers != (int64_t)a.seqs.T / a.segment + a.seqs.B) fail("chunks: segments");
  if ((int64_t)a.numbers * a.Hq >= 1 << 24 || a.heads < 1 || a.heads > 2 || a.G % a.heads) fail("chunks: grid");
  check_divisor(a.by_turns, a.G / a.heads, "chunks: by_turns");
  if (31 * a.q_stride_n * 2 + 2 * d > 0x7fffffff || 31 * a.kv_stride_n * 2 + 2 * d > 0x7fffffff) fail("chunks: offsets beyond 31 bits");
  check_divisor(a.by_segment, a.segment, "chunks: by_segment");
  if (a.part) {
    in_ws(a.part, (size_t)a.numbers * a.Hkv * d * d * 4, "chunks: part");
    in_ws(a.part_log, (size_t)a.numbers * a.Hkv * 8, "chunks: part_log");
  }
  // what any kernel may hand on has a place: several segments, the heads of a group
  if (!a.part && (a.max_len > a.segment || (a.out && a.G > a.heads))) fail("chunks: nowhere for states to go");
}
hipError_t launch_linear_step(const LinearArgs &a, int d, hipStream_t) {
  ++g_steps;
  check_linear(a, d);
  if (a.max_len > STS_LINEAR_STEP || (int64_t)a.seqs.B * a.Hkv * (d / 32) >= 1 << 24) fail("step: grid");
  return hipSuccess;
}
hipError_t launch_linear_sums(const LinearArgs &a, int d, hipStream_t) { ++g_sums; check_chunks(a, d); return hipSuccess; }
hipError_t launch_linear_carry(const LinearArgs &a, int d, hipStream_t) {
  ++g_carries;
  check_chunks(a, d);
  if (!a.part) fail("carry: nothing to carry");
  if ((int64_t)a.seqs.B * a.Hkv * (d * d / 1024) >= 1 << 24) fail("carry: grid");
  return hipSuccess;
}
hipError_t launch_linear_chunks(const LinearArgs &a, int d, hipStream_t) {
  ++g_chunks;
  check_chunks(a, d);
  if (!a.out) fail("results that nobody asked for");
  return hipSuccess;
}

static unsigned char *const fake = reinterpret_cast<unsigned char *>(uintptr_t(1) << 40);
static unsigned char *const ws = reinterpret_cast<unsigned char *>(uintptr_t(2) << 40);

static long launches() { return g_prompts + g_steps + g_sums + g_carries + g_chunks; }

int main() {
  long calls = 0, accepted = 0;
  const int Bs[] = {0, 1, 2, 64, 65, 5000, 1 << 20, 0x7fffffff - 65536}, Ts[] = {0, 1, 16, 17, 129, 8192, 1000000, 0x7fffffff - 65536, 0x7fffffff};
  for (int B : Bs) for (int T : Ts) for (int d : {64, 96, 128}) for (int Hkv : {1, 2, 3, 8, 16, 256}) for (int G : {1, 3, 4, 16}) for (int64_t stride : {0ll, 1ll << 24, 1ll << 25}) {
    const int Hq = Hkv * G;
    g_d = d;
    sts_prompt_params p;
    memset(&p, 0, sizeof(p));
    p.B = B; p.T = T; p.Hq = Hq; p.Hkv = Hkv; p.d = d;
    p.q = fake; p.k = fake; p.v = fake; p.out = fake; p.starts = reinterpret_cast<const int32_t *>(fake);
    p.q_stride_n = stride ? stride : Hq * d; p.q_stride_h = d; p.kv_stride_n = stride ? stride : Hkv * d; p.kv_stride_h = d;
    p.scale = 0.1f;
    const long before = launches();
    const sts_status rc = sts_prompt_attn(&p, nullptr);
    if (launches() - before != (rc == STS_OK && B && T ? 1 : 0)) fail("prompt: launches");
    if ((d == 96 || Hq > 256 || stride > 1 << 24) && rc != STS_EUNSUPPORTED) fail("prompt: accepted what it cannot");
    accepted += rc == STS_OK;
    ++calls;
    for (int max_len : {0, 1, 16, 17, 100, 3000, 0x7fffffff})
      for (int kind = 0; kind < 4; ++kind) {
        sts_linear_params l;
        memset(&l, 0, sizeof(l));
        l.B = B; l.T = T; l.Hq = Hq; l.Hkv = Hkv; l.d = d; l.max_len = max_len;
        l.k = fake; l.v = fake; l.decay = reinterpret_cast<const float *>(fake); l.decay_rows = kind & 1;
        l.q_stride_n = p.q_stride_n; l.q_stride_h = d; l.kv_stride_n = p.kv_stride_n; l.kv_stride_h = d;
        if (kind != 1) { l.q = fake; l.out = fake; }
        if (kind != 2) { l.state_out = reinterpret_cast<float *>(fake); l.state_out_stride = (int64_t)Hkv * d * d; l.num_slots_out = B; }
        if (kind != 3) l.starts = reinterpret_cast<const int32_t *>(fake);
        l.scale = 1.f;
        const size_t need = sts_linear_attn_workspace_bytes(&l);
        l.workspace = ws;
        l.workspace_bytes = need;
        g_ws_lo = ws;
        g_ws_hi = ws + need;
        const long first = launches();
        const sts_status got = sts_linear_attn(&l, nullptr);
        if (got == STS_OK && need == 0) fail("linear: the size query and the call disagree");
        if (got != STS_OK && launches() != first) fail("linear: kernels enqueued before a refusal");
        if (got == STS_EWORKSPACE) fail("linear: the workspace that was asked for is refused");
        if (got == STS_OK && B > 0 && launches() == first) fail("linear: nothing was done");
        if (got == STS_OK && B > 0 && need > 256) {
          const long then = launches();
          l.workspace_bytes = need - 257;
          if (sts_linear_attn(&l, nullptr) != STS_EWORKSPACE || launches() != then) fail("linear: short workspace accepted");
        }
        accepted += got == STS_OK;
        ++calls;
      }
  }
  if (!accepted || !g_prompts || !g_steps || !g_sums || !g_carries || !g_chunks) fail("a launcher was not reached: the driver does not check it");
  printf("host checks done: %ld calls, %ld accepted, %ld stub launches\n", calls, accepted, launches());
  return 0;
}
