// Host side of the layers over packed batches: sts_prompt_attn, sts_linear_attn. Argument checks, launch plans, workspaces.
#include <math.h>
#include <string.h>

#include "layers.h"

namespace {

inline size_t align256(size_t x) { return (x + 255) & ~(size_t)255; }
inline bool aligned(const void *p, size_t to) { return reinterpret_cast<uintptr_t>(p) % to == 0; }

// rows of bf16 heads: 16-byte loads, and offsets within 64 rows (a tile of keys) below 2^31 bytes
bool strides_ok(int64_t n, int64_t h, int d) { return n >= d && n % 8 == 0 && n <= (int64_t)1 << 24 && h >= 0 && h % 8 == 0; }

// what the calls have in common
sts_status validate(int B, int T, int Hq, int Hkv, int d, int out_dtype, float scale, int64_t kv_n, int64_t kv_h) {
  if (B < 0 || T < 0 || Hq < 1 || Hkv < 1 || Hq % Hkv != 0) return STS_EINVAL;
  if (d != 64 && d != 128) return STS_EUNSUPPORTED;
  if (Hq > STS_MAX_HEADS || Hq / Hkv > STS_MAX_GROUP) return STS_EUNSUPPORTED;
  if (out_dtype != STS_BF16 && out_dtype != STS_F32) return STS_EINVAL;
  if (!isfinite(scale * 1.44269504088896340736f)) return STS_EINVAL;
  if (!strides_ok(kv_n, kv_h, d)) return STS_EUNSUPPORTED;
  if ((int64_t)T * (Hq / Hkv) > 0x7fffffffll - 65536 || B > 0x7fffffff - 65536) return STS_EUNSUPPORTED;
  return STS_OK;
}

constexpr int64_t MOST_GROUPS = 1 << 24;      // workgroups of 256 threads that a grid's dimension holds

struct LinearPlan {
  bool step;                 // the recurrent form
  int32_t each, max_len;     // rows of a sequence without starts; rows of the longest
  int32_t segment, heads, numbers;
  bool several;              // a sequence may have more than one segment
  bool carry;                // states are handed on: between segments, and to the workgroups of a group
  size_t part_bytes, log_bytes;
  size_t total() const { return part_bytes + log_bytes ? part_bytes + log_bytes : 256; }
};

sts_status plan_linear(const sts_linear_params *p, LinearPlan &pl) {
  if (!p) return STS_EINVAL;
  const sts_status v = validate(p->B, p->T, p->Hq, p->Hkv, p->d, p->out_dtype, p->scale, p->kv_stride_n, p->kv_stride_h);
  if (v != STS_OK) return v;
  memset(&pl, 0, sizeof(pl));
  if (p->max_len < 0 || (!p->starts && p->B > 0 && p->T % p->B != 0)) return STS_EINVAL;
  pl.each = p->B > 0 ? p->T / p->B : 0;
  pl.max_len = !p->starts ? pl.each : p->max_len == 0 || p->max_len > p->T ? p->T : p->max_len;
  // Row by row up to 16 rows, by chunks (of 32, whose time hardly depends on how many rows there are) behind that. 16 rows of 32 heads in us, row by row
  // and by chunks: 8 sequences with groups of four heads 12.8 and 15.9, without groups 16.8 and 12.9; 64 sequences 44.8 and 53.6, 93 and 72; 12 rows of 64
  // 37.4 and 57.3, 80 and 72; 8 rows 29.2 and 52.8, 67 and 71. So batches without groups lose up to a quarter between 10 and 16 rows. They stay row by row, too: a
  // block's results are right to fp32 then, whatever the batch beside it, where those of chunks hold weights and states as bf16.
  pl.step = pl.max_len <= STS_LINEAR_STEP;
  if ((int64_t)p->B * p->Hkv * (p->d * p->d / 1024) >= MOST_GROUPS) return STS_EUNSUPPORTED;
  if (pl.step) return STS_OK;
  // Segments: as many as the chip runs workgroups at once, two on a compute unit (four of half the waves), less half a one for each sequence (its last is
  // not whole), but no fewer than half as many, and of 128 rows at least. In us, with so many, twice, three quarters and half as many: 8192 rows with 32 heads 119,
  // 144, 127, 117; six prompts of 77 to 6001 rows, 32 heads in groups of four, 90, 105, 100, 105, and six of 1000 to 12000 202, 213, 234, 284; sixteen
  // of 500 to 4000 rows, 16 heads of 64, 100, 106, 107, 121. (Where the rows divide evenly a segment has a chunk more than it need have.)
  // Two heads of a group go to one workgroup where groups are even.
  pl.heads = p->Hq / p->Hkv % 2 == 0 ? 2 : 1;
  const int64_t at_once = (int64_t)(p->d == 128 ? 2 : 4) * sts_cu_count() * pl.heads / p->Hq, left = at_once - p->B / 2 > at_once / 2 ? at_once - p->B / 2 : at_once / 2;
  int64_t segment = (p->T / (left > 0 ? left : 1) + STS_LINEAR_CHUNK) / STS_LINEAR_CHUNK * STS_LINEAR_CHUNK;
  if (segment < 128) segment = 128;
  const int64_t numbers = piece_numbers(p->T, segment, p->B);
  if (numbers * p->Hq + STS_XCDS * STS_MAX_GROUP >= MOST_GROUPS) return STS_EUNSUPPORTED;
  pl.segment = (int32_t)segment;
  pl.numbers = (int32_t)numbers;
  pl.several = pl.max_len > segment;
  pl.carry = pl.several || (p->out && p->Hq / p->Hkv > pl.heads);
  if (pl.carry) {
    pl.part_bytes = align256((size_t)numbers * p->Hkv * p->d * p->d * sizeof(float));
    pl.log_bytes = align256((size_t)numbers * p->Hkv * sizeof(double));
  }
  return STS_OK;
}

// a pool of states: its slots must hold one, and there must be one for every sequence where no list says which
sts_status validate_states(const void *pool, int64_t stride, int num_slots, const int32_t *slots, const sts_linear_params *p) {
  if (!pool) return slots ? STS_EINVAL : STS_OK;
  if (num_slots < 0 || (!slots && num_slots < p->B)) return STS_EINVAL;
  if (stride < (int64_t)p->Hkv * p->d * p->d || stride % 4 || !aligned(pool, 16)) return STS_EUNSUPPORTED;
  return STS_OK;
}

}  // namespace

extern "C" {

sts_status sts_prompt_attn(const sts_prompt_params *p, void *stream) {
  if (!p) return STS_EINVAL;
  const sts_status v = validate(p->B, p->T, p->Hq, p->Hkv, p->d, p->out_dtype, p->scale, p->kv_stride_n, p->kv_stride_h);
  if (v != STS_OK) return v;
  if (!strides_ok(p->q_stride_n, p->q_stride_h, p->d)) return STS_EUNSUPPORTED;
  const int G = p->Hq / p->Hkv;
  const int64_t numbers = piece_numbers((int64_t)p->T * G, STS_PROMPT_ROWS, p->B);
  if (numbers * p->Hkv >= MOST_GROUPS) return STS_EUNSUPPORTED;
  if (p->B == 0 || p->T == 0) return STS_OK;
  if (!p->q || !p->k || !p->v || !p->starts || !p->out) return STS_EINVAL;
  if (!aligned(p->q, 16) || !aligned(p->k, 16) || !aligned(p->v, 16) || !aligned(p->out, 16)) return STS_EUNSUPPORTED;
  PromptArgs a;
  memset(&a, 0, sizeof(a));
  a.q = static_cast<const uint16_t *>(p->q);
  a.k = static_cast<const uint16_t *>(p->k);
  a.v = static_cast<const uint16_t *>(p->v);
  a.q_stride_n = p->q_stride_n; a.q_stride_h = p->q_stride_h; a.kv_stride_n = p->kv_stride_n; a.kv_stride_h = p->kv_stride_h;
  a.seqs = {p->starts, p->B, p->T, 0};
  a.Hq = p->Hq; a.Hkv = p->Hkv; a.G = G;
  a.numbers = (int32_t)numbers;
  a.scale = p->scale;
  a.scale_log2 = p->scale * 1.44269504088896340736f;
  a.by_numbers = divide_by(a.numbers);
  a.by_group = divide_by(G);
  a.out = p->out;
  a.lse_out = p->lse_out;
  a.out_dtype = p->out_dtype;
  hipStream_t s = static_cast<hipStream_t>(stream);
  return sts_run_kernel(STS_K_PROMPT, s, [&] { return launch_prompt_attn(a, p->d, s); }) == hipSuccess ? STS_OK : STS_EHIP;
}

size_t sts_linear_attn_workspace_bytes(const sts_linear_params *p) {
  LinearPlan pl;
  return plan_linear(p, pl) == STS_OK ? pl.total() : 0;
}

sts_status sts_linear_attn(const sts_linear_params *p, void *stream) {
  LinearPlan pl;
  sts_status v = plan_linear(p, pl);
  if (v != STS_OK) return v;
  if ((p->q == nullptr) != (p->out == nullptr)) return STS_EINVAL;
  if (p->q && !strides_ok(p->q_stride_n, p->q_stride_h, p->d)) return STS_EUNSUPPORTED;
  v = validate_states(p->state, p->state_stride, p->num_slots, p->slots, p);
  if (v != STS_OK) return v;
  v = validate_states(p->state_out, p->state_out_stride, p->num_slots_out, p->slots_out, p);
  if (v != STS_OK) return v;
  if (!aligned(p->q, 16) || !aligned(p->k, 16) || !aligned(p->v, 16) || !aligned(p->out, 16)) return STS_EUNSUPPORTED;
  if (p->B == 0) return STS_OK;
  if (p->T > 0 && (!p->k || !p->v || !p->decay)) return STS_EINVAL;
  if (!p->out && !p->state_out) return STS_OK;         // nothing is asked for
  LinearArgs a;
  memset(&a, 0, sizeof(a));
  a.q = static_cast<const uint16_t *>(p->q);
  a.k = static_cast<const uint16_t *>(p->k);
  a.v = static_cast<const uint16_t *>(p->v);
  a.q_stride_n = p->q_stride_n; a.q_stride_h = p->q_stride_h; a.kv_stride_n = p->kv_stride_n; a.kv_stride_h = p->kv_stride_h;
  a.decay = p->decay;
  a.decay_rows = p->decay_rows;
  a.seqs = {p->starts, p->B, p->T, pl.each};
  a.lens = p->lens;
  a.max_len = pl.max_len;
  a.Hq = p->Hq; a.Hkv = p->Hkv; a.G = p->Hq / p->Hkv;
  a.scale = p->scale;
  a.state = p->state; a.slots = p->slots; a.state_stride = p->state_stride; a.num_slots = p->num_slots;
  a.state_out = p->state_out; a.slots_out = p->slots_out; a.state_out_stride = p->state_out_stride; a.num_slots_out = p->num_slots_out;
  a.out = p->out;
  a.out_dtype = p->out_dtype;
  a.by_heads = divide_by(a.Hkv);
  a.by_group = divide_by(a.G);
  hipStream_t s = static_cast<hipStream_t>(stream);
  const int d = p->d;
  if (pl.step) return sts_run_kernel(STS_K_LINEAR_STEP, s, [&] { return launch_linear_step(a, d, s); }) == hipSuccess ? STS_OK : STS_EHIP;
  a.segment = pl.segment;
  a.numbers = pl.numbers;
  a.by_segment = divide_by(a.segment);
  a.heads = pl.heads;
  a.by_turns = divide_by(a.G / a.heads);
  if (pl.carry) {
    if (!p->workspace || p->workspace_bytes < pl.part_bytes + pl.log_bytes || !aligned(p->workspace, 256)) return STS_EWORKSPACE;
    a.part = static_cast<float *>(p->workspace);
    a.part_log = reinterpret_cast<double *>(static_cast<unsigned char *>(p->workspace) + pl.part_bytes);
  }
  hipError_t rc = hipSuccess;
  if (pl.several || !p->out) rc = sts_run_kernel(STS_K_LINEAR_SUMS, s, [&] { return launch_linear_sums(a, d, s); });
  if (rc == hipSuccess && pl.carry) rc = sts_run_kernel(STS_K_LINEAR_CARRY, s, [&] { return launch_linear_carry(a, d, s); });
  if (rc == hipSuccess && p->out) rc = sts_run_kernel(STS_K_LINEAR_CHUNKS, s, [&] { return launch_linear_chunks(a, d, s); });
  return rc == hipSuccess ? STS_OK : STS_EHIP;
}

}  // extern "C"
