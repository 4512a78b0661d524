// Host side of the speculative decoding calls: argument checks, the tree's masks, launch
// records. Every check runs before the first launch.
#include <cstring>

#include "draft.h"
#include "host.h"

namespace tu {

namespace {

static_assert(kMaxDraft == TU_MAX_DRAFT, "draft size");

// Nothing may leave a C entry as an exception (a failed host allocation, in practice).
template <class F>
int guarded(F&& body) {
  try {
    return body();
  } catch (...) {
    return fail(TU_ERR_ARG, "out of host memory");
  }
}

int check_draft(const tu_draft* d) {
  if (!d) return fail(TU_ERR_ARG, "null draft");
  if (d->n < 0 || d->n > TU_MAX_DRAFT) return fail(TU_ERR_ARG, "a draft has 0 .. %d nodes", TU_MAX_DRAFT);
  if (d->n > 0 && !d->parent) return fail(TU_ERR_ARG, "null parent array");
  for (int i = 0; i < d->n; ++i)
    if (d->parent[i] < -1 || d->parent[i] >= i)
      return fail(TU_ERR_ARG, "node %d: parent %d is neither -1 nor an earlier node", i, (int)d->parent[i]);
  return TU_OK;
}

int check_norm(const tu_qk_norm* m) {
  if (!m) return TU_OK;
  if (m->kind != TU_NORM_NONE && m->kind != TU_NORM_RMS && m->kind != TU_NORM_L2)
    return fail(TU_ERR_ARG, "unknown norm %d", (int)m->kind);
  if (!std::isfinite(m->eps) || m->eps < 0.f) return fail(TU_ERR_ARG, "eps must be finite and not negative");
  if (!std::isfinite(m->weight_offset)) return fail(TU_ERR_ARG, "weight_offset must be finite");
  if ((m->q_weight && !aligned16(m->q_weight)) || (m->k_weight && !aligned16(m->k_weight)))
    return fail(TU_ERR_ARG, "norm weights must be 16-byte aligned");
  return TU_OK;
}

// Depths of the nodes (0: a root).
void draft_depths(const tu_draft* d, uint8_t* depth) {
  for (int i = 0; i < d->n; ++i) depth[i] = d->parent[i] < 0 ? 0 : (uint8_t)(depth[d->parent[i]] + 1);
}

void draft_masks(const tu_draft* d, DraftMasks* m) {
  for (int i = 0; i < d->n; ++i) {
    const int p = d->parent[i];
    m->m[i][0] = p < 0 ? 0 : m->m[p][0];
    m->m[i][1] = p < 0 ? 0 : m->m[p][1];
    m->m[i][i >> 6] |= 1ull << (i & 63);
  }
}

int check_rows(const char* what, const void* in, int64_t stride, int64_t heads, int head_dim, int64_t T) {
  if (!in) return fail(TU_ERR_ARG, "null %s", what);
  if (!aligned16(in)) return fail(TU_ERR_ARG, "%s must be 16-byte aligned", what);
  if (stride % 8 || stride < 0 || (T > 1 && stride < heads * head_dim) || stride > INT32_MAX)
    return fail(TU_ERR_ARG, "%s: token stride %lld (a multiple of 8, at least %lld)", what, (long long)stride,
                (long long)(heads * head_dim));
  return TU_OK;
}

// Lanes that turn the angle rates, the norm and the work of one lane group.
void norm_record(const tu_attn_params* p, const tu_qk_norm* norm, int64_t T, NormArgs* a) {
  const double r = std::max(1, (int)p->rotary_dim), log2_theta = std::log2(p->rope_theta);
  for (int l = 0; l < 16; ++l) a->turn_lane[l] = std::exp2(-16.0 * l / r * log2_theta) * 0.15915494309189535;
  for (int e = 0; e < 8; ++e) a->turn_elem[e] = std::exp2(-2.0 * e / r * log2_theta);
  a->T = (int32_t)T;
  a->rotary = p->rotary_dim;
  a->kind = norm ? norm->kind : TU_NORM_NONE;
  a->eps = norm ? norm->eps : 0.f;
  a->weight_offset = norm ? norm->weight_offset : 0.f;
  a->weight[0] = norm ? static_cast<const bf16_t*>(norm->q_weight) : nullptr;
  a->weight[1] = norm ? static_cast<const bf16_t*>(norm->k_weight) : nullptr;
  const int heads = a->heads_end[2];
  // A workgroup takes 2 or 4 tokens where that leaves the chip full of them (eight per CU fit; 16 + 2
  // heads of 256, 1, 2 or 4 a workgroup: 2,048 tokens 12.0, 12.7, 16.3 us; 4,096 21.2, 19.4, 23.1;
  // 8,191 34.0, 32.2, 31.8); with few tokens their heads go to several, so that every lane group has a row.
  const int groups = 256 * 16 / p->head_dim;
  a->tokens = T > 3 * 8 * kCus ? 4 : T > 8 * kCus ? 2 : 1;
  const int most = (heads + groups - 1) / groups;
  a->head_parts = (int32_t)std::max<int64_t>(1, std::min<int64_t>(most, 4 * kCus / T));
  a->part_heads = (heads + a->head_parts - 1) / a->head_parts;
}

// Splits of the key range and rows of a workgroup (in waves of 32) of the attention, by their estimated time.
// A workgroup holds a CU. In microseconds, as fitted to launches over 0 to 50,000 rows, trees of 1 to 128
// nodes and four head layouts (the choice is 1.6 % behind the best of the forced ones in the mean, 13 % at worst: 128
// nodes over 12,000 rows of 8 heads of 128): a stage takes 1.0 +
// 0.03 a wave with rows (0.7 of that with head_dim 64, whose stages are half as long), a wave's queries and outputs 0.1,
// those of a second wave on a SIMD 0.6, the join's launch 2.8 and its partial outputs a microsecond for 2 MB on
// their way through memory; what the tiles read again costs one for 40 MB. So short contexts take one split and small tiles (16 + 2 heads of 256, 64
// nodes over 40 rows: 9.9 us in 16 tiles of one wave, 14.5 in two of eight, 15.0 with four splits), long ones
// one tile and a split for every CU (64 nodes over 24,000 rows: 40.6 us in two tiles of eight waves, 42.8 in
// four of four; 24 nodes over 3,000: 14.2 in three tiles of two and 32 splits, as chosen, 16.2 in one of six, 20.6 with 95 splits).
struct DraftPlan {
  int splits;
  int tile_waves;
};

DraftPlan draft_plan(const tu_attn_params* p, int64_t n, int64_t len) {
  const int64_t Hkv = p->n_kv_heads, waves = std::max<int64_t>(1, (n * (p->n_q_heads / Hkv) + 31) / 32);
  const int64_t keys = draft_stage_keys(p->head_dim), stages = std::max<int64_t>(1, (len + n + keys - 1) / keys);
  // a split's rows span less than 2^31 bytes (its loads' offsets are 32 bits wide), with the stages loaded past its end
  const int64_t stage_bytes = keys * Hkv * p->head_dim * 2;
  const int64_t fewest = (stages * stage_bytes) / (INT32_MAX - 8 * stage_bytes) + 1;
  const double partial = n * p->n_q_heads * p->head_dim * 2.0 / 2.0e6;   // of a split
  const double half = p->head_dim == 64 ? 0.7 : 1.0, read = (p->head_dim == 64 ? 16 : 32) * 1024 / 40.0e6;   // of a stage
  DraftPlan best{1, 1};
  double least = 0.0;
  for (int64_t w = 1; w <= std::min<int64_t>(waves, kDraftRows / 32); ++w) {
    const int64_t tiles = (waves + w - 1) / w;
    if ((waves + tiles - 1) / tiles != w) continue;   // as many tiles of fewer waves do
    const double stage = (1.0 + 0.03 * w) * half;
    const double rows = 0.1 * std::min<int64_t>(w, 4) + 0.6 * std::max<int64_t>(0, w - 4);
    // stages of a split: with k of them the time is k stage + (stages / k) partial, but one workgroup a CU
    const int64_t most = std::max<int64_t>(1, kCus / (Hkv * tiles)), k0 = (stages + most - 1) / most;
    const int64_t k = std::max(k0, (int64_t)(std::sqrt(stages * partial / stage) + 0.5));
    const int64_t many = p->kv_splits > 0 ? p->kv_splits : k == k0 ? most : (stages + k - 1) / k;
    for (const int64_t want : {many, p->kv_splits > 0 ? many : (int64_t)1}) {
      const int64_t s = std::max<int64_t>(1, std::min<int64_t>({std::max(want, fewest), stages, kMaxDraftSplits}));
      const int64_t turns = (Hkv * tiles * s + kCus - 1) / kCus;
      const double time = turns * (rows + (stages + s - 1) / s * stage) + (s > 1 ? 2.8 + s * partial : 0.0) +
                          Hkv * tiles * stages * read;
      if (least == 0.0 || time < least) {
        least = time;
        best = {(int)s, (int)w};
      }
    }
  }
  return best;
}

// Partial rows of a split: those of whole waves.
int64_t wave_rows(const tu_attn_params* p, int64_t n) { return (n * (p->n_q_heads / p->n_kv_heads) + 31) / 32 * 32 * p->n_kv_heads; }

size_t attention_ws(const tu_attn_params* p, int64_t n, int splits) {
  if (splits <= 1) return kStatusBytes;
  const size_t rows = (size_t)splits * wave_rows(p, n);
  return kStatusBytes + align_up(rows * p->head_dim * sizeof(_Float16)) + align_up(rows * 2 * sizeof(float));
}

// At least attention_ws of every plan for 1 .. n nodes over 0 .. len rows. Neither splits nor rows of a workgroup
// rise with either number (draft_plan weighs them against each other), so its own formula for the most
// splits is taken with the fewest tiles and the longest context, for every number of nodes.
size_t attention_ws_bound(const tu_attn_params* p, int64_t n, int64_t len) {
  const int64_t Hkv = p->n_kv_heads, keys = draft_stage_keys(p->head_dim), stage_bytes = keys * Hkv * p->head_dim * 2;
  size_t most = kStatusBytes;
  for (int64_t i = 1; i <= n; ++i) {
    const int64_t waves = wave_rows(p, i) / 32 / Hkv, tiles = (waves + kDraftRows / 32 - 1) / (kDraftRows / 32);
    const int64_t stages = (len + i + keys - 1) / keys;
    const int64_t fewest = (stages * stage_bytes) / (INT32_MAX - 8 * stage_bytes) + 1;
    const int64_t many = p->kv_splits > 0 ? p->kv_splits : std::max<int64_t>(1, kCus / (Hkv * tiles));
    most = std::max(most, attention_ws(p, i, (int)std::min<int64_t>({std::max(many, fewest), stages, kMaxDraftSplits})));
  }
  return most;
}

// The delta kernels' grids and offsets are 32 bits wide.
int check_delta_heads(const tu_delta_params* p) {
  if (int e = check_delta(p)) return e;
  if (p->n_v_heads > UINT16_MAX) return fail(TU_ERR_ARG, "too many heads");
  return TU_OK;
}

int check_channels(const char* what, int i, int32_t channels) {
  if (channels <= 0 || channels % 8) return fail(TU_ERR_ARG, "%s %d: channels must be a positive multiple of 8", what, i);
  if ((int64_t)channels * TU_MAX_DRAFT > INT32_MAX) return fail(TU_ERR_ARG, "%s %d: too many channels", what, i);
  return TU_OK;
}

constexpr size_t kVerifyBytes = kStatusBytes + (kMaxDraft + 1) * kDrawMaxBlocks * sizeof(double);

int check_workspace(const void* ws, size_t bytes, size_t need) {
  if (!ws || bytes < need) return fail(TU_ERR_WORKSPACE, "workspace of %zu bytes, %zu needed", bytes, need);
  if (!aligned16(ws)) return fail(TU_ERR_WORKSPACE, "workspace must be 16-byte aligned");
  return TU_OK;
}

}  // namespace

}  // namespace tu

using namespace tu;

extern "C" {

int qk_norm_rope(const tu_attn_params* p, const tu_qk_norm* norm, const void* q, int64_t q_stride, const void* k,
                 int64_t k_stride, int64_t T, int64_t first_pos, const int32_t* pos, void* q_out, int64_t q_out_stride,
                 void* k_out, int64_t k_out_stride, void* stream) {
  return guarded([&]() -> int {
    if (int e = check_attn(p)) return e;
    if (int e = check_norm(norm)) return e;
    if (T < 0) return fail(TU_ERR_ARG, "negative T");
    if (!pos && (first_pos < 0 || first_pos > INT32_MAX - T))
      return fail(TU_ERR_ARG, "positions outside the int32 range");
    if (pos && (reinterpret_cast<uintptr_t>(pos) & 3)) return fail(TU_ERR_ARG, "misaligned positions");
    if (T * (int64_t)(p->n_q_heads + p->n_kv_heads) > INT32_MAX / 2 || T > INT32_MAX / 2)
      return fail(TU_ERR_ARG, "T too large");
    if (T == 0) return ok();
    if (!q && !k) return fail(TU_ERR_ARG, "neither queries nor keys");
    const int D = p->head_dim;
    if (q) {
      if (int e = check_rows("q", q, q_stride, p->n_q_heads, D, T)) return e;
      if (int e = check_rows("q_out", q_out, q_out_stride, p->n_q_heads, D, T)) return e;
    }
    if (k) {
      if (int e = check_rows("k", k, k_stride, p->n_kv_heads, D, T)) return e;
      if (int e = check_rows("k_out", k_out, k_out_stride, p->n_kv_heads, D, T)) return e;
    }
    NormArgs a{};
    a.in[0] = static_cast<const bf16_t*>(q);
    a.in[1] = static_cast<const bf16_t*>(k);
    a.out[0] = static_cast<bf16_t*>(q_out);
    a.out[1] = static_cast<bf16_t*>(k_out);
    a.in_stride[0] = q_stride;
    a.in_stride[1] = k_stride;
    a.out_stride[0] = q_out_stride;
    a.out_stride[1] = k_out_stride;
    a.heads_end[0] = q ? p->n_q_heads : 0;
    a.heads_end[1] = a.heads_end[0] + (k ? p->n_kv_heads : 0);
    a.heads_end[2] = a.heads_end[1];
    a.pos = pos;
    a.first_pos = first_pos;
    norm_record(p, norm, T, &a);
    hipStream_t st = static_cast<hipStream_t>(stream);
    if (int e = hip_check(timed("qk_norm_rope", st, [&] { return launch_qk_norm(a, D, st); }), "qk norm")) return e;
    return ok();
  });
}

int draft_append(const tu_seq* seq, void* k_cache, void* v_cache, const tu_attn_params* p, const tu_qk_norm* norm,
                 const tu_draft* draft, const void* q, int64_t q_stride, const void* k, int64_t k_stride,
                 const void* v, int64_t v_stride, void* q_hat, void* stream) {
  return guarded([&]() -> int {
    if (int e = check_seq(seq)) return e;
    if (int e = check_attn(p)) return e;
    if (int e = check_norm(norm)) return e;
    if (int e = check_draft(draft)) return e;
    const int n = draft->n, D = p->head_dim;
    if (seq->len + n > seq->capacity)
      return fail(TU_ERR_CAPACITY, "%lld rows + %d drafted exceed capacity %lld", (long long)seq->len, n,
                  (long long)seq->capacity);
    if (seq->next_pos + n > INT32_MAX) return fail(TU_ERR_ARG, "positions overflow int32");
    if (n == 0) return ok();
    if (!k_cache || !v_cache || !q_hat) return fail(TU_ERR_ARG, "null tensor");
    if (!aligned16(k_cache) || !aligned16(v_cache) || !aligned16(q_hat))
      return fail(TU_ERR_ARG, "tensors must be 16-byte aligned");
    if (int e = check_rows("q", q, q_stride, p->n_q_heads, D, n)) return e;
    if (int e = check_rows("k", k, k_stride, p->n_kv_heads, D, n)) return e;
    if (int e = check_rows("v", v, v_stride, p->n_kv_heads, D, n)) return e;
    NormArgs a{};
    const int64_t row = (int64_t)p->n_kv_heads * D;
    a.in[0] = static_cast<const bf16_t*>(q);
    a.in[1] = static_cast<const bf16_t*>(k);
    a.in[2] = static_cast<const bf16_t*>(v);
    a.out[0] = static_cast<bf16_t*>(q_hat);
    a.out[1] = static_cast<bf16_t*>(k_cache) + seq->len * row;
    a.out[2] = static_cast<bf16_t*>(v_cache) + seq->len * row;
    a.in_stride[0] = q_stride;
    a.in_stride[1] = k_stride;
    a.in_stride[2] = v_stride;
    a.out_stride[0] = (int64_t)p->n_q_heads * D;
    a.out_stride[1] = a.out_stride[2] = row;
    a.heads_end[0] = p->n_q_heads;
    a.heads_end[1] = a.heads_end[0] + p->n_kv_heads;
    a.heads_end[2] = a.heads_end[1] + p->n_kv_heads;
    a.first_pos = seq->next_pos;
    a.use_depth = 1;
    draft_depths(draft, a.depth);
    norm_record(p, norm, n, &a);
    hipStream_t st = static_cast<hipStream_t>(stream);
    if (int e = hip_check(timed("qk_norm_rope", st, [&] { return launch_qk_norm(a, D, st); }), "draft append")) return e;
    return ok();
  });
}

size_t draft_attention_workspace_size(const tu_attn_params* p, int32_t n, int64_t len) {
  if (check_attn(p) || n < 0 || n > TU_MAX_DRAFT || len < 0 || len > INT32_MAX / 2) return 0;
  return attention_ws(p, n, draft_plan(p, n, len).splits);
}

size_t draft_attention_workspace_bound(const tu_attn_params* p, int32_t max_n, int64_t max_len) {
  if (check_attn(p) || max_n < 0 || max_n > TU_MAX_DRAFT || max_len < 0 || max_len > INT32_MAX / 2) return 0;
  return attention_ws_bound(p, max_n, max_len);
}

int draft_attention(const tu_seq* seq, const void* k_cache, const void* v_cache, const tu_attn_params* p,
                    const tu_draft* draft, const void* q_hat, void* out, void* workspace, size_t workspace_bytes,
                    void* stream) {
  return guarded([&]() -> int {
    if (int e = check_seq(seq)) return e;
    if (int e = check_attn(p)) return e;
    if (int e = check_draft(draft)) return e;
    const int n = draft->n;
    if (seq->len + n > seq->capacity)
      return fail(TU_ERR_CAPACITY, "%lld rows + %d drafted exceed capacity %lld", (long long)seq->len, n,
                  (long long)seq->capacity);
    if (seq->len > INT32_MAX / 2) return fail(TU_ERR_ARG, "context too long");
    if ((int64_t)n * p->n_q_heads * p->head_dim * 2 > INT32_MAX) return fail(TU_ERR_ARG, "too many heads");   // out, in bytes
    if (n == 0) return ok();
    if (!k_cache || !v_cache || !q_hat || !out) return fail(TU_ERR_ARG, "null tensor");
    if (!aligned16(k_cache) || !aligned16(v_cache) || !aligned16(q_hat) || !aligned16(out))
      return fail(TU_ERR_ARG, "tensors must be 16-byte aligned");
    const DraftPlan plan = draft_plan(p, n, seq->len);
    const int splits = plan.splits;
    if (int e = check_workspace(workspace, workspace_bytes, attention_ws(p, n, splits))) return e;
    DraftAttnArgs a{};
    a.q_hat = static_cast<const bf16_t*>(q_hat);
    a.k_cache = static_cast<const bf16_t*>(k_cache);
    a.v_cache = static_cast<const bf16_t*>(v_cache);
    a.out = static_cast<bf16_t*>(out);
    Arena ar(after_status(workspace));
    if (splits > 1) {
      const size_t rows = (size_t)splits * wave_rows(p, n);
      a.part_o = static_cast<_Float16*>(ar.take(rows * p->head_dim * sizeof(_Float16)));
      a.part_ml = static_cast<float*>(ar.take(rows * 2 * sizeof(float)));
    }
    a.status = call_status(workspace);
    a.len = (int32_t)seq->len;
    a.n = n;
    a.n_q_heads = p->n_q_heads;
    a.n_kv_heads = p->n_kv_heads;
    a.group = p->n_q_heads / p->n_kv_heads;
    a.n_waves = (n * a.group + 31) / 32;
    a.tile_waves = plan.tile_waves;
    a.n_tiles = (a.n_waves + plan.tile_waves - 1) / plan.tile_waves;
    a.n_splits = splits;
    const int keys = draft_stage_keys(p->head_dim), stages = (int)((seq->len + n + keys - 1) / keys);
    a.split_stages = stages / splits;
    a.more_stages = stages % splits;
    if ((int64_t)p->n_kv_heads * splits * a.n_tiles >= 1 << 21 || n * a.group >= 1 << 21)   // quotient() in the kernel
      return fail(TU_ERR_ARG, "too many heads");
    a.scale_log2 = p->softmax_scale * 1.4426950408889634f;
    draft_masks(draft, &a.seen);
    hipStream_t st = static_cast<hipStream_t>(stream);
    const int D = p->head_dim;
    if (int e = hip_check(timed("draft_attention", st, [&] { return launch_draft_attention(a, D, st); }), "draft attention"))
      return e;
    if (splits > 1)
      if (int e = hip_check(timed("draft_merge", st, [&] { return launch_draft_merge(a, D, st); }), "draft merge")) return e;
    return ok();
  });
}

int draft_short_conv(const tu_draft* draft, const tu_conv_tensor* tensors, int32_t n, int32_t width,
                     int32_t activation, void* stream) {
  return guarded([&]() -> int {
    if (int e = check_draft(draft)) return e;
    if (n < 0 || (n > 0 && !tensors)) return fail(TU_ERR_ARG, "bad tensor array");
    if (width < 1 || width > 8) return fail(TU_ERR_ARG, "width must be 1 .. 8");
    if (activation != TU_CONV_IDENTITY && activation != TU_CONV_SILU) return fail(TU_ERR_ARG, "unknown activation");
    for (int i = 0; i < n; ++i) {
      const tu_conv_tensor& t = tensors[i];
      if (t.T != draft->n) return fail(TU_ERR_ARG, "tensor %d has %lld rows, the draft %d nodes", i, (long long)t.T, draft->n);
      if (int e = check_channels("tensor", i, t.channels)) return e;
      if (draft->n == 0) continue;
      if (!t.x || !t.weight || !t.out || (!t.state && width > 1)) return fail(TU_ERR_ARG, "tensor %d: null pointer", i);
      if (!aligned16(t.x) || !aligned16(t.weight) || !aligned16(t.out) || (t.state && !aligned16(t.state)))
        return fail(TU_ERR_ARG, "tensor %d: not 16-byte aligned", i);
    }
    if (draft->n == 0) return ok();
    hipStream_t st = static_cast<hipStream_t>(stream);
    DraftConvArgs a{};
    a.n = draft->n;
    a.width = width;
    for (int i = 0; i < draft->n; ++i)
      for (int t = 0, at = i; t < 8; ++t) {
        a.up[i][t] = (int8_t)at;
        at = at >= 0 ? draft->parent[at] : at - 1;
      }
    for (int j0 = 0; j0 < n; j0 += kMaxConvJobs) {
      a.n_jobs = std::min(kMaxConvJobs, n - j0);
      for (int j = 0; j < a.n_jobs; ++j) {
        const tu_conv_tensor& t = tensors[j0 + j];
        a.job[j] = ConvJob{};
        a.job[j].state = static_cast<bf16_t*>(t.state);
        a.job[j].x = static_cast<const bf16_t*>(t.x);
        a.job[j].w = static_cast<const bf16_t*>(t.weight);
        a.job[j].out = static_cast<bf16_t*>(t.out);
        a.job[j].C = t.channels;
        a.job[j].act = activation == TU_CONV_SILU;
      }
      if (int e = hip_check(timed("draft_conv", st, [&] { return launch_draft_conv(a, st); }), "draft convolution")) return e;
    }
    return ok();
  });
}

int draft_delta_rule(const float* state, const void* q, const void* k, const void* v, const float* beta,
                     const float* g, const tu_delta_params* p, const tu_draft* draft, float* out, void* stream) {
  return guarded([&]() -> int {
    if (int e = check_delta_heads(p)) return e;
    if (int e = check_draft(draft)) return e;
    if (draft->n == 0) return ok();
    if (!state || !q || !k || !v || !beta || !g || !out) return fail(TU_ERR_ARG, "null tensor");
    if (!aligned16(state) || !aligned16(q) || !aligned16(k) || !aligned16(v) || !aligned16(out))
      return fail(TU_ERR_ARG, "tensors must be 16-byte aligned");
    DraftDeltaArgs a{};
    a.state = state;
    a.q = static_cast<const bf16_t*>(q);
    a.k = static_cast<const bf16_t*>(k);
    a.v = static_cast<const bf16_t*>(v);
    a.beta = beta;
    a.g = g;
    a.out = out;
    a.n = draft->n;
    a.n_k_heads = p->n_k_heads;
    a.n_v_heads = p->n_v_heads;
    a.scale = p->scale;
    draft_masks(draft, &a.seen);
    hipStream_t st = static_cast<hipStream_t>(stream);
    if (int e = hip_check(timed("draft_delta", st, [&] { return launch_draft_delta(a, p->d_k, st); }), "draft delta rule"))
      return e;
    return ok();
  });
}

size_t draft_verify_workspace_size(int32_t n, int64_t vocab) {
  if (n < 0 || n > TU_MAX_DRAFT || vocab < 0 || vocab > INT32_MAX) return 0;
  return kVerifyBytes;
}

int draft_verify(const tu_draft* draft, const int32_t* tokens, const float* target, int64_t target_stride,
                 const float* proposal, int64_t proposal_stride, int64_t vocab, const float* u, int32_t* result,
                 void* workspace, size_t workspace_bytes, void* stream) {
  return guarded([&]() -> int {
    if (int e = check_draft(draft)) return e;
    const int n = draft->n;
    if (n == 0) return fail(TU_ERR_ARG, "nothing to verify: the draft has no root");
    for (int i = 1; i < n; ++i)
      if (draft->parent[i] < 0) return fail(TU_ERR_ARG, "node %d: a verified draft has one root, node 0", i);
    if (vocab < 1 || vocab > INT32_MAX / 2) return fail(TU_ERR_ARG, "vocab outside [1, 2^30)");
    if (!tokens || !target || !u || !result) return fail(TU_ERR_ARG, "null tensor");
    if (target_stride < vocab || (proposal && proposal_stride < vocab)) return fail(TU_ERR_ARG, "row stride below vocab");
    const uintptr_t bits = (uintptr_t)tokens | (uintptr_t)target | (uintptr_t)proposal | (uintptr_t)u | (uintptr_t)result;
    if (bits & 3) return fail(TU_ERR_ARG, "tensors must be 4-byte aligned");
    if (int e = check_workspace(workspace, workspace_bytes, kVerifyBytes)) return e;
    DraftVerifyArgs a{};
    a.tokens = tokens;
    a.target = target;
    a.proposal = proposal;
    a.u = u;
    a.result = result;
    a.target_stride = target_stride;
    a.proposal_stride = proposal_stride;
    a.vocab = vocab;
    Arena ar(after_status(workspace));
    a.part = static_cast<unsigned long long*>(ar.take((kMaxDraft + 1) * kDrawMaxBlocks * sizeof(double)));
    a.status = call_status(workspace);
    a.n = n;
    // as few whole blocks of a workgroup's elements a slice as kDrawMaxBlocks slices allow
    const int64_t block = kDrawThreads * kDrawPer, blocks = (vocab + block - 1) / block;
    a.slice = (blocks + kDrawMaxBlocks - 1) / kDrawMaxBlocks * block;
    a.n_blocks = (int32_t)((vocab + a.slice - 1) / a.slice);
    a.polls = kDrawPolls;
    a.wide = ((uintptr_t)target & 15) == 0 && target_stride % 4 == 0 &&
             (!proposal || (((uintptr_t)proposal & 15) == 0 && proposal_stride % 4 == 0));
    uint8_t last[kMaxDraft] = {};    // last child so far
    for (int i = 1; i < n; ++i) {
      const int up = draft->parent[i];
      a.parent[i] = (uint8_t)up;
      if (last[up]) a.sibling[last[up]] = (uint8_t)i;
      else {
        a.child[up] = (uint8_t)i;
        a.first[i >> 6] |= 1ull << (i & 63);
      }
      last[up] = (uint8_t)i;
    }
    draft_masks(draft, &a.seen);
    hipStream_t st = static_cast<hipStream_t>(stream);
    if (int e = hip_check(timed("draft_verify", st, [&] { return launch_draft_clear(a, st); }), "draft verification")) return e;
    if (int e = hip_check(timed("draft_verify", st, [&] { return launch_draft_draw(a, st); }), "draft verification")) return e;
    return ok();
  });
}

int draft_accept(tu_seq* seq, const tu_draft* draft, const int32_t* path, int32_t n_path, const tu_layer_io* layers,
                 int32_t n_layers, const tu_attn_params* attn, const tu_delta_params* delta, const tu_conv_tensor* conv,
                 int32_t n_conv, int32_t width, void* stream) {
  return guarded([&]() -> int {
    if (int e = check_seq(seq)) return e;
    if (int e = check_draft(draft)) return e;
    if (n_path < 0 || n_path > draft->n || (n_path > 0 && !path)) return fail(TU_ERR_ARG, "bad path");
    for (int j = 0; j < n_path; ++j) {
      if (path[j] < 0 || path[j] >= draft->n) return fail(TU_ERR_ARG, "path[%d] = %d is no node", j, (int)path[j]);
      if (draft->parent[path[j]] != (j ? path[j - 1] : -1))
        return fail(TU_ERR_ARG, "path[%d] = %d does not continue the path", j, (int)path[j]);
    }
    if (n_layers < 0 || (n_layers > 0 && !layers)) return fail(TU_ERR_ARG, "bad layer array");
    if (n_conv < 0 || (n_conv > 0 && !conv)) return fail(TU_ERR_ARG, "bad convolution array");
    if (n_conv > 0 && (width < 1 || width > 8)) return fail(TU_ERR_ARG, "width must be 1 .. 8");
    if (seq->len + draft->n > seq->capacity)
      return fail(TU_ERR_CAPACITY, "%lld rows + %d drafted exceed capacity %lld", (long long)seq->len, (int)draft->n,
                  (long long)seq->capacity);
    if (seq->next_pos + n_path > INT32_MAX) return fail(TU_ERR_ARG, "positions overflow int32");
    int n_attn = 0, n_delta = 0;
    for (int l = 0; l < n_layers; ++l) {
      const tu_layer_io& L = layers[l];
      if (L.kind == TU_LAYER_ATTN) {
        ++n_attn;
        if (!L.k_cache || !L.v_cache || !L.k_cache[0] || !L.v_cache[0]) return fail(TU_ERR_ARG, "layer %d: null cache", l);
        if (!aligned16(L.k_cache[0]) || !aligned16(L.v_cache[0])) return fail(TU_ERR_ARG, "layer %d: not 16-byte aligned", l);
      } else if (L.kind == TU_LAYER_DELTA) {
        ++n_delta;
        if (!L.state || !L.state[0] || !L.k || !L.v || !L.beta || !L.g) return fail(TU_ERR_ARG, "layer %d: null tensor", l);
        if (!aligned16(L.state[0]) || !aligned16(L.k) || !aligned16(L.v))
          return fail(TU_ERR_ARG, "layer %d: not 16-byte aligned", l);
      } else {
        return fail(TU_ERR_ARG, "layer %d: unknown kind", l);
      }
    }
    if (n_attn)
      if (int e = check_attn(attn)) return e;
    if (n_delta)
      if (int e = check_delta_heads(delta)) return e;
    for (int i = 0; i < n_conv; ++i) {
      const tu_conv_tensor& t = conv[i];
      if (t.T != draft->n) return fail(TU_ERR_ARG, "convolution %d has %lld rows, the draft %d nodes", i, (long long)t.T, (int)draft->n);
      if (int e = check_channels("convolution", i, t.channels)) return e;
      if (width > 1 && (!t.state || !t.x)) return fail(TU_ERR_ARG, "convolution %d: null pointer", i);
      if (width > 1 && (!aligned16(t.state) || !aligned16(t.x))) return fail(TU_ERR_ARG, "convolution %d: not 16-byte aligned", i);
    }
    std::vector<tu_interval> runs(seq->live, seq->live + seq->n_live);
    push_run(runs, seq->next_pos, seq->next_pos + n_path);
    if ((int64_t)runs.size() > seq->live_cap) return fail(TU_ERR_CAPACITY, "live-interval list full (%d)", seq->live_cap);
    if (n_path == 0) return ok();

    hipStream_t st = static_cast<hipStream_t>(stream);
    const int n_moved = width > 1 ? n_conv : 0;
    int la = 0, ld = 0, ic = 0;      // next attention layer, delta layer, convolution
    bool pos = true;
    while (pos || la < n_layers || ld < n_layers || ic < n_moved) {
      AcceptArgs a{};
      for (int j = 0; j < n_path; ++j) a.path[j] = (uint8_t)path[j];
      a.n_path = n_path;
      a.len = seq->len;
      a.next_pos = seq->next_pos;
      a.pos = pos ? seq->d_pos : nullptr;
      pos = false;
      if (n_attn) a.row_chunks = attn->n_kv_heads * attn->head_dim / 8;
      for (; la < n_layers && a.n_bufs + 2 <= kMaxAcceptBufs; ++la) {
        if (layers[la].kind != TU_LAYER_ATTN) continue;
        a.bufs[a.n_bufs++] = static_cast<bf16_t*>(layers[la].k_cache[0]);
        a.bufs[a.n_bufs++] = static_cast<bf16_t*>(layers[la].v_cache[0]);
      }
      if (n_delta) {
        a.n_k_heads = delta->n_k_heads;
        a.n_v_heads = delta->n_v_heads;
        a.d = delta->d_k;
      }
      for (; ld < n_layers && a.n_delta < kMaxAcceptDelta; ++ld) {
        const tu_layer_io& L = layers[ld];
        if (L.kind != TU_LAYER_DELTA) continue;
        a.delta[a.n_delta++] = AcceptDelta{L.state[0], static_cast<const bf16_t*>(L.k), static_cast<const bf16_t*>(L.v),
                                           L.beta, L.g};
      }
      a.width = width;
      for (; ic < n_moved && a.n_conv < kMaxAcceptConv; ++ic)
        a.conv[a.n_conv++] = AcceptConv{static_cast<bf16_t*>(conv[ic].state), static_cast<const bf16_t*>(conv[ic].x),
                                        conv[ic].channels, 0};
      if (int e = hip_check(timed("draft_accept", st, [&] { return launch_draft_accept(a, st); }), "draft acceptance"))
        return e;
    }
    commit_intervals(seq, runs);
    seq->len += n_path;
    seq->next_pos += n_path;
    return ok();
  });
}

}  // extern "C"
