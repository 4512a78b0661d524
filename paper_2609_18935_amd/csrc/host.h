// Host helpers shared by the translation units of the C ABI: error reporting, the call
// status, argument checks, the kernel timer.
#pragma once

#include <algorithm>
#include <atomic>
#include <cmath>
#include <cstdarg>
#include <cstdio>
#include <string>
#include <vector>

#include "common.h"
#include "tailupdate.h"

namespace tu {

inline thread_local std::string g_err;

inline int fail(int code, const char* fmt, ...) {
  char buf[512];
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(buf, sizeof(buf), fmt, ap);
  va_end(ap);
  g_err = buf;
  return code;
}

inline int ok() {
  g_err.clear();
  return TU_OK;
}

inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

constexpr size_t kAlign = 256;
inline size_t align_up(size_t x) { return (x + kAlign - 1) & ~(kAlign - 1); }

// Carves aligned regions out of a workspace; with base == nullptr it only measures.
struct Arena {
  char* base;
  size_t used = 0;
  explicit Arena(void* b) : base(static_cast<char*>(b)) {}
  void* take(size_t bytes) {
    void* p = base ? base + used : nullptr;
    used += align_up(bytes);
    return p;
  }
};

// The first kStatusBytes of every workspace hold the call's status: the tagged 64-bit
// word and, 64 bytes further, the number of the call that last ran there (CallStatus in
// common.h); the rest is carved by the planners.
constexpr size_t kStatusBytes = 256;
constexpr size_t kStatusLastOffset = 64;
inline std::atomic<uint32_t> g_calls{0};

// The status of a new call on workspace ws: numbers 1 .. 2^32 - 2, one per call of the process.
inline CallStatus call_status(void* ws) {
  uint32_t n;
  do n = g_calls.fetch_add(1, std::memory_order_relaxed) + 1;
  while (n == 0 || n == 0xFFFFFFFFu);
  CallStatus st{};
  st.word = static_cast<unsigned long long*>(ws);
  st.last = reinterpret_cast<uint32_t*>(static_cast<char*>(ws) + kStatusLastOffset);
  st.call = n;
  return st;
}
inline void* after_status(void* ws) { return ws ? static_cast<char*>(ws) + kStatusBytes : nullptr; }

inline int check_seq(const tu_seq* s) {
  if (!s) return fail(TU_ERR_ARG, "null context");
  if (s->len < 0 || s->capacity < s->len) return fail(TU_ERR_ARG, "len %lld outside [0, capacity %lld]",
                                                      (long long)s->len, (long long)s->capacity);
  if (s->n_live < 0 || s->n_live > s->live_cap) return fail(TU_ERR_ARG, "n_live outside [0, live_cap]");
  if (s->n_live > 0 && !s->live) return fail(TU_ERR_ARG, "null live-interval array");
  if (s->capacity > 0 && !s->d_pos) return fail(TU_ERR_ARG, "null d_pos");
  if (s->next_pos < 0 || s->next_pos > INT32_MAX) return fail(TU_ERR_ARG, "cursor outside the int32 position range");
  if (s->vt_rows < 0) return fail(TU_ERR_ARG, "negative vt_rows");
  int64_t total = 0, max_end = -1;
  for (int i = 0; i < s->n_live; ++i) {
    const tu_interval& iv = s->live[i];
    if (iv.end <= iv.begin || iv.begin < 0) return fail(TU_ERR_ARG, "empty or negative live run");
    if (i > 0 && iv.begin == s->live[i - 1].end)
      return fail(TU_ERR_ARG, "consecutive live runs %d and %d are position-contiguous (not merged)", i - 1, i);
    max_end = std::max(max_end, iv.end);
    total += iv.end - iv.begin;
  }
  if (max_end > s->next_pos) return fail(TU_ERR_ARG, "live position at or beyond the cursor");
  if (total != s->len) return fail(TU_ERR_ARG, "live runs cover %lld positions, len is %lld",
                                   (long long)total, (long long)s->len);
  std::vector<tu_interval> sorted(s->live, s->live + s->n_live);
  std::sort(sorted.begin(), sorted.end(), [](const tu_interval& x, const tu_interval& y) { return x.begin < y.begin; });
  for (size_t i = 1; i < sorted.size(); ++i)
    if (sorted[i].begin < sorted[i - 1].end) return fail(TU_ERR_ARG, "live runs overlap");
  return TU_OK;
}

// Appends a run in row order, merging it into the previous run when contiguous.
inline void push_run(std::vector<tu_interval>& iv, int64_t begin, int64_t end) {
  if (end <= begin) return;
  if (!iv.empty() && iv.back().end == begin) iv.back().end = end;
  else iv.push_back({begin, end});
}

inline int check_attn(const tu_attn_params* p) {
  if (!p) return fail(TU_ERR_ARG, "null attention parameters");
  if (p->n_kv_heads <= 0 || p->n_q_heads <= 0 || p->n_q_heads % p->n_kv_heads)
    return fail(TU_ERR_ARG, "n_q_heads must be a positive multiple of n_kv_heads");
  if (p->head_dim != 64 && p->head_dim != 128 && p->head_dim != 256)
    return fail(TU_ERR_ARG, "head_dim must be 64, 128 or 256");
  if (p->rotary_dim < 0 || p->rotary_dim > p->head_dim || (p->rotary_dim & 1))
    return fail(TU_ERR_ARG, "rotary_dim must be even and within [0, head_dim]");
  if (!(p->rope_theta > 0.0) || !std::isfinite(p->rope_theta)) return fail(TU_ERR_ARG, "rope_theta must be positive");
  if (!(p->softmax_scale > 0.f) || !std::isfinite(p->softmax_scale)) return fail(TU_ERR_ARG, "softmax_scale must be positive");
  if (p->kv_splits < 0 || p->kv_splits > 64) return fail(TU_ERR_ARG, "kv_splits must be in [0, 64]");
  if ((long)p->n_kv_heads * p->head_dim * 2 > kGatherStripeBytes) return fail(TU_ERR_ARG, "cache row too wide");
  return TU_OK;
}

inline int check_delta(const tu_delta_params* p) {
  if (!p) return fail(TU_ERR_ARG, "null delta parameters");
  if (p->n_k_heads <= 0 || p->n_v_heads <= 0 || p->n_v_heads % p->n_k_heads)
    return fail(TU_ERR_ARG, "n_v_heads must be a positive multiple of n_k_heads");
  if (p->d_k != p->d_v || (p->d_k != 64 && p->d_k != 128)) return fail(TU_ERR_ARG, "d_k = d_v must be 64 or 128");
  if (p->chunk != 16 && p->chunk != 32 && p->chunk != 64) return fail(TU_ERR_ARG, "chunk must be 16, 32 or 64");
  if (!std::isfinite(p->scale)) return fail(TU_ERR_ARG, "scale must be finite");
  return TU_OK;
}

inline int hip_check(hipError_t e, const char* what) {
  if (e != hipSuccess) return fail(TU_ERR_HIP, "%s: %s", what, hipGetErrorString(e));
  return TU_OK;
}

// ------------------------------------------------------------------ kernel timing

struct ProfRec {
  const char* name;
  hipEvent_t start;
  hipEvent_t stop;
};
inline thread_local bool g_prof = false;
inline thread_local std::vector<ProfRec> g_recs;
inline thread_local uint64_t g_launches = 0;   // kernels this thread has enqueued through timed()

// Runs `launch` (which enqueues one kernel on `st`), bracketed by events when profiling.
template <class F>
hipError_t timed(const char* name, hipStream_t st, F&& launch) {
  ++g_launches;
  if (!g_prof) return launch();
  ProfRec r{name, nullptr, nullptr};
  if (hipEventCreate(&r.start) != hipSuccess) return launch();
  if (hipEventCreate(&r.stop) != hipSuccess) {
    (void)hipEventDestroy(r.start);
    return launch();
  }
  (void)hipEventRecord(r.start, st);
  const hipError_t e = launch();
  (void)hipEventRecord(r.stop, st);
  g_recs.push_back(r);
  return e;
}

inline int commit_intervals(tu_seq* s, const std::vector<tu_interval>& iv) {
  if ((int64_t)iv.size() > s->live_cap) return fail(TU_ERR_CAPACITY, "live-interval list full (%d)", s->live_cap);
  for (size_t i = 0; i < iv.size(); ++i) s->live[i] = iv[i];
  s->n_live = (int32_t)iv.size();
  return TU_OK;
}

}  // namespace tu
