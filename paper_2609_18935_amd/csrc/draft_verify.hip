// Verification of a tree of drafted tokens against the target's probabilities.
//
// The children of a node are tried one after the other; after r rejections what is left of the
// target row is the r-fold normalised max(.. - q, 0). Unnormalised it is max(p - b q, 0) with
// one number b that grows by F = sum_t max(p(t) - b q(t), 0) with each rejection: F is all
// that a test needs of the row, so a rejection costs one pass over the rows of one node and
// an acceptance of a first child nothing. (A drafter's choice without probabilities is a
// point mass: the rejected tokens' entries are zero instead.)
//
// k_draft_clear (one workgroup) zeroes the counters of the passes. k_draft_draw: every
// workgroup reads the single probabilities that the tests need, of all nodes at once, and
// derives the same walk from them; where a node has a rejection, or no child is left to try,
// each sums its slice of the row in float64, publishes the sum, waits for the others
// (bounded; the few workgroups fit the chip many times over), and adds all of them up in one
// order. The workgroup whose slice holds the drawn token finds it. Bound by the latency of the
// passes; the rows themselves (a megabyte) are read once and stay in registers.
#include "draft.h"

namespace tu {

namespace {

constexpr long kSpinLimit = 1l << 20;   // polls of a bounded wait
constexpr int kClearThreads = kMaxDraft;
constexpr int kWaves = kDrawThreads / 64;

// What the tests of node i (as a child of its parent) need of the rows.
struct Odds {
  float p, q, u;
  int token;     // -1: outside the vocabulary
};

__device__ __forceinline__ Odds odds_of(const DraftVerifyArgs& a, int i) {
  Odds o{0.f, 1.f, 2.f, -1};
  const int up = i > 0 && i < a.n ? a.parent[i] : -1;
  if (up < 0) return o;
  const int x = a.tokens[i];
  o.u = a.u[i];
  if (x < 0 || x >= a.vocab) return o;
  o.token = x;
  o.p = a.target[up * a.target_stride + x];
  if (a.proposal) o.q = a.proposal[up * a.proposal_stride + x];
  return o;
}

__global__ __launch_bounds__(kClearThreads) void k_draft_clear(DraftVerifyArgs a) {
  status_mark(a.status);
  for (int i = threadIdx.x; i <= kMaxDraft; i += kClearThreads) a.arrived[i] = 0;
  for (int i = threadIdx.x; i < a.n + 2; i += kClearThreads) a.result[i] = i == 0 ? 0 : -1;
}

__device__ __forceinline__ double wave_sum(double x) {
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) x += __shfl_xor(x, d, 64);
  return x;
}

__global__ __launch_bounds__(kDrawThreads) void k_draft_draw(DraftVerifyArgs a) {
  __shared__ Odds s_odds[kMaxDraft];
  __shared__ uint64_t s_seen[kMaxDraft][2];
  __shared__ int s_parent[kMaxDraft];
  __shared__ unsigned long long s_first[2], s_on[2];   // accepted as first children; on the accepted path
  __shared__ double s_wave[kWaves];
  __shared__ double s_part[kDrawMaxBlocks];
  __shared__ int s_out[kMaxDraft];                     // rejected tokens of the row (point-mass drafts)
  __shared__ int s_mine[kMaxDraft];                    // those of this workgroup's slice
  __shared__ int s_found, s_best, s_expired;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int n = a.n, blk = blockIdx.x;
  const bool drawn = a.proposal != nullptr;

  if (tid < 2) s_first[tid] = 0;
  if (tid == 0) s_expired = 0;
  __syncthreads();
  if (tid < n) {
    const Odds o = odds_of(a, tid);
    s_odds[tid] = o;
    s_seen[tid][0] = a.seen.m[tid][0];
    s_seen[tid][1] = a.seen.m[tid][1];
    s_parent[tid] = a.parent[tid];
    bool first = true;   // the first child of its parent
    for (int j = 1; j < tid; ++j) first &= a.parent[j] != a.parent[tid];
    if (tid == 0 || (first && (double)o.u * (double)o.q < (double)o.p)) atomicOr(&s_first[tid >> 6], 1ull << (tid & 63));
  }
  __syncthreads();

  const int64_t lo = min(a.vocab, (int64_t)blk * a.slice), hi = min(a.vocab, lo + a.slice);
  int pass = 0;
  for (;;) {
    // the deepest node all of whose ancestors (and itself) are accepted
    if (tid < 2) s_on[tid] = 0;
    __syncthreads();
    if (tid < n && !(s_seen[tid][0] & ~s_first[0]) && !(s_seen[tid][1] & ~s_first[1]))
      atomicOr(&s_on[tid >> 6], 1ull << (tid & 63));
    __syncthreads();
    const int m = s_on[1] ? 127 - __builtin_clzll(s_on[1]) : 63 - __builtin_clzll(s_on[0]);
    const float* P = a.target + m * a.target_stride;
    const float* Q = drawn ? a.proposal + m * a.proposal_stride : nullptr;
    float pr[kDrawPer], qr[kDrawPer];
#pragma unroll
    for (int j = 0; j < kDrawPer; ++j) {
      const int64_t t = lo + (int64_t)j * kDrawThreads + tid;
      pr[j] = t < hi ? P[t] : 0.f;
      qr[j] = drawn && t < hi ? Q[t] : 0.f;
    }

    double b = 0.0, F = 1.0;
    int n_out = 0, n_mine = 0;
    // the value of element t of what is left, given the rejected tokens that may be t
    auto left = [&](float p, float q, int64_t t, const int* out, int n_out) __attribute__((always_inline)) -> double {
      if (drawn) {
        const double v = (double)p - b * (double)q;
        return v > 0.0 ? v : 0.0;
      }
      for (int k = 0; k < n_out; ++k)
        if (out[k] == t) return 0.0;
      return p > 0.f ? (double)p : 0.0;
    };
    // sum of what is left over the whole row, the same in every workgroup
    auto total = [&]() -> double {
      double x = 0.0;
#pragma unroll
      for (int j = 0; j < kDrawPer; ++j) x += left(pr[j], qr[j], lo + (int64_t)j * kDrawThreads + tid, s_mine, n_mine);
      for (int64_t t = lo + (int64_t)kDrawPer * kDrawThreads + tid; t < hi; t += kDrawThreads)
        x += left(P[t], drawn ? Q[t] : 0.f, t, s_mine, n_mine);
      x = wave_sum(x);
      if (lane == 0) s_wave[wave] = x;
      __syncthreads();
      if (tid == 0) {
        double sum = 0.0;
        for (int w = 0; w < kWaves; ++w) sum += s_wave[w];
        double* slot = a.part + (int64_t)pass * kDrawMaxBlocks + blk;
        __hip_atomic_store(slot, sum, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        __hip_atomic_fetch_add(a.arrived + pass, 1, __ATOMIC_RELEASE, __HIP_MEMORY_SCOPE_AGENT);
        long spins = 0;
        while (__hip_atomic_load(a.arrived + pass, __ATOMIC_ACQUIRE, __HIP_MEMORY_SCOPE_AGENT) < a.n_blocks) {
          __builtin_amdgcn_s_sleep(1);
          if (++spins > kSpinLimit) {
            s_expired = 1;
            break;
          }
        }
      }
      __syncthreads();
      if (tid < a.n_blocks)
        s_part[tid] = __hip_atomic_load(a.part + (int64_t)pass * kDrawMaxBlocks + tid, __ATOMIC_RELAXED,
                                        __HIP_MEMORY_SCOPE_AGENT);
      __syncthreads();
      double sum = 0.0;
      for (int w = 0; w < a.n_blocks; ++w) sum += s_part[w];
      ++pass;
      return sum;
    };

    int took = -1;
    bool tried = false;
    for (int c = m + 1; c < n && took < 0; ++c) {
      if (s_parent[c] != m) continue;
      const Odds o = s_odds[c];
      double px = 0.0;
      if (o.token >= 0) px = left(o.p, o.q, o.token, s_out, n_out);
      if ((double)o.u * (double)o.q * F < px) {
        took = c;
      } else {
        if (drawn) {
          b += F;
        } else {
          const bool mine = o.token >= lo && o.token < hi;
          __syncthreads();
          if (tid == 0) {
            s_out[n_out] = o.token;
            if (mine) s_mine[n_mine] = o.token;
          }
          __syncthreads();
          ++n_out;
          n_mine += mine;
        }
        F = total();
        tried = true;
        if (s_expired) break;
      }
    }
    if (s_expired) break;
    if (took >= 0) {
      __syncthreads();
      if (tid == 0) s_first[took >> 6] |= 1ull << (took & 63);
      __syncthreads();
      continue;
    }
    if (!tried) F = total();                 // a leaf
    if (!(F > 0.0) && !s_expired) {          // nothing left: the row itself
      b = 0.0;
      n_mine = 0;
      F = total();
    }
    if (s_expired) break;
    if (blk == 0 && tid == 0) {
      int k = 0;
      for (int i = 0; i < n; ++i)
        if (s_on[i >> 6] >> (i & 63) & 1) a.result[2 + k++] = i;
      a.result[0] = k;
    }
    // the slice that holds the drawn token: the first whose cumulative sum exceeds the target
    const double want = (double)a.u[0] * F;
    double before = 0.0;
    int owner = -1, last = -1;
    for (int w = 0; w < a.n_blocks && owner < 0; ++w) {
      if (s_part[w] > 0.0) last = w;
      if (before + s_part[w] > want) owner = w;
      else before += s_part[w];
    }
    const bool rounded = owner < 0;          // u[0] times the whole rounded up to the whole
    if (rounded) owner = last;
    if (owner == blk && F > 0.0 && F < __builtin_inf()) {
      if (tid == 0) {
        s_found = 0x7fffffff;
        s_best = -1;
      }
      __syncthreads();
      int best = -1;                         // the last element with a share, should none exceed
      for (int64_t t0 = lo; t0 < hi; t0 += kDrawThreads) {
        const int64_t t = t0 + tid;
        const double x = t < hi ? left(P[t], drawn ? Q[t] : 0.f, t, s_mine, n_mine) : 0.0;
        if (x > 0.0) best = (int)t;
        double cum = x;                      // inclusive sum within the wave
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
          const double y = __shfl_up(cum, d, 64);
          if (lane >= d) cum += y;
        }
        if (lane == 63) s_wave[wave] = cum;
        __syncthreads();
        double base = before, all = before;
        for (int w = 0; w < kWaves; ++w) {
          if (w < wave) base += s_wave[w];
          all += s_wave[w];
        }
        if (!rounded && x > 0.0 && base + cum > want) atomicMin(&s_found, (int)t);
        before = all;
        __syncthreads();
        const int found = s_found;
        __syncthreads();
        if (found != 0x7fffffff) break;
      }
      if (s_found == 0x7fffffff) atomicMax(&s_best, best);
      __syncthreads();
      if (tid == 0) a.result[1] = s_found == 0x7fffffff ? s_best : s_found;
    }
    break;
  }
  if (tid == 0 && s_expired) status_raise(a.status, kFaultWait);
}

}  // namespace

hipError_t launch_draft_clear(const DraftVerifyArgs& a, hipStream_t s) {
  hipLaunchKernelGGL(k_draft_clear, dim3(1), dim3(kClearThreads), 0, s, a);
  return hipGetLastError();
}

hipError_t launch_draft_draw(const DraftVerifyArgs& a, hipStream_t s) {
  if (a.n_blocks < 1 || a.n_blocks > kDrawMaxBlocks) return hipErrorInvalidValue;
  hipLaunchKernelGGL(k_draft_draw, dim3(a.n_blocks), dim3(kDrawThreads), 0, s, a);
  return hipGetLastError();
}

}  // namespace tu
