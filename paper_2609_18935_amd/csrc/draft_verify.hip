// Verification of a tree of drafted tokens against the target's probabilities.
//
// The children of a node are tried one after the other; after r rejections what is left of the
// target row is the r-fold normalised max(.. - q, 0). Unnormalised it is max(p - b q, 0) with
// one number b that grows by F = sum_t max(p(t) - b q(t), 0) with each rejection: F is all
// that a test needs of the row, so a rejection costs one pass over the rows of one node and
// an acceptance of a first child nothing. (A drafter's choice without probabilities is a
// point mass: the rejected tokens' entries are zero instead.)
//
// k_draft_clear empties the places of the passes' sums. k_draft_draw: every workgroup reads the
// single probabilities that the tests need, of all nodes at once, and derives the same walk
// from them; where a node has a rejection, or no child is left to try, each sums its slice of
// the row in float64 and publishes the sum, reads the others' as they appear (a bounded wait;
// the few workgroups fit the chip many times over) and adds all of them up in one order. The
// workgroup whose slice holds the drawn token finds it. Bound by latency: the odds (two
// dependent loads), the rows of a node (a load; a megabyte, kept in registers over its passes)
// and one exchange a pass; and by fetching code that runs once, so it is kept small. Measured in a graph of such
// calls over a vocabulary of 131,072: 7.9 us for one node, 8.5 for a chain of six, 10 to 11 for 64 nodes with
// several rejections (k_draft_clear 1.4 of it), 12 to 14 without proposals (more rejections; each sums its row again,
// though a point mass only takes p(x) from F).
#include <algorithm>

#include "draft.h"

namespace tu {

namespace {

constexpr int kClearThreads = 256;
static_assert(kDrawMaxBlocks == 64, "a slice's sum per lane");
constexpr int kWaves = kDrawThreads / 64;

// What the tests of node i (as a child of its parent) need of the rows.
struct Odds {
  float p, q, u;
  int token;     // -1: outside the vocabulary
};

__device__ __forceinline__ Odds odds_of(const DraftVerifyArgs& a, int i) {
  Odds o{0.f, 1.f, 2.f, -1};
  if (i == 0) return o;
  const int up = a.parent[i];
  const int x = a.tokens[i];
  o.u = a.u[i];
  if (x < 0 || x >= a.vocab) return o;
  o.token = x;
  o.p = a.target[up * a.target_stride + x];
  if (a.proposal) o.q = a.proposal[up * a.proposal_stride + x];
  return o;
}

// A sum that has not been written yet. (A sum that is not a number is written as another NaN.)
constexpr unsigned long long kEmpty = ~0ull;

__global__ __launch_bounds__(kClearThreads) void k_draft_clear(DraftVerifyArgs a) {
  status_mark(a.status);
  const int t = blockIdx.x * kClearThreads + threadIdx.x;
  for (int i = t; i < (a.n + 1) * a.n_blocks; i += gridDim.x * kClearThreads) a.part[i] = kEmpty;
  if (t < a.n + 2) a.result[t] = t == 0 ? 0 : -1;
}

// x + the value that CTRL moves here from another lane of the rows in MASK (0 elsewhere)
template <int CTRL, int MASK>
__device__ __forceinline__ double add_dpp(double x) {
  const uint64_t b = __builtin_bit_cast(uint64_t, x);
  const uint32_t lo = __builtin_amdgcn_update_dpp(0, (int)(uint32_t)b, CTRL, MASK, 0xf, false);
  const uint32_t hi = __builtin_amdgcn_update_dpp(0, (int)(uint32_t)(b >> 32), CTRL, MASK, 0xf, false);
  return x + __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}

// x + the values of the lanes before it
__device__ __forceinline__ double wave_scan(double x) {
  x = add_dpp<0x111, 0xf>(x);   // row_shr 1, 2, 4, 8: within 16 lanes
  x = add_dpp<0x112, 0xf>(x);
  x = add_dpp<0x114, 0xf>(x);
  x = add_dpp<0x118, 0xf>(x);
  x = add_dpp<0x142, 0xa>(x);   // the last lane of rows 0 and 2 to rows 1 and 3
  return add_dpp<0x143, 0xc>(x);   // lane 31 to rows 2 and 3
}

// 8 elements of a row from t on (0 from hi on, and no reads there); `wide`: the address is a multiple of 16
__device__ __forceinline__ void load_row(const float* row, int64_t t, int64_t hi, bool wide, float (&x)[kDrawPer]) {
  static_assert(kDrawPer == 8, "two vectors");
  if (wide && t + kDrawPer <= hi) {
    *(f32x4*)x = *(const f32x4*)(row + t);
    *(f32x4*)(x + 4) = *(const f32x4*)(row + t + 4);
  } else {
#pragma unroll
    for (int j = 0; j < kDrawPer; ++j) {
      const float y = row[min(t + j, hi - 1)];
      x[j] = t + j < hi ? y : 0.f;
    }
  }
}

// DRAWN: the drafter's probabilities are given. (Two instances: the code runs once, and much of the
// time goes into fetching it.)
template <bool DRAWN>
__global__ __launch_bounds__(kDrawThreads) void k_draft_draw(DraftVerifyArgs a) {
  __shared__ Odds s_odds[kMaxDraft];
  __shared__ uint64_t s_seen[kMaxDraft][2];
  __shared__ uint8_t s_child[kMaxDraft], s_sibling[kMaxDraft];
  __shared__ unsigned long long s_first[2], s_on[2];   // accepted as first children; on the accepted path
  __shared__ double s_wave[kWaves], s_before[kDrawMaxBlocks + 1];   // sums of the waves; of the slices before a slice
  __shared__ int s_out[kMaxDraft];                     // rejected tokens of the row (point-mass drafts)
  __shared__ int s_mine[kMaxDraft];                    // those of this workgroup's slice
  __shared__ int s_last, s_expired;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int n = a.n, blk = blockIdx.x;

  if (tid < 2) s_first[tid] = 0;
  if (tid == 0) s_expired = 0;
  if (tid < n) {
    s_seen[tid][0] = a.seen.m[tid][0];
    s_seen[tid][1] = a.seen.m[tid][1];
    s_child[tid] = a.child[tid];
    s_sibling[tid] = a.sibling[tid];
  }
  __syncthreads();
  if (tid < n) {
    const Odds o = odds_of(a, tid);
    s_odds[tid] = o;
    const bool first = a.first[tid >> 6] >> (tid & 63) & 1;   // the first child of its parent
    if (tid == 0 || (first && (double)o.u * (double)o.q < (double)o.p)) atomicOr(&s_first[tid >> 6], 1ull << (tid & 63));
  }

  const int64_t lo = min(a.vocab, (int64_t)blk * a.slice), hi = min(a.vocab, lo + a.slice);
  const int64_t t0 = lo + tid * kDrawPer;      // this thread's elements of the slice's first block
  const bool wide = a.wide;
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
    const float* Q = DRAWN ? a.proposal + m * a.proposal_stride : nullptr;
    float pr[kDrawPer], qr[kDrawPer] = {};
    load_row(P, t0, hi, wide, pr);
    if (DRAWN) load_row(Q, t0, hi, wide, qr);

    double b = 0.0, F = 1.0;
    int n_out = 0, n_mine = 0;
    // 8 values of what is left, from element t on, and their sum in element order
    auto left = [&](const float (&p)[kDrawPer], const float (&q)[kDrawPer], int64_t t, double (&v)[kDrawPer])
                    __attribute__((always_inline)) -> double {
      uint32_t gone = 0;   // rejected tokens among them
      if constexpr (!DRAWN)
        for (int k = 0; k < n_mine; ++k) {
          const int64_t at = s_mine[k] - t;
          if (at >= 0 && at < kDrawPer) gone |= 1u << at;
        }
      double x = 0.0;
#pragma unroll
      for (int j = 0; j < kDrawPer; ++j) {
        v[j] = DRAWN ? (double)p[j] - b * (double)q[j] : gone >> j & 1 ? 0.0 : (double)p[j];
        v[j] = v[j] > 0.0 ? v[j] : 0.0;
        x += v[j];
      }
      return x;
    };
    // sum of what is left over the whole row, the same in every workgroup
    auto total = [&]() -> double {
      double v[kDrawPer], x = left(pr, qr, t0, v);
      for (int64_t t = t0 + kDrawThreads * kDrawPer; t < hi; t += kDrawThreads * kDrawPer) {
        float p[kDrawPer], q[kDrawPer] = {};
        load_row(P, t, hi, wide, p);
        if (DRAWN) load_row(Q, t, hi, wide, q);
        x += left(p, q, t, v);
      }
      x = wave_scan(x);
      if (lane == 63) s_wave[wave] = x;
      __syncthreads();
      if (wave == 0) {
        unsigned long long* slots = a.part + (int64_t)pass * a.n_blocks;
        if (lane == 0) {
          double sum = 0.0;
#pragma unroll
          for (int w = 0; w < kWaves; ++w) sum += s_wave[w];
          const unsigned long long bits = sum == sum ? __builtin_bit_cast(unsigned long long, sum) : 0x7ff8000000000000ull;
          __hip_atomic_store(slots + blk, bits, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        }
        unsigned long long bits = 0;   // slices past the last are empty: 0.0
        int spins = 0;
        for (;;) {
          if (lane < a.n_blocks) bits = __hip_atomic_load(slots + lane, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
          if (__all(bits != kEmpty)) break;
          if (++spins > a.polls) {
            s_expired = 1;
            break;
          }
        }
        const double mine = __builtin_bit_cast(double, bits);
        const double upto = wave_scan(mine);
        if (lane < kDrawMaxBlocks) s_before[lane + 1] = upto;
        if (lane == 0) s_before[0] = 0.0;
        const uint64_t some = __ballot(mine > 0.0);
        if (lane == 0) s_last = some ? 63 - __builtin_clzll(some) : -1;   // the last slice with a share
      }
      __syncthreads();
      ++pass;
      return s_before[kDrawMaxBlocks];
    };

    int took = -1;
    bool summed = false, whole = false;   // F is a sum; of the row itself
    for (int c = s_child[m];;) {
      if (c > 0) {
        const Odds o = s_odds[c];
        double px = 0.0;
        if (o.token >= 0) {
          px = DRAWN ? (double)o.p - b * (double)o.q : (double)o.p;
          if (!(px > 0.0)) px = 0.0;
          if constexpr (!DRAWN)
            for (int k = 0; k < n_out; ++k)
              if (s_out[k] == o.token) px = 0.0;
        }
        if ((double)o.u * (double)o.q * F < px) {
          took = c;
          break;
        }
        if constexpr (DRAWN) {
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
        c = s_sibling[c];
      } else if (summed) {
        if (F > 0.0 || whole) break;
        b = 0.0;   // nothing left: the row itself
        n_mine = 0;
        whole = true;
      }
      F = total();
      summed = true;
      if (s_expired) break;
    }
    if (s_expired) break;
    if (took >= 0) {
      __syncthreads();
      if (tid == 0) s_first[took >> 6] |= 1ull << (took & 63);
      __syncthreads();
      continue;
    }
    // the slice that holds the drawn token: the first whose cumulative sum exceeds the target
    // (the last one with a share if u[0] times the whole was rounded up to the whole; without a distribution
    // there is no token)
    const bool draws = F > 0.0 && F < __builtin_inf();
    const double want = (double)a.u[0] * F;
    const uint64_t past = __ballot(lane < a.n_blocks && s_before[lane + 1] > want);
    const int owner = !draws ? 0 : past ? __builtin_ctzll(past) : s_last;
    if (owner != blk) break;
    // The owner writes all of the result: one whose wait has expired writes nothing, and the count stays 0,
    // whatever the other workgroups have seen.
    if (tid < n && (s_on[tid >> 6] >> (tid & 63) & 1)) {   // the path, in order
      const uint64_t below = (1ull << (tid & 63)) - 1;
      const int at = __popcll(s_on[0] & (tid < 64 ? below : ~0ull)) + (tid < 64 ? 0 : __popcll(s_on[1] & below));
      a.result[2 + at] = tid;
      if (tid == m) a.result[0] = at + 1;
    }
    if (!draws) break;
    double before = s_before[blk];
    int found = -1;
    for (int64_t tb = lo; tb < hi; tb += kDrawThreads * kDrawPer) {
      const int64_t t = tb + tid * kDrawPer;
      float p[kDrawPer], q[kDrawPer] = {};
      if (tb == lo) {
#pragma unroll
        for (int j = 0; j < kDrawPer; ++j) p[j] = pr[j], q[j] = qr[j];
      } else {
        load_row(P, t, hi, wide, p);
        if (DRAWN) load_row(Q, t, hi, wide, q);
      }
      double v[kDrawPer];
      const double x = left(p, q, t, v);
      const double cum = wave_scan(x);
      __syncthreads();
      if (lane == 63) s_wave[wave] = cum;
      __syncthreads();
      double base = before;
      for (int w = 0; w < kWaves; ++w) {
        if (w < wave) base += s_wave[w];
        before += s_wave[w];
      }
      // this thread's first element that takes the sum past the target, else its last with a share
      double sum = base + (cum - x);
      int first = -1, last = -1;
#pragma unroll
      for (int j = 0; j < kDrawPer; ++j) {
        sum += v[j];
        if (v[j] > 0.0) {
          last = (int)(t + j);
          if (first < 0 && sum > want) first = last;
        }
      }
      // the first thread of the block that has one; the last thread with a share otherwise
      __shared__ int s_pick[2][kWaves];
      const uint64_t has = __ballot(first >= 0), share = __ballot(last >= 0);
      if (has ? lane == __builtin_ctzll(has) : lane == 0) s_pick[0][wave] = has ? first : -1;
      if (share ? lane == 63 - __builtin_clzll(share) : lane == 0) s_pick[1][wave] = share ? last : -1;
      __syncthreads();
      const int hit = lane < kWaves ? s_pick[0][lane] : -1, near = lane < kWaves ? s_pick[1][lane] : -1;
      const uint64_t hits = __ballot(hit >= 0), nears = __ballot(near >= 0);
      if (hits) {
        found = __builtin_amdgcn_readlane(hit, __builtin_ctzll(hits));
        break;
      }
      if (nears) found = __builtin_amdgcn_readlane(near, 63 - __builtin_clzll(nears));
    }
    if (tid == 0) a.result[1] = found;
    break;
  }
  if (tid == 0 && s_expired) status_raise(a.status, kFaultWait);
}

}  // namespace

hipError_t launch_draft_clear(const DraftVerifyArgs& a, hipStream_t s) {
  const int blocks = std::max(1, std::min(16, ((a.n + 1) * a.n_blocks + kClearThreads - 1) / kClearThreads));
  hipLaunchKernelGGL(k_draft_clear, dim3(blocks), dim3(kClearThreads), 0, s, a);
  return hipGetLastError();
}

hipError_t launch_draft_draw(const DraftVerifyArgs& a, hipStream_t s) {
  if (a.n_blocks < 1 || a.n_blocks > kDrawMaxBlocks) return hipErrorInvalidValue;
  if (a.proposal) hipLaunchKernelGGL(k_draft_draw<true>, dim3(a.n_blocks), dim3(kDrawThreads), 0, s, a);
  else hipLaunchKernelGGL(k_draft_draw<false>, dim3(a.n_blocks), dim3(kDrawThreads), 0, s, a);
  return hipGetLastError();
}

}  // namespace tu
