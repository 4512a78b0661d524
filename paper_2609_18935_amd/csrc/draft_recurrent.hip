// The recurrent layers over a tree of drafted tokens: the short convolution and the gated
// delta rule along every node's path, the carried states only read.
//
// Convolution. A thread takes 8 channels of one node: the rows under the taps are the node's
// and those of its ancestors, then the carried ones; products are summed in fp32 in tap order
// and rounded once to bf16. Bound by latency and issue: a layer's rows and weights (a few MB)
// stay in L2.
//
// Delta rule. Evaluated token by token a tree needs a state (d x d fp32) per node; in the
// WY form it needs the carried state once. With D_ij = gamma_i / gamma_j where j is an ancestor
// of i or i itself, else 0 (gamma: product of the gates along the path),
//     (I + M) U = diag(beta) (V - diag(gamma) K S^T),   M = strictly-lower(diag(beta) D o K K^T)
//     O = scale (diag(gamma) Q S^T + (D o Q K^T) U).
// Rows of S are independent columns of U: a workgroup takes 16 rows of one value head, so 32
// heads of 128 rows fill the 256 CUs with one workgroup each and the state is read once. All
// node pairs are products of bf16 rows on the bf16 MFMA (exact products, fp32 sums); K S^T and
// Q S^T split S into three bf16 terms (24 bits, as many as the fp32 value has); the
// triangular solve and the last product run on the fp32 MFMA. Nothing is rounded below fp32.
//
// Nodes go in blocks of 16. Wave w forms row block w (and the mirrored one of the upper half
// when there are 8): its products with the blocks before it and with S. Then one lane per
// column inverts the diagonal blocks I + M_bb by forward substitution, and every wave solves
// for all of U (the same work on each SIMD, so that U is where the output products need it):
// an MFMA accumulator lane holds rows 4 g .. 4 g + 3 of a column, exactly the operand of the
// next 16x16x4 products if contracted index 4 g + e is fed in step e, so U never leaves the
// registers.
//
// A node whose inputs are not finite must not reach nodes of other paths (0 x NaN in a product
// of blocks): it is left out, and its outputs and its descendants' set to NaN.
#include "draft.h"

namespace tu {

namespace {

constexpr int kThreads = 256;

// ------------------------------------------------------------------ short convolution

template <int W>
__global__ __launch_bounds__(kThreads) void k_draft_conv(DraftConvArgs a) {
  const int b = blockIdx.x;
  int ji = 0;
  while (ji + 1 < a.n_jobs && a.job[ji + 1].block_begin <= b) ++ji;
  const bf16_t* state = a.job[ji].state;
  const bf16_t* x = a.job[ji].x;
  const bf16_t* w = a.job[ji].w;
  bf16_t* out = a.job[ji].out;
  const int C = a.job[ji].C, act = a.job[ji].act;
  const long item = (long)(b - a.job[ji].block_begin) * kThreads + threadIdx.x;
  const int chunks = C >> 3;
  const int node = (int)(item / chunks);
  if (node >= a.n) return;
  const int c0 = (int)(item - (long)node * chunks) * 8;

  bf16_t wt[8 * W];
#pragma unroll
  for (int i = 0; i < W; ++i) *(u32x4*)(wt + 8 * i) = *(const u32x4*)(w + (long)c0 * W + 8 * i);
  u32x4 rows[W];   // rows[t] lies under tap t
  const uint64_t up = *(const uint64_t*)a.up[node];
#pragma unroll
  for (int t = 0; t < W; ++t) {
    const int at = (int8_t)(up >> (8 * (W - 1 - t)));
    const bf16_t* row = at >= 0 ? x + (long)at * C : state + (long)(W - 1 + at) * C;
    rows[t] = *(const u32x4*)(row + c0);
  }
  bf16x8 y;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    float s = 0.f;
#pragma unroll
    for (int t = 0; t < W; ++t) {
      const uint32_t word = rows[t][e >> 1];
      s = __builtin_fmaf(bf16_to_f32(wt[e * W + t]), __uint_as_float(e & 1 ? word & 0xFFFF0000u : word << 16), s);
    }
    if (act) s = s / (1.f + __expf(-s));
    y[e] = (__bf16)s;
  }
  *(u32x4*)(out + (long)node * C + c0) = __builtin_bit_cast(u32x4, y);
}

// ------------------------------------------------------------------ delta rule

constexpr int kBlock = 16;           // nodes of a block, state rows of a workgroup
constexpr int kMStride = 20;         // floats of a row of a 16 x 16 block in LDS

// 8 fp32 values as three bf16 terms, x = t[0] + t[1] + t[2] to fp32's last bit
__device__ __forceinline__ void split3(const float* x, bf16x8 (&t)[3]) {
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const __bf16 hi = (__bf16)x[e];
    const float r1 = x[e] - (float)hi;
    const __bf16 mid = (__bf16)r1;
    t[0][e] = hi;
    t[1][e] = mid;
    t[2][e] = (__bf16)(r1 - (float)mid);
  }
}

__device__ __forceinline__ bool finite(float x) { return fabsf(x) < __builtin_inff(); }

// a + sum over the 16 contracted rows: A holds row (lane & 15), columns 4 g .. 4 g + 3
__device__ __forceinline__ f32x4 mma16(f32x4 A, f32x4 B, f32x4 acc) {
#pragma unroll
  for (int e = 0; e < 4; ++e) acc = __builtin_amdgcn_mfma_f32_16x16x4f32(A[e], B[e], acc, 0, 0, 0);
  return acc;
}

constexpr int tri(int b) { return b * (b + 1) / 2; }

template <int DK, int NB>   // NB: blocks of 16 nodes
__global__ __launch_bounds__(kThreads) void k_draft_delta(DraftDeltaArgs a) {
  constexpr int NK = DK / 32;               // 32-deep steps of a row product
  constexpr int NSL = DK / kBlock;          // workgroups of a head
  constexpr int N = NB * kBlock;
  constexpr int RB = NB > 4 ? 2 : 1;        // row blocks of a wave
  __shared__ __attribute__((aligned(16))) float s_m[tri(NB)][kBlock * kMStride];   // -M
  __shared__ __attribute__((aligned(16))) float s_a[tri(NB)][kBlock * kMStride];   // D o Q K^T
  __shared__ __attribute__((aligned(16))) float s_t[NB][kBlock * kMStride];        // (I + M_bb)^-1
  __shared__ __attribute__((aligned(16))) float s_rhs[kBlock][N + 4];              // [state row][node]
  __shared__ __attribute__((aligned(16))) bf16x8 s_k[NB][NK][64];   // K as the lanes of a product hold it
  __shared__ double s_gate[N], lg[N];       // log2 of the gates; of gamma
  __shared__ float s_beta[N];
  __shared__ unsigned long long s_bad[kBlock][2];   // nodes to leave out, for each state row

  const int Hv = a.n_v_heads, Hk = a.n_k_heads;
  const int item = xcd_remap(blockIdx.x, gridDim.x);
  if (item >= Hv * NSL) return;
  const int h = item / NSL, kh = h / (Hv / Hk);
  const int i0 = (item - h * NSL) * kBlock;
  const int n = a.n;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int g = lane >> 4, col = lane & 15;

  // ---- everything that comes from memory is asked for first: the gates (a thread a node), this
  // wave's rows of K, Q and V, the workgroup's 16 rows of S, the masks
  float gin = 1.f, bin = 0.f;
  if (tid < n) {
    gin = a.g[(long)tid * Hv + h];
    bin = a.beta[(long)tid * Hv + h];
  }
  f32x4 sx[NK][2];
  {
    const float* sp = a.state + ((long)h * DK + i0 + col) * DK + 8 * g;
#pragma unroll
    for (int s = 0; s < NK; ++s) {
      sx[s][0] = *(const f32x4*)(sp + 32 * s);
      sx[s][1] = *(const f32x4*)(sp + 32 * s + 4);
    }
  }
  bf16x8 kf[RB][NK], qf[RB][NK];
  float vf[RB][4];
  uint64_t see[RB][4][2];   // masks of this lane's nodes: rows 4 g + e of its blocks
#pragma unroll
  for (int rb = 0; rb < RB; ++rb) {
    const int b = rb ? NB - 1 - wave : wave;
    if (b >= NB) continue;
    const long at = ((long)min(b * kBlock + col, n - 1) * Hk + kh) * DK + 8 * g;   // rows past the last repeat it
#pragma unroll
    for (int s = 0; s < NK; ++s) {
      kf[rb][s] = __builtin_bit_cast(bf16x8, *(const u32x4*)(a.k + at + 32 * s));
      qf[rb][s] = __builtin_bit_cast(bf16x8, *(const u32x4*)(a.q + at + 32 * s));
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int i = b * kBlock + 4 * g + e;
      vf[rb][e] = bf16_to_f32(a.v[((long)min(i, n - 1) * Hv + h) * DK + i0 + col]);
      see[rb][e][0] = i < n ? a.seen.m[i][0] : 0;
      see[rb][e][1] = i < n && NB > 4 ? a.seen.m[i][1] : 0;
    }
  }
  // a thread's share of a node's path: PARTS neighbouring lanes a node
  constexpr int PARTS = kThreads / N, SHARE = N / PARTS;
  const int pnode = tid / PARTS, ppart = tid % PARTS;
  uint64_t pmask = 0;
  if (pnode < n) pmask = a.seen.m[pnode][ppart * SHARE >> 6] >> (ppart * SHARE & 63);

  if (tid < N) {
    const float gate = gin < 0x1p-100f ? 0x1p-100f : gin;   // as delta_rule_continue holds it
    s_gate[tid] = (double)log2f(gate);
    s_beta[tid] = bin;
  }
  if (tid < 2 * kBlock) s_bad[tid >> 1][tid & 1] = 0;
#pragma unroll
  for (int rb = 0; rb < RB; ++rb) {
    const int b = rb ? NB - 1 - wave : wave;
    if (b >= NB) continue;
#pragma unroll
    for (int s = 0; s < NK; ++s) s_k[b][s][lane] = kf[rb][s];
  }
  __syncthreads();

  // ---- log2 gamma: float64 sums of the gates along the paths
  {
    double x = 0.0;
#pragma unroll 16
    for (int j = 0; j < SHARE; ++j) {
      const double y = s_gate[ppart * SHARE + j];
      x += pmask >> j & 1 ? y : 0.0;
    }
#pragma unroll
    for (int d = 1; d < PARTS; d <<= 1) x += __shfl_xor(x, d, 64);
    if (ppart == 0) lg[pnode] = x;
  }

  // ---- products of this wave's rows with S, in three bf16 terms, the smallest first
  f32x4 yk[RB], yq[RB];
  {
    bf16x8 st[NK][3];
#pragma unroll
    for (int s = 0; s < NK; ++s) {
      float x[8];
      *(f32x4*)x = sx[s][0];
      *(f32x4*)(x + 4) = sx[s][1];
      split3(x, st[s]);
    }
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
      yk[rb] = yq[rb] = f32x4{0.f, 0.f, 0.f, 0.f};
      if ((rb ? NB - 1 - wave : wave) >= NB) continue;
#pragma unroll
      for (int p = 2; p >= 0; --p)
#pragma unroll
        for (int s = 0; s < NK; ++s) {
          yk[rb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf[rb][s], st[s][p], yk[rb], 0, 0, 0);
          yq[rb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(qf[rb][s], st[s][p], yq[rb], 0, 0, 0);
        }
    }
  }
  __syncthreads();

#pragma unroll
  for (int rb = 0; rb < RB; ++rb) {
    const int b = rb ? NB - 1 - wave : wave;
    if (b >= NB || b * kBlock >= n) continue;
    double li[4];
    float bi[4];
    uint32_t bad = 0, bad_row = 0;   // bit e: node 4 g + e has an input that is not finite; for this state row
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int i = b * kBlock + 4 * g + e;
      const bool live = i < n;
      li[e] = lg[i];
      bi[e] = s_beta[i];
      const float gam = __builtin_amdgcn_exp2f((float)li[e]);
      float rhs = bi[e] * (vf[rb][e] - gam * yk[rb][e]);
      if (!live) rhs = 0.f;
      if (!finite(rhs)) {
        bad_row |= 1u << e;
        rhs = 0.f;
      }
      s_rhs[col][i] = rhs;
      yq[rb][e] *= gam;
    }
    for (int c = 0; c <= b; ++c) {
      f32x4 kk = {0.f, 0.f, 0.f, 0.f}, qk = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int s = 0; s < NK; ++s) {
        const bf16x8 kc = s_k[c][s][lane];
        kk = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf[rb][s], kc, kk, 0, 0, 0);
        qk = __builtin_amdgcn_mfma_f32_16x16x32_bf16(qf[rb][s], kc, qk, 0, 0, 0);
      }
      const int j = c * kBlock + col;
      const double lj = lg[j];
      float* mb = s_m[tri(b) + c];
      float* ab = s_a[tri(b) + c];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int i = b * kBlock + 4 * g + e;
        const bool sees = (NB > 4 && j >= 64 ? see[rb][e][1] : see[rb][e][0]) >> (j & 63) & 1;
        const float ratio = __builtin_amdgcn_exp2f((float)(li[e] - lj));
        float m = -bi[e] * ratio * kk[e];
        if (!finite(m)) {
          if (i == j) bad |= 1u << e;
          m = 0.f;
        }
        mb[(4 * g + e) * kMStride + col] = sees && i != j ? m : 0.f;
        ab[(4 * g + e) * kMStride + col] = sees ? ratio * qk[e] : 0.f;
      }
    }
    if (bad | bad_row) {
      for (int e = 0; e < 4; ++e) {
        const int i = b * kBlock + 4 * g + e;
        if (bad_row >> e & 1) atomicOr(&s_bad[col][i >> 6], 1ull << (i & 63));
        if (bad >> e & 1)
          for (int r = 0; r < kBlock; ++r) atomicOr(&s_bad[r][i >> 6], 1ull << (i & 63));
      }
    }
  }
  __syncthreads();

  // inverses of the diagonal blocks: 16 lanes a block, lane `col` its column of (I + M)^-1
  if (tid < N) {
    const int b = tid >> 4;
    const float* mb = s_m[tri(b) + b];
    float t[kBlock];
#pragma unroll
    for (int i = 0; i < kBlock; ++i) {
      float x0 = i == col ? 1.f : 0.f, x1 = 0.f;
#pragma unroll
      for (int j = 0; j < i; ++j) {
        const float m = mb[i * kMStride + j];
        if (j & 1) x1 = __builtin_fmaf(m, t[j], x1);
        else x0 = __builtin_fmaf(m, t[j], x0);
      }
      t[i] = x0 + x1;
      s_t[b][i * kMStride + col] = t[i];
    }
  }
  __syncthreads();

  const unsigned long long bad0 = s_bad[col][0], bad1 = s_bad[col][1];
  f32x4 u[NB];
#pragma unroll
  for (int b = 0; b < NB; ++b) {
    f32x4 acc = *(const f32x4*)&s_rhs[col][b * kBlock + 4 * g];
    if (b * kBlock < n) {
#pragma unroll
      for (int c = 0; c < b; ++c) acc = mma16(*(const f32x4*)(s_m[tri(b) + c] + col * kMStride + 4 * g), u[c], acc);
      u[b] = mma16(*(const f32x4*)(s_t[b] + col * kMStride + 4 * g), acc, f32x4{0.f, 0.f, 0.f, 0.f});
    }
  }
#pragma unroll
  for (int rb = 0; rb < RB; ++rb) {
    const int b = rb ? NB - 1 - wave : wave;
    if (b >= NB || b * kBlock >= n) continue;
    f32x4 o = yq[rb];
#pragma unroll
    for (int c = 0; c < NB; ++c)
      if (c <= b) o = mma16(*(const f32x4*)(s_a[tri(b) + c] + col * kMStride + 4 * g), u[c], o);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int i = b * kBlock + 4 * g + e;
      if (i >= n) continue;
      const bool spoilt = (see[rb][e][0] & bad0) | (see[rb][e][1] & bad1);
      a.out[((long)i * Hv + h) * DK + i0 + col] = spoilt ? __builtin_nanf("") : a.scale * o[e];
    }
  }
}

template <int DK>
hipError_t delta_for(const DraftDeltaArgs& a, hipStream_t s) {
  const int blocks = (a.n_v_heads * (DK / kBlock) + 7) & ~7;   // xcd_remap wants a multiple of 8
  if (a.n <= 16) hipLaunchKernelGGL((k_draft_delta<DK, 1>), dim3(blocks), dim3(kThreads), 0, s, a);
  else if (a.n <= 32) hipLaunchKernelGGL((k_draft_delta<DK, 2>), dim3(blocks), dim3(kThreads), 0, s, a);
  else if (a.n <= 64) hipLaunchKernelGGL((k_draft_delta<DK, 4>), dim3(blocks), dim3(kThreads), 0, s, a);
  else hipLaunchKernelGGL((k_draft_delta<DK, 8>), dim3(blocks), dim3(kThreads), 0, s, a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_draft_conv(DraftConvArgs& a, hipStream_t s) {
  int blocks = 0;
  for (int j = 0; j < a.n_jobs; ++j) {
    a.job[j].block_begin = blocks;
    blocks += (int)(((long)a.n * (a.job[j].C >> 3) + kThreads - 1) / kThreads);
  }
  if (blocks <= 0) return hipSuccess;
  switch (a.width) {
#define TU_CASE(W)                                                                          \
  case W:                                                                                   \
    hipLaunchKernelGGL(k_draft_conv<W>, dim3(blocks), dim3(kThreads), 0, s, a);             \
    return hipGetLastError();
    TU_CASE(1) TU_CASE(2) TU_CASE(3) TU_CASE(4) TU_CASE(5) TU_CASE(6) TU_CASE(7) TU_CASE(8)
#undef TU_CASE
    default: return hipErrorInvalidValue;
  }
}

hipError_t launch_draft_delta(const DraftDeltaArgs& a, int d, hipStream_t s) {
  if (a.n <= 0) return hipSuccess;
  return d == 128 ? delta_for<128>(a, s) : d == 64 ? delta_for<64>(a, s) : hipErrorInvalidValue;
}

}  // namespace tu
