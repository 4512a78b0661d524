// The recurrent layers over a tree of drafted tokens: the short convolution and the gated
// delta rule along every node's path, the carried states only read.
//
// Convolution. A thread takes 8 channels of one node: the rows under the taps are the node's
// and those of its ancestors, then the carried ones; products are summed in fp32 in tap order
// and rounded once to bf16. Bound by latency and issue: a layer's rows and weights (a few MB)
// stay in L2. Measured in a graph of such calls, 8,192 channels of width 4: one node 3.1 us, 64 3.4, 128 4.2.
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
// when there are 8; of the last of four rows waves 0 and 1, which have little to do, take a block
// each): its products with the blocks before it and with S, whose three terms one wave a
// part has split for all. Then one lane per
// column inverts the diagonal blocks I + M_bb by forward substitution, and every wave solves
// for all of U (the same work on each SIMD, so that U is where the output products need it):
// an MFMA accumulator lane holds rows 4 g .. 4 g + 3 of a column, exactly the operand of the
// next 16x16x4 products if contracted index 4 g + e is fed in step e, so U never leaves the
// registers.
//
// Bound by latency, not by its bytes (2 to 6 MB) or products: one trip to memory for all operands, then
// five dependent phases (gates along the paths, products with S and between nodes, inverses, the
// solve block by block, outputs) with one wave a SIMD. Measured in a graph of such calls, 16 key and 32 value heads
// of 128: 1 node 4.7 us, 7 5.0, 16 5.3, 32 6.3, 64 8.1 (7.4 a call launched by itself), 65 11.9, 128 14.7.
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

// x + the value of the lane that CTRL pairs this one with
template <int CTRL>
__device__ __forceinline__ double add_dpp(double x) {
  const uint64_t b = __builtin_bit_cast(uint64_t, x);
  const uint32_t lo = __builtin_amdgcn_update_dpp(0, (int)(uint32_t)b, CTRL, 0xf, 0xf, true);
  const uint32_t hi = __builtin_amdgcn_update_dpp(0, (int)(uint32_t)(b >> 32), CTRL, 0xf, 0xf, true);
  return x + __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}

constexpr int tri(int b) { return b * (b + 1) / 2; }

template <int DK, int NB>   // NB: blocks of 16 nodes
__global__ __launch_bounds__(kThreads) void k_draft_delta(
    const float* state, const bf16_t* q, const bf16_t* k, const bf16_t* v, const float* beta, const float* gate_in, int n,
    uint32_t heads, DraftDeltaArgs a) {   // up to `a`: in registers from the start
  constexpr int NK = DK / 32;               // 32-deep steps of a row product
  constexpr int NSL = DK / kBlock;          // workgroups of a head
  constexpr int N = NB * kBlock;
  constexpr int RB = NB > 4 ? 2 : 1;        // row blocks of a wave
  // -M; before it is formed, the 16 rows of S in three bf16 terms as the lanes of a product hold them
  constexpr size_t kMBytes = sizeof(float) * tri(NB) * kBlock * kMStride, kSBytes = sizeof(bf16x8) * NK * 3 * 64;
  __shared__ __attribute__((aligned(16))) char s_ms[kMBytes > kSBytes ? kMBytes : kSBytes];
  auto s_m = (float(*)[kBlock * kMStride])s_ms;
  auto s_s = (bf16x8(*)[3][64])s_ms;
  __shared__ __attribute__((aligned(16))) float s_a[tri(NB)][kBlock * kMStride];   // D o Q K^T
  __shared__ __attribute__((aligned(16))) float s_t[NB][kBlock * kMStride];        // (I + M_bb)^-1
  __shared__ __attribute__((aligned(16))) float s_rhs[kBlock][N + 4];              // [state row][node]
  __shared__ __attribute__((aligned(16))) bf16x8 s_k[NB][NK][64];   // K as the lanes of a product hold it
  __shared__ __attribute__((aligned(16))) bf16x8 s_q[NB == 4 ? NK : 1][64];        // Q of the last of 4 blocks
  __shared__ double s_gate[N];              // log2 of the gates
  __shared__ float s_lg[N][2];              // log2 gamma, in two fp32 terms
  __shared__ uint64_t s_see[N][2];          // masks
  __shared__ float s_beta[N];
  __shared__ unsigned long long s_bad[kBlock][2];   // nodes to leave out, for each state row

  const int Hk = heads & 0xFFFF, Hv = heads >> 16;
  const int item = xcd_remap(blockIdx.x, Hv * NSL);
  if (item >= Hv * NSL) return;
  const int h = item / NSL, kh = h / (Hv / Hk);
  const int i0 = (item - h * NSL) * kBlock;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int g = lane >> 4, col = lane & 15;

  // ---- everything that comes from memory is asked for first: the gates (a thread a node), this
  // wave's rows of K, Q and V, the workgroup's 16 rows of S, the masks
  float gin = 1.f, bin = 0.f;
  uint64_t see0 = 0, see1 = 0;
  if (tid < n) {
    see0 = a.seen.m[tid][0];
    see1 = a.seen.m[tid][1];
    gin = gate_in[(long)tid * Hv + h];
    bin = beta[(long)tid * Hv + h];
  }
  float sx[8];   // wave s takes dims 32 s .. of S
  if (wave < NK) {
    const float* sp = state + ((long)h * DK + i0 + col) * DK + 8 * g + 32 * wave;
    *(f32x4*)sx = *(const f32x4*)sp;
    *(f32x4*)(sx + 4) = *(const f32x4*)(sp + 4);
  }
  bf16x8 kf[RB][NK], qf[RB][NK];
  float vf[RB][4];
#pragma unroll
  for (int rb = 0; rb < RB; ++rb) {
    const int b = rb ? NB - 1 - wave : wave;
    if (b >= NB) continue;
    const long at = ((long)min(b * kBlock + col, n - 1) * Hk + kh) * DK + 8 * g;   // rows past the last repeat it
#pragma unroll
    for (int s = 0; s < NK; ++s) {
      kf[rb][s] = __builtin_bit_cast(bf16x8, *(const u32x4*)(k + at + 32 * s));
      qf[rb][s] = __builtin_bit_cast(bf16x8, *(const u32x4*)(q + at + 32 * s));
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int i = b * kBlock + 4 * g + e;
      vf[rb][e] = bf16_to_f32(v[((long)min(i, n - 1) * Hv + h) * DK + i0 + col]);
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
    s_see[tid][0] = see0;
    s_see[tid][1] = see1;
  }
  if (tid < 2 * kBlock) s_bad[tid >> 1][tid & 1] = 0;
#pragma unroll
  for (int rb = 0; rb < RB; ++rb) {
    const int b = rb ? NB - 1 - wave : wave;
    if (b >= NB) continue;
#pragma unroll
    for (int s = 0; s < NK; ++s) {
      s_k[b][s][lane] = kf[rb][s];
      if (NB == 4 && b == 3) s_q[s][lane] = qf[rb][s];
    }
  }
  if (wave < NK) {
    bf16x8 t[3];
    split3(sx, t);
#pragma unroll
    for (int p = 0; p < 3; ++p) s_s[wave][p][lane] = t[p];
  }
  __syncthreads();

  // ---- log2 gamma: float64 sums of the gates along the paths
  {
    double x[2] = {0.0, 0.0};
#pragma unroll 16
    for (int j = 0; j < SHARE; ++j) {
      const double y = s_gate[ppart * SHARE + j];
      x[j & 1] += pmask >> j & 1 ? y : 0.0;
    }
    double sum = x[0] + x[1];
    if (PARTS >= 2) sum = add_dpp<0xB1>(sum);     // quad_perm 1,0,3,2
    if (PARTS >= 4) sum = add_dpp<0x4E>(sum);     // quad_perm 2,3,0,1
    if (PARTS >= 8) sum = add_dpp<0x141>(sum);    // row_half_mirror
    if (PARTS >= 16) sum = add_dpp<0x140>(sum);   // row_mirror
    if (ppart == 0) {
      // differences of two such logs lose nothing: the high terms' is exact where it matters (near
      // each other), the low terms' is added
      const float hi = (float)sum;
      s_lg[pnode][0] = hi;
      s_lg[pnode][1] = fabsf(hi) < __builtin_inff() ? (float)(sum - (double)hi) : 0.f;
    }
  }

  // ---- products of this wave's rows with S, in three bf16 terms, the smallest first
  f32x4 yk[RB], yq[RB];
  {
    bf16x8 st[NK][3];
#pragma unroll
    for (int s = 0; s < NK; ++s)
#pragma unroll
      for (int p = 0; p < 3; ++p) st[s][p] = s_s[s][p][lane];
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

  // ---- blocks of M and of D o Q K^T. A row block's wave forms its blocks; of the last of four
  // rows waves 0 and 1 take one each.
  struct Rows {   // of this lane's nodes 4 g + e of a block
    float lh[4], ll[4], beta[4];
    uint64_t see[4][NB > 4 ? 2 : 1];
  };
  auto rows_of = [&](int b) __attribute__((always_inline)) -> Rows {
    Rows r;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int i = b * kBlock + 4 * g + e;
      r.lh[e] = s_lg[i][0];
      r.ll[e] = s_lg[i][1];
      r.beta[e] = s_beta[i];
      r.see[e][0] = s_see[i][0];
      if constexpr (NB > 4) r.see[e][1] = s_see[i][1];
    }
    return r;
  };
  auto pair = [&](int b, int c, const Rows& r, const bf16x8 (&kb)[NK], const bf16x8 (&qb)[NK]) __attribute__((always_inline)) -> uint32_t {
    uint32_t bad = 0;   // bit e: node 4 g + e has a key, beta or gate that is not finite (diagonal blocks)
    f32x4 kk = {0.f, 0.f, 0.f, 0.f}, qk = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int s = 0; s < NK; ++s) {
      const bf16x8 kc = s_k[c][s][lane];
      kk = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kb[s], kc, kk, 0, 0, 0);
      qk = __builtin_amdgcn_mfma_f32_16x16x32_bf16(qb[s], kc, qk, 0, 0, 0);
    }
    const int j = c * kBlock + col;
    const float jh = s_lg[j][0], jl = s_lg[j][1];
    float* mb = s_m[tri(b) + c] + 4 * g * kMStride + col;
    float* ab = s_a[tri(b) + c] + 4 * g * kMStride + col;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const uint64_t see = NB > 4 && c >= 4 ? r.see[e][NB > 4 ? 1 : 0] : r.see[e][0];
      const bool sees = (uint32_t)(see >> (16 * (c & 3))) >> col & 1, self = b == c && 4 * g + e == col;
      const float ratio = __builtin_amdgcn_exp2f((r.lh[e] - jh) + (r.ll[e] - jl));
      float m = -r.beta[e] * ratio * kk[e];
      if (!finite(m)) {
        if (self) bad |= 1u << e;
        m = 0.f;
      }
      mb[e * kMStride] = sees && !self ? m : 0.f;
      ab[e * kMStride] = sees ? ratio * qk[e] : 0.f;
    }
    return bad;
  };
#pragma unroll
  for (int rb = 0; rb < RB; ++rb) {
    const int b = rb ? NB - 1 - wave : wave;
    if (b >= NB || b * kBlock >= n) continue;
    const Rows r = rows_of(b);
    uint32_t bad = 0, bad_row = 0;   // bad_row: for this state row
    f32x4 rhs;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float gam = __builtin_amdgcn_exp2f(r.lh[e] + r.ll[e]);
      rhs[e] = r.beta[e] * (vf[rb][e] - gam * yk[rb][e]);
      if (b * kBlock + 4 * g + e >= n) rhs[e] = 0.f;
      if (!finite(rhs[e])) {
        bad_row |= 1u << e;
        rhs[e] = 0.f;
      }
      yq[rb][e] *= gam;
    }
    *(f32x4*)&s_rhs[col][b * kBlock + 4 * g] = rhs;
    for (int c = NB == 4 && b == 3 ? 2 : 0; c <= b; ++c) bad |= pair(b, c, r, kf[rb], qf[rb]);
    if (bad | bad_row) {
      for (int e = 0; e < 4; ++e) {
        const int i = b * kBlock + 4 * g + e;
        if (bad_row >> e & 1) atomicOr(&s_bad[col][i >> 6], 1ull << (i & 63));
        if (bad >> e & 1)
          for (int x = 0; x < kBlock; ++x) atomicOr(&s_bad[x][i >> 6], 1ull << (i & 63));
      }
    }
  }
  if (NB == 4 && wave < 2 && 3 * kBlock < n) {
    bf16x8 kb[NK], qb[NK];
#pragma unroll
    for (int s = 0; s < NK; ++s) {
      kb[s] = s_k[3 < NB ? 3 : 0][s][lane];
      qb[s] = s_q[NB == 4 ? s : 0][lane];
    }
    pair(3, wave, rows_of(3 < NB ? 3 : 0), kb, qb);
  }
  __syncthreads();

  // inverses of the diagonal blocks: 16 lanes a block, lane `col` its column of (I + M)^-1
  if (tid < N) {
    const int b = tid >> 4;
    const float* mb = s_m[tri(b) + b];
    f32x4 m[kBlock][4];   // all of it first: a row's reads would hold up its step
#pragma unroll
    for (int i = 1; i < kBlock; ++i)
#pragma unroll
      for (int j = 0; j < i; j += 4) m[i][j / 4] = *(const f32x4*)(mb + i * kMStride + j);
    asm volatile("" ::: "memory");
    float t[kBlock];
#pragma unroll
    for (int i = 0; i < kBlock; ++i) {
      t[i] = i == col ? 1.f : 0.f;
      if (NB > 1 || i < n) {   // rows of no node are zeros but for the one
        float x[4] = {t[i], 0.f, 0.f, 0.f};
#pragma unroll
        for (int j = 0; j < i; ++j) x[j & 3] = __builtin_fmaf(m[i][j / 4][j & 3], t[j], x[j & 3]);
        t[i] = (x[0] + x[1]) + (x[2] + x[3]);
      }
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
      const bool spoilt = (s_see[i][0] & bad0) | (s_see[i][1] & bad1);
      a.out[((long)i * Hv + h) * DK + i0 + col] = spoilt ? __builtin_nanf("") : a.scale * o[e];
    }
  }
}

template <int DK>
hipError_t delta_for(const DraftDeltaArgs& a, hipStream_t s) {
  const int blocks = (a.n_v_heads * (DK / kBlock) + 7) & ~7;   // xcd_remap wants a multiple of 8
  const auto run = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, dim3(blocks), dim3(kThreads), 0, s, a.state, a.q, a.k, a.v, a.beta, a.g, a.n,
                       (uint32_t)a.n_k_heads | (uint32_t)a.n_v_heads << 16, a);
    return hipGetLastError();
  };
  if (a.n_v_heads > UINT16_MAX) return hipErrorInvalidValue;
  if (a.n <= 16) return run(k_draft_delta<DK, 1>);
  if (a.n <= 32) return run(k_draft_delta<DK, 2>);
  if (a.n <= 64) return run(k_draft_delta<DK, 4>);
  return run(k_draft_delta<DK, 8>);
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
