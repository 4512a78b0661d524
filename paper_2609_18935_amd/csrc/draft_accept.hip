// Keeping the accepted path of a draft: one launch for the attention layers' cache rows, the
// delta layers' states and the convolutions' carried rows.
//
// Delta states: the recurrence token by token along the path, as k_delta_step without outputs:
// 16 lanes hold a row of one value head in registers from the first token to the last, two rows
// at a time (two chains of dependent sums in flight, a token's operands read once for both).
// Bound by HBM: each state is read and written once. Measured: six tokens into 36 states of 32 heads
// of 128 x 128, 12 pairs of caches and 36 convolutions of 8,192 channels 35 us in one launch (158 MB,
// 4.5 TB/s; a copy 5.06); three tokens into three of each state and one pair of caches 5.4 us (latency: the
// tokens one behind the other).
//
// Cache rows: a thread takes one 16-byte column of a K or V buffer and moves it row by row in
// path order. Row len + j only ever overwrites rows whose own move came earlier (path[j] >= j,
// increasing), so nothing is lost in place.
//
// Convolutions: a thread takes 8 channels, reads the width - 1 rows that stay, then writes.
#include <algorithm>

#include "draft.h"

namespace tu {

namespace {

constexpr int kThreads = 256;
constexpr int kPairs = 16;             // row pairs of a workgroup
constexpr int kRows = 2 * kPairs;
constexpr int kLanes = kThreads / kPairs;
constexpr int kBatch = 8;   // cache rows in flight

template <int ROT>
__device__ __forceinline__ float add_rotated(float x) {
  return x + __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), 0x120 + ROT, 0xf, 0xf,
                                                                   true));
}
__device__ __forceinline__ float row_sum(float x) {
  return add_rotated<1>(add_rotated<2>(add_rotated<4>(add_rotated<8>(x))));
}

template <int DK>
__device__ __forceinline__ void advance(const AcceptArgs& a, int item) {
  constexpr int NC = DK / kLanes;
  constexpr int NSL = DK / kRows;
  const int Hv = a.n_v_heads, Hk = a.n_k_heads;
  const int li = item / (Hv * NSL);
  const int rem = item - li * Hv * NSL;
  const int h = rem / NSL, kh = h / (Hv / Hk);
  const int row = (rem - h * NSL) * kRows + threadIdx.x / kLanes, l = threadIdx.x % kLanes;
  const AcceptDelta L = a.delta[li];
  // a token's operands, requested a token ahead
  struct Token {
    uint32_t k[NC / 2];
    uint32_t v[2];
    float beta, g;
  };
  auto token = [&](int j) __attribute__((always_inline)) -> Token {
    Token x;
    const long t = a.path[j];
    const bf16_t* kp = L.k + (t * Hk + kh) * DK + NC * l;
    if constexpr (NC == 8) *(u32x4*)x.k = *(const u32x4*)kp;
    else *(u32x2*)x.k = *(const u32x2*)kp;
    const bf16_t* vp = L.v + (t * Hv + h) * DK + row;
    x.v[0] = vp[0];
    x.v[1] = vp[kPairs];
    x.beta = L.beta[t * Hv + h];
    x.g = L.g[t * Hv + h];
    return x;
  };
  float* sp = L.state + ((long)h * DK + row) * DK + NC * l;
  float st[2][NC];
#pragma unroll
  for (int r = 0; r < 2; ++r)
#pragma unroll
    for (int c = 0; c < NC; c += 4) {
      const f32x4 x = *(const f32x4*)(sp + r * kPairs * DK + c);
#pragma unroll
      for (int e = 0; e < 4; ++e) st[r][c + e] = x[e];
    }
  Token now = token(0);
  for (int j = 0; j < a.n_path; ++j) {
    const Token next = token(min(j + 1, a.n_path - 1));
    float kf[NC];
#pragma unroll
    for (int e = 0; e < NC / 2; ++e) {
      kf[2 * e] = __uint_as_float(now.k[e] << 16);
      kf[2 * e + 1] = __uint_as_float(now.k[e] & 0xFFFF0000u);
    }
    const float g = now.g < 0x1p-100f ? 0x1p-100f : now.g;
    float d[2][2] = {{0.f, 0.f}, {0.f, 0.f}}, u[2];
#pragma unroll
    for (int c = 0; c < NC; ++c)
#pragma unroll
      for (int r = 0; r < 2; ++r) {
        st[r][c] *= g;
        d[r][c & 1] = __builtin_fmaf(st[r][c], kf[c], d[r][c & 1]);
      }
#pragma unroll
    for (int r = 0; r < 2; ++r) u[r] = now.beta * (bf16_to_f32(now.v[r]) - row_sum(d[r][0] + d[r][1]));
#pragma unroll
    for (int c = 0; c < NC; ++c)
#pragma unroll
      for (int r = 0; r < 2; ++r) st[r][c] = __builtin_fmaf(u[r], kf[c], st[r][c]);
    now = next;
  }
#pragma unroll
  for (int r = 0; r < 2; ++r)
#pragma unroll
    for (int c = 0; c < NC; c += 4)
      *(f32x4*)(sp + r * kPairs * DK + c) = f32x4{st[r][c], st[r][c + 1], st[r][c + 2], st[r][c + 3]};
}

__device__ __forceinline__ void carry_rows(const AcceptArgs& a, int block) {
  int ci = 0;
  while (ci + 1 < a.n_conv && a.conv[ci + 1].block_begin <= block) ++ci;
  const AcceptConv C = a.conv[ci];
  const int c0 = ((block - C.block_begin) * kThreads + threadIdx.x) * 8;
  if (c0 >= C.channels) return;
  const int keep = a.width - 1;
  u32x4 rows[7];
#pragma unroll
  for (int i = 0; i < 7; ++i) {
    if (i >= keep) break;
    const int at = a.n_path + i;   // row of [carried; path]
    rows[i] = at < keep ? *(const u32x4*)(C.state + (long)at * C.channels + c0)
                        : *(const u32x4*)(C.x + (long)a.path[at - keep] * C.channels + c0);
  }
#pragma unroll
  for (int i = 0; i < 7; ++i) {
    if (i >= keep) break;
    *(u32x4*)(C.state + (long)i * C.channels + c0) = rows[i];
  }
}

__device__ __forceinline__ void move_rows(const AcceptArgs& a, int block) {
  const int bi = block / a.row_blocks;
  const int c = (block - bi * a.row_blocks) * kThreads + threadIdx.x;
  if (bi == 0 && a.pos)
    for (int j = c; j < a.n_path; j += a.row_blocks * kThreads) a.pos[a.len + j] = (int32_t)(a.next_pos + j);
  if (bi >= a.n_bufs || c >= a.row_chunks) return;
  u32x4* base = (u32x4*)a.bufs[bi] + a.len * a.row_chunks + c;
  for (int j0 = 0; j0 < a.n_path; j0 += kBatch) {
    u32x4 x[kBatch];
#pragma unroll
    for (int j = 0; j < kBatch; ++j)
      if (j0 + j < a.n_path) x[j] = base[(long)a.path[j0 + j] * a.row_chunks];
#pragma unroll
    for (int j = 0; j < kBatch; ++j)
      if (j0 + j < a.n_path && a.path[j0 + j] != j0 + j) base[(long)(j0 + j) * a.row_chunks] = x[j];
  }
}

template <int DK>
__global__ __launch_bounds__(kThreads) void k_draft_accept(AcceptArgs a) {
  const int b = blockIdx.x;
  if (b < a.delta_blocks) advance<DK>(a, b);
  else if (b < a.delta_blocks + a.conv_blocks) carry_rows(a, b - a.delta_blocks);
  else move_rows(a, b - a.delta_blocks - a.conv_blocks);
}

}  // namespace

hipError_t launch_draft_accept(AcceptArgs& a, hipStream_t s) {
  a.delta_blocks = a.n_delta > 0 ? a.n_delta * a.n_v_heads * (a.d / kRows) : 0;
  a.conv_blocks = 0;
  for (int i = 0; i < a.n_conv; ++i) {
    a.conv[i].block_begin = a.conv_blocks;
    a.conv_blocks += (a.conv[i].channels / 8 + kThreads - 1) / kThreads;
  }
  a.row_blocks = std::max(1, (a.row_chunks + kThreads - 1) / kThreads);
  const int row_total = a.row_blocks * std::max(a.n_bufs, a.pos ? 1 : 0);
  const int blocks = a.delta_blocks + a.conv_blocks + row_total;
  if (blocks <= 0) return hipSuccess;
  if (a.n_delta > 0 && a.d == 64) hipLaunchKernelGGL(k_draft_accept<64>, dim3(blocks), dim3(kThreads), 0, s, a);
  else hipLaunchKernelGGL(k_draft_accept<128>, dim3(blocks), dim3(kThreads), 0, s, a);
  return hipGetLastError();
}

}  // namespace tu
