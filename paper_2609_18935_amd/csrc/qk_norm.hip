// Norms of queries and keys for each head with the position rotation in the same pass
// (qk_norm_rope, draft_append).
//
// A row of one head is read once into registers, normed there, rotated and written: bound by
// HBM for many tokens, by latency for one. D / 16 lanes hold a row, two chunks of 8 elements
// a lane: in the rotated part the chunks j0 .. j0 + 7 and j0 + r/2 .. that form 8 pairs, so a
// pair never leaves its lane, and behind it two chunks in a row. A lane forms the sines of its
// 8 pairs once and goes through `per_group` heads of one token with them.
//
// Angles: position * theta^(-2j/r) / (2 pi) is formed in float64 (turns; the rate of pair
// 8 l + e is the product of two factors that come with the launch) and reduced to
// [-1/2, 1/2] there, so that a far position loses nothing; sine and cosine of the remaining
// fraction are fp32. Norm, weight and rotation are fp32, with one rounding to bf16.
#include "draft.h"
#include "tailupdate.h"

namespace tu {

namespace {

constexpr int kThreads = 256;

template <int CTRL>
__device__ __forceinline__ float add_dpp(float x) {
  return x + __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), CTRL, 0xf, 0xf, true));
}

// Sum over a group of 4, 8 or 16 lanes, the same bits in each of them.
template <int LANES>
__device__ __forceinline__ float group_sum(float x) {
  x = add_dpp<0xB1>(x);                              // quad_perm 1,0,3,2
  x = add_dpp<0x4E>(x);                              // quad_perm 2,3,0,1
  if constexpr (LANES >= 8) x = add_dpp<0x141>(x);   // row_half_mirror
  if constexpr (LANES >= 16) x = add_dpp<0x140>(x);  // row_mirror
  return x;
}

__device__ __forceinline__ void unpack8(u32x4 w, float* f) {
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    f[2 * e] = __uint_as_float(w[e] << 16);
    f[2 * e + 1] = __uint_as_float(w[e] & 0xFFFF0000u);
  }
}

__device__ __forceinline__ u32x4 pack8(const float* f) {
  bf16x8 b;
#pragma unroll
  for (int e = 0; e < 8; ++e) b[e] = (__bf16)f[e];
  return __builtin_bit_cast(u32x4, b);
}

__device__ __forceinline__ void turn_sincos(double turns, float& sn, float& cs) {
  const float f = (float)(turns - __builtin_rint(turns));
  sincospif(2.f * f, &sn, &cs);
}

// PAIRED: r / 2 is a multiple of 8, a lane holds whole pairs. Otherwise the normed row goes
// through LDS and every lane forms its 16 elements one by one.
template <int D, bool PAIRED>
__global__ __launch_bounds__(kThreads) void k_qk_norm(NormArgs a) {
  constexpr int LANES = D / 16;
  constexpr int kGroups = kThreads / LANES;
  __shared__ float s_row[PAIRED ? 1 : kGroups][PAIRED ? 1 : D];
  const int group = blockIdx.x * kGroups + threadIdx.x / LANES;
  const int l = threadIdx.x % LANES;
  const int t = group / a.n_groups;
  if (t >= a.T) return;
  const int h0 = (group - t * a.n_groups) * a.per_group;
  const int h1 = min(h0 + a.per_group, (int)a.heads_end[2]);
  const int r = a.rotary, half = r >> 1;
  const int turning = PAIRED ? half >> 3 : 0;   // lanes that hold pairs
  const bool turns = l < turning;
  const int ea = turns ? 8 * l : (PAIRED ? r : 0) + 16 * (l - turning);   // first elements of the two chunks
  const int eb = turns ? half + 8 * l : ea + 8;

  double p = (double)(a.first_pos + (a.use_depth ? (int)a.depth[t] : t));
  if (a.pos) p = (double)a.pos[t];
  float sn[8], cs[8];
  if (PAIRED && turns) {
    const double rate = a.turn_lane[l] * p;
#pragma unroll
    for (int e = 0; e < 8; ++e) turn_sincos(rate * a.turn_elem[e], sn[e], cs[e]);
  }

  for (int h = h0; h < h1; ++h) {
    const int which = h < a.heads_end[0] ? 0 : h < a.heads_end[1] ? 1 : 2;
    const int head = h - (which == 0 ? 0 : a.heads_end[which - 1]);
    const bf16_t* x = a.in[which] + t * a.in_stride[which] + (long)head * D;
    bf16_t* y = a.out[which] + t * a.out_stride[which] + (long)head * D;
    const u32x4 wa = *(const u32x4*)(x + ea), wb = *(const u32x4*)(x + eb);
    if (which == 2) {   // values go as they are
      *(u32x4*)(y + ea) = wa;
      *(u32x4*)(y + eb) = wb;
      continue;
    }
    float f[16];
    unpack8(wa, f);
    unpack8(wb, f + 8);
    if (a.kind != TU_NORM_NONE) {
      float ss = 0.f;
#pragma unroll
      for (int e = 0; e < 16; ++e) ss = __builtin_fmaf(f[e], f[e], ss);
      ss = group_sum<LANES>(ss);
      if (a.kind == TU_NORM_RMS) ss *= 1.f / D;
      const float inv = 1.f / sqrtf(ss + a.eps);
#pragma unroll
      for (int e = 0; e < 16; ++e) f[e] *= inv;
      if (a.kind == TU_NORM_RMS && a.weight[which]) {
        float w[16];
        unpack8(*(const u32x4*)(a.weight[which] + ea), w);
        unpack8(*(const u32x4*)(a.weight[which] + eb), w + 8);
#pragma unroll
        for (int e = 0; e < 16; ++e) f[e] *= w[e] + a.weight_offset;
      }
    }
    if constexpr (PAIRED) {
      if (turns) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float u = f[e], v = f[e + 8];
          f[e] = u * cs[e] - v * sn[e];
          f[e + 8] = v * cs[e] + u * sn[e];
        }
      }
    } else {
      // a group lies in one wave, whose LDS accesses keep their order
      float* row = s_row[threadIdx.x / LANES];
      __builtin_amdgcn_wave_barrier();
#pragma unroll
      for (int e = 0; e < 16; ++e) row[ea + e] = f[e];
      __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
      __builtin_amdgcn_wave_barrier();
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        const int d = ea + e;
        if (d < r) {
          const int j = d < half ? d : d - half;
          float s1, c1;
          turn_sincos(a.turn_lane[j >> 3] * p * a.turn_elem[j & 7], s1, c1);
          f[e] = d < half ? row[j] * c1 - row[j + half] * s1 : row[j + half] * c1 + row[j] * s1;
        }
      }
      __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
      __builtin_amdgcn_wave_barrier();
    }
    *(u32x4*)(y + ea) = pack8(f);
    *(u32x4*)(y + eb) = pack8(f + 8);
  }
}

}  // namespace

hipError_t launch_qk_norm(const NormArgs& a, int head_dim, hipStream_t s) {
  const long groups = (long)a.T * a.n_groups;
  if (groups <= 0) return hipSuccess;
  const int per_block = kThreads * 16 / head_dim;
  const long blocks = (groups + per_block - 1) / per_block;
  const bool paired = (a.rotary & 15) == 0;
  const auto run = [&](auto pairs, auto any) {
    if (paired) hipLaunchKernelGGL(pairs, dim3(blocks), dim3(kThreads), 0, s, a);
    else hipLaunchKernelGGL(any, dim3(blocks), dim3(kThreads), 0, s, a);
    return hipGetLastError();
  };
  switch (head_dim) {
    case 256: return run(k_qk_norm<256, true>, k_qk_norm<256, false>);
    case 128: return run(k_qk_norm<128, true>, k_qk_norm<128, false>);
    case 64: return run(k_qk_norm<64, true>, k_qk_norm<64, false>);
    default: return hipErrorInvalidValue;
  }
}

}  // namespace tu
