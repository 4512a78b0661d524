// Norms of queries and keys for each head with the position rotation in the same pass
// (qk_norm_rope, draft_append).
//
// A row of one head is read once into registers, normed there, rotated and written: bound by
// HBM for many tokens, by latency for one. D / 16 lanes hold a row, two chunks of 8 elements
// a lane: in the rotated part the chunks j0 .. j0 + 7 and j0 + r/2 .. that form 8 pairs, so a
// pair never leaves its lane, and behind it two chunks in a row. A workgroup forms the sines of
// its few tokens once, into LDS, while its first rows are on their way, and shares them among
// the tokens' heads.
//
// Angles: position * theta^(-2j/r) / (2 pi) is formed in float64 (turns; the rate of pair
// 8 l + e is the product of two factors that come with the launch) and reduced to
// [-1/2, 1/2] there, so that a far position loses nothing; sine and cosine of the remaining
// fraction are fp32. Norm, weight and rotation are fp32, with one rounding to bf16.
//
// Inputs are read as streams: each is read once (2,048 tokens of 16 + 2 heads of 256 12.5 -> 11.3 us,
// and what other kernels left in the caches stays). Outputs are not written so: the attention behind
// finds them in the caches (4,096 tokens: 292 us for both; 312 with streamed outputs).
// Measured, 16 + 2 heads of 256, rotated whole: 8,191 tokens 31.5 us (151 MB, 4.8 TB/s, a copy
// 5.06), 1,000 7.6, one 3.4 (latency: the launch, one trip to memory, one rotation).
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
  __shared__ __attribute__((aligned(16))) float s_cos[kNormTokens * D / 2];
  __shared__ __attribute__((aligned(16))) float s_sin[kNormTokens * D / 2];
  __shared__ float s_row[PAIRED ? 1 : kGroups][PAIRED ? 1 : D];
  const int part = blockIdx.x % a.head_parts;
  const int tok0 = blockIdx.x / a.head_parts * a.tokens, n_tok = min(a.tokens, a.T - tok0);
  const int h0 = part * a.part_heads, nh = min(a.part_heads, a.heads_end[2] - h0);
  const int g = threadIdx.x / LANES, l = threadIdx.x % LANES;
  const int r = a.rotary, half = r >> 1;
  const int turning = PAIRED ? half >> 3 : 0;   // lanes that hold pairs
  const bool turns = l < turning;
  const int ea = turns ? 8 * l : (PAIRED ? r : 0) + 16 * (l - turning);   // first elements of the two chunks
  const int eb = turns ? half + 8 * l : ea + 8;

  // rows (token, head) of the workgroup, head fastest, dealt out to the lane groups; read one
  // ahead (in place too: a row is written by the lanes that have read it; two and more ahead were slower,
  // 8,191 tokens 38 - 44 us)
  struct Row {
    u32x4 a, b;
  };
  auto row_of = [&](int h, int& which, int& head) __attribute__((always_inline)) {
    which = h < a.heads_end[0] ? 0 : h < a.heads_end[1] ? 1 : 2;
    head = h - (which == 0 ? 0 : a.heads_end[which - 1]);
  };
  auto read = [&](int tok, int h) __attribute__((always_inline)) -> Row {
    int which, head;
    row_of(h0 + h, which, head);
    const bf16_t* x = a.in[which] + (long)(tok0 + tok) * a.in_stride[which] + (long)head * D;
    return Row{__builtin_nontemporal_load((const u32x4*)(x + ea)), __builtin_nontemporal_load((const u32x4*)(x + eb))};
  };
  auto forward = [&](int& tok, int& h) __attribute__((always_inline)) {
    for (h += kGroups; h >= nh && tok < n_tok; h -= nh) ++tok;
  };
  int tok = 0, h = g;
  for (; h >= nh && tok < n_tok; h -= nh) ++tok;
  Row next{};
  if (tok < n_tok) next = read(tok, h);

  for (int i = threadIdx.x; i < n_tok * half; i += kThreads) {
    const int t = i / half, j = i - t * half;
    double p = (double)(a.first_pos + (a.use_depth ? (int)a.depth[tok0 + t] : tok0 + t));
    if (a.pos) p = (double)a.pos[tok0 + t];
    turn_sincos(p * (a.turn_lane[j >> 3] * a.turn_elem[j & 7]), s_sin[i], s_cos[i]);
  }
  __syncthreads();

  while (tok < n_tok) {
    int which, head;
    row_of(h0 + h, which, head);
    bf16_t* y = a.out[which] + (long)(tok0 + tok) * a.out_stride[which] + (long)head * D;
    const float* cs = s_cos + tok * half;
    const float* sn = s_sin + tok * half;
    const u32x4 wa = next.a, wb = next.b;
    forward(tok, h);
    if (tok < n_tok) next = read(tok, h);
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
      const float inv = __builtin_amdgcn_rsqf(ss + a.eps);   // within a step of fp32
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
        float c[8], s[8];
#pragma unroll
        for (int e = 0; e < 8; e += 4) {
          *(f32x4*)(c + e) = *(const f32x4*)(cs + 8 * l + e);
          *(f32x4*)(s + e) = *(const f32x4*)(sn + 8 * l + e);
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float u = f[e], v = f[e + 8];
          f[e] = u * c[e] - v * s[e];
          f[e + 8] = v * c[e] + u * s[e];
        }
      }
    } else {
      // a group lies in one wave, whose LDS accesses keep their order
      float* row = s_row[g];
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
          f[e] = d < half ? row[j] * cs[j] - row[j + half] * sn[j] : row[j + half] * cs[j] + row[j] * sn[j];
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
  if (a.T <= 0) return hipSuccess;
  if (a.tokens < 1 || a.tokens > kNormTokens || a.part_heads * a.head_parts < a.heads_end[2]) return hipErrorInvalidValue;
  const long blocks = (long)((a.T + a.tokens - 1) / a.tokens) * a.head_parts;
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
