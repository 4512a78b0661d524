// Attention of a tree of drafted tokens over the cache: node i sees every cached row, its
// ancestors' rows and its own.
//
// The G query heads of a KV head are packed as rows (row = node * G + h mod G). A workgroup
// takes 256 rows (8 waves of 32) of one KV head and one split of the key range. K and V come
// as they lie in the cache, in stages of 16 KB each (32 keys of 256 dims), by LDS DMA into a
// ring of four, three of them in flight: the cache is asked for far ahead whatever the number
// of rows, and waves without rows only load.
//
// S^T = K Q^T on v_mfma_f32_32x32x16_bf16, so that a lane holds 16 keys of one query and the
// running maximum and sum are per lane. P is rounded to f16 (10 stored mantissa bits; bf16's 7
// would add an error as large as the output's own rounding), so V must be f16 too: every
// thread turns the chunks that it has itself loaded into f16 in place, before the barrier that
// shows the stage to the others. O^T += V^T P^T on the f16 MFMA, V transposed on its way by
// ds_read_b64_tr_b16. Softmax sums, the running maximum (moved only when exceeded by 2^8) and
// O are fp32.
//
// A row of D dims lies in LDS as D / 8 chunks of 16 bytes, permuted within the row so that the
// rows read together fall into different banks: chunk c of K row r at c ^ (r mod 16), of V row
// r at c ^ 2 (r mod 8); less where a row has fewer chunks.
//
// The tree only matters to the units of 32 keys that reach past row len: there each lane
// shifts its node's mask to the unit and drops the keys whose bit is clear.
#include "attention_tile.h"
#include "draft.h"

namespace tu {

namespace {

constexpr int kThreads = 512;
constexpr int kStages = 4;
constexpr int kLoads = 4;   // DMA loads of a thread for a stage: two of K, two of V
constexpr int kLgkmWait0 = 15 | (7 << 4) | (0 << 8) | (3 << 14);

typedef __attribute__((__vector_size__(4 * sizeof(short)))) short s16x4;
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;

// One array per stage and tensor, so that the compiler sees that the DMA into one does not
// alias the reads of another.
__shared__ __attribute__((aligned(16))) char g_k0[kDraftStageBytes];
__shared__ __attribute__((aligned(16))) char g_k1[kDraftStageBytes];
__shared__ __attribute__((aligned(16))) char g_k2[kDraftStageBytes];
__shared__ __attribute__((aligned(16))) char g_k3[kDraftStageBytes];
__shared__ __attribute__((aligned(16))) char g_v0[kDraftStageBytes];
__shared__ __attribute__((aligned(16))) char g_v1[kDraftStageBytes];
__shared__ __attribute__((aligned(16))) char g_v2[kDraftStageBytes];
__shared__ __attribute__((aligned(16))) char g_v3[kDraftStageBytes];

template <int B>
struct IntC {
  static constexpr int value = B;
};
template <int B>
__device__ __forceinline__ char* stage_k() {
  return B == 0 ? g_k0 : B == 1 ? g_k1 : B == 2 ? g_k2 : g_k3;
}
template <int B>
__device__ __forceinline__ char* stage_v() {
  return B == 0 ? g_v0 : B == 1 ? g_v1 : B == 2 ? g_v2 : g_v3;
}

// Barrier that does not wait for the loads in flight.
__device__ __forceinline__ void wg_barrier() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt(kLgkmWait0);
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

template <int D>
__global__ __launch_bounds__(kThreads) __attribute__((amdgpu_waves_per_eu(2, 2))) void k_draft_attn(DraftAttnArgs a) {
  constexpr int NS = D / 16;                 // 16-dim steps of S^T = K Q^T
  constexpr int NDB = D / 32;                // 32-dim blocks of O^T
  constexpr int RC = D / 8;                  // 16-byte chunks per row
  constexpr int SK = draft_stage_keys(D);    // keys of a stage
  constexpr int KSWZ = RC < 16 ? RC - 1 : 15;
  constexpr int VSWZ = RC / 2 < 8 ? RC / 2 - 1 : 7;
  static_assert(SK * RC == 2 * kThreads, "two chunks of K and of V per thread and stage");

  const int item = xcd_remap(blockIdx.x, gridDim.x);
  const int Hq = a.n_q_heads, Hkv = a.n_kv_heads, G = Hq / Hkv;
  if (item >= Hkv * a.n_splits * a.n_tiles) return;
  status_mark(a.status);
  // the row tiles of one key range are neighbours: they share a die's L2
  int local = item;
  const int tile = __builtin_amdgcn_readfirstlane(local % a.n_tiles);
  local /= a.n_tiles;
  const int split = __builtin_amdgcn_readfirstlane(local % a.n_splits);
  const int hkv = __builtin_amdgcn_readfirstlane(local / a.n_splits);
  const int len = a.len, n = a.n;
  const int rows_total = n * G;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int hl = lane >> 5, col = lane & 31;
  const int r = tile * kDraftRows + wave * 32 + col;
  const bool row_ok = r < rows_total;
  const int node = row_ok ? r / G : n - 1;
  const int qh = hkv * G + (row_ok ? r - (r / G) * G : 0);
  const int n_valid = len + n;
  const int n_st = (n_valid + SK - 1) / SK;
  const int st0 = (int)((long)n_st * split / a.n_splits), st1 = (int)((long)n_st * (split + 1) / a.n_splits);
  const long rs = (long)Hkv * D;
  const bf16_t* kbase = a.k_cache + (long)hkv * D;
  const bf16_t* vbase = a.v_cache + (long)hkv * D;

  bf16x8 qf[NS];
  {
    const bf16_t* qrow = a.q_hat + ((long)node * Hq + qh) * D + 8 * hl;   // rows past the last repeat one (dropped)
#pragma unroll
    for (int s = 0; s < NS; ++s) qf[s] = __builtin_bit_cast(bf16x8, *(const u32x4*)(qrow + 16 * s));
  }

  // ---- a stage: LDS chunk i * 512 + tid of K and of V is loaded by load i of the thread.
  // The resource ends at the cache's data: rows past it, and stages past the split, are zeros.
  // The second load's row lies a multiple of 16 (of 8 with 8 chunks) rows on: the same chunk.
  constexpr int LR = kThreads / RC;
  static_assert(LR % (KSWZ + 1) == 0 && LR % (VSWZ + 1) == 0, "both loads of a thread take the same chunk");
  const int lrow = tid / RC, lc = tid % RC;
  const uint32_t koff = (uint32_t)(lrow * (int)rs * 2 + (lc ^ (lrow & KSWZ)) * 16);
  const uint32_t voff = (uint32_t)(lrow * (int)rs * 2 + (lc ^ (2 * (lrow & VSWZ))) * 16);
  const uint32_t lstep = (uint32_t)(LR * (int)rs * 2);
  auto load = [&](auto bc, int st) __attribute__((always_inline)) {
    constexpr int B = decltype(bc)::value;
    const int key0 = st * SK;
    const int bytes = st < st1 ? min(n_valid - key0, SK) * (int)rs * 2 - ((int)rs - D) * 2 : 0;
    const long off = (long)key0 * rs;
#pragma unroll
    for (int i = 0; i < 2; ++i)
      dma16(kbase + off, bytes, koff, i * lstep, stage_k<B>() + (i * kThreads + wave * 64) * 16);
#pragma unroll
    for (int i = 0; i < 2; ++i)
      dma16(vbase + off, bytes, voff, i * lstep, stage_v<B>() + (i * kThreads + wave * 64) * 16);
  };

  f32x16 o[NDB];
#pragma unroll
  for (int db = 0; db < NDB; ++db)
#pragma unroll
    for (int e = 0; e < 16; ++e) o[db][e] = 0.f;
  float m_run = -__builtin_inff(), l_run = 0.f;
  const float c2 = a.scale_log2;
  bool big = false;

  // transposing reads of V (see the unit below): block db lies 256 bytes behind block db - 4
  constexpr int NVA = NDB < 4 ? NDB : 4;
  uint32_t vaddr[NVA];
  {
    const int i = lane & 15, g = lane >> 4;
    const int row = 4 * (g >> 1) + (i >> 2);
    const int c0 = 2 * (g & 1) + ((i & 3) >> 1);
#pragma unroll
    for (int db = 0; db < NVA; ++db)
      vaddr[db] = (uint32_t)(row * D * 2 + (((4 * db + c0) ^ (2 * (row & VSWZ))) * 16) + (i & 1) * 8);
  }

  // K row `col`, chunk hl ^ (col mod 16); chunk 2 s + hl is this address ^ 32 s
  const uint32_t kaddr = (uint32_t)(col * D * 2 + ((hl ^ (col & KSWZ)) * 16));

  // ---- this thread's two chunks of V to f16, in place
  auto to_f16 = [&](auto bc) __attribute__((always_inline)) {
    constexpr int B = decltype(bc)::value;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      u32x4* at = (u32x4*)(stage_v<B>() + (i * kThreads + tid) * 16);
      const u32x4 w = *at;
      f16x8 x;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float lo = __uint_as_float(w[e] << 16), hi = __uint_as_float(w[e] & 0xFFFF0000u);
        big |= !(fabsf(lo) < 65536.f) | !(fabsf(hi) < 65536.f);
        x[2 * e] = (_Float16)lo;
        x[2 * e + 1] = (_Float16)hi;
      }
      *at = __builtin_bit_cast(u32x4, x);
    }
  };

  // Keeps n MFMAs fed by their LDS fragment reads (PER reads each), two fragments ahead: bounds the
  // fragment registers in flight (the compiler would otherwise issue every read up front).
  constexpr int kMfma = 0x008, kDsRead = 0x100;
  auto sched_reads = [&](auto nc, auto per) __attribute__((always_inline)) {
    constexpr int N = decltype(nc)::value, PER = decltype(per)::value;
    __builtin_amdgcn_sched_group_barrier(kDsRead, PER, 0);
#pragma unroll
    for (int i = 0; i < N; ++i) {
      if (i < N - 1) __builtin_amdgcn_sched_group_barrier(kDsRead, PER, 0);
      __builtin_amdgcn_sched_group_barrier(kMfma, 1, 0);
    }
  };

  // ---- 32 keys (unit u of the stage in B, first key kb0)
  auto unit = [&](auto bc, int u, int kb0) __attribute__((always_inline)) {
    constexpr int B = decltype(bc)::value;
    const char* ks = stage_k<B>() + u * 32 * D * 2;
    uint32_t kx = kaddr;
    asm volatile("" : "+v"(kx));   // formed per unit: hoisted, the 8 addresses would cost registers
    const char* vs = stage_v<B>() + u * 32 * D * 2;
    f32x16 sacc;
#pragma unroll
    for (int e = 0; e < 16; ++e) sacc[e] = 0.f;
#pragma unroll
    for (int s = 0; s < NS; ++s) {
      const bf16x8 ka = __builtin_bit_cast(bf16x8, *(const u32x4*)(ks + (kx ^ (32 * s & 16 * KSWZ)) + (32 * s & ~(16 * KSWZ))));
      sacc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(ka, qf[s], sacc, 0, 0, 0);
    }
    sched_reads(IntC<NS>{}, IntC<1>{});
    if (kb0 + 31 >= len) {   // reaches the tree (uniform)
      // bit x of `keys`: this query sees key kb0 + x
      uint32_t keys;
      const int d = kb0 - len;
      const uint64_t m0 = a.seen.m[node][0], m1 = a.seen.m[node][1];
      if (d <= 0) {
        keys = d > -32 ? (uint32_t)(m0 << -d) | ((1u << -d) - 1u) : 0xFFFFFFFFu;
      } else if (d < 64) {
        keys = (uint32_t)(m0 >> d | m1 << (64 - d));
      } else {
        keys = d < 128 ? (uint32_t)(m1 >> (d - 64)) : 0u;
      }
      keys >>= 4 * hl;
#pragma unroll
      for (int e = 0; e < 16; ++e)
        if (!(keys >> (8 * (e >> 2) + (e & 3)) & 1)) sacc[e] = -__builtin_inff();
    }
    float mx = -__builtin_inff();
#pragma unroll
    for (int e = 0; e < 16; ++e) mx = fmaxf(mx, sacc[e]);
    const auto sw = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(uint32_t, mx),
                                                     __builtin_bit_cast(uint32_t, mx), false, false);
    mx = fmaxf(__builtin_bit_cast(float, (uint32_t)sw[0]), __builtin_bit_cast(float, (uint32_t)sw[1])) * c2;
    if (__any(mx > m_run + kTau)) {
      const float m_new = fmaxf(m_run, mx);
      const float alpha = m_new == -__builtin_inff() ? 1.f : __builtin_amdgcn_exp2f(m_run - m_new);
      m_run = m_new;
      l_run *= alpha;
#pragma unroll
      for (int db = 0; db < NDB; ++db) scale_acc(o[db], alpha);
    }
    const float m_use = m_run == -__builtin_inff() ? 0.f : m_run;
    f16x8 pf[2];
    float ps[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      const float p = __builtin_amdgcn_exp2f(__builtin_fmaf(sacc[e], c2, -m_use));
      ps[e & 3] += p;
      pf[e >> 3][e & 7] = (_Float16)p;
    }
    l_run += (ps[0] + ps[1]) + (ps[2] + ps[3]);
    // lane group g reads keys 4 (g >> 1) + 0 .. 3 (+ 16 ks, + 8) at dims 32 db + 16 (g & 1) ..
#pragma unroll
    for (int k16 = 0; k16 < 2; ++k16) {
#pragma unroll
      for (int db = 0; db < NDB; ++db) {
        const s16x4 x0 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(vs + vaddr[db & 3] + (db >> 2) * 256 + (16 * k16) * D * 2));
        const s16x4 x1 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(vs + vaddr[db & 3] + (db >> 2) * 256 + (16 * k16 + 8) * D * 2));
        const u32x2 w0 = __builtin_bit_cast(u32x2, x0), w1 = __builtin_bit_cast(u32x2, x1);
        const f16x8 va = __builtin_bit_cast(f16x8, u32x4{w0[0], w0[1], w1[0], w1[1]});
        o[db] = __builtin_amdgcn_mfma_f32_32x32x16_f16(va, pf[k16], o[db], 0, 0, 0);
      }
    }
    sched_reads(IntC<2 * NDB>{}, IntC<2>{});
  };

  const bool busy = tile * kDraftRows + wave * 32 < rows_total;   // a wave without rows only loads
  auto step = [&](auto bc, int st) __attribute__((always_inline)) {
    constexpr int B = decltype(bc)::value;
    __builtin_amdgcn_s_waitcnt(vm_wait((kStages - 2) * kLoads));   // this thread's loads of the stage have landed
    asm volatile("" ::: "memory");
    to_f16(bc);
    wg_barrier();   // everyone's have; everyone is done with the stage before
    load(IntC<(B + kStages - 1) % kStages>{}, st + kStages - 1);
    if (busy) {
#pragma unroll
      for (int u = 0; u < SK / 32; ++u) {
        const int kb0 = st * SK + 32 * u;
        if (SK == 32 || kb0 < n_valid) unit(bc, u, kb0);
      }
    }
  };

  if (st0 < st1) {
    load(IntC<0>{}, st0);
    load(IntC<1>{}, st0 + 1);
    load(IntC<2>{}, st0 + 2);
    for (int st = st0; st < st1; st += kStages) {
      step(IntC<0>{}, st);
      if (st + 1 < st1) step(IntC<1>{}, st + 1);
      if (st + 2 < st1) step(IntC<2>{}, st + 2);
      if (st + 3 < st1) step(IntC<3>{}, st + 3);
    }
    __builtin_amdgcn_s_waitcnt(vm_wait(0));   // no load may outlive the workgroup
  }
  if (big) status_raise(a.status, kFaultRange);

  const auto lsw = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(uint32_t, l_run),
                                                    __builtin_bit_cast(uint32_t, l_run), false, false);
  const float l_tot = __builtin_bit_cast(float, (uint32_t)lsw[0]) + __builtin_bit_cast(float, (uint32_t)lsw[1]);
  if (!row_ok) return;
  const float inv = l_tot == 0.f ? 0.f : 1.f / l_tot;   // 0: no key of this split is seen; NaN goes on
  const long row = (long)node * Hq + qh;
  if (a.n_splits == 1) {
    bf16_t* orow = a.out + row * D;
#pragma unroll
    for (int db = 0; db < NDB; ++db)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        typedef __attribute__((__vector_size__(4 * sizeof(__bf16)))) __bf16 bf16x4;
        const bf16x4 v = {(__bf16)(o[db][4 * i] * inv), (__bf16)(o[db][4 * i + 1] * inv),
                          (__bf16)(o[db][4 * i + 2] * inv), (__bf16)(o[db][4 * i + 3] * inv)};
        *(bf16x4*)(orow + db * 32 + 8 * i + 4 * hl) = v;
      }
  } else {
    const long prow = (long)split * n * Hq + row;
    _Float16* orow = a.part_o + prow * D;
#pragma unroll
    for (int db = 0; db < NDB; ++db)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const f16x4 v = {(_Float16)(o[db][4 * i] * inv), (_Float16)(o[db][4 * i + 1] * inv),
                         (_Float16)(o[db][4 * i + 2] * inv), (_Float16)(o[db][4 * i + 3] * inv)};
        *(f16x4*)(orow + db * 32 + 8 * i + 4 * hl) = v;
      }
    if (hl == 0) {
      a.part_ml[prow * 2] = l_tot == 0.f ? -__builtin_inff() : m_run == -__builtin_inff() ? 0.f : m_run;
      a.part_ml[prow * 2 + 1] = l_tot;
    }
  }
}

// Joins the splits of one (node, head) row a workgroup: D / 4 lanes hold the row, 4 dims each,
// the lane groups take the splits in turn and are added up through LDS in a fixed order.
constexpr int kMergeThreads = 256;
template <int D>
__global__ __launch_bounds__(kMergeThreads) void k_draft_merge(DraftAttnArgs a) {
  constexpr int LANES = D / 4;
  constexpr int GROUPS = kMergeThreads / LANES;
  __shared__ float s_w[128];
  __shared__ __attribute__((aligned(16))) float s_o[GROUPS][D];
  const long row = blockIdx.x, R = (long)a.n * a.n_q_heads;
  const int tid = threadIdx.x, g = tid / LANES, l = tid % LANES;
  // weights of the splits: every wave forms them alike
  const int lane = tid & 63;
  float m[2], w[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int s = lane + 64 * i;
    m[i] = -__builtin_inff();
    w[i] = 0.f;
    if (s < a.n_splits) {
      const float* ml = a.part_ml + ((long)s * R + row) * 2;
      m[i] = ml[0];
      w[i] = ml[1];
    }
  }
  float M = fmaxf(m[0], m[1]);
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) M = fmaxf(M, __shfl_xor(M, d, 64));
  float L = 0.f;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    w[i] = m[i] == -__builtin_inff() ? 0.f : w[i] * __builtin_amdgcn_exp2f(m[i] - M);
    L += w[i];
  }
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) L += __shfl_xor(L, d, 64);
  if (tid < 64) {
    s_w[lane] = w[0];
    s_w[lane + 64] = w[1];
  }
  __syncthreads();
  f32x4 acc = {0.f, 0.f, 0.f, 0.f};
  const _Float16* po = a.part_o + row * D + 4 * l;
#pragma unroll 8
  for (int s = g; s < a.n_splits; s += GROUPS) {
    const float ws = s_w[s];
    const f16x4 v = *(const f16x4*)(po + (long)s * R * D);
    if (ws != 0.f) {
#pragma unroll
      for (int e = 0; e < 4; ++e) acc[e] += ws * (float)v[e];
    }
  }
  *(f32x4*)&s_o[g][4 * l] = acc;
  __syncthreads();
  for (int d = tid; d < D; d += kMergeThreads) {
    float sum = 0.f;
#pragma unroll
    for (int i = 0; i < GROUPS; ++i) sum += s_o[i][d];
    ((__bf16*)a.out)[row * D + d] = (__bf16)(sum / L);
  }
}

}  // namespace

hipError_t launch_draft_attention(const DraftAttnArgs& a, int head_dim, hipStream_t s) {
  const int items = a.n_kv_heads * a.n_splits * a.n_tiles;
  const int blocks = (items + kXcds - 1) / kXcds * kXcds;   // a whole number per die (xcd_remap)
  if (items <= 0) return hipSuccess;
  switch (head_dim) {
    case 256: hipLaunchKernelGGL(k_draft_attn<256>, dim3(blocks), dim3(kThreads), 0, s, a); break;
    case 128: hipLaunchKernelGGL(k_draft_attn<128>, dim3(blocks), dim3(kThreads), 0, s, a); break;
    case 64: hipLaunchKernelGGL(k_draft_attn<64>, dim3(blocks), dim3(kThreads), 0, s, a); break;
    default: return hipErrorInvalidValue;
  }
  return hipGetLastError();
}

hipError_t launch_draft_merge(const DraftAttnArgs& a, int head_dim, hipStream_t s) {
  const int rows = a.n * a.n_q_heads;
  if (rows <= 0) return hipSuccess;
  switch (head_dim) {
    case 256: hipLaunchKernelGGL(k_draft_merge<256>, dim3(rows), dim3(kMergeThreads), 0, s, a); break;
    case 128: hipLaunchKernelGGL(k_draft_merge<128>, dim3(rows), dim3(kMergeThreads), 0, s, a); break;
    case 64: hipLaunchKernelGGL(k_draft_merge<64>, dim3(rows), dim3(kMergeThreads), 0, s, a); break;
    default: return hipErrorInvalidValue;
  }
  return hipGetLastError();
}

}  // namespace tu
