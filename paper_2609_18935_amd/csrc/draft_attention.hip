// Attention of a tree of drafted tokens over the cache: node i sees every cached row, its
// ancestors' rows and its own.
//
// The G query heads of a KV head are packed as rows (row = node * G + h mod G). A workgroup
// takes up to 256 rows (8 waves of 32, two per SIMD) of one KV head and one split of the key range.
// K and V come as they lie in the cache, in stages of 16 KB each (32 keys of 256 dims), by LDS
// DMA into rings of four, two to three of them in flight: the cache is asked for far ahead whatever
// the number of rows, and waves without rows only load.
//
// S^T = K Q^T on v_mfma_f32_32x32x16_bf16, so that a lane holds 16 keys of one query and the
// running maximum and sum are per lane. P is rounded to f16 (10 stored mantissa bits; bf16's 7
// would add an error as large as the output's own rounding), so V must be f16 too: every
// thread turns the chunks that it has itself loaded into f16 in place, a barrier before anyone
// reads them. O^T += V^T P^T on the f16 MFMA, V transposed on its way by ds_read_b64_tr_b16.
// Softmax sums, the running maximum and O are fp32; partial outputs of splits are normalised and
// rounded to f16.
//
// The two waves of a SIMD take turns: while waves 0 - 3 run the matrix products of a stage (P V of
// the stage before, then K Q^T), waves 4 - 7 run the softmax of theirs, and a barrier later the
// other way round. With rows for four waves or fewer, waves 4 - 7 only load, and products and softmax of a
// stage follow one another.
//
// A row of D dims lies in LDS as D / 8 chunks of 16 bytes, permuted within the row so that the
// rows read together fall into different banks: chunk c of K row r at c ^ (r mod 16), of V row r at
// c ^ 4 (r mod 4) (four chunks of four rows at a time); less where a row has fewer chunks. With 2 (r mod 8)
// for V, 29 % of the LDS's busy cycles were conflicts; now 1 %.
//
// The tree only matters to the units of 32 keys that reach past row len: there each lane shifts its
// node's mask to the unit and drops the keys whose bit is clear.
//
// Measured with heads 16 / 2 of 256: 64 nodes over 65,536 rows 70 us at the least (135 MB, 69 GFLOP) + 8 for the
// join (34 MB of partial outputs), 78 to 86 together in a long run; 2.1 us a stage (1.17 PFLOP/s, 0.91 of what an
// 8192^3 bf16 matrix product sustains here). The matrix cores are busy in 65,600 of 124,000 cycles (53 %), the LDS
// in 41,100; fragments are read only three ahead of the products, but which waits make up the rest is not known.
// One node over 32,768 rows 15 us + 3: HBM (67 MB, 4.4 TB/s). 24 nodes over 11,907 rows 14 + 4 (two tiles of 96
// rows, 64 splits; 20 together where the cache comes from HBM): three waves' work a workgroup, each stage's
// products and softmax one behind the other, and Q (48 KB a workgroup) and its partial outputs (48 KB) half as long
// as the six stages between them. One node over 300 rows 8.5 us with the join, 24 9.6, without cached rows 6.3:
// latency. 24 nodes over 24,000 rows: heads 16 / 4 of 64 14.2 us (25 MB of K and V, 4.9 us of a copy), heads 32 / 8
// of 128 27.7 (98 MB, 19.5). One workgroup a CU there too: that of heads of 64 takes 72 KB of LDS and 137 registers
// a lane, 9 more than two workgroups would have.
#include "attention_tile.h"
#include "draft.h"

namespace tu {

namespace {

constexpr int kThreads = 512;
constexpr int kUnit = kDraftUnit;
// P is formed against a reference that lies kLift below the largest score met (log2 units) and moves
// only when that has risen by more than kRise: P stays below 2^(kLift + kRise), within f16, a key
// 2^(kLift + 14) below the largest still has all of f16's bits, and what P loses below is at most
// 2^-(kLift + 25) of the largest. (Without kLift, many keys 17 e-folds below one whose value is small
// came out as zeros. 13 and 2 move the reference more often: 64 nodes over 65,536 rows 84.2 -> 86.2 us.)
// Near kHuge and beyond, where roundings of the score and the reference reach whole units, it moves at smaller
// rises, and is the largest score itself.
constexpr float kLift = 11.f, kRise = 4.f, kHuge = 0x1p22f;
static_assert(kLift + kRise < 15.5f, "P within f16, with the roundings below kHuge");
constexpr int kLgkmWait0 = 15 | (7 << 4) | (0 << 8) | (3 << 14);

typedef __attribute__((__vector_size__(4 * sizeof(short)))) short s16x4;
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
typedef __attribute__((address_space(3))) u32x4 lds_u32x4;
typedef __attribute__((__vector_size__(4 * sizeof(__bf16)))) __bf16 bf16x4;

template <int B>
struct IntC {
  static constexpr int value = B;
};

// 16 bytes per lane from the buffer at voff to LDS at lds + 16 lane. Written out, so that
// one loop body can serve every place of the rings: for the compiler's own load it would wait
// for all loads in flight before any LDS read whose address it cannot tell apart. It has no
// output register; the kernel waits for it by count, and for all of them before it ends.
// The whole offset is the vector one: the range check compares it with the resource's size
// itself, while a scalar offset larger than a short split's rows would leave the check to a
// difference that is negative.
__device__ __forceinline__ void dma_lds(uint32_t lds, uint32_t voff, u32x4 res) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds"
               :
               : "s"(lds), "v"(voff), "s"(res)
               : "memory", "m0");
}

constexpr int kWriteThrough = 17;   // sc0 sc1

// Raw buffer resource of `bytes` bytes: reads past them give zeros.
__device__ __forceinline__ u32x4 buffer_of(const void* base, uint32_t bytes) {
  const uint64_t b = (uint64_t)base;
  return u32x4{(uint32_t)__builtin_amdgcn_readfirstlane((uint32_t)b),
               (uint32_t)__builtin_amdgcn_readfirstlane((uint32_t)(b >> 32)),
               (uint32_t)__builtin_amdgcn_readfirstlane(bytes), (uint32_t)kBufWord3};
}

// x / d for 0 <= x < 2^21: the half keeps the product off every border (the reciprocal's and the product's
// errors, 1.5 * 2^-23 of it, move it by less than x 2^-22 / d < 1 / (2 d))
__device__ __forceinline__ int quotient(int x, int d) { return (int)(((float)x + 0.5f) * __builtin_amdgcn_rcpf((float)d)); }

// Barrier that does not wait for the loads in flight.
__device__ __forceinline__ void wg_barrier() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt(kLgkmWait0);
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

// Workgroups of a launch: a whole number per die (xcd_remap).
__host__ __device__ constexpr int whole_dies(int items) { return (items + kXcds - 1) / kXcds * kXcds; }

template <int D>
__global__ __launch_bounds__(kThreads) __attribute__((amdgpu_waves_per_eu(2, 2))) void k_draft_attn(
    const bf16_t* k_cache, const bf16_t* v_cache, const bf16_t* q_hat, int len, int n, int Hkv, int G, int n_splits,
    uint32_t tiles, int split_stages, int more_stages, DraftAttnArgs a) {   // up to `a`: in registers from the start
  constexpr int NS = D / 16;                 // 16-dim steps of S^T = K Q^T
  constexpr int NDB = D / 32;                // 32-dim blocks of O^T
  constexpr int RC = D / 8;                  // 16-byte chunks per row
  constexpr int KSWZ = RC < 16 ? RC - 1 : 15;
  auto vswz = [](int row) __attribute__((always_inline)) { return RC < 16 ? (row & 2) * 2 : (row & 3) * 4; };
  constexpr int SK = draft_stage_keys(D);    // keys of a stage
  constexpr int SUB = SK / kUnit;            // units of a stage
  constexpr int UB = SK * D * 2;             // bytes of a stage of K (or V)
  constexpr int NL = UB / 16 / kThreads;     // loads of a thread for one of them
  constexpr int PER = 2 * NL;                // loads of a thread for a stage
  static_assert(NL * 16 * kThreads == UB && SUB * kUnit == SK, "whole loads and units");
  __shared__ __attribute__((aligned(4 * UB))) char g_k[4 * UB];   // the rings (aligned: addresses in them are xored)
  __shared__ __attribute__((aligned(4 * UB))) char g_v[4 * UB];
  __shared__ uint64_t s_mask[kDraftRows][2];   // masks of the rows' nodes (workgroups that reach the tree)
  __shared__ int s_row[kDraftRows];            // output rows
  __shared__ unsigned long long s_spoilt[D][2];   // nodes whose value is not finite in f16, by dim
  __shared__ int s_spoils;

  const int n_tiles = tiles & 0xFFFFFF, tile_waves = tiles >> 24;
  const int items = Hkv * n_splits * n_tiles;
  const int item = xcd_remap(blockIdx.x, whole_dies(items));
  if (item >= items) return;
  // the row tiles of one key range are neighbours: they share a die's L2
  const int range = __builtin_amdgcn_readfirstlane(quotient(item, n_tiles));
  const int tile = __builtin_amdgcn_readfirstlane(item - range * n_tiles);
  const int hkv = __builtin_amdgcn_readfirstlane(quotient(range, n_splits));
  const int split = __builtin_amdgcn_readfirstlane(range - hkv * n_splits);
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int hl = lane >> 5, col = lane & 31;
  // stages u0 .. u1 - 1: equal shares, the first `more_stages` splits one more
  const int u0 = split * split_stages + min(split, more_stages);
  const int u1 = u0 + split_stages + (split < more_stages ? 1 : 0);
  const int rs = Hkv * D;   // elements of a cache row

  // ---- a stage: LDS chunk i * 512 + tid is loaded by load i of the thread. The resources start
  // at the split's first row and end with its last one that holds data: rows past it, and
  // stages past the split, are zeros. (A split's rows span less than 2^31 bytes.) The second
  // load's row lies a multiple of 16 rows on (of 8 with 8 chunks): the same chunk.
  constexpr int LR = kThreads / RC;
  static_assert(LR % (KSWZ + 1) == 0 && LR % 4 == 0, "the loads of a thread take the same chunk");
  const long start = (long)u0 * SK * rs + (long)hkv * D;
  const uint32_t bytes = (uint32_t)(min((u1 - u0) * SK, len + n - u0 * SK) * rs * 2 - (rs - D) * 2);
  const u32x4 kres = buffer_of(k_cache + start, bytes), vres = buffer_of(v_cache + start, bytes);
  uint32_t koff, voff;   // of the next stage to load
  {
    const int lrow = tid / RC, lc = tid % RC;
    koff = (uint32_t)(lrow * rs * 2 + (lc ^ (lrow & KSWZ)) * 16);
    voff = (uint32_t)(lrow * rs * 2 + (lc ^ vswz(lrow)) * 16);
  }
  const uint32_t stage_bytes = (uint32_t)(SK * rs * 2);
  const uint32_t lds_k = (uint32_t)(uintptr_t)(lds_void*)g_k + wave * 1024;
  const uint32_t lds_v = (uint32_t)(uintptr_t)(lds_void*)g_v + wave * 1024;
  auto load_k = [&](int place) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < NL; ++i) dma_lds(lds_k + place * UB + i * kThreads * 16, koff + i * LR * rs * 2, kres);
    koff += stage_bytes;
  };
  auto load_v = [&](int place) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < NL; ++i) dma_lds(lds_v + place * UB + i * kThreads * 16, voff + i * LR * rs * 2, vres);
    voff += stage_bytes;
  };

  // the first stages are asked for before anything else; Q is waited for with the first of them
  load_k(0);
  const int Hq = Hkv * G;
  const int rows_total = n * G;
  const int first = (tile * tile_waves + wave) * 32;   // of this wave's packed rows
  const bool busy = wave < tile_waves && first < rows_total;   // a wave without rows only loads
  // Q's rows are read a line at a time (four parts of a row, 64 / LPR rows a load) and go
  // through the wave's own LDS, in a ring place that is free until the first step, into the
  // operands: lane (query, half) holds 8 dims of each 16.
  constexpr int LPR = D / 32;          // 16-byte chunks of a quarter row
  constexpr int QL = LPR / 2;          // loads of a quarter
  bf16x8 qf[NS];
  u32x4 w[NS];
  uint64_t mask = 0;
  if (busy) {
    const int r = first + col;
    const int node = min(quotient(r, G), n - 1);
    const int row = r < rows_total ? node * Hq + hkv * G + (r - node * G) : -1;
    if (hl == 0) s_row[wave * 32 + col] = row;
    const bf16_t* from[QL];
#pragma unroll
    for (int i = 0; i < QL; ++i)
      from[i] = q_hat + (long)max(s_row[wave * 32 + lane / LPR + i * (64 / LPR)], 0) * D + (lane % LPR) * 8;
#pragma unroll
    for (int b = 0; b < 4; ++b)
#pragma unroll
      for (int i = 0; i < QL; ++i) w[b * QL + i] = *(const u32x4*)(from[i] + b * (D / 4));
    if (u1 * SK > len) mask = a.seen.m[node][hl];
  }
  if (u1 * SK > len) {
    for (int i = tid; i < 2 * D; i += kThreads) s_spoilt[i >> 1][i & 1] = 0;
    if (tid == 0) s_spoils = 0;
  }
  load_v(0);
  load_k(1);
  load_v(1);
  load_k(2);
  status_mark(a.status);
  if (busy) {
    if (u1 * SK > len) s_mask[wave * 32 + col][hl] = mask;
    char* const mine = (wave < 4 ? g_k : g_v) + 3 * UB + (wave & 3) * (UB / 4);
#pragma unroll
    for (int b = 0; b < 4; ++b) {
      asm volatile("" ::: "memory");
#pragma unroll
      for (int i = 0; i < QL; ++i) {
        const int rr = lane / LPR + i * (64 / LPR);
        *(u32x4*)(mine + (rr * LPR + ((lane % LPR) ^ (rr & (LPR - 1)))) * 16) = w[b * QL + i];
      }
      asm volatile("" ::: "memory");
#pragma unroll
      for (int i = 0; i < QL; ++i)
        qf[b * QL + i] = __builtin_bit_cast(
            bf16x8, *(const u32x4*)(mine + (col * LPR + ((2 * i + hl) ^ (col & (LPR - 1)))) * 16));
    }
  }

  f32x16 o[NDB];
#pragma unroll
  for (int db = 0; db < NDB; ++db)
#pragma unroll
    for (int e = 0; e < 16; ++e) o[db][e] = 0.f;
  float m_run = -__builtin_inff(), l_run = 0.f;
  const float c2 = a.scale_log2;
  float big = 0.f;   // largest |v| met

  // transposing reads of V (see pv below): block db of 32 dims lies at this address ^ 64 db (256
  // bytes on for each four blocks)
  uint32_t vaddr;
  {
    const int i = lane & 15, g = lane >> 4;
    const int row = 4 * (g >> 1) + (i >> 2);
    const int c0 = 2 * (g & 1) + ((i & 3) >> 1);
    vaddr = (uint32_t)(uintptr_t)(lds_void*)g_v + (uint32_t)(row * D * 2 + ((c0 ^ vswz(row)) * 16) + (i & 1) * 8);
  }
  // K row `col`, chunk hl ^ (col mod 16); chunk 2 s + hl is this address ^ 32 s
  const uint32_t kaddr = (uint32_t)(uintptr_t)(lds_void*)g_k + (uint32_t)(col * D * 2 + ((hl ^ (col & KSWZ)) * 16));

  // (what is derived from these is formed per unit: hoisted, it would cost registers)
  auto fresh = [](uint32_t x) __attribute__((always_inline)) -> uint32_t {
    asm volatile("" : "+v"(x));
    return x;
  };

  // ---- this thread's loads up to V of the stage in `place` and K of the next have landed (two
  // stages of loads are newer); its chunks of that V to f16, in place
  // A value of a node that is not finite must not reach nodes that do not see it (0 x NaN in a
  // product): it becomes 0, and the outputs that do see it are set to NaN at the end.
  auto to_f16 = [&](int place, int stage) __attribute__((always_inline)) {
    __builtin_amdgcn_s_waitcnt(vm_wait(2 * PER));
    asm volatile("" ::: "memory");
    u32x4* const at = (u32x4*)(g_v + place * UB + (fresh(tid) & (kThreads - 1)) * 16);
    u32x4 w[NL];
#pragma unroll
    for (int i = 0; i < NL; ++i) w[i] = at[i * kThreads];
#pragma unroll
    for (int i = 0; i < NL; ++i) {
      f16x8 x;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float lo = __uint_as_float(w[i][e] << 16), hi = __uint_as_float(w[i][e] & 0xFFFF0000u);
        big = fmaxf(fmaxf(fabsf(lo), fabsf(hi)), big);
        x[2 * e] = (_Float16)lo;
        x[2 * e + 1] = (_Float16)hi;
      }
      at[i * kThreads] = __builtin_bit_cast(u32x4, x);
      if ((stage + 1) * SK > len) {   // uniform
        const u32x4 bits = __builtin_bit_cast(u32x4, x);
        bool odd = false;   // an exponent of ones
#pragma unroll
        for (int e = 0; e < 4; ++e) odd |= (~bits[e] & 0x7C00u) == 0 | (~bits[e] & 0x7C000000u) == 0;
        const uint32_t t = fresh(tid);
        const int row = t / RC + i * LR, node = stage * SK + row - len;
        if (odd && node >= 0 && node < n) {
          const int dim = ((t % RC) ^ vswz(row)) * 8;
          uint16_t* const half = (uint16_t*)(at + i * kThreads);
#pragma unroll 1
          for (int e = 0; e < 8; ++e)
            if ((~half[e] & 0x7C00u) == 0) {
              half[e] = 0;
              atomicOr(&s_spoilt[dim + e][node >> 6], 1ull << (node & 63));
              s_spoils = 1;
            }
        }
      }
    }
    asm volatile("" : "+v"(big));   // here, not behind the next products with the values kept until then
  };

  f32x16 sacc[SUB];
  f16x8 pf[SUB][2];

  // ---- the matrix products: O^T += V^T P^T of the stage in one ring place, then S^T of the one in
  // another (in this order P is gone when the scores come). LDS reads run kAhead fragments ahead: an
  // MFMA takes 32 cycles, a read over 100; more would not fit the registers.
  constexpr int kMfma = 0x008, kDsRead = 0x100, kAhead = 3;
  auto sched_reads = [&](auto nc, auto per) __attribute__((always_inline)) {
    constexpr int N = decltype(nc)::value, READS = decltype(per)::value;
    constexpr int AHEAD = kAhead < N ? kAhead : N;
    __builtin_amdgcn_sched_group_barrier(kDsRead, READS * AHEAD, 0);
#pragma unroll
    for (int i = 0; i < N; ++i) {
      if (i + AHEAD < N) __builtin_amdgcn_sched_group_barrier(kDsRead, READS, 0);
      __builtin_amdgcn_sched_group_barrier(kMfma, 1, 0);
    }
  };
  auto pv = [&](int place) __attribute__((always_inline)) {
    const uint32_t vx = vaddr + place * UB;
    // lane group g reads keys 4 (g >> 1) + 0 .. 3 (+ 16 k16, + 8) at dims 32 db + 16 (g & 1) .. ;
    // the blocks that share an address follow one another
#pragma unroll
    for (int u = 0; u < SUB; ++u)
#pragma unroll
      for (int lo = 0; lo < (NDB < 4 ? NDB : 4); ++lo)
#pragma unroll
        for (int k16 = 0; k16 < 2; ++k16)
#pragma unroll
          for (int db = lo; db < NDB; db += 4) {
            const uint32_t at = (vx ^ (64 * lo)) + (db >> 2) * 256 + (kUnit * u + 16 * k16) * D * 2;
            const s16x4 x0 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(uintptr_t)at);
            const s16x4 x1 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(uintptr_t)(at + 8 * D * 2));
            const u32x2 w0 = __builtin_bit_cast(u32x2, x0), w1 = __builtin_bit_cast(u32x2, x1);
            const f16x8 va = __builtin_bit_cast(f16x8, u32x4{w0[0], w0[1], w1[0], w1[1]});
            o[db] = __builtin_amdgcn_mfma_f32_32x32x16_f16(va, pf[u][k16], o[db], 0, 0, 0);
          }
    sched_reads(IntC<2 * NDB * SUB>{}, IntC<2>{});
  };
  auto qk = [&](int place) __attribute__((always_inline)) {
    const uint32_t kx = kaddr + place * UB;
#pragma unroll
    for (int u = 0; u < SUB; ++u)
#pragma unroll
      for (int e = 0; e < 16; ++e) sacc[u][e] = 0.f;
#pragma unroll
    for (int i = 0; i < NS; ++i) {
      const int s = NS == 16 ? (i >> 1) + 8 * (i & 1) : i;   // steps that share an address follow one another
#pragma unroll
      for (int u = 0; u < SUB; ++u) {
        const bf16x8 ka = __builtin_bit_cast(
            bf16x8, *(const lds_u32x4*)(uintptr_t)((kx ^ (32 * s & 16 * KSWZ)) + (32 * s & ~(16 * KSWZ)) + kUnit * u * D * 2));
        sacc[u] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(ka, qf[s], sacc[u], 0, 0, 0);
      }
    }
    sched_reads(IntC<NS * SUB>{}, IntC<1>{});
  };

  // ---- softmax of a stage: the masks, the maximum, P in f16 in the key order of the operand
  auto softmax = [&](int stage) __attribute__((always_inline)) {
#pragma unroll
    for (int u = 0; u < SUB; ++u) {
      const int d = stage * SK + u * kUnit - len;
      if (d + kUnit - 1 >= 0) {   // the unit reaches the tree (uniform)
        // bit x of `keys`: this query sees key x of the unit
        uint32_t keys;
        const uint32_t t = fresh(tid), mr = (t & ~63u) / 2 + (t & 31u);
        const uint64_t m0 = s_mask[mr][0], m1 = s_mask[mr][1];
        if (d <= 0) keys = (uint32_t)(m0 << -d) | ((1u << -d) - 1u);
        else if (d < 64) keys = (uint32_t)(m0 >> d | m1 << (64 - d));
        else keys = d < 128 ? (uint32_t)(m1 >> (d - 64)) : 0u;
        keys >>= (t & 32u) >> 3;
#pragma unroll
        for (int e = 0; e < 16; ++e)
          if (!(keys >> (8 * (e >> 2) + (e & 3)) & 1)) sacc[u][e] = -__builtin_inff();
      }
    }
    float mx = -__builtin_inff();
#pragma unroll
    for (int u = 0; u < SUB; ++u)
#pragma unroll
      for (int e = 0; e < 16; ++e) mx = fmaxf(mx, sacc[u][e]);
    const auto sw = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(uint32_t, mx),
                                                     __builtin_bit_cast(uint32_t, mx), false, false);
    mx = fmaxf(__builtin_bit_cast(float, (uint32_t)sw[0]), __builtin_bit_cast(float, (uint32_t)sw[1])) * c2;
    if (__any(mx - m_run > __builtin_fmaf(fabsf(mx), -2.f / kHuge, kLift + kRise))) {
      const float m_new = fmaxf(m_run, fabsf(mx) < kHuge ? mx - kLift : mx);
      const float alpha = m_new == -__builtin_inff() ? 1.f : __builtin_amdgcn_exp2f(m_run - m_new);
      m_run = m_new;
      l_run *= alpha;
#pragma unroll
      for (int db = 0; db < NDB; ++db) scale_acc(o[db], alpha);
    }
    const float m_use = m_run == -__builtin_inff() ? 0.f : m_run;
    float ps[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int u = 0; u < SUB; ++u)
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        const float p = __builtin_amdgcn_exp2f(__builtin_fmaf(sacc[u][e], c2, -m_use));
        ps[e & 3] += p;
        pf[u][e >> 3][e & 7] = (_Float16)p;
      }
    l_run += (ps[0] + ps[1]) + (ps[2] + ps[3]);
  };

  // ---- half-steps, a barrier before each: in half-step 2 t waves 0 - 3 form the products of stage
  // t while waves 4 - 7 run the softmax of stage t - 1, in 2 t + 1 the other way round. K of
  // stage t - 1 and V of stage t - 2 are no longer read from 2 t on: their places take stages t + 3
  // and t + 2. V of stage t is turned to f16 in 2 t and 2 t + 1 and first read in 2 t + 2.
  const int n_stages = u1 - u0;
  constexpr int UNR = 2;
  auto refill = [&](int t) __attribute__((always_inline)) {
    load_k((t + 3) & 3);
    load_v((t + 2) & 3);
  };
  auto early = [&](int t) __attribute__((always_inline)) {   // waves 0 - 3
    wg_barrier();
    refill(t);
    if (busy) {
      if (t > 0) pv((t - 1) & 3);
      qk(t & 3);
    }
    wg_barrier();
    if (busy) softmax(u0 + t);
    to_f16(t & 3, u0 + t);
  };
  auto later = [&](int t) __attribute__((always_inline)) {   // waves 4 - 7
    wg_barrier();
    refill(t);
    if (busy && t > 0) softmax(u0 + t - 1);
    to_f16(t & 3, u0 + t);
    wg_barrier();
    if (busy) {
      if (t > 0) pv((t - 1) & 3);
      qk(t & 3);
    }
  };
  auto run = [&](auto step) __attribute__((always_inline)) {
    for (int t = 0; t < n_stages; t += UNR) {
#pragma unroll
      for (int i = 0; i < UNR; ++i)
        if (i == 0 || t + i < n_stages) step(t + i);
    }
  };
  __builtin_amdgcn_s_waitcnt(vm_wait(2 * PER));   // K of the first stage
  if (wave < 4) run(early);
  else run(later);
  __builtin_amdgcn_s_waitcnt(vm_wait(0));   // the loads past the split's end: no write into LDS may come later
  wg_barrier();
  if (busy) {
    if (wave >= 4) softmax(u1 - 1);
    pv((n_stages - 1) & 3);
  }
  if (big >= 65520.f) status_raise(a.status, kFaultRange);
  wg_barrier();   // the rings are written over below
  if (!busy) return;
  const uint32_t te = fresh(tid);
  const int lane_e = te & 63, col_e = te & 31, hl_e = (te >> 5) & 1;

  const auto lsw = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(uint32_t, l_run),
                                                    __builtin_bit_cast(uint32_t, l_run), false, false);
  const float l_tot = __builtin_bit_cast(float, (uint32_t)lsw[0]) + __builtin_bit_cast(float, (uint32_t)lsw[1]);
  const bool whole = n_splits == 1;
  // 0: no key of this split is seen. A query sees its own key: over all keys a sum of 0 (scores of -infinity
  // alone) is NaN, as where splits are joined
  const float inv = l_tot == 0.f && !whole ? 0.f : 1.f / l_tot;
  const int row = s_row[wave * 32 + col_e];
  if (u1 * SK > len && s_spoils) {
    const uint64_t m0 = s_mask[wave * 32 + col_e][0], m1 = s_mask[wave * 32 + col_e][1];
#pragma unroll
    for (int c = 0; c < 4 * NDB; ++c) {
      asm volatile("" ::: "memory");   // one chunk's masks at a time
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int dim = 8 * c + 4 * hl_e + e;
        if ((s_spoilt[dim][0] & m0) | (s_spoilt[dim][1] & m1)) o[c >> 2][4 * (c & 3) + e] = __builtin_nanf("");
      }
    }
  }
  auto chunk = [&](int c) __attribute__((always_inline)) -> f32x4 {   // dims 8 c + 4 hl .. + 3
    const int db = c >> 2, i = c & 3;
    return f32x4{o[db][4 * i], o[db][4 * i + 1], o[db][4 * i + 2], o[db][4 * i + 3]} * inv;
  };
  if (!whole) {
    // A partial output as the lanes hold it, written through: the caches of the dies would
    // otherwise be written back when the kernel ends, with nothing else to do (24 nodes over 11,907
    // rows, 25 MB of partial outputs: 22.0 -> 21.1 us with the join; 64 over 65,536: 83.8 -> 82.8).
    if (row < 0) return;
    const int packed = tile * tile_waves + wave;
    const long at = (long)(split * Hkv + hkv) * a.n_waves + packed;
    const __amdgpu_buffer_rsrc_t res = __builtin_amdgcn_make_buffer_rsrc(a.part_o + at * 32 * D, 0, 64 * D, kBufWord3);
#pragma unroll
    for (int p = 0; p < 2 * NDB; ++p) {
      const f16x4 x = __builtin_convertvector(chunk(2 * p), f16x4), y = __builtin_convertvector(chunk(2 * p + 1), f16x4);
      const u32x4 xy = __builtin_bit_cast(u32x4, __builtin_shufflevector(x, y, 0, 1, 2, 3, 4, 5, 6, 7));
      __builtin_amdgcn_raw_buffer_store_b128(xy, res, lane_e * 16 + p * 1024, 0, kWriteThrough);
    }
    if (hl_e == 0) {
      float* ml = a.part_ml + ((long)((hkv * a.n_waves + packed) * 32 + col_e) * n_splits + split) * 2;
      ml[0] = l_tot == 0.f ? -__builtin_inff() : m_run == -__builtin_inff() ? 0.f : m_run;
      ml[1] = l_tot;
    }
    return;
  }
  // the wave's 32 rows through its own place of the rings, then 16 bytes a lane in whole rows
  const uint32_t mine = (uint32_t)(uintptr_t)(lds_void*)(wave < 4 ? g_k : g_v) + (wave & 3) * UB;
  const uint32_t wr = mine + col_e * D * 2 + hl_e * 8 + (col_e & KSWZ) * 16;
#pragma unroll
  for (int c = 0; c < 4 * NDB; ++c)
    *(__attribute__((address_space(3))) bf16x4*)(uintptr_t)((wr ^ (16 * c & 16 * KSWZ)) + (16 * c & ~(16 * KSWZ))) =
        __builtin_convertvector(chunk(c), bf16x4);
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt(kLgkmWait0);
  // rows past the last (s_row is -1) lie past the resource: their stores are dropped
  const __amdgpu_buffer_rsrc_t out_res = __builtin_amdgcn_make_buffer_rsrc(a.out, 0, n * Hq * D * 2, kBufWord3);
#pragma unroll
  for (int i = 0; i < kUnit * RC / 64; ++i) {
    const int q = i * 64 + lane_e, rr = q / RC, c = q % RC;
    const u32x4 x = *(const lds_u32x4*)(uintptr_t)(mine + rr * D * 2 + ((c ^ (rr & KSWZ)) * 16));
    __builtin_amdgcn_raw_buffer_store_b128(x, out_res, s_row[wave * 32 + rr] * (D * 2) + c * 16, 0, 0);
  }
}

// Joins the splits. The partial outputs lie as the lanes of k_draft_attn held them: for each split,
// KV head and 32 packed rows D / 16 pieces of 1 KB, 16 bytes a lane (half, row): dims 16 p + 4 half + e, and 8
// further on. A workgroup takes 8 rows of one piece: 16 lanes, whose 16 groups take the splits
// in turn and are added up through LDS in a fixed order. Every lane requests all of its splits
// at once, before the weights are known: one trip to memory.
constexpr int kMergeThreads = 256;
constexpr int kMergeRows = 8;
constexpr int kMergeGroups = kMergeThreads / 16;
constexpr int kMergeEach = kMaxDraftSplits / kMergeGroups;   // splits of a lane group
static_assert(kMergeThreads / 32 == kMergeRows && kMaxDraftSplits == 4 * 32, "32 lanes form a row's weights");

// `op` over 32 lanes, the same bits in each of them
template <class Op>
__device__ __forceinline__ float over_32(float x, Op op) {
  const auto moved = [&](auto ctrl) __attribute__((always_inline)) {
    return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), decltype(ctrl)::value, 0xf, 0xf, true));
  };
  x = op(x, moved(IntC<0xB1>{}));    // quad_perm 1,0,3,2
  x = op(x, moved(IntC<0x4E>{}));    // quad_perm 2,3,0,1
  x = op(x, moved(IntC<0x141>{}));   // row_half_mirror
  x = op(x, moved(IntC<0x140>{}));   // row_mirror
  return op(x, __shfl_xor(x, 16, 64));
}

template <int D>
__global__ __launch_bounds__(kMergeThreads) void k_draft_merge(const _Float16* part_o, const float* part_ml, bf16_t* to,
                                                               int n, int G, int Hkv, int ns, int n_waves) {
  constexpr int PIECES = D / 16;
  __shared__ float s_w[kMergeRows][kMaxDraftSplits + 1], s_l[kMergeRows];
  __shared__ __attribute__((aligned(16))) float s_o[kMergeGroups][kMergeRows][20];
  const int rows = n * G;
  const int piece = blockIdx.x / 4 % PIECES, part = blockIdx.x / (4 * PIECES);   // the four parts of a piece are neighbours
  const int hkv = part / n_waves, r0 = (part - hkv * n_waves) * 32 + blockIdx.x % 4 * kMergeRows;
  if (r0 >= rows) return;
  const int tid = threadIdx.x, g = tid >> 4, col = tid & 7, hl = tid >> 3 & 1;

  typedef __attribute__((__vector_size__(2 * sizeof(float)))) float f32x2;
  const int wr = tid >> 5, wl = tid & 31;   // forms weights of row r0 + wr
  f32x2 x[4];
  const f32x2* ml = (const f32x2*)part_ml + ((long)hkv * n_waves * 32 + r0 + wr) * ns;
#pragma unroll
  for (int i = 0; i < 4; ++i)
    x[i] = r0 + wr < rows && wl + 32 * i < ns ? ml[wl + 32 * i] : f32x2{-__builtin_inff(), 0.f};
  const _Float16* po = part_o + ((long)hkv * n_waves + r0 / 32) * 32 * D + piece * 512 + (hl * 32 + r0 % 32 + col) * 8;
  const long each = (long)Hkv * n_waves * 32 * D;   // of a split
  f16x8 v[kMergeEach];
#pragma unroll
  for (int i = 0; i < kMergeEach; ++i) {
    const int s = g + kMergeGroups * i;
    v[i] = s < ns && r0 + col < rows ? *(const f16x8*)(po + s * each) : f16x8{};
  }
  float M = fmaxf(fmaxf(x[0][0], x[1][0]), fmaxf(x[2][0], x[3][0]));
  M = over_32(M, [](float a, float b) { return fmaxf(a, b); });
  float L = 0.f;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float w = x[i][0] == -__builtin_inff() ? 0.f : x[i][1] * __builtin_amdgcn_exp2f(x[i][0] - M);
    s_w[wr][wl + 32 * i] = w;   // 0 past the last split
    L += w;
  }
  L = over_32(L, [](float a, float b) { return a + b; });
  if (wl == 0) s_l[wr] = L;
  __syncthreads();
  float acc[8] = {};
#pragma unroll
  for (int i = 0; i < kMergeEach; ++i) {
    const float ws = s_w[col][g + kMergeGroups * i];
#pragma unroll
    for (int e = 0; e < 8; ++e) acc[e] = __builtin_fmaf(ws, (float)v[i][e], acc[e]);
  }
  *(f32x4*)&s_o[g][col][4 * hl] = f32x4{acc[0], acc[1], acc[2], acc[3]};
  *(f32x4*)&s_o[g][col][4 * hl + 8] = f32x4{acc[4], acc[5], acc[6], acc[7]};
  __syncthreads();
  const int out = tid >> 4, r = r0 + out, d = tid & 15;   // row, dim of the piece
  if (out >= kMergeRows || r >= rows) return;
  float sum = 0.f;
#pragma unroll
  for (int i = 0; i < kMergeGroups; ++i) sum += s_o[i][out][d];
  const int node = r / G;
  ((__bf16*)to)[((long)(node * Hkv + hkv) * G + (r - node * G)) * D + 16 * piece + d] = (__bf16)(sum / s_l[out]);
}

}  // namespace

hipError_t launch_draft_attention(const DraftAttnArgs& a, int head_dim, hipStream_t s) {
  const int items = a.n_kv_heads * a.n_splits * a.n_tiles;
  if (items <= 0) return hipSuccess;
  const auto run = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, dim3(whole_dies(items)), dim3(kThreads), 0, s, a.k_cache, a.v_cache, a.q_hat, a.len, a.n,
                       a.n_kv_heads, a.group, a.n_splits, (uint32_t)a.n_tiles | (uint32_t)a.tile_waves << 24,
                       a.split_stages, a.more_stages, a);
    return hipGetLastError();
  };
  switch (head_dim) {
    case 256: return run(k_draft_attn<256>);
    case 128: return run(k_draft_attn<128>);
    case 64: return run(k_draft_attn<64>);
    default: return hipErrorInvalidValue;
  }
}

hipError_t launch_draft_merge(const DraftAttnArgs& a, int head_dim, hipStream_t s) {
  const int parts = a.n_kv_heads * a.n_waves * 4;
  if (parts <= 0) return hipSuccess;
  const auto run = [&](auto kernel, int pieces) {
    hipLaunchKernelGGL(kernel, dim3(parts * pieces), dim3(kMergeThreads), 0, s, a.part_o, a.part_ml, a.out, a.n, a.group,
                       a.n_kv_heads, a.n_splits, a.n_waves);
    return hipGetLastError();
  };
  switch (head_dim) {
    case 256: return run(k_draft_merge<256>, 16);
    case 128: return run(k_draft_merge<128>, 8);
    case 64: return run(k_draft_merge<64>, 4);
    default: return hipErrorInvalidValue;
  }
}

}  // namespace tu
