// Launch records of the speculative decoding kernels (a tree of drafted tokens over one
// context). Every kernel takes its record by value.
#pragma once

#include "common.h"

namespace tu {

constexpr int kMaxDraft = 128;   // TU_MAX_DRAFT

// Bit j of the mask of node i: node i sees node j (an ancestor, or i itself).
struct DraftMasks {
  uint64_t m[kMaxDraft][2];
};

constexpr int kNormTokens = 4;   // tokens of a norm workgroup, at most
struct NormArgs {
  const bf16_t* in[3];    // q, k, v (v is copied; draft_append only)
  bf16_t* out[3];
  int64_t in_stride[3];   // elements from one token to the next
  int64_t out_stride[3];
  const bf16_t* weight[2];  // of q, of k, or null
  const int32_t* pos;     // positions, or null: first_pos + t, or first_pos + depth[t]
  int64_t first_pos;
  double turn_lane[16];   // theta^(-16 l / r) / (2 pi): turns per position of pair 8 l
  double turn_elem[8];    // theta^(-2 e / r)
  int32_t heads_end[3];   // prefix of the head counts of q, k, v
  int32_t T;
  int32_t kind;           // TU_NORM_*
  int32_t rotary;
  float eps;
  float weight_offset;
  int32_t tokens;         // of a workgroup
  int32_t head_parts;     // workgroups that share the heads of a token
  int32_t part_heads;     // heads of each of them
  int32_t use_depth;
  uint8_t depth[kMaxDraft];
};

struct DraftAttnArgs {
  const bf16_t* q_hat;    // [n][Hq][D]
  const bf16_t* k_cache;  // [>= len + n][Hkv][D]
  const bf16_t* v_cache;
  bf16_t* out;            // [n][Hq][D]
  // unused when n_splits == 1:
  _Float16* part_o;       // [splits][Hkv][n_waves][D / 16][64][8] normalised partial outputs, as the lanes hold them
  float* part_ml;         // [Hkv][n_waves * 32][splits][2] reference max (log2 units), sum
  CallStatus status;
  int32_t len;
  int32_t n;
  int32_t n_q_heads;
  int32_t n_kv_heads;
  int32_t n_tiles;        // row tiles of a KV head
  int32_t tile_waves;     // waves of a tile that have rows, 32 each
  int32_t n_splits;
  int32_t group;          // query heads per KV head
  int32_t split_stages;   // stages of a split; the first more_stages splits have one more
  int32_t more_stages;
  float scale_log2;       // softmax_scale * log2(e)
  int32_t n_waves;        // ceil(n * G / 32): waves with rows
  DraftMasks seen;
};
constexpr int kMaxDraftSplits = 128;
constexpr int kDraftRows = 256;         // packed query rows of an attention workgroup, at most
constexpr int kDraftUnit = 32;          // keys of a unit of the products
// Keys of a stage: 16 KB of K, 16 KB of V; half of that with head_dim 64, where longer stages leave
// short contexts too few of them.
constexpr int draft_stage_keys(int head_dim) { return head_dim == 256 ? 32 : 64; }

struct DraftConvArgs {
  ConvJob job[kMaxConvJobs];   // state is only read
  int32_t n_jobs;
  int32_t n;                   // nodes
  int32_t width;
  int32_t pad;
  int8_t up[kMaxDraft][8];     // row under the t-th tap back from node i: a node, or -1, -2, .. for the carried rows, newest first
};

struct DraftDeltaArgs {
  const float* state;   // [Hv][d][d]
  const bf16_t* q;      // [n][Hk][d]
  const bf16_t* k;
  const bf16_t* v;      // [n][Hv][d]
  const float* beta;    // [n][Hv]
  const float* g;
  float* out;           // [n][Hv][d]
  int32_t n;
  int32_t n_k_heads;
  int32_t n_v_heads;
  float scale;
  DraftMasks seen;
};

constexpr int kDrawThreads = 512;
constexpr int kDrawPer = 8;       // consecutive row elements of a thread, in registers
constexpr int kDrawMaxBlocks = 64;
constexpr int kDrawPolls = 1 << 20;   // of a wait for the other workgroups, each a trip to memory
struct DraftVerifyArgs {
  const int32_t* tokens;
  const float* target;
  const float* proposal;    // or null
  const float* u;
  int32_t* result;
  int64_t target_stride;
  int64_t proposal_stride;
  int64_t vocab;
  unsigned long long* part; // [n + 1][n_blocks] sums of the passes (bits of a double)
  CallStatus status;
  int32_t n;
  int32_t n_blocks;         // workgroups of a pass, each a contiguous slice of the row
  int64_t slice;            // elements of a slice, a multiple of kDrawThreads * kDrawPer
  int32_t wide;             // every row is 16-byte aligned
  int32_t polls;            // of a bounded wait, behind the first
  uint64_t first[2];        // nodes that are their parent's first child
  uint8_t parent[kMaxDraft];
  uint8_t child[kMaxDraft];    // first child (0: none)
  uint8_t sibling[kMaxDraft];  // next child of the same parent (0: none)
  DraftMasks seen;
};

constexpr int kMaxAcceptDelta = 48;
constexpr int kMaxAcceptConv = 48;
constexpr int kMaxAcceptBufs = 64;
struct AcceptDelta {
  float* state;
  const bf16_t* k;
  const bf16_t* v;
  const float* beta;
  const float* g;
};
struct AcceptConv {
  bf16_t* state;
  const bf16_t* x;
  int32_t channels;
  int32_t block_begin;
};
struct AcceptArgs {
  AcceptDelta delta[kMaxAcceptDelta];
  AcceptConv conv[kMaxAcceptConv];
  bf16_t* bufs[kMaxAcceptBufs];   // K and V caches
  int32_t* pos;                   // d_pos, or null
  int64_t len;
  int64_t next_pos;
  int32_t n_delta;
  int32_t n_conv;
  int32_t n_bufs;
  int32_t row_chunks;             // 16-byte chunks of a cache row
  int32_t n_k_heads;
  int32_t n_v_heads;
  int32_t d;
  int32_t width;
  int32_t n_path;
  int32_t delta_blocks;           // workgroups of the three parts
  int32_t conv_blocks;
  int32_t row_blocks;             // per buffer
  uint8_t path[kMaxDraft];
};

hipError_t launch_qk_norm(const NormArgs& a, int head_dim, hipStream_t s);
hipError_t launch_draft_attention(const DraftAttnArgs& a, int head_dim, hipStream_t s);
hipError_t launch_draft_merge(const DraftAttnArgs& a, int head_dim, hipStream_t s);
hipError_t launch_draft_conv(DraftConvArgs& a, hipStream_t s);   // sets each job's block_begin, n_cblocks
hipError_t launch_draft_delta(const DraftDeltaArgs& a, int d, hipStream_t s);
hipError_t launch_draft_clear(const DraftVerifyArgs& a, hipStream_t s);
hipError_t launch_draft_draw(const DraftVerifyArgs& a, hipStream_t s);
hipError_t launch_draft_accept(AcceptArgs& a, hipStream_t s);    // sets the block counts

static_assert(sizeof(NormArgs) <= kMaxKernargBytes && sizeof(DraftAttnArgs) <= kMaxKernargBytes &&
                  sizeof(DraftConvArgs) <= kMaxKernargBytes && sizeof(DraftDeltaArgs) <= kMaxKernargBytes &&
                  sizeof(DraftVerifyArgs) <= kMaxKernargBytes && sizeof(AcceptArgs) <= kMaxKernargBytes,
              "draft launch records");

}  // namespace tu
