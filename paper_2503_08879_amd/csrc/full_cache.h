// Kernel parameters of the operators on the full cache (rotary.hip, cache_attn.hip) and their launches.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace sagekv {

// Heads of packed tokens: head h of token t begins at base + t * token + h * head (bytes).
struct TokenRows {
  char* base;
  int64_t token, head;
};

// A dense or paged cache: head c of token t of problem p begins at block * s_block + c * s_head + (t & (2^shift - 1)) * s_token (bytes), the block
// the problem itself (table null, shift 31) or table[p * pitch + (t >> shift)].
struct FullCache {
  char *K, *V;
  int64_t ks_block, ks_head, vs_block, vs_head;
  int ks_token, vs_token;  // less than 2^24
  const int32_t* table;
  int64_t pitch;
  int shift, n_blocks;
};

struct RotaryParams {
  TokenRows q, q_out, k, v;  // rotary alone: q only
  FullCache cache;           // Hkv > 0
  int64_t n_tokens, capacity;
  int Hq, Hkv, D, dtype, P;
  int r, pairs_layout;  // r = 0: no rotation
  float amplitude, sign;
  const double* freq;
  const int32_t *offsets, *lens, *positions;
};
hipError_t launch_rotary(const RotaryParams& p, hipStream_t s);

constexpr int kAttnGroups = 256;   // workgroups of an attention launch at most: one per CU,
constexpr int kAttnWaves = 1024;   // of four waves
constexpr int kRowWeight = 2;      // a row's beginning and end, in blocks
constexpr int kWholeRounds = 3;    // see Walk::start in cache_attn.hip

// Whole rows: how many waves each gets, and how many blocks the longest row's waves then take one after the other, at most.
struct RowCuts {
  int cuts, rows_each;
  __host__ __device__ explicit RowCuts(int64_t rows)
      : cuts(4 * rows <= kAttnWaves ? 4 : 2 * rows <= kAttnWaves ? 2 : 1), rows_each((int)((rows * cuts + kAttnWaves - 1) / kAttnWaves)) {}
  __host__ __device__ int64_t rounds(int64_t blocks) const { return (blocks + cuts - 1) / cuts * rows_each; }
};

// A row whose parts are to be joined, those of workgroups first (its second slot) and first + 1 .. last (their first slots).
struct JoinRecord {
  int row, first, last;  // first < 0: nothing to do
};

// Tokens of a block.
constexpr int attn_block(int dtype, int head_dim) { return dtype == 1 ? (head_dim == 128 ? 16 : 32) : (head_dim == 128 ? 32 : 64); }

struct CacheAttnParams {
  FullCache cache;
  const char* q;
  float *out, *lse;
  const int32_t* lens;
  int P, Hq, Hkv, G, D, dtype;
  int S, W, max_len;
  bool by_row;  // a join record per row, else one per workgroup
  int n_waves;
  int heads;     // of a group, a workgroup's at most
  float scale;       // 1 / sqrt(head_dim)
  float join_scale;  // the parts' maxima times this are logits: scale where they are products (bf16), 1 where they are logits (fp32)
  float* part_acc;    // [kAttnGroups][2][G][D]
  float2* part_ml;    // [kAttnGroups][2][G]
  JoinRecord* joins;  // [kAttnGroups]
};
hipError_t launch_cache_attn(const CacheAttnParams& p, bool join, hipStream_t s);

}  // namespace sagekv
