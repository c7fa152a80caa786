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
  int64_t ks_block, ks_head, ks_token, vs_block, vs_head, vs_token;
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

}  // namespace sagekv
