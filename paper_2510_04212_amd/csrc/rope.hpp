// What the entry point of the rotary positions (api_cache.hip) hands to their kernel (rope.hip).
#pragma once
#include <hip/hip_runtime.h>

// Queries or keys: element (b, h, n, k) at b*_b + h*_h + n*_n + k.  uint16_t: bf16 bits.
struct RopeSide {
  const unsigned short* in;
  unsigned short* out;
  long long in_b, in_h, in_n, out_b, out_h, out_n;
};
struct RopeArgs {
  RopeSide q, k;
  const int* positions;            // [B][N] with rows positions_stride apart; NULL: 0 .. N-1
  long long positions_stride;
  const double* frequencies;       // [rot/2], radians per position
  int B, H, H_kv, N, d, rot;
  int heads_per_block;             // set by the dispatch
  float magnitude;
  int inverse;
};
hipError_t attn_rope_dispatch(const RopeArgs&, int interleaved, hipStream_t);
