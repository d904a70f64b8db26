// What the entry point of the choice among beams (api_cache.hip) hands to its kernels (beam.hip).
#pragma once
#include <hip/hip_runtime.h>

constexpr int kMostBeams = 64, kMostChosen = 128;

struct BeamArgs {
  const void* logits;                      // token t of beam k of item b at b * stride_b + k * stride_beam + t
  long long stride_b, stride_beam;
  int wide;                                // float32; otherwise bf16
  const float* scores;                     // [B][beams]
  const unsigned char* finished;           // the same, or NULL
  int end_token;
  int *parents, *tokens;                   // [B][n]
  float* scores_out;
  unsigned char* finished_out;             // or NULL
  int B, beams, V, n;
  void* workspace;
};
size_t attn_beam_select_partial_bytes(int B, int beams, int V, int n);
hipError_t attn_beam_select_dispatch(const BeamArgs&, hipStream_t);
