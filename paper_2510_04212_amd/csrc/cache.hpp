// The cache of keys and values in 8 bits (include/attn.h describes it): what its kernels share, and what the entry
// points (api_cache.hip) hand to them (cache.hip, cache_attn.hip, cache_shared.hip, cache_copy.hip).
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>
#include "cache_shares.hpp"

constexpr int kLowestExponent = -100;      // of a scale 2^e: dequantised values stay normal bf16 numbers (2^-9 2^-100 at least)
constexpr int kHighestExponent = 119;      // and finite: 448 * 2^119 = 1.75 * 2^127

struct CacheArgs {
  unsigned char* K;                        // [B][H_kv][capacity][d]
  unsigned char* V;                        // [B][H_kv][capacity / 64][d][64]
  float* K_scale;                          // [B][H_kv][capacity / 64]
  float* V_scale;
  int capacity;
};

// rows of a bf16 tensor: element (b, h, n, k) at b*sb + h*sh + n*sn + k
struct Rows {
  const unsigned short* at;
  long long sb, sh, sn;
};

struct AppendArgs {
  CacheArgs cache;
  Rows K, V;
  const int *lengths, *counts;
  int B, H_kv, N;
};
hipError_t attn_cache_append_dispatch(const AppendArgs&, int d, hipStream_t);

struct AttendArgs {
  CacheArgs cache;
  Rows Q;
  unsigned short* O;
  long long o_sb, o_sh, o_sn;
  float* LSE;                              // [B][H][N]
  const int *lengths, *counts;
  int B, H, H_kv, N, group, causal;
  float scale;
  float* partials;                         // workspace
};
size_t attn_cache_fwd_partial_bytes(int B, int H, int H_kv, int N, int d, int capacity);
hipError_t attn_cache_fwd_dispatch(const AttendArgs&, int d, hipStream_t);

// Sequences that continue prefixes: `own` is about the sequences and their own caches, P * S of them; sequence b continues prefix b / S.
struct SharedArgs {
  AttendArgs own;
  CacheArgs prefix;                        // of P sequences
  const int* prefix_lengths;
  int P, S;
};
size_t attn_cache_fwd_shared_partial_bytes(int P, int S, int H, int H_kv, int N, int d, int prefix_capacity, int capacity);
hipError_t attn_cache_fwd_shared_dispatch(const SharedArgs&, int d, hipStream_t);

struct WeighArgs {
  CacheArgs cache;
  Rows Q;
  const float* LSE;
  const float* in;                         // [B][H_kv][capacity] or NULL
  float* out;
  const int *lengths, *counts;
  int B, H, H_kv, N, group, causal;
  float scale;
};
hipError_t attn_cache_weights_dispatch(const WeighArgs&, int d, hipStream_t);

struct EvictArgs {
  CacheArgs from, to;
  const float* weights;                    // [B][H_kv][from.capacity]
  float* weights_out;                      // [B][H_kv][to.capacity] or NULL
  int* kept;                               // [B][H_kv][budget]
  const int* lengths;
  int B, H_kv, budget, recent;
};
hipError_t attn_cache_evict_dispatch(const EvictArgs&, int d, hipStream_t);

struct ForkArgs {
  CacheArgs from, to;
  const int *sources, *lengths;            // [B_out]; [B_in]
  int* lengths_out;                        // [B_out]
  int B_in, B_out, H_kv, d;
};
hipError_t attn_cache_fork_dispatch(const ForkArgs&, hipStream_t);

struct ReorderArgs {
  CacheArgs cache;
  const int *parents, *lengths;            // [P][S] each
  int* lengths_out;
  int P, S, H_kv, d;
};
constexpr int kMostReordered = 64;         // sequences of a group
hipError_t attn_cache_reorder_dispatch(const ReorderArgs&, hipStream_t);

#ifdef __HIPCC__
#include "common.hpp"

// Tokens of sequence b that are in the cache, and how many of its queries / new tokens are real.  Whatever the device
// arrays hold, nothing outside the tensors is touched: counts are taken into [0, N], lengths into [0, capacity] where
// they bound a read.
DEVI int real_count(const int* counts, int b, int N) { return counts ? min(max(counts[b], 0), N) : N; }

// Scans over a wave in lane order by row shifts (1, 2, 4, 8 lanes within 16) and row broadcasts: vector instructions, no LDS exchange.  join(0, x) = x.
template <class F> DEVI unsigned scan_wave(unsigned x, F&& join) {
  x = join(__builtin_amdgcn_update_dpp(0, (int)x, 0x111, 0xf, 0xf, false), x);
  x = join(__builtin_amdgcn_update_dpp(0, (int)x, 0x112, 0xf, 0xf, false), x);
  x = join(__builtin_amdgcn_update_dpp(0, (int)x, 0x114, 0xf, 0xf, false), x);
  x = join(__builtin_amdgcn_update_dpp(0, (int)x, 0x118, 0xf, 0xf, false), x);
  x = join(__builtin_amdgcn_update_dpp(0, (int)x, 0x142, 0xa, 0xf, false), x);      // the last lane of row 0 to row 1, of 2 to 3
  x = join(__builtin_amdgcn_update_dpp(0, (int)x, 0x143, 0xc, 0xf, false), x);      // lane 31 to rows 2 and 3
  return x;
}
DEVI unsigned sum_to_lane(unsigned x) { return scan_wave(x, [](unsigned a, unsigned b) { return a + b; }); }
DEVI unsigned max_over_wave(unsigned x) {       // the same in all lanes
  return (unsigned)__builtin_amdgcn_readlane((int)scan_wave(x, [](unsigned a, unsigned b) { return max(a, b); }), 63);
}

// 2^e as float32, e >= -126, and the exponent of a scale
DEVI float power(int e) { return __uint_as_float((unsigned)(e + 127) << 23); }
DEVI int exponent(float scale) { return (int)((__float_as_uint(scale) >> 23) & 255) - 127; }
// the least e with amax <= 448 * 2^e (448 = 1.75 * 2^8), within the limits above
DEVI int exponent_for(float amax) {
  const unsigned u = __float_as_uint(amax);
  const int e = (int)(u >> 23) - 127 - 8 + ((u & 0x7fffffu) > 0x600000u ? 1 : 0);
  return min(max(e, kLowestExponent), kHighestExponent);
}
// Four values to E4M3: nearest, ties to even (v_cvt_pk_fp8_f32), beyond 448 to 448, NaN to NaN.
DEVI float saturate_e4m3(float x) { return x != x ? x : __builtin_amdgcn_fmed3f(x, -448.f, 448.f); }
DEVI unsigned pack4_e4m3(float a, float b, float c, float d) {
  int w = __builtin_amdgcn_cvt_pk_fp8_f32(saturate_e4m3(a), saturate_e4m3(b), 0, false);
  w = __builtin_amdgcn_cvt_pk_fp8_f32(saturate_e4m3(c), saturate_e4m3(d), w, true);
  return (unsigned)w;
}
// four codes to the values they stand for under a scale `times` larger: exact but for results below 2^-6
DEVI unsigned rescale4_e4m3(unsigned w, float times) {
  return pack4_e4m3(__builtin_amdgcn_cvt_f32_fp8((int)w, 0) * times, __builtin_amdgcn_cvt_f32_fp8((int)w, 1) * times,
                    __builtin_amdgcn_cvt_f32_fp8((int)w, 2) * times, __builtin_amdgcn_cvt_f32_fp8((int)w, 3) * times);
}
#endif
