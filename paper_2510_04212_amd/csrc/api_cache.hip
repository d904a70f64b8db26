// C ABI of the rotary positions and of the 8-bit cache (see include/attn.h): argument validation and dispatch only.
#include <hip/hip_runtime.h>
#include <stdint.h>
#include <algorithm>
#include <cmath>
#include "../../include/attn.h"
#include "cache.hpp"
#include "rope.hpp"

static_assert(kBlock == ATTN_CACHE_BLOCK, "tokens of a scale");

namespace {

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
bool aligned4(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }
// The dispatches return hipErrorInvalidConfiguration, before anything is launched, where a grid would be too large.
int launched(hipError_t e) { return e == hipSuccess ? ATTN_OK : e == hipErrorInvalidConfiguration ? ATTN_ERR_UNSUPPORTED : ATTN_ERR_LAUNCH; }

// Sizes of bf16 rows [B,H,N,d].  *empty for B * H == 0.
int check_rows(int B, int H, int N, int d, bool* empty) {
  *empty = false;
  if (B < 0 || H < 0 || N < 0 || d < 0) return ATTN_ERR_BAD_ARG;
  if (B == 0 || H == 0) { *empty = true; return ATTN_OK; }
  if (d != 32 && d != 64 && d != 96 && d != 128 && d != 256) return ATTN_ERR_UNSUPPORTED;
  if (N == 0) return ATTN_ERR_UNSUPPORTED;
  if ((double)B * H * (double)N * d >= 1099511627776.0) return ATTN_ERR_UNSUPPORTED;      // 2^40
  return ATTN_OK;
}
// Grid limits: sequences and heads are the grid's second and third dimension (65535 each), and rows of a sequence and of the batch are counted in int.
int check_cache(int B, int H_kv, int d, int capacity) {
  if (capacity <= 0 || capacity % kBlock != 0) return ATTN_ERR_BAD_ARG;
  if (capacity > (1 << 30) || B > 65535 || H_kv > 65535) return ATTN_ERR_UNSUPPORTED;
  if ((double)B * H_kv * (double)capacity * d >= 1099511627776.0) return ATTN_ERR_UNSUPPORTED;
  return ATTN_OK;
}
bool scale_ok(float s) { return s > 0.f && std::isfinite(s); }

// three strides of a tensor; least: 0 for inputs, 1 for outputs
bool strides_ok(const long long* s, long long least) {
  for (int i = 0; i < 3; ++i)
    if (s[i] < least || s[i] % 8 != 0 || s[i] >= (1ll << 40)) return false;
  return true;
}
struct Strides { long long b, h, n; };
Strides strides_of(const long long* s, int H, int N, int d) {
  return s ? Strides{s[0], s[1], s[2]} : Strides{(long long)H * N * d, (long long)N * d, d};
}
template <class... P> bool all_aligned16(P... p) { return (aligned16(p) && ...); }

}  // namespace

extern "C" int attn_rope(const void* Q, const void* K, void* Q_out, void* K_out, const long long* strides, const int* positions,
                         long long positions_stride_b, const double* frequencies, int B, int H, int H_kv, int N, int d, int rot,
                         int interleaved, float magnitude, int inverse, void* stream) {
  bool empty;
  if (H_kv < 0 || rot < 0) return ATTN_ERR_BAD_ARG;
  if ((K == nullptr) != (K_out == nullptr)) return ATTN_ERR_NULL;
  if (!K) H_kv = 0;
  if (H == 0 && H_kv > 0) {                // no queries here: the keys alone
    long long of_keys[12] = {};
    if (strides) {
      std::copy_n(strides + 3, 3, of_keys);
      std::copy_n(strides + 9, 3, of_keys + 6);
    }
    return attn_rope(K, nullptr, K_out, nullptr, strides ? of_keys : nullptr, positions, positions_stride_b, frequencies, B, H_kv, 0, N, d, rot,
                     interleaved, magnitude, inverse, stream);
  }
  int st = check_rows(B, H, N, d, &empty);
  if (st != ATTN_OK) return st;
  if (empty) return ATTN_OK;
  if (H_kv > 0 && (st = check_rows(B, H_kv, N, d, &empty)) != ATTN_OK) return st;
  if (rot < 2 || rot > d || rot % 2 != 0 || !std::isfinite(magnitude)) return ATTN_ERR_BAD_ARG;
  if ((double)H + H_kv > 65535.0 || (double)B * N >= 2147483648.0) return ATTN_ERR_UNSUPPORTED;
  if (!Q || !Q_out || !frequencies) return ATTN_ERR_NULL;
  if (!all_aligned16(Q, K, Q_out, K_out, frequencies) || !aligned4(positions)) return ATTN_ERR_BAD_ARG;
  if (positions && (positions_stride_b < 0 || positions_stride_b >= (1ll << 40))) return ATTN_ERR_BAD_ARG;
  if (strides && (!strides_ok(strides, 0) || !strides_ok(strides + 6, 1))) return ATTN_ERR_BAD_ARG;
  if (strides && K && (!strides_ok(strides + 3, 0) || !strides_ok(strides + 9, 1))) return ATTN_ERR_BAD_ARG;
  const Strides q = strides_of(strides, H, N, d), k = strides_of(strides ? strides + 3 : nullptr, H_kv, N, d);
  const Strides qo = strides_of(strides ? strides + 6 : nullptr, H, N, d), ko = strides_of(strides ? strides + 9 : nullptr, H_kv, N, d);
  auto same = [](const Strides& x, const Strides& y) { return x.b == y.b && x.h == y.h && x.n == y.n; };
  if ((Q_out == Q && !same(q, qo)) || (K && K_out == K && !same(k, ko))) return ATTN_ERR_BAD_ARG;
  if (K && (Q_out == K || K_out == Q || Q_out == K_out)) return ATTN_ERR_BAD_ARG;
  using u16 = unsigned short;
  RopeArgs a{};
  a.q = RopeSide{static_cast<const u16*>(Q), static_cast<u16*>(Q_out), q.b, q.h, q.n, qo.b, qo.h, qo.n};
  a.k = RopeSide{static_cast<const u16*>(K), static_cast<u16*>(K_out), k.b, k.h, k.n, ko.b, ko.h, ko.n};
  a.positions = positions;
  a.positions_stride = positions_stride_b;
  a.frequencies = frequencies;
  a.B = B; a.H = H; a.H_kv = H_kv; a.N = N; a.d = d; a.rot = rot;
  a.magnitude = magnitude;
  a.inverse = inverse != 0;
  return launched(attn_rope_dispatch(a, interleaved != 0, static_cast<hipStream_t>(stream)));
}

extern "C" int attn_rope_frequencies(double* out, float* magnitude, int rot, double base, int scaling, double factor,
                                     double original_length, double beta_fast, double beta_slow) {
  if (!out) return ATTN_ERR_NULL;
  if (rot < 2 || rot % 2 != 0 || rot > 256 || !(base > 0.0) || !std::isfinite(base)) return ATTN_ERR_BAD_ARG;
  if (scaling < ATTN_ROPE_NONE || scaling > ATTN_ROPE_YARN) return ATTN_ERR_BAD_ARG;
  if (scaling != ATTN_ROPE_NONE && !(factor >= 1.0 && std::isfinite(factor))) return ATTN_ERR_BAD_ARG;
  if (scaling == ATTN_ROPE_NTK) {
    if (rot < 4) return ATTN_ERR_BAD_ARG;
    base *= std::pow(factor, (double)rot / (rot - 2));
  }
  if (scaling == ATTN_ROPE_YARN &&
      (!(original_length > 0.0) || !std::isfinite(original_length) || !(beta_slow >= 0.0) || !(beta_fast > beta_slow) || !std::isfinite(beta_fast)))
    return ATTN_ERR_BAD_ARG;
  for (int i = 0; i < rot / 2; ++i) {
    const double f = std::pow(base, -2.0 * i / rot);
    out[i] = f;
    if (scaling == ATTN_ROPE_LINEAR) out[i] = f / factor;
    if (scaling == ATTN_ROPE_YARN) {
      const double turns = original_length * f / 6.283185307179586;
      const double keep = std::min(1.0, std::max(0.0, (turns - beta_slow) / (beta_fast - beta_slow)));
      out[i] = f * keep + f / factor * (1.0 - keep);
    }
  }
  if (magnitude) *magnitude = scaling == ATTN_ROPE_YARN ? (float)(0.1 * std::log(factor) + 1.0) : 1.0f;
  return ATTN_OK;
}

extern "C" int attn_cache_append(const void* K, const void* V, const long long* strides, void* K_cache, void* V_cache, float* K_scale,
                                 float* V_scale, const int* lengths, const int* counts, int B, int H_kv, int N, int d, int capacity,
                                 void* stream) {
  bool empty;
  int st = check_rows(B, H_kv, N, d, &empty);
  if (st != ATTN_OK) return st;
  if (empty) return ATTN_OK;
  if ((st = check_cache(B, H_kv, d, capacity)) != ATTN_OK) return st;
  if (!K || !V || !K_cache || !V_cache || !K_scale || !V_scale || !lengths) return ATTN_ERR_NULL;
  if (!all_aligned16(K, V, K_cache, V_cache, K_scale, V_scale) || !aligned4(lengths) || !aligned4(counts)) return ATTN_ERR_BAD_ARG;
  const void* outs[] = {K_cache, V_cache, K_scale, V_scale};
  for (int i = 0; i < 4; ++i) {
    if (outs[i] == K || outs[i] == V) return ATTN_ERR_BAD_ARG;
    for (int j = 0; j < i; ++j)
      if (outs[i] == outs[j]) return ATTN_ERR_BAD_ARG;
  }
  if (strides && (!strides_ok(strides, 0) || !strides_ok(strides + 3, 0))) return ATTN_ERR_BAD_ARG;
  const Strides k = strides_of(strides, H_kv, N, d), v = strides_of(strides ? strides + 3 : nullptr, H_kv, N, d);
  using u16 = unsigned short;
  using u8 = unsigned char;
  AppendArgs a{};
  a.cache = CacheArgs{static_cast<u8*>(K_cache), static_cast<u8*>(V_cache), K_scale, V_scale, capacity};
  a.K = Rows{static_cast<const u16*>(K), k.b, k.h, k.n};
  a.V = Rows{static_cast<const u16*>(V), v.b, v.h, v.n};
  a.lengths = lengths;
  a.counts = counts;
  a.B = B; a.H_kv = H_kv; a.N = N;
  return launched(attn_cache_append_dispatch(a, d, static_cast<hipStream_t>(stream)));
}

// Sizes of a call with H query heads over a cache of H_kv.
static int check_attend(int B, int H, int H_kv, int N, int d, int capacity, bool* empty) {
  if (H_kv < 0) return ATTN_ERR_BAD_ARG;
  int st = check_rows(B, H, N, d, empty);
  if (st != ATTN_OK || *empty) return st;
  if (H_kv < 1 || H < H_kv || H % H_kv != 0) return ATTN_ERR_BAD_ARG;
  if ((double)N * H >= 1073741824.0 || (double)B * N * H >= 274877906944.0) return ATTN_ERR_UNSUPPORTED;      // rows: counted in int per sequence
  const int st2 = check_cache(B, H_kv, d, capacity);
  if (st2 != ATTN_OK) return st2;
  // work of attn_cache_fwd is counted in int, in key blocks of row tiles (seconds of it, at this limit)
  return cache_units(B, H_kv, cache_form(B, H, H_kv, N, d, capacity), capacity) < kUnitLimit ? ATTN_OK : ATTN_ERR_UNSUPPORTED;
}

extern "C" size_t attn_cache_fwd_workspace_bytes(int B, int H, int H_kv, int N, int d, int capacity) {
  bool empty;
  if (check_attend(B, H, H_kv, N, d, capacity, &empty) != ATTN_OK || empty) return 0;
  return attn_cache_fwd_partial_bytes(B, H, H_kv, N, d, capacity);
}

extern "C" int attn_cache_fwd(const void* Q, const long long* strides, const void* K_cache, const void* V_cache, const float* K_scale,
                              const float* V_scale, const int* lengths, const int* counts, void* O, float* LSE, void* workspace,
                              size_t workspace_bytes, int B, int H, int H_kv, int N, int d, int capacity, int causal,
                              float softmax_scale, void* stream) {
  bool empty;
  int st = check_attend(B, H, H_kv, N, d, capacity, &empty);
  if (st != ATTN_OK) return st;
  if (!scale_ok(softmax_scale)) return ATTN_ERR_BAD_ARG;
  if (empty) return ATTN_OK;
  if (!Q || !K_cache || !V_cache || !K_scale || !V_scale || !lengths || !O || !LSE) return ATTN_ERR_NULL;
  if (!all_aligned16(Q, K_cache, V_cache, K_scale, V_scale, O, LSE) || !aligned4(lengths) || !aligned4(counts)) return ATTN_ERR_BAD_ARG;
  if (O == Q || O == K_cache || O == V_cache || O == LSE || LSE == K_scale || LSE == V_scale) return ATTN_ERR_BAD_ARG;
  if (strides && (!strides_ok(strides, 0) || !strides_ok(strides + 3, 1))) return ATTN_ERR_BAD_ARG;
  const size_t need = attn_cache_fwd_partial_bytes(B, H, H_kv, N, d, capacity);
  if (need > 0 && !workspace) return ATTN_ERR_NULL;
  if (need > 0 && (workspace_bytes < need || !aligned16(workspace))) return ATTN_ERR_WORKSPACE;
  const Strides q = strides_of(strides, H, N, d), o = strides_of(strides ? strides + 3 : nullptr, H, N, d);
  using u16 = unsigned short;
  using u8 = unsigned char;
  AttendArgs a{};
  a.cache = CacheArgs{static_cast<u8*>(const_cast<void*>(K_cache)), static_cast<u8*>(const_cast<void*>(V_cache)),
                      const_cast<float*>(K_scale), const_cast<float*>(V_scale), capacity};
  a.Q = Rows{static_cast<const u16*>(Q), q.b, q.h, q.n};
  a.O = static_cast<u16*>(O);
  a.o_sb = o.b; a.o_sh = o.h; a.o_sn = o.n;
  a.LSE = LSE;
  a.lengths = lengths;
  a.counts = counts;
  a.B = B; a.H = H; a.H_kv = H_kv; a.N = N; a.group = H / H_kv; a.causal = causal != 0;
  a.scale = softmax_scale;
  a.partials = static_cast<float*>(workspace);
  return launched(attn_cache_fwd_dispatch(a, d, static_cast<hipStream_t>(stream)));
}

extern "C" int attn_cache_weights(const void* Q, const long long* strides, const void* K_cache, const float* K_scale, const float* LSE,
                                  const int* lengths, const int* counts, const float* weights_in, float* weights_out, int B, int H,
                                  int H_kv, int N, int d, int capacity, int causal, float softmax_scale, void* stream) {
  bool empty;
  int st = check_attend(B, H, H_kv, N, d, capacity, &empty);
  if (st != ATTN_OK) return st;
  if (!scale_ok(softmax_scale)) return ATTN_ERR_BAD_ARG;
  if (empty) return ATTN_OK;
  if (!Q || !K_cache || !K_scale || !LSE || !lengths || !weights_out) return ATTN_ERR_NULL;
  if (!all_aligned16(Q, K_cache, K_scale, LSE, weights_in, weights_out) || !aligned4(lengths) || !aligned4(counts)) return ATTN_ERR_BAD_ARG;
  const void* out = weights_out;
  if (out == Q || out == K_cache || out == K_scale || out == LSE) return ATTN_ERR_BAD_ARG;
  if (strides && !strides_ok(strides, 0)) return ATTN_ERR_BAD_ARG;
  const Strides q = strides_of(strides, H, N, d);
  WeighArgs a{};
  a.cache = CacheArgs{static_cast<unsigned char*>(const_cast<void*>(K_cache)), nullptr, const_cast<float*>(K_scale), nullptr, capacity};
  a.Q = Rows{static_cast<const unsigned short*>(Q), q.b, q.h, q.n};
  a.LSE = LSE;
  a.in = weights_in;
  a.out = weights_out;
  a.lengths = lengths;
  a.counts = counts;
  a.B = B; a.H = H; a.H_kv = H_kv; a.N = N; a.group = H / H_kv; a.causal = causal != 0;
  a.scale = softmax_scale;
  return launched(attn_cache_weights_dispatch(a, d, static_cast<hipStream_t>(stream)));
}

extern "C" int attn_cache_evict(const void* K_cache, const void* V_cache, const float* K_scale, const float* V_scale, const float* weights,
                                const int* lengths, void* K_out, void* V_out, float* K_scale_out, float* V_scale_out,
                                float* weights_out, int* kept, int B, int H_kv, int d, int capacity, int capacity_out, int budget,
                                int recent, void* stream) {
  bool empty;
  int st = check_rows(B, H_kv, 1, d, &empty);
  if (st != ATTN_OK) return st;
  if (empty) return ATTN_OK;
  if ((st = check_cache(B, H_kv, d, capacity)) != ATTN_OK || (st = check_cache(B, H_kv, d, capacity_out)) != ATTN_OK) return st;
  if (budget < 1 || budget > capacity_out || recent < 0 || recent > budget) return ATTN_ERR_BAD_ARG;
  if (!K_cache || !V_cache || !K_scale || !V_scale || !weights || !lengths || !K_out || !V_out || !K_scale_out || !V_scale_out || !kept)
    return ATTN_ERR_NULL;
  if (!all_aligned16(K_cache, V_cache, K_scale, V_scale, weights, K_out, V_out, K_scale_out, V_scale_out, weights_out) ||
      !aligned4(lengths) || !aligned4(kept))
    return ATTN_ERR_BAD_ARG;
  const void* ins[] = {K_cache, V_cache, K_scale, V_scale, weights, lengths};
  const void* outs[] = {K_out, V_out, K_scale_out, V_scale_out, kept, weights_out};
  for (int i = 0; i < 6; ++i) {
    for (const void* p : ins)
      if (outs[i] == p) return ATTN_ERR_BAD_ARG;
    for (int j = 0; j < i; ++j)
      if (outs[i] == outs[j]) return ATTN_ERR_BAD_ARG;
  }
  using u8 = unsigned char;
  EvictArgs a{};
  a.from = CacheArgs{static_cast<u8*>(const_cast<void*>(K_cache)), static_cast<u8*>(const_cast<void*>(V_cache)),
                     const_cast<float*>(K_scale), const_cast<float*>(V_scale), capacity};
  a.to = CacheArgs{static_cast<u8*>(K_out), static_cast<u8*>(V_out), K_scale_out, V_scale_out, capacity_out};
  a.weights = weights;
  a.weights_out = weights_out;
  a.kept = kept;
  a.lengths = lengths;
  a.B = B; a.H_kv = H_kv; a.budget = budget; a.recent = recent;
  return launched(attn_cache_evict_dispatch(a, d, static_cast<hipStream_t>(stream)));
}
