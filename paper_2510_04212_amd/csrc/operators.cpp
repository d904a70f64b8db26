// Plain calls of the rotary positions, of the 8-bit cache and of the choice among beams, marshalled in C++ (host code only; every computation is behind the C ABI).
//
// What bounds a token's step is the host: rotating, appending or attending for one token takes the GPU 4 to 7 us, and the checks, ctypes
// conversions and allocations of binding.py took longer.  us a call among others, in Python -> here: rotating one token of 32 sequences
// 17.4 -> 5.7, appending it 12.4 -> 6.1, attending to 1024 tokens of one sequence 16.4 -> 5.8.
//
// Each function takes the plain case - tensors on the current GPU, of the types, shapes, strides and alignments that binding.py and the library
// accept, outputs and workspace new, on the current stream - and returns None for any other: the caller's Python code then handles it, or raises
// what it always raised.
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/utils/pybind.h>
#include <ATen/ATen.h>
#include <ATen/hip/impl/HIPStreamMasqueradingAsCUDA.h>
#include <c10/hip/HIPFunctions.h>
#include <algorithm>
#include <climits>
#include <optional>
#include <tuple>
#include <vector>
#include "../../include/attn.h"

namespace {

using at::Tensor;
using OptTensor = std::optional<Tensor>;
using Device = c10::DeviceIndex;

void* stream_of(Device device) { return static_cast<void*>(c10::hip::getCurrentHIPStreamMasqueradingAsCUDA(device).stream()); }

// (A tensor subclass that has its data elsewhere has the address NULL, which the library would take for an argument that is not there.)
bool on(const Tensor& t, Device device, at::ScalarType type) {
  return t.defined() && t.is_cuda() && t.layout() == at::kStrided && t.scalar_type() == type && t.get_device() == device && !t.is_neg() &&
         !t.is_conj() && t.data_ptr() != nullptr;
}
// bf16 rows [B,H,N,d] the library takes as they are
bool rows(const Tensor& t, Device device) {
  if (!on(t, device, at::kBFloat16) || t.dim() != 4 || t.numel() == 0 || t.stride(3) != 1) return false;
  if (reinterpret_cast<uintptr_t>(t.data_ptr()) % 16 != 0) return false;
  for (int i = 0; i < 3; ++i)
    if (t.stride(i) < 0 || t.stride(i) % 8 != 0 || t.size(i) > INT_MAX) return false;
  return t.size(3) <= INT_MAX;
}
bool dense(const Tensor& t, Device device, at::ScalarType type, at::IntArrayRef shape) {
  return on(t, device, type) && t.sizes() == shape && t.is_contiguous();
}
bool dense16(const Tensor& t, Device device, at::ScalarType type, at::IntArrayRef shape) {
  return dense(t, device, type, shape) && reinterpret_cast<uintptr_t>(t.data_ptr()) % 16 == 0;
}
// sequences' lengths, and counts if there are any
bool lengths_fit(const Tensor& lengths, const OptTensor& counts, Device device, int64_t B) {
  return dense(lengths, device, at::kInt, {B}) && (!counts || dense(*counts, device, at::kInt, {B}));
}
const int* ints(const Tensor& t) { return static_cast<const int*>(t.data_ptr()); }
const int* ints(const OptTensor& t) { return t ? ints(*t) : nullptr; }

struct Cache {
  const Tensor &K, &V, &K_scale, &V_scale;
  int64_t B = 0, H = 0, capacity = 0, d = 0;
  bool fits(Device device) {
    if (!on(K, device, at::kFloat8_e4m3fn) || K.dim() != 4 || K.numel() == 0) return false;
    B = K.size(0); H = K.size(1); capacity = K.size(2); d = K.size(3);
    const int64_t nb = capacity / ATTN_CACHE_BLOCK;
    return std::max(std::max(B, H), std::max(capacity, d)) <= INT_MAX && capacity % ATTN_CACHE_BLOCK == 0 && dense16(K, device, at::kFloat8_e4m3fn, {B, H, capacity, d}) &&
           dense16(V, device, at::kFloat8_e4m3fn, {B, H, nb, d, ATTN_CACHE_BLOCK}) && dense16(K_scale, device, at::kFloat, {B, H, nb}) &&
           dense16(V_scale, device, at::kFloat, {B, H, nb});
  }
  float* ks() const { return static_cast<float*>(K_scale.data_ptr()); }
  float* vs() const { return static_cast<float*>(V_scale.data_ptr()); }
};

void put(long long* s, const Tensor& t) {
  for (int i = 0; i < 3; ++i) s[i] = t.stride(i);
}
// The library has a reason of its own to refuse: binding.py raises it.
bool done(int status) { return status == ATTN_OK; }

std::optional<std::tuple<Tensor, OptTensor>> rope(const Tensor& q, const OptTensor& k, const Tensor& frequencies, const OptTensor& positions,
                                                  bool interleaved, double magnitude, bool inverse) {
  if (!q.defined() || !q.is_cuda()) return std::nullopt;
  const auto device = c10::hip::current_device();
  if (!rows(q, device) || (k && !rows(*k, device))) return std::nullopt;
  const int64_t B = q.size(0), H = q.size(1), N = q.size(2), d = q.size(3);
  if (k && (k->size(0) != B || k->size(2) != N || k->size(3) != d)) return std::nullopt;
  if (!on(frequencies, device, at::kDouble) || frequencies.dim() != 1 || !frequencies.is_contiguous() || 2 * frequencies.numel() > d) return std::nullopt;
  long long stride = 0;
  if (positions) {
    const Tensor& p = *positions;
    if (!on(p, device, at::kInt) || p.dim() < 1 || p.dim() > 2 || p.size(-1) != N || p.stride(-1) != 1 || (p.dim() == 2 && p.size(0) != B)) return std::nullopt;
    if (p.dim() == 2) stride = p.stride(0);
  }
  Tensor q_out = at::empty_like(q);
  OptTensor k_out;
  if (k) k_out = at::empty_like(*k);
  long long strides[12] = {};
  put(strides, q);
  put(strides + 6, q_out);
  if (k) {
    put(strides + 3, *k);
    put(strides + 9, *k_out);
  }
  if (!done(attn_rope(q.data_ptr(), k ? k->data_ptr() : nullptr, q_out.data_ptr(), k ? k_out->data_ptr() : nullptr, strides, ints(positions), stride,
                      static_cast<const double*>(frequencies.data_ptr()), (int)B, (int)H, k ? (int)k->size(1) : 0, (int)N, (int)d, (int)(2 * frequencies.numel()),
                      interleaved, (float)magnitude, inverse, stream_of(device))))
    return std::nullopt;
  return std::make_tuple(q_out, k_out);
}

bool cache_append(const Tensor& K, const Tensor& V, const Tensor& K_scale, const Tensor& V_scale, const Tensor& k, const Tensor& v,
                  const Tensor& lengths, const OptTensor& counts) {
  if (!k.defined() || !k.is_cuda()) return false;
  const auto device = c10::hip::current_device();
  Cache c{K, V, K_scale, V_scale};
  if (!c.fits(device) || !rows(k, device) || !rows(v, device) || k.sizes() != v.sizes()) return false;
  if (k.size(0) != c.B || k.size(1) != c.H || k.size(3) != c.d || !lengths_fit(lengths, counts, device, c.B)) return false;
  long long strides[6];
  put(strides, k);
  put(strides + 3, v);
  return done(attn_cache_append(k.data_ptr(), v.data_ptr(), strides, K.data_ptr(), V.data_ptr(), c.ks(), c.vs(), ints(lengths), ints(counts),
                                (int)c.B, (int)c.H, (int)k.size(2), (int)c.d, (int)c.capacity, stream_of(device)));
}

std::optional<std::tuple<Tensor, Tensor>> cache_fwd(const Tensor& K, const Tensor& V, const Tensor& K_scale, const Tensor& V_scale, const Tensor& q,
                                                    const Tensor& lengths, double scale, bool causal, const OptTensor& counts) {
  if (!q.defined() || !q.is_cuda()) return std::nullopt;
  const auto device = c10::hip::current_device();
  Cache c{K, V, K_scale, V_scale};
  if (!c.fits(device) || !rows(q, device) || q.size(0) != c.B || q.size(3) != c.d || !lengths_fit(lengths, counts, device, c.B)) return std::nullopt;
  const int B = (int)c.B, H = (int)q.size(1), N = (int)q.size(2), d = (int)c.d, capacity = (int)c.capacity;
  Tensor o = at::empty({B, H, N, d}, q.options());
  Tensor lse = at::empty({B, H, N}, q.options().dtype(at::kFloat));
  const size_t need = attn_cache_fwd_workspace_bytes(B, H, (int)c.H, N, d, capacity);
  Tensor ws;
  if (need > 0) ws = at::empty({(int64_t)need}, q.options().dtype(at::kByte));
  long long strides[6];
  put(strides, q);
  put(strides + 3, o);
  if (!done(attn_cache_fwd(q.data_ptr(), strides, K.data_ptr(), V.data_ptr(), c.ks(), c.vs(), ints(lengths), ints(counts), o.data_ptr(),
                           static_cast<float*>(lse.data_ptr()), need > 0 ? ws.data_ptr() : nullptr, need, B, H, (int)c.H, N, d, capacity, causal,
                           (float)scale, stream_of(device))))
    return std::nullopt;
  return std::make_tuple(o, lse);
}

OptTensor cache_weights(const Tensor& K, const Tensor& V, const Tensor& K_scale, const Tensor& V_scale, const Tensor& q, const Tensor& lse,
                        const Tensor& lengths, double scale, bool causal, const OptTensor& counts, const OptTensor& weights, const OptTensor& out) {
  if (!q.defined() || !q.is_cuda()) return std::nullopt;
  const auto device = c10::hip::current_device();
  Cache c{K, V, K_scale, V_scale};
  if (!c.fits(device) || !rows(q, device) || q.size(0) != c.B || q.size(3) != c.d || !lengths_fit(lengths, counts, device, c.B)) return std::nullopt;
  const int B = (int)c.B, H = (int)q.size(1), N = (int)q.size(2);
  if (!dense16(lse, device, at::kFloat, {B, H, N})) return std::nullopt;
  const int64_t shape[3] = {c.B, c.H, c.capacity};
  if ((weights && !dense16(*weights, device, at::kFloat, shape)) || (out && !dense16(*out, device, at::kFloat, shape))) return std::nullopt;
  Tensor to = out ? *out : at::empty(shape, q.options().dtype(at::kFloat));
  long long strides[3];
  put(strides, q);
  if (!done(attn_cache_weights(q.data_ptr(), strides, K.data_ptr(), c.ks(), static_cast<const float*>(lse.data_ptr()), ints(lengths), ints(counts),
                               weights ? static_cast<const float*>(weights->data_ptr()) : nullptr, static_cast<float*>(to.data_ptr()), B, H, (int)c.H, N,
                               (int)c.d, (int)c.capacity, causal, (float)scale, stream_of(device))))
    return std::nullopt;
  return to;
}

// Into the given cache; the weights of the kept tokens and their old positions.
std::optional<std::tuple<Tensor, Tensor>> cache_evict(const Tensor& K, const Tensor& V, const Tensor& K_scale, const Tensor& V_scale,
                                                      const Tensor& weights, const Tensor& lengths, const Tensor& Ko, const Tensor& Vo,
                                                      const Tensor& Kso, const Tensor& Vso, int64_t budget, int64_t recent) {
  if (!K.defined() || !K.is_cuda()) return std::nullopt;
  const auto device = c10::hip::current_device();
  Cache c{K, V, K_scale, V_scale}, o{Ko, Vo, Kso, Vso};
  if (!c.fits(device) || !o.fits(device) || o.B != c.B || o.H != c.H || o.d != c.d) return std::nullopt;
  if (budget < 1 || budget > o.capacity || recent < 0 || recent > budget) return std::nullopt;
  if (!dense16(weights, device, at::kFloat, {c.B, c.H, c.capacity}) || !lengths_fit(lengths, std::nullopt, device, c.B)) return std::nullopt;
  Tensor w = at::empty({c.B, c.H, o.capacity}, weights.options());
  Tensor kept = at::empty({c.B, c.H, budget}, lengths.options());
  if (!done(attn_cache_evict(K.data_ptr(), V.data_ptr(), c.ks(), c.vs(), static_cast<const float*>(weights.data_ptr()), ints(lengths), Ko.data_ptr(),
                             Vo.data_ptr(), o.ks(), o.vs(), static_cast<float*>(w.data_ptr()), static_cast<int*>(kept.data_ptr()), (int)c.B, (int)c.H,
                             (int)c.d, (int)c.capacity, (int)o.capacity, (int)budget, (int)recent, stream_of(device))))
    return std::nullopt;
  return std::make_tuple(w, kept);
}

std::optional<std::tuple<Tensor, Tensor>> cache_fwd_shared(const Tensor& Kp, const Tensor& Vp, const Tensor& Kps, const Tensor& Vps, const Tensor& prefix_lengths,
                                                           const Tensor& K, const Tensor& V, const Tensor& K_scale, const Tensor& V_scale, const Tensor& q,
                                                           const Tensor& lengths, double scale, bool causal, const OptTensor& counts) {
  if (!q.defined() || !q.is_cuda()) return std::nullopt;
  const auto device = c10::hip::current_device();
  Cache p{Kp, Vp, Kps, Vps}, c{K, V, K_scale, V_scale};
  if (!c.fits(device) || !p.fits(device) || p.H != c.H || p.d != c.d || c.B % p.B != 0) return std::nullopt;
  if (!rows(q, device) || q.size(0) != c.B || q.size(3) != c.d || !lengths_fit(lengths, counts, device, c.B) ||
      !lengths_fit(prefix_lengths, std::nullopt, device, p.B))
    return std::nullopt;
  const int P = (int)p.B, S = (int)(c.B / p.B), H = (int)q.size(1), N = (int)q.size(2), d = (int)c.d;
  const size_t need = attn_cache_fwd_shared_workspace_bytes(P, S, H, (int)c.H, N, d, (int)p.capacity, (int)c.capacity);
  Tensor o = at::empty({c.B, H, N, d}, q.options());
  Tensor lse = at::empty({c.B, H, N}, q.options().dtype(at::kFloat));
  Tensor ws;
  if (need > 0) ws = at::empty({(int64_t)need}, q.options().dtype(at::kByte));
  long long strides[6];
  put(strides, q);
  put(strides + 3, o);
  if (!done(attn_cache_fwd_shared(q.data_ptr(), strides, Kp.data_ptr(), Vp.data_ptr(), p.ks(), p.vs(), ints(prefix_lengths), K.data_ptr(), V.data_ptr(), c.ks(),
                                  c.vs(), ints(lengths), ints(counts), o.data_ptr(), static_cast<float*>(lse.data_ptr()), need > 0 ? ws.data_ptr() : nullptr,
                                  need, P, S, H, (int)c.H, N, d, (int)p.capacity, (int)c.capacity, causal, (float)scale, stream_of(device))))
    return std::nullopt;
  return std::make_tuple(o, lse);
}

// Into the given cache; its lengths.
OptTensor cache_fork(const Tensor& K, const Tensor& V, const Tensor& K_scale, const Tensor& V_scale, const Tensor& sources, const Tensor& lengths,
                     const Tensor& Ko, const Tensor& Vo, const Tensor& Kso, const Tensor& Vso) {
  if (!K.defined() || !K.is_cuda()) return std::nullopt;
  const auto device = c10::hip::current_device();
  Cache c{K, V, K_scale, V_scale}, o{Ko, Vo, Kso, Vso};
  if (!c.fits(device) || !o.fits(device) || o.H != c.H || o.d != c.d) return std::nullopt;
  if (!lengths_fit(lengths, std::nullopt, device, c.B) || !lengths_fit(sources, std::nullopt, device, o.B)) return std::nullopt;
  Tensor left = at::empty({o.B}, lengths.options());
  if (!done(attn_cache_fork(K.data_ptr(), V.data_ptr(), c.ks(), c.vs(), ints(sources), ints(lengths), Ko.data_ptr(), Vo.data_ptr(), o.ks(), o.vs(),
                            static_cast<int*>(left.data_ptr()), (int)c.B, (int)o.B, (int)c.H, (int)c.d, (int)c.capacity, (int)o.capacity, stream_of(device))))
    return std::nullopt;
  return left;
}

OptTensor cache_reorder(const Tensor& K, const Tensor& V, const Tensor& K_scale, const Tensor& V_scale, const Tensor& parents, const Tensor& lengths) {
  if (!K.defined() || !K.is_cuda()) return std::nullopt;
  const auto device = c10::hip::current_device();
  Cache c{K, V, K_scale, V_scale};
  if (!c.fits(device) || !parents.defined() || parents.dim() != 2 || parents.numel() != c.B) return std::nullopt;
  if (!dense(parents, device, at::kInt, parents.sizes()) || !lengths_fit(lengths, std::nullopt, device, c.B)) return std::nullopt;
  Tensor left = at::empty({c.B}, lengths.options());
  if (!done(attn_cache_reorder(K.data_ptr(), V.data_ptr(), c.ks(), c.vs(), ints(parents), ints(lengths), static_cast<int*>(left.data_ptr()),
                               (int)parents.size(0), (int)parents.size(1), (int)c.H, (int)c.d, (int)c.capacity, stream_of(device))))
    return std::nullopt;
  return left;
}

std::optional<std::tuple<Tensor, Tensor, Tensor, Tensor>> beam_select(const Tensor& logits, const Tensor& scores, int64_t n, const OptTensor& finished,
                                                                      const std::optional<int64_t>& end_token) {
  if (!logits.defined() || !logits.is_cuda()) return std::nullopt;
  const auto device = c10::hip::current_device();
  const bool wide = logits.scalar_type() == at::kFloat;
  if (!on(logits, device, wide ? at::kFloat : at::kBFloat16) || logits.dim() != 3 || logits.numel() == 0 || logits.stride(2) != 1) return std::nullopt;
  const int64_t B = logits.size(0), beams = logits.size(1), V = logits.size(2);
  if (std::max(std::max(B, beams), V) > INT_MAX || n < 1 || n > INT_MAX || logits.stride(0) < 0 || logits.stride(1) < 0) return std::nullopt;
  if (!dense(scores, device, at::kFloat, {B, beams}) || (finished && (!end_token || !dense(*finished, device, at::kBool, {B, beams})))) return std::nullopt;
  if (end_token && (*end_token < 0 || *end_token >= V)) return std::nullopt;
  const size_t need = attn_beam_select_workspace_bytes((int)B, (int)beams, (int)V, (int)n);
  if (need == 0) return std::nullopt;      // refused
  const auto ints_of = logits.options().dtype(at::kInt);
  Tensor parents = at::empty({B, n}, ints_of), tokens = at::empty({B, n}, ints_of), sums = at::empty({B, n}, scores.options());
  Tensor ended = at::empty({B, n}, logits.options().dtype(at::kBool)), ws = at::empty({(int64_t)need}, logits.options().dtype(at::kByte));
  if (!done(attn_beam_select(logits.data_ptr(), wide ? ATTN_LOGITS_FLOAT32 : ATTN_LOGITS_BF16, logits.stride(0), logits.stride(1),
                             static_cast<const float*>(scores.data_ptr()), finished ? static_cast<const unsigned char*>(finished->data_ptr()) : nullptr,
                             end_token ? (int)*end_token : -1, static_cast<int*>(parents.data_ptr()), static_cast<int*>(tokens.data_ptr()),
                             static_cast<float*>(sums.data_ptr()), static_cast<unsigned char*>(ended.data_ptr()), ws.data_ptr(), need, (int)B, (int)beams,
                             (int)V, (int)n, stream_of(device))))
    return std::nullopt;
  return std::make_tuple(parents, tokens, sums, ended);
}

}  // namespace

PYBIND11_MODULE(_operators, m) {
  m.def("rope", &rope, "attn_rope; None: not a plain case");
  m.def("cache_append", &cache_append, "attn_cache_append; False: not a plain case");
  m.def("cache_fwd", &cache_fwd, "attn_cache_fwd; None: not a plain case");
  m.def("cache_weights", &cache_weights, "attn_cache_weights; None: not a plain case");
  m.def("cache_evict", &cache_evict, "attn_cache_evict; None: not a plain case");
  m.def("cache_fwd_shared", &cache_fwd_shared, "attn_cache_fwd_shared; None: not a plain case");
  m.def("cache_fork", &cache_fork, "attn_cache_fork; None: not a plain case");
  m.def("cache_reorder", &cache_reorder, "attn_cache_reorder; None: not a plain case");
  m.def("beam_select", &beam_select, "attn_beam_select; None: not a plain case");
}
