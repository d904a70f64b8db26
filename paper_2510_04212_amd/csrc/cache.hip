// Writing the 8-bit cache: new tokens quantised into it (attn_cache_append of include/attn.h), and a cache cut down to the
// tokens that got the most attention (attn_cache_evict).
#include "cache.hpp"

namespace {

constexpr int kThreads = 256;

DEVI unsigned max_over_wave(unsigned x) {
#pragma unroll
  for (int i = 32; i; i >>= 1) x = max(x, (unsigned)__shfl_xor((int)x, i));
  return x;
}

// ---- append.  One work-group per (sequence, head, block of the cache that gets tokens): it alone reads and writes that
// block and its scales.  With amax the largest finite magnitude of the block's new tokens, the block's exponent is
//   e = max(exponent_for(amax), e of the tokens that are already in it),
// a new code is the E4M3 number nearest to x 2^-e, and where e grew the older codes are multiplied by 2^(e_old - e): exact, E4M3
// being a floating-point format, but for results below its normal range (2^-6 of 448 2^e).  No token's code depends on how
// tokens were split into calls but for that.
//
// Bound by bytes: 2 read and 1 written per element.  All loads of a thread are in flight before the maximum is taken; K
// is handled in rows (a wave reads 1 KB and writes 512 consecutive bytes), V in pieces of 4 tokens x 8 columns, so that four
// codes of one column are one 4-byte store and 16 lanes write a column's 64 consecutive bytes.
DEVI unsigned magnitude(unsigned bits16) {                 // of a finite bf16 number; 0 for infinities and NaN
  const unsigned m = bits16 & 0x7fffu;
  return m < 0x7f80u ? m : 0u;
}
DEVI unsigned largest8(u32x4 x) {
  unsigned m = 0;
#pragma unroll
  for (int j = 0; j < 4; ++j) m = max(m, max(magnitude(x[j] & 0xffffu), magnitude(x[j] >> 16)));
  return m;
}
DEVI unsigned any_nan8(u32x4 x) {
  unsigned m = 0;
#pragma unroll
  for (int j = 0; j < 4; ++j) m |= (unsigned)((x[j] & 0x7fffu) > 0x7f80u) | (unsigned)((x[j] & 0x7fffffffu) > 0x7f80ffffu);
  return m;
}
DEVI float bf16_at(u32x4 x, int j) { return __uint_as_float((j & 1) ? x[j / 2] & 0xffff0000u : x[j / 2] << 16); }

template <int D> __global__ __launch_bounds__(kThreads) void attn_cache_append_kernel(AppendArgs p) {
  constexpr int CH = D / 8;                                // 16-byte chunks of a bf16 row
  constexpr int NK = kBlock * CH / kThreads;               // chunks per thread
  constexpr int UNITS = kBlock / 4 * CH, NU = (UNITS + kThreads - 1) / kThreads;
  const int b = blockIdx.z, h = blockIdx.y, tid = threadIdx.x;
  const int n = real_count(p.counts, b, p.N);
  const long long length = p.lengths[b], first = length - n;            // position of the first new token
  const long long blk = (max(first, 0ll) >> 6) + blockIdx.x, base = blk * kBlock;
  if (n == 0 || base >= min(length, (long long)p.cache.capacity)) return;
  const bool fresh = base >= first;
  const size_t bh = (size_t)b * p.H_kv + h;
  const size_t at_scale = bh * (p.cache.capacity / kBlock) + blk;
  unsigned char* K = p.cache.K + (bh * p.cache.capacity + base) * D;
  unsigned char* V = p.cache.V + at_scale * (D * kBlock);
  const unsigned short* Kn = p.K.at + b * p.K.sb + h * p.K.sh;
  const unsigned short* Vn = p.V.at + b * p.V.sb + h * p.V.sh;
  auto index = [&](int t) { return base + t - first; };                 // of the block's token t among the new ones
  auto is_new = [&](int t) { return index(t) >= 0 && index(t) < n; };

  u32x4 xk[NK], xv[NU][4];
  unsigned mk = 0, mv = 0, nan = 0;
#pragma unroll
  for (int k = 0; k < NK; ++k) {
    const int v = tid + k * kThreads, t = v / CH, c = v % CH;
    xk[k] = u32x4{0, 0, 0, 0};
    if (is_new(t)) xk[k] = *reinterpret_cast<const u32x4*>(Kn + index(t) * p.K.sn + c * 8);
  }
#pragma unroll
  for (int k = 0; k < NU; ++k) {
    const int unit = tid + k * kThreads, u = unit & 15, c = unit >> 4;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      xv[k][j] = u32x4{0, 0, 0, 0};
      if (unit < UNITS && is_new(4 * u + j)) xv[k][j] = *reinterpret_cast<const u32x4*>(Vn + index(4 * u + j) * p.V.sn + c * 8);
    }
  }
  const int old_k = fresh ? kLowestExponent : exponent(p.cache.K_scale[at_scale]);
  const float was_v = fresh ? power(kLowestExponent) : p.cache.V_scale[at_scale];
  const int old_v = exponent(was_v);
#pragma unroll
  for (int k = 0; k < NK; ++k) mk = max(mk, largest8(xk[k]));
#pragma unroll
  for (int k = 0; k < NU; ++k)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      mv = max(mv, largest8(xv[k][j]));
      nan |= any_nan8(xv[k][j]);
    }
  __shared__ unsigned most[2][kThreads / 64], nans[kThreads / 64];
  mk = max_over_wave(mk);
  mv = max_over_wave(mv);
  nan = __any(nan != 0) ? 1u : 0u;
  if ((tid & 63) == 0) { most[0][tid >> 6] = mk; most[1][tid >> 6] = mv; nans[tid >> 6] = nan; }
  __syncthreads();                                         // (every thread has read the old scales, too)
#pragma unroll
  for (int w = 0; w < kThreads / 64; ++w) { mk = max(mk, most[0][w]); mv = max(mv, most[1][w]); nan |= nans[w]; }
  const int ek = max(exponent_for(__uint_as_float(mk << 16)), old_k), ev = max(exponent_for(__uint_as_float(mv << 16)), old_v);
  if (tid == 0) { p.cache.K_scale[at_scale] = power(ek); p.cache.V_scale[at_scale] = nan || was_v < 0.f ? -power(ev) : power(ev); }

  // whole: every code of the block is written, zeros behind the last token; otherwise the new tokens' alone
  const bool whole_k = fresh || ek != old_k, whole_v = fresh || ev != old_v;
  const float to_k = power(-ek), to_v = power(-ev);
  const float times_k = power(max(old_k - ek, -126)), times_v = power(max(old_v - ev, -126));
#pragma unroll
  for (int k = 0; k < NK; ++k) {
    const int v = tid + k * kThreads, t = v / CH, c = v % CH;
    const bool fills = is_new(t);
    if (!fills && !whole_k) continue;
    uint2 w = make_uint2(0, 0);
    uint2* to = reinterpret_cast<uint2*>(K + t * D + c * 8);
    if (fills) {
      w.x = pack4_e4m3(bf16_at(xk[k], 0) * to_k, bf16_at(xk[k], 1) * to_k, bf16_at(xk[k], 2) * to_k, bf16_at(xk[k], 3) * to_k);
      w.y = pack4_e4m3(bf16_at(xk[k], 4) * to_k, bf16_at(xk[k], 5) * to_k, bf16_at(xk[k], 6) * to_k, bf16_at(xk[k], 7) * to_k);
    } else if (index(t) < 0) {
      w = *to;
      w.x = rescale4_e4m3(w.x, times_k);
      w.y = rescale4_e4m3(w.y, times_k);
    }
    *to = w;
  }
#pragma unroll
  for (int k = 0; k < NU; ++k) {
    const int unit = tid + k * kThreads, u = unit & 15, c = unit >> 4;
    if (unit >= UNITS) continue;
    unsigned fills = 0, keeps = 0;                         // 0xff in the byte of a new / an older token
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      fills |= is_new(4 * u + j) ? 0xffu << (8 * j) : 0u;
      keeps |= index(4 * u + j) < 0 ? 0xffu << (8 * j) : 0u;
    }
    if (!fills && !whole_v) continue;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      unsigned* to = reinterpret_cast<unsigned*>(V + (c * 8 + i) * kBlock + 4 * u);
      unsigned w = pack4_e4m3(bf16_at(xv[k][0], i) * to_v, bf16_at(xv[k][1], i) * to_v, bf16_at(xv[k][2], i) * to_v,
                              bf16_at(xv[k][3], i) * to_v) & fills;
      if (fills != 0xffffffffu) {
        if (!whole_v) w |= *to & ~fills;
        else if (keeps) w |= rescale4_e4m3(*to, times_v) & keeps;
      }
      *to = w;
    }
  }
}

// ---- evict, first kernel: which tokens stay.  One work-group per (sequence, head).  The need-th largest of the weights in front of
// the recent tokens is found digit by digit (11, 11 and 10 bits of an order-preserving integer form) with a histogram in LDS, then the
// tokens above it and the first of those equal to it are written in ascending order: positions are prefix counts.
constexpr int kSelectThreads = 1024;
constexpr int kBins = 2048;

// larger weight <=> larger key; -0 = +0, NaN above everything
DEVI unsigned sort_key(float w) {
  const unsigned u = __float_as_uint(w);
  if (w != w) return 0xffffffffu;
  if (w == 0.f) return 0x80000000u;
  return (u & 0x80000000u) ? ~u : u | 0x80000000u;
}

// inclusive sum over the work-group in thread order; every thread gets the total as well
DEVI unsigned scan_sum(unsigned x, unsigned* waves, unsigned& total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
  for (int i = 1; i < 64; i <<= 1) {
    const unsigned y = (unsigned)__shfl_up((int)x, i);
    if (lane >= i) x += y;
  }
  __syncthreads();
  if (lane == 63) waves[wave] = x;
  __syncthreads();
  unsigned before = 0;
  total = 0;
#pragma unroll
  for (int w = 0; w < kSelectThreads / 64; ++w) {
    if (w < wave) before += waves[w];
    total += waves[w];
  }
  return x + before;
}

__global__ __launch_bounds__(kSelectThreads) void attn_cache_select_kernel(EvictArgs p) {
  __shared__ unsigned bins[kBins];
  __shared__ unsigned waves[kSelectThreads / 64];
  __shared__ unsigned found[2];
  const int b = blockIdx.y, h = blockIdx.x, tid = threadIdx.x;
  const size_t bh = (size_t)b * p.H_kv + h;
  int* kept = p.kept + bh * p.budget;
  const int length = min(max(p.lengths[b], 0), p.from.capacity);
  const int stay = min(length, p.budget);
  for (int i = stay + tid; i < p.budget; i += kSelectThreads) kept[i] = -1;
  if (length <= p.budget) {
    for (int i = tid; i < length; i += kSelectThreads) kept[i] = i;
    return;
  }
  const int old = length - p.recent, need = p.budget - p.recent;      // need < old
  for (int i = tid; i < p.recent; i += kSelectThreads) kept[need + i] = old + i;
  if (need == 0) return;
  const float* weights = p.weights + bh * p.from.capacity;

  unsigned prefix = 0, known = 0;                          // the digits found so far, and the bits they cover
  unsigned left = (unsigned)need;                          // wanted among the keys that have these digits
#pragma unroll 1
  for (int pass = 0; pass < 3; ++pass) {
    const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0;
    const unsigned digits = pass == 2 ? 1023u : 2047u;
    for (int i = tid; i < kBins; i += kSelectThreads) bins[i] = 0;
    __syncthreads();
    for (int i = tid; i < old; i += kSelectThreads) {
      const unsigned key = sort_key(weights[i]);
      if ((key & known) == prefix) atomicAdd(&bins[(key >> shift) & digits], 1u);
    }
    __syncthreads();
    // from the top: thread t holds bins (2047 - 2t) and the one below
    const int top = kBins - 1 - 2 * tid;
    const unsigned upper = bins[top], lower = bins[top - 1];
    unsigned total;
    const unsigned to = scan_sum(upper + lower, waves, total), from = to - upper - lower;
    if (from < left && left <= to) {
      const bool in_upper = left <= from + upper;
      found[0] = (unsigned)(in_upper ? top : top - 1);
      found[1] = left - (in_upper ? from : from + upper);
    }
    __syncthreads();
    prefix |= found[0] << shift;
    known |= digits << shift;
    left = found[1];
    __syncthreads();
  }
  // key == prefix: of these the first `left` stay
  unsigned above = 0, equal = 0;                           // before the present stretch
  for (int i0 = 0; i0 < old; i0 += 4 * kSelectThreads) {
    const int i = i0 + 4 * tid;
    unsigned more[4], same[4], count = 0;                  // (above, equal) as 16 + 16 bits: 4096 at most each
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const unsigned key = i + j < old ? sort_key(weights[i + j]) : 0u;
      more[j] = i + j < old && key > prefix;
      same[j] = i + j < old && key == prefix;
      count += more[j] | same[j] << 16;
    }
    unsigned total;
    const unsigned before = scan_sum(count, waves, total) - count;
    unsigned a = above + (before & 0xffffu), e = equal + (before >> 16);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      if (more[j] || (same[j] && e < left)) kept[a + min(e, left)] = i + j;
      a += more[j];
      e += same[j];
    }
    above += total & 0xffffu;
    equal += total >> 16;
  }
}

// ---- evict, second kernel: one work-group per block of the new cache.  Its scales are the largest of its tokens' old ones, so that
// codes are only ever multiplied by powers of two <= 1.  V's codes are gathered one by one (its blocks hold columns).
template <int D> __global__ __launch_bounds__(kThreads) void attn_cache_gather_kernel(EvictArgs p) {
  const int b = blockIdx.z, h = blockIdx.y, j = blockIdx.x, tid = threadIdx.x;
  const size_t bh = (size_t)b * p.H_kv + h;
  const int stay = min(min(max(p.lengths[b], 0), p.from.capacity), p.budget);
  const int here = min(stay - j * kBlock, kBlock);         // tokens of this block
  __shared__ int source[kBlock];
  __shared__ float times[2][kBlock];
  __shared__ int moved[2];                                 // does any code change?
  if (tid < kBlock) {
    const bool real = tid < here;
    const int t = real ? p.kept[bh * p.budget + j * kBlock + tid] : 0;
    if (p.weights_out)
      p.weights_out[bh * p.to.capacity + j * kBlock + tid] = real ? p.weights[bh * p.from.capacity + t] : 0.f;
    const size_t at = bh * (p.from.capacity / kBlock) + t / kBlock;
    const float vs = real ? p.from.V_scale[at] : 0.f;      // (its sign: NaN among the block's codes)
    const int ek = real ? exponent(p.from.K_scale[at]) : -127, ev = real ? exponent(vs) : -127;
    const bool nan = __any(vs < 0.f);
    const int mk = (int)max_over_wave((unsigned)(ek + 127)) - 127, mv = (int)max_over_wave((unsigned)(ev + 127)) - 127;
    source[tid] = t;
    times[0][tid] = power(max(ek - mk, -126));
    times[1][tid] = power(max(ev - mv, -126));
    const bool any_k = __any(real && ek != mk), any_v = __any(real && ev != mv);
    if (tid == 0 && here > 0) {
      moved[0] = any_k;
      moved[1] = any_v;
      const size_t to = bh * (p.to.capacity / kBlock) + j;
      p.to.K_scale[to] = power(mk);
      p.to.V_scale[to] = nan ? -power(mv) : power(mv);
    }
  }
  if (here <= 0) return;
  __syncthreads();
  const unsigned char* K = p.from.K + bh * p.from.capacity * D;
  unsigned char* K_to = p.to.K + (bh * p.to.capacity + j * kBlock) * D;
  constexpr int CH = D / 16;
#pragma unroll
  for (int k = 0; k < (kBlock * CH + kThreads - 1) / kThreads; ++k) {
    const int v = tid + k * kThreads, t = v / CH, c = v % CH;
    if (v >= kBlock * CH) break;
    u32x4 w{0, 0, 0, 0};
    if (t < here) {
      w = *reinterpret_cast<const u32x4*>(K + (size_t)source[t] * D + c * 16);
      if (moved[0]) {
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = rescale4_e4m3(w[i], times[0][t]);
      }
    }
    *reinterpret_cast<u32x4*>(K_to + t * D + c * 16) = w;
  }
  const unsigned char* V = p.from.V + bh * p.from.capacity * D;
  unsigned char* V_to = p.to.V + (bh * p.to.capacity + j * kBlock) * D;
  const int u = tid & 15;
  size_t from[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) from[i] = (size_t)(source[4 * u + i] / kBlock) * (D * kBlock) + source[4 * u + i] % kBlock;
#pragma unroll 4
  for (int c = tid >> 4; c < D; c += kThreads / 16) {
    unsigned w = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (4 * u + i < here) w |= (unsigned)V[from[i] + c * kBlock] << (8 * i);
    if (moved[1])
      w = pack4_e4m3(__builtin_amdgcn_cvt_f32_fp8((int)w, 0) * times[1][4 * u], __builtin_amdgcn_cvt_f32_fp8((int)w, 1) * times[1][4 * u + 1],
                     __builtin_amdgcn_cvt_f32_fp8((int)w, 2) * times[1][4 * u + 2], __builtin_amdgcn_cvt_f32_fp8((int)w, 3) * times[1][4 * u + 3]);
    *reinterpret_cast<unsigned*>(V_to + c * kBlock + 4 * u) = w;
  }
}

template <class F> hipError_t by_head_size(int d, F&& f) {
  switch (d) {
    case 32: return f(std::integral_constant<int, 32>{});
    case 64: return f(std::integral_constant<int, 64>{});
    case 96: return f(std::integral_constant<int, 96>{});
    case 128: return f(std::integral_constant<int, 128>{});
    default: return f(std::integral_constant<int, 256>{});
  }
}

}  // namespace

hipError_t attn_cache_append_dispatch(const AppendArgs& p, int d, hipStream_t stream) {
  // N tokens touch at most this many blocks, wherever they begin
  const dim3 grid((unsigned)((p.N + kBlock - 2) / kBlock + 1), (unsigned)p.H_kv, (unsigned)p.B);
  return by_head_size(d, [&](auto D) {
    attn_cache_append_kernel<D><<<grid, kThreads, 0, stream>>>(p);
    return hipGetLastError();
  });
}

hipError_t attn_cache_evict_dispatch(const EvictArgs& p, int d, hipStream_t stream) {
  attn_cache_select_kernel<<<dim3((unsigned)p.H_kv, (unsigned)p.B), kSelectThreads, 0, stream>>>(p);
  if (const hipError_t e = hipGetLastError(); e != hipSuccess) return e;
  const dim3 grid((unsigned)(p.to.capacity / kBlock), (unsigned)p.H_kv, (unsigned)p.B);
  return by_head_size(d, [&](auto D) {
    attn_cache_gather_kernel<D><<<grid, kThreads, 0, stream>>>(p);
    return hipGetLastError();
  });
}
