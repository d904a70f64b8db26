// Writing the 8-bit cache: new tokens quantised into it (attn_cache_append of include/attn.h), and a cache cut down to the
// tokens that got the most attention (attn_cache_evict).
#include "cache.hpp"
#include <algorithm>

namespace {

constexpr int kThreads = 256;

// ---- append.  One work-group per (sequence, head, block of the cache that gets tokens): it alone reads and writes that
// block and its scales.  With amax the largest finite magnitude of the block's new tokens, the block's exponent is
//   e = max(exponent_for(amax), e of the tokens that are already in it),
// a new code is the E4M3 number nearest to x 2^-e, and where e grew the older codes are multiplied by 2^(e_old - e): exact, E4M3
// being a floating-point format, but for results below its normal range (2^-6 of 448 2^e).  No token's code depends on how
// tokens were split into calls but for that.
//
// Bound by bytes: 2 read and 1 written per element.  All loads of a thread are in flight before the maximum is taken; K
// is handled in rows (a wave reads 1 KB and writes 512 consecutive bytes), V in pieces of 4 tokens x 8 columns, so that four
// codes of one column are one 4-byte store and 16 lanes write a column's 64 consecutive bytes.  2 sequences of up to 8192 tokens,
// 8 heads, d 128: 21 us, 3.9 TB/s.
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
      unsigned char* to = V + (c * 8 + i) * kBlock + 4 * u;
      unsigned w = pack4_e4m3(bf16_at(xv[k][0], i) * to_v, bf16_at(xv[k][1], i) * to_v, bf16_at(xv[k][2], i) * to_v,
                              bf16_at(xv[k][3], i) * to_v) & fills;
      if (whole_v || fills == 0xffffffffu) {
        if (keeps) w |= rescale4_e4m3(*reinterpret_cast<unsigned*>(to), times_v) & keeps;
        *reinterpret_cast<unsigned*>(to) = w;
      } else {                             // single bytes: nothing has to be read first
#pragma unroll
        for (int j = 0; j < 4; ++j)
          if (fills >> (8 * j) & 0xffu) to[j] = (unsigned char)(w >> (8 * j));
      }
    }
  }
}

// ---- evict, first kernel: which tokens stay.  One work-group per (sequence, head).  The need-th largest of the weights in front of
// the recent tokens is found digit by digit (11, 11 and 10 bits of an order-preserving integer form) with a histogram in LDS, then the
// tokens above it and the first of those equal to it are written in ascending order: positions are prefix counts.
//
// Bound by latency (a work-group has a head's weights for itself): keys stay in LDS, loaded once, where ROOM holds them, and loops are not
// unrolled, as the first pass over an instruction costs more than the jump.  us of 8 heads of 32768 and 128 of 4400 weights: 43 and
// 12.2 with the weights read again in every pass, 30 and 20 with the keys in registers and all loops unrolled, 22.8 and 8.8 so.
constexpr int kSelectThreads = 1024;
constexpr int kBins = 2048;

// larger weight <=> larger key; -0 = +0, NaN above everything.  No weight's key is below that of -infinity, 0x7fffff.
DEVI unsigned sort_key(float w) {
  const unsigned u = __float_as_uint(w);
  if (w != w) return 0xffffffffu;
  if (w == 0.f) return 0x80000000u;
  return (u & 0x80000000u) ? ~u : u | 0x80000000u;
}

template <int ROOM> __global__ __launch_bounds__(kSelectThreads) void attn_cache_select_kernel(EvictArgs p) {
  __shared__ u32x4 keys[ROOM / 4];
  __shared__ unsigned bins[kBins];
  __shared__ unsigned waves[2][kSelectThreads / 64];
  __shared__ unsigned found[2];
  const int b = blockIdx.y, h = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
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
  const f32x4* weights = reinterpret_cast<const f32x4*>(p.weights + bh * p.from.capacity);       // (rows of a multiple of 64)
  // Four keys to a thread at a time, whole work-groups of them: behind the last, keys are 0, which is no weight's, falls into the lowest bin, and is
  // neither above nor equal to one that is looked for.
  const int quads = (old + 4 * kSelectThreads - 1) / (4 * kSelectThreads) * kSelectThreads;
  auto from_memory = [&](int quad) {
    u32x4 k{0, 0, 0, 0};
    if (4 * quad < old) {
      const f32x4 w = weights[quad];
#pragma unroll
      for (int i = 0; i < 4; ++i) k[i] = 4 * quad + i < old ? sort_key(w[i]) : 0u;
    }
    return k;
  };
  static_assert(ROOM % (4 * kSelectThreads) == 0, "whole work-groups of keys");
  const bool stays = old <= ROOM;          // the keys do
  auto key = [&](int quad) { return stays ? keys[quad] : from_memory(quad); };
  if (stays) {
#pragma unroll 4
    for (int i = tid; i < quads; i += kSelectThreads) keys[i] = from_memory(i);
  }
  auto sum_before = [&](const unsigned* of_waves) {        // of the waves in front of this one
    const unsigned x = sum_to_lane(lane < wave ? of_waves[lane & (kSelectThreads / 64 - 1)] : 0u);
    return (unsigned)__builtin_amdgcn_readlane((int)x, 63);
  };

  unsigned prefix = 0, known = 0;                          // the digits found so far, and the bits they cover
  unsigned left = (unsigned)need;                          // wanted among the keys that have these digits
#pragma unroll 1
  for (int pass = 0; pass < 3; ++pass) {
    const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0;
    const unsigned digits = pass == 2 ? 1023u : 2047u;
    for (int i = tid; i < kBins; i += kSelectThreads) bins[i] = 0;
    __syncthreads();
#pragma unroll 1
    for (int quad = tid; quad < quads; quad += kSelectThreads) {
      const u32x4 k = key(quad);
      // keys that differ in a digit before: nothing to count, as for nearly all of them in the later passes
      if (__all(((k[0] ^ prefix) & known) != 0 && ((k[1] ^ prefix) & known) != 0 && ((k[2] ^ prefix) & known) != 0 && ((k[3] ^ prefix) & known) != 0))
        continue;
      // a wave of equal keys adds to one bin at once
      const unsigned leader = (unsigned)__builtin_amdgcn_readfirstlane((int)k[0]);
      if (__all(((k[0] ^ leader) | (k[1] ^ leader) | (k[2] ^ leader) | (k[3] ^ leader)) == 0)) {
        if (lane == 0) atomicAdd(&bins[(leader >> shift) & digits], 256u);
        continue;
      }
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (((k[i] ^ prefix) & known) == 0) atomicAdd(&bins[(k[i] >> shift) & digits], 1u);
    }
    __syncthreads();
    // from the top: thread t holds bins (2047 - 2t) and the one below
    const int top = kBins - 1 - 2 * tid;
    const unsigned upper = bins[top], lower = bins[top - 1];
    unsigned to = sum_to_lane(upper + lower);
    if (lane == 63) waves[0][wave] = to;
    __syncthreads();
    to += sum_before(waves[0]);
    const unsigned from = to - upper - lower;
    if (from < left && left <= to) {
      const bool in_upper = left <= from + upper;
      found[0] = (unsigned)(in_upper ? top : top - 1);
      found[1] = left - (in_upper ? from : from + upper);
    }
    __syncthreads();
    prefix |= found[0] << shift;
    known |= digits << shift;
    left = found[1];
  }
  // key == prefix: of these the first `left` stay.  kSelectThreads quads at a time; the counts' exchange alternates between two places.
  unsigned above = 0, equal = 0;                           // in front of them
#pragma unroll 1
  for (int first = 0, odd = 0; first < quads; first += kSelectThreads, odd ^= 1) {
    const int quad = first + tid;
    unsigned count = 0;                                    // (above, equal) as 16 + 16 bits: 4096 at most each
    const u32x4 k = key(quad);
#pragma unroll
    for (int i = 0; i < 4; ++i) count += (k[i] > prefix ? 1u : 0u) + (k[i] == prefix ? 0x10000u : 0u);
    const unsigned to = sum_to_lane(count);
    if (lane == 63) waves[odd][wave] = to;
    __syncthreads();
    const unsigned x = to - count + sum_before(waves[odd]);
    unsigned a = above + (x & 0xffffu), e = equal + (x >> 16);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const bool bigger = k[i] > prefix, tie = k[i] == prefix;
      if (bigger || (tie && e < left)) kept[a + min(e, left)] = 4 * quad + i;
      a += bigger;
      e += tie;
    }
    if (tid == kSelectThreads - 1) {
      bins[2 * odd] = a;
      bins[2 * odd + 1] = e;
    }
    __syncthreads();
    above = bins[2 * odd];
    equal = bins[2 * odd + 1];
  }
}

// ---- evict, second kernel: one work-group per block of the new cache.  Its scales are the largest of its tokens' old ones, so that
// codes are only ever multiplied by powers of two <= 1.  V's blocks hold columns: of each, four tokens' codes are picked from 8 bytes where the four
// lie so near each other (nearly all do while most tokens stay), and one by one elsewhere.  Bound by bytes: 4096 of 4400 tokens of 128 heads, d 128: 71 us,
// 3.8 TB/s.
//
// Two loads one after the other, the kept positions and what they lead to: all of a thread's codes are on their way before anything waits.  The old K is
// read once and past the caches (the whole call 86.1 -> 83.4 us, with a token's attention behind it 119.4 -> 116.7); not V, whose lines neighbouring blocks share (100), nor
// what is written, which attention reads next (4 sequences of 8192: 50.5 -> 53 with it, though 512 heads, 0.5 GB, gain 8 %).
template <int D> __global__ __launch_bounds__(kThreads) void attn_cache_gather_kernel(EvictArgs p) {
  const int b = blockIdx.z, h = blockIdx.y, j = blockIdx.x, tid = threadIdx.x;
  const size_t bh = (size_t)b * p.H_kv + h;
  const int* kept = p.kept + bh * p.budget + j * kBlock;
  const int room = min(p.budget - j * kBlock, kBlock);     // of the list: -1 behind the last kept token
  auto source = [&](int t) { return t < room ? kept[t] : -1; };
  constexpr int CH = D / 16, NK = (kBlock * CH + kThreads - 1) / kThreads, NV = D / 16;
  const int u = tid & 15;
  int from_k[NK], from_v[4];
#pragma unroll
  for (int k = 0; k < NK; ++k) from_k[k] = source((tid + k * kThreads) / CH);
#pragma unroll
  for (int i = 0; i < 4; ++i) from_v[i] = source(4 * u + i);
  const int one = tid < kBlock ? source(tid) : -1;

  const unsigned char* K = p.from.K + bh * p.from.capacity * D;
  const unsigned char* V = p.from.V + bh * p.from.capacity * D;
  u32x4 xk[NK];
#pragma unroll
  for (int k = 0; k < NK; ++k) {
    xk[k] = u32x4{0, 0, 0, 0};
    if (from_k[k] >= 0) xk[k] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(K + (size_t)from_k[k] * D + (tid + k * kThreads) % CH * 16));
  }
  const int first = max(from_v[0], 0), window = min(first % kBlock & ~3, kBlock - 8);       // of the source block's tokens: 8 from here
  unsigned pick = 0;                       // of those, v_perm's selector: 12 is a zero
  bool near = true;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const bool real = from_v[i] >= 0;
    const int at = from_v[i] % kBlock - window;
    near &= !real || (from_v[i] / kBlock == first / kBlock && at < 8);
    pick |= (real ? (unsigned)(at & 7) : 12u) << (8 * i);
  }
  unsigned lo[NV], hi[NV];
  if (near) {
    const unsigned char* eight = V + (size_t)(first / kBlock) * (D * kBlock) + (tid >> 4) * kBlock + window;
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      const unsigned* at = reinterpret_cast<const unsigned*>(eight + k * (kThreads / 16) * kBlock);
      lo[k] = at[0];
      hi[k] = at[1];
    }
  }
  // scales: the largest of the block's tokens', and what each token's codes are multiplied by
  __shared__ float times[2][kBlock];
  __shared__ int moved[2];                 // does any code change?
  if (tid < kBlock) {
    const bool real = one >= 0;
    const size_t at = bh * (p.from.capacity / kBlock) + max(one, 0) / kBlock;
    const float vs = real ? p.from.V_scale[at] : 0.f;      // (its sign: NaN among the block's codes)
    const int ek = real ? exponent(p.from.K_scale[at]) : -127, ev = real ? exponent(vs) : -127;
    if (p.weights_out) p.weights_out[bh * p.to.capacity + j * kBlock + tid] = real ? p.weights[bh * p.from.capacity + one] : 0.f;
    const bool nan = __any(vs < 0.f);
    const int mk = (int)max_over_wave((unsigned)(ek + 127)) - 127, mv = (int)max_over_wave((unsigned)(ev + 127)) - 127;
    times[0][tid] = power(max(ek - mk, -126));
    times[1][tid] = power(max(ev - mv, -126));
    const bool any_k = __any(real && ek != mk), any_v = __any(real && ev != mv), any = __any(real);
    if (tid == 0) {
      moved[0] = any_k;
      moved[1] = any_v;
      if (any) {
        const size_t to = bh * (p.to.capacity / kBlock) + j;
        p.to.K_scale[to] = power(mk);
        p.to.V_scale[to] = nan ? -power(mv) : power(mv);
      }
    }
  }
  __syncthreads();
  if (room <= 0 || kept[0] < 0) return;    // a block behind the last kept token stays as it is
  unsigned char* K_to = p.to.K + (bh * p.to.capacity + j * kBlock) * D;
  unsigned char* V_to = p.to.V + (bh * p.to.capacity + j * kBlock) * D;
#pragma unroll
  for (int k = 0; k < NK; ++k) {
    const int v = tid + k * kThreads, t = v / CH;
    if (v >= kBlock * CH) break;
    if (moved[0]) {
#pragma unroll
      for (int i = 0; i < 4; ++i) xk[k][i] = rescale4_e4m3(xk[k][i], times[0][t]);
    }
    *reinterpret_cast<u32x4*>(K_to + t * D + v % CH * 16) = xk[k];
  }
#pragma unroll
  for (int k = 0; k < NV; ++k) {
    const int c = (tid >> 4) + k * (kThreads / 16);
    unsigned w = 0;
    if (near) {
      w = __builtin_amdgcn_perm(hi[k], lo[k], pick);
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (from_v[i] >= 0) w |= (unsigned)V[(size_t)(from_v[i] / kBlock) * (D * kBlock) + c * kBlock + from_v[i] % kBlock] << (8 * i);
    }
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
  // N tokens touch at most this many blocks, wherever they begin; there are not more than the capacity's
  const long long blocks = std::min(((long long)p.N + kBlock - 2) / kBlock + 1, (long long)(p.cache.capacity / kBlock));
  if (!grid_fits(blocks, kThreads)) return hipErrorInvalidConfiguration;
  const dim3 grid((unsigned)blocks, (unsigned)p.H_kv, (unsigned)p.B);
  return by_head_size(d, [&](auto D) {
    attn_cache_append_kernel<D><<<grid, kThreads, 0, stream>>>(p);
    return hipGetLastError();
  });
}

hipError_t attn_cache_evict_dispatch(const EvictArgs& p, int d, hipStream_t stream) {
  if (!grid_fits(p.to.capacity / kBlock, kThreads)) return hipErrorInvalidConfiguration;         // (of the second kernel)
  // room for the longest sequence's keys if there is any, so that as many work-groups as possible share a compute unit (the whole call, 128 heads of 4400
  // weights: 84.0 us, and 86.4 with room for 32768; 512 of 8192: 391 and 395)
  const dim3 heads((unsigned)p.H_kv, (unsigned)p.B);
  if (p.from.capacity <= 8192) attn_cache_select_kernel<8192><<<heads, kSelectThreads, 0, stream>>>(p);
  else attn_cache_select_kernel<32768><<<heads, kSelectThreads, 0, stream>>>(p);
  if (const hipError_t e = hipGetLastError(); e != hipSuccess) return e;
  const dim3 grid((unsigned)(p.to.capacity / kBlock), (unsigned)p.H_kv, (unsigned)p.B);
  return by_head_size(d, [&](auto D) {
    attn_cache_gather_kernel<D><<<grid, kThreads, 0, stream>>>(p);
    return hipGetLastError();
  });
}
