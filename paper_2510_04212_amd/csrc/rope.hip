// Rotary positions (attn_rope of include/attn.h): the first `rot` columns of every query and key row are rot/2 pairs,
// and pair i of the token at position p turns by the angle p * frequency[i]:
//   (x, y) -> magnitude * (x cos - y sin, x sin + y cos),     the inverse with -sin.
// Both directions are this kernel: the rotation is linear and its transpose is the inverse (times the same magnitude).
//
// Angles.  p * frequency reaches 10^6 radians, of which float32 would keep one digit after the point: the product and its
// reduction to a fraction of a turn are float64 (a position and a pair once, for all heads), sine and cosine of what is
// left float32.  The products are float32 and rounded to bf16 once.
//
// What bounds it: bytes, 2 read and 2 written per element.  A thread keeps one slot (W pairs, or W columns that pass) of one token
// and walks over the heads with its sines and cosines in registers, kUnroll rows of loads in flight.  4 x 4096 tokens, H 32/32, d 128, one
// direction: 107 us, 5.0 TB/s.
#include "common.hpp"
#include "rope.hpp"
#include <algorithm>

namespace {

constexpr int kThreads = 256;
constexpr int kUnroll = 4;

template <int W> struct Vec;
template <> struct Vec<4> { typedef unsigned long long type; };
template <> struct Vec<1> { typedef unsigned short type; };

template <int W> union Bits {
  typename Vec<W>::type v;
  bf16_t x[W];
};

// The pairs of one row's slot, `valid` of them (interleaved: the last slot's columns from rot on pass, whatever their bits).
template <int W, bool INTERLEAVED>
DEVI void turn(const Bits<W>& a, const Bits<W>& b, Bits<W>& u, Bits<W>& w, const float (&c)[W], const float (&s)[W], int valid) {
  if constexpr (INTERLEAVED) {
#pragma unroll
    for (int j = 0; j < W; j += 2) {
      if (j / 2 >= valid) break;
      const float x = (float)a.x[j], y = (float)a.x[j + 1];
      u.x[j] = (bf16_t)(x * c[j / 2] - y * s[j / 2]);
      u.x[j + 1] = (bf16_t)(x * s[j / 2] + y * c[j / 2]);
    }
  } else {
#pragma unroll
    for (int j = 0; j < W; ++j) {
      const float x = (float)a.x[j], y = (float)b.x[j];
      u.x[j] = (bf16_t)(x * c[j] - y * s[j]);
      w.x[j] = (bf16_t)(x * s[j] + y * c[j]);
    }
  }
}

template <int W, bool INTERLEAVED>
__global__ __launch_bounds__(kThreads) void attn_rope_kernel(RopeArgs p) {
  // slots of a row: those with pairs (W pairs in the half layout, W / 2 in the interleaved one), then those that pass
  const int half = p.rot / 2;
  const int turning = INTERLEAVED ? (p.rot + W - 1) / W : half / W;
  const int slots = INTERLEAVED ? p.d / W : half / W + (p.d - p.rot) / W;
  const int per_block = kThreads / slots;
  const int slot = threadIdx.x % slots, local = threadIdx.x / slots;
  const long long token = (long long)blockIdx.x * per_block + local;
  if (local >= per_block || token >= (long long)p.B * p.N) return;
  const int b = (int)(token / p.N), n = (int)(token % p.N);
  const bool pairs = slot < turning;
  // columns of the slot: first (and, half layout, first + half)
  const int first = INTERLEAVED || pairs ? slot * W : p.rot + (slot - turning) * W;

  constexpr int PAIRS = INTERLEAVED ? W / 2 : W;
  const int pair0 = slot * PAIRS;
  const int valid = pairs ? min(PAIRS, half - pair0) : 0;
  float c[W], s[W];
  const double at = p.positions ? (double)p.positions[b * p.positions_stride + n] : (double)n;
#pragma unroll
  for (int j = 0; j < PAIRS; ++j) {
    if (j >= valid) break;
    const double turns = at * p.frequencies[pair0 + j] * 0.15915494309189533577;      // 1 / (2 pi)
    sincospif(2.0f * (float)(turns - rint(turns)), &s[j], &c[j]);
    c[j] *= p.magnitude;
    s[j] *= p.inverse ? -p.magnitude : p.magnitude;
  }

  const int heads = p.H + p.H_kv;
  const int j0 = blockIdx.y * p.heads_per_block, j1 = min(heads, j0 + p.heads_per_block);
  const bool two = !INTERLEAVED && pairs;
  auto address = [&](int j, long long& in, long long& out) -> const RopeSide& {
    const RopeSide& t = j < p.H ? p.q : p.k;
    const int h = j < p.H ? j : j - p.H;
    in = b * t.in_b + h * t.in_h + n * t.in_n + first;
    out = b * t.out_b + h * t.out_h + n * t.out_n + first;
    return t;
  };
  for (int j = j0; j < j1; j += kUnroll) {
    Bits<W> x[kUnroll], y[kUnroll];
#pragma unroll
    for (int i = 0; i < kUnroll; ++i) {
      if (j + i >= j1) break;
      long long in, out;
      const RopeSide& t = address(j + i, in, out);
      x[i].v = *reinterpret_cast<const typename Vec<W>::type*>(t.in + in);
      if (two) y[i].v = *reinterpret_cast<const typename Vec<W>::type*>(t.in + in + half);
    }
#pragma unroll
    for (int i = 0; i < kUnroll; ++i) {
      if (j + i >= j1) break;
      long long in, out;
      const RopeSide& t = address(j + i, in, out);
      Bits<W> u = x[i], w = y[i];
      if (pairs) turn<W, INTERLEAVED>(x[i], y[i], u, w, c, s, valid);
      *reinterpret_cast<typename Vec<W>::type*>(t.out + out) = u.v;
      if (two) *reinterpret_cast<typename Vec<W>::type*>(t.out + out + half) = w.v;
    }
  }
}

template <int W, bool INTERLEAVED> hipError_t launch(RopeArgs p, hipStream_t stream) {
  const int slots = INTERLEAVED ? p.d / W : p.rot / 2 / W + (p.d - p.rot) / W;
  const int per_block = kThreads / slots;
  const long long blocks = ((long long)p.B * p.N + per_block - 1) / per_block;
  if (!grid_fits(blocks, kThreads)) return hipErrorInvalidConfiguration;
  // Heads are shared out to several blocks until the grid fills the chip.  us, H 32/8, d 128, all heads in one block / as many blocks as 512 / 2048: 1 x 2048
  // tokens 23 / 10.5 / 9.9, 2 x 4096 - / 36 / 31, 1 x 512 19 / 4.4 / 5.0 (sines and cosines are formed again in each).
  const int heads = p.H + p.H_kv;
  const long long shares = std::min<long long>(heads, (2048 + blocks - 1) / blocks);
  p.heads_per_block = (int)((heads + shares - 1) / shares);
  const dim3 grid((unsigned)blocks, (unsigned)((heads + p.heads_per_block - 1) / p.heads_per_block));
  attn_rope_kernel<W, INTERLEAVED><<<grid, kThreads, 0, stream>>>(p);
  return hipGetLastError();
}

}  // namespace

hipError_t attn_rope_dispatch(const RopeArgs& p, int interleaved, hipStream_t stream) {
  // 8 bytes a load: 16 take twice the registers and half the threads (H 32/8, d 128: 8 x 4096 tokens 131 us, 125 so; one token 3.6 and 2.8), 2 bytes 158.
  if (interleaved) return launch<4, true>(p, stream);
  // half layout: both halves of a slot have to be aligned for the load
  if (p.rot / 2 % 4 == 0) return launch<4, false>(p, stream);
  return launch<1, false>(p, stream);
}
