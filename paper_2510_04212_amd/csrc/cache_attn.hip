// Attention over the 8-bit cache (attn_cache_fwd of include/attn.h) and the attention weight that each cached token got
// (attn_cache_weights).
//
// Products.  v_mfma_f32_16x16x32_bf16 on codes widened to bf16 in registers: an E4M3 number times a power of two is a bf16 number, and
// v_cvt_scalef32_pk_bf16_fp8 forms two of them in one instruction, so that scores and outputs need no scale factor of their own.
// Nothing passes through LDS on the way: the tile is computed transposed, S^T = K Q^T and O^T += V^T P^T, and both
// operands from the cache are 16 consecutive bytes per lane as they lie in memory (K in rows, V's blocks in columns):
//   tile i of 16 tokens (i = 0..3) of a block: the lane of row slot r holds token 16 (r / 4) + 4 i + (r % 4), columns 16 g .. + 15 of every 64,
//   so that S^T leaves lane group g with the 16 consecutive tokens 16 g .. 16 g + 15 of the block, which are the k-slots that V's
//   16 bytes of column 16 dt + r have: 8 of them make one instruction's, the other 8 the next one's.
// The row sum adds the float32 probabilities, not the rounded ones that are multiplied with V: LSE is exact to float32, as the weights
// exp(S - LSE) need it.
//
// Rows.  All query heads of a key/value head share its cache: their queries are one list of rows, row = query * group + head of the
// group, cut into tiles of M = 16 RT 4 / KW rows.  A work-group's four waves take KW shares of the key blocks of 4 / KW row groups.
#include "cache.hpp"
#include <algorithm>
#include <cmath>

namespace {

constexpr int kThreads = 256;

// d = 32 c + 8 half + ... of the columns: 16-byte chunks serve 64 columns (lane group g: 16 g ..), an 8-byte one the last 32 (8 g ..)
template <int D> struct Cols {
  static constexpr int C64 = D / 64, KC = D / 32;          // whole chunks, and instructions of K Q^T
  static constexpr bool ODD = D % 64 != 0;
};

DEVI bf16x8 widen8(unsigned lo, unsigned hi, float scale) {
  union { bf16x2 p[4]; bf16x8 v; } u;
  u.p[0] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, false);
  u.p[1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, true);
  u.p[2] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, false);
  u.p[3] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, true);
  return u.v;
}

// K codes of one lane for a block: 4 tiles of 16 tokens
template <int D> struct KCodes {
  u32x4 c[4][Cols<D>::C64 ? Cols<D>::C64 : 1];
  uint2 odd[4];
  // at: the block's first byte + the lane's offset (key_offset)
  DEVI void load(const unsigned char* at, int g) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
#pragma unroll
      for (int k = 0; k < Cols<D>::C64; ++k) c[i][k] = *reinterpret_cast<const u32x4*>(at + i * 4 * D + k * 64 + g * 16);
      if constexpr (Cols<D>::ODD) odd[i] = *reinterpret_cast<const uint2*>(at + i * 4 * D + Cols<D>::C64 * 64 + g * 8);
    }
  }
  // fragment k (of KC) of tile i
  DEVI bf16x8 frag(int i, int k, float scale) const {
    if (k < 2 * Cols<D>::C64) return (k & 1) ? widen8(c[i][k / 2][2], c[i][k / 2][3], scale) : widen8(c[i][k / 2][0], c[i][k / 2][1], scale);
    return widen8(odd[i].x, odd[i].y, scale);
  }
};
DEVI int key_offset(int r, int D) { return ((r >> 2) * 16 + (r & 3)) * D; }

// the columns of a query row that go with fragment k: 8 consecutive from here
template <int D> DEVI int query_column(int k, int g) {
  return k < 2 * Cols<D>::C64 ? (k >> 1) * 64 + g * 16 + (k & 1) * 8 : Cols<D>::C64 * 64 + g * 8;
}

DEVI float max_over_groups(float x) {
  unsigned u = __float_as_uint(x);
  auto a = __builtin_amdgcn_permlane32_swap(u, u, false, false);
  u = __float_as_uint(fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1])));
  a = __builtin_amdgcn_permlane16_swap(u, u, false, false);
  return fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
}
DEVI int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }
DEVI long long uniform(long long x) {
  return (long long)(((unsigned long long)(unsigned)uniform((int)(x >> 32)) << 32) | (unsigned)uniform((int)x));
}

// ---- The list of key blocks (cache_shares.hpp): sums of cost over runs of (sequence, tile) items, in LDS; before[k]: items 0 .. k run - 1.
struct Prefix {
  const Problem& q;
  int items, run;
  const long long* before;
  DEVI long long operator()(int item) const {
    const int k = item / run;
    long long s = before[k];
    for (int i = k * run; i < item; ++i) s += q.cost(i / q.tiles, i % q.tiles);
    return uniform(s);
  }
};
DEVI Prefix make_prefix(const Problem& q, int B, long long* before, long long* waves) {
  const int items = B * q.tiles, run = (items + kThreads - 1) / kThreads;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  long long x = 0;
  for (int i = tid * run; i < min(items, (tid + 1) * run); ++i) x += q.cost(i / q.tiles, i % q.tiles);
#pragma unroll
  for (int i = 1; i < 64; i <<= 1) {
    const long long y = __shfl_up(x, i);
    if (lane >= i) x += y;
  }
  if (lane == 63) waves[wave] = x;
  __syncthreads();
  for (int w = 0; w < wave; ++w) x += waves[w];
  before[tid + 1] = x;
  if (tid == 0) before[0] = 0;
  __syncthreads();
  return Prefix{q, items, run, before};
}

// ---- state of a wave's rows: lane (r, g) has row r of each of its RT tiles, output columns 16 dt + 4 g .. + 3
template <int D, int RT> struct Acc {
  f32x4 o[RT][D / 16];
  float l[RT];                    // sum of the probabilities of the lane's own tokens (of all four groups' after join_groups)
  float m[RT];                    // running maximum of the scores, in units of log 2; the same in the four groups
  DEVI void clear() {
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
      m[rt] = -INFINITY;
      l[rt] = 0.f;
#pragma unroll
      for (int dt = 0; dt < D / 16; ++dt) o[rt][dt] = f32x4{0, 0, 0, 0};
    }
  }
  DEVI void join_groups() {
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) l[rt] = sum_over_groups(l[rt]);
  }
  DEVI void scale(int rt, float by) {
    l[rt] *= by;
#pragma unroll
    for (int dt = 0; dt < D / 16; ++dt) o[rt][dt] *= by;
  }
};
template <int D, int RT, int KW> constexpr int kSlotFloats = (4 / KW) * RT * (D / 16 * 256 + 32);

template <int RT> struct RowsOf {
  int row[RT], query[RT], head[RT];       // row < 0: none
  int limit[RT];                          // tokens it sees; no row: all, so that it asks for no masking
  bool empty[RT];                         // a row whose output is 0
};

// O and LSE of row r of tile rt, from the sum and the maximum
template <int D, int RT>
DEVI void store_rows(const AttendArgs& p, const RowsOf<RT>& rows, int b, int h, Acc<D, RT>& a, int g) {
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    if (rows.row[rt] < 0) continue;
    const int head = h * p.group + rows.head[rt];
    unsigned short* to = p.O + b * p.o_sb + head * p.o_sh + rows.query[rt] * p.o_sn;
    const float l = a.l[rt];
    const Divisor by = make_divisor(l);
#pragma unroll
    for (int dt = 0; dt < D / 16; ++dt) {
      union { bf16x4 v; uint2 w; } u;
#pragma unroll
      for (int i = 0; i < 4; ++i) u.v[i] = rows.empty[rt] ? (bf16_t)0.f : (bf16_t)divide(a.o[rt][dt][i], by);
      *reinterpret_cast<uint2*>(to + dt * 16 + g * 4) = u.w;
    }
    if (g == 0)
      p.LSE[((size_t)b * p.H + head) * p.N + rows.query[rt]] = rows.empty[rt] ? -INFINITY : (a.m[rt] + log2f(l)) * 0.6931471805599453f;
  }
}
template <int RT>
DEVI void find_rows(RowsOf<RT>& rows, const AttendArgs& p, int b, int first, int r) {
  const int n = real_count(p.counts, b, p.N);
  const long long length = p.lengths[b];
  const long long all = max(0ll, min(length, (long long)p.cache.capacity));
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    const int row = first + rt * 16 + r;
    const bool there = row < p.N * p.group;
    const int query = there ? row / p.group : 0;
    rows.row[rt] = there ? row : -1;
    rows.query[rt] = query;
    rows.head[rt] = there ? row - query * p.group : 0;
    const long long seen = p.causal ? min(all, length - n + query + 1) : all;
    rows.empty[rt] = there && (query >= n || seen <= 0);
    rows.limit[rt] = there && query < n ? (int)max(0ll, seen) : 0x7fffffff;
  }
}

// bytes of w that are 0x7f or 0xff, E4M3's NaN: 0x80 in each of them
DEVI unsigned nan_codes(unsigned w) { return ((w & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u; }

// A masked block whose V holds NaN: 0 * NaN must not reach the rows that do not see that token.  The codes are cleared, and an
// output to which a row's visible tokens bring a NaN is made one: that count is a product, too, of ones.
template <int D, int RT>
DEVI void take_out_nan(Acc<D, RT>& a, u32x4 (&v)[D / 16], const RowsOf<RT>& rows, int t0, int g) {
  bf16x8 seen[RT][2];
#pragma unroll
  for (int rt = 0; rt < RT; ++rt)
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
      for (int e = 0; e < 8; ++e) seen[rt][j][e] = (bf16_t)(t0 + 16 * g + 8 * j + e < rows.limit[rt] ? 1.f : 0.f);
#pragma unroll
  for (int dt = 0; dt < D / 16; ++dt)
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const unsigned lo = nan_codes(v[dt][2 * j]), hi = nan_codes(v[dt][2 * j + 1]);
      bf16x8 bad;
#pragma unroll
      for (int e = 0; e < 8; ++e) bad[e] = (bf16_t)((((e < 4 ? lo : hi) >> (8 * (e & 3))) & 0x80u) ? 1.f : 0.f);
      v[dt][2 * j] &= ~((lo >> 7) * 0xffu);
      v[dt][2 * j + 1] &= ~((hi >> 7) * 0xffu);
#pragma unroll
      for (int rt = 0; rt < RT; ++rt) {
        f32x4 count{0, 0, 0, 0};
        count = mfma16(bad, seen[rt][j], count);
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (count[i] > 0.f) a.o[rt][dt][i] = NAN;
      }
    }
}

// One block of 64 tokens for a wave's rows.  masked (the same in all lanes): some row does not see all of it.  after_scores() is called when
// K's codes have been used.
template <int D, int RT, class F>
DEVI void block_step(Acc<D, RT>& a, const bf16x8 (&q)[RT][D / 32], const KCodes<D>& k, u32x4 (&v)[D / 16], float k_scale, float v_scale,
                     float scale_log2, const RowsOf<RT>& rows, bool masked, int t0, int g, F&& after_scores) {
  f32x4 s[RT][4];
#pragma unroll
  for (int rt = 0; rt < RT; ++rt)
#pragma unroll
    for (int i = 0; i < 4; ++i) s[rt][i] = f32x4{0, 0, 0, 0};
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int c = 0; c < D / 32; ++c) {
      const bf16x8 kf = k.frag(i, c, k_scale);
#pragma unroll
      for (int rt = 0; rt < RT; ++rt) s[rt][i] = mfma16(kf, q[rt][c], s[rt][i]);
    }
  after_scores();
  if (masked) {
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
      const int seen = rows.limit[rt] - t0 - 16 * g;
#pragma unroll
      for (int i = 0; i < 16; ++i)
        if (i >= seen) s[rt][i / 4][i % 4] = -INFINITY;
    }
    bool bad = false;
#pragma unroll
    for (int dt = 0; dt < D / 16; ++dt)
#pragma unroll
      for (int i = 0; i < 4; ++i) bad |= nan_codes(v[dt][i]) != 0;
    if (__any(bad)) take_out_nan<D, RT>(a, v, rows, t0, g);
  }
  bf16x8 pr[RT][2];
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    float most = -INFINITY;
#pragma unroll
    for (int i = 0; i < 16; ++i) most = fmaxf(most, s[rt][i / 4][i % 4]);
    const float m = fmaxf(a.m[rt], max_over_groups(most) * scale_log2);
    const float use = m == -INFINITY ? 0.f : m;            // nothing seen so far: exp2(-inf) = 0
    if (__any(m != a.m[rt])) {
      a.scale(rt, __builtin_amdgcn_exp2f(a.m[rt] - use));
      a.m[rt] = m;
    }
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float x = __builtin_amdgcn_exp2f(__builtin_fmaf(s[rt][2 * j + e / 4][e % 4], scale_log2, -use));
        a.l[rt] += x;
        pr[rt][j][e] = (bf16_t)x;
      }
  }
#pragma unroll
  for (int dt = 0; dt < D / 16; ++dt)
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const bf16x8 vf = widen8(v[dt][2 * j], v[dt][2 * j + 1], v_scale);
#pragma unroll
      for (int rt = 0; rt < RT; ++rt) a.o[rt][dt] = mfma16(vf, pr[rt][j], a.o[rt][dt]);
    }
}

// SPLIT: shares of the list of blocks; otherwise one segment per work-group (blockIdx: head, tile, sequence), nothing to merge.
template <int D, int RT, int KW, bool SPLIT>
__global__ __launch_bounds__(kThreads, D == 256 ? 1 : 2) void attn_cache_fwd_kernel(AttendArgs p, int tiles, int most_shares) {
  constexpr int RG = 4 / KW, M = 16 * RT * RG;
  __shared__ long long before[SPLIT ? kThreads + 1 : 1], wave_sums[4];
  __shared__ f32x4 joined[KW > 1 ? RG * KW / 2 * RT * (D / 16) * 64 : 1];
  __shared__ float joined_ml[KW > 1 ? 2 * 4 * RT * 16 : 1];
  const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6);
  const int r = lane & 15, g = lane >> 4;
  const int kw = wave % KW, rg = wave / KW;
  const Problem q{p.lengths, p.counts, p.cache.capacity, p.N, p.group, p.causal, tiles, M};
  const int nb = p.cache.capacity / kBlock;
  const float scale_log2 = p.scale * kLog2e;

  Segment seg;
  long long pos, end;
  int w = 0;
  if constexpr (SPLIT) {
    const Prefix f = make_prefix(q, p.B, before, wave_sums);
    const long long total = p.H_kv * f(f.items);
    const int shares = shares_of(total, most_shares, kLeastBlocks<KW>);
    w = share_of(blockIdx.x, shares);
    if (w < 0) return;
    pos = share_begin(total, shares, w);
    end = share_begin(total, shares, w + 1);
    seg = locate(q, f, p.B, p.H_kv, pos);
  } else {
    seg.b = blockIdx.z;
    seg.h = blockIdx.x;
    seg.t = blockIdx.y;
    seg.begin = 0;
    seg.blocks = q.blocks(seg.b, seg.t);
    seg.cost = max(1, seg.blocks);
    pos = 0;
    end = seg.cost;
  }

  while (true) {
    const int blk0 = (int)(pos - seg.begin), blk1 = (int)(min(end, seg.begin + seg.cost) - seg.begin);
    const int blk_end = min(blk1, seg.blocks);
    RowsOf<RT> rows;
    find_rows(rows, p, seg.b, seg.t * M + rg * RT * 16, r);
    int least = 0x7fffffff;
    bf16x8 qf[RT][D / 32];
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
      least = min(least, rows.limit[rt]);
      const unsigned short* from = p.Q.at + seg.b * p.Q.sb + (seg.h * p.group + rows.head[rt]) * p.Q.sh + rows.query[rt] * p.Q.sn;
#pragma unroll
      for (int c = 0; c < D / 32; ++c) qf[rt][c] = *reinterpret_cast<const bf16x8*>(from + query_column<D>(c, g));
    }
#pragma unroll
    for (int i = 1; i < 16; i <<= 1) least = min(least, __shfl_xor(least, i));
    least = uniform(least);

    Acc<D, RT> a;
    a.clear();
    const size_t bh = (size_t)seg.b * p.H_kv + seg.h;
    const unsigned char* K = p.cache.K + bh * p.cache.capacity * D + key_offset(r, D);
    const unsigned char* V = p.cache.V + bh * p.cache.capacity * D + r * kBlock + g * 16;
    const float* Ks = p.cache.K_scale + bh * nb;
    const float* Vs = p.cache.V_scale + bh * nb;
    int blk = blk0 + kw;
    KCodes<D> k;
    if (blk < blk_end) k.load(K + (size_t)blk * (kBlock * D), g);
    for (; blk < blk_end; blk += KW) {
      u32x4 v[D / 16];
#pragma unroll
      for (int dt = 0; dt < D / 16; ++dt)
        v[dt] = *reinterpret_cast<const u32x4*>(V + (size_t)blk * (kBlock * D) + dt * 16 * kBlock);
      const float k_scale = Ks[blk], v_scale = Vs[blk];
      block_step<D, RT>(a, qf, k, v, k_scale, v_scale, scale_log2, rows, blk * kBlock + kBlock > least, blk * kBlock, g, [&] {
        if (blk + KW < blk_end) k.load(K + (size_t)(blk + KW) * (kBlock * D), g);
      });
    }

    a.join_groups();
    // the KW waves of a row group: one maximum, then two halves at a time
    if constexpr (KW > 1) {
      if (g == 0)
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) joined_ml[(wave * RT + rt) * 16 + r] = a.m[rt];
      __syncthreads();
#pragma unroll
      for (int rt = 0; rt < RT; ++rt) {
        float m = -INFINITY;
#pragma unroll
        for (int o = 0; o < KW; ++o) m = fmaxf(m, joined_ml[((rg * KW + o) * RT + rt) * 16 + r]);
        a.scale(rt, __builtin_amdgcn_exp2f(a.m[rt] - (m == -INFINITY ? 0.f : m)));
        a.m[rt] = m;
      }
      float* joined_l = joined_ml + 4 * RT * 16;
#pragma unroll
      for (int half = KW / 2; half >= 1; half /= 2) {
        f32x4* mine = joined + (rg * (KW / 2) + (kw & (half - 1))) * RT * (D / 16) * 64 + lane;
        if (kw >= half && kw < 2 * half) {
#pragma unroll
          for (int rt = 0; rt < RT; ++rt) {
#pragma unroll
            for (int dt = 0; dt < D / 16; ++dt) mine[(rt * (D / 16) + dt) * 64] = a.o[rt][dt];
            if (g == 0) joined_l[(wave * RT + rt) * 16 + r] = a.l[rt];
          }
        }
        __syncthreads();
        if (kw < half) {
#pragma unroll
          for (int rt = 0; rt < RT; ++rt) {
#pragma unroll
            for (int dt = 0; dt < D / 16; ++dt) a.o[rt][dt] += mine[(rt * (D / 16) + dt) * 64];
            a.l[rt] += joined_l[((wave + half) * RT + rt) * 16 + r];
          }
        }
        __syncthreads();
      }
    }
    if (kw == 0) {
      if (!SPLIT || (blk0 == 0 && blk1 == seg.cost)) {
        store_rows<D, RT>(p, rows, seg.b, seg.h, a, g);
      } else {
        float* slot = p.partials + (size_t)(2 * w + (blk0 == 0 ? 1 : 0)) * kSlotFloats<D, RT, KW>;
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
          const int tile = rg * RT + rt;
#pragma unroll
          for (int dt = 0; dt < D / 16; ++dt) reinterpret_cast<f32x4*>(slot)[(tile * (D / 16) + dt) * 64 + lane] = a.o[rt][dt];
          float* ml = slot + RG * RT * (D / 16 * 256) + tile * 32;
          if (g == 0) {
            ml[r] = a.m[rt];
            ml[16 + r] = a.l[rt];
          }
        }
      }
    }
    if constexpr (!SPLIT) break;
    pos = seg.begin + blk1;
    if (pos >= end) break;
    next_segment(q, p.H_kv, seg);
  }
}

// Joins the parts of a segment that was split between shares: the work-group of the first share that begins inside it.  blockIdx.y is one row tile
// of 16 and COLS / 16 of the D / 16 column tiles; the four waves take every fourth part and join theirs in LDS.
template <int D, int RT, int KW, int DT>
__global__ __launch_bounds__(kThreads) void attn_cache_merge_kernel(AttendArgs p, int tiles, int most_shares) {
  constexpr int RG = 4 / KW, M = 16 * RT * RG, PARTS = D / 16 / DT;
  __shared__ long long before[kThreads + 1], wave_sums[4];
  __shared__ f32x4 joined[4][DT][64];
  __shared__ float joined_ml[2][4][16];
  const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6);
  const int r = lane & 15, g = lane >> 4;
  const Problem q{p.lengths, p.counts, p.cache.capacity, p.N, p.group, p.causal, tiles, M};
  const Prefix f = make_prefix(q, p.B, before, wave_sums);
  const long long total = p.H_kv * f(f.items);
  const int shares = shares_of(total, most_shares, kLeastBlocks<KW>);
  const int w = blockIdx.x + 1;
  if (w >= shares) return;
  const long long begin = share_begin(total, shares, w);
  const Segment seg = locate(q, f, p.B, p.H_kv, begin);
  if (seg.begin == begin || share_begin(total, shares, w - 1) > seg.begin) return;
  const long long seg_end = seg.begin + seg.cost;
  const int tile = blockIdx.y / PARTS, dt0 = (blockIdx.y % PARTS) * DT;

  f32x4 o[DT];
  float m = -INFINITY, l = 0.f;
#pragma unroll
  for (int i = 0; i < DT; ++i) o[i] = f32x4{0, 0, 0, 0};
  for (int part = wave;; part += 4) {
    const int share = w - 1 + part;
    if (share >= shares || share_begin(total, shares, share) >= seg_end) break;
    const float* slot = p.partials + (size_t)(2 * share + (part == 0 ? 1 : 0)) * kSlotFloats<D, RT, KW>;
    const float* ml = slot + RG * RT * (D / 16 * 256) + tile * 32;
    f32x4 x[DT];
#pragma unroll
    for (int i = 0; i < DT; ++i) x[i] = reinterpret_cast<const f32x4*>(slot)[(tile * (D / 16) + dt0 + i) * 64 + lane];
    const float mp = ml[r], lp = ml[16 + r];
    const float most = fmaxf(m, mp), use = most == -INFINITY ? 0.f : most;
    const float mine = __builtin_amdgcn_exp2f(m - use), theirs = __builtin_amdgcn_exp2f(mp - use);
    l = l * mine + lp * theirs;
#pragma unroll
    for (int i = 0; i < DT; ++i) o[i] = o[i] * mine + x[i] * theirs;
    m = most;
  }
  if (g == 0) { joined_ml[0][wave][r] = m; joined_ml[1][wave][r] = l; }
#pragma unroll
  for (int i = 0; i < DT; ++i) joined[wave][i][lane] = o[i];
  __syncthreads();
  if (wave != 0) return;
  float most = -INFINITY;
#pragma unroll
  for (int k = 0; k < 4; ++k) most = fmaxf(most, joined_ml[0][k][r]);
  const float use = most == -INFINITY ? 0.f : most;
  l = 0.f;
#pragma unroll
  for (int i = 0; i < DT; ++i) o[i] = f32x4{0, 0, 0, 0};
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const float by = __builtin_amdgcn_exp2f(joined_ml[0][k][r] - use);
    l += joined_ml[1][k][r] * by;
#pragma unroll
    for (int i = 0; i < DT; ++i) o[i] += joined[k][i][lane] * by;
  }
  RowsOf<1> rows;
  find_rows(rows, p, seg.b, seg.t * M + tile * 16, r);
  if (rows.row[0] < 0) return;
  const int head = seg.h * p.group + rows.head[0];
  unsigned short* to = p.O + seg.b * p.o_sb + head * p.o_sh + rows.query[0] * p.o_sn;
  const Divisor by = make_divisor(l);
#pragma unroll
  for (int i = 0; i < DT; ++i) {
    union { bf16x4 v; uint2 w; } u;
#pragma unroll
    for (int c = 0; c < 4; ++c) u.v[c] = rows.empty[0] ? (bf16_t)0.f : (bf16_t)divide(o[i][c], by);
    *reinterpret_cast<uint2*>(to + (dt0 + i) * 16 + g * 4) = u.w;
  }
  if (dt0 == 0 && g == 0)
    p.LSE[((size_t)seg.b * p.H + head) * p.N + rows.query[0]] = rows.empty[0] ? -INFINITY : (most + log2f(l)) * 0.6931471805599453f;
}

template <int D, int RT, int KW> hipError_t launch_fwd(const AttendArgs& p, const CacheForm& f, hipStream_t stream) {
  if (!f.split) {
    attn_cache_fwd_kernel<D, RT, KW, false><<<dim3((unsigned)p.H_kv, (unsigned)f.tiles, (unsigned)p.B), kThreads, 0, stream>>>(p, f.tiles, 0);
    return hipGetLastError();
  }
  attn_cache_fwd_kernel<D, RT, KW, true><<<(unsigned)((f.shares + 7) / 8 * 8), kThreads, 0, stream>>>(p, f.tiles, f.shares);
  if (const hipError_t e = hipGetLastError(); e != hipSuccess || f.shares == 1) return e;
  constexpr int DT = KW == 4 ? 2 : D / 16;
  attn_cache_merge_kernel<D, RT, KW, DT><<<dim3((unsigned)(f.shares - 1), (4 / KW) * RT * (D / 16 / DT)), kThreads, 0, stream>>>(p, f.tiles, f.shares);
  return hipGetLastError();
}
template <int D> hipError_t launch_fwd(const AttendArgs& p, hipStream_t stream) {
  const CacheForm f = cache_form(p.B, p.H, p.H_kv, p.N, D, p.cache.capacity);
  if (f.RT == 1) return launch_fwd<D, 1, 4>(p, f, stream);
  if (f.KW == 4) return launch_fwd<D, 2, 4>(p, f, stream);
  if (f.KW == 2) return launch_fwd<D, 2, 2>(p, f, stream);
  return launch_fwd<D, 2, 1>(p, f, stream);
}

// ---- weights.  The wave's tile is S^T again: lane (r, g) adds up exp(S - LSE) of row r of every row tile for the 16 tokens of its
// group, and the 16 lanes of a group are added at the end.  A block's tokens belong to one wave (WG = false: few row tiles) or to
// one work-group whose four waves take the row tiles in turn: no atomics.
template <int D, bool WG> __global__ __launch_bounds__(kThreads, 2) void attn_cache_weights_kernel(WeighArgs p) {
  __shared__ float joined[WG ? 4 : 1][kBlock];
  const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6);
  const int r = lane & 15, g = lane >> 4;
  const int nb = p.cache.capacity / kBlock;
  const int blk = WG ? blockIdx.x : blockIdx.x * 4 + wave, h = blockIdx.y, b = blockIdx.z;
  if (blk >= nb) return;
  const size_t bh = (size_t)b * p.H_kv + h;
  const int n = real_count(p.counts, b, p.N), rows = n * p.group;
  const long long length = p.lengths[b];
  const int all = (int)max(0ll, min(length, (long long)p.cache.capacity));
  const int t0 = blk * kBlock;
  float sum[16];
#pragma unroll
  for (int i = 0; i < 16; ++i) sum[i] = 0.f;
  if (t0 < all && rows > 0) {
    KCodes<D> k;
    k.load(p.cache.K + (bh * p.cache.capacity + t0) * D + key_offset(r, D), g);
    const float k_scale = p.cache.K_scale[bh * nb + blk], scale_log2 = p.scale * kLog2e;
    bf16x8 kf[4][D / 32];
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int c = 0; c < D / 32; ++c) kf[i][c] = k.frag(i, c, k_scale);
    // the first row that sees the block's first token
    const long long from = p.causal ? max(0ll, t0 - (length - n)) * p.group : 0;
    for (long long tile = from / 16 + (WG ? wave : 0); tile * 16 < rows; tile += WG ? 4 : 1) {
      const int row = (int)(tile * 16) + r;
      const bool there = row < rows;
      const int query = there ? row / p.group : 0, head = h * p.group + (there ? row - query * p.group : 0);
      const unsigned short* at = p.Q.at + b * p.Q.sb + head * p.Q.sh + query * p.Q.sn;
      bf16x8 qf[D / 32];
#pragma unroll
      for (int c = 0; c < D / 32; ++c) qf[c] = *reinterpret_cast<const bf16x8*>(at + query_column<D>(c, g));
      const float lse = p.LSE[((size_t)b * p.H + head) * p.N + query];
      const long long seen = p.causal ? min((long long)all, length - n + query + 1) : all;
      // a row that is not there, or sees nothing, adds nothing
      const int limit = there && lse != -INFINITY ? (int)max(0ll, seen) : 0;
      const float less = limit > 0 ? lse * kLog2e : 0.f;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        f32x4 s{0, 0, 0, 0};
#pragma unroll
        for (int c = 0; c < D / 32; ++c) s = mfma16(kf[i][c], qf[c], s);
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          const float x = __builtin_amdgcn_exp2f(__builtin_fmaf(s[c], scale_log2, -less));
          sum[4 * i + c] += t0 + 16 * g + 4 * i + c < limit ? x : 0.f;
        }
      }
    }
  }
  float mine = 0.f;                                        // of token 16 g + r
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    float x = sum[i];
#pragma unroll
    for (int d = 1; d < 16; d <<= 1) x += __shfl_xor(x, d);
    mine = r == i ? x : mine;
  }
  if constexpr (WG) {
    joined[wave][lane] = mine;
    __syncthreads();
    if (wave != 0) return;
    mine = joined[0][lane] + joined[1][lane] + joined[2][lane] + joined[3][lane];
  }
  const int t = t0 + lane;
  const size_t at = bh * p.cache.capacity + t;
  // a token of this call's has no weight yet
  p.out[at] = t >= all ? 0.f : (p.in && t < length - n ? p.in[at] : 0.f) + mine;
}

template <int D> hipError_t launch_weights(const WeighArgs& p, hipStream_t stream) {
  const unsigned nb = (unsigned)(p.cache.capacity / kBlock);
  if ((long long)p.N * p.group <= 64)
    attn_cache_weights_kernel<D, false><<<dim3((nb + 3) / 4, (unsigned)p.H_kv, (unsigned)p.B), kThreads, 0, stream>>>(p);
  else
    attn_cache_weights_kernel<D, true><<<dim3(nb, (unsigned)p.H_kv, (unsigned)p.B), kThreads, 0, stream>>>(p);
  return hipGetLastError();
}

}  // namespace

size_t attn_cache_fwd_partial_bytes(int B, int H, int H_kv, int N, int d, int capacity) {
  const CacheForm f = cache_form(B, H, H_kv, N, d, capacity);
  return f.split && f.shares > 1 ? 2 * (size_t)f.shares * f.slot_floats(d) * sizeof(float) : 0;
}

hipError_t attn_cache_fwd_dispatch(const AttendArgs& p, int d, hipStream_t stream) {
  switch (d) {
    case 32: return launch_fwd<32>(p, stream);
    case 64: return launch_fwd<64>(p, stream);
    case 96: return launch_fwd<96>(p, stream);
    case 128: return launch_fwd<128>(p, stream);
    default: return launch_fwd<256>(p, stream);
  }
}

hipError_t attn_cache_weights_dispatch(const WeighArgs& p, int d, hipStream_t stream) {
  switch (d) {
    case 32: return launch_weights<32>(p, stream);
    case 64: return launch_weights<64>(p, stream);
    case 96: return launch_weights<96>(p, stream);
    case 128: return launch_weights<128>(p, stream);
    default: return launch_weights<256>(p, stream);
  }
}
