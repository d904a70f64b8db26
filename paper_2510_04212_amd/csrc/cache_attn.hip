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
// exp(S - LSE) need it.  P is rounded to bf16 for that product because the matrix unit takes 16-bit operands: O's relative error (root mean square, against
// 64 bits) is 0.0022, and 0.0017, O's own rounding, with P in float32, which would take a second product of every tile.
//
// Rows.  All query heads of a key/value head share its cache: their queries are one list of rows, row = query * group + head of the
// group, cut into tiles of M = 16 RT 4 / KW rows.  A work-group's four waves take KW shares of the key blocks of 4 / KW row groups.
#include "cache.hpp"
#include <algorithm>
#include <cmath>

namespace {

constexpr int kThreads = 256;
typedef __attribute__((ext_vector_type(2))) unsigned int u32x2;

// d = 32 c + 8 half + ... of the columns: 16-byte chunks serve 64 columns (lane group g: 16 g ..), an 8-byte one the last 32 (8 g ..)
template <int D> struct Cols {
  static constexpr int C64 = D / 64;       // whole chunks
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

// Codes of one lane for a block, 16 bytes (or 8: the last 32 columns of d = 32, 96) each: K's of tile i, columns 64 c ..; V's of column tile dt.
// From memory into registers: every wave reads its own blocks.  K + V: 2 d registers / 8.
template <int D> struct KCodes {
  u32x4 c[4][Cols<D>::C64 ? Cols<D>::C64 : 1];
  u32x2 odd[4];
  // block: its first byte, the same in all lanes; at: the lane's offset
  DEVI void load(const unsigned char* block, unsigned at, unsigned at_odd) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
#pragma unroll
      for (int k = 0; k < Cols<D>::C64; ++k) c[i][k] = *reinterpret_cast<const u32x4*>(block + at + (i * 4 * D + k * 64));
      if constexpr (Cols<D>::ODD) odd[i] = *reinterpret_cast<const u32x2*>(block + at_odd + (i * 4 * D + Cols<D>::C64 * 64));
    }
  }
};
template <int D> struct VCodes {
  u32x4 c[D / 16];
  DEVI void load(const unsigned char* block, unsigned at) {
#pragma unroll
    for (int dt = 0; dt < D / 16; ++dt) c[dt] = *reinterpret_cast<const u32x4*>(block + at + dt * 1024);
  }
};
// From LDS, where a block's codes are shared by the four waves of a work-group.  Pieces of 1 KB, one transfer instruction each: 16 rows (tokens of
// a tile, or columns of V) x 64 bytes, the four 16-byte chunks of row r permuted by slot_mask(r / 4) (common.hpp: 16 lanes reading
// chunk g of 16 rows then meet all banks once); two tiles' 32 bytes a row for the last columns of d = 32, 96.
template <int D> struct Staged {
  static constexpr int KP = 4 * Cols<D>::C64 + (Cols<D>::ODD ? 2 : 0), PIECES = KP + D / 16;
  static constexpr int kBytes = PIECES * 1024;
  // the byte of the block that lane `lane` of piece i fetches, K's (i < KP) and V's
  static DEVI unsigned source(int i, int lane) {
    if (i < 4 * Cols<D>::C64) {
      const int r = lane >> 2, tile = i / (Cols<D>::C64 ? Cols<D>::C64 : 1), c = i % (Cols<D>::C64 ? Cols<D>::C64 : 1);
      return (unsigned)(((r >> 2) * 16 + tile * 4 + (r & 3)) * D + c * 64 + (((lane & 3) ^ slot_mask(r >> 2)) << 4));
    }
    if (i < KP) {
      const int r = (lane >> 1) & 15, tile = 2 * (i - 4 * Cols<D>::C64) + (lane >> 5);
      return (unsigned)(((r >> 2) * 16 + tile * 4 + (r & 3)) * D + Cols<D>::C64 * 64 + ((lane & 1) << 4));
    }
    const int r = lane >> 2;
    return (unsigned)(((i - KP) * 16 + r) * kBlock + (((lane & 3) ^ slot_mask(r >> 2)) << 4));
  }
};
typedef __attribute__((address_space(3))) const u32x4 lds_u32x4;
typedef __attribute__((address_space(3))) const u32x2 lds_u32x2;
// at, at_odd: LDS addresses, the buffer's + the lane's
template <int D> DEVI void read_staged(KCodes<D>& k, int at, int at_odd) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
#pragma unroll
    for (int c = 0; c < Cols<D>::C64; ++c) k.c[i][c] = *reinterpret_cast<lds_u32x4*>((unsigned long)(unsigned)(at + (i * Cols<D>::C64 + c) * 1024));
    if constexpr (Cols<D>::ODD) k.odd[i] = *reinterpret_cast<lds_u32x2*>((unsigned long)(unsigned)(at_odd + 4 * Cols<D>::C64 * 1024 + i * 512));
  }
}
template <int D> DEVI void read_staged(VCodes<D>& v, int at) {
#pragma unroll
  for (int dt = 0; dt < D / 16; ++dt) v.c[dt] = *reinterpret_cast<lds_u32x4*>((unsigned long)(unsigned)(at + (Staged<D>::KP + dt) * 1024));
}
// 64 lanes' 16 bytes each from block + at into LDS at `to` .. + 1023; `block` and `to` the same in all lanes.  Inline assembly as in common.hpp's
// TileLoader, and for its reasons; waited for with wait_vmem().
DEVI void fetch_piece(const unsigned char* block, unsigned at, unsigned to) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" : : "s"(to), "v"(at), "s"(block) : "m0");
}
DEVI bf16x8 key_frag(const u32x4& w, int half, float scale) { return widen8(w[2 * half], w[2 * half + 1], scale); }

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

// ---- The list of segments (cache_shares.hpp): every thread sums up the units of a run of (sequence, tile) items, for one head; a scan over the threads.
struct Runs {
  int before[kThreads + 1];                // units in front of thread t's run
  int waves[kThreads / 64];
  Segment segment;
};
// units of all items
DEVI int scan_units(const Problem& q, int items, int run, Runs& runs) {
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  int x = 0;
  for (int i = tid * run; i < min(items, (tid + 1) * run); ++i) x += q.cost(i / q.tiles, i % q.tiles);
  x = (int)sum_to_lane((unsigned)x);
  if (lane == 63) runs.waves[wave] = x;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < kThreads / 64 - 1; ++w) x += w < wave ? runs.waves[w] : 0;
  runs.before[tid + 1] = x;
  if (tid == 0) runs.before[0] = 0;
  __syncthreads();
  return uniform(runs.before[kThreads]);
}
// The segment of unit `pos`, found by the thread whose run holds it.
DEVI Segment find_segment(const Problem& q, int B, int H_kv, int run, int pos, Runs& runs) {
  auto units_before = [&](int item) {      // in front of an item
    int x = runs.before[item / run];
    for (int i = item / run * run; i < item; ++i) x += q.cost(i / q.tiles, i % q.tiles);
    return x;
  };
  const int tid = threadIdx.x;
  int b = -1, first = 0, each = 0, here = runs.before[tid];
  for (int i = tid * run; i < min(B * q.tiles, (tid + 1) * run); ++i) {
    if (i / q.tiles != b) {
      b = i / q.tiles;
      first = units_before(b * q.tiles);
      each = units_before((b + 1) * q.tiles) - first;
    }
    Segment s;
    if (locate(q, b, i % q.tiles, first, each, here - first, H_kv, pos, &s)) runs.segment = s;
    here += q.cost(b, i % q.tiles);
  }
  __syncthreads();
  Segment s = runs.segment;
  s.b = uniform(s.b);
  s.h = uniform(s.h);
  s.t = uniform(s.t);
  s.begin = uniform(s.begin);
  return s;
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

// A row of the list: which query and head it is, and how many tokens it sees.
struct Row {
  int query, head, limit;
  bool there, empty;                    // empty: its output is 0
};
DEVI Row find_row(const AttendArgs& p, int b, int row) {
  const int n = real_count(p.counts, b, p.N);
  const long long length = p.lengths[b];
  const long long all = max(0ll, min(length, (long long)p.cache.capacity));
  Row x;
  x.there = row < p.N * p.group;
  x.query = x.there ? row / p.group : 0;
  x.head = x.there ? row - x.query * p.group : 0;
  const long long seen = p.causal ? min(all, length - n + x.query + 1) : all;
  x.empty = x.query >= n || seen <= 0;
  x.limit = x.there && x.query < n ? (int)max(0ll, seen) : 0x7fffffff;       // a row that nobody asks for needs no masking
  return x;
}
// O and LSE of a row: DT column tiles from dt0 on
template <int DT>
DEVI void store_row(const AttendArgs& p, const Row& x, int b, int h, const f32x4* o, float m, float l, int dt0, int g) {
  if (!x.there) return;
  const int head = h * p.group + x.head;
  unsigned short* to = p.O + b * p.o_sb + head * p.o_sh + x.query * p.o_sn + dt0 * 16 + g * 4;
  const Divisor by = make_divisor(l);
#pragma unroll
  for (int i = 0; i < DT; ++i) {
    union { bf16x4 v; u32x2 w; } u;
#pragma unroll
    for (int c = 0; c < 4; ++c) u.v[c] = x.empty ? (bf16_t)0.f : (bf16_t)divide(o[i][c], by);
    *reinterpret_cast<u32x2*>(to + i * 16) = u.w;
  }
  if (dt0 == 0 && g == 0) p.LSE[((size_t)b * p.H + head) * p.N + x.query] = x.empty ? -INFINITY : (m + log2f(l)) * 0.6931471805599453f;
}

// bytes of w that are 0x7f or 0xff, E4M3's NaN: 0x80 in each of them
DEVI unsigned nan_codes(unsigned w) { return ((w & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u; }

// A masked block whose V holds NaN: 0 * NaN must not reach the rows that do not see that token.  The codes are made 0, and an
// output to which a row's visible tokens bring a NaN is made one: that count is a product, too, of ones.
template <int D, int RT>
DEVI void take_out_nan(Acc<D, RT>& a, VCodes<D>& v, const int (&limit)[RT], int t0, int g) {
  int seen[RT];
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    seen[rt] = limit[rt] - t0 - 16 * g;
    settle(seen[rt]);                      // (a copy: or the masks are formed for both uses at once, and kept)
  }
#pragma unroll
  for (int dt = 0; dt < D / 16; ++dt)
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const unsigned lo = nan_codes(v.c[dt][2 * j]), hi = nan_codes(v.c[dt][2 * j + 1]);
      v.c[dt][2 * j] &= ~((lo >> 7) * 0xffu);
      v.c[dt][2 * j + 1] &= ~((hi >> 7) * 0xffu);
      bf16x8 ones;
#pragma unroll
      for (int e = 0; e < 8; ++e) ones[e] = (bf16_t)((((e < 4 ? lo : hi) >> (8 * (e & 3))) & 0x80u) ? 1.f : 0.f);
#pragma unroll
      for (int rt = 0; rt < RT; ++rt) {
        bf16x8 sees;
#pragma unroll
        for (int e = 0; e < 8; ++e) sees[e] = (bf16_t)(8 * j + e < seen[rt] ? 1.f : 0.f);
        const f32x4 count = mfma16(ones, sees, f32x4{0, 0, 0, 0});
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (count[i] > 0.f) a.o[rt][dt][i] = NAN;
      }
    }
}

// One block of 64 tokens for a wave's rows.  masked (the same in all lanes): some row does not see all of it.  after_scores() is called when
// K's codes have been used.
//
// The maximum that probabilities are taken relative to is let fall behind the true one by up to kSlack (a factor of 2^kSlack, harmless in float32 and
// bf16 alike), so that the accumulators are hardly ever rescaled.
//
// Of the two waves that share a SIMD, the one that multiplies goes first, so that the other's softmax fills in (2048 queries over 16384 tokens, H 32/8,
// d 128: 534 -> 493 us; 16 queries of 64 sequences of 4300: 126 -> 121; d = 64, 4096 queries of 4 sequences: 441 -> 413; with one wave a SIMD, d = 256, even:
// not there).
constexpr float kSlack = 8.f;
template <int D, int RT, class F>
DEVI void block_step(Acc<D, RT>& a, const bf16x8 (&q)[RT][D / 32], const KCodes<D>& k, VCodes<D>& v, float k_scale, float v_scale, float scale_log2,
                     const int (&limit)[RT], bool masked, int t0, int g, F&& after_scores) {
  constexpr bool kMultipliesFirst = D < 256;
  f32x4 s[RT][4];
#pragma unroll
  for (int rt = 0; rt < RT; ++rt)
#pragma unroll
    for (int i = 0; i < 4; ++i) s[rt][i] = f32x4{0, 0, 0, 0};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
#pragma unroll
    for (int c = 0; c < Cols<D>::C64; ++c) {
      const u32x4 w = k.c[i][c];
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        const bf16x8 kf = key_frag(w, half, k_scale);
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) s[rt][i] = mfma16(kf, q[rt][2 * c + half], s[rt][i]);
      }
    }
    if constexpr (Cols<D>::ODD) {
      const u32x2 w = k.odd[i];
      const bf16x8 kf = widen8(w.x, w.y, k_scale);
#pragma unroll
      for (int rt = 0; rt < RT; ++rt) s[rt][i] = mfma16(kf, q[rt][D / 32 - 1], s[rt][i]);
    }
  }
  if (kMultipliesFirst) __builtin_amdgcn_s_setprio(0);
  after_scores();
  if (masked) {
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
      const int seen = limit[rt] - t0 - 16 * g;
#pragma unroll
      for (int i = 0; i < 16; ++i)
        if (i >= seen) s[rt][i / 4][i % 4] = -INFINITY;
    }
    if (v_scale < 0.f) take_out_nan<D, RT>(a, v, limit, t0, g);          // V's scale is negative: a code of the block is NaN
  }
  v_scale = __builtin_fabsf(v_scale);
  bf16x8 pr[RT][2];
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    float most = s[rt][0][0];
#pragma unroll
    for (int i = 1; i < 16; ++i) most = fmaxf(most, s[rt][i / 4][i % 4]);
    most = max_over_groups(most) * scale_log2;
    if (__any(most > a.m[rt] + kSlack)) {
      const float m = most > a.m[rt] + kSlack ? most : a.m[rt];
      a.scale(rt, __builtin_amdgcn_exp2f(a.m[rt] - (m == -INFINITY ? 0.f : m)));
      a.m[rt] = m;
    }
    const float use = a.m[rt] == -INFINITY ? 0.f : a.m[rt];            // nothing seen so far: exp2(-inf) = 0
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float x = __builtin_amdgcn_exp2f(__builtin_fmaf(s[rt][2 * j + e / 4][e % 4], scale_log2, -use));
        a.l[rt] += x;
        pr[rt][j][e] = (bf16_t)x;
      }
  }
  if (kMultipliesFirst) __builtin_amdgcn_s_setprio(1);
#pragma unroll
  for (int dt = 0; dt < D / 16; ++dt) {
    const u32x4 w = v.c[dt];
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const bf16x8 vf = widen8(w[2 * j], w[2 * j + 1], v_scale);
#pragma unroll
      for (int rt = 0; rt < RT; ++rt) a.o[rt][dt] = mfma16(vf, pr[rt][j], a.o[rt][dt]);
    }
  }
}

// SPLIT: shares of the list of blocks; otherwise one segment per work-group (blockIdx: head, tile, sequence), nothing to merge.
//
// KW = 4, few rows: bound by bytes; every wave reads blocks of its own straight into registers, K's a block ahead (one token of 64 sequences of 4300, H 32/8, d
// 128: 100 us, 5.6 TB/s).  KW = 1, many rows: bound by
// the vector and matrix units; the four waves share a block through LDS, filled by asynchronous transfers a block ahead (three blocks ahead, in four
// buffers: 16 queries of 64 sequences of 4300 tokens, H 32/8, d 128, 139 us; one ahead, in two: 125.  2048 queries over 16384: 636 and 620; these with the
// loop of that time, which takes 121 and 493 now).
template <int D, int RT, int KW, bool SPLIT>
__global__ __launch_bounds__(kThreads, D == 256 ? 1 : 2) void attn_cache_fwd_kernel(AttendArgs p, int tiles, int most_shares, bool notes_by_segment) {
  constexpr int RG = 4 / KW, M = 16 * RT * RG;
  static_assert(KW == 1 || KW == 4, "the four waves have rows of their own, or blocks");
  __shared__ Runs runs;
  __shared__ f32x4 joined[KW == 4 ? 4 * RT * (D / 16) * 64 : 1];         // [wave][RT][D / 16][lane]
  __shared__ float joined_m[KW == 4 ? 4 * RT * 16 : 1], joined_l[KW == 4 ? 4 * RT * 16 : 1];
  __shared__ __attribute__((aligned(1024))) char staged[KW == 1 ? 2 * Staged<D>::kBytes : 16];
  const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6);
  const int r = lane & 15, g = lane >> 4;
  const int kw = wave % KW, rg = wave / KW;
  const Problem q{p.lengths, p.counts, p.cache.capacity, p.N, p.group, p.causal, tiles, M};
  const int nb = p.cache.capacity / kBlock;
  const float scale_log2 = p.scale * kLog2e;

  Segment seg;
  int pos, end, w = 0;
  Shares all{1, 0, 0};
  Join* notes = reinterpret_cast<Join*>(p.partials);
  if constexpr (SPLIT) {
    const int items = p.B * tiles, run = (items + kThreads - 1) / kThreads;
    all = shares_of(p.H_kv * scan_units(q, items, run, runs), most_shares, kLeastUnits<KW>);
    w = share_of(blockIdx.x, all.number);
    if (w < 0) return;
    pos = uniform(all.begin(w));
    end = uniform(all.begin(w + 1));
    seg = find_segment(q, p.B, p.H_kv, run, pos, runs);
    if (tid == 0 && !notes_by_segment) notes[w] = note_of_share(all, w, seg, p.H_kv, tiles);
  } else {
    seg.b = blockIdx.z;
    seg.h = blockIdx.x;
    seg.t = blockIdx.y;
    seg.begin = 0;
    seg.blocks = q.blocks(seg.b, seg.t);
    pos = 0;
    end = seg.end();
  }
  seg.blocks = uniform(seg.blocks);

  while (true) {
    const int to = min(end, seg.end());
    if (SPLIT && notes_by_segment && tid == 0 && pos == seg.begin)
      notes[segment_number(seg, p.H_kv, tiles)] = note_of_segment(all, w, seg, p.H_kv, tiles);
    const int b = seg.b, h = seg.h, first_row = seg.t * M + rg * RT * 16;
    const int blk0 = seg.block_at(pos), blk_end = seg.block_at(to);
    const size_t bh = (size_t)b * p.H_kv + h;
    const unsigned char* K = p.cache.K + bh * p.cache.capacity * D;
    const unsigned char* V = p.cache.V + bh * p.cache.capacity * D;
    const float* Ks = p.cache.K_scale + bh * nb;
    const float* Vs = p.cache.V_scale + bh * nb;
    // a wave of few rows: its first block is on its way while the queries are looked for
    const unsigned at = ((r >> 2) * 16 + (r & 3)) * D + g * 16, at_odd = ((r >> 2) * 16 + (r & 3)) * D + g * 8, at_v = r * kBlock + g * 16;
    KCodes<D> k;
    float k_scale = 0.f, next_v = 0.f;     // loaded with K's codes: a load behind V's would have V waited for
    auto load_key = [&](int blk) {
      if (blk >= blk_end) return;
      k_scale = Ks[blk];
      next_v = Vs[blk];
      k.load(K + (size_t)blk * (kBlock * D), at, at_odd);
    };
    if constexpr (KW == 4) load_key(blk0 + kw);
    int least = 0x7fffffff, limit[RT];
    bf16x8 qf[RT][D / 32];
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
      const Row x = find_row(p, b, first_row + rt * 16 + r);
      limit[rt] = x.limit;
      least = min(least, x.limit);
      const unsigned short* from = p.Q.at + b * p.Q.sb + (h * p.group + x.head) * p.Q.sh + x.query * p.Q.sn;
#pragma unroll
      for (int c = 0; c < D / 32; ++c) qf[rt][c] = *reinterpret_cast<const bf16x8*>(from + query_column<D>(c, g));
    }
#pragma unroll
    for (int i = 1; i < 16; i <<= 1) least = min(least, __shfl_xor(least, i));
    least = uniform(least);

    Acc<D, RT> a;
    a.clear();
    if constexpr (KW == 1) {
      // a wave fetches every fourth piece; PIECES is a multiple of 4
      constexpr int MINE = Staged<D>::PIECES / 4;
      const unsigned buffers = uniform(lds_address(staged));
      unsigned from[MINE];
#pragma unroll
      for (int i = 0; i < MINE; ++i) from[i] = Staged<D>::source(wave + 4 * i, lane);
      auto fetch = [&](int blk, int buffer) {
#pragma unroll
        for (int i = 0; i < MINE; ++i) {
          const int piece = wave + 4 * i;
          fetch_piece((piece < Staged<D>::KP ? K : V) + (size_t)blk * (kBlock * D), from[i], buffers + buffer * Staged<D>::kBytes + piece * 1024);
        }
      };
      const int in_piece = r * 64 + ((g ^ slot_mask(r >> 2)) << 4), in_odd = r * 32 + g * 8;
      const bool rows_here = first_row < p.N * p.group;
      // Scales: 64 blocks' at a time, one in each lane.
      float k_scales = 0.f, v_scales = 0.f;
      auto load_scales = [&](int blk) {
        const int mine = min(blk + lane, nb - 1);
        k_scales = Ks[mine];
        v_scales = Vs[mine];
        settle(k_scales);
        settle(v_scales);
      };
      __syncthreads();                                     // nobody reads the last segment's blocks any more
      if (blk0 < blk_end) {
        fetch(blk0, 0);
        load_scales(blk0);
      }
      // What the compiler has loaded is settled here: waits that it placed inside the loop, where it knows nothing of the transfers, would wait for these.
#pragma unroll
      for (int rt = 0; rt < RT; ++rt)
#pragma unroll
        for (int c = 0; c < D / 32; ++c) settle(qf[rt][c]);
      int buffer = 0;
      for (int blk = blk0; blk < blk_end; ++blk) {
        wait_vmem();
        __syncthreads();                                   // this block has landed for all waves, and all have read the one before
        if (blk + 1 < blk_end) fetch(blk + 1, buffer ^ 1);
        if (rows_here) {
          if (blk > blk0 && ((blk - blk0) & 63) == 0) load_scales(blk);
          const float ks = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(k_scales), (blk - blk0) & 63));
          const float vs = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(v_scales), (blk - blk0) & 63));
          const int base = (int)buffers + buffer * Staged<D>::kBytes;
          VCodes<D> v;
          read_staged<D>(k, base + in_piece, base + in_odd);
          block_step<D, RT>(a, qf, k, v, ks, vs, scale_log2, limit, blk * kBlock + kBlock > least, blk * kBlock, g,
                            [&] { read_staged<D>(v, base + in_piece); });
        }
        buffer ^= 1;
      }
    } else {
      for (int blk = blk0 + kw; blk < blk_end; blk += KW) {
        VCodes<D> v;
        v.load(V + (size_t)blk * (kBlock * D), at_v);
        block_step<D, RT>(a, qf, k, v, k_scale, next_v, scale_log2, limit, blk * kBlock + kBlock > least, blk * kBlock, g,
                          [&] { load_key(blk + KW); });
      }
    }

    a.join_groups();
    const bool whole = !SPLIT || (pos == seg.begin && to == seg.end());
    float* slot = p.partials + most_shares * (sizeof(Join) / sizeof(float)) + (size_t)(2 * w + (pos == seg.begin ? 1 : 0)) * kSlotFloats<D, RT, KW>;
    // O and LSE of a finished row, or this part of them: column tiles dt0 .. dt0 + DT - 1 of row tile `tile`
    auto put = [&](auto DT, int tile, const f32x4* o, float m, float l, int dt0) {
      if (whole) {
        store_row<DT>(p, find_row(p, b, seg.t * M + tile * 16 + r), b, h, o, m, l, dt0, g);
        return;
      }
#pragma unroll
      for (int i = 0; i < DT; ++i) reinterpret_cast<f32x4*>(slot)[(tile * (D / 16) + dt0 + i) * 64 + lane] = o[i];
      float* ml = slot + RG * RT * (D / 16 * 256) + tile * 32;
      if (g == 0 && dt0 == 0) {
        ml[r] = m;
        ml[16 + r] = l;
      }
    };
    if constexpr (KW == 1) {
#pragma unroll
      for (int rt = 0; rt < RT; ++rt) put(std::integral_constant<int, D / 16>{}, rg * RT + rt, a.o[rt], a.m[rt], a.l[rt], 0);
    } else {
      // Four waves have four sums of the same rows: all go to LDS as they are, and each wave joins RT * D / 64 of the RT * D / 16 tiles
      // (d = 32: the first two).
      __syncthreads();                                     // the last segment's have been read
#pragma unroll
      for (int rt = 0; rt < RT; ++rt) {
#pragma unroll
        for (int dt = 0; dt < D / 16; ++dt) joined[((wave * RT + rt) * (D / 16) + dt) * 64 + lane] = a.o[rt][dt];
        if (g == 0) {
          joined_m[(wave * RT + rt) * 16 + r] = a.m[rt];
          joined_l[(wave * RT + rt) * 16 + r] = a.l[rt];
        }
      }
      __syncthreads();
      constexpr int EACH = D / 16 >= 4 ? D / 16 / 4 : 1, REST = D / 16 - 4 * EACH;       // column tiles per wave (d = 96: 1, and 2 that are left)
#pragma unroll
      for (int rt = 0; rt < RT; ++rt) {
        float by[4], m = -INFINITY, l = 0.f;
#pragma unroll
        for (int x = 0; x < 4; ++x) m = fmaxf(m, joined_m[(x * RT + rt) * 16 + r]);
        const float use = m == -INFINITY ? 0.f : m;
#pragma unroll
        for (int x = 0; x < 4; ++x) {
          by[x] = __builtin_amdgcn_exp2f(joined_m[(x * RT + rt) * 16 + r] - use);
          l += joined_l[(x * RT + rt) * 16 + r] * by[x];
        }
        auto join = [&](auto DT, int dt0) {
          f32x4 o[DT];
#pragma unroll
          for (int i = 0; i < DT; ++i) {
            o[i] = f32x4{0, 0, 0, 0};
#pragma unroll
            for (int x = 0; x < 4; ++x) o[i] += joined[((x * RT + rt) * (D / 16) + dt0 + i) * 64 + lane] * by[x];
          }
          put(DT, rt, o, m, l, dt0);
        };
        if (wave * EACH < D / 16) join(std::integral_constant<int, EACH>{}, wave * EACH);
        if (REST > 0 && wave < REST) join(std::integral_constant<int, 1>{}, 4 * EACH + wave);
      }
    }
    if constexpr (!SPLIT) break;
    pos = to;
    if (pos >= end) break;
    next_segment(q, p.H_kv, seg);
    seg.blocks = uniform(seg.blocks);
  }
}

// Joins the parts of the segments that were split between shares.  blockIdx.x is a note; blockIdx.y one row tile of 16 and DT of the D / 16 column
// tiles; the NW waves take every NW-th part, kAhead of them in flight, and join theirs in LDS.
template <int D, int RT, int KW, int NW, int DT>
__global__ __launch_bounds__(64 * NW) void attn_cache_merge_kernel(AttendArgs p, int tiles, int shares_room, bool notes_by_segment) {
  constexpr int RG = 4 / KW, M = 16 * RT * RG, PARTS = D / 16 / DT, kAhead = NW == 16 ? 8 : DT <= 8 ? 2 : 1;
  __shared__ f32x4 joined[NW][DT][64];
  __shared__ float joined_ml[2][NW][16];
  const int lane = threadIdx.x & 63, wave = uniform((int)(threadIdx.x >> 6));
  const int r = lane & 15, g = lane >> 4;
  const int note = blockIdx.x + (notes_by_segment ? 0 : 1);
  const Join* notes = reinterpret_cast<const Join*>(p.partials);
  const int shares = notes[0].parts;
  const Join j = notes[note];              // there is room for it, whether there is such a share or not
  if ((!notes_by_segment && note >= shares) || j.parts == 0) return;
  const int b = j.segment / tiles / p.H_kv, h = j.segment / tiles % p.H_kv, t = j.segment % tiles;
  const float* slots = p.partials + shares_room * (sizeof(Join) / sizeof(float));
  const int tile = blockIdx.y / PARTS, dt0 = (blockIdx.y % PARTS) * DT;

  f32x4 o[DT];
  float m = -INFINITY, l = 0.f;
#pragma unroll
  for (int i = 0; i < DT; ++i) o[i] = f32x4{0, 0, 0, 0};
  for (int part = wave; part < j.parts; part += NW * kAhead) {
    f32x4 x[kAhead][DT];
    float mp[kAhead], lp[kAhead];
#pragma unroll
    for (int a = 0; a < kAhead; ++a) {
      mp[a] = -INFINITY;
      lp[a] = 0.f;
#pragma unroll
      for (int i = 0; i < DT; ++i) x[a][i] = f32x4{0, 0, 0, 0};
      if (part + a * NW >= j.parts) continue;
      const float* slot = slots + (size_t)joined_slot(j.first, part + a * NW) * kSlotFloats<D, RT, KW>;
      const float* ml = slot + RG * RT * (D / 16 * 256) + tile * 32;
#pragma unroll
      for (int i = 0; i < DT; ++i) x[a][i] = reinterpret_cast<const f32x4*>(slot)[(tile * (D / 16) + dt0 + i) * 64 + lane];
      mp[a] = ml[r];
      lp[a] = ml[16 + r];
    }
    float most = m;
#pragma unroll
    for (int a = 0; a < kAhead; ++a) most = fmaxf(most, mp[a]);
    const float use = most == -INFINITY ? 0.f : most, mine = __builtin_amdgcn_exp2f(m - use);
    l *= mine;
#pragma unroll
    for (int i = 0; i < DT; ++i) o[i] *= mine;
#pragma unroll
    for (int a = 0; a < kAhead; ++a) {
      const float theirs = __builtin_amdgcn_exp2f(mp[a] - use);
      l += lp[a] * theirs;
#pragma unroll
      for (int i = 0; i < DT; ++i) o[i] += x[a][i] * theirs;
    }
    m = most;
  }
  if (g == 0) { joined_ml[0][wave][r] = m; joined_ml[1][wave][r] = l; }
#pragma unroll
  for (int i = 0; i < DT; ++i) joined[wave][i][lane] = o[i];
  __syncthreads();
  if (wave != 0) return;
  float most = -INFINITY;
#pragma unroll
  for (int k = 0; k < NW; ++k) most = fmaxf(most, joined_ml[0][k][r]);
  const float use = most == -INFINITY ? 0.f : most;
  l = 0.f;
#pragma unroll
  for (int i = 0; i < DT; ++i) o[i] = f32x4{0, 0, 0, 0};
#pragma unroll 4
  for (int k = 0; k < NW; ++k) {
    const float by = __builtin_amdgcn_exp2f(joined_ml[0][k][r] - use);
    l += joined_ml[1][k][r] * by;
#pragma unroll
    for (int i = 0; i < DT; ++i) o[i] += joined[k][i][lane] * by;
  }
  store_row<DT>(p, find_row(p, b, t * M + tile * 16 + r), b, h, o, most, l, dt0, g);
}

template <int D, int RT, int KW> hipError_t launch_fwd(const AttendArgs& p, const CacheForm& f, hipStream_t stream) {
  if (!f.split) {
    attn_cache_fwd_kernel<D, RT, KW, false><<<dim3((unsigned)p.H_kv, (unsigned)f.tiles, (unsigned)p.B), kThreads, 0, stream>>>(p, f.tiles, 0, false);
    return hipGetLastError();
  }
  attn_cache_fwd_kernel<D, RT, KW, true><<<(unsigned)((f.shares + 7) / 8 * 8), kThreads, 0, stream>>>(p, f.tiles, f.shares, f.many_parts);
  if (const hipError_t e = hipGetLastError(); e != hipSuccess) return e;
  const unsigned joins = (unsigned)(f.shares - 1), row_tiles = (4 / KW) * RT;
  if (f.many_parts)
    attn_cache_merge_kernel<D, RT, KW, 16, 2><<<dim3((unsigned)(p.B * p.H_kv * f.tiles), row_tiles * (D / 32)), 1024, 0, stream>>>(p, f.tiles, f.shares, true);
  else
    attn_cache_merge_kernel<D, RT, KW, 2, D / 16><<<dim3(joins, row_tiles), 128, 0, stream>>>(p, f.tiles, f.shares, false);
  return hipGetLastError();
}
template <int D> hipError_t launch_fwd(const AttendArgs& p, hipStream_t stream) {
  const CacheForm f = cache_form(p.B, p.H, p.H_kv, p.N, D, p.cache.capacity);
  if (f.KW == 4) return launch_fwd<D, 1, 4>(p, f, stream);
  if (f.RT == 1) return launch_fwd<D, 1, 1>(p, f, stream);
  return launch_fwd<D, 2, 1>(p, f, stream);
}

// ---- weights.  The wave's tile is S^T again: lane (r, g) adds up exp(S - LSE) of row r of every row tile for the 16 tokens of its
// group, and the 16 lanes of a group are added at the end: a block's tokens belong to one wave or one work-group, no atomics.
//
// Few row tiles: bound by K's bytes; a wave takes up to 8 blocks one after the other, the next one's codes on their way (one token of 32
// sequences of 2000 to 4160 tokens, H 32/8, d 128: 25 us with a block per wave, 22.6 with 2, 21.4 with 8).  Many: by the exponentials and the products, and by what a row
// tile costs besides (addresses, loads), which two blocks share (500 queries, H 32/8, over 16384 tokens: 142 us with one block, 80 with two);
// the four waves of a work-group take the row tiles in turn.
DEVI float sum_over_16_lanes(float x) {        // the same in all 16: four rotations of the row
  x += __uint_as_float((unsigned)__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(x), 0x128, 0xf, 0xf, false));
  x += __uint_as_float((unsigned)__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(x), 0x124, 0xf, 0xf, false));
  x += __uint_as_float((unsigned)__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(x), 0x122, 0xf, 0xf, false));
  x += __uint_as_float((unsigned)__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(x), 0x121, 0xf, 0xf, false));
  return x;
}
// What a (sequence, head) is to a wave.
struct Weighed {
  int b, h, n, rows, all;                  // queries, rows of the list; tokens in the cache
  long long length;
  int lead;                                // query i sees max(0, min(all, lead + i)) tokens (all without causal); |lead| <= 2^30
  size_t first;                            // element of weights of the head's first token
  DEVI Weighed(const WeighArgs& p, int b_, int h_) : b(b_), h(h_) {
    n = uniform(real_count(p.counts, b, p.N));
    rows = n * p.group;
    length = uniform(p.lengths[b]);
    all = (int)max(0ll, min(length, (long long)p.cache.capacity));
    lead = p.causal ? (int)max(-(1ll << 30), min(length - n + 1, 1ll << 30)) : all;
    first = ((size_t)b * p.H_kv + h) * p.cache.capacity;
  }
  // what token t had: one of this call's has no weight yet
  DEVI float had(const WeighArgs& p, int t) const { return p.in && t < all && t < length - n ? p.in[first + t] : 0.f; }
};
// one row tile's queries: fragments, LSE in units of log 2, tokens that the lane's row sees (none where it is not there or sees nothing)
template <int D> struct QueryTile {
  bf16x8 q[D / 32];
  float less;
  int limit;
  // (limit in 64 bits: d = 256, 256 rows of 8 sequences of 4096 tokens 75 us, and 98 with `sees` in the kernel for few rows)
  DEVI void load(const WeighArgs& p, const Weighed& x, bool there, int query, int member, int g) {
    const int head = x.h * p.group + (there ? member : 0), i = there ? query : 0;
    const unsigned short* at = p.Q.at + x.b * p.Q.sb + head * p.Q.sh + i * p.Q.sn;
    load_queries(at, g);
    const float lse = p.LSE[((size_t)x.b * p.H + head) * p.N + i];
    limit = there && lse != -INFINITY ? (p.causal ? (int)max(0ll, min((long long)x.all, x.length - x.n + i + 1)) : x.all) : 0;
    less = limit > 0 ? lse * kLog2e : 0.f;
  }
  DEVI void load_queries(const unsigned short* at, int g) {
#pragma unroll
    for (int c = 0; c < D / 32; ++c) q[c] = *reinterpret_cast<const bf16x8*>(at + query_column<D>(c, g));
  }
  DEVI void sees(const Weighed& x, bool there, int query, float lse) {
    limit = there && lse != -INFINITY ? max(0, min(x.all, x.lead + query)) : 0;
    less = limit > 0 ? lse * kLog2e : 0.f;
  }
};
template <int D> DEVI void widen_keys(bf16x8 (&kf)[4][D / 32], const KCodes<D>& k, float scale) {
#pragma unroll
  for (int j = 0; j < 4; ++j)
#pragma unroll
    for (int c = 0; c < D / 32; ++c)
      kf[j][c] = c < 2 * Cols<D>::C64 ? key_frag(k.c[j][c / 2], c & 1, scale) : widen8(k.odd[j].x, k.odd[j].y, scale);
}
// a row tile's probabilities for the 16 tokens from `seen_from` on
template <int D> DEVI void add_weights(float (&sum)[16], const bf16x8 (&kf)[4][D / 32], const QueryTile<D>& tile, float scale_log2, int seen_from) {
  const int seen = tile.limit - seen_from;
  const bool whole = __all(seen >= 16);
  f32x4 s[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) s[j] = f32x4{0, 0, 0, 0};
#pragma unroll
  for (int c = 0; c < D / 32; ++c)
#pragma unroll
    for (int j = 0; j < 4; ++j) s[j] = mfma16(kf[j][c], tile.q[c], s[j]);
#pragma unroll
  for (int i = 0; i < 16; ++i) s[i / 4][i % 4] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[i / 4][i % 4], scale_log2, -tile.less));
  if (!whole) {
#pragma unroll
    for (int i = 0; i < 16; ++i)
      if (i >= seen) s[i / 4][i % 4] = 0.f;
  }
#pragma unroll
  for (int i = 0; i < 16; ++i) sum[i] += s[i / 4][i % 4];
}
// of token 16 g + r: the sum over the 16 lanes that have some of it
DEVI float own_sum(const float (&sum)[16], int r) {
  float mine = 0.f;
#pragma unroll
  for (int j = 0; j < 16; ++j) {
    const float x = sum_over_16_lanes(sum[j]);
    mine = r == j ? x : mine;
  }
  return mine;
}

template <int D> __global__ __launch_bounds__(kThreads, D == 256 ? 1 : 2) void attn_cache_weights_few_kernel(WeighArgs p, int per_wave) {
  const int lane = threadIdx.x & 63, wave = uniform((int)(threadIdx.x >> 6)), r = lane & 15, g = lane >> 4;
  const int nb = p.cache.capacity / kBlock, first = uniform((int)(blockIdx.x * 4 + wave) * per_wave);
  if (first >= nb) return;
  const Weighed x(p, blockIdx.z, blockIdx.y);
  const int end = min(nb, first + per_wave);
  const int keys_end = x.rows > 0 ? min(end, (x.all + kBlock - 1) / kBlock) : first;       // blocks with something to add
  const unsigned token = (r >> 2) * 16 + (r & 3);
  const unsigned char* K = p.cache.K + x.first * D;
  const float* Ks = p.cache.K_scale + x.first / kBlock;
  KCodes<D> k;
  float k_scale = 0.f, had = x.had(p, first * kBlock + lane);
  QueryTile<D> tile;
  auto load_key = [&](int blk) {
    if (blk >= keys_end) return;
    k_scale = Ks[blk];
    k.load(K + (size_t)blk * (kBlock * D), token * D + g * 16, token * D + g * 8);
  };
  auto load_tile = [&](int row) { tile.load(p, x, row < x.rows, row / p.group, row % p.group, g); };
  load_key(first);
  if (first < keys_end) load_tile(r);
  const float scale_log2 = p.scale * kLog2e;
#pragma unroll 1
  for (int blk = first; blk < end; ++blk) {
    const int t = blk * kBlock + lane;
    float sum[16];
#pragma unroll
    for (int j = 0; j < 16; ++j) sum[j] = 0.f;
    const float was = had;
    if (blk + 1 < end) had = x.had(p, t + kBlock);
    if (blk < keys_end) {
      bf16x8 kf[4][D / 32];
      widen_keys<D>(kf, k, k_scale);
      load_key(blk + 1);
      add_weights<D>(sum, kf, tile, scale_log2, blk * kBlock + 16 * g);
      if (x.rows > 16) {
        for (int row = 16; row < x.rows; row += 16) {
          load_tile(row + r);
          add_weights<D>(sum, kf, tile, scale_log2, blk * kBlock + 16 * g);
        }
        load_tile(r);
      }
    }
    const float mine = own_sum(sum, r);
    p.out[x.first + t] = t >= x.all ? 0.f : was + mine;
  }
}

template <int D, int NB> __global__ __launch_bounds__(kThreads, 2) void attn_cache_weights_many_kernel(WeighArgs p) {
  __shared__ float joined[4][NB * kBlock];
  const int lane = threadIdx.x & 63, wave = uniform((int)(threadIdx.x >> 6)), r = lane & 15, g = lane >> 4;
  const int nb = p.cache.capacity / kBlock, blk = blockIdx.x * NB, t0 = blk * kBlock;
  const Weighed x(p, blockIdx.z, blockIdx.y);
  float sum[NB][16];
#pragma unroll
  for (int i = 0; i < NB; ++i)
#pragma unroll
    for (int j = 0; j < 16; ++j) sum[i][j] = 0.f;
  if (t0 < x.all && x.rows > 0) {
    const unsigned token = (r >> 2) * 16 + (r & 3);
    // rows from the tile of the first that sees the first of these tokens on
    const long long hidden = p.causal ? max(0ll, t0 - (x.length - x.n)) * p.group : 0;
    constexpr int kStep = 64;
    int row = (int)min(hidden / 16 * 16, (long long)x.rows) + wave * 16 + r;
    int query = row / p.group, member = row - query * p.group;
    const int step_query = kStep / p.group, step_member = kStep - step_query * p.group;
    const unsigned short* queries = p.Q.at + x.b * p.Q.sb + x.h * p.group * p.Q.sh;
    const float* lse = p.LSE + ((size_t)x.b * p.H + x.h * p.group) * p.N;
    // where the row lies, moved on rather than multiplied out for each
    long long at = query * p.Q.sn + member * p.Q.sh;
    int at_lse = member * p.N + query;
    const long long step = step_query * p.Q.sn + step_member * p.Q.sh, wrap = p.Q.sn - p.group * p.Q.sh;
    const int step_lse = step_member * p.N + step_query, wrap_lse = 1 - p.group * p.N;
    QueryTile<D> next;
    auto load_tile = [&]() {                               // and on to the one after it
      const bool there = row < x.rows;
      next.load_queries(queries + (there ? at : 0), g);
      next.sees(x, there, query, lse[there ? at_lse : 0]);
      row += kStep;
      query += step_query;
      member += step_member;
      at += step;
      at_lse += step_lse;
      if (member >= p.group) {
        member -= p.group;
        ++query;
        at += wrap;
        at_lse += wrap_lse;
      }
    };
    int tile = uniform(row - r);
    bf16x8 kf[NB][4][D / 32];
#pragma unroll
    for (int i = 0; i < NB; ++i) {
      const int from = min(blk + i, nb - 1);               // a block past the end: the last one again, for nothing
      KCodes<D> k;
      k.load(p.cache.K + (x.first + (size_t)from * kBlock) * D, token * D + g * 16, token * D + g * 8);
      widen_keys<D>(kf[i], k, p.cache.K_scale[x.first / kBlock + from]);
    }
    const float scale_log2 = p.scale * kLog2e;
    if (tile < x.rows) load_tile();
    for (; tile < x.rows; tile += kStep) {
      const QueryTile<D> now = next;
      if (tile + kStep < x.rows) load_tile();
#pragma unroll
      for (int i = 0; i < NB; ++i) add_weights<D>(sum[i], kf[i], now, scale_log2, t0 + i * kBlock + 16 * g);
    }
  }
#pragma unroll
  for (int i = 0; i < NB; ++i) joined[wave][i * kBlock + lane] = own_sum(sum[i], r);
  __syncthreads();
  for (int i = wave; i < NB && blk + i < nb; i += 4) {
    const int at = i * kBlock + lane, t = t0 + at;
    p.out[x.first + t] = t >= x.all ? 0.f : x.had(p, t) + joined[0][at] + joined[1][at] + joined[2][at] + joined[3][at];
  }
}

template <int D> hipError_t launch_weights(const WeighArgs& p, hipStream_t stream) {
  const unsigned nb = (unsigned)(p.cache.capacity / kBlock);
  constexpr int NB = D <= 128 ? 2 : 1;       // (a lane's registers hold one block's keys of d = 256)
  // The crossing point is where the second block's widened keys are paid for, later the more there are of them.  us, few / many, 32 sequences of 4096
  // (d = 96, 128; 16 of d = 32, 64; 8 of d = 256): d = 128: 256 rows 141 / 159, 320 171 / 177, 384 202 / 199, 448 232 / 226, 512 264 / 246; d = 32: 96 rows
  // 18.3 / 19.5, 128 22.8 / 21.7; d = 64: 160 32.6 / 33.7, 192 37.6 / 36.5, 256 47 / 43; d = 96: 288 123 / 126, 320 135 / 133.  At d = 256 it lies beyond
  // the rule's 768: 512 133 / 151, 768 194 / 208, 896 225 / 237.
  if ((long long)p.N * p.group <= 3 * D) {
    // a block per wave until the waves are two to a SIMD, then more, up to 8
    const long long blocks = (long long)p.B * p.H_kv * nb;
    const unsigned per_wave = (unsigned)std::min(8ll, std::max(1ll, blocks / 2048)), per_group = 4 * per_wave;
    attn_cache_weights_few_kernel<D><<<dim3((nb + per_group - 1) / per_group, (unsigned)p.H_kv, (unsigned)p.B), kThreads, 0, stream>>>(p, (int)per_wave);
  } else {
    if (!grid_fits((nb + NB - 1) / NB, kThreads)) return hipErrorInvalidConfiguration;
    attn_cache_weights_many_kernel<D, NB><<<dim3((nb + NB - 1) / NB, (unsigned)p.H_kv, (unsigned)p.B), kThreads, 0, stream>>>(p);
  }
  return hipGetLastError();
}

}  // namespace

size_t attn_cache_fwd_partial_bytes(int B, int H, int H_kv, int N, int d, int capacity) {
  return cache_form(B, H, H_kv, N, d, capacity).workspace_bytes(d);
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
