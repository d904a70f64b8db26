// Attention over the 8-bit cache: what the kernels of attn_cache_fwd (cache_attn.hip) and attn_cache_fwd_shared (cache_shared.hip) do with a
// segment, a (sequence, key/value head, tile of query rows) and its key blocks.
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
#pragma once
#include "cache.hpp"

namespace {

constexpr int kAttendThreads = 256;
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
  int before[kAttendThreads + 1];                // units in front of thread t's run
  int waves[kAttendThreads / 64];
  Segment segment;
};
// A thread's units, summed over the threads in front of it in its wave and with its own.
DEVI int own_units(const Problem& q, int items, int run) {
  const int tid = threadIdx.x;
  int x = 0;
  for (int i = tid * run; i < min(items, (tid + 1) * run); ++i) x += q.cost(i / q.tiles, i % q.tiles);
  return x;
}
DEVI int scan_in_wave(int x, Runs& runs) {
  const int tid = threadIdx.x;
  x = (int)sum_to_lane((unsigned)x);
  if ((tid & 63) == 63) runs.waves[tid >> 6] = x;
  return x;
}
// behind a barrier; another one, and runs.before is there for all
DEVI void scan_waves(int x, Runs& runs) {
  const int tid = threadIdx.x, wave = tid >> 6;
#pragma unroll
  for (int w = 0; w < kAttendThreads / 64 - 1; ++w) x += w < wave ? runs.waves[w] : 0;
  runs.before[tid + 1] = x;
  if (tid == 0) runs.before[0] = 0;
}
// units of all items
DEVI int scan_units(const Problem& q, int items, int run, Runs& runs) {
  const int x = scan_in_wave(own_units(q, items, run), runs);
  __syncthreads();
  scan_waves(x, runs);
  __syncthreads();
  return uniform(runs.before[kAttendThreads]);
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
  s.start = q.start;
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

// A prefix's tokens in front of a sequence's own: its codes and scales for a head, its blocks and tokens.
struct Before {
  const unsigned char *K, *V;
  const float *K_scale, *V_scale;
  int blocks, length;
};

// What a work-group has to do: units pos .. end - 1 of a list, beginning in `seg`, as share w of `all`.
struct Work {
  Segment seg;
  int pos, end, w;
  Shares all;
};
// Where the parts of split segments go, and the notes about them.
struct Parts {
  Join* notes;
  float* slots;
  bool by_segment;                         // a note for each segment
};

// What the segments are over: a call's queries and its cache.
struct PlainCall {
  static constexpr bool kJoint = false, kHeads = false, kRealRows = false;
  const AttendArgs& p;
  // a row of the list
  DEVI const unsigned short* query(int b, int head, int query) const { return p.Q.at + b * p.Q.sb + head * p.Q.sh + query * p.Q.sn; }
  // column tiles dt0 .. dt0 + DT - 1 of a finished row tile, the segment's `tile`-th
  template <int DT, int M> DEVI void store(const Segment& s, int tile, const f32x4* o, float m, float l, int dt0, int lane) const {
    store_row<DT>(p, find_row(p, s.b, s.t * M + tile * 16 + (lane & 15)), s.b, s.h, o, m, l, dt0, lane >> 4);
  }
};

// LDS of a work-group: sums of the four waves to be joined, or two blocks' codes.
template <int D, int RT, int KW, bool HEADS = false>
constexpr int kAttendBytes = KW == 4 ? 4 * RT * (D / 16) * 64 * 16 + 2 * 4 * RT * 16 * 4 : HEADS ? 0 : 2 * Staged<D>::kBytes;

// SPLIT: a share of the list of blocks; otherwise one segment, nothing to merge.
//
// KW = 4, few rows: bound by bytes; every wave reads blocks of its own straight into registers, K's a block ahead (one token of 64 sequences of 4300, H 32/8, d
// 128: 100 us, 5.6 TB/s).  KW = 1, many rows: bound by
// the vector and matrix units; the four waves share a block through LDS, filled by asynchronous transfers a block ahead (three blocks ahead, in four
// buffers: 16 queries of 64 sequences of 4300 tokens, H 32/8, d 128, 139 us; one ahead, in two: 125.  2048 queries over 16384: 636 and 620; these with the
// loop of that time, which takes 121 and 493 now).
//
// Call::kJoint: a segment's blocks are those of its sequence's prefix, then its own.
// Call::kHeads (KW = 1, few rows): a segment is the same rows of four key/value heads, one for each wave, which reads that head's blocks straight into
// registers: short segments are begun and ended four at a time, and nothing is joined in LDS.
// Call::kRealRows: parts hold the real queries' rows alone (few of 16 or 64 rows may be real, and short segments have many parts).
// staged: kAttendBytes of LDS, 1 KB aligned.
template <int D, int RT, int KW, bool SPLIT, class Call>
DEVI void attend(const Call& call, const Problem& q, Work& work, const Parts& parts, char* staged) {
  constexpr int RG = 4 / KW, M = 16 * RT * (Call::kHeads ? 1 : RG);
  constexpr bool DIRECT = KW == 4 || Call::kHeads;
  static_assert(KW == 1 || (KW == 4 && !Call::kHeads), "the four waves have rows of their own, or heads, or blocks");
  f32x4* joined = reinterpret_cast<f32x4*>(staged);        // KW == 4: [wave][RT][D / 16][lane]
  float *joined_m = reinterpret_cast<float*>(joined + 4 * RT * (D / 16) * 64), *joined_l = joined_m + 4 * RT * 16;
  const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6);
  const int r = lane & 15, g = lane >> 4;
  const int kw = wave % KW, rg = wave / KW;
  const AttendArgs& p = call.p;
  const int nb = p.cache.capacity / kBlock, tiles = q.tiles, w = work.w, end = work.end, heads = Call::kHeads ? (p.H_kv + 3) / 4 : p.H_kv;
  const float scale_log2 = p.scale * kLog2e;
  Segment& seg = work.seg;
  int pos = work.pos;

  while (true) {
    const int to = min(end, seg.end());
    if (SPLIT && parts.by_segment && tid == 0 && pos == seg.begin)
      parts.notes[segment_number(seg, heads, tiles)] = note_of_segment(work.all, w, seg, heads, tiles);
    const bool idle = Call::kHeads && 4 * seg.h + wave >= p.H_kv;          // there is no such head
    const int b = seg.b, h = Call::kHeads ? min(4 * seg.h + wave, p.H_kv - 1) : seg.h, first_row = seg.t * M + (Call::kHeads ? 0 : rg * RT * 16);
    const int blk0 = seg.block_at(pos), blk_end = idle ? blk0 : seg.block_at(to);
    const size_t bh = (size_t)b * p.H_kv + h;
    const unsigned char* K = p.cache.K + bh * p.cache.capacity * D;
    const unsigned char* V = p.cache.V + bh * p.cache.capacity * D;
    const float* Ks = p.cache.K_scale + bh * nb;
    const float* Vs = p.cache.V_scale + bh * nb;
    [[maybe_unused]] Before before;
    if constexpr (Call::kJoint) before = call.before(b, h, D);
    // block blk of the segment: its codes, its place among the 64 blocks' scales, its first token, and the tokens there are
    auto codes = [&](const unsigned char* own, const unsigned char* prefix, int blk) {
      if constexpr (Call::kJoint) return blk < before.blocks ? prefix + (size_t)blk * (kBlock * D) : own + (size_t)(blk - before.blocks) * (kBlock * D);
      else return own + (size_t)blk * (kBlock * D);
    };
    auto scale_of = [&](const float* own, const float* prefix, int blk) {
      if constexpr (Call::kJoint) return blk < before.blocks ? prefix[blk] : own[blk - before.blocks];
      else return own[blk];
    };
    // a wave of few rows: its first block is on its way while the queries are looked for
    const unsigned at = ((r >> 2) * 16 + (r & 3)) * D + g * 16, at_odd = ((r >> 2) * 16 + (r & 3)) * D + g * 8, at_v = r * kBlock + g * 16;
    KCodes<D> k;
    float k_scale = 0.f, next_v = 0.f;     // loaded with K's codes: a load behind V's would have V waited for
    auto load_key = [&](int blk) {
      if (blk >= blk_end) return;
      k_scale = scale_of(Ks, before.K_scale, blk);
      next_v = scale_of(Vs, before.V_scale, blk);
      k.load(codes(K, before.K, blk), at, at_odd);
    };
    if constexpr (DIRECT) load_key(blk0 + kw);
    int least = 0x7fffffff, limit[RT];
    bf16x8 qf[RT][D / 32];
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
      const Row x = find_row(p, b, first_row + rt * 16 + r);
      limit[rt] = x.limit;
      least = min(least, x.limit);
      const unsigned short* from = call.query(b, h * p.group + x.head, x.query);
#pragma unroll
      for (int c = 0; c < D / 32; ++c) qf[rt][c] = *reinterpret_cast<const bf16x8*>(from + query_column<D>(c, g));
    }
#pragma unroll
    for (int i = 1; i < 16; i <<= 1) least = min(least, __shfl_xor(least, i));
    least = uniform(least);

    const int real_rows = (Call::kRealRows ? uniform(q.count(b)) : p.N) * p.group;
    Acc<D, RT> a;
    a.clear();
    auto step = [&](const KCodes<D>& k, VCodes<D>& v, float k_scale, float v_scale, int blk, auto&& after_scores) {
      if constexpr (Call::kJoint) {
        const bool prefix = blk < before.blocks;
        const int t0 = (prefix ? blk : blk - before.blocks) * kBlock;
        int seen[RT];
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) seen[rt] = prefix ? before.length : limit[rt];
        block_step<D, RT>(a, qf, k, v, k_scale, v_scale, scale_log2, seen, t0 + kBlock > (prefix ? before.length : least), t0, g, after_scores);
      } else {
        block_step<D, RT>(a, qf, k, v, k_scale, v_scale, scale_log2, limit, blk * kBlock + kBlock > least, blk * kBlock, g, after_scores);
      }
    };
    if constexpr (!DIRECT) {
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
          const bool key = piece < Staged<D>::KP;
          fetch_piece(codes(key ? K : V, key ? before.K : before.V, blk), from[i], buffers + buffer * Staged<D>::kBytes + piece * 1024);
        }
      };
      const int in_piece = r * 64 + ((g ^ slot_mask(r >> 2)) << 4), in_odd = r * 32 + g * 8;
      const bool rows_here = first_row < real_rows;
      // Scales: 64 blocks' at a time, one in each lane.
      float k_scales = 0.f, v_scales = 0.f;
      auto load_scales = [&](int blk) {
        const int mine = min(blk + lane, (Call::kJoint ? before.blocks : 0) + nb - 1);
        k_scales = scale_of(Ks, before.K_scale, mine);
        v_scales = scale_of(Vs, before.V_scale, mine);
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
          step(k, v, ks, vs, blk, [&] { read_staged<D>(v, base + in_piece); });
        }
        buffer ^= 1;
      }
    } else {
      for (int blk = blk0 + kw; blk < blk_end; blk += KW) {
        VCodes<D> v;
        v.load(codes(V, before.V, blk), at_v);
        step(k, v, k_scale, next_v, blk, [&] { load_key(blk + KW); });
      }
    }

    a.join_groups();
    const bool whole = !SPLIT || (pos == seg.begin && to == seg.end());
    float* slot = parts.slots + (size_t)(2 * w + (pos == seg.begin ? 1 : 0)) * kSlotFloats<D, RT, KW>;
    // O and LSE of a finished row, or this part of them: column tiles dt0 .. dt0 + DT - 1 of row tile `tile`
    auto put = [&](auto DT, int tile, const f32x4* o, float m, float l, int dt0) {
      if (whole) {
        call.template store<DT, M>(seg, tile, o, m, l, dt0, lane);
        return;
      }
      if (Call::kRealRows && seg.t * M + (Call::kHeads ? 0 : tile * 16) + r >= real_rows) return;
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
    next_segment(q, heads, seg);
    seg.blocks = uniform(seg.blocks);
  }
}

}  // namespace
