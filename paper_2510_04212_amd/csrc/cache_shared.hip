// Attention of sequences that continue prefixes they share with others (attn_cache_fwd_shared of include/attn.h).
#include "cache_attend.hpp"
#include <algorithm>
#include <cmath>

namespace {

// Every segment reads its sequence's prefix, then its own blocks.
struct JointCall {
  static constexpr bool kJoint = true, kHeads = false, kRealRows = false;
  const AttendArgs& p;
  const SharedArgs& all;
  DEVI int length(int b) const { return uniform(min(max(all.prefix_lengths[b / all.S], 0), all.prefix.capacity)); }
  DEVI Before before(int b, int h, int d) const {
    const size_t ph = (size_t)(b / all.S) * p.H_kv + h, at = ph * all.prefix.capacity;
    const int tokens = length(b);
    return Before{all.prefix.K + at * d, all.prefix.V + at * d, all.prefix.K_scale + at / kBlock, all.prefix.V_scale + at / kBlock,
                  (tokens + kBlock - 1) / kBlock, tokens};
  }
  DEVI const unsigned short* query(int b, int head, int query) const { return p.Q.at + b * p.Q.sb + head * p.Q.sh + query * p.Q.sn; }
  template <int DT, int M> DEVI void store(const Segment& s, int tile, const f32x4* o, float m, float l, int dt0, int lane) const {
    Row x = find_row(p, s.b, s.t * M + tile * 16 + (lane & 15));
    if (length(s.b) > 0) x.empty = x.query >= real_count(p.counts, s.b, p.N);
    store_row<DT>(p, x, s.b, s.h, o, m, l, dt0, lane >> 4);
  }
};

template <int D, int RT, int KW>
__global__ __launch_bounds__(kAttendThreads, D == 256 ? 1 : 2) void attn_cache_joint_kernel(SharedArgs a, int tiles) {
  constexpr int M = 16 * RT * 4 / KW;
  const AttendArgs& p = a.own;
  const Problem q{p.lengths, p.counts, p.cache.capacity, p.N, p.group, p.causal, tiles, M};
  const JointCall call{p, a};
  Work work{{}, 0, 0, 0, {1, 0, 0}};
  work.seg.b = blockIdx.z;
  work.seg.h = blockIdx.x;
  work.seg.t = blockIdx.y;
  work.seg.begin = 0;
  const int b = work.seg.b, t = work.seg.t;
  const int before = t * M < q.count(b) * p.group ? (call.length(b) + kBlock - 1) / kBlock : 0;
  work.seg.blocks = uniform(q.blocks(b, t) + before);
  work.end = work.seg.end();
  __shared__ __attribute__((aligned(1024))) char staged[kAttendBytes<D, RT, KW>];
  attend<D, RT, KW, false>(call, q, work, Parts{}, staged);
}

// ---- shared: two lists of segments in one launch, the prefixes' (rows: the real queries of a prefix's sequences, one after the other) and the sequences'
// own.  Every segment leaves its rows' sums, whole or in parts, for the joining kernel.  The prefixes' are shared out to work-groups as in
// attn_cache_fwd, to as many of those that run at once as what their units cost against the own ones' says; own ones have a work-group each, or, where they are
// long, are shared out to the rest.
//
// Bound by bytes up to 64 rows (128 beams of 16 prompts: 47 us, 3.9 TB/s with 12 us of finding work and parts), by the matrix and vector units above (16 answers about 131072
// tokens: 51.7 us, 660 TFLOP/s), where with 128-row tiles at d = 128 both lists' state does not fit beside attend's: 14 vector registers and some 400 scalar ones spill, 24 and 513
// where own tiles have 128 rows, too (64 queries each of 2 x 8: 89 us, 690 TFLOP/s); a plain call's kernel spills 7 and 258 and reaches 1070.
struct List {
  Join* notes;                             // one for each segment
  float* slots;                            // parts of segments: two for each work-group
  float* whole;                            // whole segments
  int heads, tiles;                        // segments of a sequence: so many (key/value heads, or fours of them) times so many (tiles of rows)
  int cost;                                // of a unit
  __host__ __device__ int segment(int b, int h, int t) const { return (b * heads + h) * tiles + t; }
};
struct SharedPlan {
  AttendArgs prefix;                       // the prefixes as sequences: P of them, of up to S * N queries each
  const int* starts;                       // [P * S]: real queries of its prefix's sequences in front of this one; NULL: all are taken
  int groups;                              // work-groups that the lists are shared out to: a multiple of 8, 16 at least
  bool own_split;                          // the own list is; otherwise a work-group for each of its segments follows
  List prefixes, own;
};

// What four heads' segments cost to begin and end, in blocks of theirs.
constexpr int kHeadsStart = 1;
template <int KW, bool HEADS> constexpr int kLeast = HEADS ? kHeadsStart + 1 : kLeastUnits<KW>;

// 16-row tiles of a slot: sums of their rows, then maxima and sums of probabilities
template <int D> constexpr int kTileFloats = D / 16 * 256 + 32;

template <int D, int TILES, bool PREFIX, bool HEADS> struct ListCall {
  static constexpr bool kJoint = false, kHeads = HEADS, kRealRows = true;
  const AttendArgs& p;
  const SharedPlan& plan;
  int N, S;                                // (of the prefixes)
  DEVI const List& list() const { return PREFIX ? plan.prefixes : plan.own; }
  DEVI const unsigned short* query(int b, int head, int query) const {
    long long s = b;
    int i = query;
    if constexpr (PREFIX) {
      int at = 0;
      if (plan.starts) {                   // the last sequence that begins at or in front of it (those without queries in front of it, too)
        const int* starts = plan.starts + (size_t)b * S;
        for (int end = S; end - at > 1;) {
          const int mid = (at + end) / 2;
          if (starts[mid] <= query) at = mid;
          else end = mid;
        }
        i = min(query - starts[at], N - 1);                // (a row behind the last real one: any query)
      } else {
        at = query / N;
        i = query - at * N;
      }
      s = (long long)b * S + at;
    }
    return p.Q.at + s * p.Q.sb + head * p.Q.sh + i * p.Q.sn;
  }
  template <int DT, int M> DEVI void store(const Segment& s, int tile, const f32x4* o, float m, float l, int dt0, int lane) const {
    const int r = lane & 15;
    if (s.t * M + (HEADS ? 0 : tile * 16) + r >= p.N * p.group) return;
    float* slot = list().whole + (size_t)list().segment(s.b, s.h, s.t) * (TILES * kTileFloats<D>);
#pragma unroll
    for (int i = 0; i < DT; ++i) reinterpret_cast<f32x4*>(slot)[(tile * (D / 16) + dt0 + i) * 64 + lane] = o[i];
    float* ml = slot + TILES * (D / 16 * 256) + tile * 32;
    if (lane < 16 && dt0 == 0) {
      ml[r] = m;
      ml[16 + r] = l;
    }
  }
};

// Where a padded batch's real queries begin, prefix by prefix, and how many there are.
__global__ __launch_bounds__(kAttendThreads) void attn_cache_starts_kernel(const int* counts, int S, int N, int* starts, int* totals) {
  __shared__ int waves[kAttendThreads / 64];
  const int p = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int run = (S + kAttendThreads - 1) / kAttendThreads, first = min(S, tid * run), end = min(S, first + run);
  counts += (size_t)p * S;
  starts += (size_t)p * S;
  int sum = 0;
  for (int s = first; s < end; ++s) sum += real_count(counts, s, N);
  int x = (int)sum_to_lane((unsigned)sum);
  if (lane == 63) waves[wave] = x;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < kAttendThreads / 64; ++w) x += w < wave ? waves[w] : 0;
  if (tid == kAttendThreads - 1) totals[p] = x;
  x -= sum;
  for (int s = first; s < end; ++s) {
    starts[s] = x;
    x += real_count(counts, s, N);
  }
}

template <int D, int RT, int KW, int ORT, int OKW, bool HEADS>
__global__ __launch_bounds__(kAttendThreads, D == 256 ? 1 : 2) void attn_cache_shared_kernel(SharedArgs a, SharedPlan plan) {
  constexpr int BYTES = kAttendBytes<D, RT, KW>, OWN_BYTES = kAttendBytes<D, ORT, OKW, HEADS>;
  __shared__ __attribute__((aligned(1024))) char staged[BYTES > OWN_BYTES ? BYTES : OWN_BYTES];       // a work-group is in one of the two
  __shared__ Runs runs, own_runs;
  const AttendArgs &p = plan.prefix, &o = a.own;
  const Problem q{p.lengths, p.counts, p.cache.capacity, p.N, p.group, 0, plan.prefixes.tiles, 16 * RT * 4 / KW};
  const Problem own{o.lengths, o.counts, o.cache.capacity, o.N, o.group, o.causal, plan.own.tiles, HEADS ? 16 : 16 * ORT * 4 / OKW, HEADS ? kHeadsStart : kStart};
  const int run = (p.B * q.tiles + kAttendThreads - 1) / kAttendThreads, own_run = (o.B * own.tiles + kAttendThreads - 1) / kAttendThreads;
  Work work;
  if ((int)blockIdx.x >= plan.groups) {    // an own segment
    const int i = blockIdx.x - plan.groups;
    work.seg = Segment{i / own.tiles / plan.own.heads, i / own.tiles % plan.own.heads, i % own.tiles, 0, 0, own.start};
    work.seg.blocks = uniform(own.blocks(work.seg.b, work.seg.t));
    work.pos = 0;
    work.end = work.seg.end();
    work.w = 0;
    work.all = Shares{1, work.end, 0};
  } else {
    int x = own_units(q, p.B * q.tiles, run), own_x = own_units(own, o.B * own.tiles, own_run);          // (both lists' loads at once)
    x = scan_in_wave(x, runs);
    own_x = scan_in_wave(own_x, own_runs);
    __syncthreads();
    scan_waves(x, runs);
    scan_waves(own_x, own_runs);
    __syncthreads();
    const int units = plan.prefixes.heads * uniform(runs.before[kAttendThreads]), own_all = plan.own.heads * uniform(own_runs.before[kAttendThreads]);
    const int eighths = plan.groups / 8;
    const long long cost = (long long)units * plan.prefixes.cost, own_cost = (long long)own_all * plan.own.cost;
    const int groups = 8 * uniform(min(max((int)((eighths * cost + (cost + own_cost) / 2) / (cost + own_cost)), 1), eighths - 1));
    const bool of_prefix = (int)blockIdx.x < groups;
    if (!of_prefix && !plan.own_split) return;
    work.all = of_prefix ? shares_of(units, groups, kLeastUnits<KW>) : shares_of(own_all, plan.groups - groups, kLeast<OKW, HEADS>);
    work.w = share_of(of_prefix ? blockIdx.x : blockIdx.x - groups, work.all.number);
    if (work.w < 0) return;
    work.pos = uniform(work.all.begin(work.w));
    work.end = uniform(work.all.begin(work.w + 1));
    work.seg = of_prefix ? find_segment(q, p.B, plan.prefixes.heads, run, work.pos, runs) : find_segment(own, o.B, plan.own.heads, own_run, work.pos, own_runs);
    work.seg.blocks = uniform(work.seg.blocks);
    if (of_prefix) {
      attend<D, RT, KW, true>(ListCall<D, RT * 4 / KW, true, false>{p, plan, o.N, a.S}, q, work, Parts{plan.prefixes.notes, plan.prefixes.slots, true}, staged);
      return;
    }
  }
  attend<D, ORT, OKW, true>(ListCall<D, ORT * 4 / OKW, false, HEADS>{o, plan, 0, 0}, own, work, Parts{plan.own.notes, plan.own.slots, true}, staged);
}

// Joins a row's parts: those of its prefix's segment and those of its own.  blockIdx: 16 rows of a prefix's sequences, padding included; the head, and DT of
// the D / 16 column tiles; the prefix.  NW waves take every NW-th part and join theirs in LDS.
template <int D, int RT, int KW, int ORT, int OKW, bool HEADS, int NW, int DT>
__global__ __launch_bounds__(64 * NW) void attn_cache_shared_merge_kernel(SharedArgs a, SharedPlan plan) {
  constexpr int TILES = RT * 4 / KW, OTILES = ORT * 4 / OKW, PARTS = D / 16 / DT, kAhead = DT <= 2 ? 4 : DT <= 8 ? 2 : 1;
  __shared__ f32x4 joined[NW][DT][64];
  __shared__ float joined_ml[2][NW][16];
  const AttendArgs& p = a.own;
  const int lane = threadIdx.x & 63, wave = uniform((int)(threadIdx.x >> 6));
  const int r = lane & 15, g = lane >> 4;
  const int h = blockIdx.y / PARTS, dt0 = blockIdx.y % PARTS * DT, item = blockIdx.z;
  const int own_rows = p.N * p.group, rows = a.S * own_rows, there = blockIdx.x * 16 + r < (unsigned)rows;
  const int row = there ? blockIdx.x * 16 + r : 0, s = row / own_rows, own_row = row - s * own_rows, b = item * a.S + s;
  const bool real = there && own_row < real_count(p.counts, b, p.N) * p.group;
  const int in_prefix = plan.starts ? plan.starts[b] * p.group + own_row : row;             // its row of the prefix's list

  // where the row's parts lie: in its prefix's segment, then in its own
  constexpr int OM = HEADS ? 16 : 16 * OTILES;
  const int t = in_prefix / (16 * TILES), at = in_prefix % (16 * TILES), own_tile = HEADS ? h % 4 : own_row % OM / 16;
  const int segment = plan.prefixes.segment(item, h, t), own_segment = plan.own.segment(b, HEADS ? h / 4 : h, own_row / OM);
  Join j{0, 0, 0, 0}, k{0, 0, 0, 0};
  if (real) {
    j = plan.prefixes.notes[segment];
    k = plan.own.notes[own_segment];
  }
  const int parts = real ? max(j.parts, 1) : 0, all = real ? parts + max(k.parts, 1) : 0;
  auto slot_of = [&](int part) {
    if (part < parts)
      return j.parts == 0 ? plan.prefixes.whole + (size_t)segment * (TILES * kTileFloats<D>)
                          : plan.prefixes.slots + (size_t)joined_slot(j.first, part) * (TILES * kTileFloats<D>);
    return k.parts == 0 ? plan.own.whole + (size_t)own_segment * (OTILES * kTileFloats<D>)
                        : plan.own.slots + (size_t)joined_slot(k.first, part - parts) * (OTILES * kTileFloats<D>);
  };
  f32x4 o[DT];
  float m = -INFINITY, l = 0.f;
#pragma unroll
  for (int i = 0; i < DT; ++i) o[i] = f32x4{0, 0, 0, 0};
  for (int part = wave; __any(part < all); part += NW * kAhead) {
    f32x4 x[kAhead][DT];
    float mp[kAhead], lp[kAhead];
#pragma unroll
    for (int a = 0; a < kAhead; ++a) {
      mp[a] = -INFINITY;
      lp[a] = 0.f;
#pragma unroll
      for (int i = 0; i < DT; ++i) x[a][i] = f32x4{0, 0, 0, 0};
      const int this_part = part + a * NW;
      if (this_part >= all) continue;
      const bool first = this_part < parts;
      const float* slot = slot_of(this_part);
      const int tile = first ? at / 16 : own_tile, in_tile = first ? at % 16 : own_row % 16;
#pragma unroll
      for (int i = 0; i < DT; ++i) x[a][i] = reinterpret_cast<const f32x4*>(slot)[(tile * (D / 16) + dt0 + i) * 64 + 16 * g + in_tile];
      const float* ml = slot + (first ? TILES : OTILES) * (D / 16 * 256) + tile * 32;
      mp[a] = ml[in_tile];
      lp[a] = ml[16 + in_tile];
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
  if (wave != 0 || !there) return;
  float most = -INFINITY;
#pragma unroll
  for (int w = 0; w < NW; ++w) most = fmaxf(most, joined_ml[0][w][r]);
  const float use = most == -INFINITY ? 0.f : most;
  l = 0.f;
#pragma unroll
  for (int i = 0; i < DT; ++i) o[i] = f32x4{0, 0, 0, 0};
#pragma unroll 4
  for (int w = 0; w < NW; ++w) {
    const float by = __builtin_amdgcn_exp2f(joined_ml[0][w][r] - use);
    l += joined_ml[1][w][r] * by;
#pragma unroll
    for (int i = 0; i < DT; ++i) o[i] += joined[w][i][lane] * by;
  }
  Row x = find_row(p, b, own_row);
  if (a.prefix_lengths[item] > 0) x.empty = x.query >= real_count(p.counts, b, p.N);
  store_row<DT>(p, x, b, h, o, most, l, dt0, g);
}

// Which form serves a call, and what it needs.
struct SharedForm {
  CacheForm prefix, own;
  bool shared, own_split, heads;           // heads: four key/value heads of a sequence's own make a segment
  int own_heads, groups;
  long long segments, own_segments;
  // notes, parts, whole segments, starts and totals of real queries
  size_t workspace_bytes(int d, int P, int S) const {
    if (!shared) return 0;
    const size_t slot = prefix.slot_floats(d) * sizeof(float), own_slot = slot_floats_own(d) * sizeof(float);
    return (size_t)(segments + own_segments) * sizeof(Join) + (2 * (size_t)groups + segments) * slot + (2 * (size_t)groups + own_segments) * own_slot +
           ((size_t)P * S + P + 3) / 4 * 16;
  }
  size_t slot_floats_own(int d) const { return heads ? 4 * (size_t)(d / 16 * 256 + 32) : own.slot_floats(d); }
};
// Estimates in us, from capacities.  Joint: one launch, bound by a segment's chain of blocks, by all segments' reads through the caches (10.5 TB/s), by
// what has to come from memory (5.2; 6.2 where one work-group reads it), or by the vector and matrix units.  Shared: finding the work, parts and a second launch cost
// 12 us and more, and then a prefix is read once.  us, joint / shared, P x S, H 32/8, d 128, own 16 to 128 tokens of 128: prefixes of 1024: 1x4 10.3 / 13.8, 1x16 10.3 / 17.1,
// 8x4 11.5 / 16.7, 1x64 17.6 / 21.3, 4x32 32.1 / 25.7, 16x8 32.2 / 25.3;  of 2048: 1x4 15.7 / 14.8, 8x4 16.7 / 19.7, 1x64 28.1 / 22.5, 16x8 55.6 / 33.5;  of 512: 16x8 22.0 / 22.7;
// 16 queries, 1x8 of 1024: 23.7 / 25.3;  64 queries, 2x4 of 2048: 58.5 / 49.9;  d 64, H 12/12: 1x4 of 2048 10.2 / 12.7, 16x8 of 1024 22.2 / 17.9.
// S = 1, 2, own capacity 256, full prefixes: of 4096: 16x1 27.5 / 36.0, 64x1 96.9 / 116, 8x2 27.4 / 22.8, 64x2 120 / 125;  64 queries each: 64x1 324 / 402.
//
// What the estimates do not know is how long the prefixes are: where one is full and the others are short, the joint form takes its chain all the same.  So that
// may be up to twice what the shared form costs beside its bytes, where there is more than one prefix (a single one of 4096, 4 x 512 queries: 171 / 190).  One full prefix among
// 500 tokens each, and all full: 16x1 of 131072 694 / 70 and 840 / 704, of 8192 48.1 / 24.6 and 52.5 / 56.1;  128x1 of 8192 70.1 / 48.5 and 359 / 384, of 4096 49.8 / 47.1 and
// 189 / 213;  16 queries, 64x1 of 8192 146 / 49.9 and 236 / 259;  256 queries, 16x1 of 8192 248 / 162 and 563 / 657;  d 32, H 16/8, 16x1 of 32768 64.5 / 18.9 and 94.5 / 49.4;
// 16 queries of it, 16x1 of 8192 72.1 / 17.8 and 73.5 / 33.8 (small blocks take longer than their bytes).
bool joint_is_faster(const CacheForm& prefix, const CacheForm& own, double rows, double P, double S, double H_kv, int d, int prefix_blocks, int blocks) {
  const double wide = d / 128.0, megabytes = 128e-6 * d, segments = P * S * H_kv * own.tiles, all = prefix_blocks + blocks;
  auto busy = [&](const CacheForm& f, double number) { return number * wide * (f.KW == 4 ? 0.7 : f.RT == 1 ? 1.3 : 2.0) / 512; };
  const double chain = all * (own.KW == 4 ? std::max(0.33 * wide, 0.115) : own.RT == 1 ? 0.4 + 0.65 * wide : 0.6 + wide);
  const double begin = 12 + (own.KW == 4 ? 0 : 8) + wide * (1.5 + 0.006 * P * S * H_kv * std::ceil(rows / 16));        // parts of 16 rows: 32 KB through memory
  if (P > 1 && chain > 2 * begin) return false;
  const double once = P * H_kv * ((double)prefix_blocks + S * blocks) * megabytes;
  const double joint =
      4.5 + std::max(std::max(chain, segments * all * megabytes / 10.5), std::max(once / (S == 1 ? 6.2 : 5.2), own.KW == 4 ? 0.0 : busy(own, segments * all)));
  const double shared = begin + std::max(once / 6, busy(prefix, P * H_kv * prefix.tiles * prefix_blocks) + busy(own, segments * blocks));
  return joint < shared;
}
// Own segments of up to 16 rows have a work-group each where attn_cache_fwd's rule says so; up to four blocks, four heads have one (us, four heads / one: 16 x 8 of
// 1024, own 128: 25.3 / 29.5; of 4096, own 512: 58 / 55.5).  More rows are shared out (64 queries each of 2 x 8, prefixes of 8192, own 1024: 108 us, and 124 whole).
// Prefixes of more than 64 rows: two row tiles a wave where a share has ten blocks or so (256 rows of 8192: 39.8 us, and 31.9 with one; 128 of 131072: 60 and 66).
SharedForm shared_form(int P, int S, int H, int H_kv, int N, int d, int prefix_capacity, int capacity) {
  SharedForm f;
  const long long rows = (long long)N * (H / H_kv);
  const int room = d == 256 ? 256 : 512;   // as many work-groups run at once
  f.prefix = row_form(rows * S);
  f.own = cache_form(P * S, H, H_kv, N, d, capacity);
  if (f.prefix.RT == 2 && f.own.RT == 1 && cache_units(P, H_kv, f.prefix, prefix_capacity) < 10.0 * room) f.prefix.set_rows(rows * S, 1);
  f.heads = f.own.KW == 4 && H_kv >= 3 && (f.own.split || capacity <= 4 * kBlock);
  f.own_heads = f.heads ? (H_kv + 3) / 4 : H_kv;
  f.segments = (long long)P * H_kv * f.prefix.tiles;
  f.own_segments = (long long)P * S * f.own_heads * f.own.tiles;
  f.own_split = f.own.split || f.own.KW == 1 || f.own_segments > 1 << 20;
  f.shared = !joint_is_faster(f.prefix, f.own, (double)rows, P, S, H_kv, d, prefix_capacity / kBlock, capacity / kBlock);
  auto shares = [&](const CacheForm& form, bool heads, int B, int H_kv, int capacity) {
    return cache_units(B, H_kv, form, capacity, heads ? kHeadsStart : kStart) / (heads ? kLeast<1, true> : form.KW == 4 ? kLeast<4, false> : kLeast<1, false>);
  };
  const double most = shares(f.prefix, false, P, H_kv, prefix_capacity) + shares(f.own, f.heads, P * S, f.own_heads, capacity) + 16;
  f.groups = most >= room ? room : (int)most / 8 * 8;
  return f;
}
// What a unit costs a work-group, roughly: with as many running as fit, the block of a segment of up to 16 rows takes 0.7 us at d = 128, of 64 rows 1.3, of 128 rows 2.0.
// Few own segments are a matter of their chains' latency, and get twice the work-groups, or they would end after the prefixes' (16 answers about 131072 tokens:
// 59.8 us, and 64.8 without).
int unit_cost(const CacheForm& f, bool heads, bool few) { return heads ? 4 : f.KW == 4 ? (few ? 2 : 1) : f.RT == 1 ? 2 : 3; }

template <int D, int RT, int KW, int ORT, int OKW, bool HEADS> hipError_t launch_shared(const SharedArgs& a, const SharedForm& f, hipStream_t stream) {
  SharedPlan plan{};
  const AttendArgs& p = a.own;
  int* integers;
  {
    char* at = reinterpret_cast<char*>(p.partials);
    auto take = [&](size_t bytes) { char* x = at; at += bytes; return x; };
    auto floats = [&](size_t n) { return reinterpret_cast<float*>(take(n * sizeof(float))); };
    plan.prefixes.notes = reinterpret_cast<Join*>(take(f.segments * sizeof(Join)));
    plan.own.notes = reinterpret_cast<Join*>(take(f.own_segments * sizeof(Join)));
    plan.prefixes.slots = floats(2 * (size_t)f.groups * f.prefix.slot_floats(D));
    plan.prefixes.whole = floats((size_t)f.segments * f.prefix.slot_floats(D));
    plan.own.slots = floats(2 * (size_t)f.groups * f.slot_floats_own(D));
    plan.own.whole = floats((size_t)f.own_segments * f.slot_floats_own(D));
    integers = reinterpret_cast<int*>(at);
  }
  plan.prefix = p;
  plan.prefix.cache = a.prefix;
  plan.prefix.lengths = a.prefix_lengths;
  // Padded queries are left out of a prefix's rows, for a launch that finds where the real ones begin (5 us); with one query a sequence, those that have ended are not
  // worth it.
  const bool padded = p.counts && p.N > 1;
  plan.prefix.counts = padded ? integers + (size_t)a.P * a.S : nullptr;
  plan.prefix.B = a.P;
  plan.prefix.N = a.S * p.N;
  plan.prefix.causal = 0;
  plan.starts = padded ? integers : nullptr;
  plan.groups = f.groups;
  plan.own_split = f.own_split;
  plan.prefixes.heads = p.H_kv;
  plan.prefixes.tiles = f.prefix.tiles;
  plan.prefixes.cost = unit_cost(f.prefix, false, true);
  plan.own.heads = f.own_heads;
  plan.own.tiles = f.own.tiles;
  plan.own.cost = unit_cost(f.own, f.heads, f.own_segments < 256);
  const unsigned row_tiles = (unsigned)(((long long)a.S * p.N * p.group + 15) / 16);
  if (!grid_fits(row_tiles, 128)) return hipErrorInvalidConfiguration;     // (with more threads, there are fewer than 128 segments)
  if (padded) {
    attn_cache_starts_kernel<<<(unsigned)a.P, kAttendThreads, 0, stream>>>(p.counts, a.S, p.N, integers, integers + (size_t)a.P * a.S);
    if (const hipError_t e = hipGetLastError(); e != hipSuccess) return e;
  }
  attn_cache_shared_kernel<D, RT, KW, ORT, OKW, HEADS><<<(unsigned)(f.groups + (f.own_split ? 0 : f.own_segments)), kAttendThreads, 0, stream>>>(a, plan);
  if (const hipError_t e = hipGetLastError(); e != hipSuccess) return e;
  if (f.groups > 4 * f.segments)
    attn_cache_shared_merge_kernel<D, RT, KW, ORT, OKW, HEADS, 8, 2><<<dim3(row_tiles, (unsigned)(p.H_kv * (D / 32)), (unsigned)a.P), 512, 0, stream>>>(a, plan);
  else
    attn_cache_shared_merge_kernel<D, RT, KW, ORT, OKW, HEADS, 2, D / 16><<<dim3(row_tiles, (unsigned)p.H_kv, (unsigned)a.P), 128, 0, stream>>>(a, plan);
  return hipGetLastError();
}

template <int D, int RT, int KW> hipError_t launch_joint(const SharedArgs& a, const CacheForm& f, hipStream_t stream) {
  const AttendArgs& p = a.own;
  attn_cache_joint_kernel<D, RT, KW><<<dim3((unsigned)p.H_kv, (unsigned)f.tiles, (unsigned)p.B), kAttendThreads, 0, stream>>>(a, f.tiles);
  return hipGetLastError();
}
template <int D> hipError_t launch(const SharedArgs& a, hipStream_t stream) {
  const AttendArgs& p = a.own;
  const SharedForm f = shared_form(a.P, a.S, p.H, p.H_kv, p.N, D, a.prefix.capacity, p.cache.capacity);
  if (f.shared) {
    if (f.heads) {
      if (f.prefix.KW == 4) return launch_shared<D, 1, 4, 1, 1, true>(a, f, stream);
      if (f.prefix.RT == 1) return launch_shared<D, 1, 1, 1, 1, true>(a, f, stream);
      return launch_shared<D, 2, 1, 1, 1, true>(a, f, stream);
    }
    if (f.own.KW == 4) {
      if (f.prefix.KW == 4) return launch_shared<D, 1, 4, 1, 4, false>(a, f, stream);
      if (f.prefix.RT == 1) return launch_shared<D, 1, 1, 1, 4, false>(a, f, stream);
      return launch_shared<D, 2, 1, 1, 4, false>(a, f, stream);
    }
    if (f.own.RT == 1) return f.prefix.RT == 1 ? launch_shared<D, 1, 1, 1, 1, false>(a, f, stream) : launch_shared<D, 2, 1, 1, 1, false>(a, f, stream);
    return launch_shared<D, 2, 1, 2, 1, false>(a, f, stream);
  }
  if (f.own.KW == 4) return launch_joint<D, 1, 4>(a, f.own, stream);
  if (f.own.RT == 1) return launch_joint<D, 1, 1>(a, f.own, stream);
  return launch_joint<D, 2, 1>(a, f.own, stream);
}

}  // namespace

size_t attn_cache_fwd_shared_partial_bytes(int P, int S, int H, int H_kv, int N, int d, int prefix_capacity, int capacity) {
  return shared_form(P, S, H, H_kv, N, d, prefix_capacity, capacity).workspace_bytes(d, P, S);
}

hipError_t attn_cache_fwd_shared_dispatch(const SharedArgs& a, int d, hipStream_t stream) {
  switch (d) {
    case 32: return launch<32>(a, stream);
    case 64: return launch<64>(a, stream);
    case 96: return launch<96>(a, stream);
    case 128: return launch<128>(a, stream);
    default: return launch<256>(a, stream);
  }
}
