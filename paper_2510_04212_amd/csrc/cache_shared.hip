// Attention of sequences that continue prefixes they share with others (attn_cache_fwd_shared of include/attn.h).
#include "cache_attend.hpp"

namespace {

// Every segment reads its sequence's prefix, then its own blocks.
struct JointCall {
  static constexpr bool kJoint = true, kHeads = false;
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
// own.  The work-groups are dealt to the lists by what their units cost, and every segment leaves its rows' sums, whole or in parts, for the joining kernel.
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
  const int* starts;                       // [P * S]: real queries of its prefix's sequences in front of this one; NULL: all are real
  int groups;                              // work-groups: a multiple of 8, 16 at least
  List prefixes, own;
};

// 16-row tiles of a slot: sums of their rows, then maxima and sums of probabilities
template <int D> constexpr int kTileFloats = D / 16 * 256 + 32;

template <int D, int TILES, bool PREFIX, bool HEADS> struct ListCall {
  static constexpr bool kJoint = false, kHeads = HEADS;
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
  const Problem own{o.lengths, o.counts, o.cache.capacity, o.N, o.group, o.causal, plan.own.tiles, HEADS ? 16 : 16 * ORT * 4 / OKW};
  const int run = (p.B * q.tiles + kAttendThreads - 1) / kAttendThreads, own_run = (o.B * own.tiles + kAttendThreads - 1) / kAttendThreads;
  const int units = plan.prefixes.heads * scan_units(q, p.B * q.tiles, run, runs), own_units = plan.own.heads * scan_units(own, o.B * own.tiles, own_run, own_runs);
  const int eighths = plan.groups / 8;
  const long long cost = (long long)units * plan.prefixes.cost, own_cost = (long long)own_units * plan.own.cost;
  const int groups = 8 * uniform(min(max((int)((eighths * cost + (cost + own_cost) / 2) / (cost + own_cost)), 1), eighths - 1));
  auto begin = [&](const Problem& problem, const List& list, int B, int total, int most, int least, int runs_of, Runs& runs, int group, Work& work) {
    work.all = shares_of(total, most, least);
    work.w = share_of(group, work.all.number);
    if (work.w < 0) return false;
    work.pos = uniform(work.all.begin(work.w));
    work.end = uniform(work.all.begin(work.w + 1));
    work.seg = find_segment(problem, B, list.heads, runs_of, work.pos, runs);
    work.seg.blocks = uniform(work.seg.blocks);
    return true;
  };
  Work work;
  if ((int)blockIdx.x < groups) {
    if (!begin(q, plan.prefixes, p.B, units, groups, kLeastUnits<KW>, run, runs, blockIdx.x, work)) return;
    attend<D, RT, KW, true>(ListCall<D, RT * 4 / KW, true, false>{p, plan, o.N, a.S}, q, work, Parts{plan.prefixes.notes, plan.prefixes.slots, true}, staged);
  } else {
    if (!begin(own, plan.own, o.B, own_units, plan.groups - groups, kLeastUnits<OKW>, own_run, own_runs, blockIdx.x - groups, work)) return;
    attend<D, ORT, OKW, true>(ListCall<D, ORT * 4 / OKW, false, HEADS>{o, plan, 0, 0}, own, work, Parts{plan.own.notes, plan.own.slots, true}, staged);
  }
}

// Joins a row's parts: those of its prefix's segment and those of its own.  blockIdx: 16 rows of a prefix's sequences, padding included; the head, and DT of
// the D / 16 column tiles; the prefix.  NW waves take every NW-th part and join theirs in LDS.
template <int D, int RT, int KW, int ORT, int OKW, bool HEADS, int NW, int DT>
__global__ __launch_bounds__(64 * NW) void attn_cache_shared_merge_kernel(SharedArgs a, SharedPlan plan) {
  constexpr int TILES = RT * 4 / KW, OTILES = ORT * 4 / OKW, PARTS = D / 16 / DT;
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

  f32x4 o[DT];
  float m = -INFINITY, l = 0.f;
#pragma unroll
  for (int i = 0; i < DT; ++i) o[i] = f32x4{0, 0, 0, 0};
  // the parts of row `at` of a list's segment, in its 16-row tile `tile`
  auto add = [&](const List& list, int tiles, int segment, int tile, int at, int first) {
    Join j{0, 0, 0, 0};
    if (real) j = list.notes[segment];
    const int parts = !real ? 0 : j.parts == 0 ? 1 : j.parts;
    for (int part = first; __any(part < parts); part += NW) {
      const float* slot = j.parts == 0 ? list.whole + (size_t)segment * (tiles * kTileFloats<D>)
                                       : list.slots + (size_t)joined_slot(j.first, part) * (tiles * kTileFloats<D>);
      f32x4 x[DT];
      float mp = -INFINITY, lp = 0.f;
#pragma unroll
      for (int i = 0; i < DT; ++i) x[i] = f32x4{0, 0, 0, 0};
      if (part < parts) {
#pragma unroll
        for (int i = 0; i < DT; ++i) x[i] = reinterpret_cast<const f32x4*>(slot)[(tile * (D / 16) + dt0 + i) * 64 + 16 * g + at];
        const float* ml = slot + tiles * (D / 16 * 256) + tile * 32;
        mp = ml[at];
        lp = ml[16 + at];
      }
      const float most = fmaxf(m, mp), use = most == -INFINITY ? 0.f : most;
      const float mine = __builtin_amdgcn_exp2f(m - use), theirs = __builtin_amdgcn_exp2f(mp - use);
      l = l * mine + lp * theirs;
#pragma unroll
      for (int i = 0; i < DT; ++i) o[i] = o[i] * mine + x[i] * theirs;
      m = most;
    }
  };
  const int t = in_prefix / (16 * TILES), at = in_prefix % (16 * TILES);
  add(plan.prefixes, TILES, plan.prefixes.segment(item, h, t), at / 16, at % 16, wave);
  constexpr int OM = HEADS ? 16 : 16 * OTILES;             // (the waves without a prefix's part first)
  add(plan.own, OTILES, plan.own.segment(b, HEADS ? h / 4 : h, own_row / OM), HEADS ? h % 4 : own_row % OM / 16, own_row % 16, NW - 1 - wave);

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
  bool shared, heads;                      // heads: four key/value heads of a sequence's own make a segment
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
SharedForm shared_form(int P, int S, int H, int H_kv, int N, int d, int prefix_capacity, int capacity) {
  SharedForm f;
  const long long rows = (long long)N * (H / H_kv);
  f.prefix = row_form(rows * S);
  f.own = row_form(rows);
  f.heads = f.own.KW == 4 && H_kv >= 3;
  f.own_heads = f.heads ? (H_kv + 3) / 4 : H_kv;
  f.segments = (long long)P * H_kv * f.prefix.tiles;
  f.own_segments = (long long)P * S * f.own_heads * f.own.tiles;
  f.shared = true;
  auto shares = [](const CacheForm& form, bool heads, double units) { return units / (form.KW == 4 && !heads ? kLeastUnits<4> : kLeastUnits<1>); };
  const double most = shares(f.prefix, false, cache_units(P, H_kv, f.prefix, prefix_capacity)) + shares(f.own, f.heads, cache_units(P * S, f.own_heads, f.own, capacity)) + 16;
  const int room = d == 256 ? 256 : 512;   // as many as run at once
  f.groups = most >= room ? room : (int)most / 8 * 8;
  return f;
}
int unit_cost(const CacheForm& f, bool heads) { return heads ? 4 : f.KW == 4 ? 2 : f.RT == 1 ? 2 : 3; }

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
  plan.prefix.counts = p.counts ? integers + (size_t)a.P * a.S : nullptr;
  plan.prefix.B = a.P;
  plan.prefix.N = a.S * p.N;
  plan.prefix.causal = 0;
  plan.starts = p.counts ? integers : nullptr;
  plan.groups = f.groups;
  plan.prefixes.heads = p.H_kv;
  plan.prefixes.tiles = f.prefix.tiles;
  plan.prefixes.cost = unit_cost(f.prefix, false);
  plan.own.heads = f.own_heads;
  plan.own.tiles = f.own.tiles;
  plan.own.cost = unit_cost(f.own, f.heads);
  const unsigned row_tiles = (unsigned)(((long long)a.S * p.N * p.group + 15) / 16);
  if (!grid_fits(row_tiles, 128)) return hipErrorInvalidConfiguration;     // (with more threads, there are fewer than 128 segments)
  if (p.counts) {
    attn_cache_starts_kernel<<<(unsigned)a.P, kAttendThreads, 0, stream>>>(p.counts, a.S, p.N, integers, integers + (size_t)a.P * a.S);
    if (const hipError_t e = hipGetLastError(); e != hipSuccess) return e;
  }
  attn_cache_shared_kernel<D, RT, KW, ORT, OKW, HEADS><<<(unsigned)f.groups, kAttendThreads, 0, stream>>>(a, plan);
  if (const hipError_t e = hipGetLastError(); e != hipSuccess) return e;
  if (f.groups > 4 * f.segments)
    attn_cache_shared_merge_kernel<D, RT, KW, ORT, OKW, HEADS, 16, 2><<<dim3(row_tiles, (unsigned)(p.H_kv * (D / 32)), (unsigned)a.P), 1024, 0, stream>>>(a, plan);
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
  if (f.own.tiles > 65535) return hipErrorInvalidConfiguration;
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
