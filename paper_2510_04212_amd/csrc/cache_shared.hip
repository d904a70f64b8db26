// Attention of sequences that continue prefixes they share with others (attn_cache_fwd_shared of include/attn.h).
#include "cache_attend.hpp"

namespace {

// Every segment reads its sequence's prefix, then its own blocks.
struct JointCall {
  static constexpr bool kJoint = true;
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
  attend<D, RT, KW, false>(call, q, work, Parts{});
}


// ---- shared: two lists of segments in one launch, the prefixes' (rows: all queries of a prefix's sequences, one after the other) and the sequences' own.
// The work-groups are dealt to the lists by their units, and every segment leaves its rows' sums, whole or in parts, for the joining kernel.
struct SharedPlan {
  AttendArgs prefix;                       // the prefixes as sequences: P of them, of S * N queries each
  int tiles, own_tiles, groups;            // work-groups: a multiple of 8, 16 at least
  Join *notes, *own_notes;                 // one for each segment
  float *slots, *own_slots;                // parts of segments: two for each work-group
  float *whole, *own_whole;                // whole segments
};

// Segments whose rows are joined later.
template <int SLOT> struct ListCall {
  static constexpr bool kJoint = false;
  const AttendArgs& p;
  int N;                                   // queries of a sequence
  int S;                                   // sequences of a list's item, one after the other
  float* whole;
  DEVI const unsigned short* query(int b, int head, int query) const {
    const int s = S == 1 ? 0 : query / N;
    return p.Q.at + ((long long)b * S + s) * p.Q.sb + head * p.Q.sh + (query - s * N) * p.Q.sn;
  }
  template <int DT, int M> DEVI void store(const Segment& s, int tile, const f32x4* o, float m, float l, int dt0, int lane) const {
    const int r = lane & 15;
    if (s.t * M + tile * 16 + r >= p.N * p.group) return;
    constexpr int DTILES = (SLOT / (M / 16) - 32) / 256;
    float* slot = whole + (size_t)segment_number(s, p.H_kv, (p.N * p.group + M - 1) / M) * SLOT;
#pragma unroll
    for (int i = 0; i < DT; ++i) reinterpret_cast<f32x4*>(slot)[(tile * DTILES + dt0 + i) * 64 + lane] = o[i];
    float* ml = slot + M / 16 * DTILES * 256 + tile * 32;
    if (lane < 16 && dt0 == 0) {
      ml[r] = m;
      ml[16 + r] = l;
    }
  }
};

template <int D, int RT, int KW, int ORT, int OKW>
__global__ __launch_bounds__(kAttendThreads, D == 256 ? 1 : 2) void attn_cache_shared_kernel(SharedArgs a, SharedPlan plan) {
  __shared__ Runs runs, own_runs;
  const AttendArgs &p = plan.prefix, &o = a.own;
  const Problem q{p.lengths, nullptr, p.cache.capacity, p.N, p.group, 0, plan.tiles, 16 * RT * 4 / KW};
  const Problem own{o.lengths, o.counts, o.cache.capacity, o.N, o.group, o.causal, plan.own_tiles, 16 * ORT * 4 / OKW};
  const int run = (p.B * q.tiles + kAttendThreads - 1) / kAttendThreads, own_run = (o.B * own.tiles + kAttendThreads - 1) / kAttendThreads;
  const int units = p.H_kv * scan_units(q, p.B * q.tiles, run, runs), own_units = o.H_kv * scan_units(own, o.B * own.tiles, own_run, own_runs);
  const int eighths = plan.groups / 8;
  const int groups = 8 * uniform(min(max((int)((long long)eighths * units / (units + own_units)), 1), eighths - 1));
  auto begin = [&](const Problem& problem, int B, int total, int most, int least, int runs_of, Runs& runs, int group, Work& work) {
    work.all = shares_of(total, most, least);
    work.w = share_of(group, work.all.number);
    if (work.w < 0) return false;
    work.pos = uniform(work.all.begin(work.w));
    work.end = uniform(work.all.begin(work.w + 1));
    work.seg = find_segment(problem, B, p.H_kv, runs_of, work.pos, runs);
    work.seg.blocks = uniform(work.seg.blocks);
    return true;
  };
  Work work;
  if ((int)blockIdx.x < groups) {
    constexpr int SLOT = kSlotFloats<D, RT, KW>;
    if (!begin(q, p.B, units, groups, kLeastUnits<KW>, run, runs, blockIdx.x, work)) return;
    attend<D, RT, KW, true>(ListCall<SLOT>{p, o.N, a.S, plan.whole}, q, work, Parts{plan.notes, plan.slots, true});
  } else {
    constexpr int SLOT = kSlotFloats<D, ORT, OKW>;
    if (!begin(own, o.B, own_units, plan.groups - groups, kLeastUnits<OKW>, own_run, own_runs, blockIdx.x - groups, work)) return;
    attend<D, ORT, OKW, true>(ListCall<SLOT>{o, o.N, 1, plan.own_whole}, own, work, Parts{plan.own_notes, plan.own_slots, true});
  }
}

// Joins a row's parts: those of its prefix's segment and those of its own.  blockIdx: 16 rows of a prefix's list; DT of the D / 16 column tiles, and the head; the prefix.
template <int D, int RT, int KW, int ORT, int OKW, int NW, int DT>
__global__ __launch_bounds__(64 * NW) void attn_cache_shared_merge_kernel(SharedArgs a, SharedPlan plan) {
  constexpr int M = 16 * RT * 4 / KW, OM = 16 * ORT * 4 / OKW, SLOT = kSlotFloats<D, RT, KW>, OSLOT = kSlotFloats<D, ORT, OKW>;
  constexpr int PARTS = D / 16 / DT;
  __shared__ f32x4 joined[NW][DT][64];
  __shared__ float joined_ml[2][NW][16];
  const AttendArgs& p = a.own;
  const int lane = threadIdx.x & 63, wave = uniform((int)(threadIdx.x >> 6));
  const int r = lane & 15, g = lane >> 4;
  const int h = blockIdx.y / PARTS, dt0 = blockIdx.y % PARTS * DT, item = blockIdx.z;
  const int row0 = blockIdx.x * 16, t = row0 / M, tile = row0 % M / 16;
  const int own_rows = p.N * p.group, row = min(row0 + r, a.S * own_rows - 1);
  const int s = row / own_rows, own_row = row - s * own_rows, b = item * a.S + s;

  f32x4 o[DT];
  float m = -INFINITY, l = 0.f;
#pragma unroll
  for (int i = 0; i < DT; ++i) o[i] = f32x4{0, 0, 0, 0};
  // one more part: its tile of a slot, the row's lane in it
  auto add = [&](const float* slot, int tiles, int tile, int at, bool there) {
    f32x4 x[DT];
    float mp = -INFINITY, lp = 0.f;
#pragma unroll
    for (int i = 0; i < DT; ++i) x[i] = f32x4{0, 0, 0, 0};
    if (there) {
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
  };
  const int segment = (item * p.H_kv + h) * plan.tiles + t;
  const Join j = plan.notes[segment];
  if (j.parts == 0) {
    if (wave == 0) add(plan.whole + (size_t)segment * SLOT, M / 16, tile, r, true);
  } else {
    for (int part = wave; part < j.parts; part += NW) add(plan.slots + (size_t)joined_slot(j.first, part) * SLOT, M / 16, tile, r, true);
  }
  const int own_segment = (b * p.H_kv + h) * plan.own_tiles + own_row / OM, own_tile = own_row % OM / 16;
  const Join k = plan.own_notes[own_segment];
  const int parts = k.parts == 0 ? 1 : k.parts;
  for (int part = NW - 1 - wave; __any(part < parts); part += NW)        // (the waves without a prefix's part first)
    add(k.parts == 0 ? plan.own_whole + (size_t)own_segment * OSLOT : plan.own_slots + (size_t)joined_slot(k.first, part) * OSLOT, OM / 16, own_tile, own_row & 15,
        part < parts);

  if (g == 0) { joined_ml[0][wave][r] = m; joined_ml[1][wave][r] = l; }
#pragma unroll
  for (int i = 0; i < DT; ++i) joined[wave][i][lane] = o[i];
  __syncthreads();
  if (wave != 0 || row0 + r >= a.S * own_rows) return;
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
  bool shared;
  int groups;
  long long segments, own_segments;
  // notes, parts, whole segments
  size_t workspace_bytes(int d) const {
    if (!shared) return 0;
    const size_t slot = prefix.slot_floats(d) * sizeof(float), own_slot = own.slot_floats(d) * sizeof(float);
    return (size_t)(segments + own_segments) * sizeof(Join) + (2 * (size_t)groups + segments) * slot + (2 * (size_t)groups + own_segments) * own_slot;
  }
};
SharedForm shared_form(int P, int S, int H, int H_kv, int N, int d, int prefix_capacity, int capacity) {
  SharedForm f;
  const long long rows = (long long)N * (H / H_kv);
  f.prefix = row_form(rows * S);
  f.own = row_form(rows);
  f.segments = (long long)P * H_kv * f.prefix.tiles;
  f.own_segments = (long long)P * S * H_kv * f.own.tiles;
  f.shared = true;
  auto shares = [](const CacheForm& form, double units) { return units / (form.KW == 4 ? kLeastUnits<4> : kLeastUnits<1>); };
  const double most = shares(f.prefix, cache_units(P, H_kv, f.prefix, prefix_capacity)) + shares(f.own, cache_units(P * S, H_kv, f.own, capacity)) + 16;
  const int room = d == 256 ? 256 : 512;   // as many as run at once
  f.groups = most >= room ? room : (int)most / 8 * 8;
  return f;
}

template <int D, int RT, int KW, int ORT, int OKW> hipError_t launch_shared(const SharedArgs& a, const SharedForm& f, hipStream_t stream) {
  SharedPlan plan{};
  const AttendArgs& p = a.own;
  plan.prefix = p;
  plan.prefix.cache = a.prefix;
  plan.prefix.lengths = a.prefix_lengths;
  plan.prefix.counts = nullptr;
  plan.prefix.B = a.P;
  plan.prefix.N = a.S * p.N;
  plan.prefix.causal = 0;
  plan.tiles = f.prefix.tiles;
  plan.own_tiles = f.own.tiles;
  plan.groups = f.groups;
  plan.notes = reinterpret_cast<Join*>(p.partials);
  plan.own_notes = plan.notes + f.segments;
  plan.slots = reinterpret_cast<float*>(plan.own_notes + f.own_segments);
  plan.whole = plan.slots + 2 * (size_t)f.groups * f.prefix.slot_floats(D);
  plan.own_slots = plan.whole + (size_t)f.segments * f.prefix.slot_floats(D);
  plan.own_whole = plan.own_slots + 2 * (size_t)f.groups * f.own.slot_floats(D);
  const unsigned row_tiles = (unsigned)(((long long)a.S * p.N * p.group + 15) / 16);
  if (!grid_fits(row_tiles, 128)) return hipErrorInvalidConfiguration;     // (with more threads, there are fewer than 128 segments)
  attn_cache_shared_kernel<D, RT, KW, ORT, OKW><<<(unsigned)f.groups, kAttendThreads, 0, stream>>>(a, plan);
  if (const hipError_t e = hipGetLastError(); e != hipSuccess) return e;
  if (f.groups > 4 * f.segments)
    attn_cache_shared_merge_kernel<D, RT, KW, ORT, OKW, 16, 2><<<dim3(row_tiles, (unsigned)(p.H_kv * (D / 32)), (unsigned)a.P), 1024, 0, stream>>>(a, plan);
  else
    attn_cache_shared_merge_kernel<D, RT, KW, ORT, OKW, 2, D / 16><<<dim3(row_tiles, (unsigned)p.H_kv, (unsigned)a.P), 128, 0, stream>>>(a, plan);
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
    if (f.own.KW == 4) {
      if (f.prefix.KW == 4) return launch_shared<D, 1, 4, 1, 4>(a, f, stream);
      if (f.prefix.RT == 1) return launch_shared<D, 1, 1, 1, 4>(a, f, stream);
      return launch_shared<D, 2, 1, 1, 4>(a, f, stream);
    }
    if (f.own.RT == 1) return f.prefix.RT == 1 ? launch_shared<D, 1, 1, 1, 1>(a, f, stream) : launch_shared<D, 2, 1, 1, 1>(a, f, stream);
    return launch_shared<D, 2, 1, 2, 1>(a, f, stream);
  }
  if (f.own.tiles > 65535) return hipErrorInvalidConfiguration;
  if (f.own.KW == 4) return launch_joint<D, 1, 4>(a, f.own, stream);
  if (f.own.RT == 1) return launch_joint<D, 1, 1>(a, f.own, stream);
  return launch_joint<D, 2, 1>(a, f.own, stream);
}

}  // namespace

size_t attn_cache_fwd_shared_partial_bytes(int P, int S, int H, int H_kv, int N, int d, int prefix_capacity, int capacity) {
  return shared_form(P, S, H, H_kv, N, d, prefix_capacity, capacity).workspace_bytes(d);
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
