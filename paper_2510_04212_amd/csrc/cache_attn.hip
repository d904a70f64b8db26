// Attention over the 8-bit cache (attn_cache_fwd of include/attn.h) and the attention weight that each cached token got
// (attn_cache_weights).
#include "cache_attend.hpp"
#include <algorithm>
#include <cmath>

namespace {

constexpr int kThreads = kAttendThreads;

// Many rows whose segments are whole, of 32 blocks at most (cache_form): attend's loop over staged blocks with nothing to share out or to join, and a segment's scales in
// one load.  2048 queries of 4 sequences of 2048 tokens, H 16/8, d 32 and 64, 32/8, 96 and 128, 16/4, 256: 70.0, 70.3, 152, 171 and 259 us, and 73.2, 74.1, 155, 178 and 264
// as an instance of attend.
template <int D, int RT>
__global__ __launch_bounds__(kThreads, D == 256 ? 1 : 2) void attn_cache_whole_kernel(AttendArgs p, int tiles) {
  constexpr int M = 64 * RT;
  __shared__ __attribute__((aligned(1024))) char staged[2 * Staged<D>::kBytes];
  const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6);
  const int r = lane & 15, g = lane >> 4;
  const Problem q{p.lengths, p.counts, p.cache.capacity, p.N, p.group, p.causal, tiles, M};
  const int nb = p.cache.capacity / kBlock;
  const float scale_log2 = p.scale * kLog2e;
  const int b = blockIdx.z, h = blockIdx.x, t = blockIdx.y, first_row = t * M + wave * RT * 16;
  // (the compiler knows nothing of a copy's range, and orders the loop less well then: d 256 259 us, and 262 with the copy alone)
  const int counted = q.blocks(b, t), blocks = max(min(counted, uniform(counted)), 0);
  const size_t bh = (size_t)b * p.H_kv + h;
  const unsigned char* K = p.cache.K + bh * p.cache.capacity * D;
  const unsigned char* V = p.cache.V + bh * p.cache.capacity * D;
  const float* Ks = p.cache.K_scale + bh * nb;
  const float* Vs = p.cache.V_scale + bh * nb;
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
  constexpr int MINE = Staged<D>::PIECES / 4;              // a wave fetches every fourth piece
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
  float k_scales = 0.f, v_scales = 0.f;    // one block's in each lane
  if (blocks > 0) {
    fetch(0, 0);
    k_scales = Ks[min(lane, nb - 1)];
    v_scales = Vs[min(lane, nb - 1)];
    settle(k_scales);
    settle(v_scales);
  }
  // what the compiler has loaded is settled in front of the loop, as in attend
#pragma unroll
  for (int rt = 0; rt < RT; ++rt)
#pragma unroll
    for (int c = 0; c < D / 32; ++c) settle(qf[rt][c]);
  KCodes<D> k;
  int buffer = 0;
  for (int blk = 0; blk < blocks; ++blk) {
    wait_vmem();
    __syncthreads();                                       // this block has landed for all waves, and all have read the one before
    if (blk + 1 < blocks) fetch(blk + 1, buffer ^ 1);
    if (rows_here) {
      const float ks = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(k_scales), blk));
      const float vs = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(v_scales), blk));
      const int base = (int)buffers + buffer * Staged<D>::kBytes;
      VCodes<D> v;
      read_staged<D>(k, base + in_piece, base + in_odd);
      block_step<D, RT>(a, qf, k, v, ks, vs, scale_log2, limit, blk * kBlock + kBlock > least, blk * kBlock, g,
                        [&] { read_staged<D>(v, base + in_piece); });
    }
    buffer ^= 1;
  }
  a.join_groups();
  auto put = [&](int tile, const f32x4* o, float m, float l) {
    store_row<D / 16>(p, find_row(p, b, t * M + tile * 16 + r), b, h, o, m, l, 0, g);
  };
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) put(wave * RT + rt, a.o[rt], a.m[rt], a.l[rt]);
}

// SPLIT: shares of the list of blocks; otherwise (up to 16 rows) one segment per work-group (blockIdx: head, tile, sequence), nothing to merge.
template <int D, int RT, int KW, bool SPLIT>
__global__ __launch_bounds__(kThreads, D == 256 ? 1 : 2) void attn_cache_fwd_kernel(AttendArgs p, int tiles, int most_shares, bool notes_by_segment) {
  __shared__ __attribute__((aligned(1024))) char staged[kAttendBytes<D, RT, KW>];
  __shared__ Runs runs;
  const Problem q{p.lengths, p.counts, p.cache.capacity, p.N, p.group, p.causal, tiles, 16 * RT * 4 / KW};
  const PlainCall call{p};
  Work work{{}, 0, 0, 0, {1, 0, 0}};
  Parts parts{reinterpret_cast<Join*>(p.partials), p.partials + most_shares * (sizeof(Join) / sizeof(float)), notes_by_segment};
  if constexpr (SPLIT) {
    const int items = p.B * tiles, run = (items + kThreads - 1) / kThreads;
    work.all = shares_of(p.H_kv * scan_units(q, items, run, runs), most_shares, kLeastUnits<KW>);
    work.w = share_of(blockIdx.x, work.all.number);
    if (work.w < 0) return;
    work.pos = uniform(work.all.begin(work.w));
    work.end = uniform(work.all.begin(work.w + 1));
    work.seg = find_segment(q, p.B, p.H_kv, run, work.pos, runs);
    if (threadIdx.x == 0 && !notes_by_segment) parts.notes[work.w] = note_of_share(work.all, work.w, work.seg, p.H_kv, tiles);
  } else {
    work.seg.b = blockIdx.z;
    work.seg.h = blockIdx.x;
    work.seg.t = blockIdx.y;
    work.seg.begin = 0;
    work.seg.blocks = q.blocks(work.seg.b, work.seg.t);
    work.end = work.seg.end();
  }
  work.seg.blocks = uniform(work.seg.blocks);
  attend<D, RT, KW, SPLIT>(call, q, work, parts, staged);
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
    const dim3 grid((unsigned)p.H_kv, (unsigned)f.tiles, (unsigned)p.B);
    if constexpr (KW == 1) attn_cache_whole_kernel<D, RT><<<grid, kThreads, 0, stream>>>(p, f.tiles);
    else attn_cache_fwd_kernel<D, RT, KW, false><<<grid, kThreads, 0, stream>>>(p, f.tiles, 0, false);
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
