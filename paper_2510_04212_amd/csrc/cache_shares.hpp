// How the work of an attn_cache_fwd call is shared out, and which form of its kernels serves it.
//
// A call is a list of segments (sequence, key/value head, tile of query rows), in this order, of so many key blocks each, and
// `shares` work-groups take equal parts of all those blocks, wherever segments begin and end: sequences may differ in length
// by any factor, and lengths are known on the device only.  A part of a segment is left in the workspace, in slot 2w + 1 of share w where
// it begins the segment, 2w otherwise (a share ends inside one segment and begins inside one at most), and a second kernel
// joins the parts: the first share that begins inside a segment leaves a note for it (Join).  A segment that sees nothing counts as one block, so that somebody writes its rows.
//
// Plain C++ (host and device).
#pragma once
#include <stddef.h>

#ifdef __HIPCC__
#define SHARES_FN __host__ __device__ __forceinline__
#else
#define SHARES_FN inline
#endif

constexpr int kBlock = 64;                 // tokens that share a scale; the header's ATTN_CACHE_BLOCK

struct Problem {
  const int *lengths, *counts;             // counts may be NULL
  int capacity, N, group, causal, tiles, M;     // M rows (query * group + head of the group) per tile
  // of the N queries, those that sequence b really has
  SHARES_FN int count(int b) const {
    if (!counts) return N;
    const int c = counts[b];
    return c < 0 ? 0 : c > N ? N : c;
  }
  // key blocks that tile t of sequence b has to look at
  SHARES_FN int blocks(int b, int t) const {
    const int n = count(b), rows = n * group, first = t * M;
    if (first >= rows) return 0;
    const int last = (rows - first < M ? rows : first + M) - 1;
    const long long length = lengths[b], all = length < capacity ? length : capacity;
    long long seen = causal ? length - n + last / group + 1 : length;
    if (seen > all) seen = all;
    return seen > 0 ? (int)((seen + kBlock - 1) / kBlock) : 0;
  }
  SHARES_FN int cost(int b, int t) const {
    const int n = blocks(b, t);
    return n > 0 ? n : 1;
  }
};

struct Segment {
  int b, h, t;
  long long begin;                         // of its blocks in the whole list
  int blocks, cost;
};

// The segment that block `pos` of the list belongs to.  before(item): cost of the items (b, t), item = b * tiles + t, in front of
// one, for one head; it is called with 0 .. B * tiles.
template <class F> SHARES_FN Segment locate(const Problem& q, F&& before, int B, int H_kv, long long pos) {
  Segment s;
  s.b = 0;
  for (int hi = B; hi - s.b > 1;) {        // the last sequence that begins at or before pos
    const int mid = s.b + (hi - s.b) / 2;
    if (H_kv * before(mid * q.tiles) <= pos) s.b = mid; else hi = mid;
  }
  const long long first = before(s.b * q.tiles), each = before((s.b + 1) * q.tiles) - first;
  long long rest = pos - H_kv * first;
  s.h = (int)(rest / each);
  rest -= s.h * each;
  s.t = 0;
  for (int hi = q.tiles; hi - s.t > 1;) {
    const int mid = s.t + (hi - s.t) / 2;
    if (before(s.b * q.tiles + mid) - first <= rest) s.t = mid; else hi = mid;
  }
  s.begin = pos - (rest - (before(s.b * q.tiles + s.t) - first));
  s.blocks = q.blocks(s.b, s.t);
  s.cost = s.blocks > 0 ? s.blocks : 1;
  return s;
}
// The one behind it; there is one.
SHARES_FN void next_segment(const Problem& q, int H_kv, Segment& s) {
  s.begin += s.cost;
  if (++s.t == q.tiles) {
    s.t = 0;
    if (++s.h == H_kv) {
      s.h = 0;
      ++s.b;
    }
  }
  s.blocks = q.blocks(s.b, s.t);
  s.cost = s.blocks > 0 ? s.blocks : 1;
}

// Shares that `total` blocks are worth, and where share w begins.
SHARES_FN int shares_of(long long total, int most, int least_blocks) {
  const long long s = total / least_blocks;
  return s < 1 ? 1 : s > most ? most : (int)s;
}
SHARES_FN long long share_begin(long long total, int shares, int w) { return total * w / shares; }
// What share w >= 1, which begins in s, notes for the joining kernel: parts of s, in shares w - 1 and the following; 0 where it is not the
// first to begin inside s.  Note 0 holds the number of shares in `parts`.
struct alignas(16) Join { int b, h, t, parts; };
SHARES_FN Join join_of(long long total, int shares, int w, const Segment& s) {
  Join j{s.b, s.h, s.t, 0};
  if (w == 0) j.parts = shares;
  else if (s.begin < share_begin(total, shares, w) && share_begin(total, shares, w - 1) <= s.begin)
    j.parts = (int)(((s.begin + s.cost) * shares + total - 1) / total) - (w - 1);     // up to the first share that begins at its end or later
  return j;
}
// Slot of part i of them.
SHARES_FN int joined_slot(int w, int i) { return 2 * (w - 1 + i) + (i == 0 ? 1 : 0); }
// Share of a work-group, or -1: neighbours in the list go to one XCD (work-groups are dealt to the eight in turn), as they read the
// same head's cache.  The grid has a multiple of 8 work-groups, at least `shares`.
SHARES_FN int share_of(int group, int shares) {
  const int per = (shares + 7) / 8, w = (group & 7) * per + (group >> 3);
  return (group >> 3) < per && w < shares ? w : -1;
}

// ---- forms.  Four waves take 4 / KW groups of RT tiles of 16 rows, and KW shares of the key blocks of a group.
struct CacheForm {
  int RT, KW, tiles, shares;
  bool split;                              // shared out; otherwise a work-group per segment and nothing to join
  int rows() const { return 16 * RT * 4 / KW; }
  size_t slot_floats(int d) const { return (size_t)(4 / KW) * RT * (d / 16 * 256 + 32); }
  bool many_parts;                         // few segments for the shares: each is in many parts
  // notes, then slots
  size_t workspace_bytes(int d) const { return split && shares > 1 ? shares * sizeof(Join) + 2 * (size_t)shares * slot_floats(d) * sizeof(float) : 0; }
};
template <int KW> constexpr int kLeastBlocks = KW == 4 ? 4 : 8;
inline CacheForm cache_form(int B, int H, int H_kv, int N, int d, int capacity) {
  const long long rows = (long long)N * (H / H_kv);
  CacheForm f;
  f.RT = rows <= 16 ? 1 : 2;
  f.KW = rows <= 32 ? 4 : 1;
  f.tiles = (int)((rows + f.rows() - 1) / f.rows());
  const int nb = capacity / kBlock;
  f.split = nb > 16 || f.tiles > 65535;    // (the grid's second dimension)
  const double blocks = (double)B * H_kv * f.tiles * nb / (f.KW == 4 ? kLeastBlocks<4> : kLeastBlocks<1>);
  const int most = d == 256 ? 256 : 512;
  f.shares = blocks >= most ? most : blocks < 1 ? 1 : (int)blocks;
  f.many_parts = f.shares > 4.0 * B * H_kv * f.tiles;
  return f;
}
