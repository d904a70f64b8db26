// How the work of an attn_cache_fwd call is shared out, and which form of its kernels serves it.
//
// A call is a list of segments (sequence, key/value head, tile of query rows), in this order, of so many units of work each: kStart to
// begin and end one, then one for each of its key blocks.  `shares` work-groups take equal parts of all units, wherever segments begin and
// end: sequences may differ in length by any factor, and lengths are known on the device only.  A part of a segment is left in the
// workspace, in slot 2w + 1 of share w where it begins the segment, 2w otherwise (a share ends inside one segment and begins inside one at
// most), and a second kernel joins the parts, as the notes say that the shares leave for it (Join).
//
// Plain C++ (host and device).
#pragma once
#include <stddef.h>

#ifdef __HIPCC__
#define SHARES_FN __host__ __device__ __forceinline__
#else
#define SHARES_FN inline
#endif

// Reading the queries, filling the pipeline, joining the waves and storing takes a work-group about as long as kStart key blocks: without
// it, the shares of short sequences take longer than the others (one token of 64 sequences of 64 to 8192 tokens, H 32/8, d 128: 160 us
// at 0, 139 at 1, 121 at 3, 117 at 5 and at 8).
constexpr int kStart = 5;
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
  SHARES_FN int cost(int b, int t) const { return kStart + blocks(b, t); }
};

// Units of a call, counted in int: below this (where the entry point refuses the call), so that sums of two stay in range.
constexpr double kUnitLimit = 1073741824.0;

struct Segment {
  int b, h, t;
  int begin;                               // of its units in the whole list
  int blocks;
  SHARES_FN int end() const { return begin + kStart + blocks; }
  SHARES_FN int block_at(int pos) const {  // the first block at or behind a unit of it
    const int i = pos - begin - kStart;
    return i > 0 ? i : 0;
  }
};

// Does unit `pos` of the list belong to item (b, t) of some head?  Of the units of one head, `first` stand in front of sequence b, `each` are b's,
// and `at` of those stand in front of tile t.  If so, *s is the segment.  Exactly one item says yes: all are asked at once.
SHARES_FN bool locate(const Problem& q, int b, int t, int first, int each, int at, int H_kv, int pos, Segment* s) {
  int rest = pos - H_kv * first;
  if (rest < at || rest - at >= H_kv * each) return false;          // (not in front of the item in the first head, nor behind b)
  const int h = rest / each;
  rest -= h * each;
  const int blocks = q.blocks(b, t);
  if (rest < at || rest >= at + kStart + blocks) return false;
  *s = Segment{b, h, t, pos - (rest - at), blocks};
  return true;
}
// The one behind it; there is one.
SHARES_FN void next_segment(const Problem& q, int H_kv, Segment& s) {
  s.begin = s.end();
  if (++s.t == q.tiles) {
    s.t = 0;
    if (++s.h == H_kv) {
      s.h = 0;
      ++s.b;
    }
  }
  s.blocks = q.blocks(s.b, s.t);
}

// `total` units shared out: the first `longer` shares have one more than `each`.
struct Shares {
  int number, each, longer;
  SHARES_FN int begin(int w) const { return w * each + (w < longer ? w : longer); }
  // the first share that begins at or behind unit `pos`
  SHARES_FN int at_or_behind(int pos) const {
    const int edge = longer * (each + 1);
    return pos <= edge ? (pos + each) / (each + 1) : longer + (pos - edge + each - 1) / each;
  }
};
SHARES_FN Shares shares_of(int total, int most, int least) {
  const int n = total / least;
  Shares s;
  s.number = n < 1 ? 1 : n > most ? most : n;
  s.each = total / s.number;
  s.longer = total - s.each * s.number;
  return s;
}
// A note for the joining kernel: the segment's number in the list and its parts, in shares `first` and the following (none: it is whole).  Where segments
// are more than a quarter of the shares, there is one note for each share, of the segment that it begins inside if it is the first to do so, and
// note 0 holds the number of shares in `parts`; otherwise one for each segment, by the share that begins it.
struct alignas(16) Join { int segment, first, parts, unused; };
SHARES_FN int segment_number(const Segment& s, int H_kv, int tiles) { return (s.b * H_kv + s.h) * tiles + s.t; }
SHARES_FN Join note_of_share(const Shares& all, int w, const Segment& s, int H_kv, int tiles) {
  Join j{segment_number(s, H_kv, tiles), w - 1, 0, 0};
  if (w == 0) j.parts = all.number;
  else if (s.begin < all.begin(w) && all.begin(w - 1) <= s.begin) j.parts = all.at_or_behind(s.end()) - (w - 1);
  return j;
}
// share w begins s
SHARES_FN Join note_of_segment(const Shares& all, int w, const Segment& s, int H_kv, int tiles) {
  const int parts = all.at_or_behind(s.end()) - w;
  return Join{segment_number(s, H_kv, tiles), w, parts > 1 ? parts : 0, 0};
}
// Slot of part i.
SHARES_FN int joined_slot(int first, int i) { return 2 * (first + i) + (i == 0 ? 1 : 0); }
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
  size_t workspace_bytes(int d) const { return split ? shares * sizeof(Join) + 2 * (size_t)shares * slot_floats(d) * sizeof(float) : 0; }
};
// No share is smaller.  Four waves that share the blocks out: one block; sharing them: two (20 rows of 4 sequences of 1000 tokens, H 32/8, d 128: 24.7 us
// at eight blocks, 21.5 at four, 19.7 at two; 64 rows of 32768: 33.3, 28.7, 29.6; 8400 rows of 2100: 70.8, 73.6, 73.9).
template <int KW> constexpr int kLeastUnits = kStart + (KW == 4 ? 1 : 2);
inline double cache_units(int B, int H_kv, const CacheForm& f, int capacity) {
  return (double)B * H_kv * f.tiles * (kStart + capacity / kBlock);
}
// Figures come in pairs, both sides measured on the code of that step; later steps made both faster.
// Rows.  Up to 16: each wave takes blocks of its own (one token of 64 sequences of 4300, H 32/8, d 128: 102 us, and 116 with the blocks
// shared through LDS; of 4 sequences of 1000: 13 and 24).  From 17 on the blocks would be read and widened once for each row tile: the waves share
// them (32 rows of 64 x 4300: 132 us with blocks of a wave's own, 118 shared; 64 rows: 164 and 123).  From 65 on two row tiles a wave (68 rows:
// 284 us with one, 169 with two; 128 rows: 274 and 184).
//
// Split.  Sharing out costs 5 to 10 us (finding the segment, the second kernel) and pays where the longest segment alone takes longer than all bytes
// together, that is for few segments, long ones, and lengths far apart.  Whole / split, us, H 32/8:
//   up to 16 rows, a segment's length counted in blocks of 16 KB of d = 128: from 16 (few segments) over 28 to 64, the more segments there are.
//     d = 128, one token, capacity 1024: 1 sequence 8.8 / 14.8;  2048: 1 15.6 / 14.5, 16 15.3 / 22.7;  2112: 6 15.5 / 16.6, 24 20.7 / 30.5;  3008: 6 19.6 / 18.1,
//     12 19.8 / 24.7;  4096: 1 25.0 / 13.3, 12 28.9 / 30.5 (25.4 / 22.2 at lengths of 256 to 4096), 24 36.8 / 48.4 (30.4 / 32.0), 64 91 / 98 (60 / 66);
//     8192: 32 91 / 115 full, 61 / 61 ragged, 51 / 35 with one sequence in eight full.  d = 64, 4096: 4 12.1 / 15.3, 24 16.9 / 24.2
//   more rows, shared blocks: 16, 32 where there is a segment for every work-group that runs at once.  64 rows: 1024: 1 19 / 23;  2048: 4 33 / 24, 64 59 / 63;
//     4096: 4 61 / 28.  2048 queries of 2048 tokens 65 / 71, 4096 of 4096 197 / 175.
inline CacheForm cache_form(int B, int H, int H_kv, int N, int d, int capacity) {
  const long long rows = (long long)N * (H / H_kv);
  CacheForm f;
  f.RT = rows <= 64 ? 1 : 2;
  f.KW = rows <= 16 ? 4 : 1;
  f.tiles = (int)((rows + f.rows() - 1) / f.rows());
  const double most_shares = cache_units(B, H_kv, f, capacity) / (f.KW == 4 ? kLeastUnits<4> : kLeastUnits<1>);
  const int most = d == 256 ? 256 : 512;   // as many as run at once
  const double segments = (double)B * H_kv * f.tiles;
  const int nb = capacity / kBlock;
  bool whole = nb <= (f.KW == 1 && segments >= most ? 32 : 16);
  if (f.KW == 4 && segments >= most / 16) {
    const double limit = 28 + 102 * segments / most;
    whole = nb <= 64 && nb * (d / 128.0) <= (limit < 64 ? limit : 64);
  }
  f.split = !whole || f.tiles > 65535;     // (the grid's second dimension)
  f.shares = most_shares >= most ? most : most_shares < 1 ? 1 : (int)most_shares;
  f.many_parts = f.shares > 4 * segments;
  return f;
}
