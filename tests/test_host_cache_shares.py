"""CPU-only check of how a call over the 8-bit cache is shared out (csrc/cache_shares.hpp), compiled with g++: every key block of every
segment is taken once, parts go to slots of their own, and the part that joins a segment is found once."""
import os
import random
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER_DIR = os.path.join(ROOT, "paper_2510_04212_amd", "csrc")

MAIN = r"""
#include "cache_shares.hpp"
#include <cstdio>
#include <cstdlib>
#include <map>
#include <tuple>
#include <vector>
// stdin: B H_kv N group causal capacity M most least, then B lengths, then B counts (-9: none)
int main() {
  int B, H, N, group, causal, capacity, M, most, least;
  while (scanf("%d %d %d %d %d %d %d %d %d", &B, &H, &N, &group, &causal, &capacity, &M, &most, &least) == 9) {
    std::vector<int> lengths(B), counts(B);
    for (int& x : lengths) scanf("%d", &x);
    for (int& x : counts) scanf("%d", &x);
    const int tiles = (N * group + M - 1) / M;
    const Problem q{lengths.data(), counts[0] == -9 ? nullptr : counts.data(), capacity, N, group, causal, tiles, M};
    std::vector<int> sums{0};
    for (int i = 0; i < B * tiles; ++i) sums.push_back(sums.back() + q.cost(i / tiles, i % tiles));
    auto locate_one = [&](int pos) {
      Segment found{-1, 0, 0, 0, 0};
      int times = 0;
      for (int i = 0; i < B * tiles; ++i) {
        const int b = i / tiles, first = sums.at(b * tiles);
        Segment s;
        if (locate(q, b, i % tiles, first, sums.at((b + 1) * tiles) - first, sums[i] - first, H, pos, &s)) { found = s; ++times; }
      }
      if (times != 1) { printf("found %d times\n", times); exit(1); }
      return found;
    };
    const int total = H * sums.back();
    const Shares all = shares_of(total, most, least);
    const int shares = all.number;
    if (shares < 1 || shares > most || all.begin(0) != 0 || all.begin(shares) != total) { printf("shares\n"); return 1; }
    for (int pos = 0; pos <= total; pos += 1 + total / 1000) {
      const int s = all.at_or_behind(pos);
      if (s < 0 || s > shares || all.begin(s) < pos || (s > 0 && all.begin(s - 1) >= pos)) { printf("at or behind\n"); return 1; }
    }
    std::vector<int> seen(shares, 0);
    for (int g = 0; g < (shares + 7) / 8 * 8; ++g)
      if (const int w = share_of(g, shares); w >= 0) ++seen.at(w);
    for (int x : seen) if (x != 1) { printf("share taken %d times\n", x); return 1; }
    std::map<std::tuple<int, int, int>, std::vector<std::pair<int, int>>> parts;      // segment -> [from, to)
    std::map<std::tuple<int, int, int>, std::vector<int>> slots;
    std::vector<int> used(2 * shares, 0);
    for (int w = 0; w < shares; ++w) {
      int pos = all.begin(w);
      const int end = all.begin(w + 1);
      if (end <= pos) { printf("empty share\n"); return 1; }
      Segment s = locate_one(pos);
      while (true) {
        if (s.b >= B || s.h >= H || s.t >= tiles || s.begin > pos || s.end() <= pos) { printf("wrong segment\n"); return 1; }
        if (s.blocks != q.blocks(s.b, s.t) || s.blocks > capacity / kBlock) { printf("wrong blocks\n"); return 1; }
        const int to = end < s.end() ? end : s.end();
        const auto key = std::make_tuple(s.b, s.h, s.t);
        parts[key].push_back({s.block_at(pos), s.block_at(to)});
        if (pos != s.begin || to != s.end()) {
          const int slot = 2 * w + (pos == s.begin ? 1 : 0);
          ++used.at(slot);
          slots[key].push_back(slot);
        }
        pos = to;
        if (pos >= end) break;
        next_segment(q, H, s);
      }
    }
    for (int x : used) if (x > 1) { printf("slot used twice\n"); return 1; }
    if ((long long)parts.size() != (long long)B * H * tiles) { printf("segments missing\n"); return 1; }
    for (auto& [key, list] : parts) {
      int at = 0;
      for (auto [from, to] : list) { if (from != at || to < from) { printf("hole\n"); return 1; } at = to; }
      if (at != q.blocks(std::get<0>(key), std::get<2>(key))) { printf("end missing\n"); return 1; }
    }
    // the joining kernel's view: the notes of shares 1 .., and those of all segments
    auto key_of = [&](int number) { return std::make_tuple(number / tiles / H, number / tiles % H, number % tiles); };
    std::map<std::tuple<int, int, int>, int> joined;
    auto check = [&](const Join& j) {
      ++joined[key_of(j.segment)];
      std::vector<int> mine;
      for (int i = 0; i < j.parts; ++i) mine.push_back(joined_slot(j.first, i));
      if (mine != slots[key_of(j.segment)]) { printf("other parts joined\n"); exit(1); }
    };
    std::map<std::tuple<int, int, int>, Join> of_segment;
    for (int w = 0; w < shares; ++w) {
      int pos = all.begin(w);
      const int end = all.begin(w + 1);
      Segment s = locate_one(pos);
      const Join j = note_of_share(all, w, s, H, tiles);
      if (w == 0 && j.parts != shares) { printf("first note\n"); return 1; }
      if (w > 0 && j.parts > 0) check(j);
      while (true) {
        if (pos == s.begin) of_segment[std::make_tuple(s.b, s.h, s.t)] = note_of_segment(all, w, s, H, tiles);
        pos = end < s.end() ? end : s.end();
        if (pos >= end) break;
        next_segment(q, H, s);
      }
    }
    if ((long long)of_segment.size() != (long long)B * H * tiles) { printf("notes missing\n"); return 1; }
    auto once = joined;
    joined.clear();
    for (auto& [key, j] : of_segment) {
      if (key_of(j.segment) != key || (j.parts == 0) != (slots.count(key) == 0)) { printf("wrong note\n"); return 1; }
      if (j.parts > 0) check(j);
    }
    if (joined != once) { printf("notes differ\n"); return 1; }
    for (auto& [key, list] : slots) if (joined[key] != 1) { printf("not joined once\n"); return 1; }
    if (joined.size() != slots.size()) { printf("joined for nothing\n"); return 1; }
    printf("ok %d\n", shares);
  }
  return 0;
}
"""

FORMS = r"""
#include "cache_shares.hpp"
#include <cstdio>
int main() {
  int B, H, Hkv, N, d, cap;
  while (scanf("%d %d %d %d %d %d", &B, &H, &Hkv, &N, &d, &cap) == 6) {
    const CacheForm f = cache_form(B, H, Hkv, N, d, cap);
    printf("%d %d %d %d %d %zu %d\n", f.RT, f.KW, f.tiles, f.shares, (int)f.split, f.slot_floats(d), (int)f.many_parts);
  }
}
"""


def _build(tmp_path_factory, text):
    d = tmp_path_factory.mktemp("shares")
    (d / "main.cpp").write_text(text)
    subprocess.run(["g++", "-std=c++17", "-O1", "-fsanitize=undefined", "-fno-sanitize-recover=all", "-I", HEADER_DIR, str(d / "main.cpp"),
                    "-o", str(d / "main")], check=True)
    return str(d / "main")


def test_every_block_is_taken_once_and_every_part_joined(tmp_path_factory):
    exe = _build(tmp_path_factory, MAIN)
    rng = random.Random(4)
    cases = []
    for _ in range(400):
        B, H, N = rng.choice((1, 1, 2, 5, 17, 70)), rng.choice((1, 2, 3, 8)), rng.choice((1, 1, 2, 7, 40, 300))
        group, capacity = rng.choice((1, 2, 4, 7)), 64 * rng.choice((1, 2, 5, 40, 300))
        M = rng.choice((16, 32, 64, 128))
        # lengths and counts as a caller may hold them, valid or not
        lengths = [rng.choice((0, 1, 63, 64, 65, capacity - 1, capacity, capacity + 1, rng.randint(0, capacity), -5, 2**31 - 1)) for _ in range(B)]
        counts = [-9] * B if rng.random() < 0.5 else [rng.choice((0, 1, N, rng.randint(0, N), -3, 2**31 - 1)) for _ in range(B)]
        cases.append([B, H, N, group, rng.randint(0, 1), capacity, M, rng.choice((1, 3, 8, 100, 512, 768)), rng.choice((1, 4, 6, 13))] + lengths + counts)
    r = subprocess.run([exe], input="\n".join(" ".join(map(str, c)) for c in cases), capture_output=True, text=True)
    assert r.returncode == 0, r.stdout[-200:] + r.stderr[-500:]
    assert r.stdout.count("ok") == len(cases)


@pytest.mark.parametrize("d", (32, 64, 96, 128, 256))
def test_the_form_covers_the_rows_and_the_workspace_is_what_the_library_says(tmp_path_factory, d):
    from paper_2510_04212_amd import binding
    exe = _build(tmp_path_factory, FORMS)
    cases = [(B, Hkv * g, Hkv, N, d, cap) for B in (1, 3, 64) for Hkv in (1, 8) for g in (1, 4, 16) for N in (1, 2, 5, 16, 100, 2048)
             for cap in (64, 1024, 1088, 16384, 262144)]
    out = subprocess.run([exe], input="\n".join(" ".join(map(str, c)) for c in cases), check=True, capture_output=True, text=True).stdout
    kinds, many_parts = set(), set()
    for c, line in zip(cases, out.splitlines()):
        RT, KW, tiles, shares, split, slot, many = map(int, line.split())
        rows, M = c[3] * c[1] // c[2], 64 * RT // KW
        assert tiles * M >= rows > (tiles - 1) * M and 1 <= shares <= 768
        assert binding.cache_fwd_workspace_bytes(*c) == (16 * shares + 2 * shares * slot * 4 if split and shares > 1 else 0)
        kinds.add((RT, KW, bool(split)))
        many_parts.add((RT, KW, bool(many)))
    assert kinds == many_parts == {(RT, KW, s) for RT, KW in ((1, 4), (1, 1), (2, 1)) for s in (False, True)}


def test_whole_segments_of_shared_blocks_are_short(tmp_path_factory):
    """One lane of a wave holds a block's scales there: a whole segment of more than 16 rows has at most 32 blocks, however many segments there are."""
    exe = _build(tmp_path_factory, FORMS)
    cases = [(B, Hkv * g, Hkv, N, d, cap) for B in (1, 60, 65535) for Hkv in (1, 8, 64) for g in (1, 4) for N in (5, 17, 70, 5000) for d in (32, 128, 256)
             for cap in (1024, 2048, 2112, 4096, 8192, 1 << 20) if B * Hkv * N < 1 << 24]
    out = subprocess.run([exe], input="\n".join(" ".join(map(str, c)) for c in cases), check=True, capture_output=True, text=True).stdout
    whole = [c[5] for c, line in zip(cases, out.splitlines()) if line.split()[1] == "1" and line.split()[4] == "0"]
    assert max(whole) == 32 * 64
