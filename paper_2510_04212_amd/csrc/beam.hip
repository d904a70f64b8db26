// The choice among beams (attn_beam_select of include/attn.h): the n best of all continuations of an item's beams.
//
// A beam's log-probabilities log softmax(x) = x - log(sum(exp(x))) keep the order of its logits, so that the first kernel, with a work-group for each
// chunk of a beam's logits, needs no sum of the others': it leaves the chunk's n best, its maximum m and the sum of exp(x - m).  The second, with a
// work-group for each item, has the beams' sums from those and takes the n best of what the chunks left.
//
// Numbers.  Candidates of different beams may be closer to one another than float32 tells: sums are compared in float64.  exp(x - m) is float32 (within
// |x - m| 2^-23, of the difference and of log2(e), and the hardware exponential's 2^-23), a thread's sum too (of up to 32 terms), everything after it float64.
#include "beam.hpp"
#include "cache.hpp"
#include <type_traits>

namespace {

constexpr int kThreads = 256;
typedef unsigned long long u64;
typedef u32x4 __attribute__((aligned(4))) At4;
typedef u32x4 __attribute__((aligned(2))) At2;

// Larger <=> better, of one beam: by value, then by index, the lower first; -0 = +0.  0: none.
DEVI unsigned order(float x) {
  const unsigned u = __float_as_uint(x);
  if (x == 0.f) return 0x80000000u;
  return (u & 0x80000000u) ? ~u : u | 0x80000000u;
}
DEVI u64 order(double x) {
  const u64 u = (u64)__double_as_longlong(x == 0.0 ? 0.0 : x);
  return (u >> 63) ? ~u : u | 1ull << 63;
}
DEVI u64 key_of(float x, int token) { return x > -INFINITY ? (u64)order(x) << 32 | (0xffffffffu - (unsigned)token) : 0; }
DEVI float value_of(u64 key) {
  const unsigned u = (unsigned)(key >> 32);
  return __uint_as_float((u & 0x80000000u) ? u & 0x7fffffffu : ~u);
}
DEVI int token_of(u64 key) { return (int)(0xffffffffu - (unsigned)key); }

struct Stat { double sum; float m; };      // the sum is NaN where the chunk holds NaN or +infinity

// A chunk is 256 threads' 8 or 32 elements.  The smaller one fills the chip for few rows; the larger one leaves fewer lists, and less is spent on each beside its
// elements.  us a call, 8 / 32: beams 1 x 4 of 32000, n 8: 8.6 / 10.5;  6 x 5 of 50257 (bf16), n 5: 10.8 / 13.2;  8 x 8 of 32000, n 8: 11.0 / 11.9;  32 x 8 of
// 32000, n 16: 20.6 / 18.9;  1 x 8 of 131072, n 16: 16.6 / 11.7;  1 x 32 of 32000, n 64: 45.8 / 27.7;  32 x 8 of 131072, n 16: 53 / 34.5.
struct ScanForm {
  int per_thread, chunks;
  long long rows;
  __host__ __device__ size_t lists_at() const { return (size_t)rows * chunks * sizeof(Stat); }
  size_t bytes(int n) const { return lists_at() + (size_t)rows * chunks * n * sizeof(u64); }
};
ScanForm scan_form(int B, int beams, int V, int n) {
  ScanForm l;
  l.rows = (long long)B * beams;
  auto chunks = [&](int per_thread) { return (V + kThreads * per_thread - 1) / (kThreads * per_thread); };
  l.per_thread = l.rows * V <= 1 << 22 && (long long)beams * chunks(8) * n <= 4096 ? 8 : 32;
  l.chunks = chunks(l.per_thread);
  return l;
}

DEVI u64 best_in_wave(u64 x) {
#pragma unroll
  for (int i = 1; i < 64; i <<= 1) {
    const u64 y = __shfl_xor(x, i);
    x = y > x ? y : x;
  }
  return x;
}
// of four neighbouring lanes, the same in all of them
DEVI unsigned max_of_4(unsigned x) {
  x = max(x, (unsigned)__builtin_amdgcn_update_dpp(0, (int)x, 0xb1, 0xf, 0xf, false));
  return max(x, (unsigned)__builtin_amdgcn_update_dpp(0, (int)x, 0x4e, 0xf, 0xf, false));
}
// Largest t, as far as the upper BITS bits go, such that at least n of the lanes' values reach it: a wave's search, two bits at a time.
template <int BITS, int EACH> DEVI unsigned reached_by(const unsigned (&x)[EACH], int n) {
  static_assert(BITS % 2 == 0, "two bits at a time");
  unsigned t = 0;
#pragma unroll
  for (int bit = 30; bit >= 32 - BITS; bit -= 2) {
    unsigned next = t;
#pragma unroll
    for (unsigned c = 1; c < 4; ++c) {
      int reach = 0;
#pragma unroll
      for (int i = 0; i < EACH; ++i) reach += __popcll(__ballot(x[i] >= (t | c << bit)));
      if (reach >= n) next = t | c << bit;
    }
    t = next;
  }
  return t;
}

// Few are chosen of many, so most are left out at once: the n-th largest of the maxima of 64 or 256 groups of elements is a bound that the n best
// reach, and hardly any others (64 groups, n = 16: 18 elements).  Those that do are gathered in LDS, and each finds its place by counting the better ones.
// Where too many reach it, the best is taken n times: equal values, or, as the bound has 16 bits (a bf16 step), many logits far from 0 together (32 x 8 x 131072, n 16:
// 32 us; 192 with 1000 added to all; 491 with all but one in 1000 at -10000).
//
// Bound by bytes for large rows of float32 (32 x 8 x 131072, n 16: 27.3 us, 4.9 TB/s; 181 with the best taken n times), by the work on a chunk beside them
// otherwise (the same in bf16: 17.9 us, 3.7 TB/s).  Without exponentials it takes as long, without the search for the best 25 and 13.
constexpr int kFewGroups = 32;             // n up to here: 64 groups
constexpr int kGathered = kThreads;

// over the wave, to lane 63: the steps of scan_wave
template <int CONTROL, int ROWS> DEVI double add_shifted(double x) {
  const u64 u = (u64)__double_as_longlong(x);
  const unsigned lo = (unsigned)__builtin_amdgcn_update_dpp(0, (int)(unsigned)u, CONTROL, ROWS, 0xf, false);
  const unsigned hi = (unsigned)__builtin_amdgcn_update_dpp(0, (int)(unsigned)(u >> 32), CONTROL, ROWS, 0xf, false);
  return x + __longlong_as_double((long long)((u64)hi << 32 | lo));
}
DEVI double sum_to_last_lane(double x) {
  x = add_shifted<0x111, 0xf>(x);
  x = add_shifted<0x112, 0xf>(x);
  x = add_shifted<0x114, 0xf>(x);
  x = add_shifted<0x118, 0xf>(x);
  x = add_shifted<0x142, 0xa>(x);
  return add_shifted<0x143, 0xc>(x);
}

template <int PER, bool WIDE>
__global__ __launch_bounds__(kThreads, 5) void attn_beam_scan_kernel(BeamArgs p, int chunks, Stat* stats, u64* lists) {
  constexpr int VEC = WIDE ? 4 : 8, LOADS = PER / VEC, SIZE = WIDE ? 4 : 2, WAVES = kThreads / 64;
  __shared__ unsigned tops[kThreads];
  __shared__ u64 gathered[kGathered], best[WAVES];
  __shared__ double sums[WAVES];
  __shared__ int count;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const unsigned row = blockIdx.x / (unsigned)chunks;
  const int chunk = (int)(blockIdx.x - row * chunks);
  if (p.finished && p.finished[row]) return;
  if (!(__builtin_fabsf(p.scores[row]) < INFINITY)) return;
  const int b = (int)(row / (unsigned)p.beams), k = (int)(row - (unsigned)(b * p.beams));
  const char* at = static_cast<const char*>(p.logits) + (b * p.stride_b + k * p.stride_beam) * SIZE;
  // The thread's elements, 16 bytes at a time, by their tokens, wherever the row begins: sums in another order would be others in their last bits, and equal
  // beams' no longer equal.  Loads of 16 bytes from any address cost nothing (32 x 8 rows of 131072 n 16: 34.2 us, and 34.3 at a pitch of 131073; bf16 26.8 and 27.9).
  using Anywhere = std::conditional_t<WIDE, At4, At2>;
  const int chunk0 = chunk * (kThreads * PER), first = chunk0 + tid * VEC;                 // (V <= 2^24)
  auto index = [&](int i) { return first + i / VEC * (kThreads * VEC) + i % VEC; };
  auto load = [&](int e) {
    if (e >= p.V) return -INFINITY;
    return WIDE ? reinterpret_cast<const float*>(at)[e] : __uint_as_float((unsigned)reinterpret_cast<const unsigned short*>(at)[e] << 16);
  };
  float x[PER];
  {
    u32x4 w[LOADS];
    const bool whole = chunk0 + kThreads * PER <= p.V;
#pragma unroll
    for (int j = 0; j < LOADS; ++j) {      // all in flight at once
      const int e = index(j * VEC);
      if (whole || e + VEC <= p.V) w[j] = *reinterpret_cast<const Anywhere*>(at + (long long)e * SIZE);
    }
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const unsigned bits = WIDE ? w[i / VEC][i % 4] : w[i / VEC][i % VEC / 2];
      x[i] = __uint_as_float(WIDE ? bits : (i & 1) ? bits & 0xffff0000u : bits << 16);
    }
    if (!whole)                            // the row's last elements one by one (32 x 8 rows of 131000: 34.4 us, and 46.4 with the whole last chunk so)
#pragma unroll
      for (int i = 0; i < PER; ++i)
        if (index(i - i % VEC) + VEC > p.V) x[i] = load(index(i));
  }
  float of_load[LOADS], mine = -INFINITY;  // (maxima pass over NaN; the sum below does not)
#pragma unroll
  for (int j = 0; j < LOADS; ++j) {
    of_load[j] = x[j * VEC];
#pragma unroll
    for (int i = 1; i < VEC; ++i) of_load[j] = fmaxf(of_load[j], x[j * VEC + i]);
    mine = fmaxf(mine, of_load[j]);
  }
  const bool few = p.n <= kFewGroups;
  const unsigned top = order(mine);
  if (few) {
    const unsigned of_4 = max_of_4(top);
    if ((lane & 3) == 0) tops[tid >> 2] = of_4;
  } else {
    tops[tid] = top;
  }
  if (tid == 0) count = 0;
  __syncthreads();
  unsigned reach, most_key;
  if (few) {
    const unsigned t[1] = {tops[lane]};
    most_key = max_over_wave(t[0]);
    reach = reached_by<16>(t, p.n);
  } else {
    const unsigned t[4] = {tops[lane], tops[lane + 64], tops[lane + 128], tops[lane + 192]};
    most_key = max_over_wave(max(max(t[0], t[1]), max(t[2], t[3])));
    reach = reached_by<16>(t, p.n);
  }
  const float most = value_of((u64)most_key << 32);
  const float bound = reach > order(-INFINITY) ? value_of((u64)reach << 32) : -3.40282347e38f;       // no -infinity
  const float from = most == -INFINITY ? 0.f : most;
  float sum = 0.f;
#pragma unroll
  for (int i = 0; i < PER; ++i) sum += __builtin_amdgcn_exp2f((x[i] - from) * kLog2e);
  const double wide = sum_to_last_lane(sum);
  if (lane == 63) sums[wave] = wide;
  if (mine >= bound) {                     // a few threads, an element or two each
#pragma unroll
    for (int j = 0; j < LOADS; ++j) {
      if (of_load[j] < bound) continue;
#pragma unroll
      for (int i = j * VEC; i < (j + 1) * VEC; ++i)
        if (x[i] >= bound) {
          const int to = atomicAdd(&count, 1);
          if (to < kGathered) gathered[to] = key_of(x[i], index(i));
        }
    }
  }
  __syncthreads();
  const double total = sums[0] + sums[1] + sums[2] + sums[3];
  if (tid == 0) stats[(size_t)row * chunks + chunk] = Stat{total, most};
  if (total != total) return;              // nobody asks for the rest
  // a beam's lists lie side by side: the best of all its chunks, then the second ...
  u64* list = lists + (size_t)row * p.n * chunks + chunk;
  const int found = count;
  if (found <= kGathered) {
    if (wave * 64 < found) {
      const u64 key = tid < found ? gathered[tid] : 0;
      int place = 0;
#pragma unroll 8
      for (int i = 0; i < found; ++i) place += gathered[i] > key ? 1 : 0;
      if (tid < found && place < p.n) list[place * chunks] = key;
    }
    for (int i = found + tid; i < p.n; i += kThreads) list[i * chunks] = 0;
    return;
  }
  u64 last = ~0ull;
  for (int i = 0; i < p.n; ++i) {
    u64 left = 0;
#pragma unroll 1
    for (int j = 0; j < PER; ++j) {        // (read again: there are no registers for all keys)
      const u64 key = key_of(load(index(j)), index(j));
      left = key < last && key > left ? key : left;
    }
    left = best_in_wave(left);
    __syncthreads();
    if (lane == 0) best[wave] = left;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < WAVES; ++w) left = best[w] > left ? best[w] : left;
    if (tid == 0) list[i * chunks] = left;
    last = left;                           // (0: nothing is below it)
  }
}

// A candidate of an item: larger sum, then lower beam, then what is better within the beam.
struct Candidate {
  double sum;
  u64 key;
  int beam;
};
DEVI bool better(const Candidate& a, const Candidate& b) {
  if (a.sum != b.sum) return a.sum > b.sum;
  if (a.beam != b.beam) return a.beam < b.beam;
  return a.key > b.key;
}

// The same again: a bound from 64 or 256 groups of candidates, by their sums rounded to float32 (which keeps their order), and the places of those that reach it.
constexpr int kChooseThreads = 1024, kHeld = 4;
__global__ __launch_bounds__(kChooseThreads) void attn_beam_choose_kernel(BeamArgs p, int chunks, const Stat* stats, const u64* lists) {
  // A logit's sum is (x - most) + rest, as logits can be so large that the rest would be lost next to them; rest = -infinity: no candidates
  __shared__ float most[kMostBeams];
  __shared__ double rest[kMostBeams];
  __shared__ unsigned tops[kChooseThreads];
  __shared__ Candidate gathered[kChooseThreads], best[kChooseThreads / 64];
  __shared__ u64 sums[kChooseThreads];     // of the gathered, in order
  __shared__ unsigned shared_reach;
  __shared__ int count;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, b = blockIdx.x;
  const long long row0 = (long long)b * p.beams;
  // Numbers of candidates, and so groups, such that neither a beam's best ones nor all beams' share a group: a beam's run through all of its chunks' best,
  // then the second ..., and the next beam begins as many groups behind as there are chunks.
  const int per_beam = chunks * p.n, stride = (per_beam + 63) / 64 * 64 + chunks, all = p.beams * stride;
  auto listed = [&](int j, int k) { return j < all && j - k * stride < per_beam ? lists[(row0 + k) * per_beam + (j - k * stride)] : 0; };
  // a thread's first candidates are on their way while the sums are formed
  u64 held[kHeld];
#pragma unroll
  for (int i = 0; i < kHeld; ++i) held[i] = listed(tid + i * kChooseThreads, (tid + i * kChooseThreads) / stride);
  if (tid == 0) count = 0;
  for (int k = wave; k < p.beams; k += kChooseThreads / 64) {
    const Stat* s = stats + (row0 + k) * chunks;
    const Stat own = s[min(lane, chunks - 1)];             // (whatever is there, until it is known to be wanted)
    const float score = p.scores[row0 + k];
    const bool finite = __builtin_fabsf(score) < INFINITY;
    float m = 0.f;
    double to = finite ? (double)score : -INFINITY;
    if (finite && !(p.finished && p.finished[row0 + k])) {
      bool bad = own.sum != own.sum;
      m = own.m;
      for (int c = lane + 64; c < chunks; c += 64) {
        bad |= s[c].sum != s[c].sum;
        m = fmaxf(m, s[c].m);
      }
#pragma unroll
      for (int i = 1; i < 64; i <<= 1) m = fmaxf(m, __shfl_xor(m, i));
      double sum = lane < chunks && own.m > -INFINITY ? own.sum * exp((double)own.m - m) : 0.0;
      for (int c = lane + 64; c < chunks; c += 64)
        if (s[c].m > -INFINITY) sum += s[c].sum * exp((double)s[c].m - m);
#pragma unroll
      for (int i = 1; i < 64; i <<= 1) sum += __shfl_xor(sum, i);
      to = __any(bad) || m == -INFINITY ? -INFINITY : to - log(sum);
    }
    if (lane == 0) { most[k] = m; rest[k] = to; }
  }
  __syncthreads();
  // candidate j of the item, its key as it was read; one that is none has the key 0
  auto candidate = [&](int j, u64 key) {
    const int k = j / stride;
    Candidate c{rest[k], key, k};
    if (c.sum == -INFINITY) {
      c.key = 0;
    } else if (p.finished && p.finished[row0 + k]) {
      c.key = j == k * stride ? key_of(0.f, p.end_token) : 0;
    } else if (key != 0) {
      c.sum += (double)value_of(key) - most[k];
    }
    return c;
  };
  auto for_all = [&](auto&& f) {
#pragma unroll
    for (int i = 0; i < kHeld; ++i)
      if (tid + i * kChooseThreads < all) {
        const Candidate c = candidate(tid + i * kChooseThreads, held[i]);
        if (c.key != 0) f(c);
      }
    for (int j = tid + kHeld * kChooseThreads; j < all; j += kChooseThreads) {
      const Candidate c = candidate(j, listed(j, j / stride));
      if (c.key != 0) f(c);
    }
  };
  unsigned top = 0;
  for_all([&](const Candidate& c) { top = max(top, order((float)c.sum)); });
  tops[tid] = top;
  __syncthreads();
  if (wave == 0) {
    unsigned t[4] = {0, 0, 0, 0};          // of 256 groups
#pragma unroll
    for (int w = 0; w < kChooseThreads / 64; ++w) t[w % 4] = max(t[w % 4], tops[w * 64 + lane]);
    unsigned bound;
    if (p.n <= kFewGroups) {
      const unsigned one[1] = {max(max(t[0], t[1]), max(t[2], t[3]))};
      bound = reached_by<24>(one, p.n);
    } else {
      bound = reached_by<24>(t, p.n);
    }
    if (lane == 0) shared_reach = bound;
  }
  __syncthreads();
  const unsigned reach = shared_reach;
  if (top >= reach)
    for_all([&](const Candidate& c) {
      if (order((float)c.sum) < reach) return;
      const int i = atomicAdd(&count, 1);
      if (i < kChooseThreads) {
        gathered[i] = c;
        sums[i] = order(c.sum);
      }
    });
  auto put = [&](int i, const Candidate& c) {
    const long long to = (long long)b * p.n + i;
    const bool there = c.key != 0;
    const int token = there ? token_of(c.key) : -1;
    p.parents[to] = there ? c.beam : -1;
    p.tokens[to] = token;
    p.scores_out[to] = there ? (float)c.sum : -INFINITY;
    if (p.finished_out) p.finished_out[to] = there && (token == p.end_token || (p.finished && p.finished[row0 + c.beam]));
  };
  __syncthreads();
  const int found = count;
  if (found <= kChooseThreads) {
    if (wave * 64 < found) {
      const int at = min(tid, found - 1);
      const Candidate mine = gathered[at];
      const u64 sum = sums[at];
      int place = 0, equal = 0;
#pragma unroll 8
      for (int i = 0; i < found; ++i) {
        place += sums[i] > sum ? 1 : 0;
        equal += sums[i] == sum ? 1 : 0;
      }
      if (equal > 1)
        for (int i = 0; i < found; ++i) place += sums[i] == sum && better(gathered[i], mine) ? 1 : 0;
      if (tid < found && place < p.n) put(place, mine);
    }
    for (int i = found + tid; i < p.n; i += kChooseThreads) put(i, Candidate{-INFINITY, 0, 0});
    return;
  }
  Candidate last{INFINITY, ~0ull, -1};
  for (int i = 0; i < p.n; ++i) {
    Candidate next{-INFINITY, 0, kMostBeams};
    for_all([&](const Candidate& c) {
      if (better(last, c) && better(c, next)) next = c;
    });
#pragma unroll
    for (int j = 1; j < 64; j <<= 1) {
      const Candidate other{__shfl_xor(next.sum, j), __shfl_xor(next.key, j), __shfl_xor(next.beam, j)};
      if (better(other, next)) next = other;
    }
    __syncthreads();
    if (lane == 0) best[wave] = next;
    __syncthreads();
    for (int w = 0; w < kChooseThreads / 64; ++w)
      if (better(best[w], next)) next = best[w];
    last = next;
    if (tid == 0) put(i, next);
  }
}

}  // namespace

size_t attn_beam_select_partial_bytes(int B, int beams, int V, int n) {
  return scan_form(B, beams, V, n).bytes(n);
}

hipError_t attn_beam_select_dispatch(const BeamArgs& p, hipStream_t stream) {
  const ScanForm l = scan_form(p.B, p.beams, p.V, p.n);
  if (!grid_fits(l.rows * l.chunks, kThreads)) return hipErrorInvalidConfiguration;
  Stat* stats = static_cast<Stat*>(p.workspace);
  u64* lists = reinterpret_cast<u64*>(static_cast<char*>(p.workspace) + l.lists_at());
  const unsigned grid = (unsigned)(l.rows * l.chunks);
  auto scan = [&](auto PER, auto WIDE) { attn_beam_scan_kernel<PER, WIDE><<<grid, kThreads, 0, stream>>>(p, l.chunks, stats, lists); };
  using std::bool_constant, std::integral_constant;
  if (l.per_thread == 8) p.wide ? scan(integral_constant<int, 8>{}, bool_constant<true>{}) : scan(integral_constant<int, 8>{}, bool_constant<false>{});
  else p.wide ? scan(integral_constant<int, 32>{}, bool_constant<true>{}) : scan(integral_constant<int, 32>{}, bool_constant<false>{});
  if (const hipError_t e = hipGetLastError(); e != hipSuccess) return e;
  attn_beam_choose_kernel<<<(unsigned)p.B, kChooseThreads, 0, stream>>>(p, l.chunks, stats, lists);
  return hipGetLastError();
}
