// The choice among beams (attn_beam_select of include/attn.h): the n best of all continuations of an item's beams.
//
// A beam's log-probabilities log softmax(x) = x - log(sum(exp(x))) keep the order of its logits, so that the first kernel, with a work-group for each
// chunk of a beam's logits, needs no sum of the others': it leaves the chunk's n best, its maximum m and the sum of exp(x - m).  The second, with a
// work-group for each item, has the beams' sums from those and takes the n best of what the chunks left.
//
// Numbers.  Candidates of different beams may be closer to one another than float32 tells: sums are compared in float64.  exp(x - m) is float32 (within
// |x - m| 2^-24 and the hardware exponential's 2^-23), a thread's sum too (of up to 32 terms), everything after it float64.
#include "beam.hpp"
#include "common.hpp"
#include <algorithm>

namespace {

constexpr int kThreads = 256;
typedef unsigned long long u64;

// Larger <=> better, of one beam: by value, then by index, the lower first; -0 = +0.  0: none.
DEVI unsigned order(float x) {
  const unsigned u = __float_as_uint(x);
  if (x == 0.f) return 0x80000000u;
  return (u & 0x80000000u) ? ~u : u | 0x80000000u;
}
DEVI u64 key_of(float x, int token) { return x > -INFINITY ? (u64)order(x) << 32 | (0xffffffffu - (unsigned)token) : 0; }
DEVI float value_of(u64 key) {
  const unsigned u = (unsigned)(key >> 32);
  return __uint_as_float((u & 0x80000000u) ? u & 0x7fffffffu : ~u);
}
DEVI int token_of(u64 key) { return (int)(0xffffffffu - (unsigned)key); }

struct Stat { double sum; float m; };      // m: NaN where the chunk holds NaN or +infinity

struct ScanForm {
  int per_thread, chunks;
  long long rows;
  __host__ __device__ size_t lists_at() const { return (size_t)rows * chunks * sizeof(Stat); }
  size_t bytes(int n) const { return lists_at() + (size_t)rows * chunks * n * sizeof(u64); }
};
// (a row begins up to 7 elements behind a 16-byte boundary)
ScanForm scan_form(int B, int beams, int V) {
  ScanForm l;
  l.rows = (long long)B * beams;
  l.per_thread = l.rows * V <= 1 << 20 ? 8 : 32;
  l.chunks = (int)(((long long)V + 7 + kThreads * l.per_thread - 1) / (kThreads * l.per_thread));
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

template <int PER, bool WIDE>
__global__ __launch_bounds__(kThreads) void attn_beam_scan_kernel(BeamArgs p, int chunks, Stat* stats, u64* lists) {
  constexpr int VEC = WIDE ? 4 : 8, LOADS = PER / VEC;
  __shared__ u64 best[kThreads / 64];
  __shared__ float mosts[kThreads / 64];
  __shared__ double sums[kThreads / 64];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int chunk = blockIdx.x % (unsigned)chunks;
  const long long row = blockIdx.x / (unsigned)chunks;
  if (p.finished && p.finished[row]) return;
  if (!(__builtin_fabsf(p.scores[row]) < INFINITY)) return;
  const int b = (int)(row / p.beams), k = (int)(row % p.beams);
  const char* at = static_cast<const char*>(p.logits) + (b * p.stride_b + k * p.stride_beam) * (WIDE ? 4 : 2);
  const int shift = (int)((reinterpret_cast<uintptr_t>(at) & 15) / (WIDE ? 4 : 2));        // elements behind a 16-byte boundary
  // the thread's elements, 16 bytes at a time from such boundaries on
  float x[PER];
  int first[LOADS];
#pragma unroll
  for (int j = 0; j < LOADS; ++j) {
    const long long e0 = (long long)chunk * (kThreads * PER) + (j * kThreads + tid) * VEC - shift;
    first[j] = (int)min(e0, (long long)p.V);
    if (e0 >= 0 && e0 + VEC <= p.V) {
      const u32x4 w = *reinterpret_cast<const u32x4*>(at + e0 * (WIDE ? 4 : 2));
#pragma unroll
      for (int i = 0; i < VEC; ++i)
        x[j * VEC + i] = WIDE ? __uint_as_float(w[i % 4]) : __uint_as_float((i & 1) ? w[i / 2] & 0xffff0000u : w[i / 2] << 16);
    } else {
#pragma unroll
      for (int i = 0; i < VEC; ++i) {
        x[j * VEC + i] = -INFINITY;
        if (e0 + i >= 0 && e0 + i < p.V)
          x[j * VEC + i] = WIDE ? reinterpret_cast<const float*>(at)[e0 + i] : __uint_as_float((unsigned)reinterpret_cast<const unsigned short*>(at)[e0 + i] << 16);
      }
    }
  }
  float most = -INFINITY;
  bool bad = false;
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    most = fmaxf(most, x[i]);
    bad |= !(x[i] < INFINITY);
  }
#pragma unroll
  for (int i = 1; i < 64; i <<= 1) most = fmaxf(most, __shfl_xor(most, i));
  if (__any(bad)) most = INFINITY;         // (stands for both)
  if (lane == 0) mosts[wave] = most;
  __syncthreads();
  most = fmaxf(fmaxf(mosts[0], mosts[1]), fmaxf(mosts[2], mosts[3]));
  const long long slot = row * chunks + chunk;
  u64* list = lists + slot * p.n;
  if (!(most < INFINITY)) {                // (the same in all threads)
    if (tid == 0) stats[slot] = Stat{0.0, NAN};
    for (int i = tid; i < p.n; i += kThreads) list[i] = 0;
    return;
  }
  constexpr float kLog2eRest = 1.92596303e-8f;             // log2(e) - kLog2e
  const float from = most == -INFINITY ? 0.f : most;
  float sum = 0.f;
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const float d = x[i] - from;
    sum += __builtin_amdgcn_exp2f(__builtin_fmaf(d, kLog2e, d * kLog2eRest));
  }
  double wide = sum;
#pragma unroll
  for (int i = 1; i < 64; i <<= 1) wide += __shfl_xor(wide, i);
  if (lane == 0) sums[wave] = wide;
  __syncthreads();
  if (tid == 0) stats[slot] = Stat{sums[0] + sums[1] + sums[2] + sums[3], most};

  u64 last = ~0ull;
  for (int i = 0; i < p.n; ++i) {
    u64 mine = 0;
#pragma unroll
    for (int j = 0; j < PER; ++j) {
      const u64 key = key_of(x[j], first[j / VEC] + j % VEC);
      mine = key < last && key > mine ? key : mine;
    }
    mine = best_in_wave(mine);
    __syncthreads();
    if (lane == 0) best[wave] = mine;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kThreads / 64; ++w) mine = best[w] > mine ? best[w] : mine;
    if (tid == 0) list[i] = mine;
    last = mine;                           // (0: nothing is below it)
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

constexpr int kChooseThreads = 1024;
__global__ __launch_bounds__(kChooseThreads) void attn_beam_choose_kernel(BeamArgs p, int chunks, const Stat* stats, const u64* lists) {
  // A logit's sum is (x - most) + rest, as logits can be so large that the rest would be lost next to them; rest = -infinity: no candidates
  __shared__ float most[kMostBeams];
  __shared__ double rest[kMostBeams];
  __shared__ Candidate best[kChooseThreads / 64];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, b = blockIdx.x;
  const long long row0 = (long long)b * p.beams;
  for (int k = wave; k < p.beams; k += kChooseThreads / 64) {
    const float score = p.scores[row0 + k];
    const bool finite = __builtin_fabsf(score) < INFINITY;
    float m = 0.f;
    double to = finite ? (double)score : -INFINITY;
    if (finite && !(p.finished && p.finished[row0 + k])) {
      const Stat* s = stats + (row0 + k) * chunks;
      m = -INFINITY;
      bool bad = false;
      for (int c = lane; c < chunks; c += 64) {
        bad |= s[c].m != s[c].m;
        m = fmaxf(m, s[c].m);
      }
#pragma unroll
      for (int i = 1; i < 64; i <<= 1) m = fmaxf(m, __shfl_xor(m, i));
      double sum = 0.0;
      for (int c = lane; c < chunks; c += 64)
        if (s[c].m > -INFINITY) sum += s[c].sum * exp((double)s[c].m - m);
#pragma unroll
      for (int i = 1; i < 64; i <<= 1) sum += __shfl_xor(sum, i);
      to = __any(bad) || m == -INFINITY ? -INFINITY : to - log(sum);
    }
    if (lane == 0) { most[k] = m; rest[k] = to; }
  }
  __syncthreads();
  const int per_beam = chunks * p.n, all = p.beams * per_beam;
  Candidate last{INFINITY, ~0ull, -1};
  for (int i = 0; i < p.n; ++i) {
    Candidate mine{-INFINITY, 0, kMostBeams};
    for (int j = tid; j < all; j += kChooseThreads) {
      const int k = j / per_beam, at = j - k * per_beam;
      if (rest[k] == -INFINITY) continue;
      Candidate c{rest[k], 0, k};
      if (p.finished && p.finished[row0 + k]) {
        c.key = at == 0 ? key_of(0.f, p.end_token) : 0;
      } else {
        c.key = lists[(row0 + k) * per_beam + at];
        c.sum += (double)value_of(c.key) - most[k];
      }
      if (c.key != 0 && better(last, c) && better(c, mine)) mine = c;
    }
#pragma unroll
    for (int j = 1; j < 64; j <<= 1) {
      const Candidate other{__shfl_xor(mine.sum, j), __shfl_xor(mine.key, j), __shfl_xor(mine.beam, j)};
      if (better(other, mine)) mine = other;
    }
    __syncthreads();
    if (lane == 0) best[wave] = mine;
    __syncthreads();
    for (int w = 0; w < kChooseThreads / 64; ++w)
      if (better(best[w], mine)) mine = best[w];
    last = mine;
    if (tid == 0) {
      const long long to = (long long)b * p.n + i;
      const bool there = mine.key != 0;
      const int token = there ? token_of(mine.key) : -1;
      p.parents[to] = there ? mine.beam : -1;
      p.tokens[to] = token;
      p.scores_out[to] = there ? (float)mine.sum : -INFINITY;
      if (p.finished_out) p.finished_out[to] = there && (token == p.end_token || (p.finished && p.finished[row0 + mine.beam]));
    }
  }
}

}  // namespace

size_t attn_beam_select_partial_bytes(int B, int beams, int V, int n) { return scan_form(B, beams, V).bytes(n); }

hipError_t attn_beam_select_dispatch(const BeamArgs& p, hipStream_t stream) {
  const ScanForm l = scan_form(p.B, p.beams, p.V);
  if (!grid_fits(l.rows * l.chunks, kThreads)) return hipErrorInvalidConfiguration;
  Stat* stats = static_cast<Stat*>(p.workspace);
  u64* lists = reinterpret_cast<u64*>(static_cast<char*>(p.workspace) + l.lists_at());
  const unsigned grid = (unsigned)(l.rows * l.chunks);
  if (p.wide) {
    if (l.per_thread == 8) attn_beam_scan_kernel<8, true><<<grid, kThreads, 0, stream>>>(p, l.chunks, stats, lists);
    else attn_beam_scan_kernel<32, true><<<grid, kThreads, 0, stream>>>(p, l.chunks, stats, lists);
  } else {
    if (l.per_thread == 8) attn_beam_scan_kernel<8, false><<<grid, kThreads, 0, stream>>>(p, l.chunks, stats, lists);
    else attn_beam_scan_kernel<32, false><<<grid, kThreads, 0, stream>>>(p, l.chunks, stats, lists);
  }
  if (const hipError_t e = hipGetLastError(); e != hipSuccess) return e;
  attn_beam_choose_kernel<<<(unsigned)p.B, kChooseThreads, 0, stream>>>(p, l.chunks, stats, lists);
  return hipGetLastError();
}
