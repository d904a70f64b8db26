// Sequences of a cache copied whole: into another cache (attn_cache_fork of include/attn.h), or to other places of their group in the same
// one (attn_cache_reorder).  Blocks that hold tokens are moved as they are, codes and scales.
#include "cache.hpp"
#include <algorithm>

namespace {

constexpr int kThreads = 256;
constexpr int kPiece = 16;                 // bytes of a load

DEVI int blocks_of(int tokens) { return (tokens + kBlock - 1) / kBlock; }

// ---- fork.  Work-groups of a (sequence of the new cache, head) take chunks of its codes in turn; bound by bytes.
constexpr int kChunk = kThreads * 4;       // pieces of K and as many of V
__global__ __launch_bounds__(kThreads) void attn_cache_fork_kernel(ForkArgs p) {
  const int i = blockIdx.z, h = blockIdx.y, tid = threadIdx.x;
  const int from = p.sources[i];
  const int tokens = from >= 0 && from < p.B_in ? min(max(p.lengths[from], 0), min(p.from.capacity, p.to.capacity)) : 0;
  if (blockIdx.x == 0 && h == 0 && tid == 0) p.lengths_out[i] = tokens;
  if (tokens == 0) return;
  const int blocks = blocks_of(tokens);
  const size_t sh = (size_t)from * p.H_kv + h, th = (size_t)i * p.H_kv + h;
  const size_t at = sh * p.from.capacity * p.d, to = th * p.to.capacity * p.d;
  const u32x4 *K = reinterpret_cast<const u32x4*>(p.from.K + at), *V = reinterpret_cast<const u32x4*>(p.from.V + at);
  u32x4 *K_to = reinterpret_cast<u32x4*>(p.to.K + to), *V_to = reinterpret_cast<u32x4*>(p.to.V + to);
  const long long pieces = (long long)blocks * kBlock * p.d / kPiece;
  for (long long first = (long long)blockIdx.x * kChunk; first < pieces; first += (long long)gridDim.x * kChunk) {
    u32x4 k[kChunk / kThreads], v[kChunk / kThreads];
#pragma unroll
    for (int j = 0; j < kChunk / kThreads; ++j) {
      const long long x = first + j * kThreads + tid;
      if (x < pieces) {
        k[j] = K[x];
        v[j] = V[x];
      }
    }
#pragma unroll
    for (int j = 0; j < kChunk / kThreads; ++j) {
      const long long x = first + j * kThreads + tid;
      if (x < pieces) {
        K_to[x] = k[j];
        V_to[x] = v[j];
      }
    }
  }
  if (blockIdx.x == 0) {
    const size_t sb = sh * (p.from.capacity / kBlock), tb = th * (p.to.capacity / kBlock);
    for (int blk = tid; blk < blocks; blk += kThreads) {
      p.to.K_scale[tb + blk] = p.from.K_scale[sb + blk];
      p.to.V_scale[tb + blk] = p.from.V_scale[sb + blk];
    }
  }
}

// ---- reorder.  A thread has the same piece of all sequences of a group: it reads those that go elsewhere before it writes over them, and no other
// thread touches what it reads or writes, so that neither cycles nor copies need memory of their own.

// What sequence `s` of the group gets: the sequence's number (-1: it stays, or there is no such place) and its blocks.
struct Gets { int source, blocks; };
DEVI Gets look_up(const ReorderArgs& p, size_t first, int s, bool writes_length) {
  if (s >= p.S) return Gets{-1, 0};
  int from = p.parents[first + s];
  if (from < 0 || from >= p.S) from = s;
  const int tokens = p.lengths[first + from];
  if (writes_length) p.lengths_out[first + s] = tokens;
  return from == s ? Gets{-1, 0} : Gets{from, blocks_of(min(max(tokens, 0), p.cache.capacity))};
}
// f(K, V, x, pieces of a block) for the thread's pieces x of a head's codes, up to `most` blocks, and for its scales; K, V: those of the group's first sequence
template <class F> DEVI void for_pieces(const ReorderArgs& p, size_t first, int h, int most, F&& f) {
  const int per_block = kBlock * p.d / kPiece;
  const size_t at = (first * p.H_kv + h) * (p.cache.capacity / kBlock);    // blocks in front of the head's
  u32x4 *K = reinterpret_cast<u32x4*>(p.cache.K) + at * per_block, *V = reinterpret_cast<u32x4*>(p.cache.V) + at * per_block;
  const long long pieces = (long long)most * per_block;
  for (long long x = (long long)blockIdx.x * kThreads + threadIdx.x; x < pieces; x += (long long)gridDim.x * kThreads) f(K, V, x, per_block);
  if (blockIdx.x == 0)
    for (int blk = threadIdx.x; blk < most; blk += kThreads) f(p.cache.K_scale + at, p.cache.V_scale + at, blk, 1);
}

// Few sequences: all are read, then all are written.  Four: 60.2 us, 4.3 TB/s (32 x 4 sequences of 300 to 2048 tokens, 8 heads, d 128), and 64.5 with the order
// below; four young ones (12 heads of d 64, 16 to 256 tokens) 3.9 and 5.4.
constexpr int kFew = 4;
__global__ __launch_bounds__(kThreads) void attn_cache_reorder_kernel(ReorderArgs p) {
  constexpr int S = kFew;
  __shared__ Gets gets[S];
  const int h = blockIdx.y, tid = threadIdx.x;
  const size_t first = (size_t)blockIdx.z * p.S;
  if (tid < S) gets[tid] = look_up(p, first, tid, blockIdx.x == 0 && h == 0);
  __syncthreads();
  int source[S], blocks[S], most = 0;
#pragma unroll
  for (int s = 0; s < S; ++s) {
    source[s] = __builtin_amdgcn_readfirstlane(gets[s].source);
    blocks[s] = __builtin_amdgcn_readfirstlane(gets[s].blocks);
    most = max(most, blocks[s]);
  }
  for_pieces(p, first, h, most, [&](auto* K, auto* V, long long x, int a_block) {
    const size_t stride = (size_t)p.H_kv * (p.cache.capacity / kBlock) * a_block;
    std::remove_reference_t<decltype(*K)> k[S], v[S];
#pragma unroll
    for (int s = 0; s < S; ++s)
      if (x < (long long)blocks[s] * a_block) {
        k[s] = K[source[s] * stride + x];
        v[s] = V[source[s] * stride + x];
      }
#pragma unroll
    for (int s = 0; s < S; ++s)
      if (x < (long long)blocks[s] * a_block) {
        K[s * stride + x] = k[s];
        V[s * stride + x] = v[s];
      }
  });
}

// More: the moves in an order in which no sequence is written that a later move reads, eight at a time, read together and then written.  First
// those to places that nobody reads, then those to places that only they read, and so on; what is left are cycles, of which the first place's sequence is
// held until the last one gets it.  16 x 8 sequences of 300 to 2048 tokens, 8 heads, d 128: 50.9 us, 3.8 TB/s (with all pieces in registers 61); 8 x 16, 4 x 32 and 2 x 64 of
// them: 58, 90 and 91 us (81, 137 and 188).
struct alignas(16) Move { int to, from, blocks, held; };   // from: -1: what is held;  held: blocks of `to` that are held before it is written
constexpr int kAtOnce = 8;
__global__ __launch_bounds__(kThreads) void attn_cache_reorder_many_kernel(ReorderArgs p) {
  __shared__ Move moves[kMostReordered];
  __shared__ volatile int flags[kMostReordered];           // (lanes of one wave write and read them in turn)
  __shared__ int number, most_blocks;
  const int h = blockIdx.y, tid = threadIdx.x;
  const size_t first = (size_t)blockIdx.z * p.S;
  static_assert(kMostReordered == 64, "a lane for each sequence");
  if (tid < 64) {
    const Gets mine = look_up(p, first, tid, blockIdx.x == 0 && h == 0);
    unsigned long long left = __ballot(mine.source >= 0);
    int count = 0;
    while (left != 0) {
      const bool goes = left >> tid & 1;
      flags[tid] = 0;
      __builtin_amdgcn_wave_barrier();
      if (goes) flags[mine.source] = 1;
      __builtin_amdgcn_wave_barrier();
      const unsigned long long now = __ballot(goes && flags[tid] == 0);
      if (now == 0) break;
      if (now >> tid & 1) moves[count + __popcll(now & ((1ull << tid) - 1))] = Move{tid, mine.source, mine.blocks, 0};
      count += __popcll(now);
      left &= ~now;
    }
    while (left != 0) {
      const int begin = __ffsll((long long)left) - 1;
      // whoever gets the first place's sequence knows how many blocks it has
      const unsigned long long last = __ballot((left >> tid & 1) && mine.source == begin);
      const int held = __builtin_amdgcn_readlane(mine.blocks, __ffsll((long long)last) - 1);
      for (int s = begin;;) {
        const int from = __builtin_amdgcn_readlane(mine.source, s), blocks = __builtin_amdgcn_readlane(mine.blocks, s);
        if (tid == 0) moves[count] = Move{s, from == begin ? -1 : from, blocks, s == begin ? held : 0};
        ++count;
        left &= ~(1ull << s);
        if (from == begin) break;
        s = from;
      }
    }
    const int most = (int)max_over_wave((unsigned)mine.blocks);
    if (tid == 0) { number = count; most_blocks = most; }
  }
  __syncthreads();
  const int count = __builtin_amdgcn_readfirstlane(number);
  for_pieces(p, first, h, __builtin_amdgcn_readfirstlane(most_blocks), [&](auto* K, auto* V, long long x, int a_block) {
    using Piece = std::remove_reference_t<decltype(*K)>;
    const size_t stride = (size_t)p.H_kv * (p.cache.capacity / kBlock) * a_block;
    K += x;
    V += x;
    Piece held_k{}, held_v{};
    for (int i = 0; i < count; i += kAtOnce) {
      Piece k[kAtOnce], v[kAtOnce];
      int to[kAtOnce], blocks[kAtOnce];
#pragma unroll
      for (int j = 0; j < kAtOnce; ++j) {
        const Move m = moves[min(i + j, count - 1)];
        to[j] = __builtin_amdgcn_readfirstlane(m.to);
        blocks[j] = i + j < count ? __builtin_amdgcn_readfirstlane(m.blocks) : 0;
        const int from = __builtin_amdgcn_readfirstlane(m.from), held = __builtin_amdgcn_readfirstlane(m.held);
        if (i + j < count && x < (long long)held * a_block) {
          held_k = K[to[j] * stride];
          held_v = V[to[j] * stride];
        }
        if (x < (long long)blocks[j] * a_block) {
          k[j] = from < 0 ? held_k : K[from * stride];
          v[j] = from < 0 ? held_v : V[from * stride];
        }
      }
#pragma unroll
      for (int j = 0; j < kAtOnce; ++j)
        if (x < (long long)blocks[j] * a_block) {
          K[to[j] * stride] = k[j];
          V[to[j] * stride] = v[j];
        }
    }
  });
}

// Work-groups of a (sequence or group, head): enough for the chip several times over, and no more than there is work for.
unsigned per_head(long long chunks, long long heads) { return (unsigned)std::min(chunks, std::max(1ll, 8192 / heads)); }

}  // namespace

hipError_t attn_cache_fork_dispatch(const ForkArgs& p, hipStream_t stream) {
  const long long capacity = std::min(p.from.capacity, p.to.capacity), chunks = (capacity * p.d / kPiece + kChunk - 1) / kChunk;
  const dim3 grid(per_head(chunks, (long long)p.B_out * p.H_kv), (unsigned)p.H_kv, (unsigned)p.B_out);
  attn_cache_fork_kernel<<<grid, kThreads, 0, stream>>>(p);
  return hipGetLastError();
}

hipError_t attn_cache_reorder_dispatch(const ReorderArgs& p, hipStream_t stream) {
  const long long chunks = ((long long)p.cache.capacity * p.d / kPiece + kThreads - 1) / kThreads;
  const dim3 grid(per_head(chunks, (long long)p.P * p.H_kv), (unsigned)p.H_kv, (unsigned)p.P);
  if (p.S <= kFew) attn_cache_reorder_kernel<<<grid, kThreads, 0, stream>>>(p);
  else attn_cache_reorder_many_kernel<<<grid, kThreads, 0, stream>>>(p);
  return hipGetLastError();
}
