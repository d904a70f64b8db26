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

// ---- reorder.  A thread has the same piece of all sequences of a group: it reads those that go elsewhere, then writes them, and no other thread
// touches what it reads or writes, so that neither cycles nor copies need memory of their own.
template <int S>
__global__ __launch_bounds__(kThreads) void attn_cache_reorder_kernel(ReorderArgs p) {
  __shared__ int parent[S], blocks[S];     // where sequence s comes from (-1: it stays), and how many blocks
  __shared__ int most;
  const int group = blockIdx.z, h = blockIdx.y, tid = threadIdx.x;
  const size_t first = (size_t)group * p.S;
  if (tid == 0) most = 0;
  __syncthreads();
  if (tid < S) {
    int from = -1, n = 0;
    if (tid < p.S) {
      from = p.parents[first + tid];
      if (from < 0 || from >= p.S) from = tid;
      const int tokens = p.lengths[first + from];
      if (blockIdx.x == 0 && h == 0) p.lengths_out[first + tid] = tokens;
      n = blocks_of(min(max(tokens, 0), p.cache.capacity));
      if (from == tid) from = -1;
    }
    parent[tid] = from;
    blocks[tid] = n;
    if (from >= 0) atomicMax(&most, n);
  }
  __syncthreads();
  const size_t per_sequence = (size_t)p.H_kv * p.cache.capacity * p.d / kPiece, per_block = (size_t)kBlock * p.d / kPiece;
  const size_t at = (first * p.H_kv + h) * p.cache.capacity * p.d / kPiece;
  const long long pieces = (long long)most * per_block;
  auto move = [&](auto* base, size_t stride, long long x, size_t a_block) {
    std::remove_reference_t<decltype(*base)> held[S];
#pragma unroll
    for (int s = 0; s < S; ++s)
      if (parent[s] >= 0 && x < (long long)(blocks[s] * a_block)) held[s] = base[parent[s] * stride + x];
#pragma unroll
    for (int s = 0; s < S; ++s)
      if (parent[s] >= 0 && x < (long long)(blocks[s] * a_block)) base[s * stride + x] = held[s];
  };
  for (long long x = (long long)blockIdx.x * kThreads + tid; x < pieces; x += (long long)gridDim.x * kThreads) {
    move(reinterpret_cast<u32x4*>(p.cache.K) + at, per_sequence, x, per_block);
    move(reinterpret_cast<u32x4*>(p.cache.V) + at, per_sequence, x, per_block);
  }
  if (blockIdx.x == 0) {
    const size_t nb = p.cache.capacity / kBlock, of_scales = (first * p.H_kv + h) * nb;
    for (int blk = tid; blk < most; blk += kThreads) {
      move(p.cache.K_scale + of_scales, p.H_kv * nb, blk, 1);
      move(p.cache.V_scale + of_scales, p.H_kv * nb, blk, 1);
    }
  }
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
  if (p.S <= 4) attn_cache_reorder_kernel<4><<<grid, kThreads, 0, stream>>>(p);
  else if (p.S <= 8) attn_cache_reorder_kernel<8><<<grid, kThreads, 0, stream>>>(p);
  else if (p.S <= 16) attn_cache_reorder_kernel<16><<<grid, kThreads, 0, stream>>>(p);
  else if (p.S <= 32) attn_cache_reorder_kernel<32><<<grid, kThreads, 0, stream>>>(p);
  else attn_cache_reorder_kernel<64><<<grid, kThreads, 0, stream>>>(p);
  return hipGetLastError();
}
