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

template <int D, int RT, int KW> hipError_t launch_joint(const SharedArgs& a, const CacheForm& f, hipStream_t stream) {
  const AttendArgs& p = a.own;
  attn_cache_joint_kernel<D, RT, KW><<<dim3((unsigned)p.H_kv, (unsigned)f.tiles, (unsigned)p.B), kAttendThreads, 0, stream>>>(a, f.tiles);
  return hipGetLastError();
}
template <int D> hipError_t launch(const SharedArgs& a, hipStream_t stream) {
  const AttendArgs& p = a.own;
  const CacheForm f = cache_form(p.B, p.H, p.H_kv, p.N, D, p.cache.capacity);
  if (f.tiles > 65535) return hipErrorInvalidConfiguration;
  if (f.KW == 4) return launch_joint<D, 1, 4>(a, f, stream);
  if (f.RT == 1) return launch_joint<D, 1, 1>(a, f, stream);
  return launch_joint<D, 2, 1>(a, f, stream);
}

}  // namespace

size_t attn_cache_fwd_shared_partial_bytes(int, int, int, int, int, int, int, int) { return 0; }

hipError_t attn_cache_fwd_shared_dispatch(const SharedArgs& a, int d, hipStream_t stream) {
  switch (d) {
    case 32: return launch<32>(a, stream);
    case 64: return launch<64>(a, stream);
    case 96: return launch<96>(a, stream);
    case 128: return launch<128>(a, stream);
    default: return launch<256>(a, stream);
  }
}
