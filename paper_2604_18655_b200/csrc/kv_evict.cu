// Eviction from the streams' own segments by the totals of attention weight that their keys have gathered.
//
// Of the S rows of a (stream, kv head) the B = budget that stay are the first in the order: rows no older than `recent`
// positions, then falling total (NaN lowest, -0 = +0), then rising index.  The cache is a set as far as attention goes (a key
// carries its position in its rotation), so nothing is shifted: the kept rows behind index B, in rising order, take the places
// of the dropped rows before it, in rising order.  What moves is at most min(B, S - B) rows -- one row for a segment that is one
// over its budget -- and sources (>= B) and destinations (< B) are disjoint, so all rows move at once, in place.
//
// kv_select_kernel: one CTA per (stream, kv head) finds the B-th row of that order.  Totals as order-preserving 32-bit images, held
// in registers from one read (up to 16 a thread); then 2048-way histograms over what is left of the range between the smallest and
// the largest image (not over fixed bits: the leading 11 bits of totals of one scale are a few dozen values, on whose counters the
// shared-memory atomics queue up).  At most three rounds; holes and movers are ranked by ballots.  Few moves are carried out by the same
// CTA, many by kv_move_kernel, for which the whole GPU takes the rows of all lists.
#include "../../include/mlora.h"
#include "cache_ops.cuh"

namespace mlora {

constexpr int EV_BINS = 2048;

__device__ __forceinline__ uint32_t ev_image(float w) {
  if (w == 0.f) w = 0.f;
  const uint32_t b = __float_as_uint(w);
  return (w != w) ? 0u : ((b & 0x80000000u) ? ~b : (b | 0x80000000u));
}

// 16 bytes a lane; HD / 8 lanes move a K row, as many its V row; FLY rows on their way at a time
template <int HD, int FLY>
__device__ __forceinline__ void ev_move(const EvictArgs& p, const int2* list, int count, int pair, int first, int step, int l) {
  constexpr int LANES = HD / 4;
  const size_t base = (size_t)pair * p.cap;
  __half* const c = (l < LANES / 2 ? p.own_k : p.own_v) + base * HD + (l % (LANES / 2)) * 8;
  for (int j = first; j < count; j += FLY * step) {
    int2 m[FLY];
    uint4 x[FLY];
#pragma unroll
    for (int f = 0; f < FLY; ++f) m[f] = j + f * step < count ? list[j + f * step] : make_int2(-1, -1);
#pragma unroll
    for (int f = 0; f < FLY; ++f)
      if (m[f].x >= 0) x[f] = __ldcs(reinterpret_cast<const uint4*>(c + (size_t)m[f].x * HD));
#pragma unroll
    for (int f = 0; f < FLY; ++f) {
      if (m[f].x < 0) continue;
      *reinterpret_cast<uint4*>(c + (size_t)m[f].y * HD) = x[f];
      if (l == 0) p.out_weight[base + m[f].y] = p.weight[base + m[f].x];
      if (l == 1 && p.position != nullptr) p.out_position[base + m[f].y] = p.position[base + m[f].x];
      if (l == 2 && p.out_source != nullptr) p.out_source[(size_t)pair * p.budget + m[f].y] = m[f].x;
    }
  }
}

// KPT: rows a thread holds in registers (0: any number, read again each time).  Warp w has the rows from w * 32 * KPT on (KPT = 0:
// an even share), lane l every 32nd of them.
template <int THREADS, int KPT>
__global__ void __launch_bounds__(THREADS) kv_select_kernel(const EvictArgs p, const int move_here) {
  constexpr int WARPS = THREADS / 32, PER = EV_BINS / THREADS;
  __shared__ int hist[EV_BINS];
  __shared__ int s_w[2][WARPS];
  __shared__ uint32_t s_lo[WARPS], s_hi[WARPS];
  __shared__ int s_bin, s_above, s_count;
  const int kh = blockIdx.x, s = blockIdx.y, pair = s * p.Hkv + kh;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const size_t base = (size_t)pair * p.cap;
  const float* const w = p.weight + base;
  const int32_t* const pos = p.position != nullptr ? p.position + base : nullptr;
  const bool recency = p.recent > 0 && pos != nullptr;
  int S = p.suffix_len[s];
  const long long from = recency ? (long long)p.newest[s] - p.recent : 0;
  if (S < 0 || S > p.bound) {                              // stay in bounds, report
    if (tid == 0 && kh == 0) atomicCAS(p.status, 0, MLORA_ERR_ARG);
    S = S < 0 ? 0 : p.bound;
  }
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  const int B = p.budget;
  if (tid == 0 && kh == 0) p.out_len[s] = min(S, B);
  int2* const list = p.moves + (size_t)pair * p.max_moves;
  if (S <= B) {                                            // nothing to drop
    if (tid == 0) p.counts[pair] = 0;
    for (int i = tid; i < S; i += THREADS) {
      if (p.out_weight != p.weight) p.out_weight[base + i] = w[i];
      if (pos != nullptr && p.out_position != p.position) p.out_position[base + i] = pos[i];
      if (p.out_source != nullptr) p.out_source[(size_t)pair * B + i] = i;
    }
    return;
  }
  // ---- the rows: image of the total, and which are new
  const int seg = KPT > 0 ? 32 * KPT : (S + WARPS * 32 - 1) / (WARPS * 32) * 32;
  const int i0 = warp * seg + lane, n_j = KPT > 0 ? KPT : seg / 32;
  uint32_t key[KPT > 0 ? KPT : 1];
  uint32_t fresh = 0u;                                     // bit j: row j of the thread is new
  if constexpr (KPT > 0) {
    constexpr int FLY = KPT < 8 ? KPT : 8;                 // reads on their way at a time
#pragma unroll
    for (int j0 = 0; j0 < KPT; j0 += FLY) {
      float x[FLY];
      int32_t q[FLY];
#pragma unroll
      for (int j = 0; j < FLY; ++j) {
        const int i = i0 + (j0 + j) * 32;
        x[j] = i < S ? w[i] : 0.f;
        q[j] = recency && i < S ? pos[i] : INT32_MIN;
      }
#pragma unroll
      for (int j = 0; j < FLY; ++j) {
        key[j0 + j] = ev_image(x[j]);
        fresh |= (uint32_t)(recency && (long long)q[j] > from && i0 + (j0 + j) * 32 < S) << (j0 + j);
      }
    }
  }
  auto is_new = [&](int j) { return KPT > 0 ? (bool)((fresh >> j) & 1u) : (recency && (long long)pos[i0 + j * 32] > from); };
  auto image = [&](int j) { if constexpr (KPT > 0) return key[j]; else return ev_image(w[i0 + j * 32]); };
  auto rows = [&](auto&& f) {                              // the thread's rows in turn; f(j, index, there)
    if constexpr (KPT > 0) {
#pragma unroll
      for (int j = 0; j < KPT; ++j) f(j, i0 + j * 32, i0 + j * 32 < S);
    } else {
      for (int j = 0; j < n_j; ++j) f(j, i0 + j * 32, i0 + j * 32 < S);
    }
  };
  int phase = 0;
  // what the warps before this one have in all (v: this warp's count, the same in every lane), and the total
  auto before = [&](int v, int& total) {
    int* const at = s_w[phase ^= 1];
    if (lane == 0) at[warp] = v;
    __syncthreads();
    const int c = lane < WARPS ? at[lane] : 0;
    total = __reduce_add_sync(0xffffffffu, c);
    return __reduce_add_sync(0xffffffffu, lane < warp ? c : 0);
  };
  // ---- the class in which the order is decided: the new rows where they alone fill the budget, else the others
  bool among_new = false;
  int want = B;
  if (recency) {
    int mine = 0, n_new;
    rows([&](int j, int, bool there) { mine += there && is_new(j); });
    before(__reduce_add_sync(0xffffffffu, mine), n_new);
    among_new = n_new >= B;
    want = among_new ? B : B - n_new;                      // rows of the class that stay (may be 0)
  }
  const bool none = want == 0;
  // ---- the range of the class's images, then the bin of the want-th largest, again within that bin, ...
  uint32_t lo = 0xffffffffu, hi = 0u;
  rows([&](int j, int, bool there) {
    if (there && is_new(j) == among_new) { const uint32_t k = image(j); lo = min(lo, k); hi = max(hi, k); }
  });
  lo = __reduce_min_sync(0xffffffffu, lo); hi = __reduce_max_sync(0xffffffffu, hi);
  if (lane == 0) { s_lo[warp] = lo; s_hi[warp] = hi; }
  for (int i = tid; i < EV_BINS; i += THREADS) hist[i] = 0;
  __syncthreads();
  lo = __reduce_min_sync(0xffffffffu, s_lo[lane < WARPS ? lane : 0]); hi = __reduce_max_sync(0xffffffffu, s_hi[lane < WARPS ? lane : 0]);
  bool all_equal_stay = none;                              // the rows at `lo` all stay: nothing to count among them
  while (!none) {
    const int shift = max(0, 32 - __clz(hi - lo) - 11);    // (hi - lo) >> shift < 2048
    rows([&](int j, int, bool there) {
      if (there && is_new(j) == among_new) { const uint32_t k = image(j); if (k >= lo && k <= hi) atomicAdd(&hist[(k - lo) >> shift], 1); }
    });
    __syncthreads();
    // bins from the top, PER a thread: 2047 - PER tid - i
    int b[PER], inc = 0;
#pragma unroll
    for (int i = 0; i < PER; ++i) { b[i] = hist[EV_BINS - 1 - PER * tid - i]; inc += b[i]; }
    const int mine = inc;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) { const int x = __shfl_up_sync(0xffffffffu, inc, o); if (lane >= o) inc += x; }
    int total;
    int above = before(__shfl_sync(0xffffffffu, inc, 31), total) + inc - mine;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      hist[EV_BINS - 1 - PER * tid - i] = 0;
      if (above < want && want <= above + b[i]) { s_bin = EV_BINS - 1 - PER * tid - i; s_above = above; s_count = b[i]; }
      above += b[i];
    }
    __syncthreads();
    want -= s_above;
    lo += (uint32_t)s_bin << shift;
    hi = min(hi, lo + ((1u << shift) - 1u));
    all_equal_stay = want == s_count;
    if (all_equal_stay || lo == hi) break;                 // (a whole bin stays, or one value is left)
  }
  // ---- rows of the class at or above `lo` stay -- of those equal to it the first `want`, where not all do
  int eq_before = 0;
  if (!all_equal_stay) {
    int eq = 0, total;
    rows([&](int j, int, bool there) { eq += __popc(__ballot_sync(0xffffffffu, there && is_new(j) == among_new && image(j) == lo)); });
    eq_before = before(eq, total);
  }
  auto walk = [&](auto&& use) {
    int seen = eq_before;
    rows([&](int j, int i, bool there) {
      bool stay = false;
      if (there) {
        const bool nw = is_new(j);
        stay = nw != among_new ? nw : !none && image(j) >= lo;
      }
      if (!all_equal_stay) {
        const bool e = there && is_new(j) == among_new && image(j) == lo;
        const unsigned em = __ballot_sync(0xffffffffu, e);
        if (e && seen + __popc(em & ((1u << lane) - 1)) >= want) stay = false;
        seen += __popc(em);
      }
      use(j, i, stay, __ballot_sync(0xffffffffu, there && i < B && !stay), __ballot_sync(0xffffffffu, there && i >= B && stay));
    });
  };
  int holes = 0, movers = 0;
  walk([&](int, int, bool, unsigned hm, unsigned mm) { holes += __popc(hm); movers += __popc(mm); });
  int n_moves;
  int h_at = before(holes, n_moves), m_at = before(movers, n_moves);
  if (tid == 0) p.counts[pair] = n_moves;
  walk([&](int j, int i, bool stay, unsigned hm, unsigned mm) {
    const unsigned below = (1u << lane) - 1;
    if ((hm >> lane) & 1u) list[h_at + __popc(hm & below)].y = i;
    if ((mm >> lane) & 1u) list[m_at + __popc(mm & below)].x = i;
    h_at += __popc(hm); m_at += __popc(mm);
    if (stay && i < B) {
      if (p.out_weight != p.weight) p.out_weight[base + i] = w[i];
      if (pos != nullptr && p.out_position != p.position) p.out_position[base + i] = pos[i];
      if (p.out_source != nullptr) p.out_source[(size_t)pair * B + i] = i;
    }
  });
  if (move_here) {
    __syncthreads();                                       // (the list, through global memory, within the CTA)
    if (p.hd == 64) ev_move<64, 4>(p, list, n_moves, pair, tid / 16, THREADS / 16, tid % 16);
    else ev_move<128, 4>(p, list, n_moves, pair, tid / 32, THREADS / 32, tid % 32);
  }
}

template <int HD>
__global__ void __launch_bounds__(256) kv_move_kernel(const EvictArgs p) {
  constexpr int LANES = HD / 4, PER = 256 / LANES;         // lanes of a move, moves of a CTA at a time
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const int pair = blockIdx.y, first = blockIdx.x * PER * 4;
  ev_move<HD, 4>(p, p.moves + (size_t)pair * p.max_moves, min(p.counts[pair], first + PER * 4), pair, first + threadIdx.x / LANES, PER, threadIdx.x % LANES);
}

template <int THREADS, int KPT>
static cudaError_t ev_select(const EvictArgs& a, int move_here, cudaStream_t st) {
  kv_select_kernel<THREADS, KPT><<<dim3(a.Hkv, a.n), THREADS, 0, st>>>(a, move_here);
  return cudaGetLastError();
}

cudaError_t launch_kv_evict(const EvictArgs& a, cudaStream_t st) {
  const int move_here = a.max_moves <= 256;
  cudaError_t e;
  if (a.bound <= 1024) e = ev_select<256, 4>(a, move_here, st);
  else if (a.bound <= 4096) e = ev_select<1024, 4>(a, move_here, st);
  else if (a.bound <= 8192) e = ev_select<1024, 8>(a, move_here, st);
  else if (a.bound <= 16384) e = ev_select<1024, 16>(a, move_here, st);
  else e = ev_select<1024, 0>(a, move_here, st);
  if (e != cudaSuccess || move_here) return e;
  cudaLaunchConfig_t cfg{};
  const int per = 4 * (256 / (a.hd / 4));
  cfg.gridDim = dim3((unsigned)((a.max_moves + per - 1) / per), (unsigned)(a.n * a.Hkv));
  cfg.blockDim = dim3(256); cfg.stream = st;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr; cfg.numAttrs = 1;
  return a.hd == 64 ? cudaLaunchKernelEx(&cfg, kv_move_kernel<64>, a) : cudaLaunchKernelEx(&cfg, kv_move_kernel<128>, a);
}

}  // namespace mlora
