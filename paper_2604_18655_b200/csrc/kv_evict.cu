// Eviction from the streams' own segments by the totals of attention weight that their keys have gathered.
//
// Of the S rows of a (stream, kv head) the B = budget that stay are the first in the order: rows no older than `recent`
// positions, then falling total (NaN lowest, -0 = +0), then rising index.  The cache is a set as far as attention goes (a key
// carries its position in its rotation), so nothing is shifted: the kept rows behind index B, in rising order, take the places
// of the dropped rows before it, in rising order.  What moves is at most min(B, S - B) rows -- one row for a segment that is one
// over its budget -- and sources (>= B) and destinations (< B) are disjoint, so all rows move at once, in place.
//
// kv_select_kernel: one CTA per (stream, kv head) finds the B-th row of that order by radix selection over order-preserving
// 32-bit images of the totals (11 + 11 + 10 bits, histograms in shared memory), ranks holes and movers by counting, and writes
// the list of moves.  kv_move_kernel: the whole GPU moves the rows of all lists.
#include "../../include/mlora.h"
#include "cache_ops.cuh"

namespace mlora {

constexpr int EV_THREADS = 1024, EV_WARPS = 32;

__device__ __forceinline__ uint32_t ev_image(float w) {
  if (w == 0.f) w = 0.f;
  const uint32_t b = __float_as_uint(w);
  return (w != w) ? 0u : ((b & 0x80000000u) ? ~b : (b | 0x80000000u));
}

// sum over the CTA, known to every thread
__device__ __forceinline__ int ev_total(int v, int* s_w) {
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  v = __reduce_add_sync(0xffffffffu, v);
  __syncthreads();
  if (lane == 0) s_w[warp] = v;
  __syncthreads();
  return __reduce_add_sync(0xffffffffu, s_w[lane]);
}
// what the warps before this one have in all (v: this warp's count, the same in every lane), and the total
__device__ __forceinline__ int ev_before(int v, int* s_w, int& total) {
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  __syncthreads();
  if (lane == 0) s_w[warp] = v;
  __syncthreads();
  const int c = s_w[lane];
  total = __reduce_add_sync(0xffffffffu, c);
  return __reduce_add_sync(0xffffffffu, lane < warp ? c : 0);
}

__global__ void __launch_bounds__(EV_THREADS) kv_select_kernel(const EvictArgs p) {
  __shared__ int hist[2048];
  __shared__ int s_w[EV_WARPS];
  __shared__ int s_bin, s_above;
  const int kh = blockIdx.x, s = blockIdx.y, pair = s * p.Hkv + kh;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const size_t base = (size_t)pair * p.cap;
  const float* w = p.weight + base;
  const int32_t* pos = p.position != nullptr ? p.position + base : nullptr;
  int S = p.suffix_len[s];
  if (S < 0 || S > p.bound) {                              // stay in bounds, report
    if (tid == 0 && kh == 0) atomicCAS(p.status, 0, MLORA_ERR_ARG);
    S = S < 0 ? 0 : p.bound;
  }
  const int B = p.budget;
  if (tid == 0 && kh == 0) p.out_len[s] = min(S, B);
  const bool recency = p.recent > 0 && pos != nullptr;
  const long long from = recency ? (long long)p.newest[s] - p.recent : 0;
  auto is_new = [&](int i) { return recency && (long long)pos[i] > from; };
  if (S <= B) {                                            // nothing to drop
    if (tid == 0) p.counts[pair] = 0;
    for (int i = tid; i < S; i += EV_THREADS) {
      if (p.out_weight != p.weight) p.out_weight[base + i] = w[i];
      if (pos != nullptr && p.out_position != p.position) p.out_position[base + i] = pos[i];
    }
    if (p.out_source != nullptr)
      for (int i = tid; i < S; i += EV_THREADS) p.out_source[(size_t)pair * B + i] = i;
    return;
  }
  // ---- the class in which the order is decided: the new rows where they alone fill the budget, else the others
  int mine = 0;
  for (int i = tid; i < S; i += EV_THREADS) mine += is_new(i);
  const int n_new = ev_total(mine, s_w);
  const bool among_new = n_new >= B;
  int want = among_new ? B : B - n_new;                    // rows of the class that stay (may be 0)
  // ---- radix selection: `prefix` = the leading bits of the want-th largest image of the class
  uint32_t prefix = 0;
  const int shift[3] = {21, 10, 0}, bits[3] = {11, 11, 10};
  for (int ps = 0; ps < 3 && want > 0; ++ps) {
    for (int i = tid; i < 2048; i += EV_THREADS) hist[i] = 0;
    __syncthreads();
    const int top = shift[ps] + bits[ps];
    for (int i = tid; i < S; i += EV_THREADS) {
      const uint32_t k = ev_image(w[i]);
      if (is_new(i) == among_new && (top == 32 || (k >> top) == (prefix >> top))) atomicAdd(&hist[(k >> shift[ps]) & ((1 << bits[ps]) - 1)], 1);
    }
    __syncthreads();
    // bins from the top: thread i has bins 2047 - 2i and 2046 - 2i
    const int b1 = hist[2047 - 2 * tid], b0 = hist[2046 - 2 * tid];
    int inc = b1 + b0;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) { const int x = __shfl_up_sync(0xffffffffu, inc, o); if (lane >= o) inc += x; }
    int total;
    const int before = ev_before(__shfl_sync(0xffffffffu, inc, 31), s_w, total) + inc - b1 - b0;
    if (before < want && want <= before + b1) { s_bin = 2047 - 2 * tid; s_above = before; }
    else if (before + b1 < want && want <= before + b1 + b0) { s_bin = 2046 - 2 * tid; s_above = before + b1; }
    __syncthreads();
    prefix |= (uint32_t)s_bin << shift[ps];
    want -= s_above;
    __syncthreads();
  }
  // now: images of the class above `prefix` stay, and the first `want` equal to it
  const bool none = (among_new ? B : B - n_new) == 0;
  const int seg = (S + EV_WARPS * 32 - 1) / (EV_WARPS * 32) * 32, i0 = warp * seg, i1 = min(S, i0 + seg);
  int eq = 0;
  for (int i = i0 + lane; i - lane < i1; i += 32) {
    const bool e = i < i1 && !none && is_new(i) == among_new && ev_image(w[i]) == prefix;
    eq += __popc(__ballot_sync(0xffffffffu, e));
  }
  int total;
  const int eq_before = ev_before(eq, s_w, total);
  // ---- holes and movers, counted, then listed
  auto walk = [&](auto&& use) {
    int seen = eq_before;
    for (int i = i0 + lane; i - lane < i1; i += 32) {
      bool stay = false, e = false;
      if (i < i1) {
        const bool nw = is_new(i);
        const uint32_t k = ev_image(w[i]);
        if (nw != among_new) stay = nw;
        else if (!none) { stay = k > prefix; e = k == prefix; }
      }
      const unsigned em = __ballot_sync(0xffffffffu, e);
      if (e && seen + __popc(em & ((1u << lane) - 1)) < want) stay = true;
      seen += __popc(em);
      use(i, stay, __ballot_sync(0xffffffffu, i < i1 && i < B && !stay), __ballot_sync(0xffffffffu, i < i1 && i >= B && stay));
    }
  };
  int holes = 0, movers = 0;
  walk([&](int, bool, unsigned hm, unsigned mm) { holes += __popc(hm); movers += __popc(mm); });
  int n_moves;
  int h_at = ev_before(holes, s_w, n_moves), m_at = ev_before(movers, s_w, n_moves);
  if (tid == 0) p.counts[pair] = n_moves;
  int2* list = p.moves + (size_t)pair * p.max_moves;
  walk([&](int i, bool stay, unsigned hm, unsigned mm) {
    const unsigned below = (1u << lane) - 1;
    if ((hm >> lane) & 1u) list[h_at + __popc(hm & below)].y = i;
    if ((mm >> lane) & 1u) list[m_at + __popc(mm & below)].x = i;
    h_at += __popc(hm); m_at += __popc(mm);
    if (i < i1 && i < B && stay) {
      if (p.out_weight != p.weight) p.out_weight[base + i] = w[i];
      if (pos != nullptr && p.out_position != p.position) p.out_position[base + i] = pos[i];
      if (p.out_source != nullptr) p.out_source[(size_t)pair * B + i] = i;
    }
  });
}

// 16 bytes a lane; HD / 8 lanes move a K row, as many its V row
template <int HD>
__global__ void __launch_bounds__(256) kv_move_kernel(const EvictArgs p) {
  constexpr int LANES = HD / 4, PER = 256 / LANES;         // lanes of a move, moves of a CTA at a time
  const int pair = blockIdx.y, count = p.counts[pair];
  const int l = threadIdx.x % LANES;
  const size_t base = (size_t)pair * p.cap;
  for (int j = blockIdx.x * PER + threadIdx.x / LANES; j < count; j += gridDim.x * PER) {
    const int2 m = p.moves[(size_t)pair * p.max_moves + j];
    __half* c = (l < LANES / 2 ? p.own_k : p.own_v) + (l % (LANES / 2)) * 8;
    *reinterpret_cast<uint4*>(c + (base + m.y) * HD) = *reinterpret_cast<const uint4*>(c + (base + m.x) * HD);
    if (l == 0) p.out_weight[base + m.y] = p.weight[base + m.x];
    if (l == 1 && p.position != nullptr) p.out_position[base + m.y] = p.position[base + m.x];
    if (l == 2 && p.out_source != nullptr) p.out_source[(size_t)pair * p.budget + m.y] = m.x;
  }
}

cudaError_t launch_kv_evict(const EvictArgs& a, cudaStream_t st) {
  kv_select_kernel<<<dim3(a.Hkv, a.n), EV_THREADS, 0, st>>>(a);
  cudaError_t e = cudaGetLastError();
  if (e != cudaSuccess || a.max_moves == 0) return e;
  const int per = 256 / (a.hd / 4);
  int gx = (a.max_moves + per - 1) / per;
  if (gx > 256) gx = 256;
  const dim3 grid((unsigned)gx, (unsigned)(a.n * a.Hkv));
  if (a.hd == 64) kv_move_kernel<64><<<grid, 256, 0, st>>>(a);
  else kv_move_kernel<128><<<grid, 256, 0, st>>>(a);
  return cudaGetLastError();
}

}  // namespace mlora
