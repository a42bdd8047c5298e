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
// shared-memory atomics queue up).  At most three rounds; holes and movers are ranked by ballots.  A long segment is shared by a
// cluster of up to eight CTAs, which read each other's histograms and counts through distributed shared memory.  Few moves are
// carried out by the same CTAs, many by kv_move_kernel, for which the whole GPU takes the rows of all lists.
#include "../../include/mlora.h"
#include "cache_ops.cuh"

namespace mlora {

constexpr int EV_BINS = 2048;
constexpr int EV_FEW = 4;                                  // up to so many rows too many are found one by one

__device__ __forceinline__ uint32_t ev_image(float w) {
  if (w == 0.f) w = 0.f;
  const uint32_t b = __float_as_uint(w);
  return (w != w) ? 0u : ((b & 0x80000000u) ? ~b : (b | 0x80000000u));
}

// 16 bytes a lane; HD / 8 lanes move a K row, as many its V row; FLY rows on their way at a time.  What is written is marked to leave L2
// first -- the few rows of a stream at its budget excepted -- and so is what is read where L2 cannot hold the moves: 64 segments 16384 ->
// 8192 rows of 64 features 43.1 us, writes alone marked 55.1, reads alone 52.9, neither 55.4; 32 segments 30.7, 28.8, 29.9 and 32.8.
template <int HD, int FLY>
__device__ __forceinline__ void ev_move(const EvictArgs& p, const int2* list, int count, int pair, int first, int step, int l) {
  constexpr int LANES = HD / 4;
  const size_t base = (size_t)pair * p.cap;
  __half* const c = (l < LANES / 2 ? p.own_k : p.own_v) + base * HD + (l % (LANES / 2)) * 8;
  const uint32_t* const from = l == 0 ? reinterpret_cast<const uint32_t*>(p.weight) + base : (l == 1 && p.position != nullptr ? reinterpret_cast<const uint32_t*>(p.position) + base : nullptr);
  uint32_t* const to = l == 0   ? reinterpret_cast<uint32_t*>(p.out_weight) + base
                       : l == 1 ? (p.position != nullptr ? reinterpret_cast<uint32_t*>(p.out_position) + base : nullptr)
                       : l == 2 && p.out_source != nullptr ? reinterpret_cast<uint32_t*>(p.out_source) + (size_t)pair * p.budget
                                                           : nullptr;
  int2 m[FLY], next[FLY];
  auto ahead = [&](int j) {                                // (the list a round ahead of the rows)
#pragma unroll
    for (int f = 0; f < FLY; ++f) next[f] = j + f * step < count ? list[j + f * step] : make_int2(-1, -1);
  };
  ahead(first);
  for (int j = first; j < count; j += FLY * step) {
    uint4 x[FLY];
    uint32_t side[FLY];                                    // lane 0: the total, lane 1: the position, lane 2: the index
#pragma unroll
    for (int f = 0; f < FLY; ++f) m[f] = next[f];
#pragma unroll
    for (int f = 0; f < FLY; ++f) {
      if (m[f].x < 0) continue;
      const uint4* const row = reinterpret_cast<const uint4*>(c + (size_t)m[f].x * HD);
      x[f] = p.past_l2 ? __ldcs(row) : *row;
      side[f] = from != nullptr ? from[m[f].x] : (uint32_t)m[f].x;
    }
    ahead(j + FLY * step);
#pragma unroll
    for (int f = 0; f < FLY; ++f) {
      if (m[f].x < 0) continue;
      if constexpr (FLY == 1) *reinterpret_cast<uint4*>(c + (size_t)m[f].y * HD) = x[f];
      else __stcs(reinterpret_cast<uint4*>(c + (size_t)m[f].y * HD), x[f]);
      if (to != nullptr) to[m[f].y] = side[f];
    }
  }
}

__device__ __forceinline__ void ev_cluster_sync() {
  asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// the word at `own` in the shared memory of the cluster's CTA `rank`
__device__ __forceinline__ uint32_t ev_remote(const void* own, int rank) {
  uint32_t at, v;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"((uint32_t)__cvta_generic_to_shared(own)), "r"(rank));
  asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(at) : "memory");
  return v;
}

__device__ __forceinline__ int4 ev_remote4(const void* own, int rank) {
  uint32_t at;
  int4 v;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"((uint32_t)__cvta_generic_to_shared(own)), "r"(rank));
  asm volatile("ld.shared::cluster.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(at) : "memory");
  return v;
}

// KPT: rows a thread holds in registers (0: any number, read again each time).  CL: the CTAs of a cluster share the segment.  Warp w of
// CTA c has the rows from (c * WARPS + w) * 32 * KPT on (KPT = 0: an even share), lane l every 32nd of them.  FEW: at most EV_FEW rows are
// too many, which the CTA always moves itself (no list in global memory).
template <int THREADS, int KPT, bool CL, bool FEW>
__global__ void __launch_bounds__(THREADS) kv_select_kernel(const EvictArgs p, const int move_here) {
  constexpr int WARPS = THREADS / 32, PER = EV_BINS / THREADS;
  __shared__ __align__(16) int hist[EV_BINS];
  __shared__ int s_w[2][WARPS];
  __shared__ uint32_t s_lo[WARPS], s_hi[WARPS];
  __shared__ int s_found[3], s_got[3];                     // bin, rows of the class above it, rows in it
  __shared__ uint32_t s_few[2][3][WARPS];                  // few rows too many: a warp's last row (class, image, index)
  __shared__ int s_gone[EV_FEW], s_few_moves;
  __shared__ int2 s_few_list[EV_FEW];
  __shared__ int s_cta[2];
  __shared__ uint32_t s_range[2];
  int rank = 0, ctas = 1;
  if constexpr (CL) {
    asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
    asm("mov.u32 %0, %%cluster_nctaid.x;" : "=r"(ctas));
  }
  const int kh = blockIdx.x / ctas, s = blockIdx.y, pair = s * p.Hkv + kh;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const size_t base = (size_t)pair * p.cap;
  const float* const w = p.weight + base;
  const int32_t* const pos = p.position != nullptr ? p.position + base : nullptr;
  const bool recency = p.recent > 0 && pos != nullptr;
  int S = p.suffix_len[s];
  const long long from = recency ? (long long)p.newest[s] - p.recent : 0;
  if (S < 0 || S > p.bound) {                              // stay in bounds, report
    if (tid == 0 && blockIdx.x == 0) atomicCAS(p.status, 0, MLORA_ERR_ARG);
    S = S < 0 ? 0 : p.bound;
  }
  if (!FEW && !move_here) asm volatile("griddepcontrol.launch_dependents;" ::: "memory");   // (kv_move_kernel, which waits for this one)
  const int B = p.budget;
  if (tid == 0 && blockIdx.x == 0) p.out_len[s] = min(S, B);
  int2* const list = p.moves + (size_t)pair * p.max_moves;
  if (S <= B) {                                            // nothing to drop
    if (!FEW && tid == 0 && rank == 0) p.counts[pair] = 0;
    for (int i = rank * THREADS + tid; i < S; i += ctas * THREADS) {
      if (p.out_weight != p.weight) p.out_weight[base + i] = w[i];
      if (pos != nullptr && p.out_position != p.position) p.out_position[base + i] = pos[i];
      if (p.out_source != nullptr) p.out_source[(size_t)pair * B + i] = i;
    }
    return;
  }
  // ---- the rows, CH of a thread at a time (KPT > 0: all of them, once): images of the totals; bit j of a mask is row i0 + 32 j
  constexpr int CH = KPT > 0 ? KPT : 8, FLY = CH < 8 ? CH : 8;           // (FLY: reads on their way at a time)
  const int seg = KPT > 0 ? 32 * KPT : (S + ctas * WARPS * 32 - 1) / (ctas * WARPS * 32) * 32;
  const int first = (rank * WARPS + warp) * seg + lane, end = min(S, first - lane + seg), chunks = KPT > 0 ? 1 : (seg / 32 + CH - 1) / CH;
  uint32_t key[CH], there = 0u, fresh = 0u;                // in range; new
  int i0 = first;
  auto low_bits = [](int n) { return n >= 32 ? 0xffffffffu : n <= 0 ? 0u : (1u << n) - 1u; };
  auto up_to = [&](int limit) { return low_bits(min(CH, (limit - i0 + 31) >> 5)); };   // rows below index `limit`
  auto fetch = [&](int c) {
    i0 = first + c * CH * 32;
    there = up_to(end);
    fresh = 0u;
#pragma unroll
    for (int j0 = 0; j0 < CH; j0 += FLY) {
      float x[FLY];
      int32_t q[FLY];
#pragma unroll
      for (int j = 0; j < FLY; ++j) {
        const bool ok = (there >> (j0 + j)) & 1u;
        x[j] = ok ? w[i0 + (j0 + j) * 32] : 0.f;
        q[j] = ok && recency ? pos[i0 + (j0 + j) * 32] : INT32_MIN;
      }
#pragma unroll
      for (int j = 0; j < FLY; ++j) {
        key[j0 + j] = ev_image(x[j]);
        if (recency) fresh |= (uint32_t)((long long)q[j] > from) << (j0 + j);
      }
    }
    fresh &= there;
  };
  if (KPT > 0) fetch(0);
  auto pass = [&](auto&& f) {
    for (int c = 0; c < chunks; ++c) {
      if (KPT == 0) fetch(c);
      f();
    }
  };
  int phase = 0;
  // what the warps before this one (of the whole cluster) have in all (v: this warp's count, the same in every lane), and the total
  auto before = [&](int v, int& total) {
    int* const at = s_w[phase ^= 1];
    if (lane == 0) at[warp] = v;
    __syncthreads();
    const int c = lane < WARPS ? at[lane] : 0;
    total = __reduce_add_sync(0xffffffffu, c);
    int sum = __reduce_add_sync(0xffffffffu, lane < warp ? c : 0);
    if constexpr (CL) {
      if (tid == 0) s_cta[phase] = total;
      ev_cluster_sync();
      const int x = lane < ctas ? (int)ev_remote(&s_cta[phase], lane) : 0;
      total = __reduce_add_sync(0xffffffffu, x);
      sum += __reduce_add_sync(0xffffffffu, lane < rank ? x : 0);
    }
    return sum;
  };
  const bool copy_w = p.out_weight != p.weight, copy_p = pos != nullptr && p.out_position != p.position, copies = copy_w || copy_p || p.out_source != nullptr;
  auto copy = [&](uint32_t same) {                         // what stays where it is (all of a batch's reads ahead of its writes)
#pragma unroll
    for (int j0 = 0; j0 < CH; j0 += FLY) {
      float x[FLY];
      int32_t q[FLY];
#pragma unroll
      for (int j = 0; j < FLY; ++j) {
        const int i = i0 + (j0 + j) * 32;
        const bool ok = (same >> (j0 + j)) & 1u;
        x[j] = ok && copy_w ? w[i] : 0.f;
        q[j] = ok && copy_p ? pos[i] : 0;
      }
#pragma unroll
      for (int j = 0; j < FLY; ++j) {
        const int i = i0 + (j0 + j) * 32;
        if (!((same >> (j0 + j)) & 1u)) continue;
        if (copy_w) p.out_weight[base + i] = x[j];
        if (copy_p) p.out_position[base + i] = q[j];
        if (p.out_source != nullptr) p.out_source[(size_t)pair * B + i] = i;
      }
    }
  };
  // ---- a row or a few too many (a stream that decodes at its budget): the last of the order, one after the other -- the smallest image of
  // the rows that are not new, or of the new ones where there are no others; of equals the highest index
  if constexpr (FEW) {
    const int drop = S - B;
    uint32_t alive = there;
    for (int d = 0; d < drop; ++d) {
      uint32_t lowest = 0xffffffffu, lowest_new = 0xffffffffu;
      bool any = false;
#pragma unroll
      for (int j = 0; j < CH; ++j)
        if ((alive >> j) & 1u) {
          if ((fresh >> j) & 1u) lowest_new = min(lowest_new, key[j]);
          else { lowest = min(lowest, key[j]); any = true; }
        }
      lowest = __reduce_min_sync(0xffffffffu, lowest); lowest_new = __reduce_min_sync(0xffffffffu, lowest_new);
      any = __any_sync(0xffffffffu, any);
      // (images reach 0xff800000 at most: 0xffffffff stands for no row)
      const uint32_t mine = any ? lowest : lowest_new;
      int at = -1;
#pragma unroll
      for (int j = 0; j < CH; ++j)
        if (((alive >> j) & 1u) && (bool)((fresh >> j) & 1u) != any && key[j] == mine) at = max(at, i0 + j * 32);
      at = __reduce_max_sync(0xffffffffu, at);
      if (lane == 0) { s_few[d & 1][0][warp] = any ? 0u : 1u; s_few[d & 1][1][warp] = mine; s_few[d & 1][2][warp] = (uint32_t)at; }
      __syncthreads();
      const uint32_t c = lane < WARPS ? s_few[d & 1][0][lane] : 1u, k = lane < WARPS ? s_few[d & 1][1][lane] : 0xffffffffu;
      const int i = lane < WARPS ? (int)s_few[d & 1][2][lane] : -1;
      const uint32_t c_min = __reduce_min_sync(0xffffffffu, c);        // (a warp without rows has class 1 and no image)
      const uint32_t k_min = __reduce_min_sync(0xffffffffu, c == c_min ? k : 0xffffffffu);
      const int gone = __reduce_max_sync(0xffffffffu, c == c_min && k == k_min ? i : -1);
      if (tid == 0) s_gone[d] = gone;
#pragma unroll
      for (int j = 0; j < CH; ++j)
        if (i0 + j * 32 == gone) alive &= ~(1u << j);
    }
    __syncthreads();
    if (copies) copy(alive & up_to(B));
    if (tid == 0) {                                        // the places before the budget, and the rows behind it that stay
      int n_moves = 0, m = B;
      for (int h = 0; h < drop; ++h) {                     // (in rising order: the smallest place not taken yet)
        int place = B;
        for (int d = 0; d < drop; ++d)
          if (s_gone[d] < place && (n_moves == 0 || s_gone[d] > s_few_list[n_moves - 1].y)) place = s_gone[d];
        if (place >= B) break;
        bool gone = true;
        while (m < S && gone) {
          gone = false;
          for (int d = 0; d < drop; ++d) gone = gone || s_gone[d] == m;
          if (gone) ++m;
        }
        s_few_list[n_moves++] = make_int2(m++, place);
      }
      s_few_moves = n_moves;
    }
    __syncthreads();
    if (p.hd == 64) ev_move<64, 1>(p, s_few_list, s_few_moves, pair, tid / 16, THREADS / 16, tid % 16);
    else ev_move<128, 1>(p, s_few_list, s_few_moves, pair, tid / 32, THREADS / 32, tid % 32);
  } else {
  // ---- the class in which the order is decided: the new rows where they alone fill the budget, else the others
  // -- and the range of all images, in which the histograms start.  One exchange for both.
  uint32_t lo = 0xffffffffu, hi = 0u;
  int n_new = 0;
  pass([&] {
    n_new += __popc(fresh);
#pragma unroll
    for (int j = 0; j < CH; ++j)
      if ((there >> j) & 1u) { lo = min(lo, key[j]); hi = max(hi, key[j]); }
  });
  lo = __reduce_min_sync(0xffffffffu, lo); hi = __reduce_max_sync(0xffffffffu, hi); n_new = __reduce_add_sync(0xffffffffu, n_new);
  if (lane == 0) { s_lo[warp] = lo; s_hi[warp] = hi; s_w[0][warp] = n_new; }     // (phase is 0: `before` starts with the other)
  for (int i = tid; i < EV_BINS; i += THREADS) hist[i] = 0;
  __syncthreads();
  lo = __reduce_min_sync(0xffffffffu, s_lo[lane < WARPS ? lane : 0]); hi = __reduce_max_sync(0xffffffffu, s_hi[lane < WARPS ? lane : 0]);
  n_new = __reduce_add_sync(0xffffffffu, lane < WARPS ? s_w[0][lane] : 0);
  if constexpr (CL) {
    if (tid == 0) { s_range[0] = lo; s_range[1] = hi; s_cta[0] = n_new; }
    ev_cluster_sync();
    const int c = lane < ctas ? lane : 0;
    lo = __reduce_min_sync(0xffffffffu, ev_remote(&s_range[0], c)); hi = __reduce_max_sync(0xffffffffu, ev_remote(&s_range[1], c));
    n_new = __reduce_add_sync(0xffffffffu, lane < ctas ? (int)ev_remote(&s_cta[0], lane) : 0);
  }
  const bool among_new = n_new >= B;
  int want = among_new ? B : B - n_new;                    // rows of the class that stay (at least one)
  auto of_class = [&] { return among_new ? fresh : there & ~fresh; };
  // ---- the bin of the want-th largest of the class, again within that bin, ...
  bool all_equal_stay = false;                             // the rows at `lo` all stay: nothing to count among them
  if (tid == 0) s_got[0] = s_got[1] = s_got[2] = 0;
  // (32 bits of range by 11 a round: three are enough; the bound, and those on the list below, hold even if another stream writes the
  // totals meanwhile)
  for (int round = 0; round < 3 && lo < hi; ++round) {
    const int shift = max(0, 32 - __clz(hi - lo) - 11);    // (hi - lo) >> shift < 2048
    pass([&] {
      const uint32_t cls = of_class();
#pragma unroll
      for (int j = 0; j < CH; ++j)
        if (((cls >> j) & 1u) && key[j] - lo <= hi - lo) atomicAdd(&hist[(key[j] - lo) >> shift], 1);
    });
    if constexpr (CL) {
      // every CTA adds up a slice of the bins over all CTAs (16 bytes a read), then the slices' sums tell which one goes on
      ev_cluster_sync();
      const int slice = EV_BINS / ctas, top = (ctas - rank) * slice;   // bins top - slice .. top - 1: the higher, the lower the rank
      int b[4] = {0, 0, 0, 0};
      const bool mine = tid < slice / 4;
      const int at = top - 4 - 4 * tid;
      if (mine)
        for (int c = 0; c < ctas; ++c) {
          const int4 x = ev_remote4(&hist[at], c);
          b[0] += x.w; b[1] += x.z; b[2] += x.y; b[3] += x.x;
        }
      const int sum = b[0] + b[1] + b[2] + b[3];
      int inc = sum, all;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) { const int x = __shfl_up_sync(0xffffffffu, inc, o); if (lane >= o) inc += x; }
      int above = before(__shfl_sync(0xffffffffu, inc, 31), all) + inc - sum;   // (with the slices of lower rank)
      if (mine) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          if (above < want && want <= above + b[i]) { s_found[0] = at + 3 - i; s_found[1] = above; s_found[2] = b[i]; }
          above += b[i];
        }
      }
      for (int i = tid; i < EV_BINS; i += THREADS) hist[i] = 0;        // (read by all: `before` has waited for them)
      // which rank has found it: that of the last slice whose higher ones hold less than is wanted
      int winner;
      {
        const int x = lane < ctas ? (int)ev_remote(&s_cta[phase], lane) : 0;
        int up = x;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) { const int y = __shfl_up_sync(0xffffffffu, up, o); if (lane >= o) up += y; }
        winner = __ffs(__ballot_sync(0xffffffffu, up >= want)) - 1;
      }
      ev_cluster_sync();
      if (tid < 3) s_got[tid] = (int)ev_remote(&s_found[tid], winner);
      __syncthreads();
    } else {
      __syncthreads();
      // bins from the top, PER a thread: 2047 - PER tid - i
      int b[PER], inc = 0;
#pragma unroll
      for (int i = 0; i < PER; ++i) { b[i] = hist[EV_BINS - 1 - PER * tid - i]; inc += b[i]; }
      const int sum = inc;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) { const int x = __shfl_up_sync(0xffffffffu, inc, o); if (lane >= o) inc += x; }
      int all;
      int above = before(__shfl_sync(0xffffffffu, inc, 31), all) + inc - sum;
#pragma unroll
      for (int i = 0; i < PER; ++i) {
        hist[EV_BINS - 1 - PER * tid - i] = 0;
        if (above < want && want <= above + b[i]) { s_got[0] = EV_BINS - 1 - PER * tid - i; s_got[1] = above; s_got[2] = b[i]; }
        above += b[i];
      }
      __syncthreads();
    }
    want -= s_got[1];
    lo += (uint32_t)s_got[0] << shift;
    hi = min(hi, lo + ((1u << shift) - 1u));
    all_equal_stay = want == s_got[2];
    if (all_equal_stay || lo == hi) break;                 // (a whole bin stays, or one value is left)
  }
  // ---- rows of the class at or above `lo` stay -- of those equal to it the first `want`, where not all do
  int seen = 0, total;                                     // rows equal to `lo` ahead of the warp's next one
  if (!all_equal_stay) {
    int eq = 0;
    pass([&] {
      const uint32_t cls = of_class();
#pragma unroll
      for (int j = 0; j < CH; ++j) eq += ((cls >> j) & 1u) && key[j] == lo;
    });
    seen = before(__reduce_add_sync(0xffffffffu, eq), total);
  }
  const unsigned below = (1u << lane) - 1;
  const int seen0 = seen;
  auto stay_bits = [&] {                                   // (once a pass and chunk, in order)
    const uint32_t cls = of_class();
    uint32_t stay = 0u;
#pragma unroll
    for (int j = 0; j < CH; ++j) stay |= (uint32_t)(key[j] >= lo) << j;
    stay &= cls;
    if (!all_equal_stay) {
#pragma unroll
      for (int j = 0; j < CH; ++j) {
        const bool e = ((cls >> j) & 1u) && key[j] == lo;
        const unsigned em = __ballot_sync(0xffffffffu, e);
        if (e && seen + __popc(em & below) >= want) stay &= ~(1u << j);
        seen += __popc(em);
      }
    }
    return among_new ? stay : stay | fresh;
  };
  // holes and movers: counted, ranked, listed
  uint32_t stay = 0u;
  int holes = 0, movers = 0;
  pass([&] {
    stay = stay_bits();
    const uint32_t b = up_to(B);
    holes += __popc(there & b & ~stay); movers += __popc(stay & ~b);
  });
  holes = __reduce_add_sync(0xffffffffu, holes); movers = __reduce_add_sync(0xffffffffu, movers);
  int n_h, n_m;
  int h_at = before(holes, n_h), m_at = before(movers, n_m);
  const int n_moves = min(min(n_h, n_m), p.max_moves);     // (the three agree: see above)
  if (tid == 0 && rank == 0) p.counts[pair] = n_moves;
  seen = seen0;
  pass([&] {
    if (KPT == 0) stay = stay_bits();
    const uint32_t b = up_to(B), h = there & b & ~stay, m = stay & ~b, same = stay & b;
    if (holes + movers > 0) {
#pragma unroll
      for (int j = 0; j < CH; ++j) {
        const unsigned hm = __ballot_sync(0xffffffffu, (h >> j) & 1u), mm = __ballot_sync(0xffffffffu, (m >> j) & 1u);
        const int hj = h_at + __popc(hm & below), mj = m_at + __popc(mm & below);
        if (((h >> j) & 1u) && hj < p.max_moves) list[hj].y = i0 + j * 32;
        if (((m >> j) & 1u) && mj < p.max_moves) list[mj].x = i0 + j * 32;
        h_at += __popc(hm); m_at += __popc(mm);
      }
    }
    if (copies) copy(same);
  });
  // the list, through global memory; and no CTA of a cluster ends while another may read its counts
  if constexpr (CL) ev_cluster_sync(); else __syncthreads();
  if (move_here) {
    if (p.hd == 64) ev_move<64, 4>(p, list, n_moves, pair, rank * (THREADS / 16) + tid / 16, ctas * (THREADS / 16), tid % 16);
    else ev_move<128, 4>(p, list, n_moves, pair, rank * (THREADS / 32) + tid / 32, ctas * (THREADS / 32), tid % 32);
  }
  }
}

template <int HD>
__global__ void __launch_bounds__(256) kv_move_kernel(const EvictArgs p) {
  constexpr int LANES = HD / 4, PER = 256 / LANES;         // lanes of a move, moves of a CTA at a time
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const int pair = blockIdx.y;
  ev_move<HD, 4>(p, p.moves + (size_t)pair * p.max_moves, p.counts[pair], pair, blockIdx.x * PER + threadIdx.x / LANES, gridDim.x * PER, threadIdx.x % LANES);
}

template <int THREADS, int KPT, bool CL, bool FEW = false>
static cudaError_t ev_select(const EvictArgs& a, int ctas, int move_here, cudaStream_t st) {
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3((unsigned)(a.Hkv * ctas), (unsigned)a.n); cfg.blockDim = dim3(THREADS); cfg.stream = st;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = (unsigned)ctas; attr[0].val.clusterDim.y = 1; attr[0].val.clusterDim.z = 1;
  cfg.attrs = attr; cfg.numAttrs = CL ? 1 : 0;
  return cudaLaunchKernelEx(&cfg, kv_select_kernel<THREADS, KPT, CL, FEW>, a, move_here);
}

cudaError_t launch_kv_evict(const EvictArgs& args, cudaStream_t st) {
  EvictArgs a = args;
  // The selecting CTAs move the rows themselves where these are few, or where the segments fill the SMs (one CTA each) to 60% in every
  // wave: 256 segments 4096 -> 2048 rows 36.9 us, 40.6 by a kernel of their own (96 segments 14.6 and 15.2 in a graph; 160 segments 30.9 and 28.7,
  // 16 segments 16.4 and 11.6; of 128 segments with 128 features and up to 8192 rows 54.1 and 51.3: the largest moves lose a little).
  const int pairs = a.n * a.Hkv, waves = (pairs + 147) / 148;
  const int move_here = a.max_moves <= 256 || pairs * 5 >= waves * 148 * 3;
  // About half of the worst case moves, from somewhere to somewhere else: as many bytes as this, of 126 MB.  (67 and 84 MB gain by keeping
  // what is read, 134 MB lose.)
  a.past_l2 = (size_t)pairs * a.max_moves * a.hd * 4 > 100000000;
  const bool few = a.bound - a.budget <= EV_FEW;           // (one row of 257 in eight segments: 2.9 us, 4.3 by histograms)
  cudaError_t e;
  if (few && a.bound <= 1024) e = ev_select<256, 4, false, true>(a, 1, move_here, st);
  else if (few && a.bound <= 4096) e = ev_select<1024, 4, false, true>(a, 1, move_here, st);
  else if (few && a.bound <= 8192) e = ev_select<1024, 8, false, true>(a, 1, move_here, st);
  else if (few && a.bound <= 16384) e = ev_select<1024, 16, false, true>(a, 1, move_here, st);
  else if (a.bound <= 1024) e = ev_select<256, 4, false>(a, 1, move_here, st);
  else if (a.bound <= 4096) e = ev_select<1024, 4, false>(a, 1, move_here, st);
  else if (a.bound <= 8192) e = ev_select<1024, 8, false>(a, 1, move_here, st);
  else if (a.bound <= 16384) e = ev_select<1024, 16, false>(a, 1, move_here, st);
  else if (a.bound <= 131072) e = ev_select<1024, 16, true>(a, a.bound <= 32768 ? 2 : (a.bound <= 65536 ? 4 : 8), move_here, st);
  else e = ev_select<1024, 0, true>(a, 8, move_here, st);
  if (e != cudaSuccess || move_here) return e;             // (always so for the FEW kernels: max_moves is at most EV_FEW)
  cudaLaunchConfig_t cfg{};
  const int per = 4 * (256 / (a.hd / 4)), most = (a.max_moves + per - 1) / per;
  // (as many CTAs as fit, 32 segments 8192 -> 4096 rows 15.4 and 16.8 us by twice as many; twice as many past L2, 64 segments 16384 ->
  // 8192 rows 41.6 and 42.9)
  const int want = ((a.past_l2 ? 2 : 1) * 148 * 8 + pairs - 1) / pairs;
  cfg.gridDim = dim3((unsigned)(most < want ? most : want), (unsigned)pairs);
  cfg.blockDim = dim3(256); cfg.stream = st;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr; cfg.numAttrs = 1;
  return a.hd == 64 ? cudaLaunchKernelEx(&cfg, kv_move_kernel<64>, a) : cudaLaunchKernelEx(&cfg, kv_move_kernel<128>, a);
}

}  // namespace mlora
