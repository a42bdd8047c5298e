// Attention over shared prefix, own segment and draft tree (Sec. 3.4, 3.5, App. A) that also totals, for every key of the
// cache, the softmax weight that the pass's rows and the query heads of its group gave it: what eviction decides by.
//
//   s[v][j] = q_v . k_j / sqrt(hd)     v = (stream, node, query head of the group), j = key the row sees
//   p[v][j] = exp(s[v][j] - m_v) / sum_j exp(s[v][j] - m_v),   out_v = sum_j p[v][j] V_j,   total_j += sum_v p[v][j]
//
// A key's weight needs the row's maximum and sum over ALL keys, which no CTA of a split key axis knows.  So the first kernel
// (scored_rows_kernel: online softmax over a chunk of keys, partial results as in any split attention) also leaves the scores
// in scratch, and the second one (scored_finish_kernel) joins the partials and sums exp(s - m) / sum over the rows of a key.
// The scores are 4 bytes a row and key against 4 hd bytes of K and V: little where few rows share a KV head.
#include <cuda.h>
#include <cudaTypedefs.h>

#include <type_traits>

#include "../../include/mlora.h"
#include "cache_ops.cuh"
#include "tc.cuh"

namespace mlora {

constexpr int SC_WARPS = 4;

__device__ __forceinline__ float sc_ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// The ancestor-or-self mask of node c of stream s.  A parent that is not an earlier node counts as the root and is reported, as is a root
// that has one.
__device__ __forceinline__ unsigned long long sc_ancestors(const ScoredArgs& p, int s, int c) {
  if (p.parent == nullptr) return c >= 63 ? ~0ull : (1ull << (c + 1)) - 1;
  const int32_t* par = p.parent + (size_t)s * p.T;
  unsigned long long mask = 1ull;
  bool bad = par[0] != -1;
  for (int it = 0; it < 64 && c > 0; ++it) {
    mask |= 1ull << c;
    int pc = par[c];
    if (pc < 0 || pc >= c) { bad = true; pc = 0; }
    c = pc;
  }
  if (bad) atomicCAS(p.status, 0, MLORA_ERR_ARG);
  return mask;
}

// One CTA: 16 query rows of a kv head against a chunk of keys, the warps taking 32 keys (16 of 128 features) in turn, each through a ring of its own
// in shared memory that it fills with 16-byte asynchronous copies (keys past the end as zeros): STAGES - 1 steps ahead, and no warp
// waits for another before the end.  The pieces of a row lie as with the 128-byte swizzle: piece i of key k at i ^ (k mod 8).
// From there to the fragments of mma.m16n8k16 with 16-byte reads, free of bank conflicts.  A product does not depend on the
// order of its features, nor an output on the order of its columns, so both are dealt to suit them:
//   S:  lane (g, t) holds, of key g, the pieces 2 t + j of each 64 features; a piece feeds two k-steps (q is dealt the same way)
//   PV: lane (g, t) holds, of keys 2t, 2t + 1, 2t + 8, 2t + 9, piece g of each 64 features; column g of n-tile i is feature 8 g + i
// Long segments are bound by the bytes of K and V (eight streams of 16384 rows of 8 heads of 128: 85 us, 95% of the copy rate), short ones by the
// length of a step's chain: two products with their exponentials between them take 0.6 us whether a step has 16 keys or 32 (heads of 64,
// eight ragged streams of up to 2048 rows: 14.3 us by 16, 12.3 by 32; at 128 features 32 keys leave an SM one CTA: 12.0 and 14.6 us for
// 8 x 16 nodes).
template <int HD> struct ScCfg {
  static constexpr int KEYS = HD == 64 ? 32 : 16, ROUND = SC_WARPS * KEYS;       // keys of a warp's step, of all warps' (chunks are multiples)
  static constexpr int STAGES = HD == 64 ? 2 : 3, CTAS = HD == 64 ? 3 : 2;       // ring of a warp; CTAs an SM
  static constexpr int STEP = 2 * KEYS * HD * 2;                                 // bytes of a step: its K and V
  static constexpr size_t SMEM = (size_t)SC_WARPS * STAGES * STEP;
};

template <int HD>
__global__ void __launch_bounds__(SC_WARPS * 32, ScCfg<HD>::CTAS) scored_rows_kernel(const ScoredArgs p, const float scale_log2) {
  using C = ScCfg<HD>;
  constexpr int HALVES = HD / 64, KP = 2 * HALVES;         // 64-feature halves; K pieces of a lane and key
  extern __shared__ __align__(128) unsigned char sc_smem[];
  __shared__ float2 ml_s[SC_WARPS][16];
  __shared__ unsigned long long anc_s[16];
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");      // (scored_finish_kernel, which waits for this one)
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, t = lane & 3;
  const int kh = blockIdx.y, G = p.Hq / p.Hkv, R_all = p.n * p.T * G, slots = p.n_prefix_chunks + p.n_own_chunks;
  // ---- which rows, which keys
  int item = blockIdx.x, v0, v1, k0, k1, S = 0, slot, ld;
  const __half *kb, *vb;
  float* sc;
  bool own = false;
  int32_t lone_parent = -1;
  if (item < p.n_prefix_chunks * p.rt_prefix) {
    slot = item / p.rt_prefix;
    v0 = (item - slot * p.rt_prefix) * 16; v1 = min(v0 + 16, R_all);
    k0 = slot * p.prefix_chunk; k1 = min(p.P, k0 + p.prefix_chunk);
    kb = p.prefix_k + (size_t)kh * p.P * HD; vb = p.prefix_v + (size_t)kh * p.P * HD;
    sc = p.sc_prefix; ld = p.ld_prefix;
  } else {
    own = true;
    item -= p.n_prefix_chunks * p.rt_prefix;
    const int rt = item % p.rt_own, chunk = item / p.rt_own % p.n_own_chunks, s = item / (p.rt_own * p.n_own_chunks);
    v0 = s * p.T * G + rt * 16; v1 = min(v0 + 16, (s + 1) * p.T * G);
    S = p.suffix_len[s];
    if (S < 0 || S > p.suffix_bound) {                     // stay in bounds, report
      if (tid == 0) atomicCAS(p.status, 0, MLORA_ERR_ARG);
      S = S < 0 ? 0 : p.suffix_bound;
    }
    slot = p.n_prefix_chunks + chunk;
    k0 = chunk * p.own_chunk; k1 = min(S + p.T, k0 + p.own_chunk);
    if (k1 <= k0) return;                                  // nothing here (the second kernel skips this slot too)
    const size_t seg = ((size_t)s * p.Hkv + kh) * p.cap * HD;
    kb = p.own_k + seg; vb = p.own_v + seg;
    sc = p.sc_own; ld = p.ld_own;
    // (a single row has no mask to make; what its parent says is reported all the same, at the end: nothing waits for it)
    if (p.T == 1 && p.parent != nullptr && k1 > S && tid == 0) lone_parent = p.parent[s];
    if (p.T > 1 && k1 > S && tid < 16) {                   // ancestor-or-self masks of the tile's nodes
      anc_s[tid] = v0 + tid < v1 ? sc_ancestors(p, s, (v0 + tid) / G - s * p.T) : 0ull;
    }
    if (p.T > 1 && k1 > S) __syncthreads();
  }
  // ---- the ring: a lane copies one piece of every RPI-th row
  const uint32_t ring = tc_smem_u32(sc_smem) + warp * C::STAGES * C::STEP;
  constexpr int LPR = HD / 8, RPI = 32 / LPR;              // lanes a row, rows an instruction
  const int c_row = lane / LPR, c_piece = lane % LPR;
  const int steps = (k1 - k0 - warp * C::KEYS + C::ROUND - 1) / C::ROUND;           // (may be negative: none)
  const size_t c_first = (size_t)(k0 + warp * C::KEYS + c_row) * HD + c_piece * 8;
  const __half *c_k = kb + c_first, *c_v = vb + c_first;
  uint32_t c_at[C::KEYS / RPI];                            // where the lane's rows go within a step's K
#pragma unroll
  for (int r = 0; r < C::KEYS; r += RPI) c_at[r / RPI] = (c_piece >> 3) * (C::KEYS * 128) + (r + c_row) * 128 + (((c_piece & 7) ^ ((r + c_row) & 7)) << 4);
  uint32_t c_stage = 0;
  auto copy = [&](int i) {                                 // step i of this warp (in turn)
    if (i < steps) {
      const int left = k1 - (k0 + (i * SC_WARPS + warp) * C::KEYS) - c_row;       // the lane's rows from there on
      const uint32_t dst = ring + c_stage;
      c_stage = c_stage + C::STEP == C::STAGES * C::STEP ? 0 : c_stage + C::STEP;
      if (left + c_row >= C::KEYS) {
#pragma unroll
        for (int r = 0; r < C::KEYS; r += RPI) {
          asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst + c_at[r / RPI]), "l"(c_k + r * HD) : "memory");
          asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst + c_at[r / RPI] + C::KEYS * HD * 2), "l"(c_v + r * HD) : "memory");
        }
      } else {
#pragma unroll
        for (int r = 0; r < C::KEYS; r += RPI) {
          const int n = r < left ? 16 : 0;                 // (nothing is read where the count is 0; the address stays in the segment)
          const size_t back = r < left ? (size_t)r * HD : 0;
          const __half *fk = left > 0 ? c_k + back : kb, *fv = left > 0 ? c_v + back : vb;
          asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst + c_at[r / RPI]), "l"(fk), "r"(n) : "memory");
          asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst + c_at[r / RPI] + C::KEYS * HD * 2), "l"(fv), "r"(n) : "memory");
        }
      }
      c_k += (size_t)C::ROUND * HD; c_v += (size_t)C::ROUND * HD;
    }
    asm volatile("cp.async.commit_group;" ::: "memory");   // (one a step, empty ones too: the count stays)
  };
#pragma unroll
  for (int i = 0; i < C::STAGES - 1; ++i) copy(i);
  // ---- q, rows g and g + 8
  const int va = v0 + g, vz = v0 + g + 8;
  const bool ok_a = va < v1, ok_z = vz < v1;
  uint32_t qf[KP * 2][4];
  auto q_row = [&](int v) { const int m = v / G; return p.q + ((size_t)m * p.Hq + kh * G + (v - m * G)) * HD; };
#pragma unroll
  for (int j = 0; j < KP; ++j) {
    const int f = (j >> 1) * 64 + (2 * t + (j & 1)) * 8;
    uint4 a = make_uint4(0, 0, 0, 0), z = a;
    if (ok_a) a = *reinterpret_cast<const uint4*>(q_row(va) + f);
    if (ok_z) z = *reinterpret_cast<const uint4*>(q_row(vz) + f);
    qf[2 * j][0] = a.x; qf[2 * j][1] = z.x; qf[2 * j][2] = a.y; qf[2 * j][3] = z.y;
    qf[2 * j + 1][0] = a.z; qf[2 * j + 1][1] = z.z; qf[2 * j + 1][2] = a.w; qf[2 * j + 1][3] = z.w;
  }
  unsigned long long anc_a = ~0ull, anc_z = ~0ull;
  const bool tree = own && p.T > 1 && k1 > S;
  if (tree) { anc_a = anc_s[g]; anc_z = anc_s[g + 8]; }
  float o[HALVES * 8][4];
#pragma unroll
  for (int i = 0; i < HALVES * 8; ++i) o[i][0] = o[i][1] = o[i][2] = o[i][3] = 0.f;
  float m_a = -INFINITY, m_z = -INFINITY, l_a = 0.f, l_z = 0.f;
  float* sc_a = sc + ((size_t)kh * R_all + va) * ld + k0 + warp * C::KEYS + 2 * t;
  float* sc_z = sc + ((size_t)kh * R_all + vz) * ld + k0 + warp * C::KEYS + 2 * t;
  const bool high = v0 + 8 < v1;                           // (the same for the whole CTA)
  auto piece = [&](uint32_t tile, int row, int h, int i) {
    uint4 x;
    asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(x.x), "=r"(x.y), "=r"(x.z), "=r"(x.w)
                 : "r"(tile + h * (C::KEYS * 128) + row * 128 + ((i ^ (row & 7)) << 4)) : "memory");
    return x;
  };
  uint32_t r_stage = 0;
  for (int i = 0; i < steps; ++i) {
    const int key0 = k0 + (i * SC_WARPS + warp) * C::KEYS;
    asm volatile("cp.async.wait_group %0;" ::"n"(C::STAGES - 2) : "memory");
    __syncwarp();                                          // (step i is there for all lanes; step i - 1's stage is free)
    copy(i + C::STAGES - 1);
    const uint32_t kt = ring + r_stage, vt = kt + C::KEYS * HD * 2;
    r_stage = r_stage + C::STEP == C::STAGES * C::STEP ? 0 : r_stage + C::STEP;
    float s[C::KEYS / 8][4];
#pragma unroll
    for (int nt = 0; nt < C::KEYS / 8; ++nt) {
      s[nt][0] = s[nt][1] = s[nt][2] = s[nt][3] = 0.f;
#pragma unroll
      for (int j = 0; j < KP; ++j) {
        const uint4 kf = piece(kt, nt * 8 + g, j >> 1, 2 * t + (j & 1));
        mma_16816(s[nt], qf[2 * j], kf.x, kf.y);
        mma_16816(s[nt], qf[2 * j + 1], kf.z, kf.w);
      }
    }
    // rows 8 .. 15 of the tile are left out where there are none (one row a stream has as many as its KV heads have query heads)
    float mx_a = -INFINITY, mx_z = -INFINITY;
#pragma unroll
    for (int nt = 0; nt < C::KEYS / 8; ++nt)
#pragma unroll
      for (int e = 0; e < 4; ++e) s[nt][e] *= scale_log2;
    if (key0 + C::KEYS > k1 || (tree && key0 + C::KEYS > S)) {          // the end of the chunk, or the pass's own rows
#pragma unroll
      for (int nt = 0; nt < C::KEYS / 8; ++nt)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const int key = key0 + nt * 8 + 2 * t + e;
          bool see_a = key < k1, see_z = see_a;
          if (tree && key >= S) { see_a = see_a && ((anc_a >> (key - S)) & 1ull); see_z = see_z && ((anc_z >> (key - S)) & 1ull); }
          if (!see_a) s[nt][e] = -INFINITY;
          if (!see_z) s[nt][2 + e] = -INFINITY;
        }
    }
#pragma unroll
    for (int nt = 0; nt < C::KEYS / 8; ++nt) mx_a = fmaxf(mx_a, fmaxf(s[nt][0], s[nt][1]));
    if (ok_a) {
#pragma unroll
      for (int nt = 0; nt < C::KEYS / 8; ++nt) *reinterpret_cast<float2*>(sc_a + nt * 8) = make_float2(s[nt][0], s[nt][1]);
    }
    sc_a += C::ROUND;
    if (high) {
#pragma unroll
      for (int nt = 0; nt < C::KEYS / 8; ++nt) mx_z = fmaxf(mx_z, fmaxf(s[nt][2], s[nt][3]));
      if (ok_z) {
#pragma unroll
        for (int nt = 0; nt < C::KEYS / 8; ++nt) *reinterpret_cast<float2*>(sc_z + nt * 8) = make_float2(s[nt][2], s[nt][3]);
      }
      sc_z += C::ROUND;
    }
#pragma unroll
    for (int x = 1; x <= 2; x <<= 1) {
      mx_a = fmaxf(mx_a, __shfl_xor_sync(0xffffffffu, mx_a, x));
      if (high) mx_z = fmaxf(mx_z, __shfl_xor_sync(0xffffffffu, mx_z, x));
    }
    if (__any_sync(0xffffffffu, mx_a > m_a || mx_z > m_z)) {             // a new maximum: what there is is scaled down
      const float n_a = fmaxf(m_a, mx_a), n_z = fmaxf(m_z, mx_z);
      const float c_a = n_a == -INFINITY ? 1.f : sc_ex2(m_a - n_a), c_z = n_z == -INFINITY ? 1.f : sc_ex2(m_z - n_z);
      m_a = n_a; m_z = n_z;
      l_a *= c_a; l_z *= c_z;
#pragma unroll
      for (int i = 0; i < HALVES * 8; ++i) { o[i][0] *= c_a; o[i][1] *= c_a; o[i][2] *= c_z; o[i][3] *= c_z; }
    }
    const float b_a = m_a == -INFINITY ? 0.f : m_a;
    uint32_t pf[C::KEYS / 16][4] = {};
#pragma unroll
    for (int nt = 0; nt < C::KEYS / 8; ++nt) {
      const float e0 = sc_ex2(s[nt][0] - b_a), e1 = sc_ex2(s[nt][1] - b_a);
      l_a += e0 + e1;
      pf[nt >> 1][(nt & 1) * 2] = h2_as_u32(__floats2half2_rn(e0, e1));   // (weights up to 1 as fp16 for mma: off by 2^-11 of each at most, 2^-25 below 2^-14; l adds up the 32-bit ones)
    }
    if (high) {
      const float b_z = m_z == -INFINITY ? 0.f : m_z;
#pragma unroll
      for (int nt = 0; nt < C::KEYS / 8; ++nt) {
        const float e2 = sc_ex2(s[nt][2] - b_z), e3 = sc_ex2(s[nt][3] - b_z);
        l_z += e2 + e3;
        pf[nt >> 1][(nt & 1) * 2 + 1] = h2_as_u32(__floats2half2_rn(e2, e3));
      }
    }
#pragma unroll
    for (int q = 0; q < C::KEYS / 16; ++q)
#pragma unroll
      for (int h = 0; h < HALVES; ++h) {
        const int r = q * 16 + 2 * t;
        const uint4 x0 = piece(vt, r, h, g), x1 = piece(vt, r + 1, h, g), x2 = piece(vt, r + 8, h, g), x3 = piece(vt, r + 9, h, g);
        const uint32_t w0[4] = {x0.x, x0.y, x0.z, x0.w}, w1[4] = {x1.x, x1.y, x1.z, x1.w};
        const uint32_t w2[4] = {x2.x, x2.y, x2.z, x2.w}, w3[4] = {x3.x, x3.y, x3.z, x3.w};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          mma_16816(o[h * 8 + 2 * e], pf[q], __byte_perm(w0[e], w1[e], 0x5410), __byte_perm(w2[e], w3[e], 0x5410));
          mma_16816(o[h * 8 + 2 * e + 1], pf[q], __byte_perm(w0[e], w1[e], 0x7632), __byte_perm(w2[e], w3[e], 0x7632));
        }
      }
  }
  asm volatile("cp.async.wait_group 0;" ::: "memory");
  __syncthreads();                                         // the rings become the warps' outputs, [SC_WARPS][16][HD]
  float* const o_s = reinterpret_cast<float*>(sc_smem);
  auto o_at = [&](int w, int r, int f) -> float& { return o_s[(w * 16 + r) * HD + f]; };
  // ---- the warps' results joined
#pragma unroll
  for (int x = 1; x <= 2; x <<= 1) {
    l_a += __shfl_xor_sync(0xffffffffu, l_a, x);
    l_z += __shfl_xor_sync(0xffffffffu, l_z, x);
  }
#pragma unroll
  for (int h = 0; h < HALVES; ++h)
#pragma unroll
    for (int i = 0; i < 8; ++i) {                          // columns 2t, 2t + 1 of n-tile i: features 16 t + i, 16 t + 8 + i
      const int f = h * 64 + 16 * t + i;
      o_at(warp, g, f) = o[h * 8 + i][0]; o_at(warp, g, f + 8) = o[h * 8 + i][1];
      o_at(warp, g + 8, f) = o[h * 8 + i][2]; o_at(warp, g + 8, f + 8) = o[h * 8 + i][3];
    }
  if (t == 0) { ml_s[warp][g] = make_float2(m_a, l_a); ml_s[warp][g + 8] = make_float2(m_z, l_z); }
  __syncthreads();
  for (int i = tid; i < (v1 - v0) * (HD / 4); i += SC_WARPS * 32) {
    const int r = i / (HD / 4), c = i % (HD / 4) * 4;
    float M = -INFINITY;
#pragma unroll
    for (int x = 0; x < SC_WARPS; ++x) M = fmaxf(M, ml_s[x][r].x);
    const float Mb = M == -INFINITY ? 0.f : M;
    float L = 0.f;
    float4 a = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int x = 0; x < SC_WARPS; ++x) {
      const float2 ml = ml_s[x][r];
      const float f = sc_ex2(ml.x - Mb);
      const float4 b = *reinterpret_cast<const float4*>(&o_at(x, r, c));
      L += f * ml.y;
      a.x += f * b.x; a.y += f * b.y; a.z += f * b.z; a.w += f * b.w;
    }
    const size_t at = ((size_t)kh * R_all + v0 + r) * slots + slot;
    *reinterpret_cast<float4*>(p.part_o + at * HD + c) = a;
    if (c == 0) *reinterpret_cast<float2*>(p.part_ml + at * 2) = make_float2(M, L);
  }
  if (lone_parent != -1) atomicCAS(p.status, 0, MLORA_ERR_ARG);
}

constexpr int FIN_THREADS = 128, FIN_WARPS = FIN_THREADS / 32, FIN_KEYS = 128;   // keys of a warp, four a lane
constexpr int FIN_ROWS = 512;                              // rows whose maximum and 1 / sum are held at a time
constexpr int FIN_FLY = 8, FIN_ONE = 16;                   // 16-byte, 4-byte reads of a thread on their way at a time

__device__ __forceinline__ int sc_len(const ScoredArgs& p, int s) {
  const int S = p.suffix_len[s];
  return S < 0 ? 0 : (S > p.suffix_bound ? p.suffix_bound : S);
}
// slots of a row of stream s that were written
__device__ __forceinline__ int sc_slots(const ScoredArgs& p, int s) {
  return p.n_prefix_chunks + min(p.n_own_chunks, (sc_len(p, s) + p.T + p.own_chunk - 1) / p.own_chunk);
}

// One warp: row w = kv head * R_all + v joined from its first `ns` slots and written; returns (maximum, 1 / sum).
template <int HD>
__device__ __forceinline__ float2 sc_join_row(const ScoredArgs& p, int w, int R_all, int slots, int lane, int ns) {
  constexpr int N = HD / 32;                               // features of a lane
  const int G = p.Hq / p.Hkv, kh = w / R_all, v = w - kh * R_all, m = v / G;
  const size_t at = (size_t)w * slots;
  const float2* const ml_at = reinterpret_cast<const float2*>(p.part_ml) + at;
  float M = -INFINITY, L = 0.f, a[N] = {};
  for (int i0 = 0; i0 < ns; i0 += FIN_FLY) {               // FIN_FLY slots at a time, in order
    float x[FIN_FLY][N];
    float2 ml[FIN_FLY];
#pragma unroll
    for (int i = 0; i < FIN_FLY; ++i) {
      const int k = i0 + i;
      ml[i] = make_float2(-INFINITY, 0.f);
      if (k >= slots) continue;                            // (a slot that was not written is read and not used)
      asm volatile("ld.global.cg.v2.f32 {%0, %1}, [%2];" : "=f"(ml[i].x), "=f"(ml[i].y) : "l"(ml_at + k) : "memory");
      const float* po = p.part_o + (at + k) * HD + lane * N;
      if constexpr (N == 4) asm volatile("ld.global.cg.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(x[i][0]), "=f"(x[i][1]), "=f"(x[i][2]), "=f"(x[i][3]) : "l"(po) : "memory");
      else asm volatile("ld.global.cg.v2.f32 {%0, %1}, [%2];" : "=f"(x[i][0]), "=f"(x[i][1]) : "l"(po) : "memory");
    }
    float Mn = M;
#pragma unroll
    for (int i = 0; i < FIN_FLY; ++i) Mn = i0 + i < ns ? fmaxf(Mn, ml[i].x) : Mn;
    const float Mb = Mn == -INFINITY ? 0.f : Mn, f0 = sc_ex2(M - Mb);
    M = Mn;
    L *= f0;
#pragma unroll
    for (int j = 0; j < N; ++j) a[j] *= f0;
#pragma unroll
    for (int i = 0; i < FIN_FLY; ++i)
      if (i0 + i < ns) {
        const float f = sc_ex2(ml[i].x - Mb);
        L = fmaf(f, ml[i].y, L);
#pragma unroll
        for (int j = 0; j < N; ++j) a[j] = fmaf(f, x[i][j], a[j]);
      }
  }
  const float inv = 1.f / L;
  __half2* dst = reinterpret_cast<__half2*>(p.out + ((size_t)m * p.Hq + kh * G + (v - m * G)) * HD + lane * N);
#pragma unroll
  for (int j = 0; j < N / 2; ++j) dst[j] = __floats2half2_rn(a[2 * j] * inv, a[2 * j + 1] * inv);
  return make_float2(M == -INFINITY ? 0.f : M, inv);
}

// Blocks: rows of the output (one warp a row), then the prefix keys, then the own keys.  Of up to eight rows a warp takes all, for 128
// keys (four a lane); of more every fourth, for the block's 128 keys, or 32 (one a lane; ONE) where there would be few blocks.
// Bound by the length of its chain of reads, so everything that can goes out first: lengths before the kernel ahead has ended, scores before
// the maxima and sums that say what they count for.
template <int HD, bool ONE>
__global__ void __launch_bounds__(FIN_THREADS, 5) scored_finish_kernel(const ScoredArgs p, const int out_blocks, const int prefix_blocks, const int own_blocks,
                                                                    const int prefix_keys, const int own_keys) {
  __shared__ float2 row_s[FIN_ROWS];
  __shared__ __align__(16) float sum_s[FIN_WARPS][FIN_KEYS];
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, G = p.Hq / p.Hkv, R = p.T * G, R_all = p.n * R, slots = p.n_prefix_chunks + p.n_own_chunks;
  int b = blockIdx.x;
  if (b < out_blocks) {
    const int w = b * FIN_WARPS + warp;
    if (w >= p.Hkv * R_all) return;
    const int ns = sc_slots(p, w % R_all / R);
    asm volatile("griddepcontrol.wait;" ::: "memory");
    sc_join_row<HD>(p, w, R_all, slots, lane, ns);
    return;
  }
  b -= out_blocks;
  const bool own = b >= p.Hkv * prefix_blocks;
  int kh, s = 0, key0, v0, v1, ld, limit;
  const int keys = own ? own_keys : prefix_keys;           // of the block: 512 (few rows), 128 or 32
  const int step = (own ? own_blocks : prefix_blocks) * keys;          // the block's next keys are so many on
  const float* sc;
  float* dst;
  if (!own) {
    kh = b / prefix_blocks; key0 = (b - kh * prefix_blocks) * keys;
    v0 = 0; v1 = R_all; ld = p.ld_prefix; sc = p.sc_prefix; limit = p.P;
    dst = p.prefix_weight + (size_t)kh * p.P;
  } else {
    b -= p.Hkv * prefix_blocks;
    const int seg = b / own_blocks;
    kh = seg % p.Hkv; s = seg / p.Hkv; key0 = (b - seg * own_blocks) * keys;
    v0 = s * R; v1 = v0 + R; ld = p.ld_own; sc = p.sc_own;
    dst = p.own_weight + ((size_t)s * p.Hkv + kh) * p.cap;
    limit = sc_len(p, s) + p.T;
    if (key0 >= limit) return;
  }
  // (the slots of the row that the thread joins first: the lengths are an input)
  const int r_first = min(FIN_ROWS, v1 - v0) <= 2 * FIN_THREADS / 8 ? tid >> 3 : tid;
  const int ns_first = sc_slots(p, (v0 + min(r_first, v1 - v0 - 1)) / R);
  const bool all_rows = keys > FIN_KEYS, one = ONE && keys < FIN_KEYS;
  // (and so are the totals of a warp's first keys, where every warp has its own: 0.2 us of 5.3 for a single stream, 0.6 of 45.6 for sixteen)
  float old4[4];
  auto totals = [&](int k) {
#pragma unroll
    for (int i = 0; i < 4; ++i) old4[i] = k + i < limit ? dst[k + i] : 0.f;
  };
  if (all_rows) totals(key0 + warp * FIN_KEYS + 4 * lane);
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const int r_step = all_rows ? 1 : FIN_WARPS;
  float x[4 * FIN_FLY];                                    // scores: four keys of FIN_FLY rows, or one key of FIN_ONE rows
  auto fetch = [&](int k0, int r0, int rows, int r) {      // the lane's keys from k0 on, of rows r0 + r, r0 + r + r_step, ...
    // (a scratch row is a multiple of 32 keys long; what lies past the last key is read and not used)
    const float* const at = sc + ((size_t)kh * R_all + r0) * ld + (one ? min(k0 + lane, ld - 1) : min(k0 + 4 * lane, ld - 4));
    if (one) {
#pragma unroll
      for (int i = 0; i < FIN_ONE; ++i)
        if (r + i * FIN_WARPS < rows) asm volatile("ld.global.cg.f32 %0, [%1];" : "=f"(x[i]) : "l"(at + (size_t)(r + i * FIN_WARPS) * ld) : "memory");
    } else {
#pragma unroll
      for (int i = 0; i < FIN_FLY; ++i)
        if (r + i * r_step < rows)
          asm volatile("ld.global.cg.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(x[4 * i]), "=f"(x[4 * i + 1]), "=f"(x[4 * i + 2]), "=f"(x[4 * i + 3])
                       : "l"(at + (size_t)(r + i * r_step) * ld) : "memory");
    }
  };
  // Eight lanes a row where there are few rows, else one.
  auto normalise = [&](auto lanes_c, int r0, int rows) {
    constexpr int lanes = decltype(lanes_c)::value, per = FIN_THREADS / lanes;
    const int l = tid & (lanes - 1);
    for (int r = tid / lanes; r < (rows + per - 1) / per * per; r += per) {
      const int v = r0 + min(r, rows - 1), ns = r0 == v0 && r == r_first ? ns_first : sc_slots(p, v / R);
      const float2* const ml_at = reinterpret_cast<const float2*>(p.part_ml) + ((size_t)kh * R_all + v) * slots;
      float M = -INFINITY, L = 0.f;
#pragma unroll 4
      for (int i = l; i < ns; i += lanes) {
        const float2 ml = __ldcg(ml_at + i);
        const float Mn = fmaxf(M, ml.x), Mb = Mn == -INFINITY ? 0.f : Mn;
        L = L * sc_ex2(M - Mb) + ml.y * sc_ex2(ml.x - Mb);
        M = Mn;
      }
#pragma unroll
      for (int o = 1; o < lanes; o <<= 1) {
        const float Mo = __shfl_xor_sync(0xffffffffu, M, o), Lo = __shfl_xor_sync(0xffffffffu, L, o);
        const float Mn = fmaxf(M, Mo), Mb = Mn == -INFINITY ? 0.f : Mn;
        L = L * sc_ex2(M - Mb) + Lo * sc_ex2(Mo - Mb);
        M = Mn;
      }
      if (l == 0 && r < rows) row_s[r] = make_float2(M == -INFINITY ? 0.f : M, 1.f / L);
    }
  };
  auto normalisers = [&](int r0, int rows) {
    if (rows <= 2 * FIN_THREADS / 8) normalise(std::integral_constant<int, 8>{}, r0, rows);
    else normalise(std::integral_constant<int, 1>{}, r0, rows);
  };
  if (all_rows) {
    const int rows = v1 - v0;
    const int mine = key0 + warp * FIN_KEYS;
    fetch(mine, v0, rows, 0);
    normalise(std::integral_constant<int, 8>{}, v0, rows);
    __syncthreads();
    for (int k0 = mine; k0 < limit; k0 += step) {
      const int k = k0 + 4 * lane;
      if (k0 != mine) { fetch(k0, v0, rows, 0); totals(k); }
      float sum[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int i = 0; i < FIN_FLY; ++i)
        if (i < rows) {
          const float2 ml = row_s[i];
#pragma unroll
          for (int j = 0; j < 4; ++j) sum[j] = fmaf(sc_ex2(x[4 * i + j] - ml.x), ml.y, sum[j]);
        }
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (k + i < limit) dst[k + i] = old4[i] + sum[i];
    }
    return;
  }
  const bool once = v1 - v0 <= FIN_ROWS;                   // the rows' normalisers are made once
  for (int k0 = key0; k0 < limit; k0 += step) {
    const bool writes = tid < keys && k0 + tid < limit;
    const float old = writes ? dst[k0 + tid] : 0.f;
    float sum[4] = {0.f, 0.f, 0.f, 0.f};
    for (int r0 = v0; r0 < v1; r0 += FIN_ROWS) {
      const int rows = min(FIN_ROWS, v1 - r0);
      fetch(k0, r0, rows, warp);
      if (!once || k0 == key0) {
        __syncthreads();
        normalisers(r0, rows);
        __syncthreads();
      }
      if (one) {
        for (int r = warp; r < rows; r += FIN_WARPS * FIN_ONE) {
          if (r != warp) fetch(k0, r0, rows, r);
#pragma unroll
          for (int i = 0; i < FIN_ONE; ++i)
            if (r + i * FIN_WARPS < rows) { const float2 ml = row_s[r + i * FIN_WARPS]; sum[i & 3] = fmaf(sc_ex2(x[i] - ml.x), ml.y, sum[i & 3]); }
        }
      } else {
        for (int r = warp; r < rows; r += FIN_WARPS * FIN_FLY) {
          if (r != warp) fetch(k0, r0, rows, r);
#pragma unroll
          for (int i = 0; i < FIN_FLY; ++i)
            if (r + i * FIN_WARPS < rows) {
              const float2 ml = row_s[r + i * FIN_WARPS];
#pragma unroll
              for (int j = 0; j < 4; ++j) sum[j] = fmaf(sc_ex2(x[4 * i + j] - ml.x), ml.y, sum[j]);
            }
        }
      }
    }
    if (k0 != key0) __syncthreads();
    if (one) sum_s[warp][lane] = (sum[0] + sum[1]) + (sum[2] + sum[3]);
    else *reinterpret_cast<float4*>(&sum_s[warp][4 * lane]) = make_float4(sum[0], sum[1], sum[2], sum[3]);
    __syncthreads();
    if (writes) {
      float t = 0.f;
#pragma unroll
      for (int w = 0; w < FIN_WARPS; ++w) t += sum_s[w][tid];
      dst[k0 + tid] = old + t;
    }
  }
}

// ----------------------------------------------------------------------------- many rows a KV head (trees, wide groups)
// Attention as mlora_attention runs it (attn_tc_kernel), its partial results joined by scored_join_kernel, which leaves every row's
// maximum and 1 / sum; a second pass over K alone makes the scores again, on the tensor cores, and sums the weights key by key.  For
// 96 rows a KV head the scores in scratch would be 768 bytes of traffic a key, K is 256.
// scored_weights_kernel: 128 keys of a segment against up to 128 of the rows that see them at a time.  S^T = K Q^T with the keys as
// the rows of the accumulator: a thread owns a key (its tensor-memory lane), so that sums over query rows stay in the thread and no
// order of work can change them.  A CTA keeps one operand and streams the other: a tile of prefix keys against all blocks of rows,
// or a stream's rows (where they are one block) against several tiles of its own keys.  Two accumulators: the next product is made
// while this one's exponentials are.  Many blocks of rows of a prefix tile are shared by a cluster of two CTAs, the second of which hands its
// sums to the first.
// Its floor would be the exponentials, 8 clocks an SM for a row of a tile (16 a clock); it takes three times that: one warpgroup reads an
// accumulator and makes its exponentials in turn, while the other accumulator waits for it (8 x 32 nodes of llama3b heads: exponential unit
// 30% busy, issue 26%, tensor pipe 15%).
constexpr int SW_KEYS = 128, SW_ROWS = 128, SW_THREADS = 160;
template <int HD> struct SwCfg {
  static constexpr uint32_t TILE = SW_KEYS * HD * 2;
  static constexpr size_t SMEM = 3 * (size_t)TILE + 1024;
};

constexpr int JOIN_THREADS = 128;
template <int HD>
__global__ void __launch_bounds__(JOIN_THREADS) scored_join_kernel(const ScoredArgs p) {
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");      // (scored_weights_kernel, which waits for this one)
  const int w = blockIdx.x * (JOIN_THREADS / 32) + (threadIdx.x >> 5), lane = threadIdx.x & 31, R = p.T * (p.Hq / p.Hkv), R_all = p.n * R;
  const AttnArgs& t = p.attn;
  const int ns = w < p.Hkv * R_all ? t.n_prefix_chunks + min(t.n_own_chunks, (sc_len(p, w % R_all / R) + p.T + t.own_chunk - 1) / t.own_chunk) : 0;
  asm volatile("griddepcontrol.wait;" ::: "memory");
  if (w >= p.Hkv * R_all) return;
  const float2 ml = sc_join_row<HD>(p, w, R_all, t.n_prefix_chunks + t.n_own_chunks, lane, ns);
  if (lane == 0) p.row_ml[w] = ml;
}

template <int HD>
__global__ void __launch_bounds__(SW_THREADS, 2)
scored_weights_kernel(const __grid_constant__ ScoredArgs p, const int rb, const int prefix_ctas, const int pair, const int own_ctas, const int own_per, const float scale_log2,
                      const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_pk, const __grid_constant__ CUtensorMap map_ok) {
  constexpr int HALVES = HD / 64;
  constexpr uint32_t TILE = SwCfg<HD>::TILE, HALF = SW_KEYS * 128;
  extern __shared__ __align__(1024) unsigned char sw_smem[];
  __shared__ __align__(8) uint64_t fix_full, mov_full[2], mov_empty[2], s_full[2], s_empty[2];
  __shared__ __align__(16) float2 ml_s[2][SW_ROWS];
  __shared__ unsigned long long anc_s[2][SW_ROWS];
  __shared__ uint32_t tmem_s;
  __shared__ float half_s[SW_KEYS];                        // the second CTA's sums
  const uint32_t fix_sm = (tc_smem_u32(sw_smem) + 1023u) & ~1023u, mov_sm = fix_sm + TILE;
  const int tid = threadIdx.x, warp = __shfl_sync(0xffffffffu, tid >> 5, 0), lane = tid & 31;
  const int kh = blockIdx.y, G = p.Hq / p.Hkv, R = p.T * G, R_all = p.n * R;
  const bool own = (int)blockIdx.x >= prefix_ctas, shared = pair && !own;
  const int second = shared ? blockIdx.x & 1 : 0;          // (its rank in the cluster)
  int s = 0, key0, limit, v_lo = 0, v_hi = R_all, S = 0, units;
  bool mov_k = false;                                      // the keys are what moves
  if (!own) {
    key0 = (blockIdx.x >> pair) * SW_KEYS; limit = p.P;
    units = (R_all + rb - 1) / rb;
    if (shared) {
      const int mine = (units + 1) / 2;
      if (second) { v_lo = mine * rb; units -= mine; } else { units = mine; v_hi = min(R_all, mine * rb); }
    }
  } else {
    const int i = blockIdx.x - prefix_ctas;
    if (i >= p.n * own_ctas) return;                       // (the grid is made of whole clusters)
    s = i / own_ctas; key0 = (i - s * own_ctas) * own_per * SW_KEYS;
    S = sc_len(p, s); limit = S + p.T;
    v_lo = s * R; v_hi = v_lo + R;
    if (key0 >= limit) return;
    mov_k = R <= rb;                                       // (else own_per is 1)
    units = mov_k ? min(own_per, (limit - key0 + SW_KEYS - 1) / SW_KEYS) : (R + rb - 1) / rb;
  }
  if (tid == 0) {
    TC_MBAR_INIT(&fix_full, 1);
    for (int i = 0; i < 2; ++i) { TC_MBAR_INIT(mov_full + i, 1); TC_MBAR_INIT(mov_empty + i, 1); TC_MBAR_INIT(s_full + i, 1); TC_MBAR_INIT(s_empty + i, 4); }
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 4) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(tc_smem_u32(&tmem_s)), "r"(256u) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
  __syncthreads();
  asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
  const uint32_t tmem = __shfl_sync(0xffffffffu, tmem_s, 0);
  float total = 0.f;
  bool complete = false;
  if (warp == 4) {
    // ---- copies and MMAs, by one thread.  Neither K nor q is written by the kernels of this call.
    if (tc_elect()) {
      auto load_q = [&](uint32_t dst, int b, uint32_t bar) {
        tc_expect_tx(bar, HALVES * (uint32_t)rb * 128u);
#pragma unroll
        for (int h = 0; h < HALVES; ++h) at_copy3(dst + h * HALF, &map_q, h * 64, kh * G, (v_lo + b * rb) / G, bar);
      };
      auto load_k = [&](uint32_t dst, int i, uint32_t bar) {
        tc_expect_tx(bar, TILE);
#pragma unroll
        for (int h = 0; h < HALVES; ++h) {
          if (own) at_copy4(dst + h * HALF, &map_ok, h * 64, key0 + i * SW_KEYS, kh, s, bar);
          else at_copy3(dst + h * HALF, &map_pk, h * 64, key0 + i * SW_KEYS, kh, bar);
        }
      };
      auto load = [&](int u) {
        const uint32_t bar = tc_smem_u32(mov_full + (u & 1)), dst = mov_sm + (u & 1) * TILE;
        if (mov_k) load_k(dst, u, bar); else load_q(dst, u, bar);
      };
      if (mov_k) load_q(fix_sm, 0, tc_smem_u32(&fix_full)); else load_k(fix_sm, 0, tc_smem_u32(&fix_full));
      load(0);
      if (units > 1) load(1);
      constexpr uint64_t DESC = ((uint64_t)1 << 46) | ((uint64_t)2 << 61) | ((uint64_t)(1024 >> 4) << 32) | ((uint64_t)1 << 16);
      auto desc = [](uint32_t a) { return DESC | (uint64_t)((a & 0x3FFFF) >> 4); };
      int loaded = units > 1 ? 2 : 1;
      bool alive = tc_wait(tc_smem_u32(&fix_full), 0u, p.status);
      for (int u = 0; u < units && alive; ++u) {
        const int st = u & 1; const uint32_t ph = (uint32_t)((u >> 1) & 1);
        alive = tc_wait(tc_smem_u32(mov_full + st), ph, p.status) && tc_wait(tc_smem_u32(s_empty + st), ph ^ 1u, p.status);
        if (!alive) break;
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        const int n_rows = mov_k ? R : min(rb, v_hi - v_lo - u * rb);
        const uint32_t idesc = (1u << 4) | ((uint32_t)((n_rows + 15) / 16 * 2) << 17) | ((SW_KEYS >> 4) << 24);
        const uint32_t mov = mov_sm + st * TILE, k_sm = mov_k ? mov : fix_sm, q_sm = mov_k ? fix_sm : mov;
#pragma unroll
        for (int kk = 0; kk < HD / 16; ++kk) {
          const uint32_t off = (kk >> 2) * HALF + (kk & 3) * 32;
          asm volatile(
              "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
              "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}"
              ::"r"(tmem + st * 128), "l"(desc(k_sm + off)), "l"(desc(q_sm + off)), "r"(idesc), "r"(kk > 0 ? 1u : 0u) : "memory");
        }
        tc_commit(tc_smem_u32(s_full + st));
        tc_commit(tc_smem_u32(mov_empty + st));
        if (u + 2 < units) {
          alive = tc_wait(tc_smem_u32(mov_empty + st), ph, p.status);
          if (alive) { load(u + 2); loaded = u + 3; }
        }
      }
      // no copy may be in flight when the CTA ends (passes at once unless a wait gave up somewhere)
      if (!alive) {
        tc_wait(tc_smem_u32(&fix_full), 0u, p.status);
        for (int u = loaded > 2 ? loaded - 2 : 0; u < loaded; ++u) tc_wait(tc_smem_u32(mov_full + (u & 1)), (uint32_t)((u >> 1) & 1), p.status);
      }
    }
    __syncwarp();
  } else {
    // ---- weights: thread = key; a block's rows' normalisers are brought by the same threads, one row each, a unit ahead
    asm volatile("griddepcontrol.wait;" ::: "memory");
    float* const dst = own ? p.own_weight + ((size_t)s * p.Hkv + kh) * p.cap : p.prefix_weight + (size_t)kh * p.P;
    const bool tree = own && p.T > 1;
    bool alive = true;
    float2 next = make_float2(0.f, 0.f);
    unsigned long long next_anc = 0ull;
    auto fetch = [&](int b) {
      const int v = v_lo + b * rb + tid;
      next = make_float2(0.f, 0.f);
      if (tid < rb && v < v_hi) {
        asm volatile("ld.global.cg.v2.f32 {%0, %1}, [%2];" : "=f"(next.x), "=f"(next.y) : "l"(p.row_ml + (size_t)kh * R_all + v) : "memory");
        if (tree) next_anc = p.anc[v / G];
      }
    };
    fetch(0);
    float sum[4] = {0.f, 0.f, 0.f, 0.f};
    for (int u = 0; u < units; ++u) {
      const int st = u & 1, ms = mov_k ? 0 : st; const uint32_t ph = (uint32_t)((u >> 1) & 1);
      if (!mov_k || u == 0) {
        ml_s[ms][tid] = next;
        if (tree) anc_s[ms][tid] = next_anc;
        asm volatile("bar.sync 1, 128;" ::: "memory");
        if (!mov_k && u + 1 < units) fetch(u + 1);
      }
      const int tile0 = mov_k ? key0 + u * SW_KEYS : key0, key = tile0 + tid, d = key - S;
      const bool masked = tree && tile0 + SW_KEYS > S;                 // (the same for the whole CTA)
      if (alive) alive = tc_wait(tc_smem_u32(s_full + st), ph, p.status);
      alive = __all_sync(0xffffffffu, alive);                          // (no way out: the other warps wait at the barrier)
      asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
      const int n_rows = !alive ? 0 : mov_k ? R : min(rb, v_hi - v_lo - u * rb);
      const uint32_t at = tmem + st * 128 + ((uint32_t)(warp * 32) << 16);
      // 32 columns at a time, the next ones on their way meanwhile; every step over all of them, so that no exponential waits for
      // the one before (written one column after the other it took 45 clocks a column, eight times the exponential unit's)
      float xs[2][32];
      auto columns = [&](int c0, float (&x)[32], float (&following)[32]) {
        asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
        if (c0 + 32 < n_rows) at_ld32(at + c0 + 32, following);
#pragma unroll
        for (int h = 0; h < 32; h += 16) {
          float m[16], w[16];
#pragma unroll
          for (int i = 0; i < 16; i += 2) {
            const float4 ml = *reinterpret_cast<const float4*>(&ml_s[ms][c0 + h + i]);
            m[i] = ml.x; w[i] = ml.y; m[i + 1] = ml.z; w[i + 1] = ml.w;
          }
#pragma unroll
          for (int i = 0; i < 16; ++i) x[h + i] = fmaf(x[h + i], scale_log2, -m[i]);
          // rows past the end (whatever their accumulator columns hold) and nodes that do not see this key weigh nothing
          if (c0 + 32 > n_rows) {
#pragma unroll
            for (int i = 0; i < 16; ++i) x[h + i] = c0 + h + i < n_rows ? x[h + i] : -INFINITY;
          }
          if (masked) {
            const uint32_t* const words = reinterpret_cast<const uint32_t*>(&anc_s[ms][c0 + h]) + (d >= 32 ? 1 : 0);
            const uint32_t always = d >= 0 ? 0u : 1u;
            uint32_t see[16];
#pragma unroll
            for (int i = 0; i < 16; ++i) see[i] = ((words[2 * i] >> (d & 31)) | always) & 1u;
#pragma unroll
            for (int i = 0; i < 16; ++i) x[h + i] = see[i] ? x[h + i] : -INFINITY;
          }
#pragma unroll
          for (int i = 0; i < 16; ++i) x[h + i] = sc_ex2(x[h + i]);
#pragma unroll
          for (int i = 0; i < 16; ++i) sum[i & 3] = fmaf(x[h + i], w[i], sum[i & 3]);
        }
      };
      if (n_rows > 0) at_ld32(at, xs[0]);
      for (int c0 = 0; c0 < n_rows; c0 += 64) {
        columns(c0, xs[0], xs[1]);
        if (c0 + 32 < n_rows) columns(c0 + 32, xs[1], xs[0]);
      }
      asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
      __syncwarp();
      if (lane == 0) tc_arrive(tc_smem_u32(s_empty + st));
      if (mov_k) {
        if (alive && key < limit) dst[key] += (sum[0] + sum[1]) + (sum[2] + sum[3]);
        sum[0] = sum[1] = sum[2] = sum[3] = 0.f;
      }
    }
    if (!mov_k) {
      total = (sum[0] + sum[1]) + (sum[2] + sum[3]);
      if (shared) half_s[tid] = total;
      else if (alive && key0 + tid < limit) dst[key0 + tid] += total;
    }
    complete = alive;
  }
  asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
  if (shared) {
    asm volatile("barrier.cluster.arrive.release;\n\tbarrier.cluster.wait.acquire;" ::: "memory");
    if (!second && warp < 4) {
      uint32_t at;
      float x;
      asm volatile("mapa.shared::cluster.u32 %0, %1, 1;" : "=r"(at) : "r"(tc_smem_u32(&half_s[tid])));
      asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(x) : "r"(at) : "memory");
      if (complete && key0 + tid < limit) p.prefix_weight[(size_t)kh * p.P + key0 + tid] += total + x;
    }
    asm volatile("barrier.cluster.arrive.release;\n\tbarrier.cluster.wait.acquire;" ::: "memory");   // (read before its owner ends)
  }
  __syncthreads();
  if (warp == 4) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(256u) : "memory");
}

// What the tcgen05 kernels read of the pass: every node's ancestor-or-self mask.  Reports malformed parents and lengths out of their bound.
__global__ void scored_prep_kernel(const ScoredArgs p) {
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");      // (the attention kernel, which waits for this one)
  const int i = blockIdx.x * blockDim.x + threadIdx.x;
  if (i < p.n) {
    const int S = p.suffix_len[i];
    if (S < 0 || S > p.suffix_bound) atomicCAS(p.status, 0, MLORA_ERR_ARG);
  }
  if (i >= p.n * p.T) return;
  const int s = i / p.T;
  p.anc[i] = sc_ancestors(p, s, i - s * p.T);
}

template <int HD>
static cudaError_t sw_launch(const ScoredArgs& a, cudaStream_t st) {
  const int rows = a.n * a.T, G = a.Hq / a.Hkv, rb = G * (SW_ROWS / G);
  scored_prep_kernel<<<(rows + 127) / 128, 128, 0, st>>>(a);
  cudaError_t e = cudaGetLastError();
  if (e != cudaSuccess) return e;
  AttnArgs t = a.attn;
  t.q = a.q; t.prefix_k = a.prefix_k; t.prefix_v = a.prefix_v; t.prefix_head_stride = (size_t)a.P * HD;
  t.own_k = a.own_k; t.own_v = a.own_v; t.own_head_stride = (size_t)a.cap * HD; t.own_stream_stride = t.own_head_stride * a.Hkv;
  // (its CTAs start while the masks are made)
  t.pdl = 1; t.anc_late = 1; t.len_limit = a.suffix_bound + 1; t.suffix_len = a.suffix_len; t.anc = a.anc; t.out = a.out; t.status = a.status; t.part_o = a.part_o; t.part_ml = a.part_ml;
  if ((e = launch_attention(t, st)) != cudaSuccess) return e;
  cudaLaunchConfig_t cfg{};
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr; cfg.numAttrs = 1; cfg.stream = st;
  cfg.gridDim = dim3((unsigned)((rows * a.Hq + JOIN_THREADS / 32 - 1) / (JOIN_THREADS / 32))); cfg.blockDim = dim3(JOIN_THREADS);
  if ((e = cudaLaunchKernelEx(&cfg, scored_join_kernel<HD>, a)) != cudaSuccess) return e;
  const cuuint64_t H = sizeof(__half);
  CUtensorMap mq, mpk, mok;
  {
    const cuuint64_t d[3] = {HD, (cuuint64_t)a.Hq, (cuuint64_t)rows}, s[2] = {HD * H, a.Hq * HD * H};
    const cuuint32_t b[3] = {64, (cuuint32_t)G, (cuuint32_t)(rb / G)};
    if ((e = at_map(a.q, 3, d, s, b, &mq)) != cudaSuccess) return e;
  }
  mpk = mq;
  if (a.P > 0) {
    const cuuint64_t d[3] = {HD, (cuuint64_t)a.P, (cuuint64_t)a.Hkv}, s[2] = {HD * H, t.prefix_head_stride * H};
    const cuuint32_t b[3] = {64, SW_KEYS, 1};
    if ((e = at_map(a.prefix_k, 3, d, s, b, &mpk)) != cudaSuccess) return e;
  }
  {
    const cuuint64_t d[4] = {HD, (cuuint64_t)a.cap, (cuuint64_t)a.Hkv, (cuuint64_t)a.n}, s[3] = {HD * H, t.own_head_stride * H, t.own_stream_stride * H};
    const cuuint32_t b[4] = {64, SW_KEYS, 1, 1};
    if ((e = at_map(a.own_k, 4, d, s, b, &mok)) != cudaSuccess) return e;
  }
  const int prefix_tiles = a.prefix_weight != nullptr ? (a.P + SW_KEYS - 1) / SW_KEYS : 0, own_tiles = (a.suffix_bound + a.T + SW_KEYS - 1) / SW_KEYS;
  // Prefix tiles with several blocks of rows: one CTA each or two; own keys: so many tiles a CTA in turn.  By a CTA's time (a unit is 128
  // keys by a block of rows, three units' worth of fixed cost) and the waves that all CTAs make, two an SM.  (8 x 32 nodes of llama3b
  // heads: one wave of 7 and 5 units 17 us, two waves of 4 and 4 26.)
  const int blocks = (rows * G + rb - 1) / rb;
  int pair = 0, own_per = 1;
  long long cost = -1;
  for (int two = 0; two <= (prefix_tiles > 0 && blocks > 2 ? 1 : 0); ++two)
    for (int per = 1; per <= (a.T * G > rb ? 1 : (own_tiles < 16 ? own_tiles : 16)); ++per) {
      const long long ctas = (long long)a.Hkv * ((prefix_tiles << two) + a.n * ((own_tiles + per - 1) / per));
      const int own_units = a.T * G > rb ? (a.T * G + rb - 1) / rb : per, prefix_units = prefix_tiles > 0 ? (blocks + two) >> two : 0;
      const long long c = (ctas + 2 * 148 - 1) / (2 * 148) * (3 + (own_units > prefix_units ? own_units : prefix_units));
      if (cost < 0 || c < cost) { cost = c; pair = two; own_per = per; }
    }
  const int prefix_ctas = prefix_tiles << pair, own_ctas = (own_tiles + own_per - 1) / own_per;
  cfg.gridDim = dim3((unsigned)((prefix_ctas + a.n * own_ctas + pair) >> pair << pair), (unsigned)a.Hkv);
  cfg.blockDim = dim3(SW_THREADS); cfg.dynamicSmemBytes = SwCfg<HD>::SMEM;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = 2; attr[1].val.clusterDim.y = 1; attr[1].val.clusterDim.z = 1;
  cfg.numAttrs = 1 + pair;
  return cudaLaunchKernelEx(&cfg, scored_weights_kernel<HD>, a, rb, prefix_ctas, pair, own_ctas, own_per, 1.4426950408889634f / sqrtf((float)HD), mq, mpk, mok);
}

cudaError_t init_scored() {
  cudaError_t e;
  if ((e = full_carveout(scored_weights_kernel<64>)) != cudaSuccess || (e = full_carveout(scored_weights_kernel<128>)) != cudaSuccess) return e;
  if ((e = full_carveout(scored_rows_kernel<64>)) != cudaSuccess || (e = full_carveout(scored_rows_kernel<128>)) != cudaSuccess) return e;
  if ((e = full_carveout(scored_finish_kernel<64, false>)) != cudaSuccess || (e = full_carveout(scored_finish_kernel<128, false>)) != cudaSuccess ||
      (e = full_carveout(scored_finish_kernel<64, true>)) != cudaSuccess || (e = full_carveout(scored_finish_kernel<128, true>)) != cudaSuccess) return e;
  if ((e = cudaFuncSetAttribute(scored_rows_kernel<64>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)ScCfg<64>::SMEM)) != cudaSuccess) return e;
  if ((e = cudaFuncSetAttribute(scored_rows_kernel<128>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)ScCfg<128>::SMEM)) != cudaSuccess) return e;
  if ((e = cudaFuncSetAttribute(scored_weights_kernel<64>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)SwCfg<64>::SMEM)) != cudaSuccess) return e;
  return cudaFuncSetAttribute(scored_weights_kernel<128>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)SwCfg<128>::SMEM);
}

// ----------------------------------------------------------------------------- plan
// Which kernels.  A stream with more than 16 rows a KV head: those for few rows while their scores in scratch are few, up to 3 million
// words (heads of 64 features; 0.85 of 128), and up to 256 rows share the prefix.  Few rows / tcgen05, us: heads of 64, 16 nodes of one
// stream, 512 + 64 keys (0.3 M words) 8.2 / 10.5, 8 x 8 nodes, 512 + 1000 keys (3.1 M) 17.8 / 18.3, 2048 + 200 keys (4.6 M) 25.0 / 19.2, 8 x 16
// nodes, 512 + 64 keys (512 rows) 24.0 / 16.2, 16 x 6 nodes, no prefix 11.1 / 12.3; heads of 128, 4 x 8 nodes, 512 + 64 keys (0.4 M) 11.5 / 12.2,
// 8 x 8 (0.9 M) 19.9 / 14.8.
// Up to 16 rows (decode): the tcgen05 ones only for many streams behind a long prefix with own segments so short that it does not matter that
// these fill a few of 128 accumulator columns.  Heads of 64: 32 streams, 8192 + 100 keys (8.4 M words of prefix) 42.4 / 30.7, 16 streams (4.2 M)
// 22.1 / 25.8, 64 streams, 8192 + 500 keys 68.2 / 68.4; heads of 128: 32 streams, 4096 + 100 keys (3.1 M) 37.6 / 27.6, 4096 + 1000 keys 47.0 / 50.6.
static int sc_round(const ScoredArgs& a) { return a.hd == 64 ? ScCfg<64>::ROUND : ScCfg<128>::ROUND; }
static int sc_resident(const ScoredArgs& a, int sm_count) { return sm_count * (a.hd == 64 ? ScCfg<64>::CTAS : ScCfg<128>::CTAS); }
static size_t sc_rows(const ScoredArgs& a) { return (size_t)a.n * a.T * a.Hq; }
static bool sc_tc_possible(const ScoredArgs& a) {          // at some bound
  const int G = a.Hq / a.Hkv;
  if (G > SW_ROWS || !tensor_maps_available()) return false;
  return a.T * G > 16 || ((long long)a.n * a.T * G >= 48 && (long long)sc_rows(a) * a.P >= (a.hd == 64 ? 6000000ll : 2500000ll));
}
// where the tcgen05 kernels are possible: the shortest and longest own segments that they take (longest < shortest: none)
static void sc_tc_bounds(const ScoredArgs& a, int sm_count, long long& lo, long long& hi) {
  const int G = a.Hq / a.Hkv;
  lo = 0; hi = 1ll << 40;
  if (a.T * G <= 16) { hi = 512ll / ((long long)a.n * a.Hkv) * SW_KEYS - a.T; return; }
  if ((a.P > 0 && (long long)a.n * a.T * G > 256) || (long long)a.Hkv * a.n * ((a.T * G + 15) / 16) > sc_resident(a, sm_count)) return;
  const long long few = (a.hd == 64 ? 3000000ll : 850000ll) / (long long)sc_rows(a) - a.P - a.T;
  lo = few < 0 ? 0 : few + 1;
}
static bool sc_tc(const ScoredArgs& a, int sm_count) {
  if (!sc_tc_possible(a)) return false;
  long long lo, hi;
  sc_tc_bounds(a, sm_count, lo, hi);
  return a.suffix_bound >= lo && a.suffix_bound <= hi;
}

// Few rows: the keys in chunks of m rounds, m by a CTA's time (half a microsecond a round, four rounds' worth of fixed cost) and the waves
// that all CTAs make.
static long long sc_ctas(const ScoredArgs& a, long long chunk) {
  auto up = [](long long x, long long y) { return (x + y - 1) / y; };
  return a.Hkv * (a.rt_prefix * up(a.P, chunk) + a.n * (long long)a.rt_own * up((long long)a.suffix_bound + a.T, chunk));
}
static int sc_chunk(const ScoredArgs& a, int sm_count) {
  const long long resident = sc_resident(a, sm_count), round = sc_round(a), own_keys = (long long)a.suffix_bound + a.T;
  const long long most = ((a.P > own_keys ? a.P : own_keys) + round - 1) / round;
  long long best = most, cost = -1;
  for (long long m = most; m >= 1; m -= 1 + m / 16) {
    const long long ctas = sc_ctas(a, m * round);
    if (m < most && ctas > 4 * resident) break;
    const long long c = (ctas + resident - 1) / resident * (4 + m);
    if (cost < 0 || c <= cost) { cost = c; best = m; }
  }
  return (int)(best * round);
}

// Many rows: prefix and own segments in chunks of at most `m` tiles of 128 keys, m by a CTA's time (about 2 us a tile and two and a
// half tiles' worth of fixed cost) and the waves that all CTAs make, two an SM.  (The plan of mlora_attention cuts the prefix first and
// the own segments then: at 8 x 32 nodes, 2048 + 1056 keys, it leaves own segments whole and takes 28 us, this 19.)
static long long sw_ctas(const ScoredArgs& a, int m) {
  const int G = a.Hq / a.Hkv, rb = G * (SW_ROWS / G);
  const long long blocks = ((long long)a.n * a.T * G + rb - 1) / rb, rb_own = (a.T * G + rb - 1) / rb;
  const long long tiles = (a.P + SW_KEYS - 1) / SW_KEYS, own = (a.suffix_bound + a.T + SW_KEYS - 1) / SW_KEYS;
  return a.Hkv * ((tiles + m - 1) / m * blocks + (own + m - 1) / m * a.n * rb_own);
}
static void sw_chunks(ScoredArgs& a, int sm_count) {
  const int tiles = (a.P + SW_KEYS - 1) / SW_KEYS, own = (a.suffix_bound + a.T + SW_KEYS - 1) / SW_KEYS, most = tiles > own ? tiles : own;
  int best = most;
  double cost = 0.0;
  for (int m = most; m >= 1; m -= 1 + m / 16) {
    const long long ctas = sw_ctas(a, m);
    if (m < most && ctas > 4ll * sm_count) break;
    const double c = (double)((ctas + 2 * sm_count - 1) / (2 * sm_count)) * (2.5 + m);
    if (m == most || c < cost) { cost = c; best = m; }
  }
  a.attn.n_prefix_chunks = (tiles + best - 1) / best;
  a.attn.prefix_chunk = (tiles > 0 ? (tiles + a.attn.n_prefix_chunks - 1) / a.attn.n_prefix_chunks : 1) * SW_KEYS;
  a.attn.n_own_chunks = (own + best - 1) / best;
  a.attn.own_chunk = (own + a.attn.n_own_chunks - 1) / a.attn.n_own_chunks * SW_KEYS;
  // (evened out, the last chunks may be empty)
  if (tiles > 0) a.attn.n_prefix_chunks = (tiles * SW_KEYS + a.attn.prefix_chunk - 1) / a.attn.prefix_chunk;
  a.attn.n_own_chunks = (own * SW_KEYS + a.attn.own_chunk - 1) / a.attn.own_chunk;
}

static void sc_plan_few(ScoredArgs& a, int sm_count) {
  const int G = a.Hq / a.Hkv;
  const long long own_keys = (long long)a.suffix_bound + a.T;
  a.tc = 0;
  a.rt_own = (a.T * G + 15) / 16;
  a.rt_prefix = (a.n * a.T * G + 15) / 16;
  const int chunk = sc_chunk(a, sm_count);
  a.prefix_chunk = a.own_chunk = chunk;
  a.n_prefix_chunks = (a.P + chunk - 1) / chunk;
  a.n_own_chunks = (int)((own_keys + chunk - 1) / chunk);
  a.ld_prefix = (a.P + 31) / 32 * 32;
  a.ld_own = (int)((own_keys + 31) / 32 * 32);
}

void scored_plan(ScoredArgs& a, int sm_count) {
  if (!sc_tc(a, sm_count)) { sc_plan_few(a, sm_count); return; }
  a.tc = 1;
  a.attn = AttnArgs{};
  a.attn.P = a.P; a.attn.n = a.n; a.attn.T = a.T; a.attn.Hq = a.Hq; a.attn.Hkv = a.Hkv; a.attn.hd = a.hd; a.attn.suffix_bound = a.suffix_bound;
  a.attn.tc_nq = 1;
  sw_chunks(a, sm_count);
}

// tcgen05 form, behind the partial results: the rows' normalisers and masks (two floats a node), on 16-byte boundaries
static size_t sw_floats(const ScoredArgs& a, size_t slots) { return sc_rows(a) * slots * (a.hd + 2) + 4 + sc_rows(a) * 2 + (size_t)a.n * a.T * 2; }
static size_t sc_floats(const ScoredArgs& a) {
  return sc_rows(a) * ((size_t)(a.n_prefix_chunks + a.n_own_chunks) * (a.hd + 2) + (size_t)a.ld_prefix + a.ld_own);
}
size_t scored_workspace_floats(const ScoredArgs& a) {
  return a.tc ? sw_floats(a, (size_t)a.attn.n_prefix_chunks + a.attn.n_own_chunks) : sc_floats(a);
}

// Each form needs more for a longer bound: the longest up to this one that goes by it counts.
size_t scored_workspace_most(const ScoredArgs& given, int sm_count) {
  ScoredArgs a = given;
  size_t most = 0;
  long long lo = 1ll << 40, hi = -1;                       // bounds that go by the tcgen05 kernels
  if (sc_tc_possible(a)) sc_tc_bounds(a, sm_count, lo, hi);
  if (lo <= given.suffix_bound && lo <= hi) {
    a.suffix_bound = (int)(hi < given.suffix_bound ? hi : given.suffix_bound);
    // a CTA writes at most 128 rows of partial results; there are no more than four an SM, or one for each item, or one a tile
    const long long items = sw_ctas(a, 1 << 28), all = sw_ctas(a, 1), four = 4ll * sm_count;
    const long long ctas = all < four ? all : (items > four ? items : four);
    most = sw_floats(a, 0) + (size_t)(SW_ROWS * ctas) * (a.hd + 2);
  }
  const long long few = given.suffix_bound >= lo && given.suffix_bound <= hi ? lo - 1 : given.suffix_bound;
  if (few >= 0) {
    a.suffix_bound = (int)few;
    sc_plan_few(a, sm_count);
    // a CTA writes 16 rows of partial results; there are no more than four waves of CTAs, or one for each item, or one for each round
    const long long items = sc_ctas(a, 1ll << 40), all = sc_ctas(a, sc_round(a)), four = 4ll * sc_resident(a, sm_count);
    const long long ctas = all < four ? all : (items > four ? items : four);
    const size_t f = (size_t)(16 * ctas) * (a.hd + 2) + sc_rows(a) * ((size_t)a.ld_prefix + a.ld_own);
    most = f > most ? f : most;
  }
  return most;
}

void scored_carve(ScoredArgs& a, float* ws) {              // ws: 16-byte aligned
  a.part_o = ws;
  if (a.tc) {
    const size_t parts = sc_rows(a) * ((size_t)a.attn.n_prefix_chunks + a.attn.n_own_chunks);
    a.part_ml = ws + parts * a.hd;
    float* const at = a.part_ml + (parts * 2 + 3) / 4 * 4;
    a.row_ml = (float2*)at;
    a.anc = (unsigned long long*)(a.row_ml + sc_rows(a));
    return;
  }
  const size_t parts = sc_rows(a) * ((size_t)a.n_prefix_chunks + a.n_own_chunks);
  a.sc_prefix = a.part_o + parts * a.hd;
  a.sc_own = a.sc_prefix + sc_rows(a) * a.ld_prefix;
  a.part_ml = a.sc_own + sc_rows(a) * a.ld_own;
}

template <int HD>
static cudaError_t sc_launch(const ScoredArgs& a, cudaStream_t st) {
  const float scale_log2 = 1.4426950408889634f / sqrtf((float)HD);
  scored_rows_kernel<HD><<<dim3((unsigned)(a.n_prefix_chunks * a.rt_prefix + a.n * a.n_own_chunks * a.rt_own), (unsigned)a.Hkv), SC_WARPS * 32, ScCfg<HD>::SMEM, st>>>(a, scale_log2);
  cudaError_t e = cudaGetLastError();
  if (e != cudaSuccess) return e;
  const int out_blocks = (a.n * a.T * a.Hq + FIN_WARPS - 1) / FIN_WARPS;
  // keys of a block (32 where 128 would leave SMs idle: 8 x 16 rows 512 + 64 keys 16.7 and 13.5 us with 128 and 32, but one row of eight streams
  // behind 4096 keys 10.9 and 14.7), and blocks: one for all keys only as far as that fills the machine, the rest in turns
  auto keys_of = [](long long keys, long long segments, int rows) {
    return rows <= FIN_FLY ? FIN_WARPS * FIN_KEYS : (segments * ((keys + FIN_KEYS - 1) / FIN_KEYS) < 100 ? 32 : FIN_KEYS);
  };
  auto blocks_of = [](long long keys, long long segments, int per) {
    const long long all = (keys + per - 1) / per, fill = (148 * 8 + segments - 1) / segments;
    return (int)(all < fill ? all : fill);
  };
  const int G = a.Hq / a.Hkv, own_all = a.suffix_bound + a.T;
  const int prefix_keys = keys_of(a.P, a.Hkv, a.n * a.T * G), own_keys = keys_of(own_all, (long long)a.n * a.Hkv, a.T * G);
  const int prefix_blocks = a.prefix_weight != nullptr ? blocks_of(a.P, a.Hkv, prefix_keys) : 0;
  const int own_blocks = blocks_of(own_all, (long long)a.n * a.Hkv, own_keys);
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3((unsigned)(out_blocks + a.Hkv * prefix_blocks + a.n * a.Hkv * own_blocks)); cfg.blockDim = dim3(FIN_THREADS); cfg.stream = st;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr; cfg.numAttrs = 1;
  const bool one = prefix_keys < FIN_KEYS || own_keys < FIN_KEYS;
  return cudaLaunchKernelEx(&cfg, one ? scored_finish_kernel<HD, true> : scored_finish_kernel<HD, false>, a, out_blocks, prefix_blocks, own_blocks, prefix_keys, own_keys);
}

cudaError_t launch_attention_scored(const ScoredArgs& a, cudaStream_t st) {
  if (a.tc) return a.hd == 64 ? sw_launch<64>(a, st) : sw_launch<128>(a, st);
  return a.hd == 64 ? sc_launch<64>(a, st) : sc_launch<128>(a, st);
}

}  // namespace mlora
