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
#include "../../include/mlora.h"
#include "cache_ops.cuh"

namespace mlora {

constexpr int SC_WARPS = 4, SC_STEP = 16;                  // warps of a CTA, keys of a warp's step
constexpr int SC_KEYS = SC_WARPS * SC_STEP;                // keys of a CTA's round; chunks are multiples of it

__device__ __forceinline__ float sc_ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// One CTA: 16 query rows of a kv head against a chunk of keys, the warps taking 16 keys in turn.
// K and V go straight from global memory to the fragments of mma.m16n8k16.  A product does not depend on the order of its
// features, nor an output on the order of its columns, so both are dealt such that a lane reads 16 bytes at a time:
//   S:  lane (g, t) holds, of key g, the pieces 4 j + t of 8 features; a piece feeds two k-steps (q is dealt the same way)
//   PV: lane (g, t) holds, of keys 2t, 2t + 1, 2t + 8, 2t + 9, piece g of each 64 features; column g of n-tile i is feature 8 g + i
template <int HD>
__global__ void __launch_bounds__(SC_WARPS * 32) scored_rows_kernel(const ScoredArgs p, const float scale_log2) {
  constexpr int KP = HD / 32, HALVES = HD / 64;            // K pieces of a lane and key, 64-feature halves of V
  __shared__ float o_s[SC_WARPS][16][HD];
  __shared__ float2 ml_s[SC_WARPS][16];
  __shared__ unsigned long long anc_s[16];
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, t = lane & 3;
  const int kh = blockIdx.y, G = p.Hq / p.Hkv, R_all = p.n * p.T * G, slots = p.n_prefix_chunks + p.n_own_chunks;
  // ---- which rows, which keys
  int item = blockIdx.x, v0, v1, k0, k1, S = 0, slot, ld;
  const __half *kb, *vb;
  float* sc;
  bool own = false;
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
    if (p.T > 1 && k1 > S && tid < 16) {                   // ancestor-or-self masks of the tile's nodes
      unsigned long long mask = 0ull;
      if (v0 + tid < v1) {
        int c = (v0 + tid) / G - s * p.T;
        if (p.parent == nullptr) mask = c >= 63 ? ~0ull : (1ull << (c + 1)) - 1;
        else {
          const int32_t* par = p.parent + (size_t)s * p.T;
          bool bad = par[0] != -1;
          for (int it = 0; it < 64 && c > 0; ++it) {
            mask |= 1ull << c;
            int pc = par[c];
            if (pc < 0 || pc >= c) { bad = true; pc = 0; }
            c = pc;
          }
          mask |= 1ull;
          if (bad) atomicCAS(p.status, 0, MLORA_ERR_ARG);
        }
      }
      anc_s[tid] = mask;
    }
    if (p.T > 1 && k1 > S) __syncthreads();
  }
  // ---- q, rows g and g + 8
  const int va = v0 + g, vz = v0 + g + 8;
  const bool ok_a = va < v1, ok_z = vz < v1;
  uint32_t qf[KP * 2][4];
  auto q_row = [&](int v) { const int m = v / G; return p.q + ((size_t)m * p.Hq + kh * G + (v - m * G)) * HD; };
#pragma unroll
  for (int j = 0; j < KP; ++j) {
    uint4 a = make_uint4(0, 0, 0, 0), z = a;
    if (ok_a) a = *reinterpret_cast<const uint4*>(q_row(va) + j * 32 + t * 8);
    if (ok_z) z = *reinterpret_cast<const uint4*>(q_row(vz) + j * 32 + t * 8);
    qf[2 * j][0] = a.x; qf[2 * j][1] = z.x; qf[2 * j][2] = a.y; qf[2 * j][3] = z.y;
    qf[2 * j + 1][0] = a.z; qf[2 * j + 1][1] = z.z; qf[2 * j + 1][2] = a.w; qf[2 * j + 1][3] = z.w;
  }
  unsigned long long anc_a = ~0ull, anc_z = ~0ull;
  const bool tree = own && p.T > 1 && k1 > S;
  if (tree) { anc_a = anc_s[g]; anc_z = anc_s[g + 8]; }
  // ---- keys
  uint4 kf[2][KP], vf[4][HALVES];
  const uint4 zero = make_uint4(0, 0, 0, 0);
  auto load_k = [&](int key0) {
#pragma unroll
    for (int nt = 0; nt < 2; ++nt) {
      const int key = key0 + nt * 8 + g;
#pragma unroll
      for (int j = 0; j < KP; ++j)
        kf[nt][j] = key < k1 ? __ldcs(reinterpret_cast<const uint4*>(kb + (size_t)key * HD + j * 32 + t * 8)) : zero;
    }
  };
  auto load_v = [&](int key0) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int key = key0 + 2 * t + (i & 1) + (i >> 1) * 8;
#pragma unroll
      for (int h = 0; h < HALVES; ++h)
        vf[i][h] = key < k1 ? __ldcs(reinterpret_cast<const uint4*>(vb + (size_t)key * HD + h * 64 + g * 8)) : zero;
    }
  };
  float o[HALVES * 8][4];
#pragma unroll
  for (int i = 0; i < HALVES * 8; ++i) o[i][0] = o[i][1] = o[i][2] = o[i][3] = 0.f;
  float m_a = -INFINITY, m_z = -INFINITY, l_a = 0.f, l_z = 0.f;
  float* const sc_a = sc + ((size_t)kh * R_all + va) * ld;
  float* const sc_z = sc + ((size_t)kh * R_all + vz) * ld;
  int key0 = k0 + warp * SC_STEP;
  if (key0 < k1) { load_k(key0); load_v(key0); }
  for (; key0 < k1; key0 += SC_KEYS) {
    float s[2][4];
#pragma unroll
    for (int nt = 0; nt < 2; ++nt) {
      s[nt][0] = s[nt][1] = s[nt][2] = s[nt][3] = 0.f;
#pragma unroll
      for (int j = 0; j < KP; ++j) {
        mma_16816(s[nt], qf[2 * j], kf[nt][j].x, kf[nt][j].y);
        mma_16816(s[nt], qf[2 * j + 1], kf[nt][j].z, kf[nt][j].w);
      }
    }
    const int next = key0 + SC_KEYS;
    if (next < k1) load_k(next);
    float mx_a = -INFINITY, mx_z = -INFINITY;
#pragma unroll
    for (int nt = 0; nt < 2; ++nt)
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const int key = key0 + nt * 8 + 2 * t + e;
        bool see_a = key < k1, see_z = see_a;
        if (tree && key >= S) { see_a = see_a && ((anc_a >> (key - S)) & 1ull); see_z = see_z && ((anc_z >> (key - S)) & 1ull); }
        s[nt][e] = see_a ? s[nt][e] * scale_log2 : -INFINITY;
        s[nt][2 + e] = see_z ? s[nt][2 + e] * scale_log2 : -INFINITY;
        mx_a = fmaxf(mx_a, s[nt][e]); mx_z = fmaxf(mx_z, s[nt][2 + e]);
      }
#pragma unroll
    for (int nt = 0; nt < 2; ++nt) {
      const int key = key0 + nt * 8 + 2 * t;
      if (ok_a) *reinterpret_cast<float2*>(sc_a + key) = make_float2(s[nt][0], s[nt][1]);
      if (ok_z) *reinterpret_cast<float2*>(sc_z + key) = make_float2(s[nt][2], s[nt][3]);
    }
#pragma unroll
    for (int x = 1; x <= 2; x <<= 1) {
      mx_a = fmaxf(mx_a, __shfl_xor_sync(0xffffffffu, mx_a, x));
      mx_z = fmaxf(mx_z, __shfl_xor_sync(0xffffffffu, mx_z, x));
    }
    const float n_a = fmaxf(m_a, mx_a), n_z = fmaxf(m_z, mx_z);
    const float b_a = n_a == -INFINITY ? 0.f : n_a, b_z = n_z == -INFINITY ? 0.f : n_z;
    const float c_a = sc_ex2(m_a - b_a), c_z = sc_ex2(m_z - b_z);
    m_a = n_a; m_z = n_z;
    l_a *= c_a; l_z *= c_z;
#pragma unroll
    for (int i = 0; i < HALVES * 8; ++i) { o[i][0] *= c_a; o[i][1] *= c_a; o[i][2] *= c_z; o[i][3] *= c_z; }
    uint32_t pf[4];
#pragma unroll
    for (int nt = 0; nt < 2; ++nt) {
      const float e0 = sc_ex2(s[nt][0] - b_a), e1 = sc_ex2(s[nt][1] - b_a), e2 = sc_ex2(s[nt][2] - b_z), e3 = sc_ex2(s[nt][3] - b_z);
      l_a += e0 + e1; l_z += e2 + e3;
      pf[nt * 2] = h2_as_u32(__floats2half2_rn(e0, e1));   // (weights up to 1 as fp16: half a step of 2^-11 of each)
      pf[nt * 2 + 1] = h2_as_u32(__floats2half2_rn(e2, e3));
    }
#pragma unroll
    for (int h = 0; h < HALVES; ++h) {
      const uint32_t w0[4] = {vf[0][h].x, vf[0][h].y, vf[0][h].z, vf[0][h].w}, w1[4] = {vf[1][h].x, vf[1][h].y, vf[1][h].z, vf[1][h].w};
      const uint32_t w2[4] = {vf[2][h].x, vf[2][h].y, vf[2][h].z, vf[2][h].w}, w3[4] = {vf[3][h].x, vf[3][h].y, vf[3][h].z, vf[3][h].w};
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        mma_16816(o[h * 8 + 2 * i], pf, __byte_perm(w0[i], w1[i], 0x5410), __byte_perm(w2[i], w3[i], 0x5410));
        mma_16816(o[h * 8 + 2 * i + 1], pf, __byte_perm(w0[i], w1[i], 0x7632), __byte_perm(w2[i], w3[i], 0x7632));
      }
    }
    if (next < k1) load_v(next);
  }
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
      o_s[warp][g][f] = o[h * 8 + i][0]; o_s[warp][g][f + 8] = o[h * 8 + i][1];
      o_s[warp][g + 8][f] = o[h * 8 + i][2]; o_s[warp][g + 8][f + 8] = o[h * 8 + i][3];
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
      const float4 b = *reinterpret_cast<const float4*>(&o_s[x][r][c]);
      L += f * ml.y;
      a.x += f * b.x; a.y += f * b.y; a.z += f * b.z; a.w += f * b.w;
    }
    const size_t at = ((size_t)kh * R_all + v0 + r) * slots + slot;
    *reinterpret_cast<float4*>(p.part_o + at * HD + c) = a;
    if (c == 0) *reinterpret_cast<float2*>(p.part_ml + at * 2) = make_float2(M, L);
  }
}

constexpr int FIN_THREADS = 128;
constexpr int FIN_ROWS = 256;                              // rows whose maximum and 1 / sum are held at a time

// slots of row v that were written
__device__ __forceinline__ int sc_slots(const ScoredArgs& p, int s) {
  int S = p.suffix_len[s];
  S = S < 0 ? 0 : (S > p.suffix_bound ? p.suffix_bound : S);
  return p.n_prefix_chunks + min(p.n_own_chunks, (S + p.T + p.own_chunk - 1) / p.own_chunk);
}

// blocks: rows of the output (one warp a row), then the prefix keys (one thread a key), then the own keys
template <int HD>
__global__ void __launch_bounds__(FIN_THREADS) scored_finish_kernel(const ScoredArgs p, const int out_blocks, const int prefix_blocks, const int own_blocks) {
  __shared__ float2 row_s[FIN_ROWS];
  const int tid = threadIdx.x, lane = tid & 31, G = p.Hq / p.Hkv, R = p.T * G, R_all = p.n * R, slots = p.n_prefix_chunks + p.n_own_chunks;
  const float2* const ml_all = reinterpret_cast<const float2*>(p.part_ml);
  int b = blockIdx.x;
  if (b < out_blocks) {
    const int w = b * (FIN_THREADS / 32) + (tid >> 5);
    if (w >= p.Hkv * R_all) return;
    const int kh = w / R_all, v = w - kh * R_all, m = v / G, ns = sc_slots(p, m / p.T);
    const size_t at = (size_t)w * slots;
    float M = -INFINITY, L = 0.f;
    for (int i = 0; i < ns; ++i) M = fmaxf(M, ml_all[at + i].x);
    const float Mb = M == -INFINITY ? 0.f : M;
    float a[HD / 32] = {};
    for (int i = 0; i < ns; ++i) {
      const float2 ml = ml_all[at + i];
      const float f = sc_ex2(ml.x - Mb);
      L += f * ml.y;
#pragma unroll
      for (int j = 0; j < HD / 32; ++j) a[j] += f * p.part_o[(at + i) * HD + lane * (HD / 32) + j];
    }
    const float inv = 1.f / L;
    __half2* dst = reinterpret_cast<__half2*>(p.out + ((size_t)m * p.Hq + kh * G + (v - m * G)) * HD + lane * (HD / 32));
#pragma unroll
    for (int j = 0; j < HD / 64; ++j) dst[j] = __floats2half2_rn(a[2 * j] * inv, a[2 * j + 1] * inv);
    return;
  }
  b -= out_blocks;
  int kh, s = 0, key, v0, v1, ld, limit;
  const float* sc;
  float* dst;
  if (b < p.Hkv * prefix_blocks) {
    kh = b / prefix_blocks; key = (b - kh * prefix_blocks) * FIN_THREADS + tid;
    v0 = 0; v1 = R_all; ld = p.ld_prefix; sc = p.sc_prefix; limit = p.P;
    dst = p.prefix_weight + (size_t)kh * p.P;
  } else {
    b -= p.Hkv * prefix_blocks;
    const int seg = b / own_blocks;
    kh = seg % p.Hkv; s = seg / p.Hkv; key = (b - seg * own_blocks) * FIN_THREADS + tid;
    v0 = s * R; v1 = v0 + R; ld = p.ld_own; sc = p.sc_own;
    int S = p.suffix_len[s];
    limit = (S < 0 ? 0 : (S > p.suffix_bound ? p.suffix_bound : S)) + p.T;
    if (key - tid >= limit) return;
    dst = p.own_weight + ((size_t)s * p.Hkv + kh) * p.cap;
  }
  float sum = 0.f;
  for (int r0 = v0; r0 < v1; r0 += FIN_ROWS) {
    const int rows = min(FIN_ROWS, v1 - r0);
    __syncthreads();
    for (int r = tid; r < rows; r += FIN_THREADS) {
      const int v = r0 + r, ns = sc_slots(p, v / R);
      const size_t at = ((size_t)kh * R_all + v) * slots;
      float M = -INFINITY, L = 0.f;
      for (int i = 0; i < ns; ++i) M = fmaxf(M, ml_all[at + i].x);
      const float Mb = M == -INFINITY ? 0.f : M;
      for (int i = 0; i < ns; ++i) { const float2 ml = ml_all[at + i]; L += sc_ex2(ml.x - Mb) * ml.y; }
      row_s[r] = make_float2(Mb, 1.f / L);
    }
    __syncthreads();
    if (key < limit) {
      const float* at = sc + ((size_t)kh * R_all + r0) * ld + key;
#pragma unroll 4
      for (int r = 0; r < rows; ++r) { const float2 ml = row_s[r]; sum = fmaf(sc_ex2(at[(size_t)r * ld] - ml.x), ml.y, sum); }
    }
  }
  if (key < limit) dst[key] += sum;
}

// Chunks: a wave or so of CTAs, from one round of keys to eight
void scored_plan(ScoredArgs& a, int sm_count) {
  const int G = a.Hq / a.Hkv;
  a.rt_own = (a.T * G + 15) / 16;
  a.rt_prefix = (a.n * a.T * G + 15) / 16;
  const long long own_keys = (long long)a.suffix_bound + a.T;
  const long long units = a.Hkv * (a.rt_prefix * (long long)a.P + (long long)a.n * a.rt_own * own_keys);
  long long chunk = units / (sm_count * 4) / SC_KEYS * SC_KEYS;
  chunk = chunk < SC_KEYS ? SC_KEYS : (chunk > 8 * SC_KEYS ? 8 * SC_KEYS : chunk);
  a.prefix_chunk = a.own_chunk = (int)chunk;
  a.n_prefix_chunks = (int)((a.P + chunk - 1) / chunk);
  a.n_own_chunks = (int)((own_keys + chunk - 1) / chunk);
  a.ld_prefix = (a.P + 15) / 16 * 16;
  a.ld_own = (int)((own_keys + 15) / 16 * 16);
}

static size_t sc_parts(const ScoredArgs& a) { return (size_t)a.n * a.T * a.Hq * (a.n_prefix_chunks + a.n_own_chunks); }
size_t scored_workspace_floats(const ScoredArgs& a) {
  return sc_parts(a) * (a.hd + 2) + (size_t)a.n * a.T * a.Hq * ((size_t)a.ld_prefix + a.ld_own);
}
void scored_carve(ScoredArgs& a, float* ws) {              // ws: 16-byte aligned
  a.part_o = ws;
  a.sc_prefix = a.part_o + sc_parts(a) * a.hd;
  a.sc_own = a.sc_prefix + (size_t)a.n * a.T * a.Hq * a.ld_prefix;
  a.part_ml = a.sc_own + (size_t)a.n * a.T * a.Hq * a.ld_own;
}

template <int HD>
static cudaError_t sc_launch(const ScoredArgs& a, cudaStream_t st) {
  const float scale_log2 = 1.4426950408889634f / sqrtf((float)HD);
  scored_rows_kernel<HD><<<dim3((unsigned)(a.n_prefix_chunks * a.rt_prefix + a.n * a.n_own_chunks * a.rt_own), (unsigned)a.Hkv), SC_WARPS * 32, 0, st>>>(a, scale_log2);
  cudaError_t e = cudaGetLastError();
  if (e != cudaSuccess) return e;
  const int out_blocks = (a.n * a.T * a.Hq + FIN_THREADS / 32 - 1) / (FIN_THREADS / 32);
  const int prefix_blocks = a.prefix_weight != nullptr ? (a.P + FIN_THREADS - 1) / FIN_THREADS : 0;
  const int own_blocks = (a.suffix_bound + a.T + FIN_THREADS - 1) / FIN_THREADS;
  scored_finish_kernel<HD><<<out_blocks + a.Hkv * prefix_blocks + a.n * a.Hkv * own_blocks, FIN_THREADS, 0, st>>>(a, out_blocks, prefix_blocks, own_blocks);
  return cudaGetLastError();
}

cudaError_t launch_attention_scored(const ScoredArgs& a, cudaStream_t st) { return a.hd == 64 ? sc_launch<64>(a, st) : sc_launch<128>(a, st); }

}  // namespace mlora
