// Rotary positions of a pass's rows and the append of its K/V rows (Sec. 3.1 attention block; the kernel-level counterpart of
// what the model passes do inside their attention kernels and projection epilogues).
//
// A pair (a, b) of a row at position p turns by the angle p * f:  a' = a c - b s,  b' = b c + a s,  c = gain cos, s = gain sin.
// Pairs are (i, i + rotary/2) or (2i, 2i + 1), i < rotary/2; features from `rotary` on pass through; v passes through.
// Angles: p * f / 2 pi in 64 bits, its fraction of a turn (exact) rounded to 32 bits, sincospi of twice that: good to 2^-22
// rad at any position (p = 10^6 in 32 bits would be off by 0.06 rad).
// Bound by bytes: every feature is read and written once, 16 bytes at a time.  A CTA first fills a table of its rows' cos and
// sin (one thread a pair, shared by all heads), the loads of its first features being on their way meanwhile.
#include "../../include/mlora.h"
#include "cache_ops.cuh"

namespace mlora {

constexpr int ROPE_THREADS = 256;
constexpr int ROPE_ROWS = 4;                               // rows of a CTA in large calls

// 8 features as loaded: fp16 (4 words) or fp32 (8 words)
template <bool F32> struct RopeVec;
template <> struct RopeVec<false> {
  uint4 u;
  __device__ __forceinline__ void load(const void* base, long long at) { u = __ldg(reinterpret_cast<const uint4*>(reinterpret_cast<const __half*>(base) + at)); }
  __device__ __forceinline__ void get(float (&f)[8]) const {
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) { const float2 x = __half22float2(u32_as_h2(w[i])); f[2 * i] = x.x; f[2 * i + 1] = x.y; }
  }
};
template <> struct RopeVec<true> {
  float4 a, b;
  __device__ __forceinline__ void load(const void* base, long long at) {
    const float4* p = reinterpret_cast<const float4*>(reinterpret_cast<const float*>(base) + at);
    a = __ldg(p); b = __ldg(p + 1);
  }
  __device__ __forceinline__ void get(float (&f)[8]) const {
    f[0] = a.x; f[1] = a.y; f[2] = a.z; f[3] = a.w; f[4] = b.x; f[5] = b.y; f[6] = b.z; f[7] = b.w;
  }
};

__device__ __forceinline__ uint4 rope_pack(const float (&f)[8]) {
  return make_uint4(h2_as_u32(__floats2half2_rn(f[0], f[1])), h2_as_u32(__floats2half2_rn(f[2], f[3])),
                    h2_as_u32(__floats2half2_rn(f[4], f[5])), h2_as_u32(__floats2half2_rn(f[6], f[7])));
}

// An item is 16 features of a head: two pieces of 8 that hold the two halves of 8 pairs (half-split), or 16 neighbours.
template <bool F32, int HD, int ROWS>
__global__ void __launch_bounds__(ROPE_THREADS) rope_append_kernel(const RopeArgs p) {
  constexpr int IH = HD / 16;                              // items of a head
  __shared__ float2 cs[ROWS][HD / 2];
  __shared__ int s_at[ROWS];                               // the row's place in its own segment, -1: none
  const int tid = threadIdx.x, rows = p.n * p.T, row0 = blockIdx.x * ROWS, half = p.rotary >> 1;
  const int H = p.Hq + 2 * p.Hkv;
  const int in_rows = min(ROWS, rows - row0);
  if (tid < in_rows && p.own_k != nullptr) {
    const int row = row0 + tid, s = row / p.T, t = row - s * p.T, S = p.suffix_len[s];
    const bool ok = S >= 0 && S <= p.cap - p.T;
    if (!ok) atomicCAS(p.status, 0, MLORA_ERR_CAPACITY);
    s_at[tid] = ok ? S + t : -1;
  }
  for (int i = tid; i < in_rows * half; i += ROPE_THREADS) {
    const int r = i / half, j = i - r * half;
    const double turns = (double)p.positions[row0 + r] * p.freq[j] * 0.15915494309189533577;
    const float x = (float)(2.0 * (turns - rint(turns)));
    float sn, cn;
    sincospif(x, &sn, &cn);
    cs[r][j] = make_float2(cn * p.gain, sn * p.gain);
  }
  __syncthreads();
  for (int i = tid; i < in_rows * H * IH; i += ROPE_THREADS) {
    const int it = i % IH, u = i / IH, r = u / H, h = u - r * H, row = row0 + r;
    const bool is_q = h < p.Hq, is_v = h >= p.Hq + p.Hkv;
    if (is_q ? p.q_out == nullptr : (p.own_k == nullptr || s_at[r] < 0)) continue;
    const void* src = is_q ? p.q : (is_v ? p.v : p.k);
    const int hh = is_q ? h : (is_v ? h - p.Hq - p.Hkv : h - p.Hq);
    const long long from = row * (is_q ? p.q_stride : (is_v ? p.v_stride : p.k_stride)) + hh * HD;
    // offsets of the two pieces
    const bool turn = !is_v && it * 16 < p.rotary;
    const bool split = turn && !p.interleaved;
    const int o0 = split ? it * 8 : it * 16, o1 = split ? it * 8 + half : it * 16 + 8;
    RopeVec<F32> va, vb;
    va.load(src, from + o0); vb.load(src, from + o1);
    float a[8], b[8];
    va.get(a); vb.get(b);
    if (split) {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float2 c = cs[r][it * 8 + e];
        const float x = a[e], y = b[e];
        a[e] = x * c.x - y * c.y; b[e] = y * c.x + x * c.y;
      }
    } else if (turn) {
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float2 c = cs[r][it * 8 + e], d = cs[r][it * 8 + 4 + e];
        float x = a[2 * e], y = a[2 * e + 1];
        a[2 * e] = x * c.x - y * c.y; a[2 * e + 1] = y * c.x + x * c.y;
        x = b[2 * e]; y = b[2 * e + 1];
        b[2 * e] = x * d.x - y * d.y; b[2 * e + 1] = y * d.x + x * d.y;
      }
    }
    __half* dst;
    if (is_q) dst = p.q_out + ((size_t)row * p.Hq + hh) * HD;
    else {
      const size_t seg = (size_t)(row / p.T) * p.Hkv + hh;
      dst = (is_v ? p.own_v : p.own_k) + (seg * p.cap + s_at[r]) * HD;
      if (is_v && it == 0) {
        if (p.own_weight != nullptr) p.own_weight[seg * p.cap + s_at[r]] = 0.f;
        if (p.own_position != nullptr) p.own_position[seg * p.cap + s_at[r]] = p.positions[row];
      }
    }
    *reinterpret_cast<uint4*>(dst + o0) = rope_pack(a);
    *reinterpret_cast<uint4*>(dst + o1) = rope_pack(b);
  }
}

template <bool F32, int HD>
static cudaError_t rope_launch(const RopeArgs& a, cudaStream_t st) {
  const int rows = a.n * a.T;
  if (rows < 148 * 8) rope_append_kernel<F32, HD, 1><<<rows, ROPE_THREADS, 0, st>>>(a);
  else rope_append_kernel<F32, HD, ROPE_ROWS><<<(rows + ROPE_ROWS - 1) / ROPE_ROWS, ROPE_THREADS, 0, st>>>(a);
  return cudaGetLastError();
}

cudaError_t launch_rope_append(const RopeArgs& a, cudaStream_t st) {
  if (a.hd == 64) return a.in_fp32 ? rope_launch<true, 64>(a, st) : rope_launch<false, 64>(a, st);
  return a.in_fp32 ? rope_launch<true, 128>(a, st) : rope_launch<false, 128>(a, st);
}

}  // namespace mlora
