// Rotary positions of a pass's rows and the append of its K/V rows (Sec. 3.1 attention block; the kernel-level counterpart of
// what the model passes do inside their attention kernels and projection epilogues).
//
// A pair (a, b) of a row at position p turns by the angle p * f:  a' = a c - b s,  b' = b c + a s,  c = gain cos, s = gain sin.
// Pairs are (i, i + rotary/2) or (2i, 2i + 1), i < rotary/2; features from `rotary` on pass through; v passes through.
// Angles: p * f / 2 pi in 64 bits with the products' rounding errors carried along, its fraction of a turn rounded to 32 bits, sincospi
// of twice that: good to 2^-22 rad at any 32-bit position and frequencies up to 2^16 (p = 10^6 in 32 bits would be off by 0.06 rad; 64 bits
// without the errors by 2^-21 at 2^31).
// Bound by bytes: every feature is read and written once, 16 bytes at a time (81% of the copy rate for 16384 fp16 rows, 76% for 5003
// fp32 rows; in a graph 88% and 81%).  A CTA first fills a table of its rows' cos and sin (one thread a pair, shared by all heads), the loads
// of its first features being on their way meanwhile.  fp16: 64 registers, so that four CTAs share an SM (16384 rows with 100 registers and
// twice the reads in flight: 41 us); fp32: 76 to 80, three CTAs.
#include "../../include/mlora.h"
#include "cache_ops.cuh"

namespace mlora {

constexpr int ROPE_THREADS = 256;

// 8 features as loaded: fp16 (4 words) or fp32 (8 words)
template <bool F32> struct RopeVec;
template <> struct RopeVec<false> {
  uint4 u;
  __device__ __forceinline__ void load(const unsigned char* row, int at) { u = *reinterpret_cast<const uint4*>(row + at * 2); }
  __device__ __forceinline__ void get(float (&f)[8]) const {
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) { const float2 x = __half22float2(u32_as_h2(w[i])); f[2 * i] = x.x; f[2 * i + 1] = x.y; }
  }
};
template <> struct RopeVec<true> {
  float4 a, b;
  __device__ __forceinline__ void load(const unsigned char* row, int at) {
    const float4* p = reinterpret_cast<const float4*>(row + at * 4);
    a = p[0]; b = p[1];
  }
  __device__ __forceinline__ void get(float (&f)[8]) const {
    f[0] = a.x; f[1] = a.y; f[2] = a.z; f[3] = a.w; f[4] = b.x; f[5] = b.y; f[6] = b.z; f[7] = b.w;
  }
};

__device__ __forceinline__ uint4 rope_pack(const float (&f)[8]) {
  return make_uint4(h2_as_u32(__floats2half2_rn(f[0], f[1])), h2_as_u32(__floats2half2_rn(f[2], f[3])),
                    h2_as_u32(__floats2half2_rn(f[4], f[5])), h2_as_u32(__floats2half2_rn(f[6], f[7])));
}

// The angle p f as half turns in [-1, 1]: 1 / 2 pi as a sum of two doubles, the errors of both products by fma
__device__ __forceinline__ float rope_half_turns(double p, double f) {
  constexpr double INV = 0.15915494309189533577, INV_REST = -9.8393383375912429e-18;
  const double a = p * f, a_rest = fma(p, f, -a), t = a * INV;
  const double rest = fma(a_rest, INV, fma(a, INV_REST, fma(a, INV, -t)));
  return (float)(2.0 * ((t - rint(t)) + rest));
}

// An item is 16 features of a head: two pieces of 8 that hold the two halves of 8 pairs (half-split), or 16 neighbours.  Which 16 is
// fixed for a thread; it goes through the CTA's (row, head) in steps of ROPE_THREADS / items-of-a-head, without divisions, FLY items' reads
// on their way at a time, the first before the table is filled.  Addresses of several rows come from shared memory.
template <bool F32, int HD, int ROWS, int FLY>
__global__ void __launch_bounds__(ROPE_THREADS) rope_append_kernel(const RopeArgs p) {
  constexpr int IH = HD / 16, STEP = ROPE_THREADS / IH, SIZE = F32 ? 4 : 2;
  __shared__ __align__(16) float2 cs[ROWS][HD / 2];
  __shared__ const unsigned char* s_src[ROWS][3];          // the row's q, k, v
  __shared__ __half* s_dst[ROWS][3];                       // where they go: head 0 of q_out's row, of its place in the own segments; null: nowhere
  const int tid = threadIdx.x, rows = p.n * p.T, row0 = blockIdx.x * ROWS, half = p.rotary >> 1;
  const int H = p.Hq + 2 * p.Hkv, in_rows = min(ROWS, rows - row0);
  auto row_of = [&](int x, int what) {
    const long long stride = what == 0 ? p.q_stride : (what == 1 ? p.k_stride : p.v_stride);
    const void* base = what == 0 ? p.q : (what == 1 ? p.k : p.v);
    return reinterpret_cast<const unsigned char*>(base) + (row0 + x) * stride * SIZE;
  };
  if constexpr (ROWS > 1)
    for (int i = tid; i < in_rows * 3; i += ROPE_THREADS) s_src[i / 3][i % 3] = row_of(i / 3, i % 3);
  const int it = tid % IH;
  const bool in_turn = it * 16 < p.rotary, split = in_turn && !p.interleaved;
  const int o0 = split ? it * 8 : it * 16, o1 = split ? o0 + half : o0 + 8;      // offsets of the two pieces (v: split is undone below)
  const int v0 = it * 16;
  // (r, h): the item's row and head, h counted through q, k, v
  const int dr = STEP / H, dh = STEP - dr * H;
  int r = (tid / IH) / H, h = tid / IH - r * H;
  auto advance = [&](int& r, int& h) {
    r += dr; h += dh;
    if (h >= H) { h -= H; ++r; }
  };
  RopeVec<F32> va[FLY], vb[FLY];
  int fr[FLY], fh[FLY];
  auto fetch = [&] {
#pragma unroll
    for (int f = 0; f < FLY; ++f) {
      fr[f] = r; fh[f] = h;
      if (r < in_rows) {
        const int what = (h >= p.Hq) + (h >= p.Hq + p.Hkv), hh = h - (what == 0 ? 0 : (what == 1 ? p.Hq : p.Hq + p.Hkv));
        const unsigned char* src = ROWS == 1 ? row_of(0, what) : s_src[r][what];
        va[f].load(src, hh * HD + (what == 2 ? v0 : o0)); vb[f].load(src, hh * HD + (what == 2 ? v0 + 8 : o1));
      }
      advance(r, h);
    }
  };
  if constexpr (ROWS > 1) __syncthreads();
  fetch();
  for (int i = ROPE_THREADS - 1 - tid; i < in_rows * 3; i += ROPE_THREADS) {
    const int x = i / 3, what = i - x * 3, row = row0 + x;
    __half* dst = nullptr;
    if (what == 0) {
      if (p.q_out != nullptr) dst = p.q_out + (size_t)row * p.Hq * HD;
    } else if (p.own_k != nullptr) {
      const int s = row / p.T, S = p.suffix_len[s];
      if (S >= 0 && S <= p.cap - p.T) dst = (what == 1 ? p.own_k : p.own_v) + ((size_t)s * p.Hkv * p.cap + S + (row - s * p.T)) * HD;
      else atomicCAS(p.status, 0, MLORA_ERR_CAPACITY);
    }
    s_dst[x][what] = dst;
  }
  for (int i = tid; i < in_rows * half; i += ROPE_THREADS) {
    const int x = ROWS == 1 ? 0 : i / half, j = i - x * half;
    const float t = rope_half_turns((double)p.positions[row0 + x], p.freq[j]);
    float sn, cn;
    sincospif(t, &sn, &cn);
    cs[x][j] = make_float2(cn * p.gain, sn * p.gain);
  }
  __syncthreads();
  // a total of 0 and the position of every appended row and KV head, rows side by side
  if (p.own_weight != nullptr || p.own_position != nullptr)
    for (int i = tid; i < p.Hkv * ROWS; i += ROPE_THREADS) {
      const int x = i % ROWS;
      if (x >= in_rows || s_dst[x][1] == nullptr) continue;
      const size_t at = (size_t)(s_dst[x][1] - p.own_k) / HD + (size_t)(i / ROWS) * p.cap;
      if (p.own_weight != nullptr) p.own_weight[at] = 0.f;
      if (p.own_position != nullptr) p.own_position[at] = p.positions[row0 + x];
    }
  while (true) {
#pragma unroll
    for (int f = 0; f < FLY; ++f) {
      if (fr[f] >= in_rows) break;
      const int what = (fh[f] >= p.Hq) + (fh[f] >= p.Hq + p.Hkv), hh = fh[f] - (what == 0 ? 0 : (what == 1 ? p.Hq : p.Hq + p.Hkv));
      __half* dst = s_dst[fr[f]][what];
      if (dst == nullptr) continue;
      dst += (size_t)hh * (what == 0 ? HD : p.cap * (long long)HD);
      float a[8], b[8];
      va[f].get(a); vb[f].get(b);
      if (what == 2) {
        *reinterpret_cast<uint4*>(dst + v0) = rope_pack(a);
        *reinterpret_cast<uint4*>(dst + v0 + 8) = rope_pack(b);
        continue;
      }
      if (in_turn) {
        float2 c[8];
#pragma unroll
        for (int e = 0; e < 8; e += 2) {
          const float4 x = *reinterpret_cast<const float4*>(&cs[fr[f]][it * 8 + e]);
          c[e] = make_float2(x.x, x.y); c[e + 1] = make_float2(x.z, x.w);
        }
        if (split) {
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const float x = a[e], y = b[e];
            a[e] = x * c[e].x - y * c[e].y; b[e] = y * c[e].x + x * c[e].y;
          }
        } else {
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            float x = a[2 * e], y = a[2 * e + 1];
            a[2 * e] = x * c[e].x - y * c[e].y; a[2 * e + 1] = y * c[e].x + x * c[e].y;
            x = b[2 * e]; y = b[2 * e + 1];
            b[2 * e] = x * c[4 + e].x - y * c[4 + e].y; b[2 * e + 1] = y * c[4 + e].x + x * c[4 + e].y;
          }
        }
      }
      *reinterpret_cast<uint4*>(dst + o0) = rope_pack(a);
      *reinterpret_cast<uint4*>(dst + o1) = rope_pack(b);
    }
    if (r >= in_rows) break;
    fetch();
  }
}

template <bool F32, int HD>
static cudaError_t rope_launch(const RopeArgs& a, cudaStream_t st) {
  const int rows = a.n * a.T;
  // Few rows: a CTA each.  Many: as many as make a sector of totals (8 rows of fp16: 16384 rows of 48 heads of 64 in 37.2 us, 4 rows
  // 39.8; 38.4 since angles carry their rounding errors), or of the same bytes (4 rows of fp32: 5003 rows of 40 heads of 128 in 30.9 us, 8 rows 33.3).
  constexpr int ROWS = F32 ? 4 : 8;
  if (rows < 148 * 8) rope_append_kernel<F32, HD, 1, 2><<<rows, ROPE_THREADS, 0, st>>>(a);
  else rope_append_kernel<F32, HD, ROWS, 2><<<(rows + ROWS - 1) / ROWS, ROPE_THREADS, 0, st>>>(a);
  return cudaGetLastError();
}

cudaError_t launch_rope_append(const RopeArgs& a, cudaStream_t st) {
  if (a.hd == 64) return a.in_fp32 ? rope_launch<true, 64>(a, st) : rope_launch<false, 64>(a, st);
  return a.in_fp32 ? rope_launch<true, 128>(a, st) : rope_launch<false, 128>(a, st);
}

}  // namespace mlora
