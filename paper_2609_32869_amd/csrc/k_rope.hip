// Rotary positions of queries and keys.
//
// A pair (a, b) of a head at position p becomes A (a cos t - b sin t, b cos t + a sin t) with
// t = 2 pi p f.  Far positions need the angle's whole turns taken off exactly: p f in 64 bits
// and its fraction, then sine and cosine of at most an eighth of a turn as polynomials in 32.
#include <algorithm>

#include "wf_ops.h"

namespace wf {

// cos and sin of 2 pi x for x = p f in 64 bits, times `amp`: x = quarter / 4 + rest with |rest| <=
// 1/8, Taylor series of sine and cosine at 2 pi rest (last terms 2e-9 and 2e-9 at an eighth of a turn).
__device__ __forceinline__ float2 turn(double x, float amp) {
  x -= rint(x);
  const double quarter = rint(4.0 * x);
  const float t = (float)(x - 0.25 * quarter) * 6.28318530717958647693f, u = t * t;
  float s = 2.7557319e-6f, c = -2.7557319e-7f;
  s = fmaf(s, u, -1.98412698e-4f);
  c = fmaf(c, u, 2.48015873e-5f);
  s = fmaf(s, u, 8.33333333e-3f);
  c = fmaf(c, u, -1.38888889e-3f);
  s = fmaf(s, u, -0.166666667f);
  c = fmaf(c, u, 4.16666667e-2f);
  s = fmaf(t * u, s, t);
  c = fmaf(c, u, -0.5f);
  c = fmaf(c, u, 1.0f);
  const int q = (int)quarter;  // -2 .. 2
  const float co = q & 1 ? s : c, si = q & 1 ? c : s;
  // a quarter on: (cos, sin) -> (-sin, cos); two: (-cos, -sin); three: (sin, -cos)
  return make_float2(((q + 1) & 2 ? -co : co) * amp, (q & 2 ? -si : si) * amp);
}

// `N` consecutive elements of a row as fp32 and back.
template <int N>
__device__ __forceinline__ void ld(const float* p, float* o) {
  if constexpr (N == 4) {
    const float4 v = *reinterpret_cast<const float4*>(p);
    o[0] = v.x; o[1] = v.y; o[2] = v.z; o[3] = v.w;
  } else o[0] = p[0];
}
template <int N>
__device__ __forceinline__ void ld(const bf16* p, float* o) {
  if constexpr (N == 8) ld8(p, o);
  else o[0] = to_f(p[0]);
}
template <int N>
__device__ __forceinline__ void st(float* p, const float* v) {
  if constexpr (N == 4) *reinterpret_cast<float4*>(p) = make_float4(v[0], v[1], v[2], v[3]);
  else p[0] = v[0];
}
template <int N>
__device__ __forceinline__ void st(bf16* p, const float* v) {
  if constexpr (N == 8)
    *reinterpret_cast<uint4*>(p) = make_uint4(pack2_bf16(v[0], v[1]), pack2_bf16(v[2], v[3]), pack2_bf16(v[4], v[5]), pack2_bf16(v[6], v[7]));
  else p[0] = from_f<bf16>(v[0]);
}

// Block: `tb` tokens.  First their sines and cosines into LDS, then every (token, head, unit of N
// elements): a unit of halves is N elements and their partners, one of interleaved pairs N (one
// element: the pair) elements, the units behind `dims` are copied.
template <typename T, int N>
__global__ void __launch_bounds__(256) k_rotary(RotaryArgs a) {
  extern __shared__ float2 cs[];
  const int half = a.dims >> 1, t0 = (blockIdx.x + gridDim.x * blockIdx.z) * a.tb, nt = min(a.tb, a.tokens - t0);
  if (nt <= 0) return;
  for (int i = threadIdx.x; i < nt * half; i += 256) {
    const int t = i / half, j = i - t * half;
    float2 z = turn((double)a.positions[t0 + t] * a.turns[j], a.amplitude);
    if (a.transposed) z.y = -z.y;
    cs[i] = z;
  }
  __syncthreads();
  const int tu = N == 1 ? half : a.interleaved ? a.dims / N : half / N, units = tu + (a.copies ? (a.width - a.dims) / N : 0);
  const int heads = a.rows[0].heads + (a.n_rows > 1 ? a.rows[1].heads : 0), total = nt * heads * units;
  for (int i = blockIdx.y * 256 + threadIdx.x; i < total; i += gridDim.y * 256) {
    const int r = i / units, u = i - r * units, t = r / heads;
    int h = r - t * heads;
    const bool second = h >= a.rows[0].heads;
    const RotaryRows& w = a.rows[second];
    if (second) h -= a.rows[0].heads;
    const T* x = reinterpret_cast<const T*>(w.x) + (t0 + t) * w.xt + h * w.xh;
    T* y = reinterpret_cast<T*>(w.y) + (t0 + t) * w.yt + h * w.yh;
    const float2* z = cs + t * half;
    if (u >= tu) {
      const int at = a.dims + (u - tu) * N;
      float v[N];
      ld<N>(x + at, v);
      st<N>(y + at, v);
    } else if (!a.interleaved) {
      float p[N], q[N], o[N], s[N];
      ld<N>(x + u * N, p);
      ld<N>(x + half + u * N, q);
#pragma unroll
      for (int j = 0; j < N; ++j) {
        const float2 c = z[u * N + j];
        o[j] = fmaf(p[j], c.x, -(q[j] * c.y));
        s[j] = fmaf(q[j], c.x, p[j] * c.y);
      }
      st<N>(y + u * N, o);
      st<N>(y + half + u * N, s);
    } else if constexpr (N == 1) {
      float p, q;
      ld<1>(x + 2 * u, &p);
      ld<1>(x + 2 * u + 1, &q);
      const float2 c = z[u];
      const float o = fmaf(p, c.x, -(q * c.y)), s = fmaf(q, c.x, p * c.y);
      st<1>(y + 2 * u, &o);
      st<1>(y + 2 * u + 1, &s);
    } else {
      float p[N];
      ld<N>(x + u * N, p);
#pragma unroll
      for (int j = 0; j < N; j += 2) {
        const float2 c = z[(u * N + j) >> 1];
        const float o = fmaf(p[j], c.x, -(p[j + 1] * c.y));
        p[j + 1] = fmaf(p[j + 1], c.x, p[j] * c.y);
        p[j] = o;
      }
      st<N>(y + u * N, p);
    }
  }
}

void rotary(const RotaryArgs& a0, hipStream_t st) {
  RotaryArgs a = a0;
  const int half = a.dims / 2, heads = a.rows[0].heads + (a.n_rows > 1 ? a.rows[1].heads : 0);
  const int nv = a.bf16_data ? 8 : 4;
  const bool vec = a.vec && a.dims % (a.interleaved ? nv : 2 * nv) == 0 && (a.width - a.dims) % nv == 0;
  const int n = vec ? nv : 1;
  a.tb = (int)std::max<long long>(1, std::min<long long>(std::min(16, 1024 / half), (1 << 24) / ((long long)heads * a.width)));
  const long long items = (long long)a.tb * heads * (a.width / n);
  const int blocks = (a.tokens + a.tb - 1) / a.tb, bx = std::min(blocks, 1 << 20);  // a grid's x holds 2^32 threads
  const dim3 grid(bx, (unsigned)std::min<long long>(16, std::max<long long>(1, items / 2048)), (blocks + bx - 1) / bx);
  const size_t lds = (size_t)a.tb * half * sizeof(float2);
  if (a.bf16_data) {
    if (vec) k_rotary<bf16, 8><<<grid, 256, lds, st>>>(a);
    else k_rotary<bf16, 1><<<grid, 256, lds, st>>>(a);
  } else {
    if (vec) k_rotary<float, 4><<<grid, 256, lds, st>>>(a);
    else k_rotary<float, 1><<<grid, 256, lds, st>>>(a);
  }
}

}  // namespace wf
