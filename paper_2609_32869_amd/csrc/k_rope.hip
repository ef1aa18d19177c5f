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

// N consecutive elements of a row as they lie in memory, and their values.
template <typename T, int N>
struct Raw;
template <>
struct Raw<float, 4> {
  float4 v;
  __device__ __forceinline__ void get(float* o) const { o[0] = v.x; o[1] = v.y; o[2] = v.z; o[3] = v.w; }
  __device__ __forceinline__ void set(const float* o) { v = make_float4(o[0], o[1], o[2], o[3]); }
};
template <>
struct Raw<float, 2> {
  float2 v;
  __device__ __forceinline__ void get(float* o) const { o[0] = v.x; o[1] = v.y; }
  __device__ __forceinline__ void set(const float* o) { v = make_float2(o[0], o[1]); }
};
template <>
struct Raw<bf16, 4> {
  uint2 v;
  __device__ __forceinline__ void get(float* o) const {
    o[0] = __uint_as_float(v.x << 16);
    o[1] = __uint_as_float(v.x & 0xffff0000u);
    o[2] = __uint_as_float(v.y << 16);
    o[3] = __uint_as_float(v.y & 0xffff0000u);
  }
  __device__ __forceinline__ void set(const float* o) { v = make_uint2(pack2_bf16(o[0], o[1]), pack2_bf16(o[2], o[3])); }
};
template <>
struct Raw<bf16, 2> {
  uint32_t v;
  __device__ __forceinline__ void get(float* o) const {
    o[0] = __uint_as_float(v << 16);
    o[1] = __uint_as_float(v & 0xffff0000u);
  }
  __device__ __forceinline__ void set(const float* o) { v = pack2_bf16(o[0], o[1]); }
};
template <>
struct Raw<float, 1> {
  float v;
  __device__ __forceinline__ void get(float* o) const { o[0] = v; }
  __device__ __forceinline__ void set(const float* o) { v = o[0]; }
};
template <>
struct Raw<bf16, 8> {
  uint4 v;
  __device__ __forceinline__ void get(float* o) const {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      o[2 * j] = __uint_as_float(w[j] << 16);
      o[2 * j + 1] = __uint_as_float(w[j] & 0xffff0000u);
    }
  }
  __device__ __forceinline__ void set(const float* o) {
    v = make_uint4(pack2_bf16(o[0], o[1]), pack2_bf16(o[2], o[3]), pack2_bf16(o[4], o[5]), pack2_bf16(o[6], o[7]));
  }
};
template <>
struct Raw<bf16, 1> {
  bf16 v;
  __device__ __forceinline__ void get(float* o) const { o[0] = to_f(v); }
  __device__ __forceinline__ void set(const float* o) { v = from_f<bf16>(o[0]); }
};

// Units of N elements of a head: of halves N elements and their partners each, of interleaved pairs N elements (N = 1: a pair),
// of which the last may reach past `dims`; the units behind are copied.
struct Units {
  int turning, copied, from;  // copied ones start at element `from`
};
template <int N>
__host__ __device__ __forceinline__ Units units_of(const RotaryArgs& a) {
  const int half = a.dims / 2, turning = N == 1 ? half : a.interleaved ? (a.dims + N - 1) / N : half / N;
  const int from = a.interleaved && N > 1 ? turning * N : a.dims;
  return Units{turning, a.copies ? (a.width - from) / N : 0, from};
}
// Block: `tb` tokens.  Their sines and cosines into LDS, then every (token, head, unit).  A thread takes I units at a time, all
// loaded before the first is used, the first I before the sines are formed.
template <typename T, int N, int I>
__global__ void __launch_bounds__(256) k_rotary(RotaryArgs a) {
  extern __shared__ float2 cs[];
  typedef Raw<T, N> R;
  const int half = a.dims >> 1, t0 = (blockIdx.x + gridDim.x * blockIdx.z) * a.tb, nt = min(a.tb, a.tokens - t0);
  if (nt <= 0) return;
  const Units of = units_of<N>(a);
  const int tu = of.turning, units = tu + of.copied;
  const int heads = a.rows[0].heads + (a.n_rows > 1 ? a.rows[1].heads : 0), total = nt * heads * units;
  // quotients of numbers below 2^22 as products: (i + 1/2) / n is 1 / (2 n) off a whole number at least, more than its two
  // roundings, 2^-23 of it; larger ones by division
  const float iu = 1.f / units, ih = 1.f / heads;
  const bool small = total <= 1 << 22;
  R p[I], q[I];
  T* y[I];
  int at[I], z[I];  // first element, its partner's distance is `apart`; index of its sine, -1: a copy, -2: nothing
  const int apart = a.interleaved ? (N == 1 ? 1 : 0) : half;
  auto load = [&](int first) {
#pragma unroll
    for (int k = 0; k < I; ++k) {
      const int i = first + k * 256;
      z[k] = -2;
      if (i >= total) continue;
      const int r = small ? (int)((i + 0.5f) * iu) : i / units, u = i - r * units, t = small ? (int)((r + 0.5f) * ih) : r / heads;
      int h = r - t * heads;
      const bool second = h >= a.rows[0].heads;
      if (second) h -= a.rows[0].heads;
      const long long xt = second ? a.rows[1].xt : a.rows[0].xt, xh = second ? a.rows[1].xh : a.rows[0].xh;
      const long long yt = second ? a.rows[1].yt : a.rows[0].yt, yh = second ? a.rows[1].yh : a.rows[0].yh;
      const T* x = reinterpret_cast<const T*>(second ? a.rows[1].x : a.rows[0].x) + (t0 + t) * xt + h * xh;
      y[k] = reinterpret_cast<T*>(second ? a.rows[1].y : a.rows[0].y) + (t0 + t) * yt + h * yh;
      const bool turns = u < tu;
      at[k] = !turns ? of.from + (u - tu) * N : a.interleaved && N == 1 ? 2 * u : u * N;
      z[k] = !turns ? -1 : t * half + (a.interleaved && N > 1 ? u * N / 2 : u * N);
      p[k] = *reinterpret_cast<const R*>(x + at[k]);
      if (apart) q[k] = *reinterpret_cast<const R*>(x + (turns ? at[k] + apart : at[k]));
    }
  };
  int first = blockIdx.y * 256 * I + threadIdx.x;
  load(first);
  for (int i = threadIdx.x; i < nt * half; i += 256) {
    const int t = i / half, j = i - t * half;
    float2 c = turn((double)a.positions[t0 + t] * a.turns[j], a.amplitude);
    if (a.transposed) c.y = -c.y;
    cs[i] = c;
  }
  __syncthreads();
  for (;;) {
#pragma unroll
    for (int k = 0; k < I; ++k) {
      if (z[k] == -2) continue;
      R* o = reinterpret_cast<R*>(y[k] + at[k]);
      if (z[k] < 0) {
        *o = p[k];
        continue;
      }
      const float2* c = cs + z[k];
      float u[N], v[N];
      p[k].get(u);
      if (apart) {
        float s[N], w[N];
        q[k].get(v);
#pragma unroll
        for (int j = 0; j < N; ++j) {
          s[j] = fmaf(u[j], c[j].x, -(v[j] * c[j].y));
          w[j] = fmaf(v[j], c[j].x, u[j] * c[j].y);
        }
        p[k].set(s);
        q[k].set(w);
        *o = p[k];
        *reinterpret_cast<R*>(y[k] + at[k] + apart) = q[k];
      } else if constexpr (N > 1) {
#pragma unroll
        for (int j = 0; j < N; j += 2) {
          if (at[k] + j >= a.dims) break;
          const float2 d = c[j >> 1];
          const float s = fmaf(u[j], d.x, -(u[j + 1] * d.y));
          u[j + 1] = fmaf(u[j + 1], d.x, u[j] * d.y);
          u[j] = s;
        }
        p[k].set(u);
        *o = p[k];
      }
    }
    first += gridDim.y * 256 * I;
    if (first - (int)threadIdx.x >= total) break;
    load(first);
  }
}

template <typename T, int N>
static void rotary_launch(RotaryArgs& a, hipStream_t st) {
  const int half = a.dims / 2, heads = a.rows[0].heads + (a.n_rows > 1 ? a.rows[1].heads : 0);
  const Units of = units_of<N>(a);
  const int units = of.turning + of.copied;
  // Tokens of a block: units for every thread, more where there are blocks enough to fill the chip with them; sines
  // within LDS; at most 2^24 units
  const long long each = (long long)heads * units, all = each * a.tokens;
  const long long want = all > 256ll * 256 * 16 ? 2048 : 256;
  a.tb = (int)std::max<long long>(1, std::min<long long>({(want + each - 1) / each, 2048 / half, (1 << 24) / each, 64}));
  const int blocks = (a.tokens + a.tb - 1) / a.tb, bx = std::min(blocks, 1 << 20);  // a grid's x holds 2^32 threads
  const unsigned by = (unsigned)std::min<long long>(1024, (a.tb * each + 2047) / 2048);
  const dim3 grid(bx, by, (blocks + bx - 1) / bx);
  const size_t lds = (size_t)a.tb * half * sizeof(float2);
  if (want > 256) k_rotary<T, N, 4><<<grid, 256, lds, st>>>(a);
  else k_rotary<T, N, 1><<<grid, 256, lds, st>>>(a);
}
// The widest units that the parts of a head hold whole and that all rows are aligned to.
void rotary(const RotaryArgs& a0, hipStream_t st) {
  RotaryArgs a = a0;
  auto fits = [&](int n) {
    if (a.align < n * (a.bf16_data ? 2 : 4)) return false;
    return a.interleaved ? a.width % n == 0 : a.dims % (2 * n) == 0 && (a.width - a.dims) % n == 0;
  };
  if (a.bf16_data) {
    if (fits(8)) rotary_launch<bf16, 8>(a, st);
    else if (fits(4)) rotary_launch<bf16, 4>(a, st);
    else if (fits(2)) rotary_launch<bf16, 2>(a, st);
    else rotary_launch<bf16, 1>(a, st);
  } else {
    if (fits(4)) rotary_launch<float, 4>(a, st);
    else if (fits(2)) rotary_launch<float, 2>(a, st);
    else rotary_launch<float, 1>(a, st);
  }
}

}  // namespace wf
