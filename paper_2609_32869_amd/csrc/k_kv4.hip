// Acoustic keys and values in 4 bits, and attention over them.
//
// Elements are e2m1 (0, 0.5, 1, 1.5, 2, 3, 4, 6 and their negatives) in blocks of 32 that
// share a power-of-two scale; a block lies along the axis that its product sums over
// (keys: 32 of a frame's 64 dims; values: 32 frames of one dim), so the eight elements
// that a lane gives a matrix instruction have one scale and one instruction turns two
// codes and the scale into two bf16 values, exactly.
#include "wf_operand.h"
#include "wf_ops.h"

namespace wf {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

// Smallest 2^e, e >= -120, with amax <= 6 * 2^e, as a biased exponent: amax = m 2^x with
// 1 <= m < 2 is <= 6 * 2^e = 1.5 * 2^(e + 2) for e = x - 2 where m <= 1.5, else x - 1.
// 0xff where amax is not finite.
__device__ __forceinline__ uint32_t scale_of(float amax) {
  const uint32_t u = __float_as_uint(amax);
  const int e = (int)(u >> 23) - ((u & 0x7fffffu) <= 0x400000u ? 2 : 1);
  return (u >> 23) == 255u ? 255u : (uint32_t)max(e, 7);
}

// 8 values -> 8 codes, element i in nibble i.
__device__ __forceinline__ uint32_t codes8(const float* x, float s) {
  uint32_t r = 0;
  r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, x[0], x[1], s, 0);
  r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, x[2], x[3], s, 1);
  r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, x[4], x[5], s, 2);
  return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, x[6], x[7], s, 3);
}

// 8 codes -> the 8 bf16 values they stand for.
__device__ __forceinline__ bf16x8 values8(uint32_t c, float s) {
  const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, s, 0);
  const bf16x2 b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, s, 1);
  const bf16x2 d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, s, 2);
  const bf16x2 e = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, s, 3);
  return bf16x8{a[0], a[1], b[0], b[1], d[0], d[1], e[0], e[1]};
}

// max |x| that keeps a NaN (fmaxf would drop it): |x| as integers, NaN above infinity
__device__ __forceinline__ uint32_t umax(uint32_t a, uint32_t b) { return a > b ? a : b; }
__device__ __forceinline__ uint32_t mag(float x) { return __float_as_uint(x) & 0x7fffffffu; }
__device__ __forceinline__ float scale_f(uint32_t byte) { return __uint_as_float(byte << 23); }

// ---------------------------------------------------------------- store
// A wave per (entry, head, 32-frame group); frames at or beyond the request's length are
// not read and stand for zero.
template <typename T>
__global__ void __launch_bounds__(256) k_kv4_store(Kv4StoreArgs a) {
  const int lane = threadIdx.x & 63, n = lane & 15, kg = lane >> 4;
  const int g = blockIdx.x * 4 + (threadIdx.x >> 6), head = blockIdx.y, r = blockIdx.z;
  if (g >= a.c.groups) return;
  const int len = a.lens ? min(max(a.lens[r], 0), a.c.frames) : a.c.frames;
  uint8_t* out = a.c.base + (((size_t)(a.slot0 + r) * a.c.n_head + head) * a.c.groups + g) * kKv4Group;
  const T* K = reinterpret_cast<const T*>(a.k) + r * a.kr + head * a.kh;
  const T* V = reinterpret_cast<const T*>(a.v) + r * a.vr + head * a.vh;
#pragma unroll
  for (int t = 0; t < 2; ++t) {
    const int f = g * 32 + 16 * t + n;
    float x[16];
    uint32_t m = 0;
#pragma unroll
    for (int j = 0; j < 16; ++j) {
      x[j] = f < len ? to_f(K[(long long)f * a.kf + 16 * kg + j]) : 0.f;
      m = umax(m, mag(x[j]));
    }
    m = umax(m, (uint32_t)__shfl_xor((int)m, 16));
    const uint32_t sb = scale_of(__uint_as_float(m));
    const float s = scale_f(sb);
    uint2 c = make_uint2(codes8(x, s), codes8(x + 8, s));
    *reinterpret_cast<uint2*>(out + 16 * lane + 8 * t) = c;
    if ((kg & 1) == 0) out[kKv4KeyScale + 32 * (kg >> 1) + 2 * n + t] = (uint8_t)sb;
  }
#pragma unroll
  for (int dt = 0; dt < 4; ++dt) {
    float x[8];
    uint32_t m = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int f = g * 32 + 8 * kg + j;
      x[j] = f < len ? to_f(V[(long long)f * a.vf + 16 * dt + n]) : 0.f;
      m = umax(m, mag(x[j]));
    }
    m = umax(m, (uint32_t)__shfl_xor((int)m, 16));
    m = umax(m, (uint32_t)__shfl_xor((int)m, 32));
    const uint32_t sb = scale_of(__uint_as_float(m));
    *reinterpret_cast<uint32_t*>(out + kKv4Values + 16 * lane + 4 * dt) = codes8(x, scale_f(sb));
    if (kg == 0) out[kKv4ValueScale + 4 * n + dt] = (uint8_t)sb;
  }
}

void kv4_store(const Kv4StoreArgs& a, hipStream_t st) {
  const dim3 grid((a.c.groups + 3) / 4, a.c.n_head, a.n);
  if (a.bf16_src) k_kv4_store<bf16><<<grid, 256, 0, st>>>(a);
  else k_kv4_store<float><<<grid, 256, 0, st>>>(a);
}

// ---------------------------------------------------------------- load
template <typename T>
__global__ void __launch_bounds__(256) k_kv4_load(Kv4LoadArgs a) {
  const int lane = threadIdx.x & 63, n = lane & 15, kg = lane >> 4;
  const int g = blockIdx.x * 4 + (threadIdx.x >> 6), head = blockIdx.y, r = blockIdx.z;
  if (g >= a.c.groups) return;
  const uint8_t* in = a.c.base + (((size_t)(a.slot0 + r) * a.c.n_head + head) * a.c.groups + g) * kKv4Group;
  T* K = reinterpret_cast<T*>(a.k);
  T* V = reinterpret_cast<T*>(a.v);
  auto at = [&](int f, int d) { return (((size_t)r * a.c.frames + f) * a.c.n_head + head) * kHeadDim + d; };
#pragma unroll
  for (int t = 0; t < 2; ++t) {
    const int f = g * 32 + 16 * t + n;
    const float s = scale_f(in[kKv4KeyScale + 32 * (kg >> 1) + 2 * n + t]);
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const bf16x8 x = values8(*reinterpret_cast<const uint32_t*>(in + 16 * lane + 8 * t + 4 * h), s);
      if (f < a.c.frames)
#pragma unroll
        for (int j = 0; j < 8; ++j) K[at(f, 16 * kg + 8 * h + j)] = from_f<T>((float)x[j]);
    }
  }
#pragma unroll
  for (int dt = 0; dt < 4; ++dt) {
    const bf16x8 x = values8(*reinterpret_cast<const uint32_t*>(in + kKv4Values + 16 * lane + 4 * dt),
                             scale_f(in[kKv4ValueScale + 4 * n + dt]));
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int f = g * 32 + 8 * kg + j;
      if (f < a.c.frames) V[at(f, 16 * dt + n)] = from_f<T>((float)x[j]);
    }
  }
}

void kv4_load(const Kv4LoadArgs& a, hipStream_t st) {
  const dim3 grid((a.c.groups + 3) / 4, a.c.n_head, a.n);
  if (a.bf16_out) k_kv4_load<bf16><<<grid, 256, 0, st>>>(a);
  else k_kv4_load<float><<<grid, 256, 0, st>>>(a);
}

// ---------------------------------------------------------------- attention
// Block (head, request, 16 query rows), four waves; a wave takes every fourth group.
// bf16 terms of a query value (fp32: exact) and of a probability (fp32 output: exact;
// bf16 output: 2^-16 relative, against the output's own 2^-9).
template <typename T>
struct Terms {
  static constexpr int q = sizeof(T) == 4 ? 3 : 1, p = sizeof(T) == 4 ? 3 : 2;
};
// Eight values as N bf16 terms.
template <int N>
__device__ __forceinline__ void split_terms(const float* v, bf16x8 (&t)[N]) {
  uint4 u[3];
  if constexpr (N == 3) split3x8(v, u[0], u[1], u[2]);
  else if constexpr (N == 2) split2x8(v, u[0], u[1]);
  else u[0] = make_uint4(pack2_bf16(v[0], v[1]), pack2_bf16(v[2], v[3]), pack2_bf16(v[4], v[5]), pack2_bf16(v[6], v[7]));
#pragma unroll
  for (int i = 0; i < N; ++i) t[i] = __builtin_bit_cast(bf16x8, u[i]);
}
template <int N>
__device__ __forceinline__ floatx4 mfma_terms(bf16x8 x, const bf16x8 (&t)[N], floatx4 acc) {
#pragma unroll
  for (int i = 0; i < N; ++i) acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x, t[i], acc, 0, 0, 0);
  return acc;
}

template <typename T>
__global__ void __launch_bounds__(256) k_kv4_attend(Kv4AttendArgs a) {
  constexpr int QT = Terms<T>::q, PT = Terms<T>::p;
  __shared__ float wm[4][16], wl[4][16], wo[4][16][68];
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, n = lane & 15, kg = lane >> 4;
  const int head = blockIdx.x, r = blockIdx.y, row = blockIdx.z * 16 + n;
  const int len = a.lens ? min(max(a.lens[r], 0), a.c.frames) : a.c.frames;
  const uint8_t* in = a.c.base + ((size_t)(a.slot0 + r) * a.c.n_head + head) * a.c.groups * kKv4Group;
  bf16x8 qt[2][QT];
  {
    const T* q = reinterpret_cast<const T*>(a.q) + r * a.sr + (long long)min(row, a.rows - 1) * a.si + head * a.sh + 16 * kg;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      float x[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) x[j] = row < a.rows ? 0.125f * to_f(q[8 * h + j]) : 0.f;
      split_terms<QT>(x, qt[h]);
    }
  }
  float m = -INFINITY, l = 0.f;
  floatx4 o[4];
#pragma unroll
  for (int dt = 0; dt < 4; ++dt) o[dt] = floatx4{0.f, 0.f, 0.f, 0.f};
  for (int g = w; g * 32 < len; g += 4) {
    const uint8_t* p = in + (size_t)g * kKv4Group;
    const uint4 kc = *reinterpret_cast<const uint4*>(p + 16 * lane), vc = *reinterpret_cast<const uint4*>(p + kKv4Values + 16 * lane);
    const uint32_t ks = *reinterpret_cast<const uint16_t*>(p + kKv4KeyScale + 32 * (kg >> 1) + 2 * n);
    const uint32_t vs = *reinterpret_cast<const uint32_t*>(p + kKv4ValueScale + 4 * n);
    floatx4 s[2];
    float mx = -INFINITY;
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const float sc = scale_f(ks >> (8 * t) & 255);
      const bf16x8 k0 = values8(t ? kc.z : kc.x, sc), k1 = values8(t ? kc.w : kc.y, sc);
      floatx4 acc = mfma_terms<QT>(k1, qt[1], mfma_terms<QT>(k0, qt[0], floatx4{0.f, 0.f, 0.f, 0.f}));
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if (g * 32 + 16 * t + 4 * kg + i >= len) acc[i] = -INFINITY;
        mx = fmaxf(mx, acc[i]);
      }
      s[t] = acc;
    }
    mx = fmaxf(mx, __shfl_xor(mx, 16));
    mx = fmaxf(mx, __shfl_xor(mx, 32));
    const float mn = fmaxf(m, mx), f = m == -INFINITY ? 0.f : __expf(m - mn);
    const float base = mn == -INFINITY ? 0.f : mn;
    m = mn;
    l *= f;
#pragma unroll
    for (int dt = 0; dt < 4; ++dt) o[dt] *= f;
    float pb[8];
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        s[t][i] = __expf(s[t][i] - base);
        l += s[t][i];
      }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const auto x = __builtin_amdgcn_permlane32_swap(__float_as_uint(s[0][i]), __float_as_uint(s[1][i]), false, false);
      const auto y = __builtin_amdgcn_permlane16_swap(x[0], x[1], false, false);
      pb[i] = __uint_as_float(y[0]);
      pb[4 + i] = __uint_as_float(y[1]);
    }
    bf16x8 pt[PT];
    split_terms<PT>(pb, pt);
    const uint32_t vw[4] = {vc.x, vc.y, vc.z, vc.w};
#pragma unroll
    for (int dt = 0; dt < 4; ++dt) {
      const bf16x8 v = values8(vw[dt], scale_f(vs >> (8 * dt) & 255));
      o[dt] = mfma_terms<PT>(v, pt, o[dt]);
    }
  }
  l += __shfl_xor(l, 16);
  l += __shfl_xor(l, 32);
  if (lane < 16) {
    wm[w][lane] = m;
    wl[w][lane] = l;
  }
#pragma unroll
  for (int dt = 0; dt < 4; ++dt)
#pragma unroll
    for (int i = 0; i < 4; ++i) wo[w][n][16 * dt + 4 * kg + i] = o[dt][i];
  __syncthreads();
  for (int t = threadIdx.x; t < 16 * 64; t += 256) {
    const int i = t >> 6, d = t & 63, out_row = blockIdx.z * 16 + i;
    if (out_row >= a.rows) break;
    float M = wm[0][i], L = 0.f, O = 0.f;
    for (int j = 1; j < 4; ++j) M = fmaxf(M, wm[j][i]);
    for (int j = 0; j < 4; ++j) {
      const float f = wm[j][i] == -INFINITY && wl[j][i] == 0.f ? 0.f : __expf(wm[j][i] - M);
      L = fmaf(f, wl[j][i], L);
      O = fmaf(f, wo[j][i][d], O);
    }
    reinterpret_cast<T*>(a.out)[(((size_t)r * a.rows + out_row) * a.c.n_head + head) * kHeadDim + d] =
        from_f<T>(L == 0.f ? 0.f : O / L);
  }
}

void kv4_attend(const Kv4AttendArgs& a, hipStream_t st) {
  const dim3 grid(a.c.n_head, a.n, (a.rows + 15) / 16);
  if (a.bf16_q) k_kv4_attend<bf16><<<grid, 256, 0, st>>>(a);
  else k_kv4_attend<float><<<grid, 256, 0, st>>>(a);
}

}  // namespace wf
