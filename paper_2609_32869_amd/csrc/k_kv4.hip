// Acoustic keys and values in 4 bits, and attention over them.
//
// Elements are e2m1 (0, 0.5, 1, 1.5, 2, 3, 4, 6 and their negatives) in blocks of 32 that
// share a power-of-two scale; a block lies along the axis that its product sums over
// (keys: 32 of a frame's 64 dims; values: 32 frames of one dim), so the eight elements
// that a lane gives a matrix instruction have one scale and one instruction turns two
// codes and the scale into two bf16 values, exactly.
#include <algorithm>

#include "wf_kv4.h"
#include "wf_operand.h"
#include "wf_ops.h"

namespace wf {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

// 8 codes -> the 8 bf16 values they stand for.
__device__ __forceinline__ bf16x8 values8(uint32_t c, float s) {
  const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, s, 0);
  const bf16x2 b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, s, 1);
  const bf16x2 d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, s, 2);
  const bf16x2 e = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, s, 3);
  return bf16x8{a[0], a[1], b[0], b[1], d[0], d[1], e[0], e[1]};
}

// ---------------------------------------------------------------- store
// A wave per (entry, head, 32-frame group), four heads a block: their rows lie beside each
// other.  Every load is issued before the first use and without a condition (frames at or
// beyond the length re-read the last given one and count as zero); a load under one would
// make each wait for the one before (16 ragged entries: 101 us against 53).  Memory bounds
// it: 96 entries of 1500 frames, 20 heads, fp32, 357 us or 4.7 TB/s, the copy rate.
template <int N>
__device__ __forceinline__ void ld_vals(const float* p, int vec, float* o) {
  if (vec) {
#pragma unroll
    for (int j = 0; j < N; j += 4) *reinterpret_cast<float4*>(o + j) = *reinterpret_cast<const float4*>(p + j);
  } else {
#pragma unroll
    for (int j = 0; j < N; ++j) o[j] = p[j];
  }
}
// bf16: raw bits, two values a word
template <int N>
__device__ __forceinline__ void ld_bits(const bf16* p, int vec, uint32_t* o) {
  if (vec) {
    if constexpr (N == 4) *reinterpret_cast<uint2*>(o) = *reinterpret_cast<const uint2*>(p);
    else
#pragma unroll
      for (int j = 0; j < N / 2; j += 4) *reinterpret_cast<uint4*>(o + j) = *reinterpret_cast<const uint4*>(p + 2 * j);
  } else {
#pragma unroll
    for (int j = 0; j < N; j += 2) o[j / 2] = (uint32_t)p[j].u | (uint32_t)p[j + 1].u << 16;
  }
}
// N consecutive source elements as they were loaded, converted where they are used.
template <typename T, int N>
struct Raw;
template <int N>
struct Raw<float, N> {
  float v[N];
  __device__ __forceinline__ void load(const float* p, int vec) { ld_vals<N>(p, vec, v); }
  __device__ __forceinline__ float get(int j) const { return v[j]; }
};
template <int N>
struct Raw<bf16, N> {
  uint32_t v[N / 2];
  __device__ __forceinline__ void load(const bf16* p, int vec) { ld_bits<N>(p, vec, v); }
  __device__ __forceinline__ float get(int j) const { return __uint_as_float(j & 1 ? v[j / 2] & 0xffff0000u : v[j / 2] << 16); }
};

// A group's key or value codes and scales from the lane's values (16 dims of frames n, 16 + n; 8 frames of dims
// 4 n .. + 3), of which those that are not `in` count as zero.
template <typename In>
__device__ __forceinline__ void put_keys(uint8_t* out, const In& in, float (&x)[2][16]) {
  const int lane = threadIdx.x & 63, n = lane & 15, kg = lane >> 4;
  uint2 c[2];
  uint32_t s[2];
#pragma unroll
  for (int t = 0; t < 2; ++t) {
    const bool ok = in(16 * t + n);
    uint32_t m = 0;
#pragma unroll
    for (int j = 0; j < 16; ++j) {
      x[t][j] = ok ? x[t][j] : 0.f;
      m = umax(m, mag(x[t][j]));
    }
    m = umax(m, (uint32_t)__shfl_xor((int)m, 16));  // the block's other 16 dims
    s[t] = scale_of(__uint_as_float(m));
    c[t] = make_uint2(codes8(x[t], scale_f(s[t])), codes8(x[t] + 8, scale_f(s[t])));
  }
  *reinterpret_cast<uint4*>(out + 16 * lane) = make_uint4(c[0].x, c[0].y, c[1].x, c[1].y);
  if ((kg & 1) == 0) *reinterpret_cast<uint16_t*>(out + kKv4KeyScale + 32 * (kg >> 1) + 2 * n) = (uint16_t)(s[0] | s[1] << 8);
}
template <typename In>
__device__ __forceinline__ void put_values(uint8_t* out, const In& in, float (&x)[4][8]) {
  const int lane = threadIdx.x & 63, n = lane & 15, kg = lane >> 4;
  uint32_t c[4], s = 0;
#pragma unroll
  for (int dt = 0; dt < 4; ++dt) {
    uint32_t m = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      x[dt][j] = in(8 * kg + j) ? x[dt][j] : 0.f;
      m = umax(m, mag(x[dt][j]));
    }
    m = umax(m, (uint32_t)__shfl_xor((int)m, 16));
    m = umax(m, (uint32_t)__shfl_xor((int)m, 32));
    const uint32_t sb = scale_of(__uint_as_float(m));
    c[dt] = codes8(x[dt], scale_f(sb));
    s |= sb << (8 * dt);
  }
  *reinterpret_cast<uint4*>(out + kKv4Values + 16 * lane) = make_uint4(c[0], c[1], c[2], c[3]);
  if (kg == 0) *reinterpret_cast<uint32_t*>(out + kKv4ValueScale + 4 * n) = s;
}

template <typename T>
__global__ void __launch_bounds__(256) k_kv4_store(Kv4StoreArgs a) {
  const int lane = threadIdx.x & 63, n = lane & 15, kg = lane >> 4;
  const int g = blockIdx.y, head = blockIdx.x * 4 + (threadIdx.x >> 6), r = blockIdx.z;
  if (head >= a.c.n_head) return;
  const int len = a.lens ? min(max(a.lens[r], 0), a.c.frames) : a.c.frames, top = max(len - 1, 0);
  uint8_t* out = a.c.base + (((size_t)(a.slot0 + r) * a.c.n_head + head) * a.c.groups + g) * kKv4Group;
  const T* K = reinterpret_cast<const T*>(a.k) + r * a.kr + head * a.kh + 16 * kg;
  const T* V = reinterpret_cast<const T*>(a.v) + r * a.vr + head * a.vh + 4 * n;
  if (g * 32 >= len) {  // uniform: nothing given (scales of 2^-120, as a block of zeros has)
    const uint4 z = make_uint4(0, 0, 0, 0);
    *reinterpret_cast<uint4*>(out + 16 * lane) = z;
    *reinterpret_cast<uint4*>(out + kKv4Values + 16 * lane) = z;
    if (lane < 32) *reinterpret_cast<uint32_t*>(out + kKv4KeyScale + 4 * lane) = 0x07070707u;
    return;
  }
  Raw<T, 16> k[2];
  Raw<T, 4> v[8];
#pragma unroll
  for (int t = 0; t < 2; ++t) k[t].load(K + min(g * 32 + 16 * t + n, top) * a.kf, a.vec);
#pragma unroll
  for (int j = 0; j < 8; ++j) v[j].load(V + min(g * 32 + 8 * kg + j, top) * a.vf, a.vec);
  auto in = [&](int f) { return g * 32 + f < len; };
  float x[2][16], y[4][8];
#pragma unroll
  for (int t = 0; t < 2; ++t)
#pragma unroll
    for (int j = 0; j < 16; ++j) x[t][j] = k[t].get(j);
#pragma unroll
  for (int dt = 0; dt < 4; ++dt)
#pragma unroll
    for (int j = 0; j < 8; ++j) y[dt][j] = v[j].get(dt);
  put_keys(out, in, x);
  put_values(out, in, y);
}

void kv4_store(const Kv4StoreArgs& a, hipStream_t st) {
  const dim3 grid((a.c.n_head + 3) / 4, a.c.groups, a.n);
  if (a.bf16_src) k_kv4_store<bf16><<<grid, 256, 0, st>>>(a);
  else k_kv4_store<float><<<grid, 256, 0, st>>>(a);
}

// ---------------------------------------------------------------- load
// The store's waves and lanes; the results' rows leave 16 bytes a lane: 16 entries of 1500
// frames into fp32 54 us, 5.1 TB/s (keys and values in waves of their own: 76).
__device__ __forceinline__ void st8(float* p, bf16x8 x) {
  *reinterpret_cast<float4*>(p) = make_float4((float)x[0], (float)x[1], (float)x[2], (float)x[3]);
  *reinterpret_cast<float4*>(p + 4) = make_float4((float)x[4], (float)x[5], (float)x[6], (float)x[7]);
}
__device__ __forceinline__ void st8(bf16* p, bf16x8 x) { *reinterpret_cast<uint4*>(p) = __builtin_bit_cast(uint4, x); }
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
__device__ __forceinline__ void st4(float* p, bf16x4 x) {
  *reinterpret_cast<float4*>(p) = make_float4((float)x[0], (float)x[1], (float)x[2], (float)x[3]);
}
__device__ __forceinline__ void st4(bf16* p, bf16x4 x) { *reinterpret_cast<uint2*>(p) = __builtin_bit_cast(uint2, x); }

template <typename T>
__global__ void __launch_bounds__(256) k_kv4_load(Kv4LoadArgs a) {
  const int lane = threadIdx.x & 63, n = lane & 15, kg = lane >> 4;
  const int g = blockIdx.y, head = blockIdx.x * 4 + (threadIdx.x >> 6), r = blockIdx.z;
  if (head >= a.c.n_head) return;
  const uint8_t* in = a.c.base + (((size_t)(a.slot0 + r) * a.c.n_head + head) * a.c.groups + g) * kKv4Group;
  const uint4 k = *reinterpret_cast<const uint4*>(in + 16 * lane), v = *reinterpret_cast<const uint4*>(in + kKv4Values + 16 * lane);
  const uint32_t ks = *reinterpret_cast<const uint16_t*>(in + kKv4KeyScale + 32 * (kg >> 1) + 2 * n);
  const uint32_t vs = *reinterpret_cast<const uint32_t*>(in + kKv4ValueScale + 4 * n);
  const size_t pitch = (size_t)a.c.n_head * kHeadDim, at = ((size_t)r * a.c.frames + g * 32) * pitch + head * kHeadDim;
  T* K = reinterpret_cast<T*>(a.k) + at + 16 * kg;
  T* V = reinterpret_cast<T*>(a.v) + at + 4 * n;
#pragma unroll
  for (int t = 0; t < 2; ++t) {
    const int f = 16 * t + n;
    const float s = scale_f(t ? ks >> 8 : ks & 255);
    if (g * 32 + f < a.c.frames) {
      st8(K + f * pitch, values8(t ? k.z : k.x, s));
      st8(K + f * pitch + 8, values8(t ? k.w : k.y, s));
    }
  }
  bf16x8 x[4];
  const uint32_t vw[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int dt = 0; dt < 4; ++dt) x[dt] = values8(vw[dt], scale_f(vs >> (8 * dt) & 255));
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const int f = 8 * kg + j;
    if (g * 32 + f < a.c.frames) st4(V + f * pitch, bf16x4{x[0][j], x[1][j], x[2][j], x[3][j]});
  }
}

void kv4_load(const Kv4LoadArgs& a, hipStream_t st) {
  const dim3 grid((a.c.n_head + 3) / 4, a.c.groups, a.n);
  if (a.bf16_out) k_kv4_load<bf16><<<grid, 256, 0, st>>>(a);
  else k_kv4_load<float><<<grid, 256, 0, st>>>(a);
}

// ---------------------------------------------------------------- a decoder's keys and values
// The values that the prompt pass's attention reads, in the request-time product's bf16
// layout, whose values lie transposed: a lane's eight frames of a dim are 16 consecutive
// bytes.  Grid z: entries.  Memory bounds it: about ten slots of 1,500 frames, 20 heads, 22 us.
__global__ void __launch_bounds__(256) k_kv4_unpack(Kv4UnpackArgs a) {
  const int lane = threadIdx.x & 63, n = lane & 15, kg = lane >> 4;
  const int g = blockIdx.x * 4 + (threadIdx.x >> 6), head = blockIdx.y, slot = a.slot0 + blockIdx.z, H = a.c.n_head, F = a.c.frames;
  if (g >= a.c.groups) return;
  const uint8_t* in = a.c.base + (((size_t)slot * H + head) * a.c.groups + g) * kKv4Group;
  const uint4 k = *reinterpret_cast<const uint4*>(in + 16 * lane), v = *reinterpret_cast<const uint4*>(in + kKv4Values + 16 * lane);
  const uint32_t ks = *reinterpret_cast<const uint16_t*>(in + kKv4KeyScale + 32 * (kg >> 1) + 2 * n);
  const uint32_t vs = *reinterpret_cast<const uint32_t*>(in + kKv4ValueScale + 4 * n);
  bf16* dst = a.kv + (size_t)slot * a.stride;
  bf16* K = dst + (size_t)head * F * kHeadDim + 16 * kg;
  bf16* V = dst + ((size_t)H * F + (size_t)head * a.vt_frames) * kHeadDim;
#pragma unroll
  for (int t = 0; t < 2; ++t) {
    const int f = g * 32 + 16 * t + n;
    const float s = scale_f(t ? ks >> 8 : ks & 255);
    if (f < F) {
      st8(K + (size_t)f * kHeadDim, values8(t ? k.z : k.x, s));
      st8(K + (size_t)f * kHeadDim + 8, values8(t ? k.w : k.y, s));
    }
  }
  const uint32_t vw[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int dt = 0; dt < 4; ++dt)  // frames past the last are zeros, as the layout has them
    st8(V + vt_index(4 * n + dt, g * 32 + 8 * kg), values8(vw[dt], scale_f(vs >> (8 * dt) & 255)));
}
void kv4_unpack(const Kv4UnpackArgs& a, hipStream_t st) {
  k_kv4_unpack<<<dim3((a.c.groups + 3) / 4, a.c.n_head, a.n), 256, 0, st>>>(a);
}

// ---------------------------------------------------------------- attention
// Block (head, request, chunk of the groups) x (16 query rows), eight waves; a wave takes
// steps of two groups, the next step's codes in flight while it multiplies the current one.
//   scores   S^T = K q^T per 16-frame tile (v_mfma_f32_16x16x32_bf16): lane 16 kg + n gets
//            row n of frames 4 kg .. + 3.  The queries' smallest terms first, so that two of
//            the six roundings are to the score's own size (one row of 131,072 frames whose
//            scores reach 15: off by 4.4e-7 in the 2-norm, largest first 1.7e-6)
//   softmax  running maximum and sum per row, one rescaling per step; the difference to the
//            maximum first, then powers of two: right at any magnitude of the scores
//   values   O^T = V^T P^T per group: two lane swaps turn the group's two score tiles into
//            the operand (lane: row n, frames 8 kg .. + 7)
//   output   waves joined in LDS; one chunk: O / l, else the chunk's (max, l, O) record for
//            the merge kernel

// bf16 terms of a query value and of a probability: as many as hold it exactly (an fp32 query three, a bf16 one one,
// a probability three).  Two terms of a probability, 2^-16 of it, are a tenth faster with bf16 rows (16 x 5 rows of ragged
// memories 10.7 us against 11.7) and round 0.24% of the bf16 outputs to the other side of 64 bits, three 0.017%, as sums
// in 32 bits do.  A decoder step's operands hold an fp32 value to 2^-16 themselves: two terms of each.
enum { KV4_ROWS = 0, KV4_OPERAND = 1, KV4_RECORDS = 2 };
template <typename T, int OUT>
struct Terms {
  static constexpr int q = sizeof(T) == 2 ? 1 : OUT == KV4_ROWS ? 3 : 2;
  static constexpr int p = OUT == KV4_ROWS ? 3 : 2;
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
__device__ __forceinline__ floatx4 mfma16(bf16x8 a, bf16x8 b, floatx4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ float swap_max(float v) {
  const auto x = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  v = fmaxf(__uint_as_float(x[0]), __uint_as_float(x[1]));
  const auto y = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return fmaxf(__uint_as_float(y[0]), __uint_as_float(y[1]));
}
__device__ __forceinline__ float swap_sum(float v) {
  const auto x = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  v = __uint_as_float(x[0]) + __uint_as_float(x[1]);
  const auto y = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return __uint_as_float(y[0]) + __uint_as_float(y[1]);
}

// Codes and scales of KS groups.
template <int KS>
struct KvStep {
  uint4 k[KS], v[KS];
  uint32_t ks[KS], vs[KS];
};
// Groups g .. g + KS - 1 (those from `end` on re-read group end - 1, masked below).
template <int KS>
__device__ __forceinline__ void kv_load(const uint8_t* in, int g, int end, KvStep<KS>& s) {
  const int lane = threadIdx.x & 63, n = lane & 15, kg = lane >> 4;
#pragma unroll
  for (int u = 0; u < KS; ++u) {
    const uint8_t* p = in + (size_t)min(g + u, end - 1) * kKv4Group;
    s.k[u] = *reinterpret_cast<const uint4*>(p + 16 * lane);
    s.v[u] = *reinterpret_cast<const uint4*>(p + kKv4Values + 16 * lane);
    s.ks[u] = *reinterpret_cast<const uint16_t*>(p + kKv4KeyScale + 32 * (kg >> 1) + 2 * n);
    s.vs[u] = *reinterpret_cast<const uint32_t*>(p + kKv4ValueScale + 4 * n);
  }
}
constexpr float kLog2e = 1.44269504088896f;
// exp(x - m) for a maximum m that is -inf where there is no x yet: 0 there.
__device__ __forceinline__ float no_inf(float m) { return m == -INFINITY ? 0.f : m; }
__device__ __forceinline__ float exp_to(float x, float base) { return __builtin_amdgcn_exp2f((x - base) * kLog2e); }
// A row's running state: maximum of the scores, the lane's share of the sum, O^T.  (Rescaling only where the maximum
// moves by more than a few powers costs registers past 64, a block per CU fewer: 68 us against 52 at 96 x 9 rows.)
struct RowState {
  float m, l;
  floatx4 o[4];
};
template <int KS, int QT, int PT>
__device__ __forceinline__ void kv_step(KvStep<KS>& c, int g, int len, const bf16x8 (&qt)[2][QT], RowState& st) {
  const int kg = (threadIdx.x & 63) >> 4;
  floatx4 s[2 * KS];
#pragma unroll
  for (int t = 0; t < 2 * KS; ++t) {
    const int u = t >> 1;
    const float sc = scale_f(t & 1 ? c.ks[u] >> 8 : c.ks[u] & 255);
    const bf16x8 k0 = values8(t & 1 ? c.k[u].z : c.k[u].x, sc), k1 = values8(t & 1 ? c.k[u].w : c.k[u].y, sc);
    s[t] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = QT - 1; i >= 0; --i)
      s[t] = mfma16(k1, qt[1][i], mfma16(k0, qt[0][i], s[t]));
  }
  if ((g + KS) * kKv4Frames > len) {  // uniform: the last step
#pragma unroll
    for (int t = 0; t < 2 * KS; ++t)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (g * kKv4Frames + 16 * t + 4 * kg + i >= len) s[t][i] = -INFINITY;
#pragma unroll
    for (int u = 0; u < KS; ++u) {  // values past the length may stand for infinity: 0 instead
      const int left = len - (g + u) * kKv4Frames - 8 * kg;
      const uint32_t in = left >= 8 ? ~0u : left <= 0 ? 0u : (1u << 4 * left) - 1;
      c.v[u].x &= in;
      c.v[u].y &= in;
      c.v[u].z &= in;
      c.v[u].w &= in;
    }
  }
  float mx = -INFINITY;
#pragma unroll
  for (int t = 0; t < 2 * KS; ++t)
#pragma unroll
    for (int i = 0; i < 4; ++i) mx = fmaxf(mx, s[t][i]);
  const float m = fmaxf(st.m, swap_max(mx)), base = no_inf(m);
  const float f = exp_to(st.m, base);  // 0 at first
  st.m = m;
  float l = 0.f;
#pragma unroll
  for (int t = 0; t < 2 * KS; ++t)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      s[t][i] = exp_to(s[t][i], base);
      l += s[t][i];
    }
  st.l = fmaf(st.l, f, l);
#pragma unroll
  for (int dt = 0; dt < 4; ++dt) st.o[dt] *= f;
#pragma unroll
  for (int u = 0; u < KS; ++u) {
    float pb[8];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const auto x = __builtin_amdgcn_permlane32_swap(__float_as_uint(s[2 * u][i]), __float_as_uint(s[2 * u + 1][i]), false, false);
      const auto y = __builtin_amdgcn_permlane16_swap(x[0], x[1], false, false);
      pb[i] = __uint_as_float(y[0]);
      pb[4 + i] = __uint_as_float(y[1]);
    }
    bf16x8 pt[PT];
    split_terms<PT>(pb, pt);
    const uint32_t vw[4] = {c.v[u].x, c.v[u].y, c.v[u].z, c.v[u].w};
#pragma unroll
    for (int dt = 0; dt < 4; ++dt) {
      const bf16x8 x = values8(vw[dt], scale_f(c.vs[u] >> (8 * dt) & 255));
#pragma unroll
      for (int i = PT - 1; i >= 0; --i) st.o[dt] = mfma16(x, pt[i], st.o[dt]);
    }
  }
}

// The lane's 16 query values (dims 16 kg ..) of row `row`, times 1 / sqrt(64).
template <typename T>
__device__ __forceinline__ void q_load(const Kv4AttendArgs& a, int r, int row, int head, float* x) {
  const int kg = (threadIdx.x & 63) >> 4;
  const T* q = reinterpret_cast<const T*>(a.q) + r * a.sr + (long long)min(row, a.rows - 1) * a.si + head * a.sh + 16 * kg;
  if (a.vec) {
#pragma unroll
    for (int j = 0; j < 16; j += 8) ld8(q + j, x + j);
  } else {
#pragma unroll
    for (int j = 0; j < 16; ++j) x[j] = to_f(q[j]);
  }
#pragma unroll
  for (int j = 0; j < 16; ++j) x[j] = row < a.rows ? 0.125f * x[j] : 0.f;
}

// Waves a block and groups a step.  us a replayed call (20 heads; fp32 1 x 9 rows, 96 x 9 rows of 1,500 frames, one row of
// 131,072; bf16 16 x 5 rows of ragged memories): 8 waves of 2: 8.5, 50, 39.7, 11.7; of 1: 6.9, 50, 40.3, 13.1; of 3: 8.7,
// 61, 50, 11.2; 4 waves of 2: 7.0, 50, 41.3, 12.5; 16 of 2: 8.8, 67, 53, 11.9.
constexpr int kAttWaves = 8, kAttStep = 2;
constexpr int kKv4Record = 32 + 16 * 64;  // max [16], sum [16], O [16][64]

template <typename T, int OUT, int NW = kAttWaves, int KS = kAttStep>
__global__ void __launch_bounds__(NW * 64) k_kv4_attend(Kv4AttendArgs a) {
  constexpr int QT = Terms<T, OUT>::q, PT = Terms<T, OUT>::p, S = NW * KS;
  StampScope stamp_scope(OUT == KV4_ROWS ? nullptr : a.stamp, NW * 64);
  __shared__ float wm[NW][16], wl[NW][16], wo[NW][16][68];
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, n = lane & 15, kg = lane >> 4;
  const int head = blockIdx.x % a.c.n_head, chunk = blockIdx.x / a.c.n_head, r = blockIdx.y, row = blockIdx.z * 16 + n;
  const int len = a.lens ? min(max(a.lens[r], 0), a.c.frames) : a.c.frames;
  const uint8_t* in = a.c.base + ((size_t)(a.slot0 + r) * a.c.n_head + head) * a.c.groups * kKv4Group;
  const int end = min((chunk + 1) * a.cgroups, (len + kKv4Frames - 1) / kKv4Frames);
  const int lim = min(len, end * kKv4Frames);  // a step that reaches past the chunk holds its last group again
  int g = chunk * a.cgroups + w * KS;
  RowState st;
  st.m = -INFINITY;
  st.l = 0.f;
#pragma unroll
  for (int dt = 0; dt < 4; ++dt) st.o[dt] = floatx4{0.f, 0.f, 0.f, 0.f};
  if (g < end) {
    KvStep<KS> A, B;
    kv_load<KS>(in, g, end, A);
    float x[16];
    q_load<T>(a, r, row, head, x);
    bf16x8 qt[2][QT];
    split_terms<QT>(x, qt[0]);
    split_terms<QT>(x + 8, qt[1]);
    for (;;) {
      kv_load<KS>(in, g + S, end, B);
      kv_step<KS, QT, PT>(A, g, lim, qt, st);
      g += S;
      if (g >= end) break;
      kv_load<KS>(in, g + S, end, A);
      kv_step<KS, QT, PT>(B, g, lim, qt, st);
      g += S;
      if (g >= end) break;
    }
  }
  const float l = swap_sum(st.l);
  if (lane < 16) {
    wm[w][lane] = st.m;
    wl[w][lane] = l;
  }
  // value tile dt holds dims 4 m + dt: o[dt][i] of the lane is dim 16 kg + 4 i + dt
#pragma unroll
  for (int i = 0; i < 4; ++i)
    *reinterpret_cast<floatx4*>(&wo[w][n][16 * kg + 4 * i]) = floatx4{st.o[0][i], st.o[1][i], st.o[2][i], st.o[3][i]};
  __syncthreads();
  const int nr = min(16, a.rows - (int)blockIdx.z * 16);
  for (int t = threadIdx.x; t < nr * 64; t += NW * 64) {
    const int i = t >> 6, d = t & 63;
    float M = wm[0][i], L = 0.f, O = 0.f;
#pragma unroll
    for (int j = 1; j < NW; ++j) M = fmaxf(M, wm[j][i]);
    const float base = no_inf(M);
#pragma unroll
    for (int j = 0; j < NW; ++j) {
      const float f = exp_to(wm[j][i], base);  // 0 for a wave of no frames
      L = fmaf(f, wl[j][i], L);
      O = fmaf(f, wo[j][i][d], O);
    }
    if constexpr (OUT == KV4_OPERAND) {
      put_op<bf16>(a.op, a.nsplit, a.R9, a.row0 + r * a.rows + i, head * kHeadDim + d, O / L);
    } else if constexpr (OUT == KV4_RECORDS) {
      float* rec = a.part + (((size_t)r * a.c.n_head + head) * a.nchunk + chunk) * kXrPart;
      rec[32 + t] = O;
      if (d == 0) {
        rec[i] = M;
        rec[16 + i] = L;
      }
    } else if (a.nchunk == 1) {
      reinterpret_cast<T*>(a.out)[(((size_t)r * a.rows + blockIdx.z * 16 + i) * a.c.n_head + head) * kHeadDim + d] =
          from_f<T>(L == 0.f ? 0.f : O / L);
    } else {
      float* rec = a.part + ((((size_t)r * gridDim.z + blockIdx.z) * a.c.n_head + head) * a.nchunk + chunk) * kKv4Record;
      rec[32 + t] = O;
      if (d == 0) {
        rec[i] = M;
        rec[16 + i] = L;
      }
    }
  }
}

// Joins the chunks of one row of a (head, request): 16 threads (4 dims each) take every
// sixteenth chunk, so that a few loads per thread are in flight at once, and meet in LDS.
template <typename T>
__global__ void __launch_bounds__(256) k_kv4_merge(Kv4AttendArgs a) {
  __shared__ float wm[16], wl[16], wo[16][64];
  const int head = blockIdx.x, r = blockIdx.y, row = blockIdx.z, tile = row >> 4, i = row & 15, tiles = (a.rows + 15) >> 4;
  const int t = threadIdx.x, q = t >> 4, d = 4 * (t & 15);
  const float* rec = a.part + (((size_t)r * tiles + tile) * a.c.n_head + head) * a.nchunk * kKv4Record;
  float M = -INFINITY, L = 0.f;
  floatx4 O = {0.f, 0.f, 0.f, 0.f};
  constexpr int U = 4;
  for (int c0 = q; c0 < a.nchunk; c0 += 16 * U) {
    float m[U], l[U];
    floatx4 o[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const float* p = rec + (size_t)min(c0 + 16 * u, a.nchunk - 1) * kKv4Record;
      m[u] = p[i];
      l[u] = p[16 + i];
      o[u] = *reinterpret_cast<const floatx4*>(p + 32 + i * 64 + d);
    }
    float Mn = M;
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (c0 + 16 * u < a.nchunk) Mn = fmaxf(Mn, m[u]);
    const float base = no_inf(Mn), f0 = exp_to(M, base);
    M = Mn;
    L *= f0;
    O *= f0;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (c0 + 16 * u < a.nchunk) {
        const float f = exp_to(m[u], base);
        L = fmaf(f, l[u], L);
        O += f * o[u];
      }
    }
  }
  *reinterpret_cast<floatx4*>(&wo[q][d]) = O;
  if (d == 0) {
    wm[q] = M;
    wl[q] = L;
  }
  __syncthreads();
  if (t < 64) {
    float m = wm[0], l = 0.f, o = 0.f;
#pragma unroll
    for (int j = 1; j < 16; ++j) m = fmaxf(m, wm[j]);
    const float base = no_inf(m);
#pragma unroll
    for (int j = 0; j < 16; ++j) {
      const float f = exp_to(wm[j], base);
      l = fmaf(f, wl[j], l);
      o = fmaf(f, wo[j][t], o);
    }
    reinterpret_cast<T*>(a.out)[(((size_t)r * a.rows + row) * a.c.n_head + head) * kHeadDim + t] = from_f<T>(l == 0.f ? 0.f : o / l);
  }
}

// Groups of a chunk: a long memory over about four blocks per CU, so that requests of different lengths share the
// chip, in whole steps of a block's waves (16 groups, the nearest).  us a replayed call of 4,500 frames, 20 heads, split
// against one block per (head, request): 20 pairs 7.6 / 18.1, 80 pairs 13.1 / 18.5, 320 pairs 28.3 / 33.4; of 131,072 frames:
// 20 pairs 39.9 / 418, 160 pairs 306 / 424.  Not split: up to 1,536 frames (20 pairs, 1,500 frames: 7.2 / 8.2, but the merge's
// launch costs the caller more); from 480 pairs; and, below 8,192 frames, pairs that give each CU as many blocks within a
// fifth (240 pairs, 4,500 frames: 25.6 / 20.2; 460 pairs: 41.3 / 34.0).  Towards 512 blocks instead of 1,024 equal lengths
// are a tenth faster at times (168 pairs, 13,512 frames: 38.5 against 43.1; 160 of 4,500: 18.4 against 20.4) and mixed ones
// far slower (160 pairs of up to 16,384: 41 against 32; 40 of up to 131,072: 73 against 42).
static int kv4_chunk(int n, int rows, int n_head, int frames) {
  constexpr int step = kAttWaves * kAttStep, cus = 256;
  const int pairs = (int)std::min<long long>((long long)n * n_head * ((rows + 15) / 16), 1 << 20), groups = kv4_groups(frames);
  const bool even = 5 * pairs >= 4 * ((pairs + cus - 1) / cus * cus);
  if (groups <= 3 * step || pairs >= 480 || (even && groups < 256)) return groups;
  const int chunks = 1024 / pairs, each = (groups + chunks - 1) / chunks;
  return std::max(step, (each + step / 2) / step * step);
}
static int kv4_chunks(int n, int rows, int n_head, int frames) {
  const int each = kv4_chunk(n, rows, n_head, frames);
  return (kv4_groups(frames) + each - 1) / each;
}
size_t kv4_workspace(int n, int rows, int n_head, int frames) {
  const int nc = kv4_chunks(n, rows, n_head, frames);
  return nc == 1 ? 0 : (size_t)n * n_head * ((rows + 15) / 16) * nc * kKv4Record * 4;
}

template <typename T>
static void attend_launch(const Kv4AttendArgs& a, hipStream_t st) {
  const int tiles = (a.rows + 15) / 16;
  k_kv4_attend<T, KV4_ROWS><<<dim3(a.c.n_head * a.nchunk, a.n, tiles), kAttWaves * 64, 0, st>>>(a);
  if (a.nchunk > 1) k_kv4_merge<T><<<dim3(a.c.n_head, a.n, a.rows), 256, 0, st>>>(a);
}
void kv4_attend(const Kv4AttendArgs& a0, hipStream_t st) {
  Kv4AttendArgs a = a0;
  a.cgroups = kv4_chunk(a.n, a.rows, a.c.n_head, a.c.frames);
  a.nchunk = kv4_chunks(a.n, a.rows, a.c.n_head, a.c.frames);
  if (a.bf16_q) attend_launch<bf16>(a, st);
  else attend_launch<float>(a, st);
}

void kv4_attend_operand(const Kv4AttendArgs& a0, hipStream_t st) {
  Kv4AttendArgs a = a0;
  a.nchunk = 1;
  a.cgroups = a.c.groups;
  k_kv4_attend<float, KV4_OPERAND><<<dim3(a.c.n_head, a.n, (a.rows + 15) / 16), kAttWaves * 64, 0, st>>>(a);
}
// Four waves of a group each: the chunks of 128 frames that the step of one slot takes.
void kv4_attend_records(const Kv4AttendArgs& a0, hipStream_t st) {
  static_assert(kXrPart == 32 + kRows * 64, "records hold nine rows");
  Kv4AttendArgs a = a0;
  a.cgroups = cross_mx_chunk(1) / kKv4Frames;
  a.nchunk = cross_mx_chunks(1, a.c.frames);
  k_kv4_attend<float, KV4_RECORDS, 4, 1><<<dim3(a.c.n_head * a.nchunk, a.n), 256, 0, st>>>(a);
}

}  // namespace wf
