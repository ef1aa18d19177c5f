// A paged self-attention cache in 8 bits, and attention over it.
//
// Elements are e4m3 with a power-of-two scale for the keys and one for the values of a page (16
// positions) and head, so one instruction turns two codes and the scale into two bf16 values,
// exactly, and a page whose scale grows keeps its values unless they fall below the new scale's
// smallest normal one.
#include <algorithm>

#include "wf_kv4.h"
#include "wf_operand.h"
#include "wf_ops.h"

namespace wf {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

// Smallest 2^e, e >= -100, with amax <= 448 * 2^e = 1.75 * 2^(e + 8), as a biased exponent.
__device__ __forceinline__ uint32_t scale8_of(float amax) {
  const uint32_t u = __float_as_uint(amax);
  const int e = (int)(u >> 23) - ((u & 0x7fffffu) <= 0x600000u ? 8 : 7);
  return (uint32_t)max(e, 27);
}
// 4 values -> 4 codes, element i in byte i; `inv` the scale's inverse.  No |x| inv passes 448.  What is
// not finite becomes NaN.
__device__ __forceinline__ uint32_t codes8x4(const float* x, float inv) {
  float y[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) y[j] = mag(x[j]) >= 0x7f800000u ? __uint_as_float(0x7fc00000u) : x[j] * inv;
  int r = __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], 0, false);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], r, true);
}
// 4 codes -> the 4 values they stand for.
__device__ __forceinline__ void values8x4(uint32_t c, float s, float* x) {
  const auto a = __builtin_amdgcn_cvt_pk_f32_fp8((int)c, false), b = __builtin_amdgcn_cvt_pk_f32_fp8((int)c, true);
  x[0] = a[0] * s;
  x[1] = a[1] * s;
  x[2] = b[0] * s;
  x[3] = b[1] * s;
}
__device__ __forceinline__ uint32_t mag_finite(float x) { return mag(x) >= 0x7f800000u ? 0u : mag(x); }
// 2^(127 - byte) of a scale byte in [27, 247]
__device__ __forceinline__ float inverse_f(uint32_t byte) { return __uint_as_float((254u - byte) << 23); }

// The whole wave's maxima of two non-negative numbers, as floats' bits.
template <int CTRL>
__device__ __forceinline__ uint32_t umax_dpp(uint32_t v) {
  return umax(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xf, 0xf, false));
}
__device__ __forceinline__ uint32_t umax16(uint32_t v) {
  return umax_dpp<kDppMirror>(umax_dpp<kDppHalfMirror>(umax_dpp<kDppXor2>(umax_dpp<kDppXor1>(v))));
}
__device__ __forceinline__ void wave_umax(uint32_t& a, uint32_t& b) {
  a = umax16(a);
  b = umax16(b);
  auto lane = [](uint32_t v, int l) { return (uint32_t)__builtin_amdgcn_readlane((int)v, l); };
  a = umax(umax(lane(a, 0), lane(a, 16)), umax(lane(a, 32), lane(a, 48)));
  b = umax(umax(lane(b, 0), lane(b, 16)), umax(lane(b, 32), lane(b, 48)));
}
// Four consecutive elements.
__device__ __forceinline__ void ld4(const float* p, int vec, float* o) {
  if (vec) {
    const float4 v = *reinterpret_cast<const float4*>(p);
    o[0] = v.x; o[1] = v.y; o[2] = v.z; o[3] = v.w;
  } else {
#pragma unroll
    for (int j = 0; j < 4; ++j) o[j] = p[j];
  }
}
__device__ __forceinline__ void ld4(const bf16* p, int vec, float* o) {
  if (vec) {
    const uint2 v = *reinterpret_cast<const uint2*>(p);
    o[0] = __uint_as_float(v.x << 16);
    o[1] = __uint_as_float(v.x & 0xffff0000u);
    o[2] = __uint_as_float(v.y << 16);
    o[3] = __uint_as_float(v.y & 0xffff0000u);
  } else {
#pragma unroll
    for (int j = 0; j < 4; ++j) o[j] = to_f(p[j]);
  }
}
// In the store and the load, lane 16 kg + n has dims 4 n .. + 3 of positions 4 kg .. + 3, so that a wave reads and writes
// whole rows.  The code words: of its keys, dims 4 n .. of position 4 kg + j; of its values, those positions of dim 4 n + j.
__device__ __forceinline__ int key_code(int lane, int j) { return 256 * ((lane & 15) >> 2) + 16 * (4 * (lane >> 4) + j) + 4 * (lane & 3); }
__device__ __forceinline__ int value_code(int lane, int j) {
  return kKv8Values + 32 * (16 * (lane >> 5) + (lane & 15)) + 8 * j + 4 * ((lane >> 4) & 1);
}

// ---------------------------------------------------------------- store
// A wave per (page that a request writes, head): the page's scale is the maximum of 1,024 elements, so a wave holds it whole
// and reads and writes it once.  Bytes bound it: 8 x 8,192 rows of 8 heads, fp32, 335 MB, in 64 us store after store (5.2 TB/s, a
// large copy's rate), 95 behind a load that has just written 537 MB.  Nine rows of each of 96 requests, 20 heads, 9.4 us (10.9 behind
// a load): positions, page numbers, kept codes, scales, one trip to memory after the other.  Where a request's pages lie in the
// grid: request r's first page has number starts[r] / 16 + 2 r (packed), which leaves room for every page that its rows can touch, or r * per (padded).
template <typename T>
__global__ void __launch_bounds__(256) k_kv8_store(Kv8StoreArgs a, int per, int hb) {
  // neighbouring blocks take neighbouring heads of one page, whose rows lie beside each other; by grid y where there are too many
  const int unit = gridDim.y > 1 ? blockIdx.x : blockIdx.x / (unsigned)hb, hq = gridDim.y > 1 ? blockIdx.y : blockIdx.x - unit * hb;
  const int lane = threadIdx.x & 63, head = __builtin_amdgcn_readfirstlane(hq * 4 + (threadIdx.x >> 6));
  if (head >= a.c.n_head) return;
  int r, col, first, count;
  if (a.starts) {
    int lo = 0, hi = a.n;  // the last request whose first number is <= the block's
    auto at = [&](int i) { return min(max(a.starts[i], 0), a.rows); };
    while (hi - lo > 1) {
      const int m = (lo + hi) >> 1;
      if (at(m) / 16 + 2 * m <= unit) lo = m;
      else hi = m;
    }
    r = lo;
    first = at(r);
    count = at(r + 1) - first;
    col = unit - (first / 16 + 2 * r);
  } else {
    r = unit / (unsigned)per;
    col = unit - r * per;
    first = 0;
    count = a.counts ? min(max(a.counts[r], 0), a.rows) : a.rows;
  }
  const long long pos = a.positions[r], begin = max(pos, 0ll);  // first position stored
  const long long page0 = (begin >> 4) + col;                    // this wave's page of the request
  if (col < 0 || count <= 0 || page0 >= a.max_pages || page0 * 16 >= pos + count) return;
  const int page = a.tables[r * a.ts + page0];
  const long long skip = page0 * 16 - pos;  // row of position 0 of the page (negative: kept positions before the rows)
  const int kept = (int)max(-skip, 0ll);    // positions [0, kept) stay, [kept, end) are rows
  const int end = (int)min(count - skip, 16ll);
  // Every load is issued before the first use and without a condition (positions that are no row's take the nearest
  // row and are replaced): a load under one would make each wait for the one before.
  const int n = lane & 15, kg = lane >> 4;
  const T* K = reinterpret_cast<const T*>(a.k) + (a.starts ? 0 : r * a.kr) + head * a.kh + 4 * n;
  const T* V = reinterpret_cast<const T*>(a.v) + (a.starts ? 0 : r * a.vr) + head * a.vh + 4 * n;
  float x[4][4], y[4][4];  // [position 4 kg + j][dim 4 n + ..]
  if (kept == 0 && end == 16) {  // a page of rows alone
    const T *k = K + (first + skip) * a.ki + 4 * kg * a.ki, *v = V + (first + skip) * a.vi + 4 * kg * a.vi;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      ld4(k + j * a.ki, a.vec, x[j]);
      ld4(v + j * a.vi, a.vec, y[j]);
    }
  } else {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const long long row = first + min(max(skip + 4 * kg + j, 0ll), (long long)count - 1);
      ld4(K + row * a.ki, a.vec, x[j]);
      ld4(V + row * a.vi, a.vec, y[j]);
    }
  }
  if (page < 0 || page >= a.c.n_pages) return;
  uint8_t* out = a.c.base + page * a.c.page + (size_t)head * kKv8Head;
  uint8_t* sc = a.c.base + page * a.c.page + (size_t)a.c.n_head * kKv8Head + 2 * head;
#pragma unroll
  for (int j = 0; j < 4; ++j)
#pragma unroll
    for (int d = 0; d < 4; ++d) {
      x[j][d] = 4 * kg + j < end ? x[j][d] : 0.f;
      y[j][d] = 4 * kg + j < end ? y[j][d] : 0.f;
    }
  if (kept) {  // uniform
    const uint32_t old = *reinterpret_cast<const uint16_t*>(sc);
    uint32_t kc[4], vc[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      kc[j] = *reinterpret_cast<const uint32_t*>(out + key_code(lane, j));
      vc[j] = *reinterpret_cast<const uint32_t*>(out + value_code(lane, j));
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      float p[4], q[4];
      values8x4(kc[j], scale_f(old & 255), p);
      values8x4(vc[j], scale_f(old >> 8), q);
#pragma unroll
      for (int d = 0; d < 4; ++d) {
        x[j][d] = 4 * kg + j < kept ? p[d] : x[j][d];
        y[d][j] = 4 * kg + d < kept ? q[d] : y[d][j];
      }
    }
  }
  uint32_t m = 0, m2 = 0;
#pragma unroll
  for (int j = 0; j < 16; ++j) {
    m = umax(m, mag_finite(x[j >> 2][j & 3]));
    m2 = umax(m2, mag_finite(y[j >> 2][j & 3]));
  }
  wave_umax(m, m2);
  const uint32_t ks = scale8_of(__uint_as_float(m)), vs = scale8_of(__uint_as_float(m2));
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const float q[4] = {y[0][j], y[1][j], y[2][j], y[3][j]};
    *reinterpret_cast<uint32_t*>(out + key_code(lane, j)) = codes8x4(x[j], inverse_f(ks));
    *reinterpret_cast<uint32_t*>(out + value_code(lane, j)) = codes8x4(q, inverse_f(vs));
  }
  if (lane == 0) *reinterpret_cast<uint16_t*>(sc) = (uint16_t)(ks | vs << 8);
}

void kv8_store(const Kv8StoreArgs& a, hipStream_t st) {
  const int per = (a.rows + 30) / 16;  // pages that a request's rows can touch
  const long long units = a.starts ? a.rows / 16 + 2ll * a.n + 1 : (long long)per * a.n;
  const int hb = (a.c.n_head + 3) / 4;
  const dim3 grid = units * hb < 1 << 24 ? dim3((unsigned)(units * hb)) : dim3((unsigned)units, hb);
  if (a.bf16_src) k_kv8_store<bf16><<<grid, 256, 0, st>>>(a, per, hb);
  else k_kv8_store<float><<<grid, 256, 0, st>>>(a, per, hb);
}

// ---------------------------------------------------------------- load
__device__ __forceinline__ void st4(float* p, const float* x) { *reinterpret_cast<float4*>(p) = make_float4(x[0], x[1], x[2], x[3]); }
__device__ __forceinline__ void st4(bf16* p, const float* x) {
  *reinterpret_cast<uint2*>(p) = make_uint2(pack2_bf16(x[0], x[1]), pack2_bf16(x[2], x[3]));
}
// A wave per (request, column of its table, head).  Bytes bound it: 8 x 8,192 positions of 8 heads into fp32 604 MB, 99 us
// (6.1 TB/s, nine tenths of them writes).
template <typename T>
__global__ void __launch_bounds__(256) k_kv8_load(Kv8LoadArgs a) {
  const int lane = threadIdx.x & 63, head = blockIdx.y * 4 + (threadIdx.x >> 6), n = lane & 15, kg = lane >> 4;
  if (head >= a.c.n_head) return;
  const int r = blockIdx.x / a.max_pages, col = blockIdx.x - r * a.max_pages;
  const int page = a.tables[r * a.ts + col];
  const int len = min(max(a.lens[r], 0), 16 * a.max_pages) - 16 * col;  // positions of this page
  const bool there = page >= 0 && page < a.c.n_pages && len > 0;
  const size_t pitch = (size_t)a.c.n_head * kHeadDim, at = ((size_t)blockIdx.x * 16 + 4 * kg) * pitch + head * kHeadDim + 4 * n;
  T* K = reinterpret_cast<T*>(a.k) + at;
  T* V = reinterpret_cast<T*>(a.v) + at;
  float x[4][4], y[4][4];  // x[j]: dims 4 n .. of position 4 kg + j; y[dt]: dim 4 n + dt of those positions
  if (there) {             // uniform
    const uint8_t* in = a.c.base + page * a.c.page + (size_t)head * kKv8Head;
    const uint32_t s = *reinterpret_cast<const uint16_t*>(a.c.base + page * a.c.page + (size_t)a.c.n_head * kKv8Head + 2 * head);
    uint32_t c[4], v[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      c[j] = *reinterpret_cast<const uint32_t*>(in + key_code(lane, j));
      v[j] = *reinterpret_cast<const uint32_t*>(in + value_code(lane, j));
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      values8x4(c[j], scale_f(s & 255), x[j]);
      values8x4(v[j], scale_f(s >> 8), y[j]);
    }
  }
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const bool in = there && 4 * kg + j < len;
    const float p[4] = {in ? x[j][0] : 0.f, in ? x[j][1] : 0.f, in ? x[j][2] : 0.f, in ? x[j][3] : 0.f};
    const float q[4] = {in ? y[0][j] : 0.f, in ? y[1][j] : 0.f, in ? y[2][j] : 0.f, in ? y[3][j] : 0.f};
    st4(K + j * pitch, p);
    st4(V + j * pitch, q);
  }
}

void kv8_load(const Kv8LoadArgs& a, hipStream_t st) {
  const dim3 grid((unsigned)((long long)a.n * a.max_pages), (a.c.n_head + 3) / 4);
  if (a.bf16_out) k_kv8_load<bf16><<<grid, 256, 0, st>>>(a);
  else k_kv8_load<float><<<grid, 256, 0, st>>>(a);
}

// ---------------------------------------------------------------- attention
// A key and value head's query columns are the rows of its group's heads: column c is row c / group,
// head c % group of the group.  Block (key and value head, request, 16 columns, chunk of the
// positions) x NW waves; a wave takes steps of 32 positions (two pages), every NW-th.
//   scores   S^T = K q^T per page (v_mfma_f32_16x16x32_bf16): lane 16 kg + n gets column n of
//            positions 4 kg .. + 3
//   softmax  per column a reference, which moves up to the maximum where a score passes it by kRaise (as every
//            time a maximum moves, most steps of a short context rescaled), in steps with values above 448 where a score
//            passes it at all: such values meet probabilities of at most 1, so that n of up to 3.4e38 / n have finite
//            sums; and the sum
//   values   O^T = V^T P^T per step: two lane swaps turn its two score tiles into the operand
//            (lane: column n, positions 8 kg .. + 7)
//   output   waves joined in LDS; one chunk: O / l, else the chunk's (reference, l, O) record for the
//            merge kernel
// A step's codes, scales and page numbers are loaded while the one before is multiplied.  Bytes bound long contexts: four
// requests of one row at 131,071, 8 heads of four each, 538 MB in 99 us (5.4 TB/s; the merge 5 us more).  Vector
// instructions bound many rows, whose every 16 columns turn the codes into values anew: 185 x 29 at 0 to 2,069, 32 heads over 8, 186 us.
// Of many short ones, 96 x 9 rows at 0 to 438, 20 heads (17.0 us, the bytes 12), the start and end of 1,920 blocks are the rest.  Two
// tiles of 16 columns to a block would share the conversion of their keys and values, but leave half the blocks and 156
// registers: with probabilities in two terms four x nine rows from 65,536 on, 32 heads over 8, 190 us for 143, 32 x nine at 0 to
// 4,000 56 for 41.
namespace {
constexpr float kScale = 0.125f * 1.44269504088896f;  // exp(s / 8) = 2^(kScale s)
constexpr float kRaise = 8.f / kScale;
constexpr int kRecord = 32 + 16 * 64;  // reference [16], sum [16], O [16][64]

__device__ __forceinline__ float no_inf(float m) { return m == -INFINITY ? 0.f : m; }
__device__ __forceinline__ float exp_to(float x, float base) { return __builtin_amdgcn_exp2f((x - base) * kScale); }
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
// Eight values as N bf16 terms: three hold an fp32 value exactly, one a bf16 value.
template <int N>
__device__ __forceinline__ void split_terms(const float* v, bf16x8 (&t)[N]) {
  uint4 u[3];
  if constexpr (N == 3) split3x8(v, u[0], u[1], u[2]);
  else u[0] = make_uint4(pack2_bf16(v[0], v[1]), pack2_bf16(v[2], v[3]), pack2_bf16(v[4], v[5]), pack2_bf16(v[6], v[7]));
#pragma unroll
  for (int i = 0; i < N; ++i) t[i] = __builtin_bit_cast(bf16x8, u[i]);
}
// 8 codes -> the 8 bf16 values they stand for.
__device__ __forceinline__ bf16x8 bf8(uint32_t lo, uint32_t hi, float s) {
  const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, s, false), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, s, true);
  const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, s, false), d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, s, true);
  return bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}
// The bytes of a word whose codes stand for no finite value, as 0xff each: low seven bits from 0x80 less a byte of `step` on.  kNan:
// NaN; kInfinite: codes from 256 on as well, which the largest scale, 2^120, takes past 32 bits' range.
constexpr uint32_t kNan = 0x01010101u, kInfinite = 0x08080808u;
__device__ __forceinline__ uint32_t odd_bytes(uint32_t c, uint32_t step) {
  const uint32_t x = (c & 0x7f7f7f7fu) + step;
  return ((x & 0x80808080u) >> 7) * 255u;
}
__device__ __forceinline__ uint32_t negative_bytes(uint32_t c) { return ((c & 0x80808080u) >> 7) * 255u; }
// The bytes of positions below `left` in the two words of eight positions.
__device__ __forceinline__ void cut(uint32_t& lo, uint32_t& hi, int left) {
  lo &= left >= 4 ? ~0u : left <= 0 ? 0u : (1u << 8 * left) - 1;
  hi &= left >= 8 ? ~0u : left <= 4 ? 0u : (1u << 8 * (left - 4)) - 1;
}

// a / b of numbers below 2^21: (a + 1/2) / b is 1 / (2 b) off a whole number at least, more than its roundings (a division
// of integers is forty instructions)
__device__ __forceinline__ int quotient(int a, int b) { return (int)((a + 0.5f) * __builtin_amdgcn_rcpf((float)b)); }
// Codes and scales of two pages; there: bit t set where page t's number is good and it holds a position that a row sees.
struct Step {
  uint4 k[2], v[2];
  uint32_t s[2], there;
};
struct State {
  float m, l;
  floatx4 o[4];
};
}  // namespace

// Positions p0 .. p0 + 31; `lim`: this lane's column sees positions below it; all columns see those below `low`, none
// those from `top` on.
template <int QT, int PT>
__device__ __forceinline__ void kv8_step(Step& c, int p0, int lim, int low, int top, const bf16x8 (&qt)[2][QT], State& st) {
  const int kg = (threadIdx.x & 63) >> 4;
  floatx4 s[2];
#pragma unroll
  for (int t = 0; t < 2; ++t) {
    const float sc = scale_f(c.s[t] & 255);
    const bf16x8 k0 = bf8(c.k[t].x, c.k[t].y, sc), k1 = bf8(c.k[t].z, c.k[t].w, sc);
    s[t] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = QT - 1; i >= 0; --i) s[t] = mfma16(k1, qt[1][i], mfma16(k0, qt[0][i], s[t]));
  }
  uint32_t vw[4][2] = {{c.v[0].x, c.v[0].y}, {c.v[0].z, c.v[0].w}, {c.v[1].x, c.v[1].y}, {c.v[1].z, c.v[1].w}};
  const uint32_t vs = (kg >> 1 ? c.s[1] : c.s[0]) >> 8;
  const bool masked = p0 + 32 > low || c.there != 3;
  uint32_t odd = 0, hidden = 0;  // hidden: bit 4 t + i
  const uint32_t step = vs == 247 ? kInfinite : kNan;
  if (masked) {  // uniform
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (p0 + 16 * t + 4 * kg + i >= lim || !(c.there >> t & 1)) {
          s[t][i] = -INFINITY;
          hidden |= 1u << (4 * t + i);
        }
    const int left = c.there >> (kg >> 1) & 1 ? top - p0 - 8 * kg : 0;
#pragma unroll
    for (int dt = 0; dt < 4; ++dt) {
      cut(vw[dt][0], vw[dt][1], left);
      odd |= odd_bytes(vw[dt][0], step) | odd_bytes(vw[dt][1], step);
    }
  }
  float mx = -INFINITY;
#pragma unroll
  for (int t = 0; t < 2; ++t)
#pragma unroll
    for (int i = 0; i < 4; ++i) mx = fmaxf(mx, s[t][i]);
  const float above = (c.s[0] | c.s[1]) & 0x8000u ? 0.f : kRaise;  // a value scale of 2 or more
  if (__builtin_amdgcn_ballot_w64(mx - st.m > above)) {
    const float top = swap_max(mx), m = top - st.m > above ? top : st.m, f = exp_to(st.m, no_inf(m));  // 0 at first
    st.m = m;
    st.l *= f;
#pragma unroll
    for (int dt = 0; dt < 4; ++dt) st.o[dt] *= f;
  }
  const float base = no_inf(st.m);
  float l = 0.f;
#pragma unroll
  for (int t = 0; t < 2; ++t)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      s[t][i] = exp_to(s[t][i], base);
      l += s[t][i];
    }
  st.l += l;
  auto operand = [&](const floatx4 (&x)[2], float* pb) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const auto u = __builtin_amdgcn_permlane32_swap(__float_as_uint(x[0][i]), __float_as_uint(x[1][i]), false, false);
      const auto y = __builtin_amdgcn_permlane16_swap(u[0], u[1], false, false);
      pb[i] = __uint_as_float(y[0]);
      pb[4 + i] = __uint_as_float(y[1]);
    }
  };
  // A NaN or an infinity times a probability of 0 would reach the columns that do not see it: such values leave
  // the product and are counted, for the columns that do, by two products of ones.
  if (__builtin_amdgcn_ballot_w64(odd != 0)) {
    floatx4 sees[2];
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int i = 0; i < 4; ++i) sees[t][i] = hidden >> (4 * t + i) & 1 ? 0.f : 1.f;
    float pb[8];
    operand(sees, pb);
    bf16x8 one[1];
    split_terms<1>(pb, one);
#pragma unroll
    for (int dt = 0; dt < 4; ++dt) {
      uint32_t up[2], down[2];
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const uint32_t c = vw[dt][j], any = odd_bytes(c, step), nan = odd_bytes(c, kNan), neg = negative_bytes(c);
        up[j] = (nan | (any & ~neg)) & 0x38383838u;  // 0x38: the code of 1
        down[j] = (nan | (any & neg)) & 0x38383838u;
        vw[dt][j] &= ~any;
      }
      const floatx4 z = mfma16(bf8(up[0], up[1], 1.f), one[0], floatx4{0.f, 0.f, 0.f, 0.f});
      const floatx4 y = mfma16(bf8(down[0], down[1], 1.f), one[0], floatx4{0.f, 0.f, 0.f, 0.f});
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if (z[i] > 0.f) st.o[dt][i] += INFINITY;
        if (y[i] > 0.f) st.o[dt][i] -= INFINITY;
      }
    }
  }
  float pb[8];
  operand(s, pb);
  bf16x8 pt[PT];
  split_terms<PT>(pb, pt);
#pragma unroll
  for (int dt = 0; dt < 4; ++dt) {
    const bf16x8 x = bf8(vw[dt][0], vw[dt][1], scale_f(vs));
#pragma unroll
    for (int i = PT - 1; i >= 0; --i) st.o[dt] = mfma16(x, pt[i], st.o[dt]);
  }
}

// Position of request r's first row and its rows, as far as they matter: positions far outside the tables count as the
// nearest that behave alike.
__device__ __forceinline__ void kv8_rows(const Kv8AttendArgs& a, int r, int& pos, int& count) {
  count = a.counts ? min(max(a.counts[r], 0), a.rows) : a.rows;
  pos = min(max(a.positions[r], -(1 << 20)), 16 * a.max_pages);
}

template <typename T, int NW>  // four waves a SIMD: 128 registers, where fp32 with eight waves took 129 and a block less (52 us for 60: 64 x 5 rows below)
__global__ void __launch_bounds__(NW * 64, 4) k_kv8_attend(Kv8AttendArgs a) {
  // bf16 terms of a query value and of a probability: as many as hold it exactly.  Two terms of a probability, 2^-16 of it, would
  // save a bf16 call 2% (96 x 9 rows at 0 to 438, 22.4 us a replay for 22.9) to 9% (185 x 29, 177 for 193)
  constexpr int QT = sizeof(T) == 2 ? 1 : 3, PT = 3;
  __shared__ float wm[NW][16], wl[NW][16];
  __shared__ alignas(16) float wo[NW][16][68];
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), n = lane & 15, kg = lane >> 4;
  const int cols = a.rows * a.group, cap = 16 * a.max_pages, tiles = (cols + 15) >> 4;
  int chunk = quotient(blockIdx.x, a.c.n_head), head = blockIdx.x - chunk * a.c.n_head, r = blockIdx.y, tile = blockIdx.z;
  if (a.units) {  // eight (request, chunk, head)s' first tiles, their second ones, ...
    const int eight = quotient(blockIdx.x, 8 * tiles), rest = blockIdx.x - 8 * tiles * eight, unit = 8 * eight + (rest & 7);
    if (unit >= a.units) return;
    tile = rest >> 3;
    const int part = quotient(unit, a.c.n_head);
    head = unit - part * a.c.n_head;
    r = quotient(part, a.nchunk);
    chunk = part - r * a.nchunk;
  }
  const int c0 = tile * 16;
  const int* table = a.tables + r * a.ts;
  // Before the request's position is known: the query, and the page numbers of the wave's first 32 steps (two a step) where
  // the positions are not split.
  const int col = c0 + n, i = quotient(col, a.group);
  int ahead = table[min(2 * (w + (lane >> 1) * NW) + (lane & 1), a.max_pages - 1)];
  const T* q = reinterpret_cast<const T*>(a.q) + r * a.sr + (long long)min(i, a.rows - 1) * a.si + (head * a.group + col - i * a.group) * a.sh + 16 * kg;
  float x[16];
  if (a.vec) {
    ld8(q, x);
    ld8(q + 8, x + 8);
  } else {
#pragma unroll
    for (int j = 0; j < 16; ++j) x[j] = to_f(q[j]);
  }
  int pos, count;
  kv8_rows(a, r, pos, count);
  // columns of rows from `count` on, and of rows that see nothing, run along unmasked and are written as zeros
  const int i0 = quotient(c0, a.group), i1 = min(quotient(min(cols, c0 + 16) - 1, a.group), count - 1);  // rows of this tile
  const bool live = col < cols && i < count && pos + i >= 0;
  const int top = i0 < count ? min(max(pos + i1 + 1, 0), cap) : 0;
  const int low = min(max(pos + i0, 0) + 1, top), lim = live ? min(pos + i + 1, cap) : cap;
  const int groups = (top + 31) / 32, each = a.nchunk == 1 ? groups : (int)((groups + a.nchunk - 1u) / (unsigned)a.nchunk);
  const int end = min((chunk + 1) * each, groups), g0 = chunk * each + w;
  State st;
  st.m = -INFINITY;
  st.l = 0.f;
#pragma unroll
  for (int dt = 0; dt < 4; ++dt) st.o[dt] = floatx4{0.f, 0.f, 0.f, 0.f};
  const int steps = g0 < end ? (end - g0 + NW - 1) / NW : 0;
  auto load = [&](int i, Step& s) {  // the wave's step i, or its last again
    if ((i & 31) == 0 && i < steps && (i > 0 || a.nchunk > 1))
      ahead = table[min(2 * (g0 + (i + (lane >> 1)) * NW) + (lane & 1), a.max_pages - 1)];
    i = min(i, steps - 1);
    int p[2];
    s.there = 0;
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      p[t] = __builtin_amdgcn_readlane(ahead, 2 * (i & 31) + t);
      // nothing need ever have been stored in the page behind the last position: its scales may be anything
      if (p[t] >= 0 && p[t] < a.c.n_pages && 32 * (g0 + i * NW) + 16 * t < top) s.there |= 1u << t;
      else p[t] = 0;
    }
    const uint8_t* in[2];
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      in[t] = a.c.base + p[t] * a.c.page + (size_t)head * kKv8Head;
      s.k[t] = *reinterpret_cast<const uint4*>(in[t] + 16 * lane);
      s.s[t] = *reinterpret_cast<const uint16_t*>(a.c.base + p[t] * a.c.page + (size_t)a.c.n_head * kKv8Head + 2 * head);
      if (!(s.there >> t & 1)) s.s[t] = 0x7f7f;  // another page's scales may be anything: 1
    }
    const uint8_t* values = (kg >> 1 ? in[1] : in[0]) + kKv8Values + 32 * (lane & 31);
    s.v[0] = *reinterpret_cast<const uint4*>(values);
    s.v[1] = *reinterpret_cast<const uint4*>(values + 16);
  };
  if (steps > 0) {
    Step A, B;
    load(0, A);
    bf16x8 qt[2][QT];
    split_terms<QT>(x, qt[0]);
    split_terms<QT>(x + 8, qt[1]);
    for (int i = 0;;) {
      load(i + 1, B);
      kv8_step<QT, PT>(A, 32 * (g0 + i * NW), lim, low, top, qt, st);
      if (++i >= steps) break;
      load(i + 1, A);
      kv8_step<QT, PT>(B, 32 * (g0 + i * NW), lim, low, top, qt, st);
      if (++i >= steps) break;
    }
  }
  const float l = swap_sum(st.l);
  if (lane < 16) {
    wm[w][lane] = st.m;
    wl[w][lane] = l;
  }
  // value tile dt holds dims 4 m + dt: o[dt][i] of the lane is dim 16 kg + 4 i + dt
#pragma unroll
  for (int e = 0; e < 4; ++e)
    *reinterpret_cast<floatx4*>(&wo[w][n][16 * kg + 4 * e]) = floatx4{st.o[0][e], st.o[1][e], st.o[2][e], st.o[3][e]};
  __syncthreads();
  const int nc = min(16, cols - c0);
  for (int t = threadIdx.x; t < nc * 16; t += NW * 64) {
    const int c = t >> 4, d = 4 * (t & 15), ci = quotient(c0 + c, a.group);
    float M = wm[0][c], L = 0.f;
    floatx4 O = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int j = 1; j < NW; ++j) M = fmaxf(M, wm[j][c]);
    const float base = no_inf(M);
#pragma unroll
    for (int j = 0; j < NW; ++j) {
      const float f = exp_to(wm[j][c], base);  // 0 for a wave of no positions
      L = fmaf(f, wl[j][c], L);
      O += f * *reinterpret_cast<const floatx4*>(&wo[j][c][d]);
    }
    if (a.nchunk == 1) {
      const float inv = ci < count && pos + ci >= 0 && L != 0.f ? 1.f / L : 0.f;
      const float o[4] = {inv == 0.f ? 0.f : O[0] * inv, inv == 0.f ? 0.f : O[1] * inv, inv == 0.f ? 0.f : O[2] * inv, inv == 0.f ? 0.f : O[3] * inv};
      st4(reinterpret_cast<T*>(a.out) + ((((size_t)r * a.rows + ci) * a.c.n_head + head) * a.group + c0 + c - ci * a.group) * kHeadDim + d, o);
    } else {
      float* rec = a.part + ((((size_t)r * tiles + tile) * a.c.n_head + head) * a.nchunk + chunk) * kRecord;
      *reinterpret_cast<floatx4*>(rec + 32 + c * 64 + d) = O;
      if (d == 0) {
        rec[c] = M;
        rec[16 + c] = L;
      }
    }
  }
}

// Joins the chunks of one column: 16 threads (4 dims each) take every sixteenth chunk and meet in LDS.
template <typename T>
__global__ void __launch_bounds__(256) k_kv8_merge(Kv8AttendArgs a) {
  __shared__ float wm[16], wl[16];
  __shared__ alignas(16) float wo[16][64];
  const int cols = a.rows * a.group, tiles = (cols + 15) >> 4;
  const int head = blockIdx.x, r = blockIdx.y, c = blockIdx.z, tile = c >> 4, i = c & 15;
  const int t = threadIdx.x, q = t >> 4, d = 4 * (t & 15);
  const float* rec = a.part + (((size_t)r * tiles + tile) * a.c.n_head + head) * a.nchunk * kRecord;
  float M = -INFINITY, L = 0.f;
  floatx4 O = {0.f, 0.f, 0.f, 0.f};
  for (int k = q; k < a.nchunk; k += 16) {
    const float* p = rec + (size_t)k * kRecord;
    const float m = p[i], Mn = fmaxf(M, m), base = no_inf(Mn), f0 = exp_to(M, base), f = exp_to(m, base);
    M = Mn;
    L = fmaf(f, p[16 + i], L * f0);
    O = O * f0 + f * *reinterpret_cast<const floatx4*>(p + 32 + i * 64 + d);
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
    int pos, count;
    kv8_rows(a, r, pos, count);
    const int ci = c / a.group;
    const bool some = ci < count && pos + ci >= 0 && l != 0.f;
    reinterpret_cast<T*>(a.out)[((((size_t)r * a.rows + ci) * a.c.n_head + head) * a.group + c % a.group) * kHeadDim + t] =
        from_f<T>(some ? o / l : 0.f);
  }
}

// Waves of a block: fewer where the positions are few and the blocks many, whose start and end then weigh more than a wave's
// steps.  The table's width stands for the positions, which are not known here: of contexts far below it a call takes up to a
// fifth more (64 rows at 0 to 500, 32 heads over 8, table of 2,048 pages 19.4 us, of 32 17.3).  us a call of a graph of one, replayed
// again and again (some 5 us more than among a stream's other calls), bf16, probabilities in two terms:
//   one wave / four   256 requests of one row at 0 to 64, 20 heads, 15.6 / 22.4, of nine at 0 to 100, 32 heads over 8, 22.7 / 30.3
//   four / eight      20 heads: 96 of nine rows at 0 to 438 21.7 / 24.5, 256 of one at 0 to 447 36 / 47; 32 over 8: 185 of 29 at 0 to
//                     2,069 175 / 201; but 64 of one at 4,000, 20 heads, 127 / 118, 256 of one at 0 to 4,000 252 / 239
static int kv8_waves(long long blocks, int max_pages) {
  if (max_pages <= 8 && blocks > 1024) return 1;
  return (max_pages <= 64 && blocks > 256) || (max_pages <= 192 && blocks >= 3584) ? 4 : 8;
}
// Chunks of the positions: towards four blocks a compute unit, each of two steps of every wave at least.
static int kv8_chunks(int n, int rows, int group, int n_head, int max_pages) {
  const long long blocks = (long long)n * n_head * ((rows * group + 15) / 16), groups = (max_pages + 1) / 2;
  return (int)std::max<long long>(1, std::min<long long>(1024 / blocks, groups / 16));
}
size_t kv8_workspace(int n, int rows, int group, int n_head, int max_pages) {
  const int nc = kv8_chunks(n, rows, group, n_head, max_pages);
  return nc == 1 ? 0 : (size_t)n * n_head * ((rows * group + 15) / 16) * nc * kRecord * 4;
}

template <typename T>
static void attend_launch(Kv8AttendArgs& a, hipStream_t st) {
  // The tiles of the same keys and values one behind the other on one XCD (every eighth block), the later ones then read them
  // from its L2.  us a replayed call, probabilities in two terms, tiles by grid z / so: four x nine rows from 65,536 on, 32 heads over 8, 217 / 143; one x 17
  // at 130,000, 20 heads, 124 / 91; 64 x five at 0 to 4,000, 32 over 8, 59 / 51; but 64 x 17 at 0 to 600, 20 heads, 30.6 / 32.2.
  const int cols = a.rows * a.group, tiles = (cols + 15) / 16;
  const long long units = (long long)a.n * a.nchunk * a.c.n_head, x = (units + 7) / 8 * 8 * tiles;
  if (tiles > 1 && x <= 1 << 20) a.units = (int)units;
  const dim3 grid = a.units ? dim3((unsigned)x) : dim3(a.c.n_head * a.nchunk, a.n, tiles);
  const int waves = kv8_waves((long long)grid.x * grid.y * grid.z, a.max_pages);
  if (waves == 1) k_kv8_attend<T, 1><<<grid, 64, 0, st>>>(a);
  else if (waves == 4) k_kv8_attend<T, 4><<<grid, 256, 0, st>>>(a);
  else k_kv8_attend<T, 8><<<grid, 512, 0, st>>>(a);
  if (a.nchunk > 1) k_kv8_merge<T><<<dim3(a.c.n_head, a.n, cols), 256, 0, st>>>(a);
}
void kv8_attend(const Kv8AttendArgs& a0, hipStream_t st) {
  Kv8AttendArgs a = a0;
  a.nchunk = kv8_chunks(a.n, a.rows, a.group, a.c.n_head, a.max_pages);
  if (a.bf16_q) attend_launch<bf16>(a, st);
  else attend_launch<float>(a, st);
}

}  // namespace wf
