// Causal attention of packed prompts.
//
// Rows of all sequences lie one after the other; row t sees the rows of its own sequence up to
// itself, an interval [lo, t] of the packed rows.  A block takes 32 consecutive rows of one
// head, whichever sequences they belong to, and the keys from its first row's lo to its last
// row: short sequences share a block, and neither lengths nor their tiles have to be known on
// the host.  Scores outside a row's interval are replaced by -inf.
#include <algorithm>

#include "wf_operand.h"
#include "wf_ops.h"

namespace wf {

namespace {
constexpr float kScale = 0.125f * 1.44269504088896340736f;  // exp(s / 8) = 2^(kScale s)

__device__ __forceinline__ float pair_max(float v) {  // over the two half-waves
  const auto x = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return fmaxf(__uint_as_float(x[0]), __uint_as_float(x[1]));
}
__device__ __forceinline__ float pair_sum(float v) {
  const auto x = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return __uint_as_float(x[0]) + __uint_as_float(x[1]);
}
__device__ __forceinline__ bool finite(float v) { return (__float_as_uint(v) & 0x7f800000u) != 0x7f800000u; }

// Borders near a block's rows, in LDS: `base` is the index of the last border at or before the block's first row (0: before
// all), the window holds `size` of them from there on.
constexpr int kWindow = 512;
struct Borders {
  int base, size, begin, end;  // begin, end: the rows of all sequences
};
// The block's 256 threads narrow the borders 256-fold a round (none up to 511 sequences) and load the window:
// one round trip to memory, where a search of 96 borders by every row takes seven.
__device__ __forceinline__ Borders borders_near(const int* starts, int n, int q0, int* window, int* counts) {
  int base = 0, size = n + 1;
  while (size > kWindow) {
    const int stride = (size + 255) / 256, i = threadIdx.x * stride;
    const bool before = i < size && starts[base + i] <= q0;
    const int c = __popcll(__builtin_amdgcn_ballot_w64(before));
    if ((threadIdx.x & 63) == 0) counts[threadIdx.x >> 6] = c;
    __syncthreads();
    const int at = max(counts[0] + counts[1] + counts[2] + counts[3] - 1, 0) * stride;
    __syncthreads();
    size = min(stride, size - at);
    base += at;
  }
  base = min(base, n);
  size = min(kWindow, n + 1 - base);
  for (int i = threadIdx.x; i < size; i += 256) window[i] = starts[base + i];
  const Borders b{base, size, starts[0], starts[n]};
  __syncthreads();
  return b;
}
// First key of row t: the largest border <= t, where t lies in a sequence; t + 1 (no key) elsewhere.
__device__ __forceinline__ int first_key(const int* starts, int n, const int* window, const Borders& b, int t) {
  if (t < b.begin || t >= b.end) return t + 1;
  const bool near = b.base + b.size > n || window[b.size - 1] > t;
  int lo = 0, hi = near ? b.size - 1 : n - b.base;  // the border of lo is <= t, that of hi > t
  while (hi - lo > 1) {
    const int m = (lo + hi) >> 1;
    if ((near ? window[m] : starts[b.base + m]) <= t) lo = m;
    else hi = m;
  }
  return min(max(near ? window[lo] : starts[b.base + lo], 0), t + 1);
}

// N consecutive elements of a row.
template <int N>
__device__ __forceinline__ void ld(const float* p, int vec, float* o) {
  if (vec) {
#pragma unroll
    for (int j = 0; j < N; j += 4) *reinterpret_cast<floatx4*>(o + j) = *reinterpret_cast<const floatx4*>(p + j);
  } else {
#pragma unroll
    for (int j = 0; j < N; ++j) o[j] = p[j];
  }
}
template <int N>
__device__ __forceinline__ void ld(const bf16* p, int vec, float* o) {
  if (vec) {
    if constexpr (N == 8) {
      ld8(p, o);
    } else {
      const uint2 v = *reinterpret_cast<const uint2*>(p);
      o[0] = __uint_as_float(v.x << 16);
      o[1] = __uint_as_float(v.x & 0xffff0000u);
      o[2] = __uint_as_float(v.y << 16);
      o[3] = __uint_as_float(v.y & 0xffff0000u);
    }
  } else {
#pragma unroll
    for (int j = 0; j < N; ++j) o[j] = to_f(p[j]);
  }
}
__device__ __forceinline__ floatx16 mfma32(bf16x8 a, bf16x8 b, floatx16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }

// Eight values as N bf16 terms: three hold an fp32 value exactly (the first its top eight bits, the others what
// is left, rounded), one a bf16 value.
template <int N>
__device__ __forceinline__ void terms8(const float* v, bf16x8 (&t)[N]) {
  uint32_t h[4], m[4], l[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const float a = v[2 * e], b = v[2 * e + 1];
    if constexpr (N == 1) {
      h[e] = pack2_bf16(a, b);
    } else {
      h[e] = pack2_hi(a, b);
      const float ra = a - __uint_as_float(__float_as_uint(a) & 0xffff0000u), rb = b - __uint_as_float(__float_as_uint(b) & 0xffff0000u);
      m[e] = pack2_bf16(ra, rb);
      l[e] = pack2_bf16(ra - __uint_as_float(m[e] << 16), rb - __uint_as_float(m[e] & 0xffff0000u));
    }
  }
  t[0] = __builtin_bit_cast(bf16x8, make_uint4(h[0], h[1], h[2], h[3]));
  if constexpr (N == 3) {
    t[1] = __builtin_bit_cast(bf16x8, make_uint4(m[0], m[1], m[2], m[3]));
    t[2] = __builtin_bit_cast(bf16x8, make_uint4(l[0], l[1], l[2], l[3]));
  }
}
// The product of two such sums, its smallest parts first; what three terms leave out is below 2^-22 of it.
template <int N>
__device__ __forceinline__ floatx16 product(const bf16x8 (&a)[N], const bf16x8 (&b)[N], floatx16 c) {
  if constexpr (N == 3) {
    c = mfma32(a[2], b[0], c);
    c = mfma32(a[0], b[2], c);
    c = mfma32(a[1], b[1], c);
    c = mfma32(a[1], b[0], c);
    c = mfma32(a[0], b[1], c);
  }
  return mfma32(a[0], b[0], c);
}
}  // namespace

// Block: (32 rows, head), four waves that take every fourth tile of 32 keys, each on its own from memory
// to registers, and join their maxima, sums and outputs in LDS at the end.  fp32 values enter the products as three
// bf16 terms, six products of the 2,500 TFLOP/s kind for one of the 157 of v_mfma_f32_32x32x2_f32.
//   S^T = K q^T  a lane gets keys 8 (v / 4) + 4 (lane / 32) + v % 4 of row lane % 32
//   O^T += V^T P^T  the half-waves' eight values of an instruction are taken as those keys, so the probabilities
//                are the operand as they are, and a lane's values are V[those keys][lane % 32 + 32 d]
// The next tile's keys are loaded once this one's are multiplied, the values likewise.
template <typename T>
__global__ void __launch_bounds__(256, 2) k_prompt32(PromptArgs a, int tiles, int per) {
  constexpr int N = sizeof(T) == 4 ? 3 : 1;
  __shared__ float wm[4][32], wl[4][32], wo[4][32][68];
  const int at = (blockIdx.x & 7) * per + (blockIdx.x >> 3);  // as in k_prompt16
  if (at >= tiles * a.heads) return;
  const int head = at / tiles, q0 = (tiles - 1 - at % tiles) * 32;
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, lr = lane & 31, lk = lane >> 5;
  const int row = min(q0 + lr, a.tokens - 1);
  const T* Q = reinterpret_cast<const T*>(a.q) + row * a.qt + head * a.qh + 8 * lk;
  float q[4][8];
#pragma unroll
  for (int s = 0; s < 4; ++s) ld<8>(Q + 16 * s, a.vec, q[s]);
  int* window = reinterpret_cast<int*>(wo);
  const Borders near = borders_near(a.starts, a.n, q0, window, reinterpret_cast<int*>(wm));
  const int lo = first_key(a.starts, a.n, window, near, row), hi = lo > row ? lo : row + 1;  // keys [lo, hi)
  // the keys that any of the rows sees, and those that all see
  int k0 = hi > lo ? lo : a.tokens, k1 = hi > lo ? hi : 0, f0 = lo, f1 = hi;
#pragma unroll
  for (int m = 1; m < 32; m <<= 1) {
    k0 = min(k0, __shfl_xor(k0, m));
    k1 = max(k1, __shfl_xor(k1, m));
    f0 = max(f0, __shfl_xor(f0, m));
    f1 = min(f1, __shfl_xor(f1, m));
  }
  k0 = __builtin_amdgcn_readfirstlane(k0);
  k1 = __builtin_amdgcn_readfirstlane(k1);
  f0 = __builtin_amdgcn_readfirstlane(f0);
  f1 = __builtin_amdgcn_readfirstlane(f1);
  const T* K = reinterpret_cast<const T*>(a.k) + (head / a.group) * a.kh + 8 * lk;
  const T* V = reinterpret_cast<const T*>(a.v) + (head / a.group) * a.vh + lr;
  float kx[4][8], vx[2][2][8];  // a tile: keys' dims 16 s + 8 lk .. + 7 of key lr; values [dim half][sixteen keys]
  auto load_keys = [&](int kt) {
    const T* p = K + min(kt + lr, a.tokens - 1) * a.kt;
#pragma unroll
    for (int s = 0; s < 4; ++s) ld<8>(p + 16 * s, a.vec, kx[s]);
  };
  auto load_values = [&](int kt) {
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const T* p = V + min(kt + 8 * (i >> 2) + 4 * lk + (i & 3), a.tokens - 1) * a.vt;
      vx[0][i >> 3][i & 7] = to_f(p[0]);
      vx[1][i >> 3][i & 7] = to_f(p[32]);
    }
  };
  int kt = k0 + 32 * w;
  if (kt < k1) {
    load_keys(kt);
    load_values(kt);
  }
  bf16x8 qt[4][N];
#pragma unroll
  for (int s = 0; s < 4; ++s) terms8<N>(q[s], qt[s]);
  float m = -INFINITY, l = 0.f;
  floatx16 o[2];
#pragma unroll
  for (int d = 0; d < 2; ++d)
#pragma unroll
    for (int v = 0; v < 16; ++v) o[d][v] = 0.f;
  for (; kt < k1; kt += 128) {
    floatx16 s;
#pragma unroll
    for (int v = 0; v < 16; ++v) s[v] = 0.f;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      bf16x8 t[N];
      terms8<N>(kx[i], t);
      s = product<N>(t, qt[i], s);
    }
    if (kt + 128 < k1) load_keys(kt + 128);
    const bool masked = kt < f0 || kt + 32 > f1;  // uniform: some row does not see some key
    uint32_t out = 0;                             // bit v: the row does not see the key
    if (masked) {
#pragma unroll
      for (int v = 0; v < 16; ++v) {
        const int key = kt + 8 * (v >> 2) + 4 * lk + (v & 3);
        const bool hidden = key < lo || key >= hi;
        s[v] = hidden ? -INFINITY : s[v];
        out |= hidden ? 1u << v : 0u;
      }
    }
    float mx = -INFINITY;
#pragma unroll
    for (int v = 0; v < 16; ++v) mx = fmaxf(mx, s[v]);
    const float mn = fmaxf(m, pair_max(mx)), base = mn == -INFINITY ? 0.f : mn;
    const float f = __builtin_amdgcn_exp2f((m - base) * kScale);
    m = mn;
    l *= f;
#pragma unroll
    for (int d = 0; d < 2; ++d)
#pragma unroll
      for (int v = 0; v < 16; ++v) o[d][v] *= f;
    float p[2][8];
#pragma unroll
    for (int v = 0; v < 16; ++v) {
      p[v >> 3][v & 7] = __builtin_amdgcn_exp2f((s[v] - base) * kScale);
      l += p[v >> 3][v & 7];
    }
    // A NaN or an infinity times a probability of 0 would reach the rows that do not see it (and an infinity in terms is
    // NaN): such values leave the product and are counted, for the rows that do, by two products of ones.
    float odd = 0.f;
#pragma unroll
    for (int i = 0; i < 32; ++i) odd = fmaf(vx[i >> 4][(i >> 3) & 1][i & 7], 0.f, odd);
    if (__builtin_amdgcn_ballot_w64(odd != 0.f)) {
#pragma unroll
      for (int d = 0; d < 2; ++d) {
        floatx16 up, down;
#pragma unroll
        for (int v = 0; v < 16; ++v) up[v] = down[v] = 0.f;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          bf16x8 plus, minus, sees;
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const float y = vx[d][i][e];
            plus[e] = (__bf16)(y != y || y == INFINITY ? 1.f : 0.f);
            minus[e] = (__bf16)(y != y || y == -INFINITY ? 1.f : 0.f);
            sees[e] = (__bf16)(out >> (8 * i + e) & 1 ? 0.f : 1.f);
            vx[d][i][e] = finite(y) ? y : 0.f;
          }
          up = mfma32(plus, sees, up);
          down = mfma32(minus, sees, down);
        }
#pragma unroll
        for (int v = 0; v < 16; ++v) {
          if (up[v] > 0.f) o[d][v] += INFINITY;
          if (down[v] > 0.f) o[d][v] -= INFINITY;
        }
      }
    }
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      bf16x8 pt[N];
      terms8<N>(p[i], pt);
#pragma unroll
      for (int d = 0; d < 2; ++d) {
        bf16x8 t[N];
        terms8<N>(vx[d][i], t);
        o[d] = product<N>(t, pt, o[d]);
      }
    }
    if (kt + 128 < k1) load_values(kt + 128);
  }
  l = pair_sum(l);
  __syncthreads();  // the window lies where the outputs go
  if (lane < 32) {
    wm[w][lr] = m;
    wl[w][lr] = l;
  }
  // lane: row lr, dims 32 d + 8 (v / 4) + 4 lk + v % 4
#pragma unroll
  for (int d = 0; d < 2; ++d)
#pragma unroll
    for (int g = 0; g < 4; ++g)
      *reinterpret_cast<floatx4*>(&wo[w][lr][32 * d + 8 * g + 4 * lk]) =
          floatx4{o[d][4 * g], o[d][4 * g + 1], o[d][4 * g + 2], o[d][4 * g + 3]};
  __syncthreads();
#pragma unroll
  for (int t = threadIdx.x; t < 32 * 64; t += 256) {
    const int i = t >> 6, d = t & 63, r = q0 + i;
    if (r >= a.tokens) break;
    float M = wm[0][i], L = 0.f, O = 0.f;
#pragma unroll
    for (int j = 1; j < 4; ++j) M = fmaxf(M, wm[j][i]);
    const float base = M == -INFINITY ? 0.f : M;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const float f = __builtin_amdgcn_exp2f((wm[j][i] - base) * kScale);
      L = fmaf(f, wl[j][i], L);
      O = fmaf(f, wo[j][i][d], O);
    }
    if (!a.clear && (r < near.begin || r >= near.end)) continue;
    reinterpret_cast<T*>(a.out)[((size_t)r * a.heads + head) * kHeadDim + d] = from_f<T>(L == 0.f ? 0.f : O / L);
  }
}

// ---------------------------------------------------------------- bf16
// Block: (128 NQ rows, head), four waves of 32 NQ rows.  Keys and values stream through three LDS
// stages in tiles of 64 rows, copied straight from memory (global_load_lds_dwordx4) two tiles
// ahead of their use.  Per 32 keys and 32 rows a wave forms S^T = K q^T on
// v_mfma_f32_32x32x16_bf16, so a lane holds 16 keys of one row (keys 8 (v / 4) + 4 (lane / 32) +
// v % 4): reference and sum are per lane (one swap of half-waves joins a row's two lanes) and
// the probabilities, rounded to bf16 in place, are the B operand of O^T += V^T P^T if the half-waves'
// eight values of an instruction are taken as those keys.  The A operand then is, for a dim, keys 4
// and 4 together, what ds_read_b64_tr_b16 makes of rows as they lie in memory.  The sum is taken of
// the rounded probabilities.
namespace {
typedef __attribute__((address_space(3))) void lds_void;
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
constexpr int kTile = 64, kStage = 1024;  // keys of a tile; 16-byte chunks of a stage
// A stage: chunk c (8 dims) of key r at 8 r + (c ^ (r & 7)), then the values in the same way.
constexpr int kWaitNext = (4 & 15) | (7 << 4);  // vmcnt <= 4: the copies of the tile behind the next; lgkmcnt 0
constexpr int kWaitAll = (0 & 15) | (7 << 4) | (15 << 8);

__device__ __forceinline__ float dot2(uint32_t a, uint32_t b, float c) {
  return __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16v2, a), __builtin_bit_cast(bf16v2, b), c, false);
}
// two bf16 values, zero where they are not finite
__device__ __forceinline__ uint32_t finite2(uint32_t x) {
  return ((x & 0x7f80u) == 0x7f80u ? 0u : x & 0xffffu) | ((x & 0x7f800000u) == 0x7f800000u ? 0u : x & 0xffff0000u);
}
}  // namespace

// Keys and values k0 .. k0 + 63 (rows past the last are the last) into a stage.
__device__ __forceinline__ void prompt_copy(const bf16* K, const bf16* V, const PromptArgs& a, int k0, uint4* stage) {
  const int w = threadIdx.x >> 6, lane = threadIdx.x & 63;
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    const int slot = (w * 2 + j) * 64 + lane, r = slot >> 3, ch = (slot & 7) ^ (r & 7);
    __builtin_amdgcn_global_load_lds((const void*)(K + min(k0 + r, a.tokens - 1) * a.kt + 8 * ch), (lds_void*)&stage[(w * 2 + j) * 64], 16, 0, 0);
  }
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    const int slot = (w * 2 + j) * 64 + lane, r = slot >> 3, ch = (slot & 7) ^ (r & 7);
    __builtin_amdgcn_global_load_lds((const void*)(V + min(k0 + r, a.tokens - 1) * a.vt + 8 * ch), (lds_void*)&stage[512 + (w * 2 + j) * 64], 16, 0, 0);
  }
}

template <int NQ>
__global__ void __launch_bounds__(256, 2) k_prompt16(PromptArgs a, int tiles, int per) {
  __shared__ uint4 st0[kStage], st1[kStage], st2[kStage];
  // The blocks that one XCD gets (every eighth) are neighbours: one head's, whose keys and values its L2 then
  // holds, those with the most keys first.
  const int at = (blockIdx.x & 7) * per + (blockIdx.x >> 3);
  if (at >= tiles * a.heads || (int)(blockIdx.x >> 3) >= per) return;
  const int head = at / tiles, q0 = (tiles - 1 - at % tiles) * 128 * NQ;
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, lr = lane & 31, lk = lane >> 5;
  const bf16* Q = reinterpret_cast<const bf16*>(a.q) + head * a.qh;
  const bf16* K = reinterpret_cast<const bf16*>(a.k) + (head / a.group) * a.kh;
  const bf16* V = reinterpret_cast<const bf16*>(a.v) + (head / a.group) * a.vh;
  __shared__ int window[kWindow], first[4], last[4], from[4], to[4], odd[4];  // odd: the last tile of a stage that held a NaN or an infinity
  const Borders near = borders_near(a.starts, a.n, q0, window, first);
  // the wave's rows, the keys [lo, hi) that each sees, and those that any or all of the wave's do
  int row[NQ], lo[NQ], hi[NQ], w0 = a.tokens, w1 = 0, f0 = 0, f1 = a.tokens;
  bf16x8 qf[NQ][4];
#pragma unroll
  for (int u = 0; u < NQ; ++u) {
    row[u] = q0 + (w * NQ + u) * 32 + lr;
    const int r = min(row[u], a.tokens - 1);
    lo[u] = first_key(a.starts, a.n, window, near, r);
    hi[u] = lo[u] > r ? lo[u] : r + 1;
    if (lo[u] < hi[u]) {
      w0 = min(w0, lo[u]);
      w1 = max(w1, hi[u]);
    }
    f0 = max(f0, lo[u]);
    f1 = min(f1, hi[u]);
#pragma unroll
    for (int s = 0; s < 4; ++s) qf[u][s] = *reinterpret_cast<const bf16x8*>(Q + r * a.qt + 16 * s + 8 * lk);
  }
#pragma unroll
  for (int m = 1; m < 32; m <<= 1) {
    w0 = min(w0, __shfl_xor(w0, m));
    w1 = max(w1, __shfl_xor(w1, m));
    f0 = max(f0, __shfl_xor(f0, m));
    f1 = min(f1, __shfl_xor(f1, m));
  }
  if (lane == 0) {
    first[w] = w0;
    last[w] = w1;
    from[w] = f0;
    to[w] = f1;
    odd[w] = -1;
  }
  __syncthreads();
  w0 = __builtin_amdgcn_readfirstlane(w0);
  w1 = __builtin_amdgcn_readfirstlane(w1);
  f0 = __builtin_amdgcn_readfirstlane(f0);
  f1 = __builtin_amdgcn_readfirstlane(f1);
  const int k0 = __builtin_amdgcn_readfirstlane(min(min(first[0], first[1]), min(first[2], first[3])));
  const int k1 = __builtin_amdgcn_readfirstlane(max(max(last[0], last[1]), max(last[2], last[3])));
  const int b0 = __builtin_amdgcn_readfirstlane(max(max(from[0], from[1]), max(from[2], from[3])));
  const int b1 = __builtin_amdgcn_readfirstlane(min(min(to[0], to[1]), min(to[2], to[3])));
  const int nt = k1 > k0 ? (k1 - k0 + kTile - 1) / kTile : 0;
  // Scores are formed less a reference of their row (the products' accumulators start at its negative,
  // `nref`), so p = 2^(kScale s) with no rounding of the reference in it.  It becomes the maximum of the first tile
  // with a score above -inf, then moves only when a score passes it by kRaise: p stays below 2^8
  constexpr float kRaise = 8.f / kScale;
  constexpr int KB = NQ == 1 ? 2 : 1;  // halves of a tile at a time, as registers allow
  float raise[NQ], l[NQ], nref[NQ];
  floatx16 o[NQ][2];
#pragma unroll
  for (int u = 0; u < NQ; ++u) {
    raise[u] = -INFINITY;
    l[u] = nref[u] = 0.f;
#pragma unroll
    for (int d = 0; d < 2; ++d)
#pragma unroll
      for (int v = 0; v < 16; ++v) o[u][d][v] = 0.f;
  }
  auto step = [&](int t, uint4* cur, uint4* nxt) {
    __builtin_amdgcn_s_waitcnt(kWaitNext);
    const int kt = k0 + t * kTile;
    const bool cut = t < nt && (kt < b0 || kt + kTile > b1);  // some row of the block does not see some key
    if (cut) {
      // A NaN or an infinity times a probability of 0 would reach the rows that do not see it: such values
      // leave the tile, each wave looking at what it copied, and are added to the rows that do below.
      uint4* own = cur + 512 + 128 * w + lane;
      const uint4 x[2] = {own[0], own[64]};
      float z = 0.f;
#pragma unroll
      for (int j = 0; j < 2; ++j) z = dot2(x[j].x, 0u, dot2(x[j].y, 0u, dot2(x[j].z, 0u, dot2(x[j].w, 0u, z))));
      if (__builtin_amdgcn_ballot_w64(z != 0.f)) {
#pragma unroll
        for (int j = 0; j < 2; ++j) own[64 * j] = make_uint4(finite2(x[j].x), finite2(x[j].y), finite2(x[j].z), finite2(x[j].w));
        if (lane == 0) odd[t & 3] = t;
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup");
      }
    }
    __builtin_amdgcn_s_barrier();
    prompt_copy(K, V, a, k0 + min(t + 2, nt - 1) * kTile, nxt);  // every step issues its copies: exact wait counts
    if (t >= nt || kt >= w1 || kt + kTile <= w0) return;
#pragma unroll 1
    for (int h0 = 0; h0 < 2; h0 += KB) {
      floatx16 sc[NQ][KB];
#pragma unroll
      for (int kb = 0; kb < KB; ++kb) {
#pragma unroll
        for (int u = 0; u < NQ; ++u)
#pragma unroll
          for (int v = 0; v < 16; ++v) sc[u][kb][v] = nref[u];
#pragma unroll
        for (int s = 0; s < 4; ++s) {
          const int r = (h0 + kb) * 32 + lr;
          const bf16x8 kf = __builtin_bit_cast(bf16x8, cur[r * 8 + ((2 * s + lk) ^ (r & 7))]);
#pragma unroll
          for (int u = 0; u < NQ; ++u) sc[u][kb] = mfma32(kf, qf[u][s], sc[u][kb]);
        }
      }
      if (kt < f0 || kt + kTile > f1) {  // uniform: some row does not see some key
#pragma unroll
        for (int u = 0; u < NQ; ++u)
#pragma unroll
          for (int kb = 0; kb < KB; ++kb)
#pragma unroll
            for (int v = 0; v < 16; ++v) {
              const int key = kt + (h0 + kb) * 32 + 8 * (v >> 2) + 4 * lk + (v & 3);
              sc[u][kb][v] = (uint32_t)(key - lo[u]) < (uint32_t)(hi[u] - lo[u]) ? sc[u][kb][v] : -INFINITY;
            }
      }
      uint32_t pk[NQ][KB][8];
#pragma unroll
      for (int u = 0; u < NQ; ++u) {
        float mx = sc[u][0][0];
#pragma unroll
        for (int kb = 0; kb < KB; ++kb)
#pragma unroll
          for (int v = 0; v < 16; ++v) mx = fmaxf(mx, sc[u][kb][v]);
        mx = pair_max(mx);
        if (__builtin_amdgcn_ballot_w64(mx > raise[u])) {
          const float d = mx > raise[u] ? mx : 0.f;
          const float f = raise[u] > 0.f ? __builtin_amdgcn_exp2f(-d * kScale) : 0.f;  // no score yet: l and o are 0
          if (mx > raise[u]) raise[u] = kRaise;
          l[u] *= f;
#pragma unroll
          for (int e = 0; e < 2; ++e)
#pragma unroll
            for (int v = 0; v < 16; ++v) o[u][e][v] *= f;
#pragma unroll
          for (int kb = 0; kb < KB; ++kb)
#pragma unroll
            for (int v = 0; v < 16; ++v) sc[u][kb][v] -= d;
          nref[u] -= d;
        }
#pragma unroll
        for (int kb = 0; kb < KB; ++kb)
#pragma unroll
          for (int v = 0; v < 16; v += 2) {
            pk[u][kb][v >> 1] = pack2_bf16(__builtin_amdgcn_exp2f(sc[u][kb][v] * kScale), __builtin_amdgcn_exp2f(sc[u][kb][v + 1] * kScale));
            l[u] = dot2(pk[u][kb][v >> 1], 0x3f803f80u, l[u]);
          }
      }
#pragma unroll
      for (int kb = 0; kb < KB; ++kb)
#pragma unroll
        for (int s = 0; s < 2; ++s)
#pragma unroll
          for (int d = 0; d < 2; ++d) {
            // eight keys 4 lk + 8 h + .. of sixteen for the lane's dim: a lane reads row lane / 4 % 4 of them, the 8-byte piece lane % 4
            // of sixteen dims
            uint2 x[2];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              const int r = (h0 + kb) * 32 + 16 * s + 8 * h + 4 * lk + ((lane >> 2) & 3), c = 4 * d + 2 * ((lane >> 4) & 1) + ((lane >> 1) & 1);
              const char* p = reinterpret_cast<const char*>(cur + 512 + r * 8 + (c ^ (r & 7))) + 8 * (lane & 1);
              x[h] = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)p));
            }
            const bf16x8 vf = __builtin_bit_cast(bf16x8, make_uint4(x[0].x, x[0].y, x[1].x, x[1].y));
#pragma unroll
            for (int u = 0; u < NQ; ++u) {
              const uint4 p = make_uint4(pk[u][kb][4 * s], pk[u][kb][4 * s + 1], pk[u][kb][4 * s + 2], pk[u][kb][4 * s + 3]);
              o[u][d] = mfma32(vf, __builtin_bit_cast(bf16x8, p), o[u][d]);
            }
          }
    }
    if (cut && __builtin_amdgcn_readfirstlane(odd[t & 3]) == t) {  // what left the tile, for the rows that see it
#pragma unroll 1
      for (int key = kt; key < min(kt + kTile, k1); ++key) {
        const bf16* vp = V + key * a.vt + 4 * lk;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          float x[4];
          ld<4>(vp + 8 * e, 1, x);
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const float y = finite(x[i]) ? 0.f : x[i];
#pragma unroll
            for (int u = 0; u < NQ; ++u) o[u][e >> 2][4 * (e & 3) + i] += (uint32_t)(key - lo[u]) < (uint32_t)(hi[u] - lo[u]) ? y : 0.f;
          }
        }
      }
    }
  };
  if (nt > 0) {
    prompt_copy(K, V, a, k0, st0);
    prompt_copy(K, V, a, k0 + min(1, nt - 1) * kTile, st1);
    for (int t = 0; t < nt; t += 3) {
      step(t, st0, st2);
      step(t + 1, st1, st0);
      step(t + 2, st2, st1);
    }
    __builtin_amdgcn_s_waitcnt(kWaitAll);  // no copy may land in LDS after the block has left
  }
#pragma unroll
  for (int u = 0; u < NQ; ++u) {
    const float total = pair_sum(l[u]), inv = total == 0.f ? 0.f : 1.f / total;
    if (row[u] >= a.tokens) continue;
    if (!a.clear && (row[u] < near.begin || row[u] >= near.end)) continue;
    // O^T: lane holds row lr, dims 32 d + 8 (v / 4) + 4 lk + v % 4
    bf16* op = reinterpret_cast<bf16*>(a.out) + ((size_t)row[u] * a.heads + head) * kHeadDim;
#pragma unroll
    for (int d = 0; d < 2; ++d)
#pragma unroll
      for (int g = 0; g < 4; ++g)
        *reinterpret_cast<uint2*>(op + d * 32 + 8 * g + 4 * lk) =
            make_uint2(pack2_bf16(o[u][d][4 * g] * inv, o[u][d][4 * g + 1] * inv), pack2_bf16(o[u][d][4 * g + 2] * inv, o[u][d][4 * g + 3] * inv));
  }
}
template <int NQ>
static void prompt16(const PromptArgs& a, hipStream_t st) {
  const int tiles = (a.tokens + 128 * NQ - 1) / (128 * NQ), per = (int)(((long long)tiles * a.heads + 7) / 8);
  k_prompt16<NQ><<<8 * per, 256, 0, st>>>(a, tiles, per);
}

template <typename T>
static void prompt32(const PromptArgs& a, hipStream_t st) {
  const int tiles = (a.tokens + 31) / 32, per = (int)(((long long)tiles * a.heads + 7) / 8);
  k_prompt32<T><<<8 * per, 256, 0, st>>>(a, tiles, per);
}

void prompt_attend(const PromptArgs& a, hipStream_t st) {
  if (!a.bf16_data) return prompt32<float>(a, st);
  if (!a.vec) return prompt32<bf16>(a, st);
  if (a.tokens > 4096) return prompt16<2>(a, st);
  prompt16<1>(a, st);
}

}  // namespace wf
