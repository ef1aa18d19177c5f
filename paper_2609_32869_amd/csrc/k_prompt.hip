// Causal attention of packed prompts.
//
// Rows of all sequences lie one after the other; row t sees the rows of its own sequence up to
// itself, an interval [lo, t] of the packed rows.  A block takes consecutive rows of one head,
// whichever sequences they belong to, and the keys from its own last row back to its first row's
// lo: short sequences share a block, and neither lengths nor their tiles have to be known on
// the host.  Scores outside a row's interval are replaced by -inf.  One pass over the keys:
// scores, their exponentials less a running reference, and the product with the values stay in
// registers.
//
// The matrix and the vector units bound it together: per 32 rows and 32 keys 8 products (bf16, 256
// cycles) and 16 exponentials a lane with four instructions about each (340 cycles).
#include <algorithm>

#include "wf_operand.h"
#include "wf_ops.h"

namespace wf {

namespace {
constexpr float kScale = 0.125f * 1.44269504088896340736f;  // exp(s / 8) = 2^(kScale s)
// The reference of a row's probabilities p = 2^(kScale (s - reference)) moves where a score passes its old maximum by this, so that p
// would reach 2^8.  p or the values are taken 2^-8 of themselves: n values of up to 3.4e38 / n have finite sums.
constexpr float kRaise = 8.f / kScale;

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
// The block's NT threads narrow the borders NT-fold a round (none up to 511 sequences) and load the window:
// one round trip to memory, where a search of 96 borders by every row takes seven.  meanwhile() runs while
// the window is on its way.  counts: a word a wave.
template <int NT, typename F>
__device__ __forceinline__ Borders borders_near(const int* starts, int n, int q0, int* window, int* counts, const F& meanwhile) {
  const int tid = threadIdx.x;
  int base = 0, size = n + 1;
  while (size > kWindow) {
    const int stride = (size + NT - 1) / NT, i = tid * stride;
    const int c = __popcll(__builtin_amdgcn_ballot_w64(i < size && starts[base + i] <= q0));
    if ((tid & 63) == 0) counts[tid >> 6] = c;
    __syncthreads();
    int at = -1;
    for (int w = 0; w < NT / 64; ++w) at += counts[w];
    at = max(at, 0) * stride;
    __syncthreads();
    size = min(stride, size - at);
    base += at;
  }
  base = min(base, n);
  int x[kWindow / NT];
#pragma unroll
  for (int j = 0; j < kWindow / NT; ++j) x[j] = starts[min(base + NT * j + tid, n)];
  const Borders b{base, min(kWindow, n + 1 - base), starts[0], starts[n]};
  meanwhile();
#pragma unroll
  for (int j = 0; j < kWindow / NT; ++j) window[NT * j + tid] = x[j];
  __syncthreads();
  return b;
}
// First key of row t: the largest border <= t, where t lies in a sequence; t + 1 (no key) elsewhere.
__device__ __forceinline__ int first_key(const int* starts, int n, const int* window, const Borders& b, int t) {
  if (t < b.begin || t >= b.end) return t + 1;
  int lo = 0, hi = b.size - 1;  // the border of lo is <= t, that of hi > t
  if (b.base + b.size > n || window[hi] > t) {
    while (hi - lo > 1) {
      const int m = (lo + hi) >> 1;
      if (window[m] <= t) lo = m;
      else hi = m;
    }
    return min(max(window[lo], 0), t + 1);
  }
  lo = b.base;
  hi = n;
  while (hi - lo > 1) {
    const int m = (lo + hi) >> 1;
    if (starts[m] <= t) lo = m;
    else hi = m;
  }
  return min(max(starts[lo], 0), t + 1);
}

// Which head and tile of rows a block takes.  An XCD gets every eighth block; so that its L2 holds few heads' keys and values
// and all XCDs have equal work, each head's tiles are dealt to S = 2^shift parts (heads * S a multiple of 8), and the
// XCD takes `parts` = heads * S / 8 of them that follow each other, those of the longest tiles first.  Contiguous
// eighths of all (head, tile) pairs instead leave one XCD 1.75 heads' work and the next 1.25 (12 heads of 8,192 rows: 181 us).
struct Grid {
  int tiles, parts, shift, blocks;
};
static Grid grid_of(int tokens, int rows, int heads) {
  const int tiles = (tokens + rows - 1) / rows, shift = heads % 8 == 0 ? 0 : heads % 4 == 0 ? 1 : heads % 2 == 0 ? 2 : 3;
  const int parts = (heads << shift) / 8;
  return Grid{tiles, parts, shift, 8 * parts * ((tiles + (1 << shift) - 1) >> shift)};
}
__device__ __forceinline__ bool block_of(const Grid& g, int& head, int& tile) {
  const unsigned x = blockIdx.x & 7, j = blockIdx.x >> 3, k = j / (unsigned)g.parts, part = x * g.parts + (j - k * g.parts);
  const int t = (k << g.shift) + (part & ((1 << g.shift) - 1));
  head = part >> g.shift;
  tile = g.tiles - 1 - t;
  return t < g.tiles;
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

// ---------------------------------------------------------------- few rows, and rows of any alignment
// Block: (32 rows, head), four waves that take every fourth tile of 32 keys, each on its own from memory
// to registers, and join their maxima, sums and outputs in LDS at the end.  fp32 values enter the products as three
// bf16 terms: six products of v_mfma_f32_32x32x16_bf16, each a sixteenth of the time of the same product by
// v_mfma_f32_32x32x2_f32 (9,001 rows of 12 heads 262 us against 471).
//   S^T = K q^T  a lane gets keys 8 (v / 4) + 4 (lane / 32) + v % 4 of row lane % 32
//   O^T += V^T P^T  the half-waves' eight values of an instruction are taken as those keys, so the probabilities
//                are the operand as they are, and a lane's values are V[those keys][lane % 32 + 32 d]
// The next tile's keys are loaded once this one's are multiplied, the values likewise.  One prompt of 224 rows, 20 heads: 10.5 us
// a call among others, 8.0 of the host; the way of a block's first loads, its two tiles and the joining bounds it.
template <typename T>
__global__ void __launch_bounds__(256, 2) k_prompt32(PromptArgs a, Grid grid) {
  constexpr int N = sizeof(T) == 4 ? 3 : 1;
  __shared__ float wm[4][32], wl[4][32];
  __shared__ alignas(16) float wo[4][32][68];
  int head, tile;
  if (!block_of(grid, head, tile)) return;
  const int q0 = tile * 32;
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, lr = lane & 31, lk = lane >> 5;
  const int row = min(q0 + lr, a.tokens - 1);
  const T* Q = reinterpret_cast<const T*>(a.q) + row * a.qt + head * a.qh + 8 * lk;
  float q[4][8];
#pragma unroll
  for (int s = 0; s < 4; ++s) ld<8>(Q + 16 * s, a.vec, q[s]);
  const T* K = reinterpret_cast<const T*>(a.k) + (head / a.group) * a.kh + 8 * lk;
  const T* V = reinterpret_cast<const T*>(a.v) + (head / a.group) * a.vh + lr;
  const int last = a.tokens - 1;
  float kx[4][8], vx[2][2][8];  // a tile: keys' dims 16 s + 8 lk .. + 7 of key lr; values [dim half][sixteen keys]
  auto load_keys = [&](int kt) {
    const T* p = K + min(max(kt + lr, 0), last) * a.kt;
#pragma unroll
    for (int s = 0; s < 4; ++s) ld<8>(p + 16 * s, a.vec, kx[s]);
  };
  auto load_values = [&](int kt) {
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const T* p = V + min(max(kt + 8 * (i >> 2) + 4 * lk + (i & 3), 0), last) * a.vt;
      vx[0][i >> 3][i & 7] = to_f(p[0]);
      vx[1][i >> 3][i & 7] = to_f(p[32]);
    }
  };
  // Tile t: keys e - 32 (t + 1) .. e - 32 t - 1, from the block's own rows back to its first sequence's first row, so that
  // the waves' first tiles are under way before the borders are known.
  const int e = min(q0 + 32, a.tokens);
  int kt = e - 32 * (w + 1);
  int* window = reinterpret_cast<int*>(wo);
  const Borders near = borders_near<256>(a.starts, a.n, q0, window, reinterpret_cast<int*>(wm), [&] {
    load_keys(kt);
    load_values(kt);
  });
  const int lo = first_key(a.starts, a.n, window, near, row);  // the row sees keys [lo, row]
  // first keys do not decrease along the rows
  const int k0 = __builtin_amdgcn_readlane(lo, 0), f0 = __builtin_amdgcn_readlane(lo, 31);
  bf16x8 qt[4][N];
#pragma unroll
  for (int s = 0; s < 4; ++s) terms8<N>(q[s], qt[s]);
  float m = -INFINITY, l = 0.f;
  floatx16 o[2];
#pragma unroll
  for (int d = 0; d < 2; ++d)
#pragma unroll
    for (int v = 0; v < 16; ++v) o[d][v] = 0.f;
  for (; kt + 32 > k0; kt -= 128) {
    floatx16 s;
#pragma unroll
    for (int v = 0; v < 16; ++v) s[v] = 0.f;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      bf16x8 t[N];
      terms8<N>(kx[i], t);
      s = product<N>(t, qt[i], s);
    }
    if (kt - 96 > k0) load_keys(kt - 128);
    const bool masked = kt < f0 || kt + 31 > q0;  // uniform: some row does not see some key
    uint32_t out = 0;                             // bit v: the row does not see the key
    if (masked) {
#pragma unroll
      for (int v = 0; v < 16; ++v) {
        const int key = kt + 8 * (v >> 2) + 4 * lk + (v & 3);
        const bool hidden = key < lo || key > row;
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
    if (kt - 96 > k0) load_values(kt - 128);
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
// Block: (128 NQ rows, head), G groups of four waves of 32 NQ rows; group g takes tiles g, g + G, ...  Keys and values
// stream through NS LDS stages a group in tiles of 64 rows, copied straight from memory
// (global_load_lds_dwordx4) NS - 1 tiles ahead of their use.  KB x 32 keys at a time a wave forms S^T = K q^T on
// v_mfma_f32_32x32x16_bf16, so a lane holds 16 of 32 keys of one row (keys 8 (v / 4) + 4 (lane / 32) + v % 4):
// reference and sum are per lane (one swap of half-waves joins a row's two lanes) and the probabilities, rounded to
// bf16 in place (2^-9 of each, as the results' own rounding: an error of 0.0019 of the 2-norm where that alone leaves 0.0014;
// two terms of each would take 43% more time, 6.8 ms for 4.8 of 32,768 rows of 32 heads, 14% more for 96 short prompts),
// are the B operand of O^T += V^T P^T if the half-waves'
// eight values of an instruction are taken as those keys.  The A operand then is, for a dim, keys 4 and 4 together,
// what ds_read_b64_tr_b16 makes of rows as they lie in memory.  The sum is taken of the rounded probabilities.
// 32,768 rows, 32 heads over 8: 4.7 to 5.3 ms by the card, whose clock falls under this load, 940 to 830 TFLOP/s, 78 to 72%
// of what a library's large product reaches on it; 96 prompts of 1 to 447 rows, 20 heads: 73 us, where the bytes alone are
// 43.  Raising the waves' priority, around the products or of every other wave, changes nothing.
namespace {
typedef __attribute__((address_space(3))) void lds_void;
constexpr int kTile = 64, kStage = 1024;  // keys of a tile; 16-byte chunks of a stage
// LDS stages.  Reads form their addresses by xor within a row's 128 bytes, so a row starts on a border of as many.
template <int CHUNKS>
struct alignas(128) Stages {
  uint4 chunk[CHUNKS];
};
// A stage: chunk c (8 dims) of key r at 8 r + (c ^ (r & 7)), then of its values at 8 r + (c ^ 2 (r & 3)): the four rows that sixteen
// lanes read two chunks of by ds_read_b64_tr_b16 then lie in different banks (as the keys lie, two and two shared them).
// lgkmcnt 0 and vmcnt the copies of the tiles behind the next, four each
template <int NS>
constexpr int kWaitNext = (4 * (NS - 2)) | (7 << 4);
constexpr int kWaitAll = (0 & 15) | (7 << 4) | (15 << 8);

// where chunk c of row r lies in its row of a stage, and which one lies there
__device__ __forceinline__ int key_chunk(int r, int c) { return (c ^ r) & 7; }
__device__ __forceinline__ int value_chunk(int r, int c) { return (c ^ 2 * (r & 3)) & 7; }
__device__ __forceinline__ float dot2(uint32_t a, uint32_t b, float c) {
  return __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16v2, a), __builtin_bit_cast(bf16v2, b), c, false);
}
// two bf16 values, zero where they are not finite
__device__ __forceinline__ uint32_t finite2(uint32_t x) {
  return ((x & 0x7f80u) == 0x7f80u ? 0u : x & 0xffffu) | ((x & 0x7f800000u) == 0x7f800000u ? 0u : x & 0xffff0000u);
}
}  // namespace

// A pointer that is the same in every lane, kept out of their registers.
__device__ __forceinline__ const char* in_sgpr(const void* p) {
  const uint64_t x = reinterpret_cast<uint64_t>(p);
  const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)x), hi = __builtin_amdgcn_readfirstlane((uint32_t)(x >> 32));
  return reinterpret_cast<const char*>((uint64_t)hi << 32 | lo);
}
// Where a lane's chunks of a tile lie: rows w * 16 + 8 j + lane / 8 (j = 0, 1), bytes from the tile's first row.
struct Chunks {
  uint32_t k, v;
};
// Reads of a tile in asm, for the compiler would wait for every copy under way before each of them.
// 32 keys as the operands of four products: the lane's dims 16 s + 8 lk .. + 7 lie at `at` ^ 32 s.
__device__ __forceinline__ void read_keys(uint32_t at, bf16x8 (&x)[4]) {
  asm volatile(
      "ds_read_b128 %0, %4\n\t"
      "ds_read_b128 %1, %5\n\t"
      "ds_read_b128 %2, %6\n\t"
      "ds_read_b128 %3, %7\n\t"
      "s_waitcnt lgkmcnt(0)"
      : "=&v"(x[0]), "=&v"(x[1]), "=&v"(x[2]), "=&v"(x[3])
      : "v"(at), "v"(at ^ 32u), "v"(at ^ 64u), "v"(at ^ 96u)
      : "memory");
}
// Joins two groups' parts of the same rows (a wave of each has them in the same lanes): the reference m of a part's
// probabilities, -inf where it saw no score, its sum and outputs.  The first group's waves get the whole and true.
__device__ __forceinline__ bool join(int g, int w, float* lds, float m, float& l, floatx16 (&o)[2]) {
  float* p = lds + w * 34 * 64 + (threadIdx.x & 63);
  if (g) {
    p[0] = m;
    p[64] = l;
#pragma unroll
    for (int v = 0; v < 32; ++v) p[(2 + v) * 64] = o[v >> 4][v & 15];
  }
  __syncthreads();
  if (g) return false;
  const float m1 = p[0], top = fmaxf(m, m1), base = top == -INFINITY ? 0.f : top;
  const float f = __builtin_amdgcn_exp2f((m - base) * kScale), f1 = __builtin_amdgcn_exp2f((m1 - base) * kScale);
  l = l * f + p[64] * f1;
#pragma unroll
  for (int v = 0; v < 32; ++v) o[v >> 4][v & 15] = o[v >> 4][v & 15] * f + p[(2 + v) * 64] * f1;
  return true;
}
// The values of 32 keys as the operands of four products, [sixteen keys][dim half]; `at` ^ 64: the other half.  The wait falls into
// the time that the scores' products take.
__device__ __forceinline__ void read_values(uint32_t at, bf16x8 (&x)[2][2]) {
  uint2 r[8];
  asm volatile(
      "ds_read_b64_tr_b16 %0, %8\n\t"
      "ds_read_b64_tr_b16 %1, %8 offset:0x400\n\t"
      "ds_read_b64_tr_b16 %2, %9\n\t"
      "ds_read_b64_tr_b16 %3, %9 offset:0x400\n\t"
      "ds_read_b64_tr_b16 %4, %8 offset:0x800\n\t"
      "ds_read_b64_tr_b16 %5, %8 offset:0xc00\n\t"
      "ds_read_b64_tr_b16 %6, %9 offset:0x800\n\t"
      "ds_read_b64_tr_b16 %7, %9 offset:0xc00\n\t"
      "s_waitcnt lgkmcnt(0)"
      : "=&v"(r[0]), "=&v"(r[1]), "=&v"(r[2]), "=&v"(r[3]), "=&v"(r[4]), "=&v"(r[5]), "=&v"(r[6]), "=&v"(r[7])
      : "v"(at), "v"(at ^ 64u)
      : "memory");
#pragma unroll
  for (int i = 0; i < 4; ++i) x[i >> 1][i & 1] = __builtin_bit_cast(bf16x8, make_uint4(r[2 * i].x, r[2 * i].y, r[2 * i + 1].x, r[2 * i + 1].y));
}

// Keys and values k0 .. k0 + 63 (rows outside the tensors are the nearest) into a stage: the tile's address is the wave's, a
// lane adds its constant chunk.
__device__ __forceinline__ void prompt_copy(const bf16* K, const bf16* V, const PromptArgs& a, int k0, const Chunks& c, uint4* stage, int w) {
  const int lane = threadIdx.x & 63;
  // (the instruction's own offset would move both addresses)
  lds_void *ks0 = (lds_void*)&stage[w * 128], *ks1 = (lds_void*)&stage[w * 128 + 64];
  lds_void *vs0 = (lds_void*)&stage[512 + w * 128], *vs1 = (lds_void*)&stage[512 + w * 128 + 64];
  if (k0 >= 0 && k0 + kTile <= a.tokens) {
    const char *kp = in_sgpr(K + k0 * a.kt), *vp = in_sgpr(V + k0 * a.vt);
    __builtin_amdgcn_global_load_lds((const void*)(kp + c.k), ks0, 16, 0, 0);
    __builtin_amdgcn_global_load_lds((const void*)(in_sgpr(kp + 16 * a.kt) + c.k), ks1, 16, 0, 0);
    __builtin_amdgcn_global_load_lds((const void*)(vp + c.v), vs0, 16, 0, 0);
    __builtin_amdgcn_global_load_lds((const void*)(in_sgpr(vp + 16 * a.vt) + c.v), vs1, 16, 0, 0);
  } else {
    const int r = w * 16 + (lane >> 3), ch = 8 * key_chunk(lane >> 3, lane), cv = 8 * value_chunk(lane >> 3, lane), last = a.tokens - 1;
    const int r0 = min(max(k0 + r, 0), last), r1 = min(max(k0 + r + 8, 0), last);
    __builtin_amdgcn_global_load_lds((const void*)(K + r0 * a.kt + ch), ks0, 16, 0, 0);
    __builtin_amdgcn_global_load_lds((const void*)(K + r1 * a.kt + ch), ks1, 16, 0, 0);
    __builtin_amdgcn_global_load_lds((const void*)(V + r0 * a.vt + cv), vs0, 16, 0, 0);
    __builtin_amdgcn_global_load_lds((const void*)(V + r1 * a.vt + cv), vs1, 16, 0, 0);
  }
}

template <int NQ, int KB, int WAVES, int G, int NS>
__global__ void __launch_bounds__(256 * G, WAVES) k_prompt16(PromptArgs a, Grid grid) {
  __shared__ Stages<G * NS * kStage> shared;
  static_assert(alignof(decltype(shared)) % 128 == 0, "reads xor addresses up to 127");
  int head, tile;
  if (!block_of(grid, head, tile)) return;
  const int q0 = tile * 128 * NQ;
  const int w = __builtin_amdgcn_readfirstlane((threadIdx.x >> 6) & 3), g = __builtin_amdgcn_readfirstlane(threadIdx.x >> 8);
  const int lane = threadIdx.x & 63, lr = lane & 31, lk = lane >> 5;
  uint4* const stages = shared.chunk + g * NS * kStage;
  const bf16* Q = reinterpret_cast<const bf16*>(a.q) + head * a.qh;
  const bf16* K = reinterpret_cast<const bf16*>(a.k) + (head / a.group) * a.kh;
  const bf16* V = reinterpret_cast<const bf16*>(a.v) + (head / a.group) * a.vh;
  __shared__ int window[kWindow], odd[8];  // odd: the last tile of a group's stage that held a NaN or an infinity
  // Tile t: keys e - 64 (t + 1) .. e - 64 t - 1, from the block's own rows back to its first sequence's first row, so
  // that the first is copied before the borders are known.
  const int rows = 128 * NQ, e = min(q0 + rows, a.tokens), r0 = q0 + w * 32 * NQ;
  const uint32_t crow = w * 16 + (lane >> 3);
  const Chunks chunks{crow * 2 * (uint32_t)a.kt + 16 * key_chunk(lane >> 3, lane), crow * 2 * (uint32_t)a.vt + 16 * value_chunk(lane >> 3, lane)};
  int row[NQ], lo[NQ];  // a row and the first key that it sees (the row + 1: none)
  bf16x8 qf[NQ][4];
#pragma unroll
  for (int u = 0; u < NQ; ++u) {
    row[u] = min(r0 + u * 32 + lr, a.tokens - 1);
#pragma unroll
    for (int s = 0; s < 4; ++s) qf[u][s] = *reinterpret_cast<const bf16x8*>(Q + row[u] * a.qt + 16 * s + 8 * lk);
  }
  auto copy_first = [&] {
#pragma unroll 1
    for (int i = 0; i < NS - 1; ++i) prompt_copy(K, V, a, e - (i * G + g + 1) * kTile, chunks, stages + i * kStage, w);
    if (threadIdx.x < 8) odd[threadIdx.x] = -1;
  };
  const Borders near = borders_near<256 * G>(a.starts, a.n, q0, window, odd, copy_first);
  // first keys do not decrease along the rows: of the wave's rows, and of the block's first and last
  int first = 0, bound = 0;
#pragma unroll 1
  for (int i = 0; i < 2; ++i) {
    const int x = first_key(a.starts, a.n, window, near, i == 0 ? min(r0 + lane, a.tokens - 1) : lane & 1 ? e - 1 : q0);
    first = i == 0 ? x : first;
    bound = x;
  }
#pragma unroll
  for (int u = 0; u < NQ; ++u) lo[u] = __shfl(first, 32 * u + lr);
  const int k0 = __builtin_amdgcn_readlane(bound, 0), b0 = __builtin_amdgcn_readlane(bound, 1);
  const int w0 = __builtin_amdgcn_readlane(first, 0), f0 = __builtin_amdgcn_readlane(first, 32 * NQ - 1);
  const int nt = (e - min(k0, e) + kTile - 1) / kTile;
  // Scores are formed less a reference of their row (the products' accumulators start at its negative, `nref`), so p =
  // 2^(kScale s).  It lies kRaise above the maximum of the first tile with a score above -inf, then moves only when a
  // score passes it: p stays below 1 (its exponent's rounding, 2^-21, is far below p's own).  raise: -inf before, 0 from then on
  float raise[NQ], l[NQ];
  constexpr int NR = WAVES == 4 ? 1 : 16;  // at four waves a SIMD the reference is subtracted instead, for sixteen registers
  float nref[NQ][NR];
  floatx16 o[NQ][2];
  auto clear = [&] {
#pragma unroll
    for (int u = 0; u < NQ; ++u) {
      raise[u] = -INFINITY;
      l[u] = 0.f;
#pragma unroll
      for (int v = 0; v < 16; ++v) nref[u][v % NR] = o[u][0][v] = o[u][1][v] = 0.f;
    }
  };
  clear();
  bool careful = false;
  // a lane's key lk (chunk) of row lr; its part of sixteen keys by sixteen dims, as ds_read_b64_tr_b16 turns them: row
  // 4 lk + lane / 4 % 4 (and 8 on), the 8-byte piece lane % 4 of dims 16 (lane / 16 % 2) ..
  const int vrow = 4 * lk + ((lane >> 2) & 3), vchunk = value_chunk(vrow, 2 * ((lane >> 4) & 1) + ((lane >> 1) & 1));
  const uint32_t kat = 128 * lr + 16 * (lk ^ (lr & 7)), vat = 8192 + 128 * vrow + 16 * vchunk + 8 * (lane & 1);
  auto step = [&](int i, uint4* cur, uint4* nxt) {
    const int t = i * G + g;
    const uint32_t lds = (uint32_t)(uintptr_t)(lds_void*)cur;
    __builtin_amdgcn_s_waitcnt(kWaitNext<NS>);
    const int kt = e - (t + 1) * kTile;
    const bool cut = careful && t < nt && (kt < b0 || kt + kTile > q0 + 1);  // some row of the block does not see some key
    if (cut) {  // what is not finite among the values leaves the tile, each wave looking at what it copied
      uint4* own = cur + 512 + 128 * w + lane;
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const uint4 x = own[64 * j], y = make_uint4(finite2(x.x), finite2(x.y), finite2(x.z), finite2(x.w));
        if (__builtin_amdgcn_ballot_w64(((x.x ^ y.x) | (x.y ^ y.y) | (x.z ^ y.z) | (x.w ^ y.w)) != 0)) {
          own[64 * j] = y;
          if (lane == 0) odd[4 * g + (i & 3)] = t;
        }
      }
      __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup");
    }
    __builtin_amdgcn_s_barrier();
    prompt_copy(K, V, a, e - min(t + (NS - 1) * G + 1, nt) * kTile, chunks, nxt, w);  // in every step: exact wait counts
    if (t >= nt || kt >= r0 + 32 * NQ || kt + kTile <= w0) return;
#pragma unroll 1
    for (int h0 = 0; h0 < 2; h0 += KB) {
      const int kh = kt + 32 * h0;
      if (kh >= r0 + 32 * NQ || kh + 32 * KB <= w0) continue;
      floatx16 sc[NQ][KB];
#pragma unroll
      for (int kb = 0; kb < KB; ++kb) {
        bf16x8 kf[4];
        read_keys(lds + 4096 * (h0 + kb) + kat, kf);
#pragma unroll
        for (int s = 0; s < 4; ++s)
#pragma unroll
          for (int u = 0; u < NQ; ++u) {
            if (s == 0) {
#pragma unroll
              for (int v = 0; v < 16; ++v) sc[u][kb][v] = NR == 16 ? nref[u][v % NR] : 0.f;
            }
            sc[u][kb] = mfma32(kf[s], qf[u][s], sc[u][kb]);
          }
      }
      bf16x8 vf[KB][2][2];
#pragma unroll
      for (int kb = 0; kb < KB; ++kb) read_values(lds + 4096 * (h0 + kb) + vat, vf[kb]);
      auto masked = [&](int u, floatx16 (&x)[KB]) {  // and their maximum
        if (kh + 32 * KB > r0 + 1) {                 // uniform: some row of the wave does not see some key behind it
#pragma unroll
          for (int kb = 0; kb < KB; ++kb)
#pragma unroll
            for (int v = 0; v < 16; ++v)
              x[kb][v] = 32 * kb + 8 * (v >> 2) + (v & 3) <= row[u] - kh - 4 * lk ? x[kb][v] : -INFINITY;
        }
        if (kh < f0) {  // nor keys of the sequence before
#pragma unroll
          for (int kb = 0; kb < KB; ++kb)
#pragma unroll
            for (int v = 0; v < 16; ++v)
              x[kb][v] = 32 * kb + 8 * (v >> 2) + (v & 3) >= lo[u] - kh - 4 * lk ? x[kb][v] : -INFINITY;
        }
        float mx = x[0][0];
#pragma unroll
        for (int kb = 0; kb < KB; ++kb)
#pragma unroll
          for (int v = 0; v < 16; ++v) mx = fmaxf(mx, x[kb][v]);
        return pair_max(mx);
      };
      uint32_t pk[NQ][KB][8];
#pragma unroll
      for (int u = 0; u < NQ; ++u) {
        float mx = masked(u, sc[u]);
        const bool up = (NR == 1 ? mx + nref[u][0] : mx) > raise[u];
        if (__builtin_amdgcn_ballot_w64(up)) {
          // Sums that began at a reference hold its roundings, however far below the new one it lies: the scores of such rows again
          if (NR == 16 && __builtin_amdgcn_ballot_w64(up && raise[u] == 0.f)) {
            floatx16 x[KB];
#pragma unroll
            for (int kb = 0; kb < KB; ++kb) {
              bf16x8 kf[4];
              read_keys(lds + 4096 * (h0 + kb) + kat, kf);
#pragma unroll
              for (int v = 0; v < 16; ++v) x[kb][v] = 0.f;
#pragma unroll
              for (int s = 0; s < 4; ++s) x[kb] = mfma32(kf[s], qf[u][s], x[kb]);
            }
            mx = masked(u, x);
#pragma unroll
            for (int kb = 0; kb < KB; ++kb)
#pragma unroll
              for (int v = 0; v < 16; ++v) sc[u][kb][v] = up ? x[kb][v] : sc[u][kb][v];
          }
          const float next = up ? -(mx + kRaise) : nref[u][0];
          const float f = !up ? 1.f : raise[u] == 0.f ? __builtin_amdgcn_exp2f(fminf(next - nref[u][0], 0.f) * kScale) : 0.f;  // no score yet: l and o are 0
          if (up) raise[u] = 0.f;
          l[u] *= f;
#pragma unroll
          for (int e = 0; e < 2; ++e)
#pragma unroll
            for (int v = 0; v < 16; ++v) o[u][e][v] *= f;
          if constexpr (NR == 16) {
#pragma unroll
            for (int kb = 0; kb < KB; ++kb)
#pragma unroll
              for (int v = 0; v < 16; ++v) sc[u][kb][v] += up ? next : 0.f;
          }
#pragma unroll
          for (int v = 0; v < NR; ++v) nref[u][v] = next;
        }
        if constexpr (NR == 1) {
#pragma unroll
          for (int kb = 0; kb < KB; ++kb)
#pragma unroll
            for (int v = 0; v < 16; ++v) sc[u][kb][v] += nref[u][0];
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
#pragma unroll
            for (int u = 0; u < NQ; ++u) {
              const uint4 p = make_uint4(pk[u][kb][4 * s], pk[u][kb][4 * s + 1], pk[u][kb][4 * s + 2], pk[u][kb][4 * s + 3]);
              o[u][d] = mfma32(vf[kb][s][d], __builtin_bit_cast(bf16x8, p), o[u][d]);
            }
          }
    }
    if (cut && __builtin_amdgcn_readfirstlane(odd[4 * g + (i & 3)]) == t) {  // and is added for the rows that see it
#pragma unroll 1
      for (int key = max(kt, 0); key < kt + kTile; ++key) {
        const bf16* vp = V + key * a.vt + 4 * lk;
#pragma unroll
        for (int b = 0; b < 8; ++b) {
          float x[4];
          ld<4>(vp + 8 * b, 1, x);
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const float y = finite(x[j]) ? 0.f : x[j];
#pragma unroll
            for (int u = 0; u < NQ; ++u) o[u][b >> 2][4 * (b & 3) + j] += key >= lo[u] && key <= row[u] ? y : 0.f;
          }
        }
      }
    }
  };
  for (;;) {
    uint4 *cur = stages, *nxt = stages + (NS - 1) * kStage;
    for (int i = 0; i * G < nt; ++i) {
      step(i, cur, nxt);
      nxt = cur;
      cur = cur == stages + (NS - 1) * kStage ? stages : cur + kStage;
    }
    __builtin_amdgcn_s_waitcnt(kWaitAll);  // no copy may land in LDS after the block has left
    if (careful) break;
    // A NaN or an infinity among the values reaches rows that do not see it, as its product with a probability of 0.
    // Where a result is not finite the block starts again and keeps such values out of the tiles that are not whole.
    float z = 0.f;
#pragma unroll
    for (int u = 0; u < NQ; ++u)
#pragma unroll
      for (int v = 0; v < 32; ++v) z = fmaf(o[u][v >> 4][v & 15], 0.f, z);
    if (__builtin_amdgcn_ballot_w64(z != 0.f) && lane == 0) window[0] = -1 - kWindow;
    __syncthreads();
    if (__builtin_amdgcn_readfirstlane(window[0]) != -1 - kWindow) break;
    careful = true;
    clear();
    copy_first();
    __syncthreads();
  }
  if constexpr (G == 2) {
    static_assert(NQ == 1, "one tile of rows a wave");
    __syncthreads();
    if (!join(g, w, reinterpret_cast<float*>(shared.chunk), raise[0] == 0.f ? -nref[0][0] : -INFINITY, l[0], o[0])) return;
  }
#pragma unroll
  for (int u = 0; u < NQ; ++u) {
    const float total = pair_sum(l[u]), inv = total == 0.f ? 0.f : 1.f / total;
    if (r0 + u * 32 + lr >= a.tokens) continue;
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
template <int NQ, int KB, int WAVES, int G, int NS>
static void prompt16(const PromptArgs& a, hipStream_t st) {
  const Grid g = grid_of(a.tokens, 128 * NQ, a.heads);
  k_prompt16<NQ, KB, WAVES, G, NS><<<g.blocks, 256 * G, 0, st>>>(a, g);
}


// ---------------------------------------------------------------- fp32, many rows
// Block: (128 rows, head), G groups of four waves of 32 rows; group g takes tiles g, g + G, ... of 32 keys.  A group's 256
// threads load 8 dims of a key and of a value row each, split them into three bf16 terms once for the whole block and
// write them to one of two LDS stages while the other is multiplied; the next tile's loads are under way
// meanwhile.  A stage holds six planes of 32 rows of 64 dims (keys' terms, values' terms) in k_prompt16's order.  Products as in
// k_prompt32 (six a pair of operands, a plane at a time, the smallest first), softmax as in k_prompt16.  32,768 rows, 32
// heads: 22.9 ms, 192 TFLOP/s, where a library's fp32 product reaches 152; 9,001 rows of five prompts, 12 heads: 229 us.
constexpr int kPlane = 4096, kStage3 = 6 * kPlane;
template <int G>
__global__ void __launch_bounds__(256 * G, 2) k_prompt3(PromptArgs a, Grid grid) {
  __shared__ Stages<G * 2 * kStage3 / 16> shared;
  static_assert(alignof(decltype(shared)) % 128 == 0, "reads xor addresses up to 127");
  __shared__ int window[kWindow], odd[8];  // odd: the last tile of a group's stage that held a NaN or an infinity
  int head, tile;
  if (!block_of(grid, head, tile)) return;
  const int q0 = tile * 128;
  const int w = __builtin_amdgcn_readfirstlane((threadIdx.x >> 6) & 3), g = __builtin_amdgcn_readfirstlane(threadIdx.x >> 8);
  const int lane = threadIdx.x & 63, lr = lane & 31, lk = lane >> 5;
  uint4* const stages = shared.chunk + g * 2 * kStage3 / 16;
  const int e = min(q0 + 128, a.tokens), r0 = q0 + w * 32, row = min(r0 + lr, a.tokens - 1);
  const float* Q = reinterpret_cast<const float*>(a.q) + row * a.qt + head * a.qh + 8 * lk;
  const float* V = reinterpret_cast<const float*>(a.v) + (head / a.group) * a.vh;
  const int cr = (threadIdx.x & 255) >> 3, cc = threadIdx.x & 7;  // the thread's row of its group's tile and its eight dims
  const float *Kc = reinterpret_cast<const float*>(a.k) + (head / a.group) * a.kh + 8 * cc, *Vc = V + 8 * cc;
  float q[4][8], kx[8], vx[8];
#pragma unroll
  for (int s = 0; s < 4; ++s) ld<8>(Q + 16 * s, a.vec, q[s]);
  auto load = [&](int t) {
    const int r = min(max(e - (t + 1) * 32 + cr, 0), a.tokens - 1);
    ld<8>(Kc + r * a.kt, a.vec, kx);
    ld<8>(Vc + r * a.vt, a.vec, vx);
  };
  const uint32_t lds = (uint32_t)(uintptr_t)(lds_void*)stages, put = 128 * cr + 16 * key_chunk(cr, cc), putv = 3 * kPlane + 128 * cr + 16 * value_chunk(cr, cc);
  auto stage = [&](int i) {  // the group's tile i, its terms from the registers
    // What is not finite among the values leaves the tile and is added for the rows that see it: its product with a
    // probability of 0 would reach those that do not (and an infinity in terms is NaN).
    float z = 0.f;
#pragma unroll
    for (int j = 0; j < 8; ++j) z = fmaf(vx[j], 0.f, z);
    if (__builtin_amdgcn_ballot_w64(z != 0.f)) {
#pragma unroll
      for (int j = 0; j < 8; ++j) vx[j] = finite(vx[j]) ? vx[j] : 0.f;
      if (lane == 0) odd[2 * g + (i & 1)] = i;
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) vx[j] *= 0x1p-8f;
    char* to = reinterpret_cast<char*>(stages) + (i & 1) * kStage3;
    bf16x8 k3[3], v3[3];
    terms8<3>(kx, k3);
    terms8<3>(vx, v3);
#pragma unroll
    for (int j = 0; j < 3; ++j) {
      *reinterpret_cast<bf16x8*>(to + put + j * kPlane) = k3[j];
      *reinterpret_cast<bf16x8*>(to + putv + j * kPlane) = v3[j];
    }
  };
  const Borders near = borders_near<256 * G>(a.starts, a.n, q0, window, odd, [&] { load(g); });
  // first keys do not decrease along the rows: of the wave's rows, and of the block's first
  const int lo = first_key(a.starts, a.n, window, near, row), bound = first_key(a.starts, a.n, window, near, q0);
  const int k0 = __builtin_amdgcn_readfirstlane(bound), w0 = __builtin_amdgcn_readlane(lo, 0), f0 = __builtin_amdgcn_readlane(lo, 31);
  const int nt = (e - min(k0, e) + 31) / 32;
  bf16x8 qt[4][3];
#pragma unroll
  for (int s = 0; s < 4; ++s) terms8<3>(q[s], qt[s]);
  float raise = -INFINITY, l = 0.f;  // as in k_prompt16, but for a reference at the maximum: raise is kRaise from the first on
  floatx16 nref, o[2];
#pragma unroll
  for (int v = 0; v < 16; ++v) nref[v] = o[0][v] = o[1][v] = 0.f;
  const int vrow = 4 * lk + ((lane >> 2) & 3), vchunk = value_chunk(vrow, 2 * ((lane >> 4) & 1) + ((lane >> 1) & 1));
  const uint32_t kat = lds + 128 * lr + 16 * (lk ^ (lr & 7)), vat = lds + 3 * kPlane + 128 * vrow + 16 * vchunk + 8 * (lane & 1);
  if (threadIdx.x < 4) odd[threadIdx.x] = -1;
  __syncthreads();
  stage(0);
  __syncthreads();
  for (int i = 0; i * G < nt; ++i) {
    const int t = i * G + g, kt = e - (t + 1) * 32;
    const bool more = (i + 1) * G < nt;
    if (more) load(t + G);
    if (t < nt && kt < r0 + 32 && kt + 32 > w0) {  // uniform
      const uint32_t half = (i & 1) * kStage3;
      auto scores = [&](floatx16& x) {  // onto x, and their maximum
#pragma unroll
        for (int b = 2; b >= 0; --b) {
          bf16x8 kf[4];
          read_keys(kat + half + b * kPlane, kf);
#pragma unroll
          for (int j = 2 - b; j >= 0; --j)
#pragma unroll
            for (int s = 0; s < 4; ++s) x = mfma32(kf[s], qt[s][j], x);
        }
        if (kt + 31 > r0) {
#pragma unroll
          for (int v = 0; v < 16; ++v) x[v] = 8 * (v >> 2) + (v & 3) <= row - kt - 4 * lk ? x[v] : -INFINITY;
        }
        if (kt < f0) {
#pragma unroll
          for (int v = 0; v < 16; ++v) x[v] = 8 * (v >> 2) + (v & 3) >= lo - kt - 4 * lk ? x[v] : -INFINITY;
        }
        float mx = x[0];
#pragma unroll
        for (int v = 1; v < 16; ++v) mx = fmaxf(mx, x[v]);
        return pair_max(mx);
      };
      floatx16 sc = nref;
      float mx = scores(sc);
      const bool up = mx > raise;
      if (__builtin_amdgcn_ballot_w64(up)) {
        if (__builtin_amdgcn_ballot_w64(up && raise > 0.f)) {
          floatx16 x;
#pragma unroll
          for (int v = 0; v < 16; ++v) x[v] = 0.f;
          mx = scores(x);
#pragma unroll
          for (int v = 0; v < 16; ++v) sc[v] = up ? x[v] : sc[v];
        }
        const float next = up ? -mx : nref[0];
        const float f = !up ? 1.f : raise > 0.f ? __builtin_amdgcn_exp2f(fminf(next - nref[0], 0.f) * kScale) : 0.f;
        if (up) raise = kRaise;
        l *= f;
#pragma unroll
        for (int v = 0; v < 16; ++v) {
          o[0][v] *= f;
          o[1][v] *= f;
          sc[v] += up ? next : 0.f;
          nref[v] = next;
        }
      }
      bf16x8 pt[2][3];
#pragma unroll
      for (int s = 0; s < 2; ++s) {
        float p[8];
#pragma unroll
        for (int v = 0; v < 8; ++v) {
          p[v] = __builtin_amdgcn_exp2f(sc[8 * s + v] * kScale);
          l += p[v];
        }
        terms8<3>(p, pt[s]);
      }
#pragma unroll
      for (int b = 2; b >= 0; --b) {
        bf16x8 vf[2][2];
        read_values(vat + half + b * kPlane, vf);
#pragma unroll
        for (int j = 2 - b; j >= 0; --j)
#pragma unroll
          for (int s = 0; s < 2; ++s)
#pragma unroll
            for (int d = 0; d < 2; ++d) o[d] = mfma32(vf[s][d], pt[s][j], o[d]);
      }
      if (__builtin_amdgcn_readfirstlane(odd[2 * g + (i & 1)]) == i) {
#pragma unroll 1
        for (int key = max(kt, 0); key < min(kt + 32, a.tokens); ++key) {
          const float* vp = V + key * a.vt + 4 * lk;
#pragma unroll
          for (int b = 0; b < 8; ++b) {
            float x[4];
            ld<4>(vp + 8 * b, a.vec, x);
#pragma unroll
            for (int j = 0; j < 4; ++j) o[b >> 2][4 * (b & 3) + j] += !finite(x[j]) && key >= lo && key <= row ? x[j] : 0.f;
          }
        }
      }
    }
    if (more) stage(i + 1);
    __syncthreads();
  }
  if (G == 2 && !join(g, w, reinterpret_cast<float*>(shared.chunk), raise > 0.f ? -nref[0] : -INFINITY, l, o)) return;
  const float total = pair_sum(l), inv = total == 0.f ? 0.f : 256.f / total;
  if (r0 + lr >= a.tokens || (!a.clear && (row < near.begin || row >= near.end))) return;
  float* op = reinterpret_cast<float*>(a.out) + ((size_t)row * a.heads + head) * kHeadDim + 4 * lk;
#pragma unroll
  for (int d = 0; d < 2; ++d)
#pragma unroll
    for (int g = 0; g < 4; ++g)
      *reinterpret_cast<floatx4*>(op + d * 32 + 8 * g) =
          floatx4{o[d][4 * g] * inv, o[d][4 * g + 1] * inv, o[d][4 * g + 2] * inv, o[d][4 * g + 3] * inv};
}

template <typename T>
static void prompt32(const PromptArgs& a, hipStream_t st) {
  const Grid g = grid_of(a.tokens, 32, a.heads);
  k_prompt32<T><<<g.blocks, 256, 0, st>>>(a, g);
}

template <int G>
static void prompt3(const PromptArgs& a, hipStream_t st) {
  const Grid g = grid_of(a.tokens, 128, a.heads);
  k_prompt3<G><<<g.blocks, 256 * G, 0, st>>>(a, g);
}

// By the blocks of 128 rows and the mean length, whose causes are: few blocks leave compute units waiting for the longest, and
// then a block's own tiles one after the other are the call's time; many keep all busy, and then what a row costs counts.
// us a call of a graph of one, replayed again and again (small ones take 4 to 8 us more so than among a stream's other calls;
// sequences x rows x heads), bf16:
//   few blocks of long sequences: two groups of waves share a block's keys, 64 keys at a time (2,048 x 20: 32; one group 42;
//     2 x 4,000 x 8: 68 / 92; but 10 x 512 x 14: 37 / 28)
//   up to some more: two groups of 32 keys at a time and four waves a SIMD (4 x 4,200 x 8, 1,056 blocks: 126, one group 163; 4 x
//     1,813 x 20: 61 / 69; 6 x 8,533 x 8: 687 / 707; but 9 x 1,896 x 24, 3,200 blocks: 176 / 166; one sequence, 810 blocks of
//     10,294 x 10: 206 / 224, 1,024 of 4,096 x 32: 104 / 105, but 1,944 of 10,294 x 24: 422 / 414)
//   very many of very long sequences: 256 rows a block, half the reads from LDS (32,768 x 32: 4,690 / 4,860; but 16,384 x 6:
//     446 / 277)
//   others: one group, 32 keys at a time, four waves a SIMD (96 of 224 x 20: 62; 64 keys and two waves 84)
// fp32: two groups as above (2 x 3,200 x 8: 166 / 216; but 2,800 x 32, 704 blocks: 210 / 197); below 256 blocks 32 rows a block,
// its waves taking its keys in turn (224 x 20: 16.4, k_prompt3 20.3; 1,000 x 32: 49 / 53).
void prompt_attend(const PromptArgs& a, hipStream_t st) {
  const long long blocks = (a.tokens + 127) / 128 * (long long)a.heads, mean = a.tokens / a.n;
  const bool few = blocks <= (a.bf16_data ? 256 : 384), some = blocks <= (a.bf16_data ? 640 : 576);
  const bool shared = few ? mean >= 256 : some && mean >= (a.bf16_data ? 1536 : 1024);
  if (!a.bf16_data) {
    if (blocks < 256) return prompt32<float>(a, st);
    if (shared) return prompt3<2>(a, st);
    return prompt3<1>(a, st);
  }
  // k_prompt16 reads 16 bytes at a time, 64 rows by 32-bit offsets; rows off a 16-byte border take single elements and 32-row blocks
  // (8,192 x 12: 813 us for 166, 96 of 224 x 20: 322 / 59, 224 x 20: 16.7 / 16.1)
  if (!a.vec || std::max(a.kt, a.vt) > 1 << 24) return prompt32<bf16>(a, st);
  if (shared) return prompt16<1, 2, 2, 2, 2>(a, st);
  if (mean >= 16384 && blocks >= 4096) return prompt16<2, 1, 2, 1, 3>(a, st);
  if (blocks <= (mean < 256 ? 0 : mean < 1024 ? 512 : a.n == 1 ? 1024 : mean < 4096 ? 1536 : 3584)) return prompt16<1, 1, 4, 2, 2>(a, st);
  prompt16<1, 1, 4, 1, 2>(a, st);
}

}  // namespace wf
