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

// First key of row t: the largest border <= t, where t lies in a sequence; t + 1 (no key) elsewhere.
__device__ __forceinline__ int first_key(const int* starts, int n, int t) {
  if (t < starts[0] || t >= starts[n]) return t + 1;
  int a = 0, b = n;  // starts[a] <= t < starts[b]
  while (b - a > 1) {
    const int m = (a + b) >> 1;
    if (starts[m] <= t) a = m;
    else b = m;
  }
  return min(max(starts[a], 0), t + 1);
}

// 4 consecutive elements of a row.
template <typename T>
__device__ __forceinline__ floatx4 ld4(const T* p, int vec) {
  if (!vec) return floatx4{to_f(p[0]), to_f(p[1]), to_f(p[2]), to_f(p[3])};
  if constexpr (sizeof(T) == 4) {
    return *reinterpret_cast<const floatx4*>(p);
  } else {
    const uint2 v = *reinterpret_cast<const uint2*>(p);
    return floatx4{__uint_as_float(v.x << 16), __uint_as_float(v.x & 0xffff0000u), __uint_as_float(v.y << 16),
                   __uint_as_float(v.y & 0xffff0000u)};
  }
}
}  // namespace

// Block: (32 rows, head), four waves that take every fourth tile of 32 keys and join their
// maxima, sums and outputs in LDS at the end.  Products on v_mfma_f32_32x32x2_f32:
//   S^T = K q^T  step s: dims s (lanes 0..31) and 32 + s (lanes 32..63); a lane gets keys
//                8 (v / 4) + 4 (lane / 32) + v % 4 of row lane % 32
//   O^T += V^T P^T  step v: the two half-waves' keys of element v, so the probabilities are the
//                operand as they are, and a lane's value is V[key][lane % 32 + 32 nt]
template <typename T>
__global__ void __launch_bounds__(256) k_prompt32(PromptArgs a) {
  __shared__ float wm[4][32], wl[4][32], wo[4][32][68];
  const int head = blockIdx.y, q0 = (gridDim.x - 1 - blockIdx.x) * 32;
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, lr = lane & 31, lk = lane >> 5;
  const int row = min(q0 + lr, a.tokens - 1);
  const int lo = first_key(a.starts, a.n, row), hi = lo > row ? lo : row + 1;  // keys [lo, hi)
  int k0 = hi > lo ? lo : a.tokens, k1 = hi > lo ? hi : 0;
#pragma unroll
  for (int m = 1; m < 32; m <<= 1) {
    k0 = min(k0, __shfl_xor(k0, m));
    k1 = max(k1, __shfl_xor(k1, m));
  }
  k0 = __builtin_amdgcn_readfirstlane(k0);
  k1 = __builtin_amdgcn_readfirstlane(k1);
  const T* Q = reinterpret_cast<const T*>(a.q) + row * a.qt + head * a.qh + 32 * lk;
  const T* K = reinterpret_cast<const T*>(a.k) + (head / a.group) * a.kh + 32 * lk;
  const T* V = reinterpret_cast<const T*>(a.v) + (head / a.group) * a.vh;
  floatx4 q[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) q[j] = ld4(Q + 4 * j, a.vec);
  float m = -INFINITY, l = 0.f;
  floatx16 o[2];
#pragma unroll
  for (int nt = 0; nt < 2; ++nt)
#pragma unroll
    for (int v = 0; v < 16; ++v) o[nt][v] = 0.f;
  for (int kt = k0 + 32 * w; kt < k1; kt += 128) {
    floatx16 s;
#pragma unroll
    for (int v = 0; v < 16; ++v) s[v] = 0.f;
    const T* kp = K + min(kt + lr, a.tokens - 1) * a.kt;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const floatx4 x = ld4(kp + 4 * j, a.vec);
#pragma unroll
      for (int e = 0; e < 4; ++e) s = __builtin_amdgcn_mfma_f32_32x32x2f32(x[e], q[j][e], s, 0, 0, 0);
    }
    uint32_t out = 0;  // bit v: the row does not see the key
    float mx = -INFINITY;
#pragma unroll
    for (int v = 0; v < 16; ++v) {
      const int key = kt + 8 * (v >> 2) + 4 * lk + (v & 3);
      if (key < lo || key >= hi) {
        s[v] = -INFINITY;
        out |= 1u << v;
      }
      mx = fmaxf(mx, s[v]);
    }
    const float mn = fmaxf(m, pair_max(mx)), base = mn == -INFINITY ? 0.f : mn;
    const float f = __builtin_amdgcn_exp2f((m - base) * kScale);
    m = mn;
    l *= f;
#pragma unroll
    for (int nt = 0; nt < 2; ++nt)
#pragma unroll
      for (int v = 0; v < 16; ++v) o[nt][v] *= f;
#pragma unroll
    for (int v = 0; v < 16; ++v) {
      s[v] = __builtin_amdgcn_exp2f((s[v] - base) * kScale);
      l += s[v];
    }
    float x[2][16];
    bool odd = false;
#pragma unroll
    for (int v = 0; v < 16; ++v) {
      const T* vp = V + min(kt + 8 * (v >> 2) + 4 * lk + (v & 3), a.tokens - 1) * a.vt + lr;
      x[0][v] = to_f(vp[0]);
      x[1][v] = to_f(vp[32]);
      odd |= !finite(x[0][v]) || !finite(x[1][v]);
    }
    // A NaN or an infinity times a probability of 0 would reach the rows that do not see it: such
    // values leave the product and are counted, for the rows that do, by two products of ones.
    if (__builtin_amdgcn_ballot_w64(odd) && __builtin_amdgcn_ballot_w64(out != 0)) {
#pragma unroll
      for (int nt = 0; nt < 2; ++nt) {
        floatx16 up, down;
#pragma unroll
        for (int v = 0; v < 16; ++v) up[v] = down[v] = 0.f;
#pragma unroll
        for (int v = 0; v < 16; ++v) {
          const float y = x[nt][v], sees = out >> v & 1 ? 0.f : 1.f;
          up = __builtin_amdgcn_mfma_f32_32x32x2f32(y != y || y == INFINITY ? 1.f : 0.f, sees, up, 0, 0, 0);
          down = __builtin_amdgcn_mfma_f32_32x32x2f32(y != y || y == -INFINITY ? 1.f : 0.f, sees, down, 0, 0, 0);
          x[nt][v] = finite(y) ? y : 0.f;
        }
#pragma unroll
        for (int v = 0; v < 16; ++v) {
          if (up[v] > 0.f) o[nt][v] += INFINITY;
          if (down[v] > 0.f) o[nt][v] -= INFINITY;
        }
      }
    }
#pragma unroll
    for (int nt = 0; nt < 2; ++nt)
#pragma unroll
      for (int v = 0; v < 16; ++v) o[nt] = __builtin_amdgcn_mfma_f32_32x32x2f32(x[nt][v], s[v], o[nt], 0, 0, 0);
  }
  l = pair_sum(l);
  if (lane < 32) {
    wm[w][lr] = m;
    wl[w][lr] = l;
  }
  // lane: row lr, dims 32 nt + 8 (v / 4) + 4 lk + v % 4
#pragma unroll
  for (int nt = 0; nt < 2; ++nt)
#pragma unroll
    for (int g = 0; g < 4; ++g)
      *reinterpret_cast<floatx4*>(&wo[w][lr][32 * nt + 8 * g + 4 * lk]) =
          floatx4{o[nt][4 * g], o[nt][4 * g + 1], o[nt][4 * g + 2], o[nt][4 * g + 3]};
  __syncthreads();
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
    if (!a.clear && (r < a.starts[0] || r >= a.starts[a.n])) continue;
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
__device__ __forceinline__ floatx16 mfma32(bf16x8 a, bf16x8 b, floatx16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
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
  // the wave's rows, the keys [lo, hi) that each sees, and those that any or all of the wave's do
  int row[NQ], lo[NQ], hi[NQ], w0 = a.tokens, w1 = 0, f0 = 0, f1 = a.tokens;
  bf16x8 qf[NQ][4];
#pragma unroll
  for (int u = 0; u < NQ; ++u) {
    row[u] = q0 + (w * NQ + u) * 32 + lr;
    const int r = min(row[u], a.tokens - 1);
    lo[u] = first_key(a.starts, a.n, r);
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
  __shared__ int first[4], last[4], from[4], to[4], odd[4];  // odd: the last tile of a stage that held a NaN or an infinity
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
          const floatx4 x = ld4(vp + 8 * e, 1);
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
    if (!a.clear && (row[u] < a.starts[0] || row[u] >= a.starts[a.n])) continue;
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

void prompt_attend(const PromptArgs& a, hipStream_t st) {
  const dim3 grid((a.tokens + 31) / 32, a.heads);
  if (a.bf16_data && a.vec) {
    if (a.tokens > 4096) return prompt16<2>(a, st);
    return prompt16<1>(a, st);
  }
  if (a.bf16_data) k_prompt32<bf16><<<grid, 256, 0, st>>>(a);
  else k_prompt32<float><<<grid, 256, 0, st>>>(a);
}

}  // namespace wf
