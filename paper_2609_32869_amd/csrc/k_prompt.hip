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

void prompt_attend(const PromptArgs& a, hipStream_t st) {
  const dim3 grid((a.tokens + 31) / 32, a.heads);
  if (a.bf16_data) k_prompt32<bf16><<<grid, 256, 0, st>>>(a);
  else k_prompt32<float><<<grid, 256, 0, st>>>(a);
}

}  // namespace wf
