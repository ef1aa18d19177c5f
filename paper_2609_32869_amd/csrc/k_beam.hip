// Beam search: the k best continuations over a request's beams and vocabulary, and the
// page tables of the beams that were chosen.
#include <algorithm>
#include <type_traits>

#include "wf_operand.h"
#include "wf_ops.h"

namespace wf {

// ---------------------------------------------------------------- selection
// score(b, v) = s_b + x_bv - log sum_u exp(x_bu).  A beam's order over v is the order of
// its logits, so the row kernel keeps the k best logits of each piece of a row beside the
// piece's maximum and sum of exponentials; the beams meet in 64-bit scores in the merge.
//
// Row kernel: a block per (piece of kBeamPiece columns, row), one read of the logits into
// registers, 32 per thread, a wave's columns together.  With the block's lanes in k groups
// or more, the least of the groups' maxima bounds the piece's k-th best from below; the
// few values that reach it go to LDS and are ranked by counting.  Where a wave has many of
// them (near-equal logits; pieces so short that some groups hold nothing and all is kept),
// the wave's own bound is the k-th best of its lanes' maxima, found bit by bit with ballots,
// equal ones by column: KL lanes at most, whose values fit its KL * R places with any number of
// ties.  Not waiting for the places to run out, a call of 62 x 8 rows of 367 logits, 3 best,
// takes 12.4 us instead of 22.9, of 20 x 16 rows of 4,624, 32 best, 20.4 instead of 55.8.
// 768 rows of 51,864 logits: fp32 32 us, the copy rate of 4.9 TB/s.  bf16 33.6 us, half that rate: a wave's 525 vector
// instructions (16 a logit of a lane, the exponential four of them; 32 are the exponentials themselves) take about 60% of
// the SIMDs' time, and for half of its own a wave waits, for its logits before and at the barriers after them.  64 logits a
// thread: 34 and 41 us, fewer waves a SIMD.
constexpr int kBeamRegs = 32, kBeamPiece = 256 * kBeamRegs;

// Larger value, larger integer, both zeros alike; NaN and -inf (no candidates) at 0.
__device__ __forceinline__ uint32_t order_of(float x) {
  const uint32_t u = __float_as_uint(x + 0.f);  // -0 + 0 = +0
  return !(x > -INFINITY) ? 0u : u >> 31 ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float value_of(uint32_t o) { return __uint_as_float(o >> 31 ? o & 0x7fffffffu : ~o); }

// Bits of the r-th largest of the active lanes' words, from `high` down to `low`, appended to
// t; r becomes the rank among the lanes that hold those bits.
template <int high, int low>
__device__ __forceinline__ void wave_kth(uint32_t w, bool active, uint32_t& t, int& r) {
#pragma unroll
  for (int bit = high; bit >= low; --bit) {
    const int c = __popcll(__ballot(active && (w >> bit) == (t >> bit | 1u)));
    const bool up = c >= r;
    t = up ? t | 1u << bit : t;
    r = up ? r : r - c;
  }
}
__device__ __forceinline__ float max8(float v) {  // over 8 lanes, in each of them
  v = fmaxf(v, dpp<kDppXor1>(v));
  v = fmaxf(v, dpp<kDppXor2>(v));
  return fmaxf(v, dpp<kDppHalfMirror>(v));
}
// sum over a row of 16 lanes by DPP moves of the two halves, in every lane of the row
template <int CTRL>
__device__ __forceinline__ double dpp_d(double v) {
  const uint64_t u = __builtin_bit_cast(uint64_t, v);
  const uint32_t lo = __builtin_amdgcn_update_dpp(0, (int)(uint32_t)u, CTRL, 0xf, 0xf, false);
  const uint32_t hi = __builtin_amdgcn_update_dpp(0, (int)(u >> 32), CTRL, 0xf, 0xf, false);
  return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}
__device__ __forceinline__ double sum16d(double v) {
  v += dpp_d<kDppXor1>(v);
  v += dpp_d<kDppXor2>(v);
  v += dpp_d<kDppHalfMirror>(v);
  return v + dpp_d<kDppMirror>(v);
}
__device__ __forceinline__ double lane_d(double v, int l) {
  const uint64_t u = __builtin_bit_cast(uint64_t, v);
  const uint32_t lo = __builtin_amdgcn_readlane((int)(uint32_t)u, l), hi = __builtin_amdgcn_readlane((int)(u >> 32), l);
  return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}
// whole-wave sum, uniform result
__device__ __forceinline__ double wave_sum_d(double v) {
  v = sum16d(v);
  return (lane_d(v, 0) + lane_d(v, 16)) + (lane_d(v, 32) + lane_d(v, 48));
}

// 8 consecutive logits or suppression bytes.  Rows start anywhere (every second bf16 row of
// an odd vocabulary lies off 4 bytes), so the loads are 16 bytes at the elements'
// alignment: columns are grouped by number, not by address, and rows of equal values have
// equal sums.
template <typename T>
struct Eight {
  T v[8];
  __device__ __forceinline__ void load(const T* p) { __builtin_memcpy(v, p, sizeof(v)); }
};

// The thread's R logits: eights from columns v0 + 512 i on, of which the row's last, partial
// one is read as the row's last eight columns (eight_at) and keeps those that are its own.
// The loads are issued together, without a condition.  Columns past the row and suppressed
// ones are -inf.
__device__ __forceinline__ int eight_at(int v, int vocab) { return max(min(v, vocab - 8), 0); }
template <typename T, int R>
__device__ __forceinline__ void load_logits(const T* x, const uint8_t* sup, int v0, int vocab, float* y) {
  constexpr int N = R / 8;
  if (vocab >= 8) {
    Eight<T> e[N];
#pragma unroll
    for (int i = 0; i < N; ++i) e[i].load(x + eight_at(v0 + 512 * i, vocab));
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int i = 0; i < R; ++i) y[i] = to_f(e[i / 8].v[i % 8]);
  } else {  // a row shorter than an eight
#pragma unroll
    for (int i = 0; i < R; ++i) y[i] = i < 8 ? to_f(x[min(i, vocab - 1)]) : -INFINITY;
  }
  if (__builtin_amdgcn_readfirstlane(v0) + 64 * R > vocab) {  // the row's last columns
#pragma unroll
    for (int i = 0; i < R; ++i) {
      const int v = v0 + 512 * (i / 8), c = eight_at(v, vocab) + i % 8;
      if (c < v || c >= vocab) y[i] = -INFINITY;
    }
  }
  if (sup) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const uint8_t* p = sup + eight_at(v0 + 512 * i, vocab);
      uint64_t m = 0;
      if (vocab >= 8) __builtin_memcpy(&m, p, 8);
      else
        for (int j = 0; j < vocab; ++j) m |= (uint64_t)p[j] << (8 * j);
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (m >> (8 * j) & 255) y[8 * i + j] = -INFINITY;
    }
  }
}

// KL: groups of the block's lanes, and lanes of a wave that survive at most; k <= KL
template <typename T, int KL>
__global__ void __launch_bounds__(256) k_beam_rows(BeamSelectArgs a) {
  constexpr int R = kBeamRegs, kSeg = KL * R;  // a wave's survivors
  constexpr int kMany = 64;
  static_assert(kMany <= kSeg, "a wave's survivors fit their places");
  __shared__ __align__(16) uint64_t keys[4 * kSeg];
  __shared__ float gm[KL], wm[4];
  __shared__ double ws[4];
  __shared__ int wn[4];
  const int r = blockIdx.x, b = blockIdx.z, row = r * a.beams + b, t = threadIdx.x, lane = t & 63;
  const int w = __builtin_amdgcn_readfirstlane(t >> 6);
  const T* x = reinterpret_cast<const T*>(a.logits) + r * a.sr + b * a.sb + (b < kRows ? 0 : a.far);
  const int v0 = blockIdx.y * 256 * R + w * 64 * R + 8 * lane;
  float y[R];
  load_logits<T, R>(x, a.suppress, v0, a.vocab, y);
  float m = -INFINITY;
#pragma unroll
  for (int i = 0; i < R; ++i) m = fmaxf(m, y[i]);
  // maxima of the block's KL groups of 256 / KL lanes
  {
    const float g = KL == 16 ? max16(m) : max8(m);
    if (lane % (256 / KL) == 0) gm[t / (256 / KL)] = g;
  }
  // sum of exponentials relative to the lane's maximum, eight at a time in 32 bits, then 64.  Powers of two, m log2(e)
  // rounded once and what that took put back on the sum.  It took up to half a step of m log2(e), a quarter at 2^22 and
  // at 1e10 more powers of two than there are, so larger logits go by difference
  constexpr float log2e = 1.44269504088896f;
  const float base = m == -INFINITY ? 0.f : m;
  double sum = 0;
  if (__ballot(fabsf(base) > 0x1p22f) == 0) {
    const float mc = base * log2e, took = fmaf(base, log2e, -mc);
#pragma unroll
    for (int i = 0; i < R; i += 8) {
      float p = 0.f;
#pragma unroll
      for (int e = 0; e < 8; ++e) p += __builtin_amdgcn_exp2f(fmaf(y[i + e], log2e, -mc));
      sum += (double)p;
    }
    sum *= (double)__builtin_amdgcn_exp2f(-took);
  } else {
#pragma unroll
    for (int i = 0; i < R; i += 8) {
      float p = 0.f;
#pragma unroll
      for (int e = 0; e < 8; ++e) p += __builtin_amdgcn_exp2f((y[i + e] - base) * log2e);
      sum += (double)p;
    }
  }
  // to the wave's maximum; a lane of no values holds 0, or NaN, which stays
  const float M = wave_max(m);
  if (m != -INFINITY) sum *= (double)__builtin_amdgcn_exp2f((m - M) * log2e);
  sum = wave_sum_d(sum);
  if (lane == 0) {
    wm[w] = M;
    ws[w] = sum;
  }
  __syncthreads();
  // the least of KL groups' maxima, or of half or a quarter as many groups where k allows it
  float g[KL];
#pragma unroll
  for (int i = 0; i < KL; ++i) g[i] = gm[i];
  float least = INFINITY;
  if (a.k <= KL / 4) {
#pragma unroll
    for (int i = 0; i < KL; i += 4) least = fminf(least, fmaxf(fmaxf(g[i], g[i + 1]), fmaxf(g[i + 2], g[i + 3])));
  } else if (a.k <= KL / 2) {
#pragma unroll
    for (int i = 0; i < KL; i += 2) least = fminf(least, fmaxf(g[i], g[i + 1]));
  } else {
#pragma unroll
    for (int i = 0; i < KL; ++i) least = fminf(least, g[i]);
  }
  least = fmaxf(least, -__FLT_MAX__);  // a group of no values: every value is kept
  uint64_t lanes = __ballot(m >= least);
  uint32_t col = ~0u;
  int over = 0;
  if (__popcll(lanes) > KL || least == -__FLT_MAX__) {
#pragma unroll
    for (int i = 0; i < R; ++i) over += __popcll(__ballot(y[i] >= least));
  }
  if (over > kMany && __popcll(lanes) >= a.k) {  // fewer lanes than k: all their values fit
    const uint32_t best = order_of(m);
    uint32_t bound = 0;
    int need = a.k;
    bool active = best != 0;
    wave_kth<31, 0>(best, active, bound, need);
    least = value_of(bound);
    lanes = __ballot(m >= least);
    if (__popcll(lanes) > KL) {  // more equal maxima than that: the first of them by column
      int at = 0;
#pragma unroll
      for (int i = R - 1; i >= 0; --i)
        if (y[i] == m) at = eight_at(v0 + 512 * (i / 8), a.vocab) + i % 8;
      uint32_t inv = 0;
      active = best == bound;
      wave_kth<31, 0>(~(uint32_t)at, active, inv, need);
      col = ~inv;
      lanes = __ballot(m > least || (m == least && (uint32_t)at <= col));
    }
  }
  // the wave's survivors: value and place first, as little as possible per value, then made into keys in place
  int mine = 0;
  if (lanes != 0) {
    uint2* seg = reinterpret_cast<uint2*>(keys + w * kSeg);
    auto gather = [&](auto ties) {
#pragma unroll
      for (int i = 0; i < R; ++i) {
        bool in = y[i] >= least;
        if constexpr (decltype(ties)::value)
          in = in && (y[i] > least || (uint32_t)(eight_at(v0 + 512 * (i / 8), a.vocab) + i % 8) <= col);
        const uint64_t mask = __ballot(in);
        if (mask != 0) {  // uniform, and rare
          const int at = __builtin_amdgcn_mbcnt_hi((uint32_t)(mask >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)mask, mine));
          if (in) seg[at] = make_uint2(__float_as_uint(y[i]), i << 6 | lane);
          mine += __popcll(mask);
        }
      }
    };
    if (col == ~0u) gather(std::false_type{});
    else gather(std::true_type{});
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    for (int u = lane; u < mine; u += 64) {
      const uint2 e = seg[u];
      const int i = e.y >> 6, v = v0 - 8 * lane + 8 * (int)(e.y & 63) + 512 * (i / 8), c = eight_at(v, a.vocab) + i % 8;
      keys[w * kSeg + u] = (uint64_t)order_of(__uint_as_float(e.x)) << 32 | (uint32_t)~c;
    }
  }
  if (lane == 0) wn[w] = mine;
  __syncthreads();
  const size_t piece = (size_t)row * gridDim.y + blockIdx.y;
  // rank by counting larger keys (a larger value, then a lower column)
  int n = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) n += wn[i];
  for (int i = t; i < n; i += 256) {
    int s = i, q = 0;
#pragma unroll
    for (int j = 0; j < 3; ++j)
      if (q == j && s >= wn[j]) {
        s -= wn[j];
        q = j + 1;
      }
    const uint64_t key = keys[q * kSeg + s];
    int rank = 0;
    for (int j = 0; j < 4; ++j) {
      const int e = wn[j];
      for (int u = 0; u < e; u += 4) {  // entries past e lie in the segment (kSeg is a multiple of 4) and do not count
        uint64_t z[4];
#pragma unroll
        for (int d = 0; d < 4; ++d) z[d] = keys[j * kSeg + u + d];
#pragma unroll
        for (int d = 0; d < 4; ++d) rank += u + d < e && z[d] > key;
      }
    }
    if (rank < a.k) {
      a.pv[piece * a.k + rank] = value_of((uint32_t)(key >> 32));
      a.pi[piece * a.k + rank] = (int)~(uint32_t)key;
    }
  }
  for (int i = n + t; i < a.k; i += 256) {
    a.pv[piece * a.k + i] = -INFINITY;
    a.pi[piece * a.k + i] = -1;
  }
  if (t == 0) {
    float mm = wm[0];
    for (int i = 1; i < 4; ++i) mm = fmaxf(mm, wm[i]);
    double total = 0;
    for (int i = 0; i < 4; ++i)
      total += ws[i] * (double)__expf((wm[i] == -INFINITY ? mm : wm[i]) - (mm == -INFINITY ? 0.f : mm));
    a.pm[piece] = mm;
    a.ps[piece] = total;
  }
}

// Merge: a block per request.  16 lanes a row join its pieces' sums; then the pieces'
// candidates by 64-bit score, the first M of a thread held in registers (2 below 512
// candidates, 4 up to 1,024, else 16: 3,584 of 16 beams, 32 best, 16.7 us with 4, 13.1 with 16).
// The k-th best is bounded by the best of the waves' k-th best lanes; from 512 candidates on
// they are mixed over the waves and the least of the waves' k/4-th best lanes bounds it more
// closely (3,584 candidates: 13 us instead of 41; 350: 4.8 instead of 4.5).  Scores for that are rounded to 32 bits, which keeps
// the order, and cut to 24 (with 16, cumulative scores of some hundred lie too close, 350
// candidates all survive: 42 us instead of 7).  More survivors than the array holds, which
// takes that many nearly equal scores, are chosen one by one.  One request of five beams
// 4.8 us, 96 of eight 7.2: a chain of short phases between barriers, not bytes (1.3 MB of
// candidates at 96).
constexpr int kMergeList = 1024;
// ties: order = beam * 2^20 + column
__device__ __forceinline__ bool ahead(double s, int o, double t, int p) { return s > t || (s == t && o < p); }

template <int M, bool MIX>
__global__ void __launch_bounds__(256) k_beam_merge(BeamSelectArgs a, int np) {
  __shared__ double top[kMaxBeams], rest[kMaxBeams], ls[kMergeList], bs[4];
  __shared__ int lo[kMergeList], bo[4], count;
  __shared__ uint32_t tv[4];
  const int r = blockIdx.x, t = threadIdx.x, lane = t & 63, w = t >> 6;
  const int per = np * a.k, total = a.beams * per;
  const size_t first = (size_t)r * total;
  // MIX: candidates in turn over the waves and, each time elsewhere, over their lanes
  auto place = [&](int u) {
    const int l = (lane + 9 * u) & 63;
    return 256 * u + (MIX ? 4 * l + ((w + l) & 3) : t);
  };
  float xv[M];
  int xi[M];
#pragma unroll
  for (int i = 0; i < M; ++i) {
    const size_t at = first + min(place(i), total - 1);
    xv[i] = a.pv[at];
    xi[i] = a.pi[at];
  }
  {
    const int b = min(t >> 4, a.beams - 1), p0 = t & 15;
    const size_t row = ((size_t)r * a.beams + b) * np;
    const float sc = a.scores[(size_t)r * a.beams + b], m0 = a.pm[row + min(p0, np - 1)];
    const double s0 = a.ps[row + min(p0, np - 1)];
    float m = m0;
    for (int p = p0 + 16; p < np; p += 16) m = fmaxf(m, a.pm[row + p]);
    m = max16(m);
    auto part = [&](float pm, double ps) { return pm == -INFINITY && ps == 0 ? 0 : ps * exp((double)pm - (double)m); };
    double s = p0 < np ? part(m0, s0) : 0;
    for (int p = p0 + 16; p < np; p += 16) s += part(a.pm[row + p], a.ps[row + p]);
    s = sum16d(s);
    // score = (x - m) + (s_b - log sum): the difference is exact enough at any magnitude; NaN where the row or the
    // beam offers nothing
    if (p0 == 0 && t >> 4 < a.beams) {
      top[b] = m;
      rest[b] = sc < INFINITY ? (double)sc - log(s) : NAN;
    }
  }
  if (t == 0) count = 0;
  __syncthreads();
  // score and order of candidate i, whose logit and column are x and c; false: none
  auto score = [&](int i, float x, int c, double& s, int& o) {
    const int b = min(i, total - 1) / per;
    s = ((double)x - top[b]) + rest[b];
    o = b << 20 | c;
    return i < total && c >= 0 && s > -INFINITY;
  };
  double rs[M];
  int ro[M];
  bool rl[M];
  uint32_t best = 0;
#pragma unroll
  for (int i = 0; i < M; ++i) {
    rl[i] = score(place(i), xv[i], xi[i], rs[i], ro[i]);
    if (rl[i]) best = max(best, order_of((float)rs[i]));
  }
  for (int i = t + 256 * M; i < total; i += 256) {
    double s;
    int o;
    if (score(i, a.pv[first + i], a.pi[first + i], s, o)) best = max(best, order_of((float)s));
  }
  const bool active = best != 0;
  uint32_t bound = 0;
  int need = MIX ? (a.k + 3) / 4 : a.k;
  if (__popcll(__ballot(active)) >= need) wave_kth<31, 8>(best, active, bound, need);
  if (lane == 0) tv[w] = bound;
  __syncthreads();
  bound = MIX ? min(min(tv[0], tv[1]), min(tv[2], tv[3])) : max(max(tv[0], tv[1]), max(tv[2], tv[3]));
  auto keep = [&](double s, int o) {
    const int j = atomicAdd(&count, 1);
    if (j < kMergeList) {
      ls[j] = s;
      lo[j] = o;
    }
  };
#pragma unroll
  for (int i = 0; i < M; ++i)
    if (rl[i] && order_of((float)rs[i]) >= bound) keep(rs[i], ro[i]);
  for (int i = t + 256 * M; i < total; i += 256) {
    double s;
    int o;
    if (score(i, a.pv[first + i], a.pi[first + i], s, o) && order_of((float)s) >= bound) keep(s, o);
  }
  __syncthreads();
  const int n = count;
  auto put = [&](int rank, double s, int o) {
    a.out_score[(size_t)r * a.k + rank] = (float)s;
    a.out_beam[(size_t)r * a.k + rank] = o < 0 ? -1 : o >> 20;
    a.out_token[(size_t)r * a.k + rank] = o < 0 ? -1 : o & ((1 << 20) - 1);
  };
  if (n <= kMergeList) {
    for (int i = t; i < n; i += 256) {
      const double s = ls[i];
      const int o = lo[i];
      int rank = 0;
      for (int j = 0; j < n; j += 4) {  // entries past n lie in the array and do not count
        double z[4];
        int q[4];
#pragma unroll
        for (int d = 0; d < 4; ++d) {
          z[d] = ls[j + d];
          q[d] = lo[j + d];
        }
#pragma unroll
        for (int d = 0; d < 4; ++d) rank += j + d < n && ahead(z[d], q[d], s, o);
      }
      if (rank < a.k) put(rank, s, o);
    }
    for (int i = n + t; i < a.k; i += 256) put(i, -INFINITY, -1);
    return;
  }
  double ps = INFINITY;
  int po = -1;
  for (int j = 0; j < a.k; ++j) {
    double s1 = -INFINITY;
    int o1 = 0x7fffffff;
    for (int i = t; i < total; i += 256) {
      double s;
      int o;
      if (score(i, a.pv[first + i], a.pi[first + i], s, o) && ahead(ps, po, s, o) && ahead(s, o, s1, o1)) {
        s1 = s;
        o1 = o;
      }
    }
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const double s2 = __shfl_xor(s1, o);
      const int o2 = __shfl_xor(o1, o);
      if (ahead(s2, o2, s1, o1)) {
        s1 = s2;
        o1 = o2;
      }
    }
    if (lane == 0) {
      bs[w] = s1;
      bo[w] = o1;
    }
    __syncthreads();
    for (int i = 0; i < 4; ++i)
      if (ahead(bs[i], bo[i], s1, o1)) {
        s1 = bs[i];
        o1 = bo[i];
      }
    ps = s1;
    po = o1;
    if (t == 0) put(j, s1, o1);
    __syncthreads();
  }
}

int beam_pieces(int vocab) { return (vocab + kBeamPiece - 1) / kBeamPiece; }

static size_t up256(size_t v) { return (v + 255) / 256 * 256; }
size_t beam_space_bytes(int n, int beams, int vocab, int k) {
  const size_t pieces = (size_t)n * beams * beam_pieces(vocab);
  return up256(pieces * 8) + up256(pieces * 4) + 2 * up256(pieces * k * 4);
}
void beam_space(BeamSelectArgs& a, char* space) {
  const size_t pieces = (size_t)a.n * a.beams * beam_pieces(a.vocab);
  a.ps = reinterpret_cast<double*>(space);
  a.pm = reinterpret_cast<float*>(space += up256(pieces * 8));
  a.pv = reinterpret_cast<float*>(space += up256(pieces * 4));
  a.pi = reinterpret_cast<int*>(space += up256(pieces * a.k * 4));
}

void beam_select(const BeamSelectArgs& a, hipStream_t st) {
  const int np = beam_pieces(a.vocab);
  const dim3 grid(a.n, np, a.beams);
  auto launch = [&](auto tag) {
    using T = decltype(tag);
    if (a.k <= 16) k_beam_rows<T, 16><<<grid, 256, 0, st>>>(a);
    else k_beam_rows<T, kMaxCand><<<grid, 256, 0, st>>>(a);
  };
  if (a.bf16_logits) launch(bf16{});
  else launch(0.f);
  const int total = a.beams * np * a.k;
  if (total < 512) k_beam_merge<2, false><<<a.n, 256, 0, st>>>(a, np);
  else if (total <= 1024) k_beam_merge<4, true><<<a.n, 256, 0, st>>>(a, np);
  else k_beam_merge<16, true><<<a.n, 256, 0, st>>>(a, np);
}

// ---------------------------------------------------------------- page tables
// Beam j continues beam parents[j] of its request: it keeps that beam's pages.  Full
// pages are never written again, so beams share them.  The page of the next position
// is one beam's own: the first beam that keeps a part-filled page goes on in it, every
// other one gets the pool's next unreferenced page and a copy.
//
// Grid (region x part of a page, request).  Every block works the request's pages out for
// itself (a few hundred table entries, a bit per page of the cache in LDS), so that one
// launch does it all.  The first block writes the tables, each copies its part of the
// copied pages in its region.  64 regions of 40 KB pages, 5 beams: one request 6.7 us, four
// dependent round trips; eight requests 11.4 us, the copied pages' bytes (floor 8.9).
constexpr int kReorderThreads = 256;
__global__ void __launch_bounds__(kReorderThreads) k_cache_reorder(ReorderArgs a, int parts) {
  __shared__ unsigned used[kMaxPages / 32];
  __shared__ int parent[kMaxBeams], mine[kMaxBeams], fresh[kMaxBeams];
  __shared__ int2 copy[kMaxBeams];  // (source, destination)
  __shared__ int ncopy;
  const int r = blockIdx.y, t = threadIdx.x;
  const bool lead = blockIdx.x == 0;
  const int* T = a.tables + r * a.tr;
  int* N = a.new_tables + r * a.nr;
  const int* pool = a.pool + (size_t)r * a.pool_pages;
  // independent loads first
  const int p0 = pool[0], q0 = pool[min(t, a.pool_pages - 1)], raw = a.lens[r];
  if (t < kMaxBeams) {
    const int p = t < a.beams ? a.parents[(size_t)r * a.beams + t] : -1;
    parent[t] = p < a.beams ? p : -1;
    fresh[t] = -1;
  }
  for (int i = t; i < (a.n_pages + 31) / 32; i += kReorderThreads) used[i] = 0;
  __syncthreads();
  const int len = (int)min((long long)max(raw, 0), (long long)a.max_pages * a.page_tokens);
  const int last = len / a.page_tokens, part = len % a.page_tokens, kept = last + (part ? 1 : 0);
  const int entries = a.beams * (lead ? a.max_pages : kept), width = lead ? a.max_pages : max(kept, 1);
  for (int i = t; i < entries; i += kReorderThreads) {
    const int j = i / width, c = i - j * width, p = parent[j];
    const bool keep = p >= 0 && c < kept;
    const int page = keep ? T[p * a.tb + c] : p0;
    if (keep && page >= 0 && page < a.n_pages) atomicOr(&used[page >> 5], 1u << (page & 31));
    if (keep && c == last) mine[j] = page;
    if (lead && !(c == last && p >= 0)) N[j * a.nb + c] = page;
  }
  __syncthreads();
  if (t < 64) {  // the first wave: which beams need a page, and the pool's free ones in order
    const int j = min(t, a.beams - 1);
    bool need = t < a.beams && parent[j] >= 0 && last < a.max_pages, again = false;
    if (need && part)
      for (int i = 0; i < j; ++i) again = again || (parent[i] >= 0 && mine[i] == mine[j]);
    need = need && (part == 0 || again);
    const uint64_t below = ((uint64_t)1 << t) - 1, who = __ballot(need);
    const int want = __popcll(who), rank = __popcll(who & below);
    for (int i0 = 0, found = 0; i0 < a.pool_pages && found < want; i0 += 64) {
      const int i = i0 + t;
      const int q = i0 == 0 ? q0 : i < a.pool_pages ? pool[i] : -1;
      const bool free = i < a.pool_pages && q >= 0 && q < a.n_pages && !(used[max(q, 0) >> 5] >> (q & 31) & 1);
      const uint64_t m = __ballot(free);
      const int f = found + __popcll(m & below);
      if (free && f < want) fresh[f] = q;
      found += __popcll(m);
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");  // fresh[] was written by other lanes
    const int page = need ? fresh[rank] : -1;
    const bool moved = need && page >= 0 && part && mine[j] >= 0 && mine[j] < a.n_pages;
    const uint64_t mv = __ballot(moved);
    if (moved) copy[__popcll(mv & below)] = make_int2(mine[j], page);
    if (t == 0) ncopy = __popcll(mv);
    if (lead && t < a.beams && parent[j] >= 0 && last < a.max_pages)
      N[j * a.nb + last] = need ? (page >= 0 ? page : part ? mine[j] : p0) : mine[j];
  }
  __syncthreads();
  const int nc = ncopy, region = blockIdx.x / parts, share = blockIdx.x % parts;
  char* base = a.cache + (size_t)region * a.region_stride;
  const size_t per = a.page_bytes / 16, i0 = per * share / parts, i1 = per * (share + 1) / parts;
  for (int j = 0; j < nc; ++j) {
    const uint4* s = reinterpret_cast<const uint4*>(base + (size_t)copy[j].x * a.page_bytes);
    uint4* d = reinterpret_cast<uint4*>(base + (size_t)copy[j].y * a.page_bytes);
    for (size_t i = i0 + t; i < i1; i += kReorderThreads) d[i] = s[i];
  }
}

void cache_reorder(const ReorderArgs& a, hipStream_t st) {
  // pages cut into parts of at least 4 KB until about four blocks per compute unit copy (eight
  // requests: towards 512 blocks 14.2 us, 1,024 11.2, 2,048 12.5, 4,096 16.4: each block repeats the tables' work)
  const long long have = (long long)a.regions * a.n;
  int parts = (int)std::max<long long>(1, std::min<long long>(1024 / have, (long long)(a.page_bytes / 4096)));
  k_cache_reorder<<<dim3((unsigned)(a.regions * parts), a.n), kReorderThreads, 0, st>>>(a, parts);
}

// ---------------------------------------------------------------- beam search on a handle's slots
// A block per request; what a request decides is a few dozen dependent choices of one
// thread, everything per beam or page is spread over the block.

// Every beam starts on the leader's prompt with its last token unread (the first step
// reads it and gives the first choice); only beam 0 runs until then.
__global__ void __launch_bounds__(256) k_beam_begin(BeamArgs a) {
  const int r = blockIdx.x, t = threadIdx.x, B = a.beams, P = a.pages, leader = a.slot0 + r;
  const int* lead = a.state + leader * kStateInts;
  const int L = lead[ST_LEN] - 1, anchor = a.last[r];
  __syncthreads();  // the leader's state is read before it is written
  for (int i = t; i < B * P; i += 256) {
    const int b = i / P, j = i - b * P;
    a.pool[(size_t)r * B * P + i] = j * a.max_batch + a.slot0 + b * a.n + r;
    a.page_table[(size_t)(a.slot0 + b * a.n + r) * P + j] = j * a.max_batch + leader;
  }
  if (t < B) {
    int* st = a.state + (a.slot0 + t * a.n + r) * kStateInts;
    st[ST_L] = L;
    st[ST_ANCHOR] = anchor;
    st[ST_EMITTED] = 0;
    st[ST_MAX_NEW] = 1 << 30;  // the search keeps its own budget
    st[ST_DONE] = t > 0;
    st[ST_STEP] = 0;
    st[ST_NV] = 0;
    st[ST_HN] = 0;
    st[ST_LEN] = L + 1;
    st[ST_LIVE] = 1;
    a.scores[r * B + t] = t == 0 ? 0.f : -INFINITY;
    a.parents[r * B + t] = 0;
  }
  if (t == 0) {
    int* q = a.req + r * kBeamReq;
    q[BR_L] = L;
    q[BR_STEPS] = 0;
    q[BR_FIN] = 0;
    q[BR_DONE] = 0;
    q[BR_MAX_NEW] = a.max_new[r];
    q[BR_LIVE] = 1;
  }
}
void beam_start(const BeamArgs& a, hipStream_t st) { k_beam_begin<<<a.n, 256, 0, st>>>(a); }

// ---------------------------------------------------------------- self-attention of the beams' rows
// Block (head, row): one query over at most 448 positions, so a few hundred keys and values of
// 64: 8 lanes a key (16 bytes or two a lane), a lane a dim of the values, the loads of three
// keys or pages in flight at once.  The row's own key and value come from the product's
// rows, rounded to the cache's type, and go into the cache; positions of the last page past it
// hold anything and are left out.  bf16, 20 heads: 5 rows at 130 positions 6.5 us, two
// dependent memory round trips; 80 rows at 190 positions 13.6 us, registers (eight waves a SIMD;
// four keys or pages in flight, six waves: 6.0 and 14.9 us; two: 6.4 and 13.6).  The nine rows
// of a (head, request) on one XCD: no faster.
template <typename S>
__global__ void __launch_bounds__(256) k_beam_attn(BeamAttnArgs a) {
  StampScope stamp_scope(a.stamp, 256);
  __shared__ float sc[kMaxCtx], newv[kHeadDim], red[4], sum[4], acc[4][kHeadDim];
  __shared__ int pts[kMaxCtx / kPage];
  const int head = blockIdx.x, p = blockIdx.y / kRows, i = blockIdx.y % kRows, row = a.rows.slot0 * kRows + blockIdx.y;
  const int t = threadIdx.x, lane = t & 63, w = t >> 6, slot = a.rows.slot_of(p, i), H = a.n_head;
  const int* st = a.state + max(slot, 0) * kStateInts;
  const int L = st[ST_L];
  float* q = a.qkv + (size_t)row * a.ldq + head * kHeadDim;
  if (slot < 0 || !st[ST_LIVE] || st[ST_DONE] || L < 0 || L >= a.n_ctx) {  // uniform: a row of no beam
    if (t < kHeadDim) put_op<S>(a.out, a.nsplit, a.R9, row, head * kHeadDim + t, 0.f);
    return;
  }
  if (t < a.pages) pts[t] = a.page_table[(size_t)slot * a.pages + t];
  const int g = lane & 7, kl = lane >> 3, d = H * kHeadDim;
  float q8[8], k8[8];
  ld8(q + 8 * g, q8);
  ld8(q + d + 8 * g, k8);
  float own = 0.f;  // the score of the row's own key
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    q8[e] *= 0.125f;
    own = fmaf(q8[e], to_f(from_f<S>(k8[e])), own);
  }
  own = sum8(own);
  __syncthreads();
  S* K = reinterpret_cast<S*>(a.kcache);
  S* V = reinterpret_cast<S*>(a.vcache);
  constexpr bool vt = sizeof(S) == 2;  // values of a page: [head][dim][position], fp32 [head][position][dim]
  if (t < kHeadDim) {
    const size_t ph = (size_t)pts[L / kPage] * H + head;
    const S v = from_f<S>(q[2 * d + t]);
    newv[t] = to_f(v);
    K[(ph * kPage + L % kPage) * kHeadDim + t] = from_f<S>(q[d + t]);
    V[vt ? (ph * kHeadDim + t) * kPage + L % kPage : (ph * kPage + L % kPage) * kHeadDim + t] = v;
  }
  // scores of the L cached keys: 32 of the block at a time, B times that in flight
  constexpr int B = 3;
  float mx = own;
  for (int j0 = 0; j0 < L; j0 += 32 * B) {
    float kx[B][8];
#pragma unroll
    for (int u = 0; u < B; ++u) {
      const int j = min(j0 + 32 * u + 8 * w + kl, L - 1);
      ld8(K + (((size_t)pts[j / kPage] * H + head) * kPage + j % kPage) * kHeadDim + 8 * g, kx[u]);
    }
#pragma unroll
    for (int u = 0; u < B; ++u) {
      float s = 0.f;
#pragma unroll
      for (int e = 0; e < 8; ++e) s = fmaf(q8[e], kx[u][e], s);
      s = sum8(s);
      const int j = j0 + 32 * u + 8 * w + kl;
      if (j < L) {
        mx = fmaxf(mx, s);
        if (g == 0) sc[j] = s;
      }
    }
  }
  mx = wave_max(mx);
  if (lane == 0) red[w] = mx;
  __syncthreads();
  mx = fmaxf(fmaxf(red[0], red[1]), fmaxf(red[2], red[3]));
  // probabilities in place, zero behind the last position
  const int np = (L + kPage - 1) / kPage;
  float l = 0.f;
  for (int j = t; j < np * kPage; j += 256) {
    const float pr = j < L ? __expf(sc[j] - mx) : 0.f;
    sc[j] = pr;
    l += pr;
  }
  l = wave_sum(l);
  if (lane == 0) sum[w] = l;
  __syncthreads();
  // values: a wave every fourth page, a lane a dim
  float o = 0.f;
  for (int c0 = w; c0 < np; c0 += 4 * B) {
    float v[B][kPage];
#pragma unroll
    for (int u = 0; u < B; ++u) {
      const size_t ph = (size_t)pts[min(c0 + 4 * u, np - 1)] * H + head;
      if constexpr (vt) {
        ld8(V + (ph * kHeadDim + lane) * kPage, v[u]);
        ld8(V + (ph * kHeadDim + lane) * kPage + 8, v[u] + 8);
      } else {
#pragma unroll
        for (int e = 0; e < kPage; ++e) v[u][e] = to_f(V[(ph * kPage + e) * kHeadDim + lane]);
      }
    }
#pragma unroll
    for (int u = 0; u < B; ++u) {
      const int c = c0 + 4 * u;
      if (c >= np) break;
#pragma unroll
      for (int e = 0; e < kPage; ++e) {
        const int j = kPage * c + e;
        o = fmaf(sc[j], j < L ? v[u][e] : 0.f, o);
      }
    }
  }
  acc[w][lane] = o;
  if (a.clear_q && t < kHeadDim) q[t] = 0.f;  // every wave has read its queries
  __syncthreads();
  if (t < kHeadDim) {
    const float pr = __expf(own - mx), all = (sum[0] + sum[1]) + (sum[2] + sum[3]) + pr;
    put_op<S>(a.out, a.nsplit, a.R9, row, head * kHeadDim + t,
              fmaf(pr, newv[t], (acc[0][t] + acc[1][t]) + (acc[2][t] + acc[3][t])) / all);
  }
}
template <typename S>
void beam_attn(const BeamAttnArgs& a, hipStream_t st) {
  k_beam_attn<S><<<dim3(a.n_head, a.rows.slots() * kRows), 256, 0, st>>>(a);
}
template void beam_attn<float>(const BeamAttnArgs&, hipStream_t);
template void beam_attn<bf16>(const BeamAttnArgs&, hipStream_t);

// After the selection: candidates in order, those that end with the end-of-transcript token
// become finished hypotheses and the others beams, until there are as many beams.  Leaves
// the tables as they were for the reordering.
__global__ void __launch_bounds__(256) k_beam_advance(BeamArgs a) {
  __shared__ int par[kMaxBeams], tok[kMaxBeams], fin_all;
  __shared__ float sc[kMaxBeams];
  const int r = blockIdx.x, t = threadIdx.x, B = a.beams, P = a.pages;
  int* q = a.req + r * kBeamReq;
  const bool was_done = q[BR_DONE] != 0;
  const int L = q[BR_L], step = q[BR_STEPS];
  for (int i = t; i < B * P; i += 256) {
    const int b = i / P;
    a.tables[(size_t)r * B * P + i] = a.page_table[(size_t)(a.slot0 + b * a.n + r) * P + (i - b * P)];
  }
  if (t < B) par[t] = -1;
  __syncthreads();
  if (t == 0 && !was_done) {
    int live = 0, nf = q[BR_FIN];
    for (int j = 0; j < a.k && live < B; ++j) {
      const int b = a.cand_beam[r * a.k + j], v = a.cand_token[r * a.k + j];
      const float s = a.cand_score[r * a.k + j];
      if (b < 0) break;
      if (v == a.eos) {
        if (nf < B) {
          a.fscore[r * B + nf] = s;
          a.fstep[r * B + nf] = step;
          a.fbeam[r * B + nf] = b;
          ++nf;
        }
      } else {
        par[live] = b;
        tok[live] = v;
        sc[live] = s;
        ++live;
      }
    }
    const bool done = nf >= B || live == 0 || step + 1 >= q[BR_MAX_NEW] || L + 1 >= a.n_ctx;
    q[BR_L] = L + 1;
    q[BR_STEPS] = step + 1;
    q[BR_FIN] = nf;
    q[BR_DONE] = done;
    q[BR_LIVE] = live;
    fin_all = done;
  }
  __syncthreads();
  if (!was_done && t < B) {
    const bool on = par[t] >= 0;
    int* st = a.state + (a.slot0 + t * a.n + r) * kStateInts;
    st[ST_L] = L + 1;
    if (on) st[ST_ANCHOR] = tok[t];
    st[ST_DONE] = !on || fin_all;
    st[ST_STEP] = step + 1;
    a.scores[r * B + t] = on ? sc[t] : -INFINITY;
    const size_t at = ((size_t)step * a.n + r) * B + t;
    a.bt[at] = on ? tok[t] : -1;
    a.bp[at] = par[t];
  }
  if (t < B) a.parents[r * B + t] = was_done ? -1 : par[t];
  if (t == 0) {
    a.lens[r] = L + 1;
    if (a.done) a.done[r] = was_done || fin_all;
  }
}
void beam_advance(const BeamArgs& a, hipStream_t st) { k_beam_advance<<<a.n, 256, 0, st>>>(a); }

// The hypotheses, best first by score / length^penalty: the finished ones and, where those
// are fewer than the beams, the best live ones.  Then the slots are given back.
__global__ void __launch_bounds__(256) k_beam_end(BeamArgs a) {
  __shared__ float sc[kMaxBeams], val[kMaxBeams];
  __shared__ int hs[kMaxBeams], hb[kMaxBeams], he[kMaxBeams], order[kMaxBeams], nh;
  const int r = blockIdx.x, t = threadIdx.x, B = a.beams, P = a.pages;
  const int* q = a.req + r * kBeamReq;
  if (t == 0) {
    int n = 0;
    for (int i = 0; i < q[BR_FIN]; ++i, ++n) {  // the path of fbeam up to the step before, then the closing token
      sc[n] = a.fscore[r * B + i];
      hs[n] = a.fstep[r * B + i] - 1;
      hb[n] = a.fbeam[r * B + i];
      he[n] = 1;
    }
    if (q[BR_STEPS] > 0)
      for (int b = 0; b < q[BR_LIVE] && n < B; ++b, ++n) {  // beams come best first
        sc[n] = a.scores[r * B + b];
        hs[n] = q[BR_STEPS] - 1;
        hb[n] = b;
        he[n] = 0;
      }
    for (int i = 0; i < n; ++i) {
      val[i] = sc[i] / powf((float)(hs[i] + 1 + he[i]), a.length_penalty);
      int j = i;
      for (; j > 0 && val[order[j - 1]] < val[i]; --j) order[j] = order[j - 1];
      order[j] = i;
    }
    nh = n;
  }
  __syncthreads();
  if (t < B) {
    int* out = a.tokens + ((size_t)r * B + t) * a.len_max;
    int len = 0;
    if (t < nh) {
      const int h = order[t];
      int b = hb[h];
      len = hs[h] + 1 + he[h];
      if (he[h] && len - 1 < a.len_max) out[len - 1] = a.eos;
      for (int s = hs[h]; s >= 0; --s) {
        const size_t at = ((size_t)s * a.n + r) * B + b;
        if (s < a.len_max) out[s] = a.bt[at];
        b = a.bp[at];
      }
    }
    for (int s = len; s < a.len_max; ++s) out[s] = -1;
    a.out_len[r * B + t] = len;
    a.out_score[r * B + t] = t < nh ? sc[order[t]] : -INFINITY;
  }
  for (int i = t; i < B * P; i += 256) {
    const int b = i / P, j = i - b * P, slot = a.slot0 + b * a.n + r;
    a.page_table[(size_t)slot * P + j] = j * a.max_batch + slot;
  }
  if (t < B) {
    int* st = a.state + (a.slot0 + t * a.n + r) * kStateInts;
    st[ST_LIVE] = 0;
    st[ST_DONE] = 1;
  }
}
void beam_end(const BeamArgs& a, hipStream_t st) { k_beam_end<<<a.n, 256, 0, st>>>(a); }

}  // namespace wf
