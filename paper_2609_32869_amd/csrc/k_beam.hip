// Beam search: the k best continuations over a request's beams and vocabulary, and the
// page tables of the beams that were chosen.
#include "wf_ops.h"

namespace wf {

// ---------------------------------------------------------------- selection
// score(b, v) = s_b + x_bv - log sum_u exp(x_bu).  A beam's order over v is the order of
// its logits, so each row keeps its k best logits; the beams meet in 64-bit scores.

template <typename T>
__device__ __forceinline__ float logit(const T* x, const uint8_t* sup, int v) {
  return sup && sup[v] ? -INFINITY : to_f(x[v]);
}

template <typename T>
__global__ void __launch_bounds__(256) k_beam_rows(BeamSelectArgs a) {
  __shared__ float sv[256];
  __shared__ int si[256];
  __shared__ double sd[256];
  const int row = blockIdx.x, r = row / a.beams, b = row % a.beams, t = threadIdx.x;
  const T* x = reinterpret_cast<const T*>(a.logits) + r * a.sr + b * a.sb;
  float last = INFINITY;
  int li = -1;
  for (int j = 0; j < a.k; ++j) {
    float bv = -INFINITY;
    int bi = a.vocab;
    for (int v = t; v < a.vocab; v += 256) {
      const float y = logit(x, a.suppress, v);
      if ((y < last || (y == last && v > li)) && y > -INFINITY && better(y, v, bv, bi)) {
        bv = y;
        bi = v;
      }
    }
    sv[t] = bv;
    si[t] = bi;
    __syncthreads();
    for (int o = 128; o > 0; o >>= 1) {
      if (t < o && better(sv[t + o], si[t + o], sv[t], si[t])) {
        sv[t] = sv[t + o];
        si[t] = si[t + o];
      }
      __syncthreads();
    }
    last = sv[0];
    li = si[0];
    __syncthreads();
    if (j == 0) {
      double sum = 0;
      for (int v = t; v < a.vocab; v += 256) {
        const float y = logit(x, a.suppress, v);
        if (!(y == -INFINITY)) sum += (double)expf(y - last);
      }
      sd[t] = sum;
      __syncthreads();
      for (int o = 128; o > 0; o >>= 1) {
        if (t < o) sd[t] += sd[t + o];
        __syncthreads();
      }
      if (t == 0) a.lse[row] = (double)last + log(sd[0]);
    }
    if (t == 0) {
      a.pv[(size_t)row * a.k + j] = last;
      a.pi[(size_t)row * a.k + j] = li;
    }
    if (li >= a.vocab) {  // nothing left (uniform)
      last = -INFINITY;
      li = a.vocab;
    }
  }
}

__global__ void __launch_bounds__(64) k_beam_merge(BeamSelectArgs a) {
  const int r = blockIdx.x;
  if (threadIdx.x != 0) return;
  int at[kMaxBeams];
  for (int b = 0; b < a.beams; ++b) at[b] = 0;
  for (int j = 0; j < a.k; ++j) {
    double best = -INFINITY;
    int bb = -1;
    for (int b = 0; b < a.beams; ++b) {
      if (at[b] >= a.k) continue;
      const size_t row = (size_t)r * a.beams + b;
      const double s = (double)a.scores[row] + ((double)a.pv[row * a.k + at[b]] - a.lse[row]);
      if (s > best && s < INFINITY) {
        best = s;
        bb = b;
      }
    }
    a.out_score[(size_t)r * a.k + j] = (float)best;
    a.out_beam[(size_t)r * a.k + j] = bb;
    a.out_token[(size_t)r * a.k + j] = bb < 0 ? -1 : a.pi[((size_t)r * a.beams + bb) * a.k + at[bb]];
    if (bb >= 0) ++at[bb];
  }
}

void beam_select(const BeamSelectArgs& a, hipStream_t st) {
  if (a.bf16_logits) k_beam_rows<bf16><<<a.n * a.beams, 256, 0, st>>>(a);
  else k_beam_rows<float><<<a.n * a.beams, 256, 0, st>>>(a);
  k_beam_merge<<<a.n, 64, 0, st>>>(a);
}

// ---------------------------------------------------------------- page tables
// Beam j continues beam parents[j] of its request: it keeps that beam's pages.  Full
// pages are never written again, so beams share them.  The page of the next position
// is one beam's own: the first beam that keeps a part-filled page goes on in it, every
// other one gets the pool's next unreferenced page and a copy.
//
// Grid (region, request).  Every block works the request's pages out for itself (a few
// hundred table entries, a bit per page of the cache in LDS); the first one writes the
// tables, each copies the pages of its region.
__global__ void __launch_bounds__(256) k_cache_reorder(ReorderArgs a) {
  __shared__ unsigned used[kMaxPages / 32];
  __shared__ int2 copy[kMaxBeams];  // (source, destination), destination -1: none
  const int r = blockIdx.y, t = threadIdx.x;
  const bool lead = blockIdx.x == 0;
  for (int i = t; i < (a.n_pages + 31) / 32; i += 256) used[i] = 0;
  __syncthreads();
  const int len = (int)min((long long)max(a.lens[r], 0), (long long)a.max_pages * a.page_tokens);
  const int last = len / a.page_tokens, part = len % a.page_tokens, kept = last + (part ? 1 : 0);
  const int* T = a.tables + r * a.tr;
  int* N = a.new_tables + r * a.tr;
  const int* pool = a.pool + (size_t)r * a.pool_pages;
  const int* parents = a.parents + (size_t)r * a.beams;
  for (int j = 0; j < a.beams; ++j) {
    const int p = parents[j];
    const bool live = p >= 0 && p < a.beams;
    for (int c = t; c < a.max_pages; c += 256) {
      const int page = live && c < kept ? T[p * a.tb + c] : pool[0];
      if (lead) N[j * a.tb + c] = page;
      if (live && c < kept && page >= 0 && page < a.n_pages) atomicOr(&used[page >> 5], 1u << (page & 31));
    }
  }
  __syncthreads();
  if (t == 0) {
    int at = 0;
    for (int j = 0; j < a.beams; ++j) {
      const int p = parents[j];
      int2 cp = make_int2(-1, -1);
      if (p >= 0 && p < a.beams && last < a.max_pages) {
        bool need = part == 0;
        const int mine = T[p * a.tb + last];
        for (int i = 0; i < j && !need; ++i) {
          const int pi = parents[i];
          need = pi >= 0 && pi < a.beams && T[pi * a.tb + last] == mine;
        }
        if (need) {
          int page = -1;
          for (; at < a.pool_pages && page < 0; ++at) {
            const int q = pool[at];
            if (q >= 0 && q < a.n_pages && !(used[q >> 5] >> (q & 31) & 1)) page = q;
          }
          if (page >= 0) {
            if (lead) N[j * a.tb + last] = page;
            if (part && mine >= 0 && mine < a.n_pages) cp = make_int2(mine, page);
          }
        }
      }
      copy[j] = cp;
    }
  }
  __syncthreads();
  char* base = a.cache + (size_t)blockIdx.x * a.region_stride;
  for (int j = 0; j < a.beams; ++j) {
    if (copy[j].y < 0) continue;
    const uint4* s = reinterpret_cast<const uint4*>(base + (size_t)copy[j].x * a.page_bytes);
    uint4* d = reinterpret_cast<uint4*>(base + (size_t)copy[j].y * a.page_bytes);
    for (size_t i = t; i < a.page_bytes / 16; i += 256) d[i] = s[i];
  }
}

void cache_reorder(const ReorderArgs& a, hipStream_t st) {
  k_cache_reorder<<<dim3(a.regions, a.n), 256, 0, st>>>(a);
}

}  // namespace wf
