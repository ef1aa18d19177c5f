// Argument blocks and launchers of the stateless operators (internal): beam selection
// and page reordering (k_beam.hip), the 4-bit acoustic cache (k_kv4.hip).
#pragma once
#include <hip/hip_runtime.h>
#include <string>

#include "wf_common.h"
#include "wf_kernels.h"

namespace wf {

// Records the message of a call without a handle (wf_last_error(NULL)); returns code.
int op_fail(int code, const char* msg);

// ---------------------------------------------------------------- beam selection
constexpr int kMaxBeams = 16;       // beams of one request
constexpr int kMaxCand = 32;        // candidates kept per request
constexpr int kMaxVocab = 1 << 20;  // columns of a logits row
struct BeamSelectArgs {
  const void* logits;  // element (r, b, v) at r * sr + b * sb + (b < kRows ? 0 : far) + v
  int bf16_logits;
  long long sr, sb, far;  // far: more of it for the beams from kRows on (a handle's logits)
  const float* scores;      // (r, b) at r * beams + b
  const uint8_t* suppress;  // [vocab] nonzero: the column is left out, or null
  int n, beams, vocab, k;
  // per piece of a logits row ((r * beams + b) * pieces + piece): its k best as (logit, column; -1: none),
  // its maximum and its sum of exponentials relative to that
  float* pv;
  int* pi;
  float* pm;
  double* ps;
  float* out_score;  // [n][k]
  int* out_beam;
  int* out_token;
};
int beam_pieces(int vocab);  // pieces of a row
// bytes of the row kernel's results, and the pointers to them in `space` (of a with its sizes set)
size_t beam_space_bytes(int n, int beams, int vocab, int k);
void beam_space(BeamSelectArgs& a, char* space);
void beam_select(const BeamSelectArgs& a, hipStream_t st);

// ---------------------------------------------------------------- page tables after a choice of beams
constexpr int kMaxPages = 1 << 18;  // pages of a cache (a bit each in LDS)
struct ReorderArgs {
  char* cache;  // [regions] of region_stride bytes, each n_pages pages of page_bytes
  int regions;
  size_t region_stride, page_bytes;
  int n_pages;
  const int* tables;   // (r, b, c) at r * tr + b * tb + c
  int* new_tables;     // other memory: (r, b, c) at r * nr + b * nb + c
  long long tr, tb, nr, nb;
  const int* parents;  // [n][beams]
  const int* lens;     // [n]
  const int* pool;     // [n][pool_pages]
  int n, beams, max_pages, pool_pages, page_tokens;
};
void cache_reorder(const ReorderArgs& a, hipStream_t st);

// ---------------------------------------------------------------- beam search on a handle's slots
// Request r's beam b is slot slot0 + b * n + r.  Per request: BR_* words.
enum { BR_L = 0, BR_STEPS = 1, BR_FIN = 2, BR_DONE = 3, BR_MAX_NEW = 4, BR_LIVE = 5, kBeamReq = 8 };
struct BeamArgs {
  int* state;       // the handle's slots
  int* page_table;  // [slot][pages]
  int slot0, n, beams, pages, max_batch, eos, n_ctx, k;
  int* req;         // [n][kBeamReq]
  float* scores;    // [n][beams] cumulative log-probabilities
  const float* cand_score;  // [n][k] candidates of the step, best first
  const int* cand_beam;
  const int* cand_token;
  int* parents;     // [n][beams] of the step (-1: no beam)
  int* lens;        // [n] positions cached after it
  int* pool;        // [n][beams * pages] the request's own pages
  int* tables;      // [n][beams][pages] the page tables before the step's choice
  int* bt;          // [step][n][beams] token and parent of every beam
  int* bp;
  float* fscore;    // [n][beams] finished hypotheses: score, step of the closing token, beam before it
  int* fstep;
  int* fbeam;
  const int* last;  // begin: last prompt token of each request
  const int* max_new;
  int* done;        // step: [n] or null
  // end: [n][beams][len_max], [n][beams], [n][beams]
  int* tokens;
  int* out_len;
  float* out_score;
  int len_max;
  float length_penalty;
};
void beam_start(const BeamArgs& a, hipStream_t st);
void beam_advance(const BeamArgs& a, hipStream_t st);
void beam_end(const BeamArgs& a, hipStream_t st);
// Self-attention of the beams' rows, each over its own page table, after putting its new key
// and value into its page.
struct BeamAttnArgs {
  BeamRows rows;
  float* qkv;  // q | k | v of the pass's rows, [row][ldq]
  int ldq;
  void *kcache, *vcache;
  const int* state;
  const int* page_table;
  Operand out;
  int n_head, n_ctx, pages, nsplit, R9;
  int clear_q;  // as in AttnArgs
  unsigned long long* stamp;
};
template <typename S>
void beam_attn(const BeamAttnArgs& a, hipStream_t st);

// ---------------------------------------------------------------- acoustic keys and values in 4 bits
// Per (entry, head), groups of 32 frames one after the other, kKv4Group bytes each: the
// keys' and the values' codes in the order in which a wave's lanes multiply them, then
// their scales' biased exponents (0xff: the block stands for NaN).
//   keys    lane l = 16 kg + n, byte 8 t + j: dims 16 kg + 2 j, + 1 of frame 16 t + n
//   values  lane l = 16 kg + n, byte 4 dt + j: frames 8 kg + 2 j, + 1 of dim 4 n + dt
//   scales  keys: byte 32 half + 2 n + t: dims 32 half .. + 31 of frame 16 t + n;
//           values: a byte per dim
// Low nibble first.  A wave reads a group's codes as two 16-byte loads per lane.
constexpr int kKv4Frames = 32;
constexpr int kKv4Values = 1024, kKv4KeyScale = 2048, kKv4ValueScale = 2112, kKv4Group = 2176;
constexpr int kKv4MaxFrames = 1 << 20;
__host__ __device__ inline int kv4_groups(int frames) { return (frames + kKv4Frames - 1) / kKv4Frames; }
struct Kv4 {
  uint8_t* base;
  int n_head, groups, frames;
};
struct Kv4StoreArgs {
  Kv4 c;
  const void *k, *v;  // element (r, f, h, d) at r * sr + f * sf + h * sh + d
  int bf16_src;
  long long kr, kf, kh, vr, vf, vh;
  const int* lens;  // [n] or null
  int slot0, n;
  int vec;  // rows may be read 16 bytes at a time
};
void kv4_store(const Kv4StoreArgs& a, hipStream_t st);
struct Kv4LoadArgs {
  Kv4 c;
  void *k, *v;  // [n][frames][n_head][64]
  int bf16_out, slot0, n;
};
void kv4_load(const Kv4LoadArgs& a, hipStream_t st);
// A decoder's acoustic keys and values in the bf16 layout of the request-time product (keys
// [head][frame][64], values [head][frame / 256][dim][256]).
struct Kv4UnpackArgs {
  Kv4 c;
  bf16* kv;  // entry i at i * stride elements
  size_t stride;
  int vt_frames;
  int slot0, n;
};
void kv4_unpack(const Kv4UnpackArgs& a, hipStream_t st);
struct Kv4AttendArgs {
  Kv4 c;
  const void* q;  // element (r, i, h, d) at r * sr + i * si + h * sh + d
  long long sr, si, sh;
  int bf16_q, vec;
  void* out;  // [n][rows][n_head][64], the query's type
  const int* lens;
  int slot0, n, rows;
  float* part;  // chunk records (nchunk > 1)
  int nchunk, cgroups;  // chunks of the groups and groups of a chunk (set by the launcher)
  Operand op;  // a decoder step's output: row i of request r is operand row row0 + r * rows + i
  int nsplit, R9, row0;
  unsigned long long* stamp;  // launch timing slot (profiled calls), or null
};
size_t kv4_workspace(int n, int rows, int n_head, int frames);
void kv4_attend(const Kv4AttendArgs& a, hipStream_t st);
// A decoder step's rows (fp32 queries as two bf16 terms, like the step's other products):
// into the next product's operand, or as the records of cross_mx_chunks(1) chunks for
// attn_cross_merge (one request of at most nine rows).
void kv4_attend_operand(const Kv4AttendArgs& a, hipStream_t st);
void kv4_attend_records(const Kv4AttendArgs& a, hipStream_t st);

}  // namespace wf
