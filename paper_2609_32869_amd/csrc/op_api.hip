// C entries of the operators without a handle: argument checks and launches.
#include <cstdint>

#include "../../include/wf.h"
#include "wf_ops.h"

using namespace wf;

namespace {

int bad(const char* msg) { return op_fail(WF_EINVAL, msg); }

bool aligned(const void* p, size_t a) { return reinterpret_cast<uintptr_t>(p) % a == 0; }

bool overlap(const void* a, size_t na, const void* b, size_t nb) {
  const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
  return x < y + nb && y < x + na;
}

int launched() {
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? WF_OK : op_fail(WF_EHIP, hipGetErrorString(e));
}

constexpr int kMaxGrid = 65535;  // blocks along a grid's y and z

int check_dtype(int dtype, size_t& e) {
  if (dtype != WF_F32 && dtype != WF_BF16) return bad("dtype must be WF_F32 or WF_BF16");
  e = dtype == WF_F32 ? 4 : 2;
  return WF_OK;
}

int check_select(int n, int beams, int vocab, int k) {
  if (n < 1 || n > kMaxGrid) return bad("n must be in [1, 65535]");
  if (beams < 1 || beams > kMaxBeams) return bad("beams must be in [1, 16]");
  if (vocab < 1 || vocab > kMaxVocab) return bad("n_vocab must be in [1, 2^20]");
  if (k < 1 || k > kMaxCand) return bad("k must be in [1, 32]");
  return WF_OK;
}

int check_cache(const wf_kv4* c, bool data = true) {
  if (!c) return bad("null cache");
  if (c->entries < 1 || c->entries > kMaxGrid) return bad("entries must be in [1, 65535]");
  if (c->n_head < 1 || c->n_head > kMaxGrid) return bad("n_head must be in [1, 65535]");
  if (c->n_frames < 1 || c->n_frames > kKv4MaxFrames) return bad("n_frames must be in [1, 2^20]");
  if (data && (!c->data || !aligned(c->data, 16))) return bad("cache data must be 16-byte aligned");
  return WF_OK;
}
int check_range(const wf_kv4* c, int slot0, int n) {
  if (n < 1 || slot0 < 0 || slot0 > c->entries - n) return bad("entries out of range");
  return WF_OK;
}
Kv4 geometry(const wf_kv4* c) {
  return Kv4{static_cast<uint8_t*>(c->data), c->n_head, kv4_groups(c->n_frames), c->n_frames};
}
// Strides of three axes before the last; vec: every row starts on 16 bytes.
int check_strides(const void* p, const int64_t* s, size_t e, int& vec) {
  if (!p || !s) return bad("null argument");
  if (!aligned(p, e)) return bad("a tensor must be aligned to its elements");
  for (int i = 0; i < 3; ++i)
    if (s[i] < 0 || s[i] > ((int64_t)1 << 40)) return bad("stride out of range");
  if (!aligned(p, 16) || (s[0] * e) % 16 || (s[1] * e) % 16 || (s[2] * e) % 16) vec = 0;
  return WF_OK;
}

}  // namespace

extern "C" {

int wf_beam_select_workspace_bytes(int n, int beams, int n_vocab, int k, size_t* bytes) {
  if (int r = check_select(n, beams, n_vocab, k)) return r;
  if (!bytes) return bad("null bytes");
  *bytes = beam_space_bytes(n, beams, n_vocab, k);
  return WF_OK;
}

int wf_beam_select(const void* logits, int dtype, int64_t req_stride, int64_t beam_stride, const float* scores,
                   const uint8_t* suppress, int n, int beams, int n_vocab, int k, float* out_score, int32_t* out_beam,
                   int32_t* out_token, void* workspace, size_t ws_bytes, void* stream) {
  size_t e;
  if (int r = check_select(n, beams, n_vocab, k)) return r;
  if (int r = check_dtype(dtype, e)) return r;
  if (!logits || !scores || !out_score || !out_beam || !out_token) return bad("null argument");
  if (!aligned(logits, e) || !aligned(scores, 4) || !aligned(out_score, 4) || !aligned(out_beam, 4) || !aligned(out_token, 4))
    return bad("a tensor must be aligned to its elements");
  if (req_stride < 0 || beam_stride < 0 || req_stride > ((int64_t)1 << 40) || beam_stride > ((int64_t)1 << 40))
    return bad("stride out of range");
  if (!workspace || !aligned(workspace, 256)) return bad("workspace must be 256-byte aligned");
  if (ws_bytes < beam_space_bytes(n, beams, n_vocab, k)) return op_fail(WF_ESIZE, "workspace too small");
  BeamSelectArgs a{};
  a.logits = logits;
  a.bf16_logits = dtype == WF_BF16;
  a.sr = req_stride;
  a.sb = beam_stride;
  a.scores = scores;
  a.suppress = suppress;
  a.n = n;
  a.beams = beams;
  a.vocab = n_vocab;
  a.k = k;
  beam_space(a, static_cast<char*>(workspace));
  a.out_score = out_score;
  a.out_beam = out_beam;
  a.out_token = out_token;
  beam_select(a, static_cast<hipStream_t>(stream));
  return launched();
}

int wf_cache_reorder(void* cache, int n_regions, size_t region_stride, int n_pages, size_t page_bytes,
                     const int32_t* tables, int32_t* new_tables, int n, int beams, int max_pages, int page_tokens,
                     const int32_t* parents, const int32_t* lens, const int32_t* pool, int pool_pages, void* stream) {
  if (!cache || !tables || !new_tables || !parents || !lens || !pool) return bad("null argument");
  if (n < 1 || n > kMaxGrid) return bad("n must be in [1, 65535]");
  if (beams < 1 || beams > kMaxBeams) return bad("beams must be in [1, 16]");
  if (n_regions < 1 || n_regions > kMaxGrid) return bad("n_regions must be in [1, 65535]");
  if (n_pages < 1 || n_pages > kMaxPages) return bad("n_pages must be in [1, 2^18]");
  if (max_pages < 1 || max_pages > kMaxPages) return bad("max_pages must be in [1, 2^18]");
  if (page_tokens < 1 || page_tokens > (1 << 20)) return bad("page_tokens must be in [1, 2^20]");
  if (pool_pages < 1 || pool_pages > kMaxPages) return bad("pool_pages must be in [1, 2^18]");
  if (!aligned(cache, 16) || page_bytes == 0 || page_bytes % 16 || page_bytes > ((size_t)1 << 40) || region_stride % 16)
    return bad("cache, page_bytes and region_stride must be multiples of 16 bytes");
  if (n_regions > 1 && region_stride / page_bytes < (size_t)n_pages) return bad("regions overlap");
  if (!aligned(tables, 4) || !aligned(new_tables, 4) || !aligned(parents, 4) || !aligned(lens, 4) || !aligned(pool, 4))
    return bad("a tensor must be aligned to its elements");
  // every block reads all of these, and the first one of a request writes its new tables
  const size_t nb = (size_t)n * beams, tb = nb * max_pages * 4;
  if (overlap(new_tables, tb, tables, tb) || overlap(new_tables, tb, parents, nb * 4) || overlap(new_tables, tb, lens, (size_t)n * 4) ||
      overlap(new_tables, tb, pool, (size_t)n * pool_pages * 4))
    return bad("new_tables must not share memory with another argument");
  ReorderArgs a{};
  a.cache = static_cast<char*>(cache);
  a.regions = n_regions;
  a.region_stride = region_stride;
  a.page_bytes = page_bytes;
  a.n_pages = n_pages;
  a.tables = tables;
  a.new_tables = new_tables;
  a.tb = a.nb = max_pages;
  a.tr = a.nr = (long long)beams * max_pages;
  a.parents = parents;
  a.lens = lens;
  a.pool = pool;
  a.n = n;
  a.beams = beams;
  a.max_pages = max_pages;
  a.pool_pages = pool_pages;
  a.page_tokens = page_tokens;
  cache_reorder(a, static_cast<hipStream_t>(stream));
  return launched();
}

int wf_kv4_bytes(int entries, int n_head, int n_frames, size_t* bytes) {
  const wf_kv4 c{nullptr, entries, n_head, n_frames};
  if (int r = check_cache(&c, false)) return r;
  if (!bytes) return bad("null bytes");
  *bytes = (size_t)entries * n_head * kv4_groups(n_frames) * kKv4Group;
  return WF_OK;
}

int wf_kv4_store(const wf_kv4* c, int slot0, int n, const void* k, const int64_t* k_stride, const void* v,
                 const int64_t* v_stride, int dtype, const int32_t* lens, void* stream) {
  size_t e;
  int vec = 1;
  if (int r = check_cache(c)) return r;
  if (int r = check_range(c, slot0, n)) return r;
  if (int r = check_dtype(dtype, e)) return r;
  if (int r = check_strides(k, k_stride, e, vec)) return r;
  if (int r = check_strides(v, v_stride, e, vec)) return r;
  if (!aligned(lens, 4)) return bad("lens must be aligned to its elements");
  Kv4StoreArgs a{};
  a.c = geometry(c);
  a.k = k;
  a.v = v;
  a.bf16_src = dtype == WF_BF16;
  a.kr = k_stride[0];
  a.kf = k_stride[1];
  a.kh = k_stride[2];
  a.vr = v_stride[0];
  a.vf = v_stride[1];
  a.vh = v_stride[2];
  a.lens = lens;
  a.slot0 = slot0;
  a.n = n;
  a.vec = vec;
  kv4_store(a, static_cast<hipStream_t>(stream));
  return launched();
}

int wf_kv4_load(const wf_kv4* c, int slot0, int n, void* k, void* v, int dtype, void* stream) {
  size_t e;
  if (int r = check_cache(c)) return r;
  if (int r = check_range(c, slot0, n)) return r;
  if (int r = check_dtype(dtype, e)) return r;
  if (!k || !v) return bad("null argument");
  if (!aligned(k, 16) || !aligned(v, 16)) return bad("outputs must be 16-byte aligned");
  Kv4LoadArgs a{};
  a.c = geometry(c);
  a.k = k;
  a.v = v;
  a.bf16_out = dtype == WF_BF16;
  a.slot0 = slot0;
  a.n = n;
  kv4_load(a, static_cast<hipStream_t>(stream));
  return launched();
}

int wf_kv4_attend_workspace_bytes(const wf_kv4* c, int n, int rows, size_t* bytes) {
  if (int r = check_cache(c, false)) return r;
  if (int r = check_range(c, 0, n)) return r;
  if (rows < 1 || rows > (1 << 19)) return bad("rows must be in [1, 2^19]");
  if (!bytes) return bad("null bytes");
  *bytes = kv4_workspace(n, rows, c->n_head, c->n_frames);
  return WF_OK;
}

int wf_kv4_attend(const wf_kv4* c, int slot0, int n, const void* q, const int64_t* q_stride, int rows, int dtype,
                  const int32_t* lens, void* out, void* workspace, size_t ws_bytes, void* stream) {
  size_t e, need;
  int vec = 1;
  if (int r = check_cache(c)) return r;
  if (int r = check_range(c, slot0, n)) return r;
  if (int r = check_dtype(dtype, e)) return r;
  if (int r = wf_kv4_attend_workspace_bytes(c, n, rows, &need)) return r;
  if (int r = check_strides(q, q_stride, e, vec)) return r;
  if (!out || !aligned(out, 16)) return bad("out must be 16-byte aligned");
  if (!aligned(lens, 4)) return bad("lens must be aligned to its elements");
  if (need > 0 && (!workspace || !aligned(workspace, 256))) return bad("workspace must be 256-byte aligned");
  if (ws_bytes < need) return op_fail(WF_ESIZE, "workspace too small");
  Kv4AttendArgs a{};
  a.c = geometry(c);
  a.q = q;
  a.sr = q_stride[0];
  a.si = q_stride[1];
  a.sh = q_stride[2];
  a.bf16_q = dtype == WF_BF16;
  a.vec = vec;
  a.out = out;
  a.lens = lens;
  a.slot0 = slot0;
  a.n = n;
  a.rows = rows;
  a.part = static_cast<float*>(workspace);
  kv4_attend(a, static_cast<hipStream_t>(stream));
  return launched();
}

}  // extern "C"
