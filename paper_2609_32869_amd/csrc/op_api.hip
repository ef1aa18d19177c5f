// C entries of the operators without a handle: argument checks and launches.
#include <cmath>
#include <cstdint>
#include <utility>

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
// Strides of the `axes` axes before the last; vec: every row starts on 16 bytes.
int check_strides(const void* p, const int64_t* s, size_t e, int& vec, int axes = 3) {
  if (!p || !s) return bad("null argument");
  if (!aligned(p, e)) return bad("a tensor must be aligned to its elements");
  if (!aligned(p, 16)) vec = 0;
  for (int i = 0; i < axes; ++i) {
    if (s[i] < 0 || s[i] > ((int64_t)1 << 40)) return bad("stride out of range");
    if ((s[i] * e) % 16) vec = 0;
  }
  return WF_OK;
}
// Rows of `width` elements at t * s[0] + h * s[1] that overlap.
bool rows_overlap(const int64_t* s, int tokens, int heads, int width) {
  const int64_t a = tokens > 1 ? s[0] : INT64_MAX, b = heads > 1 ? s[1] : INT64_MAX;
  if (a < width || b < width) return true;
  if (tokens <= 1 || heads <= 1) return false;
  return a < b ? b / a < tokens : a / b < heads;
}
// Two such tensors of equal tokens that share memory, or that lie in one another in a way that is not looked into: rows of
// one token beside each other, as slices of one buffer, do not.
bool tensors_overlap(const char* a, const int64_t* as, int ah, const char* b, const int64_t* bs, int bh, int tokens, int width, size_t e) {
  auto row = [&](const int64_t* s, int heads) { return (uint64_t)((heads > 1 ? (heads - 1) * s[1] : 0) + width) * e; };
  auto all = [&](const int64_t* s, int heads) { return (tokens > 1 ? (uint64_t)(tokens - 1) * s[0] * e : 0) + row(s, heads); };
  if (!overlap(a, all(as, ah), b, all(bs, bh))) return false;
  if (tokens <= 1 || as[0] != bs[0]) return true;
  if (b < a) {
    std::swap(a, b);
    std::swap(as, bs);
    std::swap(ah, bh);
  }
  const uint64_t pitch = as[0] * e, apart = (uint64_t)(b - a) % pitch;
  return apart < row(as, ah) || apart + row(bs, bh) > pitch;
}
int check_heads(int n_head, int n_kv_head) {
  if (n_kv_head < 1 || n_head < 1 || n_head > kMaxGrid || n_head % n_kv_head)
    return bad("n_head must be in [1, 65535] and a multiple of the key and value heads");
  return WF_OK;
}

int check_cache8(const wf_kv8* c, bool data = true) {
  if (!c) return bad("null cache");
  if (c->n_pages < 1 || c->n_pages > kKv8MaxPages) return bad("n_pages must be in [1, 2^24]");
  if (c->n_head < 1 || c->n_head > kKv8MaxHeads) return bad("n_head must be in [1, 4096]");
  if (data && (!c->data || !aligned(c->data, 16))) return bad("cache data must be 16-byte aligned");
  return WF_OK;
}
int check_tables(int n, const int32_t* tables, int64_t stride, int max_pages) {
  if (n < 1 || n > kMaxGrid) return bad("n must be in [1, 65535]");
  if (max_pages < 1 || max_pages > kKv8MaxPages) return bad("max_pages must be in [1, 2^24]");
  if (!tables || !aligned(tables, 4)) return bad("tables must be aligned to its elements");
  if (stride < 0 || stride > ((int64_t)1 << 40)) return bad("stride out of range");
  return WF_OK;
}
Kv8 geometry(const wf_kv8* c) { return Kv8{static_cast<uint8_t*>(c->data), c->n_pages, c->n_head, kv8_page_bytes(c->n_head)}; }
constexpr int kMaxUnits = (1 << 24) - 1;  // blocks of 256 threads along a grid's x

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

int wf_rotary_turns(int dims, double base, int scaling, double factor, double context, double low, double high,
                    double* turns, float* amplitude) {
  if (dims < 2 || dims > 4096 || dims % 2) return bad("dims must be even and in [2, 4096]");
  if (!(base > 1.0) || !std::isfinite(base)) return bad("base must be above 1");
  if (scaling < WF_ROTARY_PLAIN || scaling > WF_ROTARY_RAMP) return bad("unknown scaling");
  if (scaling != WF_ROTARY_PLAIN && !(factor >= 1.0 && std::isfinite(factor))) return bad("factor must be 1 or more");
  if (scaling == WF_ROTARY_BASE && dims < 4) return bad("scaling the base needs dims above 2");
  if (scaling == WF_ROTARY_RAMP && !(context > 0.0 && std::isfinite(context))) return bad("context must be above 0");
  if (scaling == WF_ROTARY_RAMP && !(low >= 0.0 && low < high && std::isfinite(high))) return bad("low must be in [0, high)");
  if (!turns || !amplitude) return bad("null argument");
  if (scaling == WF_ROTARY_BASE) base *= std::pow(factor, dims / (dims - 2.0));
  for (int i = 0; i < dims / 2; ++i) {
    double f = std::pow(base, -2.0 * i / dims) / (2.0 * 3.14159265358979323846);
    if (scaling == WF_ROTARY_LINEAR) f /= factor;
    if (scaling == WF_ROTARY_RAMP) {
      const double w = std::fmin(std::fmax((f * context - low) / (high - low), 0.0), 1.0);
      f *= w + (1.0 - w) / factor;
    }
    turns[i] = f;
  }
  *amplitude = scaling == WF_ROTARY_RAMP ? (float)(0.1 * std::log(factor) + 1.0) : 1.f;
  return WF_OK;
}

int wf_rotary(const double* turns, int dims, int interleaved, float amplitude, int transposed, const int32_t* positions,
              int tokens, int width, int dtype, const void* q, const int64_t* q_stride, int q_heads, void* q_out,
              const int64_t* q_out_stride, const void* k, const int64_t* k_stride, int k_heads, void* k_out,
              const int64_t* k_out_stride, void* stream) {
  size_t e;
  if (width < 2 || width > 4096) return bad("width must be in [2, 4096]");
  if (dims < 2 || dims > width || dims % 2) return bad("dims must be even and in [2, width]");
  if (tokens < 0 || tokens > (1 << 28)) return bad("tokens must be in [0, 2^28]");
  if (int r = check_dtype(dtype, e)) return r;
  if (!turns || !positions) return bad("null argument");
  if (!aligned(turns, 8) || !aligned(positions, 4)) return bad("a tensor must be aligned to its elements");
  if (!std::isfinite(amplitude)) return bad("amplitude must be finite");
  RotaryArgs a{};
  a.turns = turns;
  a.dims = dims;
  a.interleaved = interleaved != 0;
  a.transposed = transposed != 0;
  a.width = width;
  a.amplitude = amplitude;
  a.positions = positions;
  a.tokens = tokens;
  a.bf16_data = dtype == WF_BF16;
  a.n_rows = k ? 2 : 1;
  a.align = 16;
  int vec = 1;
  const struct {
    const void* x;
    const int64_t* xs;
    void* y;
    const int64_t* ys;
    int heads;
  } rows[2] = {{q, q_stride, q_out, q_out_stride, q_heads}, {k, k_stride, k_out, k_out_stride, k_heads}};
  for (int i = 0; i < a.n_rows; ++i) {
    const auto& w = rows[i];
    if (w.heads < 1 || w.heads > kMaxGrid) return bad("heads must be in [1, 65535]");
    if (int r = check_strides(w.x, w.xs, e, vec, 2)) return r;
    if (int r = check_strides(w.y, w.ys, e, vec, 2)) return r;
    const uint64_t all = reinterpret_cast<uintptr_t>(w.x) | reinterpret_cast<uintptr_t>(w.y) | e * (w.xs[0] | w.xs[1] | w.ys[0] | w.ys[1]);
    while (all % a.align) a.align /= 2;
    if (rows_overlap(w.ys, tokens, w.heads, width)) return bad("rows of a result overlap");
    if (w.x == w.y) {
      if ((tokens > 1 && w.xs[0] != w.ys[0]) || (w.heads > 1 && w.xs[1] != w.ys[1])) return bad("in place, strides must be equal");
    } else {
      a.copies = 1;  // of a tensor in place: onto itself
    }
    a.rows[i] = RotaryRows{w.x, w.y, w.xs[0], w.xs[1], w.ys[0], w.ys[1], w.heads};
  }
  if (k && tokens > 0 &&
      tensors_overlap(static_cast<const char*>(q_out), q_out_stride, q_heads, static_cast<const char*>(k_out), k_out_stride, k_heads, tokens, width, e))
    return bad("the results overlap");
  if (tokens == 0) return WF_OK;
  rotary(a, static_cast<hipStream_t>(stream));
  return launched();
}

int wf_prompt_attend(const void* q, const int64_t* q_stride, const void* k, const int64_t* k_stride, const void* v,
                     const int64_t* v_stride, int dtype, const int32_t* starts, int n, int tokens, int n_head,
                     int n_kv_head, void* out, int clear, void* stream) {
  size_t e;
  if (int r = check_dtype(dtype, e)) return r;
  if (int r = check_heads(n_head, n_kv_head)) return r;
  if (n < 1 || n > (1 << 24)) return bad("n must be in [1, 2^24]");
  if (tokens < 0 || (long long)tokens * n_head > (1 << 28)) return bad("tokens * n_head must be in [0, 2^28]");
  if (!starts || !aligned(starts, 4)) return bad("starts must be aligned to its elements");
  PromptArgs a{};
  a.vec = 1;
  if (int r = check_strides(q, q_stride, e, a.vec, 2)) return r;
  if (int r = check_strides(k, k_stride, e, a.vec, 2)) return r;
  if (int r = check_strides(v, v_stride, e, a.vec, 2)) return r;
  if (!out || !aligned(out, 16)) return bad("out must be 16-byte aligned");
  if (tokens == 0) return WF_OK;
  auto extent = [&](const int64_t* t, int heads) { return ((tokens - 1) * (uint64_t)t[0] + (heads - 1) * (uint64_t)t[1] + kHeadDim) * e; };
  const uint64_t written = (uint64_t)tokens * n_head * kHeadDim * e;
  if (overlap(out, written, q, extent(q_stride, n_head)) || overlap(out, written, k, extent(k_stride, n_kv_head)) ||
      overlap(out, written, v, extent(v_stride, n_kv_head)))
    return bad("out overlaps q, k or v");
  a.q = q;
  a.k = k;
  a.v = v;
  a.qt = q_stride[0];
  a.qh = q_stride[1];
  a.kt = k_stride[0];
  a.kh = k_stride[1];
  a.vt = v_stride[0];
  a.vh = v_stride[1];
  a.bf16_data = dtype == WF_BF16;
  a.starts = starts;
  a.n = n;
  a.tokens = tokens;
  a.heads = n_head;
  a.group = n_head / n_kv_head;
  a.out = out;
  a.clear = clear != 0;
  prompt_attend(a, static_cast<hipStream_t>(stream));
  return launched();
}

int wf_kv8_page_bytes(int n_head, size_t* bytes) {
  const wf_kv8 c{nullptr, 1, n_head};
  if (int r = check_cache8(&c, false)) return r;
  if (!bytes) return bad("null bytes");
  *bytes = kv8_page_bytes(n_head);
  return WF_OK;
}

int wf_kv8_store(const wf_kv8* c, int n, const void* k, const int64_t* k_stride, const void* v, const int64_t* v_stride,
                 int dtype, int rows, const int32_t* starts, const int32_t* counts, const int32_t* tables,
                 int64_t table_stride, int max_pages, const int32_t* positions, void* stream) {
  size_t e;
  if (int r = check_cache8(c)) return r;
  if (int r = check_tables(n, tables, table_stride, max_pages)) return r;
  if (int r = check_dtype(dtype, e)) return r;
  if (starts && counts) return bad("starts and counts exclude each other");
  if (rows < 0 || (starts ? rows > (1 << 27) : rows > (1 << 20) || (long long)n * ((rows + 30) / 16) > kMaxUnits))
    return bad("rows out of range");
  Kv8StoreArgs a{};
  a.vec = 1;
  if (int r = check_strides(k, k_stride, e, a.vec)) return r;
  if (int r = check_strides(v, v_stride, e, a.vec)) return r;
  if (!aligned(starts, 4) || !aligned(counts, 4) || !positions || !aligned(positions, 4))
    return bad("starts, counts and positions must be aligned to their elements");
  if (rows == 0) return WF_OK;
  a.c = geometry(c);
  a.k = k;
  a.v = v;
  a.bf16_src = dtype == WF_BF16;
  a.kr = k_stride[0];
  a.ki = k_stride[1];
  a.kh = k_stride[2];
  a.vr = v_stride[0];
  a.vi = v_stride[1];
  a.vh = v_stride[2];
  a.rows = rows;
  a.starts = starts;
  a.counts = counts;
  a.tables = tables;
  a.ts = table_stride;
  a.max_pages = max_pages;
  a.n = n;
  a.positions = positions;
  kv8_store(a, static_cast<hipStream_t>(stream));
  return launched();
}

int wf_kv8_load(const wf_kv8* c, int n, const int32_t* tables, int64_t table_stride, int max_pages, const int32_t* lens,
                void* k, void* v, int dtype, void* stream) {
  size_t e;
  if (int r = check_cache8(c)) return r;
  if (int r = check_tables(n, tables, table_stride, max_pages)) return r;
  if ((long long)n * max_pages > kMaxUnits) return bad("n * max_pages must be below 2^24");
  if (int r = check_dtype(dtype, e)) return r;
  if (!lens || !aligned(lens, 4)) return bad("lens must be aligned to its elements");
  if (!k || !v || !aligned(k, 16) || !aligned(v, 16)) return bad("outputs must be 16-byte aligned");
  Kv8LoadArgs a{};
  a.c = geometry(c);
  a.tables = tables;
  a.ts = table_stride;
  a.max_pages = max_pages;
  a.n = n;
  a.lens = lens;
  a.k = k;
  a.v = v;
  a.bf16_out = dtype == WF_BF16;
  kv8_load(a, static_cast<hipStream_t>(stream));
  return launched();
}

int wf_kv8_attend_workspace_bytes(const wf_kv8* c, int n, int rows, int n_q_head, int max_pages, size_t* bytes) {
  if (int r = check_cache8(c, false)) return r;
  if (n < 1 || n > kMaxGrid) return bad("n must be in [1, 65535]");
  if (int r = check_heads(n_q_head, c->n_head)) return r;
  const int group = n_q_head / c->n_head;
  if (rows < 1 || rows > (1 << 19) / group) return bad("rows times a group's heads must be in [1, 2^19]");
  if (max_pages < 1 || max_pages > kKv8MaxPages) return bad("max_pages must be in [1, 2^24]");
  if (!bytes) return bad("null bytes");
  *bytes = kv8_workspace(n, rows, group, c->n_head, max_pages);
  return WF_OK;
}

int wf_kv8_attend(const wf_kv8* c, int n, const void* q, const int64_t* q_stride, int rows, int n_q_head, int dtype,
                  const int32_t* tables, int64_t table_stride, int max_pages, const int32_t* positions,
                  const int32_t* counts, void* out, void* workspace, size_t ws_bytes, void* stream) {
  size_t e, need;
  if (int r = check_cache8(c)) return r;
  if (int r = check_tables(n, tables, table_stride, max_pages)) return r;
  if (int r = check_dtype(dtype, e)) return r;
  if (int r = wf_kv8_attend_workspace_bytes(c, n, rows, n_q_head, max_pages, &need)) return r;
  Kv8AttendArgs a{};
  a.vec = 1;
  if (int r = check_strides(q, q_stride, e, a.vec)) return r;
  if (!positions || !aligned(positions, 4) || !aligned(counts, 4)) return bad("positions and counts must be aligned to their elements");
  if (!out || !aligned(out, 16)) return bad("out must be 16-byte aligned");
  if (need > 0 && (!workspace || !aligned(workspace, 256))) return bad("workspace must be 256-byte aligned");
  if (ws_bytes < need) return op_fail(WF_ESIZE, "workspace too small");
  a.c = geometry(c);
  a.q = q;
  a.sr = q_stride[0];
  a.si = q_stride[1];
  a.sh = q_stride[2];
  a.bf16_q = dtype == WF_BF16;
  a.rows = rows;
  a.group = n_q_head / c->n_head;
  a.n = n;
  a.tables = tables;
  a.ts = table_stride;
  a.max_pages = max_pages;
  a.positions = positions;
  a.counts = counts;
  a.out = out;
  a.part = static_cast<float*>(workspace);
  kv8_attend(a, static_cast<hipStream_t>(stream));
  return launched();
}

}  // extern "C"
