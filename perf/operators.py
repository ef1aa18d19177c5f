"""The calls a program makes of this library's stateless operators, as cases to time.

Four kinds of pass, all of decoding with several hypotheses (beams) per recording and
acoustic keys and values held in 4 bits:

  select   the k best continuations of every recording's beams, by cumulative
           log-probability: log-softmax over the vocabulary and the choice over beams and
           vocabulary in one call;
  reorder  the beams' page tables after a choice: beam j continues beam parents[j], full
           pages are shared, and the page that is written next is copied where two beams
           continue one;
  store    acoustic keys and values into the 4-bit cache, and the values that it then holds;
  attend   attention of a few query rows per recording over its part of the 4-bit cache.

The 4-bit form: e2m1 elements (0, 0.5, 1, 1.5, 2, 3, 4, 6 and their negatives, nearest with
ties to the even code) in blocks of 32 with a power-of-two scale, the smallest 2^e (e >= -120)
with max |x| <= 6 * 2^e.  A key's blocks lie along its 64 dimensions (two per frame), a
value's along 32 frames of one dimension.
"""
import math

import torch

own = False

HEAD = 64      # head width
PAGE = 16      # positions of a cache page
BLOCK = 32     # elements that share a scale


def listed():
    return [
        # one recording, five beams: the interactive case, where latency counts
        {"name": "select_1x5", "kind": "select", "n": 1, "beams": 5, "vocab": 51866, "k": 10, "dtype": "f32", "rows": 1,
         "suppress": False},
        # a batch engine's head output: every ninth row of a [slots * 9, vocab] buffer, suppressed tokens
        {"name": "select_16x5", "kind": "select", "n": 16, "beams": 5, "vocab": 51866, "k": 10, "dtype": "f32", "rows": 9,
         "suppress": True},
        # the whole batch with eight beams, logits in bf16, an odd vocabulary
        {"name": "select_96x8", "kind": "select", "n": 96, "beams": 8, "vocab": 51865, "k": 16, "dtype": "bf16", "rows": 1,
         "suppress": False},
        # one recording's beams, large-v3 caches: 32 blocks' keys and values, pages of 16 positions of 20 heads
        {"name": "reorder_1x5", "kind": "reorder", "n": 1, "beams": 5, "regions": 64, "heads": 20, "pages": 28, "lo": 117,
         "hi": 117},
        # eight recordings at ragged lengths
        {"name": "reorder_8x5", "kind": "reorder", "n": 8, "beams": 5, "regions": 64, "heads": 20, "pages": 28, "lo": 0,
         "hi": 447},
        # a new recording's keys and values of one decoder block
        {"name": "store_1", "kind": "store", "n": 1, "heads": 20, "frames": 1500, "lo": 1500, "dtype": "bf16"},
        # recordings of different lengths, fp32 sources
        {"name": "store_16", "kind": "store", "n": 16, "heads": 20, "frames": 1500, "lo": 1, "dtype": "f32"},
        # plain decoding of one recording: a single query row
        {"name": "attend_1x1", "kind": "attend", "n": 1, "rows": 1, "heads": 20, "frames": 1500, "lo": 1500, "dtype": "f32"},
        # a verification pass of one recording: anchor and eight candidates
        {"name": "attend_1x9", "kind": "attend", "n": 1, "rows": 9, "heads": 20, "frames": 1500, "lo": 1500, "dtype": "f32"},
        # five beams of each of 16 recordings read one acoustic memory; ragged, some of no frames
        {"name": "attend_16x5", "kind": "attend", "n": 16, "rows": 5, "heads": 20, "frames": 1500, "lo": 0, "dtype": "bf16"},
        # a verification pass of the whole batch
        {"name": "attend_96x9", "kind": "attend", "n": 96, "rows": 9, "heads": 20, "frames": 1500, "lo": 1500,
         "dtype": "f32"},
        # a long recording in one memory (131,072 frames, 44 minutes), a single row
        {"name": "attend_long", "kind": "attend", "n": 1, "rows": 1, "heads": 20, "frames": 131072, "lo": 131072,
         "dtype": "f32"},
    ]


def log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo - 0.49), math.log(hi + 0.49)))))))


def draw(rng):
    kind = rng.choice(["select", "select", "reorder", "store", "attend", "attend", "attend"])
    if kind == "select":
        beams = rng.randint(1, 16)
        vocab = log_int(rng, 64, 51866)
        n = log_int(rng, 1, min(256, 96 * 8 * 51865 // (2 * beams * vocab)))
        return {"kind": kind, "n": n, "beams": beams, "vocab": vocab, "k": rng.randint(1, min(32, 2 * beams)),
                "dtype": rng.choice(["f32", "bf16"]), "rows": rng.choice([1, 1, 9]) if n * beams < 100 else 1,
                "suppress": rng.random() < 0.4}
    if kind == "reorder":
        pages = rng.choice([4, 28])
        lo = rng.randint(0, PAGE * pages)
        return {"kind": kind, "n": log_int(rng, 1, 8), "beams": rng.randint(1, 5), "regions": rng.choice([4, 8, 24, 64]),
                "heads": rng.choice([2, 6, 12, 20]), "pages": pages, "lo": lo, "hi": rng.randint(lo, PAGE * pages)}
    heads = rng.choice([2, 6, 8, 12, 20])
    if kind == "store":
        frames = log_int(rng, 1, 4096)
        n = log_int(rng, 1, max(1, 16 * 20 * 1500 // (heads * frames)))
        return {"kind": kind, "n": min(n, 256), "heads": heads, "frames": frames, "lo": rng.choice([0, frames]),
                "dtype": rng.choice(["f32", "bf16"])}
    frames = log_int(rng, 1, 131072)
    n = log_int(rng, 1, min(256, max(1, 96 * 20 * 1500 // (heads * frames))))
    return {"kind": kind, "n": n, "rows": rng.choice([1, 1, 5, 9, rng.randint(2, 16), rng.randint(17, 48)]), "heads": heads,
            "frames": frames, "lo": rng.choice([0, frames]), "dtype": rng.choice(["f32", "bf16"])}


def dtype_of(case):
    return torch.float32 if case["dtype"] == "f32" else torch.bfloat16


def work(case):
    n = case["n"]
    if case["kind"] == "select":
        e = 4 if case["dtype"] == "f32" else 2
        size = n * case["beams"] * case["vocab"]
        return {"bytes": e * size + (case["vocab"] if case["suppress"] else 0) + n * (4 * case["beams"] + 12 * case["k"]),
                "flops": 4 * size}
    if case["kind"] == "reorder":
        # the beams that continue a parent after another one copy a page (read and written; as many as the parents'
        # distribution gives on average); the tables are read and written
        page, B = PAGE * case["heads"] * HEAD * 2, case["beams"]
        distinct = sum(1 - (1 - math.sqrt((p + 1) / B) + math.sqrt(p / B)) ** B for p in range(B))
        copies = round(sum(1 for v in positions(case) if v % PAGE) * (B - distinct))
        return {"bytes": 2 * copies * case["regions"] * page + 8 * n * case["beams"] * case["pages"], "flops": 0}
    e = 4 if case["dtype"] == "f32" else 2
    lens = lengths(case)
    elems = 2 * HEAD * case["heads"] * sum(lens)             # keys and values
    held = elems // 2 + elems // BLOCK
    if case["kind"] == "store":
        # the source read, the cache written; the values that it holds read back and written whole
        return {"bytes": e * elems + 2 * held + 4 * 2 * HEAD * case["heads"] * n * case["frames"], "flops": 0}
    return {"bytes": held + 2 * e * n * case["rows"] * case["heads"] * HEAD,
            "flops": 2 * elems * case["rows"]}


# ---------------------------------------------------------------- inputs

def lengths(case):
    """Frames of each recording: evenly over [lo, frames]."""
    n, lo, hi = case["n"], case["lo"], case["frames"]
    return [hi if n == 1 else lo + round(i * (hi - lo) / (n - 1)) for i in range(n)]


def positions(case):
    """Cached positions of each recording's beams: evenly over [lo, hi]."""
    n, lo, hi = case["n"], case["lo"], case["hi"]
    return [hi if n == 1 else lo + round(i * (hi - lo) / (n - 1)) for i in range(n)]


def generator(seed, case):
    g = torch.Generator(device="cuda")
    g.manual_seed(1000003 * seed + 7919 * case["n"] + 31)
    return g


def acoustic(case, seed):
    """Keys and values [n, frames, heads, 64] in the case's type, and each recording's frames.  Widths differ by
    dimension, as a projection's do, and some blocks are zero."""
    g = generator(seed, case)
    shape = (case["n"], case["frames"], case["heads"], HEAD)
    out = []
    for _ in range(2):
        width = torch.exp(0.7 * torch.randn((case["heads"], HEAD), device="cuda", generator=g))
        x = torch.empty(shape, dtype=dtype_of(case), device="cuda")
        for i in range(case["n"]):
            x[i] = torch.randn(shape[1:], device="cuda", generator=g) * width
        out.append(x)
    out[1][:, :, 0, :3] = 0
    lens = torch.tensor(lengths(case), dtype=torch.int32)
    lens = lens[torch.randperm(case["n"], generator=torch.Generator().manual_seed(seed))]
    return out[0], out[1], lens.cuda()


def queries(case, seed):
    g = generator(seed + 77, case)
    return torch.randn((case["n"], case["rows"], case["heads"], HEAD), device="cuda", generator=g).to(dtype_of(case))


def beam_tables(case, seed):
    """Page tables that a search leaves: the beams of a recording share a first part, the page in writing is each
    beam's own; pages are spread over the pool.  Parents favour the better beams."""
    n, B, P = case["n"], case["beams"], case["pages"]
    g = torch.Generator().manual_seed(seed * 31 + n)
    total = n * B * P
    pool = torch.randperm(total, generator=g).view(n, B * P)
    lens = torch.tensor(positions(case))
    tables = pool[:, :1].repeat(1, B * P).view(n, B, P).clone()
    for i in range(n):
        used = -(-int(lens[i]) // PAGE)
        if used == 0:
            continue
        shared = int(torch.randint(0, used, (1,), generator=g))
        tables[i, :, :shared] = pool[i, :shared]
        tables[i, :, shared:used] = pool[i, shared:shared + B * (used - shared)].view(B, used - shared)
    parents = (torch.rand((n, B), generator=g) ** 2 * B).long().clamp(max=B - 1)
    as32 = lambda t: t.to(torch.int32).cuda()  # noqa: E731
    return as32(tables), as32(parents), as32(lens), as32(pool)


def prepare(case, seed):
    kind = case["kind"]
    if kind == "select":
        g = generator(seed, case)
        n, B, V = case["n"], case["beams"], case["vocab"]
        # a language model's logits: most of the mass on a few tokens
        buf = torch.empty((n, B, case["rows"], V), dtype=dtype_of(case), device="cuda")
        for i in range(n):
            buf[i] = 3.0 * torch.randn(buf.shape[1:], device="cuda", generator=g)
        logits = buf[:, :, 0]
        scores = -20.0 * torch.rand((n, B), device="cuda", generator=g)
        if case["n"] > 1:
            scores[0, 1:] = -math.inf  # a recording's first choice: one beam lives
        mask = (torch.rand(V, device="cuda", generator=g) < 0.03).to(torch.uint8) if case["suppress"] else None
        return {"kind": kind, "k": case["k"], "logits": logits, "scores": scores, "suppress": mask}
    if kind == "reorder":
        g = generator(seed, case)
        tables, parents, lens, pool = beam_tables(case, seed)
        shape = (case["regions"], pool.numel(), PAGE * case["heads"] * HEAD)
        cache = torch.empty(shape, dtype=torch.bfloat16, device="cuda")
        for r in range(shape[0]):
            cache[r] = torch.randn(shape[1:], device="cuda", generator=g)
        return {"kind": kind, "cache": cache, "tables": tables, "parents": parents, "lens": lens, "pool": pool}
    k, v, lens = acoustic(case, seed)
    full = case["lo"] == case["frames"]
    state = {"kind": kind, "lens": None if full else lens, "frames": case["frames"]}
    if own:
        from paper_2609_32869_amd import AcousticCache4
        state["cache"] = AcousticCache4(case["n"], case["heads"], case["frames"])
    if kind == "store":
        state.update(k=k, v=v)
        return state
    state["q"] = queries(case, seed)
    # what a request's set-up left: the library's cache, or the same codes and scales as plain tensors
    if own:
        state["cache"].store(0, k, v, state["lens"])
    else:
        state["held"] = plain_store(k, v, state["lens"])
    return state


# ---------------------------------------------------------------- the operators in elementary operations

def run(state):
    if own:
        return run_own(state)
    kind = state["kind"]
    if kind == "select":
        return plain_select(state["logits"], state["scores"], state["k"], state["suppress"])
    if kind == "reorder":
        return plain_reorder(state["cache"], state["tables"], state["parents"], state["lens"], state["pool"])
    if kind == "store":
        return plain_values(*plain_store(state["k"], state["v"], state["lens"]), state["frames"])
    return plain_attend(state["q"], *state["held"], state["lens"], state["frames"])


def run_own(state):
    import paper_2609_32869_amd as wf
    kind = state["kind"]
    if kind == "select":
        return wf.beam_select(state["logits"], state["scores"], state["k"], suppress=state["suppress"])
    if kind == "reorder":
        new = wf.cache_reorder(state["cache"], state["tables"], state["parents"], state["lens"], state["pool"], PAGE)
        return new, state["cache"]
    if kind == "store":
        state["cache"].store(0, state["k"], state["v"], state["lens"])
        return state["cache"].load(0, len(state["k"]))
    return state["cache"].attend(0, state["q"], state["lens"])


def plain_select(logits, scores, k, suppress):
    """64 bits: a candidate's rank is a border, and sums of exponentials over a vocabulary set it."""
    n, B, V = logits.shape
    x = logits.double()
    if suppress is not None:
        x = torch.where(suppress.bool(), -math.inf, x)
    top = x.amax(-1, keepdim=True)
    lse = top + torch.log(torch.exp(x - top).sum(-1, keepdim=True))
    flat = (scores.double()[:, :, None] + (x - lse)).reshape(n, B * V)
    value, index = [], []
    for _ in range(k):                                       # argmax gives the first of equal values
        at = flat.argmax(-1, keepdim=True)
        value.append(flat.gather(1, at))
        index.append(at)
        flat.scatter_(1, at, -math.inf)
    value, index = torch.cat(value, 1), torch.cat(index, 1)
    none = value == -math.inf
    return value.float(), torch.where(none, -1, index // V).int(), torch.where(none, -1, index % V).int()


def plain_reorder(cache, tables, parents, lens, pool):
    n, B, P = tables.shape
    L = lens.long()[:, None]
    last, part = L // PAGE, L % PAGE > 0
    column = torch.arange(P, device=tables.device)[None, None]
    kept = tables.gather(1, parents.long()[:, :, None].expand(n, B, P)).long()
    held = column * PAGE < L[:, :, None]
    flags = torch.zeros(cache.shape[1] + 1, dtype=torch.int32, device=tables.device)
    flags[torch.where(held, kept, cache.shape[1]).flatten()] = 1
    free = pool.long().gather(1, torch.sort(flags[pool.long()], dim=1, stable=True).indices)
    mine = kept.gather(2, last.clamp(max=P - 1)[:, :, None].expand(n, B, 1))[:, :, 0]
    again = ((mine[:, :, None] == mine[:, None, :]) & torch.ones((B, B), device=mine.device).tril(-1).bool()).any(-1)
    need = (last < P) & (~part | again)
    fresh = free.gather(1, (need.long().cumsum(1) - 1).clamp(min=0))
    new = torch.where(held, kept, pool.long()[:, :1, None])
    new = torch.where((column == last[:, :, None]) & need[:, :, None], fresh[:, :, None], new)
    # every beam's page of the next position; those that are not copied go to themselves
    to = torch.where(need, fresh, mine).flatten()
    cache[:, to] = cache[:, torch.where(need & part, mine, to.view(n, B)).flatten()]
    return new.int(), cache


def plain_quantise(x):
    """Codes (uint8, 0..15) and exponents of blocks along the last axis of 32."""
    mag = x.abs()
    m, e = torch.frexp(mag.amax(-1, keepdim=True))
    e = torch.where(m <= 0.75, e - 3, e - 2).clamp(min=-120)
    y = torch.ldexp(mag, -e)
    half = torch.round(y * 2)                                # codes 0..3 in steps of one half, ties to even
    code = torch.where(y < 2, half, torch.where(y < 4, torch.round(y) + 2, torch.round(y / 2) + 4))
    return (code.to(torch.uint8) + 8 * torch.signbit(x).to(torch.uint8)), e.squeeze(-1).to(torch.int8)


def pack(code):
    return code[..., 0::2] + 16 * code[..., 1::2]


def unpack(packed, e):
    code = torch.stack((packed & 15, packed >> 4), -1).flatten(-2)
    grid = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6], device=packed.device)
    grid = torch.cat((grid, -grid))
    return torch.ldexp(grid[code.long()], e.unsqueeze(-1).int())


def plain_store(k, v, lens):
    n, F, H, _ = k.shape
    groups = -(-F // BLOCK)
    if lens is not None:
        live = (torch.arange(F, device=k.device)[None] < lens[:, None])[:, :, None, None]
        k, v = torch.where(live, k, 0), torch.where(live, v, 0)
    kc, ke = plain_quantise(k.float().permute(0, 2, 1, 3).reshape(n, H, F, HEAD // BLOCK, BLOCK))
    vp = torch.zeros((n, groups * BLOCK, H, HEAD), device=k.device)
    vp[:, :F] = v
    vc, ve = plain_quantise(vp.view(n, groups, BLOCK, H, HEAD).permute(0, 3, 1, 4, 2))
    return pack(kc), ke, pack(vc), ve


def plain_heads(kc, ke, vc, ve, frames):
    """Keys and values [n, heads, frames, 64]."""
    n, H = kc.shape[:2]
    k = unpack(kc, ke).reshape(n, H, frames, HEAD)
    v = unpack(vc, ve).permute(0, 1, 2, 4, 3).reshape(n, H, -1, HEAD)[:, :, :frames]
    return k, v


def plain_values(kc, ke, vc, ve, frames):
    k, v = plain_heads(kc, ke, vc, ve, frames)
    return k.transpose(1, 2).contiguous(), v.transpose(1, 2).contiguous()


def plain_attend(q, kc, ke, vc, ve, lens, frames):
    k, v = plain_heads(kc, ke, vc, ve, frames)
    s = 0.125 * torch.matmul(q.float().transpose(1, 2), k.transpose(2, 3).contiguous())
    if lens is not None:
        live = (torch.arange(frames, device=q.device)[None] < lens[:, None])[:, None, None]
        s = torch.where(live, s, -math.inf)
    top = s.amax(-1, keepdim=True)
    p = torch.exp(s - torch.where(top == -math.inf, 0, top))
    total = p.sum(-1, keepdim=True)
    o = torch.matmul(p, v.contiguous()) / torch.where(total == 0, 1, total)
    return o.transpose(1, 2).contiguous().to(q.dtype)


# ---------------------------------------------------------------- the definitions in 64 bits

def exact(case, seed):
    kind = case["kind"]
    if kind == "select":
        s = prepare(case, seed)
        out = [exact_select(x, sc, case["k"], s["suppress"]) for x, sc in zip(s["logits"], s["scores"])]
        return tuple(torch.stack([torch.tensor([c[j] for c in o], dtype=torch.float64 if j == 0 else torch.int32) for o in out])
                     for j in range(3))
    if kind == "reorder":
        return exact_tables(*beam_tables(case, seed)), None
    k, v, lens = acoustic(case, seed)
    inside = torch.arange(case["frames"], device="cuda").view(1, -1, 1, 1) < lens.view(-1, 1, 1, 1)
    k, v = k.double() * inside, v.double() * inside
    k = nearest(k.unflatten(-1, (2, BLOCK)), -1).flatten(-2)
    short = -case["frames"] % BLOCK
    v = nearest(torch.nn.functional.pad(v, (0, 0, 0, 0, 0, short)).unflatten(1, (-1, BLOCK)), 2).flatten(1, 2)[:, :case["frames"]]
    if kind == "store":
        return k, v
    q = queries(case, seed).double()
    out = torch.zeros_like(q)
    for i in range(case["n"]):
        m = int(lens[i])
        if m == 0:
            continue
        for h in range(case["heads"]):
            w = torch.softmax(q[i, :, h] @ k[i, :m, h].T / 8.0, -1)
            out[i, :, h] = w @ v[i, :m, h]
    return out


def exact_select(x, scores, k, suppress):
    """(score, beam, token) of one recording's k best, from every beam's own best."""
    found = []
    for b in range(len(x)):
        row = x[b].double()
        if suppress is not None:
            row = row.masked_fill(suppress != 0, -math.inf)
        logp = torch.log_softmax(row, 0) + scores[b].double()
        keep = min(len(row), k)
        value, index = torch.sort(logp, descending=True, stable=True)
        found += [(p, b, t) for p, t in zip(value[:keep].tolist(), index[:keep].tolist()) if p > -math.inf]
    found.sort(key=lambda c: (-c[0], c[1], c[2]))
    return (found + [(-math.inf, -1, -1)] * k)[:k]


def exact_tables(tables, parents, lens, pool):
    out = []
    for T, par, L, Q in zip(tables.tolist(), parents.tolist(), lens.tolist(), pool.tolist()):
        P, last = len(T[0]), L // PAGE
        rows = [[T[p][c] if c * PAGE < L else Q[0] for c in range(P)] for p in par]
        taken = {r[c] for r in rows for c in range(P) if c * PAGE < L}
        spare = [page for page in Q if page not in taken]
        for j, r in enumerate(rows):
            if last < P and (L % PAGE == 0 or r[last] in [rows[i][last] for i in range(j)]):
                r[last] = spare.pop(0)
        out.append(rows)
    return torch.tensor(out, dtype=torch.int32)


def nearest(x, axis):
    """The 4-bit grid's value nearest to each element, the even code of two; `axis`: the 32 that share a scale."""
    grid = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6], dtype=torch.float64, device=x.device)
    peak = x.abs().amax(axis, keepdim=True)
    step = torch.full_like(peak, 2.0 ** -120)
    need = peak / 6 > step
    up = torch.exp2(torch.ceil(torch.log2(torch.where(need, peak / 6, torch.ones_like(peak)))))
    up = torch.where(peak <= 3 * up, up / 2, up)             # where the logarithm's rounding went past a border
    up = torch.where(peak > 6 * up, up * 2, up)
    step = torch.where(need, up, step)
    y = x.abs() / step
    low = (torch.searchsorted(grid, y.contiguous(), right=True) - 1).clamp(0, 6)
    below, above = y - grid[low], grid[low + 1] - y
    code = torch.where((above < below) | ((above == below) & (low % 2 == 1)), low + 1, low)
    return torch.copysign(grid[code], x) * step
