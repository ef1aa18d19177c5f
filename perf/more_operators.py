"""The calls a program makes for a decoder's self-attention, from the prompt to single tokens, as
cases to time.

Four kinds of pass:

  rotary  rotary positions of queries and keys in one call: halves or interleaved pairs, the
          whole head or its first part, frequencies scaled for long contexts;
  prompt  causal attention of packed prompts of different lengths, heads in groups that share a
          key and value head;
  store   keys and values into a paged cache in 8 bits, appended to what its pages hold, and the
          values that the written pages then stand for;
  attend  attention of one or a few rows per request over its pages.

The 8-bit form: e4m3 elements (nearest, ties to the even code) with one power-of-two scale for
the keys and one for the values of a page (16 positions) and head, the smallest 2^e (e >= -100)
with max |x| <= 448 * 2^e.  Appending to a page that is part-filled rounds the values that it
stands for and the new ones to their common scale; positions behind the last hold zeros.
"""
import math

import torch

own = False

HEAD = 64      # head width
PAGE = 16      # positions of a cache page
LOWEST = -100  # smallest exponent of a scale


def listed():
    return [
        # one new token's query and key in plain decoding: latency
        {"name": "rotary_1", "kind": "rotary", "tokens": 1, "heads": 20, "kv": 20, "dims": 64, "pairs": "halves",
         "scaling": "none", "far": 447, "dtype": "f32"},
        # a verification pass of a whole batch: 96 recordings' anchors and eight candidates
        {"name": "rotary_864", "kind": "rotary", "tokens": 864, "heads": 20, "kv": 20, "dims": 64, "pairs": "halves",
         "scaling": "linear", "far": 447, "dtype": "bf16"},
        # a long prompt far past the trained context: half of the head, interleaved, scaled by parts
        {"name": "rotary_long", "kind": "rotary", "tokens": 65536, "heads": 32, "kv": 8, "dims": 32, "pairs": "interleaved",
         "scaling": "ramp", "far": 1 << 20, "dtype": "bf16"},
        # one recording's prompt with the text before it (half the context), fp32
        {"name": "prompt_224", "kind": "prompt", "n": 1, "tokens": 224, "lo": 224, "heads": 20, "kv": 20, "rest": 0, "dtype": "f32"},
        # a batch's prompts, packed: one token to the context, rows of no prompt behind the last
        {"name": "prompt_96", "kind": "prompt", "n": 96, "tokens": 21504, "lo": 1, "heads": 20, "kv": 20, "rest": 67, "dtype": "bf16"},
        # fp32 prompts of ragged lengths, grouped heads
        {"name": "prompt_f32", "kind": "prompt", "n": 5, "tokens": 9001, "lo": 300, "heads": 12, "kv": 6, "rest": 0, "dtype": "f32"},
        # one long document
        {"name": "prompt_long", "kind": "prompt", "n": 1, "tokens": 32768, "lo": 32768, "heads": 32, "kv": 8, "rest": 0, "dtype": "bf16"},
        # a verification pass's nine rows appended to every recording's pages
        {"name": "store_96x9", "kind": "store", "n": 96, "rows": 9, "packed": False, "at": 430, "kv": 20, "dtype": "bf16"},
        # packed prompts into an empty cache
        {"name": "store_prompts", "kind": "store", "n": 8, "rows": 8192, "packed": True, "at": 0, "kv": 8, "dtype": "f32"},
        # plain decoding of one recording at the end of its context
        {"name": "attend_1x1", "kind": "attend", "n": 1, "rows": 1, "lo": 447, "hi": 447, "heads": 20, "kv": 20, "dtype": "f32"},
        # a verification pass of the whole batch at ragged positions
        {"name": "attend_96x9", "kind": "attend", "n": 96, "rows": 9, "lo": 0, "hi": 438, "heads": 20, "kv": 20, "dtype": "bf16"},
        # four long contexts, one token each, grouped heads
        {"name": "attend_long", "kind": "attend", "n": 4, "rows": 1, "lo": 131071, "hi": 131071, "heads": 32, "kv": 8, "dtype": "bf16"},
    ]


def log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo - 0.49), math.log(hi + 0.49)))))))


def draw(rng):
    kind = rng.choice(["rotary", "rotary", "prompt", "prompt", "prompt", "store", "store", "attend", "attend", "attend"])
    dtype = rng.choice(["f32", "bf16"])
    heads, kv = rng.choice([(2, 2), (6, 6), (6, 1), (8, 8), (8, 2), (12, 12), (12, 6), (14, 2), (20, 20), (32, 8), (32, 4), (24, 1)])
    if kind == "rotary":
        return {"kind": kind, "tokens": log_int(rng, 1, 65536 * 40 // (heads + kv) // (2 if dtype == "f32" else 1)), "heads": heads,
                "kv": kv, "dims": rng.choice([2, 16, 32, 48, 64, 64, 64, 2 * rng.randint(2, 32)]),
                "pairs": rng.choice(["halves", "interleaved"]),
                "scaling": rng.choice(["none", "linear", "base", "ramp"]), "far": log_int(rng, 1, 1 << 20), "dtype": dtype}
    if kind == "prompt":
        tokens = log_int(rng, 1, 16384 if dtype == "bf16" else 6000)
        n = log_int(rng, 1, min(tokens, 256))
        return {"kind": kind, "n": n, "tokens": tokens, "lo": rng.randint(0, tokens // n), "heads": heads, "kv": kv,
                "rest": rng.choice([0, 0, rng.randint(1, 200)]), "dtype": dtype}
    if kind == "store":
        packed = rng.random() < 0.5
        rows = log_int(rng, 1, 8192) if packed else rng.choice([1, 1, 9, rng.randint(2, 48)])
        n = log_int(rng, 1, min(256, max(1, 8 * 8 * 8192 // (kv * rows))))
        return {"kind": kind, "n": n, "rows": rows, "packed": packed, "at": rng.choice([0, rng.randint(1, 900)]), "kv": kv,
                "dtype": dtype}
    hi = log_int(rng, 1, 131071)
    n = log_int(rng, 1, min(256, max(1, 4 * 131072 * 8 // (kv * (hi + 64)))))
    return {"kind": kind, "n": n, "rows": rng.choice([1, 1, 1, 5, 9, rng.randint(2, 16), rng.randint(17, 48)]),
            "lo": rng.choice([0, hi, hi // 2]), "hi": hi, "heads": heads, "kv": kv, "dtype": dtype}


def dtype_of(case):
    return torch.float32 if case["dtype"] == "f32" else torch.bfloat16


def work(case):
    kind, e = case["kind"], 4 if case["dtype"] == "f32" else 2
    if kind == "rotary":
        size = case["tokens"] * (case["heads"] + case["kv"])
        return {"bytes": 2 * e * size * HEAD + 4 * case["tokens"], "flops": 3 * size * case["dims"]}
    if kind == "prompt":
        pairs = sum(m * (m + 1) // 2 for m in lengths(case))
        rows = case["tokens"]
        return {"bytes": e * HEAD * (rows * (2 * case["heads"] + 2 * case["kv"])), "flops": 4 * HEAD * case["heads"] * pairs}
    KV = case["kv"]
    if kind == "store":
        # the new rows read, the pages' kept values read, the pages written; the pages read back and their values written
        counts, at = counts_of(case), starts_at(case)
        pages = sum(-(-(p % PAGE + c) // PAGE) for p, c in zip(at, counts) if c)
        kept = sum(p % PAGE for p, c in zip(at, counts) if c)
        held = pages * KV * (2 * PAGE * HEAD + 2)
        values = 4 * 2 * HEAD * KV * case["n"] * PAGE * columns(case)
        return {"bytes": 2 * e * HEAD * KV * sum(counts) + 2 * HEAD * KV * kept + 2 * held + values, "flops": 0}
    sees = [p + case["rows"] for p in starts_at(case)]
    rows = case["n"] * case["rows"] * case["heads"]
    pairs = sum(case["rows"] * p + case["rows"] * (case["rows"] + 1) // 2 for p in starts_at(case))
    return {"bytes": sum(2 * HEAD * KV * m + 2 * KV * -(-m // PAGE) for m in sees) + 2 * e * rows * HEAD,
            "flops": 4 * HEAD * case["heads"] * pairs}


# ---------------------------------------------------------------- inputs

def spread(n, lo, hi):
    """n whole numbers evenly over [lo, hi]; the last alone where n is 1."""
    return [hi if n == 1 else lo + round(i * (hi - lo) / (n - 1)) for i in range(n)]


def lengths(case):
    """Rows of each packed prompt: from `lo` on and growing evenly, `tokens` in all."""
    n, lo = case["n"], case["lo"]
    more = case["tokens"] - n * lo
    ends = [more * i * (i + 1) // (n * (n + 1)) for i in range(n + 1)]
    return [lo + b - a for a, b in zip(ends, ends[1:])]


def counts_of(case):
    """Rows that each request appends: all of them, packed prompts from 1 to twice the mean."""
    return spread(case["n"], 1, 2 * case["rows"] - 1) if case["packed"] and case["n"] > 1 else [case["rows"]] * case["n"]


def starts_at(case):
    """Positions before a request's first row."""
    return spread(case["n"], 0, case["at"]) if case["kind"] == "store" else spread(case["n"], case["lo"], case["hi"])


def columns(case):
    """Pages of a request that a store can touch."""
    return (max(counts_of(case)) + 2 * PAGE - 2) // PAGE


def generator(seed, case):
    g = torch.Generator(device="cuda")
    g.manual_seed(1000003 * seed + 7919 * case.get("n", 1) + case["heads" if "heads" in case else "kv"])
    return g


def order(values, seed):
    """The values in an order of the seed's."""
    at = torch.randperm(len(values), generator=torch.Generator().manual_seed(seed)).tolist()
    return [values[i] for i in at]


def as32(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def running(counts):
    out = [0]
    for c in counts:
        out.append(out[-1] + c)
    return out


def rows_like(case, g, shape):
    """Keys or values: widths differ by dimension, as a projection's do."""
    width = torch.exp(0.7 * torch.randn(shape[-2:], device="cuda", generator=g))
    x = torch.empty(shape, dtype=dtype_of(case), device="cuda")
    for part, size in zip(x.split(65536), (s.shape for s in x.split(65536))):
        part.copy_(torch.randn(size, device="cuda", generator=g) * width)
    return x


def packed_rows(case, seed):
    """Queries, keys and values of packed prompts, as slices of one projection's output, and the prompts' borders."""
    g = generator(seed, case)
    T, H, KV = case["tokens"] + case["rest"], case["heads"], case["kv"]
    qkv = torch.empty((T, H + 2 * KV, HEAD), dtype=dtype_of(case), device="cuda")
    qkv[:, :H] = torch.randn((T, H, HEAD), device="cuda", generator=g)
    qkv[:, H:H + KV] = torch.randn((T, KV, HEAD), device="cuda", generator=g)
    qkv[:, H + KV:] = rows_like(case, g, (T, KV, HEAD))
    starts = as32(running(order(lengths(case), seed)))
    return qkv[:, :H], qkv[:, H:H + KV], qkv[:, H + KV:], starts


def page_tables(n, width, seed):
    """Pages spread over a pool that holds as many as the tables name."""
    g = torch.Generator().manual_seed(31 * seed + n)
    return torch.randperm(n * width, generator=g).view(n, width).to(torch.int32).cuda()


def cache_rows(case, seed):
    """What a request's pages hold before the pass and what the pass appends."""
    g = generator(seed + 5, case)
    n, KV = case["n"], case["kv"]
    at = order(starts_at(case), seed)
    if case["kind"] == "attend":
        longest = max(at) + case["rows"]
        tables = page_tables(n, -(-longest // PAGE), seed)
        return {"at": as32(at), "tables": tables, "old": [rows_like(case, g, (n, longest, KV, HEAD)) for _ in range(2)],
                "held": as32([p + case["rows"] for p in at]), "longest": longest}
    counts = order(counts_of(case), seed + 1)
    tables = page_tables(n, max(p // PAGE for p in at) + columns(case), seed)
    out = {"at": as32(at), "tables": tables, "old": [rows_like(case, g, (n, max(1, max(at)), KV, HEAD)) for _ in range(2)],
           "held": as32(at), "longest": max(1, max(at)), "most": max(counts)}
    if case["packed"]:
        out["starts"] = as32(running(counts))
        out["new"] = [rows_like(case, g, (sum(counts), KV, HEAD)) for _ in range(2)]
    else:
        out["new"] = [rows_like(case, g, (n, case["rows"], KV, HEAD)) for _ in range(2)]
    first = torch.tensor([p // PAGE for p in at], device="cuda")
    wide = first[:, None] + torch.arange(columns(case), device="cuda")
    out["touched"] = tables.gather(1, wide).contiguous()
    out["written"] = as32([p % PAGE + c for p, c in zip(at, counts)])
    return out


def frequencies(case):
    """Turns a position of every pair, in 64 bits, and the amplitude."""
    dims, base, factor, context = case["dims"], 10000.0, 8.0, 4096.0
    if case["scaling"] == "base" and dims > 2:
        base *= factor ** (dims / (dims - 2))
    f = [base ** (-2 * i / dims) / (2 * math.pi) for i in range(dims // 2)]
    if case["scaling"] == "linear":
        f = [x / factor for x in f]
    if case["scaling"] == "ramp":
        mix = [min(max((x * context - 1.0) / (32.0 - 1.0), 0.0), 1.0) for x in f]
        f = [x * (w + (1 - w) / factor) for x, w in zip(f, mix)]
    return f, 0.1 * math.log(factor) + 1 if case["scaling"] == "ramp" else 1.0


def rotary_rows(case, seed):
    g = generator(seed, case)
    T, H, KV = case["tokens"], case["heads"], case["kv"]
    qkv = torch.randn((T, H + 2 * KV, HEAD), device="cuda", generator=g).to(dtype_of(case))
    at = torch.randint(0, case["far"] + 1, (T,), device="cuda", generator=g, dtype=torch.int32)
    return qkv[:, :H], qkv[:, H:H + KV], at


def prepare(case, seed):
    kind = case["kind"]
    if kind == "rotary":
        q, k, at = rotary_rows(case, seed)
        state = {"kind": kind, "q": q, "k": k, "at": at}
        if own:
            from paper_2609_32869_amd import Rotary
            scaling = {"none": {}, "linear": {"scaling": "linear", "factor": 8.0}, "base": {"scaling": "base", "factor": 8.0},
                       "ramp": {"scaling": "ramp", "factor": 8.0, "context": 4096}}[case["scaling"]]
            if case["dims"] == 2 and case["scaling"] == "base":
                scaling = {}                                     # one frequency of 1 at any base
            state["rotary"] = Rotary(case["dims"], interleaved=case["pairs"] == "interleaved", **scaling)
        else:
            f, state["amplitude"] = frequencies(case)
            state["turns"] = torch.tensor(f, dtype=torch.float64, device="cuda")
            state["pairs"] = case["pairs"]
        return state
    if kind == "prompt":
        q, k, v, starts = packed_rows(case, seed)
        state = {"kind": kind, "q": q, "k": k, "v": v, "starts": starts}
        if not own:
            state["borders"] = running(order(lengths(case), seed))
        return state
    state = dict(cache_rows(case, seed), kind=kind, kv=case["kv"], n=case["n"])
    pages = state["tables"].numel()
    zero = torch.zeros(case["n"], dtype=torch.int32, device="cuda")
    old = state.pop("old")
    if own:
        from paper_2609_32869_amd import PagedCache8
        state["cache"] = PagedCache8(pages, case["kv"])
        state["cache"].store(*old, state["tables"], zero, counts=state["held"])
    else:
        # one page more than the tables name: what is to be written nowhere goes there
        form = [(torch.zeros((pages + 1, PAGE, case["kv"], HEAD), device="cuda").to(torch.float8_e4m3fn),
                 torch.full((pages + 1, case["kv"]), LOWEST, dtype=torch.int32, device="cuda")) for _ in range(2)]
        state["form"] = form
        for (code, e), x in zip(form, old):
            plain_store(code, e, x.flatten(0, 1), state["tables"], zero, torch.arange(case["n"], device="cuda") * state["longest"],
                        state["held"], state["longest"])
    if kind == "attend":
        g = generator(seed + 77, case)
        state["q"] = torch.randn((case["n"], case["rows"], case["heads"], HEAD), device="cuda", generator=g).to(dtype_of(case))
    return state


# ---------------------------------------------------------------- the operators in elementary operations

def run(state):
    if own:
        return run_own(state)
    kind = state["kind"]
    if kind == "rotary":
        return plain_rotary(state)
    if kind == "prompt":
        return plain_prompt(state["q"], state["k"], state["v"], state["borders"])
    if kind == "store":
        n, out = state["n"], []
        for (code, e), x in zip(state["form"], state["new"]):
            if "starts" in state:
                first, counts = state["starts"][:-1].long(), state["starts"].diff()
            else:
                first = torch.arange(n, device=x.device) * x.shape[1]
                counts, x = torch.full_like(state["at"], x.shape[1]), x.flatten(0, 1)
            plain_store(code, e, x, state["tables"], state["at"], first, counts, state["most"])
            out.append(plain_values(code, e, state["touched"], state["written"]))
        return out
    return plain_attend(state["q"], state["form"], state["tables"], state["at"])


def run_own(state):
    import paper_2609_32869_amd as wf
    kind = state["kind"]
    if kind == "rotary":
        return state["rotary"].rotate(state["at"], state["q"], state["k"])
    if kind == "prompt":
        return wf.prompt_attention(state["q"], state["k"], state["v"], state["starts"])
    if kind == "store":
        state["cache"].store(*state["new"], state["tables"], state["at"], starts=state.get("starts"))
        return state["cache"].load(state["touched"], state["written"])
    return state["cache"].attend(state["q"], state["tables"], state["at"])


def plain_rotary(state):
    angle = state["at"].double()[:, None] * state["turns"] * (2 * math.pi)
    c = (state["amplitude"] * torch.cos(angle)).float()[:, None]
    s = (state["amplitude"] * torch.sin(angle)).float()[:, None]
    half = c.shape[-1]
    out = []
    for x in (state["q"], state["k"]):
        y = x.float().clone()
        if state["pairs"] == "halves":
            a, b = slice(0, half), slice(half, 2 * half)
        else:
            a, b = slice(0, 2 * half, 2), slice(1, 2 * half, 2)
        u, w = y[..., a].clone(), y[..., b].clone()
        y[..., a], y[..., b] = u * c - w * s, w * c + u * s
        out.append(y.to(x.dtype))
    return out


def softmax_rows(s):
    top = s.amax(-1, keepdim=True)
    p = torch.exp(s - torch.where(top == -math.inf, 0, top))
    total = p.sum(-1, keepdim=True)
    return p / torch.where(total == 0, 1, total)


def plain_prompt(q, k, v, borders):
    H, KV = q.shape[1], k.shape[1]
    out = torch.zeros(q.shape, device=q.device)
    for a, b in zip(borders, borders[1:]):
        if a == b:
            continue
        m = b - a
        hidden = torch.ones((m, m), dtype=torch.bool, device=q.device).triu(1)
        each = max(1, min(H, (1 << 29) // (m * m)))              # heads at a time: scores of 2 GB
        for h in range(0, H, each):
            heads = torch.arange(h, min(h + each, H), device=q.device)
            x = q[a:b, h:h + each].float().transpose(0, 1).contiguous()
            y = k[a:b].float()[:, heads // (H // KV)].permute(1, 2, 0).contiguous()
            s = torch.matmul(x, y).mul_(0.125).masked_fill_(hidden, -math.inf)
            z = v[a:b].float()[:, heads // (H // KV)].transpose(0, 1).contiguous()
            out[a:b, h:h + each] = torch.matmul(softmax_rows(s), z).transpose(0, 1)
    return out.to(q.dtype)


def plain_round(x):
    """x: [..., PAGE, heads, HEAD] -> the nearest values with a scale for each (PAGE, HEAD), in units of it, and its exponent."""
    top = x.abs().amax((-3, -1))
    m, e = torch.frexp(top)                                      # top = m 2^e, 0.5 <= m < 1; 448 = 0.875 2^9
    e = torch.where(m <= 0.875, e - 9, e - 8).clamp(min=LOWEST)
    y = torch.ldexp(x, -e[..., None, :, None])
    step = (torch.frexp(y)[1] - 4).clamp(min=-9)                 # three bits behind the first, from 2^-6 on
    return torch.ldexp(torch.round(torch.ldexp(y, -step)), step), e


def plain_store(code, e, x, tables, at, first, counts, most):
    """x: [rows, heads, HEAD], of which request r appends counts[r] (at most `most`) from first[r] on at position at[r]."""
    n, P = tables.shape
    cols = (most + 2 * PAGE - 2) // PAGE
    start = (at % PAGE).long()[:, None]
    slot = torch.arange(cols * PAGE, device=x.device)[None]
    t = slot - start
    fresh = (t >= 0) & (t < counts[:, None])
    kept = t < 0
    column = (at // PAGE).long()[:, None] + torch.arange(cols, device=x.device)
    live = (torch.arange(cols, device=x.device)[None] * PAGE < start + counts[:, None]) & (counts[:, None] > 0)
    page = torch.where(live, tables.gather(1, column.clamp(max=P - 1)).long(), code.shape[0] - 1)
    rows = x[(first[:, None] + t).clamp(0, len(x) - 1)].float()
    old = torch.ldexp(code[page].float(), e[page][:, :, None, :, None]).flatten(1, 2)
    y = torch.where(fresh[:, :, None, None], rows, torch.where(kept[:, :, None, None], old, 0))
    y, exponent = plain_round(y.unflatten(1, (cols, PAGE)))
    code[page], e[page] = y.to(code.dtype), exponent


def plain_values(code, e, tables, lens):
    x = torch.ldexp(code[tables.long()].float(), e[tables.long()][:, :, None, :, None]).flatten(1, 2)
    live = torch.arange(x.shape[1], device=x.device)[None] < lens[:, None]
    return torch.where(live[:, :, None, None], x, 0)


def plain_attend(q, form, tables, at):
    n, rows, H, _ = q.shape
    k, v = (torch.ldexp(code[tables.long()].float(), e[tables.long()][:, :, None, :, None]).flatten(1, 2) for code, e in form)
    KV, L = k.shape[2], k.shape[1]
    sees = at[:, None] + torch.arange(rows, device=q.device)
    live = torch.arange(L, device=q.device) <= sees[:, :, None]                       # [n, rows, L]
    v = torch.where(live[:, -1, :, None, None], v, 0)            # places that nothing was stored in may hold anything
    x = q.float().view(n, rows, KV, H // KV, HEAD).permute(0, 2, 3, 1, 4).reshape(n, KV, -1, HEAD)
    s = torch.matmul(x, k.permute(0, 2, 3, 1).contiguous()).mul_(0.125).view(n, KV, H // KV, rows, L)
    p = softmax_rows(torch.where(live[:, None, None], s, -math.inf)).view(n, KV, -1, L)
    o = torch.matmul(p, v.transpose(1, 2).contiguous()).view(n, KV, H // KV, rows, HEAD)
    return o.permute(0, 3, 1, 2, 4).reshape(n, rows, H, HEAD).to(q.dtype)


# ---------------------------------------------------------------- the definitions in 64 bits

def exact(case, seed):
    kind = case["kind"]
    if kind == "rotary":
        q, k, at = rotary_rows(case, seed)
        return [exact_rotary(case, x.double(), at) for x in (q, k)]
    if kind == "prompt":
        q, k, v, starts = packed_rows(case, seed)
        return exact_prompt(q, k, v, starts.tolist(), case["heads"] // case["kv"])
    s = cache_rows(case, seed)
    at, tables = s["at"].tolist(), s["tables"]
    if kind == "store":
        counts = s["starts"].diff().tolist() if case["packed"] else [case["rows"]] * case["n"]
        offset = s["starts"].tolist() if case["packed"] else [case["rows"] * r for r in range(case["n"])]
        out = []
        for old, new in zip(s["old"], s["new"]):
            new = new.reshape(-1, case["kv"], HEAD)
            whole = torch.zeros((case["n"], columns(case) * PAGE, case["kv"], HEAD), dtype=torch.float64, device="cuda")
            for r, (p, c) in enumerate(zip(at, counts)):
                m = p % PAGE
                if m:
                    whole[r, :m] = nearest(old[r, p - m:p].double())
                whole[r, m:m + c] = new[offset[r]:offset[r] + c].double()
                used = -(-(m + c) // PAGE) * PAGE
                for a in range(0, used, PAGE * 256):
                    part = whole[r, a:min(used, a + PAGE * 256)]
                    part.copy_(nearest(part))
            out.append(whole)
        return out
    g = generator(seed + 77, case)
    q = torch.randn((case["n"], case["rows"], case["heads"], HEAD), device="cuda", generator=g).to(dtype_of(case)).double()
    out = torch.zeros_like(q)
    group = case["heads"] // case["kv"]
    for r, p in enumerate(at):
        L = p + case["rows"]
        k, v = (nearest(x[r, :L].double()) for x in s["old"])
        hidden = torch.arange(L, device="cuda")[None] > p + torch.arange(case["rows"], device="cuda")[:, None]
        for h in range(case["heads"]):
            w = q[r, :, h] @ k[:, h // group].T / 8.0
            out[r, :, h] = torch.softmax(w.masked_fill(hidden, -math.inf), -1) @ v[:, h // group]
    return out


def exact_rotary(case, x, at):
    f, amplitude = frequencies(case)
    z = torch.exp(2j * math.pi * (at.double()[:, None] * torch.tensor(f, dtype=torch.float64, device=x.device))) * amplitude
    dims, out = case["dims"], x.clone()
    if case["pairs"] == "halves":
        w = torch.complex(x[..., :dims // 2].contiguous(), x[..., dims // 2:dims].contiguous()) * z[:, None]
        out[..., :dims] = torch.cat((w.real, w.imag), -1)
    else:
        w = torch.view_as_complex(x[..., :dims].unflatten(-1, (-1, 2)).contiguous()) * z[:, None]
        out[..., :dims] = torch.view_as_real(w).flatten(-2)
    return out


def exact_prompt(q, k, v, borders, group):
    out = torch.zeros(q.shape, dtype=torch.float64, device=q.device)
    for a, b in zip(borders, borders[1:]):
        for h in range(q.shape[1]):
            y, z = k[a:b, h // group].double(), v[a:b, h // group].double()
            for i in range(a, b, 8192):                          # rows at a time
                j = min(b, i + 8192)
                s = q[i:j, h].double() @ y[:j - a].T / 8.0
                s = s.masked_fill(torch.arange(a, j, device=q.device)[None] > torch.arange(i, j, device=q.device)[:, None], -math.inf)
                out[i:j, h] = torch.softmax(s, -1) @ z[:j - a]
    return out


def nearest(x):
    """The 8-bit form's values nearest to x [positions, heads, HEAD], whose pages begin at its first position."""
    L = len(x)
    x = torch.nn.functional.pad(x, (0, 0, 0, 0, 0, -L % PAGE)).unflatten(0, (-1, PAGE))
    grid = torch.tensor([m * 2.0 ** -9 for m in range(8)] + [(8 + m) * 2.0 ** (e - 3) for e in range(-6, 9) for m in range(8)][:-1],
                        dtype=torch.float64, device=x.device)
    peak = x.abs().amax((1, 3), keepdim=True)
    scale = torch.exp2(torch.ceil(torch.log2(torch.clamp(peak / 448, min=2.0 ** LOWEST))))
    scale = torch.where((peak <= 224 * scale) & (scale > 2.0 ** LOWEST), scale / 2, scale)   # where the logarithm's rounding went past
    scale = torch.where(peak > 448 * scale, scale * 2, scale)
    y = x.abs() / scale
    low = (torch.searchsorted(grid, y.contiguous(), right=True) - 1).clamp(0, len(grid) - 2)
    below, above = y - grid[low], grid[low + 1] - y
    code = torch.where((above < below) | ((above == below) & (low % 2 == 1)), low + 1, low)
    return (torch.copysign(grid[code], x) * scale).flatten(0, 1)[:L]
