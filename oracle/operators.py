"""Plain 64-bit forms of the operators without a handle: beam selection, page tables
after a choice of beams, acoustic keys and values in 4 bits and attention over them."""
import numpy as np

GRID = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6])


def beam_select(logits, scores, k, suppress=None):
    """logits [n, beams, vocab], scores [n, beams] -> (score f64, beam, token), each [n, k]: the k best of
    score + log softmax, equal ones by lower beam, then lower token; -inf, -1, -1 where there are fewer."""
    n, B, V = logits.shape
    x = np.asarray(logits, np.float64).copy()
    if suppress is not None:
        x[:, :, np.asarray(suppress) != 0] = -np.inf
    out = np.full((n, k), -np.inf), np.full((n, k), -1), np.full((n, k), -1)
    for r in range(n):
        every = np.full((B, V), -np.inf)
        for b in range(B):
            s, row = float(scores[r][b]), x[r, b]
            if not np.isfinite(s) or np.isnan(row).any() or np.isposinf(row).any() or np.isneginf(row).all():
                continue
            m = row.max()
            every[b] = s + ((row - m) - np.log(np.exp(row - m).sum()))
        order = np.argsort(-every, axis=None, kind="stable")[:k]
        for j, i in enumerate(order):
            if every.flat[i] > -np.inf:
                out[0][r, j], out[1][r, j], out[2][r, j] = every.flat[i], i // V, i % V
    return out


def cache_reorder(tables, parents, lens, pool, page_tokens):
    """(new tables, copies): copies holds per request the (source, destination) pages."""
    n, B, P = tables.shape
    new, copies = np.empty_like(tables), []
    for r in range(n):
        L = min(max(int(lens[r]), 0), P * page_tokens)
        last, part = divmod(L, page_tokens)
        kept = last + (part > 0)
        live = [0 <= p < B for p in parents[r]]
        for j, p in enumerate(parents[r]):
            new[r, j] = pool[r][0]
            if live[j]:
                new[r, j, :kept] = tables[r, p, :kept]
        used = {int(page) for j in range(B) if live[j] for page in new[r, j, :kept]}
        fresh = iter([int(page) for page in pool[r] if page not in used])
        todo, owned = [], set()
        for j in range(B):
            if not live[j] or last >= P:
                continue
            mine = int(new[r, j, last])
            if part and mine not in owned:
                owned.add(mine)
                continue
            new[r, j, last] = next(fresh)
            if part:
                todo.append((mine, int(new[r, j, last])))
        copies.append(todo)
    return new, copies


def quantise(x, axis):
    """The values that blocks along `axis` (whole blocks of 32) stand for: nearest of the grid times the smallest
    2^e, e >= -120, with max |x| <= 6 * 2^e; ties to the even code; NaN where a block holds a non-finite value."""
    x = np.moveaxis(np.asarray(x, np.float64), axis, -1)
    shape = x.shape
    x = x.reshape(shape[:-1] + (-1, 32))
    peak = np.abs(x).max(-1, keepdims=True)
    bad = ~np.isfinite(peak)
    e = np.full(peak.shape, -120)
    for step in range(-119, 128):
        e = np.where(np.where(bad, 0, peak) > 6 * np.ldexp(1.0, step - 1), step, e)
    y = np.abs(np.where(bad, 0, x)) / np.ldexp(1.0, e)
    d = np.abs(y[..., None] - GRID)
    best = d.min(-1, keepdims=True)
    first = (d == best).argmax(-1)
    second = 7 - (d == best)[..., ::-1].argmax(-1)
    code = np.where(first % 2 == 0, first, second)
    out = np.copysign(GRID[code], x) * np.ldexp(1.0, e)
    out = np.where(np.abs(out) >= 2.0 ** 128, np.copysign(np.inf, x), out)   # 4 * 2^126 in 32 bits
    out = np.where(bad, np.nan, out)
    return np.moveaxis(out.reshape(shape), -1, axis)


def kv4_values(k, v, lens):
    """What [n, F, H, 64] keys and values stand for in 4 bits, of which lens[r] frames are given."""
    n, F = k.shape[:2]
    inside = (np.arange(F)[None] < np.asarray(lens)[:, None])[:, :, None, None]
    k, v = np.where(inside, k, 0.0), np.where(inside, v, 0.0)
    pad = np.zeros((n, -F % 32) + v.shape[2:])
    return quantise(k, 3), quantise(np.concatenate([v, pad], 1), 1)[:, :F]


def attend(q, k, v, lens):
    """softmax(q k^T / 8) v over the first lens[r] frames; zeros for a request of none.  [n, rows, H, 64]."""
    out = np.zeros(q.shape)
    for r in range(q.shape[0]):
        m = int(lens[r])
        if m == 0:
            continue
        for h in range(q.shape[2]):
            s = np.asarray(q[r, :, h], np.float64) @ k[r, :m, h].T / 8
            p = np.exp(s - s.max(-1, keepdims=True))
            out[r, :, h] = p @ v[r, :m, h] / p.sum(-1, keepdims=True)
    return out


# ---------------------------------------------------------------- a decoder's self-attention

def rotary_turns(dims, base=10000.0, scaling=None, factor=1.0, context=0.0, low=1.0, high=32.0):
    """(turns a position of every pair, amplitude)."""
    i = np.arange(dims // 2)
    if scaling == "base":
        base = base * factor ** (dims / (dims - 2))
    f = base ** (-2.0 * i / dims) / (2 * np.pi)
    if scaling == "linear":
        f = f / factor
    if scaling == "ramp":
        w = np.clip((f * context - low) / (high - low), 0, 1)
        return f * (w + (1 - w) / factor), 0.1 * np.log(factor) + 1
    return f, 1.0


def rotary(x, positions, turns, amplitude, interleaved, transposed=False):
    """x [tokens, heads, width]: the pairs of the first 2 len(turns) elements turned by positions' angles."""
    y, d = np.array(x, np.float64), 2 * len(turns)
    part = np.asarray(positions, np.float64)[:, None] * turns
    angle = 2 * np.pi * (part - np.rint(part)) * (-1 if transposed else 1)
    z = (amplitude * np.exp(1j * angle))[:, None]
    a, b = (slice(0, d, 2), slice(1, d, 2)) if interleaved else (slice(0, d // 2), slice(d // 2, d))
    w = (y[..., a] + 1j * y[..., b]) * z
    y[..., a], y[..., b] = w.real, w.imag
    return y


def seen_attention(q, k, v, sees):
    """softmax(q k^T / 8) v of rows q [rows, heads, 64] over k, v [keys, kv heads, 64], row i over its keys sees[i] (bool
    [rows, keys]); rows that see none: zeros.  Also sum p |v| and the largest |q| |k| / 8 of a seen key (for bounds)."""
    rows, H, _ = q.shape
    G = H // k.shape[1]
    out, spread, size = np.zeros(q.shape), np.zeros(q.shape), np.zeros((rows, H))
    q, k, v = (np.asarray(x, np.float64) for x in (q, k, v))
    for h in range(H):
        for i in range(rows):
            at = np.flatnonzero(sees[i])
            if not len(at):
                continue
            kk, vv = k[at, h // G], v[at, h // G]
            s = kk @ q[i, h] / 8
            with np.errstate(invalid="ignore", over="ignore"):
                p = np.exp(s - s.max())
                p = p / p.sum()
                out[i, h], spread[i, h] = p @ vv, p @ np.abs(vv)
            size[i, h] = (np.abs(kk) @ np.abs(q[i, h]) / 8).max()
    return out, spread, size


def prompt_attention(q, k, v, starts):
    rows = np.arange(len(q))
    first = np.full(len(q), -1)
    for a, b in zip(starts, starts[1:]):
        first[max(a, 0):max(b, 0)] = max(a, 0)
    sees = (first[:, None] >= 0) & (rows[None] >= first[:, None]) & (rows[None] <= rows[:, None])
    return seen_attention(q, k, v, sees)


E4M3 = np.array([m * 2.0 ** -9 for m in range(8)] + [(8 + m) * 2.0 ** (e - 3) for e in range(-6, 9) for m in range(8)][:-1])


def quantise8(x):
    """A page's keys or values of one head [16, 64] -> the values that its codes stand for; what is not finite: NaN."""
    fine = np.isfinite(x)
    top = np.abs(np.where(fine, x, 0)).max()
    e = -100
    while top > 448 * 2.0 ** e:
        e += 1
    y = np.abs(np.where(fine, x, 0)) / 2.0 ** e
    low = np.clip(np.searchsorted(E4M3, y, side="right") - 1, 0, len(E4M3) - 2)
    below, above = y - E4M3[low], E4M3[low + 1] - y
    code = np.where((above < below) | ((above == below) & (low % 2 == 1)), low + 1, low)
    return np.where(fine, np.copysign(E4M3[code], x) * 2.0 ** e, np.nan)


class PagedCache8:
    """The values that a paged 8-bit cache stands for: k, v [pages, heads, 16, 64]."""

    def __init__(self, pages, heads):
        self.pages, self.heads = pages, heads
        self.k, self.v = np.zeros((pages, heads, 16, 64)), np.zeros((pages, heads, 16, 64))

    def store(self, k, v, tables, positions):
        """k, v: a list of [rows, heads, 64] for every request."""
        for r, at in enumerate(positions):
            count = len(k[r])
            for c in range(len(tables[r])):
                page = int(tables[r][c])
                a, b = max(16 * c, at, 0), min(16 * c + 16, at + count)
                if a >= b or not 0 <= page < self.pages:
                    continue
                for held, new in ((self.k, k[r]), (self.v, v[r])):
                    x = np.zeros((self.heads, 16, 64))
                    keep = min(max(at - 16 * c, 0), 16)
                    x[:, :keep] = held[page][:, :keep]
                    x[:, a - 16 * c:b - 16 * c] = np.moveaxis(new[a - at:b - at], 0, 1)
                    for h in range(self.heads):
                        held[page][h] = quantise8(x[h])

    def rows(self, table, length):
        """(k, v [length, heads, 64], which of them lie in a page)."""
        k, v, there = np.zeros((length, self.heads, 64)), np.zeros((length, self.heads, 64)), np.zeros(length, bool)
        for c in range(min(len(table), -(-length // 16))):
            page, m = int(table[c]), min(16, length - 16 * c)
            if 0 <= page < self.pages:
                k[16 * c:16 * c + m] = np.moveaxis(self.k[page][:, :m], 0, 1)
                v[16 * c:16 * c + m] = np.moveaxis(self.v[page][:, :m], 0, 1)
                there[16 * c:16 * c + m] = True
        return k, v, there

    def attend(self, q, table, at, count):
        """One request's rows q [rows, heads, 64]."""
        rows, most = len(q), 16 * len(table)
        length = min(max(at + count, 0), most)
        k, v, there = self.rows(table, length)
        sees = (np.arange(length)[None] <= at + np.arange(rows)[:, None]) & there[None] & (np.arange(rows)[:, None] < count)
        return seen_attention(q, k, v, sees)
