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
