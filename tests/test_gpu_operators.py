"""The operators without a handle on the GPU against their plain 64-bit forms (oracle/operators.py)."""
import numpy as np
import pytest
import torch

from oracle import operators as plain

pytestmark = pytest.mark.gpu
INF = float("inf")


def lib():
    import paper_2609_32869_amd as wf
    return wf


# ---------------------------------------------------------------- beam selection

def check_select(logits, scores, k, suppress=None, stream=None):
    """Beams and tokens equal; scores: the row's sum of exponentials is off by at most 2^-20 relative (32-bit
    exponentials, 2^-22 each, and partial sums of a few values), then one rounding of the score to 32 bits."""
    got = [t.cpu().numpy() for t in lib().beam_select(logits, scores, k, suppress=suppress, stream=stream)]
    want = plain.beam_select(logits.float().cpu().numpy(), scores.cpu().numpy(), k,
                             None if suppress is None else suppress.cpu().numpy())
    assert np.array_equal(got[1], want[1])
    assert np.array_equal(got[2], want[2])
    fine = np.isfinite(want[0])
    assert np.array_equal(fine, np.isfinite(got[0])) and (got[0][~fine] == -np.inf).all()
    err = np.abs(got[0][fine] - want[0][fine])
    assert (err <= 2.0 ** -20 + 2.0 ** -24 * np.abs(want[0][fine])).all(), err.max()


@pytest.mark.parametrize("n,B,V,k,dtype", [
    (1, 1, 1, 1, torch.float32), (1, 1, 1, 4, torch.bfloat16), (2, 3, 5, 32, torch.float32), (1, 5, 64, 10, torch.float32),
    (3, 16, 65, 32, torch.bfloat16), (1, 5, 51866, 10, torch.float32), (2, 8, 51865, 16, torch.bfloat16),
    (7, 2, 1023, 7, torch.float32), (5, 4, 4097, 8, torch.bfloat16), (300, 5, 777, 10, torch.float32),
    (1, 16, 51866, 32, torch.float32), (1, 2, 300001, 5, torch.float32), (130, 4, 9001, 32, torch.bfloat16),
    (62, 8, 367, 3, torch.float32), (20, 16, 4624, 32, torch.float32), (4, 3, 40, 4, torch.bfloat16), (6, 9, 8200, 16, torch.float32),
    (1, 16, 300001, 32, torch.float32)])
def test_select(n, B, V, k, dtype):
    g = torch.Generator("cuda").manual_seed(n * 1000 + V)
    logits = (3 * torch.randn((n, B, V), device="cuda", generator=g)).to(dtype)
    scores = -10 * torch.rand((n, B), device="cuda", generator=g)
    check_select(logits, scores, k)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("offset", [0, 1, 3])
def test_select_rows_of_a_larger_buffer(dtype, offset):
    """Every ninth row, starting off a 16-byte border, beams before requests in memory."""
    g = torch.Generator("cuda").manual_seed(offset)
    buf = torch.randn(offset + 3 * 4 * 9 * 1031, device="cuda", generator=g).to(dtype)
    logits = buf[offset:].view(4, 3, 9, 1031)[:, :, 0].transpose(0, 1)[:, :, :1030]
    check_select(logits, torch.zeros((3, 4), device="cuda"), 9)


@pytest.mark.parametrize("V", [63, 5000])
@pytest.mark.parametrize("shape", ["equal", "ascending", "descending", "few"])
def test_select_ties_and_orders(V, shape):
    """Equal values go to the lower beam, then the lower token, wherever they lie."""
    x = {"equal": torch.zeros(V), "ascending": torch.arange(V) / 64.0, "descending": -torch.arange(V) / 64.0,
         "few": (torch.arange(V) % 7 == 3).float()}[shape]
    logits = x.cuda().expand(2, 5, V).contiguous()
    check_select(logits, torch.zeros((2, 5), device="cuda"), 32)
    check_select(logits.bfloat16(), torch.tensor([[-1.0, -2, -1, -2, -1]] * 2, device="cuda"), 17)


@pytest.mark.parametrize("levels", [1, 3])
def test_select_more_equal_candidates_than_a_block_lists(levels):
    """16 beams of equal rows, 32 best of each of 7 pieces: 3,584 candidates of one score, or of three."""
    logits = (torch.arange(51866, device="cuda") % levels).float().expand(2, 16, 51866)
    check_select(logits, torch.zeros((2, 16), device="cuda"), 32)
    check_select(logits, torch.tensor([[0.0, -INF] * 8, [-1.0] * 16], device="cuda"), 31)


def test_select_empty_beams_and_suppressed_tokens():
    g = torch.Generator("cuda").manual_seed(3)
    logits = torch.randn((4, 5, 1000), device="cuda", generator=g)
    scores = torch.tensor([[0, -INF, -INF, -INF, -INF], [-INF] * 5, [-1, -2, -3, -4, -5], [0, -1, -INF, -3, -4.0]], device="cuda")
    some = (torch.rand(1000, device="cuda", generator=g) < 0.5).to(torch.uint8)
    check_select(logits, scores, 10, some)
    check_select(logits, scores, 10, torch.ones(1000, dtype=torch.uint8, device="cuda"))
    one = torch.ones(1000, dtype=torch.uint8, device="cuda")
    one[777] = 0
    check_select(logits, scores, 10, one)
    logits[2, :, 3:] = -INF          # fewer candidates than k
    logits[3, 1] = -INF              # a row of nothing
    check_select(logits, scores, 32)
    logits[2] = torch.finfo(torch.float32).min   # masked with the type's lowest value: an ordinary value
    check_select(logits, scores, 32)


def test_select_non_finite_rows_offer_nothing():
    g = torch.Generator("cuda").manual_seed(4)
    logits = torch.randn((3, 4, 3000), device="cuda", generator=g)
    logits[0, 0, 2999] = float("nan")
    logits[0, 1, 5] = INF
    logits[1, 2, :] = float("nan")
    scores = torch.tensor([[0.0, 0, -1, -2], [0, 0, 0, 0], [float("nan"), INF, -1, 0]], device="cuda")
    check_select(logits, scores, 12)
    mask = torch.zeros(3000, dtype=torch.uint8, device="cuda")
    mask[2999] = mask[5] = 1         # suppressed places may hold anything
    check_select(logits, scores, 12, mask)


def test_select_peaked_and_far_logits():
    """One token with nearly all the mass, and logits of 1e4: the sum is what the top leaves over."""
    logits = torch.full((2, 2, 51866), -30.0, device="cuda")
    logits[:, :, 100] = 12.0
    logits[:, 1, 40000] = 11.5
    logits[1] += 1e4
    g = torch.Generator("cuda").manual_seed(5)
    logits += torch.rand(logits.shape, device="cuda", generator=g)
    check_select(logits, torch.tensor([[-3.0, -3.25], [-100, -99]], device="cuda"), 4)


HUGE = [1e6, 4.19e6, 4.2e6, 1e9, 3e9, 5e9, 1e10, 1e11, 1e12, 1e20, 9e29, 1e30, 3e38]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("size", HUGE)
def test_select_runs_of_huge_logits(size, dtype):
    """Columns masked with a large negative value beside ordinary ones: a wave's lanes that hold nothing else, a whole wave
    (2,048 columns), the last, partial one; a single lane (8 columns); and suppressed places with the value of either sign."""
    g = torch.Generator("cuda").manual_seed(9)
    V = 51866
    logits = (3 * torch.randn((3, 2, V), device="cuda", generator=g)).to(dtype)
    logits[0, 0, 50365:] = -size
    logits[0, 1, 4096:6144] = -size
    logits[1, 0, 16:24] = -size
    logits[1, 1, 100:] = -size
    sup = torch.zeros(V, dtype=torch.uint8, device="cuda")
    scores = torch.tensor([[-1.0, -2], [-1.5, -1], [0, -3]], device="cuda")
    check_select(logits, scores, 10)
    sup[30000:40000] = 1
    logits[2, 0, 30000:35000], logits[2, 1, 30000:40000] = size, -size
    check_select(logits, scores, 10, sup)


@pytest.mark.parametrize("sign", [1, -1])
@pytest.mark.parametrize("size", HUGE)
def test_select_rows_of_huge_logits(size, sign):
    """Whole rows about one large value: equal ones, and ones a few of its steps apart."""
    g = torch.Generator("cuda").manual_seed(10)
    logits = torch.full((2, 3, 9000), sign * size, device="cuda")
    logits[:, 1, 1234] += size * 2.0 ** -20     # by itself a logit of over 30 above the rest, or next to them
    logits[:, 2] *= 1 - 2.0 ** -24 * torch.randint(0, 3, (2, 9000), device="cuda", generator=g)
    check_select(logits, torch.tensor([[0.0, -1, -2], [-7, -INF, -7]], device="cuda"), 6)
    check_select(logits.bfloat16(), torch.zeros((2, 3), device="cuda"), 6)


# ---------------------------------------------------------------- page tables

def search_tables(rng, n, B, P, page_tokens, lens):
    """Tables as a search leaves them: a shared first part, then each beam's own pages; pages in mixed order."""
    order = rng.permutation(n * B * P).astype(np.int32)
    pool = order.reshape(n, B * P)
    tables = np.repeat(pool[:, :1], B * P, 1).reshape(n, B, P).copy()
    for r in range(n):
        used = -(-int(lens[r]) // page_tokens)
        shared = int(rng.integers(0, used + 1)) if lens[r] % page_tokens == 0 else int(rng.integers(0, max(used, 1)))
        tables[r, :, :shared] = pool[r, :shared]
        own = pool[r, shared:shared + B * (used - shared)].reshape(B, used - shared)
        tables[r, :, shared:used] = own
    return tables, pool


def check_reorder(cache, tables, parents, lens, pool, page_tokens, stream=None):
    up = lambda a: torch.from_numpy(np.ascontiguousarray(a, np.int32)).cuda()  # noqa: E731
    before = cache.clone()
    got = lib().cache_reorder(cache, up(tables), up(parents), up(lens), up(pool), page_tokens, stream=stream)
    new, copies = plain.cache_reorder(tables, parents, lens, pool, page_tokens)
    assert np.array_equal(got.cpu().numpy(), new)
    for request in copies:
        for s, d in request:
            before[:, d] = before[:, s]
    assert torch.equal(cache, before)    # the copies, and nothing else
    return new


@pytest.mark.parametrize("n,B,P,page_tokens,regions,dtype", [
    (1, 1, 1, 16, 1, torch.bfloat16), (1, 5, 28, 16, 6, torch.bfloat16), (3, 2, 4, 16, 2, torch.float32),
    (9, 16, 28, 16, 3, torch.bfloat16), (4, 3, 7, 1, 2, torch.float32), (2, 8, 300, 5, 4, torch.bfloat16)])
def test_reorder(n, B, P, page_tokens, regions, dtype):
    rng = np.random.default_rng(n * 100 + B)
    cache = torch.randn((regions, n * B * P, 24), device="cuda").to(dtype)
    for lens in (rng.integers(0, P * page_tokens + 1, n), np.zeros(n, int), np.full(n, P * page_tokens),
                 np.full(n, page_tokens * (P // 2))):
        tables, pool = search_tables(rng, n, B, P, page_tokens, lens)
        check_reorder(cache, tables, rng.integers(0, B, (n, B)), lens, pool, page_tokens)
        check_reorder(cache, tables, np.tile(np.arange(B), (n, 1)), lens, pool, page_tokens)
        check_reorder(cache, tables, np.zeros((n, B), int), lens, pool, page_tokens)


def test_reorder_fork_and_dropped_beams():
    """A first choice: every beam holds the same pages, the part-filled one among them; beams without a parent."""
    rng = np.random.default_rng(7)
    P, B = 6, 4
    cache = torch.randn((3, 2 * B * P, 40), device="cuda")
    pool = rng.permutation(2 * B * P).astype(np.int32).reshape(2, B * P)
    tables = np.repeat(pool[:, None, :P], B, 1)
    check_reorder(cache, tables, np.array([[0, 0, 0, 0], [1, -1, 2, 4]]), np.array([37, 48]), pool, 16)
    check_reorder(cache, tables, np.array([[-1, -1, -1, -1], [3, 2, 1, 0]]), np.array([1, 95]), pool, 16)


def test_reorder_search_of_many_steps():
    """Sixty choices in a row: what a beam reads through its table is always what its own path wrote."""
    rng = np.random.default_rng(8)
    n, B, P, T = 2, 5, 8, 8
    cache = torch.zeros((2, n * B * P, T * 4), device="cuda")
    pool = np.arange(n * B * P, dtype=np.int32).reshape(n, B * P)
    tables = np.repeat(pool[:, None, :P], B, 1)
    parents = np.zeros((n, B), int)
    lens = np.zeros(n, int)
    paths = [[[] for _ in range(B)] for _ in range(n)]
    for step in range(60):
        tables = check_reorder(cache, tables, parents, lens, pool, T)
        paths = [[list(paths[r][p]) for p in parents[r]] for r in range(n)]
        for r in range(n):
            for b in range(B):
                mark = float(1 + step * 100 + r * 10 + b)
                c, o = divmod(int(lens[r]), T)
                cache[:, tables[r, b, c], 4 * o:4 * o + 4] = mark
                paths[r][b].append(mark)
        lens += 1
        host = cache.cpu().numpy()
        for r in range(n):
            for b in range(B):
                read = [host[1, tables[r, b, p // T], 4 * (p % T)] for p in range(int(lens[r]))]
                assert read == paths[r][b]
        parents = (B * rng.random((n, B)) ** 2).astype(int)


def test_reorder_bad_pages_stay_inside_the_cache():
    """Page numbers and lengths that no search leaves are carried over or clamped; nothing outside is touched."""
    P, B = 4, 3
    cache = torch.randn((2, 12, 8), device="cuda")
    pool = np.array([[99, -5, 3, 3, 4, 5, 6, 7, 8, 9, 10, 11]], np.int32)
    tables = np.array([[[1000000, 2, -7, 0], [0, 1, 2, 77], [2, 2, 2, 2]]], np.int32)
    up = lambda a: torch.from_numpy(np.ascontiguousarray(a, np.int32)).cuda()  # noqa: E731
    for length in (-3, 0, 5, 63, 64, 10 ** 6, 2 ** 31 - 1):
        before = cache.clone()
        new = lib().cache_reorder(cache, up(tables), up([[0, 0, 1]]), up([length]), up(pool), 16).cpu().numpy()
        kept = -(-min(max(length, 0), 64) // 16)
        full = min(max(length, 0), 64) // 16
        assert (new[0, 0, :full] == tables[0, 0, :full]).all() and (new[0, 2, :full] == tables[0, 1, :full]).all()
        assert (new[0, :, max(kept, full + 1):] == 99).all()
        changed = (cache != before).any(-1).any(0).cpu().numpy().nonzero()[0]
        assert set(changed) <= {3, 4, 5, 6, 7, 8, 9, 10, 11}


# ---------------------------------------------------------------- 4-bit keys and values

def source(n, F, H, dtype, seed):
    g = torch.Generator("cuda").manual_seed(seed)
    width = torch.exp(torch.randn((H, 64), device="cuda", generator=g))
    k = (torch.randn((n, F, H, 64), device="cuda", generator=g) * width).to(dtype)
    v = (torch.randn((n, F, H, 64), device="cuda", generator=g) * width.flip(-1)).to(dtype)
    v[:, :, 0, :5] = 0
    return k, v


def num(t):
    return t.double().cpu().numpy()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("n,F,H", [(1, 1, 1), (2, 31, 3), (1, 32, 2), (3, 33, 2), (2, 100, 6), (1, 1500, 20), (4, 257, 1)])
def test_store_and_load(n, F, H, dtype):
    wf = lib()
    k, v = source(n, F, H, dtype, F)
    cache = wf.AcousticCache4(n + 2, H, F)
    cache.data.fill_(0x5a)
    keep = cache.data.clone().view(n + 2, -1)
    cache.store(1, k, v)
    data = cache.data.view(n + 2, -1)
    assert torch.equal(data[0], keep[0]) and torch.equal(data[-1], keep[-1])   # the neighbours' entries
    want = plain.kv4_values(num(k), num(v), [F] * n)
    for out in (torch.float32, torch.bfloat16):
        for g, w in zip(cache.load(1, n, out), want):
            assert g.dtype == out and np.array_equal(num(g), w)


def test_store_lengths():
    wf = lib()
    n, F, H = 5, 70, 2
    k, v = source(n, F, H, torch.float32, 1)
    lens = torch.tensor([0, 1, 33, 70, 64], dtype=torch.int32, device="cuda")
    for r, m in enumerate(lens.tolist()):
        k[r, m:] = float("nan")     # frames past a length are not read
        v[r, m:] = INF
    cache = wf.AcousticCache4(n, H, F)
    cache.store(0, k, v, lens)
    want = plain.kv4_values(num(k), num(v), lens.tolist())
    for g, w in zip(cache.load(0, n), want):
        assert np.array_equal(num(g), w)
    cache.store(0, k, v, torch.tensor([-4, -1, 33, 2 ** 31 - 1, 64], dtype=torch.int32, device="cuda"))
    want = plain.kv4_values(num(k), num(v), [0, 0, 33, 70, 64])
    for g, w in zip(cache.load(0, n), want):
        assert np.array_equal(num(g), w)


def test_store_borders_and_extremes():
    """Every border between two codes, both signs, and peaks at a scale's border; tiny, huge, zero and non-finite blocks."""
    wf = lib()
    y = np.array([0, 0.25, 0.5, 0.75, 1, 1.25, 1.5, 1.75, 2, 2.5, 3, 3.5, 4, 5, 6])
    y = np.concatenate([y, np.nextafter(y, 9, dtype=np.float32), np.nextafter(y, -1, dtype=np.float32)]).astype(np.float32)
    F = 64
    k = np.zeros((1, F, 1, 64), np.float32)
    for f in range(F):
        s = np.float32(2.0) ** (f - 30)
        part = y[f % 3 * 15:f % 3 * 15 + 15]
        k[0, f, 0, :30] = np.concatenate([part, -part]) * s
        k[0, f, 0, 30:32] = np.float32(6) * s
        k[0, f, 0, 32:62] = np.concatenate([-part, part]) * s
        k[0, f, 0, 62] = np.nextafter(np.float32(6) * s, np.float32(9e9))   # the next scale
    k[0, 0] = 0
    k[0, 1, 0, :32] = 3.4e38
    k[0, 2, 0, 32:] = 1e-38
    k[0, 3, 0, 5] = np.nan
    k[0, 4, 0, 40] = -np.inf
    k[0, 5, 0, :32] = 6 * 2.0 ** -120 * np.linspace(0, 1, 32)
    v = np.swapaxes(k, 1, 3).copy()
    kt, vt = torch.from_numpy(k).cuda(), torch.from_numpy(v).cuda()
    cache = wf.AcousticCache4(1, 1, F)
    cache.store(0, kt, vt)
    want = plain.kv4_values(k, v, [F])
    for g, w in zip(cache.load(0, 1), want):
        assert np.array_equal(num(g), w, equal_nan=True)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_store_strides(dtype):
    """Heads before frames, rows off a 16-byte border, keys and values interleaved, one source for all entries."""
    wf = lib()
    n, F, H = 2, 45, 3
    k, v = source(n, F, H, dtype, 2)
    want = plain.kv4_values(num(k), num(v), [F] * n)
    both = torch.empty((n, H, F, 2, 64), dtype=dtype, device="cuda")
    both[:, :, :, 0], both[:, :, :, 1] = k.transpose(1, 2), v.transpose(1, 2)
    odd = [torch.empty(1 + n * F * H * 67, dtype=dtype, device="cuda")[1:].view(n, F, H, 67)[..., 1:65] for _ in range(2)]
    odd[0].copy_(k)
    odd[1].copy_(v)
    cache = wf.AcousticCache4(n, H, F)
    for ks, vs in ((both[:, :, :, 0].transpose(1, 2), both[:, :, :, 1].transpose(1, 2)), odd):
        cache.data.fill_(0)
        cache.store(0, ks, vs)
        for g, w in zip(cache.load(0, n), want):
            assert np.array_equal(num(g), w)
    cache.store(0, k[:1].expand(n, F, H, 64), v[:1].expand(n, F, H, 64))
    for g, w in zip(cache.load(0, n), want):
        assert np.array_equal(num(g), np.repeat(w[:1], n, 0))


# ---------------------------------------------------------------- attention over them

def check_attend(cache, slot0, q, k, v, lens, lens_arg, stream=None):
    """Against 64 bits on the values that the cache holds.  A score is the sum of up to 192 products, each sum rounded
    to 32 bits: off by at most 192 * 2^-24 < 2^-16 of sum |q k| / 8; a probability by twice that, relative (its own
    score and the sum's), plus 2^-15 for its terms (2^-16 in bf16), its exponential and the sums; the output by as
    much of max |v|, then the output type's rounding.  Roundings of 32 bits go both ways and partial sums of 64 products
    of either sign are about a sixth of `mass`, the sum of |q k| / 8, so in the 2-norm an fp32 result is off by far less:
    a score by sqrt(192 / 3) * 2^-24 * mass / 6 < 2^-23.5 * mass, a probability by as much relative, which is 2^-18 at a
    mass of 45 and grows with it (two bf16 terms in place of three would take 2^-17 at any mass)."""
    got = cache.attend(slot0, q, lens_arg, stream=stream)
    assert got.dtype == q.dtype and got.shape == q.shape and got.is_contiguous()
    qn, got = num(q), num(got)
    want = plain.attend(qn, k, v, lens)
    half = 2.0 ** -9 if q.dtype == torch.bfloat16 else 2.0 ** -24
    most = 45
    for r, m in enumerate(lens):
        if m == 0:
            assert (got[r] == 0).all()
            continue
        for h in range(q.shape[2]):
            mass = (np.abs(qn[r, :, h]) @ np.abs(k[r, :m, h]).T).max(-1, keepdims=True) / 8
            tol = (2 * (2.0 ** -16 + 2.0 ** -18) * mass + 2.0 ** -15) * np.abs(v[r, :m, h]).max() + 2 * half * np.abs(want[r, :, h])
            err = np.abs(got[r, :, h] - want[r, :, h])
            assert (err <= tol).all(), (r, h, err.max(), tol.min())
            most = max(most, mass.max())
    if q.dtype == torch.float32 and max(lens) > 0:
        assert np.linalg.norm(got - want) <= 2.0 ** -18 * most / 45 * np.linalg.norm(want)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("n,rows,F,H", [
    (1, 1, 1, 1), (1, 1, 1500, 20), (1, 9, 1500, 20), (2, 16, 33, 2), (3, 17, 100, 2), (1, 40, 64, 3), (5, 5, 257, 6),
    (40, 9, 200, 20), (2, 3, 5000, 2), (100, 1, 40, 2), (1, 40, 5000, 2)])
def test_attend(n, rows, F, H, dtype):
    wf = lib()
    k, v = source(n, F, H, dtype, rows)
    cache = wf.AcousticCache4(n + 1, H, F)
    cache.store(1, k, v)
    held = plain.kv4_values(num(k), num(v), [F] * n)
    g = torch.Generator("cuda").manual_seed(rows)
    q = torch.randn((n, rows, H, 64), device="cuda", generator=g).to(dtype)
    check_attend(cache, 1, q, *held, [F] * n, None)
    lens = torch.randint(0, F + 1, (n,), device="cuda", generator=g, dtype=torch.int32)
    lens[0] = min(F, 33)
    check_attend(cache, 1, q, *held, lens.tolist(), lens)


def test_attend_lengths():
    """Each length around a group's and a wave's borders, none among them, and lengths outside the cache."""
    wf = lib()
    some = [0, 1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 191, 192, 255, 256, 257, 500, 511, 512, 513, 699, 700]
    n, F, H = len(some), 700, 2
    k, v = source(n, F, H, torch.float32, 9)
    cache = wf.AcousticCache4(n, H, F)
    cache.store(0, k, v)
    held = plain.kv4_values(num(k), num(v), [F] * n)
    q = torch.randn((n, 3, H, 64), device="cuda")
    check_attend(cache, 0, q, *held, some, torch.tensor(some, dtype=torch.int32, device="cuda"))
    wild = torch.tensor([-1, 701, -2 ** 31, 2 ** 31 - 1] + some[4:], dtype=torch.int32, device="cuda")
    check_attend(cache, 0, q, *held, [0, F, 0, F] + some[4:], wild)


def test_attend_masked_places_may_hold_anything():
    """Frames past a length that were stored as NaN blocks, and entries never stored."""
    wf = lib()
    n, F, H = 2, 400, 2
    k, v = source(n, F, H, torch.float32, 10)
    k[:, 224:] = float("nan")
    v[:, 224:] = INF
    cache = wf.AcousticCache4(n + 1, H, F)
    cache.data.fill_(0xff)
    cache.store(0, k, v)
    held = plain.kv4_values(num(k), num(v), [224] * n)
    q = torch.randn((n, 9, H, 64), device="cuda")
    lens = torch.tensor([224, 200], dtype=torch.int32, device="cuda")
    check_attend(cache, 0, q, *held, [224, 200], lens)
    assert (cache.attend(2, q[:1], torch.zeros(1, dtype=torch.int32, device="cuda")) == 0).all()
    lens[1] = 225
    got = cache.attend(0, q, lens)
    assert got[0].isfinite().all() and got[1].isnan().all()     # a non-finite frame inside shows


def test_attend_infinite_values_in_masked_places():
    """Values that stand for infinity behind the length, in a group with frames inside it: they count for nothing, also
    where a wave's last step holds that group twice."""
    wf = lib()
    n, F, H = 4, 600, 2
    for dtype in (torch.float32, torch.bfloat16):
        k, v = source(n, F, H, dtype, 20)
        v[:, 200:224] = 3.3e38
        v[:, 520:] = -3.3e38
        cache = wf.AcousticCache4(n, H, F)
        cache.store(0, k, v)
        held = plain.kv4_values(num(k), num(v), [F] * n)
        assert np.isinf(held[1][:, 200:224]).all()
        lens = [200, 193, 197, 1]
        q = torch.randn((n, 5, H, 64), device="cuda").to(dtype)
        check_attend(cache, 0, q, *held, lens, torch.tensor(lens, dtype=torch.int32, device="cuda"))


@pytest.mark.parametrize("size", [1e10, 7e20, 3e38])
@pytest.mark.parametrize("F", [45, 1500, 6000])
def test_attend_scores_of_any_magnitude(F, size):
    """Queries of one dim and keys of powers of two there: every score is exact, and so far apart that the best frames
    share the weight evenly.  Their mean takes at most 600 sums in 32 bits: 600 * 2^-24 of the largest value."""
    wf = lib()
    g = torch.Generator("cuda").manual_seed(F)
    k = torch.zeros((1, F, 2, 64), device="cuda")
    k[..., 0] = 2.0 ** torch.randint(-1, 3, (1, F, 2), device="cuda", generator=g) * \
        (1 - 2 * torch.randint(0, 2, (1, F, 2), device="cuda", generator=g))
    v = torch.randn((1, F, 2, 64), device="cuda", generator=g)
    cache = wf.AcousticCache4(1, 2, F)
    cache.store(0, k, v)
    held = plain.kv4_values(num(k), num(v), [F])
    assert np.array_equal(held[0], num(k))
    for dtype in (torch.float32, torch.bfloat16):
        q = torch.zeros((1, 3, 2, 64), device="cuda", dtype=dtype)
        q[..., 0] = torch.tensor([size, -size, size / 64], device="cuda")[None, :, None]
        got, want = num(cache.attend(0, q)), plain.attend(num(q), *held, [F])
        half = 2.0 ** -9 if dtype == torch.bfloat16 else 2.0 ** -24
        assert (np.abs(got - want) <= 600 * 2.0 ** -24 * np.abs(held[1]).max() + 2 * half * np.abs(want)).all()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_attend_probabilities_are_exact_in_the_products(dtype):
    """Two frames of scores d and 0 and of values 6 and -6: 6 (1 - p) / (1 + p) with p = exp(-d), which for a small d is
    what the last bits of p leave.  p is off by 2^-23 (its exponential, an ulp, and the rounding of d log2(e)), the result by
    3 times that, and by at most six roundings to 2^-24 of 6 (three terms' sums, the sum of both, its inverse, the product):
    under 2^-18, then half a step of the type.  (Two bf16 terms leave up to 2^-17 of p: 2^-15.4.)"""
    wf = lib()
    d = 2.0 ** torch.arange(-13, 1, 0.125, dtype=torch.float64)
    q = torch.zeros((1, len(d), 1, 64), device="cuda", dtype=dtype)
    q[0, :, 0, 0] = (8 * d).to(q)
    k, v = torch.zeros((1, 2, 1, 64), device="cuda"), torch.full((1, 2, 1, 64), 6.0, device="cuda")
    k[0, 0, 0, 0] = 1
    v[0, 1] = -6
    cache = wf.AcousticCache4(1, 1, 2)
    cache.store(0, k, v)
    p = np.exp(-num(q)[0, :, 0, :1] / 8)
    want, got = 6 * (1 - p) / (1 + p), num(cache.attend(0, q))[0, :, 0]
    half = torch.finfo(dtype).eps / 2
    assert (np.abs(got - want) <= 2.0 ** -18 + half * want).all(), (np.abs(got - want) / (2.0 ** -18 + half * want)).max()


def pair_errors(cache, q, k, v, F):
    """2-norm of each (request, head) pair's error over its result's, and the largest sum of |q k| / 8 of its rows."""
    qn, got = num(q), num(cache.attend(0, q))
    want = plain.attend(qn, k, v, [F] * len(qn))
    off = np.linalg.norm(got - want, axis=(1, 3)) / np.linalg.norm(want, axis=(1, 3))
    mass = np.array([[(np.abs(qn[r, :, h]) @ np.abs(k[r, :, h]).T).max() / 8 for h in range(q.shape[2])] for r in range(len(qn))])
    return off, mass


@pytest.mark.parametrize("F,rows,size", [(4000, 1, 3), (1500, 9, 1), (600, 3, 8), (20000, 1, 2)])
def test_attend_fp32_every_pair(F, rows, size):
    """Every (request, head) pair by its own scores.  Products of query terms and codes are exact and the smaller terms'
    sums come first, so a score is off by the two sums of its largest terms, half a step each: in the 2-norm 2^-24 * 0.4 of
    a partial sum, which for the frames that carry the weight is up to half of mass: sqrt(2) * 0.4 * 2^-25 * mass, under
    2^-25 * mass; the probability by as much, and 2^-21 for its exponential and the sums over the frames.  (With the largest
    terms first, all six sums are of that size, and more is lost: 0.46 to 0.61 of 2^-24 * mass on average.)"""
    wf = lib()
    n, H = 6, 8
    g = torch.Generator("cuda").manual_seed(F)
    width = torch.exp(0.7 * torch.randn((2, H, 64), device="cuda", generator=g))
    k, v = [torch.randn((n, F, H, 64), device="cuda", generator=g) * w for w in width]
    cache = wf.AcousticCache4(n, H, F)
    cache.store(0, k, v)
    held = [num(x) for x in cache.load(0, n)]
    q = size * torch.randn((n, rows, H, 64), device="cuda", generator=g)
    off, mass = pair_errors(cache, q, *held, F)
    assert (off <= 2.0 ** -25 * mass + 2.0 ** -21).all(), ((off / (2.0 ** -25 * mass + 2.0 ** -21)).max(), mass.max())


@pytest.mark.parametrize("F", [130, 5000])
def test_attend_fp32_exact_scores_forty_times_as_large(F):
    """Queries of one dim, keys of a few steps there: scores are exact at any size, so what is left is the exponential's
    difference times log2(e), half a step of up to 2^-23 * 16 (beyond 16 a weight is under 2^-23), and 2^-21 for the
    exponential and the sums."""
    wf = lib()
    n, H = 3, 4
    g = torch.Generator("cuda").manual_seed(F)
    k = torch.zeros((n, F, H, 64), device="cuda")
    k[..., 5] = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6], device="cuda")[torch.randint(0, 8, (n, F, H), device="cuda", generator=g)]
    v = torch.randn((n, F, H, 64), device="cuda", generator=g)
    cache = wf.AcousticCache4(n, H, F)
    cache.store(0, k, v)
    held = [num(x) for x in cache.load(0, n)]
    q = torch.zeros((n, 5, H, 64), device="cuda")
    q[..., 5] = 40 * torch.randn((n, 5, H), device="cuda", generator=g).bfloat16()   # times a code: 10 bits
    off, _ = pair_errors(cache, q, *held, F)
    assert (off <= 2.0 ** -20 + 2.0 ** -21).all(), off.max()


def test_attend_strides_and_large_scores():
    """Rows as beams of a slot-major buffer, one row for all requests, bases off 16 bytes; scores of a few hundred."""
    wf = lib()
    n, F, H = 3, 130, 2
    k, v = source(n, F, H, torch.float32, 11)
    cache = wf.AcousticCache4(n, H, F)
    cache.store(0, k, v)
    held = plain.kv4_values(num(k), num(v), [F] * n)
    for dtype in (torch.float32, torch.bfloat16):
        buf = torch.randn((5, n, 9, 3 * H * 64), device="cuda").to(dtype)
        q = buf[:, :, 0, :H * 64].view(5, n, H, 64).transpose(0, 1)
        check_attend(cache, 0, q, *held, [F] * n, None)
        check_attend(cache, 0, q[:1, :1].expand(n, 7, H, 64), *held, [F] * n, None)
        odd = torch.empty(1 + n * 4 * H * 65, dtype=dtype, device="cuda")[1:].view(n, 4, H, 65)[..., :64]
        odd.copy_(40 * buf[:4, :, 1, :H * 64].view(4, n, H, 64).transpose(0, 1))
        check_attend(cache, 0, odd, *held, [F] * n, None)


def test_attend_long_memory():
    """70,000 frames: many chunks joined; the last frames carry the weight."""
    wf = lib()
    F, H = 70000, 2
    k, v = source(1, F, H, torch.bfloat16, 12)
    k[0, -40:] *= 4
    cache = wf.AcousticCache4(1, H, F)
    cache.store(0, k, v)
    held = plain.kv4_values(num(k), num(v), [F])
    q = torch.randn((1, 2, H, 64), device="cuda")
    check_attend(cache, 0, q, *held, [F], None)
    check_attend(cache, 0, q, *held, [69001], torch.tensor([69001], dtype=torch.int32, device="cuda"))


@pytest.mark.parametrize("n,F", [(340, 1600), (230, 1600), (50, 9000), (7, 3000)])
def test_attend_mixed_lengths_of_long_memories(n, F):
    """Many requests, split into chunks and not, some ending in the first chunk, some of no frames."""
    wf = lib()
    g = torch.Generator("cuda").manual_seed(n)
    k = torch.randn((n, F, 1, 64), device="cuda", generator=g).bfloat16()
    cache = wf.AcousticCache4(n, 1, F)
    cache.store(0, k, k.flip(1))
    held = [num(x) for x in cache.load(0, n)]
    lens = torch.randint(0, F + 1, (n,), dtype=torch.int32, device="cuda", generator=g)
    lens[0], lens[n // 2], lens[n - 1] = F, 0, 1
    q = torch.randn((n, 2, 1, 64), device="cuda", generator=g)
    check_attend(cache, 0, q, *held, lens.tolist(), lens)


def test_attend_offsets_past_32_bits():
    """A cache of over 4 GiB: the last entries lie past a 32-bit offset."""
    wf = lib()
    H, F = 20, 4096
    entries = 2 ** 32 // (H * (F // 32) * 2176) + 2
    cache = wf.AcousticCache4(entries, H, F)
    assert cache.data.numel() > 2 ** 32
    k, v = source(2, F, H, torch.bfloat16, 13)
    cache.store(entries - 2, k, v)
    held = [num(x) for x in cache.load(entries - 2, 2)]
    assert np.array_equal(held[0][:, :64, :1], plain.kv4_values(num(k[:, :64, :1]), num(v[:, :64, :1]), [64] * 2)[0])
    q = torch.randn((2, 1, H, 64), device="cuda")
    check_attend(cache, entries - 2, q, *held, [F] * 2, None)


def test_gradients_are_refused_not_lost():
    """Inputs that require gradients give the same results, which raise on backward() also where another branch has one."""
    wf = lib()
    k, v = source(1, 40, 2, torch.float32, 30)
    cache = wf.AcousticCache4(1, 2, 40)
    cache.store(0, k, v)
    g = torch.Generator("cuda").manual_seed(30)
    q, x = torch.randn((1, 3, 2, 64), device="cuda", generator=g), torch.randn((1, 2, 50), device="cuda", generator=g)
    s, w = torch.zeros((1, 2), device="cuda"), torch.ones((), device="cuda", requires_grad=True)
    want, best = cache.attend(0, q), wf.beam_select(x, s, 4)
    q, s, other = q.requires_grad_(), s.requires_grad_(), torch.cuda.Stream()
    other.wait_stream(torch.cuda.current_stream())
    for stream in (None, other):
        out = cache.attend(0, q, stream=stream)
        got = wf.beam_select(x, s, 4, stream=stream)
        torch.cuda.synchronize()
        assert torch.equal(out.detach(), want) and all(torch.equal(a.detach(), b) for a, b in zip(got, best))
        assert not got[1].requires_grad and not got[2].requires_grad
        got[0].add_(1)
        for result, name in ((out, "attend"), (got[0], "beam_select")):
            with pytest.raises(wf.WfError, match=f"{name} has no backward"):
                (w * 2 + result.sum()).backward()
    with torch.no_grad():
        assert not cache.attend(0, q).requires_grad


# ---------------------------------------------------------------- streams, graphs, several calls at once

def one_of_each(seed, dtype=torch.float32):
    """Inputs of a small search step and the call that makes it."""
    wf = lib()
    n, B, V, H, F = 3, 5, 3001, 4, 150
    g = torch.Generator("cuda").manual_seed(seed)
    k, v = source(n, F, H, dtype, seed)
    cache = wf.AcousticCache4(n, H, F)
    pages = torch.randn((4, n * B * 6, 64), device="cuda", generator=g)
    rng = np.random.default_rng(seed)
    lens = np.array([37, 48, 5])
    tables, pool = search_tables(rng, n, B, 6, 16, lens)
    up = lambda a: torch.from_numpy(np.ascontiguousarray(a, np.int32)).cuda()  # noqa: E731
    tables, pool, lens = up(tables), up(pool), up(lens)
    q = torch.randn((n, B, H, 64), device="cuda", generator=g).to(dtype)
    w = torch.randn((V, H * 64), device="cuda", generator=g)
    scores = -5 * torch.rand((n, B), device="cuda", generator=g)

    def call(stream=None):
        cache.store(0, k, v, stream=stream)
        o = cache.attend(0, q, stream=stream)
        logits = torch.matmul(o.float().view(n * B, H * 64), w.t()).view(n, B, V)
        s, b, t = wf.beam_select(logits, scores, B, stream=stream)
        new = wf.cache_reorder(pages, tables, b, lens, pool, stream=stream)
        return o, s, b, t, new, pages

    return call


def test_operators_together_on_other_streams():
    """Two searches on two streams at once give what each gives alone."""
    calls = [one_of_each(1), one_of_each(2)]
    want = [[t.clone() for t in c()] for c in calls]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in calls]
    got = [None, None]
    for _ in range(20):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                got[i] = calls[i]()
    torch.cuda.synchronize()
    for w, g in zip(want, got):
        for x, y in zip(w, g):
            assert torch.equal(x, y)


def test_operators_on_a_given_stream():
    wf = lib()
    s = torch.cuda.Stream()
    logits = torch.randn((2, 3, 999), device="cuda")
    scores = torch.zeros((2, 3), device="cuda")
    torch.cuda.synchronize()
    got = wf.beam_select(logits, scores, 6, stream=s)
    s.synchronize()
    for x, y in zip(got, wf.beam_select(logits, scores, 6)):
        assert torch.equal(x, y)


def test_a_given_streams_results_take_that_streams_memory():
    """Memory freed on the current stream, whose work on it has not run, is not what a call on another stream writes."""
    wf = lib()
    s = torch.cuda.Stream()
    logits, scores = torch.randn((2, 3, 999), device="cuda"), torch.zeros((2, 3), device="cuda")
    k, v = source(2, 64, 2, torch.float32, 30)
    cache = wf.AcousticCache4(2, 2, 64)
    cache.store(0, k, v)
    q = torch.randn((2, 3, 2, 64), device="cuda")

    def call(stream=None):
        return [*wf.beam_select(logits, scores, 6, stream=stream), cache.attend(0, q, stream=stream),
                *cache.load(0, 2, stream=stream)]
    want = call()
    call(s)
    torch.cuda.synchronize()
    x = torch.randn((4096, 4096), device="cuda")
    for _ in range(5):
        for _ in range(20):
            x = x @ x * 1e-4
        stale = [torch.full_like(t, 7) for t in want for _ in range(4)]     # runs long after the calls on s
        del stale
        got = call(s)
        torch.cuda.synchronize()
        for a, b in zip(got, want):
            assert torch.equal(a, b)


def test_operators_captured_into_a_graph():
    """Two searches captured into two graphs, replayed in turn with eager work between: every replay gives the
    eager result."""
    calls = [one_of_each(3), one_of_each(4)]
    want = [[t.clone() for t in c()] for c in calls]
    torch.cuda.synchronize()
    graphs, outs = [], []
    for c in calls:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(c())
        graphs.append(g)
    for _ in range(4):
        for g, o, w in zip(graphs, outs, want):
            for t in o[:5]:
                t.fill_(0)
            g.replay()
            torch.cuda.synchronize()
            for x, y in zip(o, w):
                assert torch.equal(x, y)
        calls[0]()
        torch.cuda.synchronize()


def test_results_do_not_vary():
    """The same call twenty times: the same bits."""
    call = one_of_each(5, torch.bfloat16)
    first = [t.clone() for t in call()]
    for _ in range(20):
        for x, y in zip(first, call()):
            assert torch.equal(x, y)
