"""Attention over packed prompts and the 8-bit cache where values or scores are far apart: large values behind small
references, infinities that a row does not see, a row's own keys far below the earlier ones."""
import numpy as np
import pytest
import torch

from oracle import operators as plain
from test_gpu_selfattn import BF16, F32, INF, NAN, borders, bound, check_attend, check_rows, i32, lib, num, random_tables

pytestmark = pytest.mark.gpu

# (rows, heads, key and value heads, prompts, type, elements off a 16-byte border): each kind of tiles
KINDS = [(300, 2, 1, 2, F32, 0), (12000, 3, 1, 2, F32, 0), (12345, 9, 3, 97, F32, 0), (300, 2, 1, 2, BF16, 1), (300, 2, 1, 4, BF16, 0), (700, 2, 1, 1, BF16, 0),
         (12345, 4, 4, 30, BF16, 0), (33000, 20, 5, 1, BF16, 0)]


def slices(T, H, KV, dtype, offset):
    """Queries, keys and values of zeros, as slices of one buffer."""
    buf = torch.zeros(offset + T * (H + 2 * KV) * 64, device="cuda", dtype=dtype)
    x = buf[offset:].view(T, H + 2 * KV, 64)
    return x[:, :H], x[:, H:H + KV], x[:, H + KV:]


@pytest.mark.parametrize("T,H,KV,n,dtype,offset", KINDS)
def test_prompt_large_values_behind_a_small_reference(T, H, KV, n, dtype, offset):
    """A key five nats above the others' scores with values of 3e36: results are below that, whatever was seen before."""
    q, k, v = slices(T, H, KV, dtype, offset)
    g = torch.Generator("cuda").manual_seed(T)
    v.copy_(torch.randn(v.shape, device="cuda", generator=g))
    q[:, :, 0] = 8
    starts = [T * i // n for i in range(n)] + [T]
    rows = set()
    for a, b in zip(starts[:3], starts[1:4]):
        at = a + (b - a) // 5
        k[at, :, 0], v[at, :, 3], v[at, :, 4] = 5, 3e36, -3e36
        rows |= {i for i in (at - 1, at, at + 1, at + 64, at + 128, at + 200, b - 1) if a <= i < b}
    got = lib().prompt_attention(q, k, v, i32(starts))
    assert torch.isfinite(got).all()
    check_rows(q, k, v, got, starts, sorted(rows))


@pytest.mark.parametrize("dtype,offset", [(F32, 0), (BF16, 0), (BF16, 1)])
@pytest.mark.parametrize("T", [100, 29000])
def test_prompt_large_values_of_every_key(T, dtype, offset):
    """100 keys a prompt, all values 3.3e36, scores of any order: sums of probabilities times values stay below 3.4e38."""
    q, k, v = slices(T, 2, 1, dtype, offset)
    g = torch.Generator("cuda").manual_seed(T)
    q.copy_(torch.randn(q.shape, device="cuda", generator=g))
    k.copy_(2 * torch.randn(k.shape, device="cuda", generator=g))
    v.fill_(3.3e36)
    starts = list(range(0, T + 1, 100))
    got = lib().prompt_attention(q, k, v, i32(starts))
    assert torch.isfinite(got).all()
    check_rows(q, k, v, got, starts, [0, 1, 50, 99, T - 100, T - 1])


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("n,heads,group,width", [(1, 2, 1, 28), (1, 1, 8, 200), (300, 1, 1, 28), (260, 4, 1, 8)])
def test_attend8_large_values_behind_a_small_reference(n, heads, group, width, dtype):
    """The same of the cache's: one, four or eight waves a block, and chunks."""
    rng, rows, length = np.random.default_rng(width), 2, 16 * width
    cache, model = lib().PagedCache8(n * width, heads), plain.PagedCache8(n * width, heads)
    tables = random_tables(rng, n, width, n * width)
    k = torch.zeros((n, length, heads, 64), device="cuda")
    v = torch.from_numpy(rng.standard_normal(k.shape)).float().cuda()
    for at in {40, 259, length - 40}:
        if at < length - rows:
            k[:, at, :, 0], v[:, at, :, 3], v[:, at, :, 4] = 5, 3e36, -3e36
    cache.store(k, v, i32(tables), i32([0] * n))
    q = torch.zeros((n, rows, heads * group, 64), device="cuda", dtype=dtype)
    q[..., 0] = 8
    at = [length - rows] * n
    got = cache.attend(q, i32(tables), i32(at))
    assert torch.isfinite(got).all()
    some = sorted({0, n // 2, n - 1})
    model.store(num(k[some]), num(v[some]), tables[some], [0] * len(some))
    check_attend(cache, model, q[some], tables[some], at[:len(some)], got=got[some])


@pytest.mark.parametrize("T,H,KV,n,dtype,offset", KINDS)
@pytest.mark.parametrize("below", [1e4, 1e6, 1e8])
def test_prompt_own_keys_far_below(T, H, KV, n, dtype, offset, below):
    """A row's own tiles score -below, earlier keys around 0: those keep all weight, at their own scores' accuracy.  Of 64 products
    one is what sets the near keys apart: the far keys' is a product with 0, and adds neither size nor error."""
    q, k, v = slices(T, H, KV, dtype, offset)
    g = torch.Generator("cuda").manual_seed(T)
    for t in (q, k, v):
        t.copy_(torch.randn(t.shape, device="cuda", generator=g))
    starts = [T * i // n for i in range(n)] + [T]
    q[:, :, 0], k[:, :, 0] = 256, 0
    rows = []
    for a, b in zip(starts, starts[1:]):
        near = b - min(140, (b - a) // 2)                    # more than a block's own tiles of keys where the prompt is long
        k[near:b, :, 0] = -below / 32
        rows.append((a, near, b))
    got = lib().prompt_attention(q, k, v, i32(starts))
    for a, near, b in rows[:2] + rows[-1:]:
        for i in {near, (near + b) // 2, b - 1}:
            # the weights of the near keys, exp(-below / 2) at most, are zeros in 64 bits too
            assert below / 2 > 800
            want, spread, size = plain.seen_attention(num(q[i:i + 1]), num(k[a:near]), num(v[a:near]), np.ones((1, near - a), bool))
            assert size.max() < 64
            err = np.abs(num(got[i:i + 1]) - want)
            assert (err <= bound(want, spread, size, near - a, dtype, dtype == BF16)).all(), (i, err.max())


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("n,heads,group,width", [(2, 2, 1, 28), (1, 1, 8, 200), (260, 4, 1, 8)])
def test_attend8_first_keys_far_below(n, heads, group, width, dtype):
    """The cache's positions are taken from the first on: those score far below, the last ones around 0."""
    rng, rows, length = np.random.default_rng(width), 2, 16 * width
    cache, model = lib().PagedCache8(n * width, heads), plain.PagedCache8(n * width, heads)
    tables = random_tables(rng, n, width, n * width)
    k, v = (torch.from_numpy(rng.standard_normal((n, length, heads, 64))).float().cuda() for _ in range(2))
    k[..., 0] = 0
    far = length - 48
    k[:, :far, :, 0] = -2.0 ** 15                            # exact in 8 bits; what lies beside it in a page is rounded coarsely
    cache.store(k, v, i32(tables), i32([0] * n))
    q = torch.from_numpy(rng.standard_normal((n, rows, heads * group, 64))).to(dtype).cuda()
    q[..., 0] = 256
    got = cache.attend(q, i32(tables), i32([length - rows] * n))
    model.store(num(k[:1]), num(v[:1]), tables[:1], [0])
    kk, vv, _ = model.rows(tables[0], length)
    sees = np.arange(far, length)[None] <= length - rows + np.arange(rows)[:, None]
    want, spread, size = plain.seen_attention(num(q[0]), kk[far:], vv[far:], sees)
    assert size.max() < 64
    assert (np.abs(num(got[0]) - want) <= bound(want, spread, size, 48, dtype)).all()


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("width,where", [(3, 16), (3, 32), (60, 896), (200, 3008)])
def test_attend8_infinities_that_a_row_does_not_see(dtype, width, where):
    """Values of 3.35e38, which the cache holds as infinity: rows before them are as without them, those from them on infinite of their
    sign, NaN where a row sees both."""
    rng, n, heads = np.random.default_rng(where), 3, 2
    cache, model = lib().PagedCache8(n * width, heads), plain.PagedCache8(n * width, heads)
    cache.data.fill_(0xff)
    tables = random_tables(rng, n, width, n * width)
    k, v = (torch.from_numpy(rng.standard_normal((n, where, heads, 64))).float().cuda() for _ in range(2))
    cache.store(k, v, i32(tables), i32([0] * n))
    model.store(num(k), num(v), tables, [0] * n)
    q = torch.from_numpy(0.3 * rng.standard_normal((n, 7, 2 * heads, 64))).to(dtype).cuda()
    at = [where - 3] * n
    clean = cache.attend(q, i32(tables), i32(at), counts=i32([3] * n))
    x, y = (torch.from_numpy(rng.standard_normal((n, 4, heads, 64))).float().cuda() for _ in range(2))
    y[0, 0, 0, 7], y[0, 1, 1, 9], y[0, 2, 0, 7], y[0, 3, 0, 11] = 3.35e38, -3.35e38, -3.4e38, NAN     # of several rows and heads
    y[1, 3] = 3.35e38                                                # the last row only
    y[2, 2, :, :32] = 247 * 2.0 ** 120                               # the largest finite ones beside them
    cache.store(x, y, i32(tables), i32([where] * n))
    model.store(num(x), num(y), tables, [where] * n)
    got = cache.attend(q, i32(tables), i32(at))
    assert torch.equal(got[:, :3], clean[:, :3])
    for r in range(n):
        kk, vv, _ = model.rows(tables[r], where + 4)
        vv = np.where(np.abs(vv) >= 2.0 ** 128, np.copysign(INF, vv), vv)
        sees = np.arange(where + 4)[None] <= at[r] + np.arange(7)[:, None]
        want, spread, size = plain.seen_attention(num(q[r]), kk, vv, sees)
        g = num(got[r])
        bad = ~np.isfinite(want)
        assert np.array_equal(np.isnan(g), np.isnan(want)) and np.array_equal(g[np.isinf(want)], want[np.isinf(want)])
        assert bad.any() == (r < 2)
        tol = bound(np.where(bad, 0, want), np.where(bad, 0, spread), size, where + 4, dtype)
        assert (np.abs(np.where(bad, 0, g) - np.where(bad, 0, want)) <= tol).all()


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("width", [1, 70])
def test_attend8_probabilities_are_exact_in_the_products(dtype, width):
    """Two positions of scores d and 0 and of values 6 and -6: 6 (1 - p) / (1 + p) with p = exp(-d), which for a small d is what
    the last bits of p leave.  The scores are exact; p is off by 2^-23 for its exponential and 2^-23 for the rounding of d log2(e)
    and of its factor, the result by 3 times that (12 p / (1 + p)^2 <= 3), and by at most six roundings to 2^-24 of 6: under 2^-18,
    then half a step of the type.  (Two bf16 terms leave up to 2^-16 of p: 2^-14.4.)"""
    d = 2.0 ** torch.arange(-13, 1, 0.125, dtype=torch.float64)
    n = len(d)
    q = torch.zeros((n, 1, 1, 64), device="cuda", dtype=dtype)
    q[:, 0, 0, 0] = (8 * d).to(q)
    k, v = torch.zeros((1, 2, 1, 64), device="cuda"), torch.full((1, 2, 1, 64), 6.0, device="cuda")
    k[0, 0, 0, 0] = 1
    v[0, 1] = -6
    cache = lib().PagedCache8(width, 1)
    table = i32([list(range(width))])
    cache.store(k, v, table, i32([0]))
    got = num(cache.attend(q, table.expand(n, width), i32([1] * n)))[:, 0, 0]
    p = np.exp(-num(q)[:, 0, 0, :1] / 8)
    want = 6 * (1 - p) / (1 + p)
    tol = 2.0 ** -18 + torch.finfo(dtype).eps / 2 * want
    assert (np.abs(got - want) <= tol).all(), (np.abs(got - want) / tol).max()
