"""Rotary positions, packed prompts and the 8-bit paged cache, as far as no GPU is needed: refusals before anything
is enqueued (the pointers here point at nothing), frequencies, page sizes, and pins of the plain forms."""
import ctypes

import numpy as np
import pytest
import torch

from oracle import operators as plain
from test_operators_cpu import P, S3, _lib, varied

S2 = ctypes.c_int64 * 2


def turns_of(dims, base, scaling, factor, context, low, high):
    binding, lib = _lib()
    t, a = (ctypes.c_double * max(1, dims // 2))(), ctypes.c_float()
    rc = lib.wf_rotary_turns(dims, base, scaling, factor, context, low, high, t, ctypes.byref(a))
    return rc, np.array(t), a.value


@pytest.mark.parametrize("dims", [2, 4, 20, 64, 128, 4096])
@pytest.mark.parametrize("name,scaling", [(None, 0), ("linear", 1), ("base", 2), ("ramp", 3)])
def test_turns(dims, name, scaling):
    """Powers and quotients in 64 bits: a few roundings each."""
    if name == "base" and dims == 2:
        assert turns_of(dims, 1e4, scaling, 4.0, 0, 0, 0)[0] == -1
        return
    rc, t, a = turns_of(dims, 5e5, scaling, 4.0, 2048, 1.0, 32.0)
    want, amplitude = plain.rotary_turns(dims, 5e5, name, 4.0, 2048, 1.0, 32.0)
    assert rc == 0 and np.allclose(t, want, rtol=1e-13, atol=0) and abs(a - amplitude) <= 2.0 ** -24 * amplitude


def test_turns_of_scalings():
    """A factor of 1 changes nothing; the ramp keeps fast pairs, divides slow ones and mixes those between."""
    one = turns_of(64, 1e4, 0, 0, 0, 0, 0)[1]
    for scaling in (1, 2, 3):
        rc, t, a = turns_of(64, 1e4, scaling, 1.0, 4096, 1, 32)
        assert rc == 0 and np.allclose(t, one, rtol=1e-14) and a == 1.0
    t = turns_of(64, 1e4, 3, 8.0, 4096, 1, 32)[1]
    fast, slow = one * 4096 >= 32, one * 4096 <= 1
    assert fast.any() and slow.any() and (~fast & ~slow).any()
    assert np.array_equal(t[fast], one[fast]) and np.allclose(t[slow], one[slow] / 8, rtol=1e-15)
    mid = ~fast & ~slow
    assert (t[mid] < one[mid]).all() and (t[mid] > one[mid] / 8).all()
    base = turns_of(64, 1e4, 2, 8.0, 0, 0, 0)[1]
    assert base[0] == one[0] and np.isclose(base[-1], one[-1] / 8, rtol=1e-13)   # the slowest pair divided by the factor


def test_turns_refusals():
    nan, inf = float("nan"), float("inf")
    for bad in [dict(dims=0), dict(dims=3), dict(dims=4098), dict(dims=-2), dict(base=1.0), dict(base=nan), dict(base=inf),
                dict(scaling=-1), dict(scaling=4), dict(scaling=1, factor=0.5), dict(scaling=2, factor=nan),
                dict(scaling=3, factor=inf), dict(scaling=3, context=0.0), dict(scaling=3, context=nan),
                dict(scaling=3, low=32.0), dict(scaling=3, low=-1.0), dict(scaling=3, high=inf), dict(scaling=3, low=nan)]:
        a = dict(dict(dims=64, base=1e4, scaling=0, factor=2.0, context=4096.0, low=1.0, high=32.0), **bad)
        assert turns_of(a["dims"], a["base"], a["scaling"], a["factor"], a["context"], a["low"], a["high"])[0] == -1, bad
    binding, lib = _lib()
    assert lib.wf_rotary_turns(64, 1e4, 0, 1, 0, 0, 0, None, None) == -1


def test_rotary_refusals():
    binding, lib = _lib()
    xs, ys = S2(60 * 64, 64), S2(20 * 64, 64)

    def call(lib, a):
        return lib.wf_rotary(a["turns"], a["dims"], 0, a["amp"], 0, a["at"], a["tokens"], a["width"], a["dtype"], a["q"], a["qs"], a["qh"],
                             a["qo"], a["qos"], a["k"], a["ks"], a["kh"], a["ko"], a["kos"], None)
    good = dict(turns=P, dims=64, amp=1.0, at=P, tokens=7, width=64, dtype=0, q=P, qs=xs, qh=20, qo=P + (1 << 16), qos=ys,
                k=P, ks=xs, kh=20, ko=P + (1 << 18), kos=ys)
    bad = {"turns": [(None, -1), (P + 4, -1)], "dims": [(0, -1), (1, -1), (66, -1), (-64, -1)], "amp": [(float("nan"), -1), (float("inf"), -1)],
           "at": [(None, -1), (P + 2, -1)], "tokens": [(-1, -1), ((1 << 28) + 1, -1)], "width": [(1, -1), (62, -1), (4098, -1)], "dtype": [(2, -1)],
           "q": [(None, -1), (P + 2, -1), (P + (1 << 16), -1)]}                       # the last: in place with other strides
    for x in "qk":
        bad.update({x + "s": [(None, -1), (S2(-1, 64), -1), (S2(0, 1 << 41), -1)], x + "h": [(0, -1), (70000, -1)], x + "o": [(None, -1), (P + 1, -1)],
                    x + "os": [(S2(0, 64), -1), (S2(20 * 64, 32), -1), (S2(19 * 64, 64), -1), (S2(64, 6 * 64), -1), (None, -1)]})
    varied(call, good, bad)
    assert call(lib, dict(good, tokens=0)) == 0
    assert call(lib, dict(good, tokens=0, k=None, ks=None, kh=0, ko=None, kos=None)) == 0
    # results over each other: the same memory, heads of one buffer that meet, rows that reach into the next token's
    rows = S2(30 * 64, 64)
    wide = dict(good, qos=rows, kos=rows, kh=10)
    for apart, bad_ in ((0, True), (19 * 64, True), (20 * 64, False), (20 * 64 + 8, True), (-10 * 64, False), (-9 * 64, True), (30 * 64 + 20 * 64, False),
                        (30 * 64, True), (7 * 30 * 64, False), (6 * 30 * 64 + 20 * 64 - 8, True)):
        a = dict(wide, qo=P + (1 << 16), ko=P + (1 << 16) + 4 * apart)
        # a call that is fine is not made: a width of no good makes it refused for another reason
        assert call(lib, a if bad_ else dict(a, dtype=9)) == -1
        assert (b"results overlap" in lib.wf_last_error(None)) == bad_, apart
    assert call(lib, dict(wide, qo=P + (1 << 16), ko=P + (1 << 16) + 4 * 20 * 64, kos=S2(31 * 64, 64))) == -1
    # layouts that do not overlap: heads before tokens, one head
    for strides in (S2(64, 7 * 64), S2(64, 9 * 64)):
        assert call(lib, dict(good, qos=strides, tokens=0)) == 0
    assert call(lib, dict(good, qh=1, qos=S2(64, 0), tokens=0)) == 0


def test_prompt_refusals():
    s, o = S2(60 * 64, 64), S2(20 * 64, 64)

    def call(lib, a):
        return lib.wf_prompt_attend(a["q"], a["qs"], a["k"], a["ks"], a["v"], a["vs"], a["dtype"], a["starts"], a["n"], a["tokens"],
                                    a["heads"], a["kv"], a["out"], 1, None)
    strides = [(None, -1), (S2(-1, 64), -1), (S2(0, 1 << 41), -1)]
    good = dict(q=P, qs=s, k=P, ks=s, v=P, vs=o, dtype=1, starts=P, n=3, tokens=100, heads=20, kv=10, out=P)
    varied(call, good, {
        "q": [(None, -1), (P + 1, -1)], "k": [(None, -1), (P + 1, -1)], "v": [(None, -1)], "qs": strides, "ks": strides, "vs": strides,
        "dtype": [(2, -1), (-1, -1)], "starts": [(None, -1), (P + 2, -1)], "n": [(0, -1), ((1 << 24) + 1, -1)],
        "tokens": [(-1, -1), ((1 << 28) + 1, -1)], "heads": [(0, -1), (15, -1), (70000, -1)], "kv": [(0, -1), (3, -1), (40, -1)],
        "out": [(None, -1), (P + 8, -1)]})
    binding, lib = _lib()
    assert call(lib, dict(good, tokens=0)) == 0
    # 100 tokens of 20 heads in rows of 60 (q) or 20 (k, v) heads: results over any of them
    far = dict(good, k=P + (1 << 30), v=P + (2 << 30), dtype=0)
    for out in (P, P + 100 * 20 * 64 * 4, P + (99 * 60 + 20) * 256 - 16, P + (1 << 30) - 16, P + (2 << 30) + 99 * 20 * 256):
        assert call(lib, dict(far, out=out)) == -1 and b"overlaps" in lib.wf_last_error(None)


def test_cache8_refusals():
    binding, lib = _lib()

    def cache(**kw):
        f = dict(data=P, pages=50, heads=2)
        f.update(kw)
        return ctypes.byref(binding.WfKv8(f["data"], f["pages"], f["heads"]))
    caches = [(None, -1), (cache(data=None), -1), (cache(data=P + 8), -1), (cache(pages=0), -1), (cache(pages=(1 << 24) + 1), -1),
              (cache(heads=0), -1), (cache(heads=4097), -1)]
    table = dict(n=[(0, -1), (70000, -1)], tables=[(None, -1), (P + 2, -1)], ts=[(-1, -1), (1 << 41, -1)], most=[(0, -1), ((1 << 24) + 1, -1)])
    strides = [(None, -1), (S3(-1, 0, 0), -1), (S3(0, 1 << 41, 0), -1)]

    def store(lib, a):
        return lib.wf_kv8_store(a["c"], a["n"], a["k"], a["ks"], a["v"], a["vs"], a["dtype"], a["rows"], a["starts"], a["counts"],
                                a["tables"], a["ts"], a["most"], a["at"], None)
    s = S3(9 * 128, 128, 64)
    good = dict(c=cache(), n=3, k=P, ks=s, v=P, vs=s, dtype=0, rows=9, starts=None, counts=None, tables=P, ts=8, most=8, at=P)
    varied(store, good, dict(c=caches, k=[(None, -1), (P + 2, -1)], v=[(None, -1)], ks=strides, vs=strides, dtype=[(2, -1)],
                             rows=[(-1, -1), ((1 << 20) + 1, -1)], starts=[(P + 2, -1)], counts=[(P + 1, -1)], at=[(None, -1), (P + 2, -1)], **table))
    assert store(lib, dict(good, rows=0)) == 0
    assert store(lib, dict(good, starts=P, counts=P)) == -1
    assert store(lib, dict(good, starts=P, rows=(1 << 27) + 1)) == -1
    assert store(lib, dict(good, n=65535, rows=1 << 20)) == -1

    def load(lib, a):
        return lib.wf_kv8_load(a["c"], a["n"], a["tables"], a["ts"], a["most"], a["lens"], a["k"], a["v"], a["dtype"], None)
    varied(load, dict(c=cache(), n=3, tables=P, ts=8, most=8, lens=P, k=P, v=P, dtype=1),
           dict(c=caches, lens=[(None, -1), (P + 2, -1)], k=[(None, -1), (P + 4, -1)], v=[(None, -1)], dtype=[(3, -1)], **table))
    assert load(lib, dict(c=cache(), n=65535, tables=P, ts=8, most=300, lens=P, k=P, v=P, dtype=1)) == -1

    def attend(lib, a):
        return lib.wf_kv8_attend(a["c"], a["n"], a["q"], a["qs"], a["rows"], a["heads"], a["dtype"], a["tables"], a["ts"], a["most"], a["at"],
                                 a["counts"], a["out"], a["ws"], a["bytes"], None)
    good = dict(c=cache(), n=3, q=P, qs=S3(9 * 512, 512, 64), rows=9, heads=8, dtype=0, tables=P, ts=8000, most=8000, at=P, counts=None, out=P, ws=P,
                bytes=1 << 40)
    varied(attend, good, dict(c=caches, q=[(None, -1), (P + 2, -1)], qs=strides, rows=[(0, -1), ((1 << 17) + 1, -1)],
                              heads=[(0, -1), (7, -1), (1, -1), (65536, -1)], dtype=[(2, -1)], at=[(None, -1), (P + 2, -1)], counts=[(P + 2, -1)],
                              out=[(None, -1), (P + 8, -1)], ws=[(None, -1), (P + 16, -1)], bytes=[(0, -3), (100, -3)], **table))


def test_cache8_sizes():
    binding, lib = _lib()
    n = ctypes.c_size_t()
    for heads in (1, 2, 8, 9, 20, 4096):
        assert lib.wf_kv8_page_bytes(heads, ctypes.byref(n)) == 0
        assert n.value % 16 == 0 and 2050 * heads <= n.value < 2050 * heads + 16
    assert lib.wf_kv8_page_bytes(0, ctypes.byref(n)) == -1 and lib.wf_kv8_page_bytes(1, None) == -1
    c = binding.WfKv8(None, 100, 8)
    assert lib.wf_kv8_attend_workspace_bytes(ctypes.byref(c), 1, 1, 8, 8192, ctypes.byref(n)) == 0 and n.value > 0
    assert lib.wf_kv8_attend_workspace_bytes(ctypes.byref(c), 96, 9, 160, 28, ctypes.byref(n)) == 0 and n.value == 0
    assert lib.wf_kv8_attend_workspace_bytes(ctypes.byref(c), 96, 9, 160, 28, None) == -1


def test_binding_refuses():
    """Before the library is asked: tensors elsewhere, of other types and of other shapes."""
    from paper_2609_32869_amd import PagedCache8, Rotary, WfError, prompt_attention
    _lib()
    x = torch.zeros((4, 2, 64))
    with pytest.raises(WfError, match="on the GPU"):
        prompt_attention(x, x, x, torch.zeros(2, dtype=torch.int32))
    for bad in (dict(dims=63), dict(dims=64, scaling="ramp"), dict(dims=64, scaling="ntk"), dict(dims=64, scaling="linear", factor=0.5),
                dict(dims=2 ** 40), dict(dims=64, device="cpu")):
        with pytest.raises(WfError):
            Rotary(**dict(dict(device="cpu"), **bad))
    for bad in (dict(pages=0), dict(pages=2 ** 33), dict(n_head=0), dict(layers=0), dict(n_head=-1)):
        with pytest.raises(WfError):
            PagedCache8(**dict(dict(pages=4, n_head=2, device="cpu"), **bad))
    with pytest.raises(WfError, match="GPU"):
        PagedCache8(4, 2, device="cpu")


# ---------------------------------------------------------------- the plain forms

def test_plain_rotary_is_a_rotation():
    rng = np.random.default_rng(0)
    x = rng.standard_normal((5, 3, 64))
    at = np.array([0, 1, 1000, -7, 2 ** 31 - 1])
    for inter in (False, True):
        for dims in (2, 24, 64):
            t, _ = plain.rotary_turns(dims)
            y = plain.rotary(x, at, t, 1.0, inter)
            assert np.array_equal(y[0], x[0]) and np.array_equal(y[..., dims:], x[..., dims:])
            assert np.allclose((y ** 2).sum(-1), (x ** 2).sum(-1))
            assert np.allclose(plain.rotary(y, at, t, 1.0, inter, transposed=True), x, atol=1e-12)
            a = np.zeros((1, 1, 64))
            a[0, 0, 0] = 1                       # the first pair turns by one radian a position
            z = plain.rotary(a, [1], t, 1.0, inter)[0, 0]
            assert np.isclose(z[0], np.cos(1)) and np.isclose(z[1 if inter else dims // 2], np.sin(1))


def test_plain_prompt_against_a_library():
    rng = np.random.default_rng(1)
    q, k, v = rng.standard_normal((20, 4, 64)), rng.standard_normal((20, 2, 64)), rng.standard_normal((20, 2, 64))
    got = plain.prompt_attention(q, k, v, [2, 2, 9, 18])[0]
    for a, b in ((2, 9), (9, 18)):
        t = [torch.from_numpy(x[a:b]).transpose(0, 1) for x in (q, k.repeat(2, 1), v.repeat(2, 1))]
        want = torch.nn.functional.scaled_dot_product_attention(*t, is_causal=True).transpose(0, 1).numpy()
        assert np.allclose(got[a:b], want, atol=1e-12)
    assert not got[:2].any() and not got[18:].any()


def test_plain_quantise8():
    """Every code and tie of the grid against the type of the same name, and the scale's minimality."""
    assert np.array_equal(plain.E4M3, np.sort(np.unique(np.abs(torch.arange(256).to(torch.uint8).view(torch.float8_e4m3fn).float().numpy()[:127]))))
    rng = np.random.default_rng(2)
    x = rng.standard_normal((16, 64)) * np.exp(3 * rng.standard_normal((16, 64)))
    x[0, 0] = 448.0 * 2 ** 5
    x[np.abs(x) > 448 * 2 ** 5] = 1.0
    mid = (plain.E4M3[:-1] + plain.E4M3[1:]) / 2 * 2.0 ** 5
    x.flat[64:64 + len(mid)] = mid
    want = (torch.from_numpy(x) / 2 ** 5).float().to(torch.float8_e4m3fn).double().numpy() * 2 ** 5
    assert np.array_equal(plain.quantise8(x), want)
    x[0, 0] = 448.0 * 2 ** 5 + 1                  # the next scale: 224.03 of it, code 224
    assert plain.quantise8(x)[0, 0] == 224.0 * 2 ** 6
    z = np.full((16, 64), 1.0)
    z[3, 3], z[4, 4] = np.inf, np.nan
    r = plain.quantise8(z)
    assert np.isnan(r[3, 3]) and np.isnan(r[4, 4]) and np.isnan(r).sum() == 2 and (r[0] == 1).all()
    assert not plain.quantise8(np.zeros((16, 64))).any()


def test_plain_cache8_appends():
    """Values that were stored stay the same while the scale does; one larger value doubles the spacing at most once a step."""
    rng = np.random.default_rng(3)
    c = plain.PagedCache8(3, 1)
    x = rng.standard_normal((1, 40, 1, 64))
    c.store([x[0, :5]], [x[0, :5]], [[2, 0, 1]], [0])
    was = c.k[2, 0, :5].copy()
    c.store([x[0, 5:40] * 0.1], [x[0, 5:40]], [[2, 0, 1]], [5])
    assert np.array_equal(c.k[2, 0, :5], was)
    k, v, there = c.rows([2, 0, 1], 40)
    assert there.all() and np.abs(v - x[0]).max() < np.abs(x).max() / 16
    assert not c.k[1, 0, 8:].any()
    c.store([x[0, :1] * 100], [x[0, :1]], [[2, 0, 1]], [3])          # a rollback: what followed is gone
    scale = 2.0 ** np.ceil(np.log2(np.abs(100 * x[0, 0]).max() / 448))   # values below 2^-6 of it lie 2^-9 of it apart
    assert not c.k[2, 0, 4:].any() and np.allclose(c.k[2, 0, :3], was[:3], rtol=2.0 ** -4, atol=2.0 ** -10 * scale)
