"""The operators without a handle and the beam search, as far as no GPU is needed: every refusal before
anything is enqueued (the pointers here point at nothing), workspace sizes, and pins of the plain forms."""
import ctypes
import itertools
import os
import subprocess
import sys

import numpy as np
import pytest
import torch

from oracle import OracleOpts, Target, operators as plain
from oracle.beam import beam_search, last_logits
from wf_fixtures import VOCAB64, make_memory, make_prefix, make_weights


def _lib():
    from paper_2609_32869_amd import binding
    if not os.path.exists(binding.LIB_PATH):
        pytest.skip("libwf.so not built")
    return binding, binding.load_library()


P = 1 << 20   # a well-aligned address that is never followed
S3 = ctypes.c_int64 * 3


def varied(call, good, bad):
    """call(**good) is never made; every single bad value is refused with its code and a message."""
    binding, lib = _lib()
    for name, values in bad.items():
        for value, code in values:
            args = dict(good)
            args[name] = value
            assert call(lib, args) == code, (name, value)
            assert lib.wf_last_error(None)


def test_select_refusals():
    good = dict(logits=P, dtype=0, sr=500, sb=100, scores=P, sup=None, n=2, beams=5, vocab=100, k=10, s=P, b=P, t=P, ws=P,
                bytes=1 << 30)

    def call(lib, a):
        return lib.wf_beam_select(a["logits"], a["dtype"], a["sr"], a["sb"], a["scores"], a["sup"], a["n"], a["beams"],
                                  a["vocab"], a["k"], a["s"], a["b"], a["t"], a["ws"], a["bytes"], None)
    varied(call, good, {
        "logits": [(None, -1), (P + 2, -1)], "dtype": [(2, -1), (-1, -1)], "sr": [(-1, -1), (1 << 50, -1)], "sb": [(-5, -1)],
        "scores": [(None, -1), (P + 1, -1)], "n": [(0, -1), (-1, -1), (70000, -1)], "beams": [(0, -1), (17, -1)],
        "vocab": [(0, -1), ((1 << 20) + 1, -1)], "k": [(0, -1), (33, -1)], "s": [(None, -1), (P + 2, -1)],
        "b": [(None, -1)], "t": [(None, -1)], "ws": [(None, -1), (P + 16, -1)], "bytes": [(0, -3), (1000, -3)]})


def test_reorder_refusals():
    good = dict(cache=P, regions=2, stride=4096, pages=4, page=1024, tables=P, new=P + 4096, n=1, beams=2, most=2, tokens=16,
                parents=P, lens=P, pool=P, pool_pages=4)

    def call(lib, a):
        return lib.wf_cache_reorder(a["cache"], a["regions"], a["stride"], a["pages"], a["page"], a["tables"], a["new"], a["n"],
                                    a["beams"], a["most"], a["tokens"], a["parents"], a["lens"], a["pool"], a["pool_pages"], None)
    varied(call, good, {
        "cache": [(None, -1), (P + 8, -1)], "regions": [(0, -1), (70000, -1)], "stride": [(4000, -1), (2048, -1), (4097, -1)],
        "pages": [(0, -1), ((1 << 18) + 1, -1)], "page": [(0, -1), (1000, -1)], "tables": [(None, -1), (P + 2, -1), (P + 4096 + 4, -1)],
        "new": [(None, -1), (P, -1), (P + 12, -1)], "n": [(0, -1)], "beams": [(0, -1), (17, -1)], "most": [(0, -1)],
        "tokens": [(0, -1)], "parents": [(None, -1)], "lens": [(None, -1)], "pool": [(None, -1)], "pool_pages": [(0, -1)]})


def test_reorder_refuses_new_tables_over_what_it_reads():
    """Sizes 3 x 4 x 5 tables: 240 bytes; parents 48, lens 12, pool 3 x 20 words."""
    binding, lib = _lib()
    new = P + (1 << 16)
    far = dict(tables=P, parents=P + 4096, lens=P + 8192, pool=P + 12288)
    size = dict(tables=240, parents=48, lens=12, pool=240)

    def call(a, tokens=16):
        return lib.wf_cache_reorder(P << 4, 2, 1 << 20, 64, 1024, a["tables"], new, 3, 4, 5, tokens, a["parents"], a["lens"], a["pool"],
                                    20, None)
    for name in far:
        for at in (new - size[name] + 4, new, new + 236):
            assert call(dict(far, **{name: at})) == -1 and b"share memory" in lib.wf_last_error(None), (name, at)
        for at in (new - size[name], new + 240):      # side by side: refused for another reason, a bad page size, alone
            assert call(dict(far, **{name: at}), 0) == -1 and b"page_tokens" in lib.wf_last_error(None), (name, at)


def test_cache4_refusals():
    binding, lib = _lib()

    def cache(**kw):
        f = dict(data=P, entries=3, n_head=2, n_frames=100)
        f.update(kw)
        return ctypes.byref(binding.WfKv4(f["data"], f["entries"], f["n_head"], f["n_frames"]))
    bad_caches = [(None, -1), (cache(data=None), -1), (cache(data=P + 8), -1), (cache(entries=0), -1), (cache(n_head=0), -1),
                  (cache(n_frames=0), -1), (cache(n_frames=(1 << 20) + 1), -1)]
    ranges = dict(slot0=[(-1, -1), (3, -1), (2, -1)], n=[(0, -1), (4, -1)])
    strides = [(None, -1), (S3(-1, 0, 0), -1), (S3(0, 1 << 41, 0), -1)]

    def store(lib, a):
        return lib.wf_kv4_store(a["c"], a["slot0"], a["n"], a["k"], a["ks"], a["v"], a["vs"], a["dtype"], a["lens"], None)
    varied(store, dict(c=cache(), slot0=0, n=2, k=P, ks=S3(12800, 128, 64), v=P, vs=S3(12800, 128, 64), dtype=0, lens=None),
           dict(c=bad_caches, k=[(None, -1), (P + 2, -1)], v=[(None, -1)], ks=strides, vs=strides, dtype=[(2, -1), (7, -1)],
                lens=[(P + 2, -1)], **ranges))

    def load(lib, a):
        return lib.wf_kv4_load(a["c"], a["slot0"], a["n"], a["k"], a["v"], a["dtype"], None)
    varied(load, dict(c=cache(), slot0=0, n=2, k=P, v=P, dtype=1),
           dict(c=bad_caches, k=[(None, -1), (P + 4, -1)], v=[(None, -1)], dtype=[(-1, -1)], **ranges))

    def attend(lib, a):
        return lib.wf_kv4_attend(a["c"], a["slot0"], a["n"], a["q"], a["qs"], a["rows"], a["dtype"], a["lens"], a["out"], a["ws"],
                                 a["bytes"], None)
    long = cache(n_frames=100000)
    varied(attend, dict(c=long, slot0=0, n=2, q=P, qs=S3(128, 128, 64), rows=1, dtype=0, lens=None, out=P, ws=P, bytes=1 << 30),
           dict(c=bad_caches, q=[(None, -1), (P + 3, -1)], qs=strides, rows=[(0, -1), ((1 << 19) + 1, -1)], dtype=[(2, -1)],
                lens=[(P + 1, -1)], out=[(None, -1), (P + 8, -1)], ws=[(None, -1), (P + 64, -1)], bytes=[(0, -3)], **ranges))
    n = ctypes.c_size_t()
    assert lib.wf_kv4_bytes(3, 2, 100, ctypes.byref(n)) == 0 and n.value == 3 * 2 * 4 * 2176
    assert lib.wf_kv4_bytes(3, 2, 100, None) == -1
    assert lib.wf_kv4_attend_workspace_bytes(long, 2, 1, ctypes.byref(n)) == 0 and n.value > 0
    assert lib.wf_kv4_attend_workspace_bytes(cache(), 2, 1, ctypes.byref(n)) == 0 and n.value == 0
    assert lib.wf_kv4_attend_workspace_bytes(cache(), 2, 1, None) == -1


def test_binding_refuses_tensors_of_another_kind():
    """Before the library is asked: CPU tensors, types, shapes."""
    import paper_2609_32869_amd as wf
    x = torch.zeros((1, 2, 8))
    with pytest.raises(wf.WfError, match="on the GPU"):
        wf.beam_select(x, torch.zeros((1, 2)), 2)
    with pytest.raises(wf.WfError, match="must be a tensor"):
        wf.beam_select(None, torch.zeros((1, 2)), 2)
    i = torch.zeros((1, 2, 4), dtype=torch.int32)
    with pytest.raises(wf.WfError, match="on the GPU"):
        wf.cache_reorder(torch.zeros((1, 8, 16)), i, i[0, :1], i[0, 0, :1], i[0])


def test_results_without_a_backward_pass():
    """A result whose input requires a gradient is the same tensor, may be changed in place, and raises when a gradient is
    asked of it; others, and all without autograd, are left alone."""
    import paper_2609_32869_amd as wf
    from paper_2609_32869_amd.operators import _without_backward
    q, other = torch.ones(3, requires_grad=True), torch.ones(3, requires_grad=True)
    for make in (lambda: torch.arange(3.0),
                 lambda: torch.empty(0).set_(torch.arange(6.0).untyped_storage(), 0, (3,), (1,))):
        out = make()
        got = _without_backward("attend", out, q)
        assert got.data_ptr() == out.data_ptr() and torch.equal(got.detach(), torch.arange(3.0))
        got += 1
        with pytest.raises(wf.WfError, match="attend has no backward pass"):
            (got * other).sum().backward()
        assert q.grad is None
        plain_out = make()
        assert _without_backward("attend", plain_out, q.detach()) is plain_out
        with torch.no_grad():
            assert _without_backward("attend", plain_out, q) is plain_out
        assert not plain_out.requires_grad


def test_import_without_private_names_of_torch():
    """The package imports where PyTorch lacks the shortcuts, and takes the stream and device by the public calls."""
    code = ("import torch\n"
            "for name in ('_cuda_getCurrentRawStream', '_cuda_getDevice'):\n"
            "    if hasattr(torch._C, name): delattr(torch._C, name)\n"
            "import paper_2609_32869_amd as wf\n"
            "from paper_2609_32869_amd import operators\n"
            "torch.cuda.current_stream = lambda index: type('S', (), {'cuda_stream': 70 + index})()\n"
            "assert operators._raw_stream(3) == 73 and operators._device is torch.cuda.current_device\n")
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    subprocess.run([sys.executable, "-c", code], cwd=root, check=True, timeout=300)


def test_binding_refuses_sizes_past_32_bits():
    """What a C int would cut off to a size that is allowed."""
    import paper_2609_32869_amd as wf
    from paper_2609_32869_amd import operators
    for sizes in ((1, 5, 2 ** 32 + 100, 5), (1, 5, 100, 2 ** 32 + 5), (2 ** 32 + 1, 5, 100, 5), (1, 2 ** 32 + 5, 100, 5)):
        with pytest.raises(wf.WfError, match="out of range"):
            operators._select_bytes(*sizes)
    for sizes in ((2 ** 32 + 1, 2, 100), (1, 2 ** 32 + 2, 100), (1, 2, 2 ** 32 + 100)):
        with pytest.raises(wf.WfError, match="out of range"):
            wf.AcousticCache4(*sizes)


class Search:
    """A handle's beam calls without a library: which were made."""

    def __new__(cls, n=2, beams=3):
        from paper_2609_32869_amd import WhisperFlash
        eng = WhisperFlash.__new__(WhisperFlash)
        eng.searches, eng.made = {4: (n, beams, torch.empty(8, dtype=torch.uint8))}, []
        eng.lib = type("Lib", (), {"wf_beam_step": lambda *a: eng.made.append("step") or 0})()
        eng.h = None
        return eng


def test_beam_step_refuses_what_it_cannot_write_done_to():
    """n whole int32 of the handle's device: anything else would be written past its end."""
    import paper_2609_32869_amd as wf
    eng = Search()
    good = torch.zeros(2, dtype=torch.int32)
    for done, what in ((good.bool(), "int32"), (good.to(torch.uint8), "int32"), (good.long(), "int32"), (good[:1], "shape"),
                       (torch.zeros(3, dtype=torch.int32), "shape"), (good[None], "shape"), ([0, 0], "tensor"),
                       (torch.zeros(4, dtype=torch.int32)[::2], "contiguous"), (good.to("meta"), "on cpu")):
        with pytest.raises(wf.WfError, match=what):
            eng.beam_step(4, done)
    assert eng.made == []


def test_beam_begin_takes_one_budget_a_request():
    import paper_2609_32869_amd as wf
    last = type("T", (), {"dtype": torch.int32, "dim": lambda s: 1, "is_contiguous": lambda s: True, "is_cuda": True, "shape": (2,)})()
    for budget in ([5], [5, 5, 5], []):
        with pytest.raises(wf.WfError, match="max_new"):
            Search().beam_begin(0, 3, last, budget)


@pytest.mark.parametrize("error", [RuntimeError, KeyboardInterrupt, MemoryError])
def test_beam_search_gives_the_slots_back_on_any_error(error):
    from paper_2609_32869_amd import WhisperFlash
    eng = Search()
    ended = []

    def step(*a, **k):
        raise error("in the middle")
    eng.prefill = lambda *a, **k: None
    eng.beam_begin = lambda *a, **k: None
    eng.beam_step = step
    eng.beam_end = lambda slot0: ended.append(slot0) or (_ for _ in ()).throw(RuntimeError("and so does this"))
    eng.cfg = type("Cfg", (), {"n_ctx": 9})()
    zeros, torch.zeros = torch.zeros, lambda *a, **k: torch.ones(1)
    try:
        with pytest.raises(error, match="in the middle"):
            WhisperFlash.beam_search(eng, 4, torch.ones((1, 3), dtype=torch.int32), [3], [5], 2)
    finally:
        torch.zeros = zeros
    assert ended == [4]


def test_beam_calls_on_a_null_handle():
    binding, lib = _lib()
    n = ctypes.c_size_t()
    assert lib.wf_beam_bytes(None, 1, 1, ctypes.byref(n)) == -1
    assert lib.wf_beam_begin(None, 0, 1, 1, P, None, 1.0, P, 1 << 30, None) == -1
    assert lib.wf_beam_step(None, 0, None, 0, None) == -1
    assert lib.wf_beam_end(None, 0, P, 1, P, P, None) == -1


def test_kv4_configurations():
    binding, lib = _lib()
    from wf_fixtures import LARGE_V3, MICRO
    sizes = {}
    for bits in (16, 4):
        n = ctypes.c_size_t()
        assert lib.wf_workspace_bytes(ctypes.byref(binding.make_config(LARGE_V3, 96, bits)), ctypes.byref(n)) == 0
        sizes[bits] = n.value
    # 34 blocks of 20 heads: 47 groups of 2176 bytes against 1500 + 1536 frames of 128, and one block of all slots in transit
    per = 34 * 20 * ((1500 + 1536) * 128 - 47 * 2176)
    transit = 96 * 20 * (1500 + 1536) * 128
    assert abs((sizes[16] - sizes[4]) - (96 * per - transit)) < 1 << 20
    with pytest.raises(binding.WfError):
        binding.make_config(MICRO, 1, 4)      # fp32 storage
    with pytest.raises(binding.WfError):
        binding.make_config(LARGE_V3, 1, 8)


# ---------------------------------------------------------------- pins of the plain forms

def test_plain_quantise():
    """Representable values come back; every value goes to a nearest one, ties to the even code; blocks are apart."""
    rng = np.random.default_rng(0)
    grid = np.concatenate([plain.GRID, -plain.GRID])
    x = rng.choice(grid, (5, 64)) * 0.25
    x[:, 0] = x[:, 32] = 1.5                              # 6 * 0.25: the scale is that one
    assert np.array_equal(plain.quantise(x, 1), x)
    x = rng.standard_normal((7, 96))
    q = plain.quantise(x, 1)
    for b in range(3):
        blk, out = x[:, 32 * b:32 * b + 32], q[:, 32 * b:32 * b + 32]
        for r in range(7):
            s = min(2.0 ** e for e in range(-10, 10) if np.abs(blk[r]).max() <= 6 * 2.0 ** e)
            assert np.allclose(np.abs(out[r] - blk[r]), np.abs(blk[r][:, None] - s * grid).min(-1), atol=1e-12)
    ties = np.zeros(32)
    ties[:8] = [6, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5]
    assert plain.quantise(ties, 0)[:8].tolist() == [6, 0, 1, 1, 2, 2, 4, 4]
    ties[9] = np.nan
    assert np.isnan(plain.quantise(ties, 0)).all()


def test_plain_select_against_every_candidate():
    rng = np.random.default_rng(1)
    x, s = rng.standard_normal((3, 4, 11)), -rng.random((3, 4))
    score, beam, tok = plain.beam_select(x, s, 44)
    for r in range(3):
        p = np.exp(x[r]) / np.exp(x[r]).sum(-1, keepdims=True)
        every = s[r][:, None] + np.log(p)
        assert sorted(zip(beam[r], tok[r])) == list(itertools.product(range(4), range(11)))
        assert np.allclose(score[r], every[beam[r], tok[r]]) and (np.diff(score[r]) <= 0).all()


def test_plain_reorder_keeps_what_beams_read():
    """Any choice: what a beam reads through its new table is what its parent read, and the next position's page is its own."""
    rng = np.random.default_rng(2)
    n, B, P, T = 2, 4, 5, 3
    cache = np.arange(n * B * P * T).reshape(-1, T)
    pool = rng.permutation(n * B * P).reshape(n, B * P)
    for L in range(P * T + 1):
        used = -(-L // T)
        tables = np.repeat(pool[:, :1], B * P, 1).reshape(n, B, P).copy()
        tables[:, :, :used] = pool[:, :B * used].reshape(n, B, used)
        parents = rng.integers(0, B, (n, B))
        new, copies = plain.cache_reorder(tables, parents, [L] * n, pool, T)
        after = cache.copy()
        for req in copies:
            for s, d in req:
                after[d] = cache[s]
        for r in range(n):
            for j in range(B):
                was = [cache[tables[r, parents[r, j], p // T], p % T] for p in range(L)]
                assert [after[new[r, j, p // T], p % T] for p in range(L)] == was
            if L < P * T:
                own = new[r, :, L // T]
                assert len(set(own)) == B
                others = [page for j in range(B) for page in new[r, j, :L // T]]
                assert not set(own) & set(others)


def test_plain_attend_against_a_library():
    rng = np.random.default_rng(3)
    q, k, v = rng.standard_normal((2, 3, 2, 64)), rng.standard_normal((2, 9, 2, 64)), rng.standard_normal((2, 9, 2, 64))
    got = plain.attend(q, k, v, [9, 4])
    for r, m in ((0, 9), (1, 4)):
        t = [torch.from_numpy(a).permute(1, 0, 2) for a in (q[r], k[r, :m], v[r, :m])]
        want = torch.nn.functional.scaled_dot_product_attention(*t).permute(1, 0, 2).numpy()
        assert np.abs(got[r] - want).max() < 1e-12


def test_plain_beam_search_with_every_beam_is_exhaustive():
    """64 beams of a 64-token vocabulary, two steps: the best pair of tokens is found, and one beam is greedy."""
    cfg = VOCAB64
    T = Target(cfg, make_weights(cfg).values, OracleOpts(dtype=np.float64))
    xkv, prompt = T.cross_kv(make_memory(cfg, 0)), list(make_prefix(cfg, 0, 5))

    def logp(tokens):
        x = last_logits(T, xkv, tokens)
        return x - x.max() - np.log(np.exp(x - x.max()).sum())
    first = logp(prompt)
    pairs = {(a, b): first[a] + p for a in range(64) for b, p in enumerate(logp(prompt + [a]))}
    want = sorted(pairs, key=lambda t: -pairs[t])[:64]
    got = beam_search(T, xkv, prompt, 2, 64, 0.0)
    assert [tuple(h[0]) for h in got] == want
    greedy = list(prompt)
    for _ in range(6):
        greedy.append(int(np.argmax(last_logits(T, xkv, greedy))))
    assert beam_search(T, xkv, prompt, 6, 1)[0][0] == greedy[5:]
