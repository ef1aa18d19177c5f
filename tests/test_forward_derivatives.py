"""Forward-mode derivatives of the operators without a handle: the rotation has them, the others refuse tangents."""
import pytest
import torch
from torch.autograd import forward_ad


class Turner:
    """A stand-in for Rotary on the CPU: pairs (i, i + width / 2) turned by the position, and a record of the calls."""

    def __init__(self):
        self.calls = []

    def _turn(self, positions, tensors, transposed, in_place, stream):
        self.calls.append((transposed, in_place, stream))
        assert all(t.stride(-1) == 1 for t in tensors)
        c, s = (f(positions.to(tensors[0].dtype))[:, None, None] for f in (torch.cos, torch.sin))
        s = -s if transposed else s
        out = []
        for t in tensors:
            a, b = t.detach().chunk(2, -1)
            out.append(torch.cat((a * c - b * s, b * c + a * s), -1))
        return tuple(out)


def test_rotation_of_tangents():
    """The tangent of a rotation is the tangent rotated; an input without one has none; reverse over forward mode goes on."""
    from paper_2609_32869_amd.operators import _Rotate
    f, at = Turner(), torch.tensor([0, 1, 5], dtype=torch.int32)
    q, k, t = (torch.randn((3, 2, 4), dtype=torch.float64) for _ in range(3))
    with forward_ad.dual_level():
        dual = forward_ad.make_dual(q, t.permute(2, 1, 0).contiguous().permute(2, 1, 0))   # a tangent of other strides
        y, z = _Rotate.apply(f, at, False, None, dual, k)
        y, dy = forward_ad.unpack_dual(y)
        z, dz = forward_ad.unpack_dual(z)
        assert torch.equal(y, f._turn(at, (q,), False, False, None)[0]) and torch.equal(z, f._turn(at, (k,), False, False, None)[0])
        assert torch.equal(dy, f._turn(at, (t,), False, False, None)[0]) and not dz.any()
        w = t.clone().requires_grad_()
        _, dy = forward_ad.unpack_dual(_Rotate.apply(f, at, True, None, forward_ad.make_dual(q, w))[0])
        (g,) = torch.autograd.grad(dy, w, t)
        assert torch.equal(g, f._turn(at, (t,), False, False, None)[0])     # the transpose of the transposed rotation


def test_tangents_are_found_and_refused():
    from paper_2609_32869_amd import WfError
    from paper_2609_32869_amd.operators import _dual, _refuse_tangents
    q = torch.ones(3)
    _refuse_tangents("attend", q, None)
    with forward_ad.dual_level():
        d = forward_ad.make_dual(q, q)
        assert _dual(None, q, d) and not _dual(None, q)
        _refuse_tangents("attend", q, None)
        with pytest.raises(WfError, match="attend has no forward-mode derivative"):
            _refuse_tangents("attend", q, d)
    assert not _dual(q)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("own_stream", [False, True])
def test_rotary_tangents(dtype, own_stream):
    """The tangent of q's rotation is the rotation of its tangent, bit for bit (the operator is linear); k has none."""
    import paper_2609_32869_amd as wf
    g = torch.Generator("cuda").manual_seed(0)
    rot, at = wf.Rotary(48, interleaved=True), torch.tensor([3, 0, 77777], dtype=torch.int32, device="cuda")
    q, t, k = (torch.randn((3, h, 64), device="cuda", generator=g).to(dtype) for h in (4, 4, 2))
    stream = torch.cuda.Stream() if own_stream else None
    torch.cuda.synchronize()
    want, wk = rot.rotate(at, q, k)
    for tangent in (t, torch.empty((64, 4, 3), dtype=dtype, device="cuda").permute(2, 1, 0).copy_(t)):
        torch.cuda.synchronize()
        for context in (torch.enable_grad, torch.no_grad):
            with context(), forward_ad.dual_level():
                a, b = rot.rotate(at, forward_ad.make_dual(q, tangent), k, stream=stream)
                a, da = forward_ad.unpack_dual(a)
                b, db = forward_ad.unpack_dual(b)
            torch.cuda.synchronize()
            assert torch.equal(a, want) and torch.equal(b, wk)
            assert torch.equal(da, rot.rotate(at, t)) and (db is None or not db.any())
    with forward_ad.dual_level():
        assert forward_ad.unpack_dual(rot.rotate(at, q)).tangent is None
        with pytest.raises(wf.WfError, match="tangents are not changed in place"):
            rot.rotate(at, q, forward_ad.make_dual(k, k), in_place=True)


@pytest.mark.gpu
def test_operators_refuse_tangents():
    import paper_2609_32869_amd as wf
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    q, k = torch.randn((4, 2, 64), device="cuda"), torch.randn((4, 2, 64), device="cuda")
    starts, tables, at = i32([0, 4]), i32([[0, 1]]), i32([0])
    paged, acoustic = wf.PagedCache8(2, 2), wf.AcousticCache4(1, 2, 20)
    paged.store(k, k, tables, at, starts=starts)
    memory = torch.randn((1, 20, 2, 64), device="cuda")
    acoustic.store(0, memory, memory)
    logits, scores = torch.randn((1, 2, 50), device="cuda"), torch.zeros((1, 2), device="cuda")
    with forward_ad.dual_level():
        def dual(t):
            return forward_ad.make_dual(t, torch.ones_like(t))
        for name, call in (("prompt_attention", lambda: wf.prompt_attention(dual(q), k, k, starts)), ("prompt_attention", lambda: wf.prompt_attention(q, dual(k), k, starts)),
                           ("prompt_attention", lambda: wf.prompt_attention(q, k, dual(k), starts)),
                           ("prompt_attention", lambda: wf.prompt_attention(q, k, k, starts, out=dual(torch.empty_like(q)))),
                           ("attend", lambda: paged.attend(dual(q[None]), tables, at)), ("attend", lambda: acoustic.attend(0, dual(q[None]))),
                           ("beam_select", lambda: wf.beam_select(dual(logits), scores, 3)), ("beam_select", lambda: wf.beam_select(logits, dual(scores), 3))):
            with pytest.raises(wf.WfError, match=f"{name} has no forward-mode derivative"):
                call()
        assert torch.isfinite(wf.prompt_attention(q, k, k, starts)).all() and torch.isfinite(paged.attend(q[None], tables, at)).all()
        assert torch.isfinite(acoustic.attend(0, q[None])).all() and len(wf.beam_select(logits, scores, 3)) == 3
