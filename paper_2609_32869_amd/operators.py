"""Operators without a handle (include/wf.h): beam selection, page-table reordering,
acoustic keys and values held in 4 bits, and a decoder's self-attention: rotary positions,
attention over packed prompts and a paged cache in 8 bits.

Argument marshalling as in ``binding``: shapes, types and devices are checked here, sizes
and ranges by the library.  Every call enqueues on ``stream`` (default: the current stream
of the tensors' device) and returns without waiting; a given stream has to be ordered
behind the work that fills the tensors.  Workspaces and results come from PyTorch's
allocator for the call's stream, so concurrent calls and captured graphs each have their
own.

Rotary positions have a backward pass and forward-mode derivatives, the others neither: their
results of inputs that require gradients raise where a gradient is asked of them, and inputs with
a tangent are refused; what a cache stores or copies has no history.
"""
import ctypes
import functools

import torch
from torch.autograd import forward_ad

from .binding import WF_BF16, WF_F32, WfError, WfKv4, WfKv8, _refuse, _tensor, load_library

try:  # torch.cuda.current_stream() and current_device() without their objects and checks (2.7 and 0.1 us)
    from torch._C import _cuda_getCurrentRawStream as _raw_stream, _cuda_getDevice as _device
except ImportError:  # a PyTorch without these names
    from torch.cuda import current_device as _device

    def _raw_stream(index):
        return torch.cuda.current_stream(index).cuda_stream

_DTYPES = {torch.float32: WF_F32, torch.bfloat16: WF_BF16}
_F32, _I32, _U8 = torch.float32, torch.int32, torch.uint8


def _check(rc):
    if rc != 0:
        lib = load_library()
        msg = lib.wf_last_error(None)
        raise WfError(f"{lib.wf_strerror(rc).decode()} ({rc}): {msg.decode() if msg else ''}")


_INTS = 2 ** 31  # sizes from here on would be cut off by the C entries' 32 bits; smaller ones are the library's to check


def _gpu(t, name, dims):
    """The device of a GPU tensor of `dims` axes."""
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        _refuse(f"{name} must be a tensor on the GPU")
    if t.dim() != dims:
        _refuse(f"{name} must have {dims} axes, not {t.dim()}")
    return t.device


def _type(t, name):
    code = _DTYPES.get(t.dtype)
    if code is None:
        _refuse(f"{name} must be float32 or bfloat16, not {str(t.dtype)[6:]}")
    return code


def _enqueue(device, stream, call, *tensors):
    """call(raw stream, empty) with `device` current; empty: as torch.empty.  With a given stream the call's tensors are
    freed only behind the work that it has for them, and empty takes memory of that stream: memory of the current one
    may still be in use there, by work that the given stream is not ordered behind."""
    index = device.index
    if stream is None:
        raw, empty = _raw_stream(index), torch.empty
    else:
        if stream.device != device:
            _refuse("stream is of another device than the tensors")
        raw = stream.cuda_stream
        for t in tensors:
            if t is not None:
                t.record_stream(stream)

        current = torch.cuda.current_stream(device)

        def empty(shape, dtype, device):
            with torch.cuda.stream(stream):
                t = torch.empty(shape, dtype=dtype, device=device)
            t.record_stream(current)
            return t
    if _device() == index:
        return call(raw, empty)
    with torch.cuda.device(index):
        return call(raw, empty)


def _like(t, empty):
    """A contiguous result of t's shape, type and device, of call's `empty`: torch's own way (1.0 us of the host, torch.empty 2.1)
    where that is the current stream's."""
    if empty is torch.empty:
        return torch.empty_like(t, memory_format=torch.contiguous_format)
    return empty(t.shape, dtype=t.dtype, device=t.device)


class _NoBackward(torch.autograd.Function):
    """A result, as a function of the tensors that it came from."""

    @staticmethod
    def forward(ctx, name, result, *tensors):
        ctx.name = name
        return result.t

    @staticmethod
    def backward(ctx, *grads):
        raise WfError(f"{ctx.name} has no backward pass")


class _Held:
    """Keeps a result out of the function's inputs: what it returns is the tensor itself."""

    def __init__(self, t):
        self.t = t


def _without_backward(name, result, *tensors):
    """`result`, a tensor of its own memory, which raises on backward() where one of `tensors` wants a gradient."""
    if torch.is_grad_enabled() and any(t.requires_grad for t in tensors):
        return _NoBackward.apply(name, _Held(result), *tensors)
    return result


def _dual(*tensors):
    """Whether one of the call's tensors has a forward-mode tangent.  Outside of forward_ad's levels none has: looked at first
    (0.06 us of the host, a tensor's tangent 0.3)."""
    if getattr(forward_ad, "_current_level", 0) < 0:
        return False
    return any(isinstance(t, torch.Tensor) and forward_ad.unpack_dual(t).tangent is not None for t in tensors)


def _refuse_tangents(name, *tensors):
    if _dual(*tensors):
        _refuse(f"{name} has no forward-mode derivative")


@functools.lru_cache(maxsize=256)
def _select_bytes(n, beams, vocab, k):
    if max(n, beams, vocab, abs(k)) >= _INTS:
        _refuse("a size is out of range")
    nbytes = ctypes.c_size_t()
    _check(load_library().wf_beam_select_workspace_bytes(n, beams, vocab, k, ctypes.byref(nbytes)))
    return nbytes.value


def beam_select(logits, scores, k, suppress=None, stream=None):
    """The k best continuations of each request's beams: wf_beam_select.

    logits: fp32 or bf16 [n, beams, vocab], the last axis contiguous; scores: fp32 [n, beams];
    suppress: uint8 [vocab] or None.  Returns (score fp32, beam int32, token int32), each [n, k].
    """
    lib = load_library()
    _refuse_tangents("beam_select", logits, scores)
    dev = _gpu(logits, "logits", 3)
    dtype = _type(logits, "logits")
    n, beams, vocab = logits.shape
    sr, sb, sv = logits.stride()
    if vocab > 1 and sv != 1:
        _refuse("logits must be contiguous along the vocabulary")
    _tensor(scores, "scores", _F32, (n, beams), dev)
    if suppress is not None:
        _tensor(suppress, "suppress", _U8, (vocab,), dev)
    k = int(k)
    nbytes = _select_bytes(n, beams, vocab, k)

    def call(raw, empty):
        out = empty((3, n, k), dtype=_I32, device=dev)
        ws = empty(nbytes, dtype=_U8, device=dev)
        p, step = out.data_ptr(), 4 * n * k
        _check(lib.wf_beam_select(logits.data_ptr(), dtype, sr, sb, scores.data_ptr(),
                                  None if suppress is None else suppress.data_ptr(), n, beams, vocab, k, p, p + step,
                                  p + 2 * step, ws.data_ptr(), nbytes, raw))
        return out

    score, beam, token = _enqueue(dev, stream, call, logits, scores, suppress).unbind()
    score = score.view(_F32)
    if logits.requires_grad or scores.requires_grad:  # not as a view, which autograd would not let change in place
        own = torch.empty(0, dtype=_F32, device=dev).set_(score.untyped_storage(), score.storage_offset(), score.shape, score.stride())
        score = _without_backward("beam_select", own, logits, scores)
    return score, beam, token


def cache_reorder(cache, tables, parents, lens, pool, page_tokens=16, stream=None):
    """Page tables (and page copies, in place) after a choice of beams: wf_cache_reorder.

    cache: [regions, pages, ...] contiguous, pages of a multiple of 16 bytes; tables: int32
    [n, beams, max_pages]; parents: int32 [n, beams]; lens: int32 [n]; pool: int32 [n, pool_pages].
    Returns the new tables.
    """
    lib = load_library()
    if not isinstance(cache, torch.Tensor) or not cache.is_cuda or cache.dim() < 3 or not cache.is_contiguous():
        _refuse("cache must be a contiguous tensor [regions, pages, ...] on the GPU")
    dev = _gpu(tables, "tables", 3)
    n, beams, max_pages = tables.shape
    if dev != cache.device:
        _refuse("tables must be on the cache's device")
    _gpu(pool, "pool", 2)
    pool_pages = pool.shape[1]
    _tensor(tables, "tables", _I32, (n, beams, max_pages), dev)
    _tensor(parents, "parents", _I32, (n, beams), dev)
    _tensor(lens, "lens", _I32, (n,), dev)
    _tensor(pool, "pool", _I32, (n, pool_pages), dev)
    regions, pages = cache.shape[:2]
    if regions == 0 or pages == 0:
        _refuse("cache must hold a page")
    page_tokens = int(page_tokens)
    if max(n, beams, max_pages, regions, pages, pool_pages, abs(page_tokens)) >= _INTS:
        _refuse("a size is out of range")
    region = cache.numel() // regions * cache.element_size()

    def call(raw, empty):
        new = empty((n, beams, max_pages), dtype=_I32, device=dev)
        _check(lib.wf_cache_reorder(cache.data_ptr(), regions, region, pages, region // pages, tables.data_ptr(), new.data_ptr(),
                                    n, beams, max_pages, page_tokens, parents.data_ptr(), lens.data_ptr(),
                                    pool.data_ptr(), pool_pages, raw))
        return new

    return _enqueue(dev, stream, call, cache, tables, parents, lens, pool)


_Strides = ctypes.c_int64 * 3


class AcousticCache4:
    """Keys and values of `entries` acoustic memories in 4 bits (wf_kv4): n_frames frames of n_head heads of 64."""

    def __init__(self, entries, n_head, n_frames, device="cuda"):
        self.lib = load_library()
        self.entries, self.n_head, self.n_frames = int(entries), int(n_head), int(n_frames)
        if max(abs(self.entries), abs(self.n_head), abs(self.n_frames)) >= _INTS:
            _refuse("a size is out of range")
        nbytes = ctypes.c_size_t()
        _check(self.lib.wf_kv4_bytes(self.entries, self.n_head, self.n_frames, ctypes.byref(nbytes)))
        self.data = torch.empty(nbytes.value, dtype=_U8, device=device)
        if not self.data.is_cuda:
            _refuse("device must be a GPU")
        self.device = self.data.device
        self._c = WfKv4(self.data.data_ptr(), self.entries, self.n_head, self.n_frames)
        self._ref = ctypes.byref(self._c)
        self._spaces = {}  # workspace bytes of (n, rows)

    def _lens(self, lens, n):
        if lens is None:
            return None
        _tensor(lens, "lens", _I32, (n,), self.device)
        return lens.data_ptr()

    def _rows(self, t, name, axis1):
        """Type and strides of [n, axis1 (None: any), n_head, 64] with the last axis contiguous."""
        if _gpu(t, name, 4) != self.device:
            _refuse(f"{name} must be on {self.device}, not {t.device}")
        shape = t.shape
        if shape[2] != self.n_head or shape[3] != 64 or (axis1 is not None and shape[1] != axis1):
            _refuse(f"{name} must have shape (n, {'rows' if axis1 is None else axis1}, {self.n_head}, 64), not {tuple(shape)}")
        s = t.stride()
        if s[3] != 1:
            _refuse(f"{name} must be contiguous along its last axis")
        return _type(t, name), _Strides(*s[:3])

    def store(self, slot0, k, v, lens=None, stream=None):
        """Entries slot0 .. from k, v: fp32 or bf16 [n, n_frames, n_head, 64] (any strides but the last), of which the
        first lens[r] frames (int32 [n], None: all) are given and the others hold zeros."""
        dtype, ks = self._rows(k, "k", self.n_frames)
        vtype, vs = self._rows(v, "v", self.n_frames)
        n = k.shape[0]
        if vtype != dtype or v.shape[0] != n:
            _refuse("v must have k's type and shape")
        if not 0 <= slot0 <= self.entries - n:
            _refuse("entries out of range")
        plens = self._lens(lens, n)
        _enqueue(self.device, stream, lambda raw, empty: _check(self.lib.wf_kv4_store(
            self._ref, int(slot0), n, k.data_ptr(), ks, v.data_ptr(), vs, dtype, plens, raw)), k, v, lens, self.data)

    def load(self, slot0, n, dtype=torch.float32, stream=None):
        """The keys and values that entries slot0 .. slot0 + n - 1 hold: two tensors [n, n_frames, n_head, 64]."""
        if dtype not in _DTYPES:
            _refuse("dtype must be float32 or bfloat16")
        if not (0 < n <= self.entries and 0 <= slot0 <= self.entries - n):
            _refuse("entries out of range")

        def call(raw, empty):
            k = empty((n, self.n_frames, self.n_head, 64), dtype=dtype, device=self.device)
            v = empty((n, self.n_frames, self.n_head, 64), dtype=dtype, device=self.device)
            _check(self.lib.wf_kv4_load(self._ref, int(slot0), n, k.data_ptr(), v.data_ptr(), _DTYPES[dtype], raw))
            return k, v

        return _enqueue(self.device, stream, call, self.data)

    def attend(self, slot0, q, lens=None, stream=None):
        """softmax(q k^T / 8) v of q (fp32 or bf16 [n, rows, n_head, 64], any strides but the last) over the first lens[r]
        frames (int32 [n], None: all) of entries slot0 ..: [n, rows, n_head, 64] in q's type."""
        _refuse_tangents("attend", q)
        dtype, qs = self._rows(q, "q", None)
        n, rows = q.shape[:2]
        if not 0 <= slot0 <= self.entries - n:
            _refuse("entries out of range")
        need = self._spaces.get((n, rows))
        if need is None:
            if rows >= _INTS:
                _refuse("rows out of range")
            nbytes = ctypes.c_size_t()
            _check(self.lib.wf_kv4_attend_workspace_bytes(self._ref, n, rows, ctypes.byref(nbytes)))
            need = self._spaces[n, rows] = nbytes.value
        plens = self._lens(lens, n)

        def call(raw, empty):
            out = empty((n, rows, self.n_head, 64), dtype=q.dtype, device=self.device)
            ws = empty(need, dtype=_U8, device=self.device) if need else None
            _check(self.lib.wf_kv4_attend(self._ref, int(slot0), n, q.data_ptr(), qs, rows, dtype, plens, out.data_ptr(),
                                          ws.data_ptr() if need else None, need, raw))
            return out

        out = _enqueue(self.device, stream, call, q, lens, self.data)
        return _without_backward("attend", out, q) if q.requires_grad else out


_Strides2 = ctypes.c_int64 * 2
_SCALINGS = {None: 0, "linear": 1, "base": 2, "ramp": 3}


class _Layouts(dict):
    """What the checks of a call's tensors found, by the tensors' layouts: a call with layouts that were checked before
    goes without (one token's rotation 5 us less of the host).  At most 1,024."""

    @staticmethod
    def of(*tensors):
        """A key, or None where an argument is not a tensor (which the checks refuse)."""
        try:
            return tuple([None if t is None else (t.shape, t.stride(), t.dtype, t.get_device()) for t in tensors])
        except (AttributeError, RuntimeError):
            return None

    def keep(self, key, found):
        if len(self) >= 1024:
            self.clear()
        self[key] = found
        return found


def _heads(t, name, axes, width=64):
    """Device, type and strides of [..., heads, width] of `axes` axes, the last one contiguous."""
    dev = _gpu(t, name, axes)
    if width is not None and t.shape[-1] != width:
        _refuse(f"{name} must have a last axis of {width}, not {t.shape[-1]}")
    s = t.stride()
    if s[-1] != 1 and t.shape[-1] > 1:
        _refuse(f"{name} must be contiguous along its last axis")
    if max(t.shape) >= _INTS:
        _refuse("a size is out of range")
    return dev, _type(t, name), s[:-1]


def _vector(t, name, n, device):
    if not isinstance(t, torch.Tensor):
        _refuse(f"{name} must be a tensor")
    _tensor(t, name, _I32, (n,), device)


def _changed(t):
    """Counts the change of a tensor that a kernel wrote, as autograd's own operations do."""
    if not t.is_inference():
        torch.autograd.graph.increment_version(t)


class _Rotate(torch.autograd.Function):
    """Rotated tensors as a function of them; the gradient turns the other way, a tangent the same."""

    @staticmethod
    def forward(ctx, rotary, positions, transposed, stream, *tensors):
        ctx.rotary, ctx.transposed, ctx.stream = rotary, transposed, stream
        ctx.save_for_backward(positions)
        ctx.save_for_forward(positions)
        return rotary._turn(positions, tensors, transposed, False, stream)

    @staticmethod
    def jvp(ctx, *tangents):
        (positions,) = ctx.saved_tensors
        if ctx.stream is not None:  # as the results; an input without a tangent comes with zeros that the current stream has just made
            ctx.stream.wait_stream(torch.cuda.current_stream(ctx.stream.device))
        with torch.cuda.stream(ctx.stream):
            rows = [t if t.stride(-1) == 1 or t.shape[-1] == 1 else t.contiguous() for t in tangents[4:]]
        return _Rotate.apply(ctx.rotary, positions, ctx.transposed, ctx.stream, *rows)

    @staticmethod
    def backward(ctx, *grads):
        (positions,) = ctx.saved_tensors
        need = [i for i in range(len(grads)) if ctx.needs_input_grad[4 + i]]
        rows = [g if g.stride(-1) == 1 or g.shape[-1] == 1 else g.contiguous() for g in (grads[i] for i in need)]
        out = [None] * len(grads)
        for i, t in zip(need, _Rotate.apply(ctx.rotary, positions, not ctx.transposed, None, *rows)):
            out[i] = t
        return (None, None, None, None, *out)


class Rotary:
    """Rotary positions of heads' first `dims` elements (wf_rotary): pairs (i, i + dims / 2) or, interleaved,
    (2 i, 2 i + 1).  scaling for long contexts: None, "linear" or "base" by `factor`, or "ramp" (by parts, from pairs
    that turn `low` times within `context` positions to those that turn `high` times): wf_rotary_turns."""

    def __init__(self, dims, base=10000.0, interleaved=False, scaling=None, factor=1.0, context=0, low=1.0, high=32.0, device="cuda"):
        self.lib = load_library()
        self.dims, self.interleaved = int(dims), bool(interleaved)
        if abs(self.dims) >= _INTS:
            _refuse("a size is out of range")
        if scaling not in _SCALINGS:
            _refuse("scaling must be None, 'linear', 'base' or 'ramp'")
        turns = (ctypes.c_double * (max(2, min(self.dims, 4096)) // 2))()
        amplitude = ctypes.c_float()
        _check(self.lib.wf_rotary_turns(self.dims, base, _SCALINGS[scaling], factor, context, low, high, turns, ctypes.byref(amplitude)))
        self.amplitude = amplitude.value
        self.turns = torch.tensor(list(turns), dtype=torch.float64, device=device)
        if not self.turns.is_cuda:
            _refuse("device must be a GPU")
        self.device = self.turns.device
        self._plans = _Layouts()

    def rotate(self, positions, q, k=None, in_place=False, stream=None):
        """q, and k beside it, at their positions: q, k fp32 or bf16 [tokens, heads, width] of the same tokens, width and
        type (any strides but the last); positions int32 [tokens].  Returns new tensors, or the given ones changed in place
        (without gradients and tangents): the rotated q, or (q, k)."""
        tensors = (q,) if k is None else (q, k)
        dual = _dual(q, k)
        if dual or torch.is_grad_enabled() and (isinstance(q, torch.Tensor) and q.requires_grad or isinstance(k, torch.Tensor) and k.requires_grad):
            if in_place:
                _refuse(f"tensors that {'have tangents' if dual else 'require gradients'} are not changed in place")
            out = _Rotate.apply(self, positions, False, stream, *tensors)
        else:
            out = self._turn(positions, tensors, False, in_place, stream)
        return out[0] if k is None else out

    def _plan(self, positions, tensors):
        """Tokens, width, type; for each tensor its strides, its result's and its heads."""
        first, parts = tensors[0], []
        for t, name in zip(tensors, "qk"):
            dev, dtype, s = _heads(t, name, 3, None)
            if dev != self.device:
                _refuse(f"{name} must be on {self.device}, not {dev}")
            if t.shape[0] != first.shape[0] or t.shape[2] != first.shape[2] or t.dtype != first.dtype:
                _refuse("k must have q's tokens, width and type")
            parts.append((_Strides2(*s), _Strides2(t.shape[1] * t.shape[2], t.shape[2]), t.shape[1]))
        _vector(positions, "positions", first.shape[0], self.device)
        return first.shape[0], first.shape[2], dtype, parts

    def _turn(self, positions, tensors, transposed, in_place, stream):
        key = _Layouts.of(positions, *tensors)
        plan = self._plans.get(key) or self._plans.keep(key, self._plan(positions, tensors))
        tokens, width, dtype, parts = plan

        def call(raw, empty):
            q, qs, qo, heads = tensors[0], *parts[0]
            a = q if in_place else _like(q, empty)
            if len(tensors) == 1:
                b, rest, result = None, (None, None, 0, None, None), (a,)
            else:
                k, ks, ko, kv = tensors[1], *parts[1]
                b = k if in_place else _like(k, empty)
                rest, result = (k.data_ptr(), ks, kv, b.data_ptr(), ks if in_place else ko), (a, b)
            if tokens:
                _check(self.lib.wf_rotary(self.turns.data_ptr(), self.dims, self.interleaved, self.amplitude, transposed,
                                          positions.data_ptr(), tokens, width, dtype, q.data_ptr(), qs, heads, a.data_ptr(),
                                          qs if in_place else qo, *rest, raw))
            return result

        result = _enqueue(self.device, stream, call, positions, self.turns, *tensors)
        if in_place:
            for t in tensors:
                _changed(t)
        return result


_prompt_plans = _Layouts()


def _prompt_plan(q, k, v, starts):
    dev, dtype, qs = _heads(q, "q", 3)
    tokens, heads, _ = q.shape
    strides = []
    for t, name in ((k, "k"), (v, "v")):
        d, code, s = _heads(t, name, 3)
        if d != dev or code != dtype or t.shape[0] != tokens or t.shape[1] != k.shape[1]:
            _refuse("k and v must have q's device, type and tokens, and as many heads")
        strides.append(_Strides2(*s))
    if _gpu(starts, "starts", 1) != dev or starts.shape[0] < 2:
        _refuse(f"starts must hold two borders at least, on {dev}")
    n = starts.shape[0] - 1
    _tensor(starts, "starts", _I32, (n + 1,), dev)
    return dev, dtype, tokens, heads, k.shape[1], n, _Strides2(*qs), *strides


def prompt_attention(q, k, v, starts, out=None, stream=None):
    """Causal attention of packed prompts: wf_prompt_attend.

    q: fp32 or bf16 [tokens, n_head, 64]; k, v: [tokens, n_kv_head, 64] in the same type (any strides but the last);
    starts: int32 [n + 1], sequence s holds the rows starts[s] .. starts[s + 1] - 1.  Returns [tokens, n_head, 64]: rows of
    no sequence are zeros, or stay as they are in a given contiguous `out`.
    """
    lib = load_library()
    _refuse_tangents("prompt_attention", q, k, v, out)
    key = _Layouts.of(q, k, v, starts)
    plan = _prompt_plans.get(key) or _prompt_plans.keep(key, _prompt_plan(q, k, v, starts))
    dev, dtype, tokens, heads, kv, n, qs, ks, vs = plan
    wants = torch.is_grad_enabled() and (q.requires_grad or k.requires_grad or v.requires_grad)
    if out is not None:
        _tensor(out, "out", q.dtype, (tokens, heads, 64), dev)
        if wants or out.requires_grad:
            _refuse("prompt_attention into a given tensor has no gradient")

    def call(raw, empty):
        o = out if out is not None else _like(q, empty)
        if tokens:
            _check(lib.wf_prompt_attend(q.data_ptr(), qs, k.data_ptr(), ks, v.data_ptr(), vs, dtype, starts.data_ptr(), n, tokens, heads,
                                        kv, o.data_ptr(), out is None, raw))
        return o

    o = _enqueue(dev, stream, call, q, k, v, starts, out)
    if out is not None:
        _changed(out)
    return _without_backward("prompt_attention", o, q, k, v) if wants else o


class PagedCache8:
    """Self-attention keys and values in 8 bits (wf_kv8): `layers` layers of `pages` pages of 16 positions of n_head heads of
    64.  data: uint8 [layers, pages, bytes of a page], what cache_reorder takes as its cache (up to 2^18 pages); requests' page
    numbers lie in tables, int32 [n, max_pages] (rows of any stride), the same for every layer."""

    PAGE = 16

    def __init__(self, pages, n_head, layers=1, device="cuda"):
        self.lib = load_library()
        self.pages, self.n_head, self.layers = int(pages), int(n_head), int(layers)
        if max(abs(self.pages), abs(self.n_head), abs(self.layers)) >= _INTS:
            _refuse("a size is out of range")
        nbytes = ctypes.c_size_t()
        _check(self.lib.wf_kv8_page_bytes(self.n_head, ctypes.byref(nbytes)))
        if not 1 <= self.pages <= 1 << 24 or self.layers < 1:
            _refuse("pages must be in [1, 2^24] and layers 1 or more")
        self.data = torch.empty((self.layers, self.pages, nbytes.value), dtype=_U8, device=device)
        if not self.data.is_cuda:
            _refuse("device must be a GPU")
        self.device = self.data.device
        base, layer = self.data.data_ptr(), self.pages * nbytes.value
        self._c = [WfKv8(base + i * layer, self.pages, self.n_head) for i in range(self.layers)]
        self._refs = [ctypes.byref(c) for c in self._c]
        self._stores, self._loads, self._attends = _Layouts(), _Layouts(), _Layouts()

    def _layer(self, layer):
        if not 0 <= layer < self.layers:
            _refuse(f"layer must be in [0, {self.layers})")
        return self._refs[layer]

    def _tables(self, tables):
        """Requests, pages of a row and its stride."""
        if _gpu(tables, "tables", 2) != self.device or tables.dtype != _I32:
            _refuse(f"tables must be int32 on {self.device}")
        n, most = tables.shape
        if most > 1 and tables.stride(1) != 1:
            _refuse("tables must be contiguous along its last axis")
        if max(n, most) >= _INTS:
            _refuse("a size is out of range")
        return n, most, tables.stride(0)

    def _store_plan(self, k, v, tables, positions, starts, counts):
        n, most, ts = self._tables(tables)
        axes = 4 if starts is None else 3
        strides = []
        for t, name in ((k, "k"), (v, "v")):
            dev, code, s = _heads(t, name, axes)
            if dev != self.device or t.shape != k.shape or t.dtype != k.dtype or t.shape[-2] != self.n_head:
                _refuse(f"k and v must have equal shapes and types, {self.n_head} heads, and lie on {self.device}")
            strides.append(_Strides(*s) if starts is None else _Strides(0, *s))
        if starts is None and k.shape[0] != n:
            _refuse(f"k must hold {n} requests, not {k.shape[0]}")
        if starts is not None:
            if counts is not None:
                _refuse("starts and counts exclude each other")
            _vector(starts, "starts", n + 1, self.device)
        elif counts is not None:
            _vector(counts, "counts", n, self.device)
        _vector(positions, "positions", n, self.device)
        return n, most, ts, code, k.shape[-3], *strides

    def store(self, k, v, tables, positions, starts=None, counts=None, layer=0, stream=None):
        """Append rows to requests' pages from positions (int32 [n]) on.  k, v: fp32 or bf16, any strides but the last:
        packed [rows, n_head, 64] with starts (int32 [n + 1]), or [n, rows, n_head, 64], of which request r's first counts[r]
        (int32 [n], None: all) are given."""
        ref = self._layer(layer)
        args = (k, v, tables, positions, starts, counts)
        key = _Layouts.of(*args)
        n, most, ts, code, rows, ks, vs = self._stores.get(key) or self._stores.keep(key, self._store_plan(*args))
        if rows == 0:
            return
        _enqueue(self.device, stream, lambda raw, empty: _check(self.lib.wf_kv8_store(
            ref, n, k.data_ptr(), ks, v.data_ptr(), vs, code, rows, None if starts is None else starts.data_ptr(),
            None if counts is None else counts.data_ptr(), tables.data_ptr(), ts, most, positions.data_ptr(), raw)), *args, self.data)

    def _load_plan(self, tables, lens):
        n, most, ts = self._tables(tables)
        _vector(lens, "lens", n, self.device)
        return n, most, ts

    def load(self, tables, lens, dtype=torch.float32, layer=0, stream=None):
        """The keys and values that the first lens[r] (int32 [n]) positions of requests' pages hold: two tensors
        [n, 16 max_pages, n_head, 64], zeros behind them."""
        ref = self._layer(layer)
        code = _DTYPES.get(dtype)
        if code is None:
            _refuse("dtype must be float32 or bfloat16")
        key = _Layouts.of(tables, lens)
        n, most, ts = self._loads.get(key) or self._loads.keep(key, self._load_plan(tables, lens))

        def call(raw, empty):
            k = empty((n, 16 * most, self.n_head, 64), dtype=dtype, device=self.device)
            v = _like(k, empty)
            _check(self.lib.wf_kv8_load(ref, n, tables.data_ptr(), ts, most, lens.data_ptr(), k.data_ptr(), v.data_ptr(), code, raw))
            return k, v

        return _enqueue(self.device, stream, call, tables, lens, self.data)

    def _attend_plan(self, q, tables, positions, counts):
        n, most, ts = self._tables(tables)
        dev, dtype, s = _heads(q, "q", 4)
        if dev != self.device or q.shape[0] != n:
            _refuse(f"q must hold {n} requests on {self.device}")
        rows, heads = q.shape[1:3]
        nbytes = ctypes.c_size_t()
        _check(self.lib.wf_kv8_attend_workspace_bytes(self._refs[0], n, rows, heads, most, ctypes.byref(nbytes)))
        _vector(positions, "positions", n, self.device)
        if counts is not None:
            _vector(counts, "counts", n, self.device)
        return n, most, ts, dtype, rows, heads, _Strides(*s), nbytes.value

    def attend(self, q, tables, positions, counts=None, layer=0, stream=None):
        """softmax(q k^T / 8) v of q (fp32 or bf16 [n, rows, heads, 64], any strides but the last; heads a multiple of the
        cache's): row i of request r stands at positions[r] + i (int32 [n]) and sees positions up to its own.  Rows from
        counts[r] (int32 [n], None: all) on give zeros.  Returns [n, rows, heads, 64] in q's type."""
        _refuse_tangents("attend", q)
        ref = self._layer(layer)
        args = (q, tables, positions, counts)
        key = _Layouts.of(*args)
        n, most, ts, dtype, rows, heads, qs, need = self._attends.get(key) or self._attends.keep(key, self._attend_plan(*args))

        def call(raw, empty):
            out = _like(q, empty)
            ws = empty(need, dtype=_U8, device=self.device) if need else None
            _check(self.lib.wf_kv8_attend(ref, n, q.data_ptr(), qs, rows, heads, dtype, tables.data_ptr(), ts, most, positions.data_ptr(),
                                          None if counts is None else counts.data_ptr(), out.data_ptr(),
                                          ws.data_ptr() if need else None, need, raw))
            return out

        out = _enqueue(self.device, stream, call, *args, self.data)
        return _without_backward("attend", out, q) if q.requires_grad else out
