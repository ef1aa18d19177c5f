"""Operators without a handle (include/wf.h): beam selection, page-table reordering and
acoustic keys and values held in 4 bits.

Argument marshalling as in ``binding``: shapes, types and devices are checked here, sizes
and ranges by the library.  Every call enqueues on ``stream`` (default: the current stream
of the tensors' device) and returns without waiting; a given stream has to be ordered
behind the work that fills the tensors.  Workspaces and results come from PyTorch's
allocator for the call's stream, so concurrent calls and captured graphs each have their
own.

There are no backward passes.  Results of inputs that require gradients raise where a
gradient is asked of them; what a cache stores or copies has no history.
"""
import ctypes
import functools

import torch

from .binding import WF_BF16, WF_F32, WfError, WfKv4, _refuse, _tensor, load_library

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
