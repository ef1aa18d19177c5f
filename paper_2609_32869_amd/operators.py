"""Operators without a handle (include/wf.h): beam selection, page-table reordering and
acoustic keys and values held in 4 bits.

Argument marshalling as in ``binding``: shapes, types and devices are checked here, sizes
and ranges by the library.  Every call enqueues on ``stream`` (default: the current stream
of the tensors' device) and returns without waiting; workspaces and results come from
PyTorch's allocator, so concurrent calls and captured graphs each have their own.
"""
import ctypes

import torch

from .binding import WF_BF16, WF_F32, WfError, WfKv4, _ptr, load_library

_DTYPES = {torch.float32: WF_F32, torch.bfloat16: WF_BF16}


def _check(lib, rc):
    if rc != 0:
        msg = lib.wf_last_error(None)
        raise WfError(f"{lib.wf_strerror(rc).decode()} ({rc}): {msg.decode() if msg else ''}")


def _need(ok, what):
    if not ok:
        raise WfError(f"invalid argument (-1): {what}")


def _tensor(t, name, dtypes, shape=None, device=None, contiguous=True):
    """Refuse a tensor of another kind; shape entries of None match any size."""
    _need(isinstance(t, torch.Tensor), f"{name} must be a tensor")
    dtypes = dtypes if isinstance(dtypes, tuple) else (dtypes,)
    _need(t.dtype in dtypes, f"{name} must be {' or '.join(str(d)[6:] for d in dtypes)}, not {str(t.dtype)[6:]}")
    if shape is not None:
        _need(t.dim() == len(shape) and all(s is None or s == g for s, g in zip(shape, t.shape)),
              f"{name} must have shape {tuple('any' if s is None else s for s in shape)}, not {tuple(t.shape)}")
    _need(t.is_cuda, f"{name} must be on the GPU")
    _need(device is None or t.device == device, f"{name} is on another device")
    _need(not contiguous or t.is_contiguous(), f"{name} must be contiguous")
    return t


class _On:
    """The tensors' device made current and a stream of it, for the length of a call."""

    def __init__(self, device, stream):
        _need(stream is None or stream.device == device, "stream is of another device than the tensors")
        self.guard, self.device, self.stream = torch.cuda.device(device), device, stream

    def __enter__(self):
        self.guard.__enter__()
        s = self.stream if self.stream is not None else torch.cuda.current_stream(self.device)
        self.other = self.stream is not None and s != torch.cuda.current_stream(self.device)
        self.s = s
        return self

    def __exit__(self, *exc):
        return self.guard.__exit__(*exc)

    def ptr(self):
        return ctypes.c_void_p(self.s.cuda_stream)

    def empty(self, shape, dtype):
        """Memory for this call's work: freed or reused only behind it on its stream."""
        t = torch.empty(shape, dtype=dtype, device=self.device)
        if self.other:
            t.record_stream(self.s)
        return t


def beam_select(logits, scores, k, suppress=None, stream=None):
    """The k best continuations of each request's beams: wf_beam_select.

    logits: fp32 or bf16 [n, beams, vocab], the last axis contiguous; scores: fp32 [n, beams];
    suppress: uint8 [vocab] or None.  Returns (score fp32, beam int32, token int32), each [n, k].
    """
    lib = load_library()
    _tensor(logits, "logits", tuple(_DTYPES), (None, None, None), contiguous=False)
    n, beams, vocab = logits.shape
    dev = logits.device
    _need(vocab <= 1 or logits.stride(2) == 1, "logits must be contiguous along the vocabulary")
    _tensor(scores, "scores", torch.float32, (n, beams), dev)
    if suppress is not None:
        _tensor(suppress, "suppress", torch.uint8, (vocab,), dev)
    k = int(k)
    nbytes = ctypes.c_size_t()
    _check(lib, lib.wf_beam_select_workspace_bytes(n, beams, vocab, k, ctypes.byref(nbytes)))
    with _On(dev, stream) as on:
        score, beam = on.empty((n, k), torch.float32), on.empty((n, k), torch.int32)
        token, ws = on.empty((n, k), torch.int32), on.empty(nbytes.value, torch.uint8)
        _check(lib, lib.wf_beam_select(_ptr(logits), _DTYPES[logits.dtype], logits.stride(0), logits.stride(1), _ptr(scores),
                                       _ptr(suppress), n, beams, vocab, k, _ptr(score), _ptr(beam), _ptr(token), _ptr(ws),
                                       nbytes.value, on.ptr()))
    return score, beam, token


def cache_reorder(cache, tables, parents, lens, pool, page_tokens=16, stream=None):
    """Page tables (and page copies, in place) after a choice of beams: wf_cache_reorder.

    cache: [regions, pages, ...] contiguous, pages of a multiple of 16 bytes; tables: int32
    [n, beams, max_pages]; parents: int32 [n, beams]; lens: int32 [n]; pool: int32 [n, pool_pages].
    Returns the new tables.
    """
    lib = load_library()
    _need(isinstance(cache, torch.Tensor) and cache.is_cuda, "cache must be a tensor on the GPU")
    _need(cache.dim() >= 3 and cache.is_contiguous() and cache.numel() > 0, "cache must be contiguous [regions, pages, ...]")
    dev = cache.device
    _tensor(tables, "tables", torch.int32, (None, None, None), dev)
    n, beams, max_pages = tables.shape
    _tensor(parents, "parents", torch.int32, (n, beams), dev)
    _tensor(lens, "lens", torch.int32, (n,), dev)
    _tensor(pool, "pool", torch.int32, (n, None), dev)
    regions, pages = cache.shape[:2]
    page = cache[0, 0].numel() * cache.element_size()
    with _On(dev, stream) as on:
        new = on.empty((n, beams, max_pages), torch.int32)
        _check(lib, lib.wf_cache_reorder(_ptr(cache), regions, pages * page, pages, page, _ptr(tables), _ptr(new), n, beams,
                                         max_pages, int(page_tokens), _ptr(parents), _ptr(lens), _ptr(pool), pool.shape[1],
                                         on.ptr()))
    return new


class AcousticCache4:
    """Keys and values of `entries` acoustic memories in 4 bits (wf_kv4): n_frames frames of n_head heads of 64."""

    def __init__(self, entries, n_head, n_frames, device="cuda"):
        self.lib = load_library()
        self.entries, self.n_head, self.n_frames = int(entries), int(n_head), int(n_frames)
        nbytes = ctypes.c_size_t()
        _check(self.lib, self.lib.wf_kv4_bytes(self.entries, self.n_head, self.n_frames, ctypes.byref(nbytes)))
        self.data = torch.empty(nbytes.value, dtype=torch.uint8, device=device)
        _need(self.data.is_cuda, "device must be a GPU")
        self.device = self.data.device
        self.c = WfKv4(self.data.data_ptr(), self.entries, self.n_head, self.n_frames)

    def _lens(self, lens, n):
        if lens is not None:
            _tensor(lens, "lens", torch.int32, (n,), self.device)
        return _ptr(lens)

    def _rows(self, t, name, shape, dtypes=tuple(_DTYPES)):
        _tensor(t, name, dtypes, shape, self.device, contiguous=False)
        _need(t.stride(3) == 1, f"{name} must be contiguous along its last axis")
        return (ctypes.c_int64 * 3)(*t.stride()[:3])

    def store(self, slot0, k, v, lens=None, stream=None):
        """Entries slot0 .. from k, v: fp32 or bf16 [n, n_frames, n_head, 64] (any strides but the last), of which the
        first lens[r] frames (int32 [n], None: all) are given and the others hold zeros."""
        shape = (None, self.n_frames, self.n_head, 64)
        ks = self._rows(k, "k", shape)
        vs = self._rows(v, "v", (k.shape[0],) + shape[1:], k.dtype)
        with _On(self.device, stream) as on:
            _check(self.lib, self.lib.wf_kv4_store(ctypes.byref(self.c), int(slot0), k.shape[0], _ptr(k), ks, _ptr(v), vs,
                                                   _DTYPES[k.dtype], self._lens(lens, k.shape[0]), on.ptr()))

    def load(self, slot0, n, dtype=torch.float32, stream=None):
        """The keys and values that entries slot0 .. slot0 + n - 1 hold: two tensors [n, n_frames, n_head, 64]."""
        _need(dtype in _DTYPES, "dtype must be float32 or bfloat16")
        _need(0 < n <= self.entries and 0 <= slot0 <= self.entries - n, "entries out of range")
        with _On(self.device, stream) as on:
            k = on.empty((n, self.n_frames, self.n_head, 64), dtype)
            v = on.empty((n, self.n_frames, self.n_head, 64), dtype)
            _check(self.lib, self.lib.wf_kv4_load(ctypes.byref(self.c), int(slot0), n, _ptr(k), _ptr(v), _DTYPES[dtype],
                                                  on.ptr()))
        return k, v

    def attend(self, slot0, q, lens=None, stream=None):
        """softmax(q k^T / 8) v of q (fp32 or bf16 [n, rows, n_head, 64], any strides but the last) over the first lens[r]
        frames (int32 [n], None: all) of entries slot0 ..: [n, rows, n_head, 64] in q's type."""
        qs = self._rows(q, "q", (None, None, self.n_head, 64))
        n, rows = q.shape[:2]
        nbytes = ctypes.c_size_t()
        _check(self.lib, self.lib.wf_kv4_attend_workspace_bytes(ctypes.byref(self.c), n, rows, ctypes.byref(nbytes)))
        with _On(self.device, stream) as on:
            out, ws = on.empty((n, rows, self.n_head, 64), q.dtype), on.empty(max(nbytes.value, 1), torch.uint8)
            _check(self.lib, self.lib.wf_kv4_attend(ctypes.byref(self.c), int(slot0), n, _ptr(q), qs, rows, _DTYPES[q.dtype],
                                                    self._lens(lens, n), _ptr(out), _ptr(ws), nbytes.value, on.ptr()))
        return out
