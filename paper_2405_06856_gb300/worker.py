"""A worker's decode step over torch tensors: a thin layer on the C ABI's
``aladdin_worker_*`` calls (``include/aladdin.h``), reached as ``aladdin.Worker``,
``aladdin.make_kv`` and ``aladdin.make_tokens``.

A step of a few microseconds should not wait for Python, so each function looks at
what it needs once, in one condition, and looks for what is wrong only when that
fails; that pointers are device memory of the worker's GPU is checked by the library.
"""
from __future__ import annotations

import ctypes as C

import torch

from . import aladdin as A

_lib = A._lib
_I32, _F32 = torch.int32, torch.float32
_LOGITS = {torch.bfloat16: A.BF16, torch.float16: A.F16, torch.float32: A.F32}
_KINDS = {"bf16": (A.BF16, torch.bfloat16), "f16": (A.F16, torch.float16)}


def _fail(what, *tensors):
    """Raise for a condition on (name, tensor, type) that failed: TypeError where a tensor is
    none or has another type or no GPU, else ValueError."""
    for name, x, kind in tensors:
        if x is None:
            continue
        if not isinstance(x, torch.Tensor) or not x.is_cuda:
            raise TypeError("%s must be a CUDA tensor" % name)
        if x.dtype is not kind:
            raise TypeError("%s must be %s, got %s" % (name, kind, x.dtype))
    raise ValueError(what)


def make_kv(k, v, table, length, weight=None, pos=None, next_pos=None):
    """An aladdin_kv over torch tensors (kept alive by the returned object).

    k, v: [pages, kv_heads, page_tokens, head_dim], any strides with contiguous channels
    (a pool in [page, token, head, channel] order is passed transposed(1, 2));
    table: int32 [requests, pages a request may have], a row in memory for each request
    (not an expanded one: their pages may be the same, their entries not); length, next_pos: int32
    [requests]; weight (float32), pos (int32): [pages, kv_heads, page_tokens]."""
    try:
        kind, shape, st = k.dtype, k.shape, k.stride()
        pages, heads, tokens, dim = shape
        n, width = table.shape
        row = table.stride()
        meta = shape[:3]
        ok = (k.is_cuda and v.dtype is kind and v.shape == shape and v.stride() == st and st[3] == 1
              and table.dtype is _I32 and (row[1] == 1 or width == 1) and (n < 2 or row[0] >= width)
              and length.dtype is _I32 and length.shape == (n,) and length.is_contiguous()
              and (weight is None or (weight.dtype is _F32 and weight.shape == meta
                                      and weight.is_contiguous()))
              and (pos is None or (pos.dtype is _I32 and pos.shape == meta and pos.is_contiguous()))
              and (next_pos is None or (next_pos.dtype is _I32 and next_pos.shape == (n,)
                                        and next_pos.is_contiguous())))
    except (AttributeError, TypeError, ValueError):
        ok = False
    if not ok:
        _fail("k and v must be [pages, kv_heads, page_tokens, head_dim] with equal strides and contiguous "
              "channels, table [requests, pages] with contiguous rows that share no memory, length and next_pos contiguous "
              "[requests], weight and pos contiguous [pages, kv_heads, page_tokens]",
              ("k", k, getattr(k, "dtype", None)), ("v", v, getattr(k, "dtype", None)), ("table", table, _I32),
              ("length", length, _I32), ("weight", weight, _F32), ("pos", pos, _I32), ("next_pos", next_pos, _I32))
    # the stride of a dimension of one entry may be anything in torch
    kv = A.aladdin_kv(k.data_ptr(), v.data_ptr(), st[0] if pages > 1 else heads * tokens * dim,
                      st[1] if heads > 1 else tokens * dim, st[2], pages, width,
                      row[0] if n > 1 else width, table.data_ptr(), length.data_ptr(),
                      None if weight is None else weight.data_ptr(),
                      None if pos is None else pos.data_ptr(),
                      None if next_pos is None else next_pos.data_ptr())
    kv._shape = (kind, heads, tokens, dim)
    kv._n = n
    kv._keep = (k, v, table, length, weight, pos, next_pos)
    return kv


def make_tokens(off, q, k, v, parent=None):
    """An aladdin_tokens over torch tensors (kept alive by the returned object).

    off: int32 [requests + 1]; q: [tokens, q_heads, head_dim], k, v: [tokens, kv_heads,
    head_dim], heads and channels contiguous, any token stride (slices of one
    projection's output); q may be None where no call needs it; parent: int32 [tokens]."""
    try:
        kind, shape, ks, vs = k.dtype, k.shape, k.stride(), v.stride()
        n, heads, dim = shape
        q_heads = qs = 0
        ok = (k.is_cuda and v.dtype is kind and v.shape == shape and off.dtype is _I32 and off.dim() == 1
              and off.shape[0] > 0 and off.is_contiguous()
              and (n == 0 or (ks[2] == vs[2] == 1 and (heads == 1 or ks[1] == vs[1] == dim)))
              and (parent is None or (parent.dtype is _I32 and parent.shape == (n,)
                                      and parent.is_contiguous())))
        if ok and q is not None:
            qn, q_heads, qd = q.shape
            st = q.stride()
            # the stride of one row may be anything in torch: the row itself then
            qs = st[0] if n > 1 else q_heads * dim
            ok = (q.dtype is kind and qn == n and qd == dim
                  and (n == 0 or (st[2] == 1 and (q_heads == 1 or st[1] == dim))))
    except (AttributeError, TypeError, ValueError):
        ok = False
    if not ok:
        _fail("q, k and v must be [tokens, heads, head_dim] with contiguous heads and channels, k and v of one "
              "shape, off contiguous [requests + 1], parent contiguous [tokens]",
              ("k", k, getattr(k, "dtype", None)), ("v", v, getattr(k, "dtype", None)),
              ("q", q, getattr(k, "dtype", None)), ("off", off, _I32), ("parent", parent, _I32))
    tok = A.aladdin_tokens(off.shape[0] - 1, n, off.data_ptr(),
                           None if parent is None else parent.data_ptr(),
                           None if q is None else q.data_ptr(), k.data_ptr(), v.data_ptr(), qs,
                           ks[0] if n > 1 else heads * dim, vs[0] if n > 1 else heads * dim)
    tok._shape = (kind, q_heads, heads, dim)
    tok._keep = (off, parent, q, k, v)
    return tok


class Worker:
    """A worker's decode step over torch tensors.

    kind: "bf16" or "f16". The worker is bound to a stream (default: torch's current
    one at its creation); a call made while another stream is torch's current one
    waits for what was launched there before, and what is launched there afterwards
    waits for the call."""

    def __init__(self, kind, q_heads, kv_heads, head_dim, page_tokens, stream=None):
        self.handle = None
        if kind not in _KINDS:
            raise ValueError("kind must be one of %s" % sorted(_KINDS))
        torch.cuda.init()
        self._index = torch.cuda.current_device()
        self.device = torch.device("cuda", self._index)
        self.stream = torch.cuda.current_stream().cuda_stream if stream is None else stream
        number, self.dtype = _KINDS[kind]
        self.q_heads, self.kv_heads = int(q_heads), int(kv_heads)
        self.head_dim, self.page_tokens = int(head_dim), int(page_tokens)
        self._kv_shape = (self.dtype, self.kv_heads, self.page_tokens, self.head_dim)
        self._tok_shape = (self.dtype, self.q_heads, self.kv_heads, self.head_dim)
        self._tok_bare = (self.dtype, 0, self.kv_heads, self.head_dim)  # without queries
        self.handle = A.aladdin_worker_create(
            A.aladdin_worker_shape(number, self.q_heads, self.kv_heads, self.head_dim, self.page_tokens),
            self.stream)

    def close(self):
        if getattr(self, "handle", None):
            A.aladdin_worker_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def __enter__(self):
        return self

    def __exit__(self, *a):
        self.close()

    def status(self):
        return A.aladdin_worker_status(self.handle)

    def _call(self, name, *args):
        """The library's function in the order of torch's current stream."""
        if torch._C._cuda_getCurrentRawStream(self._index) == self.stream:
            rc = getattr(_lib, name)(self.handle, *args)
        else:
            current = torch.cuda.current_stream(self.device)
            mine = torch.cuda.ExternalStream(self.stream, self.device)
            mine.wait_stream(current)
            rc = getattr(_lib, name)(self.handle, *args)
            current.wait_stream(mine)
        if rc:
            raise A.AladdinError(rc, name)

    def _check(self, kv, tok, bare):
        if kv._shape != self._kv_shape:
            raise ValueError("the cache does not have the worker's type or shape: %s, not %s"
                             % (kv._shape, self._kv_shape))
        if tok._shape != self._tok_shape and not (bare and tok._shape == self._tok_bare):
            raise ValueError("the tokens do not have the worker's type or heads: %s, not %s"
                             % (tok._shape, self._tok_shape))
        if kv._n != tok.n_req:
            raise ValueError("the cache has %d requests, the tokens %d" % (kv._n, tok.n_req))

    def attend(self, kv, tok, scale=None, out=None, lse=None):
        """(out [tokens, q_heads, head_dim], lse [tokens, q_heads]); scale defaults to
        head_dim ** -0.5."""
        self._check(kv, tok, False)
        n = tok.n_tok
        stride = self.q_heads * self.head_dim
        if out is None:
            out = torch.empty((n, self.q_heads, self.head_dim), dtype=self.dtype, device=self.device)
        else:
            if out.dtype is not self.dtype or out.shape != (n, self.q_heads, self.head_dim) or \
                    out.stride(2) != 1 or (self.q_heads > 1 and out.stride(1) != self.head_dim):
                _fail("out must be [tokens, q_heads, head_dim], heads and channels contiguous",
                      ("out", out, self.dtype))
            if n > 1:
                stride = out.stride(0)
        if lse is None:
            lse = torch.empty((n, self.q_heads), dtype=_F32, device=self.device)
        elif lse.dtype is not _F32 or lse.shape != (n, self.q_heads) or not lse.is_contiguous():
            _fail("lse must be contiguous [tokens, q_heads]", ("lse", lse, _F32))
        self._call("aladdin_worker_attend", C.byref(kv), C.byref(tok),
                   self.head_dim ** -0.5 if scale is None else scale, out.data_ptr(), stride, lse.data_ptr())
        return out, lse

    def accept(self, kv, tok, scale=None, lse=None, acc_off=None, acc=None):
        """Keep tokens (all of them without acc_off and acc) in the cache, in place;
        with the lse of the tokens' attention the cache's weights grow by what the kept
        rows attended to."""
        self._check(kv, tok, lse is None)
        n = 0
        if acc_off is not None or acc is not None:
            if acc_off is None or acc is None or acc_off.dtype is not _I32 or acc.dtype is not _I32 or \
                    acc_off.shape != (tok.n_req + 1,) or acc.dim() != 1 or not acc_off.is_contiguous() or \
                    not acc.is_contiguous():
                _fail("acc_off and acc come together, contiguous [requests + 1] and [kept tokens]",
                      ("acc_off", acc_off, _I32), ("acc", acc, _I32))
            n, acc_off, acc = acc.shape[0], acc_off.data_ptr(), acc.data_ptr()
        if lse is not None:
            if kv.weight is None:
                raise ValueError("the cache has no weights to add to")
            if lse.dtype is not _F32 or lse.shape != (tok.n_tok, self.q_heads) or not lse.is_contiguous():
                _fail("lse must be contiguous [tokens, q_heads]", ("lse", lse, _F32))
            lse = lse.data_ptr()
        self._call("aladdin_worker_accept", C.byref(kv), C.byref(tok),
                   self.head_dim ** -0.5 if scale is None else scale, lse, acc_off, acc, n)

    def evict(self, kv, budget, recent=0):
        """Reduce the cache's requests to budget (int32 [requests]) tokens, in place."""
        if kv._shape != self._kv_shape:
            raise ValueError("the cache does not have the worker's type or shape: %s, not %s"
                             % (kv._shape, self._kv_shape))
        if kv.weight is None or kv.pos is None or kv.next is None:
            raise ValueError("eviction needs weight, pos and next_pos")
        if budget.dtype is not _I32 or budget.shape != (kv._n,) or not budget.is_contiguous():
            _fail("budget must be contiguous [requests]", ("budget", budget, _I32))
        if not 0 <= recent < 1 << 31:
            raise ValueError("recent must be at least 0 and fit in 32 bits")
        self._call("aladdin_worker_evict", C.byref(kv), kv._n, budget.data_ptr(), recent)

    def logprobs(self, logits, token=None, top=0):
        """(logprob, entropy, rank, top_id, top_logprob) of logits [rows, vocab] (contiguous
        vocabulary) at token int32 [rows]; without token logprob and rank are None, with top 0
        the alternatives."""
        kind = _LOGITS.get(logits.dtype)
        if kind is None or logits.dim() != 2 or not logits.is_cuda:
            if kind is not None and logits.is_cuda:
                raise ValueError("logits must be [rows, vocab]")
            raise TypeError("logits must be a CUDA tensor of bfloat16, float16 or float32")
        n, vocab = logits.shape
        st = logits.stride()
        if (vocab > 1 and st[1] != 1) or (n > 1 and st[0] < vocab):
            raise ValueError("the rows of logits must be contiguous and share no memory")
        if not 0 <= top < 1 << 31:
            raise ValueError("top must be at least 0 and fit in 32 bits")
        dev, empty = self.device, torch.empty
        logprob = rank = ids = tops = None
        lp = rk = ip = tp = tk = None
        if token is not None:
            if token.dtype is not _I32 or token.shape != (n,) or not token.is_contiguous():
                _fail("token must be contiguous [rows]", ("token", token, _I32))
            logprob, rank = empty(n, dtype=_F32, device=dev), empty(n, dtype=_I32, device=dev)
            tk, lp, rk = token.data_ptr(), logprob.data_ptr(), rank.data_ptr()
        entropy = empty(n, dtype=_F32, device=dev)
        if top:
            ids, tops = empty((n, top), dtype=_I32, device=dev), empty((n, top), dtype=_F32, device=dev)
            ip, tp = ids.data_ptr(), tops.data_ptr()
        self._call("aladdin_worker_logprobs", kind, n, vocab, logits.data_ptr(),
                   st[0] if n > 1 else vocab, tk, top, lp, entropy.data_ptr(), rk, ip, tp)
        return logprob, entropy, rank, ids, tops
