"""A worker's decode step over torch tensors: a thin layer on the C ABI's
``aladdin_worker_*`` calls (``include/aladdin.h``), reached as ``aladdin.Worker``,
``aladdin.make_kv``, ``aladdin.make_kv8``, ``aladdin.make_tokens`` and ``aladdin.make_rope``.

A step of a few microseconds should not wait for Python, so each function looks at
what it needs once, in one condition, and looks for what is wrong only when that
fails; that pointers are device memory of the worker's GPU is checked by the library.
"""
from __future__ import annotations

import ctypes as C

import torch

from . import aladdin as A

_lib = A._lib
_I32, _F32, _F8 = torch.int32, torch.float32, torch.float8_e4m3fn
_LOGITS = {torch.bfloat16: A.BF16, torch.float16: A.F16, torch.float32: A.F32}
_LAYOUTS = {"half": A.ROPE_HALF, "interleaved": A.ROPE_INTERLEAVED}
_SCALINGS = {None: A.ROPE_NONE, "linear": A.ROPE_LINEAR, "base": A.ROPE_BASE, "parts": A.ROPE_PARTS}
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


def make_kv8(k, v, k_scale, v_scale, table, length, next_pos=None):
    """An aladdin_kv8 over torch tensors (kept alive by the returned object).

    k, v: float8_e4m3fn [pages, kv_heads, page_tokens, head_dim], strides as for make_kv; k_scale, v_scale: contiguous
    float32 [pages, kv_heads, page_tokens / block], of the tokens [i block, (i + 1) block) of a page; table, length,
    next_pos as for make_kv."""
    try:
        shape, st = k.shape, k.stride()
        pages, heads, tokens, dim = shape
        n, width = table.shape
        row = table.stride()
        meta = k_scale.shape
        ok = (k.is_cuda and k.dtype is _F8 and v.dtype is _F8 and v.shape == shape and v.stride() == st and st[3] == 1
              and k_scale.dtype is _F32 and v_scale.dtype is _F32 and v_scale.shape == meta
              and k_scale.is_contiguous() and v_scale.is_contiguous()
              and meta[:2] == shape[:2] and len(meta) == 3 and meta[2] > 0 and tokens % meta[2] == 0
              and table.dtype is _I32 and (row[1] == 1 or width == 1) and (n < 2 or row[0] >= width)
              and length.dtype is _I32 and length.shape == (n,) and length.is_contiguous()
              and (next_pos is None or (next_pos.dtype is _I32 and next_pos.shape == (n,)
                                        and next_pos.is_contiguous())))
    except (AttributeError, TypeError, ValueError):
        ok = False
    if not ok:
        _fail("k and v must be [pages, kv_heads, page_tokens, head_dim] with equal strides and contiguous "
              "channels, k_scale and v_scale contiguous [pages, kv_heads, page_tokens / block], table [requests, pages] with "
              "contiguous rows that share no memory, length and next_pos contiguous [requests]",
              ("k", k, _F8), ("v", v, _F8), ("k_scale", k_scale, _F32), ("v_scale", v_scale, _F32),
              ("table", table, _I32), ("length", length, _I32), ("next_pos", next_pos, _I32))
    kv = A.aladdin_kv8(k.data_ptr(), v.data_ptr(), st[0] if pages > 1 else heads * tokens * dim,
                       st[1] if heads > 1 else tokens * dim, st[2], pages, width, row[0] if n > 1 else width,
                       table.data_ptr(), length.data_ptr(), None if next_pos is None else next_pos.data_ptr(),
                       k_scale.data_ptr(), v_scale.data_ptr(), tokens // meta[2])
    kv._shape = ("e4m3", heads, tokens, dim)
    kv._n = n
    kv._keep = (k, v, k_scale, v_scale, table, length, next_pos)
    return kv


def make_rope(dim, base=10000.0, layout="half", scaling=None, factor=1.0, original=None, slow=1.0, fast=32.0,
              freq=None, scale=None, device=None):
    """Rotary positions of the first ``dim`` channels of a head (an aladdin_rope, its frequencies on the GPU).

    layout: "half" (channels c, c + dim / 2 form a pair) or "interleaved" (2 c, 2 c + 1). Frequencies are base^(-2 c / dim),
    scaled for long contexts by ``factor``: "linear", "base", or "parts" (of a model made for ``original`` positions: pairs
    that turn fewer than ``slow`` times in them are slowed down, those of more than ``fast`` times are left, and in
    between in proportion to the turns; a model with a ramp over the pairs' index gives ``freq``);
    or ``freq``, dim / 2 numbers in radians a position. ``scale`` multiplies rotated channels (default: 1, for "parts"
    0.1 ln(factor) + 1)."""
    if layout not in _LAYOUTS:
        raise ValueError("layout must be one of %s" % sorted(_LAYOUTS))
    if scaling not in _SCALINGS:
        raise ValueError("scaling must be None or one of %s" % sorted(s for s in _SCALINGS if s))
    if dim < 2 or dim % 2:
        raise ValueError("dim must be even and at least 2")
    if scaling is None and factor != 1.0:
        raise ValueError("factor needs a scaling that it belongs to")
    if freq is None:
        if scaling == "parts" and original is None:
            raise ValueError("scaling by parts needs the positions that the model was made for (original)")
        freq, own = A.aladdin_rope_frequencies(dim, base, _SCALINGS[scaling], factor, original or 0.0, slow, fast)
    else:
        if scaling is not None:
            raise ValueError("freq and scaling exclude each other")
        freq, own = torch.as_tensor(freq, dtype=torch.float64).cpu().numpy(), 1.0
        if freq.shape != (dim // 2,):
            raise ValueError("freq must have dim / 2 numbers")
    turn = torch.from_numpy(A.aladdin_rope_turns(freq).view("int64")).to("cuda" if device is None else device)
    rope = A.aladdin_rope(dim, _LAYOUTS[layout], own if scale is None else scale, turn.data_ptr())
    rope._keep = turn
    return rope


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
        self._kv8_shape = ("e4m3", self.kv_heads, self.page_tokens, self.head_dim)
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

    def _check(self, kv, tok, bare, eight=False):
        if kv._shape != self._kv_shape and not (eight and kv._shape == self._kv8_shape):
            raise ValueError("the cache does not have the worker's type or shape: %s, not %s"
                             % (kv._shape, self._kv_shape))
        if tok._shape != self._tok_shape and not (bare and tok._shape == self._tok_bare):
            raise ValueError("the tokens do not have the worker's type or heads: %s, not %s"
                             % (tok._shape, self._tok_shape))
        if kv._n != tok.n_req:
            raise ValueError("the cache has %d requests, the tokens %d" % (kv._n, tok.n_req))

    def attend(self, kv, tok, scale=None, out=None, lse=None):
        """(out [tokens, q_heads, head_dim], lse [tokens, q_heads]); scale defaults to
        head_dim ** -0.5. kv: a cache of 16 or (make_kv8) of 8 bits."""
        self._check(kv, tok, False, True)
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
        self._call("aladdin_worker_attend8" if kv._shape[0] == "e4m3" else "aladdin_worker_attend", C.byref(kv), C.byref(tok),
                   self.head_dim ** -0.5 if scale is None else scale, out.data_ptr(), stride, lse.data_ptr())
        return out, lse

    def rotate(self, rope, tok, next_pos=None, pos=None, q_out=None, k_out=None):
        """(q, k) of the tokens rotated to their positions: ``pos`` (int32 [tokens]), or ``next_pos`` (int32 [requests];
        None: 0) plus a token's depth in its tree. q_out, k_out: None for a new tensor, the tokens' own tensor (in place),
        another one, or False to leave them out. Without ``pos`` tokens that no request has (padding) are not written."""
        if tok._shape != self._tok_shape and not (q_out is False and tok._shape == self._tok_bare):
            raise ValueError("the tokens do not have the worker's type or heads: %s, not %s"
                             % (tok._shape, self._tok_shape))
        n = tok.n_tok
        if (next_pos is not None and (next_pos.dtype is not _I32 or next_pos.shape != (tok.n_req,)
                                      or not next_pos.is_contiguous())) or \
                (pos is not None and (pos.dtype is not _I32 or pos.shape != (n,) or not pos.is_contiguous())):
            _fail("next_pos must be contiguous [requests], pos contiguous [tokens]",
                  ("next_pos", next_pos, _I32), ("pos", pos, _I32))
        args = []
        outs = []
        for out, heads in ((q_out, self.q_heads), (k_out, self.kv_heads)):
            stride = heads * self.head_dim
            if out is None:
                out = torch.empty((n, heads, self.head_dim), dtype=self.dtype, device=self.device)
            elif out is not False:
                if out.dtype is not self.dtype or out.shape != (n, heads, self.head_dim) or \
                        out.stride(2) != 1 or (heads > 1 and out.stride(1) != self.head_dim):
                    _fail("q_out and k_out must be [tokens, heads, head_dim], heads and channels contiguous",
                          ("out", out, self.dtype))
                if n > 1:
                    stride = out.stride(0)
            outs.append(None if out is False else out)
            args += [None if out is False else out.data_ptr(), stride]
        self._call("aladdin_worker_rotate", C.byref(rope), C.byref(tok),
                   None if next_pos is None else next_pos.data_ptr(), None if pos is None else pos.data_ptr(), *args)
        return tuple(outs)

    def append(self, kv, tok, rope=None, acc_off=None, acc=None):
        """Append tokens (all of them, any number, without acc_off and acc) to a cache of 16 or (make_kv8) of 8 bits, in
        place; with ``rope`` keys are rotated to their positions on the way."""
        self._check(kv, tok, True, True)
        n, acc_off, acc = self._choice(tok, acc_off, acc)
        self._call("aladdin_worker_append8" if kv._shape[0] == "e4m3" else "aladdin_worker_append", C.byref(kv),
                   C.byref(tok), None if rope is None else C.byref(rope), acc_off, acc, n)

    @staticmethod
    def _choice(tok, acc_off, acc):
        """Number and addresses of the chosen tokens."""
        if acc_off is None and acc is None:
            return 0, None, None
        if acc_off is None or acc is None or acc_off.dtype is not _I32 or acc.dtype is not _I32 or \
                acc_off.shape != (tok.n_req + 1,) or acc.dim() != 1 or not acc_off.is_contiguous() or \
                not acc.is_contiguous():
            _fail("acc_off and acc come together, contiguous [requests + 1] and [kept tokens]",
                  ("acc_off", acc_off, _I32), ("acc", acc, _I32))
        return acc.shape[0], acc_off.data_ptr(), acc.data_ptr()

    def accept(self, kv, tok, scale=None, lse=None, acc_off=None, acc=None):
        """Keep tokens (all of them without acc_off and acc) in the cache, in place;
        with the lse of the tokens' attention the cache's weights grow by what the kept
        rows attended to."""
        self._check(kv, tok, lse is None)
        n, acc_off, acc = self._choice(tok, acc_off, acc)
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
