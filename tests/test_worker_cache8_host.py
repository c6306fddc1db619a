"""Rotary positions and the cache of 8 bits on the host: struct layouts, frequencies, refusals that need no GPU, the tests'
own definitions by hand, and what the torch layer hands to the library."""
import ctypes
import math

import numpy as np
import pytest
import torch

import worker8_ref as ref8


class OnGpu(torch.Tensor):
    is_cuda = property(lambda self: True)


def put(x):
    return x.as_subclass(OnGpu)


@pytest.fixture(scope="module")
def lib():
    from paper_2405_06856_gb300 import build
    build.build()
    from paper_2405_06856_gb300 import aladdin as A
    return A


@pytest.fixture(scope="module")
def W(lib):
    from paper_2405_06856_gb300 import worker
    return worker


def test_struct_layout(lib):
    assert ctypes.sizeof(lib.aladdin_rope) == 24 and lib.aladdin_rope.turn.offset == 16
    assert ctypes.sizeof(lib.aladdin_kv8) == 104
    assert lib.aladdin_kv8.table.offset == 56 and lib.aladdin_kv8.k_scale.offset == 80 and lib.aladdin_kv8.block.offset == 96


def test_null_arguments(lib):
    L = lib._lib
    assert L.aladdin_worker_rotate(None, None, None, None, None, None, 0, None, 0) == lib.ERR_ARG
    assert L.aladdin_worker_append(None, None, None, None, None, None, 0) == lib.ERR_ARG
    assert L.aladdin_worker_append8(None, None, None, None, None, None, 0) == lib.ERR_ARG
    assert L.aladdin_worker_attend8(None, None, None, 1.0, None, 0, None) == lib.ERR_ARG
    assert L.aladdin_rope_turns(1, None, None) == lib.ERR_ARG
    assert L.aladdin_rope_turns(-1, None, None) == lib.ERR_ARG and L.aladdin_rope_turns(0, None, None) == 0
    assert L.aladdin_rope_frequencies(8, 10000.0, 0, 1.0, 0.0, 1.0, 32.0, None, None) == lib.ERR_ARG


@pytest.mark.parametrize("bad", [dict(dim=0), dict(dim=7), dict(dim=-2), dict(base=1.0), dict(base=math.nan), dict(base=math.inf),
                                 dict(scaling=4), dict(scaling=-1), dict(scaling=1, factor=0.5), dict(scaling=1, factor=math.nan),
                                 dict(scaling=2, dim=2, factor=2.0), dict(scaling=2, factor=1e300), dict(scaling=3, factor=2.0, original=0.0),
                                 dict(scaling=3, factor=2.0, original=100.0, slow=2.0, fast=2.0),
                                 dict(scaling=3, factor=2.0, original=100.0, slow=0.0)])
def test_frequencies_refused(lib, bad):
    with pytest.raises(lib.AladdinError):
        lib.aladdin_rope_frequencies(**{"dim": 8, **bad})


@pytest.mark.parametrize("dim", [2, 10, 64, 128])
def test_frequencies(lib, dim):
    plain = np.array([10000.0 ** (-2.0 * c / dim) for c in range(dim // 2)])
    got, s = lib.aladdin_rope_frequencies(dim)
    assert np.allclose(got, plain, rtol=1e-14, atol=0) and s == 1.0
    got, s = lib.aladdin_rope_frequencies(dim, 10000.0, lib.ROPE_LINEAR, 4.0)
    assert np.allclose(got, plain / 4, rtol=1e-14, atol=0) and s == 1.0
    if dim > 2:
        got, s = lib.aladdin_rope_frequencies(dim, 10000.0, lib.ROPE_BASE, 4.0)
        assert got[0] == 1.0 and np.isclose(got[-1], plain[-1] / 4, rtol=1e-13) and s == 1.0  # the slowest is interpolated
    got, s = lib.aladdin_rope_frequencies(dim, 10000.0, lib.ROPE_PARTS, 8.0, 4096.0, 1.0, 32.0)
    assert np.isclose(s, 0.1 * math.log(8.0) + 1.0, rtol=1e-7)
    for f, p in zip(got, plain):
        turns = 4096.0 * p / (2 * math.pi)
        want = p if turns >= 32 else p / 8 if turns <= 1 else p / 8 + (p - p / 8) * (turns - 1) / 31
        assert np.isclose(f, want, rtol=1e-13)


def test_turns(lib):
    """p turn mod 2^64 is the angle: of whole and of negative turns, and far positions of others."""
    freq = np.array([0.0, 2 * math.pi, -2 * math.pi, math.pi, -math.pi, 1.0, -1.0, 1e-4, 7.3, -1e-300])
    turn = lib.aladdin_rope_turns(freq)
    assert turn[:5].tolist() == [0, 0, 0, 1 << 63, 1 << 63] and turn[-1] == 0
    for f, t in zip(freq, turn.tolist()):
        for p in (0, 1, -1, 1000, 131071, -70000):
            angle = (p * t % (1 << 64)) / 2.0 ** 64 * 2 * math.pi
            assert abs(math.remainder(angle - p * f, 2 * math.pi)) <= abs(p * f) * 2.0 ** -51 + 2.0 ** -48, (f, p)
    for bad in (math.inf, math.nan):
        with pytest.raises(lib.AladdinError):
            lib.aladdin_rope_turns([1.0, bad])


def test_codes_by_hand():
    v = ref8.VALUES
    assert v[1] == 2.0 ** -9 and v[7] == 7 * 2.0 ** -9 and v[8] == 2.0 ** -6 and v[126] == 448 and np.all(np.diff(v) > 0)
    x = np.array([0.0, -0.0, 448, -448, 1.0, 1.0625, 1.1875, 2.0 ** -10, 1.5 * 2.0 ** -9, np.nan, np.inf, -2.0 ** -6])
    # halfway between 1 and 1.125, 1.125 and 1.25, 0 and 2^-9, 2^-9 and 2^-8: the even one
    assert ref8.code(x).tolist() == [0, 128, 126, 254, 56, 56, 58, 0, 2, 127, 127, 136]
    want = torch.from_numpy(np.linspace(-448, 448, 4097)).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    assert np.array_equal(ref8.code(np.linspace(-448, 448, 4097)), want)
    assert np.array_equal(ref8.value(ref8.code(v)), v)
    assert ref8.scale_of(448.0) == 1 and ref8.scale_of(449.0) == 2 and ref8.scale_of(0.0) == 2.0 ** -126
    assert ref8.scale_of(224.0) == 0.5


def test_rotation_by_hand():
    x = np.array([[[1.0, 2.0, 3.0, 4.0, 5.0]]])
    for layout, pairs in (("half", [(0, 2), (1, 3)]), ("interleaved", [(0, 1), (2, 3)])):
        y = ref8.rotate(x, [3], [math.pi / 2, math.pi / 6], layout, 2.0)  # 3/4 of a turn, 1/4 of a turn
        (a, b), (c, d) = pairs
        want = x[0, 0].copy()
        want[[a, b, c, d]] = 2 * x[0, 0, b], -2 * x[0, 0, a], -2 * x[0, 0, d], 2 * x[0, 0, c]
        assert np.allclose(y[0, 0], want)
    assert ref8.depths([0, 3, 3, 5], np.array([-1, 0, 0, -1, -1])).tolist() == [0, 1, 1, 0, 0]
    assert ref8.depths([0, 3], None).tolist() == [0, 1, 2]


def cache(n=4, width=8, pages=6, per_page=1, **more):
    k = put(torch.zeros(pages, 2, 16, 64).to(torch.float8_e4m3fn))
    x = dict(k=k, v=put(torch.zeros(pages, 2, 16, 64).to(torch.float8_e4m3fn)), k_scale=put(torch.ones(pages, 2, per_page)),
             v_scale=put(torch.ones(pages, 2, per_page)), table=put(torch.zeros(n, width, dtype=torch.int32)),
             length=put(torch.zeros(n, dtype=torch.int32)))
    x.update(more)
    return x


def test_make_kv8(W):
    c = cache()
    kv = W.make_kv8(**c)
    assert (kv.k, kv.v, kv.k_scale, kv.v_scale) == tuple(c[x].data_ptr() for x in ("k", "v", "k_scale", "v_scale"))
    assert (kv.page_stride, kv.head_stride, kv.token_stride, kv.block, kv.pages) == (2048, 1024, 64, 16, 6)
    wide = put(torch.zeros(6, 16, 2, 64).to(torch.float8_e4m3fn).transpose(1, 2))
    kv = W.make_kv8(**cache(k=wide, v=put(wide.clone())))
    assert (kv.page_stride, kv.head_stride, kv.token_stride) == (2048, 64, 128)
    z = torch.zeros
    for bad, kind in ((dict(k=put(z(6, 2, 16, 64, dtype=torch.bfloat16))), TypeError), (dict(v=put(z(6, 2, 16, 64))), TypeError),
                      (dict(k=z(6, 2, 16, 64).to(torch.float8_e4m3fn)), TypeError), (dict(k_scale=put(z(6, 2, 1).double())), TypeError),
                      (dict(k_scale=put(z(6, 2))), ValueError), (dict(k_scale=put(z(6, 1, 1))), ValueError),
                      (dict(v_scale=put(z(6, 2, 2))), ValueError), (dict(k_scale=put(z(6, 2, 3)), v_scale=put(z(6, 2, 3))), ValueError),
                      (dict(k_scale=put(z(6, 2, 0)), v_scale=put(z(6, 2, 0))), ValueError),
                      (dict(length=put(z(3, dtype=torch.int32))), ValueError), (dict(next_pos=put(z(4, dtype=torch.int64))), TypeError),
                      (dict(table=put(z(1, 8, dtype=torch.int32)).expand(4, -1)), ValueError), (dict(k=None), ValueError)):
        with pytest.raises(kind):
            W.make_kv8(**cache(**bad))


@pytest.fixture
def worker(W):
    w = W.Worker.__new__(W.Worker)
    w.handle = None
    w.device = torch.device("cpu")
    w.calls = []
    w._call = lambda name, *args: w.calls.append((name,) + args)
    w.dtype, w.q_heads, w.kv_heads, w.head_dim, w.page_tokens = torch.bfloat16, 4, 2, 64, 16
    w._kv_shape, w._kv8_shape = (torch.bfloat16, 2, 16, 64), ("e4m3", 2, 16, 64)
    w._tok_shape, w._tok_bare = (torch.bfloat16, 4, 2, 64), (torch.bfloat16, 0, 2, 64)
    return w


def tokens(W, n=4, q=True):
    x = put(torch.zeros(n, 8, 64, dtype=torch.bfloat16))
    return W.make_tokens(put(torch.zeros(5, dtype=torch.int32)), x[:, :4] if q else None, x[:, 4:6], x[:, 6:]), x


def test_calls_go_by_the_kind_of_cache(W, worker):
    kv8 = W.make_kv8(**cache())
    tok, _ = tokens(W)
    k = put(torch.zeros(6, 2, 16, 64, dtype=torch.bfloat16))
    kv = W.make_kv(k, put(k.clone()), cache()["table"], cache()["length"])
    for c in (kv, kv8):
        worker.attend(c, tok)
        worker.append(c, tok)
    assert [c[0] for c in worker.calls] == ["aladdin_worker_attend", "aladdin_worker_append", "aladdin_worker_attend8",
                                            "aladdin_worker_append8"]
    # a pool of 8 bits without scales is none of both, and weights are kept beside 16 bits only
    raw = W.make_kv(cache()["k"], cache()["v"], cache()["table"], cache()["length"])
    for call in (lambda: worker.attend(raw, tok), lambda: worker.append(raw, tok), lambda: worker.accept(kv8, tok),
                 lambda: worker.evict(kv8, cache()["length"])):
        with pytest.raises(ValueError):
            call()
    assert len(worker.calls) == 4


def test_rotate_arguments(W, worker):
    tok, x = tokens(W)
    rope = W.A.aladdin_rope(64, 0, 1.0, 0)
    q, k = worker.rotate(rope, tok)
    assert q.shape == (4, 4, 64) and k.shape == (4, 2, 64)
    q, k = worker.rotate(rope, tok, q_out=x[:, :4], k_out=False)
    assert k is None and worker.calls[-1][5:] == (x.data_ptr(), 8 * 64, None, 2 * 64)
    bare, _ = tokens(W, q=False)
    assert worker.rotate(rope, bare, q_out=False)[0] is None
    ints = lambda n: put(torch.zeros(n, dtype=torch.int32))
    worker.rotate(rope, tok, ints(4), ints(4))
    seen = len(worker.calls)
    for bad in (dict(next_pos=ints(5)), dict(pos=ints(3)), dict(q_out=x[:, :3]), dict(k_out=x[:3, 4:6]), dict(k_out=x[:, 4:8:2])):
        with pytest.raises(ValueError):
            worker.rotate(rope, tok, **bad)
    for bad in (dict(next_pos=ints(4).long()), dict(pos=ints(4).float()), dict(q_out=x[:, :4].float())):
        with pytest.raises(TypeError):
            worker.rotate(rope, tok, **bad)
    with pytest.raises(ValueError):
        worker.rotate(rope, bare)
    assert len(worker.calls) == seen


def test_make_rope_refusals(W):
    for bad in (dict(layout="pairs"), dict(scaling="ntk"), dict(dim=5), dict(dim=0), dict(scaling="parts", factor=2.0),
                dict(freq=[1.0, 0.5]), dict(freq=[1.0] * 4, scaling="linear")):
        with pytest.raises(ValueError):
            W.make_rope(**{"dim": 8, "device": "cpu", **bad})
    r = W.make_rope(8, freq=[1.0, 0.5, 0.25, 0.0], scale=2.0, device="cpu")
    assert (r.dim, r.layout, r.scale) == (8, 0, 2.0) and r._keep.tolist()[3] == 0
    r = W.make_rope(8, layout="interleaved", scaling="parts", factor=8.0, original=4096, device="cpu")
    assert r.layout == 1 and abs(r.scale - (0.1 * math.log(8.0) + 1.0)) < 1e-6
