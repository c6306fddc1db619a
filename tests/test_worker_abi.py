"""The worker step's C ABI on the host: struct layouts and refusals that need no GPU."""
import ctypes

import numpy as np
import pytest

import worker_ref as ref


@pytest.fixture(scope="module")
def lib():
    from paper_2405_06856_gb300 import build
    build.build()
    from paper_2405_06856_gb300 import aladdin as A
    return A


def test_struct_layout(lib):
    assert ctypes.sizeof(lib.aladdin_worker_shape) == 20
    assert ctypes.sizeof(lib.aladdin_kv) == 2 * 8 + 3 * 8 + 2 * 4 + 8 + 5 * 8
    assert lib.aladdin_kv.table.offset == 56 and lib.aladdin_kv.next.offset == 88
    assert ctypes.sizeof(lib.aladdin_tokens) == 2 * 4 + 5 * 8 + 3 * 8
    assert lib.aladdin_tokens.q_stride.offset == 48


@pytest.mark.parametrize("bad", [(2, 8, 2, 64, 16), (-1, 8, 2, 64, 16), (0, 0, 1, 64, 16), (0, 8, 0, 64, 16),
                                 (0, 8, 3, 64, 16), (0, 2048, 2, 64, 16), (0, 8, 2, 80, 16), (0, 8, 2, 0, 16),
                                 (0, 8, 2, 64, 8), (0, 8, 2, 64, 48), (0, 8, 2, 64, 512), (0, 2, 8, 64, 16)])
def test_create_rejects_bad_shapes(lib, bad):
    h = ctypes.c_void_p(5)
    s = lib.aladdin_worker_shape(*bad)
    assert lib._lib.aladdin_worker_create(ctypes.byref(s), None, ctypes.byref(h)) == lib.ERR_ARG and not h.value


def test_null_arguments(lib):
    L = lib._lib
    s = lib.aladdin_worker_shape(0, 8, 2, 64, 16)
    assert L.aladdin_worker_create(ctypes.byref(s), None, None) == lib.ERR_ARG
    h = ctypes.c_void_p()
    assert L.aladdin_worker_create(None, None, ctypes.byref(h)) == lib.ERR_ARG
    assert L.aladdin_worker_destroy(None) == lib.ERR_ARG
    assert L.aladdin_worker_status(None) == lib.ERR_ARG
    assert L.aladdin_worker_attend(None, None, None, 1.0, None, 0, None) == lib.ERR_ARG
    assert L.aladdin_worker_accept(None, None, None, 1.0, None, None, None, 0) == lib.ERR_ARG
    assert L.aladdin_worker_evict(None, None, 0, None, 0) == lib.ERR_ARG
    assert L.aladdin_worker_logprobs(None, 0, 0, 1, None, 0, None, 0, None, None, None, None, None) == lib.ERR_ARG


def test_reference_attention_by_hand():
    """Two cached tokens and a tree of three whose softmax is known: equal scores give plain means."""
    case = dict(page=16, table=np.zeros((1, 1), np.int32), len=[2], off=[0, 3], parent=np.array([-1, 0, -1]),
                scale=0.5, k=np.zeros((1, 1, 16, 4)), v=np.zeros((1, 1, 16, 4)), q=np.ones((3, 1, 4)),
                k_new=np.zeros((3, 1, 4)), v_new=np.arange(12.0).reshape(3, 1, 4))
    case["v"][0, 0, :2] = [[1, 1, 1, 1], [3, 3, 3, 3]]
    out, lse = ref.attend(case)
    v = case["v_new"][:, 0]
    assert np.allclose(out[0, 0], (4 + v[0]) / 3) and np.allclose(out[1, 0], (4 + v[0] + v[1]) / 4)
    assert np.allclose(out[2, 0], (4 + v[2]) / 3) and np.allclose(lse[:, 0], np.log([3, 4, 3]))


def test_reference_eviction_by_hand():
    case = dict(page=16, table=np.zeros((1, 1), np.int32), len=[6], next=[6],
                k=np.arange(16.0).reshape(1, 1, 16, 1), v=-np.arange(16.0).reshape(1, 1, 16, 1),
                weight=np.array([1, 5, 2, 2, 0.5, 0] + [0] * 10, np.float32).reshape(1, 1, 16),
                pos=np.arange(16, dtype=np.int32).reshape(1, 1, 16))
    k, v, weight, pos, length = ref.evict(case, [3], 1)
    # slot 5 is recent, slot 1 has 5, slots 2 and 3 have 2: the lower one stays; slot 5 moves into slot 0
    assert k[0, 0, :3, 0].tolist() == [5, 1, 2] and v[0, 0, :3, 0].tolist() == [-5, -1, -2]
    assert weight[0, 0, :3].tolist() == [0, 5, 2] and pos[0, 0, :3].tolist() == [5, 1, 2] and length == [3]


def test_reference_logprobs_by_hand():
    lp, ent, rank, ids, tlp = ref.logprobs(np.log(np.array([[0.5, 0.25, 0.25], [0.2, 0.2, 0.6]])), [2, 0], 2)
    assert np.allclose(lp, np.log([0.25, 0.2])) and rank.tolist() == [2, 0 + 1]
    assert np.allclose(ent[0], 1.5 * np.log(2)) and ids.tolist() == [[0, 1], [2, 0]]
    assert np.allclose(tlp, np.log([[0.5, 0.25], [0.6, 0.2]]))
