"""What the worker's torch layer hands to the library, on the host: tensors that say that they are on a GPU, and a
call that is recorded in place of the library's."""
import pytest
import torch


class OnGpu(torch.Tensor):
    is_cuda = property(lambda self: True)


def put(x):
    return x.as_subclass(OnGpu)


@pytest.fixture(scope="module")
def W():
    from paper_2405_06856_gb300 import build
    build.build()
    from paper_2405_06856_gb300 import worker
    return worker


@pytest.fixture
def worker(W):
    w = W.Worker.__new__(W.Worker)
    w.handle = None
    w.device = torch.device("cpu")
    w.calls = []
    w._call = lambda name, *args: w.calls.append(args)
    w._kv_shape = (torch.bfloat16, 2, 16, 64)
    return w


def test_rows_of_logits_keep_their_stride(worker):
    x = put(torch.zeros(4, 40))
    for logits, stride in ((x, 40), (x[:, :33], 40), (x[::2], 80), (x[:1], 40), (x[:1].expand(1, -1), 40),
                           (put(torch.zeros(40)).as_strided((1, 40), (3, 1)), 40)):
        worker.logprobs(logits)
        n, vocab, at, got = worker.calls[-1][1:5]
        assert (n, vocab, at) == (*logits.shape, logits.data_ptr()) and got == (stride if n > 1 else vocab)
    seen = len(worker.calls)
    # rows that share memory have a stride below their width: read with another one they would lie outside
    for logits in (x[:1].expand(8, -1), x.as_strided((3, 40), (39, 1)), put(torch.zeros(1, 1)).expand(2, 1)):
        with pytest.raises(ValueError, match="rows"):
            worker.logprobs(logits)
    assert len(worker.calls) == seen


def cache(n, width, pages=6):
    k = put(torch.zeros(pages, 2, 16, 64, dtype=torch.bfloat16))
    table = put(torch.zeros(n, width, dtype=torch.int32))
    length = put(torch.zeros(n, dtype=torch.int32))
    return k, table, length


def test_rows_of_the_page_table_keep_their_stride(W):
    k, table, length = cache(4, 8)
    for t, stride in ((table, 8), (table[:, :5], 8), (table[:, 3:], 8), (table[:, :1], 8)):
        kv = W.make_kv(k, k.clone(), t, length)
        assert (kv.table, kv.table_width, kv.table_stride) == (t.data_ptr(), t.shape[1], stride)
    kv = W.make_kv(k, k.clone(), table[:1].expand(1, -1), length[:1])
    assert kv.table_stride == 8
    # requests that share their pages by one row of the table: read with the row's width they would lie outside
    for t in (table[:1].expand(4, -1), table[:1, :1].expand(4, 1), table.as_strided((4, 8), (7, 1))):
        with pytest.raises(ValueError, match="table"):
            W.make_kv(k, k.clone(), t, length)


def test_numbers_that_32_bits_do_not_hold(W, worker):
    """The library's arguments are 32-bit: others are refused, not cut down to what they hold."""
    k, table, length = cache(4, 8)
    zeros = lambda t: put(torch.zeros(6, 2, 16, dtype=t))
    kv = W.make_kv(k, k.clone(), table, length, zeros(torch.float32), zeros(torch.int32), put(length.clone()))
    worker.evict(kv, length, 2 ** 31 - 1)
    assert worker.calls[-1][-1] == 2 ** 31 - 1
    x = put(torch.zeros(2, 40))
    worker.logprobs(x, None, 3)
    assert len(worker.calls) == 2
    for recent in (2 ** 31, 2 ** 32, 2 ** 40 + 7, -1):
        with pytest.raises(ValueError, match="recent"):
            worker.evict(kv, length, recent)
    for top in (2 ** 32 + 3, 2 ** 31, -1):
        with pytest.raises(ValueError, match="top"):
            worker.logprobs(x[:0], None, top)
    assert len(worker.calls) == 2
