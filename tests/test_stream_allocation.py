"""Where the calls on a given stream allocate, without a GPU: results and workspace come from that
stream's part of the caching allocator.  On the current stream's part they could be a block that work
pending on the current stream still writes.  (Tensors are the CPU's, said to be on a GPU; the library is
asked for sizes only.)"""
import contextlib

import pytest
import torch

from paper_2609_04910_amd import attention as at
from paper_2609_04910_amd import gauss_sum as gs

H = torch.float16


class Stream:
    cuda_stream = 7
    device = torch.device("cpu")               # the tensors'


@pytest.fixture
def where(monkeypatch):
    """The handle of the stream on which each allocation was made, in turn."""
    current, seen, empty = [0], [], torch.empty

    @contextlib.contextmanager
    def switch(stream):
        before, current[0] = current[0], stream.cuda_stream
        yield
        current[0] = before

    def allocate(*args, **kw):
        seen.append(current[0])
        return empty(*args, **kw)

    real = gs.load()

    class Sizes:
        def __getattr__(self, name):
            return getattr(real, name) if name.endswith("_size") else lambda *args: 0

    monkeypatch.setattr(torch.cuda, "stream", switch)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda *args: Stream())
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda device: current[0], raising=False)
    monkeypatch.setattr(torch.Tensor, "is_cuda", property(lambda self: True))
    monkeypatch.setattr(torch.Tensor, "record_stream", lambda self, stream: None)
    monkeypatch.setattr(torch, "empty", allocate)
    monkeypatch.setattr(at, "_launch", lambda *args: None)
    monkeypatch.setattr(gs, "load", lambda *args: Sizes())
    return seen


def z(*shape, dtype=H):
    return torch.zeros(shape, dtype=dtype)


def i32(*x):
    return torch.tensor(x, dtype=torch.int32)


QKV = (z(1, 5, 2, 64), z(1, 5000, 2, 64), z(1, 5000, 2, 64))
PAGES = (z(8, 64, 2, 64), z(8, 64, 2, 64))
ATTENTION = {
    "fwd": (lambda **kw: at.attention_fwd(*QKV, **kw), 3),
    "bwd": (lambda **kw: at.attention_bwd(*QKV, QKV[0], torch.zeros(1, 2, 5), QKV[0], **kw), 4),
    "paged": (lambda **kw: at.attention_paged(z(1, 2, 64), *PAGES, torch.zeros((1, 99), dtype=torch.int32), i32(9),
                                              return_lse=True, **kw), 3),
    "paged, no sequences": (lambda **kw: at.attention_paged(z(2, 2, 64), *PAGES, torch.zeros((0, 9), dtype=torch.int32),
                                                            i32(), q_offsets=i32(0), return_lse=True, **kw), 2),
}


@pytest.mark.parametrize("name", ATTENTION)
def test_attention_allocates_on_the_given_stream(where, name):
    call, count = ATTENTION[name]
    call(stream=Stream())
    n = len(where)
    assert n >= count and where == [7] * n
    del where[:]
    call()
    assert where == [0] * n


X, V = z(40, 16), torch.zeros(40, 3)
XB, VB = z(2, 40, 16), torch.zeros(2, 40, 3)
GAUSS = {
    "fwd": lambda **kw: gs.gauss_sum_fwd(X, X, V, 1.0, **kw),
    "bwd": lambda **kw: gs.gauss_sum_bwd(X, X, V, 1.0, V, **kw),
    "fwd_bwd": lambda **kw: gs.gauss_sum_fwd_bwd(X, X, V, 1.0, V, **kw),
    "fwd_batched": lambda **kw: gs.gauss_sum_fwd_batched(XB, XB, VB, 1.0, **kw),
    "bwd_batched": lambda **kw: gs.gauss_sum_bwd_batched(XB, XB, VB, 1.0, VB, **kw),
    "fwd_bwd_batched": lambda **kw: gs.gauss_sum_fwd_bwd_batched(XB, XB, VB, 1.0, VB, **kw),
    "mmd_flow": lambda **kw: gs.gauss_sum_mmd_flow(X, V[:, :1].contiguous(), 1.0, **kw),
    "svgd": lambda **kw: gs.gauss_sum_svgd(X, torch.zeros(40, 16), 1.0, **kw),
}


@pytest.mark.parametrize("name", GAUSS)
def test_gauss_sums_allocate_on_the_given_stream(where, name):
    GAUSS[name](stream=Stream())
    assert where and set(where) == {7}
    n = len(where)
    del where[:]
    GAUSS[name]()
    assert where == [0] * n


def test_attention_refuses_a_stream_of_another_gpu(where):
    other = Stream()
    other.device = torch.device("cuda", 1)
    table, lens = torch.zeros((1, 9), dtype=torch.int32), i32(9)
    for call in [call for call, _ in ATTENTION.values()] + [
            lambda **kw: at.attention_append(z(1, 2, 64), z(1, 2, 64), *PAGES, table, lens, **kw)]:
        with pytest.raises(ValueError, match="stream must be on"):
            call(stream=other)
    assert not where
