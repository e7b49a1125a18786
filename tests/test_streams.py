"""Calls on another stream than the current one: whose memory the results are, and who is told that tensors are in use (with stand-ins for
torch's streams: no GPU)."""
import contextlib

import pytest
import torch

import paper_2512_08537_b200 as ardiff


class Stream:
    def __init__(self, handle, device_index=0):
        self.cuda_stream, self.device_index = handle, device_index


class Tensor:
    device = "cuda:?"

    def __init__(self, index=0):
        self.index, self.seen = index, []

    def get_device(self):
        return self.index

    def record_stream(self, stream):
        self.seen.append(stream.cuda_stream)


@pytest.fixture
def current(monkeypatch):
    """The handle of the current stream, in a list: 5, or what `with torch.cuda.stream` makes it."""
    now = [5]

    @contextlib.contextmanager
    def switch(stream):
        now.append(stream.cuda_stream)
        yield
        now.pop()
    monkeypatch.setattr(torch.cuda, "stream", switch)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda index=None: Stream(now[-1]))
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda index: now[-1], raising=False)
    return now


def test_results_are_made_on_the_stream_and_all_tensors_marked(current):
    a, b, made = Tensor(), Tensor(), Tensor()
    where = []

    def call(x, number, y, nothing):
        where.append(current[-1])
        return made, None, y
    out = ardiff._beside(call, Stream(9), a, 3, b, None)
    assert out == (made, None, b) and where == [9] and current == [5]
    assert a.seen == [9] and b.seen == [9, 5] and made.seen == [5]
    assert ardiff._beside(lambda x: made, Stream(9), a) is made


def test_the_current_stream_itself_changes_nothing(current):
    a, made = Tensor(), Tensor()
    assert ardiff._beside(lambda x: made, Stream(5), a) is made
    assert a.seen == [] and made.seen == []


def test_a_stream_of_another_device_is_refused(current):
    with pytest.raises(AssertionError):
        ardiff._beside(lambda x: x, Stream(9, device_index=1), Tensor(0))
    with pytest.raises(AssertionError):
        ardiff.ardiff_sample_tokens(torch.zeros((4, 8)), torch.zeros(4), stream=Stream(9))


def test_every_call_that_allocates_goes_that_way(current, monkeypatch):
    seen = []
    monkeypatch.setattr(ardiff, "_beside", lambda fn, stream, *args: seen.append((fn.__name__, len(args))))
    t = Tensor()
    for fn, n in ((ardiff.ardiff_entropy_gate, 2), (ardiff.ardiff_entropy_gate_stats, 1), (ardiff.ardiff_entropy_gate_blocks, 4),
                  (ardiff.ardiff_tau_calibrate, 1), (ardiff.ardiff_accept_prefix, 3), (ardiff.ardiff_sample_tokens, 2),
                  (ardiff.ardiff_pages_extend, 7), (ardiff.ardiff_pages_truncate, 6), (ardiff.ardiff_distill_topk, 3),
                  (ardiff.ardiff_distill_topk_backward, 5), (ardiff.ardiff_distill_topk_step, 4)):
        fn(*[t] * n, stream=Stream(9))
        # every parameter but the stream is passed on, in order
        assert seen.pop() == (fn.__name__, fn.__code__.co_argcount - 1)
