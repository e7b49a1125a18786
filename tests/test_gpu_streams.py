"""Calls on another stream than the current one, whose tensors are dropped while they run."""
import pytest
import torch

import paper_2512_08537_b200 as ardiff
from gpu_util import require_cuda

pytestmark = pytest.mark.gpu


def make():
    d = require_cuda()
    g = torch.Generator(device=d).manual_seed(3)
    x = torch.randn((64, 9000), device=d, generator=g).to(torch.bfloat16)
    teacher, ids = x.float().topk(16, dim=1)
    length = torch.full((64,), 40, dtype=torch.int32, device=d)
    return dict(x=x, u=torch.rand((64,), device=d, generator=g), teacher=teacher, ids=ids.to(torch.int32), weight=torch.ones(64, device=d),
                stats=torch.zeros((64, 2), device=d), length=length, add=torch.full_like(length, 5), target=length - 20,
                table=torch.arange(64 * 8, dtype=torch.int32, device=d).reshape(64, 8),
                free=torch.arange(512, 1536, dtype=torch.int32, device=d), count=torch.full((1,), 600, dtype=torch.int32, device=d),
                slot=torch.zeros(400, dtype=torch.int64, device=d), feat=torch.randn((960, 256), device=d, generator=g).to(torch.bfloat16),
                entropy=torch.rand(960, device=d, generator=g), r=torch.rand(960, device=d, generator=g))


# a call, and which of the tensors above it takes, in order
CALLS = {
    "sample": (lambda s, *t: ardiff.ardiff_sample_tokens(*t, stream=s), "x u"),
    "distill": (lambda s, *t: ardiff.ardiff_distill_topk(*t, stream=s), "x teacher ids"),
    "distill_backward": (lambda s, *t: ardiff.ardiff_distill_topk_backward(*t, stream=s), "x teacher ids stats weight"),
    "distill_step": (lambda s, *t: ardiff.ardiff_distill_topk_step(*t, stream=s), "x teacher ids weight"),
    "extend": (lambda s, *t: ardiff.ardiff_pages_extend(*t[:5], 16, t[5], stream=s), "length add table free count slot"),
    "truncate": (lambda s, *t: ardiff.ardiff_pages_truncate(*t, 16, stream=s), "length target table free count"),
    "gate": (lambda s, *t: ardiff.ardiff_entropy_gate(*t, 5.0, want_entropy=True, stream=s), "feat"),
    "gate_stats": (lambda s, *t: ardiff.ardiff_entropy_gate_stats(*t, 5.0, stream=s), "feat"),
    "gate_blocks": (lambda s, *t: ardiff.ardiff_entropy_gate_blocks(*t, 1, 5, 5.0, stream=s), "feat"),
    "calibrate": (lambda s, *t: ardiff.ardiff_tau_calibrate(*t, stream=s), "entropy"),
    "accept": (lambda s, *t: ardiff.ardiff_accept_prefix(*t, 5, stream=s), "r entropy"),
}


def results(out):
    """A call's results, in full: of the ascending ids of a gate only their number is."""
    out = [v for v in (out if isinstance(out, tuple) else (out,)) if v is not None]
    return out, [i for i, v in enumerate(out) if not (i == 1 and out[0].dtype is torch.uint8)]


@pytest.mark.parametrize("name", sorted(CALLS))
def test_no_memory_is_given_out_while_a_call_on_another_stream_uses_it(name):
    """The other stream is kept busy for a tenth of a second in front of the call; meanwhile inputs and results are dropped and as
    much is allocated and written on the current stream."""
    call, takes = CALLS[name]
    want, whole = results(call(None, *[make()[k] for k in takes.split()]))
    kept = [torch.empty_like(v, device="cpu").pin_memory() for v in want]
    side = torch.cuda.Stream()
    for cycles in (1000, 200_000_000):                           # the first time loads kernels and gets memory, which may wait for all streams
        t = (lambda m: [m[k] for k in takes.split()])(make())
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            torch.cuda._sleep(cycles)
        out, _ = results(call(side, *t))
        with torch.cuda.stream(side):
            for k, v in zip(kept, out):
                k.copy_(v, non_blocking=True)
        used = t + out
        places, sizes = {v.data_ptr() for v in used}, [v.numel() * v.element_size() for v in used]
        del t, out, used, v
        others = [torch.full((n,), 255, dtype=torch.uint8, device="cuda") for n in sizes for _ in range(2)]
        running = not side.query()
        torch.cuda.synchronize()
    assert running                                               # nothing of it had run yet
    assert not places & {o.data_ptr() for o in others}
    for i in whole:
        assert torch.equal(kept[i], want[i].cpu()), i


def test_a_captured_graph_with_a_call_on_a_second_stream():
    """The call lies on a branch of the graph; its results are the graph's memory and follow the inputs at every replay."""
    t = make()
    x, u = t["x"], t["u"]
    side = torch.cuda.Stream()
    want = [v.clone() for v in ardiff.ardiff_sample_tokens(x, u, stream=side)]
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        here = torch.cuda.current_stream()
        side.wait_stream(here)
        token, logprob = ardiff.ardiff_sample_tokens(x, u, stream=side)
        ardiff.ardiff_entropy_gate_stats(t["feat"], 5.0, stream=side)          # dropped at once
        here.wait_stream(side)
        twice = 2 * token
    x0 = x.clone()
    for flip in (False, True, False):
        x.copy_(x0.flip(0) if flip else x0)
        graph.replay()
        again = want if not flip else ardiff.ardiff_sample_tokens(x, u)
        torch.cuda.synchronize()
        assert torch.equal(token, again[0]) and torch.equal(logprob, again[1]) and torch.equal(twice, 2 * again[0])
