"""Rounds of speculation with the draft model's operators around the gate, as a decoder runs them: the cache is extended by a
draft block a request, its tokens are drawn, the gate ends blocks early, the verification accepts prefixes, the rest is taken back.
Nothing is read on the host between the calls, so a round can be captured into one graph."""
import numpy as np
import pytest
import torch

import paper_2512_08537_b200 as ardiff
from gpu_util import require_cuda

pytestmark = pytest.mark.gpu
R, GAMMA, PAGE, WIDTH, V, D = 13, 5, 8, 12, 3001, 256


class Round:
    def __init__(self):
        d = require_cuda()
        z = lambda *s, t=torch.int32: torch.zeros(s, dtype=t, device=d)  # noqa: E731
        self.length, self.count, self.status = z(R), torch.full((1,), R * WIDTH, dtype=torch.int32, device=d), z(2)
        self.table = torch.full((R, WIDTH), -1, dtype=torch.int32, device=d)
        self.free = torch.randperm(R * WIDTH, device=d).to(torch.int32)
        self.add = torch.full((R,), GAMMA, dtype=torch.int32, device=d)
        self.slot, self.position, self.request = z(R * GAMMA, t=torch.int64), z(R * GAMMA), z(R * GAMMA)
        self.offset, self.after = z(R + 1), z(R)
        self.q = z(R * GAMMA, V, t=torch.bfloat16)
        self.p = z(R * GAMMA, V, t=torch.bfloat16)
        self.feat = z(R * GAMMA, D, t=torch.bfloat16)
        self.u, self.r = z(R * GAMMA, t=torch.float32), z(R * GAMMA, t=torch.float32)
        self.T = torch.full((R * GAMMA,), 0.9, device=d)
        self.top_k = torch.full((R * GAMMA,), 40, dtype=torch.int32, device=d)

    def inputs(self, seed):
        g = torch.Generator(device=self.q.device).manual_seed(seed)
        self.q.copy_(2.5 * torch.randn(self.q.shape, device=self.q.device, generator=g))
        self.p.copy_(self.q + 0.3 * torch.randn(self.q.shape, device=self.q.device, generator=g))
        self.feat.copy_(torch.randn(self.feat.shape, device=self.q.device, generator=g))
        self.u.copy_(torch.rand(self.u.shape, device=self.q.device, generator=g))
        self.r.copy_(torch.rand(self.r.shape, device=self.q.device, generator=g))

    def run(self, tau):
        ardiff.ardiff_pages_extend(self.length, self.add, self.table, self.free, self.count, PAGE, self.slot, self.position,
                                   self.request, self.offset, self.after, self.count, self.status[:1])
        self.token, self.logq = ardiff.ardiff_sample_tokens(self.q, self.u, self.T, self.top_k)
        _, _, _, self.block_len, _, _ = ardiff.ardiff_entropy_gate_blocks(self.feat, 1, GAMMA, tau)
        logp = torch.log_softmax(self.p.float() / 0.9, 1).gather(1, self.token.long()[:, None])[:, 0]
        self.ratio = torch.exp(logp - self.logq)
        self.accepted = ardiff.ardiff_accept_prefix(self.r, self.ratio, GAMMA, self.block_len)
        target = self.length + self.accepted
        ardiff.ardiff_pages_truncate(self.after, target, self.table, self.free, self.count, PAGE, self.count, self.status[1:])
        self.length.copy_(target)


def check_round(s, length0):
    """What must hold after a round, whatever was drawn."""
    assert s.status.tolist() == [0, 0]
    accepted, block_len = s.accepted.tolist(), s.block_len.tolist()
    r, ratio = s.r.tolist(), s.ratio.tolist()
    for b in range(R):
        n = 0
        while n < block_len[b] and not r[b * GAMMA + n] > ratio[b * GAMMA + n]:
            n += 1
        assert accepted[b] == n
    length = s.length.tolist()
    assert length == [a + b for a, b in zip(length0, accepted)]
    assert s.offset.tolist() == [GAMMA * i for i in range(R + 1)]
    assert s.position.tolist() == [length0[i // GAMMA] + i % GAMMA for i in range(R * GAMMA)]
    held = [-(-n // PAGE) for n in length]
    assert int(s.count) == R * WIDTH - sum(held)
    pages = [v for row, h in zip(s.table.tolist(), held) for v in row[:h]] + s.free[:int(s.count)].tolist()
    assert sorted(pages) == list(range(R * WIDTH))             # every page held once or free
    assert bool((s.token >= 0).all()) and bool((s.token < V).all()) and bool((s.logq <= 0).all())


def test_rounds_of_speculation_with_the_gate():
    torch.manual_seed(0)
    s = Round()
    for step in range(8):
        s.inputs(step)
        before = s.length.tolist()
        s.run(tau=5.0)
        check_round(s, before)
    assert max(s.length.tolist()) > 0


def test_a_captured_round_replays_like_the_same_calls():
    torch.manual_seed(1)
    a, b = Round(), Round()
    b.free.copy_(a.free)
    a.inputs(100)
    a.run(tau=5.0)                                             # loads the kernels
    b.inputs(100)
    b.run(tau=5.0)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        b.run(tau=5.0)
    for step in range(4):
        a.inputs(step)
        b.inputs(step)
        before = a.length.tolist()
        a.run(tau=5.0)
        graph.replay()
        torch.cuda.synchronize()
        check_round(a, before)
        for name in ("length", "table", "free", "count", "slot", "position", "request", "offset", "token", "logq", "accepted"):
            assert torch.equal(getattr(a, name), getattr(b, name)), (step, name)


def test_the_draft_learns_from_the_rows_it_draws_from():
    """The target's largest logits of a round's rows, and a step of the draft's logits against them: entries, loss and gradient come
    from the same rows that sampling reads, in place in a wider buffer."""
    s = Round()
    s.inputs(3)
    teacher, ids = s.p.float().topk(32, dim=1)
    weight = torch.full((R * GAMMA,), 1.0 / (R * GAMMA), device=s.q.device)
    loss, _, grad = ardiff.ardiff_distill_topk_step(s.q, teacher, ids.to(torch.int32), weight, 0.9)
    assert bool((loss >= 0).all()) and bool(torch.isfinite(grad).all())
    # the gradient of a row sums to 0 (both sides are distributions): V roundings of bf16 to half a step each
    total = grad.double().sum(1).abs()
    assert bool((total <= grad.double().abs().sum(1) * 2.0 ** -8).all())
    token, _ = ardiff.ardiff_sample_tokens(s.q, s.u, s.T, s.top_k)
    assert np.all(token.cpu().numpy() >= 0)


def test_kernels_launched_early_read_what_the_kernel_before_them_wrote():
    """A step of the distillation writes its gradient in the place of the logits, and lets the next kernel start at once; that one reads them.
    Small and large rows, on one stream and in a captured graph, against the same calls one at a time."""
    d = require_cuda()
    for n, width, k in ((4, 1001, 8), (64, 40000, 32), (700, 9000, 16)):
        g = torch.Generator(device=d).manual_seed(n)
        x0 = (4 * torch.randn((n, width), device=d, generator=g)).to(torch.bfloat16)
        teacher, ids = (x0.float() + 0.5 * torch.randn((n, width), device=d, generator=g)).topk(k, dim=1)
        ids = ids.to(torch.int32)
        weight = 50.0 + torch.rand((n,), device=d, generator=g)
        u = torch.rand((n,), device=d, generator=g)
        top_p = torch.full((n,), 0.95, device=d)
        x, out = x0.clone(), {}

        def calls(wait):
            wait()
            out["loss"], _, _ = ardiff.ardiff_distill_topk_step(x, teacher, ids, weight, grad=x)
            wait()
            out["token"], out["logprob"] = ardiff.ardiff_sample_tokens(x, u, top_p=top_p)
            wait()
            out["loss 2"], out["stats"], _ = ardiff.ardiff_distill_topk_step(x, teacher, ids, weight, 0.5, grad=x)
            wait()
            out["loss 3"], _ = ardiff.ardiff_distill_topk(x, teacher, ids, 2.0)
            wait()
            out["back"] = ardiff.ardiff_distill_topk_backward(x, teacher, ids, out["stats"], weight, grad=x).clone()

        calls(torch.cuda.synchronize)
        want = {name: v.clone() for name, v in out.items()}
        for _ in range(5):
            x.copy_(x0)
            calls(lambda: None)
            for name, v in want.items():
                assert torch.equal(out[name], v), (n, name)
        graph = torch.cuda.CUDAGraph()
        torch.cuda.synchronize()
        with torch.cuda.graph(graph):
            calls(lambda: None)
        for _ in range(5):
            x.copy_(x0)
            graph.replay()
            for name, v in want.items():
                assert torch.equal(out[name], v), (n, name)
