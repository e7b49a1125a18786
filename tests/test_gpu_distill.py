"""Distillation from a teacher's largest logits against the definition in 64 bits, through the C ABI.

Tolerances count roundings (u = 2^-24, half a step of fp32). With y = (x - m) / T and e = exp(y): the subtraction, the constant
log2(e) / T and the product with it are off by u each, 3 u |y| in the exponent; ex2.approx by 2^-22 = 4 u; so e is off by
e (4 + 3 |y|) u. Z adds to the mean of these, under the weights e, one rounding for each term that a thread adds (at most
V / 512 + 8, with a few rescalings) and for each of the merges behind them (each with another ex2): 64 u cover those. ln Z is off by
what Z is off by, and by the rounding of the stored number. The teacher's side has expf and logf (2 u) and the same exponent."""
import math

import numpy as np
import pytest
import torch

import paper_2512_08537_b200 as ardiff
from gpu_util import require_cuda

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}


def make(n, V, k, dtype, seed, spread=3.0, pad=0, teacher_dtype=torch.float32, offset=0):
    g = torch.Generator().manual_seed(seed)
    buf = torch.zeros(n * (V + pad) + offset, dtype=dtype)
    x = buf[offset:].reshape(n, V + pad)[:, :V]
    x.copy_((spread * torch.randn((n, V), generator=g)).to(dtype))
    ids = torch.stack([torch.randperm(V, generator=g)[:k] for _ in range(n)]).to(torch.int32) if k <= V else \
        torch.randint(0, V, (n, k), generator=g, dtype=torch.int32)
    teacher = (2.0 + spread * torch.randn((n, k), generator=g)).to(teacher_dtype)
    weight = 0.25 + torch.rand((n,), generator=g)
    d = require_cuda()
    xd = buf.to(d)[offset:].reshape(n, V + pad)[:, :V]
    return xd, teacher.to(d), ids.to(d), weight.to(d)


def exact(x, teacher, ids, weight, T):
    """(loss, (m, ln Z), gradient, and how far each may be off, without the last rounding of the gradient)."""
    x, t, ids, weight = x.double().cpu(), teacher.double().cpu() / T, ids.long().cpu(), weight.double().cpu()
    n, V = x.shape
    k = ids.shape[1]
    valid = (ids >= 0) & (ids < V) & ~(t == -math.inf)
    some = valid.any(1)
    t = t.masked_fill(~valid, -math.inf)
    lnq = (t - torch.logsumexp(t, 1, keepdim=True)).masked_fill(~valid, -math.inf)
    q = lnq.exp().masked_fill(~valid, 0.0)
    m = x.max(1, keepdim=True).values
    y = (x - m) / T
    z = y.exp().sum(1, keepdim=True)
    p = y.exp() / z
    lp = y.gather(1, ids.clamp(0, V - 1)) - z.log()
    live = ~(q == 0)                      # a NaN stays
    term = torch.where(live, q * (lnq - lp), torch.zeros_like(q))
    loss = torch.where(some, term.sum(1), torch.zeros(n, dtype=torch.float64))
    stats = torch.cat([m.masked_fill(z.isnan(), math.nan), z.log()], 1).masked_fill(~some[:, None], 0.0)
    g = torch.where(some[:, None], p, torch.zeros_like(p))
    qs = torch.zeros_like(p).scatter_add_(1, ids.clamp(0, V - 1), q)
    grad = (g - qs) * weight[:, None] / T
    # roundings
    py = torch.where(p > 0, p * y.abs(), torch.zeros_like(p)).sum(1)
    dz = (4 + 3 * py + V / 512 + 8 + 64) * U
    dlnz = dz + U * (2 + stats[:, 1].abs())
    top = torch.where(some[:, None], t.max(1, keepdim=True).values, torch.zeros_like(t[:, :1]))
    ty = torch.where(live, (t - top).abs(), torch.zeros_like(t))
    dq = (16 + k / 32 + 4 * ty + lnq.masked_fill(~live, 0.0).abs()) * U          # of ln q, and relative of q
    each = (lp.abs() + lnq.abs() + 4) * 4 * U + dlnz[:, None] + dq * (1 + (lnq - lp).abs())
    dloss = torch.where(live, q * each, torch.zeros_like(q)).sum(1) + (k / 512 + 32) * U * term.abs().sum(1)
    dp = torch.where(p > 0, p * ((8 + 4 * y.abs()) * U + dlnz[:, None] * 2), torch.zeros_like(p))
    dgrad = (dp + torch.where(qs > 0, qs * (dq.amax(1, keepdim=True) + (k + 4) * U), torch.zeros_like(qs))) * weight[:, None] / T + 8 * U * grad.abs() + 1e-44
    return loss, stats, grad, dloss, dlnz, dgrad


def near(got, want, tol, what):
    got, want = got.double().cpu(), want
    nan = want.isnan()
    assert torch.equal(got.isnan(), nan), what
    inf = want.isinf()
    assert torch.equal(got[inf], want[inf]) and not bool(got[~inf & ~nan].isinf().any()), what
    fine = ~nan & ~inf
    over = ((got - want).abs() - tol)[fine]
    assert over.numel() == 0 or float(over.max()) <= 0, (what, float(over.max()), float(tol[fine].min()))


def check(x, teacher, ids, weight, T):
    dtype = x.dtype
    loss_w, stats_w, grad_w, dloss, dlnz, dgrad = exact(x, teacher, ids, weight, T)
    # the gradient's own rounding; below the type's smallest normal number half of its smallest step
    tiny = torch.finfo(dtype).smallest_normal * torch.finfo(dtype).eps / 2
    tol = dgrad + (grad_w.abs() + dgrad) * (torch.finfo(dtype).eps / 2) + tiny
    loss, stats = ardiff.ardiff_distill_topk(x, teacher, ids, T)
    near(loss, loss_w, dloss, "loss")
    near(stats[:, 0], stats_w[:, 0], torch.zeros(len(loss_w)), "largest")
    near(stats[:, 1], stats_w[:, 1], dlnz, "ln Z")
    near(ardiff.ardiff_distill_topk_backward(x, teacher, ids, stats, weight, T), grad_w, tol, "backward")
    loss2, stats2, grad = ardiff.ardiff_distill_topk_step(x, teacher, ids, weight, T)
    near(loss2, loss_w, dloss, "loss of the step")             # (by other threads, so in another order of sums)
    near(stats2[:, 0], stats_w[:, 0], torch.zeros(len(loss_w)), "largest of the step")
    near(stats2[:, 1], stats_w[:, 1], dlnz, "ln Z of the step")
    near(grad, grad_w, tol, "step")
    return loss_w, grad_w


@pytest.mark.parametrize("dtype", sorted(DTYPES))
@pytest.mark.parametrize("n,V,k,T", [
    (1, 1, 1, 1.0), (3, 2, 2, 0.5), (5, 7, 3, 1.0), (2, 8, 8, 2.0), (4, 9, 4, 1.0), (2, 100, 1, 1.0), (7, 257, 33, 4.0),
    (3, 1000, 1000, 1.0), (150, 777, 64, 1.0), (1, 8191, 20, 1.0), (2, 50001, 100, 0.5), (300, 16384, 128, 1.0),
    (1, 131072, 256, 1.0), (9, 40000, 1024, 2.0)])
def test_against_the_definition(dtype, n, V, k, T):
    check(*make(n, V, k, DTYPES[dtype], seed=V + k), T)


@pytest.mark.parametrize("dtype", sorted(DTYPES))
@pytest.mark.parametrize("n,V,pad,offset", [(5, 500, 3, 0), (4, 501, 0, 1), (3, 33000, 11, 5), (200, 1003, 7, 3)])
def test_rows_at_any_place(dtype, n, V, pad, offset):
    check(*make(n, V, 16, DTYPES[dtype], seed=V, pad=pad, offset=offset), 1.0)


@pytest.mark.parametrize("teacher_dtype", sorted(DTYPES))
def test_types_of_the_teacher(teacher_dtype):
    check(*make(6, 3001, 40, torch.bfloat16, seed=3, teacher_dtype=DTYPES[teacher_dtype]), 1.5)


@pytest.mark.parametrize("dtype", sorted(DTYPES))
@pytest.mark.parametrize("V", [129, 20000])
def test_entries_that_are_none_and_ids_that_occur_again(dtype, V):
    x, teacher, ids, weight = make(8, V, 24, DTYPES[dtype], seed=V)
    ids[0, 5:] = -1                       # a shorter list
    ids[1] = -1                           # a row of padding
    ids[2, ::2] = V                       # beyond the vocabulary
    ids[3, ::3] = -2 ** 31
    ids[3, 1::3] = 2 ** 31 - 1
    ids[4] = V - 1                        # one id throughout
    ids[5, 12:] = ids[5, :12]             # every id twice
    teacher[6, 3:] = -math.inf
    teacher[7] = -math.inf
    x[1, 0] = math.nan                    # not read
    loss, grad = check(x, teacher, ids, weight, 1.0)
    assert float(loss[1]) == 0 and float(grad[1].abs().max()) == 0 and float(loss[7]) == 0
    both = ardiff.ardiff_distill_topk_step(x, teacher, ids, weight, 1.0)
    assert float(both[0][1]) == 0 and float(both[2][1].abs().max()) == 0


@pytest.mark.parametrize("dtype", sorted(DTYPES))
def test_masked_logits_and_rows_without_a_softmax(dtype):
    V = 1500
    x, teacher, ids, weight = make(8, V, 8, DTYPES[dtype], seed=11)
    ids[:] = torch.arange(8, device=ids.device, dtype=torch.int32) * 11
    x[0, 700:] = -math.inf                # a mask, not where the teacher has anything
    x[1, ids[1, 2].long()] = -math.inf    # where it has
    x[2, :] = -math.inf
    x[3, 4] = math.nan
    x[4, 1499] = math.inf
    x[5, 100:] = torch.finfo(x.dtype).min
    x[6, :] = torch.finfo(x.dtype).min    # all masked by the type's lowest value: uniform
    teacher[7, 2] = math.nan
    loss, grad = check(x, teacher, ids, weight, 1.0)
    assert float(loss[1]) == math.inf and all(math.isnan(float(loss[i])) for i in (2, 3, 4, 7))
    assert torch.isfinite(grad[0]).all() and torch.isfinite(grad[6]).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("shift", [300.0, 3e4])
def test_large_logits(dtype, shift):
    x, teacher, ids, weight = make(4, 5000, 32, torch.float32, seed=2)
    check((x + shift).to(DTYPES[dtype]), teacher + shift, ids, weight, 1.0)


def test_gradient_against_differences():
    """(L(x + h) - L(x - h)) / 2h is off by h^2 / 6 times the third derivative (at most 0.1 / T^3, of ln Z alone) and by the two
    losses' own errors over 2h."""
    T, h = 1.0, 0.0625
    x, teacher, ids, weight = make(1, 40, 6, torch.float32, seed=5, spread=1.0)
    _, _, grad = ardiff.ardiff_distill_topk_step(x, teacher, ids, weight, T)
    rows = x.repeat(80, 1)
    i = torch.arange(40, device=x.device)
    rows[i, i] += h
    rows[40 + i, i] -= h
    loss, _ = ardiff.ardiff_distill_topk(rows, teacher.repeat(80, 1), ids.repeat(80, 1), T)
    dloss = exact(rows, teacher.repeat(80, 1), ids.repeat(80, 1), weight.repeat(80), T)[3]
    diff = (loss[:40] - loss[40:]).double().cpu() / (2 * h) * float(weight[0])
    tol = float(weight[0]) * (0.1 * h * h / 6 + (dloss[:40] + dloss[40:] + 2 * U * h * 4) / (2 * h)) + 1e-6
    assert bool(((grad[0].double().cpu() - diff).abs() <= tol).all())


@pytest.mark.parametrize("dtype", sorted(DTYPES))
@pytest.mark.parametrize("n,V", [(3, 1001), (2, 60000), (200, 9000)])
def test_gradient_in_the_logits_place(dtype, n, V):
    x, teacher, ids, weight = make(n, V, 16, DTYPES[dtype], seed=V)
    loss, stats, grad = ardiff.ardiff_distill_topk_step(x, teacher, ids, weight, 1.0)
    back = ardiff.ardiff_distill_topk_backward(x, teacher, ids, stats, weight, 1.0)
    y = x.clone()
    out = ardiff.ardiff_distill_topk_step(y, teacher, ids, weight, 1.0, grad=y)
    assert out[2] is y and torch.equal(y, grad) and torch.equal(out[0], loss)
    y = x.clone()
    assert torch.equal(ardiff.ardiff_distill_topk_backward(y, teacher, ids, stats, weight, 1.0, grad=y), back)


def test_gradient_rows_apart_from_the_logits_and_nothing_between_them():
    x, teacher, ids, weight = make(6, 1003, 16, torch.bfloat16, seed=4)
    loss, stats, want = ardiff.ardiff_distill_topk_step(x, teacher, ids, weight, 1.0)
    buf = torch.full((6, 1024), 7.0, dtype=torch.bfloat16, device=x.device)
    for call in (lambda g: ardiff.ardiff_distill_topk_step(x, teacher, ids, weight, 1.0, grad=g)[2],
                 lambda g: ardiff.ardiff_distill_topk_backward(x, teacher, ids, stats, weight, 1.0, grad=g)):
        out = call(buf[:, 3:1006])
        assert bool((buf[:, :3] == 7).all()) and bool((buf[:, 1006:] == 7).all())
        assert float((out.float() - want.float()).abs().max()) <= float(want.float().abs().max()) * 2.0 ** -8
        buf[:, 3:1006] = 7.0


def test_captured_step_follows_its_buffers_and_streams_do_not_meet():
    x, teacher, ids, weight = make(40, 5000, 32, torch.bfloat16, seed=6)
    x2, teacher2, ids2, weight2 = make(40, 5000, 32, torch.bfloat16, seed=7)
    want = [ardiff.ardiff_distill_topk_step(x, teacher, ids, weight), ardiff.ardiff_distill_topk_step(x2, teacher2, ids2, weight2)]
    a, t, i, w = x.clone(), teacher.clone(), ids.clone(), weight.clone()
    loss, stats, grad = torch.zeros_like(want[0][0]), torch.zeros_like(want[0][1]), torch.zeros_like(want[0][2])
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ardiff.ardiff_distill_topk_step(a, t, i, w, 1.0, loss, stats, grad)
    for src, out in (((x2, teacher2, ids2, weight2), want[1]), ((x, teacher, ids, weight), want[0])):
        for to, v in zip((a, t, i, w), src):
            to.copy_(v)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(loss, out[0]) and torch.equal(stats, out[1]) and torch.equal(grad, out[2])
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    got = []
    for _ in range(3):
        got = [ardiff.ardiff_distill_topk_step(x, teacher, ids, weight, stream=streams[0]),
               ardiff.ardiff_distill_topk_step(x2, teacher2, ids2, weight2, stream=streams[1])]
    torch.cuda.synchronize()
    for g, w_ in zip(got, want):
        assert all(torch.equal(a_, b_) for a_, b_ in zip(g, w_))


def test_a_few_steps_of_training_bring_the_student_to_the_teacher():
    """Runs the loss with its gradient as a training loop does; that the loss is finite and falls at the first step's direction
    is what the gradient says (d loss = -eta |g|^2), to first order."""
    x, teacher, ids, weight = make(16, 600, 32, torch.float32, seed=8, spread=1.0)
    weight.fill_(1.0)
    loss0, _, grad = ardiff.ardiff_distill_topk_step(x, teacher, ids, weight)
    eta = 1e-2
    loss1, _ = ardiff.ardiff_distill_topk(x - eta * grad, teacher, ids)
    slope = (grad.double() ** 2).sum(1)
    # second order: the Hessian of ln Z has a largest eigenvalue of at most 1/2
    change = (loss0 - loss1).double()
    slack = 0.25 * eta * eta * slope + 4e-6
    assert bool(((change - eta * slope).abs() <= slack).all())


@pytest.mark.parametrize("what", ["type of ids", "ids by columns", "stats of another size", "rows that overlap", "columns apart", "type of logits"])
def test_tensors_that_do_not_fit_are_refused(what):
    x, teacher, ids, weight = make(4, 100, 8, torch.float32, seed=1)
    stats = torch.zeros((4, 2), device=x.device)
    if what == "type of ids":
        ids = ids.long()
    elif what == "ids by columns":
        ids = ids.t().contiguous()
    elif what == "stats of another size":
        stats = stats[:3]
    elif what == "rows that overlap":
        x = x[:1].expand(4, 100)
    elif what == "columns apart":
        x = x.repeat(1, 2)[:, ::2]
    else:
        x = x.double()
    with pytest.raises((AssertionError, ardiff.ArdiffError)):
        ardiff.ardiff_distill_topk_backward(x, teacher, ids, stats, weight)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("kind", ["equal", "rising", "falling"])
def test_long_rows_do_not_add_up_roundings(kind, dtype):
    """As many rows as give each row one CTA. ln Z may be off by 32 additions of a few pieces' values and the compensated sum of those (2),
    by exponents up to 4 octaves above 0 (4 + 3 4 ln 2 <= 13 roundings each, at most 12 times where the sum is scaled: later ones weigh 2^-48), by 16
    merges of 13 and by the number's own rounding: all of which does not depend on V."""
    n, V, k = 300, 1 << 22, 4
    d = require_cuda()
    i = torch.arange(V, device=d, dtype=torch.float64)
    for slope in ([-0.5, -0.75, -1.0, -2.5, -3.0] if kind == "equal" else [1e-6, 3e-5]):
        row = torch.full((V,), slope, dtype=torch.float64, device=d) if kind == "equal" else slope * (i if kind == "rising" else -i)
        if kind == "equal":
            row[:16384] = 0.0                                    # every thread's first pieces
        row = row.to(DTYPES[dtype])
        x = row.repeat(n, 1)
        y = row.double() - row.double().max()
        ln_z = float(torch.log(y.exp().sum()))
        mean = float((y.abs() * y.exp()).sum() / y.exp().sum())
        teacher = torch.zeros((n, k), device=d)
        ids = torch.arange(k, device=d, dtype=torch.int32).repeat(n, 1) * 1000
        weight = torch.ones(n, device=d)
        tol = (4 + 3 * (mean + 4) + 34 + 12 * 13 + 16 * 13 + 3 + 3 * abs(ln_z)) * U
        stats = ardiff.ardiff_distill_topk(x, teacher, ids)[1]
        step = ardiff.ardiff_distill_topk_step(x, teacher, ids, weight, grad=x)[1]
        for s in (stats, step):
            assert bool((s[:, 0].double() == float(row.double().max())).all())
            off = float((s[:, 1].double() - ln_z).abs().max())
            assert off <= tol, (slope, off, tol)
        del x
