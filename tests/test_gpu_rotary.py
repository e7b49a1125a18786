"""Rotary positions against rotations in 64 bits."""
import math

import pytest
import torch

import paper_2512_08537_b200 as ardiff
from gpu_util import require_cuda

pytestmark = pytest.mark.gpu
TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}


def gen(seed):
    return torch.Generator(device=require_cuda()).manual_seed(seed)


def normal(g, *shape):
    return torch.randn(shape, device=g.device, generator=g)


def turned(x, position, freq, axis, neighbours, sign=1.0):
    """[T, H, D] in 64 bits, and for every value the size of what went into it."""
    P = freq.numel()
    x = x.double()
    out, size = x.clone(), x.abs()
    for i in range(P):
        a = int(axis[i]) if axis is not None else 0
        angle = position[a].double() * freq[i].double() * sign if 0 <= a < position.shape[0] else torch.zeros_like(position[0]).double()
        c, s = torch.cos(angle)[:, None], torch.sin(angle)[:, None]
        m, n = (2 * i, 2 * i + 1) if neighbours else (i, i + P)
        out[..., m], out[..., n] = x[..., m] * c - x[..., n] * s, x[..., m] * s + x[..., n] * c
        size[..., m] = size[..., n] = x[..., m].abs() + x[..., n].abs()
    return out, size


def near(got, want, size):
    """A rounding of the result, and of what is computed in 32 bits: an angle of at most half a turn is off by pi 2^-24, sine and cosine
    by 2^-23 more, two products and a sum by 2^-24 each: together below 2^-21 of the two values' sizes."""
    eps = torch.finfo(got.dtype).eps / 2
    tiny = 2.0 ** -25 if got.dtype is torch.float16 else 0.0          # half a step of f16's smallest numbers
    err = (got.double() - want).abs()
    assert bool((err <= eps * want.abs() * (1 + 2.0 ** -10) + 2.0 ** -21 * size + tiny).all()), float((err / (size + 1e-30)).max())


def inputs(T, Hq, Hkv, D, P, axes, dtype, far, seed, pad=0):
    g = gen(seed)
    x = normal(g, T, Hq + 2 * Hkv, D + pad)[..., :D].to(TYPES[dtype]) if not pad else normal(g, T, Hq + 2 * Hkv, D + pad).to(TYPES[dtype])[..., :D]
    position = torch.randint(-far // 2, far, (axes, T), device=g.device, generator=g, dtype=torch.int32)
    freq = (10000.0 ** -(torch.arange(P, device=g.device) / max(1, P)).double()).float()
    axis = torch.arange(P, device=g.device, dtype=torch.int32) % axes
    return x[:, :Hq], x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:], position, freq, axis


@pytest.mark.parametrize("T,Hq,Hkv,D,P,axes,far,pad", [
    (1, 1, 1, 2, 1, 1, 10, 0), (3, 4, 2, 64, 32, 1, 2 ** 30, 0), (130, 3, 3, 80, 35, 3, 100, 0), (77, 8, 1, 96, 42, 2, 1000, 0),
    (301, 5, 5, 128, 64, 3, 100000, 0), (50, 2, 2, 33, 7, 2, 64, 0), (9, 2, 1, 512, 256, 4, 5000, 0), (40, 3, 2, 64, 20, 2, 50, 5),
    (17, 4, 4, 66, 33, 1, 500, 2), (5, 2, 2, 16, 0, 1, 5, 0), (2000, 2, 2, 64, 32, 2, 300, 0), (33, 1, 0, 64, 16, 1, 30, 0)])
@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("neighbours", [False, True])
def test_forward_and_backward(T, Hq, Hkv, D, P, axes, far, pad, dtype, neighbours):
    q, k, _, position, freq, axis = inputs(T, Hq, Hkv, D, P, axes, dtype, far, T + D, pad)
    for fn, sign in ((ardiff.ardiff_rotary, 1.0), (ardiff.ardiff_rotary_backward, -1.0)):
        got = fn(q, k, position, freq, axis=axis, neighbours=neighbours)
        for x, y in zip((q, k), got):
            assert y.shape == x.shape and y.dtype is x.dtype
            near(y, *turned(x, position, freq, axis, neighbours, sign))
            if 2 * P < D:
                assert torch.equal(y[..., 2 * P:], x[..., 2 * P:])


@pytest.mark.parametrize("neighbours", [False, True])
def test_in_place_and_an_axis_that_there_is_not(neighbours):
    q, k, _, position, freq, axis = inputs(60, 4, 2, 80, 35, 2, "bf16", 99, 1)
    axis[::3] = -1
    axis[1::7] = 2
    want = ardiff.ardiff_rotary(q, k, position, freq, axis=axis, neighbours=neighbours)
    near(want[0], *turned(q, position, freq, axis, neighbours))
    q2, k2 = q.clone(memory_format=torch.contiguous_format), k.clone(memory_format=torch.contiguous_format)
    ardiff.ardiff_rotary(q2, k2, position, freq, axis=axis, neighbours=neighbours, q_out=q2, k_out=k2)
    assert torch.equal(q2, want[0]) and torch.equal(k2, want[1])


def test_positions_of_one_axis_and_no_tokens():
    q, k, _, position, freq, _ = inputs(20, 4, 2, 64, 32, 1, "f32", 50, 2)
    want = ardiff.ardiff_rotary(q, k, position, freq)
    got = ardiff.ardiff_rotary(q, k, position[0], freq)
    assert torch.equal(want[0], got[0]) and torch.equal(want[1], got[1])
    q0, k0 = ardiff.ardiff_rotary(q[:0], k[:0], position[:, :0].contiguous(), freq)
    assert q0.shape == (0, 4, 64) and k0.shape == (0, 2, 64)


def test_gradient_is_that_of_the_formula_and_of_differences():
    """The forward is linear: sum(w * forward(x + h d)) - sum(w * forward(x)) = h sum(backward(w) * d), exactly but for roundings."""
    g = gen(3)
    q, k, _, position, freq, axis = inputs(40, 3, 3, 64, 24, 3, "f32", 1000, 3)
    w, d = normal(g, 40, 3, 64), normal(g, 40, 3, 64)
    y0, _ = ardiff.ardiff_rotary(q, k, position, freq, axis=axis)
    y1, _ = ardiff.ardiff_rotary((q + 0.5 * d).contiguous(), k, position, freq, axis=axis)
    grad, _ = ardiff.ardiff_rotary_backward(w, k, position, freq, axis=axis)
    left, right = float((w.double() * (y1.double() - y0.double())).sum()), 0.5 * float((grad.double() * d.double()).sum())
    # every value is off by at most 2^-20 of its size (about 4), weighted by w: 2^-18 sqrt(7680) at the most likely, 7680 2^-18 at worst
    assert abs(left - right) <= 7680 * 2.0 ** -18
    x = q.double().requires_grad_()
    out, _ = turned(q, position, freq, axis, False)
    P = 24
    cos = torch.cos(position.double()[axis.long()].t() * freq.double())[:, None]
    sin = torch.sin(position.double()[axis.long()].t() * freq.double())[:, None]
    y = torch.cat([x[..., :P] * cos - x[..., P:2 * P] * sin, x[..., :P] * sin + x[..., P:2 * P] * cos, x[..., 2 * P:]], -1)
    y.backward(w.double())
    near(grad, x.grad, turned(w, position, freq, axis, False, -1.0)[1])


@pytest.mark.parametrize("layout", ["nhd", "hnd", "both"])
@pytest.mark.parametrize("T,Hq,Hkv,D,P,page,count,dtype", [(1, 4, 1, 64, 32, 16, None, "bf16"), (200, 3, 3, 80, 35, 25, 190, "f16"),
                                                         (700, 4, 2, 128, 64, 64, 700, "bf16"), (30, 2, 2, 96, 48, 1, 0, "f32"),
                                                         (64, 1, 1, 40, 20, 7, 1000, "f16")])
def test_append_writes_the_slots_and_nothing_else(layout, T, Hq, Hkv, D, P, page, count, dtype):
    q, k, v, position, freq, axis = inputs(T, Hq, Hkv, D, P, 2, dtype, 3000, T)
    g = gen(T + 1)
    pages = -(-T // page) + 4
    if layout == "nhd":
        kc, vc = normal(g, pages, page, Hkv, D).to(q.dtype), normal(g, pages, page, Hkv, D).to(q.dtype)
    elif layout == "hnd":
        kc, vc = normal(g, pages, Hkv, page, D).to(q.dtype).transpose(1, 2), normal(g, pages, Hkv, page, D).to(q.dtype).transpose(1, 2)
    else:                                          # keys and values of a page side by side
        kv = normal(g, pages, 2, page, Hkv, D).to(q.dtype)
        kc, vc = kv[:, 0], kv[:, 1]
    slot = torch.randperm(pages * page, device=g.device, generator=g)[:T].contiguous()
    slot[::5] = torch.tensor([-1, pages * page, -2 ** 40, 2 ** 40], device=g.device).repeat(T)[:slot[::5].numel()]
    q_out = torch.full_like(q, 7.0, memory_format=torch.contiguous_format)
    k0, v0 = kc.clone(), vc.clone()
    n = T if count is None else min(T, count)
    c = None if count is None else torch.tensor([count], dtype=torch.int32, device=g.device)
    got = ardiff.ardiff_rotary_append(q, k, v, position, freq, slot, kc, vc, axis=axis, count=c, q_out=q_out)
    assert got is q_out
    want_q, want_k = ardiff.ardiff_rotary(q, k, position, freq, axis=axis)
    assert torch.equal(q_out[:n], want_q[:n]) and bool((q_out[n:] == 7.0).all())
    near(want_k, *turned(k, position, freq, axis, False))
    for t in range(n):
        s = int(slot[t])
        if 0 <= s < pages * page:
            k0[s // page, s % page], v0[s // page, s % page] = want_k[t], v[t]
    assert torch.equal(kc, k0) and torch.equal(vc, v0)


def test_on_another_stream_and_captured():
    q, k, v, position, freq, axis = inputs(64, 4, 2, 64, 32, 2, "bf16", 99, 5)
    want = ardiff.ardiff_rotary(q, k, position, freq, axis=axis)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = ardiff.ardiff_rotary(q, k, position, freq, axis=axis, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = ardiff.ardiff_rotary(q, k, position, freq, axis=axis)
        back = ardiff.ardiff_rotary_backward(*held, position, freq, axis=axis)
    position.add_(1)
    graph.replay()
    moved = ardiff.ardiff_rotary(q, k, position, freq, axis=axis)
    assert torch.equal(held[0], moved[0]) and torch.equal(held[1], moved[1])
    # there and back: two roundings of values that a rotation cannot make larger than sqrt 2 times the pair's larger one
    assert float((back[0].float() - q.float()).abs().max()) <= float(q.float().abs().max()) * 2.0 ** -8 * 4
    assert math.isfinite(float(back[1].float().sum()))


@pytest.mark.parametrize("D,P,pad", [(64, 32, 0), (80, 35, 0), (64, 20, 5), (66, 33, 2), (128, 64, 0)])
@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("neighbours", [False, True])
def test_pairs_of_no_axis_stand_still_whatever_they_hold(D, P, pad, dtype, neighbours):
    q, k, _, position, freq, axis = inputs(90, 3, 2, D, P, 2, dtype, 99, D + P, pad)
    q, k = q.clone(memory_format=torch.preserve_format), k.clone(memory_format=torch.preserve_format)
    axis[::2] = -1
    axis[4::6] = 2 ** 31 - 1
    still = ((axis < 0) | (axis >= 2)).nonzero()[:, 0]
    one, other = (2 * still, 2 * still + 1) if neighbours else (still, still + P)
    q[3::4, :, one] = math.inf
    q[2::4, :, other] = -math.inf
    k[::2, :, other] = math.nan
    k[:, :, one[1:]] = -0.0
    for fn, sign in ((ardiff.ardiff_rotary, 1.0), (ardiff.ardiff_rotary_backward, -1.0)):
        for x, y in zip((q, k), fn(q, k, position, freq, axis=axis, neighbours=neighbours)):
            kept = torch.cat([one, other])
            assert torch.equal(torch.nan_to_num(y[..., kept], nan=77.0), torch.nan_to_num(x[..., kept], nan=77.0))
            assert torch.equal(torch.signbit(y[..., kept]), torch.signbit(x[..., kept]))
            want, size = turned(torch.nan_to_num(x.float(), nan=0.0, posinf=0.0, neginf=0.0), position, freq, axis, neighbours, sign)
            rest = [i for i in range(D) if i not in set(kept.tolist())]
            near(y[..., rest], want[..., rest], size[..., rest])
