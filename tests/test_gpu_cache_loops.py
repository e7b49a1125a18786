"""The operators around a draft model's cache at sizes where their kernels' loops come round: several tiles a CTA, stages that are used again, few and many
rows one after the other, rows of many heads, keys that shared memory does not hold. Against the same loops in 64 bits as the small cases."""
import math

import pytest
import torch

import paper_2512_08537_b200 as ardiff
from gpu_util import require_cuda
from test_gpu_attend import Case, evicted, i32
from test_gpu_rotary import inputs, near, turned

pytestmark = pytest.mark.gpu


def weights_near(c, lse, score, new, first, decay, causal):
    """new [R, places] against decay * score and the weights' sums in 64 bits: scores as Case.scores says, an exponential of 2^-19 with lse times log2 e rounded
    and lse's own size, sums of n Hq terms."""
    for r in range(len(c.n)):
        f, L, t0 = first[r], c.len[r], sum(c.n[:r])
        if L <= f:
            continue
        want = torch.zeros((L,), dtype=torch.float64, device=new.device)
        tol = 2.0 ** -22 * score[r, :L].double().abs()
        old = max(0, L - c.n[r])
        want[:old] = decay * score[r, :old].double()
        if c.n[r]:
            x, off = c.scores(r, causal)
            given = lse[t0:t0 + c.n[r]].double()[..., None]
            w = torch.where(given > -math.inf, torch.exp(x - given), torch.zeros_like(x)).sum((0, 1))
            want += w
            largest = float(torch.where(given > -math.inf, given.abs(), torch.zeros_like(given)).max())
            tol = tol + w * (off + 2.0 ** -19 + 2.0 ** -23 * largest + 2.0 ** -24 * c.n[r] * c.Hq)
        err = (new[r, f:L].double() - want[f:]).abs()
        assert bool((err <= tol[f:] + 1e-30).all()), (r, float((err / (tol[f:] + 1e-30)).max()))


@pytest.mark.parametrize("D,dtype,layout,page", [(64, "f16", "nhd", 64), (80, "bf16", "hnd", 25), (96, "bf16", "nhd", 16), (128, "f16", "nhd", 25), (128, "bf16", "hnd", 128)])
@pytest.mark.parametrize("Hq,Hkv", [(8, 2), (24, 8), (3, 1)])
def test_weights_of_many_tiles_with_few_and_many_rows(D, dtype, layout, page, Hq, Hkv):
    """Some 1400 tiles, so ten a CTA: one segment after the other, of few rows (all heads at once), of many, of more than 128 rows a head, and of none."""
    n = [[1, 1, 40, 2, 0, 1, 150, 3, 5, 64][r % 10] for r in range(80)]
    length = [1300 + (r * 731) % 2000 for r in range(80)]
    c = Case(n, length, Hq, Hkv, D, page, dtype, layout, pad=2, seed=D + Hq)
    first = [[0, 0, 700, 129, 0][r % 5] for r in range(80)]
    N = c.table.shape[1] * page
    score = torch.rand((80, N), device=c.q.device, generator=c.g)
    for causal in (True, False):
        lse = c.attend(causal=causal)[1]
        new = torch.full_like(score, -4.0)
        _, status = ardiff.ardiff_attend_weights(c.q, c.k, c.table, c.length, c.offset, lse, score, first=i32(first), decay=0.75, causal=causal, new_score=new)
        assert int(status) == 0
        for r in range(80):
            assert bool((new[r, length[r]:] == -4.0).all()) and bool((new[r, :first[r]] == -4.0).all())
        weights_near(c, lse, score, new, first, 0.75, causal)
        again, _ = ardiff.ardiff_attend_weights(c.q, c.k, c.table, c.length, c.offset, lse, score, first=i32(first), decay=0.75, causal=causal)
        for r in range(80):
            assert torch.equal(again[r, first[r]:length[r]], new[r, first[r]:length[r]])


@pytest.mark.parametrize("D,dtype,page", [(64, "f16", 16), (80, "bf16", 25), (96, "f16", 64), (128, "bf16", 128), (128, "f16", 7)])
@pytest.mark.parametrize("rise", [0.0, 40.0])
def test_prompts_of_many_tiles_a_cta(D, dtype, page, rise):
    """384 units of 10 to 20 tiles on the SMs there are: whole units of many tiles, written at once, and cut ones. With `rise` scores grow along the keys, so that
    the base of the weights moves in tiles that all rows see."""
    n, length = [260 + r for r in range(24)], [1300 + 47 * r for r in range(24)]
    c = Case(n, length, 8, 8, D, page, dtype, seed=D)
    if rise:
        for r, L in enumerate(length):
            p = torch.arange(L, device=c.q.device)
            c.keys[r] = (c.keys[r].float() * (0.05 + rise * p / L)[:, None, None] * 0.2).to(c.keys[r].dtype)
            c.k[c.table[r].long()[p // page], p % page] = c.keys[r]
    for causal in (True, False):
        want = c.attend(causal=causal, most=max(n))
        assert int(want[2]) == 0
        c.check(want[0], want[1], causal)
        again = c.attend(causal=causal, most=max(n))
        assert torch.equal(again[0], want[0]) and torch.equal(again[1], want[1])


@pytest.mark.parametrize("D,dtype,page,Hq,Hkv,new", [(64, "f16", 16, 8, 4, 2), (80, "bf16", 25, 16, 8, 1), (96, "f16", 64, 8, 2, 5), (128, "bf16", 16, 8, 2, 8), (128, "f16", 7, 4, 4, 1)])
def test_few_rows_of_many_steps_a_warp(D, dtype, page, Hq, Hkv, new):
    """600 requests of 1000 to 1600 tokens: whole units of some hundred steps of 16 keys, one after the other, whose scores rise."""
    R = 600
    n, length = [new if r % 3 else 1 for r in range(R)], [1000 + r for r in range(R)]
    c = Case(n, length, Hq, Hkv, D, page, dtype, seed=D)
    for r, L in enumerate(length):
        p = torch.arange(L, device=c.q.device)
        c.keys[r] = (c.keys[r].float() * (0.05 + 6.0 * p / L)[:, None, None]).to(c.keys[r].dtype)
        c.k[c.table[r].long()[p // page], p % page] = c.keys[r]
    out, lse, status = c.attend(most=new)
    assert int(status) == 0
    c.check(out, lse)


@pytest.mark.parametrize("n", [3, 100])
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_alike_scores_far_below_zero(n, dtype):
    """Products and sums are exact here, so scores are off by their scaling alone: results are means, lse the score plus a logarithm."""
    c = Case([n], [500], 4, 2, 128, 16, dtype, seed=11)
    c.q.fill_(-30.0)
    c.k[c.table[0].long()] = 30.0
    out, lse, status = c.attend()
    assert int(status) == 0
    v = c.values[0].double().repeat_interleave(2, 1)
    eps = torch.finfo(c.q.dtype).eps / 2
    for i in range(n):
        L = 500 - n + i + 1
        want, size = v[:L].mean(0), v[:L].abs().mean(0)
        # scale, log2 e, their product and its product with the score are off by 2^-24 each; the weights' common factor, from the rounding of a score of up to 2^14 in
        # powers of two, is 2^-10 at most (half a step of 2^-10, times ln 2, and the operand may round it away); weight and result rounded
        assert bool(((out[i].double() - want).abs() <= (eps + 2.0 ** -10) * size + eps * want.abs() + 2.0 ** -20).all())
        exact = -900.0 * 128 * c.scale + math.log(L)
        assert float((lse[i].double() - exact).abs().max()) <= 7 * 2.0 ** -24 * abs(exact) + 2.0 ** -20


@pytest.mark.parametrize("T,Hq,Hkv,D,P,dtype", [(3000, 32, 8, 128, 64, "bf16"), (3000, 24, 16, 80, 35, "f16"), (2500, 40, 4, 64, 32, "f32"), (2999, 33, 7, 96, 20, "bf16")])
@pytest.mark.parametrize("neighbours", [False, True])
def test_rotary_of_many_tokens_and_heads(T, Hq, Hkv, D, P, dtype, neighbours):
    """A warp a token, some rows of it after the others; into a cache, too."""
    q, k, v, position, freq, axis = inputs(T, Hq, Hkv, D, P, 3, dtype, 5000, T + D)
    for fn, sign in ((ardiff.ardiff_rotary, 1.0), (ardiff.ardiff_rotary_backward, -1.0)):
        for x, y in zip((q, k), fn(q, k, position, freq, axis=axis, neighbours=neighbours)):
            near(y, *turned(x, position, freq, axis, neighbours, sign))
    page, pages = 16, -(-T // 16) + 3
    kc, vc = [torch.full((pages, page, Hkv, D), 5.0, device=q.device, dtype=q.dtype) for _ in range(2)]
    slot = torch.randperm(pages * page, device=q.device)[:T].contiguous()
    want = ardiff.ardiff_rotary(q, k, position, freq, axis=axis, neighbours=neighbours)
    count = T - 7
    got = ardiff.ardiff_rotary_append(q, k, v, position, freq, slot, kc, vc, axis=axis, count=i32([count]), neighbours=neighbours, q_out=torch.zeros_like(want[0]))
    assert torch.equal(got[:count], want[0][:count]) and not bool(got[count:].any())
    for cache, x in ((kc, want[1]), (vc, v)):
        flat = torch.full((pages * page, Hkv, D), 5.0, device=q.device, dtype=q.dtype)
        flat[slot[:count]] = x[:count]
        assert torch.equal(cache.view(pages * page, Hkv, D), flat)


@pytest.mark.parametrize("R,longest,budget", [(40, 45000, 41500), (40, 45000, 300), (3, 45000, 41500), (2, 340000, 330000)])
@pytest.mark.parametrize("kind", ["ties", "some"])
def test_eviction_of_more_keys_than_shared_memory_holds(R, longest, budget, kind):
    """A CTA a request (40), or a cluster; 40960 keys are held, others worked out again. In place: weights, positions and the caches' rows."""
    dev = require_cuda()
    g = torch.Generator(device=dev).manual_seed(R + budget)
    page, H, D = 64, 1, 8
    width = -(-longest // page)
    N, pages = width * page, R * width
    k, v = [torch.randn((pages, page, H, D), device=dev, generator=g).half() for _ in range(2)]
    table = torch.randperm(pages, device=dev, generator=g).to(torch.int32).view(R, width)
    length = [longest if r == 0 else 100 + 13 * r for r in range(R)]
    budgets = [budget if r == 0 else 60 + 3 * r for r in range(R)]
    first = [r % 4 for r in range(R)]
    score = torch.rand((R, N), device=dev, generator=g)
    if kind == "ties":
        score = (score * 3).floor()
    position = torch.argsort(torch.rand((R, N), device=dev, generator=g), 1).to(torch.int32).contiguous()
    s2, p2, l2, k2, v2 = score.clone(), position.clone(), i32(length), k.clone(), v.clone()
    got = ardiff.ardiff_pages_evict(l2, i32(budgets), s2, table, k2, v2, first=i32(first), position=p2, seen=i32([N] * R), recent=500, new_length=l2,
                                    new_score=s2, new_position=p2)
    assert int(got[3]) == 0 and got[0] is l2 and got[1] is s2 and got[2] is p2
    p = torch.arange(N, device=dev)
    for r in range(R):
        want = evicted(score[r].tolist(), position[r].tolist(), length[r], budgets[r], first[r], N, 500)
        m, at = len(want), torch.tensor(want, device=dev, dtype=torch.long)
        assert int(l2[r]) == m
        assert torch.equal(s2[r, :m], score[r, at]) and torch.equal(s2[r, m:], score[r, m:])
        assert torch.equal(p2[r, :m], position[r, at]) and torch.equal(p2[r, m:], position[r, m:])
        where = table[r].long()[p // page], p % page
        for old, new in ((k, k2), (v, v2)):
            rows = old[where]
            assert torch.equal(new[where][:m], rows[at]) and torch.equal(new[where][m:], rows[m:])


@pytest.mark.parametrize("kind", ["ties", "odd"])
def test_eviction_in_place(kind):
    """What stays and what moves, bit for bit, where weights and positions are their own results."""
    dev = require_cuda()
    g = torch.Generator(device=dev).manual_seed(8)
    R, page, H, D, width = 21, 7, 3, 80, 60
    N, pages = width * page, R * width
    k, v = [torch.randn((pages, H, page, D), device=dev, generator=g).bfloat16().transpose(1, 2) for _ in range(2)]
    table = torch.randperm(pages, device=dev, generator=g).to(torch.int32).view(R, width)
    length = [int(x) for x in torch.randint(1, N + 1, (R,), device=dev, generator=g)]
    budget = [int(x) for x in torch.randint(-1, N + 1, (R,), device=dev, generator=g)]
    score = torch.rand((R, N), device=dev, generator=g)
    if kind == "ties":
        score = (score * 4).floor()
    else:
        score = torch.where(score < 0.1, torch.full_like(score, math.nan), torch.where(score < 0.2, torch.full_like(score, -math.inf), score))
        score = torch.where(score > 0.9, torch.full_like(score, math.inf), torch.where(score > 0.8, -0.0 * score, score))
    for first in (None, [3 * r for r in range(R)]):
        s2, l2 = score.clone(), i32(length)
        k2, v2 = [x.transpose(1, 2).contiguous().transpose(1, 2) for x in (k, v)]
        _, _, _, status = ardiff.ardiff_pages_evict(l2, i32(budget), s2, table, k2, v2, first=None if first is None else i32(first), recent=5, new_length=l2, new_score=s2)
        assert int(status) == 0
        p = torch.arange(N, device=dev)
        for r in range(R):
            want = evicted(score[r].tolist(), list(range(N)), length[r], budget[r], 0 if first is None else first[r], length[r], 5)
            m, at = len(want), torch.tensor(want, device=dev, dtype=torch.long)
            assert int(l2[r]) == m and torch.equal(s2[r, :m].view(torch.int32), score[r, at].view(torch.int32))
            assert torch.equal(s2[r, m:].view(torch.int32), score[r, m:].view(torch.int32))
            where = table[r].long()[p // page], p % page
            for old, new in ((k, k2), (v, v2)):
                rows = old[where]
                assert torch.equal(new[where][:m], rows[at]) and torch.equal(new[where][m:], rows[m:])


@pytest.mark.parametrize("n,length,Hq,Hkv,D,groups,shared", [
    ([1], [5000], 4, 4, 64, None, None), ([1], [300], 8, 2, 128, None, None), ([3, 1], [4000, 77], 12, 4, 80, None, None), ([17], [3000], 1, 1, 64, None, None),
    ([300], [9000], 8, 8, 128, None, None), ([40, 700, 1, 9], [900, 3000, 8000, 4000], 16, 4, 96, None, None), ([1] * 300, list(range(500, 2000, 5)), 16, 4, 64, None, None),
    ([1200], [1200], 32, 8, 128, None, None), ([1] * 700, [900 + r for r in range(700)], 16, 16, 80, None, None), ([4, 9, 2], [900, 800, 850], 4, 2, 64, [0, 3], [700]),
    ([80, 1, 70], [900, 800, 850], 8, 2, 128, [0, 2], [500])])
def test_attention_stays_inside_its_workspace(monkeypatch, n, length, Hq, Hkv, D, groups, shared):
    """What lies in front of the workspace and behind it keeps its bytes; what lay in it before does not matter."""
    c = Case(n, length, Hq, Hkv, D, 16, seed=D, groups=groups, shared=shared)
    made = []

    def workspace(size, where, device):
        made.append((torch.full((size + 8192,), 0xFF, dtype=torch.uint8, device=device), size))
        return made[-1][0][4096:4096 + size]

    monkeypatch.setattr(ardiff, "_workspace", workspace)
    for most in (None, max(n)):
        out, lse, status = c.attend(most=most)
        assert int(status) == 0
        c.check(out, lse)
        x, size = made.pop()
        assert bool((x[:4096] == 0xFF).all()) and bool((x[4096 + size:] == 0xFF).all())
