"""Attention over pages, accumulated weights and eviction against loops in 64 bits, and a round of them together."""
import math

import pytest
import torch

import paper_2512_08537_b200 as ardiff
from gpu_util import require_cuda

pytestmark = pytest.mark.gpu
TYPES = {"bf16": torch.bfloat16, "f16": torch.float16}
SHAPE = ardiff.ARDIFF_ERR_SHAPE


def i32(v):
    return torch.tensor(v, dtype=torch.int32, device=require_cuda())


class Case:
    """Requests with n[r] new of length[r] tokens, the first `shared` of the requests of every group the same."""

    def __init__(self, n, length, Hq, Hkv, D, page, dtype="bf16", layout="nhd", groups=None, shared=None, pad=0, seed=0, spread=1.5,
                 q_pad=0):
        dev = require_cuda()
        g = self.g = torch.Generator(device=dev).manual_seed(seed + 17)
        self.n, self.len, self.Hq, self.Hkv, self.D, self.page = n, length, Hq, Hkv, D, page
        R, width = len(n), max(1, max(-(-x // page) for x in length)) + 1
        dt = TYPES[dtype]
        pages = R * width + 5
        ids = torch.randperm(pages, generator=torch.Generator().manual_seed(seed))[:R * width].view(R, width)
        shape = (pages, page, Hkv, D) if layout == "nhd" else (pages, Hkv, page, D)
        made = [torch.full(shape, math.nan, device=dev).to(dt) for _ in range(2)]     # nobody's places hold NaN
        self.k, self.v = made if layout == "nhd" else [x.transpose(1, 2) for x in made]
        self.keys = [torch.randn((x, Hkv, D), device=dev, generator=g).to(dt) for x in length]
        self.values = [torch.randn((x, Hkv, D), device=dev, generator=g).to(dt) for x in length]
        self.group = self.shared = None
        if groups is not None:
            self.group, self.shared = i32(groups), i32(shared)
            for j, s in enumerate(shared):
                for r in range(groups[j], groups[j + 1]):
                    have = min(s, length[r], length[groups[j]])
                    self.keys[r][:have], self.values[r][:have] = self.keys[groups[j]][:have], self.values[groups[j]][:have]
                    ids[r, :have // page] = ids[groups[j], :have // page]
        self.table = ids.to(torch.int32).to(dev).contiguous()
        for r in range(R):
            p = torch.arange(length[r], device=dev)
            at = self.table[r].long()[p // page], p % page
            self.k[at], self.v[at] = self.keys[r], self.values[r]
        self.offset = i32([sum(n[:r]) for r in range(R + 1)])
        self.length = i32(length)
        T = sum(n) + pad
        self.q = (spread * torch.randn((T, Hq, D + q_pad), device=dev, generator=g)).to(dt)[..., :D]
        self.scale = 1.0 / math.sqrt(D)

    def attend(self, **kw):
        a = dict(group=self.group, shared=self.shared)
        a.update(kw)
        return ardiff.ardiff_attend_pages(self.q, self.k, self.v, self.table, self.length, self.offset, **a)

    def scores(self, r, causal):
        """scale q.k [n, Hq, L] in 64 bits with -inf where unseen, and how far 32 bits may be off."""
        t0, G = sum(self.n[:r]), self.Hq // self.Hkv
        q = self.q[t0:t0 + self.n[r]].double()
        k = self.keys[r].double().repeat_interleave(G, 1)
        x = torch.einsum("nhd,lhd->nhl", q, k) * self.scale
        # a product's sum of D terms in 32 bits, cut off or rounded at every step
        off = torch.einsum("nhd,lhd->nhl", q.abs(), k.abs()).amax() * abs(self.scale) * self.D * 2.0 ** -23 if x.numel() else torch.zeros((), device=q.device)
        i = torch.arange(self.n[r], device=q.device)[:, None, None]
        p = torch.arange(self.len[r], device=q.device)[None, None, :]
        limit = self.len[r] - self.n[r] + i + 1 if causal else self.len[r]
        return torch.where(p < limit, x, torch.full_like(x, -math.inf)), float(off)

    def check(self, out, lse, causal=True):
        eps = torch.finfo(self.q.dtype).eps / 2
        G = self.Hq // self.Hkv
        for r in range(len(self.n)):
            t0 = sum(self.n[:r])
            if self.n[r] == 0:
                continue
            x, off = self.scores(r, causal)
            want_lse = torch.logsumexp(x, -1) if self.len[r] else torch.full(x.shape[:2], -math.inf, device=x.device).double()
            w = torch.nan_to_num(torch.exp(x - want_lse[..., None]), nan=0.0)
            v = self.values[r].double().repeat_interleave(G, 1)
            want, size = torch.einsum("nhl,lhd->nhd", w, v), torch.einsum("nhl,lhd->nhd", w, v.abs())
            got_lse, got = lse[t0:t0 + self.n[r]].double(), out[t0:t0 + self.n[r]].double()
            seen = want_lse > -math.inf
            assert torch.equal(got_lse > -math.inf, seen)
            # a weight is off by its score, by an exponential of 2^-22, by the sums of at most 2^15 weights in pieces of 64 and fewer;
            # lse by those and a rounding of its own
            err = (got_lse - want_lse).abs()[seen]
            tol = off + 2.0 ** -18 + 2.0 ** -23 * want_lse[seen].abs()
            assert bool((err <= tol).all()), ("lse", r, float((err - tol).max()))
            # two roundings: the weight as an operand, the result
            err, tol = (got - want).abs(), (eps * (1 + 2.0 ** -7) + 2 * off + 2.0 ** -17) * size + eps * want.abs() + 2.0 ** -25
            assert bool((err <= tol).all()), ("out", r, float((err / tol).max()))


MIXES = [  # n, length, Hq, Hkv, page
    ([1], [1], 1, 1, 16), ([1], [2], 4, 1, 1), ([1, 1, 1], [5, 64, 65], 8, 2, 16), ([1], [5000], 8, 2, 16), ([3, 0, 8], [3, 40, 333], 4, 4, 25),
    ([17, 1, 33, 64], [17, 700, 90, 64], 2, 2, 32), ([65, 5], [400, 5], 8, 1, 64), ([1] * 40, list(range(1, 400, 10)), 4, 2, 16),
    ([130], [130], 3, 1, 100), ([2, 2], [1000, 1], 32, 1, 256), ([1, 7], [63, 129], 24, 8, 7), ([0, 0], [10, 0], 2, 1, 4), ([300, 2], [900, 450], 8, 2, 64)]


@pytest.mark.parametrize("n,length,Hq,Hkv,page", MIXES)
@pytest.mark.parametrize("D,dtype,layout", [(64, "f16", "nhd"), (80, "bf16", "hnd"), (96, "f16", "hnd"), (128, "bf16", "nhd")])
def test_attend(n, length, Hq, Hkv, page, D, dtype, layout):
    # (n above length: causal queries in front see nothing)
    c = Case(n, length, Hq, Hkv, D, page, dtype, layout, pad=3, seed=len(n) + D)
    for causal in (True, False):
        out = torch.full_like(c.q, 9.0, memory_format=torch.contiguous_format)
        lse = torch.full((c.q.shape[0], Hq), 9.0, device=out.device)
        got = c.attend(causal=causal, out=out, lse=lse)
        assert got[0] is out and got[1] is lse and int(got[2]) == 0
        c.check(out, lse, causal)
        assert bool((out[sum(n):] == 9.0).all()) and bool((lse[sum(n):] == 9.0).all())
        again = [c.attend(causal=causal, most=max(n)) for _ in range(2)]       # (laid out in another way, perhaps)
        t = sum(n)
        c.check(again[0][0], again[0][1], causal)
        assert torch.equal(again[0][0][:t], again[1][0][:t]) and torch.equal(again[0][1][:t], again[1][1][:t])


SHARED = [  # n, length, Hq, Hkv, page, groups, shared
    ([1, 1], [200, 300], 4, 2, 16, [0, 2], [128]), ([1] * 20, list(range(700, 720)), 8, 2, 32, [0, 20], [650]),
    ([4, 0, 3, 5, 1], [800, 300, 310, 420, 99], 4, 4, 25, [0, 3, 5], [290, 70]), ([1, 2, 3], [100, 90, 80], 2, 1, 16, [0, 0, 3, 3], [5, 200, 3]),
    ([40, 30, 64], [1000, 1100, 1064], 8, 2, 64, [0, 3], [999]), ([9, 9], [520, 520], 16, 1, 16, [0, 2], [512]),
    ([1, 1, 1, 1], [600, 700, 650, 900], 8, 8, 100, [0, 1, 3], [512, 400]), ([300, 260], [1300, 1500], 8, 2, 64, [0, 2], [1000]),
    ([70] * 5, [570, 600, 640, 700, 572], 4, 1, 16, [0, 5], [500]), ([3, 2, 0], [64, 64, 64], 4, 2, 16, [0, 3], [0])]


@pytest.mark.parametrize("n,length,Hq,Hkv,page,groups,shared", SHARED)
@pytest.mark.parametrize("D,dtype,layout", [(64, "bf16", "hnd"), (80, "f16", "nhd"), (128, "bf16", "nhd")])
def test_shared_tokens(n, length, Hq, Hkv, page, groups, shared, D, dtype, layout):
    c = Case(n, length, Hq, Hkv, D, page, dtype, layout, groups, shared, pad=2, seed=D)
    for causal in (True, False):
        out, lse, status = c.attend(causal=causal, most=max(n))
        assert int(status) == 0
        c.check(out, lse, causal)


def test_shared_tokens_are_read_through_the_first_row_alone():
    c = Case([1] * 6, [600] * 6, 4, 2, 64, 16, groups=[0, 6], shared=[512], seed=3)
    want = c.attend()
    c.table[1:, :32] = -5                          # pages that are none
    got = c.attend()
    assert int(got[2]) == 0 and torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


def test_strides_and_scale():
    c = Case([5, 2], [90, 300], 6, 2, 64, 16, "f16", seed=9, q_pad=8)
    wide = torch.zeros((7, 6, 136), dtype=c.q.dtype, device=c.q.device)
    c.scale = 0.31
    out, lse, _ = c.attend(scale=0.31, out=wide[..., 72:])
    c.check(out, lse)
    assert bool((wide[..., :72] == 0).all())
    c.scale = -0.2
    out, lse, _ = c.attend(scale=-0.2)
    c.check(out, lse)
    for n, length in (([5, 2], [64, 300]), ([150], [260])):
        c = Case(n, length, 6, 2, 64, 16, "f16", seed=10)
        for scale in (0.0, -0.3):
            c.scale = scale
            out, lse, _ = c.attend(scale=scale)
            c.check(out, lse)


def test_extreme_scores():
    """Scores far apart: one key takes all; and all far below zero."""
    c = Case([3], [500], 4, 2, 128, 16, seed=11, spread=60.0)
    out, lse, _ = c.attend()
    c.check(out, lse)
    c.q.fill_(-30.0)
    c.k[c.table[0].long()] = 30.0
    for r in c.keys:
        r.fill_(30.0)
    out, lse, _ = c.attend()
    c.check(out, lse)


def test_what_is_not_finite_stays_with_the_queries_that_see_it():
    c = Case([4, 2], [100, 60], 4, 2, 64, 16, seed=12)
    want, want_lse, _ = c.attend()
    p = 98                                         # the third of four new tokens
    at = int(c.table[0, p // 16]), p % 16
    for cache in (c.k, c.v):
        for bad in (math.nan, math.inf):
            old = cache[at].clone()
            cache[at] = bad
            out, lse, status = c.attend()
            cache[at] = old
            assert int(status) == 0
            same = [0, 1, 4, 5]
            assert torch.equal(out[same], want[same]) and torch.equal(lse[same], want_lse[same])
            if cache is c.v or math.isnan(bad):
                assert not bool(torch.isfinite(out[[2, 3]].float()).all(-1).any())


@pytest.mark.parametrize("what", ["offset", "tokens", "negative", "length", "group", "shared", "most"])
def test_plans_that_are_out_of_range_compute_nothing(what):
    c = Case([2, 3], [50, 60], 4, 2, 64, 16, groups=[0, 2], shared=[32], seed=4)
    if what == "offset":
        c.offset = i32([0, 4, 3])
    elif what == "tokens":
        c.offset = i32([0, 2, 6])
    elif what == "negative":
        c.offset = i32([-1, 2, 5])
    elif what == "length":
        c.length = i32([50, 16 * c.table.shape[1] + 1])
    elif what == "group":
        c.group = i32([0, 3])
    elif what == "shared":
        c.shared = i32([-1])
    out, lse = torch.full_like(c.q, 3.0, memory_format=torch.contiguous_format), torch.full((5, 4), 3.0, device=c.q.device)
    got = c.attend(out=out, lse=lse, most=2 if what == "most" else None)
    assert int(got[2]) == SHAPE and bool((out == 3.0).all()) and bool((lse == 3.0).all())


def test_bad_pages_are_told_and_touch_no_other_request():
    c = Case([1, 2], [50, 60], 4, 2, 64, 16, seed=5)
    want, want_lse, _ = c.attend()
    c.table[0, 1] = c.k.shape[0]
    out, lse, status = c.attend()
    assert int(status) == SHAPE and torch.equal(out[1:], want[1:]) and torch.equal(lse[1:], want_lse[1:])
    score, status = ardiff.ardiff_attend_weights(c.q, c.k, c.table, c.length, c.offset, want_lse, torch.zeros((2, c.table.shape[1] * 16), device=out.device))
    assert int(status) == SHAPE


def test_what_is_not_finite_in_blocks_of_many_rows():
    """The same where 256 rows, and 300 keys in three tiles, are worked on together."""
    for D, dtype in ((64, "bf16"), (80, "f16"), (128, "bf16")):
        c = Case([200, 70], [300, 75], 4, 2, D, 16, dtype, seed=13)
        want, want_lse, _ = c.attend()
        for at_new in (0, 30, 150, 199):
            p = 100 + at_new
            at = int(c.table[0, p // 16]), p % 16
            for cache, bad in ((c.k, math.nan), (c.v, math.nan), (c.v, math.inf)):
                old = cache[at].clone()
                cache[at] = bad
                out, lse, status = c.attend()
                cache[at] = old
                assert int(status) == 0
                same = list(range(at_new)) + list(range(200, 270))
                assert torch.equal(lse[same], want_lse[same])
                # the same operands in another order of fp32 sums (of at most 300 terms: 300 2^-23 of the largest value), rounded once each
                off = (out[same].double() - want[same].double()).abs()
                tol = torch.finfo(out.dtype).eps * want[same].double().abs() + 300 * 2.0 ** -23 * float(c.values[0].abs().max())
                assert bool((off <= tol).all()) and torch.equal(out[200:], want[200:])
                assert not bool(torch.isfinite(out[at_new:200].float()).all(-1).any())


# ---- weights ------------------------------------------------------------------------------------
@pytest.mark.parametrize("n,length,Hq,Hkv,page", MIXES)
@pytest.mark.parametrize("D,dtype,layout", [(64, "f16", "nhd"), (80, "bf16", "hnd"), (96, "bf16", "nhd"), (128, "bf16", "nhd")])
def test_weights(n, length, Hq, Hkv, page, D, dtype, layout):
    c = Case(n, length, Hq, Hkv, D, page, dtype, layout, pad=1, seed=len(n) + D)
    R, N = len(n), c.table.shape[1] * page
    g = c.g
    first = [0 if r % 2 else max(0, length[r] // 3) for r in range(R)]
    for causal, use_first in ((True, True), (False, False)):
        lse = c.attend(causal=causal)[1]
        wide = torch.rand((R, N + 3), device=g.device, generator=g)
        score = wide[:, :N]
        new = torch.full((R, N), -4.0, device=g.device)
        got, status = ardiff.ardiff_attend_weights(c.q, c.k, c.table, c.length, c.offset, lse, score.contiguous(), first=i32(first) if use_first else None,
                                                   decay=0.75, causal=causal, new_score=new)
        assert got is new and int(status) == 0
        for r in range(R):
            f = first[r] if use_first else 0
            L, t0 = length[r], sum(n[:r])
            assert bool((new[r, L:] == -4.0).all()) and bool((new[r, :min(f, L)] == -4.0).all())
            if L <= f:
                continue
            want = torch.zeros((L,), dtype=torch.float64, device=g.device)
            tol = 2.0 ** -22 * score[r, :L].double()
            old = max(0, L - n[r])
            want[:old] = 0.75 * score[r, :old].double()
            if n[r]:
                x, off = c.scores(r, causal)
                given = lse[t0:t0 + n[r]].double()[..., None]
                w = torch.where(given > -math.inf, torch.exp(x - given), torch.zeros_like(x))
                want += w.sum((0, 1))
                # scores and exponential as above, lse times log2 e rounded, sums of n Hq terms
                tol = tol + w.sum((0, 1)) * (off + 2.0 ** -19 + 2.0 ** -23 * float(given[given > -math.inf].abs().max() if bool((given > -math.inf).any()) else 0)
                                             + 2.0 ** -24 * n[r] * Hq)
            err = (new[r, f:L].double() - want[f:]).abs()
            assert bool((err <= tol[f:] + 1e-30).all()), (r, float((err / (tol[f:] + 1e-30)).max()))
        # in place: the same
        ardiff.ardiff_attend_weights(c.q, c.k, c.table, c.length, c.offset, lse, score, first=i32(first) if use_first else None, decay=0.75,
                                     causal=causal, new_score=score)
        for r in range(R):
            f = first[r] if use_first else 0
            assert torch.equal(score[r, f:length[r]], new[r, f:length[r]])


def test_weights_add_up_to_the_queries():
    """Every query and head gives one in all."""
    c = Case([6, 1], [900, 300], 8, 2, 128, 64, seed=21)
    lse = c.attend()[1]
    score = torch.zeros((2, c.table.shape[1] * 64), device=lse.device)
    new, _ = ardiff.ardiff_attend_weights(c.q, c.k, c.table, c.length, c.offset, lse, score, new_score=score)
    total = new.double().sum(1).cpu()
    assert abs(float(total[0]) - 48) < 48 * 2.0 ** -12 and abs(float(total[1]) - 8) < 8 * 2.0 ** -12


@pytest.mark.parametrize("what", ["offset", "length"])
def test_weights_out_of_range_write_nothing(what):
    c = Case([2, 3], [50, 60], 4, 2, 64, 16, seed=4)
    lse = c.attend()[1]
    if what == "offset":
        c.offset = i32([0, 2, 9])
    else:
        c.length = i32([-1, 60])
    new = torch.full((2, c.table.shape[1] * 16), 5.0, device=lse.device)
    _, status = ardiff.ardiff_attend_weights(c.q, c.k, c.table, c.length, c.offset, lse, torch.zeros_like(new), new_score=new)
    assert int(status) == SHAPE and bool((new == 5.0).all())


# ---- eviction -----------------------------------------------------------------------------------
def evicted(score, position, length, budget, first, seen, recent):
    """Of one request, in lists: what is at every place below the new length."""
    keep = min(length, max(budget, 0, min(max(first, 0), length)))
    f = min(max(first, 0), length)
    weight = []
    for p in range(f, length):
        s = score[p] if score[p] == score[p] else -math.inf
        weight.append((-(math.inf if position[p] >= seen - recent else s), p))
    stays = set(range(f)) | {p for _, p in sorted(weight)[:keep - f]}
    tail = iter([p for p in sorted(stays) if p >= keep])
    return [p if p in stays else next(tail) for p in range(keep)]


@pytest.mark.parametrize("R,page,longest,D,H,dtype,kind", [
    (1, 16, 1, 64, 1, torch.bfloat16, "some"), (3, 16, 100, 64, 2, torch.float16, "some"), (5, 7, 300, 80, 3, torch.bfloat16, "ties"), (2, 64, 5000, 128, 1, torch.bfloat16, "some"),
    (4, 32, 2000, 8, 2, torch.float32, "odd"), (9, 1, 50, 64, 1, torch.bfloat16, "ties"), (1, 256, 45000, 64, 1, torch.bfloat16, "some"), (40, 25, 200, 96, 2, torch.float16, "odd")])
@pytest.mark.parametrize("layout", ["nhd", "hnd"])
def test_evict(R, page, longest, D, H, dtype, kind, layout):
    dev = require_cuda()
    g = torch.Generator(device=dev).manual_seed(R + longest)
    width = -(-longest // page) + 1
    N, pages = width * page, R * width
    shape = (pages, page, H, D) if layout == "nhd" else (pages, H, page, D)
    k, v = [torch.randn(shape, device=dev, generator=g).to(dtype) for _ in range(2)]
    if layout == "hnd":
        k, v = k.transpose(1, 2), v.transpose(1, 2)
    table = torch.randperm(pages, device=dev, generator=g).to(torch.int32).view(R, width)
    length = [int(x) for x in torch.randint(1, longest + 1, (R,), device=dev, generator=g)]
    length[0] = longest
    budget = [int(x) for x in torch.randint(-1, longest + 1, (R,), device=dev, generator=g)]
    first = [[0, 3, 10, -2, longest + 5][r % 5] for r in range(R)]
    score = torch.rand((R, N), device=dev, generator=g)
    if kind == "ties":
        score = (score * 4).floor()
    if kind == "odd":
        score = torch.where(score < 0.1, torch.full_like(score, math.nan), torch.where(score < 0.2, torch.full_like(score, -math.inf), score))
        score = torch.where(score > 0.9, torch.full_like(score, math.inf), torch.where(score > 0.8, -0.0 * score, torch.where(score > 0.7, -score, score)))
    position = torch.argsort(torch.rand((R, N), device=dev, generator=g), 1).to(torch.int32).contiguous()
    seen = i32([N + 5] * R)
    for use, recent in ((True, 30), (False, 4), (False, 0)):
        kw = dict(position=position, seen=seen) if use else {}
        k2, v2 = k.clone(), v.clone()
        if layout == "hnd":
            k2, v2 = [x.transpose(1, 2).contiguous().transpose(1, 2) for x in (k, v)]
        new_score, new_position = torch.full_like(score, -7.0), torch.full_like(position, -7) if use else None
        source = torch.full_like(position, -7)
        got = ardiff.ardiff_pages_evict(i32(length), i32(budget), score, table, k2, v2, first=i32(first), recent=recent, new_score=new_score,
                                        new_position=new_position, source=source, **kw)
        assert int(got[3]) == 0
        for r in range(R):
            pos = position[r].tolist() if use else list(range(N))
            want = evicted(score[r].tolist(), pos, length[r], budget[r], first[r], N + 5 if use else length[r], recent)
            n = len(want)
            assert int(got[0][r]) == n and source[r, :n].tolist() == want and bool((source[r, n:] == -7).all())
            at = torch.tensor(want, device=dev, dtype=torch.long)
            assert torch.equal(new_score[r, :n].view(torch.int32), score[r, at].view(torch.int32)) and bool((new_score[r, n:] == -7.0).all())
            if use:
                assert torch.equal(new_position[r, :n], position[r, at]) and bool((new_position[r, n:] == -7).all())
            p = torch.arange(N, device=dev)
            where = table[r].long()[p // page], p % page
            for old, new in ((k, k2), (v, v2)):
                rows = old[where].clone()
                assert torch.equal(new[where][:n], rows[at]) and torch.equal(new[where][n:], rows[n:])
    # in place
    s2, p2, l2 = score.clone(), position.clone(), i32(length)
    ardiff.ardiff_pages_evict(l2, i32(budget), s2, table, k.clone(), v.clone(), first=i32(first), position=p2, seen=seen, recent=30, new_length=l2,
                              new_score=s2, new_position=p2)
    for r in range(R):
        want = evicted(score[r].tolist(), position[r].tolist(), length[r], budget[r], first[r], N + 5, 30)
        at = torch.tensor(want, device=dev, dtype=torch.long)
        assert int(l2[r]) == len(want) and torch.equal(p2[r, :len(want)], position[r, at])


def test_evict_tells_lengths_and_pages_that_are_out_of_range():
    dev = require_cuda()
    k, v = [torch.randn((8, 16, 1, 64), device=dev).half() for _ in range(2)]
    table = i32([[0, 1, 2], [3, 4, 5], [6, 99, 7]])
    score = torch.arange(48, device=dev).float().repeat(3, 1)
    k0, v0 = k.clone(), v.clone()
    new, new_score, _, status = ardiff.ardiff_pages_evict(i32([49, 40, 20]), i32([10, 10, 15]), score, table, k, v, new_score=torch.zeros_like(score))
    assert int(status) == SHAPE and new.tolist() == [49, 10, 15]
    # request 2: place 15 moves to place 0 inside page 6, places 16 .. 19 would move from page 99
    k0[6, 0], v0[6, 0] = k0[6, 15], v0[6, 15]
    assert torch.equal(k[:3], k0[:3]) and torch.equal(k[6:], k0[6:]) and torch.equal(v[6:], v0[6:])
    assert torch.equal(k[3, :10], torch.cat([k0[4, 14:], k0[5, :8]]))
    assert bool((new_score[0] == 0).all())


# ---- together -----------------------------------------------------------------------------------
def test_a_round_from_extension_to_eviction_captured():
    """Pages are extended, tokens rotated into them, attended to, their weights added up, the cache cut down and pages given back: eagerly,
    and as a captured graph that is replayed; both against attention over lists that are kept on the host."""
    dev = require_cuda()
    R, Hq, Hkv, D, page, width, budget = 3, 8, 2, 64, 8, 16, 40
    dt = torch.bfloat16
    freq = (10000.0 ** -(torch.arange(32, device=dev) / 32.0)).float()

    def world():
        return dict(length=torch.zeros((R,), dtype=torch.int32, device=dev), table=torch.zeros((R, width), dtype=torch.int32, device=dev),
                    free=torch.arange(R * width, dtype=torch.int32, device=dev), count=i32([R * width]), k=torch.zeros((R * width, page, Hkv, D), dtype=dt, device=dev),
                    v=torch.zeros((R * width, page, Hkv, D), dtype=dt, device=dev), score=torch.zeros((R, width * page), device=dev),
                    position=torch.zeros((R, width * page), dtype=torch.int32, device=dev), seen=torch.zeros((R,), dtype=torch.int32, device=dev),
                    add=i32([0] * R), qkv=torch.zeros((64, Hq + 2 * Hkv, D), dtype=dt, device=dev), where=torch.zeros((1, 64), dtype=torch.int32, device=dev),
                    slot=torch.zeros((64,), dtype=torch.int64, device=dev), at=torch.zeros((64,), dtype=torch.int32, device=dev),
                    request=torch.zeros((64,), dtype=torch.int32, device=dev), out=torch.zeros((64, Hq, D), dtype=dt, device=dev), lse=torch.zeros((64, Hq), device=dev))

    def step(w):
        offset, _, _, status = ardiff.ardiff_pages_extend(w["length"], w["add"], w["table"], w["free"], w["count"], page, w["slot"], w["at"], w["request"],
                                                          new_length=w["length"], new_free_count=w["count"])
        q, k, v = w["qkv"][:, :Hq], w["qkv"][:, Hq:Hq + Hkv], w["qkv"][:, Hq + Hkv:]
        qr = ardiff.ardiff_rotary_append(q, k, v, w["where"], freq, w["slot"], w["k"], w["v"], count=offset[-1:])
        _, _, status2 = ardiff.ardiff_attend_pages(qr, w["k"], w["v"], w["table"], w["length"], offset, out=w["out"], lse=w["lse"])
        _, status3 = ardiff.ardiff_attend_weights(qr, w["k"], w["table"], w["length"], offset, w["lse"], w["score"], decay=0.5, new_score=w["score"])
        at, r = w["at"].long(), w["request"].long()
        live = torch.arange(64, device=dev) < offset[-1]
        flat = torch.where(live, r * (width * page) + at, torch.full_like(at, R * width * page))
        w["position"].copy_(torch.cat([w["position"].view(-1), w["position"].view(-1)[:1]]).index_copy(0, flat, w["where"][0])[:-1].view(R, -1))
        w["seen"].add_(w["add"])
        new, _, _, status4 = ardiff.ardiff_pages_evict(w["length"], i32_budget, w["score"], w["table"], w["k"], w["v"], position=w["position"], seen=w["seen"],
                                                       recent=6, new_score=w["score"], new_position=w["position"])
        _, status5 = ardiff.ardiff_pages_truncate(w["length"], new, w["table"], w["free"], w["count"], page, new_free_count=w["count"])
        w["length"].copy_(new)
        return torch.cat([status, status2, status3, status4, status5])

    i32_budget = i32([budget] * R)
    eager, graphed = world(), world()
    step(world())                                  # what is loaded on first use is loaded outside the capture
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        told = step(graphed)
    for name, x in world().items():
        graphed[name].copy_(x)
    tokens = [[] for _ in range(R)]                # of every request: (position, key, value, score) on the host
    g = torch.Generator(device=dev).manual_seed(5)
    for turn in range(6):
        add = [[30, 20, 1], [4, 0, 9], [8, 8, 8], [1, 1, 1], [20, 2, 7], [3, 30, 1]][turn]
        qkv = torch.randn((64, Hq + 2 * Hkv, D), device=dev, generator=g).to(dt)
        where = [len_ for r in range(R) for len_ in range(int(eager["seen"][r]), int(eager["seen"][r]) + add[r])]
        for w in (eager, graphed):
            w["add"].copy_(i32(add))
            w["qkv"].copy_(qkv)
            w["where"].zero_()
            w["where"][0, :len(where)] = i32(where)
        assert step(eager).tolist() == [0] * 5
        graph.replay()
        assert told.tolist() == [0] * 5
        n = sum(add)
        assert torch.equal(eager["out"][:n], graphed["out"][:n]) and torch.equal(eager["length"], graphed["length"])
        # the host's version
        q, k = ardiff.ardiff_rotary(qkv[:, :Hq], qkv[:, Hq:Hq + Hkv], eager["where"], freq)
        v, t = qkv[:, Hq + Hkv:], 0
        for r in range(R):
            for i in range(add[r]):
                tokens[r].append([where[t], k[t].double(), v[t].double(), 0.0])
                K, V = torch.stack([x[1] for x in tokens[r]]).repeat_interleave(4, 1), torch.stack([x[2] for x in tokens[r]]).repeat_interleave(4, 1)
                w = torch.softmax(torch.einsum("hd,lhd->hl", q[t].double(), K) / 8.0, -1)
                want, size = torch.einsum("hl,lhd->hd", w, V), torch.einsum("hl,lhd->hd", w, V.abs())
                tol = (2.0 ** -8 * 1.01 + 2.0 ** -12) * size + 2.0 ** -8 * want.abs()
                assert bool(((eager["out"][t].double() - want).abs() <= tol).all())
                t += 1
            # which tokens stayed, by their positions; those of no new token among them are the recent ones at least
            L = int(eager["length"][r])
            assert L == min(len(tokens[r]), budget)
            there = eager["position"][r, :L].tolist()
            byp = {x[0]: x for x in tokens[r]}
            assert len(set(there)) == L and set(there) <= set(byp)
            newest = max(byp, default=0)
            assert all(p in there for p in byp if p >= newest + 1 - 6)
            tokens[r] = [byp[p] for p in there]
        used = sum(-(-int(x) // page) for x in eager["length"])
        assert int(eager["count"]) == R * width - used == int(graphed["count"])


def test_a_cache_beyond_32_bits_and_keys_and_values_side_by_side():
    """Pages at the end of a pool of 9 GB whose keys and values lie side by side: tokens are rotated into it, attended to by few and by many rows, weighed,
    evicted; pages of 64 tokens (boxes) and of 60."""
    dev = require_cuda()
    for page in (64, 60):
        H, D, per = 1, 64, 2 * page * 64 * 2
        pages = (9 << 30) // per
        pool = torch.empty((pages, 2, page, H, D), dtype=torch.float16, device=dev)
        k, v = pool[:, 0], pool[:, 1]
        R, L, new, width = 3, 400, 20, 8
        table = (pages - 1 - torch.arange(R * width, device=dev, dtype=torch.int32)).view(R, width).contiguous()
        assert int(table.min()) * per > 1 << 32
        g = torch.Generator(device=dev).manual_seed(page)
        T = R * L
        x = torch.randn((T, 6, D), device=dev, generator=g).half()
        p = torch.arange(L, device=dev)
        slot = (table.long()[:, p // page] * page + p % page).reshape(-1)
        freq = torch.zeros((32,), device=dev)                              # (turned by nothing)
        q = ardiff.ardiff_rotary_append(x[:, :4], x[:, 4:5], x[:, 5:6], torch.zeros((1, T), dtype=torch.int32, device=dev), freq, slot, k, v)
        assert torch.equal(q, x[:, :4])
        for n in (2, new):                                                 # 8 rows, 80 rows
            rows = torch.cat([q.view(R, L, 4, D)[r, L - n:] for r in range(R)])
            offset, length = i32([n * r for r in range(R + 1)]), i32([L] * R)
            out, lse, status = ardiff.ardiff_attend_pages(rows, k, v, table, length, offset, most=n)
            score, status2 = ardiff.ardiff_attend_weights(rows, k, table, length, offset, lse, torch.zeros((R, width * page), device=dev))
            assert int(status) == 0 and int(status2) == 0
            for r in range(R):
                K, V = x.view(R, L, 6, D)[r, :, 4].double(), x.view(R, L, 6, D)[r, :, 5].double()
                s = torch.einsum("nhd,ld->nhl", rows[n * r:n * (r + 1)].double(), K) / 8.0
                s = s.masked_fill(torch.arange(L, device=dev)[None, None, :] > (L - n + torch.arange(n, device=dev))[:, None, None], -math.inf)
                w = torch.softmax(s, -1)
                want = torch.einsum("nhl,ld->nhd", w, V)
                # the weight and the result rounded to f16, values up to about 4
                assert float((out[n * r:n * (r + 1)].double() - want).abs().max()) <= 2.0 ** -11 * 2 * 4.5 + 2.0 ** -12
                assert float((score[r, :L].double() - w.sum((0, 1))).abs().max()) <= 2.0 ** -11
        before = torch.stack([k[table[1].long()[p // page], p % page], v[table[1].long()[p // page], p % page]]).clone()
        src = torch.zeros((R, width * page), dtype=torch.int32, device=dev)
        new_length, _, _, status = ardiff.ardiff_pages_evict(i32([L] * R), i32([50] * R), score, table, k, v, source=src)
        assert int(status) == 0 and new_length.tolist() == [50] * R
        at = src[1, :50].long()
        after = torch.stack([k[table[1].long()[p // page], p % page], v[table[1].long()[p // page], p % page]])
        assert torch.equal(after[:, :50], before[:, at]) and torch.equal(after[:, 50:], before[:, 50:])
        del pool, k, v


def test_many_requests_and_many_groups():
    """More requests than the plan keeps, a group a request or two, one after the other."""
    R = 1500
    n, length = [r % 3 for r in range(R)], [(r * 37) % 200 + r % 3 for r in range(R)]
    groups = list(range(0, R, 2)) + [R]
    shared = [80 if g % 2 else 0 for g in range(len(groups) - 1)]
    c = Case(n, length, 2, 1, 64, 16, groups=groups, shared=shared, seed=2)
    out, lse, status = c.attend()
    assert int(status) == 0
    c.check(out, lse)
    plain = c.attend(group=None, shared=None)
    c.check(plain[0], plain[1])


def test_two_graphs_and_an_eager_call_at_once():
    """Two captured calls share nothing; replayed beside each other, and beside an eager one."""
    c, d = Case([1] * 20, [500 + 9 * i for i in range(20)], 8, 2, 128, 16, seed=5), Case([100], [900], 8, 2, 128, 16, seed=6)
    want = [x.attend() for x in (c, d)]
    torch.cuda.synchronize()
    graphs, held = [], []
    for x in (c, d):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            held.append(x.attend())
        graphs.append(graph)
    streams = [torch.cuda.Stream() for _ in graphs]
    for _ in range(5):
        for graph, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                graph.replay()
        eager = c.attend()
        torch.cuda.synchronize()
        for w, x in zip(want, held):
            assert torch.equal(w[0], x[0]) and torch.equal(w[1], x[1])
        assert torch.equal(eager[0], want[0][0])


def test_calls_at_once_on_two_streams():
    cases = [Case([1] * 30, [700 + 7 * i for i in range(30)], 8, 2, 128, 16, seed=s) for s in (1, 2)]
    want = [c.attend() for c in cases]
    streams = [torch.cuda.Stream() for _ in cases]
    torch.cuda.synchronize()
    got = []
    for _ in range(10):
        got.append([c.attend(stream=s) for c, s in zip(cases, streams)])
    torch.cuda.synchronize()
    for pair in got:
        for w, x in zip(want, pair):
            assert torch.equal(w[0], x[0]) and torch.equal(w[1], x[1])


@pytest.mark.parametrize("page,n,length", [(64, [300, 40, 1], [700, 333, 500]), (25, [300, 1], [420, 90]), (16, [1, 2], [300, 40])])
def test_rows_that_lie_in_memory_once(page, n, length):
    """Caches whose heads or pages, and queries whose heads or tokens, are one another's: strides of 0."""
    c = Case(n, length, 8, 4, 128, page, seed=12)
    q, k, v = c.q, torch.nan_to_num(c.k), torch.nan_to_num(c.v)

    def results(q, k, v):
        out, lse, status = ardiff.ardiff_attend_pages(q, k, v, c.table, c.length, c.offset)
        score = torch.ones((len(n), c.table.shape[1] * page), device=q.device)
        score, status2 = ardiff.ardiff_attend_weights(q, k, c.table, c.length, c.offset, lse, score, new_score=score)
        assert int(status) == 0 and int(status2) == 0
        return out, lse, score

    for qs, ks in ((q[:, :1].expand_as(q), k), (q[:1].expand_as(q), k), (q, k[:, :, :1].expand_as(k)), (q, k[:1].expand_as(k)), (q, k[:, :1].expand_as(k))):
        vs = v if ks is k else v[:, :, 1:2].expand_as(v)
        same, apart = results(qs, ks, vs), results(qs.contiguous(), ks.contiguous(), vs.contiguous())
        for a, b in zip(same, apart):                  # (queries by boxes or by rows: the same sums)
            assert torch.equal(a, b)


@pytest.mark.parametrize("dtype,largest", [("bf16", 3e38), ("f16", 6e4)])
@pytest.mark.parametrize("n,page", [(300, 64), (300, 25), (12, 16)])
def test_the_largest_values_stay_with_the_queries_that_see_them(dtype, largest, n, page):
    c = Case([n], [n + 140], 2, 2, 64, page, dtype, seed=13)
    want = c.attend()
    last = torch.arange(n + 132, n + 140, device=c.q.device)          # seen by the last eight queries alone
    c.v[c.table[0].long()[last // page], last % page] = largest
    got = c.attend()
    assert torch.equal(got[0][:n - 8], want[0][:n - 8]) and torch.equal(got[1], want[1])


@pytest.mark.parametrize("n,length,Hq,Hkv,page,groups,shared", [
    ([1] * 7, [3, 900, 65, 64, 1, 0, 2000], 16, 16, 25, None, None), ([2, 4, 1], [700, 4, 1500], 32, 8, 16, None, None),
    ([1, 5, 3], [333, 1200, 90], 12, 6, 32, None, None), ([1, 1], [5000, 17], 12, 12, 64, None, None), ([1, 2], [900, 40], 3, 3, 7, None, None),
    ([2, 3, 1, 1], [800, 777, 900, 40], 16, 8, 25, [0, 3], [700]), ([1], [40], 16, 16, 1, None, None)])
@pytest.mark.parametrize("D,dtype,layout", [(80, "bf16", "nhd"), (96, "f16", "nhd"), (80, "f16", "hnd")])
def test_few_rows_of_heads_that_share_lines_of_memory(n, length, Hq, Hkv, page, groups, shared, D, dtype, layout):
    c = Case(n, length, Hq, Hkv, D, page, dtype, layout, groups, shared, pad=1, seed=len(n) * D)
    for most in (None, max(n)):
        out, lse, status = c.attend(most=most)
        assert int(status) == 0
        c.check(out, lse)


@pytest.mark.parametrize("D,dtype", [(64, "f16"), (96, "bf16"), (128, "bf16")])
@pytest.mark.parametrize("n,Hq,Hkv", [(8, 32, 8), (1, 8, 8), (3, 4, 1)])
def test_one_request_cut_into_many_pieces(n, Hq, Hkv, D, dtype):
    c = Case([n], [8000], Hq, Hkv, D, 64, dtype, seed=n)
    out, lse, status = c.attend(most=n)
    assert int(status) == 0
    c.check(out, lse)


@pytest.mark.parametrize("decoding,chunks,Hq,Hkv,D,page", [(40, [64], 32, 8, 128, 16), (64, [300, 9], 16, 4, 64, 64), (200, [33, 64], 8, 2, 80, 25), (30, [120], 16, 8, 128, 32)])
def test_decoding_and_prompts_in_one_batch(decoding, chunks, Hq, Hkv, D, page):
    """Many units of few rows and few of many: joined by half CTAs and by whole ones, in one call."""
    n = [1] * decoding + chunks
    length = [2000 - 13 * r for r in range(decoding // 2)] + [700 + r for r in range(decoding - decoding // 2)] + [1000 + x for x in chunks]
    c = Case(n, length, Hq, Hkv, D, page, seed=decoding)
    want = c.attend()
    assert int(want[2]) == 0
    c.check(want[0], want[1])
    for _ in range(20):
        got = c.attend()
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


@pytest.mark.parametrize("D,dtype,page", [(64, "bf16", 16), (80, "f16", 25), (128, "bf16", 64)])
def test_what_is_not_finite_where_the_maximum_rises(D, dtype, page):
    """300 new tokens behind 20000: several tiles a CTA, and scores that rise far above the first ones' in the tiles that hold a value that is not finite."""
    c = Case([300], [20300], 8, 8, D, page, dtype, seed=D)
    p = torch.arange(20000, 20300, device=c.q.device)
    c.keys[0][20000:] *= 8
    c.k[c.table[0].long()[p // page], p % page] = c.keys[0][20000:]
    want, want_lse, _ = c.attend()
    c.check(want, want_lse)
    for at_new in (40, 200, 299):
        at = int(c.table[0, (20000 + at_new) // page]), (20000 + at_new) % page
        for bad in (math.nan, math.inf):
            old = c.v[at].clone()
            c.v[at] = bad
            out, lse, status = c.attend()
            c.v[at] = old
            assert int(status) == 0 and torch.equal(lse, want_lse)
            assert not bool(torch.isfinite(out[at_new:].float()).any())
            out[at_new:] = want[at_new:]
            c.check(out, lse)


def heavy_and_light(dtype, R, n, G, causal, D, page):
    """One key has most of the weight and a value of 0; 16383 others, 2^19 to 2^20.6 times lighter each and all alike, so that their roundings add up, make
    the result; in front of R requests, that look at the same pages, so that a worker goes through all of them behind the heavy one. Results by heads, and
    the same in 64 bits."""
    dev, dt, H, L = require_cuda(), TYPES[dtype], 8, 16384
    g = torch.Generator(device=dev).manual_seed(D + n)
    pages = -(-L // page)
    k, v = torch.zeros((pages * page, H, D), device=dev), torch.zeros((pages * page, H, D), device=dev)
    k[1:L, :, 0] = -math.log(2.0) * (19.0 + 0.23 * torch.arange(H, device=dev))
    v[1:L] = 0.5 + torch.rand((L - 1, H, D), device=dev, generator=g)
    k, v = k.to(dt).view(pages, page, H, D), v.to(dt).view(pages, page, H, D)
    q = torch.zeros((R * n, H * G, D), dtype=dt, device=dev)
    q[..., 0] = 1
    table = torch.arange(pages, device=dev, dtype=torch.int32).repeat(R, 1)
    out, lse, status = ardiff.ardiff_attend_pages(q, k, v, table, i32([L] * R), i32([n * r for r in range(R + 1)]), most=n, scale=1.0, causal=causal)
    assert int(status) == 0
    w = torch.exp(k.reshape(-1, H, D)[:L, :, 0].double())
    want = torch.einsum("lh,lhd->hd", w, v.reshape(-1, H, D)[:L].double()) / w.sum(0)[:, None]
    return out.view(R * n, H, G, D).double(), lse.view(R * n, H, G).double(), want[None, :, None], torch.log(w.sum(0))[None, :, None]


HEAVY = [(160, 1, 1, True), (160, 4, 2, False), (20, 64, 4, False)]


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("R,n,G,causal", HEAVY)
@pytest.mark.parametrize("D,page", [(64, 16), (128, 25)])
def test_light_keys_behind_a_heavy_one_keep_their_bits(dtype, R, n, G, causal, D, page):
    out, _, want, _ = heavy_and_light(dtype, R, n, G, causal, D, page)
    # all values are positive, so errors are relative: the weight as an operand and the result, half a step each; an exponential of 2^-22 whose argument, up to
    # 2^5, is off by 2^-23 of it; sums in 32 bits of at most 2^14 weights, which are 2^-5 of the row's: all together below 2^-11.5 of the result in the sum that
    # it is divided by, and 2^-14 in its own, of 2^10 products of 16 keys
    eps = torch.finfo(TYPES[dtype]).eps / 2
    err = ((out - want) / want).abs()
    assert float(err.max()) <= 2 * eps + eps * eps + 2.0 ** -11.5, float(err.max())


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("R,n,G,causal", HEAVY)
@pytest.mark.parametrize("D,page", [(64, 16), (128, 25)])
def test_sums_of_weights_do_not_add_up_roundings(dtype, R, n, G, causal, D, page):
    _, lse, _, want = heavy_and_light(dtype, R, n, G, causal, D, page)
    # roundings of 2^-24 of the sum each: up to 32 in a tile or a group of steps, 32 of groups or 128 of tiles, 16 where parts are joined: 192 at the most; the heavy
    # key's exponential 2^-22, those of the light ones, 2^-5 of the sum, 2^-18; a logarithm of 2^-22 and lse's own rounding
    assert float((lse - want).abs().max()) <= 192 * 2.0 ** -24 + 2.0 ** -19


@pytest.mark.parametrize("D,dtype,page", [(64, "bf16", 16), (80, "f16", 25), (128, "bf16", 64), (128, "f16", 1)])
@pytest.mark.parametrize("shared", [200, 256, 333])
def test_what_is_not_finite_among_shared_tokens(D, dtype, page, shared):
    """Every query sees the shared tokens: a value that is +inf makes its column +inf, wherever the shared tokens end inside a tile of the own ones."""
    n = [40, 50, 20]
    c = Case(n, [700, 900, 1210], 4, 1, D, page, dtype, groups=[0, 3], shared=[shared], seed=shared, spread=0.3)
    want, want_lse, _ = c.attend()
    c.check(want, want_lse)
    for p in (shared - 1, shared - 60, 3):
        at = c.table[:, p // page].long()
        old = c.v[at, p % page].clone()
        c.v[at, p % page, :, 5] = math.inf
        for kw in ({}, dict(group=None, shared=None)):
            out, lse, status = c.attend(**kw)
            assert int(status) == 0 and bool(torch.isposinf(out[..., 5]).all())
            out[..., 5] = want[..., 5]
            c.check(out, lse)
        c.v[at, p % page] = old
