"""Token sampling against its definition in 64 bits, through the C ABI.

A token is right or wrong: the definition here sums in fp64 in another order than the kernel, so the two can differ only where a
border lies within some 1e-13 of a sum, which random inputs do not meet; rows of equal logits have whole sums, exact on both
sides. logprob = y ln 2 - ln Z is formed in fp64 and rounded once: half a step of fp32, with y and Z good to 1e-12."""
import math

import numpy as np
import pytest
import torch

import paper_2512_08537_b200 as ardiff
from gpu_util import require_cuda

pytestmark = pytest.mark.gpu
DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}


def define(x, u, T=None, k=None, p=None, mp=None):
    """(token, ln probability) of one row of float64 values."""
    T, k, p, mp = 1.0 if T is None else float(T), 0 if k is None else int(k), 1.0 if p is None else float(p), \
        0.0 if mp is None else float(mp)
    u = float(u)
    if not (0 <= u < 1 and 0 <= T < math.inf and p == p and mp == mp) or not np.isfinite(x.max()) or np.isnan(x).any():
        return -1, math.nan
    if T == 0:
        return int(np.argmax(x)), 0.0
    order = np.argsort(-x, kind="stable")
    if 0 < k < len(x):
        order = order[:k]
    with np.errstate(over="ignore", under="ignore"):
        y = (x[order] - x.max()) / T
    w = np.exp(y)
    if p < 1:
        before = np.concatenate([[0.0], np.cumsum(w)[:-1]])
        keep = before < p * w.sum()
        keep[0] = True
        order, w, y = order[keep], w[keep], y[keep]
    if mp > 0:
        keep = w >= min(mp, 1.0)
        order, w, y = order[keep], w[keep], y[keep]
    by = np.argsort(order)
    order, w, y = order[by], w[by], y[by]
    cum = np.cumsum(w)
    j = int(np.searchsorted(cum, u * cum[-1], side="right"))
    while w[j] == 0:
        j += 1
    return int(order[j]), float(y[j] - np.log(cum[-1]))


def check(x, u, T=None, k=None, p=None, mp=None):
    """x: CPU tensor [n, V] (any strides along n); settings: lists or None."""
    d = require_cuda()
    n = x.shape[0]
    f = lambda v, t=torch.float32: None if v is None else torch.tensor(v, dtype=t)  # noqa: E731
    T, k, p, mp, u = f(T), f(k, torch.int32), f(p), f(mp), f(u)
    on = lambda v: None if v is None else v.to(d)  # noqa: E731
    base = x.storage_offset()
    buf = torch.as_strided(x, (x.untyped_storage().nbytes() // x.element_size(),), (1,), 0).to(d)
    xd = torch.as_strided(buf, x.shape, x.stride(), base)
    token, logprob = ardiff.ardiff_sample_tokens(xd, on(u), on(T), on(k), on(p), on(mp))
    token, logprob = token.tolist(), logprob.double().tolist()
    rows = x.double().numpy()
    at = lambda v, i: None if v is None else v[i].item()  # noqa: E731
    for i in range(n):
        want, lp = define(rows[i], u[i].item(), at(T, i), at(k, i), at(p, i), at(mp, i))
        assert token[i] == want, (i, token[i], want, u[i].item(), at(T, i), at(k, i), at(p, i), at(mp, i))
        if want < 0:
            assert math.isnan(logprob[i])
        else:
            # half a step of fp32 of the value, and what 1e-12 in y and ln Z can move
            assert abs(logprob[i] - lp) <= abs(lp) * 2.0 ** -24 + 2e-12 * (1 + abs(lp)), (i, logprob[i], lp)
    return token


def rows(n, V, dtype, seed, kind="power", pad=0, offset=0):
    g = torch.Generator().manual_seed(seed)
    buf = torch.zeros(n * (V + pad) + offset, dtype=dtype)
    x = buf[offset:].reshape(n, V + pad)[:, :V]
    if kind == "power":                            # falls off like a power of the rank
        a = 0.5 + 1.5 * torch.rand((n, 1), generator=g)
        v = 10 - a * torch.log(torch.rand((n, V), generator=g) * V + 1) + 0.3 * torch.randn((n, V), generator=g)
    elif kind == "flat":
        v = torch.randn((n, V), generator=g)
    elif kind == "few values":
        v = torch.randint(-3, 4, (n, V), generator=g).float()
    elif kind == "equal":
        v = torch.full((n, V), 1.25)
    elif kind == "narrow":                         # differences of the last bits
        v = 1000.0 + torch.randn((n, V), generator=g) * 1e-3
    elif kind == "wide":
        v = 1e4 * torch.randn((n, V), generator=g)
    elif kind == "around zero":                    # values over many binades on both sides of 0
        v = torch.randn((n, V), generator=g).sign() * torch.exp(-20 * torch.rand((n, V), generator=g))
    x.copy_(v.to(dtype))
    return x, torch.rand((n,), generator=g).tolist()


SIZES = [(3, 1), (3, 2), (4, 5), (4, 8), (5, 100), (3, 1000), (3, 1024), (3, 1025), (4, 1500), (150, 2000), (3, 5000), (2, 32768),
         (2, 100003), (80, 66000), (1, 131072), (1, 262144)]


@pytest.mark.parametrize("dtype", sorted(DTYPES))
@pytest.mark.parametrize("n,V", SIZES)
def test_no_filter_and_largest(dtype, n, V):
    x, u = rows(n, V, DTYPES[dtype], seed=V)
    check(x, u)
    check(x, u, T=[0.7] * n)
    check(x, u, T=[0.0] * n)
    check(x, u, mp=[0.02] * n)


@pytest.mark.parametrize("dtype", sorted(DTYPES))
@pytest.mark.parametrize("n,V", SIZES)
def test_top_k_and_top_p(dtype, n, V):
    x, u = rows(n, V, DTYPES[dtype], seed=V + 1)
    check(x, u, k=[50] * n, T=[0.8] * n)
    check(x, u, k=[1] * n)
    check(x, u, p=[0.9] * n, T=[0.6] * n)
    check(x, u, p=[0.5] * n, k=[20] * n, mp=[0.05] * n)


@pytest.mark.parametrize("kind", ["power", "flat", "few values", "equal", "narrow", "wide", "around zero"])
@pytest.mark.parametrize("dtype", sorted(DTYPES))
@pytest.mark.parametrize("n,V", [(6, 700), (6, 3000), (4, 40000), (2, 150001)])
def test_every_filter_on_every_kind_of_row(kind, dtype, n, V):
    x, u = rows(n, V, DTYPES[dtype], seed=V + 2, kind=kind)
    for k in (3, 700, V // 3, V - 1):
        check(x, u, k=[k] * n)
        check(x, u, k=[k] * n, p=[0.97] * n)
    for p in (0.0, 1e-6, 0.3, 0.95, 0.999999, float(np.nextafter(np.float32(1), np.float32(0)))):
        check(x, u, p=[p] * n, T=[1.5] * n)
    for mp in (1e-4, 0.5, 1.0, 2.0):
        check(x, u, mp=[mp] * n)
        check(x, u, k=[V // 2] * n, mp=[mp] * n)
    check(x, u, k=[V // 2] * n, p=[0.8] * n, mp=[0.1] * n, T=[3.0] * n)


@pytest.mark.parametrize("dtype", sorted(DTYPES))
def test_settings_row_by_row_and_those_that_are_none(dtype):
    V, n = 5000, 24
    x, u = rows(n, V, DTYPES[dtype], seed=5)
    u[:3] = [0.0, 1 - 2.0 ** -24, 0.5]
    T = [1.0, 0.0, 0.5, 1e-30, 1e30, 1e-45, 3e38, 2.0] * 3
    k = [0, 5, -3, 5000, 6000, 1, 4999, 2 ** 31 - 1] * 3
    p = [1.0, 0.9, 2.0, -1.0, 0.0, 0.5, 0.99, 0.9] * 3
    mp = [0.0, -1.0, 0.1, 0.0, 1.5, 0.0, 0.01, 0.0] * 3
    for shift in range(3):
        turn = lambda v, s: v[s:] + v[:s]  # noqa: E731
        check(x, u, T=T, k=turn(k, shift), p=turn(p, 3 * shift), mp=turn(mp, 5 * shift))


@pytest.mark.parametrize("dtype", sorted(DTYPES))
def test_rows_and_settings_that_give_no_token(dtype):
    V, n = 3000, 16
    x, u = rows(n, V, DTYPES[dtype], seed=6)
    x[0, 7] = math.nan
    x[1, 2999] = math.inf
    x[2] = -math.inf
    x[3, 0] = math.nan
    u[4], u[5], u[6] = 1.0, -0.1, math.nan
    T, k, p, mp = [1.0] * n, [10] * n, [0.9] * n, [0.01] * n
    T[3] = 0.0
    T[7], T[8], T[9] = -1.0, math.nan, math.inf
    p[10], mp[11] = math.nan, math.nan
    got = check(x, u, T=T, k=k, p=p, mp=mp)
    assert got[:12] == [-1] * 12 and min(got[12:]) >= 0
    check(x, u)


@pytest.mark.parametrize("dtype", sorted(DTYPES))
@pytest.mark.parametrize("V", [900, 9000, 70000])
def test_masks(dtype, V):
    n = 8
    x, u = rows(n, V, DTYPES[dtype], seed=7)
    low = torch.finfo(x.dtype).min
    x[0, 1:] = -math.inf                         # one token left
    x[1, : V - 3] = -math.inf
    x[2, 1::2] = -math.inf
    x[3, 1:] = low
    x[4, 1::2] = low
    x[5] = low                                   # all by the type's lowest value: equal
    x[6] = -math.inf
    x[6, V // 2] = -3.0
    x[7] = low
    x[7, 5] = -math.inf
    for kw in (dict(), dict(k=[50] * n), dict(p=[0.9] * n), dict(mp=[0.1] * n), dict(k=[V - 1] * n, p=[0.99] * n),
               dict(T=[0.0] * n)):
        check(x, u, **kw)


@pytest.mark.parametrize("dtype", sorted(DTYPES))
def test_u_of_zero_takes_the_first_token_of_any_weight(dtype):
    """exp(-700) is a weight; exp(-800) is none in fp64."""
    x = torch.zeros((4, 2500), dtype=DTYPES[dtype])
    x[:, 0], x[:, 1] = -800, -700
    x[1, 0] = -math.inf
    x[2, :2] = -math.inf
    x[3, :2000] = -800
    got = check(x, [0.0] * 4)
    assert got == [1, 1, 2, 2000]
    check(x, [0.0] * 4, k=[2499] * 4)
    check(x, [0.0] * 4, p=[0.9999] * 4, k=[3] * 4)


@pytest.mark.parametrize("dtype", sorted(DTYPES))
@pytest.mark.parametrize("n,V,pad,offset", [(5, 500, 3, 0), (4, 501, 0, 1), (3, 33000, 11, 5), (200, 1103, 7, 3)])
def test_rows_at_any_place(dtype, n, V, pad, offset):
    x, u = rows(n, V, DTYPES[dtype], seed=8, pad=pad, offset=offset)
    if pad:
        wide = torch.as_strided(x, (n, V + pad), x.stride(), x.storage_offset())
        wide[:, V:] = 100.0                      # larger than all of the row
    check(x, u)
    check(x, u, k=[40] * n, p=[0.9] * n)
    check(x, u, T=[0.0] * n)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T", [5e-4, 1e-3, 0.02, 900.0, 1e3, 3e3])
@pytest.mark.parametrize("shift", [0.0, 5e4, -5e4, 7e4])
def test_sums_of_the_first_pass_at_any_temperature_and_height(dtype, T, shift):
    """The first pass sums relative to the first few logits of each part: those may be low, the largest far above them, all of
    them high or low, the temperature such that most weights are nothing or nearly all are alike."""
    n, V = 6, 40000
    x, u = rows(n, V, torch.float32, seed=12)
    x[1, :20000] -= 30.0                          # the reference is far below the largest
    x[2, :30000] -= 3000.0
    x[3, :39999] = -3e5
    x[4, 4096:] -= 500.0
    x = (x + shift).to(DTYPES[dtype])
    check(x, u, T=[T] * n)
    check(x, u, T=[T] * n, p=[0.9] * n)
    check(x, u, T=[T] * n, p=[0.9] * n, mp=[0.2] * n)


@pytest.mark.parametrize("n,V", [(1, 4096), (1, 20000), (40, 70000), (300, 9000), (700, 1500)])
def test_settings_that_differ_from_row_to_row_in_one_call(n, V):
    """Rows that are listed, walked, counted and drawn at once, by clusters of every size."""
    g = torch.Generator().manual_seed(V)
    x, u = rows(n, V, torch.bfloat16, seed=13)
    flat, _ = rows(n, V, torch.bfloat16, seed=14, kind="flat")
    x[::3] = flat[::3]
    pick = lambda v: [v[i] for i in torch.randint(0, len(v), (n,), generator=g).tolist()]  # noqa: E731
    check(x, u, T=pick([0.0, 0.7, 1.0, 2.0]), k=pick([0, 1, 40, 1200, V // 2]), p=pick([1.0, 0.5, 0.9, 0.99]), mp=pick([0.0, 0.0, 0.05]))


def test_largest_of_equal_ones_and_both_zeros():
    x = torch.full((4, 4000), -1.0)
    x[0, [70, 3999, 71]] = 2.0
    x[1] = 0.0
    x[1, ::2] = -0.0                              # the zeros are one value: ties by index
    x[2, 3990:] = 0.0
    x[2, 3990::2] = -0.0
    assert check(x, [0.5] * 4, T=[0.0] * 4) == [70, 0, 3990, 0]
    check(x, [0.3, 0.6, 0.9, 0.1], k=[3] * 4)
    check(x, [0.3, 0.6, 0.9, 0.1], k=[3001] * 4)


def test_draws_follow_the_probabilities():
    """u over a grid of 2^16 points: a token of probability P is drawn P 2^16 times, give or take one."""
    V, n = 300, 1 << 16
    g = torch.Generator().manual_seed(1)
    x = (2 * torch.randn((1, V), generator=g)).to(require_cuda())
    u = ((torch.arange(n, device=x.device) + 0.5) / n).float()
    token, logprob = ardiff.ardiff_sample_tokens(x.expand(n, V).contiguous(), u)
    count = torch.bincount(token.long(), minlength=V).double().cpu()
    P = torch.softmax(x[0].double().cpu(), 0)
    assert float((count - P * n).abs().max()) <= 1.0 + 1e-6
    assert bool(((logprob.double().cpu() - torch.log(P)[token.long().cpu()]).abs() <= 1e-6).all())


def test_captured_call_follows_its_buffers_and_streams_do_not_meet():
    d = require_cuda()
    x1, u1 = rows(20, 9000, torch.bfloat16, seed=9)
    x2, u2 = rows(20, 9000, torch.bfloat16, seed=10, kind="flat")
    sets = [(x.to(d), torch.tensor(u, device=d), torch.full((20,), T, device=d), torch.full((20,), k, dtype=torch.int32, device=d),
             torch.full((20,), p, device=d)) for x, u, T, k, p in ((x1, u1, 0.8, 40, 0.9), (x2, u2, 1.1, 0, 0.95))]
    want = [ardiff.ardiff_sample_tokens(*s) for s in sets]
    x, u, T, k, p = (t.clone() for t in sets[0])
    token, logprob = torch.zeros_like(want[0][0]), torch.zeros_like(want[0][1])
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ardiff.ardiff_sample_tokens(x, u, T, k, p, token=token, logprob=logprob)
    for i in (1, 0, 1):
        for to, v in zip((x, u, T, k, p), sets[i]):
            to.copy_(v)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(token, want[i][0]) and torch.equal(logprob, want[i][1])
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(5):
        got = [ardiff.ardiff_sample_tokens(*s, stream=st) for s, st in zip(sets, streams)]
    torch.cuda.synchronize()
    for a, b in zip(got, want):
        assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


def test_no_rows():
    d = require_cuda()
    token, logprob = ardiff.ardiff_sample_tokens(torch.empty((0, 50), device=d), torch.empty((0,), device=d))
    assert token.shape == (0,) and logprob.shape == (0,)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("kw", [{}, {"mp": 1e-9}, {"k": 15000}, {"p": 0.999999}])
@pytest.mark.parametrize("front", [-math.inf, -150.0, -90.0])
def test_tiny_numbers_pass_over_what_weighs_nothing(dtype, kw, front):
    """u below the 24 bits of a generator, in front of which lie masked logits, or ones whose weights are near u or far below it."""
    n, V = 8, 40000
    x, _ = rows(n, V, DTYPES[dtype], seed=15)
    x[:, :20000] = front
    u = [1e-45, 1e-38, 2.0**-126, 1e-30, 2.0**-100, 1e-20, 2.0**-25, 2.0**-24]
    check(x, u, **{name: [v] * n for name, v in kw.items()})
    check(x, u, T=[0.01] * n, **{name: [v] * n for name, v in kw.items()})


@pytest.mark.parametrize("kw", [{}, {"k": 59999}, {"mp": 1e-9}, {"p": 0.9999999}])
def test_draws_that_end_where_masked_logits_begin(kw):
    """The same logits on both sides of masked ones and u = 1/2: the border lies at the masked ones but for rounding, so that the last
    logit of weight before them and the first behind them are both right, and nothing else is."""
    n, half, gap = 256, 10000, 20000
    g = torch.Generator().manual_seed(16)
    v = torch.randn((n, half), generator=g)
    x = torch.cat([v, torch.full((n, gap), -math.inf), v, torch.full((n, gap), -math.inf)], 1)
    if "p" in kw or "mp" in kw:                    # (the borders are kept whatever the filter)
        x[:, [0, half - 1, half + gap, 2 * half + gap - 1]] = 3.0
    d = require_cuda()
    args = {"k": "top_k", "mp": "min_p", "p": "top_p"}
    kw = {args[name]: torch.tensor([w] * n, dtype=torch.int32 if name == "k" else torch.float32, device=d) for name, w in kw.items()}
    token, _ = ardiff.ardiff_sample_tokens(x.to(d), torch.full((n,), 0.5, device=d), **kw)
    assert set(token.tolist()) <= {half - 1, half + gap}


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("mp", [0.5, 0.01, 1e-8, 2.0**-60, 2.0**-61, 1e-30])
@pytest.mark.parametrize("T", [1.0, 0.1])
def test_min_p_that_keeps_more_than_a_list_holds(dtype, mp, T):
    n, V = 4, 60000
    x, u = rows(n, V, DTYPES[dtype], seed=17, kind="flat")
    x *= 8.0 * T
    check(x, u, T=[T] * n, mp=[mp] * n)
    check(x.clamp(max=T), u, T=[T] * n, mp=[mp] * n)


@pytest.mark.parametrize("dtype", sorted(DTYPES))
@pytest.mark.parametrize("u", [0.0, 2.0**-26])
def test_a_small_share_of_thousands_of_largest_ones_with_thousands_far_below(dtype, u):
    """The search by whole numbers looks at the far ones first, with many times the mass that is asked for in front of them. Sums are whole
    numbers, so the cut is exact."""
    lows = [41, 48, 50, 53, 58, 60, 66, 68, 69, 71, 73, 90]
    shares = [0.02, 0.05, 0.1, 0.35, 0.4, 0.45]
    x = torch.empty((len(lows) * len(shares), 6000))
    for i, low in enumerate(lows):
        x[i * len(shares):(i + 1) * len(shares)] = 10.0 - low
    x[:, 1000:4000] = 10.0
    got = check(x.to(DTYPES[dtype]), [u] * len(x), p=shares * len(lows))
    assert set(got) == {1000}


@pytest.mark.parametrize("dtype", sorted(DTYPES))
@pytest.mark.parametrize("u", [0.0, 2.0**-30, 2.0**-25])
def test_nuclei_that_end_below_more_zeros_than_a_list_holds(dtype, u):
    """Positive logits, thousands of zeros (of both signs), and negative ones, among which the nucleus ends."""
    x = torch.cat([torch.linspace(-1.1, -1.0, 1000), torch.ones(1), torch.linspace(0.51, 0.511, 3000), torch.zeros(20000)])
    x = x.repeat(8, 1)
    x[1::2, 10000:] = -0.0
    x[4:, :1000] *= 1e-3
    p = [0.995, 0.99, 0.982, 0.9999, 0.995, 0.99, 0.97, 0.9999]
    check(x.to(DTYPES[dtype]), [u] * 8, p=p)


@pytest.mark.parametrize("u", [0.0, 2.0**-25])
@pytest.mark.parametrize("kind", ["few values", "around zero", "flat"])
@pytest.mark.parametrize("dtype", sorted(DTYPES))
def test_tiny_numbers_and_nuclei_on_both_sides_of_zero(kind, dtype, u):
    x, _ = rows(12, 30000, DTYPES[dtype], seed=18, kind=kind)
    check(x, [u] * 12, p=[0.05, 0.2, 0.35, 0.5, 0.6, 0.7, 0.8, 0.9, 0.95, 0.98, 0.99, 0.999])


def test_a_count_that_ends_among_the_smallest_numbers_below_zero():
    """fp32's least negative numbers directly below thousands of zeros, and a largest logit from which steps of 2^22 numbers lead to the
    border between them."""
    g = torch.Generator().manual_seed(19)
    tiny = (torch.randperm((1 << 22) - 1, generator=g)[:600] + 1).to(torch.int32).view(torch.float32)
    top = torch.tensor([0x3fffffff], dtype=torch.int32).view(torch.float32)
    x = torch.cat([-tiny, torch.zeros(2000), top, torch.rand((1500,), generator=g)])
    x = x[torch.randperm(len(x), generator=g)].repeat(32, 1)
    k = [1501 + 2000 + v for v in (1, 2, 100, 300, 333, 500, 599, 600)] * 4
    check(x, torch.rand((32,), generator=g).tolist(), k=k)
    check(x, [0.0] * 32, k=k, p=[0.999] * 32)
