"""Refusals of the language-model operators: every one is made before anything is launched, so they need no GPU."""
import math

import pytest
import torch

import paper_2512_08537_b200 as ardiff

NULL, SHAPE, ALIGN, UNSUPPORTED = (ardiff.ARDIFF_ERR_NULL, ardiff.ARDIFF_ERR_SHAPE, ardiff.ARDIFF_ERR_ALIGN,
                                   ardiff.ARDIFF_ERR_UNSUPPORTED)
P = 4096                                   # an address that nothing is read from


def extend(**kw):
    a = dict(requests=4, page=16, width=8, length=P, add=P, table=P, free_pages=P, free_capacity=32, free_count=P, max_tokens=64,
             slot=P, position=P, request=P, offset=P, new_length=P, new_free_count=P, status=P, stream=None)
    assert set(kw) <= set(a)
    return ardiff.lib().ardiff_pages_extend(*{**a, **kw}.values())


@pytest.mark.parametrize("kw,code", [
    (dict(requests=-1), SHAPE), (dict(requests=(1 << 20) + 1), SHAPE), (dict(page=0), SHAPE), (dict(width=-1), SHAPE),
    (dict(free_capacity=-1), SHAPE), (dict(free_capacity=1 << 31), SHAPE), (dict(max_tokens=-1), SHAPE),
    (dict(max_tokens=1 << 31), SHAPE)] +
    [(dict([(name, None)]), NULL) for name in ("length", "add", "table", "free_pages", "free_count", "slot", "offset",
                                               "new_length", "new_free_count", "status")])
def test_pages_extend_refuses(kw, code):
    assert extend(**kw) == code


def truncate(**kw):
    a = dict(requests=4, page=16, width=8, length=P, target=P, table=P, free_pages=P, free_capacity=32, free_count=P,
             new_free_count=P, status=P, stream=None)
    assert set(kw) <= set(a)
    return ardiff.lib().ardiff_pages_truncate(*{**a, **kw}.values())


@pytest.mark.parametrize("kw,code", [
    (dict(requests=-1), SHAPE), (dict(requests=(1 << 20) + 1), SHAPE), (dict(page=0), SHAPE), (dict(page=-16), SHAPE),
    (dict(width=-1), SHAPE), (dict(free_capacity=-1), SHAPE), (dict(free_capacity=1 << 31), SHAPE)] +
    [(dict([(name, None)]), NULL) for name in ("length", "target", "table", "free_pages", "free_count", "new_free_count",
                                               "status")])
def test_pages_truncate_refuses(kw, code):
    assert truncate(**kw) == code


def distill(part, **kw):
    a = dict(logits=P, dtype=ardiff.ARDIFF_BF16, n=4, V=100, ld=100, teacher=P, teacher_dtype=ardiff.ARDIFF_F32, ids=P, k=8,
             temperature=1.0)
    a.update({"": dict(loss=P, stats=P), "_backward": dict(stats=P, weight=P, grad=P, ld_grad=100),
              "_step": dict(weight=P, loss=P, stats=P, grad=P, ld_grad=100)}[part])
    a["stream"] = None
    assert set(kw) <= set(a)
    return getattr(ardiff.lib(), "ardiff_distill_topk" + part)(*{**a, **kw}.values())


@pytest.mark.parametrize("part", ["", "_backward", "_step"])
@pytest.mark.parametrize("kw,code", [
    (dict(n=-1), SHAPE), (dict(n=1 << 28), SHAPE), (dict(V=0), SHAPE), (dict(V=(1 << 24) + 1, ld=1 << 25), SHAPE),
    (dict(ld=99), SHAPE), (dict(k=0), SHAPE), (dict(k=1025), SHAPE), (dict(temperature=0.0), SHAPE),
    (dict(temperature=-1.0), SHAPE), (dict(temperature=math.nan), SHAPE), (dict(temperature=math.inf), SHAPE),
    (dict(temperature=1e-39), SHAPE), (dict(temperature=4e-39), SHAPE), (dict(teacher=P + 2), ALIGN), (dict(dtype=3), UNSUPPORTED), (dict(dtype=-1), UNSUPPORTED),
    (dict(teacher_dtype=7), UNSUPPORTED), (dict(logits=P + 1), ALIGN),
    (dict(dtype=ardiff.ARDIFF_F32, logits=P + 2), ALIGN), (dict(logits=None), NULL), (dict(teacher=None), NULL),
    (dict(ids=None), NULL), (dict(stats=None), NULL)])
def test_distill_refuses(part, kw, code):
    assert distill(part, **kw) == code


@pytest.mark.parametrize("part,kw,code", [
    ("", dict(loss=None), NULL), ("_step", dict(loss=None), NULL), ("_step", dict(weight=None), NULL),
    ("_step", dict(grad=None), NULL), ("_backward", dict(weight=None), NULL), ("_backward", dict(grad=None), NULL),
    ("_step", dict(ld_grad=99), SHAPE), ("_backward", dict(ld_grad=99), SHAPE), ("_step", dict(grad=P + 1), ALIGN)])
def test_distill_refuses_what_one_part_needs(part, kw, code):
    assert distill(part, **kw) == code


@pytest.mark.parametrize("part", ["", "_backward", "_step"])
def test_distill_of_no_rows_is_nothing(part):
    assert distill(part, n=0, logits=None, teacher=None, ids=None, stats=None) == ardiff.ARDIFF_OK


def sample(**kw):
    a = dict(logits=P, dtype=ardiff.ARDIFF_BF16, n=4, V=100, ld=100, u=P, temperature=P, top_k=P, top_p=P, min_p=P, token=P,
             logprob=P, stream=None)
    assert set(kw) <= set(a)
    return ardiff.lib().ardiff_sample_tokens(*{**a, **kw}.values())


@pytest.mark.parametrize("kw,code", [
    (dict(n=-1), SHAPE), (dict(n=1 << 28), SHAPE), (dict(V=0), SHAPE), (dict(V=(1 << 18) + 1, ld=1 << 19), SHAPE),
    (dict(ld=99), SHAPE), (dict(dtype=3), UNSUPPORTED), (dict(dtype=-1), UNSUPPORTED), (dict(logits=P + 1), ALIGN),
    (dict(dtype=ardiff.ARDIFF_F32, logits=P + 2), ALIGN), (dict(logits=None), NULL), (dict(u=None), NULL),
    (dict(token=None), NULL), (dict(logprob=None), NULL)])
def test_sample_refuses(kw, code):
    assert sample(**kw) == code


def test_sample_of_no_rows_is_nothing():
    assert sample(n=0, logits=None, u=None, token=None, logprob=None) == ardiff.ARDIFF_OK


def test_tensors_of_the_host_are_refused():
    f, i = torch.zeros(4), torch.zeros(4, dtype=torch.int32)
    table = torch.zeros((4, 2), dtype=torch.int32)
    with pytest.raises(AssertionError):
        ardiff.ardiff_sample_tokens(torch.zeros((4, 8)), f)
    with pytest.raises(AssertionError):
        ardiff.ardiff_distill_topk(torch.zeros((4, 8)), torch.zeros((4, 2)), table)
    with pytest.raises(AssertionError):
        ardiff.ardiff_pages_extend(i, i, table, i, i[:1], 16, torch.zeros(4, dtype=torch.int64))
    with pytest.raises(AssertionError):
        ardiff.ardiff_pages_truncate(i, i, table, i, i[:1], 16)


@pytest.mark.parametrize("page", [2**32 + 16, 2**31, -2**32 + 16])
def test_page_sizes_that_32_bits_cut_off_are_refused(page):
    i = torch.zeros(4, dtype=torch.int32)
    table = torch.zeros((4, 2), dtype=torch.int32)
    with pytest.raises(AssertionError, match="32 bits"):
        ardiff.ardiff_pages_extend(i, i, table, i, i[:1], page, torch.zeros(4, dtype=torch.int64))
    with pytest.raises(AssertionError, match="32 bits"):
        ardiff.ardiff_pages_truncate(i, i, table, i, i[:1], page)


def test_shapes_that_32_bits_cut_off_are_refused():
    """(Tensors without memory: a row of 2^32 + 5 logits has 8 GB.)"""
    made = lambda *shape, t=torch.int32: torch.empty(shape, dtype=t, device="meta")  # noqa: E731
    for V in (2**31, 2**32 + 5):
        with pytest.raises(AssertionError, match="32 bits"):
            ardiff._rows(made(1, V, t=torch.bfloat16))
        with pytest.raises(AssertionError, match="32 bits"):
            ardiff.ardiff_distill_topk(made(1, 8, t=torch.bfloat16), made(1, V, t=torch.float32), made(1, V))
    one = made(1)
    with pytest.raises(AssertionError, match="32 bits"):
        ardiff.ardiff_pages_truncate(one, one, made(1, 2**32 + 4), one, one, 16)
    with pytest.raises(AssertionError, match="32 bits"):
        ardiff.ardiff_pages_truncate(one, one, made(2**32 + 1, 1), one, one, 16)
