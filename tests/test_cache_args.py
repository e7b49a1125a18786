"""Refusals of the operators around a draft model's cache: every one is made before anything is launched, so they need no GPU."""
import math
import struct

import pytest

import paper_2512_08537_b200 as ardiff

NULL, SHAPE, ALIGN, UNSUPPORTED = (ardiff.ARDIFF_ERR_NULL, ardiff.ARDIFF_ERR_SHAPE, ardiff.ARDIFF_ERR_ALIGN,
                                   ardiff.ARDIFF_ERR_UNSUPPORTED)
P = 4096                                   # an address that nothing is read from
BIG = 1 << 40


def call(name, defaults, kw):
    """The call with a structure of these fields, in their order."""
    assert set(kw) <= set(defaults), kw
    fields = {**defaults, **kw}
    stream = fields.pop("stream")
    form = "".join("d" if k in ("scale", "decay") else "q" for k in fields)
    return getattr(ardiff.lib(), name)(struct.pack(form, *(0 if v is None else v for v in fields.values())), stream)


@pytest.mark.parametrize("name", ["ardiff_rotary", "ardiff_rotary_backward", "ardiff_rotary_append", "ardiff_attend_pages",
                                  "ardiff_attend_weights", "ardiff_pages_evict"])
def test_no_structure(name):
    assert getattr(ardiff.lib(), name)(None, None) == NULL


@pytest.mark.parametrize("name,fields", [("ardiff_rotary", ["q_heads", "k_heads", "dtype", "width", "axes", "pairs"]),
                                         ("ardiff_rotary_append", ["q_heads", "k_heads", "width", "axes", "pairs", "pages", "page"]),
                                         ("ardiff_attend_pages", ["q_heads", "heads", "pages", "page", "head_width", "width", "requests", "groups", "most"]),
                                         ("ardiff_attend_weights", ["q_heads", "heads", "pages", "page", "head_width", "width", "requests"]),
                                         ("ardiff_pages_evict", ["requests", "recent", "width", "pages", "page", "heads", "head_width"])])
def test_what_32_bits_do_not_hold(name, fields):
    made = {"ardiff_rotary": turn, "ardiff_rotary_append": append, "ardiff_attend_pages": attend, "ardiff_attend_weights": weights,
            "ardiff_pages_evict": evict}[name]()
    for f in fields:
        for off in (1 << 32, -(1 << 32), 1 << 62):
            assert call(name, made, {f: made[f] + off}) == SHAPE, f


def turn(**kw):
    return dict(q=P, q_token=512, q_head=64, q_out=P, q_out_token=512, q_out_head=64, q_heads=8, k=P, k_token=128, k_head=64, k_out=P,
                k_out_token=128, k_out_head=64, k_heads=2, dtype=ardiff.ARDIFF_BF16, n=4, width=64, position=P, position_ld=4, axes=1, freq=P, axis=None,
                pairs=32, neighbours=0, stream=None)


ROTARY = [(dict(n=-1), SHAPE), (dict(n=1 << 31), SHAPE), (dict(width=0), SHAPE), (dict(width=513), SHAPE), (dict(pairs=33), SHAPE), (dict(pairs=-1), SHAPE),
          (dict(axes=0), SHAPE), (dict(q_heads=-1), SHAPE), (dict(q_heads=1025), SHAPE), (dict(k_heads=1025), SHAPE), (dict(dtype=3), UNSUPPORTED),
          (dict(dtype=-1), UNSUPPORTED), (dict(q=None), NULL), (dict(k=None), NULL), (dict(q_out=None), NULL), (dict(position=None), NULL), (dict(freq=None), NULL),
          (dict(q=P + 1), ALIGN), (dict(q_out=P + 1), ALIGN), (dict(position_ld=-1), SHAPE)]


@pytest.mark.parametrize("name", ["ardiff_rotary", "ardiff_rotary_backward"])
@pytest.mark.parametrize("kw,code", ROTARY + [(dict(k_out=None), NULL), (dict(dtype=ardiff.ARDIFF_F32, k=P + 2), ALIGN)])
def test_rotary_refuses(name, kw, code):
    assert call(name, turn(), kw) == code


@pytest.mark.parametrize("name", ["ardiff_rotary", "ardiff_rotary_backward"])
def test_rotary_of_nothing(name):
    assert call(name, turn(), dict(n=0, q=None, k=None)) == 0
    assert call(name, turn(), dict(q_heads=0, k_heads=0, q=None, k=None)) == 0


def append():
    return dict(q=P, q_token=512, q_head=64, q_out=P, q_out_token=512, q_out_head=64, q_heads=8, k=P, k_token=128, k_head=64, v=P, v_token=128, v_head=64,
                k_heads=2, dtype=ardiff.ARDIFF_BF16, n=4, width=64, position=P, position_ld=4, axes=1, freq=P, axis=None, pairs=32, neighbours=0, slot=P,
                count=None, k_cache=P, k_cache_page=2048, k_cache_token=128, k_cache_head=64, v_cache=P, v_cache_page=2048, v_cache_token=128,
                v_cache_head=64, pages=4, page=16, stream=None)


@pytest.mark.parametrize("kw,code", ROTARY + [(dict(slot=None), NULL), (dict(v=None), NULL), (dict(k_cache=None), NULL), (dict(v_cache=None), NULL),
                                              (dict(page=0), SHAPE), (dict(pages=-1), SHAPE), (dict(v_cache=P + 1), ALIGN)])
def test_rotary_append_refuses(kw, code):
    assert call("ardiff_rotary_append", append(), kw) == code


CACHE = dict(k_cache=P, k_page=2048, k_token=128, k_head=64)


def attend():
    return dict(q=P, q_token=512, q_head=64, q_heads=8, tokens=4, dtype=ardiff.ARDIFF_BF16, **CACHE, v_cache=P, v_page=2048, v_token=128, v_head=64, pages=4,
                page=16, heads=2, head_width=64, table=P, width=4, requests=2, length=P, offset=P, groups=1, group=P, shared=P, most=1, scale=0.125, causal=1,
                out=P, out_token=512, out_head=64, lse=P, lse_token=8, status=P, workspace=P, workspace_bytes=BIG, stream=None)


ATTEND = [(dict(requests=-1), SHAPE), (dict(requests=(1 << 20) + 1), SHAPE), (dict(tokens=-1), SHAPE), (dict(tokens=1 << 28), SHAPE), (dict(heads=0), SHAPE),
          (dict(q_heads=9), SHAPE), (dict(q_heads=1), SHAPE), (dict(q_heads=2048), SHAPE), (dict(pages=-1), SHAPE), (dict(page=0), SHAPE), (dict(width=-1), SHAPE),
          (dict(page=1 << 16, width=1 << 15), SHAPE), (dict(scale=math.inf), SHAPE), (dict(scale=math.nan), SHAPE),
          (dict(dtype=ardiff.ARDIFF_F32), UNSUPPORTED), (dict(dtype=7), UNSUPPORTED), (dict(head_width=72), UNSUPPORTED), (dict(head_width=256), UNSUPPORTED),
          (dict(workspace_bytes=8), SHAPE), (dict(workspace_bytes=0), SHAPE), (dict(k_token=124), ALIGN), (dict(k_head=4), ALIGN), (dict(k_page=1), ALIGN),
          (dict(q_token=513), ALIGN), (dict(q_head=68), ALIGN), (dict(q=P + 8), ALIGN), (dict(k_cache=P + 8), ALIGN), (dict(workspace=P + 8), ALIGN)] + \
    [(dict([(name, None)]), NULL) for name in ("q", "k_cache", "table", "length", "offset", "lse", "status", "workspace")]


@pytest.mark.parametrize("kw,code", ATTEND + [(dict(most=-1), SHAPE), (dict(page=1 << 20, width=1 << 10, heads=16, q_heads=16), SHAPE), (dict(groups=-1), SHAPE), (dict(groups=(1 << 20) + 1), SHAPE), (dict(v_token=4), ALIGN), (dict(out_token=4), ALIGN),
                                              (dict(out_head=1), ALIGN), (dict(out=P + 2), ALIGN), (dict(v_cache=P + 2), ALIGN)] +
                         [(dict([(name, None)]), NULL) for name in ("v_cache", "out", "group", "shared")])
def test_attend_refuses(kw, code):
    assert call("ardiff_attend_pages", attend(), kw) == code


def weights():
    return dict(q=P, q_token=512, q_head=64, q_heads=8, tokens=4, dtype=ardiff.ARDIFF_BF16, **CACHE, pages=4, page=16, heads=2, head_width=64, table=P, width=4,
                requests=2, length=P, offset=P, first=None, lse=P, lse_token=8, score=P, ld=64, scale=0.125, decay=1.0, causal=1, new_score=P, new_ld=64,
                status=P, workspace=P, workspace_bytes=BIG, stream=None)


@pytest.mark.parametrize("kw,code", ATTEND + [(dict(decay=math.nan), SHAPE), (dict(decay=math.inf), SHAPE), (dict(ld=-1), SHAPE), (dict(new_ld=-1), SHAPE),
                                              (dict(score=None), NULL), (dict(new_score=None), NULL)])
def test_weights_refuse(kw, code):
    assert call("ardiff_attend_weights", weights(), kw) == code


def evict():
    return dict(requests=2, length=P, budget=P, first=None, score=P, ld=64, position=None, seen=None, recent=0, table=P, width=4, dtype=ardiff.ARDIFF_F16,
                **CACHE, v_cache=P, v_page=2048, v_token=128, v_head=64, pages=4, page=16, heads=2, head_width=64, new_length=P, new_score=P, new_position=None,
                source=None, new_ld=64, status=P, workspace=P, workspace_bytes=BIG, stream=None)


@pytest.mark.parametrize("kw,code", [
    (dict(requests=-1), SHAPE), (dict(requests=(1 << 20) + 1), SHAPE), (dict(page=0), SHAPE), (dict(width=-1), SHAPE), (dict(page=1 << 16, width=1 << 15), SHAPE),
    (dict(pages=-1), SHAPE), (dict(heads=0), SHAPE), (dict(head_width=0), SHAPE), (dict(head_width=1 << 20), SHAPE), (dict(recent=-1), SHAPE), (dict(ld=-1), SHAPE),
    (dict(new_ld=-1), SHAPE), (dict(dtype=5), UNSUPPORTED), (dict(head_width=4), UNSUPPORTED), (dict(k_token=4), ALIGN), (dict(v_head=12), ALIGN),
    (dict(k_cache=P + 8), ALIGN), (dict(workspace=P + 4), ALIGN), (dict(workspace_bytes=16), SHAPE)] +
    [(dict([(name, None)]), NULL) for name in ("length", "budget", "score", "table", "k_cache", "v_cache", "new_length", "new_score", "status", "workspace")])
def test_evict_refuses(kw, code):
    assert call("ardiff_pages_evict", evict(), kw) == code


def test_workspaces():
    L = ardiff.lib()
    assert L.ardiff_attend_workspace(-1, 0, 1, 1, 1, 64) == SHAPE and L.ardiff_attend_workspace(1, 0, 1, 3, 2, 64) == SHAPE
    assert L.ardiff_attend_workspace(1, 0, 1 << 31, 8, 1, 64) == SHAPE and L.ardiff_pages_evict_workspace(4, 16, -1) == SHAPE
    assert L.ardiff_attend_weights_workspace(-1) == SHAPE
    small, large = L.ardiff_attend_workspace(1, 0, 1, 8, 2, 64), L.ardiff_attend_workspace(500, 3, 4000, 8, 2, 64)
    assert 0 < small < large
    assert L.ardiff_pages_evict_workspace(3, 16, 5) > 0 and L.ardiff_attend_weights_workspace(3) >= 32


@pytest.mark.parametrize("scale", [math.inf, -math.inf, math.nan, 1e39, 3e38, -3e38])
def test_scales_that_are_not_finite_in_powers_of_two(scale):
    assert call("ardiff_attend_pages", attend(), dict(scale=scale)) == SHAPE
    assert call("ardiff_attend_weights", weights(), dict(scale=scale)) == SHAPE


def test_results_where_inputs_are():
    """Only in place: at the same distances, and not where other blocks still read them."""
    assert call("ardiff_attend_pages", attend(), {}) == UNSUPPORTED                   # q and out are both at P
    for name in ("ardiff_rotary", "ardiff_rotary_backward"):
        for kw in (dict(q_out_token=1024), dict(q_out_head=128), dict(k_out_token=256), dict(k_out_head=1024)):
            assert call(name, turn(), kw) == UNSUPPORTED, kw
    assert call("ardiff_attend_weights", weights(), dict(new_ld=80)) == SHAPE
    assert call("ardiff_pages_evict", evict(), dict(new_ld=80)) == SHAPE
    assert call("ardiff_pages_evict", evict(), dict(new_ld=80, new_score=2 * P, position=P, new_position=P)) == SHAPE


@pytest.mark.parametrize("n,heads,width,token,head,good", [
    (3, 2, 64, 128, 64, True), (3, 2, 64, 127, 64, False), (3, 2, 64, 72, 64, False), (3, 2, 64, 136, 72, True), (3, 2, 64, 135, 72, False), (3, 2, 64, 64, 192, True),
    (3, 2, 64, 64, 191, False), (3, 2, 64, 64, 136, False), (3, 2, 64, 72, 208, True), (3, 2, 64, 72, 207, False), (1, 2, 64, 8, 64, True), (3, 1, 64, 64, 8, True),
    (3, 1, 64, 56, 8, False), (1, 2, 64, 8, 56, False), (0, 2, 64, 0, 64, True), (2, 2, 1, 2, 1, True), (2, 2, 1, 1, 1, False), (2, 2, 64, 64, 64, False)])
def test_results_whose_rows_overlap_are_refused(n, heads, width, token, head, good):
    import torch
    ardiff._t()
    like = torch.empty((n, heads, width), dtype=torch.float16)
    x = torch.empty((4096,), dtype=torch.float16).as_strided((n, heads, width), (token, head, 1))
    places = [t * token + h * head + d for t in range(n) for h in range(heads) for d in range(width)]
    assert (len(set(places)) == len(places)) == good
    if good:
        assert ardiff._out_heads(x, like, -1) == (x.data_ptr(), token, head)
    else:
        with pytest.raises(AssertionError, match="overlap"):
            ardiff._out_heads(x, like, -1)


def test_caches_whose_rows_are_one_another_s_are_not_written():
    import torch
    cache = torch.empty((3, 4, 2, 64), dtype=torch.float16)
    assert ardiff._written_cache_args(cache, torch.float16, -1) == (cache.data_ptr(), 512, 128, 64)
    assert ardiff._written_cache_args(cache.transpose(1, 2), torch.float16, -1) == (cache.data_ptr(), 512, 64, 128)
    for x in (cache[:1].expand(3, 4, 2, 64), cache[:, :1].expand(3, 4, 2, 64), cache[:, :, :1].expand(3, 4, 2, 64)):
        assert 0 in ardiff._cache_args(x, torch.float16, -1)[1:]
        with pytest.raises(AssertionError, match="written"):
            ardiff._written_cache_args(x, torch.float16, -1)
    one = torch.empty((1, 1, 1, 64), dtype=torch.float16).as_strided((1, 1, 1, 64), (0, 0, 0, 1))
    assert ardiff._written_cache_args(one, torch.float16, -1) == (one.data_ptr(), 0, 0, 0)


@pytest.mark.parametrize("page,width", [(1, (1 << 31) - 1), (1, (1 << 31) - (1 << 14) + 1), (127, 16909320), ((1 << 31) - 1, 1)])
def test_places_whose_numbers_come_close_to_2_31_are_refused(page, width):
    """Kernels step through them by thousands at once, in 32 bits."""
    assert call("ardiff_attend_pages", attend(), dict(page=page, width=width)) == SHAPE
    assert call("ardiff_attend_weights", weights(), dict(page=page, width=width)) == SHAPE
    assert call("ardiff_pages_evict", evict(), dict(page=page, width=width)) == SHAPE
    assert ardiff.lib().ardiff_pages_evict_workspace(1, page, width) == SHAPE
    assert ardiff.lib().ardiff_pages_evict_workspace(1, 1, (1 << 31) - (1 << 14)) > 1 << 32


def test_workspace_of_attention_holds_what_its_pieces_need():
    L = ardiff.lib()
    # one token of one request, 32 heads: a place of 4 rows for each of 160 x 8 warps
    assert L.ardiff_attend_workspace(1, 0, 1, 32, 8, 128) < 4 << 20
    # without groups two places a worker at the most, however many tokens: 2 x 160 x (8 x 32 + 256) rows of 128 values, and the list of blocks
    for tokens in (20000, 65536):
        assert L.ardiff_attend_workspace(64, 0, tokens, 32, 8, 128) < 90 << 20
    # with groups every row may be joined, in both lists
    assert 2 * 65536 * 32 * 128 * 4 < L.ardiff_attend_workspace(64, 1, 65536, 32, 8, 128) < 2 * 65536 * 32 * 130 * 4 + (50 << 20)
    for args in ((1, 8, 1, 64), (3, 8, 2, 64), (17, 1, 1, 128)):
        assert 0 < L.ardiff_attend_workspace(2, 0, *args) <= L.ardiff_attend_workspace(2, 1, *args)


@pytest.mark.parametrize("tokens,q_heads,heads", [(1 << 61, 8, 2), (1 << 62, 4, 2), (1 << 60, 16, 16), ((1 << 61) + 1, 8, 8), (1 << 54, 1024, 1)])
def test_numbers_of_tokens_whose_products_wrap(tokens, q_heads, heads):
    assert ardiff.lib().ardiff_attend_workspace(2, 0, tokens, q_heads, heads, 64) == SHAPE
    kw = dict(tokens=tokens, q_heads=q_heads, heads=heads, workspace_bytes=(1 << 63) - 1)
    assert call("ardiff_attend_pages", attend(), dict(kw, out=2 * P)) == SHAPE
    assert call("ardiff_attend_weights", weights(), kw) == SHAPE
