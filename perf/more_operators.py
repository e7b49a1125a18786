"""What is timed of the operators around a draft model's cache: one pass through one operator a case.

  rotary   rotary positions with several axes: "append" rotates queries and keys and writes keys and values into their slots of
           a paged cache (serving); "forward" and "backward" rotate queries and keys, or their gradients back (training)
  attend   attention of new tokens over pages, the tokens that a group of requests shares read once for all of them
  weights  the attention weight that every token of the cache has got, added up over queries and heads
  evict    the tokens of least accumulated weight leave the cache, the ones behind the new end move into their places

`run()` makes the framework's calls where `own` is true; where it is false it computes the same in elementary torch
operations, in 32 bits (angles in 64: far positions have no fraction left in 32).
"""
import math

import torch

own = False

DEVICE = "cuda"
DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
# the most that one drawn pass may cost: the largest listed pass of each kind
MAX_ROTARY = 32768 * 40 * 128                 # values rotated
MAX_SCORES = 1 << 31                          # query rows times the longest request's keys
MAX_CACHE = 1 << 29                           # values of the keys that the requests' tables name
MAX_EVICT = 1 << 28                           # values of the keys of all requests


def listed():
    return [
        # decoding: one token each for four streams of text, far into them; latency is all there is
        dict(name="rotary_append_4", op="rotary", part="append", T=4, Hq=16, Hkv=4, D=128, axes=1, far=200000, pairs="half",
             dtype="bf16", page=16, layout="nhd", pad=0),
        # the tokens of 64 images of 16 x 16 (time, row, column), heads of an odd width, the batch padded to a fixed size
        dict(name="rotary_append_16500", op="rotary", part="append", T=16500, Hq=16, Hkv=16, D=80, axes=3, far=64, pairs="half",
             dtype="bf16", page=32, layout="nhd", pad=116),
        # a training step's forward in 32 bits, neighbouring values paired
        dict(name="rotary_forward_5000", op="rotary", part="forward", T=5000, Hq=20, Hkv=20, D=64, axes=2, far=256,
             pairs="neighbours", dtype="f32", page=0, layout="nhd", pad=0),
        # the backward of a video's tokens: the largest
        dict(name="rotary_backward_32768", op="rotary", part="backward", T=32768, Hq=32, Hkv=8, D=128, axes=3, far=128,
             pairs="half", dtype="f16", page=0, layout="nhd", pad=0),
        # one stream of text, one token
        dict(name="attend_1x4096", op="attend", R=1, most=1, Hq=32, Hkv=8, D=128, shared=0, longest=4096, page=16,
             dtype="bf16", layout="nhd", pad=0, causal=True),
        # 64 samples of one long prompt, one token each
        dict(name="attend_64_shared", op="attend", R=64, most=1, Hq=32, Hkv=8, D=128, shared=8192, longest=8704, page=64,
             dtype="bf16", layout="nhd", pad=0, causal=True),
        # drafts of up to 8 tokens verified for 96 requests behind one prompt, heads of 80, pages of an odd size
        dict(name="attend_96_drafts", op="attend", R=96, most=8, Hq=16, Hkv=16, D=80, shared=2000, longest=3500, page=25,
             dtype="f16", layout="hnd", pad=13, causal=True),
        # prompts of up to 1024 tokens behind a shared one of 15000: the largest
        dict(name="attend_4_prompts", op="attend", R=4, most=1024, Hq=32, Hkv=8, D=128, shared=15000, longest=16384, page=64,
             dtype="bf16", layout="nhd", pad=0, causal=True),
        # after a decoding step: a query row a head for each of 128 requests
        dict(name="weights_128_decode", op="weights", R=128, most=1, Hq=32, Hkv=8, D=128, shared=0, longest=4096, page=16,
             dtype="bf16", layout="nhd", pad=0, causal=True),
        # after a prompt: what its last 32 queries look at
        dict(name="weights_8_window", op="weights", R=8, most=32, Hq=32, Hkv=8, D=128, shared=0, longest=16384, page=64,
             dtype="bf16", layout="nhd", pad=0, causal=True),
        # decoding at the limit of the cache: a few tokens too many in each of 128 requests
        dict(name="evict_128_decode", op="evict", R=128, Hkv=8, D=128, longest=2056, budget=2048, page=16, recent=64, first=4,
             dtype="bf16", layout="nhd"),
        # prompts cut down to an eighth
        dict(name="evict_8_prompts", op="evict", R=8, Hkv=8, D=128, longest=16384, budget=2048, page=64, recent=32, first=0,
             dtype="bf16", layout="nhd"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["rotary", "rotary", "attend", "attend", "attend", "weights", "evict"])
    Hkv, D = rng.choice([1, 2, 4, 8, 16]), rng.choice([64, 80, 96, 128])
    c = dict(op=op, Hkv=Hkv, D=D, page=rng.choice([1, 16, 25, 32, 64, 100, 256]), dtype=rng.choice(["bf16", "f16"]),
             layout=rng.choice(["nhd", "nhd", "hnd"]))
    if op == "rotary":
        G = rng.choice([1, 1, 2, 4, 8])
        c.update(part=rng.choice(["append", "forward", "backward"]), Hq=min(Hkv * G, 32), axes=rng.choice([1, 2, 3]),
                 far=_log(rng, 16, 1000000), pairs=rng.choice(["half", "neighbours"]), pad=rng.choice([0, 0, 7]))
        if c["part"] != "append":
            c.update(dtype=rng.choice(sorted(DTYPES)), page=0, layout="nhd", pad=0)
        c["T"] = min(_log(rng, 1, 65536), MAX_ROTARY // ((c["Hq"] + Hkv) * D))
        return c
    if op == "evict":
        c.update(R=_log(rng, 1, 256), longest=_log(rng, 2, 32768), recent=rng.choice([0, 1, 32, 100]), first=rng.choice([0, 0, 4, 50]))
        c["longest"] = max(2, min(c["longest"], MAX_EVICT // (c["R"] * Hkv * D)))
        c["budget"] = max(1, c["longest"] - _log(rng, 1, 16)) if rng.random() < 0.4 else _log(rng, 1, c["longest"])
        return c
    G = rng.choice([1, 2, 4, 8])
    c.update(Hq=min(Hkv * G, 32), most=rng.choice([1, 1, 4, 8, _log(rng, 2, 1024)]), R=_log(rng, 1, 256), longest=_log(rng, 1, 16384),
             pad=rng.choice([0, 0, 9]), causal=rng.random() < 0.8)
    if op == "weights":
        c["most"] = min(c["most"], 64)
    c["R"] = max(1, min(c["R"], 2048 // c["most"]))
    c["longest"] = max(c["most"], min(c["longest"], MAX_CACHE // (c["R"] * Hkv * D), MAX_SCORES // (c["R"] * c["most"] * c["Hq"])))
    c["shared"] = 0
    if c["longest"] > c["most"] and rng.random() < 0.6:
        c["shared"] = _log(rng, 1, c["longest"] - c["most"])
    return c


# ---- inputs -------------------------------------------------------------------------------------
def _gen(seed):
    return torch.Generator(device=DEVICE).manual_seed(int(seed))


def _normal(gen, *shape):
    return torch.randn(shape, device=gen.device, generator=gen)


def _whole(gen, lo, hi, *shape):
    """Whole numbers lo .. hi."""
    return torch.randint(lo, hi + 1, shape, device=gen.device, generator=gen, dtype=torch.int32)


def _cache(gen, pages, case):
    """A pool of pages of keys or of values: [pages, page, heads, width], heads or tokens next to each other in memory."""
    page, H, D = case["page"], case["Hkv"], case["D"]
    shape = (pages, page, H, D) if case["layout"] == "nhd" else (pages, H, page, D)
    x = torch.empty(shape, dtype=DTYPES[case["dtype"]], device=gen.device).normal_(generator=gen)
    return x if case["layout"] == "nhd" else x.transpose(1, 2)


def _frequencies(case, dev):
    """A ladder of frequencies for every axis over its own share of the pairs; an eighth of the pairs stands still where there
    are several axes."""
    P, axes = case["D"] // 2, case["axes"]
    if axes > 1:
        P -= P // 8
    axis = torch.arange(P, device=dev, dtype=torch.int32) * axes // P
    first = torch.searchsorted(axis, axis)
    many = torch.searchsorted(axis, axis, right=True) - first
    rung = (torch.arange(P, device=dev) - first).double() / many.double()
    return torch.pow(10000.0, -rung).float(), axis


def _prepare_rotary(case, gen):
    T, Hq, Hkv, D, dev, dtype = case["T"], case["Hq"], case["Hkv"], case["D"], gen.device, DTYPES[case["dtype"]]
    freq, axis = _frequencies(case, dev)
    s = dict(position=_whole(gen, 0, case["far"], case["axes"], T), freq=freq, axis=axis, neighbours=case["pairs"] == "neighbours")
    # queries, keys and values as one product gives them: slices of a row
    qkv = _normal(gen, T, Hq + 2 * Hkv, D).to(dtype)
    s["q"], s["k"] = qkv[:, :Hq], qkv[:, Hq:Hq + Hkv]
    if case["part"] == "append":
        s["v"] = qkv[:, Hq + Hkv:]
        pages = -(-T // case["page"]) + 3
        s["k_cache"], s["v_cache"] = _cache(gen, pages, case), _cache(gen, pages, case)
        s["slot"] = torch.randperm(pages * case["page"], device=dev, generator=gen)[:T].contiguous()
        s["count"] = torch.full((1,), max(1, T - case["pad"]), dtype=torch.int32, device=dev)
        s["q_out"] = torch.zeros((T, Hq, D), dtype=dtype, device=dev)
    return s


def _new_tokens(case):
    """New tokens of every request where there are many: from half the most up to the most, as many in all whatever the seed."""
    R, most = case["R"], case["most"]
    return [most if case["op"] == "weights" else most - (r * 61 % max(1, most // 2)) for r in range(R)]


def _prepare_attend(case, gen):
    R, most, Hq, Hkv, D, dev = case["R"], case["most"], case["Hq"], case["Hkv"], case["D"], gen.device
    page, shared, longest, dtype = case["page"], case["shared"], case["longest"], DTYPES[case["dtype"]]
    n = _whole(gen, 1 if most == 1 else 0, most, R)
    if most > 8:
        n = torch.tensor(_new_tokens(case), dtype=torch.int32, device=dev)
    n[0] = most
    # every request has its new tokens and some more of its own behind the shared ones
    length = shared + n + (torch.rand((R,), device=dev, generator=gen) * (longest - shared - n + 1)).to(torch.int32)
    length = torch.minimum(length, torch.full_like(length, longest))
    offset = torch.cat([torch.zeros((1,), dtype=torch.int64, device=dev), torch.cumsum(n, 0)]).to(torch.int32)
    width, front = -(-longest // page), shared // page
    pages = front + R * (width - front)
    order = torch.randperm(pages + 5, device=dev, generator=gen).to(torch.int32)
    at = torch.arange(width, device=dev)[None, :]
    mine = front + torch.arange(R, device=dev)[:, None] * (width - front) + at - front
    table = order[torch.where(at < front, at, mine)].contiguous()
    s = dict(k_cache=_cache(gen, pages + 5, case), length=length, offset=offset, table=table, page=page, most=most, longest=longest,
             causal=case["causal"], scale=1.0 / math.sqrt(D))
    if shared > front * page:
        # the page in which the shared part ends is every request's own; its shared tokens are copies of the first one's
        s["k_cache"][table[:, front].long(), :shared - front * page] = s["k_cache"][table[:1, front].long(), :shared - front * page]
    # a few tokens each: a batch of a fixed size, its end unused
    T = (R * most if most <= 8 else sum(_new_tokens(case))) + case["pad"]
    s["q"] = (1.5 * _normal(gen, T, Hq, D)).to(dtype)
    s["status"] = torch.full((1,), -1, dtype=torch.int32, device=dev)
    if case["op"] == "attend":
        s["v_cache"] = _cache(gen, pages + 5, case)
        if shared > front * page:
            s["v_cache"][table[:, front].long(), :shared - front * page] = s["v_cache"][table[:1, front].long(), :shared - front * page]
        s["group"] = torch.tensor([0, R], dtype=torch.int32, device=dev) if shared else None
        s["shared"] = torch.tensor([shared], dtype=torch.int32, device=dev) if shared else None
        s["out"] = torch.zeros((T, Hq, D), dtype=dtype, device=dev)
        s["lse"] = torch.zeros((T, Hq), dtype=torch.float32, device=dev)
        return s
    s["v_cache"], s["out"], s["lse"] = s["k_cache"], torch.zeros_like(s["q"]), torch.zeros((T, Hq), dtype=torch.float32, device=dev)
    s["lse"] = _plain_attend(s)[1]
    del s["v_cache"], s["out"]
    s["score"] = torch.rand((R, width * page), device=dev, generator=gen)
    s["new_score"] = torch.zeros_like(s["score"])
    s["first"] = torch.full((R,), shared, dtype=torch.int32, device=dev)
    s["decay"] = 0.9
    return s


def _prepare_evict(case, gen):
    R, longest, page, dev = case["R"], case["longest"], case["page"], gen.device
    width = -(-longest // page)
    pages = R * width
    length = _whole(gen, max(1, min(longest, case["budget"] + 1)), longest, R)
    length = torch.where(torch.rand((R,), device=dev, generator=gen) < 0.1, torch.clamp(length, max=case["budget"]), length)
    # accumulated weights spread over orders of magnitude, some tokens never looked at
    score = torch.exp(2.0 * _normal(gen, R, width * page))
    score = torch.where(torch.rand((R, width * page), device=dev, generator=gen) < 0.05, torch.zeros_like(score), score)
    # positions as earlier evictions leave them: growing with gaps, the latest ones anywhere
    position = torch.cumsum(1 + (torch.rand((R, width * page), device=dev, generator=gen) < 0.2).int(), 1)
    swap = torch.argsort(torch.arange(width * page, device=dev)[None, :] + 40.0 * torch.rand((R, width * page), device=dev, generator=gen), 1)
    position = position.gather(1, swap).to(torch.int32).contiguous()
    inside = torch.arange(width * page, device=dev)[None, :] < length[:, None]
    return dict(length=length, budget=torch.full((R,), case["budget"], dtype=torch.int32, device=dev), score=score, position=position,
                seen=(torch.where(inside, position, torch.zeros_like(position)).max(1).values + 1).to(torch.int32),
                recent=case["recent"], first=torch.full((R,), case["first"], dtype=torch.int32, device=dev), page=page,
                table=torch.randperm(pages, device=dev, generator=gen).to(torch.int32).view(R, width),
                k_cache=_cache(gen, pages, case), v_cache=_cache(gen, pages, case), new_length=torch.zeros_like(length),
                new_score=torch.zeros_like(score), new_position=torch.zeros_like(position),
                source=torch.full_like(position, -1), status=torch.full((1,), -1, dtype=torch.int32, device=dev))


def prepare(case, seed):
    make = {"rotary": _prepare_rotary, "attend": _prepare_attend, "weights": _prepare_attend, "evict": _prepare_evict}
    s = make[case["op"]](case, _gen(seed))
    s["op"], s["part"] = case["op"], case.get("part")
    return s


# ---- the plain forms ----------------------------------------------------------------------------
def _turn(x, s, back=False):
    """x [T, H, D] with its pairs turned by their angles, in 32 bits."""
    T, H, D = x.shape
    P = s["freq"].numel()
    angle = s["position"].double()[s["axis"].long()].t() * s["freq"].double()[None, :]
    cos, sin = torch.cos(angle).float()[:, None, :], torch.sin(angle).float()[:, None, :]
    if back:
        sin = -sin
    x = x.float()
    if s["neighbours"]:
        pair = x[..., :2 * P].reshape(T, H, P, 2)
        a, b = pair[..., 0], pair[..., 1]
        turned = torch.stack([a * cos - b * sin, a * sin + b * cos], -1).reshape(T, H, 2 * P)
    else:
        a, b = x[..., :P], x[..., P:2 * P]
        turned = torch.cat([a * cos - b * sin, a * sin + b * cos], -1)
    return torch.cat([turned, x[..., 2 * P:]], -1)


def _plain_rotary(s):
    back = s["part"] == "backward"
    q, k = _turn(s["q"], s, back).to(s["q"].dtype), _turn(s["k"], s, back).to(s["k"].dtype)
    if s["part"] != "append":
        return q, k
    T = q.shape[0]
    pages, page, H, D = s["k_cache"].shape
    valid = torch.arange(T, device=q.device) < s["count"]
    to = torch.where(valid, s["slot"], torch.full_like(s["slot"], pages * page))
    caches = [torch.cat([c.reshape(pages * page, H, D), x[:1]]).index_copy(0, to, x)[:-1].view(pages, page, H, D)
              for c, x in ((s["k_cache"], k), (s["v_cache"], s["v"]))]
    return torch.where(valid[:, None, None], q, s["q_out"]), caches[0], caches[1]


def _rows(s):
    """The new tokens of every request, padded to the most: where they are among the queries, which are there, how many keys each
    sees."""
    R, most = s["table"].shape[0], s["most"]
    i = torch.arange(most, device=s["q"].device)[None, :]
    n = (s["offset"][1:] - s["offset"][:-1])[:, None]
    there = i < n
    token = torch.where(there, s["offset"][:-1, None] + i, torch.full_like(n, s["q"].shape[0])).long()
    limit = s["length"][:, None] - n + i + 1 if s["causal"] else s["length"][:, None].expand(R, most)
    return token, there, limit


def _gathered(cache, s):
    """The keys or values of every request, padded to the longest, in 32 bits: [R, heads, longest, width]."""
    pages, page, H, D = cache.shape
    p = torch.arange(s["longest"], device=cache.device)
    ids = s["table"][:, p // page].long()
    return cache[ids, (p % page)[None, :]].float().permute(0, 2, 1, 3)


def _scores(s, token, there, limit):
    """scale q.k for every new token, head and key, -inf where a key is not seen: [R, kv heads, most, heads a kv head, longest]."""
    R, most = token.shape
    T, Hq, D = s["q"].shape
    Hkv = s["k_cache"].shape[2]
    q = s["q"].float()[token.clamp(max=T - 1)].view(R, most, Hkv, Hq // Hkv, D).permute(0, 2, 1, 3, 4).reshape(R, Hkv, -1, D)
    x = torch.matmul(q * s["scale"], _gathered(s["k_cache"], s).transpose(2, 3)).view(R, Hkv, most, Hq // Hkv, -1)
    p = torch.arange(s["longest"], device=q.device)
    seen = (p[None, None, :] < limit[:, :, None]) & there[:, :, None]
    return x.masked_fill_(~seen[:, None, :, None, :], -math.inf)


def _plain_attend(s):
    token, there, limit = _rows(s)
    x = _scores(s, token, there, limit)
    R, Hkv, most, G, L = x.shape
    m = x.amax(-1, keepdim=True)
    m = torch.where(m > -math.inf, m, torch.zeros_like(m))
    e = torch.exp_(x.sub_(m))
    z = e.sum(-1, keepdim=True)
    o = torch.matmul(e.view(R, Hkv, most * G, L), _gathered(s["v_cache"], s)).view(R, Hkv, most, G, -1)
    o = o / torch.where(z > 0, z, torch.ones_like(z))
    lse = (m + torch.log(z))[..., 0]
    T, Hq, D = s["q"].shape
    o = o.permute(0, 2, 1, 3, 4).reshape(R * most, Hq, D).to(s["q"].dtype)
    lse = lse.permute(0, 2, 1, 3).reshape(R * most, Hq)
    to = token.reshape(-1)
    out = torch.cat([s["out"], s["out"][:1]]).index_copy(0, to, o)[:T]
    lse = torch.cat([s["lse"], s["lse"][:1]]).index_copy(0, to, lse)[:T]
    return out, lse, torch.zeros_like(s["status"])


def _plain_weights(s):
    token, there, limit = _rows(s)
    T, Hq, D = s["q"].shape
    x = _scores(s, token, there, limit)
    R, Hkv, most, G, L = x.shape
    lse = s["lse"][token.clamp(max=T - 1)].view(R, most, Hkv, G).permute(0, 2, 1, 3)[..., None]
    got = torch.where(x > -math.inf, torch.exp(x - lse), torch.zeros_like(x)).sum((1, 2, 3))
    p = torch.arange(L, device=x.device)[None, :]
    n = (s["offset"][1:] - s["offset"][:-1])[:, None]
    length = s["length"][:, None]
    before = torch.where(p < length - n, s["decay"] * s["score"][:, :L], torch.zeros_like(got))
    inside = (p >= s["first"][:, None]) & (p < length)
    new = s["new_score"].clone()
    new[:, :L] = torch.where(inside, before + got, new[:, :L])
    return new, torch.zeros_like(s["status"])


def _plain_evict(s):
    R, N = s["score"].shape
    pages, page, H, D = s["k_cache"].shape
    p = torch.arange(N, device=s["score"].device)[None, :].expand(R, N)
    length, first = s["length"][:, None], s["first"][:, None]
    keep = torch.minimum(length, torch.maximum(s["budget"][:, None], first))
    key = torch.where(torch.isnan(s["score"]), torch.full_like(s["score"], -math.inf), s["score"])
    key = torch.where((s["position"] >= s["seen"][:, None] - s["recent"]) | (p < first), torch.full_like(key, math.inf), key)
    # places that may not leave first, then by weight, then by place; a stable sort by one after the other
    order = torch.sort(key, dim=1, descending=True, stable=True).indices
    group = torch.where(p < first, torch.zeros_like(p), torch.where(p < length, torch.ones_like(p), torch.full_like(p, 2)))
    order = order.gather(1, torch.sort(group.gather(1, order), dim=1, stable=True).indices)
    rank = torch.empty_like(order).scatter_(1, order, p)
    stays = (rank < keep) & (p < length)
    hole, tail = ~stays & (p < keep), stays & (p >= keep)
    # the j-th hole takes the j-th of the tail
    behind = torch.sort(torch.where(tail, p, torch.full_like(p, N)), dim=1).values
    j = (torch.cumsum(hole, 1) - 1).clamp(min=0)
    source = torch.where(hole, behind.gather(1, j).clamp(max=N - 1), p)
    inside = p < keep
    new_score = torch.where(inside, s["score"].gather(1, source), s["new_score"])
    new_position = torch.where(inside, s["position"].gather(1, source), s["new_position"])
    from_ = s["table"].gather(1, source // page).long() * page + source % page
    to = s["table"].gather(1, p // page).long() * page + p % page
    to = torch.where(hole, to, torch.full_like(to, pages * page)).reshape(-1)
    caches = [torch.cat([c.reshape(pages * page, H, D), c[:1, 0]]).index_copy(0, to, c.reshape(pages * page, H, D)[from_.reshape(-1)])[:-1]
              .view(pages, page, H, D) for c in (s["k_cache"], s["v_cache"])]
    return dict(k_cache=caches[0], v_cache=caches[1], new_length=keep[:, 0].to(torch.int32), new_score=new_score,
                new_position=new_position, source=torch.where(inside, source.to(torch.int32), s["source"]),
                status=torch.zeros_like(s["status"]))


# ---- one pass -----------------------------------------------------------------------------------
def _own_pass(s):
    import paper_2512_08537_b200 as ardiff
    if s["op"] == "rotary":
        if s["part"] == "append":
            ardiff.ardiff_rotary_append(s["q"], s["k"], s["v"], s["position"], s["freq"], s["slot"], s["k_cache"], s["v_cache"],
                                        axis=s["axis"], count=s["count"], neighbours=s["neighbours"], q_out=s["q_out"])
            return s["q_out"], s["k_cache"], s["v_cache"]
        turn = ardiff.ardiff_rotary if s["part"] == "forward" else ardiff.ardiff_rotary_backward
        return turn(s["q"], s["k"], s["position"], s["freq"], axis=s["axis"], neighbours=s["neighbours"])
    if s["op"] == "attend":
        return ardiff.ardiff_attend_pages(s["q"], s["k_cache"], s["v_cache"], s["table"], s["length"], s["offset"], group=s["group"],
                                          shared=s["shared"], most=s["most"], scale=s["scale"], causal=s["causal"], out=s["out"],
                                          lse=s["lse"], status=s["status"])
    if s["op"] == "weights":
        return ardiff.ardiff_attend_weights(s["q"], s["k_cache"], s["table"], s["length"], s["offset"], s["lse"], s["score"],
                                            first=s["first"], decay=s["decay"], scale=s["scale"], causal=s["causal"],
                                            new_score=s["new_score"], status=s["status"])
    ardiff.ardiff_pages_evict(s["length"], s["budget"], s["score"], s["table"], s["k_cache"], s["v_cache"], first=s["first"],
                              position=s["position"], seen=s["seen"], recent=s["recent"], new_length=s["new_length"],
                              new_score=s["new_score"], new_position=s["new_position"], source=s["source"], status=s["status"])
    return {k: s[k] for k in ("k_cache", "v_cache", "new_length", "new_score", "new_position", "source", "status")}


def run(s):
    if own:
        return _own_pass(s)
    plain = {"rotary": _plain_rotary, "attend": _plain_attend, "weights": _plain_weights, "evict": _plain_evict}
    return plain[s["op"]](s)


def work(case):
    size = 4 if case["dtype"] == "f32" else 2
    Hkv, D = case["Hkv"], case["D"]
    if case["op"] == "rotary":
        # queries, keys and, where they go into a cache, values once in and once out; positions in; six operations a pair
        T, heads = case["T"] - case["pad"], case["Hq"] + Hkv * (2 if case["part"] == "append" else 1)
        return dict(bytes=max(1, T) * (2 * heads * D * size + 4 * case["axes"]), flops=max(1, T) * (case["Hq"] + Hkv) * D * 3)
    if case["op"] == "evict":
        # weights and positions of all tokens in, those that stay out; the tokens behind the new end that stay move
        R, L, B = case["R"], (case["longest"] + min(case["longest"], case["budget"] + 1)) / 2, case["budget"]
        moved = max(0.0, L - B) * min(1.0, B / L)
        return dict(bytes=R * (8 * L + 12 * min(B, L) + moved * 4 * Hkv * D * size), flops=R * L * 4)
    R, most, shared, longest = case["R"], case["most"], case["shared"], case["longest"]
    n = 1 if most == 1 else sum(_new_tokens(case)) / R if most > 8 else most / 2
    length = shared + n + (longest - shared - n) / 2
    seen = length - (n - 1) / 2 if case["causal"] else length
    rows = R * n * case["Hq"]
    if case["op"] == "attend":
        # queries in, results out, the shared tokens once, everyone's own once
        return dict(bytes=2 * rows * D * size + 4 * rows + (shared + R * (length - shared)) * 2 * Hkv * D * size, flops=4 * D * rows * seen)
    return dict(bytes=rows * (D * size + 4) + R * (length - shared) * (Hkv * D * size + 8), flops=2 * D * rows * max(1, seen - shared))


# ---- the same from the definitions, in 64 bits --------------------------------------------------
def _exact_turn(x, s, sign):
    """Every pair as a complex number, times a number on the unit circle."""
    P = s["freq"].numel()
    x = x.double()
    angle = sign * torch.stack([s["position"][int(a)].double() * float(f) for a, f in zip(s["axis"], s["freq"])], 1)
    unit = torch.polar(torch.ones_like(angle), angle)[:, None, :]
    out = x.clone()
    if s["neighbours"]:
        z = torch.complex(x[..., 0:2 * P:2], x[..., 1:2 * P:2]) * unit
        out[..., 0:2 * P:2], out[..., 1:2 * P:2] = z.real, z.imag
    else:
        z = torch.complex(x[..., :P], x[..., P:2 * P]) * unit
        out[..., :P], out[..., P:2 * P] = z.real, z.imag
    return out


def _exact_rotary(s):
    sign = -1.0 if s["part"] == "backward" else 1.0
    q, k = _exact_turn(s["q"], s, sign), _exact_turn(s["k"], s, sign)
    if s["part"] != "append":
        return q, k
    n, page = int(s["count"]), s["k_cache"].shape[1]
    slot = s["slot"][:n]
    k_cache, v_cache = s["k_cache"].double().contiguous(), s["v_cache"].double().contiguous()
    k_cache[slot // page, slot % page] = k[:n]
    v_cache[slot // page, slot % page] = s["v"][:n].double()
    return torch.cat([q[:n], s["q_out"][n:].double()]), k_cache, v_cache


def _exact_request(s, r, h):
    """Of request r: its queries of kv head h [n, G, D], its keys [L, D], which keys each query sees [n, L]; in 64 bits."""
    t0, t1, L, page = int(s["offset"][r]), int(s["offset"][r + 1]), int(s["length"][r]), s["k_cache"].shape[1]
    Hkv = s["k_cache"].shape[2]
    G = s["q"].shape[1] // Hkv
    p = torch.arange(L, device=s["q"].device)
    slots = s["table"][r].long()[p // page], p % page
    q = s["q"][t0:t1, h * G:(h + 1) * G].double()
    i = torch.arange(t1 - t0, device=p.device)[:, None]
    sees = p[None, :] <= (L - (t1 - t0) + i) if s["causal"] else torch.ones((t1 - t0, L), dtype=torch.bool, device=p.device)
    return t0, t1, G, q, slots, sees


def _exact_attend(s):
    out, lse = s["out"].double(), s["lse"].double()
    for r in range(s["table"].shape[0]):
        for h in range(s["k_cache"].shape[2]):
            t0, t1, G, q, slots, sees = _exact_request(s, r, h)
            x = torch.einsum("ngd,ld->gnl", q, s["k_cache"][slots[0], slots[1], h].double()) * s["scale"]
            x = x.masked_fill(~sees[None], -math.inf)
            norm = torch.logsumexp(x, 2)
            o = torch.einsum("gnl,ld->ngd", torch.exp(x - norm[..., None]), s["v_cache"][slots[0], slots[1], h].double())
            out[t0:t1, h * G:(h + 1) * G] = o
            lse[t0:t1, h * G:(h + 1) * G] = norm.t()
    return out, lse, None


def _exact_weights(s):
    new = s["new_score"].double()
    for r in range(s["table"].shape[0]):
        L, first = int(s["length"][r]), int(s["first"][r])
        n = int(s["offset"][r + 1]) - int(s["offset"][r])
        if first >= L:
            continue
        total = torch.zeros((L,), dtype=torch.float64, device=new.device)
        total[:L - n] = s["score"][r, :L - n].double() * s["decay"]
        for h in range(s["k_cache"].shape[2]):
            t0, t1, G, q, slots, sees = _exact_request(s, r, h)
            x = torch.einsum("ngd,ld->ngl", q, s["k_cache"][slots[0], slots[1], h].double()) * s["scale"]
            w = torch.exp(x - s["lse"][t0:t1, h * G:(h + 1) * G].double()[..., None])
            total += (w * sees[:, None, :]).sum((0, 1))
        new[r, first:L] = total[first:]
    return new, None


def _exact_evict(s):
    """Weights that stay; what is whole or copied is equal or wrong."""
    new = s["new_score"].double().cpu()
    score, position = s["score"].cpu(), s["position"].cpu()
    for r, (L, B, F, seen) in enumerate(zip(*(s[k].tolist() for k in ("length", "budget", "first", "seen")))):
        keep = min(L, max(B, F))
        free = torch.arange(min(F, L), L)
        safe = position[r, free] >= seen - s["recent"]
        weight = torch.nan_to_num(score[r, free].double(), nan=-math.inf, posinf=math.inf, neginf=-math.inf)
        weight[safe] = math.inf
        best = free[torch.argsort(-weight, stable=True)[:keep - min(F, L)]].sort().values
        stay = set(best.tolist()) | set(range(min(F, L)))
        holes = [p for p in range(keep) if p not in stay]
        tail = [p for p in sorted(stay) if p >= keep]
        new[r, :keep] = score[r, :keep].double()
        new[r, holes] = score[r, tail].double()
    return dict(k_cache=None, v_cache=None, new_length=None, new_score=new, new_position=None, source=None, status=None)


def exact(case, seed):
    s = prepare(case, seed)
    of = {"rotary": _exact_rotary, "attend": _exact_attend, "weights": _exact_weights, "evict": _exact_evict}
    return of[case["op"]](s)
