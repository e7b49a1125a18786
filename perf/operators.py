"""What is timed of the framework's language-model operators, beside cases.py: one pass through one operator a case.

  sample     the next token of every row of logits (temperature, top-k, top-p, min-p, one given uniform number a row),
             and the logarithm of the probability that it was drawn with
  distill    the divergence of a student's rows of logits from a teacher's top logits: "forward" alone, "backward" alone
             (from the forward's row statistics), or "step": both in one call, the rows' weights being known
  extend     new tokens of every request placed in a paged cache: pages taken from the free list, the block tables
             lengthened, the slot, position and request of every new token written
  truncate   rejected tokens taken back: pages that no token needs any more go back to the free list

`run()` makes the framework's calls where `own` is true; where it is false it computes the same in elementary torch
operations, in 32 bits (token sampling in 64: a token is a choice between borders that lie closer than 32 bits tell apart).
"""
import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
# the most that one drawn pass may cost: the largest listed pass of each kind
MAX_SAMPLE = 512 * 131072
MAX_DISTILL = 4096 * 131072
MAX_TOKENS = 1 << 20


def listed():
    return [
        # one stream of text, one token: latency is all there is
        dict(name="sample_1x32768", op="sample", n=1, V=32768, pad=0, dtype="bf16", filters="top_k_p", flat=False),
        # a server's batch, every request with settings of its own (greedy ones among them), some under a grammar's mask
        dict(name="sample_64x65536_mixed", op="sample", n=64, V=65536, pad=0, dtype="bf16", filters="mixed", flat=False),
        # no filter at all, rows flat enough that the tail counts; a vocabulary of odd size inside a wider buffer
        dict(name="sample_33x100003_all", op="sample", n=33, V=100003, pad=61, dtype="f16", filters="none", flat=True),
        # logits kept in 32 bits, the nucleus alone
        dict(name="sample_256x131072_top_p", op="sample", n=256, V=131072, pad=0, dtype="f32", filters="top_p", flat=False),
        # drafts of 8 tokens for 64 requests, verified together: the largest batch
        dict(name="sample_512x131072", op="sample", n=512, V=131072, pad=0, dtype="bf16", filters="top_k_p", flat=False),
        # a draft model's smallest step: few rows of a small vocabulary
        dict(name="distill_step_16x8191", op="distill", part="step", n=16, V=8191, k=20, dtype="f32", T=1.0, empty=0.0),
        # validation: the loss alone
        dict(name="distill_forward_2048x32768", op="distill", part="forward", n=2048, V=32768, k=64, dtype="bf16", T=2.0,
             empty=0.1),
        # the backward of an automatic differentiation's graph; a width that is no multiple of 8
        dict(name="distill_backward_1000x50001", op="distill", part="backward", n=1000, V=50001, k=100, dtype="f16", T=1.0,
             empty=0.0),
        # a training step of a large vocabulary
        dict(name="distill_step_4096x131072", op="distill", part="step", n=4096, V=131072, k=128, dtype="bf16", T=1.0,
             empty=0.05),
        # decoding: one token for each of 256 requests, most of which need no new page
        dict(name="extend_256_decode", op="extend", R=256, page=16, longest=8192, most=1, fresh=0.0),
        # prompts of up to 16384 tokens for 96 new requests, a million tokens at the most
        dict(name="extend_96_prompts", op="extend", R=96, page=64, longest=0, most=16384, fresh=1.0),
        # drafts of up to 8 tokens for 2048 requests, the rejected ones taken back
        dict(name="truncate_2048_drafts", op="truncate", R=2048, page=16, longest=4096, most=8, fresh=0.0),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["sample", "sample", "sample", "distill", "distill", "extend", "truncate"])
    if op == "sample":
        V = _log(rng, 100, 200000)
        n = min(_log(rng, 1, 512), MAX_SAMPLE // V)
        return dict(op=op, n=n, V=V, pad=rng.choice([0, 0, 5, 64]), dtype=rng.choice(sorted(DTYPES)),
                    filters=rng.choice(["none", "top_k_p", "top_p", "min_p", "mixed"]), flat=rng.random() < 0.3)
    if op == "distill":
        V = _log(rng, 100, 200000)
        n = min(_log(rng, 1, 4096), MAX_DISTILL // V)
        return dict(op=op, part=rng.choice(["forward", "backward", "step"]), n=n, V=V, k=min(V, _log(rng, 1, 256)),
                    dtype=rng.choice(sorted(DTYPES)), T=rng.choice([0.5, 1.0, 2.0, 4.0]), empty=rng.choice([0.0, 0.0, 0.2]))
    R = _log(rng, 1, 4096)
    c = dict(op=op, R=R, page=rng.choice([1, 16, 32, 64, 100, 256]), longest=_log(rng, 1, 16384), most=_log(rng, 1, 16384),
             fresh=rng.choice([0.0, 0.1, 1.0]))
    if op == "truncate":
        c["most"] = min(c["most"], 64)
    c["most"] = max(1, min(c["most"], MAX_TOKENS // R))
    c["longest"] = min(c["longest"], (1 << 24) // R)
    return c


# ---- inputs -------------------------------------------------------------------------------------
def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(int(seed))


def _logits(n, V, flat, gen):
    """Rows that fall off as language models' do: a power of the rank, the exponent the row's own, and noise; flat rows
    by a smaller power."""
    dev = gen.device
    x = torch.rand((n, V), device=dev, generator=gen)
    a = torch.rand((n, 1), device=dev, generator=gen)
    a = 0.3 + 0.5 * a if flat else 0.9 + 1.1 * a
    x.mul_(V).add_(1.0).log_().mul_(-a)
    step = max(1, (1 << 27) // V)
    for r0 in range(0, n, step):
        m = min(step, n - r0)
        x[r0:r0 + m] += 0.3 * torch.randn((m, V), device=dev, generator=gen)
    return x.add_(12.0)


def _prepare_sample(case, gen):
    n, V, dev = case["n"], case["V"], gen.device
    x = _logits(n, V, case["flat"], gen)
    f = case["filters"]

    def uniform(lo, hi):
        return lo + (hi - lo) * torch.rand((n,), device=dev, generator=gen)

    def some(share):
        return torch.rand((n,), device=dev, generator=gen) < share

    s = dict(u=torch.rand((n,), device=dev, generator=gen), temperature=None, top_k=None, top_p=None, min_p=None)
    if f != "none":
        s["temperature"] = uniform(0.6, 1.2)
    if f in ("top_k_p", "mixed"):
        s["top_k"] = torch.randint(20, 100, (n,), device=dev, generator=gen, dtype=torch.int32)
    if f in ("top_k_p", "top_p", "mixed"):
        s["top_p"] = uniform(0.8, 0.98)
    if f in ("min_p", "mixed"):
        s["min_p"] = uniform(0.01, 0.1)
    if f == "mixed":                                           # each filter off in some rows, a sixth of them greedy
        s["temperature"] = torch.where(some(1 / 6), torch.zeros_like(s["temperature"]), s["temperature"])
        s["top_k"] = torch.where(some(0.5), torch.zeros_like(s["top_k"]), s["top_k"])
        s["top_p"] = torch.where(some(0.5), torch.ones_like(s["top_p"]), s["top_p"])
        s["min_p"] = torch.where(some(0.5), torch.zeros_like(s["min_p"]), s["min_p"])
        masked = some(1 / 8)[:, None] & (torch.rand((n, V), device=dev, generator=gen) < 0.9)
        masked[:, V // 2] = False
        x.masked_fill_(masked, -math.inf)
    buf = torch.zeros((n, V + case["pad"]), dtype=DTYPES[case["dtype"]], device=dev)
    buf[:, :V] = x
    s["logits"] = buf[:, :V]
    s["token"] = torch.empty((n,), dtype=torch.int32, device=dev)
    s["logprob"] = torch.empty((n,), dtype=torch.float32, device=dev)
    return s


def _prepare_distill(case, gen):
    n, V, k, dev = case["n"], case["V"], case["k"], gen.device
    x = torch.empty((n, V), dtype=DTYPES[case["dtype"]], device=dev)
    ids = torch.empty((n, k), dtype=torch.int32, device=dev)
    teacher = torch.empty((n, k), dtype=torch.float32, device=dev)
    step = max(1, (1 << 26) // V)
    for r0 in range(0, n, step):
        m = min(step, n - r0)
        xs = _logits(m, V, False, gen)
        x[r0:r0 + m] = xs
        # a teacher that mostly agrees: the student's own top entries, its values another draw around them
        top, at = xs.topk(k, dim=1)
        ids[r0:r0 + m] = at
        teacher[r0:r0 + m] = top + 0.7 * torch.randn((m, k), device=dev, generator=gen)
    # rows whose teacher kept fewer entries, and rows of padding tokens, which have none
    most = torch.randint((k + 1) // 2, k + 1, (n, 1), device=dev, generator=gen)
    most = torch.where(torch.rand((n, 1), device=dev, generator=gen) < case["empty"], torch.zeros_like(most), most)
    ids.masked_fill_(torch.arange(k, device=dev)[None, :] >= most, -1)
    # a mean over the rows, each with a weight; gradients in f16 come with a loss scale, as they do in training
    weight = (0.5 + torch.rand((n,), device=dev, generator=gen)) * ((2.0 ** 14 if case["dtype"] == "f16" else 1.0) / n)
    s = dict(logits=x, teacher=teacher, ids=ids, weight=weight, T=case["T"])
    if case["part"] == "backward":
        s["stats"] = _distill_rows(s)[1]
    return s


def _prepare_pages(case, gen):
    R, page, most, dev = case["R"], case["page"], case["most"], gen.device
    longest = case["longest"]
    length = torch.randint(0, longest + 1, (R,), device=dev, generator=gen, dtype=torch.int32)
    fresh = torch.rand((R,), device=dev, generator=gen) < case["fresh"]
    length = torch.where(fresh, torch.zeros_like(length), length)
    add = torch.randint(1 if most == 1 else 0, most + 1, (R,), device=dev, generator=gen, dtype=torch.int32)
    width = -(-(longest + most) // page)
    pages = R * width + 7
    order = torch.randperm(pages, device=dev, generator=gen).to(torch.int32)
    if case["op"] == "truncate":
        length = length + add                                  # the drafts are in the cache; some of each stay
    held = (length + page - 1) // page
    at = torch.arange(width, device=dev)[None, :]
    first = torch.cumsum(held, 0) - held
    table = torch.where(at < held[:, None], order[(first[:, None] + at).clamp_(max=pages - 1).long()],
                        torch.full((1, 1), -1, dtype=torch.int32, device=dev)).contiguous()
    taken = held.sum()
    free = torch.full((pages,), -1, dtype=torch.int32, device=dev)
    rest = torch.arange(pages, device=dev)
    free = torch.where(rest < pages - taken, order[(taken + rest).clamp_(max=pages - 1)], free)
    s = dict(length=length, table=table, free=free, free_count=(pages - taken).to(torch.int32).reshape(1), page=page,
             new_free_count=torch.zeros((1,), dtype=torch.int32, device=dev),
             status=torch.full((1,), -1, dtype=torch.int32, device=dev))
    if case["op"] == "truncate":
        drop = (torch.rand((R,), device=dev, generator=gen) * (add + 1)).to(torch.int32)
        s["target"] = length - torch.minimum(drop, add)
        return s
    tokens = R * most
    s["add"] = add
    s["slot"] = torch.full((tokens,), -1, dtype=torch.int64, device=dev)
    s["position"] = torch.full((tokens,), -1, dtype=torch.int32, device=dev)
    s["request"] = torch.full((tokens,), -1, dtype=torch.int32, device=dev)
    s["offset"] = torch.zeros((R + 1,), dtype=torch.int32, device=dev)
    s["new_length"] = torch.zeros((R,), dtype=torch.int32, device=dev)
    return s


def prepare(case, seed):
    gen = _gen(seed)
    make = {"sample": _prepare_sample, "distill": _prepare_distill, "extend": _prepare_pages, "truncate": _prepare_pages}
    s = make[case["op"]](case, gen)
    s["op"], s["part"] = case["op"], case.get("part")
    return s


# ---- the plain forms ----------------------------------------------------------------------------
def _plain_sample(s):
    x = s["logits"].double()
    n, V = x.shape
    dev = x.device

    def setting(name, off):
        return s[name].double()[:, None] if s[name] is not None else torch.full((n, 1), off, dtype=torch.float64, device=dev)

    T, p, mp = setting("temperature", 1.0), setting("top_p", 1.0), setting("min_p", 0.0)
    k = setting("top_k", 0.0)
    greedy = T == 0
    values, order = torch.sort(x, dim=1, descending=True, stable=True)
    w = torch.exp((values - values[:, :1]) / torch.where(greedy, torch.ones_like(T), T))
    rank = torch.arange(V, device=dev)[None, :]
    keep = torch.where((k > 0) & ~greedy, rank < k, torch.ones_like(rank, dtype=torch.bool))
    keep = keep & ~(greedy & (rank > 0))
    w = torch.where(keep, w, torch.zeros_like(w))
    above = torch.cumsum(w, 1)
    total = above[:, -1:]
    above = torch.cat([torch.zeros_like(total), above[:, :-1]], 1)
    keep = keep & ((p >= 1) | (above < p * total) | (rank == 0)) & ((mp <= 0) | (w >= mp.clamp(max=1.0)))
    w = torch.where(keep, w, torch.zeros_like(w))
    in_order = torch.zeros_like(w).scatter_(1, order, w)
    cum = torch.cumsum(in_order, 1)
    total = cum[:, -1:]
    token = (cum <= s["u"].double()[:, None] * total).sum(1, keepdim=True).clamp_(max=V - 1)
    logprob = torch.log(in_order.gather(1, token) / total)
    return token[:, 0].to(torch.int32), logprob[:, 0].float()


def _distill_rows(s, entries=False):
    """Loss and statistics (largest logit, logarithm of the sum of exponentials above it) of every row; and, if asked for,
    what the gradient needs: probabilities, the teacher's, the valid places."""
    x = s["logits"].float()
    V, T = x.shape[1], s["T"]
    ids = s["ids"].long()
    valid = (ids >= 0) & (ids < V) & (s["teacher"] > -math.inf)
    some = valid.any(1, keepdim=True)
    t = torch.where(valid, s["teacher"].float() / T, torch.full_like(s["teacher"], -math.inf))
    t = t - torch.where(some, t.max(1, keepdim=True).values, torch.zeros_like(t[:, :1]))
    q = torch.exp(t)
    total = torch.where(some, q.sum(1, keepdim=True), torch.ones_like(t[:, :1]))
    q = q / total
    m = x.max(1, keepdim=True).values
    e = torch.exp((x - m) / T)
    z = e.sum(1, keepdim=True)
    at = ids.clamp(0, V - 1)
    lp = (x.gather(1, at) - m) / T - torch.log(z)
    loss = torch.where(q > 0, q * (t - torch.log(total) - lp), torch.zeros_like(q)).sum(1)
    stats = torch.where(some, torch.cat([m, torch.log(z)], 1), torch.zeros_like(torch.cat([m, z], 1)))
    return (loss, stats, e, z, q, at, some) if entries else (loss, stats)


def _plain_distill(s):
    if s["part"] == "forward":
        return _distill_rows(s)
    if s["part"] == "backward":
        x, T = s["logits"].float(), s["T"]
        p = torch.exp((x - s["stats"][:, :1]) / T - s["stats"][:, 1:])
        ids = s["ids"].long()
        valid = (ids >= 0) & (ids < x.shape[1]) & (s["teacher"] > -math.inf)
        some = valid.any(1, keepdim=True)
        t = torch.where(valid, s["teacher"].float() / T, torch.full_like(s["teacher"], -math.inf))
        q = torch.exp(t - torch.where(some, t.max(1, keepdim=True).values, torch.zeros_like(t[:, :1])))
        q = q / torch.where(some, q.sum(1, keepdim=True), torch.ones_like(q[:, :1]))
        at = ids.clamp(0, x.shape[1] - 1)
        g = torch.where(some, p, torch.zeros_like(p)).scatter_add_(1, at, -q)
        return (g * (s["weight"][:, None] / T)).to(s["logits"].dtype)
    loss, stats, e, z, q, at, some = _distill_rows(s, entries=True)
    g = torch.where(some, e / z, torch.zeros_like(e)).scatter_add_(1, at, -q)
    return loss, stats, (g * (s["weight"][:, None] / s["T"])).to(s["logits"].dtype)


def _plain_extend(s):
    length, add, table, free, page = s["length"], s["add"], s["table"], s["free"], s["page"]
    R, width = table.shape
    dev = table.device
    held = (length + page - 1) // page
    after = length + add
    new = (after + page - 1) // page - held
    first = torch.cumsum(new, 0) - new
    offset = torch.cat([torch.zeros((1,), dtype=torch.int64, device=dev), torch.cumsum(add, 0)])
    at = torch.arange(width, device=dev)[None, :]
    j = at - held[:, None]
    fill = (j >= 0) & (j < new[:, None])
    pick = (s["free_count"][0] - 1 - first[:, None] - j).clamp(0, free.numel() - 1)
    table = torch.where(fill, free[pick.long()], table)
    t = torch.arange(s["slot"].numel(), device=dev)
    r = torch.searchsorted(offset, t, right=True) - 1
    inside = t < offset[-1]
    r = r.clamp(max=R - 1)
    pos = length[r] + (t - offset[r])
    pos = torch.where(inside, pos, torch.zeros_like(pos))
    slot = table[r, pos // page].long() * page + pos % page
    return dict(slot=torch.where(inside, slot, s["slot"]), position=torch.where(inside, pos.to(torch.int32), s["position"]),
                request=torch.where(inside, r.to(torch.int32), s["request"]), offset=offset.to(torch.int32), table=table,
                new_length=after, new_free_count=s["free_count"] - new.sum().to(torch.int32),
                status=torch.zeros((1,), dtype=torch.int32, device=dev))


def _plain_truncate(s):
    table, free, page = s["table"], s["free"], s["page"]
    width = table.shape[1]
    dev = table.device
    stay = (s["target"] + page - 1) // page
    back = (s["length"] + page - 1) // page - stay
    first = torch.cumsum(back, 0) - back
    total = back.sum()
    j = torch.arange(width, device=dev)[None, :] - stay[:, None]
    give = (j >= 0) & (j < back[:, None])
    # pages lie on the free list in the order that makes it give them out again as it did before
    to = s["free_count"][0] + total - 1 - first[:, None] - j
    to = torch.where(give, to, torch.full_like(to, free.numel()))
    out = torch.cat([free, free[:1]]).scatter_(0, to.reshape(-1).long(), table.reshape(-1))[:-1]
    return dict(free=out, new_free_count=s["free_count"] + total.to(torch.int32),
                status=torch.zeros((1,), dtype=torch.int32, device=dev))


# ---- one pass -----------------------------------------------------------------------------------
def _own_pass(s):
    import paper_2512_08537_b200 as ardiff
    if s["op"] == "sample":
        return ardiff.ardiff_sample_tokens(s["logits"], s["u"], s["temperature"], s["top_k"], s["top_p"], s["min_p"],
                                           token=s["token"], logprob=s["logprob"])
    if s["op"] == "distill":
        if s["part"] == "forward":
            return ardiff.ardiff_distill_topk(s["logits"], s["teacher"], s["ids"], s["T"])
        if s["part"] == "backward":
            return ardiff.ardiff_distill_topk_backward(s["logits"], s["teacher"], s["ids"], s["stats"], s["weight"], s["T"])
        return ardiff.ardiff_distill_topk_step(s["logits"], s["teacher"], s["ids"], s["weight"], s["T"])
    if s["op"] == "extend":
        ardiff.ardiff_pages_extend(s["length"], s["add"], s["table"], s["free"], s["free_count"], s["page"], s["slot"],
                                   s["position"], s["request"], s["offset"], s["new_length"], s["new_free_count"],
                                   s["status"])
        return {k: s[k] for k in ("slot", "position", "request", "offset", "table", "new_length", "new_free_count", "status")}
    ardiff.ardiff_pages_truncate(s["length"], s["target"], s["table"], s["free"], s["free_count"], s["page"],
                                 s["new_free_count"], s["status"])
    return {k: s[k] for k in ("free", "new_free_count", "status")}


def run(s):
    if own:
        return _own_pass(s)
    plain = {"sample": _plain_sample, "distill": _plain_distill, "extend": _plain_extend, "truncate": _plain_truncate}
    return plain[s["op"]](s)


def work(case):
    if case["op"] == "sample":
        n, V = case["n"], case["V"]
        size = 4 if case["dtype"] == "f32" else 2
        # the row once, the settings and the answers; a comparison a logit, and an exponential and a sum where the tail counts
        return dict(bytes=n * (V * size + 28), flops=n * V * (1 if case["filters"] == "top_k_p" else 4))
    if case["op"] == "distill":
        n, V, k = case["n"], case["V"], case["k"]
        size = 4 if case["dtype"] == "f32" else 2
        rows = 1 if case["part"] == "forward" else 2
        return dict(bytes=n * (1.0 - case["empty"]) * rows * V * size + n * case["empty"] * (rows - 1) * V * size
                    + n * (8 * k + 16), flops=n * V * (4 if rows == 1 else 7))
    R, most, page = case["R"], case["most"], case["page"]
    if case["op"] == "extend":
        tokens = R * (most + (1 if most == 1 else 0)) / 2
        # lengths and tables in, a slot, position and request a token and the new pages out
        return dict(bytes=R * 20 + tokens * 16 + 8 * tokens / page + 12, flops=8 * tokens)
    return dict(bytes=R * 8 + 8 * R * (1 + most / 4 / page), flops=8 * R)


# ---- the same from the definitions, in 64 bits --------------------------------------------------
def _exact_sample(s):
    tokens, logs = [], []
    for i in range(s["logits"].shape[0]):
        x = s["logits"][i].double()
        T = 1.0 if s["temperature"] is None else float(s["temperature"][i])
        if T == 0.0:
            tokens.append(int((x == x.max()).nonzero()[0, 0]))
            logs.append(0.0)
            continue
        k = 0 if s["top_k"] is None else int(s["top_k"][i])
        p = 1.0 if s["top_p"] is None else float(s["top_p"][i])
        mp = 0.0 if s["min_p"] is None else float(s["min_p"][i])
        prob = torch.softmax(x / T, 0)
        ids = torch.argsort(-x, stable=True)
        if 0 < k < ids.numel():
            ids = ids[:k]
        mass = prob[ids]
        mass = mass / mass.sum()
        if p < 1.0:
            count = int((torch.cumsum(mass, 0) < p).sum()) + 1
            ids = ids[:count]
        ids = ids[prob[ids] >= mp * prob.max()].sort().values
        mass = prob[ids] / prob[ids].sum()
        j = min(int((torch.cumsum(mass, 0) <= float(s["u"][i])).sum()), ids.numel() - 1)
        tokens.append(int(ids[j]))
        logs.append(float(torch.log(mass[j])))
    return None, torch.tensor(logs, dtype=torch.float64)


def _exact_distill(s):
    losses, stats, grads = [], [], []
    n, V = s["logits"].shape
    step = max(1, (1 << 27) // V)
    for r0 in range(0, n, step):
        x = s["logits"][r0:r0 + step].double()
        scaled = x / s["T"]
        ids = s["ids"][r0:r0 + step].long()
        teacher = s["teacher"][r0:r0 + step].double() / s["T"]
        has = (ids >= 0) & (ids < V)
        any_ = has.any(1)
        q = torch.nan_to_num(torch.softmax(teacher.masked_fill(~has, -math.inf), 1), nan=0.0)
        lse = torch.logsumexp(scaled, 1, keepdim=True)
        lp = scaled.gather(1, ids.clamp(min=0)) - lse
        losses.append((torch.special.xlogy(q, q) - q * lp).masked_fill(~has, 0.0).sum(1))
        top = x.max(1).values
        both = torch.stack([top, lse[:, 0] - top / s["T"]], 1)
        stats.append(both.masked_fill(~any_[:, None], 0.0))
        if s["part"] != "forward":
            g = torch.exp(scaled - lse).masked_fill(~any_[:, None], 0.0)
            g.scatter_add_(1, ids.clamp(min=0), -q)
            grads.append((g * (s["weight"][r0:r0 + step].double()[:, None] / s["T"])).to(torch.float32))
    if s["part"] == "backward":
        return torch.cat(grads)
    out = (torch.cat(losses), torch.cat(stats))
    return out if s["part"] == "forward" else (*out, torch.cat(grads))


def _exact_extend(s):
    length, add, page = s["length"].tolist(), s["add"].tolist(), s["page"]
    free, table = s["free"][:int(s["free_count"])].tolist(), s["table"].tolist()
    slot, position, request, offset = [], [], [], [0]
    for r, (have, more) in enumerate(zip(length, add)):
        for page_no in range(-(-have // page), -(-(have + more) // page)):
            table[r][page_no] = free.pop()
        for pos in range(have, have + more):
            slot.append(table[r][pos // page] * page + pos % page)
            position.append(pos)
            request.append(r)
        offset.append(len(slot))
    rest = s["slot"].numel() - len(slot)
    as_ = lambda v, t: torch.tensor(v, dtype=t)  # noqa: E731
    return dict(slot=as_(slot + [-1] * rest, torch.int64), position=as_(position + [-1] * rest, torch.int32),
                request=as_(request + [-1] * rest, torch.int32), offset=as_(offset, torch.int32),
                table=as_(table, torch.int32), new_length=as_([a + b for a, b in zip(length, add)], torch.int32),
                new_free_count=as_([len(free)], torch.int32), status=as_([0], torch.int32))


def _exact_truncate(s):
    page, table = s["page"], s["table"].tolist()
    given = []
    for r, (have, stay) in enumerate(zip(s["length"].tolist(), s["target"].tolist())):
        given += table[r][-(-stay // page):-(-have // page)]
    count, free = int(s["free_count"]), s["free"].tolist()
    free[count:count + len(given)] = given[::-1]
    return dict(free=torch.tensor(free, dtype=torch.int32), new_free_count=torch.tensor([count + len(given)], dtype=torch.int32),
                status=torch.tensor([0], dtype=torch.int32))


def exact(case, seed):
    s = prepare(case, seed)
    of = {"sample": _exact_sample, "distill": _exact_distill, "extend": _exact_extend, "truncate": _exact_truncate}
    return of[case["op"]](s)
