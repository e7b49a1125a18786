"""Pages of a cache on the device against a plain Python restatement: whole numbers, so everything is equal or wrong."""
import numpy as np
import pytest
import torch

import paper_2512_08537_b200 as ardiff
from gpu_util import require_cuda

pytestmark = pytest.mark.gpu
GAP = -77                                     # what buffers hold where nothing may be written


def dev(v, dtype=torch.int32):
    return torch.tensor(v, dtype=dtype, device=require_cuda())


class Cache:
    """Tables, free list and lengths as lists; the operators' meaning in loops."""

    def __init__(self, R, page, width, pages, seed):
        self.R, self.page, self.width = R, page, width
        self.rng = np.random.default_rng(seed)
        self.free = [int(v) for v in self.rng.permutation(pages) * 3 + 5]     # any ids
        self.capacity = pages + 3
        self.length = [0] * R
        self.table = [[GAP] * width for _ in range(R)]

    def pages_of(self, tokens):
        return -(-tokens // self.page)

    def extend(self, add):
        slot, position, request, offset = [], [], [], [0]
        for r in range(self.R):
            for p in range(self.pages_of(self.length[r]), self.pages_of(self.length[r] + add[r])):
                self.table[r][p] = self.free.pop()
            for pos in range(self.length[r], self.length[r] + add[r]):
                slot.append(self.table[r][pos // self.page] * self.page + pos % self.page)
                position.append(pos)
                request.append(r)
            offset.append(len(slot))
            self.length[r] += add[r]
        return slot, position, request, offset

    def truncate(self, target):
        back = []
        for r in range(self.R):
            back += self.table[r][self.pages_of(target[r]):self.pages_of(self.length[r])]
        self.free += back[::-1]
        self.length = list(target)


class Device:
    """The same cache on the device, updated in place."""

    def __init__(self, c):
        self.page = c.page
        self.length, self.table = dev(c.length), dev(c.table).reshape(c.R, c.width)
        self.free = torch.full((c.capacity,), GAP, dtype=torch.int32, device=self.length.device)
        self.free[:len(c.free)] = dev(c.free)
        self.count = dev([len(c.free)])

    def extend(self, add, room, off=0):
        """`off` shifts the buffers away from 16-byte boundaries."""
        make = lambda t: torch.full((room + off,), GAP, dtype=t, device=self.length.device)[off:]  # noqa: E731
        slot, position, request = make(torch.int64), make(torch.int32), make(torch.int32)
        offset, new_length, count, status = ardiff.ardiff_pages_extend(
            self.length, dev(add), self.table, self.free, self.count, self.page, slot, position, request,
            new_length=self.length, new_free_count=self.count)
        assert new_length is self.length and count is self.count
        return slot.tolist(), position.tolist(), request.tolist(), offset.tolist(), int(status)

    def truncate(self, target):
        _, status = ardiff.ardiff_pages_truncate(self.length, dev(target), self.table, self.free, self.count, self.page,
                                                 new_free_count=self.count)
        self.length = dev(target)
        return int(status)


def same(c, d):
    assert d.length.tolist() == c.length
    assert d.table.tolist() == c.table
    assert int(d.count) == len(c.free)
    assert d.free[:len(c.free)].tolist() == c.free
    assert d.free[max(len(c.free), c.most_free):].tolist() == [GAP] * (c.capacity - max(len(c.free), c.most_free))


@pytest.mark.parametrize("R,page,longest,room", [
    (1, 1, 5, 8), (1, 16, 100, 128), (3, 7, 50, 200), (33, 16, 40, 2000), (257, 100, 30, 16384), (1000, 16, 12, 16000),
    (5, 64, 5000, 40000), (96, 1, 700, 70000), (4096, 16, 9, 40000), (4097, 16, 3, 16384), (9000, 4, 4, 40001), (9000, 4, 1, 16384)])
@pytest.mark.parametrize("off", [0, 1])
def test_rounds_of_speculation(R, page, longest, room, off):
    """Prompts, then drafts of which some tokens are taken back, in place on the same buffers."""
    width = -(-(longest + 24) // page)
    c = Cache(R, page, width, R * width, seed=R + page)
    c.most_free = len(c.free)
    d = Device(c)
    for step in range(4):
        most = longest if step == 0 else 8
        add = c.rng.integers(0, most + 1, R)
        add[c.rng.random(R) < 0.2] = 0                          # idle requests
        while add.sum() > room:
            add[np.argmax(add)] = 0
        add = [int(v) for v in add]
        before = list(c.length)
        want = c.extend(add)
        slot, position, request, offset, status = d.extend(add, room, off)
        assert status == ardiff.ARDIFF_OK
        n = len(want[0])
        assert offset == want[3]
        assert slot[:n] == want[0] and position[:n] == want[1] and request[:n] == want[2]
        assert slot[n:] == [GAP] * (room - n) and position[n:] == [GAP] * (room - n) and request[n:] == [GAP] * (room - n)
        same(c, d)
        if step:
            keep = [b + int(c.rng.integers(0, a + 1)) for a, b in zip(add, before)]
            c.truncate(keep)
            assert d.truncate(keep) == ardiff.ARDIFF_OK
            same(c, d)
    c.truncate([0] * R)                                         # all requests end
    assert d.truncate([0] * R) == ardiff.ARDIFF_OK
    same(c, d)
    assert len(c.free) == R * width


def test_what_is_taken_back_is_given_out_again_alike():
    c = Cache(40, 16, 9, 400, seed=1)
    c.most_free = len(c.free)
    d = Device(c)
    d.extend([37] * 40, 4000)
    table, count, length = d.table.clone(), d.count.clone(), d.length.tolist()
    for add in ([8] * 40, [0, 50] * 20, [100] + [0] * 39):
        before = d.table.clone()
        assert d.extend(add, 4000)[-1] == ardiff.ARDIFF_OK
        first = d.table.clone()
        assert d.truncate(length) == ardiff.ARDIFF_OK
        assert torch.equal(d.count, count)
        assert d.extend(add, 4000)[-1] == ardiff.ARDIFF_OK
        assert torch.equal(d.table, first)
        assert d.truncate(length) == ardiff.ARDIFF_OK
        d.table.copy_(before)
    assert torch.equal(d.table, table)


@pytest.mark.parametrize("room", [512, 20000])                  # one launch, two launches
@pytest.mark.parametrize("what,code", [
    ("negative add", ardiff.ARDIFF_ERR_SHAPE), ("negative length", ardiff.ARDIFF_ERR_SHAPE),
    ("longer than its row", ardiff.ARDIFF_ERR_SHAPE), ("length near 2^31", ardiff.ARDIFF_ERR_SHAPE),
    ("more tokens than room", ardiff.ARDIFF_ERR_SHAPE), ("free count above capacity", ardiff.ARDIFF_ERR_SHAPE),
    ("negative free count", ardiff.ARDIFF_ERR_SHAPE), ("pages run out", ardiff.ARDIFF_ERR_NOMEM)])
@pytest.mark.parametrize("R", [6, 5000])
def test_extend_takes_nothing_where_it_cannot_give_all(R, room, what, code):
    device = require_cuda()
    width, page = 4, 16
    length, add = [3] * R, [0] * R
    add[-1] = 20
    count, capacity = 10, 12
    if what == "negative add":
        add[2] = -1
    elif what == "negative length":
        length[2] = -5
    elif what == "longer than its row":
        add[3] = width * page - 2
    elif what == "length near 2^31":
        length[0], add[0] = 2 ** 31 - 1, 2 ** 31 - 1
    elif what == "more tokens than room":
        page, add[1] = 16384, room
    elif what == "free count above capacity":
        count = 13
    elif what == "negative free count":
        count = -1
    else:
        count = 0
    table = torch.arange(R * width, dtype=torch.int32, device=device).reshape(R, width)
    table0 = table.clone()
    free = torch.arange(capacity, dtype=torch.int32, device=device)
    slot = torch.full((room,), GAP, dtype=torch.int64, device=device)
    offset, new_length, new_count, status = ardiff.ardiff_pages_extend(dev(length), dev(add), table, free, dev([count]), page, slot)
    assert int(status) == code
    assert new_length.tolist() == length and int(new_count) == count
    assert offset.tolist() == [0] * (R + 1)
    assert torch.equal(table, table0) and free.tolist() == list(range(capacity))
    assert bool((slot == GAP).all())


@pytest.mark.parametrize("what", ["target above length", "negative target", "longer than its row", "no room", "negative count"])
@pytest.mark.parametrize("R", [6, 5000])
def test_truncate_gives_nothing_back_where_it_cannot_give_all(R, what):
    device = require_cuda()
    width, page = 4, 16
    length, target = [40] * R, [40] * R
    target[1] = 5
    count, capacity = 10, 12
    if what == "target above length":
        target[2] = 41
    elif what == "negative target":
        target[2] = -1
    elif what == "longer than its row":
        length[2] = 65
    elif what == "no room":
        target[-1] = 0
    else:
        count = -1
    table = torch.arange(R * width, dtype=torch.int32, device=device).reshape(R, width)
    free = torch.arange(100, 100 + capacity, dtype=torch.int32, device=device)
    new_count, status = ardiff.ardiff_pages_truncate(dev(length), dev(target), table, free, dev([count]), page)
    assert int(status) == ardiff.ARDIFF_ERR_SHAPE and int(new_count) == count
    assert free.tolist() == list(range(100, 100 + capacity))


def test_no_requests_and_slots_beyond_32_bits():
    device = require_cuda()
    empty = torch.empty((0,), dtype=torch.int32, device=device)
    table = torch.empty((0, 4), dtype=torch.int32, device=device)
    free = dev([7, 8])
    slot = torch.empty((0,), dtype=torch.int64, device=device)
    offset, _, count, status = ardiff.ardiff_pages_extend(empty, empty, table, free, dev([2]), 16, slot)
    assert offset.tolist() == [0] and int(count) == 2 and int(status) == 0
    count, status = ardiff.ardiff_pages_truncate(empty, empty, table, free, dev([2]), 16)
    assert int(count) == 2 and int(status) == 0
    # the last page of a pool of 2^31 pages of 2^20 tokens
    table = dev([[2 ** 31 - 1, -1]])
    slot = torch.empty((2,), dtype=torch.int64, device=device)
    ardiff.ardiff_pages_extend(dev([2 ** 20 - 1]), dev([2]), table, dev([2 ** 31 - 2]), dev([1]), 2 ** 20, slot)
    assert slot.tolist() == [(2 ** 31 - 1) * 2 ** 20 + 2 ** 20 - 1, (2 ** 31 - 2) * 2 ** 20]


def test_captured_extend_and_truncate_follow_their_buffers_at_every_replay():
    device = require_cuda()
    R, page, room = 50, 16, 20000
    c = Cache(R, page, 30, R * 30, seed=5)
    c.most_free = len(c.free)
    d = Device(c)
    add = torch.zeros((R,), dtype=torch.int32, device=device)
    drop = torch.zeros((R,), dtype=torch.int32, device=device)
    target = torch.zeros((R,), dtype=torch.int32, device=device)
    slot = torch.full((room,), GAP, dtype=torch.int64, device=device)
    offset = torch.zeros((R + 1,), dtype=torch.int32, device=device)
    status = torch.zeros((2,), dtype=torch.int32, device=device)

    def step():
        ardiff.ardiff_pages_extend(d.length, add, d.table, d.free, d.count, page, slot, offset=offset, new_length=d.length,
                                   new_free_count=d.count, status=status[:1])
        torch.sub(d.length, drop, out=target)
        ardiff.ardiff_pages_truncate(d.length, target, d.table, d.free, d.count, page, new_free_count=d.count, status=status[1:])
        d.length.copy_(target)

    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        step()
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        step()
    for i in range(5):
        more = [int(v) for v in c.rng.integers(0, 300 if i == 0 else 40, R)]
        less = [int(c.rng.integers(0, min(v, 40) + 1)) for v in more]
        want = c.extend(more)
        c.truncate([a - b for a, b in zip(c.length, less)])
        add.copy_(dev(more))
        drop.copy_(dev(less))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert status.tolist() == [0, 0]
        assert offset.tolist() == want[3] and slot[:len(want[0])].tolist() == want[0]
        same(c, d)


def test_calls_on_another_stream_than_the_current_one():
    c = Cache(300, 16, 40, 300 * 40, seed=9)
    d = Device(c)
    add = [int(v) for v in c.rng.integers(0, 400, 300)]
    want = c.extend(add)
    slot = torch.full((len(want[0]),), GAP, dtype=torch.int64, device=d.length.device)
    more = dev(add)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    offset, _, _, status = ardiff.ardiff_pages_extend(d.length, more, d.table, d.free, d.count, 16, slot, stream=s)
    s.synchronize()
    assert int(status) == 0 and slot.tolist() == want[0] and offset.tolist() == want[3]


def test_pages_given_back_up_to_the_last_number_of_32_bits():
    """A step of the CTA past the last page would pass 2^31."""
    W = 2**31 - 600
    table = torch.arange(W, dtype=torch.int32, device=require_cuda()).reshape(1, W)
    free = torch.full((W,), GAP, dtype=torch.int32, device=table.device)
    count, status = ardiff.ardiff_pages_truncate(dev([W]), dev([0]), table, free, dev([0]), 1)
    assert (int(count), int(status)) == (W, 0)
    step = 1 << 28
    for i in range(0, W, step):                   # the last page lowest
        n = min(step, W - i)
        assert torch.equal(free[i:i + n], table[0, W - i - n:W - i].flip(0))


@pytest.mark.parametrize("tokens", [2**31 - 1, 2**31 - 4])
def test_tokens_up_to_the_last_number_of_32_bits(tokens):
    page, width = 1 << 20, 2048
    slot = torch.full((tokens,), GAP, dtype=torch.int64, device=require_cuda())
    table, free = dev([[GAP] * width]), dev(list(range(7, 7 + width)))
    offset, length, count, status = ardiff.ardiff_pages_extend(dev([0]), dev([tokens]), table, free, dev([width]), page, slot)
    assert (offset.tolist(), int(length), int(count), int(status)) == ([0, tokens], tokens, 0, 0)
    assert table[0].tolist() == free.tolist()[::-1]
    for p in range(width):
        lo, n = p * page, min(page, tokens - p * page)
        assert torch.equal(slot[lo:lo + n], torch.arange(n, device=slot.device) + int(6 + width - p) * page)
