"""hisparse_plan_tokens against a loop over requests and tokens: every output, and the tables around what
is written, exactly."""
import random

import pytest
import torch

import step_reference as ref
from paper_2608_07009_amd import hisparse as hs

pytestmark = pytest.mark.gpu


def ints(x, dtype=torch.int32):
    return torch.tensor(x, dtype=dtype, device="cuda")


class Case:
    def __init__(self, new, kv, t, total, per, spare=3, max_chunk=None, with_free=True, used=2,
                 seed=1, pad=0):
        rng = random.Random(seed)
        self.t, self.total, self.per, self.new, self.kv = t, total, per, new, kv
        self.max_chunk = max_chunk or max(max(new), 1)
        R = len(new)
        ids = list(range(R * per + 2 * spare + 8))
        rng.shuffle(ids)
        old = kv or [0] * R
        self.table = [[-1] * (per + pad) for _ in range(R)]
        for r in range(R):
            have = (ref.clamp(old[r], 0, per * t) + t - 1) // t if with_free else per
            for e in range(have):
                self.table[r][e] = ids.pop()
            for e in range(have, per + pad):
                self.table[r][e] = -7 - e    # must stay, or be written
        self.free = None
        self.used = used if with_free else 0
        if with_free:
            begun = min(sum(max(n, 0) // t + 2 for n in new), total + 2 * R)
            self.free = [ids.pop() if ids else 10 ** 6 + i for i in range(used + begun + spare)]
        self.batch = hs.BatchDesc(R, 1, total, self.max_chunk, per, t, per + pad, 0)

    def expected(self):
        table = [row[:] for row in self.table]
        return (table,) + ref.plan(self.new, self.kv, self.t, self.max_chunk, self.per, self.total,
                                   self.free, self.used, table)

    def device(self):
        R = len(self.new)
        self.d = dict(new=ints(self.new), kv=ints(self.kv) if self.kv else None,
                      free=ints(self.free) if self.free else None,
                      used=ints([self.used]) if self.free else None, table=ints(self.table),
                      start=ints([-5] * (R + 2)), out=ints([-5] * (R + 1)), used_out=ints([-5] * 2),
                      pos=ints([-5] * (self.total + 1)),
                      slots=ints([-5] * (self.total + 1), torch.int64))

    def call(self, **kw):
        d = dict(self.d, **kw)
        hs.hisparse_plan_tokens(self.batch, d["new"], d["kv"], d["free"],
                                len(self.free) if self.free else 0, d["used"], d["table"],
                                d["start"], d["out"], d["used_out"], d["pos"], d["slots"],
                                torch.cuda.current_stream())

    def check(self):
        self.device()
        self.call()
        table, start, out, used, pos, slots = self.expected()
        R = len(self.new)
        assert self.d["start"].tolist() == start + [-5]
        assert self.d["out"].tolist() == out + [-5]
        assert self.d["used_out"].tolist() == [used, -5]
        assert self.d["pos"].tolist() == pos + [-5]
        assert self.d["slots"].tolist() == slots + [-5]
        assert self.d["table"].tolist() == table
        assert len(out) == R


def ragged(R, chunk, context, seed):
    rng = random.Random(seed)
    new = [rng.choice((0, 1, 1, rng.randint(0, chunk))) for _ in range(R)]
    return new, [rng.randint(0, context) for _ in range(R)]


@pytest.mark.parametrize("t", [1, 2, 16, 64, 4096])
@pytest.mark.parametrize("R,chunk,context", [(1, 1, 5), (3, 40, 100), (64, 1, 300), (65, 7, 90),
                                             (1025, 3, 40), (130, 200, 300)])
def test_ragged_batches(R, chunk, context, t):
    new, kv = ragged(R, chunk, context, R + t)
    per = (max(k + n for k, n in zip(kv, new)) + t - 1) // t + 1
    Case(new, kv, t, sum(new) + 5, per, pad=2).check()


def test_one_workgroup_and_many_give_the_same():
    for total in (4096, 4097, 9001):  # 4096 rows and fewer are one workgroup's
        new, kv = ragged(70, 150, 200, total)
        while sum(new) > total:
            new[new.index(max(new))] //= 2
        Case(new, kv, 16, total, 30).check()
    new, kv = ragged(4097, 2, 30, 9)  # and 4096 requests
    Case(new, kv, 16, sum(new), 4).check()


@pytest.mark.parametrize("new,kv", [([0], [0]), ([0, 0, 0], [0, 5, 64]), ([1], [0]), ([1], [63]),
                                    ([1], [64]), ([64], [64]), ([65, 1], [63, 128]),
                                    ([3, 0, 2], None)])
def test_edges(new, kv):
    for t in (1, 64):
        Case(new, kv, t, sum(new), 300 // t + 1).check()
        Case(new, kv, t, sum(new) + 3, 300 // t + 1).check()


def test_values_are_held():
    # negative lengths, chunks above the most, tables that are full, more tokens than rows
    Case([-3, 5, 9, 4], [7, -2, 30, 10 ** 9], 4, 40, 8, max_chunk=6).check()
    Case([6, 6, 6, 6, 6], [0, 3, 31, 32, 2], 4, 11, 8).check()
    Case([2 ** 31 - 1] * 5, [0] * 5, 16, 5000, 400, max_chunk=2 ** 31 - 1).check()
    Case([2 ** 31 - 1] * 1100, [3] * 1100, 16, 900, 2, max_chunk=2 ** 31 - 1).check()


def test_too_few_free_records():
    c = Case([40, 1, 33], [0, 16, 5], 16, 80, 8, spare=0)
    c.free = c.free[:4]  # two are used: two of the six that begin
    c.check()
    assert c.d["used_out"][0].item() == 2 + 6 > 4 and (c.d["slots"][:74] == -1).any()
    c = Case([40, 1, 33], [0, 16, 5], 16, 80, 8, used=99, spare=0)
    c.free = c.free[:4]  # more used than there are: none left
    c.check()


def test_tables_that_are_complete():
    for total in (60, 5000):
        c = Case([20, 0, 31], [3, 64, 100], 16, total, 12, with_free=False)
        c.table[2][7] = -1  # a record that is missing: its tokens have no slot
        c.check()
        assert (c.d["slots"] == -1).sum() > total - 51


@pytest.mark.parametrize("total", [300, 6000])
def test_lengths_and_counts_updated_in_place(total):
    """A decode loop keeps one array of lengths and one count; captured once, replayed with other new
    tokens."""
    new, kv = ragged(90, 3, 70, 5)
    c = Case(new, kv, 16, total, 12, spare=400)
    c.device()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    keep = c.d["table"].clone(), c.d["kv"].clone(), c.d["used"].clone()
    with torch.cuda.stream(side):
        c.call(out=c.d["kv"], used_out=c.d["used"])
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            c.call(out=c.d["kv"], used_out=c.d["used"])
    torch.cuda.synchronize()
    for x, y in zip((c.d["table"], c.d["kv"], c.d["used"]), keep):
        x.copy_(y)
    for step in range(4):
        c.new = [(n + step) % 4 for n in new]
        c.d["new"].copy_(ints(c.new))
        table, start, out, used, pos, slots = c.expected()
        g.replay()
        torch.cuda.synchronize()
        assert c.d["kv"].tolist() == out and c.d["used"].tolist() == [used]
        assert c.d["start"].tolist()[:-1] == start and c.d["table"].tolist() == table
        assert c.d["pos"].tolist()[:-1] == pos and c.d["slots"].tolist()[:-1] == slots
        c.table, c.kv, c.used = table, out, used


def test_optional_outputs():
    for total in (50, 5000):
        c = Case([5, 9], [2, 15], 16, total, 4)
        c.device()
        c.call(pos=None, slots=None, used_out=None)
        table, start, out, used, pos, slots = c.expected()
        assert c.d["table"].tolist() == table and c.d["out"].tolist()[:-1] == out
        c.device()
        c.call(pos=None)
        assert c.d["slots"].tolist()[:-1] == slots
        c.device()
        c.call(slots=None, used=None)
        c.used = 0
        assert c.d["pos"].tolist()[:-1] == c.expected()[4]
        assert c.d["table"].tolist() == c.expected()[0]


@pytest.mark.parametrize("n", [2047, 2048, 2049])
def test_the_border_between_one_launch_and_two(n):
    """Batches of up to 2048 rows and 2048 requests are one launch; each of the two numbers around it."""
    new, kv = ragged(70, 60, 200, n)
    while sum(new) > n - 3:
        new[new.index(max(new))] //= 2
    Case(new, kv, 16, n, 30).check()             # rows behind the last request's
    Case([n], [5], 16, n, 200).check()           # and none
    new, kv = ragged(n, 1, 30, 9)
    Case(new, kv, 4, min(sum(new), 2048), 10).check()
    new = [0] * n
    new[0] = new[-1] = 3
    Case(new, kv, 4, 6, 10).check()
    for total in (n, 7000):                      # lengths and the count updated in place
        new, kv = ragged(90, 20, 70, n)
        c = Case(new, kv, 16, total, 12, spare=400)
        c.device()
        c.call(out=c.d["kv"], used_out=c.d["used"])
        table, start, out, used, pos, slots = c.expected()
        assert c.d["kv"].tolist() == out and c.d["used"].tolist() == [used]
        assert c.d["start"].tolist()[:-1] == start and c.d["table"].tolist() == table
        assert c.d["pos"].tolist()[:-1] == pos and c.d["slots"].tolist()[:-1] == slots
