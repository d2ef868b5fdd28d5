"""hisparse_select_records: rows of every length side by side, long ones above all, and chunks around the
lengths at which another way of scoring begins. References and exactness as in test_gpu_select."""
import random

import pytest
import torch

import step_reference as ref
from test_gpu_select import BOUNDS, KEYS, MARK, MEANS, Case, randn, small_whole

pytestmark = pytest.mark.gpu


def long_data(kind):
    """Real-valued rows of any number without a randn of each: a few thousand, each but the first of a run
    scaled by a number of its own."""
    def make(shape, g):
        n = shape[0]
        x = torch.randn((min(n, 4099), *shape[1:]), generator=g)
        if kind == BOUNDS:
            x = torch.stack((x.amin(2), x.amax(2)), 2)
        x = x.repeat((n + x.shape[0] - 1) // x.shape[0], *[1] * (len(shape) - 1))[:n]
        return (x * (0.5 + torch.rand((n, 1, 1, 1), generator=g))).to(torch.bfloat16)
    return make


@pytest.mark.parametrize("kind", [KEYS, BOUNDS, MEANS])
@pytest.mark.parametrize("first,last,k", [(0, 1, 2048), (5, 3, 700), (100, 0, 101), (0, 0, 4096)])
def test_long_and_short_rows_of_one_batch(kind, first, last, k):
    t = 32 if kind == KEYS else 1
    lens = [70003, 33, 32768, 32769, 0, k, 50000, k + 1]
    c = Case(kind, t, [2, 1, 2, 1, 1, 1, 3, 1], lens, k=k, first=first, last=last, q_heads=5, seed=k, tail=2,
             data=long_data(kind))
    rng = random.Random(k)
    for r in (0, 3, 6):
        for _ in range(40):
            c.table[r, 0, rng.randrange((lens[r] + t - 1) // t)] = rng.choice((-1, c.index.shape[0]))
    if last:
        c.table[3, 0, (lens[3] - 1) // t if kind == KEYS else lens[3] - 1] = -1  # the newest one
    c.check()


@pytest.mark.parametrize("kind", [KEYS, BOUNDS, MEANS])
def test_long_rows_of_a_chunk(kind):
    """Chunks that pass the length from which rows are long, several kv heads, and workspaces of a few rows."""
    t = 16 if kind == KEYS else 1
    c = Case(kind, t, [9, 6], [32772, 40001], k=300, last=2, first=1, heads=2, q_heads=3, data=long_data(kind))
    c.check()
    whole = c.dv["sel"].clone()
    c.device(ws=lambda n: (n // c.total + 1) * 4 + 64)
    c.call()
    assert torch.equal(c.dv["sel"], whole)


@pytest.mark.parametrize("kind", [KEYS, BOUNDS, MEANS])
def test_equal_scores_in_long_rows(kind):
    """Few distinct scores: more candidates of one score than are held at once, the lower position first."""
    for zeros, k in ((0.97, 2000), (0.9999, 3000)):
        c = Case(kind, 1, [1, 1], [90000, 33000], k=k, q_heads=2, last=1, weights=False,
                 data=small_whole(-1, 1, zeros))
        c.q = torch.randint(-1, 2, c.q.shape, generator=torch.Generator().manual_seed(8)).to(torch.bfloat16)
        c.check()


@pytest.mark.parametrize("kind", [KEYS, MEANS])
def test_not_finite_scores_in_long_rows(kind):
    c = Case(kind, 1, [1], [50000], k=40, q_heads=2, weights=False, data=long_data(kind))
    c.q = c.q.abs()
    tab = c.table[0, 0].long()
    x = c.index[tab, 0, 0]
    x[100, 5] = x[45000, 7] = float("nan")
    x[200, 0] = x[201, 0] = x[40000, 3] = float("inf")
    x[50, 0] = -float("inf")
    c.index[tab, 0, 0] = x
    c.check()
    assert {100, 45000} <= set(c.dv["sel"][0, 0].tolist())


@pytest.mark.parametrize("kind", [KEYS, BOUNDS, MEANS])
def test_long_rows_captured_and_replayed(kind):
    t = 16 if kind == KEYS else 1
    c = Case(kind, t, [2, 1], [60000, 60000], k=500, last=1, q_heads=3, data=long_data(kind))
    c.device()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=side):
        c.call()
    for i, lens in enumerate(([60000, 1], [32768, 32770], [400, 45001], [60000, 59999])):
        c.lens, c.q = lens, randn(c.q.shape, i)
        c.dv["lens"].copy_(torch.tensor(lens, dtype=torch.int32))
        c.dv["q"].copy_(c.q.flatten())
        for x in ("sel", "rec", "slen"):
            c.dv[x].fill_(MARK)
        c.dv["ws"].fill_(0xEE)
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        c.compare()


@pytest.mark.parametrize("kind", [KEYS, BOUNDS, MEANS])
@pytest.mark.parametrize("q_heads", [4, 16, 20, 64, 100])
def test_chunks_of_every_length_side_by_side(kind, q_heads):
    """1 to 9 new tokens (another way of scoring from 5 on) and chunks that pass a workgroup's share."""
    t = 8
    scale = 1 if kind == KEYS else t
    new = [1, 2, 3, 4, 5, 6, 7, 8, 9, 0, 130, 4, 5, 33, 1]
    lens = [(400 + 61 * i) * scale - i for i in range(len(new))]
    lens[2], lens[6], lens[12] = 2, 3 * scale, 20 * scale
    c = Case(kind, t, new, lens, heads=2, q_heads=q_heads, k=21, last=1, first=1, seed=q_heads, tail=3)
    c.check()
    whole = c.dv["sel"].clone()
    for rows in (4, 7, 50):  # steps that end inside chunks
        c.device(ws=lambda n: (n // c.total + 1) * rows + 64)
        c.call()
        assert torch.equal(c.dv["sel"], whole)


@pytest.mark.parametrize("kind", [KEYS, BOUNDS, MEANS])
@pytest.mark.parametrize("cand,k", [(4100, 2048), (32768, 300), (20011, 7)])
def test_more_rows_than_the_chip_has_workgroups_for(kind, cand, k):
    """Rows that many choose with half the threads, as all others do."""
    t = 4 if kind == KEYS else 1
    c = Case(kind, t, [129, 1, 2], [cand, cand - 9, cand // 2], k=k, heads=2, q_heads=3, last=2, first=1,
             data=long_data(kind), tail=3)
    c.table[0, 0, 5], c.table[1, 0, 70] = -1, c.index.shape[0]
    c.check(rows=[0, 1, 63, 64, 127, 128, 129, 130, 131])
    whole = c.dv["sel"].clone()
    c.device(ws=lambda n: (n // c.total + 1) * 100 + 64)
    c.call()
    assert torch.equal(c.dv["sel"], whole)


@pytest.mark.parametrize("kind", [KEYS, BOUNDS, MEANS])
def test_thousands_of_short_rows(kind):
    for cand, k in ((1024, 100), (513, 24), (300, 1)):
        t = 4
        c = Case(kind, t, [700, 2], [cand * (1 if kind == KEYS else t), cand - 7], k=k, heads=3, q_heads=3,
                 first=int(k > 1), last=int(k > 2), tail=1)
        c.table[0, 0, 5], c.table[0, 0, 70] = -1, c.index.shape[0]
        c.check(rows=[0, 1, 350, 699, 700, 701])


@pytest.mark.parametrize("kind", [BOUNDS, MEANS])
def test_equal_scores_in_thousands_of_short_rows(kind):
    c = Case(kind, 1, [2100], [1000 + 2100], k=90, q_heads=2, last=1, weights=False, data=small_whole(-1, 1, 0.98))
    c.per = 1024
    c.table = c.table[:, :, :1024].contiguous()
    c.lens = [1024]
    c.q = torch.randint(-1, 2, c.q.shape, generator=torch.Generator().manual_seed(8)).to(torch.bfloat16)
    c.q[2007] = 0
    c.check(rows=[0, 1075, 1076, 1500, 2007, 2099])


@pytest.mark.parametrize("kind", [KEYS, BOUNDS, MEANS])
def test_equal_scores_in_many_rows(kind):
    c = Case(kind, 1, [300], [9000], k=900, q_heads=2, last=1, weights=False, data=small_whole(-1, 1, 0.9))
    c.q = torch.randint(-1, 2, c.q.shape, generator=torch.Generator().manual_seed(8)).to(torch.bfloat16)
    c.q[7], c.q[8] = 0, c.q[9]
    c.check(rows=[0, 7, 8, 150, 299])


@pytest.mark.parametrize("kind", [KEYS, BOUNDS, MEANS])
@pytest.mark.parametrize("max_chunk", [4, 5, 40])
def test_uniform_chunks(kind, max_chunk):
    t = 4
    n = 500 * (1 if kind == KEYS else t)
    Case(kind, t, [max_chunk] * 6, [n, n - 1, 3, 0, max_chunk, n // 2], k=17, last=1, uniform=True, heads=2,
         tail=2, q_heads=9).check()


@pytest.mark.parametrize("kind", [KEYS, BOUNDS, MEANS])
@pytest.mark.parametrize("t", [64, 256])
def test_padding_of_large_records(kind, t):
    n = 3000 if kind == KEYS else 300 * t
    for new in ([1, 1], [7, 5]):
        c = Case(kind, t, new, [n - 5, n], k=60, last=2, heads=2, per_head=True)
        g = torch.Generator().manual_seed(t)
        c.table[torch.rand(c.table.shape, generator=g) < 0.3] = -1
        c.check()


def test_large_norms_beyond_a_new_tokens_own_candidates():
    """Rows that only the chunk's last new token sees are above all others, infinite or NaN."""
    for value in (1e30, float("inf"), float("nan")):
        for kind in (KEYS, MEANS):
            c = Case(kind, 1, [8], [700], k=9, q_heads=2)
            tab = c.table[0, 0].long()
            c.index[tab[699], 0, 0, 3] = value
            c.check()


@pytest.mark.parametrize("kind", [KEYS, BOUNDS, MEANS])
def test_two_calls_at_once(kind):
    """Two streams, a workspace each."""
    t = 16 if kind == KEYS else 1
    a = Case(kind, t, [1, 1], [40000, 900], k=200, last=1, q_heads=4, data=long_data(kind))
    b = Case(kind, t, [40], [3000], k=64, q_heads=4, seed=2)
    a.device()
    b.device()
    torch.cuda.synchronize()
    one, two = torch.cuda.Stream(), torch.cuda.Stream()
    for _ in range(5):
        a.call(stream=one)
        b.call(stream=two)
    torch.cuda.synchronize()
    a.compare()
    b.compare()


@pytest.mark.parametrize("kind", [KEYS, BOUNDS, MEANS])
@pytest.mark.parametrize("new", [1, 9])
def test_offsets_beyond_four_gibibytes(kind, new):
    """Index records 256 MiB apart."""
    t = 16 if kind == KEYS else 1
    c = Case(kind, t, [new], [21 * t if kind == KEYS else 21], k=5, last=1, heads=2, spare=3)
    c.device()
    apart = 1 << 28
    records, row = c.index.shape[0], c.index[0].numel()
    far = torch.empty(records * apart // 2, dtype=torch.bfloat16, device="cuda").view(records, apart // 2)
    far[:, :row] = c.index.flatten(1).cuda()
    c.x.record_stride = apart
    c.call(index=far)
    torch.cuda.synchronize()
    c.compare()
