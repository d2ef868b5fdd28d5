"""hisparse_select_records where the last chosen score ends a cluster: the best candidates lie together, far
above the others or far below a single one, so that the cut falls on the edge of a bin that has to be divided
again. Choices are compared exactly. Cluster scores are whole numbers, every sum of them is exact; real-valued
rows give no equal scores in 64 bits."""
import pytest
import torch

import step_reference as ref
from paper_2608_07009_amd import hisparse as hs
from test_gpu_select import MARK, Case

pytestmark = pytest.mark.gpu
KEYS, BOUNDS, MEANS = ref.KEYS, ref.BOUNDS, ref.MEANS


def clusters(kind, cand, new, heads, size, k, level, first=0, far=0, last=0, t=1, seed=1):
    """Candidates of scores r below 200, and `size` of them, at random places that every new token sees, of
    level + r; far: the score of the first one."""
    c = Case(kind, t, [new], [cand], k=k, heads=heads, q_heads=2, weights=False, first=first, last=last,
             seed=seed, data=lambda shape, g: torch.zeros(shape, dtype=torch.bfloat16))
    g = torch.Generator().manual_seed(seed)
    x = torch.zeros((cand, heads, 2 if kind == BOUNDS else 1, 128))
    x[..., 1:60] = torch.randint(0, 2, (cand, heads, 1, 59), generator=g).float()
    if kind == BOUNDS:
        x[:, :, 1, 1:60] += torch.randint(0, 2, (cand, heads, 59), generator=g).float()
    inner = torch.arange(max(first, 1), cand - new - last)
    for h in range(heads):
        at = inner[torch.randperm(inner.numel(), generator=g)[:size]]
        x[at, h, :, 0] = level
        if far:
            x[0, h, :, 0] = far
    c.table[:] = torch.randperm(c.table.numel(), generator=g).view(c.table.shape).int()
    tab = c.table[0, 0].long()
    per = t if kind == KEYS else 1
    place = torch.arange(cand)
    if kind == KEYS:
        c.index[tab[place // per], :, place % per] = x[:, :, 0].to(torch.bfloat16)
    else:
        c.index[tab[:cand]] = x.to(torch.bfloat16)
    q = torch.zeros((c.total, heads, 2, 128))
    q[..., 0] = 1.0
    q[:, :, 1, 1:60] = 1.0
    if kind == BOUNDS:
        q[:, :, 0, 1] = -1.0
    c.q = q.view(c.total, -1).to(torch.bfloat16)
    return c


# candidates, new tokens, kv heads and the number chosen: each way in which workgroups hold rows
ROWS = {
    "one_wave": (1000, 300, 8, 128),        # bounds and means of more than 2048 rows
    "256_threads": (4000, 1, 2, 200),
    "256_threads_many_rows": (8000, 140, 2, 200),
    "512_threads": (9000, 1, 2, 300),
    "512_threads_many_rows": (20000, 140, 2, 300),
    "1024_threads": (20000, 1, 2, 300),
    "long": (50000, 1, 2, 300),
}


@pytest.mark.parametrize("kind", [KEYS, BOUNDS, MEANS])
@pytest.mark.parametrize("rows", list(ROWS))
def test_the_cut_between_two_clusters(kind, rows):
    cand, new, heads, k = ROWS[rows]
    some = sorted({0, new // 2, new - 1})
    for size in (k - 1, k, k + 1):
        # in one bin of the first division, and over several
        for level in (65536.0, 1024.0):
            clusters(kind, cand, new, heads, size, k, level, seed=size).check(rows=some)


@pytest.mark.parametrize("kind", [KEYS, BOUNDS, MEANS])
@pytest.mark.parametrize("rows", list(ROWS))
def test_the_cut_below_a_first_record_far_above(kind, rows):
    """A record that is always chosen stretches the range of the scores: the cluster shares a bin."""
    cand, new, heads, k = ROWS[rows]
    some = sorted({0, new // 2, new - 1})
    for size in (k - 2, k - 1, k):   # the cluster's last one, with the forced one, is the cut at k - 1
        clusters(kind, cand, new, heads, size, k, 4352.0, first=1, far=2.0 ** 20, seed=size).check(rows=some)
    clusters(kind, cand, new, heads, k - 3, k, 4352.0, first=1, far=2.0 ** 20, last=2, seed=7).check(rows=some)


@pytest.mark.parametrize("kind", [KEYS, BOUNDS, MEANS])
@pytest.mark.parametrize("rows", list(ROWS))
def test_the_cut_between_two_clusters_of_one_bin(kind, rows):
    """Scores 2^20 once, 70016 about k times, 69696 some 500 times and 0: the two middle ones share a bin of
    the first division, and of rows cut down to those in question. They are further apart than the error bound
    tells apart, so that the cut is made by the second division."""
    cand, new, heads, k = ROWS[rows]
    some = sorted({0, new // 2, new - 1})
    for size in (k - 1, k, k + 1):
        c = Case(kind, 1, [new], [cand], k=k, heads=heads, q_heads=2, weights=False, seed=size,
                 data=lambda shape, g: torch.zeros(shape, dtype=torch.bfloat16))
        g = torch.Generator().manual_seed(size)
        tab = c.table[0, 0].long()
        most = min(500, cand - new - size - 1)
        for h in range(heads):
            at = torch.randperm(cand - new, generator=g)[:1 + size + most]
            far, upper = tab[at[:1]], tab[at[1:1 + size - 1]]  # (the far one is of the k best as well)
            lower = tab[at[1 + size - 1:]]
            c.index[far, h, :, 0] = 2.0 ** 20
            c.index[upper, h, :, 0] = c.index[lower, h, :, 0] = 69632.0
            c.index[upper, h, :, 1] = 384.0
            c.index[lower, h, :, 1] = 64.0
        c.q.zero_()
        q = c.q.view(c.total, heads, 2, 128)
        q[:, :, 0, :2] = 1.0
        c.check(rows=some)


@pytest.mark.parametrize("kind", [KEYS, BOUNDS, MEANS])
@pytest.mark.parametrize("size,k", [(1030, 1030), (2047, 2048), (2048, 2048), (2049, 2048)])
def test_large_clusters(kind, size, k):
    for cand in (8192, 40000):
        c = clusters(kind, cand, 1, 1, size, k, 1024.0, seed=k, t=4 if kind == KEYS else 1)
        c.check()


@pytest.mark.parametrize("kind", [KEYS, BOUNDS, MEANS])
@pytest.mark.parametrize("cand,ks", [(4000, range(130, 420)), (9000, range(300, 700)),
                                     (36000, range(1500, 1800))])
def test_every_cut_of_a_row_with_an_outlier(kind, cand, ks):
    """One score hundreds of standard deviations above the others: bins of hundreds of candidates, and the
    cut at each place within them."""
    c = Case(kind, 1, [1], [cand], k=8, q_heads=2, weights=False, seed=cand)
    tab = c.table[0, 0].long()
    if kind == KEYS:   # positive parts only: a head each way ranks like a sum of absolute values
        c.q[:, 128:] = -c.q[:, :128]
    q = c.q[0, :256].float().view(2, 128)
    for row in range(c.index.shape[2]):
        part = q[0] if kind == KEYS else q.clamp(min=0).sum(0) if kind == BOUNDS and row else \
            q.clamp(max=0).sum(0) if kind == BOUNDS else q.sum(0)
        c.index[tab[77], 0, row] = (70.0 * part).to(torch.bfloat16)
    c.device()
    x = ref.scores(kind, q, None, c.index[tab, 0])
    order = torch.sort(x, descending=True, stable=True)[1]
    assert order[0] == 77
    for k in ks:
        c.k = k
        c.d = hs.SelectDesc(c.g, k, 0, 0, c.q.stride(0))
        c.dv["sel"] = torch.full((1, 1, k), MARK, dtype=torch.int32, device="cuda")
        n = hs.hisparse_select_workspace_bytes(c.x, c.b, c.d)
        assert n <= c.dv["ws"].numel()
        c.call(rec=None)
        assert c.dv["sel"][0, 0].tolist() == sorted(order[:k].tolist()), k
