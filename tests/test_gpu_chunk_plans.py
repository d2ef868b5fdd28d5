"""hisparse_chunk_attention's ways of dividing a call: chunks without starts and lengths (split, in
several row tiles, more tiles than CUs), batches padded to many more rows than they use, thousands of
requests, and what a request's result may depend on. Compared as in test_gpu_chunk_attention."""
import random

import pytest
import torch

import token_reference as ref
from paper_2608_07009_amd import hisparse as hs
from test_gpu_chunk_attention import G, MARK, TYPES, Problem, run

pytestmark = pytest.mark.gpu


def shared(kind, type_, tpr, kv_heads, q_heads, lens, T, tail=0, splits=0, uniform=False,
           max_chunk=0, seed=3):
    """A Problem whose requests all have one table of T tokens (a stride of 0 between theirs), of which
    each sees its first ones. uniform: no starts and no lengths."""
    p = Problem(kind, type_, tpr, kv_heads, q_heads, [(1, T)], splits=splits, seed=seed)
    g = torch.Generator().manual_seed(seed)
    R, H = len(lens), p.H
    p.lens, p.uniform = list(lens), uniform
    p.k, p.v, p.hole = p.k * R, p.v * R, p.hole * R
    p.starts = [0]
    for n, _ in lens:
        p.starts.append(p.starts[-1] + n)
    p.total = p.starts[-1] + tail
    p.q = torch.randn((p.total, H, ref.D_QK[kind]), generator=g).to(torch.bfloat16)
    p.qd = p.q.flatten(1).cuda()
    p.start = None if uniform else torch.tensor(p.starts, dtype=torch.int32, device="cuda")
    p.kv_len = None if uniform else torch.tensor([t for _, t in lens], dtype=torch.int32,
                                                 device="cuda")
    c = p.chunk
    c.num_requests, c.total_tokens, c.table_request_stride = R, p.total, 0
    c.max_chunk = max_chunk or max(n for n, _ in lens)
    p.out = torch.full((p.total, H * ref.D_V[kind]), MARK, dtype=torch.bfloat16, device="cuda")
    p.lse = torch.full((p.total, H), MARK, dtype=torch.float32, device="cuda")
    p.ws_bytes = hs.hisparse_chunk_workspace_bytes(p.kv, c)
    p.ws = torch.full((p.ws_bytes + 64,), 0xFF, dtype=torch.uint8, device="cuda")
    p.run()
    p.check()
    return p


@pytest.mark.parametrize("kind,type_,tpr", TYPES)
def test_one_workspace_for_the_largest_batch(kind, type_, tpr):
    """Sized for 66 requests of 4 kv heads, which fill the CUs and are not split, it serves fewer, which
    are."""
    big = shared(kind, type_, tpr, 4, 4, [(1, 384)] * 66, 384)
    assert big.ws_bytes > 0
    for n in (63, 20, 1):
        p = shared(kind, type_, tpr, 4, 4, [(1, 384)] * n, 384)
        assert 0 < p.ws_bytes <= big.ws_bytes
        p.ws, p.ws_bytes = big.ws, big.ws_bytes
        p.out.fill_(MARK)
        p.lse.fill_(MARK)
        p.run()
        p.check(f"{n} requests")


@pytest.mark.parametrize("kind,type_,tpr", TYPES)
@pytest.mark.parametrize("requests,kv_heads,q_heads,n,splits", [
    (3, 2, 4, 1, 0), (2, 1, 4, 5, 2), (3, 1, 4, 2, 3), (1, 8, 1, 1, 0), (2, 2, 16, 40, 0),
    (2, 2, 16, 40, 3), (2, 1, 16, 21, 1)])
def test_uniform_chunks_in_parts(kind, type_, tpr, requests, kv_heads, q_heads, n, splits):
    """Neither starts nor lengths: split as chosen and as asked for, in one and in several row tiles."""
    p = shared(kind, type_, tpr, kv_heads, q_heads, [(n, 1120)] * requests, 1120, splits=splits,
               uniform=True, tail=3)
    assert (p.ws_bytes > 0) == (splits != 1)


@pytest.mark.parametrize("kind,type_,tpr", TYPES)
@pytest.mark.parametrize("splits", [0, 2])
def test_more_uniform_chunks_than_cus(kind, type_, tpr, splits):
    shared(kind, type_, tpr, 2, 4, [(1, 1120)] * 131, 1120, splits=splits, uniform=True)


@pytest.mark.parametrize("kind,type_,tpr", TYPES)
@pytest.mark.parametrize("n", [1, 40])
def test_few_rows_of_a_batch_padded_to_more_tiles_than_cus(kind, type_, tpr, n):
    """Descriptors whose rows fill more tiles than there are CUs, of which the device finds a few (of
    the largest kind for 40 tokens of 64 heads); two requests without cached or new tokens."""
    p = shared(kind, type_, tpr, 1, 64, [(n, 2000), (0, 50), (2, 0)], 2000, tail=1100,
               max_chunk=1100)
    bm, d_v = (256, 128) if kind == G else (128, 512)
    tiles = 1024 // 4 if kind == G else 1024 // 2
    # the plan of a batch with more tiles than CUs: room for parts of 512 more items than row tiles
    assert p.ws_bytes >= (tiles + 512) * bm * (4 * d_v + 8)


@pytest.mark.parametrize("kind,type_,tpr", TYPES)
def test_thousands_of_requests(kind, type_, tpr):
    """2100 requests of few tokens, one of them long."""
    g = random.Random(8)
    lens = [(g.choice((0, 1, 1, 2)), g.randint(0, 40)) for _ in range(2100)]
    lens[1345] = (3, 3000)
    p = shared(kind, type_, tpr, 1, 2, lens, 3008, tail=1)
    assert p.ws_bytes > 0


@pytest.mark.parametrize("kind,type_,tpr", TYPES)
@pytest.mark.parametrize("splits", [1, 3])
def test_a_given_number_of_splits_makes_results_independent_of_the_batch(kind, type_, tpr, splits):
    """num_splits from 1 on: a request's bits do not change with its neighbours' lengths."""
    mine = (5, 900)
    p = shared(kind, type_, tpr, 2, 4, [(2, 70), mine, (1, 33)], 1120, splits=splits)
    rows = slice(p.starts[1], p.starts[2])
    a, la = p.out[rows].clone(), p.lse[rows].clone()
    o = shared(kind, type_, tpr, 2, 4, [(7, 1120)] * 9 + [mine] + [(1, 1)] * 40, 1120,
               splits=splits)
    at = slice(o.starts[9], o.starts[10])
    o.qd[at] = p.qd[rows]
    o.run()
    torch.cuda.synchronize()
    assert torch.equal(o.out[at], a) and torch.equal(o.lse[at], la)


@pytest.mark.parametrize("kind,type_,tpr", TYPES)
@pytest.mark.parametrize("splits", [0, 3])
def test_starts_that_descend_stay_inside_the_arrays(kind, type_, tpr, splits):
    """Requests that have more rows between them than there are: whatever the rows hold, nothing is
    written past them or past the workspace."""
    p = shared(kind, type_, tpr, 2, 16, [(40, 960), (3, 500), (1, 960), (40, 64)] * 3, 960,
               splits=splits)
    rows = p.total
    p.start = torch.tensor([0, 40, 0, 84, 10, 252, -9, 10 ** 9, 3, 44, 0, 84, 0], dtype=torch.int32,
                           device="cuda")
    p.out = torch.full((rows + 64, p.out.shape[1]), MARK, dtype=torch.bfloat16, device="cuda")
    p.lse = torch.full((rows + 64, p.H), MARK, dtype=torch.float32, device="cuda")
    p.run()
    torch.cuda.synchronize()
    assert bool((p.ws[p.ws_bytes:] == 0xFF).all())
    mark = torch.tensor(MARK).to(torch.bfloat16).cuda()
    assert bool((p.out[rows:] == mark).all()) and bool((p.lse[rows:] == MARK).all())


@pytest.mark.parametrize("kind,type_,tpr", TYPES)
def test_thousands_of_requests_without_starts(kind, type_, tpr):
    """Lengths only, two new tokens each; rows behind the last."""
    g = random.Random(9)
    lens = [(2, g.randint(0, 40)) for _ in range(2050)]
    lens[1500] = (2, 1100)
    p = shared(kind, type_, tpr, 1, 2, lens, 1120, tail=5)
    p.start = None
    p.out.fill_(MARK)
    p.lse.fill_(MARK)
    p.run()
    p.check()


@pytest.mark.parametrize("kind,type_,tpr", TYPES)
def test_more_requests_than_one_launch_takes_with_tables_of_their_own(kind, type_, tpr):
    g = random.Random(10)
    run(kind, type_, tpr, 1, 2, [(g.choice((0, 1, 2)), g.randint(1, 30)) for _ in range(1100)])


@pytest.mark.parametrize("kind,type_,tpr", TYPES)
def test_more_requests_than_one_launch_takes_with_pools_of_their_own(kind, type_, tpr):
    """Slot caches [request][record]: with and without lengths the same bits."""
    R, B = 1027, 2
    gen = torch.Generator().manual_seed(1)
    kk, vv = (torch.randn((R, B, tpr, d), generator=gen).to(torch.bfloat16)
              for d in ref.DIMS[kind])
    pool = ref.make_pool(kind, type_, tpr, kk, vv).cuda()
    rb = pool.shape[-1]
    kv = hs.KvDesc(kind, type_, tpr, rb, B, rb, B * rb, B * rb)
    table = torch.tensor([[r % B, (r + 1) % B] for r in range(R)], dtype=torch.int32, device="cuda")
    q = torch.randn((R, 3, ref.D_QK[kind]), generator=gen).to(torch.bfloat16).cuda()
    c = hs.ChunkDesc(R, 1, 3, R, 1, B, 3 * ref.D_QK[kind], 3 * ref.D_V[kind], B, 0, 0, 0, 0.1, 0)
    ws = torch.empty(hs.hisparse_chunk_workspace_bytes(kv, c), dtype=torch.uint8, device="cuda")
    lens = torch.full((R,), B * tpr, dtype=torch.int32, device="cuda")
    results = []
    for kv_len in (None, lens):
        out = torch.zeros((R, 3, ref.D_V[kind]), dtype=torch.bfloat16, device="cuda")
        lse = torch.zeros((R, 3), device="cuda")
        hs.hisparse_chunk_attention(kv, c, pool, table, None, kv_len, q, out, lse, ws, ws.numel(),
                                    torch.cuda.current_stream())
        results.append((out, lse))
    torch.cuda.synchronize()
    assert torch.equal(results[0][0], results[1][0]) and torch.equal(results[0][1], results[1][1])
    for r in (0, 1023, 1024, R - 1):
        rows = [x[r][table[r].long().cpu()].flatten(0, 1) for x in (kk, vv)]
        sk, sv, _ = ref.stored(kind, *rows, type_)
        e = ref.attend(kind, sk, sv, q[r:r + 1].cpu(), torch.ones((1, B * tpr), dtype=torch.bool), 0.1)
        ref.check(kind, results[1][0][r:r + 1], results[1][1][r:r + 1], e, f"request {r}")
