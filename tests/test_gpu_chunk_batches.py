"""hisparse_chunk_attention over batches as a scheduler builds them: hundreds of requests, one of them
long, long contexts, padding, chunks without starts or lengths, and a captured step of writes and
attention. Compared as in test_gpu_chunk_attention."""
import math
import random

import pytest
import torch

import token_reference as ref
from paper_2608_07009_amd import hisparse as hs
from test_gpu_chunk_attention import BF, F8, G, L, MARK, TYPES, Problem, grow, run

pytestmark = pytest.mark.gpu


def decoding(n, most, seed):
    g = random.Random(seed)
    return [(1, g.randint(1, most)) for _ in range(n)]


@pytest.mark.parametrize("kind,type_,tpr", TYPES)
@pytest.mark.parametrize("splits", [0, 2])
def test_more_requests_than_lanes(kind, type_, tpr, splits):
    """150 requests, fewer row tiles than CUs: all may be split."""
    lens = decoding(149, 300, 1)
    lens[70:70] = [(9, 700)]
    run(kind, type_, tpr, 1, 4, lens, splits=splits, tail=3)


@pytest.mark.parametrize("kind,type_,tpr", TYPES)
@pytest.mark.parametrize("at", [0, 131, 269])
def test_one_long_request_among_many(kind, type_, tpr, at):
    """More row tiles than CUs: only the long request is split, wherever it lies."""
    lens = decoding(269, 40, 2)
    lens[at:at] = [(1, 4000)]
    p = run(kind, type_, tpr, 1, 4, lens, tail=2)
    assert p.ws_bytes > 0


@pytest.mark.parametrize("kind,type_,tpr", TYPES)
@pytest.mark.parametrize("splits", [0, 3])
def test_many_requests_without_starts(kind, type_, tpr, splits):
    """Lengths only, two new tokens each; split as chosen and as asked for."""
    lens = [(2, t) for _, t in decoding(279, 40, 5)]
    lens[200] = (2, 3000)
    run(kind, type_, tpr, 1, 4, lens, uniform=True, splits=splits)


@pytest.mark.parametrize("kind,type_,tpr", TYPES)
def test_captured_batch_whose_lengths_change(kind, type_, tpr):
    """One graph of a batch for up to 270 requests, replayed with one long request, with none, and with
    few requests at all: each equals a call of its own."""
    lens = decoding(269, 40, 6)
    lens[100:100] = [(1, 2500)]
    p = Problem(kind, type_, tpr, 1, 4, lens, tail=2)
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        p.run(side)
    all_start, all_len = p.start.clone(), p.kv_len.clone()
    for turn in range(4):
        p.start.copy_(all_start)
        p.kv_len.copy_(all_len)
        p.starts, p.lens = all_start.tolist(), list(lens)
        if turn == 1:  # none is long
            p.lens[100] = (1, 17)
        if turn == 2:  # the requests behind the first 102 have no new tokens
            p.start[102:] = 102
            p.starts = p.starts[:103]
            p.lens = p.lens[:102]
        p.kv_len[100] = p.lens[100][1]
        short = Problem.__new__(Problem)
        short.__dict__.update(p.__dict__)
        if turn == 1:  # the request's first 17 tokens, in whole pages
            n = (17 + tpr - 1) // tpr * tpr
            short.k, short.v, short.hole = ([x[:n] if i == 100 else x for i, x in enumerate(y)]
                                            for y in (p.k, p.v, p.hole))
        p.out.fill_(MARK)
        p.lse.fill_(MARK)
        torch.cuda.synchronize()
        graph.replay()
        short.check(f"turn {turn}")
        out, lse = p.out.clone(), p.lse.clone()
        p.run()
        torch.cuda.synchronize()
        assert torch.equal(out, p.out) and torch.equal(lse, p.lse)


@pytest.mark.parametrize("kind,type_,tpr", TYPES)
def test_long_chunk_among_many(kind, type_, tpr):
    """The same with a chunk of many row tiles, the largest ones, and two heads."""
    lens = decoding(150, 40, 3)
    lens[80:80] = [(40, 3000)]
    run(kind, type_, tpr, 2, 16, lens)


@pytest.mark.parametrize("kind,type_,tpr", TYPES)
def test_long_request_in_a_padded_batch(kind, type_, tpr):
    """Rows for more tiles than CUs, of which one request's single token is used; others have no
    cached tokens, or no new ones."""
    run(kind, type_, tpr, 1, 64, [(1, 3000), (0, 50), (2, 0)], tail=1100)


@pytest.mark.parametrize("kind,type_,tpr", TYPES)
@pytest.mark.parametrize("q_heads,splits", [(2, 1), (2, 3), (32, 1), (32, 2)])
def test_long_contexts(kind, type_, tpr, q_heads, splits):
    """Thousands of cached tokens in one part, from few rows and from more than one row tile."""
    run(kind, type_, tpr, 1, q_heads, [(9, 1500), (1, 4999)], splits=splits)


@pytest.mark.parametrize("kind,type_,tpr", TYPES)
@pytest.mark.parametrize("splits", [0, 1, 3])
def test_long_windows(kind, type_, tpr, splits):
    run(kind, type_, tpr, 2, 16, [(30, 1900), (1, 1300)], window=700, splits=splits)


@pytest.mark.parametrize("kind,type_,tpr", TYPES)
@pytest.mark.parametrize("window", [2 ** 31 - 1, 2 ** 30, 4096])
def test_windows_longer_than_any_request(kind, type_, tpr, window):
    """Nothing is cut off, also where a request has fewer cached than new tokens."""
    lens = [(9, 700), (1, 900), (40, 3), (5, 5), (0, 9)] + decoding(60, 300, 4)
    run(kind, type_, tpr, 1, 4, lens, window=window)
    run(kind, type_, tpr, 1, 4, lens, window=window, splits=1)


@pytest.mark.parametrize("kind,type_,tpr", TYPES)
@pytest.mark.parametrize("q_heads,splits", [(2, 1), (16, 1), (16, 2)])
def test_long_contexts_whose_scores_grow(kind, type_, tpr, q_heads, splits):
    p = Problem(kind, type_, tpr, 1, q_heads, [(12, 1000), (1, 600)], splits=splits)
    grow(p)
    p.run()
    p.check()


@pytest.mark.parametrize("kind,type_,tpr", TYPES)
@pytest.mark.parametrize("bad", [math.inf, -math.inf, math.nan])
@pytest.mark.parametrize("splits", [1, 2])
def test_values_not_seen_by_some_rows_of_a_large_tile(kind, type_, tpr, bad, splits):
    """As in test_values_that_are_not_seen, for row tiles of all waves."""
    (n, t), window, g = (24, 160), 100, 16
    p = Problem(kind, type_, tpr, 1, g, [(n, t)], window=window, splits=splits)
    spoil = [159, 150, 40]
    for tok in spoil:
        page, off = int(p.table[0, tok // tpr]), tok % tpr
        rec = p.pool[page].cpu()
        for name, x in ref.views(kind, type_, tpr, rec).items():
            if name == "scales":
                x[:, off] = bad
            elif x.dtype == torch.float8_e4m3fn:
                x.view(torch.uint8)[:, off] = 0x7F
            else:
                x[:, off] = bad
        p.pool[page] = rec.cuda()
    p.run()
    torch.cuda.synchronize()
    out = p.out.cpu().unflatten(1, (p.H, ref.D_V[kind]))
    seen = ref.visible(n, t, p.k[0].shape[0], True, window)
    clean = ~seen[:, spoil].any(1)
    assert 0 < int(clean.sum()) < n
    rows = torch.arange(n)[clean]
    e = ref.attend(kind, p.k[0][:, 0], p.v[0][:, 0], p.q[rows], seen[clean], p.scale)
    ref.check(kind, out[rows], p.lse.cpu()[rows], e)
    # what sees one is not finite, or is NaN (latent)
    spoiled = out[torch.arange(n)[~clean]].float()
    if kind == L:
        assert bool(torch.isnan(spoiled).all())
    else:
        assert not bool(torch.isfinite(spoiled).all(-1).any())


@pytest.mark.parametrize("kind,type_,tpr", TYPES)
def test_lengths_without_starts(kind, type_, tpr):
    """Every request has as many new tokens, and cached ones of its own; rows behind stay."""
    run(kind, type_, tpr, 2, 4, [(3, 200), (3, 41), (3, 3), (3, 2)], uniform=True, tail=2)


@pytest.mark.parametrize("kind,type_,tpr", TYPES)
def test_starts_without_lengths(kind, type_, tpr):
    """Chunks of their own sizes, each at the end of all its records."""
    p = Problem(kind, type_, tpr, 2, 4, [(3, 8 * tpr), (7, 8 * tpr), (0, 8 * tpr), (1, 8 * tpr)],
                tail=2)
    p.kv_len = None
    p.run()
    p.check()


@pytest.mark.parametrize("kind,type_,tpr", TYPES)
def test_chunk_past_the_longest_is_held(kind, type_, tpr):
    """A chunk start that makes a chunk longer than max_chunk: its first max_chunk rows are worked
    out, as if it ended there, the others stay."""
    p = Problem(kind, type_, tpr, 1, 4, [(5, 100), (2, 64)], tail=6)
    p.start = torch.tensor([0, 11, 13], dtype=torch.int32, device="cuda")
    p.lens = p.lens[:1]
    p.starts = [0, 5]
    p.run()
    torch.cuda.synchronize()
    tail_out, tail_lse = p.out[11:13].clone(), p.lse[11:13].clone()
    p.out[11:13] = MARK
    p.lse[11:13] = MARK
    p.check()
    assert bool(torch.isfinite(tail_out.float()).all()) and not bool((tail_lse == MARK).any())


@pytest.mark.parametrize("kind,type_,tpr", TYPES)
def test_no_new_tokens(kind, type_, tpr):
    """A batch without rows, and one whose requests have none."""
    p = Problem(kind, type_, tpr, 1, 4, [(0, 40), (0, 30), (1, 50)])
    p.chunk.total_tokens = 0
    p.run()
    torch.cuda.synchronize()
    assert bool((p.out == MARK).all())
    p.chunk.total_tokens = 1
    p.start = torch.zeros(4, dtype=torch.int32, device="cuda")
    p.run()
    torch.cuda.synchronize()
    assert bool((p.out == MARK).all()) and bool((p.lse == MARK).all())


@pytest.mark.parametrize("kind,type_,tpr", TYPES)
def test_captured_step_of_writes_and_attention(kind, type_, tpr):
    """One graph that writes a step's rows into the pool and attends to them, replayed with other
    rows, lengths and queries: every replay equals the calls made one by one."""
    R, heads, g, cap = 3, 2, 4, 12 * tpr if tpr > 1 else 200
    pages, (dk, dv) = R * cap // tpr, ref.DIMS[kind]
    rb = hs.hisparse_kv_record_bytes(kind, type_, tpr)
    pool = torch.full((pages, heads, rb), 0xFF, dtype=torch.uint8, device="cuda")
    kv = hs.KvDesc(kind, type_, tpr, rb, pages, heads * rb, rb, 0)
    table = torch.arange(pages, dtype=torch.int32, device="cuda").view(R, -1)
    gen = torch.Generator().manual_seed(7)

    def normal(*shape):
        return torch.randn(shape, generator=gen).to(torch.bfloat16)

    hist_k, hist_v = normal(R, cap, heads, dk), normal(R, cap, heads, dv)
    H, n = heads * g, 2
    scale = 1 / math.sqrt(ref.D_QK[kind])
    c = hs.ChunkDesc(R, heads, g, R * n, n, cap // tpr, H * ref.D_QK[kind], H * ref.D_V[kind],
                     cap // tpr, 0, 0, 0, scale, hs.HISPARSE_CHUNK_CAUSAL)
    ws = torch.empty(hs.hisparse_chunk_workspace_bytes(kv, c), dtype=torch.uint8, device="cuda")
    out = torch.zeros((R * n, H, ref.D_V[kind]), dtype=torch.bfloat16, device="cuda")
    lse = torch.zeros((R * n, H), device="cuda")
    q = torch.zeros((R * n, H, ref.D_QK[kind]), dtype=torch.bfloat16, device="cuda")
    k = torch.zeros((R * n, heads, dk), dtype=torch.bfloat16, device="cuda")
    v = torch.zeros((R * n, heads, dv), dtype=torch.bfloat16, device="cuda")
    slots = torch.zeros(R * n, dtype=torch.int64, device="cuda")
    lens = torch.zeros(R, dtype=torch.int32, device="cuda")

    def write(kk, vv, at, stream):
        hs.hisparse_write_tokens(kv, heads, at.numel(), kk, heads * dk, vv, heads * dv, at, pool,
                                 stream)

    def step(stream):
        write(k, v, slots, stream)
        hs.hisparse_chunk_attention(kv, c, pool, table, None, lens, q, out, lse, ws, ws.numel(),
                                    stream)

    start = [100, 5, 60]
    for r in range(R):
        at = torch.arange(start[r]) + r * cap
        write(hist_k[r, :start[r]].cuda(), hist_v[r, :start[r]].cuda(), at.cuda(),
              torch.cuda.current_stream())
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    before = pool.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        step(side)
    torch.cuda.synchronize()
    assert torch.equal(pool, before)
    sk, sv, _ = ref.stored(kind, hist_k, hist_v, type_)
    for turn in range(4):
        have = [s + n * (turn + 1) for s in start]
        new = torch.stack([torch.arange(t - n, t) for t in have])
        qq = normal(R * n, H, ref.D_QK[kind])
        rows = (torch.arange(R)[:, None], new)
        k.copy_(hist_k[rows].flatten(0, 1))
        v.copy_(hist_v[rows].flatten(0, 1))
        slots.copy_((new + torch.arange(R)[:, None] * cap).flatten())
        lens.copy_(torch.tensor(have, dtype=torch.int32))
        q.copy_(qq)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        got, got_lse, got_pool = out.clone(), lse.clone(), pool.clone()
        for r in range(R):
            seen = ref.visible(n, have[r], have[r], True)
            for h in range(heads):
                mine, hh = slice(r * n, r * n + n), slice(h * g, h * g + g)
                e = ref.attend(kind, sk[r, :have[r], h], sv[r, :have[r], h], qq[mine, hh], seen,
                               scale)
                ref.check(kind, got.cpu()[mine, hh], got_lse.cpu()[mine, hh], e, f"turn {turn}")
        step(torch.cuda.current_stream())
        torch.cuda.synchronize()
        assert torch.equal(out, got) and torch.equal(lse, got_lse) and torch.equal(pool, got_pool)
