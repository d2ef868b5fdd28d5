"""hisparse_chunk_attention against 64-bit attention; tolerances by the roundings that the call
makes (token_reference.check). Bytes that no token owns (page ends, unused records, padding) hold
NaN, rows that must not be written hold a mark."""
import math
import zlib

import pytest
import torch

import token_reference as ref
from paper_2608_07009_amd import HiSparseCache, hisparse as hs

pytestmark = pytest.mark.gpu

G, L = ref.GROUPED, ref.LATENT
BF, F8 = ref.BF16, ref.FP8
MARK = 12345.0


class Problem:
    """lens: (new, cached) tokens of each request. Pages of all heads [page][head] in a shuffled
    order, a block table per request."""

    def __init__(self, kind, type_, tpr, kv_heads, q_heads, lens, causal=True, window=0, tail=0,
                 splits=0, seed=0, scale=None, uniform=False, q_gap=0, out_gap=0, holes=False,
                 sharpen=1.0):
        self.__dict__.update(kind=kind, type_=type_, tpr=tpr, kv_heads=kv_heads, q_heads=q_heads,
                             lens=lens, causal=causal, window=window, uniform=uniform)
        g = torch.Generator().manual_seed(seed + zlib.crc32(repr((kind, type_, tpr, lens)).encode()))
        R, H = len(lens), kv_heads * q_heads
        self.H = H
        dk, dv = ref.DIMS[kind]
        self.scale = scale or 1.0 / math.sqrt(ref.D_QK[kind])
        cap = max(1, max((t + tpr - 1) // tpr for _, t in lens))
        self.k, self.v, self.hole = [], [], []
        n_pages = R * cap + 3
        rb = hs.hisparse_kv_record_bytes(kind, type_, tpr)
        pool = torch.full((n_pages, kv_heads, rb), 0xFF, dtype=torch.uint8)  # NaN everywhere
        order = torch.randperm(n_pages, generator=g)
        table = torch.full((R, cap), -1, dtype=torch.int32)
        for r, (n, t) in enumerate(lens):
            pages = (t + tpr - 1) // tpr
            k = (sharpen * torch.randn((pages * tpr, kv_heads, dk), generator=g)).to(torch.bfloat16)
            v = torch.randn((pages * tpr, kv_heads, dv), generator=g).to(torch.bfloat16)
            if pages:
                kk = k.unflatten(0, (pages, tpr)).transpose(1, 2)
                vv = v.unflatten(0, (pages, tpr)).transpose(1, 2)
                rec = ref.make_pool(kind, type_, tpr, kk, vv)
                parts = ref.views(kind, type_, tpr, rec)
                for p in parts.values():  # the last page's end holds NaN
                    e = p.view(torch.uint8) if p.dtype == torch.float8_e4m3fn else p
                    if t % tpr:
                        e[-1, :, t % tpr:] = 255 if e.dtype == torch.uint8 else math.nan
                mine = order[r * cap:r * cap + pages]
                pool[mine] = rec
                table[r, :pages] = mine.int()
            sk, sv, _ = ref.stored(kind, k, v, type_)
            hole = torch.zeros(pages * tpr, dtype=torch.bool)
            if holes:
                for j in range(pages):
                    if (j * 7 + r) % 3 == 0:
                        table[r, j] = (-1, n_pages, -5)[j % 3]
                        hole[j * tpr:(j + 1) * tpr] = True
            self.k.append(sk)
            self.v.append(sv)
            self.hole.append(hole)
        total = sum(n for n, _ in lens) + tail
        self.total, self.cap = total, cap
        q = torch.randn((total, H * ref.D_QK[kind] + q_gap), generator=g).to(torch.bfloat16)
        self.q = q[:, q_gap:].unflatten(1, (H, ref.D_QK[kind]))
        self.qd = q.cuda()[:, q_gap:]
        self.pool, self.table = pool.cuda(), table.cuda()
        starts = [0]
        for n, _ in lens:
            starts.append(starts[-1] + n)
        self.starts = starts
        self.start = None if uniform else torch.tensor(starts, dtype=torch.int32, device="cuda")
        self.kv_len = torch.tensor([t for _, t in lens], dtype=torch.int32, device="cuda")
        self.kv = hs.KvDesc(kind, type_, tpr, rb, n_pages, kv_heads * rb, rb, 0)
        D = H * ref.D_V[kind]
        self.chunk = hs.ChunkDesc(R, kv_heads, q_heads, total, max(n for n, _ in lens), cap,
                                  self.qd.stride(0), D + out_gap, cap, 0, window, splits,
                                  self.scale, hs.HISPARSE_CHUNK_CAUSAL if causal else 0)
        self.out = torch.full((total, D + out_gap), MARK, dtype=torch.bfloat16, device="cuda")
        self.lse = torch.full((total, H), MARK, dtype=torch.float32, device="cuda")
        n = hs.hisparse_chunk_workspace_bytes(self.kv, self.chunk)
        self.ws = torch.full((n + 64,), 0xFF, dtype=torch.uint8, device="cuda")
        self.ws_bytes = n
        self.out_gap = out_gap

    def run(self, stream=None, lse=True):
        hs.hisparse_chunk_attention(self.kv, self.chunk, self.pool, self.table, self.start,
                                    self.kv_len, self.qd, self.out, self.lse if lse else None,
                                    self.ws, self.ws_bytes,
                                    stream or torch.cuda.current_stream())

    def check(self, what="", lse=True):
        torch.cuda.synchronize()
        assert bool((self.ws[self.ws_bytes:] == 0xFF).all()), "wrote past the workspace"
        D, d_v, g = self.H * ref.D_V[self.kind], ref.D_V[self.kind], self.q_heads
        out, got_lse = self.out.cpu(), self.lse.cpu()
        if self.out_gap:
            assert bool((out[:, D:] == torch.tensor(MARK).to(torch.bfloat16)).all())
        out = out[:, :D].unflatten(1, (self.H, d_v))
        for r, (n, t) in enumerate(self.lens):
            rows = slice(self.starts[r], self.starts[r] + n)
            seen = ref.visible(n, t, self.k[r].shape[0], self.causal, self.window)
            seen = seen & ~self.hole[r][None]
            for h in range(self.kv_heads):
                heads = slice(h * g, (h + 1) * g)
                e = ref.attend(self.kind, self.k[r][:, h], self.v[r][:, h], self.q[rows, heads],
                               seen, self.scale)
                ref.check(self.kind, out[rows, heads], got_lse[rows, heads] if lse else None, e,
                          f"{what} request {r} head {h}")
        mark = torch.tensor(MARK)
        assert bool((out[self.starts[-1]:] == mark.to(torch.bfloat16)).all())
        assert bool((got_lse[self.starts[-1]:] == mark).all())
        if not lse:
            assert bool((got_lse == mark).all())


def run(*a, **kw):
    p = Problem(*a, **kw)
    p.run()
    p.check()
    return p


TYPES = [(G, BF, 16), (G, F8, 16), (L, BF, 1), (L, F8, 1)]


@pytest.mark.parametrize("kind,type_,tpr", TYPES)
@pytest.mark.parametrize("lens", [
    [(1, 1)], [(1, 2)], [(1, 31)], [(1, 32)], [(1, 33)], [(1, 64)], [(1, 65)], [(1, 300)],
    [(2, 2)], [(3, 70)], [(5, 5)], [(17, 40)], [(33, 33)], [(64, 129)], [(100, 130)]])
def test_lengths(kind, type_, tpr, lens):
    """One request, from one cached token on, around every tile border."""
    run(kind, type_, tpr, 1, 4, lens)


@pytest.mark.parametrize("kind,type_,tpr", [(G, BF, 1), (G, BF, 4), (G, BF, 64), (G, F8, 1),
                                            (G, F8, 2), (G, F8, 32), (G, F8, 64), (G, F8, 256),
                                            (L, BF, 16), (L, BF, 64), (L, F8, 2), (L, F8, 16),
                                            (L, F8, 64)])
def test_pages(kind, type_, tpr):
    """Page sizes that end inside a tile, fill it, and span many."""
    run(kind, type_, tpr, 2, 3, [(3, 150), (1, 64), (2, 17)])


@pytest.mark.parametrize("kind,type_,tpr", TYPES)
@pytest.mark.parametrize("kv_heads,q_heads", [(1, 1), (2, 2), (1, 7), (3, 16), (1, 31), (2, 33),
                                              (1, 128), (1, 130), (1, 256)])
def test_heads(kind, type_, tpr, kv_heads, q_heads):
    run(kind, type_, tpr, kv_heads, q_heads, [(2, 50), (1, 90)])


RAGGED = [(40, 200), (1, 1), (1, 257), (0, 30), (7, 3), (3, 0), (2, 2), (65, 65), (1, 130)]


@pytest.mark.parametrize("kind,type_,tpr", TYPES)
@pytest.mark.parametrize("splits", [0, 1, 3, 64])
def test_ragged_batch(kind, type_, tpr, splits):
    """Decoding requests beside chunks of prompts; a request without new tokens, without cached
    ones, and with fewer cached than new ones (rows that see nothing); rows behind the last."""
    run(kind, type_, tpr, 2, 5, RAGGED, tail=11, splits=splits)


@pytest.mark.parametrize("kind,type_,tpr", TYPES)
@pytest.mark.parametrize("window", [1, 2, 16, 33, 64, 1000])
def test_window(kind, type_, tpr, window):
    run(kind, type_, tpr, 1, 4, [(40, 200), (1, 180), (7, 3), (130, 130)], window=window)


@pytest.mark.parametrize("kind,type_,tpr", TYPES)
@pytest.mark.parametrize("splits", [0, 1, 2])
def test_without_causal_mask(kind, type_, tpr, splits):
    run(kind, type_, tpr, 2, 4, [(3, 70), (1, 129), (5, 2)], causal=False, splits=splits)


@pytest.mark.parametrize("kind,type_,tpr", TYPES)
@pytest.mark.parametrize("causal", [True, False])
def test_padding_records(kind, type_, tpr, causal):
    """Table entries below zero and past the pool; a request all of whose records are padding."""
    run(kind, type_, tpr, 2, 4, [(9, 150), (1, 140), (1, tpr), (20, 21)], holes=True,
        causal=causal)


@pytest.mark.parametrize("kind,type_,tpr", TYPES)
def test_uniform_chunks(kind, type_, tpr):
    """No chunk starts: every request has as many new tokens; no lengths: all its records."""
    p = Problem(kind, type_, tpr, 2, 4, [(3, 8 * tpr)] * 4, uniform=True)
    p.kv_len = None
    p.run()
    p.check()


@pytest.mark.parametrize("kind,type_,tpr", TYPES)
def test_strides_and_no_lse(kind, type_, tpr):
    """Queries and outputs inside wider rows, queries at an odd element."""
    p = Problem(kind, type_, tpr, 2, 3, [(5, 77), (1, 40)], q_gap=3, out_gap=5)
    p.run(lse=False)
    p.check(lse=False)


@pytest.mark.parametrize("kind,type_,tpr", TYPES)
def test_sharp_scores(kind, type_, tpr):
    """Scores that spread over hundreds and change their maximum from tile to tile."""
    run(kind, type_, tpr, 1, 8, [(70, 400), (1, 500)], sharpen=30.0)


@pytest.mark.parametrize("kind,type_,tpr", TYPES)
def test_scores_that_grow(kind, type_, tpr):
    """Each cached token's score above the last one's by more than any slack."""
    p = Problem(kind, type_, tpr, 1, 4, [(20, 200), (1, 260)])
    grow(p)
    p.run()
    p.check()


def grow(p):
    """Replaces every request's keys by one direction times its place."""
    for r, (n, t) in enumerate(p.lens):
        for h in range(p.kv_heads):
            T = p.k[r].shape[0]
            k = torch.zeros((T, ref.DIMS[p.kind][0]))
            k[:, :64] = (torch.arange(T)[:, None] * 0.5)
            v = p.v[r][:, h].float().to(torch.bfloat16) if p.type_ == BF else \
                torch.randn((T, ref.DIMS[p.kind][1]), generator=torch.Generator().manual_seed(r)
                            ).to(torch.bfloat16)
            kk, vv = (x.to(torch.bfloat16).unflatten(0, (T // p.tpr, p.tpr)) for x in (k, v))
            rec = ref.make_pool(p.kind, p.type_, p.tpr, kk, vv)
            p.pool[p.table[r, :T // p.tpr].long(), h] = rec.cuda()
            sk, sv, _ = ref.stored(p.kind, k.to(torch.bfloat16), v, p.type_)
            p.k[r][:, h], p.v[r][:, h] = sk, sv
    p.q[..., :64] = p.q[..., :64].abs()
    p.qd.copy_(p.q.flatten(1))


@pytest.mark.parametrize("kind,type_,tpr", TYPES)
@pytest.mark.parametrize("bad", [math.inf, -math.inf, math.nan])
def test_values_that_are_not_seen(kind, type_, tpr, bad):
    """Infinities and NaN in the K and V of later tokens, of tokens before the window and of
    nobody's records: no row that does not see them changes. Rows that see one are not compared."""
    lens, window = [(40, 100), (1, 90)], 50
    p = Problem(kind, type_, tpr, 2, 4, lens, window=window)
    spoil = {0: [99, 70, 5], 1: [2, 39]}
    for r, toks in spoil.items():
        for t in toks:
            page, off = int(p.table[r, t // tpr]), t % tpr
            rec = p.pool[page].cpu()
            parts = ref.views(kind, type_, tpr, rec)
            for name, x in parts.items():
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
    for r, (n, t) in enumerate(lens):
        seen = ref.visible(n, t, p.k[r].shape[0], True, window)
        clean = ~seen[:, spoil[r]].any(1)
        assert bool(clean.any())
        rows = torch.arange(p.starts[r], p.starts[r] + n)[clean]
        for h in range(2):
            e = ref.attend(kind, p.k[r][:, h], p.v[r][:, h], p.q[rows, h * 4:h * 4 + 4],
                           seen[clean], p.scale)
            ref.check(kind, out[rows, h * 4:h * 4 + 4], p.lse.cpu()[rows, h * 4:h * 4 + 4], e)


@pytest.mark.parametrize("kind,type_,tpr", TYPES)
def test_lengths_out_of_range_are_held(kind, type_, tpr):
    """Cached lengths past the table and below zero, chunk starts past the rows: held to the
    arrays, not read past them."""
    p = Problem(kind, type_, tpr, 1, 4, [(4, 64), (3, 64), (2, 64)], tail=2)
    p.kv_len = torch.tensor([10 ** 9, 64, 64], dtype=torch.int32, device="cuda")
    p.start = torch.tensor([0, 4, 7, 9], dtype=torch.int32, device="cuda")
    if p.cap * tpr == 64:
        p.run()
        p.check()
    p.kv_len = torch.tensor([-7, 64, 64], dtype=torch.int32, device="cuda")
    p.start = torch.tensor([-5, 4, 7, 10 ** 9], dtype=torch.int32, device="cuda")
    p.out.fill_(MARK)
    p.run()
    torch.cuda.synchronize()
    assert bool((p.out[:4] == 0).all()) and bool(torch.isinf(p.lse[:4]).all())


@pytest.mark.parametrize("kind,type_", [(G, BF), (G, F8), (L, BF), (L, F8)])
def test_records_beyond_four_gib(kind, type_):
    """Records and heads whose byte offsets pass 32 bits."""
    p = Problem(kind, type_, 1, 2, 4, [(2, 40), (1, 23)])
    rb, n, far = p.kv.record_bytes, p.kv.num_records, 1 << 27
    pool = torch.full((n * far + (1 << 26) + rb,), 0xFF, dtype=torch.uint8, device="cuda")
    for r in range(n):
        for h in range(2):
            at = r * far + h * (1 << 26)
            pool[at:at + rb] = p.pool[r, h]
    p.pool = pool
    p.kv = hs.KvDesc(kind, type_, 1, rb, n, far, 1 << 26, 0)
    p.run()
    p.check()


def slots_problem(kind, type_, tpr, requests, kv_heads, q_heads, k, B, seed=1):
    """Slot caches [request][head][B] and a slot vector per unit with padding entries."""
    g = torch.Generator().manual_seed(seed)
    dk, dv = ref.DIMS[kind]
    kk = torch.randn((requests, kv_heads, B, tpr, dk), generator=g).to(torch.bfloat16)
    vv = torch.randn((requests, kv_heads, B, tpr, dv), generator=g).to(torch.bfloat16)
    pool = ref.make_pool(kind, type_, tpr, kk, vv)
    idx = torch.stack([torch.randperm(B, generator=g)[:k] for _ in range(requests * kv_heads)])
    idx = idx.view(requests, kv_heads, k).int()
    idx[torch.rand(idx.shape, generator=g) < 0.15] = -1
    idx[0, 0] = -1  # a unit without a record
    q = torch.randn((requests, kv_heads * q_heads, ref.D_QK[kind]), generator=g).to(torch.bfloat16)
    return kk, vv, pool, idx, q


@pytest.mark.parametrize("kind,type_,tpr,requests,kv_heads,q_heads,k,B", [
    (G, F8, 16, 3, 2, 4, 9, 12), (G, BF, 16, 2, 3, 5, 7, 8), (G, F8, 64, 1, 2, 16, 3, 5),
    (L, F8, 1, 3, 1, 16, 130, 200), (L, F8, 1, 2, 1, 128, 301, 400), (L, BF, 1, 2, 1, 40, 77, 90),
    (L, F8, 1, 1, 1, 1, 1, 1)])
def test_selected_records(kind, type_, tpr, requests, kv_heads, q_heads, k, B):
    """Sparse decode: one new token per request over the records of a slot vector per unit."""
    kk, vv, pool, idx, q = slots_problem(kind, type_, tpr, requests, kv_heads, q_heads, k, B)
    pool_d, idx_d, q_d = pool.cuda(), idx.cuda(), q.cuda()
    rb = pool.shape[-1]
    kv = hs.KvDesc(kind, type_, tpr, rb, B, rb, B * rb, kv_heads * B * rb)
    H, scale = kv_heads * q_heads, 0.07
    c = hs.ChunkDesc(requests, kv_heads, q_heads, requests, 1, k, H * ref.D_QK[kind],
                     H * ref.D_V[kind], kv_heads * k, k, 0, 0, scale, 0)
    out = torch.empty((requests, H, ref.D_V[kind]), dtype=torch.bfloat16, device="cuda")
    lse = torch.empty((requests, H), device="cuda")
    ws = torch.empty(hs.hisparse_chunk_workspace_bytes(kv, c), dtype=torch.uint8, device="cuda")
    hs.hisparse_chunk_attention(kv, c, pool_d, idx_d, None, None, q_d, out, lse, ws, ws.numel(),
                                torch.cuda.current_stream())
    for r in range(requests):
        for h in range(kv_heads):
            s = idx[r, h].long()
            seen = (s >= 0).repeat_interleave(tpr)[None]
            s = s.clamp(min=0)
            sk, sv, _ = ref.stored(kind, kk[r, h][s].flatten(0, 1), vv[r, h][s].flatten(0, 1),
                                   type_)
            heads = slice(h * q_heads, (h + 1) * q_heads)
            e = ref.attend(kind, sk, sv, q[r:r + 1, heads], seen, scale)
            ref.check(kind, out[r:r + 1, heads], lse[r:r + 1, heads], e, f"unit {r},{h}")


@pytest.mark.parametrize("kind,type_,tpr", TYPES)
@pytest.mark.parametrize("splits", [1, 4])
def test_placement_changes_nothing(kind, type_, tpr, splits):
    """The same records elsewhere in the pool: the same bits."""
    p = Problem(kind, type_, tpr, 2, 6, [(3, 170), (1, 99)], splits=splits)
    p.run()
    a, la = p.out.clone(), p.lse.clone()
    perm = torch.randperm(p.pool.shape[0], generator=torch.Generator().manual_seed(4)).cuda()
    moved = torch.empty_like(p.pool)
    moved[perm] = p.pool
    t = p.table.long()
    p.table = torch.where(t >= 0, perm[t.clamp(min=0)], t).int()
    p.pool = moved
    p.run()
    assert torch.equal(p.out, a) and torch.equal(p.lse, la)
    p.check()


@pytest.mark.parametrize("kind,type_,tpr", TYPES)
def test_two_streams_and_replays(kind, type_, tpr):
    """Two calls at once on streams of their own, and two captured graphs with a workspace each,
    replayed with other queries in between: all equal to calls alone."""
    a = Problem(kind, type_, tpr, 2, 4, [(5, 300), (1, 200)], splits=3)
    b = Problem(kind, type_, tpr, 1, 8, [(2, 400)], splits=4, seed=5)
    s1, s2 = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    a.run(s1)
    b.run(s2)
    a.check("stream 1")
    b.check("stream 2")
    graphs = []
    for p, s in ((a, s1), (b, s2)):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            p.run(s)
        graphs.append(g)
    for turn in range(3):
        for p in (a, b):
            p.qd.mul_(-1 if turn % 2 else 0.5)
            p.q = p.qd.cpu().unflatten(1, (p.H, ref.D_QK[kind]))
            p.out.fill_(MARK)
            p.lse.fill_(MARK)
        torch.cuda.synchronize()
        for g in graphs:
            g.replay()
        a.check(f"replay {turn} a")
        b.check(f"replay {turn} b")
        out, lse = a.out.clone(), a.lse.clone()
        a.run()
        torch.cuda.synchronize()
        assert torch.equal(out, a.out) and torch.equal(lse, a.lse)


@pytest.mark.parametrize("kind,type_,tpr", TYPES)
def test_workspace_too_small_is_refused(kind, type_, tpr):
    p = Problem(kind, type_, tpr, 1, 4, [(1, 600)], splits=4)
    if p.ws_bytes:
        with pytest.raises(hs.HisparseError) as e:
            hs.hisparse_chunk_attention(p.kv, p.chunk, p.pool, p.table, p.start, p.kv_len, p.qd,
                                        p.out, p.lse, p.ws, p.ws_bytes - 1)
        assert e.value.status == hs.HISPARSE_ERR_INVALID_ARG
    p.run()
    p.check()


@pytest.mark.parametrize("kind,tpr,heads,q_heads", [(G, 16, 2, 4), (L, 1, 1, 16)])
def test_serving_with_eight_bit_records(kind, tpr, heads, q_heads):
    """The calls together, as a server uses them: a prompt's rows written as 8-bit records into a
    device buffer and staged to the host pool, the prompt's last chunk attending to them; decode
    steps that append a written record, resolve a selection, fetch its misses and attend to the
    slots; the rows read back."""
    type_, L_, B, k, req = F8, 24, 10, 5, 2
    rb = hs.hisparse_kv_record_bytes(kind, type_, tpr)
    dk, dv = ref.DIMS[kind]
    g = torch.Generator().manual_seed(3)
    n = (L_ - 4) * tpr  # prompt tokens of each request
    k_rows = torch.randn((req, L_ * tpr, heads, dk), generator=g).to(torch.bfloat16)
    v_rows = torch.randn((req, L_ * tpr, heads, dv), generator=g).to(torch.bfloat16)
    sk, sv, _ = ref.stored(kind, k_rows, v_rows, type_)
    H, scale = heads * q_heads, 1 / math.sqrt(ref.D_QK[kind])
    s = torch.cuda.current_stream()
    with HiSparseCache(num_requests=req, num_layers=1, units_per_request=heads, capacity=B,
                       num_records=L_, top_k=k, record_bytes=rb) as cache:
        full = torch.zeros((req, heads, L_, rb), dtype=torch.uint8, device="cuda")
        kv_full = cache.kv_desc(kind, type_, tpr, host_pool=True)
        # the units' parts one after the other: request q's record r is record q * m + r
        one = hs.KvDesc(kind, type_, tpr, rb, (req - 1) * heads * L_ + L_, rb, L_ * rb, 0)
        slots = (torch.arange(req)[:, None] * heads * L_ * tpr + torch.arange(n)[None]).flatten()
        hs.hisparse_write_tokens(one, heads, req * n, k_rows[:, :n].flatten(0, 1).cuda(),
                                 heads * dk, v_rows[:, :n].flatten(0, 1).cuda(), heads * dv,
                                 slots.cuda(), full, s)
        hs.hisparse_stage(cache.handle, 0, 1, 0, req * heads, 0, L_, full, 0, s)
        # the prompt's last chunk over the records, per-unit identity tables
        c_new = 7
        q = torch.randn((req * c_new, H, ref.D_QK[kind]), generator=g).to(torch.bfloat16)
        ident = torch.arange(L_, dtype=torch.int32, device="cuda")
        chunk = hs.ChunkDesc(req, heads, q_heads, req * c_new, c_new, L_, H * ref.D_QK[kind],
                             H * ref.D_V[kind], 0, 0, 0, 0, scale, hs.HISPARSE_CHUNK_CAUSAL)
        out = torch.zeros((req * c_new, H, ref.D_V[kind]), dtype=torch.bfloat16, device="cuda")
        ws = torch.empty(hs.hisparse_chunk_workspace_bytes(kv_full, chunk), dtype=torch.uint8,
                         device="cuda")
        lens = torch.full((req,), n, dtype=torch.int32, device="cuda")
        hs.hisparse_chunk_attention(kv_full, chunk, full, ident, None, lens, q.cuda(), out, None,
                                    ws, ws.numel(), s)
        seen = ref.visible(c_new, n, n, True)
        for r in range(req):
            for h in range(heads):
                hh = slice(h * q_heads, (h + 1) * q_heads)
                rows = slice(r * c_new, (r + 1) * c_new)
                e = ref.attend(kind, sk[r, :n, h], sv[r, :n, h], q[rows, hh], seen, scale)
                ref.check(kind, out[rows, hh], None, e, f"chunk {r},{h}")
        # decode steps over the slot cache
        kv_cache = cache.kv_desc(kind, type_, tpr)
        dec = hs.ChunkDesc(req, heads, q_heads, req, 1, k, H * ref.D_QK[kind], H * ref.D_V[kind],
                           heads * k, k, 0, 0, scale, 0)
        ws2 = torch.empty(hs.hisparse_chunk_workspace_bytes(kv_cache, dec), dtype=torch.uint8,
                          device="cuda")
        kv_new = hs.KvDesc(kind, type_, tpr, rb, req * heads, rb, rb, 0)
        out1 = torch.zeros((req, H, ref.D_V[kind]), dtype=torch.bfloat16, device="cuda")
        for step in range(4):
            rec = L_ - 4 + step
            toks = slice(rec * tpr, (rec + 1) * tpr)
            # one new record per unit: its tokens' rows, requests one behind the other
            new = torch.zeros((1, req, heads, rb), dtype=torch.uint8, device="cuda")
            at = (torch.arange(req)[:, None] * heads * tpr + torch.arange(tpr)[None]).flatten()
            hs.hisparse_write_tokens(kv_new, heads, req * tpr,
                                     k_rows[:, toks].flatten(0, 1).cuda(), heads * dk,
                                     v_rows[:, toks].flatten(0, 1).cuda(), heads * dv, at.cuda(),
                                     new, s)
            pos = torch.full((req * heads,), rec, dtype=torch.int32, device="cuda")
            new_slots = torch.empty((1, req * heads), dtype=torch.int32, device="cuda")
            hs.hisparse_append(cache.handle, 0, 1, pos, new, new_slots, s)
            sel = torch.stack([torch.randperm(rec + 1, generator=g)[:k]
                               for _ in range(req * heads)]).int()
            sel[0, 2] = -1
            slots_d = torch.empty((req * heads, k), dtype=torch.int32, device="cuda")
            hs.hisparse_resolve(cache.handle, 0, sel.cuda(), slots_d, None, s)
            q = torch.randn((req, H, ref.D_QK[kind]), generator=g).to(torch.bfloat16)
            hs.hisparse_chunk_attention(kv_cache, dec, cache.layer_cache(0)[0], slots_d, None,
                                        None, q.cuda(), out1, None, ws2, ws2.numel(), s)
            for r in range(req):
                for h in range(heads):
                    ids = sel[r * heads + h].long()
                    ids = ids[ids >= 0]
                    tk = (ids[:, None] * tpr + torch.arange(tpr)[None]).flatten()
                    hh = slice(h * q_heads, (h + 1) * q_heads)
                    e = ref.attend(kind, sk[r, tk, h], sv[r, tk, h], q[r:r + 1, hh],
                                   torch.ones((1, len(tk)), dtype=torch.bool), scale)
                    ref.check(kind, out1[r:r + 1, hh], None, e, f"step {step} unit {r},{h}")
            assert cache.check_errors()[0] == hs.HISPARSE_OK
        got_k = torch.zeros((n, heads, dk), dtype=torch.bfloat16, device="cuda")
        got_v = torch.zeros((n, heads, dv), dtype=torch.bfloat16, device="cuda")
        hs.hisparse_read_tokens(one, heads, n, full, None, got_k, heads * dk, got_v, heads * dv, s)
        assert torch.equal(got_k.cpu().double(), sk[0, :n])
        assert torch.equal(got_v.cpu().double(), sv[0, :n])
