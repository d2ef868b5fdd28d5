"""hisparse_write_tokens and hisparse_read_tokens against the 64-bit reference: every stored value,
scale and byte around them is compared exactly (the one rounding, to e4m3 or none, is the
reference's)."""
import math
import zlib

import pytest
import torch

import token_reference as ref
from paper_2608_07009_amd import hisparse as hs

pytestmark = pytest.mark.gpu

G, L = ref.GROUPED, ref.LATENT
BF, F8 = ref.BF16, ref.FP8
SHAPES = [(G, F8, 16), (G, F8, 1), (G, F8, 64), (G, BF, 16), (L, F8, 1), (L, F8, 4), (L, BF, 1)]


def rows(kind, seed, n, heads):
    g = torch.Generator().manual_seed(seed)
    out = []
    for d in ref.DIMS[kind]:
        x = torch.randn((n, heads, d), generator=g)
        x *= torch.exp2(torch.randint(-20, 20, (n, heads, 1), generator=g).float())
        out.append(x.to(torch.bfloat16))
    return out


def desc(kind, type_, tpr, pool):
    """pool [record][head][bytes] on the device"""
    return hs.KvDesc(kind, type_, tpr, pool.shape[2], pool.shape[0], pool.stride(0),
                     pool.stride(1), 0)


def same(a, b):
    a, b = a.double().cpu(), b.double().cpu()
    return torch.equal(torch.isnan(a), torch.isnan(b)) and torch.equal(a.nan_to_num(7.0),
                                                                      b.nan_to_num(7.0))


def write_and_check(kind, type_, tpr, heads, k, v, slots, records, extra=0, wide=None):
    """Writes into a pool of 0xA5 bytes and checks all of it."""
    n = k.shape[0]
    R = hs.hisparse_kv_record_bytes(kind, type_, tpr) + extra
    pool = torch.full((records, heads, R), 0xA5, dtype=torch.uint8, device="cuda")
    kd, vd = (k.cuda(), v.cuda()) if wide is None else wide(k, v)
    hs.hisparse_write_tokens(desc(kind, type_, tpr, pool), heads, n, kd, kd.stride(0), vd,
                             vd.stride(0), None if slots is None else slots.cuda(), pool,
                             torch.cuda.current_stream())
    got = pool.cpu()
    want = torch.full((records, heads, R), 0xA5, dtype=torch.uint8)
    s = torch.arange(n) if slots is None else slots
    ok = (s >= 0) & (s < records * tpr)
    rec, off = s[ok] // tpr, s[ok] % tpr
    p = ref.views(kind, type_, tpr, want)
    rk, rv, sc = ref.stored(kind, k[ok], v[ok], type_)
    if type_ == BF:
        p["rows"][rec, :, off] = torch.cat((k[ok], v[ok]), -1)
    else:
        raw = p["rows"].view(torch.uint8)
        x = rk / sc[..., :1] if kind == L else torch.cat((rk / sc[..., :1], rv / sc[..., 1:]), -1)
        raw[rec, :, off] = x.float().to(torch.float8_e4m3fn).view(torch.uint8)
        if kind == L:
            p["rope"][rec, :, off] = v[ok]
        p["scales"][rec, :, off] = sc.float()
    if bool(torch.isnan(k).any() or torch.isnan(v).any()):  # NaN may carry any sign
        g, w = ref.views(kind, type_, tpr, got), p
        assert all(same(g[name].float(), w[name].float()) for name in w)
    else:
        assert torch.equal(got, want)
    return pool


@pytest.mark.parametrize("kind,type_,tpr", SHAPES)
@pytest.mark.parametrize("heads,n", [(1, 1), (3, 5), (8, 67), (2, 1031)])
def test_write(kind, type_, tpr, heads, n):
    k, v = rows(kind, 7 * n + heads, n, heads)
    g = torch.Generator().manual_seed(n)
    records = (n + tpr - 1) // tpr + 3
    slots = torch.randperm(records * tpr, generator=g)[:n]
    slots[torch.rand(n, generator=g) < 0.1] = -1
    if n > 10:
        slots[3], slots[7] = records * tpr, (1 << 62) + 5  # past the pool: padding as well
    write_and_check(kind, type_, tpr, heads, k, v, slots, records)


@pytest.mark.parametrize("kind,type_,tpr", SHAPES)
def test_write_without_slots_into_larger_records(kind, type_, tpr):
    """Identity slots, records with room behind their tokens, more tokens than the pool holds."""
    k, v = rows(kind, 3, 5 * tpr + 1, 2)
    write_and_check(kind, type_, tpr, 2, k, v, None, 5, extra=16 * tpr)


@pytest.mark.parametrize("kind,type_,tpr", SHAPES)
@pytest.mark.parametrize("lead", [0, 1, 8])
def test_write_from_a_fused_projection(kind, type_, tpr, lead):
    """Rows that are slices of a wider buffer, at any element of it."""
    n, heads = 33, 2
    k, v = rows(kind, 5, n, heads)
    dk, dv = ref.DIMS[kind]

    def wide(k, v):
        w = torch.zeros((n, lead + heads * (dk + dv) + 3), dtype=torch.bfloat16, device="cuda")
        kd = w[:, lead:lead + heads * dk].unflatten(1, (heads, dk))
        vd = w[:, lead + heads * dk:lead + heads * (dk + dv)].unflatten(1, (heads, dv))
        kd.copy_(k)
        vd.copy_(v)
        return kd, vd

    write_and_check(kind, type_, tpr, heads, k, v, None, (n + tpr - 1) // tpr, wide=wide)


def test_write_one_row_to_every_token():
    k, v = rows(G, 9, 1, 2)
    n = 40
    k, v = k.expand(n, 2, 128), v.expand(n, 2, 128)

    def wide(k, v):
        return k[:1].cuda().expand(n, 2, 128), v[:1].cuda().expand(n, 2, 128)

    write_and_check(G, F8, 16, 2, k, v, None, 3, wide=wide)


@pytest.mark.parametrize("kind,type_,tpr", SHAPES)
def test_two_rows_for_one_slot_leave_the_others_alone(kind, type_, tpr):
    n, heads, records = 33, 2, (64 + tpr - 1) // tpr
    k, v = rows(kind, 4, n, heads)
    slots = torch.arange(n) * 61 % 64  # its order shuffled, all different
    twice = torch.cat((slots, slots[5:6]))
    R = hs.hisparse_kv_record_bytes(kind, type_, tpr)
    pools = []
    for s, kk, vv in ((slots, k, v), (twice, torch.cat((k, k[:1])), torch.cat((v, v[:1])))):
        pool = torch.full((records, heads, R), 0xA5, dtype=torch.uint8, device="cuda")
        hs.hisparse_write_tokens(desc(kind, type_, tpr, pool), heads, len(s), kk.cuda(),
                                 kk.stride(0), vv.cuda(), vv.stride(0), s.cuda(), pool,
                                 torch.cuda.current_stream())
        pools.append(ref.views(kind, type_, tpr, pool.cpu()))
    rec, off = int(slots[5]) // tpr, int(slots[5]) % tpr
    for name, a in pools[0].items():
        b = pools[1][name]
        a, b = (x.view(torch.uint8) if x.dtype == torch.float8_e4m3fn else x for x in (a, b))
        a[rec, :, off] = 0
        b[rec, :, off] = 0
        assert torch.equal(a, b)


def special_rows(kind):
    """One token per special case, in both rows."""
    inf, nan, big = math.inf, math.nan, 3.3895e38  # the largest bf16 number
    cases = [[0.0], [-0.0, 1.0], [448.0, 1.0], [449.0, -224.0, 225.0], [inf, 2.0], [-inf, 0.0],
             [nan, 3.0, -5.0], [nan, inf, -inf], [nan], [big, -big, 1.0], [2.0 ** -126], [9.2e-41],
             [2.0 ** -130, -(2.0 ** -120)], [1.0, 2.0 ** -9, 2.0 ** -10, 3 * 2.0 ** -11],
             [17.0, 18.0, 19.0, 25.0, 27.0, 448.0], [1.75, 0.1], [1.7578125, 0.1]]
    out = []
    for d in ref.DIMS[kind]:
        x = torch.zeros((len(cases), 1, d))
        for i, c in enumerate(cases):
            for j in range(d):
                x[i, 0, (j * 37) % d] = c[j % len(c)]
        out.append(x.to(torch.bfloat16))
    return out


@pytest.mark.parametrize("kind,type_,tpr", SHAPES)
def test_special_values(kind, type_, tpr):
    k, v = special_rows(kind)
    n = k.shape[0]
    records = (n + tpr - 1) // tpr
    pool = write_and_check(kind, type_, tpr, 1, k, v, None, records)
    rk, rv, _ = ref.stored(kind, k, v, type_)
    for got, want, dim in zip(read(kind, type_, tpr, pool, torch.arange(n), 1), (rk, rv), "kv"):
        # a value of the last binade may round to 2^128, which bf16 cannot hold
        assert same(got, want.float().to(torch.bfloat16)), dim


def read(kind, type_, tpr, pool, slots, heads):
    n = len(slots)
    out = [torch.full((n, heads, d), 5.0, dtype=torch.bfloat16, device="cuda")
           for d in ref.DIMS[kind]]
    hs.hisparse_read_tokens(desc(kind, type_, tpr, pool), heads, n, pool, slots.cuda(), out[0],
                            out[0].stride(0), out[1], out[1].stride(0),
                            torch.cuda.current_stream())
    return out


@pytest.mark.parametrize("kind,type_,tpr", SHAPES)
@pytest.mark.parametrize("heads,n", [(1, 1), (3, 77), (8, 500)])
def test_read(kind, type_, tpr, heads, n):
    """Slots in any order, repeated, missing; written again, the rows give the same bytes."""
    g = torch.Generator().manual_seed(zlib.crc32(f"{kind}{type_}{tpr}{n}".encode()))
    records = n // tpr + 2
    k, v = rows(kind, n, records * tpr, heads)
    pool = write_and_check(kind, type_, tpr, heads, k, v, None, records)
    slots = torch.randint(0, records * tpr, (n,), generator=g)
    slots[torch.rand(n, generator=g) < 0.1] = -3
    if n > 5:
        slots[2] = records * tpr
    gk, gv = read(kind, type_, tpr, pool, slots, heads)
    rk, rv = (x.transpose(1, 2).flatten(0, 1) for x in ref.rows_of(kind, type_, tpr, pool.cpu()))
    ok = ((slots >= 0) & (slots < records * tpr))[:, None, None]
    at = slots.clamp(0, records * tpr - 1)
    assert same(gk, torch.where(ok, rk[at], 0.0)) and same(gv, torch.where(ok, rv[at], 0.0))
    allk, allv = read(kind, type_, tpr, pool, torch.arange(records * tpr), heads)
    again = torch.full_like(pool, 0xA5)
    hs.hisparse_write_tokens(desc(kind, type_, tpr, again), heads, records * tpr, allk,
                             allk.stride(0), allv, allv.stride(0), None, again,
                             torch.cuda.current_stream())
    a2, b2 = (x.cpu() for x in read(kind, type_, tpr, again, torch.arange(records * tpr), heads))
    assert torch.equal(a2, allk.cpu()) and torch.equal(b2, allv.cpu())


def test_read_into_strided_rows_leaves_the_rest():
    k, v = rows(G, 1, 40, 2)
    pool = write_and_check(G, F8, 16, 2, k, v, None, 3)
    wide = torch.full((40, 700), 9.0, dtype=torch.bfloat16, device="cuda")
    kd, vd = wide[:, 3:259], wide[:, 301:557]
    hs.hisparse_read_tokens(desc(G, F8, 16, pool), 2, 40, pool, None, kd, 700, vd, 700,
                            torch.cuda.current_stream())
    rk, rv, _ = ref.stored(G, k, v, F8)
    w = wide.cpu()
    assert same(w[:, 3:259], rk.flatten(1)) and same(w[:, 301:557], rv.flatten(1))
    w[:, 3:259] = 9.0
    w[:, 301:557] = 9.0
    assert bool((w == 9.0).all())


def test_slots_beyond_four_gib():
    """Records, heads and slots whose byte offsets pass 32 bits."""
    n, stride = 5, 1 << 28
    pool = torch.zeros(n * stride * 4 + (1 << 16), dtype=torch.uint8, device="cuda")
    d = hs.KvDesc(G, F8, 16, 4224, 4 * n, stride, 1 << 15, 0)
    k, v = rows(G, 4, 7, 2)
    slots = torch.tensor([19 * 16 + 3, 18 * 16, 17 * 16 + 15, 0, 20 * 16, 16 * 16 + 1, 5])
    s = torch.cuda.current_stream()
    hs.hisparse_write_tokens(d, 2, 7, k.cuda(), 256, v.cuda(), 256, slots.cuda(), pool, s)
    for i, sl in enumerate(slots.tolist()):
        if sl == 20 * 16:
            continue
        for h in range(2):
            at = (sl // 16) * stride + h * (1 << 15)
            kk, vv = ref.rows_of(G, F8, 16, pool[at:at + 4224].cpu())
            rk, rv, _ = ref.stored(G, k[i, h], v[i, h], F8)
            assert same(kk[sl % 16], rk) and same(vv[sl % 16], rv)
    ok, ov = (torch.zeros((7, 2, 128), dtype=torch.bfloat16, device="cuda") for _ in "kv")
    hs.hisparse_read_tokens(d, 2, 7, pool, slots.cuda(), ok, 256, ov, 256, s)
    rk, rv, _ = ref.stored(G, k, v, F8)
    rk[4] = rv[4] = 0.0
    assert same(ok, rk) and same(ov, rv)


def test_captured_write_and_read_replay():
    """Both calls captured on another stream; every replay against fresh inputs."""
    kind, type_, tpr, heads, n = G, F8, 16, 4, 50
    kd, vd = (x.cuda() for x in rows(kind, 1, n, heads))
    slots = torch.randperm(64).cuda()[:n].contiguous()
    pool = torch.zeros((4, heads, hs.hisparse_kv_record_bytes(kind, type_, tpr)),
                       dtype=torch.uint8, device="cuda")
    ok, ov = torch.zeros_like(kd), torch.zeros_like(vd)
    d = desc(kind, type_, tpr, pool)
    stream = torch.cuda.Stream()

    def both(s):
        hs.hisparse_write_tokens(d, heads, n, kd, kd.stride(0), vd, vd.stride(0), slots, pool, s)
        hs.hisparse_read_tokens(d, heads, n, pool, slots, ok, ok.stride(0), ov, ov.stride(0), s)

    stream.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        both(stream)
    for seed in range(4):
        k, v = rows(kind, 100 + seed, n, heads)
        kd.copy_(k)
        vd.copy_(v)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        rk, rv, _ = ref.stored(kind, k, v, type_)
        assert same(ok, rk) and same(ov, rv)
        ok.zero_()


@pytest.mark.parametrize("kind,type_,tpr", [(G, F8, 16), (L, F8, 1)])
def test_the_last_binade_reads_back_finite_or_as_infinity(kind, type_, tpr):
    """Of values next to the largest bf16 number, those that round below 2^128 come back, the others as
    infinities; a part of up to 448 * 2^119 has none."""
    unit = 2.0 ** 120
    cases = [[224.0, 100.0, -224.0], [225.0, 224.0, 1.0], [247.0, -247.0, 232.0], [248.0, 247.0, -64.0],
             [255.0, -248.0, 3.0], [math.inf, 224.0, -math.inf], [math.inf, 225.0, 8.0]]
    want = [[224.0, 96.0, -224.0], [224.0, 224.0, 1.0], [240.0, -240.0, 224.0],
            [math.inf, 240.0, -64.0], [math.inf, -math.inf, 3.0], [224.0, 224.0, -224.0],
            [math.inf, 224.0, 8.0]]
    n = len(cases)
    rows_, back = [], []
    for d in ref.DIMS[kind]:
        at = [c % 3 for c in range(d)]
        rows_.append((torch.tensor(cases).double()[:, at] * unit).to(torch.bfloat16)[:, None])
        back.append((torch.tensor(want).double()[:, at] * unit).to(torch.bfloat16)[:, None])
    pool = write_and_check(kind, type_, tpr, 1, *rows_, None, (n + tpr - 1) // tpr)
    got = read(kind, type_, tpr, pool, torch.arange(n), 1)
    assert same(got[0], back[0])
    assert same(got[1], back[1] if kind == G else rows_[1])  # rotary dims keep their bits
