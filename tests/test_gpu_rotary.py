"""hisparse_rotate_tokens against 64-bit arithmetic.

Tolerance: the result is rounded to bf16 once, half a step of 2^-7 at most: 2^-8 of the value. Before it, in
fp32: the angle as a fraction of a turn (2^-25 of at most half a turn, 2 pi times that in radians), cosine
and sine (4 units of 2^-24 allowed), the magnitude and its product, a product each and their sum: together
below 16 * 2^-24 of |a| + |b|, taken as 2^-20. The angle's own error in 64 bits is 2^-52 of the turns made,
below 2^-21 at position 2^31."""
import math

import pytest
import torch

import step_reference as ref
from paper_2608_07009_amd import hisparse as hs

pytestmark = pytest.mark.gpu
HALF, INTER = hs.HISPARSE_ROTARY_HALF, hs.HISPARSE_ROTARY_INTERLEAVED


def desc(dims, layout, scaling=0, flags=0, theta=1e4, factor=8.0, magnitude=1.0, low=1.0, high=32.0):
    return hs.RotaryDesc(dims, layout, scaling, flags, theta, factor, 4096.0, low, high, magnitude)


def rows_of(x, y, first=0, out_rows=None):
    """[tokens][heads][dims] views; out_rows: int64 [tokens] rows of y."""
    r = hs.RotaryRows(x.data_ptr(), y.data_ptr(), None if out_rows is None else out_rows.data_ptr(),
                      y.shape[0] if out_rows is not None else 0, x.stride(0), x.stride(1),
                      y.stride(0), y.stride(1), x.shape[1], x.shape[2], first)
    r.keep = x, y, out_rows  # the struct holds addresses only
    return r


def data(shape, seed):
    return torch.randn(shape, generator=torch.Generator().manual_seed(seed)).to(torch.bfloat16)


def positions(n, seed, far=1 << 20):
    p = torch.randint(0, far, (n,), generator=torch.Generator().manual_seed(seed)).int()
    p[:min(n, 3)] = torch.tensor([0, 1, far - 1], dtype=torch.int32)[:min(n, 3)]
    return p


def check(got, d, pos, x, first, far=False):
    want, size = ref.rotate(d, pos, x, first)
    err = (got.cpu().double() - want).abs()
    tol = want.abs() * 2.0 ** -8 + size * (2.0 ** -20 + (2.0 ** -20 if far else 0.0))
    assert bool((err <= tol).all()), (err - tol).max().item()
    rest = torch.ones(x.shape[-1], dtype=torch.bool)
    rest[first:first + d.dims] = False
    assert torch.equal(got.cpu()[..., rest], x[..., rest])


def turn(d, pos, *rows):
    n = pos.numel()
    hs.hisparse_rotate_tokens(d, n, pos.cuda(), (hs.RotaryRows * len(rows))(*rows), len(rows),
                              torch.cuda.current_stream())


@pytest.mark.parametrize("layout", [HALF, INTER])
@pytest.mark.parametrize("dims,first,whole", [(128, 0, 128), (32, 0, 128), (64, 64, 128), (64, 512, 576),
                                              (16, 32, 64), (2, 0, 2), (2, 5, 9), (20, 3, 31),
                                              (256, 0, 256), (78, 0, 128), (48, 16, 80), (64, 8, 80)])
@pytest.mark.parametrize("n,heads", [(1, 1), (3, 5), (67, 33)])
def test_shapes(layout, dims, first, whole, n, heads):
    d, pos = desc(dims, layout), positions(n, dims)
    x = data((n, heads, whole), n + dims)
    xd, y = x.cuda(), torch.full((n, heads, whole), 7.0, dtype=torch.bfloat16, device="cuda")
    turn(d, pos, rows_of(xd, y, first))
    check(y, d, pos, x, first)
    assert torch.equal(xd.cpu(), x)
    turn(d, pos, rows_of(xd, xd, first))  # in place
    assert torch.equal(xd, y)


@pytest.mark.parametrize("scaling,kw", [(0, {}), (1, {}), (2, {}), (2, dict(low=4.0, high=5.0)),
                                        (2, dict(magnitude=1.2079441541679836)),
                                        (1, dict(factor=0.5, magnitude=0.25)), (0, dict(theta=5e6))])
def test_scalings_and_far_positions(scaling, kw):
    for layout in (HALF, INTER):
        d = desc(128, layout, scaling, **kw)
        x = data((40, 3, 128), 5)
        for far in (4096, 1 << 20, (1 << 31) - 1):
            pos = positions(40, 3, far)
            y = torch.zeros((40, 3, 128), dtype=torch.bfloat16, device="cuda")
            turn(d, pos, rows_of(x.cuda(), y))
            check(y, d, pos, x, 0, far=True)


def test_negative_positions_and_the_way_back():
    x, pos = data((33, 4, 64), 1), positions(33, 2)
    for layout in (HALF, INTER):
        a, b = (torch.zeros((33, 4, 64), dtype=torch.bfloat16, device="cuda") for _ in range(2))
        turn(desc(64, layout), -pos, rows_of(x.cuda(), a))
        turn(desc(64, layout, flags=hs.HISPARSE_ROTARY_BACK), pos, rows_of(x.cuda(), b))
        assert torch.equal(a, b)
        check(b, desc(64, layout, flags=hs.HISPARSE_ROTARY_BACK), pos, x, 0)


@pytest.mark.parametrize("layout", [HALF, INTER])
def test_back_is_the_gradient(layout):
    """The call is linear in its rows, so its derivative along e is its value at e: <g, R e> = <R' g, e>
    for unit vectors e of every pair, in exact terms up to the roundings of both calls."""
    n, D = 128, 128
    d = desc(D, layout, 2, magnitude=1.25)
    back = desc(D, layout, 2, flags=hs.HISPARSE_ROTARY_BACK, magnitude=1.25)
    pos = torch.full((n,), 777, dtype=torch.int32)
    e, g = torch.eye(n, dtype=torch.bfloat16)[:, None], data((1, 1, D), 3).expand(n, 1, D).contiguous()
    Re, Rg = (torch.zeros((n, 1, D), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    turn(d, pos, rows_of(e.cuda(), Re))
    turn(back, pos, rows_of(g.cuda(), Rg))
    left = (Re.cpu().double() * g.double()).sum((1, 2))
    right = torch.diagonal(Rg.cpu().double()[:, 0])
    # two elements of R e times g, and one of R' g: each off by 2^-8 of itself and 2^-20 of its pair
    bound = (2.0 ** -8 + 2.0 ** -20) * 2 * 1.25 * 2 * g.double().abs().max()
    assert bool(((left - right).abs() <= bound).all())
    # differences: linear, so that a step of any size gives the derivative
    x = data((n, 1, D), 9)
    y0, y1 = (torch.zeros((n, 1, D), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    x1 = (x.float() + 2.0 * e.float()).to(torch.bfloat16)
    step = x1.double() - x.double()
    turn(d, pos, rows_of(x.cuda(), y0))
    turn(d, pos, rows_of(x1.cuda(), y1))
    diff = ((y1.double() - y0.double()).cpu() * g.double()).sum((1, 2))
    want = (Rg.cpu().double() * step).sum((1, 2))
    size = (y0.cpu().double().abs() + y1.cpu().double().abs()) * g.double().abs()
    tol = (size.sum((1, 2)) * 2.0 ** -8 + step.abs().sum((1, 2)) * 2.0 ** -7 *
           Rg.cpu().double().abs().amax((1, 2)) + 2.0 ** -14)
    assert bool(((diff - want).abs() <= tol).all())


def test_arrays_of_one_call_strides_and_row_maps():
    """Queries of a fused projection into the tail of wider rows, keys in place, an index key scattered into
    a pool of rows; all at odd elements."""
    n = 71
    d, pos = desc(64, INTER, 2), positions(n, 8)
    wide = data((n, 9 * 192 + 1), 1).cuda()
    q = wide[:, 1:].unflatten(1, (9, 192))[..., 128:]          # [n][9][64]
    out = data((n, 9, 577), 2).cuda()
    tail = out[..., 513:]
    keep = out.clone()
    kbuf = data((n, 2 * 100 + 3), 3).cuda()
    k = kbuf[:, 3:].unflatten(1, (2, 100))
    k_before = k.clone()
    ik = data((n, 1, 128), 4).cuda()
    pool = data((90, 1, 128), 5).cuda()
    pool_keep = pool.clone()
    where = torch.randperm(90, generator=torch.Generator().manual_seed(6))[:n]
    where[5], where[20], where[70] = -1, 90, 1 << 40
    turn(d, pos, rows_of(q, tail), rows_of(k, k, 30),
         rows_of(ik, pool, 64, where.cuda()))
    check(tail, d, pos, q.cpu(), 0)
    assert torch.equal(out[..., :513], keep[..., :513])
    check(k, d, pos, k_before.cpu(), 30)
    ok = (where >= 0) & (where < 90)
    check(pool.cpu()[where[ok]], d, pos[ok], ik.cpu()[ok], 64)
    other = torch.ones(90, dtype=torch.bool)
    other[where[ok]] = False
    assert torch.equal(pool.cpu()[other], pool_keep.cpu()[other])


@pytest.mark.parametrize("n,heads", [(3000, 40), (5, 128), (1, 1000), (20001, 1)])
def test_sizes(n, heads):
    """Many tokens of a workgroup, several workgroups of a token."""
    d, pos = desc(64, HALF), positions(n, 1)
    x = data((n, heads, 64), 2)
    y = torch.zeros((n, heads, 64), dtype=torch.bfloat16, device="cuda")
    turn(d, pos, rows_of(x.cuda(), y))
    check(y, d, pos, x, 0)


def test_large_and_odd_values():
    x = torch.tensor([0.0, -0.0, 1e30, -3e38, 1e-40, 6e-39, 65504.0, 1.0] * 8).to(torch.bfloat16)
    x = x.view(1, 1, 64).expand(5, 1, 64).contiguous()
    pos, d = positions(5, 1), desc(64, INTER, magnitude=0.5)
    y = torch.zeros((5, 1, 64), dtype=torch.bfloat16, device="cuda")
    turn(d, pos, rows_of(x.cuda(), y))
    want, size = ref.rotate(d, pos, x, 0)
    # below the normal range a step is 2^-133 whatever the value
    assert bool(((y.cpu().double() - want).abs() <= want.abs() * 2.0 ** -8 + size * 2.0 ** -20 +
                 2.0 ** -133).all())
    # a NaN or an infinity stays in its pair
    z = data((1, 1, 64), 1)
    z[0, 0, 3], z[0, 0, 40] = math.nan, math.inf
    turn(desc(64, INTER), pos[1:2], rows_of(z.cuda(), y))
    bad = ~torch.isfinite(y[0, 0].cpu())
    assert bad.nonzero().flatten().tolist() == [2, 3, 40, 41]


def test_captured_and_replayed_on_another_stream():
    d, n = desc(128, HALF, 1), 50
    x = data((n, 6, 128), 1).cuda()
    y, pos = torch.zeros_like(x), positions(n, 1).cuda()
    rows = (hs.RotaryRows * 1)(rows_of(x, y))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=side):
        hs.hisparse_rotate_tokens(d, n, pos, rows, 1, torch.cuda.current_stream())
    for seed in (5, 6, 7):
        p, v = positions(n, seed), data((n, 6, 128), seed)
        pos.copy_(p)
        x.copy_(v)
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        check(y, d, p, v, 0)


def test_offsets_beyond_four_gibibytes():
    """Rows 256 MiB apart, read there, written there, and scattered there."""
    n, apart = 20, 1 << 27
    d, pos, x = desc(64, HALF), positions(n, 1), data((n, 1, 128), 2)
    far = torch.empty(2 * n * apart, dtype=torch.bfloat16, device="cuda").view(2 * n, 1, apart)[..., :128]
    far[:n] = x.cuda()
    to = torch.arange(n, 2 * n).flip(0).cuda()
    near = torch.zeros((n, 1, 128), dtype=torch.bfloat16, device="cuda")
    turn(d, pos, rows_of(far[:n], near))
    check(near, d, pos, x, 0)
    turn(d, pos, rows_of(x.cuda(), far, 0, to))
    check(far[n:].flip(0), d, pos, x, 0)
    turn(d, pos, rows_of(far[:n], far[:n]))
    check(far[:n], d, pos, x, 0)


@pytest.mark.parametrize("layout", [HALF, INTER])
def test_more_heads_than_one_launch_has_pieces_for(layout):
    """A token of 2^20 and more heads: several launches, each of whole heads; a second array behind it."""
    heads, whole = (1 << 20) + 50001, 130
    d, pos = desc(126, layout), positions(1, 1)
    x, z = data((1, heads, whole), 3).cuda(), data((1, 3, whole), 4)
    y, zd = torch.full_like(x, 7.0), z.cuda()
    turn(d, pos, rows_of(x, y, 3), rows_of(zd, zd, 1))
    at = torch.cat((torch.arange(0, heads, 4099), torch.arange(heads - 70, heads)))
    check(y[:, at.cuda()], d, pos, x[:, at.cuda()].cpu(), 3)
    check(zd, d, pos, z, 1)
    pair = torch.full((1,), pos.item(), dtype=torch.int32)
    same = torch.empty((1, 5, whole), dtype=torch.bfloat16, device="cuda")
    for h0 in range(0, heads - 5, 99991):  # the same as a call of its own
        turn(d, pair, rows_of(x[:, h0:h0 + 5], same, 3))
        assert torch.equal(same, y[:, h0:h0 + 5])


def test_more_tokens_than_one_launch_has_workgroups_for():
    """2^24 and more tokens, a workgroup each: one row read by all of them, written where a row map says so."""
    n, dims = (1 << 24) + 77, 522
    d = desc(2, HALF)
    pos = torch.arange(n, dtype=torch.int32, device="cuda")
    x = data((1, 1, dims), 3)
    where = torch.full((n,), -1, dtype=torch.int64, device="cuda")
    at = torch.cat((torch.arange(0, n, 300007), torch.arange(n - 90, n)))
    where[at.cuda()] = torch.arange(at.numel(), device="cuda").flip(0)
    y = torch.full((at.numel() + 2, 1, dims), 7.0, dtype=torch.bfloat16, device="cuda")
    xd = x.cuda()
    r = hs.RotaryRows(xd.data_ptr(), y.data_ptr(), where.data_ptr(), at.numel(), 0, dims, dims, dims, 1, dims, 5)
    hs.hisparse_rotate_tokens(d, n, pos, r, 1, torch.cuda.current_stream())
    check(y[:-2].flip(0), d, at.int(), x.expand(at.numel(), 1, dims), 5, far=True)
    assert bool((y[-2:] == 7.0).all())
    r = hs.RotaryRows(xd.data_ptr(), y.data_ptr(), None, 0, 0, dims, dims, dims, 1, dims, 5)
    hs.hisparse_rotate_tokens(d, 3, pos, r, 1, torch.cuda.current_stream())
    check(y[:3], d, torch.arange(3).int(), x.expand(3, 1, dims), 5)


def test_a_token_map_and_rows_of_several_launches():
    """The same with an array in place beside it, tokens apart in memory and not read twice."""
    n, heads = (1 << 22) + 5, 4200
    d = desc(2, INTER)
    pos = torch.arange(n, dtype=torch.int32, device="cuda") & 1023
    x = torch.randn((n, 16), generator=torch.Generator("cuda").manual_seed(1), device="cuda").to(torch.bfloat16)
    keep = x.clone()
    wide = data((1, heads, 2), 1).cuda()
    where = torch.full((n,), -1, dtype=torch.int64, device="cuda")
    y = torch.full((3, heads, 2), 7.0, dtype=torch.bfloat16, device="cuda")
    last = torch.tensor([0, n // 2, n - 1])
    where[last.cuda()] = torch.arange(3, device="cuda")
    rows = (hs.RotaryRows * 2)(
        hs.RotaryRows(x.data_ptr(), x.data_ptr(), None, 0, 16, 0, 16, 0, 1, 16, 8),
        hs.RotaryRows(wide.data_ptr(), y.data_ptr(), where.data_ptr(), 3, 0, 2, heads * 2, 2, heads, 2, 0))
    hs.hisparse_rotate_tokens(d, n, pos, rows, 2, torch.cuda.current_stream())
    check(y, d, pos.cpu()[last], wide.cpu().expand(3, heads, 2), 0)
    at = torch.cat((torch.arange(0, n, 50021), torch.arange(n - 90, n)))
    check(x[at.cuda(), None], d, pos.cpu()[at], keep.cpu()[at][:, None], 8)
