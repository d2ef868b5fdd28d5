"""hisparse_chunk_attention over values near the ends of their range: large V under scores that outgrow
the softmax's reference, infinities and NaN in tokens that rows do see. Compared as in
test_gpu_chunk_attention."""
import math

import pytest
import torch

import token_reference as ref
from test_gpu_chunk_attention import BF, F8, G, L, TYPES, Problem

pytestmark = pytest.mark.gpu


def refill(p, rows):
    """Replaces every request's tokens by the bf16 rows (k, v) that rows(request, head, tokens) gives."""
    for r in range(len(p.lens)):
        for h in range(p.kv_heads):
            T = p.k[r].shape[0]
            k, v = (x.to(torch.bfloat16) for x in rows(r, h, T))
            kk, vv = (x.unflatten(0, (T // p.tpr, p.tpr)) for x in (k, v))
            rec = ref.make_pool(p.kind, p.type_, p.tpr, kk, vv)
            p.pool[p.table[r, :T // p.tpr].long(), h] = rec.cuda()
            sk, sv, _ = ref.stored(p.kind, k, v, p.type_)
            p.k[r][:, h], p.v[r][:, h] = sk, sv


def one_dim_query(p):
    """A query of 1 in a single dim (latent: a rotary one), so that scores are what that dim of K
    holds."""
    p.q.zero_()
    p.q[..., 512 if p.kind == L else 0] = 1.0
    p.qd.copy_(p.q.flatten(1))


def ramp(p, size):
    """Scores that rise by p.scale per token (at most 256 of them, exact in bf16) over values of
    magnitude `size`."""
    gen = torch.Generator().manual_seed(11)

    def rows(r, h, T):
        s = torch.arange(T).float()
        if p.kind == G:
            k = torch.zeros((T, 128))
            k[:, 0] = s
            return k, torch.randn((T, 128), generator=gen) * size
        rope = torch.zeros((T, 64))
        rope[:, 0] = s
        return torch.randn((T, 512), generator=gen) * size, rope

    refill(p, rows)
    one_dim_query(p)


@pytest.mark.parametrize("kind,type_,tpr", TYPES)
@pytest.mark.parametrize("size", [-100, 90, 100])
@pytest.mark.parametrize("rise", [0.05, 0.18, 2.0])
@pytest.mark.parametrize("q_heads,splits", [(2, 1), (40, 2)])
def test_large_values_under_scores_that_grow(kind, type_, tpr, size, rise, q_heads, splits):
    """Scores that end 18, 60 and 700 powers of two above the first one, values of 2^size: the result is
    an average of values and has to be finite."""
    p = Problem(kind, type_, tpr, 1, q_heads, [(20, 240), (1, 256)], splits=splits, scale=rise)
    ramp(p, 2.0 ** size)
    p.run()
    p.check(f"2^{size}")
    assert bool(torch.isfinite(p.out.float()).all())


def spoil(p, r, token, part, dim, value):
    """Writes a value into one dim of a token's K, V or rotary row in the pool (bf16 records; in 8-bit
    ones the byte of NaN)."""
    page, off = int(p.table[r, token // p.tpr]), token % p.tpr
    rec = p.pool[page].cpu()
    parts = ref.views(p.kind, p.type_, p.tpr, rec)
    if part == "rope" and p.type_ == F8:
        parts["rope"][:, off, dim] = value
    else:
        at = dim + {"k": 0, "v": 128, "rope": 512}[part]
        if p.type_ == F8:
            assert math.isnan(value)
            parts["rows"].view(torch.uint8)[:, off, at] = 0x7F
        else:
            parts["rows"][:, off, at] = value
    p.pool[page] = rec.cuda()


def expect(p, r, hidden):
    """Reference rows of request r, head 0, whose token `hidden` weighs nothing; and which of its new
    tokens see it."""
    n, t = p.lens[r]
    seen = ref.visible(n, t, p.k[r].shape[0], p.causal, p.window)
    sees = seen[:, hidden].clone()
    seen[:, hidden] = False
    rows = slice(p.starts[r], p.starts[r] + n)
    return ref.attend(p.kind, p.k[r][:, 0], p.v[r][:, 0], p.q[rows], seen, p.scale), sees


def results(p, r):
    torch.cuda.synchronize()
    rows = slice(p.starts[r], p.starts[r + 1])
    return p.out.cpu().unflatten(1, (p.H, ref.D_V[p.kind]))[rows], p.lse.cpu()[rows]


# a token that all rows of the workgroup see, one that only later rows see, and the last row's own
SEEN = [(200, 3), (200, 190), (200, 199)]


@pytest.mark.parametrize("kind,type_,part", [(G, BF, "k"), (L, BF, "rope"), (L, F8, "rope")])
@pytest.mark.parametrize("length,token", SEEN)
@pytest.mark.parametrize("q_heads,splits", [(2, 3), (12, 1)])
def test_a_score_of_minus_infinity_weighs_nothing(kind, type_, part, length, token, q_heads,
                                                  splits):
    p = Problem(kind, type_, 4, 1, q_heads, [(20, length)], splits=splits)
    dim = 3
    p.q[..., dim + (512 if part == "rope" else 0)] = 0.75  # positive: the score is -inf, not NaN
    p.qd.copy_(p.q.flatten(1))
    spoil(p, 0, token, part, dim, -math.inf)
    p.run()
    out, lse = results(p, 0)
    e, _ = expect(p, 0, token)
    ref.check(kind, out, lse, e)


@pytest.mark.parametrize("kind,type_,part", [(G, BF, "k"), (L, BF, "rope"), (L, F8, "rope")])
@pytest.mark.parametrize("splits", [1, 2])
def test_rows_that_see_nothing_but_scores_of_minus_infinity(kind, type_, part, splits):
    """They are as rows that see nothing."""
    p = Problem(kind, type_, 4, 1, 2, [(3, 100), (3, 100)], splits=splits)
    p.q[..., 3 + (512 if part == "rope" else 0)] = 0.75
    p.qd.copy_(p.q.flatten(1))
    for token in range(100):
        spoil(p, 0, token, part, 3, -math.inf)
    p.run()
    out, lse = results(p, 0)
    assert bool((out == 0).all()) and bool((lse == -math.inf).all())
    out, lse = results(p, 1)
    seen = ref.visible(3, 100, p.k[1].shape[0], True)
    ref.check(kind, out, lse, ref.attend(kind, p.k[1][:, 0], p.v[1][:, 0], p.q[3:], seen, p.scale))


@pytest.mark.parametrize("kind,type_,part,value", [
    (G, BF, "k", math.inf), (G, BF, "k", math.nan), (G, F8, "k", math.nan),
    (L, BF, "rope", math.inf), (L, BF, "rope", math.nan), (L, F8, "rope", math.inf),
    (L, BF, "k", math.inf), (L, BF, "k", math.nan), (L, F8, "k", math.nan)])
@pytest.mark.parametrize("length,token", SEEN)
@pytest.mark.parametrize("q_heads,splits", [(2, 3), (12, 1)])
def test_a_score_of_infinity_or_nan_makes_its_rows_nan(kind, type_, part, value, length, token,
                                                       q_heads, splits):
    p = Problem(kind, type_, 4, 1, q_heads, [(20, length)], splits=splits)
    p.q[..., 3 + (512 if part == "rope" else 0)] = 0.75
    p.qd.copy_(p.q.flatten(1))
    spoil(p, 0, token, part, 3, value)
    p.run()
    out, lse = results(p, 0)
    e, sees = expect(p, 0, token)
    assert bool(torch.isnan(out[sees]).all()) and bool(torch.isnan(lse[sees]).all())
    clean = ~sees
    ref.check(kind, out[clean], lse[clean], tuple(x[clean] for x in e))


@pytest.mark.parametrize("type_,value", [(BF, math.inf), (BF, -math.inf), (BF, math.nan),
                                         (F8, math.nan)])
@pytest.mark.parametrize("length,token", SEEN)
@pytest.mark.parametrize("q_heads,splits", [(2, 3), (12, 1)])
def test_a_seen_value_that_is_not_finite_stays_in_its_dim(type_, value, length, token, q_heads,
                                                          splits):
    p = Problem(G, type_, 4, 1, q_heads, [(20, length)], splits=splits)
    spoil(p, 0, token, "v", 77, value)
    p.run()
    out, lse = results(p, 0)
    seen = ref.visible(20, length, p.k[0].shape[0], True)
    sees = seen[:, token]
    assert not bool(torch.isfinite(out[sees][..., 77]).any())
    out[sees, :, 77] = 0
    v = p.v[0][:, 0].clone()
    v[:, 77] = 0
    plain = ref.attend(G, p.k[0][:, 0], p.v[0][:, 0], p.q, seen, p.scale)
    zeroed = ref.attend(G, p.k[0][:, 0], v, p.q, seen, p.scale)
    ref.check(G, out[sees], lse[sees], tuple(x[sees] for x in zeroed))
    ref.check(G, out[~sees], lse[~sees], tuple(x[~sees] for x in plain))


@pytest.mark.parametrize("length,token", SEEN)
@pytest.mark.parametrize("q_heads,splits", [(2, 3), (12, 1)])
def test_a_latent_of_minus_infinity_makes_its_dim_nan_at_least(length, token, q_heads, splits):
    """Its score is -inf and weighs nothing, but it is value too: its dim is NaN, and each other dim
    right or NaN."""
    p = Problem(L, BF, 4, 1, q_heads, [(20, length)], splits=splits)
    p.q[..., 3] = 0.75
    p.qd.copy_(p.q.flatten(1))
    spoil(p, 0, token, "k", 3, -math.inf)
    p.run()
    out, lse = results(p, 0)
    e, sees = expect(p, 0, token)
    assert bool(torch.isnan(out[sees][..., 3]).all())
    want = e[0]
    want[..., 3] = torch.where(sees[:, None], 0.0, want[..., 3])
    out[sees, :, 3] = 0
    out = torch.where(torch.isnan(out) & sees[:, None, None], want.to(out.dtype), out)
    lse = torch.where(torch.isnan(lse) & sees[:, None], e[1].float(), lse)
    ref.check(L, out, lse, e)
