"""hisparse_chunk_attention over values near the ends of their range: large V under scores that outgrow
the softmax's reference. Compared as in test_gpu_chunk_attention."""
import pytest
import torch

import token_reference as ref
from test_gpu_chunk_attention import G, L, TYPES, Problem

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
