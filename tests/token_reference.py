"""Plain 64-bit reference of the token-record operators (hisparse_write_tokens,
hisparse_read_tokens, hisparse_chunk_attention), on CPU tensors."""
from __future__ import annotations

import math

import torch

from paper_2608_07009_amd import hisparse as hs

GROUPED, LATENT = hs.HISPARSE_KV_GROUPED, hs.HISPARSE_KV_LATENT
BF16, FP8 = hs.HISPARSE_KV_BF16, hs.HISPARSE_KV_FP8
DIMS = {GROUPED: (128, 128), LATENT: (512, 64)}  # of the K and the V row
D_QK = {GROUPED: 128, LATENT: 576}
D_V = {GROUPED: 128, LATENT: 512}


def scale_of(x: torch.Tensor) -> torch.Tensor:
    """float64 [..., dims] -> the scale [..., 1] of its 8-bit form."""
    a = torch.where(torch.isfinite(x), x.abs(), torch.zeros_like(x)).amax(-1, keepdim=True)
    e = torch.full_like(a, -117.0)
    for _ in range(260):  # the least exponent from -117 on that covers the part
        e = torch.where(a > 448.0 * torch.exp2(e), e + 1.0, e)
    return torch.where(a > 0, torch.exp2(e), torch.ones_like(a))


def round_e4m3(y: torch.Tensor) -> torch.Tensor:
    """float64 -> the nearest e4m3 number (ties to even), infinities to +-448, NaN kept."""
    y = y.clamp(-448.0, 448.0)
    step = torch.exp2(torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6))) - 3.0)
    return torch.round(y / step) * step


def stored(kind: int, k: torch.Tensor, v: torch.Tensor, type_: int):
    """What records of (k, v) rows stand for (float64 rows), and their scales."""
    k, v = k.double(), v.double()
    if type_ == BF16:
        return k, v, None
    sk = scale_of(k)
    kq = round_e4m3(k / sk) * sk
    if kind == LATENT:
        return kq, v, sk
    sv = scale_of(v)
    return kq, round_e4m3(v / sv) * sv, torch.cat((sk, sv), -1)


def views(kind: int, type_: int, tpr: int, pool: torch.Tensor) -> dict:
    """The parts of records given as uint8 [..., record_bytes]."""
    R = pool.shape[-1]
    if type_ == BF16:
        return {"rows": pool.view(torch.bfloat16).unflatten(-1, (tpr, R // 2 // tpr))
                [..., :sum(DIMS[kind])]}
    e = 256 if kind == GROUPED else 512
    at = tpr * e
    out = {"rows": pool[..., :at].view(torch.float8_e4m3fn).unflatten(-1, (tpr, e))}
    if kind == LATENT:
        out["rope"] = pool[..., at:at + 128 * tpr].view(torch.bfloat16).unflatten(-1, (tpr, 64))
        at += 128 * tpr
    n = 2 if kind == GROUPED else 1
    out["scales"] = pool[..., at:at + 4 * n * tpr].view(torch.float32).unflatten(-1, (tpr, n))
    return out


def rows_of(kind: int, type_: int, tpr: int, pool: torch.Tensor):
    """float64 K and V rows [..., tpr, dims] that records hold."""
    v = views(kind, type_, tpr, pool)
    d = DIMS[kind][0]
    if type_ == BF16:
        return v["rows"][..., :d].double(), v["rows"][..., d:].double()
    x, s = v["rows"].float().double(), v["scales"].double()
    if kind == LATENT:
        return x * s, v["rope"].double()
    return x[..., :d] * s[..., :1], x[..., d:] * s[..., 1:]


def make_pool(kind: int, type_: int, tpr: int, k: torch.Tensor, v: torch.Tensor,
              record_bytes: int = 0) -> torch.Tensor:
    """uint8 [..., record_bytes] records holding bf16 rows k, v [..., tpr, dims]."""
    R = record_bytes or hs.hisparse_kv_record_bytes(kind, type_, tpr)
    pool = torch.full((*k.shape[:-2], R), 0xA5, dtype=torch.uint8)
    p = views(kind, type_, tpr, pool)
    if type_ == BF16:
        p["rows"].copy_(torch.cat((k, v), -1))
        return pool
    rk, rv, s = stored(kind, k, v, type_)
    if kind == LATENT:
        p["rows"].copy_((rk / s).to(torch.float8_e4m3fn))
        p["rope"].copy_(v)
    else:
        p["rows"].copy_(torch.cat((rk / s[..., :1], rv / s[..., 1:]), -1)
                        .to(torch.float8_e4m3fn))
    p["scales"].copy_(s)
    return pool


def attend(kind: int, k: torch.Tensor, v: torch.Tensor, q: torch.Tensor, seen: torch.Tensor,
           scale: float):
    """One (request, kv head): k, v float64 rows [T][dims], q [n][g][d_qk], seen bool [n][T].
    Returns out [n][g][d_v], lse [n][g] and what an error of the kernels' is measured by: the
    softmax-weighted |v| and the largest sum of |q_i k_i| scale of a visible token (what bounds the
    rounding of a score)."""
    if kind == LATENT:
        k, v = torch.cat((k, v), -1), k
    q = q.double()
    n, g, T = q.shape[0], q.shape[1], k.shape[0]
    d_v = v.shape[1]
    out = torch.zeros((n, g, d_v), dtype=torch.float64)
    lse = torch.full((n, g), -math.inf, dtype=torch.float64)
    absv = torch.zeros((n, g, d_v), dtype=torch.float64)
    size = torch.zeros((n, g), dtype=torch.float64)
    for i in range(n):
        j = torch.nonzero(seen[i]).flatten()
        if not len(j):
            continue
        kk, vv = k[j], v[j]
        x = scale * (q[i] @ kk.t())
        p = torch.softmax(x, 1)
        out[i], lse[i] = p @ vv, torch.logsumexp(x, 1)
        absv[i], size[i] = p @ vv.abs(), scale * (q[i].abs() @ kk.abs().t()).amax(1)
    return out, lse, absv, size


def visible(n: int, length: int, T: int, causal: bool, window: int = 0) -> torch.Tensor:
    """bool [n][T]: which cached tokens each new token sees."""
    j = torch.arange(T)[None]
    pos = length - n + torch.arange(n)[:, None]
    seen = (j < length).expand(n, T).clone()
    if causal:
        seen &= j <= pos
    if window:
        seen &= j > pos - window
    return seen


def check(kind: int, out, lse, ref, what: str = "") -> None:
    """Kernel results of one (request, kv head) against attend()'s, by the roundings it makes.

    A score is a sum of d_qk products in fp32, in any order: off by at most d_qk 2^-24 times the sum
    of the products' magnitudes; times the scale and less the maximum, two more roundings of values
    up to that size; the exponential 2^-22 of a weight. With x the sum of these, a weight is off by
    x relative to itself, the normaliser too. Each weight is rounded to bf16 (2^-8) for the product
    with V, sums stay in fp32 (T 2^-24, at most 2^-9 here: taken into x), and the result is rounded
    to bf16 (2^-8)."""
    o_ref, l_ref, absv, size = ref
    x = size * (D_QK[kind] + 8) * 2.0 ** -24 + 2.0 ** -19
    empty = torch.isinf(l_ref)
    if lse is not None:
        lse = lse.double().cpu()
        assert torch.equal(torch.isinf(lse) & (lse < 0), empty), f"{what}: empty rows differ"
        bad = (lse - l_ref).abs()[~empty] - (x + 2.0 ** -22 * l_ref.abs())[~empty]
        assert bad.numel() == 0 or float(bad.max()) <= 0, f"{what}: lse off by {float(bad.max()):.2e} more"
    out = out.double().cpu()
    lim = (absv * (2.0 ** -8 + 2 * x[..., None])) * (1 + 2.0 ** -8) + 2.0 ** -8 * o_ref.abs()
    over = (out - o_ref).abs() - lim - 2.0 ** -133
    assert bool((over <= 0).all()), \
        f"{what}: {int((over > 0).sum())} of {over.numel()} values out of bounds, worst by {float(over.max()):.2e}"
