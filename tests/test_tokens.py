"""Token records without a GPU: record sizes, descriptors, and the refusals of the calls that write,
read and attend to them (all before any device work)."""
import numpy as np
import pytest
import torch

import token_reference as ref
from paper_2608_07009_amd import HiSparseCache, hisparse as hs

G, L = hs.HISPARSE_KV_GROUPED, hs.HISPARSE_KV_LATENT
BF, F8 = hs.HISPARSE_KV_BF16, hs.HISPARSE_KV_FP8
INVALID, UNSUPPORTED = hs.HISPARSE_ERR_INVALID_ARG, hs.HISPARSE_ERR_UNSUPPORTED


def kv(layout=G, type=F8, tpr=16, **kw):
    R = kw.pop("record_bytes", hs.hisparse_kv_record_bytes(layout, type, tpr) or 16)
    d = dict(layout=layout, type=type, tokens_per_record=tpr, record_bytes=R, num_records=8,
             record_stride=2 * R, head_stride=R, request_stride=0)
    d.update(kw)
    return hs.KvDesc(**d)


def chunk(layout=G, **kw):
    d = dict(num_requests=2, kv_heads=2, q_heads=4, total_tokens=6, max_chunk=3, max_records=4,
             q_token_stride=8 * ref.D_QK[layout], out_token_stride=8 * ref.D_V[layout],
             table_request_stride=4, table_head_stride=0, window=0, num_splits=0, scale=0.1,
             flags=hs.HISPARSE_CHUNK_CAUSAL)
    d.update(kw)
    return hs.ChunkDesc(**d)


@pytest.mark.parametrize("layout,type,tpr,n", [
    (G, BF, 1, 512), (G, BF, 64, 32768), (G, F8, 1, 272), (G, F8, 2, 528), (G, F8, 16, 4224),
    (G, F8, 64, 16896), (L, BF, 1, 1152), (L, F8, 1, 656), (L, F8, 4, 2576), (L, F8, 64, 41216),
    (L, BF, 4096, 4096 * 1152), (G, F8, 3, 0), (G, F8, 0, 0), (G, F8, 8192, 0), (2, F8, 1, 0),
    (G, 2, 1, 0), (-1, BF, 1, 0)])
def test_record_bytes(layout, type, tpr, n):
    assert hs.hisparse_kv_record_bytes(layout, type, tpr) == n


def test_bf16_records_are_those_of_the_sparse_decode_attention():
    for layout, tpr, R in ((L, 1, 1152), (G, 64, 32768), (G, 16, 8192)):
        assert hs.hisparse_kv_record_bytes(layout, BF, tpr) == R
        a = hs.AttnDesc(4, ref.D_QK[layout], ref.D_V[layout], 128 if layout == G else 0, tpr, 0,
                        0.1, 0)
        assert hs.hisparse_validate_attn(R, 8, a) == hs.HISPARSE_OK


@pytest.mark.parametrize("kw", [
    dict(layout=2), dict(type=2), dict(tpr=3), dict(tpr=0), dict(record_bytes=4208),
    dict(record_bytes=4232), dict(record_bytes=(8 << 20) + 16), dict(num_records=0),
    dict(num_records=1 << 31), dict(record_stride=4208), dict(record_stride=4232),
    dict(head_stride=-16), dict(head_stride=8), dict(request_stride=-16), dict(request_stride=24),
    dict(type=BF, record_bytes=16 * 512 + 16, record_stride=1 << 20),
    dict(num_records=(1 << 31) - 1, record_stride=1 << 32)])
def test_record_descriptors_refused(kw):
    assert hs.hisparse_validate_kv(kv(**kw)) == INVALID
    assert hs.hisparse_validate_chunk(kv(**kw), chunk()) == INVALID
    assert hs.hisparse_chunk_workspace_bytes(kv(**kw), chunk()) == 0


@pytest.mark.parametrize("kw", [dict(), dict(type=BF), dict(layout=L, tpr=1),
                                dict(record_bytes=4240, record_stride=4240), dict(tpr=4096),
                                dict(type=BF, record_bytes=16 * 528, record_stride=1 << 20)])
def test_record_descriptors_accepted(kw):
    assert hs.hisparse_validate_kv(kv(**kw)) == hs.HISPARSE_OK


@pytest.mark.parametrize("kw,status", [
    (dict(num_requests=0), INVALID), (dict(kv_heads=0), INVALID), (dict(q_heads=0), INVALID),
    (dict(q_heads=257, q_token_stride=1 << 20, out_token_stride=1 << 20), INVALID),
    (dict(num_requests=1 << 20), INVALID), (dict(total_tokens=-1), INVALID),
    (dict(max_chunk=0), INVALID), (dict(max_records=0), INVALID),
    (dict(max_records=(1 << 26) + 1), INVALID), (dict(q_token_stride=-1), INVALID),
    (dict(out_token_stride=8 * 128 - 1), INVALID), (dict(table_request_stride=-1), INVALID),
    (dict(table_head_stride=-1), INVALID), (dict(window=-1), INVALID),
    (dict(window=5, flags=0), INVALID), (dict(num_splits=-1), INVALID),
    (dict(num_splits=65), INVALID), (dict(scale=0.0), INVALID), (dict(scale=-1.0), INVALID),
    (dict(scale=float("nan")), INVALID), (dict(scale=2e6), INVALID), (dict(flags=2), INVALID),
    (dict(total_tokens=1 << 28), UNSUPPORTED)])
def test_chunk_descriptors_refused(kw, status):
    assert hs.hisparse_validate_chunk(kv(), chunk(**kw)) == status
    assert hs.hisparse_chunk_workspace_bytes(kv(), chunk(**kw)) == 0
    x = np.zeros(64, np.int64)  # never reached
    with pytest.raises(hs.HisparseError) as e:
        hs.hisparse_chunk_attention(kv(), chunk(**kw), x, x, x, x, x, x, x, x, 1 << 40)
    assert e.value.status == status


def test_chunk_calls_refused():
    x = np.zeros(4096, np.uint8)
    base = (x.ctypes.data + 15) // 16 * 16

    def call(desc=None, pool=base, table=base, start=base, kv_len=base, q=base, out=base, lse=base,
             ws=base, n=1 << 40):
        with pytest.raises(hs.HisparseError) as e:
            hs.hisparse_chunk_attention(kv(), desc or chunk(), pool, table, start, kv_len, q, out,
                                        lse, ws, n)
        return e.value.status

    assert call(pool=None) == call(table=None) == call(q=None) == call(out=None) == INVALID
    assert call(pool=base + 8) == call(table=base + 2) == call(start=base + 1) == INVALID
    assert call(kv_len=base + 2) == call(q=base + 1) == call(out=base + 1) == INVALID
    assert call(lse=base + 2) == INVALID
    # uniform chunks need all their rows
    assert call(chunk(total_tokens=5), start=None) == INVALID
    # a null descriptor
    assert hs.lib().hisparse_validate_kv(None) == INVALID
    assert hs.lib().hisparse_validate_chunk(None, None) == INVALID
    # nothing to do needs no arrays
    hs.hisparse_chunk_attention(kv(), chunk(total_tokens=0), None, None, base, base, None, None,
                                None, None, 0)


@pytest.mark.parametrize("fn", ["write", "read"])
def test_token_calls_refused(fn):
    x = np.zeros(4096, np.uint8)
    base = (x.ctypes.data + 15) // 16 * 16

    def call(desc=None, heads=2, n=3, k=base, ks=256, v=base, vs=256, slots=base, pool=base):
        desc = desc or kv()
        with pytest.raises(hs.HisparseError) as e:
            if fn == "write":
                hs.hisparse_write_tokens(desc, heads, n, k, ks, v, vs, slots, pool)
            else:
                hs.hisparse_read_tokens(desc, heads, n, pool, slots, k, ks, v, vs)
        return e.value.status

    assert call(kv(tpr=3)) == call(heads=0) == call(n=-1) == INVALID
    assert call(k=None) == call(v=None) == call(pool=None) == INVALID
    assert call(k=base + 1) == call(v=base + 1) == call(pool=base + 8) == INVALID
    assert call(slots=base + 4) == call(ks=-1) == call(vs=-1) == INVALID
    assert call(kv(head_stride=4208)) == call(kv(head_stride=0)) == INVALID
    assert call(heads=1 << 16, n=1 << 16, ks=1 << 23, vs=1 << 23) == UNSUPPORTED
    if fn == "read":
        assert call(ks=255) == call(vs=255) == INVALID
    # nothing to do needs no arrays
    if fn == "write":
        hs.hisparse_write_tokens(kv(), 2, 0, None, 256, None, 256, None, None)
    else:
        hs.hisparse_read_tokens(kv(), 2, 0, None, None, None, 256, None, 256)


@pytest.mark.parametrize("layout,most", [(G, (1 << 28) - 16), (L, (1 << 26) - 4)])
def test_more_tokens_than_one_launch_takes(layout, most):
    x = np.zeros(64, np.uint8)
    base = (x.ctypes.data + 15) // 16 * 16
    d = kv(layout, tpr=1, record_bytes=656, record_stride=656, head_stride=0)
    for call in (lambda n: hs.hisparse_write_tokens(d, 1, n, base, 512, base, 512, None, base),
                 lambda n: hs.hisparse_read_tokens(d, 1, n, base, None, base, 512, base, 512)):
        for n in (most + 1, 2 ** 31 - 1):
            with pytest.raises(hs.HisparseError) as e:
                call(n)
            assert e.value.status == UNSUPPORTED


def test_more_parts_than_one_launch_takes():
    c = dict(num_requests=1, kv_heads=1, q_heads=256, total_tokens=1 << 22, max_chunk=1 << 22,
             out_token_stride=256 * 128)
    d = kv()
    assert hs.hisparse_validate_chunk(d, chunk(**c)) == hs.HISPARSE_OK
    assert hs.hisparse_validate_chunk(d, chunk(**c, num_splits=4)) == UNSUPPORTED


def test_reference_rounding_is_torch_e4m3():
    g = torch.Generator().manual_seed(1)
    x = torch.randn(20000, generator=g, dtype=torch.float64) * torch.exp2(
        torch.randint(-12, 7, (20000,), generator=g).double())
    x = torch.cat((x, torch.tensor([448.0, -448.0, 464.0, 0.0, 2.0 ** -10, 3 * 2.0 ** -10,
                                    17.0, 18.0, 19.0])))
    y = x.float().clamp(-448, 448)
    assert torch.equal(ref.round_e4m3(y.double()), y.to(torch.float8_e4m3fn).double())


def test_reference_scales():
    x = torch.tensor([[448.0, 1.0], [448.5, 0.0], [0.0, 0.0], [2.0 ** -130, 0.0], [7 / 8, -3 / 8],
                      [float("inf"), 3.0], [float("nan"), float("-inf")], [225.0, 0.0]]).double()
    want = [1.0, 2.0, 1.0, 2.0 ** -117, 2.0 ** -9, 2.0 ** -7, 1.0, 1.0]
    assert ref.scale_of(x).flatten().tolist() == want


def test_cache_descriptor_of_a_handle():
    c = HiSparseCache.__new__(HiSparseCache)
    c.handle = None
    c.desc = hs.CacheDesc(3, 1, 2, 40, 100, 8, 4224, 1, 0, 0, 0, 0)
    d = c.kv_desc(G, F8, 16)
    assert (d.num_records, d.record_stride, d.head_stride, d.request_stride) == (
        40, 4224, 40 * 4224, 80 * 4224)
    d = c.kv_desc(G, F8, 16, host_pool=True)
    assert (d.num_records, d.head_stride, d.request_stride) == (100, 100 * 4224, 200 * 4224)
    assert hs.hisparse_validate_kv(d) == hs.HISPARSE_OK
