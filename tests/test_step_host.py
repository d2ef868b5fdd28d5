"""The calls before the attention without a GPU: descriptors, frequencies, workspace sizes and refusals
(all before any device work)."""
import ctypes

import numpy as np
import pytest

import step_reference as ref
from paper_2608_07009_amd import hisparse as hs

INVALID, UNSUPPORTED, OK = hs.HISPARSE_ERR_INVALID_ARG, hs.HISPARSE_ERR_UNSUPPORTED, hs.HISPARSE_OK
X = np.zeros(4096, np.uint8)  # addresses that no refused call reaches
BASE = (X.ctypes.data + 15) // 16 * 16


def status(fn, *a):
    with pytest.raises(hs.HisparseError) as e:
        fn(*a)
    return e.value.status


def batch(**kw):
    d = dict(num_requests=2, kv_heads=2, total_tokens=6, max_chunk=3, max_records=4,
             tokens_per_record=16, table_request_stride=4, table_head_stride=0)
    d.update(kw)
    return hs.BatchDesc(**d)


def rotary(**kw):
    d = dict(dims=64, layout=0, scaling=0, flags=0, theta=1e4, factor=4.0, original_tokens=4096.0,
             low_turns=1.0, high_turns=32.0, magnitude=1.0)
    d.update(kw)
    return hs.RotaryDesc(**d)


def rows(**kw):
    d = dict(d_in=BASE, d_out=BASE + 1024, d_out_rows=None, num_out_rows=0, in_token_stride=256,
             in_head_stride=128, out_token_stride=256, out_head_stride=128, heads=2, dims=128,
             first=0)
    d.update(kw)
    return hs.RotaryRows(**d)


def index(**kw):
    d = dict(kind=ref.BOUNDS, tokens_per_record=16, num_records=8, record_stride=1024,
             head_stride=512, request_stride=0)
    d.update(kw)
    return hs.IndexDesc(**d)


def kv(**kw):
    d = dict(layout=0, type=1, tokens_per_record=16, record_bytes=4224, num_records=8,
             record_stride=2 * 4224, head_stride=4224, request_stride=0)
    d.update(kw)
    return hs.KvDesc(**d)


def select(**kw):
    d = dict(q_heads=4, top_k=8, first_records=1, last_records=1, q_token_stride=1024)
    d.update(kw)
    return hs.SelectDesc(**d)


BAD_BATCH = [dict(num_requests=0), dict(kv_heads=0), dict(num_requests=1 << 20),
             dict(total_tokens=-1), dict(max_chunk=0), dict(max_records=0),
             dict(max_records=(1 << 26) + 1), dict(tokens_per_record=3), dict(tokens_per_record=0),
             dict(tokens_per_record=8192), dict(table_request_stride=-1),
             dict(table_head_stride=-1)]


def plan_call(b=None, new=BASE, old=BASE, free=BASE, n=4, used=BASE, table=BASE, start=BASE,
              out=BASE, used_out=BASE, pos=BASE, slots=BASE):
    hs.hisparse_plan_tokens(b or batch(), new, old, free, n, used, table, start, out, used_out, pos,
                            slots)


@pytest.mark.parametrize("kw", BAD_BATCH)
def test_batch_descriptors_refused(kw):
    assert hs.hisparse_validate_batch(batch(**kw)) == INVALID
    assert status(plan_call, batch(**kw)) == INVALID
    assert hs.hisparse_validate_select(index(), batch(**kw), select()) == INVALID
    assert hs.hisparse_select_workspace_bytes(index(), batch(**kw), select()) == 0


def test_batch_descriptors_accepted():
    for kw in (dict(), dict(total_tokens=0), dict(tokens_per_record=4096), dict(tokens_per_record=1),
               dict(max_records=1 << 26), dict(num_requests=1 << 19)):
        assert hs.hisparse_validate_batch(batch(**kw)) == OK
    assert hs.lib().hisparse_validate_batch(None) == INVALID


def test_plan_calls_refused():
    def call(**kw):
        return status(lambda: plan_call(**kw))
    assert call(new=None) == call(table=None) == call(start=None) == call(out=None) == INVALID
    assert call(free=None) == call(n=0) == call(n=-1) == call(free=None, n=-1) == INVALID
    for name in ("new", "old", "free", "used", "table", "start", "out", "used_out", "pos"):
        assert call(**{name: BASE + 2}) == INVALID
    assert call(slots=BASE + 4) == INVALID
    assert call(b=batch(table_head_stride=4)) == INVALID
    assert call(b=batch(table_request_stride=3)) == INVALID  # rows that overlap, with a free list
    assert call(n=(1 << 31) - 6) == UNSUPPORTED


@pytest.mark.parametrize("kw", [
    dict(dims=0), dict(dims=3), dict(dims=258), dict(layout=2), dict(layout=-1), dict(scaling=3),
    dict(scaling=-1), dict(flags=2), dict(theta=0.0), dict(theta=-1.0), dict(theta=float("nan")),
    dict(theta=float("inf")), dict(magnitude=float("nan")), dict(scaling=1, factor=0.0),
    dict(scaling=2, factor=float("nan")), dict(scaling=2, original_tokens=0.0),
    dict(scaling=2, low_turns=32.0), dict(scaling=2, high_turns=float("inf"))])
def test_rotary_descriptors_refused(kw):
    d = rotary(**kw)
    assert hs.hisparse_validate_rotary(d) == INVALID
    assert status(hs.hisparse_rotary_frequencies, d) == INVALID
    assert status(hs.hisparse_rotate_tokens, d, 1, BASE, rows(), 1) == INVALID


@pytest.mark.parametrize("kw", [dict(), dict(dims=2), dict(dims=256, theta=5e5),
                                dict(scaling=1, factor=0.5), dict(scaling=2),
                                dict(scaling=2, low_turns=0.25, high_turns=300.0, factor=40.0),
                                dict(factor=0.0), dict(flags=1, magnitude=0.0)])
def test_rotary_frequencies(kw):
    d = rotary(**kw)
    assert hs.hisparse_validate_rotary(d) == OK
    got, want = hs.hisparse_rotary_frequencies(d), np.array(ref.frequencies(d))
    assert got.shape == want.shape
    # a power, a quotient and three products, each within a few units of 2^-53
    assert (np.abs(got - want) <= 16 * 2.0 ** -53 * want).all()
    if d.scaling == 0:
        assert got[0] == 1.0


@pytest.mark.parametrize("kw", [
    dict(heads=0), dict(first=-1), dict(first=65), dict(dims=63), dict(dims=65537, out_head_stride=1 << 17),
    dict(in_token_stride=-1), dict(in_head_stride=-1), dict(out_token_stride=-1),
    dict(out_head_stride=127), dict(out_token_stride=127), dict(d_in=BASE + 1), dict(d_out=BASE + 1),
    dict(d_out_rows=BASE + 4), dict(d_out_rows=BASE, num_out_rows=-1), dict(d_in=None),
    dict(d_out=None), dict(d_out=BASE, in_token_stride=512), dict(d_out=BASE, in_head_stride=256),
    dict(d_out=BASE, d_out_rows=BASE, num_out_rows=4), dict(first=(1 << 31) - 1)])
def test_rotary_rows_refused(kw):
    assert status(hs.hisparse_rotate_tokens, rotary(), 2, BASE, rows(**kw), 1) == INVALID


def test_rotate_calls_refused():
    call = lambda *a: status(hs.hisparse_rotate_tokens, rotary(), *a)  # noqa: E731
    two = (hs.RotaryRows * 2)(rows(), rows(heads=0))
    assert call(2, BASE, two, 2) == INVALID
    assert call(-1, BASE, rows(), 1) == call(2, None, rows(), 1) == INVALID
    assert call(2, BASE + 2, rows(), 1) == INVALID
    assert call(2, BASE, rows(), 0) == call(2, BASE, (hs.RotaryRows * 5)(), 5) == INVALID
    assert call(2, BASE, None, 1) == INVALID
    big = rows(heads=1 << 24, dims=65536, in_head_stride=65536, out_head_stride=65536,
               out_token_stride=1 << 40)
    assert call(1, BASE, big, 1) == UNSUPPORTED
    assert call((1 << 31) - 1, BASE, rows(out_token_stride=1 << 20), 1) == UNSUPPORTED
    # nothing to do needs no arrays
    hs.hisparse_rotate_tokens(rotary(), 0, None, rows(d_in=None, d_out=None), 1)


@pytest.mark.parametrize("kw", [
    dict(kind=3), dict(kind=-1), dict(tokens_per_record=5), dict(tokens_per_record=0),
    dict(num_records=0), dict(num_records=1 << 31), dict(record_stride=496),
    dict(record_stride=1 << 31), dict(record_stride=1032), dict(head_stride=-16),
    dict(head_stride=8), dict(request_stride=-16), dict(request_stride=24),
    dict(kind=ref.KEYS, record_stride=16 * 256 - 16)])
def test_index_descriptors_refused(kw):
    assert hs.hisparse_validate_index(index(**kw)) == INVALID
    assert hs.hisparse_validate_select(index(**kw), batch(), select()) == INVALID
    assert status(hs.hisparse_summarize_records, kv(), index(**kw), batch(), BASE, BASE, BASE, BASE,
                  BASE) == INVALID


def test_index_descriptors_accepted():
    for kw in (dict(), dict(kind=ref.MEANS, record_stride=256), dict(record_stride=512),
               dict(kind=ref.KEYS, record_stride=16 * 256)):
        assert hs.hisparse_validate_index(index(**kw)) == OK
    assert hs.lib().hisparse_validate_index(None) == INVALID


def test_summarize_calls_refused():
    def call(k=None, x=None, b=None, pool=BASE, table=BASE, start=BASE, lens=BASE, out=BASE):
        return status(hs.hisparse_summarize_records, k or kv(), x or index(), b or batch(), pool,
                      table, start, lens, out)
    assert call(k=kv(tokens_per_record=3)) == call(x=index(kind=ref.KEYS, record_stride=4096)) == INVALID
    assert call(x=index(tokens_per_record=8)) == call(b=batch(tokens_per_record=8)) == INVALID
    assert call(x=index(head_stride=496)) == INVALID
    assert call(pool=None) == call(out=None) == INVALID
    assert call(pool=BASE + 8) == call(out=BASE + 8) == call(table=BASE + 2) == INVALID
    assert call(start=BASE + 2) == call(lens=BASE + 1) == INVALID
    assert call(start=None, b=batch(total_tokens=5)) == INVALID
    assert call(k=kv(layout=1, record_bytes=10304, record_stride=10304)) == UNSUPPORTED
    assert call(b=batch(total_tokens=(1 << 31) - 1)) == UNSUPPORTED
    hs.hisparse_summarize_records(kv(), index(), batch(total_tokens=0), None, None, BASE, None, None)


@pytest.mark.parametrize("kw,st", [
    (dict(q_heads=0), INVALID), (dict(q_heads=257), INVALID), (dict(top_k=0), INVALID),
    (dict(top_k=4097), INVALID), (dict(first_records=-1), INVALID), (dict(last_records=-1), INVALID),
    (dict(first_records=8), INVALID), (dict(first_records=(1 << 31) - 1), INVALID),
    (dict(q_token_stride=-1), INVALID)])
def test_select_descriptors_refused(kw, st):
    assert hs.hisparse_validate_select(index(), batch(), select(**kw)) == st
    assert hs.hisparse_select_workspace_bytes(index(), batch(), select(**kw)) == 0


def test_select_calls_refused():
    keys = index(kind=ref.KEYS, record_stride=4096, head_stride=0)

    def call(x=None, b=None, d=None, idx=BASE, table=BASE, start=BASE, lens=BASE, q=BASE, w=None,
             sel=BASE, rec=BASE, slen=BASE, ws=BASE, n=1 << 40):
        return status(hs.hisparse_select_records, x or index(), b or batch(), d or select(), idx,
                      table, start, lens, q, w, sel, rec, slen, ws, n)
    assert call(d=select(top_k=0)) == call(x=index(tokens_per_record=8)) == INVALID
    assert hs.hisparse_validate_select(keys, batch(), select(q_heads=129)) == INVALID
    assert call(idx=None) == call(q=None) == call(sel=None) == call(ws=None) == INVALID
    assert call(idx=BASE + 8) == call(ws=BASE + 8) == call(table=BASE + 2) == INVALID
    assert call(start=BASE + 1) == call(lens=BASE + 2) == call(q=BASE + 1) == INVALID
    assert call(sel=BASE + 2) == call(rec=BASE + 2) == call(slen=BASE + 2) == INVALID
    assert call(x=keys, w=BASE + 2) == INVALID
    assert call(w=BASE) == INVALID                                   # weights without keys
    assert call(d=select(last_records=0)) == INVALID                 # a length without the newest
    assert call(start=None, b=batch(total_tokens=5)) == INVALID
    assert call(n=0) == INVALID
    assert call(b=batch(total_tokens=1 << 30)) == UNSUPPORTED
    assert call(x=keys, b=batch(max_records=1 << 26)) == UNSUPPORTED
    assert call(x=index(kind=ref.KEYS, record_stride=4096, num_records=1 << 27)) == UNSUPPORTED
    assert hs.lib().hisparse_validate_select(None, None, None) == INVALID
    hs.hisparse_select_records(index(), batch(total_tokens=0), select(), None, None, BASE, None, None,
                               None, None, None, None, None, 0)


def test_select_workspace_covers_smaller_batches():
    for kind, t in ((ref.KEYS, 64), (ref.BOUNDS, 16), (ref.MEANS, 64)):
        x = index(kind=kind, tokens_per_record=t, record_stride=1 << 20)
        size = lambda n, r, h: hs.hisparse_select_workspace_bytes(  # noqa: E731
            x, batch(total_tokens=n, max_records=r, kv_heads=h, tokens_per_record=t), select())
        most = size(700, 8192, 4)
        assert 0 < most
        for n, r, h in ((700, 8192, 1), (1, 8192, 4), (699, 1, 4), (3, 100, 2), (0, 1, 1)):
            got = size(n, r, h)
            assert 0 < got <= most, (kind, n, r, h)


def test_structs_have_the_header_s_sizes():
    assert ctypes.sizeof(hs.BatchDesc) == 40 and ctypes.sizeof(hs.RotaryDesc) == 64
    assert ctypes.sizeof(hs.RotaryRows) == 80 and ctypes.sizeof(hs.IndexDesc) == 40
    assert ctypes.sizeof(hs.SelectDesc) == 24
