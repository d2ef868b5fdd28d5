"""The calls before the attention together with the ones they stand beside, as a server uses them: batches
planned from their lengths, rows turned and written, index rows kept, records chosen and attended to. Each
call is checked against its 64-bit reference, on what the calls before it left; steps are eager calls and
replays of one captured graph in turn.

Tolerances: rotated rows as in test_gpu_rotary (one rounding to bf16, 2^-8, and 2^-20 of the pair for the
sums in fp32), attention as derived in token_reference.check, means as in test_gpu_summarize; everything
else is exact."""
import math

import pytest
import torch

import step_reference as ref
import token_reference as tok
from paper_2608_07009_amd import HiSparseCache, hisparse as hs

pytestmark = pytest.mark.gpu
G, L, BF, F8 = tok.GROUPED, tok.LATENT, tok.BF16, tok.FP8


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def fill(shape, value, dtype=torch.int32):
    return torch.full(shape, value, dtype=dtype, device="cuda")


def rows(x, y, first=0, out_rows=None):
    """[tokens][heads][dims] views."""
    return hs.RotaryRows(x.data_ptr(), y.data_ptr(), None if out_rows is None else out_rows.data_ptr(),
                         y.shape[0] if out_rows is not None else 0, x.stride(0), x.stride(1), y.stride(0),
                         y.stride(1), x.shape[1], x.shape[2], first)


def near(got, d, pos, x, first):
    want, size = ref.rotate(d, pos, x, first)
    tol = want.abs() * 2.0 ** -8 + size * 2.0 ** -20
    assert bool(((got.double() - want).abs() <= tol).all())


def run_steps(step, steps, before, after):
    """Eager calls and replays of a captured graph in turn."""
    graph, side = None, torch.cuda.Stream()
    for i, s in enumerate(steps):
        before(s)
        torch.cuda.synchronize()
        if i % 2 == 0:
            step()
        else:
            if graph is None:
                graph = torch.cuda.CUDAGraph()
                with torch.cuda.graph(graph, stream=side):
                    step()
            graph.replay()
        torch.cuda.synchronize()
        after(s)


@pytest.mark.parametrize("kind,type_", [(ref.BOUNDS, BF), (ref.MEANS, BF), (ref.BOUNDS, F8), (ref.MEANS, F8)])
def test_pages_chosen_by_their_index_rows(kind, type_):
    """Prompts, chunks, drafted and single tokens of four requests over one pool of pages; every new token
    attends to the pages chosen for it."""
    t, heads, q_heads, k, R, per, total, max_chunk = 16, 2, 3, 5, 4, 20, 200, 120
    H = heads * q_heads
    gen = torch.Generator().manual_seed(kind + 10 * type_)
    records = R * per - 8
    rb = hs.hisparse_kv_record_bytes(G, type_, t)
    kv = hs.KvDesc(G, type_, t, rb, records, heads * rb, rb, 0)
    pool = fill((records, heads, rb), 0xFF, torch.uint8)  # NaN
    n_rows = ref.INDEX_ROWS[kind]
    index = fill((records, heads, n_rows, 128), math.nan, torch.bfloat16)
    x = hs.IndexDesc(kind, t, records, 2 * index.stride(0), 2 * index.stride(1), 0)
    free = torch.randperm(records, generator=gen).int().cuda()
    used, table = ints([0]), fill((R, per), -1)
    new_len, kv_len, start = ints([0] * R), ints([0] * R), ints([0] * (R + 1))
    pos, slots = fill((total,), 0), fill((total,), -1, torch.int64)
    b = hs.BatchDesc(R, heads, total, max_chunk, per, t, per, 0)
    width = (H + 2 * heads) * 128
    qkv = torch.zeros((total, width), dtype=torch.bfloat16, device="cuda")
    q, keys = (qkv[:, a:c].unflatten(1, (-1, 128)) for a, c in ((0, H * 128), (H * 128, (H + heads) * 128)))
    values = qkv[:, (H + heads) * 128:]
    rot = hs.RotaryDesc(64, hs.HISPARSE_ROTARY_HALF, hs.HISPARSE_ROTARY_BY_PARTS, 0, 1e4, 8.0, 4096.0, 1.0,
                        32.0, 1.0)
    turned = (hs.RotaryRows * 2)(rows(q, q, 64), rows(keys, keys, 64))
    d = hs.SelectDesc(q_heads, k, 1, 2, width)
    sel, rec = fill((total, heads, k), -7), fill((total, heads, k), -7)
    slen = fill((total,), 0)
    ws = fill((hs.hisparse_select_workspace_bytes(x, b, d),), 0xEE, torch.uint8)
    scale = 1 / math.sqrt(128)
    chunk = hs.ChunkDesc(total, heads, q_heads, total, 1, k, width, H * 128, heads * k, k, 0, 0, scale,
                         hs.HISPARSE_CHUNK_CAUSAL)
    out = torch.zeros((total, H, 128), dtype=torch.bfloat16, device="cuda")
    ws2 = fill((max(16, hs.hisparse_chunk_workspace_bytes(kv, chunk)),), 0xEE, torch.uint8)

    def step():
        s = torch.cuda.current_stream()
        slen.zero_()
        hs.hisparse_plan_tokens(b, new_len, kv_len, free, records, used, table, start, kv_len, used, pos,
                                slots, s)
        hs.hisparse_rotate_tokens(rot, total, pos, turned, 2, s)
        hs.hisparse_write_tokens(kv, heads, total, keys, width, values, width, slots, pool, s)
        hs.hisparse_summarize_records(kv, x, b, pool, table, start, kv_len, index, s)
        hs.hisparse_select_records(x, b, d, index, table, start, kv_len, q, None, sel, rec, slen, ws,
                                   ws.numel(), s)
        hs.hisparse_chunk_attention(kv, chunk, pool, rec, None, slen, q, out, None, ws2, ws2.numel(), s)

    cached = [0] * R
    raw = torch.zeros((total, width), dtype=torch.bfloat16)
    stored = [([], []) for _ in range(R)]  # rows [heads][128] that each request's tokens are read back as
    expected_table = [[-1] * per for _ in range(R)]
    taken = [0]

    def before(new):
        raw.copy_(torch.randn((total, width), generator=gen))
        qkv.copy_(raw)
        new_len.copy_(ints(new))

    def after(new):
        want = ref.plan(new, cached, t, max_chunk, per, total, free.tolist(), taken[0], expected_table)
        got = [y.tolist() for y in (start, kv_len, used, pos, slots)]
        assert got == [want[0], want[1], [want[2]], want[3], want[4]]
        assert table.tolist() == expected_table
        cached[:], taken[0] = want[1], want[2]
        h_q, h_k, h_v = q.cpu(), keys.cpu(), values.cpu().unflatten(1, (heads, 128))
        p = pos.cpu()
        near(h_q, rot, p, raw[:, :H * 128].unflatten(1, (-1, 128)), 64)
        near(h_k, rot, p, raw[:, H * 128:(H + heads) * 128].unflatten(1, (-1, 128)), 64)
        sk, sv, _ = tok.stored(G, h_k, h_v, type_)
        h_index, h_sel, h_rec = index.cpu(), sel.cpu(), rec.cpu()
        h_slen, h_out = slen.tolist(), out.cpu()
        for r in range(R):
            for row in range(want[0][r], want[0][r + 1]):
                stored[r][0].append(sk[row])
                stored[r][1].append(sv[row])
            if not cached[r]:
                continue
            kr, vr = torch.stack(stored[r][0]), torch.stack(stored[r][1])  # [tokens][heads][128]
            pages = (cached[r] + t - 1) // t
            tab = torch.tensor(expected_table[r][:pages])
            for j in range(pages):
                part = kr[j * t:(j + 1) * t].transpose(0, 1)
                got = h_index[tab[j]].double()
                if kind == ref.BOUNDS:
                    assert torch.equal(got, torch.stack((part.amin(1), part.amax(1)), 1))
                else:
                    m = part.mean(1)
                    tol = m.abs() * (2.0 ** -8 + 2.0 ** -23) + part.abs().sum(1) * 2.0 ** -24
                    assert bool(((got[:, 0] - m).abs() <= tol).all())
            for row in range(want[0][r], want[0][r + 1]):
                at = want[3][row]
                seen = at // t + 1
                K = min(k, seen)
                assert h_slen[row] == (K - 1) * t + at % t + 1
                for h in range(heads):
                    hh = slice(h * q_heads, (h + 1) * q_heads)
                    best = ref.select_row(kind, h_q[row, hh], None, h_index[tab[:seen], h],
                                          torch.ones(seen, dtype=torch.bool), k, 1, 2)
                    assert h_sel[row, h].tolist() == best
                    assert h_rec[row, h].tolist() == [tab[j].item() if j >= 0 else -1 for j in best]
                    see = torch.cat([torch.arange(j * t, min((j + 1) * t, at + 1)) for j in best if j >= 0])
                    e = tok.attend(G, kr[see, h], vr[see, h], h_q[row:row + 1, hh],
                                   torch.ones((1, len(see)), dtype=torch.bool), scale)
                    tok.check(G, h_out[row:row + 1, hh], None, e, f"row {row} head {h}")

    run_steps(step, [[70, 33, 0, 97], [1, 20, 5, 1], [1, 1, 1, 1], [0, 1, 3, 1], [120, 0, 40, 40], [1, 1, 1, 1],
                     [4, 5, 6, 0], [1, 1, 1, 1]], before, after)


def test_tokens_chosen_by_their_index_keys():
    """Decoding over a cache of latent records: the new token's record appended, its index key written to
    the row of its position, tokens chosen by their keys, resolved, fetched and attended to."""
    R, q_heads, i_heads, k, B, cap, prompt = 3, 16, 4, 24, 40, 128, 70
    gen = torch.Generator().manual_seed(5)
    rb = hs.hisparse_kv_record_bytes(L, BF, 1)
    scale = 1 / math.sqrt(576)
    rot = hs.RotaryDesc(64, hs.HISPARSE_ROTARY_INTERLEAVED, hs.HISPARSE_ROTARY_PLAIN, 0, 1e4, 1.0, 0.0, 0.0,
                        0.0, 1.0)
    b = hs.BatchDesc(R, 1, R, 1, cap, 1, cap, 0)
    x = hs.IndexDesc(ref.KEYS, 1, cap, 256, 0, cap * 256)
    d = hs.SelectDesc(i_heads, k, 0, 1, i_heads * 128)
    table = torch.arange(R * cap, dtype=torch.int32, device="cuda").view(R, cap)
    index = fill((R * cap, 1, 128), math.nan, torch.bfloat16)
    new_len, kv_len, start = ints([1] * R), ints([prompt, prompt - 60, prompt + 9]), ints([0] * (R + 1))
    pos, slots = fill((R,), 0), fill((R,), -1, torch.int64)
    bf = lambda *s: torch.zeros(s, dtype=torch.bfloat16, device="cuda")  # noqa: E731
    q, latent, rope, iq, ik = bf(R, q_heads, 576), bf(R, 1, 512), bf(R, 1, 64), bf(R, i_heads, 128), bf(R, 1, 128)
    w = torch.zeros((R, i_heads), device="cuda")
    turned = (hs.RotaryRows * 4)(rows(q, q, 512), rows(rope, rope), rows(iq, iq, 64),
                                 rows(ik, index, 64, slots))
    one = hs.KvDesc(L, BF, 1, rb, R, rb, 0, 0)
    record = fill((1, R, rb), 0, torch.uint8)
    sel, slot, new_slot = fill((R, 1, k), -7), fill((R, k), -7), fill((1, R), -7)
    ws = fill((hs.hisparse_select_workspace_bytes(x, b, d),), 0xEE, torch.uint8)
    attn = hs.AttnDesc(q_heads, 576, 512, 0, 1, 0, scale, 0)
    out = torch.zeros((R, q_heads, 512), device="cuda")
    ws2 = fill((max(16, hs.hisparse_decode_workspace_bytes(R, k, rb, attn)),), 0xEE, torch.uint8)
    with HiSparseCache(num_requests=R, num_layers=1, units_per_request=1, capacity=B, num_records=cap, top_k=k,
                       record_bytes=rb) as cache:
        # the prompts
        lat = torch.randn((R, cap, 512), generator=gen).to(torch.bfloat16)
        rop = torch.randn((R, cap, 64), generator=gen).to(torch.bfloat16)
        idx = torch.randn((R, cap, 128), generator=gen).to(torch.bfloat16)
        have = kv_len.tolist()
        hs.hisparse_stage(cache.handle, 0, 1, 0, R, 0, cap, torch.cat((lat, rop), 2).cuda(), 0,
                          torch.cuda.current_stream())
        for r in range(R):
            index[r * cap:r * cap + have[r], 0] = idx[r, :have[r]].cuda()

        def step():
            s = torch.cuda.current_stream()
            hs.hisparse_plan_tokens(b, new_len, kv_len, None, 0, None, table, start, kv_len, None, pos, slots, s)
            hs.hisparse_rotate_tokens(rot, R, pos, turned, 4, s)
            hs.hisparse_write_tokens(one, 1, R, latent, 512, rope, 64, None, record, s)
            hs.hisparse_append(cache.handle, 0, 1, pos, record, new_slot, s)
            hs.hisparse_select_records(x, b, d, index, None, start, kv_len, iq, w, sel, None, None, ws,
                                       ws.numel(), s)
            hs.hisparse_resolve(cache.handle, 0, sel, slot, None, s)
            hs.hisparse_sparse_decode(cache.handle, 0, q, slot, out, attn, ws2, ws2.numel(), s)

        raw = {}

        def before(_):
            for name, y in (("q", q), ("latent", latent), ("rope", rope), ("iq", iq), ("ik", ik)):
                raw[name] = torch.randn(y.shape, generator=gen).to(torch.bfloat16)
                y.copy_(raw[name])
            raw["w"] = torch.randn((R, i_heads), generator=gen) + 0.3
            w.copy_(raw["w"])

        def after(i):
            p = pos.cpu()
            assert p.tolist() == [n + i for n in have] and kv_len.tolist() == [n + i + 1 for n in have]
            assert slots.tolist() == [r * cap + p[r].item() for r in range(R)]
            h_index = index.cpu().view(R, cap, 128)
            h_q, h_rope, h_iq = q.cpu(), rope.cpu(), iq.cpu()
            near(h_q, rot, p, raw["q"], 512)
            near(h_rope, rot, p, raw["rope"], 0)
            near(h_iq, rot, p, raw["iq"], 64)
            near(torch.stack([h_index[r, p[r]] for r in range(R)])[:, None], rot, p, raw["ik"], 64)
            h_sel, h_out = sel.cpu(), out.cpu()
            for r in range(R):
                at = p[r].item()
                lat[r, at], rop[r, at], idx[r, at] = raw["latent"][r, 0], h_rope[r, 0], h_index[r, at]
                assert torch.equal(h_index[r, :at + 1], idx[r, :at + 1])
                best = ref.select_row(ref.KEYS, h_iq[r], raw["w"][r], idx[r, :at + 1, None],
                                      torch.ones(at + 1, dtype=torch.bool), k, 0, 1)
                assert h_sel[r, 0].tolist() == best
                j = torch.tensor([y for y in best if y >= 0])
                e = tok.attend(L, lat[r, j].double(), rop[r, j].double(), h_q[r:r + 1],
                               torch.ones((1, len(j)), dtype=torch.bool), scale)
                tok.check(L, h_out[r:r + 1], None, e, f"step {i} request {r}")
            assert cache.check_errors()[0] == hs.HISPARSE_OK

        run_steps(step, list(range(40)), before, after)
