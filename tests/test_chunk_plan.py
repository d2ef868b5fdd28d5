"""The host's plan of hisparse_chunk_attention, without a GPU."""
import os
import random
import shutil
import subprocess

import pytest

import token_reference as ref
from paper_2608_07009_amd import hisparse as hs

G, L = ref.GROUPED, ref.LATENT
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def workspace(kind, tpr, kv_heads, q_heads, requests, total, chunk, records, window=0, splits=0):
    rb = hs.hisparse_kv_record_bytes(kind, hs.HISPARSE_KV_FP8, tpr)
    kv = hs.KvDesc(kind, hs.HISPARSE_KV_FP8, tpr, rb, 1 << 20, rb, rb, 0)
    H = kv_heads * q_heads
    c = hs.ChunkDesc(requests, kv_heads, q_heads, total, chunk, records, H * ref.D_QK[kind],
                     H * ref.D_V[kind], records, 0, window, splits, 0.1, hs.HISPARSE_CHUNK_CAUSAL)
    if hs.hisparse_validate_chunk(kv, c) != hs.HISPARSE_OK:
        return None
    return hs.hisparse_chunk_workspace_bytes(kv, c)


def test_a_batch_one_smaller_needs_no_more():
    """32 requests of 8 kv heads x 4 with up to 600 cached tokens fill the CUs, 31 do not."""
    big, small = (workspace(G, 1, 8, 4, n, n, 1, 600) for n in (32, 31))
    assert small > 0 and big >= small


@pytest.mark.parametrize("kind", [G, L])
@pytest.mark.parametrize("splits", [0, 1, 5])
def test_a_workspace_serves_every_smaller_batch(kind, splits):
    g = random.Random(17 * kind + splits)

    def up_to(most):
        return max(1, min(most, int(2 ** g.uniform(0, most.bit_length()))))

    for _ in range(4000):
        kv_heads, q_heads = up_to(300 if g.random() < 0.1 else 16), up_to(256)
        tpr, window = g.choice((1, 16, 64)), g.choice((0, 0, up_to(5000)))
        requests, chunk, records = up_to(2000), up_to(5000), up_to(40000 // tpr)
        total = up_to(2 * requests * chunk)
        small = [g.choice((x, x, max(1, x - 1), up_to(x))) for x in (requests, total, chunk, records)]
        a = workspace(kind, tpr, kv_heads, q_heads, requests, total, chunk, records, window, splits)
        if a is None:  # more than one launch takes
            continue
        b = workspace(kind, tpr, kv_heads, q_heads, *small, window, splits)
        assert b is not None and b <= a, (kv_heads, q_heads, tpr, window, (requests, total, chunk, records), small)


def check_plans(tmp_path, name, *flags):
    exe = str(tmp_path / name)
    subprocess.check_call(["g++", "-std=c++17", "-O2", *flags, "-I", os.path.join(ROOT, "include"),
                           "-I", os.path.join(ROOT, "paper_2608_07009_amd", "csrc"),
                           os.path.join(ROOT, "tests", "chunk_plan_check.cc"), "-o", exe])
    r = subprocess.run([exe], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and r.stdout.startswith("ok"), r.stdout + r.stderr[-3000:]
    return r.stdout


@pytest.mark.skipif(shutil.which("g++") is None, reason="needs g++")
def test_what_the_device_finds_fits_the_host_s_bounds(tmp_path):
    """Random batches, with the arithmetic checked for overflow."""
    out = check_plans(tmp_path, "plain", "-fsanitize=undefined", "-fno-sanitize-recover=all")
    assert int(out.split()[1]) > 10000


@pytest.mark.skipif(shutil.which("g++") is None, reason="needs g++")
@pytest.mark.skipif("fma" not in open("/proc/cpuinfo").read(), reason="needs a CPU with FMA")
def test_parts_do_not_depend_on_how_the_compiler_contracts(tmp_path):
    """The attention and the merge are compiled apart and each works out the parts."""
    assert (check_plans(tmp_path, "off", "-mfma", "-ffp-contract=off")
            == check_plans(tmp_path, "fast", "-mfma", "-ffp-contract=fast", "-O3"))
