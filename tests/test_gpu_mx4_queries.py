"""Attention on A2T_MX4 caches where the channels of queries and keys differ in size: a rotated query
is held as three 6-bit numbers an element, whose error the oracle's bound takes as 2^-14 of the largest element
of a block of 32 (two numbers, 2^-9 of it, exceed the bound: tests/test_mx4_queries_cpu.py)."""
import numpy as np
import pytest

from oracle import mx4
from synth.streams import SEG_ACOUSTIC
from tests.test_mx4_queries_cpu import uneven

pytestmark = pytest.mark.gpu


def attend_on(k, v, q, hq, hkv, d, rows, splits=None):
    """Outputs of the last `rows` of the rows k, v; one call (a decode call for one row)."""
    import torch
    import paper_2609_31224_amd as a2t
    up = lambda x: torch.from_numpy(np.ascontiguousarray(x, np.float32)).cuda().bfloat16()   # noqa: E731
    n = len(k)
    kd, vd, qd = up(k), up(v), up(q)
    c = a2t.a2t_cache_create(1, 1, hq, hkv, d, a2t.A2T_MX4, n, 0, 1024)
    old = n - rows
    for unit, at in enumerate(range(0, old, 1000)):
        part = slice(at, min(at + 1000, old))
        m = part.stop - part.start
        a2t.a2t_append(c, 0, [0], [m], kd[part], vd[part], np.full(m, SEG_ACOUSTIC, np.uint8), np.arange(at, part.stop), [unit])
    a2t.a2t_append(c, 0, [0], [rows], kd[old:], vd[old:], np.full(rows, SEG_ACOUSTIC, np.uint8), np.arange(old, n), [n])
    o = torch.full_like(qd, float("nan"))
    if rows == 1:
        a2t.a2t_decode_attn(c, 0, [0], qd, o)
    else:
        a2t.a2t_chunk_attn(c, 0, [0], [rows], qd, o)
    a2t.a2t_sync(c)
    a2t.a2t_cache_destroy(c)
    return o.float().cpu().numpy().astype(np.float64)


@pytest.mark.parametrize("wgs", [None, "1"])   # one workgroup counted: as for launches that fill the CUs
@pytest.mark.parametrize("hq,hkv,d,rows,n", [
    (8, 1, 128, 1, 700), (4, 4, 64, 1, 700),       # decode
    (4, 1, 128, 5, 600), (8, 2, 64, 12, 600),      # 20 and 48 query rows a KV head
    (4, 1, 128, 22, 600), (4, 1, 64, 22, 600),     # 88
    (2, 1, 128, 100, 2500), (4, 1, 64, 64, 2500),  # 200, 256
])
@pytest.mark.parametrize("q_spread,k_spread", [(1.0, 1.0), (20.0, 20.0), (100.0, 50.0)])
def test_uneven_channels(gpu, monkeypatch, hq, hkv, d, rows, n, q_spread, k_spread, wgs):
    if wgs:
        monkeypatch.setenv("A2T_TARGET_WGS", wgs)
    rng = np.random.default_rng(7)
    k, v, q = uneven(rng, n, rows, hq, hkv, d, q_spread, k_spread)
    got = attend_on(k, v, q, hq, hkv, d, rows)
    ref = mx4.OracleMx4Cache(hq, hkv, d, [0], theta=1e6)
    ref.append(np.full(n, SEG_ACOUSTIC), np.arange(n), 0, {0: k}, {0: v})
    want, bound = ref.attention_bound(0, q, rows)
    off = np.abs(got - want) / bound
    assert np.isfinite(off).all()
    print(f"worst error {off.max():.3f} of its bound, {np.linalg.norm(got - want) / np.linalg.norm(want):.5f} of the outputs", flush=True)
    assert off.max() <= 1.0
