"""Every kind of workgroup of attention on A2T_MX4 caches, forced and checked by the name its launches
are timed under, against the float64 oracle: one stream, uneven streams with key splits, and values of V that
fp16 does not hold."""
import numpy as np
import pytest

from oracle import mx4
from synth.streams import SEG_ACOUSTIC, SEG_DELIM, SEG_RESPONSE, SEG_TEXT, bf16_round, tiny_stream
from tests.mx4_sessions import Sessions

pytestmark = pytest.mark.gpu

NAMES = {16: "attn_mx4", 32: "attn_mx4x2", 48: "attn_mx4x3", 64: "attn_mx4_rows64", 128: "attn_mx4_rows128"}
SMALL = [SEG_ACOUSTIC] * 7 + [SEG_DELIM, SEG_TEXT, SEG_TEXT, SEG_DELIM]


def _unit(n):
    return [SEG_TEXT if r % 9 == 4 else SEG_ACOUSTIC for r in range(n)]


def launches(a2t, c):
    """{query rows of a workgroup: launches} since the last report."""
    out = {rows: a2t.a2t_kernel_time(c, name)[0] for rows, name in sorted(NAMES.items(), reverse=True)}   # "attn_mx4" last
    return {rows: n for rows, n in out.items() if n}


def force(monkeypatch, rows, splits=None):
    monkeypatch.setenv("A2T_MX4_ROWS", str(rows))
    if splits:
        monkeypatch.setenv("A2T_SPLITS", str(splits))


def drive(specs, rows, hq, hkv, d, **kw):
    import paper_2609_31224_amd as a2t
    s = Sessions(specs, hq, hkv, d, calls="fused", layers=1, **kw)
    try:
        a2t.a2t_profile_enable(s.cache, "attn_mx4")
        s.run()
        assert set(launches(a2t, s.cache)) == {rows}
    finally:
        s.close()
    print(f"worst error {s.worst:.3f} of its bound, {s.evictions} evictions", flush=True)
    return s


@pytest.mark.parametrize("d,hq,hkv", [(64, 8, 2), (128, 4, 2)])
@pytest.mark.parametrize("rows", list(NAMES))
def test_one_stream(gpu, monkeypatch, rows, d, hq, hkv):
    """Steps of 1 to 73 rows (2 to 292 query rows of a KV head, so groups that end inside a block), a ring that wraps, a
    kept region."""
    force(monkeypatch, rows)
    steps = [SMALL, _unit(73), SMALL, [SEG_RESPONSE], _unit(16), _unit(31), SMALL, _unit(64)]
    s = drive([tiny_stream(steps, prefix=300)], rows, hq, hkv, d, budgets=[340], unit_rows=400)
    assert s.evictions >= 3


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("rows,splits", [(16, 3), (32, 2), (32, None), (48, 3), (48, None), (64, 4), (64, None), (128, 2), (128, 5), (128, None)])
def test_uneven_streams(gpu, monkeypatch, rows, splits, d):
    """Streams of 1 to 90 rows onto 0 to 1,300 keys in one launch, split or not."""
    force(monkeypatch, rows, splits)
    specs = [tiny_stream([*more, SMALL, _unit(n), _unit(m)], prefix=p)
             for n, m, p, more in ((90, 5, 600, [_unit(700)]), (1, 33, 5, [[SEG_ACOUSTIC]]), (64, 1, 0, [_unit(64)]), (17, 90, 257, [SMALL]))]
    drive(specs, rows, 4, 2, d, budgets=[100000] * 4, query_rows=90, unit_rows=1700)


@pytest.mark.parametrize("exps", [[-40, 0, 0, 0], [-26, -24, -23, -22, -12, 0], [10, 12, 13, 14, 0], [-110, -20, 0, 0, 0, 100]])
@pytest.mark.parametrize("d,hq,hkv,new", [(64, 8, 2, 25), (128, 4, 1, 40)])
@pytest.mark.parametrize("rows", list(NAMES))
def test_scales_of_values_apart(gpu, monkeypatch, rows, d, hq, hkv, new, exps):
    """Blocks of V within and outside the scales that fp16 holds, and blocks of zeros; every output element within
    its own bound."""
    import torch
    import paper_2609_31224_amd as a2t
    force(monkeypatch, rows, 1)
    rng = np.random.default_rng(11)
    old = 520
    n = old + new
    scale = np.repeat(2.0 ** rng.choice(exps, (n, hkv, d // 32)), 32, -1) * np.repeat(rng.random((n, hkv, d // 32)) < 0.9, 32, -1)
    k, v, q = (bf16_round(rng.standard_normal((m, h, d))) for m, h in ((n, hkv), (n, hkv), (new, hq)))
    v = bf16_round(v * scale)
    kd, vd, qd = (torch.from_numpy(np.ascontiguousarray(x, np.float32)).cuda().bfloat16() for x in (k, v, q))
    seg = np.full(n, SEG_ACOUSTIC, np.uint8)
    c = a2t.a2t_cache_create(1, 1, hq, hkv, d, a2t.A2T_MX4, n, 0, old)
    ref = mx4.OracleMx4Cache(hq, hkv, d, [0], theta=1e6)
    o = torch.full_like(qd, float("nan"))
    a2t.a2t_append(c, 0, [0], [old], kd[:old], vd[:old], seg[:old], np.arange(old), [0])
    a2t.a2t_profile_enable(c, "attn_mx4")
    a2t.a2t_append_attn(c, 0, [0], [new], kd[old:], vd[old:], seg[old:], np.arange(old, n), [1], [new], qd, o)
    assert launches(a2t, c) == {rows: 1}
    a2t.a2t_cache_destroy(c)
    for unit, part in enumerate((slice(0, old), slice(old, n))):
        ref.append(seg[part], np.arange(n)[part], unit, {0: k[part]}, {0: v[part]})
    want, bound = ref.attention_bound(0, q, new, least=0.0)
    off = np.abs(o.float().cpu().numpy().astype(np.float64) - want) - bound
    assert np.isfinite(off).all() and (off <= 0).all(), (float(off.max()), np.unravel_index(off.argmax(), off.shape))


@pytest.mark.parametrize("streams,rows,resident,kind", [(3, 1, 100, 16), (1, 22, 4096, 32), (16, 22, 4096, 48), (1, 1024, 0, 64), (1, 1024, 4096, 128)])
def test_planned_kinds(gpu, streams, rows, resident, kind):
    """Every kind is what some launch on the whole GPU is planned with."""
    import torch
    import paper_2609_31224_amd as a2t
    hq, hkv, d = 32, 8, 128
    c = a2t.a2t_cache_create(1, streams, hq, hkv, d, a2t.A2T_MX4, resident + rows, 0, 1024)
    a2t.a2t_profile_enable(c, "attn_mx4")
    for at in [*range(0, resident, 1024), resident]:
        n = min(1024, resident - at) if at < resident else rows
        k = torch.zeros((1, n * streams, hkv, d), dtype=torch.bfloat16, device="cuda")
        a2t.a2t_append(c, a2t.A2T_ALL_LAYERS, range(streams), [n] * streams, k, k, np.full(n * streams, SEG_ACOUSTIC, np.uint8),
                       np.tile(np.arange(at, at + n), streams), [at] * streams)
    q = torch.zeros((streams * rows, hq, d), dtype=torch.bfloat16, device="cuda")
    o = torch.full_like(q, float("nan"))
    a2t.a2t_chunk_attn(c, 0, range(streams), [rows] * streams, q, o)
    assert launches(a2t, c) == {kind: 1}
    assert (o == 0).all()
    a2t.a2t_cache_destroy(c)
