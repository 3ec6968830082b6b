"""GPU parity of A2T_MX4 caches (rows held in 4 bits) against the float64 oracle: encoded rows
and rows read back exactly, attention within a bound that the oracle derives from the
roundings it is computed with.  Query rows around the 16-row blocks and the workgroups of one to
three blocks, key counts around the 32-key blocks, both head dims, one to eight query heads
per KV head, rings that wrap, kept regions, every eviction rule, key splits, batches.
"""
import numpy as np
import pytest

from oracle import mx4
from synth.streams import SEG_ACOUSTIC, SEG_DELIM, SEG_RESPONSE, SEG_TEXT, bf16_round, tiny_stream
from tests.harness import bf16_bits_to_f32
from tests.mx4_sessions import Sessions

pytestmark = pytest.mark.gpu

SMALL = [SEG_ACOUSTIC] * 7 + [SEG_DELIM, SEG_TEXT, SEG_TEXT, SEG_DELIM]


def _unit(n):
    return [SEG_TEXT if r % 9 == 4 else SEG_ACOUSTIC for r in range(n)]


def _run(*a, **kw):
    s = Sessions(*a, **kw)
    try:
        s.run()
    finally:
        s.close()
    print(f"worst error {s.worst:.3f} of its bound, {s.evictions} evictions", flush=True)
    return s


@pytest.mark.parametrize("d", [64, 128])
def test_one_row(gpu, d):
    """The smallest calls: one row of one head, then two, three rows by decode steps."""
    _run([tiny_stream([[SEG_ACOUSTIC], [SEG_RESPONSE], [SEG_RESPONSE]])], 1, 1, d, budgets=[100], layers=1)


@pytest.mark.parametrize("hq,hkv,d,rows,prefix,splits,calls,query_rows", [
    (8, 1, 128, 2, 15, None, "separate", None),     # 16 query rows: one block
    (4, 1, 64, 17, 64, "1", "fused", None),         # 68: two groups of three blocks
    (4, 1, 128, 17, 31, "2", "separate", None),
    (16, 16, 128, 33, 700, None, "all", None),      # 33: three blocks
    (32, 8, 64, 22, 900, None, "fused", None),      # 88: two groups of three
    (32, 8, 128, 22, 900, None, "fused", 5),        # the last 5 of 22 rows query: two blocks
    (6, 3, 128, 40, 130, "5", "noalloc", None),     # 80: two groups of three
    (8, 1, 64, 16, 130, "3", "noalloc", None),      # 128: three groups of three
    (2, 2, 64, 90, 3, "128", "separate", None),     # more splits asked for than tiles
    (8, 2, 128, 61, 0, "4", "all", None),           # 244: six groups of three
])
def test_chunks(gpu, monkeypatch, hq, hkv, d, rows, prefix, splits, calls, query_rows):
    if splits:
        monkeypatch.setenv("A2T_SPLITS", splits)
    spec = tiny_stream([SMALL, _unit(rows), SMALL, [SEG_RESPONSE], _unit(rows), _unit(rows + 1), SMALL, _unit(rows)], prefix=prefix)
    s = _run([spec], hq, hkv, d, budgets=[prefix + rows + 20], calls=calls, query_rows=query_rows,
             unit_rows=max(2 * rows + 40 + prefix, 80))
    assert s.evictions >= 3


@pytest.mark.parametrize("keys", [1, 2, 31, 32, 33, 63, 64, 65, 255, 256, 257, 300])
@pytest.mark.parametrize("d", [64, 128])
def test_key_counts(gpu, d, keys):
    """Blocks that end anywhere: `keys` resident rows, then steps of one, one and three rows."""
    _run([tiny_stream([[SEG_ACOUSTIC], [SEG_RESPONSE], [SEG_ACOUSTIC] * 3], prefix=keys)], 4, 2, d, budgets=[1000], layers=1)


@pytest.mark.parametrize("rule,n_sink", [("unit", 0), ("row", 0), ("sink_recent", 3)])
@pytest.mark.parametrize("d", [64, 128])
def test_rules(gpu, d, rule, n_sink):
    """Every eviction rule moves the encoded rows it keeps."""
    spec = tiny_stream([SMALL, _unit(20), SMALL, _unit(30), [SEG_RESPONSE], SMALL, _unit(25), SMALL], prefix=2 if rule != "sink_recent" else 0)
    s = _run([spec], 4, 2, d, budgets=[50], window=1 if rule != "sink_recent" else 0, rule=rule, n_sink=n_sink, unit_rows=110)
    assert s.evictions >= 3


@pytest.mark.parametrize("d,hq,hkv", [(128, 8, 2), (64, 8, 8)])
def test_batches(gpu, d, hq, hkv):
    """Streams of unequal length that join and leave, in one launch."""
    specs = [tiny_stream([_unit(n), SMALL, [SEG_RESPONSE], _unit(m), SMALL], prefix=p)
             for n, m, p in ((3, 40, 0), (22, 1, 300), (90, 22, 17), (1, 1, 0), (64, 64, 700))]
    s = _run(specs, hq, hkv, d, budgets=[40, 200, 90, 20, 720], calls="fused", offsets=[0, 2, 1, 0, 3])
    assert s.evictions >= 5


def test_many_streams(gpu):
    """More streams than one launch describes."""
    specs = [tiny_stream([[SEG_ACOUSTIC] * (1 + i % 5), [SEG_RESPONSE]], prefix=1 + i % 37) for i in range(70)]
    _run(specs, 2, 1, 64, budgets=[30] * 70, layers=1)


def test_far_positions(gpu):
    """Positions near the largest one, a non-default theta and gaps between steps."""
    spec = tiny_stream([SMALL, [SEG_RESPONSE], _unit(9)], prefix=40, start_pos=2**31 - 400, pos_gap=50)
    _run([spec], 4, 1, 128, budgets=[30], theta=1e4)


@pytest.mark.parametrize("scale", [1e-30, 1e-3, 300.0])
def test_value_ranges(gpu, scale):
    """Scores from all alike to one-hot, and rows whose scales are at the ends."""
    _run([tiny_stream([SMALL, _unit(20), [SEG_RESPONSE]], prefix=70)], 4, 2, 128, budgets=[200], kv_scale=scale)


# ------------------------------------------------------------------ encoding
def _append_read(a2t, k, v, pos=None, d=None):
    import torch
    n, h, d = k.shape
    c = a2t.a2t_cache_create(1, 1, h, h, d, a2t.A2T_MX4, n, 0, n)
    kd, vd = (torch.from_numpy(np.ascontiguousarray(x, np.float32)).cuda().to(torch.bfloat16) for x in (k, v))
    a2t.a2t_append(c, 0, [0], [n], kd, vd, np.full(n, SEG_ACOUSTIC, np.uint8), np.arange(n) if pos is None else pos, [0])
    out = a2t.a2t_read_kv(c, 0, 0)
    back = [torch.zeros_like(kd) for _ in range(2)]
    a2t.a2t_read_rows(c, 0, [0], *back)
    a2t.a2t_sync(c)
    for x, y in zip(out, back):
        assert np.array_equal(x, y.view(torch.int16).cpu().numpy().view(np.uint16))
    a2t.a2t_cache_destroy(c)
    return [bf16_bits_to_f32(x) for x in out]


@pytest.mark.parametrize("d", [64, 128])
def test_encoding_of_every_bf16_value(gpu, d):
    """Every finite bf16 number, alone in its block and beside larger ones: blocks hold one
    number x, its successors and 0, or x and a larger power of two."""
    bits = np.arange(0x7f80, dtype=np.uint32)
    x = (bits << 16).view(np.float32)
    rows = np.zeros((len(x), d), np.float32)
    rows[:, 0::7] = x[:, None] * np.where(np.arange(0, d, 7) % 2, -1, 1)
    rows[:, 3::8] = np.roll(x, 1)[:, None]
    rows[:, 32] = np.minimum(np.ldexp(1.0, np.frexp(x)[1] + 3), 2.0 ** 127)
    rows = bf16_round(rows).reshape(-1, 4, d)
    for at in range(0, len(rows), 1024):
        part = rows[at:at + 1024]
        if len(part) == 0:
            continue
        k, v = _append_read(__import__("paper_2609_31224_amd"), np.zeros_like(part), part)
        assert np.array_equal(v, mx4.hold(part)), at
        assert not k.any()


def test_borders(gpu):
    """Halfway cases go to the even code, from both sides, at many scales."""
    import paper_2609_31224_amd as a2t
    ties = np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0])
    near = np.concatenate([ties, ties * (1 - 2.0 ** -7), ties * (1 + 2.0 ** -7)])
    block = np.zeros(32)
    block[:21], block[21], block[22:29] = near, 6.0, -ties
    rows = np.stack([np.concatenate([block * 2.0 ** e, -block * 2.0 ** (e + 1)]) for e in range(-100, 101, 5)])[:, None]
    rows = bf16_round(rows)
    k, v = _append_read(a2t, np.zeros_like(rows), rows)
    want = mx4.hold(rows)
    assert np.array_equal(v, want)
    assert np.array_equal(np.abs(want[20, 0, :7]), [0, 1, 1, 2, 2, 4, 4])    # e = 0


@pytest.mark.parametrize("d", [64, 128])
def test_blocks_that_are_not_finite(gpu, d):
    import paper_2609_31224_amd as a2t
    rng = np.random.default_rng(2)
    rows = bf16_round(rng.standard_normal((40, 2, d)))
    for r, bad in ((3, np.inf), (4, -np.inf), (5, np.nan)):
        rows[r, 1, 17] = bad
        rows[r + 10, 0, d - 1] = bad
    k, v = _append_read(a2t, rows, rows, pos=np.arange(40))
    want = mx4.hold(rows)
    assert np.array_equal(v, want, equal_nan=True)
    assert np.isnan(v[3, 1, :32]).all() and np.isfinite(v[3, 1, 32:]).all() and np.isfinite(v[3, 0]).all()
    # a key's infinity meets its partner too
    with np.errstate(invalid="ignore"):
        want = mx4.hold(mx4.rotate_to_f32(rows, np.arange(40), 1e6))
    assert np.array_equal(k, want, equal_nan=True)


# ------------------------------------------------------------------ values behind the mask
@pytest.mark.parametrize("splits", ["1", "3"])
@pytest.mark.parametrize("d,rows,bad,hq,hkv", [(64, 5, 4, 4, 2), (128, 22, 21, 4, 2), (128, 40, 17, 8, 1), (64, 33, 32, 2, 2)])
def test_masked_values_stay_out(gpu, monkeypatch, d, rows, bad, hq, hkv, splits):
    """Row `bad` of the step holds infinite and NaN values: every query row before it, which
    does not see it, comes out as if they were finite; the rows that see it do not."""
    import torch
    import paper_2609_31224_amd as a2t
    monkeypatch.setenv("A2T_SPLITS", splits)
    old = 150
    g = torch.Generator(device="cuda").manual_seed(3)
    k0, v0 = (torch.randn((old, hkv, d), generator=g, device="cuda").bfloat16() for _ in range(2))
    k, v, q = (torch.randn((rows, h, d), generator=g, device="cuda").bfloat16() for h in (hkv, hkv, hq))

    def run(spoil_k, spoil_v):
        vv, kk = v.clone(), k.clone()
        if spoil_v:
            vv[bad, :, 1] = float("inf")
            vv[bad, :, 40] = float("nan")
        if spoil_k:
            kk[bad, :, 3] = float("nan")
        c = a2t.a2t_cache_create(1, 1, hq, hkv, d, a2t.A2T_MX4, old + 2 * rows, 8, max(old, rows))
        o = torch.zeros_like(q)
        a2t.a2t_append(c, 0, [0], [old], k0, v0, np.full(old, SEG_ACOUSTIC, np.uint8), np.arange(old), [0])
        a2t.a2t_evict(c, [0], [10 * old], 1)
        a2t.a2t_append_attn(c, 0, [0], [rows], kk, vv, np.full(rows, SEG_ACOUSTIC, np.uint8), np.arange(old, old + rows), [1],
                            [rows], q, o)
        a2t.a2t_sync(c)
        a2t.a2t_cache_destroy(c)
        return o.float().cpu().numpy()

    clean = run(False, False)
    assert np.isfinite(clean).all()
    for kind in ((False, True), (True, False), (True, True)):
        got = run(*kind)
        assert np.array_equal(got[:bad], clean[:bad]), kind
        if kind[0]:
            assert np.isnan(got[bad:]).all(), kind
        else:   # the blocks of 32 dims that hold them, no others
            assert np.isnan(got[bad:, :, :64]).all() and np.array_equal(got[bad:, :, 64:], clean[bad:, :, 64:])


@pytest.mark.parametrize("d", [64, 128])
def test_query_that_is_not_finite(gpu, d):
    """Its own rows of the output are NaN, no others."""
    import torch
    import paper_2609_31224_amd as a2t
    rows = 20
    g = torch.Generator(device="cuda").manual_seed(4)
    k, v, q = (torch.randn((rows, h, d), generator=g, device="cuda").bfloat16() for h in (2, 2, 4))
    outs = []
    for spoil in (False, True):
        qq = q.clone()
        if spoil:
            qq[7, 1, 5] = float("nan")
            qq[8, 3, 6] = float("inf")
        c = a2t.a2t_cache_create(1, 1, 4, 2, d, a2t.A2T_MX4, rows, 0, rows)
        o = torch.zeros_like(q)
        a2t.a2t_append_attn(c, 0, [0], [rows], k, v, np.full(rows, SEG_ACOUSTIC, np.uint8), np.arange(rows), [0], [rows], qq, o)
        a2t.a2t_sync(c)
        a2t.a2t_cache_destroy(c)
        outs.append(o.float().cpu().numpy())
    bad = np.zeros((rows, 4), bool)
    bad[7, 1] = bad[8, 3] = True
    assert np.isnan(outs[1][bad]).all() and np.array_equal(outs[0][~bad], outs[1][~bad])


@pytest.mark.parametrize("d,hq,hkv,rows,prefix", [(64, 8, 1, 23, 40), (128, 4, 2, 37, 70), (128, 16, 4, 9, 500), (64, 2, 2, 65, 0)])
def test_small_workgroups(gpu, monkeypatch, d, hq, hkv, rows, prefix):
    """Workgroups of four waves (launches with more than two of them per CU: here one CU is
    counted), whole and with forced splits."""
    monkeypatch.setenv("A2T_TARGET_WGS", "1")
    for splits in ("0", "3"):
        monkeypatch.setenv("A2T_SPLITS", splits)
        spec = tiny_stream([SMALL, _unit(rows), [SEG_RESPONSE], _unit(rows + 2), SMALL], prefix=prefix)
        _run([spec], hq, hkv, d, budgets=[prefix + rows], calls="fused", unit_rows=2 * rows + 60 + prefix)
