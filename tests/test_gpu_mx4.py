"""GPU parity of A2T_MX4 caches (rows held in 4 bits) against the float64 oracle: encoded rows
and rows read back exactly, attention within a bound that the oracle derives from the
roundings it is computed with.  Query rows around the 16-row blocks and the workgroups of one to
three blocks and of 64 and 128 rows, key counts around the 32-key blocks, both head dims, one to eight query heads
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


@pytest.mark.parametrize("hq,hkv,d,rows,prefix,splits", [
    (8, 1, 128, 32, 0, None),      # 256 rows, few keys: 64 a workgroup
    (8, 1, 64, 24, 40, "2"),       # 192
    (4, 4, 128, 61, 500, "3"),     # 61 of 64
    (4, 2, 64, 30, 1700, "5"),     # 60 of 64
    (4, 4, 128, 127, 2800, None),  # many keys: 127 of 128 a workgroup
    (8, 1, 64, 31, 2900, "3"),     # 248 of 256
    (8, 1, 128, 16, 2800, "1"),    # 128
    (8, 1, 64, 30, 2900, "7"),     # 240 of 256
])
def test_many_rows(gpu, monkeypatch, hq, hkv, d, rows, prefix, splits):
    """Workgroups of 64 and of 128 query rows (as for launches that fill the CUs: here one CU is counted), rings that
    wrap, kept regions that end inside a block."""
    import paper_2609_31224_amd as a2t
    monkeypatch.setenv("A2T_TARGET_WGS", "1")
    if splits:
        monkeypatch.setenv("A2T_SPLITS", splits)
    more = [_unit(min(900, prefix - at)) for at in range(900, prefix, 900)]
    spec = tiny_stream([*more, SMALL, _unit(rows), SMALL, [SEG_RESPONSE], _unit(rows), _unit(rows + 1), SMALL, _unit(rows)],
                       prefix=min(prefix, 900))
    s = Sessions([spec], hq, hkv, d, budgets=[prefix + rows + 20], calls="fused", query_rows=rows, layers=1,
                 unit_rows=max(4 * rows + 80 + prefix, 80))
    try:
        a2t.a2t_profile_enable(s.cache, "attn_mx4_rows")
        s.run()
        assert a2t.a2t_kernel_time(s.cache, "attn_mx4_rows")[0] >= 4
    finally:
        s.close()


@pytest.mark.parametrize("d", [64, 128])
def test_many_rows_of_uneven_streams(gpu, monkeypatch, d):
    """Streams of 1 to 140 rows in one launch of 128-row and of 64-row workgroups."""
    monkeypatch.setenv("A2T_TARGET_WGS", "1")
    for more in ([_unit(900), _unit(900), _unit(900)], []):
        specs = [tiny_stream([*m, SMALL, _unit(n), SMALL], prefix=p) for n, p, m in ((140, 600, more), (1, 5, more), (64, 0, []), (129, 700, []))]
        _run(specs, 2, 2, d, budgets=[100000] * 4, calls="fused", layers=1, query_rows=140, unit_rows=3600)


# ------------------------------------------------------------------ the calls around them
def _fill(a2t, c, ids, n, k, v, start=0, unit=0, layer=None):
    seg = np.full(int(np.sum(n)), SEG_ACOUSTIC, np.uint8)
    pos = np.concatenate([np.arange(start, start + m) for m in n])
    a2t.a2t_append(c, a2t.A2T_ALL_LAYERS if layer is None else layer, ids, n, k, v, seg, pos, [unit] * len(ids))


def _randn(*shape, seed=0, dtype=None):
    import torch
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn(shape, generator=g, device="cuda").to(dtype or torch.bfloat16)


def test_device_refusals(gpu):
    """What a device cache refuses changes nothing."""
    import paper_2609_31224_amd as a2t
    c = a2t.a2t_cache_create(2, 2, 4, 2, 64, a2t.A2T_MX4, 64, 8, 16)
    k, v, q = _randn(3, 2, 64), _randn(3, 2, 64), _randn(3, 4, 64)

    def status(fn, *a):
        try:
            fn(*a)
            return 0
        except a2t.A2TError as e:
            return e.status
    assert status(a2t.a2t_dev_begin, c) == a2t.A2T_ERR_INVALID
    meta = (np.full(3, SEG_ACOUSTIC, np.uint8), np.arange(3), [0])
    a2t.a2t_append(c, 0, [1], [3], k, v, *meta)
    before = [a2t.a2t_stream_info_get(c, s) for s in range(2)]
    o = _randn(3, 4, 64, seed=5)
    was = o.clone()
    assert status(a2t.a2t_chunk_attn, c, 1, [1], [3], q, o) == a2t.A2T_ERR_STATE       # layer not appended
    assert status(a2t.a2t_chunk_attn, c, 0, [0], [1], q, o) == a2t.A2T_ERR_STATE       # no open step
    assert status(a2t.a2t_chunk_attn, c, 0, [1], [4], q, o) == a2t.A2T_ERR_STATE       # more queries than rows
    assert status(a2t.a2t_decode_attn, c, 0, [1, 1], q, o) == a2t.A2T_ERR_INVALID
    assert status(a2t.a2t_chunk_attn, c, 0, [1], [3], q.data_ptr() + 2, o.data_ptr()) == a2t.A2T_ERR_INVALID
    assert status(a2t.a2t_append, c, 1, [1], [3], k.data_ptr() + 8, v.data_ptr(), None, None, None) == a2t.A2T_ERR_INVALID
    assert status(a2t.a2t_read_rows, c, 1, [1], k, v) == a2t.A2T_ERR_STATE
    assert status(a2t.a2t_read_rows, c, 0, [1], None, None) == a2t.A2T_ERR_INVALID
    assert status(a2t.a2t_evict, c, [1], [0], 0) == a2t.A2T_ERR_STATE
    with pytest.raises(ValueError):
        a2t.a2t_read_rows(c, 0, [1], k.float(), None)      # bfloat16 in and out
    with pytest.raises(ValueError):
        a2t.a2t_chunk_attn(c, 0, [1], [3], q.float(), o.float())
    a2t.a2t_sync(c)
    assert [a2t.a2t_stream_info_get(c, s) for s in range(2)] == before
    assert (o == was).all()
    a2t.a2t_cache_destroy(c)


@pytest.mark.parametrize("dtype", ["mx4", "bf16", "f32"])
@pytest.mark.parametrize("hkv,d", [(3, 64), (2, 128), (40, 128)])
def test_read_rows(gpu, dtype, hkv, d):
    """Rows in cache order of streams with a kept region, a wrapped ring, one row and none, for every cache type: what
    a2t_read_kv reads, no more rows than those, either output alone, one layer or all."""
    import torch
    import paper_2609_31224_amd as a2t
    t = torch.float32 if dtype == "f32" else torch.bfloat16
    L, S = 2, 4
    c = a2t.a2t_cache_create(L, S, hkv, hkv, d, {"mx4": a2t.A2T_MX4, "bf16": a2t.A2T_BF16, "f32": a2t.A2T_F32}[dtype], 70, 60, 40)
    pos = 0
    for unit in range(6):      # streams 0 and 1: some rows kept, the ring has wrapped
        n = [17, 12]
        seg = np.where(np.arange(29) % 3 == 0, SEG_TEXT, SEG_ACOUSTIC).astype(np.uint8)
        a2t.a2t_append(c, a2t.A2T_ALL_LAYERS, [0, 1], n, _randn(L, 29, hkv, d, seed=unit, dtype=t), _randn(L, 29, hkv, d, seed=50 + unit, dtype=t),
                       seg, np.concatenate([np.arange(pos, pos + 17), np.arange(pos, pos + 12)]), [unit, unit])
        a2t.a2t_evict(c, [0, 1], [30, 35], 1)
        pos += 17
    _fill(a2t, c, [2], [1], _randn(L, 1, hkv, d, seed=9, dtype=t), _randn(L, 1, hkv, d, seed=10, dtype=t))
    info = [a2t.a2t_stream_info_get(c, s) for s in range(S)]
    assert info[0]["kept"] and info[1]["kept"] and info[0]["ring_head"] and info[3]["resident"] == 0
    assert info[0]["ring_head"] + info[0]["ring"] > 70 or info[1]["ring_head"] + info[1]["ring"] > 70
    ids = [1, 3, 2, 0]
    rows = [info[s]["resident"] for s in ids]
    total = sum(rows)
    want = [[np.concatenate([a2t.a2t_read_kv(c, layer, s)[w] for s in ids]) for layer in range(L)] for w in range(2)]
    mark = 7.0

    def call(layer, which):
        shape = (L, total, hkv, d) if layer == a2t.A2T_ALL_LAYERS else (total, hkv, d)
        size = int(np.prod(shape))
        out = [torch.full((size + 64,), mark, dtype=t, device="cuda") for _ in range(2)]
        a2t.a2t_read_rows(c, layer, ids, *[x[:size] if w in which else None for w, x in enumerate(out)])
        a2t.a2t_sync(c)
        for w, x in enumerate(out):
            x, behind = x[:size].view(shape), x[size:]
            assert (behind == mark).all()
            if w not in which:
                assert (x == mark).all()
                continue
            got = x.cpu().numpy() if dtype == "f32" else x.view(torch.int16).cpu().numpy().view(np.uint16)
            for i, l in enumerate(range(L) if layer == a2t.A2T_ALL_LAYERS else [layer]):
                assert np.array_equal(got[i] if layer == a2t.A2T_ALL_LAYERS else got, want[w][l]), (layer, w, l)
    for layer in (a2t.A2T_ALL_LAYERS, 0, 1):
        for which in ((0, 1), (0,), (1,)):
            call(layer, which)
    a2t.a2t_read_rows(c, 0, [3], _randn(1, hkv, d, dtype=t), None)      # no rows at all
    a2t.a2t_sync(c)
    a2t.a2t_cache_destroy(c)


@pytest.mark.parametrize("d", [64, 128])
def test_callers_pools(gpu, d):
    """Pools of the documented size, with what is in them before: rows come out the same, nothing is
    written behind them, and the codes and scales are where the header says."""
    import torch
    import paper_2609_31224_amd as a2t
    L, S, hkv, unit_rows, kept_rows, n = 2, 3, 2, 20, 6, 9
    rows = L * S * hkv * (unit_rows + kept_rows)
    size = rows * (d // 2 + d // 32)
    pools = [torch.full((size + 256,), 0xa5, dtype=torch.uint8, device="cuda") for _ in range(2)]
    assert all(p.data_ptr() % 256 == 0 for p in pools)
    c = a2t.a2t_cache_create(L, S, hkv, hkv, d, a2t.A2T_MX4, unit_rows, kept_rows, n, k_pool=pools[0], v_pool=pools[1])
    k, v = _randn(L, 2 * n, hkv, d, seed=1), _randn(L, 2 * n, hkv, d, seed=2)
    _fill(a2t, c, [0, 2], [n, n], k, v)
    a2t.a2t_sync(c)
    for p in pools:
        assert (p[size:] == 0xa5).all()
    codes = pools[1][:rows * d // 2].cpu().numpy()[:L * S * hkv * unit_rows * d // 2].reshape(L, S, hkv, unit_rows, d // 2)
    scales = pools[1][rows * d // 2:size].cpu().numpy()[:L * S * hkv * unit_rows * d // 32].reshape(L, S, hkv, unit_rows, d // 32)
    assert (codes[:, 1] == 0xa5).all() and (codes[:, :, :, n:] == 0xa5).all() and (scales[:, :, :, n:] == 0xa5).all()
    codes, scales = codes[:, [0, 2], :, :n], scales[:, [0, 2], :, :n]
    nib = np.stack([codes & 15, codes >> 4], -1).reshape(L, 2, hkv, n, d)
    val = mx4.LEVELS[nib & 7] * np.where(nib & 8, -1, 1) * np.repeat(2.0 ** (scales.astype(int) - 127), 32, -1)
    want = mx4.hold(v.float().cpu().numpy()).reshape(L, 2, n, hkv, d).transpose(0, 1, 3, 2, 4)
    assert np.array_equal(val, want)
    a2t.a2t_cache_destroy(c)


@pytest.mark.parametrize("hq,hkv,d,rows", [(32, 8, 128, 22), (4, 1, 64, 1), (8, 2, 128, 40)])
def test_no_allocation_calls(gpu, hq, hkv, d, rows):
    """a2t_append_attn_noalloc on a cache without a workspace against a2t_append_attn: the same rows, outputs
    within the rounding of the partials (fp16: half a step of 2^-11 of values below 6 each, twice over) and of
    the output."""
    import torch
    import paper_2609_31224_amd as a2t
    mk = lambda flags: a2t.a2t_cache_create(1, 1, hq, hkv, d, a2t.A2T_MX4, 4100 + rows, 0, 1024, flags=flags)  # noqa: E731
    ca, cb = mk(0), mk(a2t.A2T_FLAG_NO_WORKSPACE)
    for i in range(4):
        k, v = _randn(1, 1000, hkv, d, seed=i), _randn(1, 1000, hkv, d, seed=20 + i)
        for c in (ca, cb):
            _fill(a2t, c, [0], [1000], k, v, start=1000 * i, unit=i)
    k, v, q = _randn(rows, hkv, d, seed=7), _randn(rows, hkv, d, seed=8), _randn(rows, hq, d, seed=9)
    seg, pos = np.full(rows, SEG_ACOUSTIC, np.uint8), np.arange(4000, 4000 + rows)
    oa, ob = torch.zeros_like(q), torch.zeros_like(q)
    a2t.a2t_append_attn(ca, 0, [0], [rows], k, v, seg, pos, [9], [rows], q, oa)
    a2t.a2t_append_attn_noalloc(cb, 0, [0], [rows], k, v, seg, pos, [9], [rows], q, ob)
    a2t.a2t_sync(ca)
    a2t.a2t_sync(cb)
    assert (oa.float() - ob.float()).abs().max() <= 2 * 6 * 2.0 ** -11 + 2 * 2.0 ** -8 * oa.float().abs().max()
    for x, y in zip(a2t.a2t_read_kv(ca, 0, 0), a2t.a2t_read_kv(cb, 0, 0)):
        assert np.array_equal(x, y)
    for c in (ca, cb):
        a2t.a2t_cache_destroy(c)


def test_other_streams(gpu):
    """A cache on a stream of its own, moved to another one, with the default stream busy."""
    import torch
    import paper_2609_31224_amd as a2t
    side, other = torch.cuda.Stream(), torch.cuda.Stream()
    spec = tiny_stream([SMALL, _unit(20), [SEG_RESPONSE], _unit(33)], prefix=100)
    busy = torch.randn(4096, 4096, device="cuda")
    torch.cuda.synchronize()
    s = Sessions([spec], 8, 2, 128, budgets=[60], calls="fused", stream=side)
    try:
        for t, st in enumerate(spec.steps):
            for _ in range(4):
                busy = busy @ busy * 1e-3
            torch.cuda.synchronize()      # the test's own uploads are on the default stream
            a2t.a2t_sync(s.cache)
            a2t.a2t_set_stream(s.cache, other if t % 2 else side)
            s._dev = lambda x, up=s.__class__._dev: (up(s, x), torch.cuda.current_stream().synchronize())[0]
            s.step([(0, st)], t)
    finally:
        s.close()


@pytest.mark.parametrize("streams,resident,rows,hq,hkv,d", [(1, 3000, 1, 32, 8, 128), (3, 500, 22, 8, 2, 64), (2, 0, 130, 8, 1, 128)])
def test_captured_calls(gpu, streams, resident, rows, hq, hkv, d):
    """Attention and a2t_read_rows of an open step captured in a graph: every replay, with eager calls, a changed query
    and synchronisations between, gives the eager result."""
    import torch
    import paper_2609_31224_amd as a2t
    side = torch.cuda.Stream()
    c = a2t.a2t_cache_create(1, streams, hq, hkv, d, a2t.A2T_MX4, resident + rows, 0, 1024, stream=side)
    at = 0
    while at < resident:
        n = min(1024, resident - at)
        k, v = _randn(1, n * streams, hkv, d, seed=at), _randn(1, n * streams, hkv, d, seed=at + 1)
        torch.cuda.synchronize()
        _fill(a2t, c, range(streams), [n] * streams, k, v, start=at, unit=at)
        at += n
    k, v = _randn(1, rows * streams, hkv, d, seed=91), _randn(1, rows * streams, hkv, d, seed=92)
    torch.cuda.synchronize()
    _fill(a2t, c, range(streams), [rows] * streams, k, v, start=resident, unit=resident + 1)
    q = _randn(rows * streams, hq, d, seed=93)
    o = torch.zeros_like(q)
    back = torch.zeros((streams * (resident + rows), hkv, d), dtype=torch.bfloat16, device="cuda")
    torch.cuda.synchronize()

    def calls():
        if rows == 1:
            a2t.a2t_decode_attn(c, 0, range(streams), q, o)
        else:
            a2t.a2t_chunk_attn(c, 0, range(streams), [rows] * streams, q, o)
        a2t.a2t_read_rows(c, 0, range(streams), None, back)
    calls()
    a2t.a2t_sync(c)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        calls()
    for i in range(5):
        q.copy_(_randn(rows * streams, hq, d, seed=200 + i))
        o.fill_(3.0)
        back.fill_(3.0)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        got = o.clone(), back.clone()
        o.fill_(4.0)
        back.fill_(4.0)
        torch.cuda.synchronize()
        calls()
        a2t.a2t_sync(c)
        assert torch.equal(got[0], o) and torch.equal(got[1], back), i
        assert torch.isfinite(o.float()).all()
    a2t.a2t_cache_destroy(c)


def test_results_do_not_vary(gpu):
    """The same call twice gives the same bits, whatever ran before it."""
    import torch
    import paper_2609_31224_amd as a2t
    c = a2t.a2t_cache_create(1, 3, 32, 8, 128, a2t.A2T_MX4, 3000, 0, 1024)
    for i in range(2):
        _fill(a2t, c, [0, 1, 2], [1000, 700, 13], _randn(1, 1713, 8, 128, seed=i), _randn(1, 1713, 8, 128, seed=5 + i), start=1000 * i, unit=i)
    q = _randn(1713, 32, 128, seed=3)
    first = None
    for _ in range(3):
        o = torch.zeros_like(q)
        a2t.a2t_chunk_attn(c, 0, [0, 1, 2], [1000, 700, 13], q, o)
        d = torch.zeros((3, 32, 128), dtype=q.dtype, device="cuda")
        a2t.a2t_decode_attn(c, 0, [2, 0, 1], q[:3].contiguous(), d)
        a2t.a2t_sync(c)
        first = first or (o, d)
        assert torch.equal(first[0], o) and torch.equal(first[1], d)
    a2t.a2t_cache_destroy(c)


@pytest.mark.parametrize("kept", [False, True])
def test_offsets_past_32_bits(gpu, kept):
    """Rows of the last head of a pool whose codes pass 4 GiB, in the ring or in the kept region: written, moved, read
    and attended where they belong."""
    import torch
    import paper_2609_31224_amd as a2t
    hq, hkv, d, unit_rows, kept_rows = 2, 1, 128, 1 << 20, 1 << 16
    S = 66      # 66 x 1,114,112 rows of 64 bytes: 4.7 GB of codes a pool
    c = a2t.a2t_cache_create(1, S, hq, hkv, d, a2t.A2T_MX4, unit_rows, kept_rows, 300)
    n, s = 300, S - 1
    k, v, q = _randn(1, n, hkv, d, seed=1), _randn(1, n, hkv, d, seed=2), _randn(1, hq, d, seed=3)
    seg = np.where(np.arange(n) % 2, SEG_TEXT, SEG_ACOUSTIC).astype(np.uint8)
    a2t.a2t_append(c, a2t.A2T_ALL_LAYERS, [s], [n], k, v, seg, np.arange(n), [0])
    live = np.arange(n)
    if kept:
        assert a2t.a2t_evict(c, [s], [0], 0)[0][0] == n // 2
        live = live[seg == SEG_TEXT]
    k1, v1 = _randn(1, 1, hkv, d, seed=4), _randn(1, 1, hkv, d, seed=5)
    a2t.a2t_append(c, a2t.A2T_ALL_LAYERS, [s], [1], k1, v1, [SEG_ACOUSTIC], [n], [1])
    o = torch.zeros_like(q)
    a2t.a2t_decode_attn(c, 0, [s], q, o)
    kr, vr = (bf16_bits_to_f32(x) for x in a2t.a2t_read_kv(c, 0, s))
    back = torch.zeros((len(live) + 1, hkv, d), dtype=torch.bfloat16, device="cuda")
    a2t.a2t_read_rows(c, 0, [s], None, back)
    a2t.a2t_sync(c)
    both = torch.cat([v[0, live], v1[0]]).float().cpu().numpy()
    assert np.array_equal(vr, mx4.hold(both)) and np.array_equal(back.float().cpu().numpy(), vr)
    keys = torch.cat([k[0, live], k1[0]]).float().cpu().numpy()
    pos = np.append(live, n)
    assert np.array_equal(kr, mx4.hold(mx4.rotate_to_f32(keys, pos, 1e6)))
    cache = mx4.OracleMx4Cache(hq, hkv, d)
    cache.append(np.full(len(pos), SEG_ACOUSTIC), pos, 0, {0: keys}, {0: both})
    want, bound = cache.attention_bound(0, q.float().cpu().numpy(), 1)
    assert (np.abs(o.float().cpu().numpy() - want) <= bound).all()
    a2t.a2t_cache_destroy(c)


@pytest.mark.parametrize("d,hq,hkv,old,rows", [(64, 4, 2, 900, 70), (128, 4, 1, 900, 70), (128, 2, 2, 900, 70), (128, 2, 2, 900, 40),
                                               (128, 4, 1, 2900, 64), (64, 8, 1, 2900, 62), (64, 2, 2, 900, 47)])
def test_values_that_are_not_finite_in_later_blocks(gpu, monkeypatch, d, hq, hkv, old, rows):
    """The same behind several key blocks a wave, in every kind of workgroup; and values of a resident
    row, which every query sees."""
    import torch
    import paper_2609_31224_amd as a2t
    monkeypatch.setenv("A2T_SPLITS", "1")
    if rows >= 60:   # workgroups of 64 rows and, with many keys, of 128
        monkeypatch.setenv("A2T_TARGET_WGS", "1")
    bad = 33
    g = torch.Generator(device="cuda").manual_seed(6)
    k0, v0 = (torch.randn((old, hkv, d), generator=g, device="cuda").bfloat16() for _ in range(2))
    k, v, q = (torch.randn((rows, h, d), generator=g, device="cuda").bfloat16() for h in (hkv, hkv, hq))

    def run(new=False, resident=None):
        vv, vr = v.clone(), v0.clone()
        if new:
            vv[bad, :, 37] = float("nan")
        if resident is not None:
            vr[resident, 0, 2] = float("-inf")
        c = a2t.a2t_cache_create(1, 1, hq, hkv, d, a2t.A2T_MX4, old + rows, 0, 900)
        o = torch.zeros_like(q)
        for at in range(0, old, 900):
            n = min(900, old - at)
            a2t.a2t_append(c, 0, [0], [n], k0[at:at + n], vr[at:at + n], np.full(n, SEG_ACOUSTIC, np.uint8), np.arange(at, at + n), [at])
        a2t.a2t_append_attn(c, 0, [0], [rows], k, vv, np.full(rows, SEG_ACOUSTIC, np.uint8), np.arange(old, old + rows), [old],
                            [rows], q, o)
        a2t.a2t_sync(c)
        a2t.a2t_cache_destroy(c)
        return o.float().cpu().numpy()

    clean = run()
    assert np.isfinite(clean).all()
    got = run(new=True)
    assert np.array_equal(got[:bad], clean[:bad])
    assert np.isnan(got[bad:, :, 32:64]).all()
    keep = np.r_[0:32, 64:d]
    assert np.array_equal(got[bad:][..., keep], clean[bad:][..., keep])
    for row in (0, 300, 899):      # the first KV head's query heads, 32 dims
        got = run(resident=row)
        mine = hq // hkv
        assert np.isnan(got[:, :mine, :32]).all()
        assert np.array_equal(got[:, :mine, 32:], clean[:, :mine, 32:]) and np.array_equal(got[:, mine:], clean[:, mine:])


@pytest.mark.parametrize("d,hq,hkv,rows,old", [(64, 4, 2, 5, 333), (128, 2, 2, 10, 333), (64, 4, 1, 64, 333), (128, 4, 1, 64, 333), (128, 4, 1, 22, 333),
                                               (128, 2, 2, 20, 333), (64, 4, 1, 64, 2900), (128, 4, 1, 64, 2900), (64, 4, 1, 22, 333)])
@pytest.mark.parametrize("exps", [[-40], [-26, -25, -24, -23, -22, -12, -11], [10, 11, 12, 13, 14, 0], [-110, -60, -20, 0, 0, 0, 20, 100],
                                  [0, 0, 0, 0, 0, 120]])
def test_scales_of_values_apart(gpu, monkeypatch, d, hq, hkv, rows, old, exps):
    """Blocks of V whose scales fp16 holds beside some it does not, blocks of zeros, and rows
    of the step that only some of its rows see; every output element within its own bound."""
    import torch
    import paper_2609_31224_amd as a2t
    monkeypatch.setenv("A2T_SPLITS", "1")
    if rows >= 60:
        monkeypatch.setenv("A2T_TARGET_WGS", "1")
    rng = np.random.default_rng(9)
    n = old + rows
    scale = np.repeat(2.0 ** rng.choice(exps, (n, hkv, d // 32)), 32, -1) * np.repeat(rng.random((n, hkv, d // 32)) < 0.9, 32, -1)
    k, v, q = (bf16_round(rng.standard_normal((m, h, d))) for m, h in ((n, hkv), (n, hkv), (rows, hq)))
    v = bf16_round(v * scale)
    kd, vd, qd = (torch.from_numpy(np.ascontiguousarray(x, np.float32)).cuda().bfloat16() for x in (k, v, q))
    seg = np.full(n, SEG_ACOUSTIC, np.uint8)
    c = a2t.a2t_cache_create(1, 1, hq, hkv, d, a2t.A2T_MX4, n, 0, 900)
    ref = mx4.OracleMx4Cache(hq, hkv, d, [0], theta=1e6)
    o = torch.full_like(qd, float("nan"))
    parts = [slice(at, min(at + 900, old)) for at in range(0, old, 900)]
    for u, part in enumerate(parts):
        a2t.a2t_append(c, 0, [0], [part.stop - part.start], kd[part], vd[part], seg[part], np.arange(n)[part], [u])
    a2t.a2t_append_attn(c, 0, [0], [rows], kd[old:], vd[old:], seg[old:], np.arange(old, n), [len(parts)], [rows], qd, o)
    a2t.a2t_sync(c)
    a2t.a2t_cache_destroy(c)
    for unit, part in enumerate([*parts, slice(old, n)]):
        ref.append(seg[part], np.arange(n)[part], unit, {0: k[part]}, {0: v[part]})
    want, bound = ref.attention_bound(0, q, rows, least=0.0)
    off = np.abs(o.float().cpu().numpy().astype(np.float64) - want) - bound
    assert np.isfinite(off).all() and (off <= 0).all(), (float(off.max()), np.unravel_index(off.argmax(), off.shape))
