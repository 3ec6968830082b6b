"""A2T_MX4 caches on a stream of their own while the default stream is busy: every call's work is on the
cache's stream, waits for nothing on the other one and gives the result that it gives alone."""
import numpy as np
import pytest

from synth.streams import SEG_ACOUSTIC, SEG_TEXT

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("d,hq,hkv,rows", [(128, 8, 2, 22), (64, 4, 4, 1), (128, 16, 2, 100)])
def test_calls_beside_a_busy_default_stream(gpu, d, hq, hkv, rows):
    import torch
    import paper_2609_31224_amd as a2t
    L, S, old = 2, 3, 700
    n = old + 2 * rows
    g = torch.Generator(device="cuda").manual_seed(8)
    rand = lambda *shape: torch.randn(shape, generator=g, device="cuda").bfloat16()   # noqa: E731
    first = [rand(L, S * old, hkv, d) for _ in range(2)]
    steps = [[rand(L, S * rows, hkv, d), rand(L, S * rows, hkv, d), rand(L, S * rows, hq, d)] for _ in range(2)]
    busy = torch.randn(8192, 8192, device="cuda")
    into = torch.empty_like(busy)
    torch.mm(busy, busy, out=into)      # the library of products sets itself up
    segs = {m: np.where(np.arange(S * m) % 3, SEG_ACOUSTIC, SEG_TEXT).astype(np.uint8) for m in (old, rows)}
    small = torch.zeros(64, device="cuda")

    def beside(stream):
        """Whether its work runs while the default stream's does: streams share a few hardware queues."""
        done = torch.cuda.Event()
        torch.cuda.synchronize()
        for _ in range(4):
            torch.mm(busy, busy, out=into)
        done.record()
        with torch.cuda.stream(stream):
            small.add_(1)
        stream.synchronize()
        alone = not done.query()
        torch.cuda.synchronize()
        return alone
    streams = [x for x in (torch.cuda.Stream() for _ in range(8)) if beside(x)][:2]
    if len(streams) < 2:
        pytest.skip("every stream shares the default one's hardware queue")

    def go(load):
        """The calls of a session, moved to another stream halfway; [outputs], and whether the load outlasted them."""
        outs = [torch.full((L, S * rows, hq, d), float("nan"), dtype=torch.bfloat16, device="cuda") for _ in steps]
        back = [torch.full((L, S * n, hkv, d), float("nan"), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
        c = a2t.a2t_cache_create(L, S, hq, hkv, d, a2t.A2T_MX4, n, n, max(old, 100), stream=streams[0])
        done = torch.cuda.Event()
        torch.cuda.synchronize()        # nothing of the test's own is in flight
        for _ in range(load):
            torch.mm(busy, busy, out=into)
        done.record()
        a2t.a2t_append(c, a2t.A2T_ALL_LAYERS, range(S), [old] * S, *first, segs[old], np.tile(np.arange(old), S), [0] * S)
        a2t.a2t_evict(c, range(S), [500] * S, 0)
        for t, ((k, v, q), o) in enumerate(zip(steps, outs)):
            pos = np.tile(np.arange(old + t * rows, old + (t + 1) * rows), S)
            for l in range(L):
                meta = (segs[rows], pos, [t + 1] * S) if l == 0 else (None, None, None)
                a2t.a2t_append_attn(c, l, range(S), [rows] * S, k[l], v[l], *meta, [rows] * S, q[l], o[l])
            if t == 0:
                a2t.a2t_evict(c, range(S), [200] * S, 1)
                a2t.a2t_sync(c)
                a2t.a2t_set_stream(c, streams[1])
        held = sum(a2t.a2t_resident(c, s)[0] for s in range(S))
        flat = [x.view(-1)[:L * held * hkv * d] for x in back]
        a2t.a2t_read_rows(c, a2t.A2T_ALL_LAYERS, range(S), *flat)
        a2t.a2t_sync(c)
        outlasted = not done.query()
        torch.cuda.synchronize()
        a2t.a2t_cache_destroy(c)
        assert all(torch.isfinite(x.float()).all() for x in (*outs, *flat))
        return [*outs, *flat], outlasted

    want, _ = go(0)
    got, outlasted = go(24)
    assert outlasted, "the products ended before the calls did"
    for x, y in zip(want, got):
        assert torch.equal(x, y)


@pytest.mark.parametrize("dtype", ["A2T_MX4", "A2T_BF16", "A2T_F32"])
def test_tensors_too_small_for_the_rows(gpu, dtype):
    """a2t_read_rows through the binding refuses them before anything is enqueued."""
    import torch
    import paper_2609_31224_amd as a2t
    L, hkv, d = 2, 2, 64
    t = torch.float32 if dtype == "A2T_F32" else torch.bfloat16
    c = a2t.a2t_cache_create(L, 2, hkv, hkv, d, getattr(a2t, dtype), 40, 0, 20)
    x = torch.randn((L, 12, hkv, d), device="cuda").to(t)
    a2t.a2t_append(c, a2t.A2T_ALL_LAYERS, [0, 1], [7, 5], x, x, np.full(12, SEG_ACOUSTIC, np.uint8), [*range(7), *range(5)], [0, 0])
    out = lambda *shape: torch.zeros((*shape, hkv, d), dtype=t, device="cuda")   # noqa: E731
    for layer, ids, k, v in ((0, [0, 1], out(11), None), (0, [0, 1], None, out(11)), (0, [0], out(7), out(6)),
                             (a2t.A2T_ALL_LAYERS, [0, 1], out(12), None), (a2t.A2T_ALL_LAYERS, [1], out(2, 5), out(5))):
        with pytest.raises(ValueError):
            a2t.a2t_read_rows(c, layer, ids, k, v)
    for ids in ([2], [-1], [0, 0]):
        with pytest.raises(a2t.A2TError) as e:
            a2t.a2t_read_rows(c, 0, ids, out(40), None)
        assert e.value.status == a2t.A2T_ERR_INVALID
    v = out(L, 12)
    a2t.a2t_read_rows(c, a2t.A2T_ALL_LAYERS, [0, 1], None, v)
    a2t.a2t_sync(c)
    assert torch.isfinite(v.float()).all() and (v[0, 0] != 0).any()
    a2t.a2t_cache_destroy(c)
