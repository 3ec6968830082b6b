"""The `until` of a session from what the cache reports of its evictions (a2t_read_last_evict), as the header
describes it, for every eviction rule: the session attended at once sees what it saw when it was served."""
import numpy as np
import pytest

from oracle.prompt import prompt_attention
from tests.test_gpu_session_training import _f64, _units

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rule", ["A2T_RULE_UNIT", "A2T_RULE_ROW", "A2T_RULE_SINK_RECENT"])
def test_until_from_the_masks(gpu, rule, dtype):
    import torch
    import paper_2609_31224_amd as a2t
    rng = np.random.default_rng(8)
    hq, hkv, d, budget, window = 4, 2, 64, 140, 3
    units = _units(rng, 20)
    n = sum(map(len, units))
    dt, code = (torch.float32, a2t.A2T_F32) if dtype == "f32" else (torch.bfloat16, a2t.A2T_BF16)
    q, k, v = (torch.from_numpy(rng.standard_normal((n, h, d)).astype(np.float32)).to("cuda").to(dt) for h in (hq, hkv, hkv))
    cache = a2t.a2t_cache_create(1, 1, hq, hkv, d, code, n, n, 128, flags=a2t.A2T_FLAG_ROTATED)
    h = a2t.a2t_prompt_create(n, hq, hkv, d, code, flags=a2t.A2T_PROMPT_UNTIL)
    served, o = torch.empty_like(q), torch.empty_like(q)
    until, resident, at, evictions = np.full(n, 2**31 - 1, np.int32), np.zeros(0, np.int64), 0, 0
    try:
        for u, seg in enumerate(units):
            w = slice(at, at + len(seg))
            out = torch.empty_like(q[w])
            a2t.a2t_append_attn(cache, 0, [0], [len(seg)], k[w], v[w], seg, np.arange(w.start, w.stop, dtype=np.int32), [u], [len(seg)], q[w], out)
            served[w] = out
            resident = np.concatenate([resident, np.arange(w.start, w.stop)])
            at = w.stop
            count, _ = a2t.a2t_evict_rule(cache, [0], budget, window, getattr(a2t, rule), n_sink=8 if rule == "A2T_RULE_SINK_RECENT" else 0)
            if count[0]:
                before, mask, slot = a2t.a2t_read_last_evict(cache, 0)
                assert before == len(resident) and mask.sum() == count[0]
                until[resident[mask == 1]] = at
                resident = resident[mask == 0]
                assert np.array_equal(slot[mask == 0], np.arange(len(resident)))
                evictions += 1
            layout, _, _ = a2t.a2t_read_layout(cache, 0)
            assert np.array_equal(layout, resident)
        assert evictions > 5 and (until < n).sum() > 100
        a2t.a2t_prompt_attn(h, [n], q, k, v, o, until=torch.from_numpy(until).to("cuda"))
        torch.cuda.synchronize()
    finally:
        a2t.a2t_prompt_destroy(h)
        a2t.a2t_cache_destroy(cache)
    u = 2.0 ** -8 if dtype == "bf16" else 2.0 ** -24
    ref = prompt_attention([n], _f64(q), _f64(k), _f64(v), until, u_store=u, u_mul=u if dtype == "bf16" else 0.0)
    assert (np.abs(_f64(o) - ref.o) <= ref.bounds["o"]).all()
    assert (np.abs(_f64(served) - _f64(o)) <= (2e-2 if dtype == "bf16" else 1e-4) + ref.bounds["o"]).all()
