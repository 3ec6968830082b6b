"""Drives an A2T_MX4 cache and the oracle together over hand-shaped streams.  Test
infrastructure; not collected by pytest."""
from __future__ import annotations

import numpy as np

from oracle.mx4 import OracleMx4Cache
from oracle.policy import EvictRule
from synth.streams import bf16_round
from tests.harness import bf16_bits_to_f32, row_bounds


class Sessions:
    """``calls``: "separate" (a2t_append, a2t_chunk_attn), "fused" (a2t_append_attn), "noalloc"
    (a2t_append_attn_noalloc), "all" (a2t_append with A2T_ALL_LAYERS, a2t_chunk_attn); steps of
    one response row run a2t_decode_attn after a separate append.  Checked in every step: outputs
    within the oracle's bound, stored rows (a2t_read_kv and a2t_read_rows) equal to the
    oracle's, the layout, eviction counts, and that eviction moved the survivors unchanged."""

    def __init__(self, specs, hq, hkv, d, *, budgets, window=0, layers=2, seed=0, calls="separate", query_rows=None,
                 rule=None, n_sink=0, unit_rows=None, theta=1e6, stream=None, flags=0, kv_scale=1.0, offsets=None):
        import paper_2609_31224_amd as a2t
        self.a2t, self.specs, self.hq, self.hkv, self.d, self.L = a2t, specs, hq, hkv, d, layers
        self.budgets, self.window, self.calls, self.query_rows = budgets, window, calls, query_rows
        self.rule, self.n_sink, self.kv_scale = rule, n_sink, kv_scale
        self.rng = np.random.default_rng(seed)
        self.offsets = offsets or [0] * len(specs)
        bounds = [row_bounds(s) for s in specs]
        self.cache = a2t.a2t_cache_create(layers, len(specs), hq, hkv, d, a2t.A2T_MX4, unit_rows or max(b[0] for b in bounds),
                                          max(b[1] for b in bounds) + n_sink + 1, max(b[2] for b in bounds), flags=flags,
                                          rope_theta=theta, stream=stream)
        self.oracles = [OracleMx4Cache(hq, hkv, d, range(layers), theta=theta) for _ in specs]
        self.evictions = 0
        self.worst = 0.0      # largest error over its bound

    def close(self):
        self.a2t.a2t_cache_destroy(self.cache)

    def _rand(self, n, heads, scale=1.0):
        return bf16_round(scale * self.rng.standard_normal((self.L, n, heads, self.d)))

    def _dev(self, x):
        import torch
        return torch.from_numpy(np.ascontiguousarray(x, np.float32)).cuda().to(torch.bfloat16)

    def run(self):
        T = max(o + len(s.steps) for o, s in zip(self.offsets, self.specs))
        for t in range(T):
            act = [(i, s.steps[t - o]) for i, (o, s) in enumerate(zip(self.offsets, self.specs)) if 0 <= t - o < len(s.steps)]
            if act:
                self.step(act, t)
        return self

    def step(self, act, t):
        a2t, c = self.a2t, self.cache
        import torch
        ids, n = [i for i, _ in act], [st.n for _, st in act]
        nq = [min(m, self.query_rows) if self.query_rows else m for m in n]
        decode = all(st.decode for _, st in act)
        k, v, q = self._rand(sum(n), self.hkv, self.kv_scale), self._rand(sum(n), self.hkv, self.kv_scale), self._rand(sum(n), self.hq)
        seg, pos = np.concatenate([st.seg for _, st in act]), np.concatenate([st.pos for _, st in act])
        unit = [st.unit for _, st in act]
        first = np.cumsum([0] + n)
        for j, (i, st) in enumerate(act):
            rows = slice(first[j], first[j + 1])
            self.oracles[i].append(st.seg, st.pos, st.unit, {l: k[l][rows] for l in range(self.L)}, {l: v[l][rows] for l in range(self.L)})
        kd, vd = self._dev(k), self._dev(v)
        torch.cuda.current_stream().synchronize()
        asks = np.concatenate([np.arange(first[j + 1] - nq[j], first[j + 1]) for j in range(len(act))])
        if self.calls == "all":
            a2t.a2t_append(c, a2t.A2T_ALL_LAYERS, ids, n, kd, vd, seg, pos, unit)
        for l in range(self.L):
            meta = (seg, pos, unit) if l == 0 else (None, None, None)
            qd = self._dev(q[l][asks])
            o = torch.full_like(qd, float("nan"))
            torch.cuda.current_stream().synchronize()   # the cache may be on another stream than the uploads and fills
            if self.calls in ("fused", "noalloc") and not decode:
                call = a2t.a2t_append_attn if self.calls == "fused" else a2t.a2t_append_attn_noalloc
                call(c, l, ids, n, kd[l], vd[l], *meta, nq, qd, o)
            else:
                if self.calls != "all":
                    a2t.a2t_append(c, l, ids, n, kd[l], vd[l], *meta)
                if decode:
                    a2t.a2t_decode_attn(c, l, ids, qd, o)
                else:
                    a2t.a2t_chunk_attn(c, l, ids, nq, qd, o)
            a2t.a2t_sync(c)
            got = o.float().cpu().numpy().astype(np.float64)
            at = 0
            for j, (i, _) in enumerate(act):
                mine = asks[at:at + nq[j]]
                want, bound = self.oracles[i].attention_bound(l, q[l][mine], nq[j])
                off = np.abs(got[at:at + nq[j]] - want) / bound
                assert np.isfinite(off).all(), (t, i, l)
                self.worst = max(self.worst, float(off.max()))
                assert off.max() <= 1.0, (t, i, l, float(off.max()), np.unravel_index(off.argmax(), off.shape))
                at += nq[j]
        before = self.check_rows(ids)
        budgets = [self.budgets[i] for i in ids]
        if self.rule:
            lib_rule = {"unit": a2t.A2T_RULE_UNIT, "row": a2t.A2T_RULE_ROW, "sink_recent": a2t.A2T_RULE_SINK_RECENT}[self.rule]
            n_ev, unmet = a2t.a2t_evict_rule(c, ids, budgets, self.window, lib_rule, self.n_sink)
        else:
            n_ev, unmet = a2t.a2t_evict(c, ids, budgets, self.window)
        for j, i in enumerate(ids):
            rec = self.oracles[i].evict(self.budgets[i], self.window, EvictRule(self.rule or "unit", self.n_sink))
            assert (int(n_ev[j]), bool(unmet[j])) == (rec.n_evicted, rec.plan.budget_unmet), (t, i)
            p, s, u = a2t.a2t_read_layout(c, i)
            assert np.array_equal(p, rec.pos) and np.array_equal(s, rec.seg) and np.array_equal(u, rec.unit), (t, i)
            if rec.n_evicted:
                self.evictions += 1
                n_pre, mask, slot = a2t.a2t_read_last_evict(c, i)
                assert np.array_equal(mask.astype(bool), rec.plan.evict_mask) and np.array_equal(slot, rec.new_slot), (t, i)
                for l in range(self.L):
                    for old, new in zip(before[i, l], a2t.a2t_read_kv(c, l, i)):
                        assert np.array_equal(new[slot[slot >= 0]], old[slot >= 0]), (t, i, l)
        self.check_rows(ids)

    def check_rows(self, ids):
        """Stored rows against the oracle's, from the host call and from the device call."""
        import torch
        a2t, c = self.a2t, self.cache
        total = sum(self.oracles[i].resident for i in ids)
        kr, vr = (torch.full((self.L, total, self.hkv, self.d), float("nan"), dtype=torch.bfloat16, device="cuda") for _ in range(2))
        torch.cuda.current_stream().synchronize()
        a2t.a2t_read_rows(c, a2t.A2T_ALL_LAYERS, ids, kr, vr)
        a2t.a2t_sync(c)
        kr, vr = (x.view(torch.int16).cpu().numpy().view(np.uint16) for x in (kr, vr))
        out, row = {}, 0
        for i in ids:
            o = self.oracles[i]
            for l in range(self.L):
                k, v = a2t.a2t_read_kv(c, l, i)
                assert np.array_equal(k, kr[l, row:row + o.resident]) and np.array_equal(v, vr[l, row:row + o.resident]), (i, l)
                assert np.array_equal(bf16_bits_to_f32(v), o.v[l]), (i, l)
                assert np.array_equal(bf16_bits_to_f32(k), o.k[l]), (i, l)
                out[i, l] = (k, v)
            row += o.resident
        return out
