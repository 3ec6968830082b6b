"""Operators of the side channel's training on whole sessions: what is measured, in plain form
and through the library.

Three operators, as one training step uses them one after the other:

* rotary encoding of packed rows (``op`` "rope": a2t_rope_apply): pairs (i, i + r/2) or (2i, 2i + 1)
  of the first r channels of a head turn by pos * f_i, the others stay; f_i = theta^(-2i/r), scaled
  for long contexts by one of the published methods ("linear", "ntk", "yarn").  The gradient turns back;
* causal attention over packed sequences (``op`` "attn": a2t_prompt_attn, a2t_prompt_attn_grad), grouped
  heads; a key may be visible for a while only (``budget``): row j is seen by the rows j <= i < until[j]
  of its sequence, which is how a session is trained under the eviction that it will be served with;
* the preference loss of paired answers (``op`` "prefer": a2t_prefer_loss): -log sigmoid of beta times
  the chosen answer's log ratio (policy to reference) less the rejected one's, with the gradient of the
  policy's logits.
"""
import ctypes as C
import math
import zlib

import numpy as np
import torch

own = False   # False: plain torch operations; True: the library's calls

DEV = "cuda:0"
THETA = 1.0e6
FOREVER = 2**31 - 1
DTYPE = {"bf16": torch.bfloat16, "f32": torch.float32}


def _case(op, **kw):
    base = {
        "rope": dict(rows=1, hq=32, hkv=8, d=128, part=128, layout="half", scaling="none", factor=1.0, first=0, dtype="bf16", grad=False),
        "attn": dict(rows=1, seqs=1, hq=32, hkv=8, d=128, budget=0, window=0, dtype="bf16", grad=False),
        "prefer": dict(pairs=1, rows=1, vocab=1000, reference=True, beta=0.1, smoothing=0.0, dtype="bf16", grad=True),
    }[op]
    return {"op": op, **base, **kw}


def listed():
    return [
        # one decoded token's query and key: latency alone
        _case("rope", name="rope_token", first=4095),
        # a packed training batch, stretched to four times the trained context
        _case("rope", name="rope_packed", rows=16384, scaling="yarn", factor=4.0),
        # gradients of an fp32 model with interleaved pairs in half of each head, an odd number of rows far into a session
        _case("rope", name="rope_grad_f32", rows=4099, hq=16, hkv=4, part=64, layout="pairs", first=1000003, dtype="f32", grad=True),
        # one listening unit without context, a draft model with a single KV head
        _case("attn", name="attn_unit", rows=22, hq=4, hkv=1, d=64),
        # 37 short answers scored together
        _case("attn", name="attn_answers", rows=4001, seqs=37, hq=16, hkv=4, d=64),
        # a long prompt read at once
        _case("attn", name="attn_prompt", rows=16384),
        # training step of packed sessions of different lengths
        _case("attn", name="attn_train_packed", rows=8192, seqs=11, grad=True),
        # training on a ten-minute session under the eviction that it is served with
        _case("attn", name="attn_train_evicted", rows=13200, budget=4096, window=30, grad=True),
        # the same in fp32, a small model, odd lengths
        _case("attn", name="attn_train_f32", rows=2051, seqs=3, hq=4, hkv=1, d=64, grad=True, dtype="f32"),
        # one pair of short answers, a small vocabulary
        _case("prefer", name="prefer_pair", rows=19, vocab=997, dtype="f32"),
        # a batch of pairs over the extended vocabulary
        _case("prefer", name="prefer_batch", pairs=16, rows=45, vocab=151938),
        # evaluation: no gradient, the reference's log probabilities known, fp32 logits
        _case("prefer", name="prefer_eval_f32", pairs=32, rows=21, vocab=32005, reference=False, smoothing=0.1, dtype="f32", grad=False),
    ]


def draw(rng):
    """One more case of the same ranges; sizes log-uniform, odd ones among them."""
    def log_int(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    op = rng.choice(["rope", "attn", "attn", "attn", "prefer"])
    hkv = rng.choice([1, 2, 4, 8])
    heads = dict(hkv=hkv, hq=hkv * rng.choice([g for g in (1, 2, 3, 4, 8) if g * hkv <= 32]))
    d, dtype = rng.choice([64, 128]), rng.choice(["bf16", "bf16", "f32"])
    if op == "rope":
        scaling = rng.choice(["none", "linear", "ntk", "yarn"])
        return _case(op, rows=log_int(1, 16384), d=d, part=rng.choice([p for p in (16, 32, 64, 96, 128) if p <= d] + [d]), layout=rng.choice(["half", "pairs"]),
                     scaling=scaling, factor=1.0 if scaling == "none" else float(rng.choice([2, 4, 8, 32])), first=rng.choice([0, log_int(1, 4000000)]),
                     dtype=dtype, grad=rng.random() < 0.4, **heads)
    if op == "attn":
        grad = rng.random() < 0.5
        # a pass of fp32 costs about as much as one of bf16 over four times the rows
        rows = log_int(1, (8192 if grad else 12288) // (4 if dtype == "f32" else 1))
        budget = max(24, int(rows * rng.uniform(0.2, 0.7))) if rows > 200 and rng.random() < 0.35 else 0
        return _case(op, rows=rows, seqs=1 if rng.random() < 0.5 else log_int(1, max(1, min(64, rows // 4))), d=d, budget=budget, window=rng.choice([0, 3, 30]) if budget else 0,
                     dtype=dtype, grad=grad, **heads)
    vocab = log_int(500, 152000)
    pairs = log_int(1, 32)
    return _case(op, pairs=pairs, rows=log_int(1, max(1, min(60, 190000000 // (2 * pairs * vocab)))), vocab=vocab, reference=rng.random() < 0.6, beta=rng.choice([0.05, 0.1, 0.5]),
                 smoothing=rng.choice([0.0, 0.1]), dtype=dtype, grad=rng.random() < 0.7)


# ------------------------------------------------------------------ a case's rows
def _numbers(case):
    """A generator of the case's structure (lengths, units), from the case alone."""
    return np.random.default_rng(zlib.crc32(repr(sorted((k, v) for k, v in case.items() if k != "name")).encode()))


def _lengths(case):
    """Rows of each sequence: uneven shares of the total, at least one row each."""
    n, s = case["rows"], case["seqs"]
    if s == 1:
        return np.array([n], np.int32)
    cut = np.sort(_numbers(case).choice(n - 1, s - 1, replace=False)) + 1
    return np.diff(np.concatenate([[0], cut, [n]])).astype(np.int32)


def _until(case, lengths):
    """First row that no longer sees each row: sessions of one-second units (17 acoustic rows, a
    transcript between two delimiters) lose the acoustic and delimiter rows of their oldest unit
    outside the window whenever more rows than the budget are resident after a unit."""
    rng, out = _numbers(case), []
    for n in lengths:
        until, units, at, resident = np.full(n, FOREVER, np.int64), [], 0, 0
        while at < n:
            t = int(rng.poisson(3))
            rows = np.concatenate([at + np.arange(18), [at + 18 + t]])
            units.append(rows[rows < n])
            resident += min(19 + t, int(n) - at)
            at += 19 + t
            while resident > case["budget"] and len(units) > case["window"] and units:
                gone = units.pop(0)
                until[gone] = at
                resident -= len(gone)
        out.append(until)
    return np.minimum(np.concatenate(out), FOREVER).astype(np.int32)


def _visible(lengths, until):
    """(query, key) pairs that attention looks at."""
    total, at = 0.0, 0
    for n in lengths.astype(np.int64):
        j = np.arange(n)
        end = np.full(n, n) if until is None else np.minimum(until[at:at + n], n)
        total += float(np.maximum(0, end - j).sum())
        at += n
    return total


def _answer_rows(case):
    """Rows of every answer, chosen and rejected in turn: around case["rows"], at least one."""
    n = case["rows"]
    return _numbers(case).integers(max(1, n // 2), n + n // 2 + 1, 2 * case["pairs"]).astype(np.int32)


def _inputs(case, seed):
    """What the operator is given, on the GPU."""
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    dt = DTYPE[case["dtype"]]

    def rand(*shape):
        return torch.randn(shape, generator=g, device=DEV)

    if case["op"] == "prefer":
        rows = _answer_rows(case)
        n, vocab = int(rows.sum()), case["vocab"]
        stride = (vocab + 7) // 8 * 8
        logits = torch.zeros((n, stride), device=DEV)
        logits[:, :vocab] = 2.0 * rand(n, vocab)
        target = torch.randint(vocab, (n,), generator=g, device=DEV, dtype=torch.int32)
        # a trained model gives its answers' tokens some weight; the policy has moved a little from the reference
        logits[torch.arange(n, device=DEV), target.long()] += 8.0
        x = dict(rows=rows, target=target, reference=logits.to(dt, copy=True))
        for r in logits.split(256):
            r[:, :vocab] += 0.25 * rand(len(r), vocab)
        x["policy"] = logits.to(dt)
        if not case["reference"]:
            ref = x.pop("reference")
            x["ref_logp"] = torch.cat([torch.log_softmax(r[:, :vocab].double(), -1).gather(1, t.long()[:, None])[:, 0].float()
                                       for r, t in zip(ref.split(256), target.split(256))])
        return x
    hq, hkv, d, n = case["hq"], case["hkv"], case["d"], case["rows"]
    # the rows of one projection: queries, keys and values side by side
    both = rand(n, hq + 2 * hkv, d).to(dt)
    x = dict(q=both[:, :hq], k=both[:, hq:hq + hkv], v=both[:, hq + hkv:])
    if case["op"] == "rope":
        x["pos"] = case["first"] + torch.arange(n, device=DEV, dtype=torch.int32)
        return x
    # queries look for some keys more than for others, as a trained model's do
    both[:, :hq] *= 1.5
    x["rows"] = _lengths(case)
    until = _until(case, x["rows"]) if case["budget"] else None
    x["until"] = None if until is None else torch.from_numpy(until).to(DEV)
    if case["grad"]:
        x["do"] = rand(n, hq, d).to(dt)
    return x


# ------------------------------------------------------------------ plain form
TRAINED, FAST, SLOW = 8192, 32.0, 1.0   # "yarn": rows that the model was trained on, turns within them at both ends of the ramp


def _frequencies(case):
    """Frequencies (64 bits) and the factor of the rotated channels."""
    r, f = case["part"], case["factor"]
    i = np.arange(r // 2)
    if case["scaling"] == "ntk":
        return (THETA * f ** (r / (r - 2.0))) ** (-2.0 * i / r), 1.0
    plain = THETA ** (-2.0 * i / r)
    if case["scaling"] == "linear":
        return plain / f, 1.0
    if case["scaling"] == "none":
        return plain, 1.0
    at = [r * math.log(TRAINED / (turns * 2 * math.pi)) / (2 * math.log(THETA)) for turns in (FAST, SLOW)]
    low, high = max(math.floor(at[0]), 0), min(math.ceil(at[1]), r - 1)
    ramp = np.clip((i - low) / max(high - low, 1e-3), 0, 1)
    return plain * (1 - ramp) + plain / f * ramp, 0.1 * math.log(f) + 1.0


def _turn(x, pos, case):
    f, m = _frequencies(case)
    angle = pos.double()[:, None, None] * torch.from_numpy(f).to(DEV)
    c, s = (m * torch.cos(angle)).float(), (m * torch.sin(angle)).float()
    if case["grad"]:
        s = -s
    r = case["part"]
    y = x.float()
    half = case["layout"] == "half"
    a, b = (y[..., :r // 2], y[..., r // 2:r]) if half else (y[..., 0:r:2], y[..., 1:r:2])
    lo, hi = a * c - b * s, b * c + a * s
    turned = torch.cat([lo, hi], -1) if half else torch.stack([lo, hi], -1).flatten(-2)
    return torch.cat([turned, y[..., r:]], -1).to(x.dtype)


def _attend(x, case):
    """Sequence by sequence, all heads at once; the gradient from the formulas of softmax."""
    hq, hkv, d = case["hq"], case["hkv"], case["d"]
    G, dt, scale = hq // hkv, x["q"].dtype, 1.0 / math.sqrt(d)
    n = len(x["q"])
    out = dict(o=torch.empty((n, hq, d), dtype=dt, device=DEV), lse=torch.empty((hq, n), device=DEV))
    if case["grad"]:
        out.update(dq=torch.empty((n, hq, d), dtype=dt, device=DEV), dk=torch.empty((n, hkv, d), dtype=dt, device=DEV),
                   dv=torch.empty((n, hkv, d), dtype=dt, device=DEV))
    at = 0
    for m in x["rows"].tolist():
        w = slice(at, at + m)
        at += m
        q = x["q"][w].float().view(m, hkv, G, d).permute(1, 2, 0, 3).reshape(hkv, G * m, d)
        k, v = (x[c][w].float().transpose(0, 1).contiguous() for c in ("k", "v"))
        i = torch.arange(m, device=DEV)
        hidden = i[None, :] > i[:, None]
        if x["until"] is not None:
            hidden |= i[:, None] >= x["until"][w][None, :]
        s = torch.bmm(q, k.transpose(1, 2).contiguous()).mul_(scale).view(hkv, G, m, m)
        s.masked_fill_(hidden, -math.inf)
        lse = torch.logsumexp(s, -1)
        p = s.sub_(lse[..., None]).exp_().view(hkv, G * m, m)
        o = torch.bmm(p, v)
        out["o"][w] = o.view(hkv, G, m, d).permute(2, 0, 1, 3).reshape(m, hq, d).to(dt)
        out["lse"][:, w] = lse.view(hq, m)
        if not case["grad"]:
            continue
        do = x["do"][w].float().view(m, hkv, G, d).permute(1, 2, 0, 3).reshape(hkv, G * m, d)
        out["dv"][w] = torch.bmm(p.transpose(1, 2), do).transpose(0, 1).to(dt)
        dp = torch.bmm(do, v.transpose(1, 2).contiguous())
        ds = dp.sub_((do * o).sum(-1, keepdim=True)).mul_(p).mul_(scale)
        out["dq"][w] = torch.bmm(ds, k).view(hkv, G, m, d).permute(2, 0, 1, 3).reshape(m, hq, d).to(dt)
        out["dk"][w] = torch.bmm(ds.transpose(1, 2), q).transpose(0, 1).to(dt)
    return out


def _prefer(x, case):
    vocab, beta, eps, pairs = case["vocab"], case["beta"], case["smoothing"], case["pairs"]
    at = x["target"].long()[:, None]
    seq = torch.repeat_interleave(torch.arange(2 * pairs, device=DEV), torch.from_numpy(x["rows"]).to(DEV).long(), output_size=len(at))

    def log_probs(logits):
        y = logits[:, :vocab].float()
        return y, torch.logsumexp(y, -1)

    y, z = log_probs(x["policy"])
    logp = y.gather(1, at)[:, 0] - z
    if "reference" in x:
        yr, zr = log_probs(x["reference"])
        ratio = logp.double() - (yr.gather(1, at)[:, 0] - zr).double()
    else:
        ratio = logp.double() - x["ref_logp"].double()
    ratios = torch.zeros(2 * pairs, dtype=torch.float64, device=DEV).index_add_(0, seq, ratio)
    h = beta * (ratios[0::2] - ratios[1::2])
    good, bad = torch.log(torch.sigmoid(h)), torch.log(torch.sigmoid(-h))
    loss = -((1 - eps) * good + eps * bad).mean()
    out = dict(losses=torch.stack([loss, h.mean(), (h > 0).double().mean()]).float(), ratios=ratios.float())
    if case["grad"]:
        c = beta * ((1 - eps) * torch.sigmoid(-h) - eps * torch.sigmoid(h)) / pairs
        c = torch.stack([c, -c], -1).flatten()[seq].float()[:, None]
        p = torch.exp(y - z[:, None])
        p.scatter_add_(1, at, torch.full_like(c, -1.0))
        grad = torch.zeros_like(x["policy"])
        grad[:, :vocab] = (c * p).to(grad.dtype)
        out["grad"] = grad
    return out


class Plain:
    def __init__(self, case, seed):
        self.case, self.x = case, _inputs(case, seed)

    def step(self):
        x, case = self.x, self.case
        if case["op"] == "rope":
            return {"q": _turn(x["q"], x["pos"], case), "k": _turn(x["k"], x["pos"], case)}
        return _attend(x, case) if case["op"] == "attn" else _prefer(x, case)


# ------------------------------------------------------------------ the library's calls
class Library:
    """The same through the library: a handle, outputs that the program keeps, arguments marshalled once."""

    def __init__(self, case, seed):
        import paper_2609_31224_amd as a2t
        self.a2t, self.case, self.x = a2t, case, _inputs(case, seed)
        x, lib = self.x, a2t.raw_lib()
        dtype = a2t.A2T_F32 if case["dtype"] == "f32" else a2t.A2T_BF16
        stream = torch.cuda.current_stream()
        p32 = lambda a: a.ctypes.data_as(C.POINTER(C.c_int32))  # noqa: E731
        self.handle = self.destroy = None
        if case["op"] == "rope":
            scaling = {"none": a2t.A2T_ROPE_PLAIN, "linear": a2t.A2T_ROPE_LINEAR, "ntk": a2t.A2T_ROPE_NTK, "yarn": a2t.A2T_ROPE_YARN}[case["scaling"]]
            self.handle = a2t.a2t_rope_create(case["d"], dtype, rotary_dim=case["part"], layout=a2t.A2T_ROPE_HALF if case["layout"] == "half" else a2t.A2T_ROPE_PAIRS,
                                              theta=THETA, scaling=scaling, factor=case["factor"], trained_rows=TRAINED, turns_fast=FAST, turns_slow=SLOW, stream=stream)
            self.destroy = a2t.a2t_rope_destroy
            self.out = {"q": torch.empty_like(x["q"], memory_format=torch.contiguous_format), "k": torch.empty_like(x["k"], memory_format=torch.contiguous_format)}
            q, k, qo, ko = x["q"], x["k"], self.out["q"], self.out["k"]
            self.calls = [(lib.a2t_rope_apply, (self.handle.ptr, len(q), x["pos"].data_ptr(), case["hq"], q.data_ptr(), q.stride(0), qo.data_ptr(), qo.stride(0),
                                                case["hkv"], k.data_ptr(), k.stride(0), ko.data_ptr(), ko.stride(0), int(case["grad"])))]
        elif case["op"] == "attn":
            n = len(x["q"])
            self.handle = a2t.a2t_prompt_create(n, case["hq"], case["hkv"], case["d"], dtype, flags=a2t.A2T_PROMPT_UNTIL if case["budget"] else 0, stream=stream)
            self.destroy = a2t.a2t_prompt_destroy
            o = torch.empty((n, case["hq"], case["d"]), dtype=x["q"].dtype, device=DEV)
            lse = torch.empty((case["hq"], n), dtype=torch.float32, device=DEV)
            self.out = {"o": o, "lse": lse}
            until = None if x["until"] is None else x["until"].data_ptr()
            given = (self.handle.ptr, len(x["rows"]), p32(x["rows"])) + tuple(a for c in "qkv" for a in (x[c].data_ptr(), x[c].stride(0))) + (until,)
            self.calls = [(lib.a2t_prompt_attn, given + (o.data_ptr(), lse.data_ptr()))]
            if case["grad"]:
                # gradients side by side, as the projection's backward pass takes them
                both = torch.empty((n, case["hq"] + 2 * case["hkv"], case["d"]), dtype=x["q"].dtype, device=DEV)
                dq, dk, dv = both[:, :case["hq"]], both[:, case["hq"]:case["hq"] + case["hkv"]], both[:, case["hq"] + case["hkv"]:]
                self.out.update(dq=dq, dk=dk, dv=dv)
                self.calls.append((lib.a2t_prompt_attn_grad, given + (o.data_ptr(), lse.data_ptr(), x["do"].data_ptr(), dq.data_ptr(), dk.data_ptr(), dv.data_ptr())))
        else:
            n = len(x["target"])
            self.handle = a2t.a2t_prefer_create(n, case["vocab"], dtype, stream=stream)
            self.destroy = a2t.a2t_prefer_destroy
            self.out = {"losses": torch.empty(3, device=DEV), "ratios": torch.empty(2 * case["pairs"], device=DEV)}
            if case["grad"]:
                self.out["grad"] = torch.empty_like(x["policy"])
            ptr = lambda t: None if t is None else t.data_ptr()  # noqa: E731
            ref = x.get("reference")
            self.calls = [(lib.a2t_prefer_loss, (self.handle.ptr, case["pairs"], p32(x["rows"]), x["policy"].data_ptr(), x["policy"].stride(0), ptr(ref),
                                                 0 if ref is None else ref.stride(0), ptr(x.get("ref_logp")), x["target"].data_ptr(), case["beta"], case["smoothing"],
                                                 self.out["losses"].data_ptr(), self.out["ratios"].data_ptr(), ptr(self.out.get("grad"))))]

    def step(self):
        for call, args in self.calls:
            rc = call(*args)
            if rc:
                raise self.a2t.A2TError(rc, call.__name__)
        return self.out

    def __del__(self):
        if getattr(self, "handle", None) is not None:
            torch.cuda.synchronize()
            self.destroy(self.handle)


# ------------------------------------------------------------------ the interface
def prepare(case, seed):
    return Library(case, seed) if own else Plain(case, seed)


def run(state):
    return state.step()


def work(case):
    """Least bytes and operations of a pass: inputs read once, outputs written once.  Rotation: ten
    operations a pair.  Attention: two products over the visible pairs, five more for the gradient, which
    also reads O, its gradient and the statistics.  The preference loss: each logit's exponential as
    four operations, twice with a gradient."""
    size = 4 if case["dtype"] == "f32" else 2
    if case["op"] == "rope":
        n = case["rows"] * (case["hq"] + case["hkv"]) * case["d"]
        return {"bytes": 2.0 * n * size + 4.0 * case["rows"], "flops": 5.0 * n * case["part"] / case["d"]}
    if case["op"] == "attn":
        lengths = _lengths(case)
        pairs = _visible(lengths, _until(case, lengths) if case["budget"] else None)
        q, kv, lse = case["rows"] * case["hq"] * case["d"] * size, 2 * case["rows"] * case["hkv"] * case["d"] * size, 4 * case["rows"] * case["hq"]
        by, fl = 2.0 * q + kv + lse, 4.0 * case["d"] * case["hq"] * pairs
        if case["grad"]:
            by, fl = by + 4.0 * q + 2.0 * kv + lse, fl * 3.5
        return {"bytes": by + (4.0 * case["rows"] if case["budget"] else 0.0), "flops": fl}
    rows = float(_answer_rows(case).sum())
    tensors = 1 + case["reference"] + case["grad"]
    return {"bytes": rows * (case["vocab"] * size * tensors + 4 + (0 if case["reference"] else 4)), "flops": rows * case["vocab"] * 4.0 * tensors}


# ------------------------------------------------------------------ 64 bits, from the definition
def _exact_rope(x, case):
    r, f = case["part"], case["factor"]
    theta = THETA * math.pow(f, r / (r - 2.0)) if case["scaling"] == "ntk" else THETA
    turns, m = [], 1.0
    for i in range(r // 2):
        w = math.exp(-2.0 * i / r * math.log(theta))
        if case["scaling"] == "linear":
            w /= f
        if case["scaling"] == "yarn":
            first = max(0, math.floor(r / 2 * math.log(TRAINED / (2 * math.pi * FAST), THETA)))
            last = min(r - 1, math.ceil(r / 2 * math.log(TRAINED / (2 * math.pi * SLOW), THETA)))
            share = min(1.0, max(0.0, (i - first) / max(1e-3, last - first)))
            w, m = w * (1.0 - share + share / f), 1.0 + 0.1 * math.log(f)
        turns.append(w)
    angle = x["pos"].double()[:, None] * torch.tensor(turns, dtype=torch.float64, device=DEV)
    by = torch.polar(torch.full_like(angle, m), -angle if case["grad"] else angle)[:, None]
    out = {}
    for c in ("q", "k"):
        y = x[c].double().clone()
        if case["layout"] == "half":
            z = torch.complex(y[..., :r // 2].contiguous(), y[..., r // 2:r].contiguous()) * by
            y[..., :r // 2], y[..., r // 2:r] = z.real, z.imag
        else:
            y[..., :r] = torch.view_as_real(torch.view_as_complex(y[..., :r].unflatten(-1, (-1, 2)).contiguous()) * by).flatten(-2)
        out[c] = y
    return out


def _exact_attn(x, case):
    hq, G, d = case["hq"], case["hq"] // case["hkv"], case["d"]
    outs = {c: [] for c in (("o", "lse", "dq", "dk", "dv") if case["grad"] else ("o", "lse"))}
    at = 0
    for m in x["rows"].tolist():
        i = torch.arange(m, device=DEV)
        see = i[None, :] <= i[:, None]
        if x["until"] is not None:
            see = see & (i[:, None] < x["until"][at:at + m][None, :])
        q, k, v = (x[c][at:at + m].double().requires_grad_(case["grad"]) for c in "qkv")
        os, ls = [], []
        dq, dk, dv = (torch.zeros(t.shape, dtype=torch.float64, device=DEV) for t in (q, k, v))
        for h in range(hq):
            score = torch.where(see, (q[:, h].contiguous() @ k[:, h // G].contiguous().t()) / d ** 0.5, -math.inf)
            o = torch.softmax(score, -1) @ v[:, h // G].contiguous()
            os.append(o.detach())
            ls.append(torch.logsumexp(score.detach(), -1))
            if case["grad"]:
                for total, part in zip((dq, dk, dv), torch.autograd.grad(o, (q, k, v), x["do"][at:at + m, h].double())):
                    total += part
        outs["o"].append(torch.stack(os, 1))
        outs["lse"].append(torch.stack(ls))
        if case["grad"]:
            for c, total in (("dq", dq), ("dk", dk), ("dv", dv)):
                outs[c].append(total)
        at += m
    return {c: torch.cat(t, 1 if c == "lse" else 0) for c, t in outs.items()}


def _exact_prefer(x, case):
    n, vocab, eps = len(x["target"]), case["vocab"], case["smoothing"]
    rows = torch.arange(n, device=DEV)
    answer = torch.from_numpy(np.repeat(np.arange(2 * case["pairs"]), x["rows"])).to(DEV)
    target = x["target"].long()

    def log_softmax(name, chunk):
        return torch.log_softmax(x[name][chunk, :vocab].double(), -1)[torch.arange(len(chunk), device=DEV), target[chunk]]

    chunks = rows.split(512)
    policy = torch.cat([log_softmax("policy", c) for c in chunks])
    ref = torch.cat([log_softmax("reference", c) for c in chunks]) if "reference" in x else x["ref_logp"].double()
    ratios = torch.stack([(policy - ref)[answer == a].sum() for a in range(2 * case["pairs"])]).requires_grad_()
    h = case["beta"] * (ratios[0::2] - ratios[1::2])
    loss = -((1 - eps) * torch.nn.functional.logsigmoid(h) + eps * torch.nn.functional.logsigmoid(-h)).mean()
    slope, = torch.autograd.grad(loss, ratios)
    out = dict(losses=torch.stack([loss, h.mean(), (h > 0).double().mean()]).detach(), ratios=ratios.detach())
    if case["grad"]:
        grad = torch.zeros(x["policy"].shape, dtype=torch.float64, device=DEV)
        for c in chunks:
            p = -torch.softmax(x["policy"][c, :vocab].double(), -1)
            p[torch.arange(len(c), device=DEV), target[c]] += 1.0
            grad[c, :vocab] = slope[answer[c]][:, None] * p
        out["grad"] = grad
    return out


def exact(case, seed):
    x = _inputs(case, seed)
    return {"rope": _exact_rope, "attn": _exact_attn, "prefer": _exact_prefer}[case["op"]](x, case)
