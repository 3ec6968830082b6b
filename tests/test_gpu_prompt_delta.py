"""dO . O of rows that see few keys: formed from fp32 scores, not from the O that was rounded to bf16, which
costs as much as all other roundings together where a row's weight is on few keys.

Element by element within the oracle's bounds without that rounding.  And in the 2-norm as far off as a replay of the
other roundings in 64 bits: fp32 errors of 2^-20 of a value move one rounding in 2^12 to the next number of bf16,
2^-7 away, 2^-13 in the 2-norm beside the 2^-9 of all roundings, 1/500 of their sum's; 1.02 of it are allowed, where
the O's rounding makes it 1.08 to 2.9 (test_oracle_prompt_delta.py)."""
import numpy as np
import pytest

from oracle.prompt import prompt_attention
from tests.test_gpu_prompt import _case, _f64, _run
from tests.test_oracle_prompt_delta import replay

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("lengths,hq,hkv,d", [([3] * 60, 2, 1, 128), ([2, 6, 1, 16, 5, 9] * 5, 4, 2, 64), ([64, 61, 33], 8, 2, 128), ([64, 64, 40], 3, 3, 64),
                                              ([128, 100, 127, 65], 4, 1, 128), ([128, 66], 2, 2, 64)])
@pytest.mark.parametrize("until,sort,splits", [(None, 1, 0), (None, 1, 3), ("random", 1 << 20, 0), ("evicted", 1, 0), ("random", 1, 2)])
def test_short_sequences(gpu, monkeypatch, until, sort, splits, lengths, hq, hkv, d):
    import paper_2609_31224_amd as a2t
    monkeypatch.setenv("A2T_PROMPT_SORT", str(sort))
    monkeypatch.setenv("A2T_PROMPT_SPLITS", str(splits))
    # sorted keys are two runs: 64 rows at most are two tiles for sure
    at_most = 64 if until and sort == 1 else 128
    lengths = [min(n, at_most) for n in lengths]
    q, k, v, do, ut = _case(lengths, hq, hkv, d, "bf16", until, seed=d + len(lengths))
    h = a2t.a2t_prompt_create(sum(lengths), hq, hkv, d, a2t.A2T_BF16, flags=0 if until is None else a2t.A2T_PROMPT_UNTIL)
    try:
        got = _run(h, lengths, q, k, v, do, ut)
    finally:
        a2t.a2t_prompt_destroy(h)
    ref = prompt_attention(lengths, _f64(q), _f64(k), _f64(v), ut, _f64(do), u_store=2.0 ** -8, u_mul=2.0 ** -8, delta_rows=at_most)
    again = dict(zip(("dq", "dk"), replay(lengths, _f64(q), _f64(k), _f64(v), _f64(do), False, ut)))
    for c, want in ref.grads.items():
        off = np.abs(_f64(got[c]) - want)
        assert (off <= ref.bounds[c] + 1e-30).all(), c
        if c in again:
            norm, least = np.linalg.norm(off), np.linalg.norm(again[c] - want)
            print(f"[delta] {c}: {norm / np.linalg.norm(want):.5f} of the 2-norm, {norm / least:.4f} of the replay's", flush=True)
            assert norm <= 1.02 * least, c


def test_whole_range_of_blocks(gpu):
    """A long sequence's first rows beside later ones: both within the bounds with the stored O, the first 128 rows'
    dQ within those without."""
    import paper_2609_31224_amd as a2t
    lengths = [700, 120]
    q, k, v, do, _ = _case(lengths, 4, 2, 128, "bf16", None, seed=5)
    h = a2t.a2t_prompt_create(820, 4, 2, 128, a2t.A2T_BF16)
    try:
        got = _run(h, lengths, q, k, v, do, None)
    finally:
        a2t.a2t_prompt_destroy(h)
    whole = prompt_attention(lengths, _f64(q), _f64(k), _f64(v), None, _f64(do), u_store=2.0 ** -8, u_mul=2.0 ** -8)
    first = prompt_attention([128], *(_f64(x[:128]) for x in (q, k, v)), None, _f64(do[:128]), u_store=2.0 ** -8, u_mul=2.0 ** -8, delta_rows=128)
    for c, want in whole.grads.items():
        assert (np.abs(_f64(got[c]) - want) <= whole.bounds[c] + 1e-30).all(), c
    assert (np.abs(_f64(got["dq"][:128]) - first.grads["dq"]) <= first.bounds["dq"] + 1e-30).all()
