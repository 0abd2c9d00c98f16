"""The framework's calls on the listed performance cases of the gated block and of 4-bit weights, at
their own sizes, against exact() in 64 bits.

Tolerances are relative to a whole output's 2-norm, for outputs of thousands of elements and more. bf16 results
are off by their own rounding: at most half a step, 2^-8 of a value, rms not over 2^-8 / sqrt(3) (uniform within
the half step). The gradients from dg and du rounded to bf16 are sums of terms that are off by as
much again, so sqrt(2) of that and with it rms 2^-8 sqrt(2 / 3) at most. fp32 sums over n products round n
times, each by at most 2^-24 of the largest partial sum; independent roundings add up as sqrt(n) 2^-24. What a
largest element may be off is tested at small sizes in test_gpu_gated.py and test_gpu_q4.py."""
import math

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from perf import more_operators as operators  # noqa: E402

CASES = {c["name"]: {k: v for k, v in c.items() if k != "name"} for c in operators.listed()}


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


@pytest.mark.parametrize("name", CASES)
def test_listed_case(monkeypatch, name):
    case, seed = CASES[name], 5
    monkeypatch.setattr(operators, "own", True)
    got = operators.run(operators.prepare(case, seed))
    ref = operators.exact(case, seed)
    if not isinstance(got, dict):
        got, ref = {"out": got}, {"out": ref}
    for k in got:
        g, r = got[k].double(), ref[k]
        assert g.shape == r.shape and bool(torch.isfinite(g).all())
        if got[k].dtype is torch.bfloat16:
            most = 2.0 ** -8 * math.sqrt((2 if case["op"] == "backward" else 1) / 3)
        else:
            sums = {"forward": case.get("d_model", 0),
                    "backward": 3 * max(2 * case.get("d_ff", 0), case["tokens"]) + case.get("d_model", 0)}
            n = sums.get(case["op"], 8 * case.get("cols", 0))  # 4-bit: terms up to 8 times as large
            most = math.sqrt(n) * 2.0 ** -24
        assert float((g - r).norm() / r.norm()) <= most, k
