"""The measure that the steps from pages are held to (tests/paged_forms.py), on the CPU: vectors as head and remainder pass it, and a
rounding of any one vector to bf16 does not, for y or for the new pair."""
import numpy as np
import pytest

from paper_2604_21215_amd import inputs as gen
from tests import paged_forms as forms

CASES = [("bf16", 256, 512, 1.0, 12), ("bf16", 512, 1024, 0.125, 6)]


def _case(d, F, scale, S, seed=3):
    rng = np.random.default_rng(seed)
    form = ("", "bf16", 0, d, F, 70, 16, 0.0, scale, [(11 * s) % 70 for s in range(S)])
    x, w, g = forms.inputs(form)
    H, caches = d // 64, []
    for n in form[9]:
        k = rng.standard_normal((n, H, 64))
        k /= np.sqrt((k * k).mean(-1, keepdims=True)) if n else 1
        caches.append((gen.round_to_bf16(k.astype(np.float32)).astype(np.float64),
                       gen.round_to_bf16((rng.standard_normal((n, H, 64)) * 0.6).astype(np.float32)).astype(np.float64)))
    f64 = lambda m: {n: t.astype(np.float64) for n, t in m.items()}  # noqa: E731
    return lambda alter=lambda name, u: u: forms.step(f64(w), f64(g), x.astype(np.float64), caches, H, scale, 0.0, alter=alter)


def _split(name, u):
    if name in ("q", "k_t", "v_t"):   # fp32 rows
        return u.astype(np.float32).astype(np.float64)
    head = forms.to_bf16(u)
    return head + np.where(u == head, 0.0, forms.to_bf16(np.where(u == head, 1.0, u - head)))


def _moved(got, want, rows):
    return [forms.moved(r(a), b, s) for a, b, (r, s) in zip(got, want, rows)]


@pytest.mark.parametrize("dtype,d,F,scale,S", CASES)
@pytest.mark.parametrize("bits", [0, 8])
def test_one_rounding_shows(dtype, d, F, scale, S, bits):
    run = _case(d, F, scale, S)
    want = run()
    rows = [(forms.to_bf16, forms.bf16_ulp(want[0]))]
    for u in want[1:]:
        s = forms.row_step(u) if bits else forms.bf16_ulp(u)
        rows.append(((lambda a, s=s: np.rint(a / s) * s) if bits else forms.to_bf16, s))
    for flips, most in _moved(run(_split), want, rows):
        assert flips <= most / 4, (flips, most)
    for vector in forms.VECTORS:
        res = _moved(run(lambda name, u: forms.to_bf16(u) if name == vector else u), want, rows)
        assert any(flips > most for flips, most in res), (vector, res)
