"""Planted mistakes in copies of the oracle's optimizer side: the pins have to notice each."""
import pytest

from test_oracle_mutations import SRC, _build, _pins_pass

PINS = "test_oracle_optimizer.py"
MUTATIONS = {
    "norm without the root": ("norm[n] = sqrt(sum);", "norm[n] = sum;"),
    "norm from the first tensor on": ("for (int s = seg_lo; s < seg_hi; ++s)\n            for (int64_t c", "for (int s = 0; s < seg_hi; ++s)\n            for (int64_t c"),
    "factor above one": ("if (c > 1.0) c = 1.0;", ""),
    "factor upside down": ("double c = max_norm / (norm + 1e-6);", "double c = norm / (max_norm + 1e-6);"),
    "decay of the first tensor for all": ("(float)hyper[4] * (float)decay[s];", "(float)hyper[4] * (float)decay[0];"),
    "momentum weighs the gradient too": ("m[idx] = fmaf(b1, m[idx], u);", "m[idx] = fmaf(b1, m[idx], keep1 * u);"),
    "nesterov always": ("u = nesterov ? fmaf(b1, m[idx], u) : m[idx];", "u = fmaf(b1, m[idx], u);"),
    "no bias correction of the first moment": ("top = first * m[idx];", "top = m[idx];"),
    "bias correction a step late": ("(long double)step + 1.0L;", "(long double)step + 2.0L;"),
    "second moment of the unclipped gradient's size": ("new2 = half * g;", "new2 = half;"),
    "eps inside the root": ("denom = fmaf(second, sqrtf(v[idx]), eps)", "denom = second * sqrtf(v[idx] + eps)"),
    "coupled decay": ("u = fmaf(wd, p, ratio);", "u = ratio;"),
    "skipped models stepped": ("if (skip && norm && !isfinite(norm[n])) continue;", ""),
}


def test_unmodified_copy_passes(tmp_path):
    with open(SRC) as f:
        text = f.read()
    lib = str(tmp_path / "same.so")
    _build(text, lib)
    ok, tail = _pins_pass(lib, PINS)
    assert ok, tail


@pytest.mark.parametrize("name", sorted(MUTATIONS))
def test_mistake_is_caught(name, tmp_path):
    old, new = MUTATIONS[name]
    with open(SRC) as f:
        text = f.read()
    assert text.count(old) == 1, "the planted mistake's place is not unique"
    lib = str(tmp_path / "mutant.so")
    _build(text.replace(old, new), lib)
    ok, _ = _pins_pass(lib, PINS)
    assert not ok, "no pin noticed: " + name
