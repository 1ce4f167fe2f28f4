"""The precision of salt_attend against the float64 oracle, with bounds close enough to show one lost bf16 term of q or
of the probabilities (tests/attend_precision.py gives them; tests/test_attend_precision.py holds them against a model of
the arithmetic with a term less)."""
import numpy as np
import pytest

from tests import attend_precision as ap

pytestmark = pytest.mark.gpu


def _attend(b):
    b.open()
    try:
        b.fill()
        b.set()
        return b.attend()
    finally:
        b.close()


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("std", [0.05, 2.0])
@pytest.mark.parametrize("kind", ap.F32)
def test_fp32_keeps_three_terms(kind, std, dim, fmt):
    print(f"\n[gpu case] attend precision f32, {kind} std={std} dim={dim} {fmt}", flush=True)
    b = ap.f32_batch(kind, std, fmt, dim)
    r = ap.ratios_f32(b, _attend(b), ap.rows_of(b, 3))
    rms = float(np.sqrt(np.mean(r ** 2)))
    print(f"largest {r.max():.3f}, root mean square {rms:.3f}", flush=True)
    assert r.max() <= 1.0 and rms <= ap.RMS_LIMIT


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
@pytest.mark.parametrize("kind", ap.BF16)
def test_bf16_keeps_its_terms(kind, fmt):
    print(f"\n[gpu case] attend precision bf16, {kind} {fmt}", flush=True)
    b = ap.bf16_batch(kind, fmt)
    terms = 1 if fmt == "e4m3" and kind.endswith("rows") else 2
    r = ap.ratios_bf16(b, _attend(b), ap.rows_of(b, 3), terms)
    print(f"largest {r.max():.3f} of the bound for {terms} terms", flush=True)
    assert r.max() <= 1.0
