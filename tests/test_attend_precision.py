"""The bounds of tests/test_gpu_attend_precision.py against a model of the kernels' arithmetic on the same batches: with
all its terms it keeps to them by a margin, with one term of q or of the probabilities less it does not."""
import numpy as np
import pytest

from tests import attend_precision as ap

_rms = lambda r: float(np.sqrt(np.mean(r ** 2)))


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("kind", ap.F32)
def test_a_lost_third_term_shows(kind, dim, fmt):
    for std, less in ((0.05, (3, 2)), (2.0, (2, 3))):
        b = ap.f32_batch(kind, std, fmt, dim)
        rows = ap.rows_of(b, 9)
        r = ap.ratios_f32(b, ap.model(b, rows, 3, 3), rows)
        assert r.max() <= 0.5 and _rms(r) <= ap.RMS_LIMIT / 2, (std, r.max(), _rms(r))
        assert _rms(ap.ratios_f32(b, ap.model(b, rows, *less), rows)) >= ap.RMS_LIMIT * 2, std


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
@pytest.mark.parametrize("kind", ap.BF16)
def test_a_lost_second_term_shows(kind, fmt):
    b = ap.bf16_batch(kind, fmt)
    rows = ap.rows_of(b, 9)
    two, one = (ap.model(b, rows, 1, n) for n in (2, 1))
    assert ap.ratios_bf16(b, two, rows, 2).max() <= 1.0 and ap.ratios_bf16(b, one, rows, 1).max() <= 1.0
    assert ap.ratios_bf16(b, one, rows, 2).max() >= 2.0
