"""Frequencies of rotary positions against their formulas, and what their calls refuse; no GPU is touched."""
import ctypes as C
import math

import pytest


def _frequencies(turned, base=10000.0, scaling=0, factor=1.0, original=0.0, low=1.0, high=32.0):
    from paper_2509_24859_amd import binding
    out, magnitude = (C.c_double * max(turned // 2, 1))(), C.c_float(-7)
    rc = binding.load_library().harp_rotary_frequencies(turned, base, scaling, factor, original, low, high, out, C.byref(magnitude))
    return rc, list(out), magnitude.value


def _close(got, want):
    """pow of the two libraries: a few units of 2^-53 each."""
    assert len(got) == len(want) and all(abs(g - w) <= 8 * 2.0 ** -53 * w for g, w in zip(got, want)), (got, want)


@pytest.mark.parametrize("turned", [2, 6, 64, 72, 128, 256])
@pytest.mark.parametrize("base", [10000.0, 500000.0])
def test_formulas(turned, base):
    plain = [base ** (-2 * i / turned) for i in range(turned // 2)]
    rc, got, magnitude = _frequencies(turned, base)
    assert rc == 0 and magnitude == 1
    _close(got, plain)
    rc, got, magnitude = _frequencies(turned, base, 1, 4.0)
    assert rc == 0 and magnitude == 1
    _close(got, [f / 4 for f in plain])
    rc, got, magnitude = _frequencies(turned, base, 3, 8.0, 4096.0, 1.0, 32.0)
    want = []
    for f in plain:
        g = min(1, max(0, (4096 * f / (2 * math.pi) - 1) / 31))
        want.append(f * ((1 - g) / 8 + g))
    assert rc == 0 and abs(magnitude - (0.1 * math.log(8) + 1)) < 2.0 ** -23
    assert all(abs(g - w) <= 64 * 2.0 ** -53 * w for g, w in zip(got, want))


@pytest.mark.parametrize("turned", [6, 64, 128])
def test_the_base_is_stretched_so_that_the_last_pair_is(turned):
    _, plain, _ = _frequencies(turned)
    rc, got, _ = _frequencies(turned, scaling=2, factor=4.0)
    assert rc == 0 and got[0] == 1
    assert abs(got[-1] - plain[-1] / 4) <= 1e-13 * plain[-1]


@pytest.mark.parametrize("kw", [dict(turned=0), dict(turned=3), dict(turned=1 << 16), dict(turned=8, base=0.0), dict(turned=8, base=math.inf),
                                dict(turned=8, base=math.nan), dict(turned=8, scaling=4), dict(turned=8, scaling=-1),
                                dict(turned=8, scaling=1, factor=0.5), dict(turned=8, scaling=1, factor=math.nan),
                                dict(turned=2, scaling=2, factor=2.0), dict(turned=8, scaling=3, factor=2.0, original=0.0),
                                dict(turned=8, scaling=3, factor=2.0, original=64.0, low=4.0, high=4.0)])
def test_refusals(kw):
    assert _frequencies(**kw)[0] < 0
