"""Attention over the 8-bit cache at the two ends of V's range, against oracle.c in 64 bits.  Tolerances are those of
test_gpu_fp8_cache.py without their absolute part, which small values would hide behind; where V has the least scale, weights
that are subnormal in bf16 add half a step of 2^-133 for each code of at most 448, and so does out."""
import numpy as np
import pytest

from oracle import fp8_model as F
from paper_2507_10069_amd import binding as B
from paper_2507_10069_amd import workloads as W
from test_gpu_fp8_cache import Batch, _dev, _f64
import torch

pytestmark = pytest.mark.gpu

WAYS = {"few rows": dict(prefix=[400, 90, 2000], new=[1, 1, 1]), "32 rows": dict(prefix=[400, 90] * 3, new=[4] * 6),
        "chunks": dict(prefix=[400, 90], new=[60, 33]), "a chunk in pieces": dict(prefix=[3000], new=[36])}


def _check(b, q, extra=0.0):
    out, lse = b.attend(q)
    want, want_lse, size = b.reference(B.DeviceWorkload.to_numpy_bits(q)[: b.T])
    got, keys = _f64(out)[: b.T], int((b.prefix + b.new).max())
    longest = [np.linalg.norm(x, axis=-1).max() for x in (_f64(q), W.bf16_bits_to_f32(b.bits("k")).astype(np.float64))]
    e = 130 * 2.0 ** -24 * b.batch.softmax_scale * longest[0] * longest[1]
    bound = (2.0 ** -8 + 2 * e + keys * 2.0 ** -24) * size + 2.0 ** -8 * np.abs(want) + extra
    assert np.isfinite(got).all() and (np.abs(got - want) <= bound).all(), float((np.abs(got - want) / bound).max())
    assert (np.abs(_f64(lse)[: b.T] - want_lse) <= e + keys * 2.0 ** -24 + 2.0 ** -22 * np.abs(want_lse) + 2.0 ** -22).all()


@pytest.mark.parametrize("way", list(WAYS))
def test_values_of_the_least_scale(way):
    print("case least scale", way, flush=True)
    b = Batch(seed=31, **WAYS[way]).fill_contexts()
    for r, c in enumerate(b.prefix + b.new):
        b.fill("v", r, 0, b.rng.uniform(225, 448, (c, 4, 128)) * b.rng.choice([-1, 1], (c, 4, 128)) * 2.0 ** F.LEAST_EXPONENT)
    assert (b.scales["v"][b.valid["v"]] == F.LEAST_EXPONENT + F.BIAS).all()
    b.to_device()
    _check(b, b.queries(2.0), (448 * int((b.prefix + b.new).max()) + 1) * 2.0 ** -134)


@pytest.mark.parametrize("way", list(WAYS))
def test_values_as_large_as_the_header_allows(way):
    """Just inside 2^16 * slots * |v| = 2^127, and with the largest weights there can be: scores of zero in the first tile, which is the
    reference, and from then on such that every weight is 2^15.94 (16 of them sum to just less than what moves it)."""
    print("case largest values", way, flush=True)
    b = Batch(seed=32, **WAYS[way]).fill_contexts()
    slots = int((b.prefix + b.new).max())
    exponent = int(np.floor(np.log2(2.0 ** 111 / slots / 448)))
    for r, c in enumerate(b.prefix + b.new):
        k = np.ones((c, 4, 128))
        k[:64] = 0
        b.fill("k", r, 0, k)
        b.fill("v", r, 0, np.full((c, 4, 128), 448.0) * 2.0 ** exponent * np.where(np.arange(128) % 3 == 0, -1, 1))
    b.to_device()
    q = _dev(np.full((b.rows, 28, 128), 250 / 256, np.float32), torch.bfloat16)
    assert 15.9 < 250 / 256 * 128 * b.batch.softmax_scale * np.log2(np.e) < 16
    _check(b, q)
