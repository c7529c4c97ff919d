"""Rotary positions and the 8-bit cache without a GPU: what the entry points answer at the edges of their arguments."""
import ctypes

import numpy as np
import pytest
import torch

from paper_2507_10069_amd import binding as B
from test_fp8_host import OK, _batch, _cache, _rope

FAR = 0x1000000


def test_given_positions_turn_rows_of_no_request():
    """A batch without requests is no empty one where positions are given: its rows are looked at like any others."""
    lib, b = B.load(), _batch(arrays=False, num_reqs=0, max_new_len=0)
    given = ctypes.byref(_rope(num_axes=1, sections=(64, 0, 0, 0), positions=OK))
    assert lib.emm_rope(b, given, None, None, 0, None, None, None) == B.EMM_ERR_NULL
    assert lib.emm_rope(b, given, OK, None, 0, None, None, None) == B.EMM_ERR_NULL
    assert lib.emm_rope(b, given, OK + 8, None, 0, FAR, None, None) == B.EMM_ERR_INVALID_ARG
    missing = ctypes.byref(_rope(num_axes=1, sections=(64, 0, 0, 0)))
    assert lib.emm_rope(b, missing, OK, None, 0, FAR, None, None) == B.EMM_ERR_NULL
    # places in requests: without requests there are none
    assert lib.emm_rope(b, ctypes.byref(_rope()), OK, None, 0, FAR, None, None) == B.EMM_OK


def test_rotation_and_write_without_requests_is_the_rotation():
    lib, b, c = B.load(), _batch(arrays=False, num_reqs=0, max_new_len=0), ctypes.byref(_cache())
    given = ctypes.byref(_rope(num_axes=1, sections=(64, 0, 0, 0), positions=OK))
    assert lib.emm_rope_kv_scatter_fp8(b, given, OK, OK, OK, 0, None, c, None) == B.EMM_ERR_NULL
    assert lib.emm_rope_kv_scatter_fp8(b, given, OK, OK, OK, 0, FAR + 4, c, None) == B.EMM_ERR_INVALID_ARG
    assert lib.emm_rope_kv_scatter_fp8(b, given, OK, OK, OK, 0, OK + 256, c, None) == B.EMM_ERR_INVALID_ARG
    assert lib.emm_rope_kv_scatter_fp8(b, ctypes.byref(_rope()), OK, OK, OK, 0, FAR, c, None) == B.EMM_OK
    assert lib.emm_kv_scatter_fp8(b, OK, OK, 0, c, None) == B.EMM_OK


def test_strides_beyond_any_memory_are_refused():
    """Rows so far apart that the bytes they span pass 2^63: refused by the check itself, which counts them."""
    lib, c = B.load(), ctypes.byref(_cache())
    b, r = _batch(total_new_tokens=1 << 25), ctypes.byref(_rope())
    for stride in (1 << 40, (1 << 40) + 8, 1 << 38, 1 << 62):
        assert lib.emm_rope(b, r, OK, None, stride, FAR, None, None) == B.EMM_ERR_INVALID_ARG, stride
        assert lib.emm_rope_kv_scatter_fp8(b, r, OK, OK, OK, stride, FAR, c, None) == B.EMM_ERR_INVALID_ARG, stride
        assert lib.emm_kv_scatter_fp8(b, OK, OK, stride, c, None) == B.EMM_ERR_INVALID_ARG, stride


def test_positions_without_axes_are_refused():
    """(as positions of the wrong type are: by the binding, before there is a descriptor)"""
    inv = torch.zeros(64, dtype=torch.float64)
    for shape in ((0, 5), (0, 0)):
        with pytest.raises(ValueError):
            B.make_rope(inv, rotary_dim=128, positions=torch.zeros(shape, dtype=torch.int32))
    five = B.make_rope(inv, rotary_dim=128, positions=torch.zeros(5, 20, dtype=torch.int32), sections=[16, 16, 16, 8, 8])
    assert B.load().emm_rope(_batch(), ctypes.byref(five), OK, None, 0, FAR, None, None) == B.EMM_ERR_INVALID_ARG


@pytest.mark.parametrize("kind", ["yarn", "bands"])
@pytest.mark.parametrize("original_len,slow,fast", [(6, 1.0, 32.0), (1, 0.5, 1.0), (100, 20.0, 32.0), (150, 24.0, 25.0)])
def test_frequencies_that_all_turn_too_seldom_are_all_divided(kind, original_len, slow, fast):
    """Even the highest frequency has fewer than `slow` turns in the trained length."""
    n, base, scale = 64, 1e4, 8.0
    plain = base ** (-2.0 * np.arange(n // 2) / n)
    assert original_len / (2 * np.pi) < slow
    inv, _ = B.emm_rope_inv_freq_host(n, base, kind, scale, original_len, slow=slow, fast=fast)
    assert np.allclose(inv, plain / scale, rtol=1e-13, atol=0)


@pytest.mark.parametrize("kind", ["yarn", "bands"])
def test_frequencies_that_all_turn_often_enough_stay(kind):
    n, base = 64, 1e4
    plain = base ** (-2.0 * np.arange(n // 2) / n)
    inv, _ = B.emm_rope_inv_freq_host(n, base, kind, 8.0, 2 ** 31 - 1, slow=1.0, fast=32.0)
    assert (2 ** 31 - 1) * plain[-1] / (2 * np.pi) > 32 and np.allclose(inv, plain, rtol=1e-13, atol=0)


@pytest.mark.parametrize("reqs", [1, 2, 600])
def test_tables_without_pages(reqs):
    """A size is told without dividing by what there is none of, and the call itself is refused."""
    n = ctypes.c_size_t(7)
    b = _batch(num_reqs=reqs, total_new_tokens=reqs, max_new_len=1, max_pages_per_req=0)
    assert B.load().emm_attn_fp8_workspace_size(b, ctypes.byref(n)) == B.EMM_OK
    assert B.load().emm_decode_attn_fp8(b, OK, ctypes.byref(_cache()), FAR, None, OK, 1 << 40, None) == B.EMM_ERR_INVALID_ARG
