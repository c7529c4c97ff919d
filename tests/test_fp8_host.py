"""Rotary positions and the 8-bit cache on a machine without a GPU: exports, descriptors, refusals before any HIP call,
and the frequencies that the host computes."""
import ctypes
import math
import os
import re
import subprocess

import numpy as np
import pytest

from paper_2507_10069_amd import binding as B

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
OK = 0x1000                                                  # a pointer that is never followed


def _batch(arrays=True, **over):
    kw = dict(num_reqs=2, num_q_heads=8, num_kv_heads=2, head_dim=128, page_size=16, num_pages=10, max_pages_per_req=4,
              total_new_tokens=20, max_new_len=12, dtype="bf16", softmax_scale=0.1)
    kw.update(over)
    b = B.make_batch(**kw)
    if arrays:
        b.page_table = b.prefix_lens = b.new_lens = b.cu_new_lens = OK
    return b


def _rope(**over):
    r = B.emm_rope_params(0, 128, 0, 0, (ctypes.c_int32 * 4)(0, 0, 0, 0), 1.0, 0, OK, None)
    for k, v in over.items():
        setattr(r, k, (ctypes.c_int32 * 4)(*v) if k == "sections" else v)
    return r


def _cache(**over):
    c = B.emm_fp8_cache(OK, OK, OK, OK)
    for k, v in over.items():
        setattr(c, k, v)
    return c


def test_exports_match_the_header():
    lib = B.load()
    with open(os.path.join(ROOT, "include", "emm_fp8.h")) as f:
        header = f.read()
    declared = sorted(set(re.findall(r"^emm_status (emm_[a-z_0-9]+)\(", header, re.M)))
    assert declared == sorted(B.FP8_EXPORTS)
    for name in declared + ["emm_rope", "emm_rope_inv_freq_host"]:
        assert hasattr(lib, name), name


def test_header_is_plain_c99_and_structs_have_its_layout(tmp_path):
    src = tmp_path / "sizes.c"
    src.write_text('#include "emm_fp8.h"\n#include <stdio.h>\nint main(void) { printf("%zu %zu %zu", sizeof(emm_rope_params), '
                   'sizeof(emm_rope_scaling), sizeof(emm_fp8_cache)); return 0; }\n')
    exe = tmp_path / "sizes"
    subprocess.run(["gcc", "-std=c99", "-pedantic", "-Wall", "-Wextra", "-Werror", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe)], check=True)
    out = subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout.split()
    assert [int(x) for x in out] == [ctypes.sizeof(t) for t in (B.emm_rope_params, B.emm_rope_scaling, B.emm_fp8_cache)]


BATCHES = [(dict(num_q_heads=7), "INVALID_ARG"), (dict(softmax_scale=0.0), "INVALID_ARG"), (dict(dtype=5), "INVALID_ARG"),
           (dict(page_size=48), "UNSUPPORTED"), (dict(head_dim=96), "UNSUPPORTED"), (dict(max_new_len=21), "INVALID_ARG")]


@pytest.mark.parametrize("over,status", BATCHES)
def test_bad_batches_are_refused_by_all(over, status):
    lib, b, want = B.load(), _batch(**over), getattr(B, "EMM_ERR_" + status)
    r, c, n = ctypes.byref(_rope()), ctypes.byref(_cache()), ctypes.c_size_t()
    assert lib.emm_rope(b, r, OK, OK, 0, 0x100000, 0x200000, None) == want
    assert lib.emm_kv_scatter_fp8(b, OK, OK, 0, c, None) == want
    assert lib.emm_rope_kv_scatter_fp8(b, r, OK, OK, OK, 0, 0x100000, c, None) == want
    assert lib.emm_kv_gather_fp8(b, c, OK, OK, None) == want
    assert lib.emm_attn_fp8_workspace_size(b, ctypes.byref(n)) == want
    assert lib.emm_prefill_attn_fp8(b, OK, c, OK, None, OK, 1 << 40, None) == want
    for name in ("emm_rope", "emm_kv_scatter_fp8", "emm_rope_kv_scatter_fp8", "emm_kv_gather_fp8"):
        fn = getattr(lib, name)
        assert fn(None, *[None if t is not ctypes.c_int64 else 0 for t in fn.argtypes[1:]]) == B.EMM_ERR_NULL


ROPES = [(dict(layout=2), "INVALID_ARG"), (dict(rotary_dim=0), "INVALID_ARG"), (dict(rotary_dim=136), "INVALID_ARG"), (dict(rotary_dim=24), "UNSUPPORTED"),
         (dict(num_axes=5), "INVALID_ARG"), (dict(inverse=2), "INVALID_ARG"), (dict(reserved=1), "INVALID_ARG"), (dict(factor=math.nan), "INVALID_ARG"),
         (dict(num_axes=2, sections=(32, 31, 0, 0), positions=OK), "INVALID_ARG"), (dict(num_axes=2, sections=(65, -1, 0, 0), positions=OK), "INVALID_ARG"),
         (dict(positions=OK), "INVALID_ARG"), (dict(num_axes=1, sections=(64, 0, 0, 0)), "NULL"), (dict(inv_freq=None), "NULL"),
         (dict(inv_freq=OK + 4), "INVALID_ARG"), (dict(num_axes=1, sections=(64, 0, 0, 0), positions=OK + 2), "INVALID_ARG")]


@pytest.mark.parametrize("over,status", ROPES)
def test_bad_rotations_are_refused(over, status):
    lib, want = B.load(), getattr(B, "EMM_ERR_" + status)
    r = ctypes.byref(_rope(**over))
    assert lib.emm_rope(_batch(), r, OK, OK, 0, 0x100000, 0x200000, None) == want
    assert lib.emm_rope_kv_scatter_fp8(_batch(), r, OK, OK, OK, 0, 0x100000, ctypes.byref(_cache()), None) == want


def test_rows_strides_and_overlaps():
    lib, b, r, c = B.load(), _batch(), ctypes.byref(_rope()), ctypes.byref(_cache())
    far, further = 0x1000000, 0x2000000
    invalid, null = B.EMM_ERR_INVALID_ARG, B.EMM_ERR_NULL
    q_row, k_row = 8 * 128, 2 * 128
    assert lib.emm_rope(b, r, OK, None, 0, None, None, None) == null           # an output is missing
    assert lib.emm_rope(b, r, None, None, 0, None, None, None) == null
    assert lib.emm_rope(b, r, None, OK, 0, far, further, None) == null
    assert lib.emm_rope(b, r, OK + 8, None, 0, far, None, None) == invalid     # alignment
    assert lib.emm_rope(b, r, OK, None, q_row - 8, far, None, None) == invalid  # rows would overlap
    assert lib.emm_rope(b, r, OK, None, q_row + 4, far, None, None) == invalid  # rows would not be aligned
    assert lib.emm_rope(b, r, OK, None, -q_row, far, None, None) == invalid
    assert lib.emm_rope(b, r, OK, None, q_row + 2 * k_row, OK, None, None) == invalid          # in place, but strided
    assert lib.emm_rope(b, r, OK, None, 0, OK + 256, None, None) == invalid    # shifted by a head
    assert lib.emm_rope(b, r, OK, far, 0, far + 16, further, None) == invalid  # q's output over k
    assert lib.emm_rope(b, r, OK, far, 0, further, further + 512, None) == invalid             # both outputs
    eight = _batch(num_kv_heads=8)
    assert lib.emm_rope(eight, r, OK, far, 0, far, OK, None) == invalid        # each the other's output
    assert lib.emm_kv_scatter_fp8(b, OK, OK, k_row - 8, c, None) == invalid
    assert lib.emm_rope_kv_scatter_fp8(b, r, OK, far, far, k_row, further, c, None) == invalid  # the stride holds k and v, not q
    assert lib.emm_rope_kv_scatter_fp8(eight, r, OK, far, far, 0, far, c, None) == invalid     # q's output over k and v
    assert lib.emm_rope_kv_scatter_fp8(b, r, None, far, far, 0, further, c, None) == null
    assert lib.emm_rope_kv_scatter_fp8(b, None, OK, far, far, 0, further, c, None) == null
    assert lib.emm_kv_gather_fp8(b, c, OK, None, None) == null


def test_caches_and_workspaces():
    lib, b, c = B.load(), _batch(), ctypes.byref(_cache())
    for name in ("k", "v", "k_scale", "v_scale"):
        for value, want in ((None, B.EMM_ERR_NULL), (OK + 8, B.EMM_ERR_INVALID_ARG)):
            bad = ctypes.byref(_cache(**{name: value}))
            assert lib.emm_kv_scatter_fp8(b, OK, OK, 0, bad, None) == want
            assert lib.emm_kv_gather_fp8(b, bad, OK, OK, None) == want
            assert lib.emm_prefill_attn_fp8(b, OK, bad, OK, None, OK, 1 << 40, None) == want
    assert lib.emm_kv_scatter_fp8(b, OK, OK, 0, None, None) == B.EMM_ERR_NULL
    assert lib.emm_prefill_attn_fp8(b, OK, None, OK, None, OK, 1 << 40, None) == B.EMM_ERR_NULL
    for over in (dict(head_dim=64), dict(dtype="f32")):
        assert lib.emm_cross_attn_fp8(_batch(**over), OK, c, OK, None, OK, 1 << 40, None) == B.EMM_ERR_UNSUPPORTED
    assert lib.emm_decode_attn_fp8(b, OK, c, OK, None, OK, 1 << 40, None) == B.EMM_ERR_INVALID_ARG      # more than one new token
    assert lib.emm_attn_fp8_workspace_size(b, None) == B.EMM_ERR_NULL
    assert lib.emm_prefill_attn_fp8(b, OK, c, None, None, OK, 1 << 40, None) == B.EMM_ERR_NULL
    assert lib.emm_prefill_attn_fp8(_batch(arrays=False), OK, c, OK, None, OK, 1 << 40, None) == B.EMM_ERR_NULL
    assert lib.emm_prefill_attn_fp8(b, OK, c, OK, OK + 2, OK, 1 << 40, None) == B.EMM_ERR_INVALID_ARG
    assert lib.emm_prefill_attn_fp8(_batch(num_pages=0), OK, c, OK, None, OK, 1 << 40, None) == B.EMM_ERR_INVALID_ARG
    big = _batch(num_pages=4096, max_pages_per_req=2048)
    need = B.emm_attn_fp8_workspace_size(big)
    if need:
        assert lib.emm_prefill_attn_fp8(big, OK, c, OK, None, None, 0, None) == B.EMM_ERR_NULL
        assert lib.emm_prefill_attn_fp8(big, OK, c, OK, None, OK, need - 1, None) == B.EMM_ERR_WORKSPACE


LARGE = [dict(total_new_tokens=2 ** 25 + 1), dict(num_q_heads=4098), dict(total_new_tokens=2 ** 24, num_q_heads=66), dict(max_pages_per_req=2 ** 27)]


@pytest.mark.parametrize("over", LARGE)
def test_batches_beyond_the_limits_are_refused(over):
    lib, b = B.load(), _batch(**over)
    r, c, n = ctypes.byref(_rope()), ctypes.byref(_cache()), ctypes.c_size_t()
    assert lib.emm_rope(b, r, OK, None, 0, 1 << 45, None, None) == B.EMM_ERR_UNSUPPORTED
    assert lib.emm_kv_scatter_fp8(b, OK, OK, 0, c, None) == B.EMM_ERR_UNSUPPORTED
    assert lib.emm_rope_kv_scatter_fp8(b, r, OK, OK, OK, 0, 1 << 45, c, None) == B.EMM_ERR_UNSUPPORTED
    assert lib.emm_kv_gather_fp8(b, c, OK, OK, None) == B.EMM_ERR_UNSUPPORTED
    assert lib.emm_attn_fp8_workspace_size(b, ctypes.byref(n)) == B.EMM_ERR_UNSUPPORTED


def test_attention_limits():
    lib, n = B.load(), ctypes.c_size_t()
    at = dict(num_reqs=2 ** 19, total_new_tokens=2 ** 19, max_new_len=1)
    assert lib.emm_attn_fp8_workspace_size(_batch(**at), ctypes.byref(n)) == B.EMM_OK            # 2^20 pairs
    at["num_reqs"] += 1
    assert lib.emm_attn_fp8_workspace_size(_batch(**at), ctypes.byref(n)) == B.EMM_ERR_UNSUPPORTED
    assert lib.emm_cross_attn_fp8(_batch(**at), OK, ctypes.byref(_cache()), OK, None, OK, 1 << 40, None) == B.EMM_ERR_UNSUPPORTED


def test_empty_batches_are_no_ops():
    lib, c, r = B.load(), ctypes.byref(_cache()), ctypes.byref(_rope())
    for b in (_batch(arrays=False, num_reqs=0, total_new_tokens=0, max_new_len=0), _batch(arrays=False, total_new_tokens=0, max_new_len=0)):
        assert lib.emm_rope(b, r, None, None, 0, None, None, None) == B.EMM_OK
        assert lib.emm_kv_scatter_fp8(b, None, None, 0, None, None) == B.EMM_OK
        assert lib.emm_rope_kv_scatter_fp8(b, r, None, None, None, 0, None, None, None) == B.EMM_OK
        assert lib.emm_kv_gather_fp8(b, None, None, None, None) == B.EMM_OK
        for name in ("emm_prefill_attn_fp8", "emm_cross_attn_fp8", "emm_decode_attn_fp8"):
            assert getattr(lib, name)(b, None, None, None, None, None, 0, None) == B.EMM_OK


def test_frequencies():
    n, base, scale, length = 128, 1e6, 4.0, 32768
    i = np.arange(n // 2)
    plain = base ** (-2.0 * i / n)

    def near(kind, want, factor=1.0, **kw):
        inv, f = B.emm_rope_inv_freq_host(n, base, kind, scale, length, **kw)
        assert np.allclose(inv, want, rtol=1e-13, atol=0) and f == pytest.approx(factor, rel=1e-7)
    near("plain", plain)
    near("linear", plain / scale)
    ntk = (base * scale ** (n / (n - 2))) ** (-2.0 * i / n)
    near("ntk", ntk)
    assert ntk[0] == 1 and np.isclose(ntk[-1], plain[-1] / scale)            # highest as it was, lowest divided by scale
    turns = length * plain / (2 * np.pi)                                     # in the trained length
    bands = np.array([f if t > 32 else f / scale if t < 1 else f * ((t - 1) / 31) + f / scale * (1 - (t - 1) / 31) for f, t in zip(plain, turns)])
    near("bands", bands, slow=1.0, fast=32.0)
    inv, f = B.emm_rope_inv_freq_host(n, base, "yarn", scale, length, slow=1.0, fast=32.0)
    assert f == pytest.approx(0.1 * math.log(scale) + 1, rel=1e-7)
    first, last = np.argmax(turns < 32), np.argmax(turns < 1)                # i where the turns fall below fast, below slow
    assert np.allclose(inv[: first], plain[: first]) and np.allclose(inv[last + 1:], plain[last + 1:] / scale)
    kept = (inv - plain / scale) / (plain - plain / scale)
    inner = kept[first:last]
    assert (np.diff(inner) < 0).all() and np.allclose(np.diff(inner), np.diff(inner)[0])       # a linear ramp over i


@pytest.mark.parametrize("kw", [dict(rotary_dim=8), dict(rotary_dim=40), dict(rotary_dim=144), dict(base=1.0), dict(base=math.inf), dict(scale=0.5), dict(kind=7),
                                dict(kind="yarn", original_len=0), dict(kind="bands", original_len=100, slow=2.0, fast=2.0),
                                dict(kind="yarn", original_len=100, slow=0.0)])
def test_frequencies_refusals(kw):
    with pytest.raises(B.EmmError) as e:
        B.emm_rope_inv_freq_host(**dict(dict(rotary_dim=64, base=1e4, scale=2.0), **kw))
    assert e.value.status == B.EMM_ERR_INVALID_ARG
    assert B.load().emm_rope_inv_freq_host(None, None, None) == B.EMM_ERR_NULL


def test_binding_checks_tensors():
    import torch
    inv = torch.zeros(64, dtype=torch.float64)
    for bad in (dict(inv_freq=inv.float()), dict(inv_freq=inv[:10]), dict(positions=torch.zeros(3, 5, dtype=torch.int64), sections=[16, 24, 24]),
                dict(positions=torch.zeros(3, 5, dtype=torch.int32)), dict(positions=torch.zeros(5, 3, dtype=torch.int32).t(), sections=[16, 24, 24])):
        with pytest.raises(ValueError):
            B.make_rope(**dict(dict(inv_freq=inv, rotary_dim=128), **bad))
    rope = B.make_rope(inv_freq=inv, rotary_dim=128, positions=torch.zeros(3, 19, dtype=torch.int32), sections=[16, 24, 24])
    for call in (lambda: B.emm_rope(_batch(), rope, None, None, None, None), lambda: B.emm_rope_kv_scatter_fp8(_batch(), rope, None, None, None, None, None)):
        with pytest.raises(ValueError):                      # 19 positions, 20 tokens
            call()
    codes = torch.zeros(4, 2, 16, 128, dtype=torch.uint8)
    with pytest.raises(ValueError):
        B.make_fp8_cache(codes.float(), codes, codes, codes)
    with pytest.raises(ValueError):
        B.make_fp8_cache(codes.transpose(1, 2), codes, codes, codes)
