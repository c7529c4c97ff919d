"""Rotary positions on the GPU where rows belong to no request, against oracle/fp8_model.py with the tolerances of
test_gpu_fp8_cache.py."""
import numpy as np
import pytest
import torch

from oracle import fp8_model as F
from paper_2507_10069_amd import binding as B
from test_gpu_fp8_cache import DEV, _check_rotated, _dev, _f64

pytestmark = pytest.mark.gpu


def test_given_positions_turn_all_rows_without_requests():
    print("case no requests", flush=True)
    rng, T, H = np.random.default_rng(1), 37, 5
    batch = B.make_batch(num_reqs=0, num_q_heads=H, num_kv_heads=H, head_dim=64, page_size=16, num_pages=1, max_pages_per_req=1, total_new_tokens=T,
                         max_new_len=0, dtype="f32", softmax_scale=1.0)
    inv, _ = B.emm_rope_inv_freq_host(64, 1e4)
    at = rng.integers(0, 5000, T).astype(np.int32)
    rope = B.make_rope(_dev(inv), rotary_dim=64, positions=_dev(at[None]))
    q, out = _dev(rng.standard_normal((T, H, 64)).astype(np.float32)), torch.full((T, H, 64), 9.0, device=DEV)
    B.emm_rope(batch, rope, q, None, out, None)
    want = F.rotate(_f64(q), np.repeat(at[:, None], 32, 1), inv, 64, "half")
    _check_rotated(_f64(out), _f64(q), want, None, 64, "half", 1.0, "f32")
