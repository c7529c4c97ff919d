"""Rotary positions on the GPU where rows belong to no request, against oracle/fp8_model.py with the tolerances of
test_gpu_fp8_cache.py."""
import numpy as np
import pytest
import torch

from oracle import fp8_model as F
from paper_2507_10069_amd import binding as B
from test_gpu_fp8_cache import DEV, Batch, _check_rotated, _dev, _f64

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


@pytest.mark.parametrize("axes", [0, 1, 3])
@pytest.mark.parametrize("requests", [True, False])
def test_rotation_and_write_has_the_bits_of_the_two_calls_in_rows_of_no_request(axes, requests):
    """A padded batch, and one that is nothing but padding: given positions turn those rows of q, places in requests leave them."""
    print("case padded rotation and write", axes, requests, flush=True)
    b = Batch([3, 100, 9], [4, 0, 30], heads=12, kv_heads=2, seed=axes, extra_rows=21)
    if not requests:
        b.batch.num_reqs = b.batch.max_new_len = 0
    inv, _ = B.emm_rope_inv_freq_host(128, 1e6)
    pos = _dev(b.rng.integers(0, 9000, (axes, b.rows)).astype(np.int32)) if axes else None
    rope = B.make_rope(_dev(inv), rotary_dim=128, positions=pos, sections=[16, 24, 24] if axes == 3 else None)
    q, k, v = (_dev(b.rng.standard_normal((b.rows, h, 128)).astype(np.float32), torch.bfloat16) for h in (12, 2, 2))
    got, want, k_two = torch.full_like(q, 5.0), torch.full_like(q, 5.0), torch.full_like(k, 5.0)
    B.emm_rope_kv_scatter_fp8(b.batch, rope, q, k, v, got, b.to_device())
    fused = {n: t.clone() for n, t in b.pools.items()}
    cache = b.to_device()
    B.emm_rope(b.batch, rope, q, k, want, k_two)
    B.emm_kv_scatter_fp8(b.batch, k_two, v, cache)
    assert torch.equal(got, want)
    for n, t in b.pools.items():
        assert torch.equal(fused[n], t), n
    turned = b.rows if axes else b.T if requests else 0
    assert (got[turned:] == 5).all() and not (got[:turned] == 5).all(dim=-1).any()


def test_rows_of_no_request_stay_and_all_others_are_turned():
    print("case rows of no request", flush=True)
    b = Batch([3, 9, 0], [4, 2, 11], heads=4, kv_heads=2, seed=5, extra_rows=5)
    inv, _ = B.emm_rope_inv_freq_host(128, 1e4)
    x = {n: _dev(b.rng.standard_normal((b.rows, h, 128)).astype(np.float32), torch.bfloat16) for n, h in (("q", 4), ("k", 2))}
    out = {n: torch.full_like(t, 5.0) for n, t in x.items()}
    B.emm_rope(b.batch, B.make_rope(_dev(inv), rotary_dim=128), x["q"], x["k"], out["q"], out["k"])
    at = np.concatenate([np.arange(p, p + n) for p, n in zip(b.prefix, b.new)])
    for n, t in out.items():
        have = _f64(x[n])[: b.T]
        _check_rotated(_f64(t)[: b.T], have, F.rotate(have, np.repeat(at[:, None], 64, 1), inv, 128, "half"), None, 128, "half", 1.0, "bf16")
        assert (t[b.T:] == 5).all()


def test_reading_back_skips_what_has_no_slot_in_both_outputs():
    """Entries of the table outside the pool, slots behind the table, rows of no request: of K and of V every row is what its slot holds or what it was."""
    print("case no slot", flush=True)
    b = Batch([10, 0, 60, 4], [8, 3, 8, 6], kv_heads=2, heads=2, seed=8, extra_rows=4)
    b.table[1, 0], b.table[3, 0] = b.num_pages + 7, -9
    b.prefix[2] = b.table.shape[1] * 16 - 3                  # its last five tokens lie behind the table
    b.table[2, -1] = b.table[2, 3]
    b.dev["table"].copy_(_dev(b.table)), b.dev["prefix"].copy_(_dev(b.prefix))
    for n in "kv":
        b.codes[n] = np.where((b.codes[n] & 0x7F) == 0x7F, 0x30 + (n == "v"), b.codes[n]).astype(np.uint8)
        b.scales[n] = b.rng.integers(100, 150, b.scales[n].shape).astype(np.uint8)
    out = {n: torch.full((b.rows, 2, 128), 3.0, dtype=torch.bfloat16, device=DEV) for n in "kv"}
    B.emm_kv_gather_fp8(b.batch, b.to_device(), out["k"], out["v"])
    for n, t in out.items():
        want = np.full((b.rows, 2, 128), 3.0)
        for r, held in ((0, 8), (2, 3)):
            pages, places = b.slots(r, int(b.prefix[r]), held)
            want[b.cu[r]:b.cu[r] + held] = F.values_of(b.codes[n][pages, :, places], b.scales[n][pages, :, places])
        assert np.array_equal(_f64(t), want), n
