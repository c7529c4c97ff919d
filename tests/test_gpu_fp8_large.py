"""The calls of the 8-bit cache and of rotary positions at the ends of what they take: contexts as long as a row of the page
table may be, batches whose rows, slots or requests make the kernels go their ways for large calls.  References and
tolerances are those of test_gpu_fp8_cache.py unless a test says otherwise."""
import math

import numpy as np
import pytest
import torch

from paper_2507_10069_amd import binding as B
from test_gpu_fp8_cache import DEV

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("heads", [20, 7], ids=["chunk kernel", "few rows"])
def test_the_longest_context(heads):
    """2^30 slots, the most that a row of the page table may hold, in two pages: every key counts, the last ones too.  Queries of
    zeros make all weights 1 and every sum exact in 32 bits: V is 1, and 2 in the last 1/128, so that out is 129 / 128 (exact in bf16)
    and lse 30 ln 2 (2^-22 of itself: one logarithm, one product)."""
    print("case longest context", heads, flush=True)
    slots, page = 1 << 30, 256
    table = torch.zeros((1, slots // page), dtype=torch.int32, device=DEV)
    table[0, slots // page // 128 * 127:] = 1
    lens = [torch.tensor(v, dtype=torch.int32, device=DEV) for v in ([slots - 1], [1], [0, 1])]
    batch = B.make_batch(num_reqs=1, num_q_heads=heads, num_kv_heads=1, head_dim=128, page_size=page, num_pages=2, max_pages_per_req=slots // page,
                         total_new_tokens=1, max_new_len=1, dtype="bf16", softmax_scale=1.0, page_table=table, prefix_lens=lens[0], new_lens=lens[1],
                         cu_new_lens=lens[2])
    k = torch.full((2, 1, page, 128), 0x31, dtype=torch.uint8, device=DEV)
    v = torch.full((2, 1, page, 128), 0x38, dtype=torch.uint8, device=DEV)                 # the code of 1
    k_scale = torch.full((2, 1, page), 127, dtype=torch.uint8, device=DEV)
    v_scale = torch.tensor([127, 128], dtype=torch.uint8, device=DEV)[:, None, None].expand(2, 1, page).contiguous()
    q, out = torch.zeros((1, heads, 128), dtype=torch.bfloat16, device=DEV), torch.zeros((1, heads, 128), dtype=torch.bfloat16, device=DEV)
    lse = torch.zeros((1, heads), device=DEV)
    workspace = torch.empty(B.emm_attn_fp8_workspace_size(batch), dtype=torch.uint8, device=DEV)
    B.emm_decode_attn_fp8(batch, q, B.make_fp8_cache(k, v, k_scale, v_scale), out, lse, workspace)
    torch.cuda.synchronize()
    assert (out == 129 / 128).all(), out.float().unique()
    assert ((lse.double() - 30 * math.log(2)).abs() <= 2.0 ** -22 * 30 * math.log(2)).all(), lse.unique()
