"""The token operators over tables, page numbers and values that a caller got wrong or meant: what is reported, what is left alone, what is
passed on.  Tolerances as in test_gpu_token_ops.py."""
import numpy as np
import pytest
import torch

from oracle import token_ops as tk
from paper_2409_15355_b200 import binding as B
from paper_2409_15355_b200 import runtime as R
from tests.test_gpu_token_ops import HALF_STEP, Batch, bf16, check_attention, context, f64, ints, make_context

pytestmark = pytest.mark.gpu


# ------------------------------------------------------------------ lists of pages that begin before their table
def inside(values, before):
    """An int32 table on the device that lies in the middle of a larger one: reads a little in front of it stay in the allocation."""
    whole = ints(list(before) + list(values) + [0] * 8)
    return whole[len(before):len(before) + len(values)], whole


def test_append_into_a_list_that_begins_before_the_table():
    """No page is taken from in front of page_idx, where this test put good ones."""
    shape = (4, 2, 64)
    c = context(shape)
    q, k, v = bf16(3, 4, 64, seed=3), bf16(3, 2, 64, seed=1), bf16(3, 2, 64, seed=2)
    page_idx, keep = inside([1, 2, 3], [7, 6, 5, 4])
    pools = [torch.full((8 * 16, 2, 64), 9.0, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    q_out, page_cu, start = torch.zeros_like(q), ints([-3, 1, 2, 3]), ints([0, 0, 0])
    B.ba_append_paged(c.ctx, q, k, v, 3, None, None, None, 0.0, None, start, 3, q_out, *pools, B.make_page_table(16, 8, page_cu, page_idx))
    assert c.device_status() == B.BA_ERR_INVALID_ARG
    assert torch.equal(q_out, q)
    for p, x in zip(pools, (k, v)):
        assert torch.equal(p[[32, 48]], x[1:])                  # (lists 1 and 2: pages 2 and 3)
        p[[32, 48]] = 9.0
        assert (p == 9).all()
    c.close()


@pytest.mark.parametrize("which", ["own", "prefix"])
def test_attention_over_a_list_that_begins_before_the_table(which):
    """Reported, nothing written; the same tables with the list in its place are taken."""
    b = Batch((4, 2, 64), [100, 50], [0, 1, 3], [1, 1, 2], [10, 20, 30], 16, False, seed=2)
    c = make_context((4, 2, 64), b)
    o, lse = torch.full((4, 4, 64), 5.0, device="cuda"), torch.full((4, 4), 6.0, device="cuda")
    own, prefix = b.table, b.prefix_table
    cu, idx = b.keep if which == "own" else b.keep2
    n_pages = b.n_pages if which == "own" else b.kv_prefix[0].shape[0] // 16
    moved, keep = inside(idx.tolist(), [0] * 4)
    bad = cu.clone()
    bad[0] = -3
    table = B.make_page_table(16, n_pages, bad, moved)
    b.table, b.prefix_table = (table, prefix) if which == "own" else (own, table)
    b.call(c, o, lse, B.BA_OUT_F32)
    assert c.device_status() == B.BA_ERR_INVALID_ARG
    assert (o == 5).all() and (lse == 6).all()
    b.table, b.prefix_table = own, prefix
    b.call(c, o, lse, B.BA_OUT_F32)
    assert c.device_status() == B.BA_OK
    check_attention(b, o, lse, B.BA_OUT_F32, 0.125)
    c.close()
