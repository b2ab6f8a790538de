"""Keys that are not finite in the prompt's attention calls: a row that sees one is NaN, and so is its log-sum-exp, whatever the launch cuts its keys
into; the rows of other KV heads and sequences keep their bits."""
import numpy as np
import pytest
import torch

from oracle import block_attention as ob
from paper_2409_15355_b200 import binding as B
from paper_2409_15355_b200 import workloads as W
from tests.test_gpu_parity import ctx_for, dev
from tests.test_gpu_tile_edges import _requests

pytestmark = pytest.mark.gpu

CASES = [_requests("cut streams", 40, 91, (4, 100, 300), (60, 200)), _requests("clusters", 5, 114, (3, 1, 500), (1, 70), heads=(8, 1, 64)),
         _requests("one query tile", 4, 142, (9, 40, 300), (1, 32), heads=(32, 8, 128)), _requests("one long prompt", 1, 120, (20, 900, 1000), (700, 700)),
         _requests("a short question to a long prompt", 1, 121, (20, 900, 1000), (64, 64), heads=(32, 8, 128))]


@pytest.mark.parametrize("w", CASES, ids=lambda w: w.name)
@pytest.mark.parametrize("fused", [False, True], ids=["reencode_then_attend", "fused"])
@pytest.mark.parametrize("value", [float("nan"), float("inf")])
def test_a_cached_key_that_is_not_finite(w, fused, value):
    c = ctx_for(w)
    seg, buf = c.segment(w.block_lens, w.seq_nblocks, B.BA_MODE_BLOCK)
    t = ob.segment_tables(w.block_lens, w.seq_nblocks, B.BA_MODE_BLOCK)
    x = W.warm_inputs(w, 0)
    Tc, Tf = t["n_cached_tokens"], t["n_final_tokens"]
    q, kf, vf, k, v = (dev(x[n]) for n in ("q_f", "k_f", "v_f", "k_cache", "v_cache"))
    q[:, :, :2] = 1.0                                            # (products with the planted pair: infinite, above zero for some rotation or NaN)
    outs = []
    for planted in (False, True):
        if planted:
            row, head = int(t["cache_cu"][1]) // 2, w.n_kv_heads - 1            # in the first block of the first sequence
            k[row, head, 0] = value
        o, lse = torch.full((Tf, w.n_q_heads, w.head_dim), 7.0, device="cuda"), torch.full((Tf, w.n_q_heads), 7.0, device="cuda")
        if fused:
            B.ba_final_attend_fused(c.ctx, q, kf, vf, Tf, k, v, Tc, None, Tc, o, lse, seg, B.BA_MODE_BLOCK, B.BA_OUT_F32)
        else:
            k_re = k.clone()
            if planted:
                k_re[row, head, 1] = value                       # (q . k is infinite or NaN: no finite term makes up for it)
            B.ba_final_attend(c.ctx, q, kf, vf, Tf, k_re, v, Tc, None, 0, o, lse, seg, B.BA_MODE_BLOCK, B.BA_OUT_F32)
        assert c.device_status() == B.BA_OK
        outs.append((o, lse))
    G, rows = w.n_q_heads // w.n_kv_heads, w.final_lens()[0]
    seen = torch.zeros(Tf, w.n_q_heads, dtype=torch.bool, device="cuda")
    seen[:rows, head * G:(head + 1) * G] = True
    (o0, l0), (o1, l1) = outs
    assert torch.equal(o1[~seen], o0[~seen]) and torch.equal(l1[~seen], l0[~seen])
    assert torch.isfinite(l0).all()
    if value != value or not fused:                              # (an infinite key turned by the fused call scores -infinity for some rows)
        assert torch.isnan(o1[seen]).all() and torch.isnan(l1[seen]).all()
    else:
        assert (torch.isnan(l1[seen]) == torch.isnan(o1[seen]).all(-1)).all() and (torch.isnan(l1[seen]) | torch.isfinite(l1[seen])).all()
    c.close()


@pytest.mark.parametrize("w", [_requests("cut final blocks", 3, 97, (7, 64, 300), (1, 200)), _requests("one", 1, 96, (9, 150, 400), (65, 65)),
                               _requests("many", 20, 98, (3, 30, 200), (30, 90))], ids=lambda w: w.name)
def test_a_prompts_key_that_is_nan(w):
    c = ctx_for(w)
    seg, buf = c.segment(w.block_lens, w.seq_nblocks, B.BA_MODE_BLOCK)
    gen = torch.Generator().manual_seed(5)
    q, k, v = (torch.randn(w.n_tokens, h, w.head_dim, generator=gen).to(torch.bfloat16).cuda() for h in (w.n_q_heads, w.n_kv_heads, w.n_kv_heads))
    first, last = w.block_lens[0], sum(w.block_lens[:w.seq_nblocks[0]])
    row, final = first // 2, last - w.block_lens[w.seq_nblocks[0] - 1]
    outs = []
    for planted in (False, True):
        if planted:
            k[row, 0, 3] = float("nan")
        o, lse = torch.zeros(w.n_tokens, w.n_q_heads, w.head_dim, device="cuda"), torch.zeros(w.n_tokens, w.n_q_heads, device="cuda")
        B.ba_block_prefill(c.ctx, q, k, v, o, lse, seg, B.BA_MODE_BLOCK, B.BA_OUT_F32)
        assert c.device_status() == B.BA_OK
        outs.append((o, lse))
    seen = torch.zeros(w.n_tokens, w.n_q_heads, dtype=torch.bool, device="cuda")
    heads = slice(0, w.n_q_heads // w.n_kv_heads)
    seen[row:first, heads] = True                                # the rest of its block, and the final block of its sequence
    seen[final:last, heads] = True
    (o0, l0), (o1, l1) = outs
    assert torch.isnan(o1[seen]).all() and torch.isnan(l1[seen]).all()
    assert (torch.isfinite(o1[~seen]).all(-1) & torch.isfinite(l1[~seen])).all()
    assert (o1[~seen] - o0[~seen]).abs().max() <= 1e-2 and (l1[~seen] - l0[~seen]).abs().max() <= 2e-3
    c.close()
