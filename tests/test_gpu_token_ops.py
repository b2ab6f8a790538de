"""Norms with rotation, their gradients, paged append and attention over shared prefixes against the fp64 oracle.

Tolerances, elementwise.  A bf16 store is off by at most 2^-8 of the value.  Rotated values: fp32 arithmetic and an angle good to 1e-7 leave
4e-6 of the pair's length.  Gradients of x: two products and two sums of up to 128 terms, 2e-5 of |h| r + |x| r^3 mean|h x|.  Gradients of w:
chains of at most a few hundred fp32 additions, 2e-5 of the terms' absolute sum.  Attention: P is rounded to bf16, each p off by at most
2^-8 of it, so o by 2^-8 of sum p |v|, and scores of 128 fp32 products leave 1e-4 of it; lse is off by the scores' 1e-4 at most.
"""
import numpy as np
import pytest
import torch

from oracle import token_ops as tk
from paper_2409_15355_b200 import binding as B
from paper_2409_15355_b200 import runtime as R

pytestmark = pytest.mark.gpu

HALF_STEP = 2.0 ** -8
SHAPES = [(4, 2, 64), (6, 2, 64), (8, 1, 128), (32, 8, 128), (5, 5, 128), (3, 1, 64)]


def bf16(*shape, seed=0, scale=1.0):
    gen = torch.Generator().manual_seed(seed)
    return (torch.randn(*shape, generator=gen) * scale).to(torch.bfloat16).cuda()


def f64(t):
    return t.detach().double().cpu().numpy()


def ints(x):
    return torch.tensor(list(x), dtype=torch.int32, device="cuda")


def context(shape, layout=0, theta=5e5, room=0):
    return R.Context(*shape, theta, rope_layout=layout, max_blocks=64, max_q_rows=64, workspace_bytes=room)


def pair_length(y, layout):
    a, b = tk._pairs(y, layout)
    n = np.hypot(a, b)
    return tk._unpair(n, n, layout)


def check_rotated(got, want, layout, rounded=True):
    got = f64(got)
    assert np.isfinite(got).all()
    err = np.abs(got - want) - (HALF_STEP * np.abs(want) if rounded else 0) - 4e-6 * pair_length(want, layout) - 1e-30
    assert err.max() <= 0, err.max()


POSITIONS = {"short": lambda n: range(n), "far": lambda n: range(99000, 99000 + n), "any": lambda n: np.random.default_rng(n).integers(-5000, 2 ** 20, n)}


@pytest.mark.parametrize("shape", SHAPES, ids=str)
@pytest.mark.parametrize("layout", [B.BA_ROPE_ADJACENT, B.BA_ROPE_HALF])
@pytest.mark.parametrize("rows,where,normed", [(1, "far", True), (3, "any", False), (50, "short", True), (333, "any", True), (2500, "far", True)])
def test_norm_rope(shape, layout, rows, where, normed):
    hq, hkv, d = shape
    c = context(shape, layout)
    qkv = bf16(rows, hq + 2 * hkv, d, seed=rows)
    q, k = qkv[:, :hq], qkv[:, hq:hq + hkv]
    pos = list(POSITIONS[where](rows))
    w_q, w_k = (bf16(d, seed=8), bf16(d, seed=9)) if normed else (None, None)
    out = [torch.full((rows + 1, h, d), 7.0, dtype=torch.bfloat16, device="cuda") for h in (hq, hkv)]
    B.ba_qk_norm_rope(c.ctx, q, k, rows, ints(pos), w_q, w_k, 1e-6, *out)
    want = [tk.norm_rope(f64(x), pos, None if w is None else f64(w), 1e-6, 5e5, layout) for x, w in ((q, w_q), (k, w_k))]
    for got, ref in zip(out, want):
        check_rotated(got[:rows], ref, layout)
        assert (got[rows] == 7).all()
    # packed inputs, one side at a time and in place: the same bits
    for side, x, w in ((0, q, w_q), (1, k, w_k)):
        y = x.contiguous()
        args = [y if side == 0 else None, y if side == 1 else None]
        B.ba_qk_norm_rope(c.ctx, *args, rows, ints(pos), w_q, w_k, 1e-6, *args)
        assert torch.equal(y, out[side][:rows])
    assert c.device_status() == B.BA_OK
    c.close()


def test_norm_rope_without_positions_or_weights_copies():
    c = context((6, 2, 64))
    q, k = bf16(9, 6, 64, seed=1), bf16(9, 2, 64, seed=2)
    out = torch.empty_like(q), torch.empty_like(k)
    B.ba_qk_norm_rope(c.ctx, q, k, 9, None, None, None, 0.0, *out)
    assert torch.equal(out[0], q) and torch.equal(out[1], k)
    B.ba_qk_norm_rope(c.ctx, q, k, 0, None, None, None, 0.0, *out)
    B.ba_qk_norm_rope(c.ctx, None, k, 9, ints([0] * 9), None, None, 0.0, None, out[1])
    assert torch.equal(out[1], k)
    c.close()


def test_norm_of_zeros_and_of_large_values():
    c = context((3, 1, 64))
    q = torch.zeros(4, 3, 64, dtype=torch.bfloat16, device="cuda")
    q[1] = 1e17
    q[2] = 1e-20
    k = torch.zeros(4, 1, 64, dtype=torch.bfloat16, device="cuda")
    w = torch.ones(64, dtype=torch.bfloat16, device="cuda")
    out = torch.empty_like(q), torch.empty_like(k)
    B.ba_qk_norm_rope(c.ctx, q, k, 4, None, w, w, 1e-6, *out)
    assert (out[0][0] == 0).all() and (out[1] == 0).all() and torch.isfinite(out[0]).all()
    assert (out[0][1] == 1).all()
    # gradients with eps 0: the lanes of a head that is not there (three heads, four to a step) add nothing
    dq, dw = torch.empty(4, 3, 64, device="cuda"), torch.empty(64, device="cuda")
    x, dy = bf16(4, 3, 64, seed=3), torch.randn(4, 3, 64, device="cuda")
    B.ba_qk_norm_rope_bwd(c.ctx, x, None, 4, None, w, None, 0.0, dy, None, dq, None, dw, None, B.BA_OUT_F32)
    assert torch.isfinite(dq).all() and torch.isfinite(dw).all()
    c.close()


@pytest.mark.parametrize("shape", SHAPES, ids=str)
@pytest.mark.parametrize("layout", [B.BA_ROPE_ADJACENT, B.BA_ROPE_HALF])
@pytest.mark.parametrize("rows,out,normed", [(1, "f32", True), (7, "bf16", True), (130, "f32", False), (1111, "f32", True), (1300, "bf16", True)])
def test_norm_rope_gradients(shape, layout, rows, out, normed):
    hq, hkv, d = shape
    c = context(shape, layout)
    kind, code = (torch.float32, B.BA_OUT_F32) if out == "f32" else (torch.bfloat16, B.BA_OUT_BF16)
    qkv = bf16(rows, hq + 2 * hkv, d, seed=rows, scale=1.7)
    x = qkv[:, :hq], qkv[:, hq:hq + hkv]
    pos = list(POSITIONS["any"](rows))
    w = (bf16(d, seed=18), bf16(d, seed=19)) if normed else (None, None)
    dy = [bf16(rows, h, d, seed=h).to(kind) for h in (hq, hkv)]
    grad = torch.full((rows, hq + 2 * hkv, d), 5.0, dtype=kind, device="cuda")
    dx = grad[:, :hq], grad[:, hq:hq + hkv]
    dw = [torch.full((d,), float("nan"), device="cuda") if normed else None for _ in range(2)]
    args = (*x, rows, ints(pos), *w, 1e-5, *dy, *dx, *dw, code)
    B.ba_qk_norm_rope_bwd(c.ctx, *args)
    assert (grad[:, hq + hkv:] == 5).all()
    for i in range(2):
        xx, ww, g = f64(x[i]), f64(w[i]) if normed else None, f64(dy[i])
        want, want_w = tk.norm_rope_backward(xx, pos, ww, 1e-5, 5e5, g, layout)
        turned = tk.rotate(g, [-p for p in pos], 5e5, layout)
        if normed:
            n = np.sqrt((xx * xx).mean(-1, keepdims=True) + 1e-5)
            h = pair_length(turned, layout) * np.abs(ww)
            size = h / n + np.abs(xx) * (h * np.abs(xx)).mean(-1, keepdims=True) / n ** 3
            terms = (pair_length(turned, layout) * np.abs(xx) / n).sum((0, 1))
            assert (np.abs(f64(dw[i]) - want_w) <= 2e-5 * terms).all()
        else:
            size = pair_length(turned, layout)
        err = np.abs(f64(dx[i]) - want) - 2e-5 * size - (HALF_STEP * np.abs(want) if out == "bf16" else 0)
        assert err.max() <= 0, err.max()
    # the same bits again, and in the place of the gradients that come in
    first = [t.clone() for t in dx], [t.clone() if normed else None for t in dw]
    inplace = [t.clone() for t in dy]
    B.ba_qk_norm_rope_bwd(c.ctx, *x, rows, ints(pos), *w, 1e-5, *inplace, *inplace, *dw, code)
    for a, b in zip(first[0], inplace):
        assert torch.equal(a, b)
    for a, b in zip(first[1], dw):
        assert a is None or torch.equal(a, b)
    assert c.device_status() == B.BA_OK
    c.close()


def test_norm_gradients_of_no_rows_are_zero():
    c = context((4, 2, 64))
    w = bf16(64, seed=1)
    t = torch.empty(1, 4, 64, device="cuda"), torch.empty(1, 2, 64, device="cuda")
    q = bf16(1, 4, 64), bf16(1, 2, 64)
    dw = torch.ones(64, device="cuda"), torch.ones(64, device="cuda")
    B.ba_qk_norm_rope_bwd(c.ctx, *q, 0, None, w, w, 1e-6, *t, *t, *dw, B.BA_OUT_F32)
    assert (dw[0] == 0).all() and (dw[1] == 0).all()
    c.close()


# ------------------------------------------------------------------ append
def page_lists(lens, page_rows, spare=2, seed=0):
    counts = [-(-n // page_rows) for n in lens]
    cu = np.concatenate([[0], np.cumsum(counts)]).astype(int)
    n_pages = int(cu[-1]) + spare
    idx = np.random.default_rng(seed).permutation(n_pages)[:cu[-1]]
    return cu, idx, n_pages, B.make_page_table(page_rows, n_pages, *(keep := (ints(cu), ints(idx if len(idx) else [0])))), keep


@pytest.mark.parametrize("shape", SHAPES[:5], ids=str)
@pytest.mark.parametrize("layout", [B.BA_ROPE_ADJACENT, B.BA_ROPE_HALF])
@pytest.mark.parametrize("lens,used,page_rows,normed", [([1], [0], 16, True), ([1, 1, 1], [15, 16, 700], 16, True), ([0, 5, 0, 33], [3, 0, 9, 31], 32, False),
                                                        ([130, 1, 257], [0, 128, 1], 128, True), ([17, 300], [1000, 3], 4096, True)], ids=str)
def test_append(shape, layout, lens, used, page_rows, normed):
    hq, hkv, d = shape
    c = context(shape, layout)
    rows, pad = sum(lens), 3
    cu, idx, n_pages, table, keep = page_lists([a + b for a, b in zip(lens, used)], page_rows)
    qkv = bf16(rows + pad, hq + 2 * hkv, d, seed=5)
    q, k, v = qkv[:, :hq], qkv[:, hq:hq + hkv], qkv[:, hq + hkv:]
    pos = [u + t + 40 for n, u in zip(lens, used) for t in range(n)] + [0] * pad
    w = (bf16(d, seed=1), bf16(d, seed=2)) if normed else (None, None)
    pools = [bf16(n_pages * page_rows, hkv, d, seed=s) for s in (6, 7)]
    before = [p.clone() for p in pools]
    q_out = torch.full((rows + pad, hq, d), 3.0, dtype=torch.bfloat16, device="cuda")
    seq_cu = ints(np.concatenate([[0], np.cumsum(lens)]))
    B.ba_append_paged(c.ctx, q, k, v, rows + pad, ints(pos), *w, 1e-6, seq_cu, ints(used), len(lens), q_out, *pools, table)
    assert c.device_status() == B.BA_OK
    at = [r for s, (n, u) in enumerate(zip(lens, used)) for r in tk.page_rows_of(cu, idx, page_rows, s, n + u)[u:]]
    ww = [None if x is None else f64(x) for x in w]
    check_rotated(pools[0][at], tk.norm_rope(f64(k[:rows]), pos[:rows], ww[1], 1e-6, 5e5, layout), layout)
    assert torch.equal(pools[1][at], v[:rows])
    check_rotated(q_out[:rows], tk.norm_rope(f64(q[:rows]), pos[:rows], ww[0], 1e-6, 5e5, layout), layout)
    assert (q_out[rows:] == 3).all()                            # rows behind the last sequence
    rest = torch.ones(n_pages * page_rows, dtype=torch.bool)
    rest[at] = False
    for p, b in zip(pools, before):
        assert torch.equal(p[rest.cuda()], b[rest.cuda()])
    # without the queries, and (one row each) without the table: the same bits
    again = [b.clone() for b in before]
    B.ba_append_paged(c.ctx, None, k, v, rows, ints(pos), None, w[1], 1e-6, seq_cu, ints(used), len(lens), None, *again, table)
    if all(n == 1 for n in lens):
        B.ba_append_paged(c.ctx, None, k, v, rows, ints(pos), None, w[1], 1e-6, None, ints(used), len(lens), None, *again, table)
    assert torch.equal(again[0], pools[0]) and torch.equal(again[1], pools[1])
    assert c.device_status() == B.BA_OK
    c.close()


def test_append_skips_and_reports_places_without_a_page():
    shape = (4, 2, 64)
    c = context(shape)
    k, v, q = bf16(4, 2, 64, seed=1), bf16(4, 2, 64, seed=2), bf16(4, 4, 64, seed=3)
    for start, page_idx in (([16, 0, 0, 0], [0, 1, 2, 3]), ([-1, 0, 0, 0], [0, 1, 2, 3]), ([2 ** 31 - 1, 0, 0, 0], [0, 1, 2, 3]),
                            ([0, 0, 0, 0], [4, 1, 2, 3]), ([0, 0, 0, 0], [-1, 1, 2, 3])):
        pools = [torch.full((64, 2, 64), 9.0, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
        q_out = torch.zeros_like(q)
        cu, idx = ints([0, 1, 2, 3, 4]), ints(page_idx)
        B.ba_append_paged(c.ctx, q, k, v, 4, None, None, None, 0.0, None, ints(start), 4, q_out, *pools, B.make_page_table(16, 4, cu, idx))
        assert c.device_status() == B.BA_ERR_INVALID_ARG
        assert torch.equal(q_out, q)
        for p, x in zip(pools, (k, v)):
            assert torch.equal(p[[16, 32, 48]], x[1:])
            p[[16, 32, 48]] = 9.0
            assert (p == 9).all()
    c.close()


def test_passages_reencoded_into_pages_equal_reencode():
    """Cached blocks (positions from zero) brought into pages with the block's delta as every row's position: the bits of ba_reencode_k."""
    shape, lens, delta = (8, 2, 128), [70, 1, 129], [0, 70, 71]
    c = context(shape)
    k, v = bf16(200, 2, 128, seed=1), bf16(200, 2, 128, seed=2)
    want = torch.empty_like(k)
    cu = ints([0, 70, 71, 200])
    B.ba_reencode_k(c.ctx, k, None, 200, want, cu, ints(delta), 3, 200)
    pcu, idx, n_pages, table, keep = page_lists(lens, 16)
    pools = [torch.zeros(n_pages * 16, 2, 128, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    pos = [p for n, p in zip(lens, delta) for _ in range(n)]
    B.ba_append_paged(c.ctx, None, k, v, 200, ints(pos), None, None, 0.0, cu, ints([0] * 3), 3, None, *pools, table)
    at = [r for s, n in enumerate(lens) for r in tk.page_rows_of(pcu, idx, 16, s, n)]
    assert torch.equal(pools[1][at], v)
    # (cos and sin come from two ways of reducing the angle: the last bit of a rounding may fall the other way)
    a, b = pools[0][at].float(), want.float()
    assert (a == b).float().mean() > 0.995 and ((a - b).abs() <= 2 * HALF_STEP * b.abs() + 1e-5).all()
    c.close()


# ------------------------------------------------------------------ shared prefixes
class Batch:
    """A batch with its caches: NaN wherever the tables say that nothing is."""

    def __init__(self, shape, prefix, group_cu, q_lens, own, page_rows, packed, seed=0, pad_rows=0, q_scale=1.0):
        hq, hkv, d = self.shape = shape
        rng = np.random.default_rng(seed)
        self.q_cu = np.concatenate([[0], np.cumsum(q_lens)]).astype(int)
        self.rows = int(self.q_cu[-1]) + pad_rows
        self.q = bf16(max(1, self.rows), hq, d, seed=seed, scale=q_scale)
        self.own, self.prefix, self.group_cu, self.packed, self.page_rows = own, prefix, group_cu, packed, page_rows
        self.group = [next((g for g in range(len(prefix)) if group_cu[g] <= s < group_cu[g + 1]), -1) for s in range(len(own))]
        self.cu, self.idx, self.n_pages, self.table, self.keep = page_lists(own, page_rows, seed=seed)
        self.pool = [torch.full((self.n_pages * page_rows, hkv, d), float("nan"), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
        for s, n in enumerate(own):
            at = tk.page_rows_of(self.cu, self.idx, page_rows, s, n)
            for i, p in enumerate(self.pool):
                p[at] = bf16(n, hkv, d, seed=seed * 100 + 2 * s + i)
        self.prefix_cu = np.concatenate([[0], np.cumsum(prefix)]).astype(int)
        self.n_prefix = int(self.prefix_cu[-1])
        if packed:
            self.prefix_table, rows = None, [list(range(self.prefix_cu[g], self.prefix_cu[g + 1])) for g in range(len(prefix))]
            size = max(1, self.n_prefix)
        else:
            cu, idx, n_pages, self.prefix_table, self.keep2 = page_lists(prefix, page_rows, seed=seed + 1)
            rows = [tk.page_rows_of(cu, idx, page_rows, g, n) for g, n in enumerate(prefix)]
            size = n_pages * page_rows
        self.kv_prefix = [torch.full((size, hkv, d), float("nan"), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
        for g, at in enumerate(rows):
            for i, p in enumerate(self.kv_prefix):
                p[at] = bf16(len(at), hkv, d, seed=seed * 1000 + 2 * g + i)
        self.prefix_rows = rows
        one_each = all(n == 1 for n in q_lens) and pad_rows == 0
        self.tables = [ints(group_cu) if len(prefix) else None, ints(self.prefix_cu), None if one_each else ints(self.q_cu), ints(own)]
        self.shared = B.make_shared_batch(len(own), len(prefix), *self.tables)

    def room(self, cfg):
        return B.ba_shared_prefix_bytes(cfg, len(self.own), len(self.prefix), self.rows)

    def call(self, c, o, lse, out_dtype, stream=None):
        B.ba_shared_prefix_attend(c.ctx, self.q, self.rows, *self.kv_prefix, self.n_prefix, self.prefix_table, *self.pool, self.table, self.shared, o,
                                  lse, out_dtype, stream)

    def reference(self, scale):
        pool, prefix = [f64(p) for p in self.pool], [f64(p) for p in self.kv_prefix]

        def rows(i):
            def of(s):
                own = pool[i][tk.page_rows_of(self.cu, self.idx, self.page_rows, s, self.own[s])]
                g = self.group[s]
                return own if g < 0 else np.concatenate([prefix[i][self.prefix_rows[g]], own])
            return of
        return tk.shared_attend(f64(self.q)[:self.rows], rows(0), rows(1), self.q_cu, self.own,
                                lambda s: self.prefix[self.group[s]] if self.group[s] >= 0 else 0, scale)


def make_context(shape, batch=None, scale=0.0):
    cfg = B.ba_config(*shape, 0, 1e4, scale, 0)
    return R.Context(*shape, 1e4, softmax_scale=scale, max_blocks=64, max_q_rows=64, workspace_bytes=batch.room(cfg) if batch else 0)


def check_attention(b, o, lse, out_dtype, scale):
    want, want_lse, size = b.reference(scale)
    got, got_lse = f64(o), f64(lse)
    n = int(b.q_cu[-1])
    assert np.isfinite(got[:n]).all()
    err = np.abs(got[:n] - want[:n]) - (HALF_STEP + 1e-4) * size[:n] - (HALF_STEP * np.abs(want[:n]) if out_dtype == B.BA_OUT_BF16 else 0)
    assert err.max() <= 0, err.max()
    empty = np.isinf(want_lse[:n])
    assert (got_lse[:n][empty] == -np.inf).all() and (got[:n][empty] == 0).all()
    assert (np.abs(got_lse[:n][~empty] - want_lse[:n][~empty]) <= 1e-4).all()
    assert (got[n:] == 5).all() and (got_lse[n:] == 6).all()      # rows behind the last sequence


CASES = {
    # name: (prefixes, group_cu, query rows, own rows, page rows, packed)
    "one token": ([], [0], [1], [1], 16, True),
    "no keys": ([0], [0, 1], [1], [0], 16, True),
    "prefix only": ([129], [0, 2], [1, 1], [0, 0], 16, True),
    "tile edges": ([], [0], [1] * 10, [15, 16, 17, 127, 128, 129, 0, 255, 256, 257], 16, True),
    "one group": ([500], [0, 5], [1] * 5, [1, 50, 128, 300, 3], 32, True),
    "groups": ([128, 0, 1, 700], [0, 3, 4, 4, 9], [1] * 9, [5, 0, 130, 0, 9, 77, 64, 1, 20], 64, False),
    "outside groups": ([300, 40], [2, 4, 6], [1] * 8, [10, 0, 20, 30, 0, 50, 60, 129], 128, True),
    "questions": ([333], [0, 4], [17, 1, 64, 33], [17, 40, 64, 200], 64, True),
    "rows before their keys": ([], [0], [9, 5, 2], [4, 0, 300], 16, True),
    "rows before their keys, prefix": ([20], [0, 3], [9, 5, 2], [4, 0, 300], 16, False),
    "no queries": ([90], [0, 4], [0, 2, 0, 3], [10, 11, 0, 300], 256, False),
    "long": ([5000], [0, 3], [1, 2, 1], [2500, 1, 700], 16, True),
    "many rows": ([3000, 130], [0, 5, 9], [20, 1, 40, 3, 60, 1, 1, 1, 1], [20, 5, 300, 3, 700, 0, 1, 128, 200], 32, False),
    "items cut often": ([9000], [0, 3], [70, 1, 2], [100, 30, 2], 16, True),
    "many rows of their own": ([], [0], [50, 40], [1000, 2000], 64, True),
    "both kinds": ([40, 2000, 3], [0, 1, 2, 40], [3, 30] + [1] * 38, [100] * 40, 128, False),
    "a thousand sequences": ([10, 300], [0, 3, 700], [1] * 1000, [(7 * i) % 33 for i in range(1000)], 16, False),
    "many": ([64, 200], [0, 70, 150], [1] * 150, [i % 140 for i in range(150)], 16, False),
}


@pytest.mark.parametrize("shape", [(4, 2, 64), (6, 2, 64), (8, 1, 128), (32, 8, 128), (3, 3, 128), (40, 1, 64)], ids=str)
@pytest.mark.parametrize("name", list(CASES))
def test_shared_attention(shape, name):
    b = Batch(shape, *CASES[name], seed=len(name), pad_rows=0 if name == "one token" else 2)
    c = make_context(shape, b)
    for out_dtype in (B.BA_OUT_F32, B.BA_OUT_BF16):
        kind = torch.float32 if out_dtype == B.BA_OUT_F32 else torch.bfloat16
        o = torch.full((b.rows, *b.q.shape[1:]), 5.0, dtype=kind, device="cuda")
        lse = torch.full((b.rows, shape[0]), 6.0, device="cuda")
        b.call(c, o, lse, out_dtype)
        assert c.device_status() == B.BA_OK
        check_attention(b, o, lse, out_dtype, shape[2] ** -0.5)
        again = torch.full_like(o, 5.0)
        b.call(c, again, None, out_dtype)                       # no lse, and the same bits
        assert torch.equal(again, o)
    c.close()


@pytest.mark.parametrize("packed", [True, False])
def test_large_and_equal_logits(packed):
    """Maxima that grow along the keys (queries 8 times as large), and queries of zero: the mean of the values."""
    shape = (8, 2, 128)
    for q_scale in (8.0, 0.0):
        b = Batch(shape, [700, 900], [0, 2, 3], [1, 3, 2], [300, 5, 140], 16, packed, seed=4, q_scale=q_scale)
        c = make_context(shape, b, scale=0.25)
        o, lse = torch.empty(6, 8, 128, device="cuda"), torch.empty(6, 8, device="cuda")
        b.call(c, o, lse, B.BA_OUT_F32)
        want, want_lse, size = b.reference(0.25)
        # (scores are up to 16 times as large as elsewhere, and so is what 128 fp32 products leave of them)
        assert (np.abs(f64(o) - want) <= (HALF_STEP + 4e-3) * size).all() and (np.abs(f64(lse) - want_lse) <= 4e-3).all()
        c.close()


def test_replays_follow_the_tables():
    """A captured decode step, replayed with other lengths, pages and groups; another stream."""
    shape = (8, 2, 64)
    b = Batch(shape, [300, 20], [0, 2, 6], [1] * 6, [200] * 6, 16, False, seed=9)
    c = make_context(shape, b)
    o, lse = torch.empty(6, 8, 64, device="cuda"), torch.empty(6, 8, device="cuda")
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        b.call(c, o, lse, B.BA_OUT_F32)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        b.call(c, o, lse, B.BA_OUT_F32)
    for own, prefix, group_cu in (([1, 200, 0, 17, 128, 129], [300, 20], [0, 2, 6]), ([200] * 6, [129, 0], [1, 5, 5]), ([0] * 6, [1, 20], [0, 6, 6])):
        b.own, b.prefix, b.group_cu = own, prefix, group_cu
        b.group = [next((g for g in range(2) if group_cu[g] <= s < group_cu[g + 1]), -1) for s in range(6)]
    
        full = Batch(shape, [300, 20], [0, 2, 6], [1] * 6, [200] * 6, 16, False, seed=9)
        b.prefix_rows = [r[:n] for r, n in zip(full.prefix_rows, prefix)]
        b.tables[0].copy_(ints(group_cu))
        b.tables[1].copy_(ints([0, prefix[0], sum(prefix)]))
        b.tables[3].copy_(ints(own))
        o.fill_(float("nan"))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert c.device_status() == B.BA_OK
        check_attention(b, o, lse, B.BA_OUT_F32, 64 ** -0.5)
    c.close()


def test_tables_that_do_not_fit_are_reported_and_nothing_is_written():
    shape = (4, 2, 64)
    good = dict(group_cu=[0, 1, 3], prefix_cu=[0, 100, 150], q_cu=[0, 1, 2, 4], own=[10, 20, 30])
    bad = [dict(group_cu=[0, 2, 1]), dict(group_cu=[-1, 1, 3]), dict(group_cu=[0, 1, 4]), dict(prefix_cu=[0, 100, 90]), dict(prefix_cu=[-5, 100, 150]),
           dict(prefix_cu=[0, 100, 151]), dict(q_cu=[0, 2, 1, 4]), dict(q_cu=[0, 1, 2, 5]), dict(q_cu=[-1, 1, 2, 4]), dict(q_cu=[0, 1, 2, -2 ** 31]), dict(q_cu=[0, 1, 2, 2 ** 31 - 1]), dict(q_cu=[0, 5, -2 ** 31, 4]), dict(own=[10, 20, -1]),
           dict(own=[10, 33, 30]), dict(own=[10, 20, 2 ** 31 - 1])]
    b = Batch(shape, [100, 50], [0, 1, 3], [1, 1, 2], [10, 20, 30], 16, True, seed=2)
    c = make_context(shape, b)
    o, lse = torch.empty(4, 4, 64, device="cuda"), torch.empty(4, 4, device="cuda")
    for change in bad:
        t = {**good, **change}
        b.tables = [ints(t[k]) for k in ("group_cu", "prefix_cu", "q_cu", "own")]
        b.shared = B.make_shared_batch(3, 2, *b.tables)
        o.fill_(5.0)
        lse.fill_(6.0)
        b.call(c, o, lse, B.BA_OUT_F32)
        assert c.device_status() == B.BA_ERR_INVALID_ARG, change
        assert (o == 5).all() and (lse == 6).all(), change
    b.tables = [ints(good[k]) for k in ("group_cu", "prefix_cu", "q_cu", "own")]
    b.shared = B.make_shared_batch(3, 2, *b.tables)
    b.call(c, o, lse, B.BA_OUT_F32)
    assert c.device_status() == B.BA_OK
    check_attention(b, o, lse, B.BA_OUT_F32, 0.125)
    c.close()


def test_pages_outside_the_pool_count_as_zeros():
    shape = (4, 2, 64)
    b = Batch(shape, [], [0], [1, 1], [40, 20], 16, True, seed=3)
    c = make_context(shape, b)
    for page in (-1, b.n_pages, 2 ** 31 - 1):
        idx = b.idx.copy()
        idx[1] = page
        keep = ints(b.cu), ints(idx)
        table, b.table = b.table, B.make_page_table(16, b.n_pages, *keep)
        o, lse = torch.empty(2, 4, 64, device="cuda"), torch.empty(2, 4, device="cuda")
        b.call(c, o, lse, B.BA_OUT_F32)
        assert c.device_status() == B.BA_ERR_INVALID_ARG
        zero = [torch.cat([p, torch.zeros_like(p[:16])]) for p in b.pool]
        pools, b.pool, real, b.idx = b.pool, zero, b.idx, idx.copy()
        b.idx[1] = b.n_pages
        check_attention(b, o, lse, B.BA_OUT_F32, 0.125)
        b.table, b.pool, b.idx = table, pools, real
    c.close()


def test_rows_beyond_32_bits_of_elements():
    """A pool of 2.2 million rows x 8 heads x 128: the sequence's pages are its last ones."""
    shape, n = (8, 8, 128), 2_200_000 // 64
    c = R.Context(*shape, 1e4, max_blocks=64, max_q_rows=64, workspace_bytes=B.ba_shared_prefix_bytes(B.ba_config(*shape, 0, 1e4, 0.0, 0), 1, 0, 1))
    pool = [torch.empty(n * 64, 8, 128, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    cu, idx = ints([0, 3]), ints([n - 1, 7, n - 2])
    table = B.make_page_table(64, n, cu, idx)
    k, v, q = bf16(150, 8, 128, seed=1), bf16(150, 8, 128, seed=2), bf16(150, 8, 128, seed=3)
    q_out = torch.empty_like(q)
    B.ba_append_paged(c.ctx, q, k, v, 150, None, None, None, 0.0, ints([0, 150]), ints([0]), 1, q_out, *pool, table)
    at = tk.page_rows_of([0, 3], [n - 1, 7, n - 2], 64, 0, 150)
    assert torch.equal(pool[0][at], k) and torch.equal(pool[1][at], v) and torch.equal(q_out, q)
    o, lse, own = torch.empty(1, 8, 128, device="cuda"), torch.empty(1, 8, device="cuda"), ints([150])
    B.ba_shared_prefix_attend(c.ctx, q[149:].clone(), 1, None, None, 0, None, *pool, table, B.make_shared_batch(1, 0, None, None, None, own), o, lse,
                              B.BA_OUT_F32)
    assert c.device_status() == B.BA_OK
    want, want_lse, size = tk.shared_attend(f64(q)[149:], lambda s: f64(k), lambda s: f64(v), [0, 1], [150], lambda s: 0, 128 ** -0.5)
    assert (np.abs(f64(o) - want) <= (HALF_STEP + 1e-4) * size).all() and (np.abs(f64(lse) - want_lse) <= 1e-4).all()
    c.close()


def test_one_pool_for_prefixes_and_sequences():
    """Prefixes and own rows on lists of one pool, the prefix's pages shared with a sequence's list."""
    shape = (8, 2, 128)
    pool = [bf16(40 * 16, 2, 128, seed=s) for s in (1, 2)]
    q = bf16(3, 8, 128, seed=3)
    keep = ints([0, 5]), ints([3, 9, 4, 11, 0]), ints([0, 2, 4, 9]), ints([20, 21, 30, 31, 3, 9, 4, 11, 0])
    cfg = B.ba_config(*shape, 0, 1e4, 0.0, 0)
    c = R.Context(*shape, 1e4, max_blocks=64, max_q_rows=64, workspace_bytes=B.ba_shared_prefix_bytes(cfg, 3, 1, 3))
    tables = ints([0, 2]), ints([0, 70]), ints([17, 32, 75])
    o, lse = torch.empty(3, 8, 128, device="cuda"), torch.empty(3, 8, device="cuda")
    B.ba_shared_prefix_attend(c.ctx, q, 3, *pool, 0, B.make_page_table(16, 40, *keep[:2]), *pool, B.make_page_table(16, 40, *keep[2:]),
                              B.make_shared_batch(3, 1, tables[0], tables[1], None, tables[2]), o, lse, B.BA_OUT_F32)
    assert c.device_status() == B.BA_OK
    prefix = tk.page_rows_of([0, 5], [3, 9, 4, 11, 0], 16, 0, 70)
    own = [tk.page_rows_of([0, 2, 4, 9], [20, 21, 30, 31, 3, 9, 4, 11, 0], 16, s, n) for s, n in enumerate((17, 32, 75))]
    rows = [prefix + own[0], prefix + own[1], own[2]]
    want, want_lse, size = tk.shared_attend(f64(q), lambda s: f64(pool[0])[rows[s]], lambda s: f64(pool[1])[rows[s]], [0, 1, 2, 3], [17, 32, 75],
                                            lambda s: 70 if s < 2 else 0, 128 ** -0.5)
    assert (np.abs(f64(o) - want) <= (HALF_STEP + 1e-4) * size).all() and (np.abs(f64(lse) - want_lse) <= 1e-4).all()
    c.close()


def test_what_lies_in_padding_rows_changes_nothing():
    """Query rows behind the last sequence share a tile with real ones: other values there, the same bits everywhere else."""
    b = Batch((8, 2, 128), [400, 900], [0, 20, 25], [1] * 25, [40] * 25, 16, False, seed=5, pad_rows=30)
    c = make_context((8, 2, 128), b)
    outs = []
    for fill in (0.0, 40.0, float("nan"), float("inf")):
        b.q[25:] = fill
        o, lse = torch.zeros(55, 8, 128, device="cuda"), torch.zeros(55, 8, device="cuda")
        b.call(c, o, lse, B.BA_OUT_F32)
        outs.append((o, lse))
    for o, lse in outs[1:]:
        assert torch.equal(o, outs[0][0]) and torch.equal(lse, outs[0][1])
    c.close()


def test_a_captured_decode_step():
    """Append and attention captured together and replayed: the tables move on between replays, as a server's would."""
    shape = (8, 2, 64)
    hq, hkv, d = shape
    cfg = B.ba_config(*shape, 0, 1e4, 0.0, 0)
    c = R.Context(*shape, 1e4, max_blocks=64, max_q_rows=64, workspace_bytes=B.ba_shared_prefix_bytes(cfg, 4, 1, 4))
    prefix = [bf16(300, hkv, d, seed=s) for s in (1, 2)]
    cu, idx, n_pages, table, keep = page_lists([40] * 4, 16)
    pools = [torch.full((n_pages * 16, hkv, d), float("nan"), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    qkv, q_out = bf16(4, hq + 2 * hkv, d, seed=3), torch.empty(4, hq, d, dtype=torch.bfloat16, device="cuda")
    w = bf16(d, seed=4)
    pos, start, own, prefix_cu = ints([300] * 4), ints([0] * 4), ints([1] * 4), ints([0, 300])
    shared = B.make_shared_batch(4, 1, None, prefix_cu, None, own)
    o, lse = torch.empty(4, hq, d, device="cuda"), torch.empty(4, hq, device="cuda")

    def step():
        B.ba_append_paged(c.ctx, qkv[:, :hq], qkv[:, hq:hq + hkv], qkv[:, hq + hkv:], 4, pos, w, w, 1e-6, None, start, 4, q_out, *pools, table)
        B.ba_shared_prefix_attend(c.ctx, q_out, 4, *prefix, 300, None, *pools, table, shared, o, lse, B.BA_OUT_F32)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        step()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        step()
    keys, values = [f64(prefix[0])], [f64(prefix[1])]
    for n in range(20):
        qkv.copy_(bf16(4, hq + 2 * hkv, d, seed=100 + n))
        pos.fill_(300 + n)
        start.fill_(n)
        own.fill_(n + 1)
        graph.replay()
        assert c.device_status() == B.BA_OK
        at = [tk.page_rows_of(cu, idx, 16, s, n + 1) for s in range(4)]
        want, want_lse, size = tk.shared_attend(f64(q_out), lambda s: np.concatenate([keys[0], f64(pools[0])[at[s]]]),
                                                lambda s: np.concatenate([values[0], f64(pools[1])[at[s]]]), [0, 1, 2, 3, 4], [n + 1] * 4, lambda s: 300,
                                                d ** -0.5)
        assert torch.equal(pools[1][[a[-1] for a in at]], qkv[:, hq + hkv:])
        assert (np.abs(f64(o) - want) <= (HALF_STEP + 1e-4) * size).all() and (np.abs(f64(lse) - want_lse) <= 1e-4).all()
    c.close()


def test_two_contexts_on_two_streams():
    """Calls of two contexts that run at the same time: each gives what it gives alone."""
    batches = [Batch((8, 2, 128), [3000, 200], [0, 20, 30], [1] * 40, [500] * 40, 16, False, seed=5), Batch((8, 2, 128), [900], [0, 3], [40, 1, 7], [40, 300, 90], 64, True, seed=6)]
    contexts = [make_context((8, 2, 128), b) for b in batches]
    alone = []
    for b, c in zip(batches, contexts):
        o, lse = torch.empty(b.rows, 8, 128, device="cuda"), torch.empty(b.rows, 8, device="cuda")
        b.call(c, o, lse, B.BA_OUT_F32)
        alone.append((o, lse))
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in batches]
    outs = [[(torch.empty_like(a[0]), torch.empty_like(a[1])) for _ in range(10)] for a in alone]
    torch.cuda.synchronize()
    for n in range(10):
        for b, c, st, out in zip(batches, contexts, streams, outs):
            b.call(c, *out[n], B.BA_OUT_F32, st)
    torch.cuda.synchronize()
    for a, out in zip(alone, outs):
        for o, lse in out:
            assert torch.equal(o, a[0]) and torch.equal(lse, a[1])
    for c in contexts:
        assert c.device_status() == B.BA_OK
        c.close()


def test_a_queued_reencoding_stays_queued():
    """The calls leave a deferred re-encoding and its table at the end of the workspace alone."""
    b = Batch((8, 2, 128), [200], [0, 3], [1] * 4, [50] * 4, 16, True, seed=7)
    cfg = B.ba_config(8, 2, 128, 0, 1e4, 0.0, 0)
    c = R.Context(8, 2, 128, 1e4, max_blocks=64, max_q_rows=64, workspace_bytes=b.room(cfg) + (1 << 20))
    k, cu, delta = bf16(90, 2, 128, seed=1), ints([0, 40, 90]), ints([0, 40])
    want, got = torch.empty_like(k), torch.zeros_like(k)
    B.ba_reencode_k(c.ctx, k, None, 90, want, cu, delta, 2, 90)
    B.ba_reencode_k_deferred(c.ctx, k, None, 90, got, cu, delta, 2, 90)
    o, lse = torch.empty(4, 8, 128, device="cuda"), torch.empty(4, 8, device="cuda")
    b.call(c, o, lse, B.BA_OUT_F32)
    w, x, dq, dw = bf16(128, seed=2), bf16(4, 8, 128, seed=3), torch.empty(4, 8, 128, device="cuda"), torch.empty(128, device="cuda")
    B.ba_qk_norm_rope_bwd(c.ctx, x, None, 4, None, w, None, 1e-6, o, None, dq, None, dw, None, B.BA_OUT_F32)
    torch.cuda.synchronize()
    assert (got == 0).all()
    B.ba_flush(c.ctx)
    assert torch.equal(got, want) and c.device_status() == B.BA_OK
    check_attention(b, o, lse, B.BA_OUT_F32, 128 ** -0.5)
    c.close()


def test_the_calls_without_the_extension(monkeypatch):
    """Through ctypes: the same bits as through the extension."""
    shape = (6, 2, 64)
    hq, hkv, d = shape
    cfg = B.ba_config(*shape, 0, 1e4, 0.0, 0)
    c = R.Context(*shape, 1e4, max_blocks=64, max_q_rows=64, workspace_bytes=B.ba_shared_prefix_bytes(cfg, 3, 0, 3))
    qkv, w = bf16(3, hq + 2 * hkv, d, seed=3), bf16(d, seed=4)
    q, k, v = qkv[:, :hq], qkv[:, hq:hq + hkv], qkv[:, hq + hkv:]
    cu, idx, n_pages, table, keep = page_lists([5, 20, 40], 16)
    start, own, pos = ints([4, 19, 39]), ints([5, 20, 40]), ints([9, 8, 7])
    shared = B.make_shared_batch(3, 0, None, None, None, own)

    def everything():
        pools = [bf16(n_pages * 16, hkv, d, seed=s) for s in (1, 2)]
        q_out, o, lse = torch.empty(3, hq, d, dtype=torch.bfloat16, device="cuda"), torch.empty(3, hq, d, device="cuda"), torch.empty(3, hq, device="cuda")
        B.ba_append_paged(c.ctx, q, k, v, 3, pos, w, w, 1e-6, None, start, 3, q_out, *pools, table)
        B.ba_shared_prefix_attend(c.ctx, q_out, 3, None, None, 0, None, *pools, table, shared, o, lse, B.BA_OUT_F32)
        qn, kn = torch.empty(3, hq, d, dtype=torch.bfloat16, device="cuda"), torch.empty(3, hkv, d, dtype=torch.bfloat16, device="cuda")
        B.ba_qk_norm_rope(c.ctx, q, k, 3, pos, w, w, 1e-6, qn, kn)
        grad = torch.zeros(3, hq + 2 * hkv, d, dtype=torch.bfloat16, device="cuda")
        dw = torch.empty(2, d, device="cuda")
        B.ba_qk_norm_rope_bwd(c.ctx, q, k, 3, pos, w, w, 1e-6, qn, kn, grad[:, :hq], grad[:, hq:hq + hkv], dw[0], dw[1], B.BA_OUT_BF16)
        return [*pools, q_out, o, lse, qn, kn, grad, dw]
    fast = everything()
    monkeypatch.setattr(B, "_marshal", B._CtypesCalls())
    for a, b in zip(fast, everything()):
        assert torch.equal(a, b)
    assert c.device_status() == B.BA_OK
    c.close()


def _refused(status, call):
    with pytest.raises(B.BaError) as e:
        call()
    assert e.value.status == status


def test_refusals():
    """Every one of these is answered on the host, before anything is launched."""
    shape = (4, 2, 64)
    c = context(shape)
    q, k, v, w = bf16(4, 4, 64), bf16(4, 2, 64), bf16(4, 2, 64), bf16(64)
    pos = ints(range(4))
    bad, shp = B.BA_ERR_INVALID_ARG, B.BA_ERR_SHAPE
    oq, okk = torch.empty_like(q), torch.empty_like(k)
    n0 = c.launches()
    norm = lambda *a: (lambda: B.ba_qk_norm_rope(c.ctx, *a))
    wide = bf16(4, 8, 64)
    _refused(bad, norm(q, k, -1, pos, w, w, 1e-6, oq, okk))
    _refused(bad, norm(None, None, 4, pos, w, w, 1e-6, None, None))
    _refused(bad, norm(q, k, 4, pos, w, w, 1e-6, oq, None))
    _refused(bad, norm(None, k, 4, pos, w, w, 1e-6, oq, okk))
    _refused(bad, norm(q.data_ptr() + 2, k, 4, pos, w, w, 1e-6, oq, okk))
    _refused(bad, norm(q, k, 4, pos, w.data_ptr() + 8, w, 1e-6, oq, okk))
    _refused(bad, norm(q, k, 4, pos, w, w, -1e-6, oq, okk))
    _refused(bad, norm(q, k, 4, pos, w, w, float("nan"), oq, okk))
    _refused(bad, norm(wide[:, :4], k, 4, pos, w, w, 1e-6, wide, okk))                     # in place in rows that lie apart
    lib = B.load_library()
    p = lambda t: t.data_ptr()
    for stride in (-256, 128, 260):
        assert lib.ba_qk_norm_rope(c.ctx, p(q), stride, p(k), 0, 4, p(pos), None, None, 0.0, p(oq), p(okk), None) == bad
    g, gk, dw = torch.empty(4, 4, 64, device="cuda"), torch.empty(4, 2, 64, device="cuda"), torch.empty(64, device="cuda")
    bwd = lambda *a: (lambda: B.ba_qk_norm_rope_bwd(c.ctx, *a))
    _refused(bad, bwd(q, k, 4, pos, w, w, 1e-6, g, gk, g, gk, dw, None, B.BA_OUT_F32))     # a norm without room for its gradient
    _refused(bad, bwd(q, k, 4, pos, None, None, 1e-6, g, gk, g, gk, dw, dw, B.BA_OUT_F32))  # and the other way round
    _refused(bad, bwd(None, k, 4, pos, w, w, 1e-6, g, gk, g, gk, dw, dw, B.BA_OUT_F32))
    _refused(bad, bwd(q, k, 4, pos, w, w, 1e-6, g, None, g, gk, dw, dw, B.BA_OUT_F32))
    _refused(bad, bwd(q, k, 4, pos, w, w, 1e-6, g, gk, g, gk, dw, dw, 2))
    tiny = B.ba_create(c.cfg, 0, 64 * 1024 + 1024)
    _refused(B.BA_ERR_WORKSPACE, lambda: B.ba_qk_norm_rope_bwd(tiny, q, k, 4, pos, w, w, 1e-6, g, gk, g, gk, dw, dw, B.BA_OUT_F32))
    kp, vp = bf16(64, 2, 64), bf16(64, 2, 64)
    cu, idx, start = ints([0, 1, 2, 3, 4]), ints(range(4)), ints([0] * 4)
    table = B.make_page_table(16, 4, cu, idx)
    app = lambda *a: (lambda: B.ba_append_paged(c.ctx, *a))
    _refused(shp, app(q, k, v, 4, pos, w, w, 1e-6, None, start, 3, oq, kp, vp, table))
    _refused(bad, app(q, k, v, 4, pos, w, w, 1e-6, None, None, 4, oq, kp, vp, table))
    _refused(bad, app(q, k, v, 4, pos, w, w, 1e-6, None, start, 4, None, kp, vp, table))
    _refused(bad, app(q, k, None, 4, pos, w, w, 1e-6, None, start, 4, oq, kp, vp, table))
    _refused(bad, app(q, k, v, 4, pos, w, w, 1e-6, None, start, 4, oq, kp, kp, table))
    _refused(bad, app(q, kp[:4], v, 4, pos, w, w, 1e-6, None, start, 4, oq, kp, vp, table))
    own = ints([1] * 4)
    sh = lambda **kw: B.make_shared_batch(*{**dict(batch=4, n_groups=0, group_cu=None, prefix_cu=None, q_cu=None, own_len=own), **kw}.values())
    att = lambda n=4, kx=None, vx=None, nx=0, px=None, k=kp, v=vp, s=None, o=oq, out=B.BA_OUT_BF16, ctx=None: (
        lambda: B.ba_shared_prefix_attend(ctx or c.ctx, q, n, kx, vx, nx, px, k, v, table, s or sh(), o, None, out))
    _refused(bad, att(s=sh(own_len=None)))
    _refused(bad, att(s=sh(batch=-1)))
    _refused(bad, att(s=sh(n_groups=1)))                                                   # no prefix table
    _refused(bad, att(s=sh(n_groups=2, prefix_cu=own), kx=kp, vx=vp, nx=64))               # two groups, no group table
    _refused(bad, att(s=sh(n_groups=1, prefix_cu=own), kx=None, vx=vp, nx=64))
    _refused(shp, att(s=sh(batch=3)))
    _refused(B.BA_ERR_UNSUPPORTED, att(s=sh(batch=B.BA_SHARED_MAX + 1, q_cu=own)))
    _refused(bad, att(o=None))
    _refused(bad, att(out=7))
    _refused(bad, att(n=-1))
    _refused(bad, att(k=kp.data_ptr() + 8))
    _refused(B.BA_ERR_WORKSPACE, att(ctx=tiny))
    B.ba_destroy(tiny)
    assert c.launches() == n0
    # nothing to do is fine
    att(n=0, s=sh(batch=0))()
    B.ba_append_paged(c.ctx, None, k, v, 0, None, None, None, 0.0, None, start, 0, None, kp, vp, table)
    c.close()


# ------------------------------------------------------------------ together
def test_a_prompt_and_its_answers():
    """Two prompts are prefilled from cached passages; each is asked three questions at once, which then decode a few tokens: the fused
    call's keys are the packed prefix, questions and tokens go through the append, attention runs over both.  Checked against the oracle's causal
    attention over everything at once, after every step."""
    shape, theta, eps = (8, 2, 64), 5e5, 1e-6
    hq, hkv, d = shape
    passages = [[60, 131, 17], [200, 5]]
    lens = [n for p in passages for n in p + [1]]                # (the tables want a final block: one token, thrown away)
    room = B.ba_shared_prefix_bytes(B.ba_config(*shape, 0, theta, 0.0, 0), 6, 2, 6 * 40)
    c = context(shape, theta=theta, room=room)
    seg, buf = c.segment(lens, [4, 3], B.BA_MODE_BLOCK)
    n_cache = sum(map(sum, passages))
    k_cached, v_cached = bf16(n_cache, hkv, d, seed=1), bf16(n_cache, hkv, d, seed=2)      # keys at positions 0 .. of their passage
    fq, fk, fv = bf16(2, hq, d, seed=3), bf16(2, hkv, d, seed=4), bf16(2, hkv, d, seed=5)
    k_prefix = torch.empty_like(k_cached)
    B.ba_final_attend_fused(c.ctx, fq, fk, fv, 2, k_cached, v_cached, n_cache, None, n_cache, torch.empty_like(fq), None, seg, B.BA_MODE_BLOCK,
                            B.BA_OUT_BF16, k_out=k_prefix)
    totals = [sum(p) for p in passages]
    start = [0, totals[0]]
    group = [0, 0, 0, 1, 1, 1]
    questions = [33, 1, 7, 40, 2, 12]
    cu, idx, n_pages, table, keep = page_lists([n + 4 for n in questions], 16)
    pools = [torch.full((n_pages * 16, hkv, d), float("nan"), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    w_q, w_k = bf16(d, seed=6), bf16(d, seed=7)
    own = [0] * 6
    keys, values = [[] for _ in range(6)], [[] for _ in range(6)]
    for step in range(4):
        new = questions if step == 0 else [1] * 6
        rows = sum(new)
        q_cu = np.concatenate([[0], np.cumsum(new)]).astype(int)
        qkv = bf16(rows, hq + 2 * hkv, d, seed=50 + step)
        q, k, v = qkv[:, :hq], qkv[:, hq:hq + hkv], qkv[:, hq + hkv:]
        pos = [totals[group[s]] + own[s] + t for s in range(6) for t in range(new[s])]
        q_out = torch.empty(rows, hq, d, dtype=torch.bfloat16, device="cuda")
        table_cu, begin = (ints(q_cu) if step == 0 else None), ints(own)
        B.ba_append_paged(c.ctx, q, k, v, rows, ints(pos), w_q, w_k, eps, table_cu, begin, 6, q_out, *pools, table)
        for s in range(6):
            sl = slice(q_cu[s], q_cu[s + 1])
            keys[s].append(tk.norm_rope(f64(k[sl]), pos[sl], f64(w_k), eps, theta))
            values[s].append(f64(v[sl]))
            own[s] += new[s]
        now, groups, pcu = ints(own), ints([0, 3, 6]), seg.cu_cache_seq
        o, lse = torch.empty(rows, hq, d, device="cuda"), torch.empty(rows, hq, device="cuda")
        B.ba_shared_prefix_attend(c.ctx, q_out, rows, k_prefix, v_cached, n_cache, None, *pools, table,
                                  B.make_shared_batch(6, 2, groups, pcu, table_cu, now), o, lse, B.BA_OUT_F32)
        assert c.device_status() == B.BA_OK
        # the oracle: re-encoding of the passages, norms and rotations in fp64, attention over all of it
        ref_prefix = []
        at = 0
        for p in passages:
            delta, ks = 0, []
            for n in p:
                ks.append(tk.rotate(f64(k_cached[at:at + n]), [delta] * n, theta))
                delta, at = delta + n, at + n
            ref_prefix.append(np.concatenate(ks))
        kk = lambda s: np.concatenate([ref_prefix[group[s]], *keys[s]])
        vv = lambda s: np.concatenate([f64(v_cached[start[group[s]]:start[group[s]] + totals[group[s]]]), *values[s]])
        qr = tk.norm_rope(f64(q), pos, f64(w_q), eps, theta)
        want, want_lse, size = tk.shared_attend(qr, kk, vv, q_cu, own, lambda s: totals[group[s]], d ** -0.5)
        # rounding of q and k to bf16 (2^-8 each) moves a score by at most 2^-7 sum|q k| / sqrt(d), which is at most |q||k| / sqrt(d)
        reach = max(np.linalg.norm(qr, axis=-1).max() * np.linalg.norm(kk(s), axis=-1).max() for s in range(6)) * d ** -0.5 * 2.0 ** -7
        assert (np.abs(f64(lse) - want_lse) <= reach + 1e-4).all()
        assert (np.abs(f64(o) - want) <= (np.expm1(2 * reach) + HALF_STEP + 1e-4) * size).all()
        fro = np.linalg.norm(f64(o) - want) / np.linalg.norm(want)
        assert fro <= 2e-2, fro                                  # (rounding of q, k and P is random: the bound above is the worst case)
    c.close()


def test_a_training_step_through_norms_rotation_and_attention():
    """Projections -> norms and rotation -> block attention -> its gradients -> gradients of projections and norm weights, against autograd in
    fp64; positions are the tables'."""
    shape, theta, eps, lens = (4, 2, 64), 1e4, 1e-5, [40, 70, 33]
    hq, hkv, d = shape
    T = sum(lens)
    c = context(shape, theta=theta)
    seg, buf = c.segment(lens, [3], B.BA_MODE_BLOCK)
    x = bf16(T, hq + 2 * hkv, d, seed=1)
    w_q, w_k = bf16(d, seed=2), bf16(d, seed=3)
    q, k = (torch.empty(T, h, d, dtype=torch.bfloat16, device="cuda") for h in (hq, hkv))
    v = x[:, hq + hkv:].contiguous()
    B.ba_qk_norm_rope(c.ctx, x[:, :hq], x[:, hq:hq + hkv], T, seg.tok_pos, w_q, w_k, eps, q, k)
    o, lse = torch.empty_like(q), torch.empty(T, hq, device="cuda")
    B.ba_block_prefill(c.ctx, q, k, v, o, lse, seg, B.BA_MODE_BLOCK, B.BA_OUT_BF16)
    dy = bf16(T, hq, d, seed=4)
    dq, dk, dv = (torch.empty(T, h, d, device="cuda") for h in (hq, hkv, hkv))
    B.ba_block_prefill_bwd(c.ctx, q, k, v, o, lse, dy, dq, dk, dv, seg, B.BA_MODE_BLOCK, B.BA_OUT_F32)
    grad = torch.zeros(T, hq + 2 * hkv, d, device="cuda")
    dw_q, dw_k = torch.empty(d, device="cuda"), torch.empty(d, device="cuda")
    B.ba_qk_norm_rope_bwd(c.ctx, x[:, :hq], x[:, hq:hq + hkv], T, seg.tok_pos, w_q, w_k, eps, dq, dk, grad[:, :hq], grad[:, hq:hq + hkv], dw_q, dw_k,
                          B.BA_OUT_F32)
    grad[:, hq + hkv:] = dv
    assert c.device_status() == B.BA_OK
    # autograd, fp64, CPU
    X = x.double().cpu().requires_grad_()
    W = [t.double().cpu().requires_grad_() for t in (w_q, w_k)]
    pos = torch.cat([torch.arange(sum(lens))]).double()
    ang = pos[:, None, None] * torch.tensor([theta ** (-2.0 * m / d) for m in range(d // 2)], dtype=torch.float64)

    def turn(y, w):
        y = y / torch.sqrt((y * y).mean(-1, keepdim=True) + eps) * w
        a, b = y[..., 0::2], y[..., 1::2]
        return torch.stack([a * ang.cos() - b * ang.sin(), a * ang.sin() + b * ang.cos()], -1).flatten(-2)
    Q, K, V = turn(X[:, :hq], W[0]), turn(X[:, hq:hq + hkv], W[1]).repeat_interleave(2, 1), X[:, hq + hkv:].repeat_interleave(2, 1)
    block = torch.repeat_interleave(torch.arange(3), torch.tensor(lens))
    sees = (torch.arange(T)[:, None] >= torch.arange(T)[None]) & ((block[:, None] == block[None]) | (block[:, None] == 2))
    P = torch.softmax((torch.einsum("ihd,jhd->hij", Q, K) * d ** -0.5).masked_fill(~sees, float("-inf")), -1)
    (torch.einsum("hij,jhd->ihd", P, V) * dy.double().cpu()).sum().backward()
    # (the library's gradients of attention are within 1e-2 of the tensor, from bf16 q, k, P and dS)
    for got, want in ((grad, X.grad), (dw_q, W[0].grad), (dw_k, W[1].grad)):
        assert np.linalg.norm(f64(got) - want.numpy()) <= 2e-2 * np.linalg.norm(want.numpy())
    c.close()
