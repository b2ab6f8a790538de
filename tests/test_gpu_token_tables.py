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


# ------------------------------------------------------------------ values that are not finite
QUESTIONS = {"few rows": [1, 2, 1], "a query tile": [20, 1, 10], "two query tiles": [70, 40, 3]}
PLANTED = [("key of the prefix", float("nan")), ("key of the prefix", float("inf")), ("key of the prefix", float("-inf")), ("every key of the prefix", float("nan")),
           ("last key of its own", float("nan")), ("last key of its own", float("inf")), ("key of a sequence alone", float("nan")),
           ("key of a sequence alone", float("inf")), ("query", float("nan")), ("query", float("inf")), ("value of the prefix", float("nan"))]


@pytest.mark.parametrize("shape", [(4, 2, 64), (8, 2, 128)], ids=str)
@pytest.mark.parametrize("questions", list(QUESTIONS))
@pytest.mark.parametrize("alone", [100, 4000], ids=["whole", "cut"])
@pytest.mark.parametrize("where,value", PLANTED, ids=str)
def test_values_that_are_not_finite_go_through(shape, questions, alone, where, value):
    """As in the formula: a row that sees a score which is NaN or +infinity is NaN, its log-sum-exp too, wherever the work is cut; every other
    row is what it would be."""
    q_lens = QUESTIONS[questions]
    b = Batch(shape, [2000], [0, 3], q_lens + [1], [300, 40, 5, alone], 16, False, seed=11)
    own = [tk.page_rows_of(b.cu, b.idx, 16, s, n) for s, n in enumerate(b.own)]
    if where == "key of the prefix":
        b.kv_prefix[0][b.prefix_rows[0][1333], 1, 5] = value
    elif where == "every key of the prefix":
        b.kv_prefix[0][b.prefix_rows[0], 1, 5] = value
    elif where == "last key of its own":
        b.pool[0][own[0][-1], 1, 5] = value
    elif where == "key of a sequence alone":
        b.pool[0][own[3][alone // 2], 1, 5] = value
    elif where == "query":
        b.q[sum(q_lens[:2]), 1, 5] = value                      # (its scores are infinite with either sign, and NaN without)
    else:
        b.kv_prefix[1][b.prefix_rows[0][1333], 1, 5] = value
    c = make_context(shape, b)
    o, lse = torch.full((b.rows, *shape[::2]), 5.0, device="cuda"), torch.full((b.rows, shape[0]), 6.0, device="cuda")
    b.call(c, o, lse, B.BA_OUT_F32)
    assert c.device_status() == B.BA_OK
    with np.errstate(all="ignore"):
        want, want_lse, size = b.reference(shape[2] ** -0.5)
    got, got_lse, fine = f64(o), f64(lse), np.isfinite(want)
    assert (np.isnan(got) == ~fine).all() and (np.isnan(got_lse) == np.isnan(want_lse)).all()
    assert fine.any() and (np.isinf(value) or not fine.all())       # (an infinite key's scores are infinite with the query's sign)
    assert (np.abs(got - want)[fine] <= (HALF_STEP + 1e-4) * size[fine]).all()
    known = ~np.isnan(want_lse)
    assert (np.abs(got_lse - want_lse)[known] <= 1e-4).all()
    c.close()


# ------------------------------------------------------------------ calls that follow one another closely
def test_results_of_calls_in_close_succession():
    """Nothing waits between the calls, and each reads what the one before has just written: the weights' sums out of the workspace, queries and
    keys out of the append, positions and lengths out of the tables' call.  Every round gives what it gives alone."""
    shape = (8, 2, 64)
    hq, hkv, d = shape
    lens = [[40, 17, 1], [9, 70, 1], [3, 2, 1]]
    n = 40
    cfg = B.ba_config(*shape, 0, 1e4, 0.0, 0)
    c = R.Context(*shape, 1e4, max_blocks=64, max_q_rows=256, workspace_bytes=B.ba_shared_prefix_bytes(cfg, n, 1, n))
    w = bf16(d, seed=1)
    prefix = [bf16(200, hkv, d, seed=s) for s in (2, 3)]
    page_cu, page_idx, start, own = ints(range(n + 1)), ints(reversed(range(n))), ints([0] * n), ints([1] * n)
    table = B.make_page_table(16, n, page_cu, page_idx)
    pools = [torch.zeros(n * 16, hkv, d, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    segments = [np.asarray(x, dtype=np.int32) for x in lens]
    buf = torch.empty(B.ba_segments_bytes(1, 3, 80), dtype=torch.uint8, device="cuda")
    q_out = torch.empty(n, hq, d, dtype=torch.bfloat16, device="cuda")

    def round_(k, out):
        x = inputs[k]
        rows = int(segments[k].sum())
        seg = B.ba_segment(c.ctx, segments[k], np.asarray([3], dtype=np.int32), 1, 3, rows, B.BA_MODE_BLOCK, buf)
        B.ba_qk_norm_rope(c.ctx, x[:rows, :hq], None, rows, seg.tok_pos, w, None, 1e-6, out["q"][:rows], None)
        B.ba_qk_norm_rope_bwd(c.ctx, x[:rows, :hq], None, rows, seg.tok_pos, w, None, 1e-6, out["q"][:rows], None, out["dq"][:rows], None, out["dw"], None,
                              B.BA_OUT_BF16)
        B.ba_append_paged(c.ctx, x[:n, :hq], x[:n, hq:hq + hkv], x[:n, hq + hkv:], n, start, w, w, 1e-6, None, start, n, q_out, *pools, table)
        shared = B.make_shared_batch(n, 1, None, seg.cu_cache_seq, None, own)           # (the prefix: the cached tokens of the tables)
        B.ba_shared_prefix_attend(c.ctx, q_out, n, *prefix, 200, None, *pools, table, shared, out["o"], out["lse"], B.BA_OUT_F32)

    inputs = [bf16(80, hq + 2 * hkv, d, seed=20 + k) for k in range(3)]
    room = lambda: {"q": torch.zeros(80, hq, d, dtype=torch.bfloat16, device="cuda"), "dq": torch.zeros(80, hq, d, dtype=torch.bfloat16, device="cuda"),
                    "dw": torch.zeros(d, device="cuda"), "o": torch.zeros(n, hq, d, device="cuda"), "lse": torch.zeros(n, hq, device="cuda")}
    alone = []
    for k in range(3):
        alone.append(room())
        torch.cuda.synchronize()
        round_(k, alone[k])
        torch.cuda.synchronize()
    outs = [room() for _ in range(30)]
    torch.cuda.synchronize()
    for i, out in enumerate(outs):
        round_(i % 3, out)
    torch.cuda.synchronize()
    assert c.device_status() == B.BA_OK
    for i, out in enumerate(outs):
        for key, want in alone[i % 3].items():
            assert torch.equal(out[key], want), (i, key)
    for key in ("q", "o", "dw"):
        assert not torch.equal(alone[0][key], alone[1][key])
    c.close()


# ------------------------------------------------------------------ a queued re-encoding
@pytest.mark.parametrize("reader", ["packed prefix", "pool of the prefix", "own pool", "append", "norm"])
def test_a_queued_reencoding_is_run_before_its_keys_are_read(reader):
    """The call that takes the queued job's k_dst finds the keys in it, without a ba_flush in between."""
    shape = (8, 2, 128)
    hq, hkv, d = shape
    cfg = B.ba_config(*shape, 0, 1e4, 0.0, 0)
    c = R.Context(*shape, 1e4, max_blocks=64, max_q_rows=64, workspace_bytes=B.ba_shared_prefix_bytes(cfg, 3, 1, 3) + (1 << 20))
    rows, page_rows = 96, 16
    k, v, q = bf16(rows, hkv, d, seed=1), bf16(rows, hkv, d, seed=2), bf16(3, hq, d, seed=3)
    cu, delta = ints([0, 40, rows]), ints([0, 40])
    tables = ints([0, 6]), ints([5, 3, 1, 0, 2, 4]), ints([0, 2, 4, 6]), ints([0, 3]), ints([0, 90]), ints([20, 30, 0]), ints([0] * rows), ints([0, rows])
    whole, apart = B.make_page_table(page_rows, 6, *tables[:2]), B.make_page_table(page_rows, 6, tables[2], tables[1])
    own = bf16(rows, hkv, d, seed=4)

    def read(keys):
        o, lse = torch.zeros(3, hq, d, device="cuda"), torch.zeros(3, hq, device="cuda")
        shared = B.make_shared_batch(3, 1, tables[3], tables[4], None, tables[5])
        if reader == "packed prefix":
            B.ba_shared_prefix_attend(c.ctx, q, 3, keys, v, rows, None, own, v, apart, shared, o, lse, B.BA_OUT_F32)
        elif reader == "pool of the prefix":
            B.ba_shared_prefix_attend(c.ctx, q, 3, keys, v, 0, whole, own, v, apart, shared, o, lse, B.BA_OUT_F32)
        elif reader == "own pool":
            B.ba_shared_prefix_attend(c.ctx, q, 3, own, v, rows, None, keys, v, apart, shared, o, lse, B.BA_OUT_F32)
        elif reader == "append":
            pools = [torch.zeros(rows, hkv, d, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
            B.ba_append_paged(c.ctx, None, keys, v, rows, None, None, None, 0.0, tables[7], tables[6], 1, None, *pools, whole)
            return pools
        else:
            out = torch.zeros(rows, hkv, d, dtype=torch.bfloat16, device="cuda")
            B.ba_qk_norm_rope(c.ctx, None, keys, rows, None, None, None, 0.0, None, out)
            return [out]
        return [o, lse]

    plain = torch.zeros_like(k)
    B.ba_reencode_k(c.ctx, k, None, rows, plain, cu, delta, 2, rows)
    want = read(plain)
    queued = torch.zeros_like(k)
    B.ba_reencode_k_deferred(c.ctx, k, None, rows, queued, cu, delta, 2, rows)
    got = read(queued)
    assert c.device_status() == B.BA_OK
    assert torch.equal(queued, plain)
    for a, b in zip(got, want):
        assert torch.equal(a, b)
    c.close()


# ------------------------------------------------------------------ pages outside the pool, on every path
@pytest.mark.parametrize("questions", [[1, 2], [20, 3], [70, 60]], ids=["few rows", "a query tile", "two query tiles"])
@pytest.mark.parametrize("which", ["own", "prefix"])
@pytest.mark.parametrize("page_rows", [16, 64, 256])
def test_pages_outside_the_pool_count_as_zeros_on_every_path(questions, which, page_rows):
    shape = (4, 2, 64)
    b = Batch(shape, [700], [0, 2], questions, [600, 300], page_rows, False, seed=13)
    c = make_context(shape, b)
    cu, idx = (b.keep if which == "own" else b.keep2)
    pool = b.pool if which == "own" else b.kv_prefix
    n_pages = pool[0].shape[0] // page_rows
    nth = 1                                                    # the second page of the first list
    zeros = [torch.cat([p, torch.zeros_like(p[:page_rows])]) for p in pool]
    for bad in (-1, n_pages, 2 ** 31 - 1):
        wrong = idx.clone()
        wrong[nth] = bad
        table = B.make_page_table(page_rows, n_pages, cu, wrong)
        o, lse = torch.full((b.rows, 4, 64), 5.0, device="cuda"), torch.full((b.rows, 4), 6.0, device="cuda")
        kept = b.table, b.prefix_table, b.pool, b.kv_prefix, b.idx, b.prefix_rows
        if which == "own":
            b.table = table
        else:
            b.prefix_table = table
        b.call(c, o, lse, B.BA_OUT_F32)
        assert c.device_status() == B.BA_ERR_INVALID_ARG
        if which == "own":                                     # the reference reads the page from behind the pool, where zeros are
            b.pool, b.idx = zeros, b.idx.copy()
            b.idx[nth] = n_pages
        else:
            b.kv_prefix = zeros
            b.prefix_rows = [[n_pages * page_rows + t % page_rows if t // page_rows == nth else r for t, r in enumerate(b.prefix_rows[0])]]
        check_attention(b, o, lse, B.BA_OUT_F32, 0.125)
        b.table, b.prefix_table, b.pool, b.kv_prefix, b.idx, b.prefix_rows = kept
    c.close()


# ------------------------------------------------------------------ more work than any launch takes
@pytest.mark.parametrize("rows", [1, 3], ids=["few rows", "many rows"])
@pytest.mark.parametrize("n_seqs,length", [(40, 2 ** 31 - 257), (15, 2 ** 31 - 257), (2, 2 ** 31 - 1)], ids=["past 32 bits", "past the limit", "one too long"])
def test_more_work_than_a_launch_takes_is_reported(rows, n_seqs, length):
    """Lists that are long by their tables alone.  Units are counted in 64 bits: the first sum is 5.4e9, which 32 bits would take for
    1.1e9.  Nothing is looked up in the lists, and nothing is written."""
    shape = (64, 8, 64)
    cfg = B.ba_config(*shape, 0, 1e4, 0.0, 0)
    n = n_seqs * rows
    c = R.Context(*shape, 1e4, max_blocks=64, max_q_rows=64, workspace_bytes=B.ba_shared_prefix_bytes(cfg, n_seqs, 0, n))
    pool = [torch.zeros(65536, 8, 64, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    page_cu, page_idx, own, q_cu = ints(32768 * s for s in range(n_seqs + 1)), ints([0] * 64), ints([length] * n_seqs), ints(range(0, n + 1, rows))
    o, lse = torch.full((n, 64, 64), 5.0, device="cuda"), torch.full((n, 64), 6.0, device="cuda")
    B.ba_shared_prefix_attend(c.ctx, bf16(n, 64, 64, seed=1), n, None, None, 0, None, *pool, B.make_page_table(65536, 1, page_cu, page_idx),
                              B.make_shared_batch(n_seqs, 0, None, None, q_cu, own), o, lse, B.BA_OUT_F32)
    assert c.device_status() == B.BA_ERR_INVALID_ARG
    assert (o == 5).all() and (lse == 6).all()
    c.close()


def test_gradients_fit_the_workspace_that_is_asked_for():
    """The smallest that ba_workspace_bytes() gives, and rows enough for every CTA: sums of both sides at once."""
    for shape in ((32, 8, 128), (64, 1, 64), (1, 1, 128)):
        hq, hkv, d = shape
        rows, cfg = 6000, B.ba_config(*shape, 0, 1e4, 0.0, 0)
        ctx = B.ba_create(cfg, 0, B.ba_workspace_bytes(cfg, 1, 0))
        q, k, dy = bf16(rows, hq, d, seed=1), bf16(rows, hkv, d, seed=2), bf16(rows, hq, d, seed=3)
        w, dw = bf16(d, seed=4), torch.full((2, d), float("nan"), device="cuda")
        B.ba_qk_norm_rope_bwd(ctx, q, k, rows, None, w, w, 1e-6, dy, dy[:, :hkv].contiguous(), torch.empty_like(q), torch.empty_like(k), dw[0], dw[1],
                              B.BA_OUT_BF16)
        assert B.ba_last_device_status(ctx) == B.BA_OK
        for got, x, g in ((dw[0], q, dy), (dw[1], k, dy[:, :hkv])):
            xn = x.double() / torch.sqrt(x.double().square().mean(-1, keepdim=True) + 1e-6)
            want, terms = (g.double() * xn).sum((0, 1)), (g.double() * xn).abs().sum((0, 1))
            assert ((got.double() - want).abs() <= 2e-5 * terms).all()
        B.ba_destroy(ctx)


# ------------------------------------------------------------------ what the documentation allows at its ends
WIDE = {"one token": ([40], [0, 1], [1], [30], 16, False), "one token alone": ([], [0], [1], [300], 16, True),
        "questions": ([500], [0, 2], [3, 1], [140, 5], 64, True), "cut": ([4000], [0, 2], [2, 1], [900, 5], 16, False)}


@pytest.mark.parametrize("shape", [(160, 1, 64), (256, 2, 128), (129, 1, 128), (128, 1, 64), (64, 1, 128), (17, 1, 64), (16, 1, 128)], ids=str)
@pytest.mark.parametrize("name", list(WIDE))
def test_many_query_heads_a_kv_head(shape, name):
    b = Batch(shape, *WIDE[name], seed=21)
    c = make_context(shape, b)
    o, lse = torch.full((b.rows, *shape[::2]), 5.0, device="cuda"), torch.full((b.rows, shape[0]), 6.0, device="cuda")
    b.call(c, o, lse, B.BA_OUT_F32)
    assert c.device_status() == B.BA_OK
    check_attention(b, o, lse, B.BA_OUT_F32, shape[2] ** -0.5)
    c.close()


@pytest.mark.parametrize("name,case", {"most entries": ([3, 0, 40, 7, 130], [0, 9, 700, 701, 1500, 2043], [1] * 2043, [(5 * i) % 23 for i in range(2043)], 16, False),
                                       "a group each": ([(7 * i) % 150 for i in range(500)], list(range(501)), [1 + i % 2 for i in range(500)], [2 + i % 30 for i in range(500)],
                                                        16, True),
                                       "a group each, many rows": ([(37 * i) % 400 for i in range(30)], list(range(31)), [9 + i for i in range(30)], [i * 20 for i in range(30)],
                                                                   32, False)}.items())
def test_as_many_sequences_and_groups_as_there_can_be(name, case):
    shape = (4, 2, 64)
    b = Batch(shape, *case, seed=22)
    c = make_context(shape, b)
    o, lse = torch.full((b.rows, 4, 64), 5.0, device="cuda"), torch.full((b.rows, 4), 6.0, device="cuda")
    b.call(c, o, lse, B.BA_OUT_F32)
    assert c.device_status() == B.BA_OK
    check_attention(b, o, lse, B.BA_OUT_F32, 0.125)
    c.close()


@pytest.mark.parametrize("packed", [True, False])
@pytest.mark.parametrize("questions", [[1, 2, 1, 1], [20, 3, 1, 70]], ids=["few rows", "many rows"])
def test_tables_that_do_not_begin_at_zero(packed, questions):
    """Cumulative tables that are windows of longer ones: query rows in front of the first sequence, prefixes behind others, a first group that begins
    later, lists of pages behind others."""
    shape = (4, 2, 64)
    b = Batch(shape, [200, 77], [1, 2, 4], questions, [90, 30, 5, 140], 16, packed, seed=23)
    c = R.Context(*shape, 1e4, max_blocks=64, max_q_rows=64, workspace_bytes=B.ba_shared_prefix_bytes(B.ba_config(*shape, 0, 1e4, 0.0, 0), 4, 2, b.rows + 5))
    shift = lambda t, n: (t + n).contiguous()
    q = torch.cat([torch.full((5, 4, 64), float("nan"), dtype=torch.bfloat16, device="cuda"), b.q])
    group_cu, prefix_cu, q_cu, own = b.tables
    q_cu = shift(ints(b.q_cu), 5)
    before = torch.full((37, 2, 64), float("nan"), dtype=torch.bfloat16, device="cuda")
    prefix = [torch.cat([before, p]) for p in b.kv_prefix] if packed else b.kv_prefix
    prefix_cu = shift(prefix_cu, 37)
    listed = lambda keep, n: (shift(keep[0], 3), torch.cat([torch.full((3,), n, dtype=torch.int32, device="cuda"), keep[1]]))   # (three pages that are not there)
    own_lists, lists = listed(b.keep, b.n_pages), None if packed else listed(b.keep2, prefix[0].shape[0] // 16)
    o, lse = torch.full((b.rows + 5, 4, 64), 5.0, device="cuda"), torch.full((b.rows + 5, 4), 6.0, device="cuda")
    B.ba_shared_prefix_attend(c.ctx, q, b.rows + 5, *prefix, b.n_prefix + 37, None if packed else B.make_page_table(16, prefix[0].shape[0] // 16, *lists), *b.pool,
                              B.make_page_table(16, b.n_pages, *own_lists), B.make_shared_batch(4, 2, group_cu, prefix_cu, q_cu, own), o, lse, B.BA_OUT_F32)
    assert c.device_status() == B.BA_OK
    assert (o[:5] == 5).all() and (lse[:5] == 6).all()
    check_attention(b, o[5:], lse[5:], B.BA_OUT_F32, 0.125)
    c.close()


def test_append_with_rows_in_front_of_the_first_sequence():
    c = context((4, 2, 64))
    q, k, v = bf16(9, 4, 64, seed=3), bf16(9, 2, 64, seed=1), bf16(9, 2, 64, seed=2)
    pools = [torch.full((64, 2, 64), 9.0, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    q_out, tables = torch.full_like(q, 3.0), (ints([2, 5, 5, 8]), ints([14, 0, 1]), ints([1, 3, 3, 4]), ints([99, 2, 0, 3]))
    B.ba_append_paged(c.ctx, q, k, v, 9, None, None, None, 0.0, *tables[:2], 3, q_out, *pools, B.make_page_table(16, 4, *tables[2:]))
    assert c.device_status() == B.BA_OK
    assert torch.equal(q_out[2:8], q[2:8]) and (q_out[:2] == 3).all() and (q_out[8:] == 3).all()
    at = [32 + 14, 32 + 15, 0, 48 + 1, 48 + 2, 48 + 3]           # (rows 2, 3, 4 of list 0 over its pages 2 and 0; rows 5, 6, 7 of list 2 on page 3)
    for p, x in zip(pools, (k, v)):
        assert torch.equal(p[at], x[2:8])
        p[at] = 9.0
        assert (p == 9).all()
    c.close()


# ------------------------------------------------------------------ outputs in one another's place
def test_outputs_in_the_place_of_others_are_refused():
    """The sides of a call run side by side: an output of one in the place of what the other reads or writes has no defined contents."""
    c = context((4, 4, 64))
    n = 4
    q, k, v, oq, ok, dyq, dyk = (bf16(n, 4, 64, seed=s) for s in range(7))
    w, dw = bf16(64, seed=9), torch.zeros(2, 64, device="cuda")
    pools, start = [torch.zeros(64, 4, 64, dtype=torch.bfloat16, device="cuda") for _ in range(2)], ints([0] * n)
    table, keep = (lambda cu, idx: (B.make_page_table(16, 4, cu, idx), (cu, idx)))(ints(range(n + 1)), ints(range(n)))
    before = c.launches()

    def refused(call):
        with pytest.raises(B.BaError) as e:
            call()
        assert e.value.status == B.BA_ERR_INVALID_ARG
    norm = lambda a, b: lambda: B.ba_qk_norm_rope(c.ctx, q, k, n, None, w, w, 1e-6, a, b)
    for a, b in ((oq, oq), (k, ok), (oq, q), (k, q)):
        refused(norm(a, b))
    bwd = lambda dq, dk, x=dw[0], y=dw[1], kind=B.BA_OUT_BF16: lambda: B.ba_qk_norm_rope_bwd(c.ctx, q, k, n, None, w, w, 1e-6, dyq, dyk, dq, dk, x, y, kind)
    for a, b in ((oq, oq), (dyk, ok), (oq, dyq), (k, ok), (oq, q)):
        refused(bwd(a, b))
    refused(bwd(oq, ok, dw[0], dw[0]))
    wide = torch.zeros(n, 8, 64, dtype=torch.bfloat16, device="cuda")
    refused(lambda: B.ba_qk_norm_rope_bwd(c.ctx, wide[:, :4], None, n, None, w, None, 1e-6, dyq, None, wide.view(2 * n, 4, 64)[:n], None, dw[0], None, B.BA_OUT_BF16))
    refused(lambda: B.ba_qk_norm_rope_bwd(c.ctx, q, None, n, None, w, None, 1e-6, torch.zeros(n, 4, 64, device="cuda"), None, q.data_ptr(), None, dw[0], None,
                                          B.BA_OUT_F32))
    for out in (pools[0], pools[1], k, v):
        refused(lambda: B.ba_append_paged(c.ctx, q, k, v, n, None, None, None, 0.0, None, start, n, out, *pools, table))
    assert c.launches() == before
    # what stays allowed: gradients in the place of the inputs
    norm(oq, ok)()
    bwd(oq, ok)()
    dws = dw.clone()
    x, y = q.clone(), k.clone()
    B.ba_qk_norm_rope_bwd(c.ctx, x, y, n, None, w, w, 1e-6, dyq, dyk, x, y, dw[0], dw[1], B.BA_OUT_BF16)
    assert torch.equal(x, oq) and torch.equal(y, ok) and torch.equal(dw, dws)
    assert c.device_status() == B.BA_OK
    c.close()
