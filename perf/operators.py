"""Operators around the attention calls, as measurable cases: what a token goes through before and after a prompt is prefilled.

  norm_rope      norms of queries and keys for each head and the position rotation, in one pass (training and prefill)
  norm_rope_bwd  its gradients: of the projections and of the norms' weights
  append         keys and values of new tokens go into a paged cache, the keys normed and rotated on the way; their queries ride along
  shared         attention of a batch whose sequences share long prefixes: a group's prefix is read once for all of its sequences,
                 every sequence goes on with rows of its own in a paged cache

Each case is one pass through one operator.  Projections are N(0, 1) in bf16, weights of the norms lie around one, angles follow
positions of up to a hundred thousand tokens, pages lie in the pool in random order.  The lengths of a case follow from its `lens_seed`.
"""
import math
import random

import torch

own = False

DEVICE = "cuda:0"
EPS = 1e-6
LLAMA = (32, 8, 128)   # attention shape of Llama-3-8B


def _case(name, op, shape, lens_seed, **more):
    c = {"op": op, "q_heads": shape[0], "kv_heads": shape[1], "head_dim": shape[2], "rope": "adjacent", "theta": 5e5, "norm": True,
         "lens_seed": lens_seed}
    c.update(more)
    if name:
        c["name"] = name
    return c


def listed():
    return [
        # a question of 50 tokens behind a prompt of 32K: one layer's projections, queries and keys views of one buffer
        _case("norm_rope_question", "norm_rope", LLAMA, 1, rows=50, pos0=32000, fused=True),
        # a cold batch of eight prompts of 16384 tokens, separate projections, rotary halves
        _case("norm_rope_batch", "norm_rope", LLAMA, 2, rows=131072, pos0=0, fused=False, rope="half"),
        # a small training step of a small model: 2777 tokens, gradients in fp32
        _case("norm_rope_train_small", "norm_rope_bwd", (6, 2, 64), 3, rows=2777, pos0=0, fused=False, out="f32", theta=1e4),
        # a training step of 32768 tokens, bf16 gradients back into one buffer of the fused projection
        _case("norm_rope_train", "norm_rope_bwd", LLAMA, 4, rows=32768, pos0=0, fused=True, out="bf16"),
        # one decode step of 16 requests: one token each, its query, key and value
        _case("append_token", "append", LLAMA, 5, batch=16, lo=1, hi=1, used_lo=50, used_hi=700, pos0=6000, page_rows=16, queries=True),
        # the questions of 24 requests, 37 to 611 tokens, no norms, rotary halves
        _case("append_question", "append", LLAMA, 6, batch=24, lo=37, hi=611, used_lo=0, used_hi=0, pos0=6000, page_rows=64,
              queries=True, norm=False, rope="half"),
        # 64 passages of about 1000 tokens fill a cache (keys and values only)
        _case("append_passages", "append", LLAMA, 7, batch=64, lo=950, hi=1050, used_lo=0, used_hi=0, pos0=0, page_rows=128, queries=False),
        # one request decodes behind ten passages, nothing shared with anybody: all latency
        _case("decode_one", "shared", (4, 2, 64), 8, groups=1, batch=1, prefix_lo=256, prefix_hi=256, own_lo=33, own_hi=33, q_lo=1, q_hi=1,
              page_rows=16, packed_prefix=True, theta=1e4),
        # sixteen requests decode over the same 32 passages of 1000 tokens, each behind a question and an answer of its own
        _case("decode_shared_32k", "shared", LLAMA, 9, groups=1, batch=16, prefix_lo=32000, prefix_hi=32000, own_lo=50, own_hi=500, q_lo=1,
              q_hi=1, page_rows=64, packed_prefix=True),
        # 160 requests in seven groups with system prompts of ragged length, long answers
        _case("decode_groups", "shared", LLAMA, 10, groups=7, batch=160, prefix_lo=300, prefix_hi=6000, own_lo=1, own_hi=2500, q_lo=1, q_hi=1,
              page_rows=16, packed_prefix=False),
        # 64 requests without a common prefix, long caches of their own: the cache is all there is to read
        _case("decode_apart", "shared", LLAMA, 11, groups=0, batch=64, prefix_lo=0, prefix_hi=0, own_lo=1500, own_hi=7000, q_lo=1, q_hi=1,
              page_rows=128, packed_prefix=False),
        # the questions of 24 requests, 17 to 64 tokens, over the same 16384 tokens: many rows a key
        _case("questions_shared_16k", "shared", LLAMA, 12, groups=1, batch=24, prefix_lo=16384, prefix_hi=16384, own_lo=64, own_hi=64, q_lo=17,
              q_hi=64, page_rows=64, packed_prefix=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    shape = rng.choice([LLAMA, (4, 2, 64), (6, 2, 64), (8, 1, 128), (32, 32, 128), (8, 2, 128), (16, 2, 64)])
    op = rng.choice(["norm_rope", "norm_rope_bwd", "append", "shared", "shared"])
    more = {"rope": rng.choice(["adjacent", "half"]), "theta": rng.choice([1e4, 5e5, 1e6]), "norm": rng.random() < 0.8}
    seed = rng.randrange(1 << 20)
    if op in ("norm_rope", "norm_rope_bwd"):
        more.update(rows=_log(rng, 1, 16384 if op == "norm_rope_bwd" else 65536), pos0=rng.choice([0, _log(rng, 1, 100000)]),
                    fused=rng.random() < 0.5)
        if op == "norm_rope_bwd":
            more["out"] = rng.choice(["bf16", "f32"])
        return _case("", op, shape, seed, **more)
    page_rows = rng.choice([16, 32, 64, 128, 256])
    if op == "append":
        batch = _log(rng, 1, 200)
        hi = _log(rng, 1, max(2, 32768 // batch))
        used = rng.choice([0, _log(rng, 1, 2000)])
        more.update(batch=batch, lo=rng.choice([1, hi]), hi=hi, used_lo=used // 3, used_hi=used, pos0=_log(rng, 1, 100000), page_rows=page_rows,
                    queries=rng.random() < 0.7)
        return _case("", op, shape, seed, **more)
    batch = _log(rng, 1, 200)
    groups = min(batch, rng.choice([0, 1, 1, 1, 2, 5, 13]))
    prefix = _log(rng, 1, 24000 if groups == 1 else 6000) if groups else 0
    q = rng.choice([1, 1, 1, _log(rng, 1, max(1, 600 // batch))])
    own_hi = _log(rng, q, max(q + 1, 100000 // batch if batch > 30 else 3000))
    more.update(groups=groups, batch=batch, prefix_lo=prefix if rng.random() < 0.5 else prefix // 4, prefix_hi=prefix,
                own_lo=rng.choice([q, own_hi, own_hi // 4 + q]), own_hi=max(own_hi, own_hi // 4 + q), q_lo=1 if q < 8 else q // 2, q_hi=q,
                page_rows=page_rows, packed_prefix=rng.random() < 0.5)
    return _case("", op, shape, seed, **more)


class _Lengths:
    """The lengths of a case, on the host."""

    def __init__(self, c):
        rng = random.Random(c["lens_seed"])
        between = lambda lo, hi, n: [rng.randint(lo, hi) for _ in range(n)]
        if c["op"] == "append":
            self.rows = between(c["lo"], c["hi"], c["batch"])
            self.used = between(c["used_lo"], c["used_hi"], c["batch"])
        elif c["op"] == "shared":
            b, g = c["batch"], c["groups"]
            self.prefix = between(c["prefix_lo"], c["prefix_hi"], g)
            self.q = between(c["q_lo"], c["q_hi"], b)
            self.own = between(c["own_lo"], c["own_hi"], b)
            cuts = sorted(rng.sample(range(1, b), g - 1)) if g > 1 else []
            self.group_cu = [0] + cuts + [b] if g else [0]
            self.group_of = [next((k for k in range(g) if self.group_cu[k] <= s < self.group_cu[k + 1]), -1) for s in range(b)]

    def sums(self, x):
        out = [0]
        for v in x:
            out.append(out[-1] + v)
        return out


class _State:
    pass


def _normal(gen, *shape):
    """N(0, 1) in bf16, made piece by piece."""
    x = torch.empty(shape, dtype=torch.bfloat16, device=DEVICE)
    flat = x.view(-1)
    for i in range(0, flat.numel(), 1 << 27):
        n = min(1 << 27, flat.numel() - i)
        flat[i:i + n] = torch.randn(n, generator=gen, device=DEVICE)
    return x


def _ints(x):
    return torch.tensor(x, dtype=torch.int32, device=DEVICE)


def _projections(s, c, gen, rows, value=True):
    """Queries, keys and values of `rows` tokens: views of one buffer of the fused projection, or tensors of their own."""
    hq, hkv, d = c["q_heads"], c["kv_heads"], c["head_dim"]
    if c.get("fused", True):
        s.qkv = _normal(gen, rows, hq + 2 * hkv, d)
        s.q, s.k, s.v = s.qkv[:, :hq], s.qkv[:, hq:hq + hkv], s.qkv[:, hq + hkv:]
    else:
        s.q, s.k = _normal(gen, rows, hq, d), _normal(gen, rows, hkv, d)


def _weights(s, c, gen):
    d = c["head_dim"]
    s.w_q = s.w_k = None
    if c["norm"]:
        s.w_q, s.w_k = (1 + 0.1 * torch.randn(2, d, generator=gen, device=DEVICE)).to(torch.bfloat16).unbind(0)
        s.w_q, s.w_k = s.w_q.clone(), s.w_k.clone()


def _pages(gen, lens, page_rows, spare=3):
    """Page lists of sequences with room for `lens` rows each: (cumulative counts, page numbers, pages in the pool)."""
    cu = [0]
    for n in lens:
        cu.append(cu[-1] + -(-n // page_rows))
    total = cu[-1] + spare
    return _ints(cu), torch.randperm(total, generator=gen, device=DEVICE).to(torch.int32)[:max(1, cu[-1])].contiguous(), total


def prepare(case, seed):
    c, s = case, _State()
    gen = torch.Generator(device=DEVICE)
    gen.manual_seed(int(seed) * 7919 + 13)
    hq, hkv, d = c["q_heads"], c["kv_heads"], c["head_dim"]
    s.case, s.lens = c, _Lengths(c)
    _weights(s, c, gen)
    room = 0
    if c["op"] in ("norm_rope", "norm_rope_bwd"):
        rows = c["rows"]
        _projections(s, c, gen, rows)
        s.pos = torch.arange(c["pos0"], c["pos0"] + rows, dtype=torch.int32, device=DEVICE)
        if c["op"] == "norm_rope":
            s.q_out, s.k_out = torch.empty(rows, hq, d, dtype=torch.bfloat16, device=DEVICE), torch.empty(rows, hkv, d, dtype=torch.bfloat16, device=DEVICE)
        else:
            s.kind = torch.float32 if c["out"] == "f32" else torch.bfloat16
            s.dy_q, s.dy_k = _normal(gen, rows, hq, d).to(s.kind), _normal(gen, rows, hkv, d).to(s.kind)
            if c["fused"]:
                s.dqkv = torch.zeros(rows, hq + 2 * hkv, d, dtype=s.kind, device=DEVICE)
                s.dq, s.dk = s.dqkv[:, :hq], s.dqkv[:, hq:hq + hkv]
            else:
                s.dq, s.dk = torch.empty(rows, hq, d, dtype=s.kind, device=DEVICE), torch.empty(rows, hkv, d, dtype=s.kind, device=DEVICE)
            s.dw_q, s.dw_k = (torch.empty(d, device=DEVICE) for _ in range(2)) if c["norm"] else (None, None)
    elif c["op"] == "append":
        L, rows = s.lens, sum(s.lens.rows)
        _projections(s, c, gen, rows)
        s.rows = rows
        s.seq_cu, s.start = _ints(L.sums(L.rows)), _ints(L.used)
        s.page_cu, s.page_idx, s.n_pages = _pages(gen, [u + r for u, r in zip(L.used, L.rows)], c["page_rows"])
        s.pos = _ints([c["pos0"] + u + t for u, r in zip(L.used, L.rows) for t in range(r)])
        s.k_pool, s.v_pool = _normal(gen, s.n_pages * c["page_rows"], hkv, d), _normal(gen, s.n_pages * c["page_rows"], hkv, d)
        s.q_out = torch.empty(rows, hq, d, dtype=torch.bfloat16, device=DEVICE) if c["queries"] else None
    else:
        L, rows = s.lens, sum(s.lens.q)
        s.rows = rows
        s.q = _normal(gen, rows, hq, d)
        s.q_cu = _ints(L.sums(L.q)) if c["q_hi"] > 1 else None
        s.own_len, s.group_cu, s.prefix_cu = _ints(L.own), _ints(L.group_cu), _ints(L.sums(L.prefix))
        s.page_cu, s.page_idx, s.n_pages = _pages(gen, L.own, c["page_rows"])
        s.k_pool, s.v_pool = _normal(gen, s.n_pages * c["page_rows"], hkv, d), _normal(gen, s.n_pages * c["page_rows"], hkv, d)
        s.prefix_rows = sum(L.prefix)
        if c["packed_prefix"]:
            s.k_prefix, s.v_prefix = _normal(gen, max(1, s.prefix_rows), hkv, d), _normal(gen, max(1, s.prefix_rows), hkv, d)
        else:
            s.prefix_page_cu, s.prefix_page_idx, s.prefix_pages = _pages(gen, L.prefix, c["page_rows"])
            s.k_prefix, s.v_prefix = (_normal(gen, s.prefix_pages * c["page_rows"], hkv, d) for _ in range(2))
        s.o = torch.empty(rows, hq, d, dtype=torch.bfloat16, device=DEVICE)
        s.lse = torch.empty(rows, hq, device=DEVICE)
    if own:                                                  # the handle and the tables that a program keeps
        from paper_2409_15355_b200 import binding as B
        layout = B.BA_ROPE_HALF if c["rope"] == "half" else B.BA_ROPE_ADJACENT
        cfg = B.ba_config(hq, hkv, d, layout, float(c["theta"]), 0.0, 0)
        if c["op"] == "shared":
            room = B.ba_shared_prefix_bytes(cfg, c["batch"], c["groups"], s.rows)
            s.shared = B.make_shared_batch(c["batch"], c["groups"], s.group_cu, s.prefix_cu, s.q_cu, s.own_len)
            s.own_table = B.make_page_table(c["page_rows"], s.n_pages, s.page_cu, s.page_idx)
            s.prefix_table = None if c["packed_prefix"] else B.make_page_table(c["page_rows"], s.prefix_pages, s.prefix_page_cu, s.prefix_page_idx)
        if c["op"] == "append":
            s.table = B.make_page_table(c["page_rows"], s.n_pages, s.page_cu, s.page_idx)
        s.context = _context(hq, hkv, d, c["theta"], layout, room)
    return s


def _context(hq, hkv, d, theta, layout, room, kept={}):
    """The library's handle for a configuration.  It knows nothing of the inputs, and a program makes it once: one is kept for every
    configuration, and made anew only where a case needs a larger workspace."""
    from paper_2409_15355_b200 import runtime as R
    key = hq, hkv, d, theta, layout
    if key not in kept or kept[key][0] < room:
        kept[key] = room, R.Context(hq, hkv, d, theta, rope_layout=layout, max_blocks=64, max_q_rows=64, workspace_bytes=room)
    return kept[key][1]


def run(state):
    return (_run_own if own else _run_plain)(state)


# ------------------------------------------------------------------ the calls a user makes
def _run_own(s):
    from paper_2409_15355_b200 import binding as B
    c, ctx = s.case, s.context.ctx
    if c["op"] == "norm_rope":
        B.ba_qk_norm_rope(ctx, s.q, s.k, c["rows"], s.pos, s.w_q, s.w_k, EPS, s.q_out, s.k_out)
        return {"q": s.q_out, "k": s.k_out}
    if c["op"] == "norm_rope_bwd":
        kind = B.BA_OUT_F32 if c["out"] == "f32" else B.BA_OUT_BF16
        B.ba_qk_norm_rope_bwd(ctx, s.q, s.k, c["rows"], s.pos, s.w_q, s.w_k, EPS, s.dy_q, s.dy_k, s.dq, s.dk, s.dw_q, s.dw_k, kind)
        return {"dq": s.dq, "dk": s.dk, "dw_q": s.dw_q, "dw_k": s.dw_k}
    if c["op"] == "append":
        B.ba_append_paged(ctx, s.q if c["queries"] else None, s.k, s.v, s.rows, s.pos, s.w_q, s.w_k, EPS, s.seq_cu, s.start, c["batch"],
                          s.q_out, s.k_pool, s.v_pool, s.table)
        return {"q": s.q_out, "k_pool": s.k_pool, "v_pool": s.v_pool}
    B.ba_shared_prefix_attend(ctx, s.q, s.rows, s.k_prefix, s.v_prefix, s.prefix_rows, s.prefix_table, s.k_pool, s.v_pool, s.own_table,
                              s.shared, s.o, s.lse, B.BA_OUT_BF16)
    return {"o": s.o, "lse": s.lse}


# ------------------------------------------------------------------ the same in elementary operations
def _angles(c, pos):
    """cos and sin of every row's angles, [rows, 1, d / 2]; 64 bits up to the last step, as positions reach a hundred thousand."""
    d = c["head_dim"]
    theta = c["theta"] ** (-torch.arange(0, d, 2, dtype=torch.float64, device=DEVICE) / d)
    a = pos.double()[:, None, None] * theta
    return a.cos().float(), a.sin().float()


def _rotate(c, x, cos, sin):
    if c["rope"] == "half":
        a, b = x.chunk(2, dim=-1)
        return torch.cat([a * cos - b * sin, a * sin + b * cos], dim=-1)
    a, b = x[..., 0::2], x[..., 1::2]
    return torch.stack([a * cos - b * sin, a * sin + b * cos], dim=-1).flatten(-2)


def _norm_rope(c, x, w, cos, sin):
    x = x.float()
    if w is not None:
        x = x * torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS) * w.float()
    return _rotate(c, x, cos, sin)


def _norm_rope_bwd(c, x, w, cos, sin, dy):
    """(dx, dw)"""
    g = _rotate(c, dy.float(), cos, -sin)
    if w is None:
        return g, None
    x = x.float()
    r = torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS)
    h = g * w.float()
    return r * h - x * r.pow(3) * (h * x).mean(-1, keepdim=True), (g * x * r).sum((0, 1))


def _place(page_cu, page_idx, page_rows, of, t):
    """Pool rows of rows `t` of lists `of`."""
    return page_idx.long()[(page_cu.long()[of] + t // page_rows).clamp(max=page_idx.numel() - 1)] * page_rows + t % page_rows


def _run_plain(s):
    c = s.case
    hq, hkv, d = c["q_heads"], c["kv_heads"], c["head_dim"]
    if c["op"] == "shared":
        return _attend_plain(s)
    cos, sin = _angles(c, s.pos)
    if c["op"] == "norm_rope":
        s.q_out.copy_(_norm_rope(c, s.q, s.w_q, cos, sin))
        s.k_out.copy_(_norm_rope(c, s.k, s.w_k, cos, sin))
        return {"q": s.q_out, "k": s.k_out}
    if c["op"] == "norm_rope_bwd":
        dq, dw_q = _norm_rope_bwd(c, s.q, s.w_q, cos, sin, s.dy_q)
        dk, dw_k = _norm_rope_bwd(c, s.k, s.w_k, cos, sin, s.dy_k)
        s.dq.copy_(dq)
        s.dk.copy_(dk)
        return {"dq": s.dq, "dk": s.dk, "dw_q": dw_q, "dw_k": dw_k}
    row = torch.arange(s.rows, device=DEVICE)
    of = torch.searchsorted(s.seq_cu.long(), row, right=True) - 1
    at = _place(s.page_cu, s.page_idx, c["page_rows"], of, s.start.long()[of] + row - s.seq_cu.long()[of])
    s.k_pool[at] = _norm_rope(c, s.k, s.w_k, cos, sin).to(torch.bfloat16)
    s.v_pool[at] = s.v
    if c["queries"]:
        s.q_out.copy_(_norm_rope(c, s.q, s.w_q, cos, sin))
    return {"q": s.q_out, "k_pool": s.k_pool, "v_pool": s.v_pool}


def _attend_plain(s):
    """A group's queries against its prefix, every sequence's against its own rows (both padded to the longest), and one softmax over
    the two."""
    c, L = s.case, s.lens
    hq, hkv, d = c["q_heads"], c["kv_heads"], c["head_dim"]
    heads = hq // hkv
    scale = 1.0 / math.sqrt(d)
    q = s.q.float().view(s.rows, hkv, heads, d)
    q_cu = s.q_cu.long() if s.q_cu is not None else torch.arange(c["batch"] + 1, device=DEVICE)

    # own rows: [batch, longest question] x [batch, longest cache]
    t = torch.arange(max(L.own), device=DEVICE)
    seq = torch.arange(c["batch"], device=DEVICE)[:, None]
    at = _place(s.page_cu, s.page_idx, c["page_rows"], seq, t[None, :].expand(c["batch"], -1))
    k, v = s.k_pool[at].float(), s.v_pool[at].float()
    i = torch.arange(max(L.q), device=DEVICE)
    count = (q_cu[1:] - q_cu[:-1])[:, None]
    row = (q_cu[:-1, None] + i).clamp(max=s.rows - 1)                        # [batch, longest question]
    sees = s.own_len.long()[:, None] - count + 1 + i                         # own rows that it sees
    score = torch.einsum("bihgd,bthd->bihgt", q[row], k) * scale
    score = score.masked_fill((t >= sees[..., None])[:, :, None, None, :], -math.inf)
    here = i < count
    top = score.amax(-1)
    p = (score - top.clamp(min=-1e30)[..., None]).exp()
    o = torch.einsum("bihgt,bthd->bihgd", p, v)[here]                        # [rows, hkv, heads, d]: row order
    den, top = p.sum(-1)[here], top[here]
    del score, p, k, v

    if c["groups"]:
        cu, group_cu = s.prefix_cu.long(), s.group_cu.long()
        t = torch.arange(max(1, max(L.prefix)), device=DEVICE)
        group = torch.arange(c["groups"], device=DEVICE)[:, None]
        t_all = t[None, :].expand(c["groups"], -1)
        if c["packed_prefix"]:
            at = (cu[:-1, None] + t_all).clamp(max=s.k_prefix.shape[0] - 1)
        else:
            at = _place(s.prefix_page_cu, s.prefix_page_idx, c["page_rows"], group, t_all)
        k, v = s.k_prefix[at].float(), s.v_prefix[at].float()
        first, last = q_cu[group_cu[:-1]], q_cu[group_cu[1:]]                # rows of each group
        most = max(sum(L.q[a:b]) for a, b in zip(L.group_cu, L.group_cu[1:]))
        i = torch.arange(most, device=DEVICE)
        row = (first[:, None] + i).clamp(max=s.rows - 1)
        here = i < (last - first)[:, None]
        score = torch.einsum("bihgd,bthd->bihgt", q[row], k) * scale
        score = score.masked_fill((t >= (cu[1:] - cu[:-1])[:, None])[:, None, None, None, :], -math.inf)
        top2 = score.amax(-1)
        p = (score - top2.clamp(min=-1e30)[..., None]).exp()
        o2, den2, top2 = torch.einsum("bihgt,bthd->bihgd", p, v)[here], p.sum(-1)[here], top2[here]
        m = torch.maximum(top, top2)
        safe = m.clamp(min=-1e30)
        a, b = (top - safe).exp(), (top2 - safe).exp()
        o, den, top = o * a[..., None] + o2 * b[..., None], den * a + den2 * b, m
    o = torch.where(den[..., None] > 0, o / den[..., None], 0.0)
    s.o.copy_(o.reshape(s.rows, hq, d))
    s.lse.copy_(torch.where(den > 0, top + den.log(), -math.inf).reshape(s.rows, hq))
    return {"o": s.o, "lse": s.lse}


# ------------------------------------------------------------------ the definition, in 64 bits
def _turned64(c, x, w, pos, back=False):
    """R(pos) of the normed x: complex multiplication by e^{i pos theta} of every pair."""
    d = c["head_dim"]
    x = x.double()
    if w is not None:
        x = w.double() * x / torch.sqrt((x * x).sum(-1, keepdim=True) / d + EPS)
    theta = torch.tensor([c["theta"] ** (-2.0 * m / d) for m in range(d // 2)], dtype=torch.float64, device=DEVICE)
    turn = torch.polar(torch.ones_like(theta), torch.zeros_like(theta))[None, :] * torch.exp(1j * (-1 if back else 1) * pos.double()[:, None] * theta)
    half = c["rope"] == "half"
    z = torch.complex(x[..., :d // 2], x[..., d // 2:]) if half else torch.view_as_complex(x.reshape(*x.shape[:-1], d // 2, 2).contiguous())
    z = z * turn[:, None, :]
    return torch.cat([z.real, z.imag], -1) if half else torch.view_as_real(z).flatten(-2)


def exact(case, seed):
    global own
    was, own = own, False
    s = prepare(case, seed)
    own = was
    c, L = case, s.lens
    hq, hkv, d = c["q_heads"], c["kv_heads"], c["head_dim"]
    pieces = lambda n, step=4096: [slice(i, min(n, i + step)) for i in range(0, n, step)]
    if c["op"] == "norm_rope":
        both = [torch.cat([_turned64(c, x[p], w, s.pos[p]) for p in pieces(c["rows"])]) for x, w in ((s.q, s.w_q), (s.k, s.w_k))]
        return {"q": both[0], "k": both[1]}
    if c["op"] == "norm_rope_bwd":
        out = {}
        for name, x, w, dy in (("q", s.q, s.w_q, s.dy_q), ("k", s.k, s.w_k, s.dy_k)):
            dx, dw = [], torch.zeros(d, dtype=torch.float64, device=DEVICE)
            for p in pieces(c["rows"]):
                g, xx = _turned64(c, dy[p], None, s.pos[p], back=True), x[p].double()
                if w is not None:                                            # y_j = w_j x_j / n, n = sqrt(|x|^2 / d + eps)
                    n = torch.sqrt((xx * xx).sum(-1, keepdim=True) / d + EPS)
                    dw += (g * xx / n).reshape(-1, d).sum(0)
                    wg = w.double() * g
                    g = (wg - xx * ((wg * xx).sum(-1, keepdim=True) / (d * n * n))) / n
                dx.append(g)
            out["d" + name], out["dw_" + name] = torch.cat(dx), dw if w is not None else None
        return out
    if c["op"] == "append":
        k, v = s.k_pool.double(), s.v_pool.double()
        page_cu, page_idx, first = s.page_cu.tolist(), s.page_idx.tolist(), 0
        for q, (used, n) in enumerate(zip(L.used, L.rows)):
            t = torch.arange(used, used + n)
            at = (torch.tensor(page_idx[page_cu[q]:page_cu[q + 1]])[t // c["page_rows"]] * c["page_rows"] + t % c["page_rows"]).to(DEVICE)
            k[at] = _turned64(c, s.k[first:first + n], s.w_k, s.pos[first:first + n])
            v[at] = s.v[first:first + n].double()
            first += n
        return {"q": _turned64(c, s.q, s.w_q, s.pos) if c["queries"] else None, "k_pool": k, "v_pool": v}
    o = torch.zeros(s.rows, hq, d, dtype=torch.float64, device=DEVICE)
    lse = torch.full((s.rows, hq), -math.inf, dtype=torch.float64, device=DEVICE)
    table = lambda cu, idx, k, n: torch.tensor([idx[cu[k] + t // c["page_rows"]] * c["page_rows"] + t % c["page_rows"] for t in range(n)],
                                               dtype=torch.long, device=DEVICE)
    page_cu, page_idx, start = s.page_cu.tolist(), s.page_idx.tolist(), L.sums(L.prefix)
    if L.prefix and not c["packed_prefix"]:
        pcu, pidx = s.prefix_page_cu.tolist(), s.prefix_page_idx.tolist()
    first, held = 0, (-1, None, None)
    for q in range(c["batch"]):
        n, g = L.q[q], L.group_of[q]
        at = table(page_cu, page_idx, q, L.own[q])
        k, v = s.k_pool[at].double().transpose(0, 1), s.v_pool[at].double().transpose(0, 1)          # [hkv, keys, d]
        if g >= 0:
            if held[0] != g:
                at = torch.arange(start[g], start[g + 1], device=DEVICE) if c["packed_prefix"] else table(pcu, pidx, g, L.prefix[g])
                held = (g, s.k_prefix[at].double().transpose(0, 1), s.v_prefix[at].double().transpose(0, 1))
            k, v = torch.cat([held[1], k], 1), torch.cat([held[2], v], 1)
        x = s.q[first:first + n].double().view(n, hkv, hq // hkv, d).permute(1, 2, 0, 3).reshape(hkv, -1, d)     # heads of a group, rows
        z = (x @ k.transpose(1, 2) / math.sqrt(d)).view(hkv, hq // hkv, n, -1)
        ahead = torch.arange(z.shape[-1], device=DEVICE)[None, :] - (z.shape[-1] - n + torch.arange(n, device=DEVICE))[:, None]
        z = z.masked_fill(ahead > 0, -math.inf)                               # the last row sees every key, the one before one fewer
        w = torch.logsumexp(z, -1)
        p = torch.where(w[..., None] > -math.inf, (z - w[..., None]).exp(), 0.0)
        o[first:first + n] = (p.view(hkv, -1, z.shape[-1]) @ v).view(hkv, -1, n, d).permute(2, 0, 1, 3).reshape(n, hq, d)
        lse[first:first + n] = w.permute(2, 0, 1).reshape(n, hq)
        first += n
    return {"o": o, "lse": lse}


def work(case):
    c, L = case, _Lengths(case)
    hq, hkv, d = c["q_heads"], c["kv_heads"], c["head_dim"]
    if c["op"] in ("norm_rope", "norm_rope_bwd"):
        n, wide = c["rows"] * (hq + hkv) * d, 4 if c.get("out") == "f32" else 2
        if c["op"] == "norm_rope":
            return {"bytes": float(4 * n + 4 * c["rows"]), "flops": 8.0 * n}
        return {"bytes": float(((2 if c["norm"] else 0) + 2 * wide) * n + 4 * c["rows"]), "flops": 18.0 * n}
    if c["op"] == "append":
        n = sum(L.rows) * d
        moved = 2 * hkv + (hq if c["queries"] else 0)
        return {"bytes": float(4 * n * moved), "flops": 8.0 * n * (moved - hkv)}
    rows = sum(L.q)
    pairs = 0
    for q, k, g in zip(L.q, L.own, L.group_of):
        pairs += q * (L.prefix[g] if g >= 0 else 0) + sum(max(0, k - i) for i in range(q))
    keys = sum(L.prefix) + sum(L.own)
    return {"bytes": float(4 * keys * hkv * d + rows * hq * (4 * d + 4)), "flops": 4.0 * d * hq * pairs}
