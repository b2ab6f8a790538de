"""Pins of the oracle of the operators around the attention calls, and what their calls refuse without a device."""
import math

import numpy as np
import pytest

from oracle import block_attention as ob
from oracle import token_ops as tk
from paper_2409_15355_b200 import binding as B


@pytest.mark.parametrize("layout", [ob.ROPE_ADJACENT, ob.ROPE_HALF])
def test_rotation_is_complex_multiplication(layout):
    rng = np.random.default_rng(1)
    x, pos = rng.standard_normal((5, 2, 8)), [0, 1, -7, 90000, 12]
    y = tk.rotate(x, pos, 1e4, layout)
    for r, p in enumerate(pos):
        for h in range(2):
            for m in range(4):
                i, j = (2 * m, 2 * m + 1) if layout == ob.ROPE_ADJACENT else (m, m + 4)
                z = complex(x[r, h, i], x[r, h, j]) * complex(math.cos(p * 1e4 ** (-m / 4)), math.sin(p * 1e4 ** (-m / 4)))
                assert abs(y[r, h, i] - z.real) < 1e-12 and abs(y[r, h, j] - z.imag) < 1e-12


def test_a_normed_head_has_unit_mean_square():
    x = np.random.default_rng(2).standard_normal((3, 2, 16)) * 7
    assert np.allclose((tk.head_norm(x, 1.0, 0.0) ** 2).mean(-1), 1)
    assert np.allclose((tk.norm_rope(x, [5, 6, 7], 1.0, 0.0, 1e4) ** 2).mean(-1), 1)


@pytest.mark.parametrize("layout", [ob.ROPE_ADJACENT, ob.ROPE_HALF])
@pytest.mark.parametrize("normed", [True, False])
def test_gradients_are_differences(layout, normed):
    rng = np.random.default_rng(3)
    x, dy, pos, eps = rng.standard_normal((3, 2, 8)), rng.standard_normal((3, 2, 8)), [0, 4, 1000], 0.1
    w = rng.standard_normal(8) if normed else None
    loss = lambda x, w: (tk.norm_rope(x, pos, w, eps, 1e4, layout) * dy).sum()
    dx, dw = tk.norm_rope_backward(x, pos, w, eps, 1e4, dy, layout)
    e = 1e-6
    for i in np.ndindex(x.shape):
        up, down = x.copy(), x.copy()
        up[i] += e
        down[i] -= e
        assert abs((loss(up, w) - loss(down, w)) / (2 * e) - dx[i]) < 1e-7
    for i in range(8 if normed else 0):
        up, down = w.copy(), w.copy()
        up[i] += e
        down[i] -= e
        assert abs((loss(x, up) - loss(x, down)) / (2 * e) - dw[i]) < 1e-7


def test_shared_attention_is_the_final_block_of_a_prompt():
    """Prefix and own rows in one list: the last rows of a prompt under the causal mask."""
    rng = np.random.default_rng(4)
    P, n, hq, hkv, d = 9, 4, 4, 2, 8
    k, v, q = rng.standard_normal((P + n, hkv, d)), rng.standard_normal((P + n, hkv, d)), rng.standard_normal((n, hq, d))
    o, lse, _ = tk.shared_attend(q, lambda s: k, lambda s: v, [0, n], [n], lambda s: P, d ** -0.5)
    want, want_lse = ob.final_attend(q, k[P:], v[P:], k[:P], v[:P], [P, n], [2])
    assert np.abs(o - want).max() < 1e-12 and np.abs(lse - want_lse).max() < 1e-12


def test_shared_attention_of_nothing_is_zero():
    q = np.ones((3, 2, 4))
    kv = np.ones((1, 1, 4))
    o, lse, _ = tk.shared_attend(q, lambda s: kv, lambda s: kv, [0, 3], [1], lambda s: 0, 0.5)
    assert (o[:2] == 0).all() and np.isinf(lse[:2]).all() and np.allclose(o[2], 1)


def test_page_rows():
    assert tk.page_rows_of([0, 2, 3], [5, 1, 7], 2, 0, 3) == [10, 11, 2] and tk.page_rows_of([0, 2, 3], [5, 1, 7], 2, 1, 1) == [14]


# ------------------------------------------------------------------ refusals that need no device
def _cfg(**kw):
    c = dict(n_q_heads=4, n_kv_heads=2, head_dim=64, rope_layout=0, rope_theta=1e4, softmax_scale=0.0, reserved=0)
    c.update(kw)
    return B.ba_config(*c.values())


def test_workspace_of_shared_attention():
    small, large = B.ba_shared_prefix_bytes(_cfg(), 1, 0, 1), B.ba_shared_prefix_bytes(_cfg(), 64, 3, 640)
    assert 64 * 1024 < small < large
    for args, status in (((0, 0, 1), B.BA_ERR_INVALID_ARG), ((1, -1, 1), B.BA_ERR_INVALID_ARG), ((1, 0, -1), B.BA_ERR_INVALID_ARG),
                         ((B.BA_SHARED_MAX, 1, 1), B.BA_ERR_UNSUPPORTED)):
        with pytest.raises(B.BaError) as e:
            B.ba_shared_prefix_bytes(_cfg(), *args)
        assert e.value.status == status
    with pytest.raises(B.BaError) as e:
        B.ba_shared_prefix_bytes(_cfg(head_dim=96), 1, 0, 1)
    assert e.value.status == B.BA_ERR_UNSUPPORTED


def _calls_without_a_context(pages):
    shared = B.make_shared_batch(1, 0, None, None, None, 0x1000)
    return {"norm": lambda: B.ba_qk_norm_rope(None, 0x1000, 0x1000, 1, None, None, None, 1e-6, 0x1000, 0x1000, stream=_Stream),
            "norm_bwd": lambda: B.ba_qk_norm_rope_bwd(None, None, None, 1, None, None, None, 1e-6, 0x1000, 0x1000, 0x1000, 0x1000, None, None, 0,
                                                      stream=_Stream),
            "append": lambda: B.ba_append_paged(None, None, 0x1000, 0x1000, 1, None, None, None, 0.0, None, 0x1000, 1, None, 0x2000, 0x3000, pages,
                                                stream=_Stream),
            "shared": lambda: B.ba_shared_prefix_attend(None, 0x1000, 1, None, None, 0, None, 0x1000, 0x1000, pages, shared, 0x1000, None, 0,
                                                        stream=_Stream)}


class _Stream:
    cuda_stream = 0x5000


@pytest.mark.parametrize("name", ["norm", "norm_bwd", "append", "shared"])
def test_calls_without_a_context_are_refused(name):
    with pytest.raises(B.BaError) as e:
        _calls_without_a_context(B.ba_page_table(16, 4, 0x1000, 0x1000))[name]()
    assert e.value.status == B.BA_ERR_INVALID_ARG


@pytest.mark.parametrize("name", ["append", "shared"])
@pytest.mark.parametrize("bad,status", [((8, 4), B.BA_ERR_UNSUPPORTED), ((48, 4), B.BA_ERR_UNSUPPORTED), ((131072, 1), B.BA_ERR_UNSUPPORTED),
                                        ((16, 0), B.BA_ERR_INVALID_ARG), ((65536, 40000), B.BA_ERR_INVALID_ARG)], ids=str)
def test_bad_page_tables_are_refused(name, bad, status):
    with pytest.raises(B.BaError) as e:
        _calls_without_a_context(B.ba_page_table(*bad, 0x1000, 0x1000))[name]()
    assert e.value.status == status


def test_structures_are_not_mixed_up():
    with pytest.raises(Exception):
        B.ba_shared_prefix_attend(None, 0, 1, None, None, 0, None, 0, 0, B.ba_page_table(16, 4, 0, 0), B.ba_page_table(), 0, None, 0, stream=_Stream)
    with pytest.raises(Exception):
        B.ba_shared_prefix_attend(None, 0, 1, None, None, 0, None, 0, 0, None, B.make_shared_batch(1, 0, None, None, None, 0), 0, None, 0,
                                  stream=_Stream)


def test_tables_on_the_host_are_refused():
    import torch
    for bad in (np.zeros(2, dtype=np.int32), torch.zeros(2, dtype=torch.int32), [0, 1]):
        with pytest.raises(ValueError):
            B.make_shared_batch(1, 1, None, bad, None, 0x1000)


def test_views_whose_heads_lie_apart_are_refused():
    import torch
    x = torch.zeros(4, 8, 64, dtype=torch.bfloat16)
    assert B._rows(x[:, 2:6], "q") == (x[:, 2:6].data_ptr(), 512)
    assert B._rows(x, "q") == (x.data_ptr(), 0)
    for bad in (x.transpose(0, 1), x[:, ::2], x[..., :32], x.view(4, 512)[:, ::2]):
        with pytest.raises(ValueError):
            B._rows(bad, "q")


def test_struct_mirror_of_the_shared_batch(tmp_path):
    """As for the library's other structures: field names, order and offsets of the header's."""
    import ctypes as C
    import os
    import re
    import shutil
    import subprocess
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(root, "include", "ba.h")).read(), flags=re.S)
    body = re.search(r"typedef struct \{([^}]*)\} ba_shared_batch;", text).group(1)
    assert re.findall(r"\b([a-z_0-9]+)\s*[,;]", body) == [f for f, _ in B.ba_shared_batch._fields_]
    if shutil.which("gcc") is None:
        pytest.skip("no C compiler")
    lines = ["#include <stdio.h>", "#include <stddef.h>", '#include "ba.h"', "int main(void) {", 'printf("%zu\\n", sizeof(ba_shared_batch));']
    lines += [f'printf("%zu\\n", offsetof(ba_shared_batch, {f}));' for f, _ in B.ba_shared_batch._fields_] + ["return 0; }"]
    (tmp_path / "s.c").write_text("\n".join(lines))
    subprocess.run(["gcc", "-I", os.path.join(root, "include"), str(tmp_path / "s.c"), "-o", str(tmp_path / "s")], check=True)
    got = [int(v) for v in subprocess.run([str(tmp_path / "s")], check=True, capture_output=True, text=True).stdout.split()]
    assert got == [C.sizeof(B.ba_shared_batch)] + [getattr(B.ba_shared_batch, f).offset for f, _ in B.ba_shared_batch._fields_]
