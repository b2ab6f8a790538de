"""What the binding makes of the arguments of the token operators, through the extension and through ctypes.  No device is needed: every call
is refused before the library looks at memory (there is no context)."""
import types

import pytest
import torch

from paper_2409_15355_b200 import binding as B

STREAM = types.SimpleNamespace(cuda_stream=0x5000)
ADDRESS = 0x1000


@pytest.fixture(params=["extension", "ctypes"])
def way(request, monkeypatch):
    B.load_library()
    if request.param == "ctypes":
        monkeypatch.setattr(B, "_marshal", B._CtypesCalls())


def _norm(q=ADDRESS, k=ADDRESS, pos=None):
    B.ba_qk_norm_rope(None, q, k, 4, pos, None, None, 0.0, ADDRESS, ADDRESS, STREAM)


def _norm_bwd(q=ADDRESS, k=ADDRESS, dq=ADDRESS, dk=ADDRESS, pos=None):
    B.ba_qk_norm_rope_bwd(None, q, k, 4, pos, None, None, 0.0, ADDRESS, ADDRESS, dq, dk, None, None, B.BA_OUT_BF16, STREAM)


def _append(q=ADDRESS, k=ADDRESS, v=ADDRESS, pos=None, seq_cu=None, seq_start=ADDRESS):
    B.ba_append_paged(None, q, k, v, 4, pos, None, None, 0.0, seq_cu, seq_start, 4, ADDRESS, 2 * ADDRESS, 3 * ADDRESS,
                      B.ba_page_table(16, 4, ADDRESS, ADDRESS), STREAM)


ROWS = [(_norm, "q"), (_norm, "k"), (_norm_bwd, "q"), (_norm_bwd, "k"), (_norm_bwd, "dq"), (_norm_bwd, "dk"), (_append, "q"), (_append, "k"),
        (_append, "v")]


def _views():
    one, many = torch.zeros(1, 8, 64, dtype=torch.bfloat16), torch.zeros(5, 8, 64, dtype=torch.bfloat16)
    return {"one row for all": one.expand(4, 8, 64), "part of one row for all": one[:, 2:6].expand(4, 4, 64),
            "rows inside one another": many.as_strided((4, 8, 64), (64, 64, 1)), "rows a little short": many.as_strided((4, 8, 64), (504, 64, 1))}


@pytest.mark.parametrize("view", list(_views()))
@pytest.mark.parametrize("call,name", ROWS, ids=lambda v: v if isinstance(v, str) else v.__name__)
def test_views_whose_rows_share_memory_are_refused(way, call, name, view):
    """A row stride of 0 means packed rows: a row that stands for all of them must not become that."""
    with pytest.raises(ValueError, match="lie apart|side by side"):
        call(**{name: _views()[view]})


@pytest.mark.parametrize("call,name", ROWS, ids=lambda v: v if isinstance(v, str) else v.__name__)
def test_packed_rows_and_rows_of_a_fused_projection_reach_the_library(way, call, name):
    whole = torch.zeros(4, 8, 64, dtype=torch.bfloat16)
    for x in (whole, whole[:, 2:6], whole[1:2, 2:3], whole[:1].expand(1, 8, 64)):
        with pytest.raises(B.BaError) as e:
            call(**{name: x})
        assert e.value.status == B.BA_ERR_INVALID_ARG


# ------------------------------------------------------------------ tables
class _OnDevice:
    """What the binding asks of a table on the device."""
    is_cuda = True

    def __init__(self, dtype=torch.int32):
        self.dtype = dtype

    def is_contiguous(self):
        return True

    def data_ptr(self):
        return ADDRESS


TABLES = [(_norm, "pos"), (_norm_bwd, "pos"), (_append, "pos"), (_append, "seq_cu"), (_append, "seq_start")]


@pytest.mark.parametrize("bad", [_OnDevice(torch.int64), _OnDevice(torch.float32), torch.arange(4), torch.arange(4, dtype=torch.int32),
                                 torch.arange(4, dtype=torch.int32).numpy(), [0, 1, 2, 3]], ids=["int64", "float", "host int64", "host int32", "numpy", "list"])
@pytest.mark.parametrize("call,name", TABLES, ids=lambda v: v if isinstance(v, str) else v.__name__)
def test_tables_of_another_type_or_on_the_host_are_refused(way, call, name, bad):
    """An int64 arange, torch's default, would be read as pairs of 32-bit positions, one on the host not at all."""
    with pytest.raises(ValueError, match="int32 tensor"):
        call(**{name: bad})


@pytest.mark.parametrize("call,name", TABLES, ids=lambda v: v if isinstance(v, str) else v.__name__)
def test_tables_on_the_device_and_addresses_reach_the_library(way, call, name):
    for good in (_OnDevice(), ADDRESS, None):
        with pytest.raises(B.BaError) as e:
            call(**{name: good})
        assert e.value.status == B.BA_ERR_INVALID_ARG
