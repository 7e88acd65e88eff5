"""What the binding of the serving operators makes of its tensors' strides (CPU: the library and the
device are stubs that record the call)."""
import contextlib

import pytest
import torch

from paper_2607_07964_amd import kronq as K

D_IN, D_OUT = 256, 64


class Lib:
    """Records the arguments of the one call."""

    def __init__(self):
        self.args = None

    def kronq_workspace_bytes(self, *a):
        return 256

    kronq_grouped_workspace_bytes = kronq_workspace_bytes

    def _call(self, *a):
        self.args = a
        return 0

    kronq_online_linear = kronq_online_grouped = _call


@pytest.fixture
def lib(monkeypatch):
    stub = Lib()
    monkeypatch.setattr(K, "load", lambda: stub)
    monkeypatch.setattr(K, "_same_device", lambda *ts: torch.device("cpu"))
    monkeypatch.setattr(K, "_guard", lambda dev: contextlib.nullcontext())
    monkeypatch.setattr(K, "_handle", lambda dev: 0)
    return stub


def call(x, y=None, residual=None, grouped=False, d_out=D_OUT):
    w = torch.zeros(d_out, D_IN // 8, dtype=torch.int32)
    s = torch.ones(d_out, D_IN // 128)
    head = (w, s, s, 4, 128, D_IN, None, None, None, None, x)
    if grouped:
        return K.kronq_online_grouped(*head, torch.tensor([0, 1], dtype=torch.int32), y,
                                      residual=residual)
    return K.kronq_online_linear(*head, y, residual=residual)


@pytest.mark.parametrize("grouped", [False, True])
@pytest.mark.parametrize("rows", [1, 2])
def test_rows_need_a_unit_column_stride(lib, rows, grouped):
    """A row of a transposed matrix is no row in memory, however many of them there are."""
    fine = {"x": torch.zeros(rows, D_IN), "y": torch.zeros(rows, D_OUT),
            "residual": torch.zeros(rows, D_OUT)}
    call(**fine, grouped=grouped)
    assert lib.args is not None
    for name, t in fine.items():
        turned = torch.zeros(t.shape[1], 64)[:, :rows].T
        assert turned.shape == t.shape and turned.stride(1) == 64
        lib.args = None
        with pytest.raises(ValueError, match="column stride"):
            call(**{**fine, name: turned}, grouped=grouped)
        assert lib.args is None


def test_strides_of_rows_are_passed_on(lib):
    """Those of several rows; one row may stand anywhere, and so may no row and a single column."""
    x, y, r = (torch.zeros(6, 2 * d)[::2, :d] for d in (D_IN, D_OUT, D_OUT))
    call(x, y, r)
    assert lib.args[16] == 4 * D_IN and lib.args[20:22] == (r.data_ptr(), 4 * D_OUT)
    assert lib.args[24] == 4 * D_OUT
    call(x[:1], y[:1], r[:1])
    assert lib.args[16] >= D_IN and lib.args[16] % 8 == 0
    assert lib.args[21] >= D_OUT and lib.args[24] >= D_OUT
    call(torch.zeros(D_IN, 64).T[:0])
    assert lib.args[17] == 0
    call(x, torch.zeros(8, 3).T[:3, :1], d_out=1)
    assert lib.args[24] == 1
