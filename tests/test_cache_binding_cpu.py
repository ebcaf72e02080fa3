"""What the binding of the position, cache and cached-attention calls refuses before the
library is asked: no device needed."""
import pytest
import torch

from paper_2301_08658_amd import binding as B

HERE = -1                   # the "device" of tensors on the CPU


def test_workspaces_are_runs_of_bytes():
    """A strided or broadcast view's number of bytes is not what lies behind its pointer."""
    ws = torch.zeros(64, dtype=torch.uint8)
    assert B._bytes(ws, HERE) == (ws.data_ptr(), 64)
    assert B._bytes(ws[16:48].view(2, 16), HERE) == (ws.data_ptr() + 16, 32)
    assert B._bytes(None, HERE) == (None, 0)
    for bad in (ws[::2], ws.view(8, 8)[:, :4], ws[:1].expand(1 << 20), ws.view(8, 8).t()):
        with pytest.raises(ValueError, match="contiguous"):
            B._bytes(bad, HERE)
