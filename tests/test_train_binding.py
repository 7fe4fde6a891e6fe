"""The training operators' workspace sizes at their largest, and the binding's checks.
No GPU is needed."""
import pytest
import torch

import paper_2010_07565_amd as bg
from paper_2010_07565_amd import _lib


def test_workspace_of_the_norm_gradients():
    """Up to 1536 columns no more than 8 KB a column, however many rows there are; wider
    rows leave a set of sums every 64 of them, and no more than one a row."""
    most = (1 << 31) - 1
    for cols in (1, 3, 64, 256, 602, 1433, 1536):
        sizes = [bg.layernorm_backward_workspace_bytes(rows, cols) for rows in
                 (1, 1000, 20000, 1000000, 20000000, most)]
        assert all(0 < s <= 8192 * cols + 256 for s in sizes), (cols, sizes)
        assert sizes == sorted(sizes)
    for cols in (1537, 2048, 4096, 8192):
        for rows in (1, 100, 1000, 20000, 1000000, most):
            sets = min(rows, rows // 64 + 1536)
            assert 0 < bg.layernorm_backward_workspace_bytes(rows, cols) <= sets * 2 * cols * 4 + 256
    assert bg.layernorm_backward_workspace_bytes(0, 64) == 0
    assert bg.layernorm_backward_workspace_bytes(most + 1, 8192) == 0    # (refused)


N, NNZ, D_IN, D_OUT = 50, 200, 100, 16


def packed_arguments():
    return dict(rowptr=torch.zeros(N + 1, dtype=torch.int64),
                colidx=torch.zeros(NNZ, dtype=torch.int32),
                hbits=torch.zeros(N, 2, dtype=torch.int64), hscale=torch.zeros(N),
                wt=torch.zeros(D_OUT, D_IN), wbits=torch.zeros(D_OUT, 2, dtype=torch.int64),
                alpha=torch.zeros(D_OUT), gout=torch.zeros(N, D_OUT), dwt=torch.zeros(D_OUT, D_IN),
                workspace=torch.zeros(1 << 20, dtype=torch.uint8),
                slot=torch.zeros(N, dtype=torch.int32), colslot=torch.zeros(NNZ, dtype=torch.int32))


@pytest.mark.parametrize("name,short", [
    ("wbits", torch.zeros(D_OUT - 1, 2, dtype=torch.int64)),
    ("wbits", torch.zeros(D_OUT, 1, dtype=torch.int64)),
    ("alpha", torch.zeros(D_OUT - 1)), ("alpha", torch.zeros(2 * D_OUT)[::2]),
    ("alpha", torch.zeros(1, D_OUT)),
    ("slot", torch.zeros(N - 1, dtype=torch.int32)),
    ("colslot", torch.zeros(NNZ - 1, dtype=torch.int32)),
    ("colidx", torch.zeros(2 * NNZ, dtype=torch.int32)[::2]),
    ("rowptr", torch.zeros(2 * N + 2, dtype=torch.int64)[::2]),
    ("hbits", torch.zeros(N, 1, dtype=torch.int64)), ("hscale", torch.zeros(N - 1)),
    ("nnz", NNZ + 1)])
def test_packed_backward_refuses_short_arguments(name, short):
    """By name, before anything is asked of the device."""
    args = packed_arguments()
    with pytest.raises(ValueError, match="rowptr must be a device tensor"):
        bg.bigcn_layer_backward_packed(**args)         # all of them right, and on the host
    args[name] = short
    with pytest.raises(ValueError, match="colidx" if name == "nnz" else name) as e:
        bg.bigcn_layer_backward_packed(**args)
    assert "device tensor" not in str(e.value)


def test_current_stream_without_the_private_functions(monkeypatch):
    """Calls without a stream take torch's current one by its public interface where a torch
    has no other."""
    class Stream:
        cuda_stream = 77

    monkeypatch.setattr(torch.cuda, "current_stream", lambda: Stream())
    for name in ("_cuda_getCurrentRawStream", "_cuda_getDevice"):
        with monkeypatch.context() as m:
            m.setattr(torch._C, "_cuda_getDevice", lambda: 0)
            m.setattr(torch._C, "_cuda_getCurrentRawStream", lambda device: 55)
            assert _lib._stream(None) == 55
            m.delattr(torch._C, name)
            assert _lib._stream(None) == 77
    assert _lib._stream(Stream()) == 77 and _lib._stream(9) == 9


def test_more_columns_than_32_bits_count():
    """Refused: the columns' low 32 bits (70 here) are not what was asked for."""
    x = torch.zeros(1, 1).expand(1, (1 << 32) + 70)
    v = torch.zeros(1)
    for call in (lambda: bg.bigcn_checkpoint_q8(x, None, None), lambda: bg.bigcn_restore_q8(None, None, x),
                 lambda: bg.bigcn_layernorm(x, y=x), lambda: bg.bigcn_layernorm_backward(x, v, v, x=x, dx=x),
                 lambda: bg.bigcn_softmax_xent(x, v.int(), loss=v)):
        with pytest.raises(ValueError, match="columns"):
            call()
