"""Layer norm, host side: configurations, workspace sizes, refusals (no GPU: every call here is refused before a launch)."""
import ctypes as C

import pytest
import torch

from paper_2604_22808_b200 import binding as B
from paper_2604_22808_b200 import build as ffbuild
from paper_2604_22808_b200.configs import LayerNormConfig


@pytest.fixture(scope="module", autouse=True)
def _built():
    ffbuild.build()


@pytest.mark.parametrize("status,cfg", [
    (0, (64, 0, 0, 1e-6)), (0, (1, 1, 1, 1e-30)), (0, (8192, 0, 0, 1.0)), (1, (0, 0, 0, 1e-6)), (1, (-4, 0, 0, 1e-6)), (2, (8193, 0, 0, 1e-6)),
    (1, (64, 2, 0, 1e-6)), (1, (64, 0, 0, 0.0)), (1, (64, 0, 0, -1e-6)), (1, (64, 0, 0, float("nan"))), (1, (64, 0, 0, float("inf"))),
])
def test_configurations(status, cfg):
    lib, c, h = B.library(), B.ff_layer_norm_config_t(*cfg), C.c_void_p()
    assert lib.ff_layer_norm_create(C.byref(c), C.byref(h)) == status
    assert bool(h) == (status == 0)
    if status:
        assert lib.ff_last_error(None)
    lib.ff_layer_norm_destroy(h)


def test_null_arguments():
    lib, n = B.library(), C.c_size_t()
    assert lib.ff_layer_norm_create(None, None) == 1 and lib.ff_layer_norm_destroy(None) == 0
    assert lib.ff_layer_norm_forward(None, 1, 1, None, None, None, 0, None, None) == 1
    assert lib.ff_layer_norm_backward(None, 1, 1, None, None, 0, None, None, None, None, None, 0, None) == 1
    assert lib.ff_layer_norm_workspace_bytes(None, 1, 1, 0, C.byref(n)) == 1


def handle(dim=64, dtype="bf16"):
    return B.LayerNorm(LayerNormConfig(dim, dtype))


def rows(address=4096, batch=640, token=64):
    return C.byref(B.ff_rows_t(address, batch, token))


def test_workspace():
    """Sums of a few blocks for each segment; none where one block has a segment, or there are no rows."""
    lib, h, n = B.library(), handle(), C.c_size_t()

    def size(batch, tokens, per_sample):
        assert lib.ff_layer_norm_workspace_bytes(h.handle, batch, tokens, per_sample, C.byref(n)) == 0
        return n.value
    assert size(0, 5, 0) == size(3, 0, 1) == size(1, 1, 0) == size(9, 1, 1) == 0
    assert size(1, 2, 0) == 2 * 2 * 64 * 4 and size(2, 2, 1) == 2 * size(1, 2, 0)
    assert size(1, 1 << 20, 0) == size(1 << 10, 1 << 10, 0) <= 1 << 20
    assert size(1 << 20, 1 << 10, 1) == 0
    for batch, tokens in ((1 << 16, 1 << 15), (1, 1 << 31), (1 << 40, 1)):
        assert lib.ff_layer_norm_workspace_bytes(h.handle, batch, tokens, 0, C.byref(n)) == 2
    assert lib.ff_layer_norm_workspace_bytes(h.handle, -1, 1, 0, C.byref(n)) == 1
    assert lib.ff_layer_norm_workspace_bytes(h.handle, 1, 1, 0, None) == 1


def test_refused_calls():
    lib, h = B.library(), handle()

    def forward(batch=10, tokens=10, x=rows(), w=4096, b=4096, y=rows()):
        return lib.ff_layer_norm_forward(h.handle, batch, tokens, x, w, b, 0, y, None)

    def backward(x=rows(), w=4096, dy=rows(), dx=rows(), dw=4096, db=4096, ws=4096, n=1 << 30):
        return lib.ff_layer_norm_backward(h.handle, 10, 10, x, w, 0, dy, dx, dw, db, ws, n, None)
    assert forward(batch=-1) == 1 and forward(tokens=-1) == 1
    assert forward(batch=1 << 16, tokens=1 << 15) == 2 and forward(tokens=1 << 40) == 2
    for bad in (None, rows(0), rows(4097), rows(batch=-640), rows(token=-64)):
        assert forward(x=bad) == 1 and forward(y=bad) == 1 and backward(x=bad) == 1 and backward(dy=bad) == 1
        assert lib.ff_layer_norm_last_error(h.handle)
    for bad in (rows(0), rows(4097), rows(batch=0), rows(token=0)):
        assert backward(dx=bad) == 1
    assert forward(y=rows(token=0)) == 1 and forward(y=rows(batch=0)) == 1
    assert forward(w=4098) == 1 and forward(b=4098) == 1 and backward(dw=4098) == 1 and backward(db=4098) == 1
    assert backward(ws=None) == 3 and backward(ws=4100) == 3 and backward(n=16) == 3
    assert forward(batch=0) == 0 and forward(tokens=0) == 0


def test_binding_refuses():
    """Tensors that are not on a GPU, of another shape or type."""
    h = handle()
    x, w = torch.zeros(2, 3, 64, dtype=torch.bfloat16), torch.ones(64)
    with pytest.raises(B.FFError, match="on a GPU"):
        h.forward(x, w, w, x)
    with pytest.raises(B.FFError, match="dtype must be"):
        B.LayerNorm(LayerNormConfig(64, "fp16"))
    fake = type("T", (), {})

    def tensor(shape, dtype=torch.bfloat16, stride=None, device="cuda:0"):
        t = fake()
        t.shape, t.dtype, t.device, t.is_cuda = torch.Size(shape), dtype, torch.device(device), True
        st = stride or tuple(torch.empty(shape, device="meta").stride())
        t.stride, t.dim, t.data_ptr = lambda: st, lambda: len(shape), lambda: 4096
        t.is_contiguous = lambda: st == tuple(torch.empty(shape, device="meta").stride())
        return t
    x = tensor((2, 3, 64))
    for y in (tensor((2, 3, 65)), tensor((2, 3, 64), torch.float32), tensor((2, 3, 64), device="cuda:1"), tensor((2, 3, 64), stride=(384, 128, 2)),
              tensor((3, 64))):
        with pytest.raises(B.FFError):
            h.forward(x, None, None, y)
    for x in (tensor((64,)), tensor((2, 3, 60)), tensor((2, 2, 3, 64)), tensor((2, 3, 64), torch.float32)):
        with pytest.raises(B.FFError):
            h.forward(x, None, None, x)
    x = tensor((2, 3, 64))
    for w in (tensor((64,)), tensor((63,), torch.float32), tensor((3, 64), torch.float32), tensor((64,), torch.float32, device="cuda:1"),
              tensor((2, 64), torch.float32, stride=(1, 2))):
        with pytest.raises(B.FFError, match="weights"):
            h.forward(x, w, None, x)
    with pytest.raises(B.FFError, match="weights"):                # one of the model, one of the samples
        h.forward(x, tensor((64,), torch.float32), tensor((2, 64), torch.float32), x)
