"""Cross attention, host side: configurations, workspace sizes, refusals (no GPU)."""
import ctypes as C
from types import SimpleNamespace

import pytest
import torch

from paper_2604_22808_b200 import binding as B
from paper_2604_22808_b200 import build as ffbuild
from paper_2604_22808_b200.configs import CrossAttentionConfig


@pytest.fixture(scope="module", autouse=True)
def _built():
    ffbuild.build()


@pytest.mark.parametrize("status,cfg", [
    (0, (64, 8, 8, 0.0)), (0, (128, 24, 6, 0.1)), (0, (8, 65536, 1, 0.0)), (1, (0, 8, 8, 0.0)), (1, (64, 0, 8, 0.0)), (1, (64, 8, 0, 0.0)),
    (1, (64, 8, 3, 0.0)), (1, (64, 4, 8, 0.0)), (1, (64, 8, 8, -1.0)), (1, (64, 8, 8, float("nan"))), (1, (64, 8, 8, float("inf"))),
    (2, (60, 8, 8, 0.0)), (2, (136, 8, 8, 0.0)), (2, (64, 65537, 1, 0.0)),
])
def test_configurations(status, cfg):
    lib, c = B.library(), B.ff_cross_attention_config_t(*cfg)
    assert lib.ff_cross_attention_validate(C.byref(c)) == status
    n, h = C.c_size_t(), C.c_void_p()
    for training in (0, 1):
        assert lib.ff_cross_attention_workspace_bytes(C.byref(c), 2, 100, 77, training, C.byref(n)) == status
    if status:
        assert lib.ff_cross_attention_create(C.byref(c), C.byref(h)) == status and not h
        assert lib.ff_last_error(None)


def test_null_handles():
    lib, n, c = B.library(), C.c_size_t(), B.ff_cross_attention_config_t(64, 8, 8, 0.0)
    assert lib.ff_cross_attention_validate(None) == 1 and lib.ff_cross_attention_destroy(None) == 0
    assert lib.ff_cross_attention_forward(None, 1, 1, 1, *[None] * 8, 0, None) == 1
    assert lib.ff_cross_attention_backward(None, 1, 1, 1, *[None] * 12, 0, None) == 1
    assert lib.ff_cross_attention_device_status(None, None) == 1
    assert lib.ff_cross_attention_create(C.byref(c), None) == 1
    assert lib.ff_cross_attention_workspace_bytes(C.byref(c), 1, 1, 1, 0, None) == 1


def size(training, batch, queries, keys, cfg=(64, 8, 8, 0.0)):
    lib, n, c = B.library(), C.c_size_t(), B.ff_cross_attention_config_t(*cfg)
    status = lib.ff_cross_attention_workspace_bytes(C.byref(c), batch, queries, keys, training, C.byref(n))
    return n.value if status == 0 else -status


def test_workspace():
    """Nothing for a forward call with many tiles; parts of the keys where tiles are few; D and the parts' sums for a backward call."""
    assert size(0, 4, 65536, 512) == 0 and size(0, 0, 10, 10) == 0 and size(0, 3, 0, 10) == 0 and size(0, 3, 10, 0) == 0
    one = size(0, 1, 1, 32768)
    assert one > 0 and one % (8 * 65 * 4) == 0 and one // (8 * 65 * 4) <= 64
    assert size(1, 4, 65536, 512) >= 4 * 8 * 65536 * 4
    assert size(1, 1, 1, 32768) >= 8 * 4
    for training in (0, 1):
        assert size(training, -1, 1, 1) == size(training, 1, -1, 1) == size(training, 1, 1, -1) == -1
        for sizes in ((1 << 31, 1, 1), (1, 1 << 31, 1), (1, 1, 1 << 31), (1 << 28, 128, 1), (1 << 20, 1 << 20, 1), (1 << 20, 1, 1 << 20), ((1 << 63) - 1, 1, 1)):
            assert size(training, *sizes) == -2, sizes
            assert B.library().ff_last_error(None)


class Fake:
    """The library with the calls of a handle answered here, for the binding's own checks."""

    def __init__(self):
        self.calls = []

    def __getattr__(self, name):
        return lambda *a: self.calls.append((name, a)) or 0


@pytest.fixture
def attention(monkeypatch):
    real = B.library()
    a = object.__new__(B.CrossAttention)
    a.cfg, a._torch, a.handle, a.device = CrossAttentionConfig(64, 8, 2), torch, None, torch.device("cuda:0")
    a._c = B.ff_cross_attention_config_t(64, 8, 2, 0.0)
    a._bf16, a._uint8, a._float32, a._int32, a._mask_types = torch.bfloat16, torch.uint8, torch.float32, torch.int32, (torch.bool, torch.uint8)
    a._lib = SimpleNamespace(ff_cross_attention_forward="forward", ff_cross_attention_backward="backward")
    a.called = []
    a._call = lambda fn, training, size, *args: a.called.append((fn, training, size, args))
    assert real
    return a


def tensor(shape, dtype=torch.bfloat16, stride=None, device="cuda:0"):
    st = stride or tuple(torch.empty(shape, device="meta").stride())
    full = tuple(torch.empty(shape, device="meta").stride())
    return SimpleNamespace(shape=torch.Size(shape), dtype=dtype, device=torch.device(device), is_cuda=True, stride=lambda: st, data_ptr=lambda: 4096,
                           is_contiguous=lambda: st == full)


def test_binding_passes_sizes_and_strides(attention):
    q, k = tensor((3, 8, 5, 64), stride=(5 * 512, 64, 512, 1)), tensor((3, 2, 7, 64), stride=(0, 64, 128, 1))
    attention.forward(q, k, k, q, lengths=tensor((3,), torch.int32), mask=tensor((3, 7), torch.bool))
    (fn, training, sizes, args), = attention.called
    assert fn == "forward" and not training and sizes == (3, 5, 7) and args[3:5] == (4096, 4096) and args[6] is None
    heads = B.ff_heads_t.from_address(args[0])
    # (the array that holds them is alive no longer; its layout is checked with one that is)
    _, at, rows = attention._heads(q, k, k, True, q, False)
    heads = [B.ff_heads_t.from_address(a) for a in at]
    assert [(h.data, h.stride_batch, h.stride_head, h.stride_token, h.heads) for h in heads] == [
        (4096, 2560, 64, 512, 8), (4096, 0, 64, 128, 2), (4096, 0, 64, 128, 2), (4096, 2560, 64, 512, 8)]
    assert C.sizeof(B.ff_heads_t) == 40


def test_binding_refuses(attention):
    q, k = tensor((3, 8, 5, 64)), tensor((3, 2, 7, 64))
    f32 = torch.float32

    def forward(q=q, k=k, v=k, out=q, **kw):
        attention.forward(q, k, v, out, **kw)
    forward(lse=tensor((3, 8, 5), f32))
    for bad in (tensor((3, 8, 5, 32)), tensor((3, 4, 5, 64)), tensor((8, 5, 64)), tensor((3, 8, 5, 64), f32), tensor((3, 8, 5, 64), device="cuda:1"),
                tensor((3, 8, 5, 64), stride=(5120, 640, 128, 2))):
        with pytest.raises(B.FFError):
            forward(q=bad)
        with pytest.raises(B.FFError):
            forward(out=bad)
    for bad in (tensor((2, 2, 7, 64)), tensor((3, 8, 7, 64)), tensor((3, 2, 7, 32)), tensor((3, 2, 7, 64), f32)):
        with pytest.raises(B.FFError):
            forward(k=bad)
    with pytest.raises(B.FFError):
        forward(v=tensor((3, 2, 8, 64)))
    for bad in (tensor((2,), torch.int32), tensor((3,), torch.int64), tensor((3,), torch.int32, device="cuda:1"), tensor((3,), torch.int32, stride=(2,))):
        with pytest.raises(B.FFError, match="lengths"):
            forward(lengths=bad)
    for bad in (tensor((3, 8), torch.bool), tensor((3, 7), f32), tensor((3, 7), torch.bool, stride=(1, 3)), tensor((7,), torch.bool)):
        with pytest.raises(B.FFError, match="mask"):
            forward(mask=bad)
    for bad in (tensor((3, 8, 6), f32), tensor((3, 8, 5)), tensor((3, 5, 8), f32)):
        with pytest.raises(B.FFError, match="lse"):
            forward(lse=bad)
    with pytest.raises(B.FFError):
        attention.backward(q, k, k, q, tensor((3, 8, 5), f32), q, dq=tensor((3, 8, 5, 64), f32))
    with pytest.raises(B.FFError):
        attention.backward(q, k, k, q, tensor((3, 8, 5), f32), q, dk=q, dv=q)
