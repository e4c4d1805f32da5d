"""The gated feed-forward block, host side: checks of the configuration and workspace sizes (no GPU)."""
import ctypes as C
from types import SimpleNamespace

import pytest

from paper_2604_22808_b200 import binding as B
from paper_2604_22808_b200 import build as ffbuild


@pytest.fixture(scope="module", autouse=True)
def _built():
    ffbuild.build()


@pytest.mark.parametrize("status,cfg", [
    (0, (64, 128, 0)), (0, (8, 8, 2)), (1, (0, 128, 0)), (1, (64, -8, 0)), (1, (64, 128, 3)), (1, (64, 128, -1)),
    (2, (60, 128, 0)), (2, (64, 129, 0)), (2, (1 << 21, 128, 0)),
])
def test_configurations(status, cfg):
    lib, c = B.library(), B.ff_ffn_config_t(*cfg)
    assert lib.ff_ffn_validate(C.byref(c)) == status
    n, h = C.c_size_t(), C.c_void_p()
    assert lib.ff_ffn_workspace_bytes(C.byref(c), 10, 0, C.byref(n)) == status
    if status:
        assert lib.ff_ffn_create(C.byref(c), C.byref(h)) == status and not h
        assert lib.ff_last_error(None)


def test_workspace():
    lib, c, n = B.library(), B.ff_ffn_config_t(64, 200, 0), C.c_size_t()
    for tokens, training, want in ((0, 0, 0), (1, 0, 512), (10, 0, 4096), (10, 1, 3 * 4096), (1 << 20, 0, 400 << 20)):
        assert lib.ff_ffn_workspace_bytes(C.byref(c), tokens, training, C.byref(n)) == 0 and n.value == want
    assert lib.ff_ffn_workspace_bytes(C.byref(c), -1, 0, C.byref(n)) == 1
    assert lib.ff_ffn_workspace_bytes(C.byref(c), 1, 0, None) == 1


def test_null_handles():
    lib = B.library()
    assert lib.ff_ffn_validate(None) == 1 and lib.ff_ffn_destroy(None) == 0
    assert lib.ff_ffn_forward(None, 1, *[None] * 8, 0, None) == 1
    assert lib.ff_ffn_backward(None, 1, *[None] * 12, 0, None) == 1
    assert lib.ff_ffn_device_status(None, None) == 1
    assert lib.ff_ffn_create(C.byref(B.ff_ffn_config_t(64, 64, 0)), None) == 1


@pytest.mark.parametrize("training", (0, 1))
def test_workspace_of_too_many_tokens(training):
    """More tokens than a call takes: refused as the call refuses them, instead of a size that has left its type."""
    lib, n = B.library(), C.c_size_t()
    for cfg, most in (((8, 8, 0), 0x7fffff00), ((64, 1 << 20, 0), 1 << 18)):
        c = B.ff_ffn_config_t(*cfg)
        assert lib.ff_ffn_workspace_bytes(C.byref(c), most, training, C.byref(n)) == 0 and n.value >= (3 if training else 1) * most * cfg[1] * 2
        for tokens in (most + 1, 1 << 40, (1 << 63) - 1):
            assert lib.ff_ffn_workspace_bytes(C.byref(c), tokens, training, C.byref(n)) == 2
            assert lib.ff_last_error(None)


@pytest.mark.parametrize("current", (0, 1))
def test_status_is_read_on_the_handles_device(monkeypatch, current):
    """device_status names its device's current stream, which may be the default one: 0 on any device.  So the call is made with that device
    current, whichever was before (a fake of torch's device functions and of the library)."""
    at, seen = [current], []

    class Device:
        def __init__(self, device):
            self.index = device.index

        def __enter__(self):
            self.before, at[0] = at[0], self.index

        def __exit__(self, *_):
            at[0] = self.before
    ffn = B.GatedFFN.__new__(B.GatedFFN)
    ffn.device, ffn.handle = SimpleNamespace(index=1), None
    ffn._torch = SimpleNamespace(cuda=SimpleNamespace(device=Device, current_device=lambda: at[0]))
    ffn._raw_stream = lambda index: 0
    monkeypatch.setattr(B, "library", lambda: SimpleNamespace(ff_ffn_device_status=lambda handle, stream: seen.append(at[0]) or 0))
    assert ffn.device_status() == 0 and seen == [1] and at == [current]
