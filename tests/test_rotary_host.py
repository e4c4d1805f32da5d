"""Rotary positions, host side: the handle's checks and frequencies (no GPU)."""
import ctypes as C
import math

import numpy as np
import pytest

from paper_2604_22808_b200 import binding as B
from paper_2604_22808_b200 import build as ffbuild
from paper_2604_22808_b200.configs import RotaryConfig


@pytest.fixture(scope="module", autouse=True)
def _built():
    ffbuild.build()


def test_plain_frequencies():
    theta, m = B.Rotary(RotaryConfig(128, 128)).frequencies()
    assert m == 1.0 and np.allclose(theta, 10000.0 ** (-np.arange(64) / 64), rtol=1e-15)


def test_axis_frequencies():
    theta, _ = B.Rotary(RotaryConfig(128, 64, axis_pairs=(8, 14, 10), base=256.0)).frequencies()
    want = np.concatenate([256.0 ** (-np.arange(p) / p) for p in (8, 14, 10)])
    assert np.allclose(theta, want, rtol=1e-15)


def test_scalings():
    plain, _ = B.Rotary(RotaryConfig(64, 64)).frequencies()
    linear, m = B.Rotary(RotaryConfig(64, 64, scaling="linear", factor=4.0)).frequencies()
    assert m == 1.0 and np.allclose(linear, plain / 4, rtol=1e-15)
    ntk, m = B.Rotary(RotaryConfig(64, 64, scaling="ntk", factor=8.0)).frequencies()
    # the fastest pair as it was, the slowest interpolated, all between
    assert m == 1.0 and ntk[0] == 1.0 and math.isclose(ntk[-1], plain[-1] / 8, rel_tol=1e-12)
    assert np.all(ntk <= plain) and np.all(ntk >= plain / 8 * (1 - 1e-12))
    parts, m = B.Rotary(RotaryConfig(64, 64, scaling="by_parts", factor=16.0, original_length=2048)).frequencies()
    turns = 2048 * plain / (2 * math.pi)
    g = np.clip((turns - 1) / 31, 0, 1)
    assert np.allclose(parts, plain * (g + (1 - g) / 16), rtol=1e-14)
    assert parts[0] == plain[0] and math.isclose(parts[-1], plain[-1] / 16, rel_tol=1e-12)
    assert math.isclose(m, 0.1 * math.log(16) + 1, rel_tol=1e-7)
    one, _ = B.Rotary(RotaryConfig(8, 2, scaling="ntk", factor=8.0)).frequencies()      # one pair
    assert one[0] == 1.0


@pytest.mark.parametrize("status,kw", [
    (1, dict(rot_dim=0)), (1, dict(rot_dim=3)), (1, dict(rot_dim=66)), (2, dict(head_dim=12, rot_dim=8)),
    (2, dict(head_dim=264)), (1, dict(dtype="fp16")), (1, dict(layout="other")), (1, dict(scaling="other")),
    (1, dict(base=0.5)), (1, dict(base=math.nan)), (1, dict(base=math.inf)), (1, dict(scaling="linear", factor=0.5)),
    (1, dict(scaling="linear", factor=math.nan)), (1, dict(scaling="by_parts", factor=2.0)),
    (1, dict(axis_pairs=(8, 8, 8))), (1, dict(axis_pairs=(40, -8, 0))), (1, dict(grid=(2, 2, 2))),
    (1, dict(axis_pairs=(8, 12, 12), grid=(2, 0, 2))), (1, dict(axis_pairs=(8, 12, 12), grid=(2, -1, 2))),
    (2, dict(axis_pairs=(8, 12, 12), grid=(1 << 11, 1 << 10, 1 << 10))),
])
def test_refused_configurations(status, kw):
    with pytest.raises(B.FFError) as e:
        B.Rotary(RotaryConfig(**{"head_dim": 64, "rot_dim": 64, **kw}))
    assert e.value.status == status and str(e.value).split(": ", 1)[1]


def _heads(ptr=4096, heads=2, sb=1024, sh=512, st=64):
    return C.byref(B.ff_heads_t(ptr, sb, sh, st, heads))


def test_refused_calls():
    """Everything the host turns down before a launch (addresses are never read)."""
    lib, h = B.library(), B.Rotary(RotaryConfig(64, 64))
    grid = B.Rotary(RotaryConfig(64, 64, axis_pairs=(8, 12, 12), grid=(2, 3, 4)))
    free = B.Rotary(RotaryConfig(64, 64, axis_pairs=(8, 12, 12)))
    inter = B.Rotary(RotaryConfig(64, 64, layout="interleaved"))

    def apply(handle, batch=1, tokens=8, pos=None, ps=0, q=_heads(), k=None, qo=_heads(), ko=None):
        return lib.ff_rotary_apply(handle, batch, tokens, pos, ps, q, k, 0, qo, ko, None)
    assert apply(None) == 1
    assert apply(h.handle, q=None) == 1 and apply(h.handle, qo=None) == 1
    assert apply(h.handle, k=_heads()) == 1 and apply(h.handle, ko=_heads()) == 1
    assert apply(h.handle, batch=-1) == 1 and apply(h.handle, tokens=-1) == 1
    assert apply(h.handle, batch=1 << 20, tokens=1 << 20) == 2
    assert apply(h.handle, q=_heads(ptr=None)) == 1 and apply(h.handle, q=_heads(ptr=4097)) == 1
    assert apply(h.handle, q=_heads(heads=0)) == 1 and apply(h.handle, q=_heads(heads=3)) == 1
    assert apply(h.handle, q=_heads(heads=1 << 20), qo=_heads(heads=1 << 20)) == 2
    assert apply(h.handle, q=_heads(st=-64)) == 1 and apply(h.handle, qo=_heads(st=0)) == 1
    assert apply(h.handle, qo=_heads(sh=0)) == 1 and apply(h.handle, batch=2, qo=_heads(sb=0)) == 1
    assert apply(h.handle, pos=4098) == 1 and apply(h.handle, pos=4096, ps=-8) == 1
    assert apply(grid.handle, tokens=23) == 1 and apply(free.handle) == 1
    assert apply(inter.handle, q=_heads(st=65)) == 2
    assert b"aligned" in lib.ff_rotary_last_error(inter.handle)

    def norm(eps):
        return lib.ff_qk_norm(h.handle, 1, 8, None, 0, _heads(), None, None, None, eps, _heads(), None, None)
    assert [norm(e) for e in (0.0, -1e-6, math.nan, math.inf)] == [1, 1, 1, 1]

    def back(g=_heads(), ws=4096, nbytes=1 << 24):
        return lib.ff_qk_norm_backward(h.handle, 1, 8, None, 0, _heads(), None, None, None, 1e-6, g, None, _heads(), None, None, None,
                                       ws, nbytes, None)
    assert back(g=None) == 1 and back(ws=None) == 3 and back(nbytes=64) == 3 and back(ws=4104) == 3
    assert lib.ff_rotary_create(None, None) == 1 and lib.ff_rotary_destroy(None) == 0
    assert lib.ff_qk_norm_workspace_bytes(None, None) == 1


def test_refused_weight_addresses():
    """Norm weights and their gradients that are not aligned to a float are turned down before a launch would read or write them."""
    lib, h = B.library(), B.Rotary(RotaryConfig(64, 64))

    def norm(wq, wk):
        return lib.ff_qk_norm(h.handle, 1, 8, None, 0, _heads(), _heads(), wq, wk, 1e-6, _heads(), _heads(), None)

    def back(*w):
        return lib.ff_qk_norm_backward(h.handle, 1, 8, None, 0, _heads(), _heads(), *w[:2], 1e-6, _heads(), _heads(), _heads(), _heads(),
                                       *w[2:], 4096, 1 << 24, None)
    for bad in (4097, 4098, 4099):
        assert norm(bad, None) == 1 and norm(4096, bad) == 1
        for i in range(4):
            w = [4096] * 4
            w[i] = bad
            assert back(*w) == 1 and b"aligned" in lib.ff_rotary_last_error(h.handle)


def test_largest_factor():
    """The header's range of the scaling factor includes both ends."""
    for scaling, length in (("linear", 0), ("ntk", 0), ("by_parts", 2048)):
        plain, _ = B.Rotary(RotaryConfig(64, 64)).frequencies()
        theta, _ = B.Rotary(RotaryConfig(64, 64, scaling=scaling, factor=1e9, original_length=length)).frequencies()
        assert math.isclose(theta[-1], plain[-1] / 1e9, rel_tol=1e-12)
        with pytest.raises(B.FFError):
            B.Rotary(RotaryConfig(64, 64, scaling=scaling, factor=math.nextafter(1e9, 2e9), original_length=length))


@pytest.mark.parametrize("dtype,size", (("bf16", 2), ("fp32", 4)))
def test_interleaved_rows_of_odd_alignment(dtype, size):
    """A pair of the interleaved layout moves as one piece: an address or a stride, in use, that is not a multiple of two elements is refused
    in every call, as the header says."""
    lib, h = B.library(), B.Rotary(RotaryConfig(64, 64, dtype, "interleaved"))
    for odd in (_heads(ptr=4096 + size), _heads(st=65), _heads(sh=513)):
        for q, g, y in ((odd, _heads(), _heads()), (_heads(), odd, _heads()), (_heads(), _heads(), odd)):
            assert lib.ff_qk_norm_backward(h.handle, 1, 8, None, 0, q, None, None, None, 1e-6, g, None, y, None, None, None, 4096, 1 << 24, None) == 2
        assert lib.ff_rotary_apply(h.handle, 1, 8, None, 0, odd, None, 0, _heads(), None, None) == 2
        assert lib.ff_qk_norm(h.handle, 1, 8, None, 0, _heads(), odd, None, None, 1e-6, _heads(), _heads(), None) == 2
        assert b"aligned to two elements" in lib.ff_rotary_last_error(h.handle)
    assert lib.ff_rotary_apply(h.handle, 2, 8, None, 0, _heads(sb=1025), None, 0, _heads(), None, None) == 2
