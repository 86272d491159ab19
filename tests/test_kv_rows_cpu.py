"""Rotary positions without a GPU: turns from radians, scaled positions; calls without a handle; the model of the GPU tests."""
import ctypes
import math
from fractions import Fraction

import numpy as np
import pytest

import paper_2606_17059_gb300 as g

torch = pytest.importorskip("torch")

# 1 / (2 pi) to 80 digits
INVERSE = 1 / (2 * Fraction(314159265358979323846264338327950288419716939937510582097494459230781640628620899862803, 10 ** 86))


def test_turns_are_the_fractions_of_a_turn():
    rng = np.random.default_rng(0)
    f = np.concatenate([[0.0, 1.0, 6.283185307179585, 1e-300, 2.0 ** -60, math.pi], rng.uniform(0, 6.28, 200), np.exp(rng.uniform(-40, 1.8, 200))])
    for x, t in zip(f, g.p2p_kv_rotation_turns(f)):
        want = Fraction(float(x)) * INVERSE * 2 ** 64
        # half a unit for the rounding, and what the two parts of the constant and the product leave out: 2^-100 of the whole
        assert abs(int(t) - want) <= Fraction(3, 4) + want / 2 ** 60, x


def test_radians_that_are_refused():
    lib = g._load()
    for x in (-1e-9, 6.283185307179586, math.inf, math.nan):
        with pytest.raises(g.P2PError) as e:
            g.p2p_kv_rotation_turns([0.5, x])
        assert e.value.code == g.P2P_E_INVAL
    assert lib.p2p_kv_rotation_turns(-1, None, None) == g.P2P_E_INVAL and lib.p2p_kv_rotation_turns(1, None, None) == g.P2P_E_INVAL
    assert lib.p2p_kv_rotation_turns(0, None, None) == g.P2P_OK


def test_scaled_positions():
    plain = g.Rope(64, device="cpu")
    assert np.allclose(plain.radians, 10000.0 ** (-np.arange(32) / 32)) and plain.amplitude == 1.0 and plain.turns.dtype == torch.int64
    assert np.allclose(g.Rope(64, scaling="linear", factor=4.0, device="cpu").radians * 4, plain.radians)
    ntk = g.Rope(64, scaling="ntk", factor=4.0, device="cpu").radians
    assert ntk[0] == 1 and math.isclose(ntk[-1] * 4, plain.radians[-1])
    parts = g.Rope(64, scaling="by_parts", factor=8.0, original=2048, device="cpu").radians
    turns = 2048 * plain.radians / (2 * math.pi)
    for p, f, t in zip(parts, plain.radians, turns):
        keep = min(max((t - 1) / 3, 0), 1)
        assert math.isclose(p, f * keep + f / 8 * (1 - keep))
    yarn = g.Rope(64, scaling="yarn", factor=8.0, original=2048, device="cpu")
    assert np.array_equal(yarn.radians[turns > 64], plain.radians[turns > 64]) and np.allclose(yarn.radians[-3:] * 8, plain.radians[-3:])
    assert np.all(np.diff(yarn.radians) < 0) and math.isclose(yarn.amplitude, 0.1 * math.log(8) + 1)
    assert g.Rope(64, scaling="yarn", factor=8.0, original=2048, amplitude=2.0, device="cpu").amplitude == 2.0
    assert np.array_equal(g.Rope(4, radians=[0.25, 3.0], device="cpu").radians, [0.25, 3.0])
    assert g.Rope(0, device="cpu").turns.numel() == 0


@pytest.mark.parametrize("args", [dict(dim=3), dict(dim=-2), dict(dim=4, scaling="other"), dict(dim=4, theta=1.0), dict(dim=4, scaling="linear", factor=0.5),
                                  dict(dim=2, scaling="ntk", factor=2.0), dict(dim=8, scaling="yarn", factor=2.0), dict(dim=4, radians=[1.0]),
                                  dict(dim=8, scaling="by_parts", factor=2.0, original=100, low=4.0, high=1.0), dict(dim=2, radians=[0.1], scaling="linear"),
                                  dict(dim=4, theta=math.nan)])
def test_positions_that_are_refused(args):
    with pytest.raises(ValueError):
        g.Rope(device="cpu", **args)


def test_calls_without_a_handle():
    lib = g._load()
    r = g.KvRotation()
    for rc in (lib.p2p_kv_write_rotated(None, 0, 1, None, None, 1, ctypes.byref(r), None, 0, 0, 1, None, None, 0, 0, 0, None, 0, 0),
               lib.p2p_kv_attend_prompt(None, 0, 1, None, None, 1, None, 0, 0, 0, 1, 1.0, 0, None, 0, 0, None),
               lib.p2p_kv_attend_shared(None, 0, 1, None, 0, None, 0, None, 0, 0, 0, 1, 1.0, 0, None, 0, 0, None, None)):
        assert rc == g.P2P_E_INVAL
    assert lib.p2p_kv_attend_shared_work(None, 1, 1) == -1


def test_the_model_rotates_as_complex_numbers_do():
    import kv_rows_model as rm
    x = torch.randn((5, 2, 12), dtype=torch.float64)
    pos, f = torch.tensor([0, 1, 7, 1000, 123456]), np.array([1.0, 0.3, 0.01])
    for interleaved in (False, True):
        got, _ = rm.rotated(x, pos, f, 1.5, interleaved)
        z = torch.complex(x[..., 0:6:2], x[..., 1:6:2]) if interleaved else torch.complex(x[..., :3], x[..., 3:6])
        z = z * 1.5 * torch.exp(1j * pos[:, None, None].double() * torch.from_numpy(f))
        want = torch.view_as_real(z).flatten(-2) if interleaved else torch.cat([z.real, z.imag], -1)
        assert torch.allclose(got[..., :6], want) and torch.equal(got[..., 6:], x[..., 6:])
    y, _ = rm.rotated(x, pos, f, 1.0, False, torch.full((12,), 2.0), 0.0)
    assert torch.allclose(y.square().mean(-1), torch.full((5, 2), 4.0, dtype=torch.float64))
