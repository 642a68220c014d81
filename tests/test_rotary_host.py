"""Frequencies and their fractions of a turn, on the CPU, and what the oracle of
the rotation is pinned to."""
from decimal import Decimal, getcontext

import numpy as np
import pytest
import torch

from oracle import rotary as R
from paper_2608_26806_amd.rotary import Rotary, rotary_frequencies

getcontext().prec = 60
PI = Decimal("3.14159265358979323846264338327950288419716939937510582097494")


@pytest.mark.parametrize("rot, base", [(16, 10000.0), (64, 500000.0), (128, 1e6)])
def test_turns_are_the_frequencies_fractions(rot, base):
    f = rotary_frequencies(rot, base)[0]
    for freqs in (f, -f, 7 * f, f / 8):
        got = Rotary(rot, freqs, device="cpu").turns.numpy().view(np.uint64)
        for x, t in zip(freqs, got):
            want = Decimal(float(x)) / (2 * PI) % 1 * 2 ** 64
            away = abs(int(t) - want) % 2 ** 64
            # a rounding to whole numbers, and the long double's quotient (2^-64 of up to 1.2 turns)
            assert min(away, 2 ** 64 - away) <= Decimal(2)


def test_turns_at_the_ends():
    # a whole turn and a hair less are no turn; half a turn either way is the same
    got = Rotary(16, [0.0, 2 * np.pi, -1e-300, np.pi, -np.pi, 1e-25, 0.0, 0.0], device="cpu").turns.numpy().view(np.uint64)
    assert got[0] == got[2] == got[5] == 0
    assert min(int(got[1]), 2 ** 64 - int(got[1])) < 2 ** 13       # (2 pi in 64 bits is off by 2.4e-16)
    assert abs(int(got[3]) - 2 ** 63) < 2 ** 13 and abs(int(got[4]) - 2 ** 63) < 2 ** 13


def test_frequencies():
    f, scale = rotary_frequencies(128, 1e4)
    assert scale == 1 and f[0] == 1 and np.isclose(f[63], 1e4 ** (-126 / 128))
    linear, _ = rotary_frequencies(128, 1e4, "linear", factor=4)
    assert np.allclose(linear, f / 4, rtol=1e-15)
    base, _ = rotary_frequencies(128, 1e4, "base", factor=4)
    assert base[0] == 1 and np.isclose(base[-1], f[-1] / 4) and (np.diff(f / base) > 0).all()
    turns = 4096 * f / (2 * np.pi)
    parts, scale = rotary_frequencies(128, 1e4, "parts", factor=4, trained=4096)
    assert np.isclose(scale, 0.1 * np.log(4) + 1)
    wave, one = rotary_frequencies(128, 1e4, "wavelength", factor=4, trained=4096, fast=4, slow=1)
    assert one == 1
    for g, fast in ((parts, 32), (wave, 4)):
        assert np.array_equal(g[turns >= fast * 1.2], f[turns >= fast * 1.2])
        assert np.allclose(g[turns <= 1 / 1.2], f[turns <= 1 / 1.2] / 4, rtol=1e-15)
        assert (np.diff(f / g) >= -1e-12).all()
    mid = (turns > 1) & (turns < 4)
    stay = (turns[mid] - 1) / 3
    assert np.allclose(wave[mid], f[mid] * stay + f[mid] / 4 * (1 - stay))


@pytest.mark.parametrize("kw", [dict(rot_dim=3), dict(rot_dim=2), dict(rot_dim=64, base=0.0), dict(rot_dim=64, factor=0.5),
                                dict(rot_dim=64, stretch="other"), dict(rot_dim=64, stretch="parts", factor=2),
                                dict(rot_dim=64, stretch="wavelength", factor=2, trained=10, fast=1, slow=2)])
def test_frequencies_refused(kw):
    with pytest.raises(ValueError):
        rotary_frequencies(**kw)


@pytest.mark.parametrize("kw", [dict(rot_dim=24), dict(rot_dim=8), dict(rot_dim=64, pairs="other"),
                                dict(rot_dim=64, freqs=[1.0] * 31), dict(rot_dim=32, freqs=[float("nan")] * 16),
                                dict(rot_dim=64, planes=[0] * 31), dict(rot_dim=64, planes=[4] * 32),
                                dict(rot_dim=64, planes=[-1] + [0] * 31)])
def test_rotations_refused(kw):
    with pytest.raises(ValueError):
        Rotary(device="cpu", **kw)


@pytest.mark.parametrize("pairs", ["half", "interleaved"])
def test_oracle(pairs):
    rng = np.random.default_rng(1)
    x = rng.standard_normal((5, 3, 64))
    rotary = Rotary(32, base=1e4, pairs=pairs, device="cpu")
    turns = rotary.turns.numpy().view(np.uint64)
    pos = np.array([[0, 1, 7, -3, 100000]])
    out, _ = R.norm_rotary(x, pos, turns, pairs)
    assert np.array_equal(out[..., 32:], x[..., 32:]) and np.allclose(out[0], x[0], atol=1e-15)
    # as products of complex numbers, from the frequencies themselves
    f = rotary_frequencies(32, 1e4)[0]
    a, b = (x[..., :16], x[..., 16:32]) if pairs == "half" else (x[..., 0:32:2], x[..., 1:32:2])
    z = (a + 1j * b) * np.exp(1j * pos[0][:, None] * f)[:, None]
    u, w = (out[..., :16], out[..., 16:32]) if pairs == "half" else (out[..., 0:32:2], out[..., 1:32:2])
    assert np.allclose(u, z.real, atol=1e-9) and np.allclose(w, z.imag, atol=1e-9)
    # products of turned rows depend on the distance alone
    q, _ = R.norm_rotary(x[:1], np.array([[12345]]), turns, pairs)
    k, _ = R.norm_rotary(x[1:2], np.array([[12300]]), turns, pairs)
    q2, _ = R.norm_rotary(x[:1], np.array([[45]]), turns, pairs)
    assert np.allclose((q * k).sum(-1), (q2 * x[1:2]).sum(-1), atol=1e-9)
    # the norm: torch's, and a scale of the rows makes no difference
    w = rng.standard_normal(64)
    y, _ = R.norm_rotary(x, np.zeros((1, 5), dtype=int), turns, pairs, weight=w, eps=1e-6)
    want = torch.nn.functional.rms_norm(torch.from_numpy(x), (64,), torch.from_numpy(w), eps=1e-6)
    assert np.allclose(y, want.numpy(), atol=1e-12)
