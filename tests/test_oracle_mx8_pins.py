"""The eight-bit oracle (oracle/mx8.py) against known codes, torch's conversions and differences of the forward formula."""
import numpy as np
import pytest

from oracle import mx8 as om

torch = pytest.importorskip("torch")


def test_codes_are_torchs():
    codes = torch.arange(127, dtype=torch.uint8)
    assert (codes.view(torch.float8_e4m3fn).double().numpy() == om.CODES).all()
    assert om.CODES[0x38] == 1.0 and om.CODES[0x7E] == 448.0 and om.CODES[1] == 2.0 ** -9


@pytest.mark.parametrize("C", [1, 31, 32, 33, 100])
def test_rounding_is_torchs(C):
    """The codes are torch's conversions of the scaled values, ties included, and reading gives them back."""
    r = np.random.default_rng(C)
    v = (r.standard_normal((40, C)) * 2.0 ** r.integers(-20, 20, (40, 1))).astype(np.float32).astype(np.float64)
    mid = (om.CODES[:-1] + om.CODES[1:]) / 2
    v[:3] = r.choice(mid, (3, C)) * r.choice([-1.0, 1.0], (3, C))
    v[:3, 0] = 448.0  # the scale 1
    code, scale = om.pack(v)
    blocks = om.blocks(C)
    assert code.shape == (40, 32 * blocks) and scale.shape == (40, blocks)
    s = np.repeat(scale.astype(np.float64) - 127, 32, -1)
    wide = np.zeros(code.shape)
    wide[:, :C] = v
    want = torch.from_numpy((wide / 2.0 ** s).astype(np.float32)).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    assert (code == want).all() and (scale[:3, 0] == 127).all()
    back = om.unpack(code, scale, C)
    assert (np.abs(back - v) <= om.half_step(np.abs(v))).all()
    again = om.pack(back)
    assert (om.unpack(*again, C) == back).all()


def test_scales():
    """The smallest power with which the largest value is at most 448, and its bounds."""
    tops = np.array([448.0, 448.0 * (1 + 2.0 ** -40), 449.0, 224.0, 1.0, 1.75, 1.7500001, 0.0, 2.0 ** -130, 3.4e38, 2.0 ** 127.9])
    v = np.zeros((len(tops), 32))
    v[:, 5] = -tops
    code, scale = om.pack(v)
    assert list(scale.reshape(-1).astype(int) - 127) == [0, 1, 1, -1, -8, -8, -7, -117, -117, 119, 119]
    assert code[0, 5] == 0xFE and code[9, 5] == 0xFE and code[7, 5] == 0x80
    v[0, 7], v[0, 8], v[0, 9] = np.inf, -np.inf, np.nan
    code, scale = om.pack(v)
    assert scale[0, 0] == 127 and (code[0, 7:10] & 127 == 127).all() and code[0, 5] == 0xFE


def test_rms_norm_gradient_by_differences():
    r = np.random.default_rng(0)
    v, g, gamma, up = r.standard_normal((3, 17)), r.standard_normal((3, 17)), r.standard_normal(17), r.standard_normal((3, 17))
    dx, dgamma = om.rms_norm_backward(g, v, gamma, 1e-3, up)
    f = lambda x, ga: (om.rms_norm(x, ga, 1e-3) * g).sum() + (x * up).sum()  # noqa: E731
    e = 1e-6
    for i in np.ndindex(v.shape):
        d = np.zeros_like(v)
        d[i] = e
        assert abs((f(v + d, gamma) - f(v - d, gamma)) / (2 * e) - dx[i]) < 1e-7
    for i in range(17):
        d = np.zeros(17)
        d[i] = e
        assert abs((f(v, gamma + d) - f(v, gamma - d)) / (2 * e) - dgamma[i]) < 1e-7
