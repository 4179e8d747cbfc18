"""The oracle of the residual block against independent statements of the same things: torch's e4m3, differences, plain sums."""
import numpy as np
import pytest
import torch

from oracle import block_oracle as K, residual_oracle as R
from tests.residual_util import U32, block_case, check_gradients


def test_codes_are_those_of_e4m3():
    every = np.arange(256, dtype=np.uint8)
    assert np.array_equal(R.decode(every), torch.from_numpy(every).view(torch.float8_e4m3fn).double().numpy(), equal_nan=True)
    rng = np.random.default_rng(0)
    v = np.concatenate([rng.uniform(-448, 448, 20000), rng.standard_normal(20000) * 2.0 ** rng.uniform(-14, 6, 20000), R.MAGNITUDES,
                        (R.MAGNITUDES[1:] + R.MAGNITUDES[:-1]) / 2, [0.0, -0.0, np.nan]]).astype(np.float32)
    v = v[~(np.abs(v) > 448)]
    want = torch.from_numpy(v).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    nan = np.isnan(v)
    assert np.array_equal(R.encode(v)[~nan], want[~nan]) and (R.encode(v)[nan] & 0x7F == 0x7F).all()


@pytest.mark.parametrize("largest,e", [(0.0, -127), (448.0, 0), (np.nextafter(np.float32(448), np.float32(500)), 1), (1.75, -8), (1.76, -7),
                                       (2.0 ** -149, -127), (3.4e38, 120), (896.0, 1), (1e-30, -108)])
def test_exponents(largest, e):
    assert R.exponent(float(largest)) == e
    assert largest <= 448 * 2.0 ** e and (e == -127 or largest > 448 * 2.0 ** (e - 1))


def test_a_block_holds_what_is_not_finite_as_nan():
    x = np.array([[1.0, np.inf, -np.inf, np.nan, -3.0] + [0.0] * 200 + [1e30]])
    q, e, _ = R.quantise_rows(x)
    v = R.values_of_rows(q, e)
    assert v[0, 0] == 1.0 and v[0, 4] == -3.0 and np.isnan(v[0, 1:4]).all() and abs(v[0, -1] / 1e30 - 1) < 2.0 ** -4
    W = np.zeros((1, 130, 129))
    W[0, 129, 128], W[0, 0, 0] = -7.0, 5e-3
    q, e = R.quantise_matrices(W)
    assert np.array_equal(e[0], [[R.exponent(5e-3), -127], [-127, -6]])
    assert R.values_of_matrices(q, e)[0, 129, 128] == -7.0


@pytest.mark.parametrize("lmax", [0, 2])
def test_norm_and_its_adjoint_by_differences(lmax):
    rng = np.random.default_rng(lmax)
    h, dy, dh = (rng.standard_normal((3, (lmax + 1) ** 2, 5)) for _ in range(3))
    gamma = 1 + 0.3 * rng.standard_normal((lmax + 1, 5))
    y = R.rms_norm(h, gamma)
    assert np.allclose(np.sqrt(((y / gamma[np.repeat(np.arange(lmax + 1), 2 * np.arange(lmax + 1) + 1)])[:, :1] ** 2).mean((1, 2))), 1, atol=1e-4)
    dx, dgamma, _, _ = R.rms_norm_backward(h, dy, gamma, dh)
    for _ in range(6):
        u, g, t = rng.standard_normal(h.shape), rng.standard_normal(gamma.shape), 1e-5
        f = lambda s: (R.rms_norm(h + s * u, gamma + s * g) * dy).sum() + ((h + s * u) * dh).sum()
        assert abs((f(t) - f(-t)) / (2 * t) - ((dx * u).sum() + (dgamma * g).sum())) < 1e-7


def test_norm_commutes_with_rotations():
    """Any orthogonal map of the components of a degree."""
    rng = np.random.default_rng(3)
    h, gamma = rng.standard_normal((4, 4, 6)), rng.standard_normal((2, 6))
    Q = np.linalg.qr(rng.standard_normal((3, 3)))[0]
    turn = lambda v: np.concatenate([v[:, :1], np.einsum("ij,njc->nic", Q, v[:, 1:])], 1)
    assert np.allclose(R.rms_norm(turn(h), gamma), turn(R.rms_norm(h, gamma)), atol=1e-13)


def test_products_of_values_of_codes():
    rng = np.random.default_rng(4)
    q, e, _ = R.quantise_rows(rng.standard_normal((7, 140)))
    w, we = R.quantise_matrices(rng.standard_normal((1, 9, 140)))
    y, _ = K.grouped_linear(R.values_of_rows(q, e), R.values_of_matrices(w, we), [0, 7])
    by_block = sum((R.decode(q[:, b:b + 128]) @ R.decode(w[0, :, b:b + 128]).T) * 2.0 ** (e[:, [b // 128]] + we[0, 0, b // 128]) for b in (0, 128))
    assert np.allclose(y, by_block, rtol=1e-14)


def test_clip():
    norm, factor, out = R.clip([np.array([3.0]), np.array([[4.0]])], 1.0)
    assert norm == 5.0 and abs(factor - 0.2) < 1e-7 and abs(out[0][0] - 0.6) < 1e-6
    assert R.clip([np.array([3.0, 4.0])], 10.0)[1] == 1.0
    norm, factor, out = R.clip([np.array([np.inf, 1.0])], 1.0)
    assert factor == 0.0 and out[0][1] == 1.0 and R.clip([np.array([np.nan])], 1.0)[1] == 0.0
    assert R.clip([np.array([2e38, 3e38])], 1.0)[1] == 0.0


MISTAKES = {
    "dx negated": lambda c, dx, dg, dW, dy: (-dx, dg, dW),
    "dgamma negated": lambda c, dx, dg, dW, dy: (dx, -dg, dW),
    "dW negated": lambda c, dx, dg, dW, dy: (dx, dg, -dW),
    "dh left out": lambda c, dx, dg, dW, dy: (dx - c["dh"], dg, dW),
    "noise for dx": lambda c, dx, dg, dW, dy: (np.random.default_rng(1).standard_normal(dx.shape), dg, dW),
    "dW transposed": lambda c, dx, dg, dW, dy: (dx, dg, dW.transpose(0, 2, 1)),
    "dW of another group": lambda c, dx, dg, dW, dy: (dx, dg, dW[::-1]),
    "dW's entries in another order": lambda c, dx, dg, dW, dy: (dx, dg, np.random.default_rng(2).permutation(dW.ravel()).reshape(dW.shape)),
    "no adjoint of the norm": lambda c, dx, dg, dW, dy: (dy + c["dh"], dg, dW),
    "the norm taken for a constant factor": lambda c, dx, dg, dW, dy: (_scaled(c, dy), dg, dW),
    "one degree's dgamma missing": lambda c, dx, dg, dW, dy: (dx, np.concatenate([dg[:-1], 0 * dg[-1:]]), dW),
    "dx a sixteenth too long": lambda c, dx, dg, dW, dy: (dx * (1 + 2.0 ** -4), dg, dW),
}


def _scaled(c, dy):
    """gamma dy / rms + dh: without the term along h."""
    out = c["dh"].copy()
    for l in range(len(c["gamma"])):
        at = slice(l * l, (l + 1) ** 2)
        out[:, at] += dy[:, at] * c["gamma"][l] / np.sqrt((c["h"][:, at] ** 2).mean((1, 2), keepdims=True) + 1e-5)
    return out


@pytest.mark.parametrize("lmax,channels,n,n_species", [(1, 32, 40, 2), (2, 16, 30, 3), (0, 130, 20, 2)])
def test_the_check_of_a_block_s_gradients_notices_mistakes(lmax, channels, n, n_species):
    case, dx, dgamma, dW, dy = block_case(np.random.default_rng(channels), lmax, channels, n, n_species)
    check_gradients(case, dx, dgamma, dW)
    rounded = [v.astype(np.float32).astype(np.float64) for v in (dx, dgamma, dW)]
    check_gradients(case, *rounded, off=64 * U32)
    for name, mistake in MISTAKES.items():
        try:
            check_gradients(case, *mistake(case, dx, dgamma, dW, dy), off=64 * U32)
        except AssertionError:
            continue
        pytest.fail(name)
