"""Tensors and bounds that the tests of the residual block's calls share."""
import numpy as np

from oracle import residual_oracle as R

U32 = 2.0 ** -24
HALF_STEP = {"float32": 2.0 ** -24, "float16": 2.0 ** -11, "bfloat16": 2.0 ** -8}
FLOOR = {"float32": 2.0 ** -150, "float16": 2.0 ** -25, "bfloat16": 2.0 ** -134}   # half a step of the smallest numbers


def values(t):
    return t.double().cpu().numpy()


def codes(q):
    """Bytes of a tensor of codes."""
    import torch
    return q.contiguous().view(torch.uint8).cpu().numpy()


def exponents(scale):
    import torch
    return scale.view(torch.uint8).cpu().numpy().astype(np.int64) - 127


def padding(q):
    """The bytes between the last code of each row and the next multiple of 16."""
    import torch
    n = q.shape[-1]
    whole = q.as_strided((*q.shape[:-1], (n + 15) // 16 * 16), q.stride())
    return whole.contiguous().view(torch.uint8)[..., n:].cpu().numpy()


def check_codes(q, scale, y, error=0.0):
    """Codes and scales of rows y [n][cols] (fp64) that the kernel knew up to error * |y|: each code is within half a step of its value."""
    want, e, on = R.quantise_rows(y)
    got = exponents(scale).reshape(e.shape)
    code = codes(q).reshape(want.shape)
    if error == 0.0:
        assert np.array_equal(got, e) and np.array_equal(code, want)
        return
    blocks = np.array([[np.abs(y[r, b * 128:(b + 1) * 128]).max() for b in range(e.shape[1])] for r in range(len(y))]).reshape(e.shape)
    beside = np.abs(blocks / (448.0 * 2.0 ** np.minimum(got, e).astype(float)) - 1) <= error       # a largest value next to where the scale changes
    assert ((got == e) | (beside & (np.abs(got - e) == 1))).all()
    on = y * np.repeat(2.0 ** -got.astype(float), 128, 1)[:, :y.shape[1]]
    size = np.maximum(np.abs(on), 2.0 ** -6)
    half = 2.0 ** (np.floor(np.log2(size)) - 4)
    assert (np.abs(R.decode(code) - on) <= half * (1 + 1e-12) + error * np.abs(on)).all()
