"""Head norms and rotation written out in 64 bits, and what fp32 arithmetic and one rounding may be off by."""
import numpy as np
import torch

# fp32 between the load and the rounding, in units of 2^-24 of |u| + |v| of a pair: the angle's rounding to 32 bits (2^-26
# turns, 2 pi times that in radians: 1.6), sine and cosine (2 units in the last place: 2), the gain (1), two products and a sum
# (2), and of the norm the mean of up to 128 squares (3 in a lane's 8, 4 across lanes: halved by the root, with its own 2), the
# root's reciprocal (2) and two products (2): under 16.
F32 = 16 * 2.0 ** -24
HALF_STEP = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}


def turned(x, weight, pos, inv_freq, rotary, pairs, gain=1.0, eps=1e-6):
    """Rows x [tokens, heads, D] (64 bits) at positions pos: (result, |u| + |v| of each element's pair)."""
    x = np.asarray(x, np.float64)
    if weight is not None:
        x = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * np.asarray(weight, np.float64)
    angle = np.asarray(pos, np.float64)[:, None] * np.asarray(inv_freq[: rotary // 2], np.float64)
    c, s = gain * np.cos(angle)[:, None, :], gain * np.sin(angle)[:, None, :]
    at = np.arange(rotary // 2)
    first, second = (2 * at, 2 * at + 1) if pairs else (at, at + rotary // 2)
    y, size = x.copy(), np.abs(x)
    u, v = x[..., first], x[..., second]
    y[..., first], y[..., second] = u * c - v * s, v * c + u * s
    size[..., first] = size[..., second] = gain * (np.abs(u) + np.abs(v))
    return y, size


def assert_rounded(got, want, size, dtype, what):
    """Every element of got (a tensor) is the rounding of something fp32 arithmetic makes of want."""
    got = got.double().cpu().numpy()
    off = np.abs(got - want)
    most = HALF_STEP[dtype] * np.abs(want) + (1 + HALF_STEP[dtype]) * F32 * size
    worst = np.max(off - most) if off.size else 0
    assert worst <= 0, f"{what}: {worst:.3g} past its bound at {np.unravel_index(np.argmax(off - most), off.shape)}"
