"""fp64 CPU oracle of the 8-bit head: quantisation with a power of two for each
block, products of such operands, the head's forward and backward.

TEST INFRASTRUCTURE ONLY, as ``aal_oracle``: a plain transcription of the
definitions in ``include/aal.h``, sharing no code with the HIP library.  Values
are handled as the numbers they stand for.
"""
from __future__ import annotations

import numpy as np

__all__ = ["FORMATS", "round_to", "quantize", "spread", "product", "magnitude"]

# digits behind the binary point, exponent of the least normal number, largest value, has infinities
FORMATS = {"e4m3": (3, -6, 448.0, False), "e5m2": (2, -14, 57344.0, True)}


def round_to(v: np.ndarray, fmt: str) -> np.ndarray:
    """v (at most the largest value, or not finite) to the format's nearest value, ties to even."""
    digits, least, _, has_inf = FORMATS[fmt]
    v = np.asarray(v, np.float64)
    fine = np.isfinite(v)
    w = np.where(fine, v, 0.0)
    _, e = np.frexp(w)
    step = np.ldexp(1.0, np.maximum(e - 1, least) - digits)
    out = np.rint(w / step) * step
    return np.where(fine, out, v if has_inf else np.nan)


def quantize(x: np.ndarray, fmt: str, block_rows: int):
    """(q [R, C], scale [ceil(R / block_rows), ceil(C / 128)])."""
    x = np.asarray(x, np.float64)
    R, C = x.shape
    scale = np.ones((-(-R // block_rows), -(-C // 128)))
    q = np.empty_like(x)
    for i in range(scale.shape[0]):
        for j in range(scale.shape[1]):
            at = np.s_[i * block_rows:(i + 1) * block_rows, j * 128:(j + 1) * 128]
            b = np.abs(x[at])
            amax = b[np.isfinite(b)].max(initial=0.0)
            if amax > 0:
                e = -126
                while amax > np.ldexp(FORMATS[fmt][2], e):
                    e += 1
                scale[i, j] = np.ldexp(1.0, e)
            q[at] = round_to(x[at] / scale[i, j], fmt)
    return q, scale


def spread(q, scale):
    """The values that q and its scales stand for."""
    q, scale = np.asarray(q, np.float64), np.asarray(scale, np.float64)
    rows = np.arange(q.shape[0]) // (1 if scale.shape[0] == q.shape[0] else 128)
    return q * scale[rows][:, np.arange(q.shape[1]) // 128]


def product(a, a_scale, b, b_scale):
    return spread(a, a_scale) @ spread(b, b_scale).T


def magnitude(a, a_scale, b, b_scale):
    """sum_k |a b| with the scales: what the error of a sum is relative to."""
    return np.abs(spread(a, np.abs(a_scale))) @ np.abs(spread(b, np.abs(b_scale))).T
