"""The linear layer's calls around the product, from their definitions in 64 bits (numpy, CPU), and how far fp32 arithmetic may be off.

A checkpoint block (32 features of a token, include/bimask.h): e is the smallest exponent with rint(max / 2^e) <= 127, found here by
trying; codes by rint.
"""
import numpy as np
from scipy.special import erfc

ACTS = ("none", "relu", "gelu", "gelu_tanh", "silu")


def act(z, a):
    with np.errstate(over="ignore"):
        return {"none": lambda: z, "relu": lambda: np.maximum(z, 0.0), "gelu": lambda: 0.5 * z * erfc(-z / np.sqrt(2.0)),
                "gelu_tanh": lambda: 0.5 * z * (1.0 + np.tanh(np.sqrt(2.0 / np.pi) * (z + 0.044715 * z ** 3))),
                "silu": lambda: z / (1.0 + np.exp(-z))}[a]()


def slope(z, a):
    with np.errstate(over="ignore"):
        if a == "none":
            return np.ones_like(z)
        if a == "relu":
            return np.where(np.isnan(z), z, (z > 0).astype(np.float64))
        if a == "gelu":
            return 0.5 * erfc(-z / np.sqrt(2.0)) + z * np.exp(-0.5 * z * z) / np.sqrt(2.0 * np.pi)
        if a == "gelu_tanh":
            c = np.sqrt(2.0 / np.pi)
            t = np.tanh(c * (z + 0.044715 * z ** 3))
            return 0.5 * (1.0 + t) + 0.5 * z * (1.0 - t * t) * c * (1.0 + 3 * 0.044715 * z * z)
        s = 1.0 / (1.0 + np.exp(-z))
        return s * (1.0 + z * (1.0 - s))


def function_error(z, a):
    """Relative error of act, and of either term of its slope, in fp32 arithmetic.  An exponential of an argument u that took three
    roundings is off by 3 |u| 2^-24, for gelu u = z^2 / 2, for the others u <= 1.6 |z| + 0.072 |z|^3; the other operations (2^x and 1/x to
    2^-22 each, ten products and sums, the tail's fit 1.5e-7 < 2^-22) stay below 2^-19 together."""
    if a in ("none", "relu"):
        return np.zeros_like(z)
    u = 0.5 * z * z if a == "gelu" else 1.6 * np.abs(z) + (0.072 * np.abs(z) ** 3 if a == "gelu_tanh" else 0.0)
    return 2.0 ** -19 + 3.0 * np.minimum(u, 120.0) * 2.0 ** -24


def coarse_gelu(z, a):
    """What bf16 results leave out of gelu on purpose, absolute: 2.5e-4 of the tail |z| Q(|z|) (2^-8 of it below Q = 2e-8), within 2.6e-4."""
    q = 0.5 * erfc(np.abs(z) / np.sqrt(2.0))
    return np.abs(z) * q * np.where(q > 2e-8, 2.6e-4, 1.0) if a == "gelu" else np.zeros_like(z)


def slope_error(z, a):
    """Absolute error of the slope: both of its terms, which may cancel, to function_error."""
    if a in ("none", "relu"):
        return np.zeros_like(z)
    return function_error(z, a) * (np.abs(act(z, a)) / np.maximum(np.abs(z), 1e-30) + np.abs(z) * 0.81 * np.exp(-np.abs(z)) + 1e-30)


def store(x):
    """(codes int8 [T, Cp], scale bytes [T, Cp/32]) of a float64 matrix."""
    T, C = x.shape
    b = np.zeros((T, -(-C // 32) * 32))
    b[:, :C] = x
    b = b.reshape(T, -1, 32)
    most = np.abs(b).max(axis=-1)
    bad = ~np.isfinite(most)
    e = np.full(most.shape, 121.0)
    for k in range(120, -127, -1):
        with np.errstate(invalid="ignore", over="ignore"):
            e = np.where(np.rint(most * 2.0 ** -k) <= 127, k, e)
    with np.errstate(invalid="ignore"):
        q = np.clip(np.rint(b * 2.0 ** -e[..., None]), -127, 127)
    q = np.where(bad[..., None], 0, q)
    return q.astype(np.int8).reshape(T, -1), np.where(bad, 255, e + 127).astype(np.uint8)


def load(codes, scales, C):
    T = codes.shape[0]
    s = np.where(scales == 255, np.nan, 2.0 ** (scales.astype(np.float64) - 127))
    return (codes.reshape(T, -1, 32).astype(np.float64) * s[..., None]).reshape(T, -1)[:, :C]


def split(buf, T, C):
    """A checkpoint's bytes as (codes, scale bytes)."""
    Cp = -(-C // 32) * 32
    return buf[:T * Cp].view(np.int8).reshape(T, Cp), buf[T * Cp:T * Cp + T * (Cp // 32)].reshape(T, Cp // 32)


def join(codes, scales):
    return np.concatenate([codes.view(np.uint8).reshape(-1), scales.reshape(-1)])
