"""The gated block, 8-bit blocks and head layout in 64 bits, from their definitions (numpy and torch on the CPU; no code of the library)."""
import math

import numpy as np
import torch

GATES = ("silu", "gelu", "relu", "sigmoid")          # in the order of us_gate


def gate_value(gate, z):
    if gate == "relu":
        return torch.clamp(z, min=0.0)
    if gate == "gelu":
        return z * torch.special.ndtr(z)
    return torch.sigmoid(z) * (z if gate == "silu" else 1.0)


def gate_slope(gate, z):
    if gate == "relu":
        return (z > 0).double()
    if gate == "gelu":
        return torch.special.ndtr(z) + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    p = torch.sigmoid(z)
    return p * torch.sigmoid(-z) if gate == "sigmoid" else p + z * p * torch.sigmoid(-z)


def keep8(x):
    """[rows, n] float64 -> (codes int8, scales uint8): blocks of 32 of a row, step 2^e, e the smallest of -24 .. 9 with max|x| < 127.5 2^e; the scale is
    e + 127, with 64 more for a block that holds a NaN."""
    x = np.asarray(x, dtype=np.float64)
    rows, n = x.shape
    nb = -(-n // 32)
    b = np.zeros((rows, nb * 32))
    b[:, :n] = x
    b = b.reshape(rows, nb, 32)
    big = np.nanmax(np.where(np.isnan(b), 0.0, np.abs(b)), axis=2)
    e = np.full(big.shape, -24)
    for k in range(-23, 10):
        e = np.where(big >= 127.5 * 2.0 ** (k - 1), k, e)
    with np.errstate(invalid="ignore"):
        q = np.clip(np.rint(b / 2.0 ** e[..., None]), -127, 127)
    q = np.where(np.isnan(b), -128, q).astype(np.int8)
    return q.reshape(rows, nb * 32)[:, :n].copy(), (e + 127 + 64 * np.isnan(b).any(2)).astype(np.uint8)


def keep8_values(codes, scales):
    n = codes.shape[1]
    step = np.repeat(2.0 ** (scales.astype(np.float64) - 127 - 64 * (scales > 136)), 32, axis=1)[:, :n]
    return np.where(codes == -128, np.nan, codes.astype(np.float64) * step)


def fp8_values(codes, e5m2):
    return codes.view(torch.float8_e5m2 if e5m2 else torch.float8_e4m3fn).double()


def turned(x, pos, freq, rot, neighbours, back=False):
    """x [tokens, heads, dh] float64; pos [tokens]; freq [rot / 2] float64."""
    if rot == 0:
        return x
    a = pos.double()[:, None, None] * freq
    c, s = torch.cos(a), torch.sin(a) * (-1 if back else 1)
    y = x.clone()
    i = torch.arange(rot // 2)
    u, v = (2 * i, 2 * i + 1) if neighbours else (i, i + rot // 2)
    y[..., u] = x[..., u] * c - x[..., v] * s
    y[..., v] = x[..., v] * c + x[..., u] * s
    return y
