"""Inputs of the 8-bit operators' tests, shared by the CPU and GPU ones."""
import numpy as np

import gen
from oracle import i8


def weight(seed, name, rows, cols):
    return i8.quantize(gen.normal(seed, name, (rows, cols), cols ** -0.5))


def tokens(seed, name, N, cols, act):
    """About normal, every 50th channel six times as large."""
    x = gen.normal(seed, name, (N, cols))
    x[:, ::50] *= 6
    return gen.to_act(x, act)


def padded(codes):
    """Codes in rows of a multiple of 128 bytes, zeros at the end."""
    rows, cols = codes.shape
    out = np.zeros((rows, (cols + 127) // 128 * 128), np.int8)
    out[:, :cols] = codes
    return out


def experts(seed, d, f, E):
    """Wg, Wu, Wd as (codes [E, rows, cols], scale [E, rows])."""
    out = []
    for name, r, c in (("Wg", f, d), ("Wu", f, d), ("Wd", d, f)):
        q, s = weight(seed, name, E * r, c)
        out.append((q.reshape(E, r, c), s.reshape(E, r)))
    return out


def routing(seed, N, E, k, choice="random"):
    """random top-k sets; null; or a list of row counts, one expert after another (k 1)."""
    z = gen.normal(seed, "z", (N, E + 1)).astype(np.float64)
    if choice == "random":
        eidx = np.sort(np.argsort(-z, axis=1, kind="stable")[:, :k], axis=1)
    elif choice == "null":
        eidx = np.zeros((N, k), np.int64)
    else:
        eidx = np.repeat(np.arange(len(choice)), choice).reshape(N, 1)
    p = np.take_along_axis(np.exp(z), eidx, axis=1)
    return eidx.astype(np.int32), (p / p.sum(axis=1, keepdims=True)).astype(np.float32)


def awkward_rows(act):
    """Rows whose codes are hard: exact borders, zeros, the smallest and largest
    magnitudes, and rows that are not finite."""
    half = np.arange(-64, 64, dtype=np.float32) + 0.5     # with a = 127: every border
    rows = [np.concatenate([[127.0], half[1:]]), np.concatenate([[254.0], 2 * half[1:]]),
            np.concatenate([[-127.0 * 2 ** -20], half[1:] * 2 ** -20]), np.zeros(128),
            np.where(np.arange(128) == 5, 1.0, 0.0), np.linspace(-1, 1, 128),
            1e-38 * np.linspace(-1, 1, 128), 2.0 ** -133 * np.arange(128),
            3e38 * np.linspace(-1, 1, 128), 2.0 ** -126 * half, np.full(128, -2.5),
            np.where(np.arange(128) == 7, np.nan, 1.0), np.where(np.arange(128) == 9, np.inf, 1.0),
            np.where(np.arange(128) == 127, -np.inf, 0.0), 0.0 * half]
    return gen.to_act(np.stack(rows).astype(np.float32), act)
