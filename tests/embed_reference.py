"""The embedding operators from their formulas, in numpy and 64 bits (words of the mask in unsigned 64-bit arithmetic)."""
import math

import numpy as np

GOLDEN = 0x9E3779B97F4A7C15
M64 = (1 << 64) - 1


def splitmix_outputs(seed, first, count):
    """Outputs first .. first + count of the SplitMix64 generator that starts at seed."""
    with np.errstate(over="ignore"):
        z = np.uint64(seed & M64) + (np.arange(first, first + count, dtype=np.uint64) + np.uint64(1)) * np.uint64(GOLDEN)
        z = (z ^ (z >> np.uint64(30))) * np.uint64(0xBF58476D1CE4E5B9)
        z = (z ^ (z >> np.uint64(27))) * np.uint64(0x94D049BB133111EB)
        return z ^ (z >> np.uint64(31))


def threshold(p):
    return int(math.floor(p * 65536 + 0.5))


def factor(scale, p):
    t = threshold(p)
    return 0.0 if t == 65536 else scale * 65536 / (65536 - t)


def keep(n, dim, p, seed):
    words = -(-dim // 4)
    draws = splitmix_outputs(seed, 0, n * words).astype("<u8").view("<u2").reshape(n, 4 * words)[:, :dim]
    return draws >= threshold(p)


def embed(slots, rows, scale, p, seed):
    """rows: float64; the result before it is rounded"""
    n, dim = len(slots), rows.shape[1]
    out = np.zeros((n, dim))
    there = slots >= 0
    with np.errstate(invalid="ignore"):
        out[there] = rows[slots[there] % len(rows)] * factor(scale, p)
    if threshold(p):
        out[~keep(n, dim, p, seed)] = 0.0
    return out


def sums(slots, grad, num_rows, scale, p, seed):
    """(rows named, ascending; their sums; the sums of the terms' absolute values; the number of terms), 64 bits"""
    g = grad.astype(np.float64)
    if threshold(p):
        g = np.where(keep(*g.shape, p, seed), g, 0.0)
    there = slots >= 0
    named, at, counts = np.unique(slots[there] % num_rows, return_inverse=True, return_counts=True)
    total, size = np.zeros((len(named), g.shape[1])), np.zeros((len(named), g.shape[1]))
    np.add.at(total, at, g[there])
    np.add.at(size, at, np.abs(g[there]))
    f = factor(scale, p)
    return named, total * f, size * abs(f), counts


def step(rows, state, named, total, lr, eps):
    """rows and state (or None) behind the step, 64 bits"""
    rows = rows.astype(np.float64).copy()
    if state is None:
        rows[named] -= lr * total
        return rows, None
    state = state.astype(np.float64).copy()
    state[named] += np.square(total).mean(1)
    rows[named] -= lr * total / (np.sqrt(state[named]) + eps)[:, None]
    return rows, state
