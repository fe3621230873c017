"""The dropout stream in whole numbers, apart from the library: SplitMix64 on a counter, 16 bits an element."""
import numpy as np
import torch

GAMMA = 0x9E3779B97F4A7C15
ALL = (1 << 64) - 1


def _mix(x):
    x ^= x >> np.uint64(30)
    x *= np.uint64(0xBF58476D1CE4E5B9)
    x ^= x >> np.uint64(27)
    x *= np.uint64(0x94D049BB133111EB)
    x ^= x >> np.uint64(31)
    return x


def _mix_one(x):
    with np.errstate(over="ignore"):
        return int(_mix(np.array([x & ALL], dtype=np.uint64))[0])


def kept(k, rows, n, p, seed, step):
    """(bool [k][rows][n], factor): what survives, and what it is multiplied by."""
    limit = int((1.0 - p) * 65536 + 0.5)
    groups = (n + 3) // 4
    out = np.empty((k, rows, 4 * groups), dtype=bool)
    with np.errstate(over="ignore"):
        at = np.arange(1, rows * groups + 1, dtype=np.uint64) * np.uint64(GAMMA)
        for w in range(k):
            key = _mix_one(_mix_one(seed + GAMMA * (w + 1)) + GAMMA * (step + 1))
            u = _mix(at + np.uint64(key))
            bits = np.stack([(u >> np.uint64(16 * q)) & np.uint64(0xFFFF) for q in range(4)], -1)
            out[w] = (bits < limit).reshape(rows, 4 * groups)
    return torch.from_numpy(out[..., :n].copy()), (65536.0 / limit if limit else 0.0)
