"""The generator that dropout takes its decisions from, written from its definition for the tests: whole numbers of Python and numpy."""
import numpy as np


def words(seed, step, c0, c1, c2, rounds=7):
    """The four 32-bit words [..., 4] of every counter (c0, c1, c2, step); the counters are broadcast against each other."""
    low = np.uint64(0xFFFFFFFF)
    c = [np.asarray(v, dtype=np.uint64) for v in np.broadcast_arrays(c0, c1, c2, step & 0xFFFFFFFF)]
    keys = [seed & 0xFFFFFFFF, (seed >> 32) & 0xFFFFFFFF]
    for r in range(rounds):
        k0, k1 = (np.uint64((k + r * w) & 0xFFFFFFFF) for k, w in zip(keys, (0x9E3779B9, 0xBB67AE85)))
        a, b = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        c = [(b >> np.uint64(32)) ^ c[1] ^ k0, b & low, (a >> np.uint64(32)) ^ c[3] ^ k1, a & low]
    return np.stack(c, -1)


def numbers(seed, step, c0, c1, c2):
    """The eight 16-bit numbers [..., 8] of every counter, as int64."""
    w = words(seed, step, c0, c1, c2).astype(np.int64)
    return np.stack((w & 0xFFFF, w >> 16), -1).reshape(*w.shape[:-1], 8)


def least(p):
    return int(np.floor(p * 65536 + 0.5))


def keep_columns(rng, n, t, dim, p):
    """Truth values [n][t][dim] of dropout."""
    seed, step = (int(v) % 2 ** 64 for v in rng)
    got = numbers(seed, step, np.arange((dim + 7) // 8), np.arange(t)[:, None], np.arange(n)[:, None, None])
    return got.reshape(n, t, -1)[..., :dim] >= least(p)


def keep_pairs(rng, rows, length, p):
    """Truth values [rows][query][key] of attention; rows: numbers of (worker, sequence, head)."""
    seed, step = (int(v) % 2 ** 64 for v in rng)
    key = np.arange(length)
    got = numbers(seed, step, np.arange((length + 15) // 16 * 2), np.arange(length)[:, None], np.asarray(rows)[:, None, None])
    return got[:, :, 2 * (key // 16) + key // 4 % 2, 4 * (key // 8 % 2) + key % 4] >= least(p)
