"""The oracle's dropout masks for whole matrices at once: Philox 4x32-10 on arrays of 64-bit integers."""
import numpy as np

LOW = np.uint64(0xFFFFFFFF)
HALF = np.uint64(32)


def keep(seed, p, M, n, call=0):
    """What oracle.tuning_oracle.keep gives, in arrays instead of Python's integers."""
    key, number = int(seed[0]) % 2 ** 64, (int(seed[1]) + call) % 2 ** 64
    rows, blocks = np.meshgrid(np.arange(M, dtype=np.uint64), np.arange((n + 7) // 8, dtype=np.uint64), indexing="ij")
    same = lambda v: np.full_like(rows, v)  # noqa: E731
    c = [blocks, rows, same(number & 0xFFFFFFFF), same(number >> 32)]
    k = [key & 0xFFFFFFFF, key >> 32]
    for _ in range(10):
        a, b = np.uint64(0xD2511F53) * c[0], np.uint64(0xCD9E8D57) * c[2]
        c = [(b >> HALF) ^ c[1] ^ np.uint64(k[0]), b & LOW, (a >> HALF) ^ c[3] ^ np.uint64(k[1]), a & LOW]
        k = [(k[0] + 0x9E3779B9) & 0xFFFFFFFF, (k[1] + 0xBB67AE85) & 0xFFFFFFFF]
    numbers = np.stack([w >> np.uint64(s) & np.uint64(0xFFFF) for w in c for s in (0, 16)], axis=-1).reshape(M, -1)[:, :n]
    limit = int(p * 65536.0 + 0.5)
    return numbers >= limit, 1.0 / (1.0 - limit / 65536.0) if limit < 65536 else 0.0
