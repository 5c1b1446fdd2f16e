"""The generator Philox4x32-10 (Salmon et al., 2011) and dropout's mask, from their definitions, in numpy."""
import numpy as np
import torch

LOW, SHIFT = np.uint64(0xFFFFFFFF), np.uint64(32)


def philox(counter, key):
    """Four words from four counter words and two of the key (arrays or numbers)."""
    c, k = [np.asarray(v, dtype=np.uint64) for v in counter], [np.asarray(v, dtype=np.uint64) for v in key]
    for _ in range(10):
        a, b = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        c = [(b >> SHIFT) ^ c[1] ^ k[0], b & LOW, (a >> SHIFT) ^ c[3] ^ k[1], a & LOW]
        k = [(k[0] + np.uint64(0x9E3779B9)) & LOW, (k[1] + np.uint64(0xBB67AE85)) & LOW]
    return c


def kept(rows, d, p, seed, step, layer):
    """Mask [len(rows), d] of elements that dropout keeps."""
    rows = np.asarray(rows, dtype=np.uint64)
    shape = (len(rows), -(-d // 8))
    full = lambda v: np.broadcast_to(np.asarray(v, dtype=np.uint64), shape)  # noqa: E731
    c = philox([full(np.arange(shape[1])[None, :]), full(rows[:, None]), full(step & 0xFFFFFFFF), full(layer)], [seed & 0xFFFFFFFF, seed >> 32 & 0xFFFFFFFF])
    words = np.stack(c, axis=2)
    numbers = np.stack([words & np.uint64(0xFFFF), words >> np.uint64(16)], axis=3).reshape(shape[0], -1)[:, :d]
    return torch.from_numpy(numbers.astype(np.int64) >= round(p * 65536))


def factor(p):
    return float(np.float32(65536 / (65536 - round(p * 65536))))
