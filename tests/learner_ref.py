"""A learner's operators in 64 bits on the CPU, from their definitions (include/ps_learner.h)."""
import math

import numpy as np
import torch


def kept(rows, cols, p, seed, offset):
    """(0/1 array, factor): Philox4x32-10 numbers by row and column against p."""
    m = np.uint64(0xFFFFFFFF)
    groups = -(-cols // 8)
    c = [np.broadcast_to(np.arange(groups, dtype=np.uint64), (rows, groups)),
         np.broadcast_to(np.arange(rows, dtype=np.uint64)[:, None], (rows, groups)),
         np.full((rows, groups), offset & 0xFFFFFFFF, np.uint64),
         np.full((rows, groups), offset >> 32, np.uint64)]
    k = [seed & 0xFFFFFFFF, seed >> 32]
    for _ in range(10):
        p0, p1 = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        c = [(p1 >> np.uint64(32)) ^ c[1] ^ np.uint64(k[0]), p1 & m,
             (p0 >> np.uint64(32)) ^ c[3] ^ np.uint64(k[1]), p0 & m]
        k = [(k[0] + 0x9E3779B9) & 0xFFFFFFFF, (k[1] + 0xBB67AE85) & 0xFFFFFFFF]
    numbers = np.stack([h for w in c for h in (w & np.uint64(0xFFFF), w >> np.uint64(16))], axis=2)
    d = math.floor(65536 * float(np.float32(p)) + 0.5)
    keep = (numbers.reshape(rows, 8 * groups)[:, :cols] >= d).astype(np.float64)
    return keep, (65536 / (65536 - d) if d < 65536 else 0.0)


def drop(x, d):
    """x (a 64-bit array) with the dropout d (p, seed, offset) or none."""
    if d is None:
        return x
    keep, up = kept(*x.shape, d.p, d.seed, d.offset)
    return np.where(keep > 0, x * up, 0.0)


def f64(t):
    return t.detach().cpu().double().numpy()


def embedding(ids, table, scale, d=None):
    ids, table = ids.cpu().numpy().reshape(-1), f64(table)
    real = (ids >= 0) & (ids < len(table))
    y = np.zeros((len(ids), table.shape[1]))
    y[real] = table[ids[real]] * scale
    y = drop(y, d)
    y[~real] = 0
    return y


def embedding_grad(ids, grad, rows, scale, d=None):
    """(gradient, sums of its terms' magnitudes, terms per row)."""
    ids, g = ids.cpu().numpy().reshape(-1), drop(f64(grad).reshape(-1, grad.shape[-1]), d)
    out, size, count = np.zeros((rows, g.shape[1])), np.zeros((rows, g.shape[1])), np.zeros(rows)
    real = (ids >= 0) & (ids < rows)
    np.add.at(out, ids[real], g[real])
    np.add.at(size, ids[real], abs(g[real]))
    np.add.at(count, ids[real], 1)
    return out * scale, size * abs(scale), count


def quantize(x, square=False):
    """(e4m3 values as 64-bit numbers, exponent of every row and block of 128 columns)."""
    x = f64(x)
    rows, cols = x.shape
    blocks = -(-cols // 128)
    q, e = np.zeros((rows, cols)), np.zeros((rows, blocks), np.int64)
    height = 128 if square else 1
    for b in range(blocks):
        for r in range(0, rows, height):
            tile = x[r:r + height, 128 * b:128 * b + 128]
            most = np.abs(tile[np.isfinite(tile)]).max(initial=0.0)
            ex = -126
            if most > 0:
                f, ex = math.frexp(most / 448)
                ex = max(ex - (f == 0.5), -126)
            e[r:r + height, b] = ex
            v = torch.from_numpy(np.where(np.isfinite(tile), tile, np.nan) * 2.0 ** -ex)
            # e4m3's numbers are 2^-3 of their power of two apart, 2^-9 below 2^-6
            step = torch.exp2((torch.frexp(v)[1] - 4).clamp(min=-9).double())
            q[r:r + height, 128 * b:128 * b + 128] = torch.where(
                torch.isfinite(v), torch.round(v / step) * step, v).numpy()
    return q, e


def values(x, square=False):
    q, e = quantize(x, square)
    return q * 2.0 ** np.repeat(e, 128, axis=1)[:, :q.shape[1]].astype(np.float64)
