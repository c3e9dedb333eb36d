"""AdamW as include/ps_learner.h defines it: m and v step by step in fp32 and what 8 bits keep of them to the bit,
the step in 64 bits."""
import numpy as np

F = np.float32


def random_words(count, t, seed):
    """Word j & 3 of Philox4x32-7 of the counter (j >> 2, t) and the key `seed`, for j below `count`."""
    mask = np.uint64(0xFFFFFFFF)
    j = np.arange(-(-count // 4), dtype=np.uint64)
    c = [j & mask, j >> np.uint64(32), np.full_like(j, t & 0xFFFFFFFF), np.full_like(j, t >> 32)]
    k = [seed & 0xFFFFFFFF, seed >> 32]
    for _ in range(7):
        p0, p1 = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        c = [(p1 >> np.uint64(32)) ^ c[1] ^ np.uint64(k[0]), p1 & mask, (p0 >> np.uint64(32)) ^ c[3] ^ np.uint64(k[1]),
             p0 & mask]
        k = [(k[0] + 0x9E3779B9) & 0xFFFFFFFF, (k[1] + 0xBB67AE85) & 0xFFFFFFFF]
    return np.stack(c, axis=1).reshape(-1)[:count].astype(np.int64)


def encode(x, r, signed):
    """(codes, bytes) of a multiple of 128 fp32 numbers, from the definition with 64-bit numbers."""
    b = x.reshape(-1, 128)
    r = r.reshape(-1, 128)
    codes, scales = np.zeros(b.shape, np.uint8), np.zeros(len(b), np.uint8)
    for i, row in enumerate(b):
        most = F(abs(row).max())
        if not np.isfinite(row).all() or most > 1.875 * 2.0 ** 127:
            scales[i] = 255
            continue
        bits = int(most.view(np.int32))
        s = (bits >> 23) + ((bits & 0x7FFFFF) > 0x700000)
        scales[i] = s
        with np.errstate(under="ignore"):
            scaled = (abs(row).astype(np.float64) * 2.0 ** ((15 if signed else 31) - s)).astype(F)
        code = (scaled.view(np.int32).astype(np.int64) + 16 * r[i]) >> 20
        if signed:
            assert (code < 128).all()
            code = code | (np.signbit(row).astype(np.int64) << 7)
        else:
            code = np.maximum(code, row > 0)
        codes[i] = code
    return codes.reshape(-1), scales


def decode(codes, scales, signed):
    c = codes.reshape(-1, 128).astype(np.int64)
    value = ((c & (127 if signed else 255)) << 20).astype(np.int32).view(F).astype(np.float64)
    with np.errstate(under="ignore"):
        value = (value * 2.0 ** (scales.astype(np.float64) - (15 if signed else 31))[:, None]).astype(F)
    value = np.where(scales[:, None] == 255, F(np.nan), value)
    return (np.where(c > 127, -value, value) if signed else value).reshape(-1)


class Reference:
    """The optimizer of one list of tensors; weights and gradients are given at each step as 64-bit arrays."""

    def __init__(self, sizes, decay, betas, eps, bits, seed):
        self.sizes, self.decay, self.betas, self.eps, self.bits, self.seed = sizes, decay, betas, eps, bits, seed
        self.at, room = [], 0
        for n in sizes:
            self.at.append(room)
            room += -(-n // 128) * 128
        self.room, self.t = room, 0
        self.m, self.v = np.zeros(room, F), np.zeros(room, F)
        if bits == 8:
            self.m, self.v = np.zeros(room, np.uint8), np.zeros(room, np.uint8)
            self.ms, self.vs = np.zeros(room // 128, np.uint8), np.zeros(room // 128, np.uint8)

    def step(self, weights, grads, lr, factor=1.0):
        """(step, tolerance) for each tensor. Of the step in fp32: two products, a root, a sum and a division of
        the first part, each 2^-24 and 2 for root and division, its factors rounded too; the decay's product and
        the sum's: 12 * 2^-24 of the parts' magnitudes."""
        self.t += 1
        b1, b2 = self.betas
        if self.bits == 8:
            m, v = decode(self.m, self.ms, True), decode(self.v, self.vs, False)
        else:
            m, v = self.m, self.v
        out = []
        with np.errstate(all="ignore"):
            for i, (w, g) in enumerate(zip(weights, grads)):
                s = slice(self.at[i], self.at[i] + self.sizes[i])
                g = g.astype(F) * F(factor)
                m[s] = F(b1) * m[s] + F(1 - b1) * g
                v[s] = F(b2) * v[s] + F(1 - b2) * (g * g)
                up, root = 1 / (1 - b1 ** self.t), 1 / (1 - b2 ** self.t)
                adam = m[s].astype(np.float64) * up / (np.sqrt(v[s].astype(np.float64) * root) + self.eps)
                step = lr * (adam + self.decay[i] * w)
                out.append((step, 12 * 2.0 ** -24 * abs(lr) * (abs(adam) + abs(self.decay[i] * w))))
            if self.bits == 8:
                r = random_words(self.room, self.t, self.seed)
                self.m, self.ms = encode(m, r & 0xFFFF, True)
                self.v, self.vs = encode(v, r >> 16, False)
        return out
