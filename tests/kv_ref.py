"""The paged 8-bit cache on the host, from its definition in q2d.h, in 64 bits."""
import numpy as np
import torch

BLOCK = 32


def exponent(m: float) -> int:
    """Smallest e >= -127 with 448 * 2^e >= m."""
    if m == 0:
        return -127
    e = int(np.ceil(np.log2(m / 448.0)))
    while 448.0 * 2.0 ** (e - 1) >= m:
        e -= 1
    while 448.0 * 2.0 ** e < m:
        e += 1
    return max(e, -127)


def encode(x: np.ndarray) -> np.ndarray:
    """E4M3 codes of |x| <= 448, to nearest, ties to even."""
    a = np.abs(x)
    q = np.maximum(np.floor(np.log2(np.where(a > 0, a, 1.0))), -6)
    n = np.rint(a / 2.0 ** (q - 3)).astype(np.int64)          # 0 .. 16 eighths of 2^q
    up = n == 16
    q, n = np.where(up, q + 1, q).astype(np.int64), np.where(up, 8, n)
    code = np.where(n >= 8, ((q + 7) << 3) | (n - 8), n)      # below 8 eighths: q = -6, subnormal
    return (code | (np.signbit(x).astype(np.int64) << 7)).astype(np.uint8)


def decode(c: np.ndarray) -> np.ndarray:
    c = c.astype(np.int64)
    e, f = (c >> 3) & 15, c & 7
    v = np.where(e == 0, f * 2.0 ** -9, (8 + f) * 2.0 ** (e - 10.0))
    v = np.where((c & 127) == 127, np.nan, v)
    return np.where(c >= 128, -v, v)


class Cache:
    """One sequence's keys or values of one head: codes [tokens rounded up, D], a byte each block."""

    def __init__(self, D):
        self.codes, self.bytes, self.n = np.zeros((0, D), np.uint8), [], 0

    def append(self, x):
        x = np.asarray(x, dtype=np.float64)
        first, total = self.n, self.n + len(x)
        while len(self.bytes) * BLOCK < total:
            self.codes = np.concatenate((self.codes, np.zeros((BLOCK, self.codes.shape[1]), np.uint8)))
            self.bytes.append(None)
        for b in range(first // BLOCK, (total + BLOCK - 1) // BLOCK if len(x) else first // BLOCK):
            lo, hi = max(first, b * BLOCK), min(total, (b + 1) * BLOCK)
            new = x[lo - first:hi - first]
            byte = exponent(float(np.abs(new).max())) + 127 if np.isfinite(new).all() else 255
            if lo > b * BLOCK:
                old = self.bytes[b]
                byte = max(byte, old)
                if byte != old:
                    held = self.codes[b * BLOCK:lo]
                    if byte == 255:
                        held[:] = 0
                    else:
                        held[:] = encode(decode(held) * 2.0 ** (old - byte))
            self.codes[lo:hi] = 0 if byte == 255 else encode(new / 2.0 ** (byte - 127))
            self.bytes[b] = byte
        self.n = total

    def values(self):
        s = np.repeat([np.nan if b == 255 else 2.0 ** (b - 127) for b in self.bytes], BLOCK)
        return (decode(self.codes) * s[:, None] if len(s) else self.codes.astype(np.float64))[:self.n]


class Paged:
    """Reference caches of some sequences beside a device cache with shuffled pages."""

    def __init__(self, q2d, batch, heads, dim, page_size=64, capacity=512, seed=0):
        per = -(-capacity // page_size)
        self.cache = q2d.KVCache(batch * per + 2, heads, dim, page_size=page_size)
        g = torch.Generator().manual_seed(seed)
        order = torch.randperm(batch * per + 2, generator=g)[:batch * per]
        self.table = order.view(batch, per).to(torch.int32)
        self.q2d, self.heads, self.dim, self.page = q2d, heads, dim, page_size
        self.k = [[Cache(dim) for _ in range(heads)] for _ in range(batch)]
        self.v = [[Cache(dim) for _ in range(heads)] for _ in range(batch)]
        # what free pages hold is anything
        for t in (self.cache.k_codes, self.cache.v_codes_t, self.cache.k_scales, self.cache.v_scales):
            t.fill_(0xFF)

    def lens(self):
        return torch.tensor([s[0].n for s in self.k], dtype=torch.int32)

    def append(self, k, v, counts):
        """k, v [tokens, heads, dim] device tensors, counts[b] rows each sequence."""
        at = 0
        for b, n in enumerate(counts):
            for h in range(self.heads):
                self.k[b][h].append(k[at:at + n, h].float().cpu().numpy())
                self.v[b][h].append(v[at:at + n, h].float().cpu().numpy())
            at += n
        off = torch.tensor(np.concatenate(([0], np.cumsum(counts))), dtype=torch.int64).cuda()
        self.q2d.q2d_kv_write(self.cache, k, v, self.table.cuda(), self.lens().cuda(), offsets=off)

    def check(self):
        """Codes of all tokens and their blocks' scale bytes, bit for bit."""
        c = {n: getattr(self.cache, n).cpu().numpy() for n in ("k_codes", "v_codes_t", "k_scales", "v_scales")}
        for b in range(len(self.k)):
            for h in range(self.heads):
                for which, ref in (("k", self.k[b][h]), ("v", self.v[b][h])):
                    for i, byte in enumerate(ref.bytes):
                        page, sub = int(self.table[b, i * BLOCK // self.page]), i % (self.page // BLOCK)
                        n = min(ref.n - i * BLOCK, BLOCK)
                        assert c[which + "_scales"][page, h, sub] == byte, (which, b, h, i)
                        got = c["k_codes"][page, h, sub * BLOCK:sub * BLOCK + n] if which == "k" else \
                            c["v_codes_t"][page, h, sub, :, :n].T
                        assert np.array_equal(got, ref.codes[i * BLOCK:i * BLOCK + n]), (which, b, h, i)

    def dense(self, b):
        """K and V [tokens, heads, dim] of a sequence in 64 bits."""
        return [torch.from_numpy(np.stack([s.values() for s in t[b]], 1)) for t in (self.k, self.v)]
