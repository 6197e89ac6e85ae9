"""Cases of the 8-bit cache's tests: pools, tables and ragged lengths."""
import numpy as np
import torch

from oracle import q8

PAGE = 16
DTYPES = {"e4m3": torch.float8_e4m3fn, "e5m2": torch.float8_e5m2}


def bf16(rng, *shape, scale=1.0):
    return torch.from_numpy(rng.standard_normal(shape) * scale).to(torch.bfloat16)


class Pool:
    """An 8-bit pool on the CPU: pages in a random order, every slot a NaN code
    until written, scales NaN."""

    def __init__(self, rng, tokens, hkv, d, fmt, spare=2, width=None):
        self.fmt, self.hkv, self.d = fmt, hkv, d
        need = [-(-int(n) // PAGE) for n in tokens]
        self.width = max(max(need, default=1), 1) if width is None else width
        total = sum(need) + spare
        perm = rng.permutation(total)
        self.table = np.zeros((len(tokens), self.width), dtype=np.int32)
        at = 0
        for b, n in enumerate(need):
            self.table[b, :n] = perm[at:at + n]
            at += n
        self.k = torch.full((total, hkv, PAGE, d), 0x7F, dtype=torch.uint8)
        self.v = torch.full((total, hkv, d, PAGE), 0x7F, dtype=torch.uint8)
        self.ks = torch.full((total, hkv), float("nan"))
        self.vs = torch.full((total, hkv), float("nan"))

    def fill(self, rng, lens, sigma=1.0):
        """The first lens[b] tokens of every sequence written (by the oracle)."""
        rows = int(sum(lens))
        k, v = bf16(rng, rows, self.hkv, self.d, scale=sigma), bf16(rng, rows, self.hkv, self.d, scale=sigma)
        self.set(q8.kv_write_q8(self.k, self.v, self.ks, self.vs, self.table, [0] * len(lens), lens, k, v, self.fmt))
        return self

    def set(self, parts):
        self.k, self.v = torch.from_numpy(parts[0]), torch.from_numpy(parts[1])
        self.ks, self.vs = torch.from_numpy(parts[2]), torch.from_numpy(parts[3])

    def on(self, dev):
        """The binding's first five arguments, as copies on the device."""
        t = DTYPES[self.fmt]
        return [self.k.to(dev).view(t), self.v.to(dev).view(t), self.ks.to(dev), self.vs.to(dev),
                torch.from_numpy(self.table).to(dev)]

    def values(self):
        """fp64 pools (torch, as the attention's oracle takes them)."""
        return (torch.from_numpy(q8.dequantise(self.k, self.ks, self.fmt)),
                torch.from_numpy(q8.dequantise(self.v, self.vs, self.fmt)))


def i32(x, dev="cpu"):
    return torch.as_tensor(np.asarray(x), dtype=torch.int32).to(dev)
