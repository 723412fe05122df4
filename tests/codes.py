"""A cache of 8-bit codes with a scale for each block and head, on both sides
(tests only): the oracle's numbers and the library's bytes."""
from __future__ import annotations

import numpy as np
import torch

from oracle import kv_codes as kc
from paper_2609_15030_amd import linattn as la

TYPES = {"e4m3": torch.float8_e4m3fn, "int8": torch.int8}


class CodeCache:
    """`blocks` blocks of `layers` layers, the second of them used; keys and values
    [blocks, heads, bt, d], scales behind all layers.  filled: codes and scales as
    writes leave them; else bytes of 0xA5, whose scales are none.  pad: bytes that
    follow in each block."""

    def __init__(self, gen, kind, heads, d, bt, table, blocks, layers=2, filled=True, pad=0, spread=3.0):
        self.kind, self.heads, self.d, self.bt = kind, heads, d, bt
        self.table = np.asarray(table, np.int32)
        self.part_bytes = heads * bt * d
        layer = layers - 1
        self.off = tuple((2 * layer + h) * self.part_bytes for h in (0, 1))
        self.scales_at = tuple(2 * layers * self.part_bytes + (2 * layer + h) * 4 * heads for h in (0, 1))
        size = -(-(2 * layers * (self.part_bytes + 4 * heads) + pad) // 16) * 16
        self.bytes = torch.full((blocks, size), 0xA5, dtype=torch.uint8)
        if filled:
            for h in (0, 1):
                x = torch.randn((blocks, heads, bt, d), generator=gen, dtype=torch.float64)
                x *= 2.0 ** (spread * torch.rand((blocks, heads, 1, 1), generator=gen, dtype=torch.float64))
                x = x.to(torch.bfloat16).double().numpy()
                scale = np.array([[kc.scale_of(np.abs(x[b, g]).max(), kind) for g in range(heads)] for b in range(blocks)])
                self.put(h, kc.codes(x / scale[:, :, None, None], kind), scale)
        self.dev = self.bytes.cuda() if torch.cuda.is_available() else None
        self.table_dev = torch.from_numpy(self.table).cuda() if torch.cuda.is_available() else None
        self.err = torch.zeros(1, dtype=torch.int32, device="cuda") if torch.cuda.is_available() else None

    def _views(self, bytes_, half):
        o, s = self.off[half], self.scales_at[half]
        return (bytes_[:, o:o + self.part_bytes].view(TYPES[self.kind]).unflatten(1, (self.heads, self.bt, self.d)),
                bytes_[:, s:s + 4 * self.heads].view(torch.float32))

    def put(self, half, code, scale):
        c, s = self._views(self.bytes, half)
        c.copy_(torch.from_numpy(code).float().to(c.dtype))
        s.copy_(torch.from_numpy(scale).float())

    def numbers(self, half, bytes_=None):
        """(codes, scales) in fp64."""
        c, s = self._views(self.bytes if bytes_ is None else bytes_, half)
        return c.double().numpy() if c.dtype is torch.int8 else c.float().double().numpy(), s.double().numpy()

    def layer(self, rows=slice(None)):
        return la.make_kv_layer(self.dev, self.table_dev[rows].contiguous(), self.bt, self.heads, self.d, TYPES[self.kind],
                                self.off[0], self.off[1], err_count=self.err, k_scales=self.scales_at[0],
                                v_scales=self.scales_at[1])

    def rows(self, seq, n, half):
        """What the first n stored keys or values of a sequence stand for; zeros without a block."""
        code, scale = self.numbers(half)
        out = np.zeros((n, self.heads, self.d))
        for x in range(n):
            j = x // self.bt
            b = int(self.table[seq, j]) if j < self.table.shape[1] else -1
            if 0 <= b < code.shape[0]:
                out[x] = code[b, :, x % self.bt] * scale[b][:, None]
        return out

    def write(self, k, v, cu, kv):
        """The oracle's write on the host's bytes."""
        for half, x in ((0, k), (1, v)):
            code, scale = self.numbers(half)
            kc.write(code, scale, self.table, self.bt, self.kind, x.double().cpu().numpy(), cu, kv)
            self.put(half, code, scale)

    def same(self, what):
        """The device's bytes are the host's, but for which of the NaN a code is."""
        dev = self.dev.cpu()
        for half in (0, 1):
            for a, b, name in zip(self.numbers(half, dev), self.numbers(half), ("codes", "scales")):
                assert np.array_equal(a, b, equal_nan=True), (what, "values" if half else "keys", name)
            if self.kind == "e4m3":
                for x in (dev, self.bytes):
                    c = self._views(x, half)[0].view(torch.uint8)
                    c.masked_fill_((c & 0x7F) == 0x7F, 0x7F)
        assert torch.equal(dev, self.bytes), (what, "bytes that are no part of the call")


def tables(gen, kv, bt, spare=3):
    """A permuted block for every 16th .. bt'th token: (table, blocks)."""
    need = [-(-max(n, 0) // bt) for n in kv]
    blocks = sum(need) + spare
    perm = torch.randperm(blocks, generator=gen).numpy()
    t = np.full((len(kv), max(need + [1])), -1, np.int32)
    at = 0
    for i, n in enumerate(need):
        t[i, :n] = perm[at:at + n]
        at += n
    return t, blocks
