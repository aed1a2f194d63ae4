"""The plain model of the paged cache (tests/cache_ref.py) with elements held in 8 bits, as include/pgxcache.h defines them: codes as numbers, in 64 bits."""
import math

import torch

from cache_ref import RefCache

BLOCK = 16


def e4m3(x):
    """the nearest e4m3 number, ties to even, in 64 bits; NaN where x is not finite"""
    _, e = torch.frexp(x)
    step = torch.exp2(torch.clamp(e.double() - 1, min=-6.0) - 3)
    return torch.where(torch.isfinite(x), torch.round(x / step) * step, torch.full_like(x, math.nan))


def scale_for(m):
    """the smallest power of two, 2^-100 or more, with m <= 448 of it"""
    e = -100
    while m > math.ldexp(448.0, e):
        e += 1
    return math.ldexp(1.0, e)


class RefCache8(RefCache):
    def __init__(self, kv, scales, table, lengths, refs):
        super().__init__(kv.float().cpu().double(), table, lengths, refs)
        self.scales = scales.cpu().double()

    def _place(self, s, t):
        return int(self.table[s, t // self.P]), t % self.P

    def _write_block(self, layer, which, head, s, t0, first, x):
        """x: [tokens][head_dim] of the tokens first ... of the block that begins with token t0"""
        page, at = self._place(s, t0)
        live = x[torch.isfinite(x)].abs()
        scale, where = scale_for(float(live.max()) if live.numel() else 0.0), (page, layer, which, head, at // BLOCK)
        block = self.kv[page, layer, which, head, at: at + BLOCK]
        if first > t0:
            was = float(self.scales[where])
            if was >= scale:
                scale = was
            else:
                block[: first - t0] = e4m3(block[: first - t0] * was / scale)
        block[first - t0: first - t0 + len(x)] = e4m3(x / scale)
        self.scales[where] = scale

    def _write_from(self, layer, s, first, k, v):
        for which, x in ((0, k), (1, v)):
            for head in range(x.shape[1]):
                t = first
                while t < first + len(x):
                    t0 = t // BLOCK * BLOCK
                    end = min(t0 + BLOCK, first + len(x))
                    self._write_block(layer, which, head, s, t0, t, x[t - first: end - first, head].cpu().double())
                    t = end

    def write(self, layer, k, v, slots):
        for i, s in enumerate(slots):
            if 0 <= s < self.slots:
                n = min(self.grown[s], k.shape[1])
                self._write_from(layer, s, int(self.lengths[s]) - self.grown[s], k[i, :n], v[i, :n])

    def write_last(self, layer, k, v, slots):
        """what attend does with k and v [n][heads][head_dim]"""
        for i, s in enumerate(slots):
            if 0 <= s < self.slots and self.grown[s] > 0:
                self._write_from(layer, s, int(self.lengths[s]) - 1, k[i][None], v[i][None])

    def fork(self, src, dst):
        before = self.lengths.tolist(), self.table.clone()
        status = super().fork(src, dst)
        for a, b, said in zip(src, dst, status):
            if said == 0 and 0 <= a < self.slots and 0 <= b < self.slots and a != b and before[0][a] % self.P:
                full, part = before[0][a] // self.P, before[0][a] % self.P
                self.scales[int(self.table[b, full]), ..., : -(-part // BLOCK)] = self.scales[int(before[1][a, full]), ..., : -(-part // BLOCK)]
        return status

    def compact(self):
        used = int((self.refs > 0).sum())
        holes = (self.refs[:used] == 0).nonzero()[:, 0].tolist()
        moved = ((self.refs[used:] > 0).nonzero()[:, 0] + used).tolist()
        for p, to in zip(moved, holes):
            self.scales[to] = self.scales[p]
        return super().compact()

    def sequence(self, s, layer):
        n = int(self.lengths[s])
        pages = self.table[s, : self._pages(n)].long()
        kv = self.kv[pages, layer] * self.scales[pages, layer].repeat_interleave(BLOCK, 3)[..., None]
        return kv.permute(1, 2, 0, 3, 4).reshape(2, kv.shape[2], -1, kv.shape[4])[:, :, :n]

    def read(self, layer, tokens, slots, first, dtype):
        """(keys, values), [n][tokens][heads][head_dim]"""
        out = torch.zeros(2, len(slots), tokens, self.kv.shape[3], self.kv.shape[5], dtype=torch.float64)
        for i, s in enumerate(slots):
            if 0 <= s < self.slots:
                held = self.sequence(s, layer).transpose(1, 2)
                for j in range(tokens):
                    if 0 <= first[i] + j < held.shape[1]:
                        out[:, i, j] = held[:, first[i] + j]
        return out.to(dtype)
