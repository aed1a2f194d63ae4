"""A plain model of the paged cache (include/pgxcache.h) on the CPU: lists of pages per slot, one entry after the other."""
import torch


class RefCache:
    def __init__(self, kv, table, lengths, refs):
        self.kv, self.table, self.lengths, self.refs = (t.cpu().clone() for t in (kv, table, lengths, refs))
        self.P, self.width, self.slots = kv.shape[4], table.shape[1], table.shape[0]
        self.grown = [0] * self.slots

    def _pages(self, tokens):
        return -(-tokens // self.P)

    def _free_pages(self):
        return (self.refs == 0).nonzero()[:, 0].tolist()

    def advance(self, slots, counts):
        status, given, free, taken = [], 0, self._free_pages(), []
        for s, more in zip(slots, counts):
            if s == -1:
                status.append(0)
                continue
            if not 0 <= s < self.slots or more < 0:
                status.append(255)
                if 0 <= s < self.slots:
                    self.grown[s] = 0
                continue
            n = int(self.lengths[s])
            if n + more > self.width * self.P:
                status.append(2)
                self.grown[s] = 0
                continue
            have, need = self._pages(n), self._pages(n + more) - self._pages(n)
            got, given = free[given: given + need], given + need
            if len(got) < need:
                status.append(1)
                self.grown[s] = 0
                continue
            for k, page in enumerate(got):
                self.table[s, have + k] = page
                taken.append(page)
            self.lengths[s] = n + more
            self.grown[s] = more
            status.append(0)
        self.refs[taken] = 1
        return status

    def write(self, layer, k, v, slots):
        k, v = k.cpu(), v.cpu()
        for i, s in enumerate(slots):
            if not 0 <= s < self.slots:
                continue
            for t in range(min(self.grown[s], k.shape[1])):
                at = int(self.lengths[s]) - self.grown[s] + t
                page = int(self.table[s, at // self.P])
                self.kv[page, layer, 0, :, at % self.P] = k[i, t]
                self.kv[page, layer, 1, :, at % self.P] = v[i, t]

    def _release(self, s):
        for k in range(self._pages(int(self.lengths[s]))):
            self.refs[self.table[s, k]] -= 1
            self.table[s, k] = -1
        self.lengths[s] = 0
        self.grown[s] = 0

    def fork(self, src, dst):
        status, free, given, held = [], self._free_pages(), 0, []
        for a, b in zip(src, dst):
            if a == -1 or b == -1:
                status.append(0)
                continue
            if not (0 <= a < self.slots and 0 <= b < self.slots):
                status.append(255)
                continue
            if a == b:
                status.append(0)
                continue
            n = int(self.lengths[a])
            full, part = n // self.P, n % self.P
            if part:
                given += 1
                if given > len(free):
                    status.append(1)
                    continue
            self._release(b)
            for k in range(full):
                self.table[b, k] = self.table[a, k]
                self.refs[self.table[a, k]] += 1
            if part:
                page = free[given - 1]
                self.table[b, full] = page
                held.append(page)
                self.kv[page, ..., :part, :] = self.kv[int(self.table[a, full]), ..., :part, :]
            self.lengths[b] = n
            status.append(0)
        self.refs[held] = 1
        return status

    def free(self, slots):
        for s in slots:
            if 0 <= s < self.slots:
                self._release(s)

    def compact(self):
        used = int((self.refs > 0).sum())
        holes = (self.refs[:used] == 0).nonzero()[:, 0].tolist()
        moved = ((self.refs[used:] > 0).nonzero()[:, 0] + used).tolist()
        where = dict(zip(moved, holes))
        for p, to in where.items():
            self.kv[to] = self.kv[p]
            self.refs[to], self.refs[p] = int(self.refs[p]), 0
        for s in range(self.slots):
            for k in range(self.width):
                self.table[s, k] = where.get(int(self.table[s, k]), int(self.table[s, k]))
        return used

    def sequence(self, s, layer):
        """(keys, values) [kv_heads][length][head_dim] in 64 bits"""
        n = int(self.lengths[s])
        pages = self.table[s, : self._pages(n)].long()
        kv = self.kv[pages, layer].double()                        # [pages][2][heads][P][D]
        return kv.permute(1, 2, 0, 3, 4).reshape(2, kv.shape[2], -1, kv.shape[4])[:, :, :n]

    def attend(self, layer, q, slots, scale):
        q = q.cpu().double()
        out, lse, spread = torch.zeros_like(q), torch.full(q.shape[:2], float("-inf"), dtype=torch.float64), torch.zeros(q.shape[:2], dtype=torch.float64)
        for i, s in enumerate(slots):
            if not 0 <= s < self.slots or not int(self.lengths[s]):
                continue
            k, v = self.sequence(s, layer)
            group = q.shape[1] // k.shape[0]
            for h in range(q.shape[1]):
                score = (k[h // group] * q[i, h]).sum(1) * scale
                p = torch.softmax(score, 0)
                out[i, h] = (p[:, None] * v[h // group]).sum(0)
                lse[i, h] = torch.logsumexp(score, 0)
                spread[i, h] = score.abs().max()
        return out, lse, spread
