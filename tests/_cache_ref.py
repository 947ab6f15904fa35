"""Plain form of the paged cache in 64 bits: attention row by row over gathered keys, bookkeeping in Python lists."""
import math

import torch


def gather(pages, ids, L, page):
    """Rows 0..L-1 of a slot from pages [n_pages, page, H, dh]; an id outside the pool is a page of zeros."""
    out = torch.zeros((L,) + tuple(pages.shape[2:]), dtype=torch.float64, device=pages.device)
    for p in range(-(-L // page)):
        n = min(page, L - p * page)
        if 0 <= ids[p] < pages.shape[0]:
            out[p * page:p * page + n] = pages[ids[p], :n].double()
    return out


def attention(K, V, table, lens, offsets, Q, slots=None, causal=True, scale=None, cap=0.0, slopes=None, begin=None, prefix=None):
    """(O, A, S) in fp64: the outputs, sum_j p_j |v_j| and the largest scale |q| |k| of each row: what roundings scale with."""
    n_pages, page, Hkv, dh = K.shape
    N, H, _ = Q.shape
    G = H // Hkv
    scale = scale or 1.0 / math.sqrt(dh)
    O = torch.zeros((N, H, dh), dtype=torch.float64, device=Q.device)
    A, S = torch.zeros_like(O), torch.zeros((N, H, 1), dtype=torch.float64, device=Q.device)
    tab, ln = table.tolist(), lens.tolist()
    for r in range(len(offsets) - 1):
        a, b = offsets[r], offsets[r + 1]
        s = slots[r] if slots is not None else r
        if a == b or not 0 <= s < len(tab):
            continue
        L = min(max(ln[s], 0), len(tab[s]) * page)
        if L == 0:
            continue
        k, v = gather(K, tab[s], L, page), gather(V, tab[s], L, page)
        j = torch.arange(L, device=Q.device)
        pos = torch.arange(L - (b - a), L, device=Q.device) if causal else torch.full((b - a,), L, device=Q.device)
        hi = torch.clamp(torch.clamp(pos + 1, min=int(prefix[r]) if prefix is not None else 0), max=L) if causal else pos
        lo = begin[a:b].long().clamp(min=0) if begin is not None else torch.zeros_like(pos)
        seen = (j[None] >= lo[:, None]) & (j[None] < hi[:, None])
        q = Q[a:b].double().view(b - a, Hkv, G, dh)
        for h in range(Hkv):
            seen_any = seen.any(0)  # keys that nobody sees may hold anything
            kh = torch.where(seen_any[:, None], k[:, h], 0.0)
            vh = torch.where(seen_any[:, None], v[:, h], 0.0)
            for g in range(G):
                x = scale * (q[:, h, g] @ kh.T)
                size = scale * (q[:, h, g].abs() @ kh.abs().T)
                if cap:
                    x = cap * torch.tanh(x / cap)
                if slopes is not None:
                    x = x - float(slopes[h * G + g]) * (pos[:, None] - j[None]).abs()
                x = torch.where(seen, x, -math.inf)
                p = torch.softmax(x, -1)
                p = torch.where(seen, p, 0.0)
                some = seen.any(1, keepdim=True)
                # a row's masked keys add nothing, whatever they hold
                bad = ~torch.isfinite(vh)
                if bad.any():
                    o = torch.stack([(p[i][seen[i]][:, None] * vh[seen[i]]).sum(0) for i in range(b - a)])
                    m = torch.stack([(p[i][seen[i]][:, None] * vh[seen[i]].abs()).sum(0) for i in range(b - a)])
                else:
                    o, m = p @ vh, p @ vh.abs()
                O[a:b, h * G + g] = torch.where(some, o, 0.0)
                A[a:b, h * G + g] = torch.where(some, m, 0.0)
                S[a:b, h * G + g, 0] = torch.where(seen, size, 0.0).amax(-1)
    return O, A, S


class Books:
    """Tables, lengths and holders as lists; every call either does all of it or returns a status."""

    def __init__(self, table, lens, refs, page):
        self.table = [list(r) for r in table]
        self.lens, self.refs, self.page = list(lens), list(refs), page
        self.width = len(self.table[0])

    def pages(self, n):
        return -(-n // self.page)

    def _slots_ok(self, slots):
        return all(0 <= s < len(self.table) for s in slots) and len(set(slots)) == len(slots)

    def extend(self, slots, counts):
        """(status, pages, first, copies [(from, to)])."""
        none = [-1] * len(slots)
        status, need = 0, []
        if not self._slots_ok(slots):
            status = 2
        for s, n in zip(slots, counts):
            if not 0 <= s < len(self.table):
                continue
            L = self.lens[s]
            if L < 0 or L + n > self.width * self.page:
                status = max(status, 3)
                continue
            copy = False
            if n > 0 and L % self.page:
                id = self.table[s][L // self.page]
                if not 0 <= id < len(self.refs):
                    status = max(status, 5)
                else:
                    copy = self.refs[id] > 1
            start = self.pages(L) - copy
            need.append((s, L, n, start, self.pages(L + n) - start if n else 0, copy))
        free = [i for i, c in enumerate(self.refs) if c == 0]
        total = sum(x[4] for x in need)
        if status == 0 and total > len(free):
            return 1, total - len(free), none, []
        if status:
            return status, 0, none, []
        copies, at = [], 0
        for s, L, n, start, count, copy in need:
            if copy:
                copies.append((self.table[s][start], free[at]))
                self.refs[self.table[s][start]] -= 1
            for k in range(count):
                self.table[s][start + k] = free[at]
                self.refs[free[at]] = 1
                at += 1
            self.lens[s] = L + n
        return 0, total, [x[1] for x in need], copies

    def fork(self, parents, children):
        status = 0
        if not self._slots_ok(children) or any(not 0 <= p < len(self.table) or p == c for p, c in zip(parents, children)):
            status = 2
        for p, c in zip(parents, children):
            if 0 <= c < len(self.table) and 0 <= p < len(self.table) and p != c and self.lens[c] != 0:
                status = max(status, 4)
        if status:
            return status, 0
        shared, lens = 0, [self.lens[p] for p in parents]
        for p, c, L in zip(parents, children, lens):
            for k in range(self.pages(L)):
                self.table[c][k] = self.table[p][k]
                self.refs[self.table[p][k]] += 1
                shared += 1
        for c, L in zip(children, lens):
            self.lens[c] = L
        return 0, shared

    def truncate(self, slots, keep=None):
        if not self._slots_ok(slots):
            return 2, 0
        given = 0
        for i, s in enumerate(slots):
            left = min(max(keep[i] if keep else 0, 0), self.lens[s])
            for k in range(self.pages(left), self.pages(self.lens[s])):
                self.refs[self.table[s][k]] -= 1
                given += 1
            self.lens[s] = left
        return 0, given

    def compact(self):
        """Moves [(from, to)]."""
        live = [i for i, c in enumerate(self.refs) if c > 0]
        line = len(live)
        moves = list(zip([i for i in live if i >= line], [i for i in range(line) if self.refs[i] == 0]))
        to = dict(moves)
        for s, L in enumerate(self.lens):
            for k in range(self.pages(L)):
                self.table[s][k] = to.get(self.table[s][k], self.table[s][k])
        for a, b in moves:
            self.refs[b], self.refs[a] = self.refs[a], 0
        return line, moves
