"""Plain statements of the operators that serving needs around a paged K/V cache: the pages, block by block in Python, and the
verification of drafted tokens in 64 bits."""
import math

import torch


def up(n, bt):
    return (n + bt - 1) // bt


class Pool:
    """The block table as lists, the counts, and the calls on them by their definitions."""

    def __init__(self, n_blocks, n_seq, cols, bt=16):
        self.table, self.ref, self.bt = [[-1] * cols for _ in range(n_seq)], [0] * n_blocks, bt

    def fork(self, source, length):
        old, cols = self.table, len(self.table[0])
        self.table = [(old[s] if s >= 0 else [])[:up(max(n, 0), self.bt)] for s, n in zip(source, length)]
        self.table = [row + [-1] * (cols - len(row)) for row in self.table]
        for rows, by in ((old, -1), (self.table, 1)):
            for e in (e for row in rows for e in row if e >= 0):
                self.ref[e] += by

    def reserve(self, length, want):
        """(got, copy_src, copy_dst)"""
        bt, before = self.bt, list(self.ref)
        free = [i for i, r in enumerate(before) if r == 0]
        got, src, dst = list(length), [-1] * len(length), [-1] * len(length)
        part = [self.table[b][n // bt] if want[b] > n and n % bt else -1 for b, n in enumerate(length)]
        part = [e if e >= 0 and before[e] > 1 else -1 for e in part]
        asked = 0
        for b, (n, w) in enumerate(zip(length, want)):
            if w <= n:
                continue
            keeps = part[b] >= 0 and part.count(part[b]) == before[part[b]] and part[b] not in part[b + 1:]
            need = [j for j in range(n // bt, up(w, bt))
                    if self.table[b][j] < 0 or before[self.table[b][j]] > 1 and not (keeps and j == n // bt)]
            first = asked
            asked += len(need)
            if asked > len(free) and (need or keeps):
                continue
            got[b] = w
            for j, new in zip(need, free[first:asked]):
                e, self.table[b][j] = self.table[b][j], new
                self.ref[new] = 1
                if e >= 0:
                    self.ref[e] -= 1
                    if j == n // bt and n % bt:
                        src[b], dst[b] = e, new
        return got, src, dst

    def compact(self):
        """(used, copy_src, copy_dst)"""
        used = [i for i, r in enumerate(self.ref) if r]
        pairs = list(zip([i for i in used if i >= len(used)], [i for i in range(len(used)) if not self.ref[i]]))
        to = dict(pairs)
        self.table = [[to.get(e, e) for e in row] for row in self.table]
        for s, d in pairs:
            self.ref[d], self.ref[s] = self.ref[s], 0
        pairs += [(-1, -1)] * (len(self.ref) // 2 - len(pairs))
        return len(used), [s for s, _ in pairs], [d for _, d in pairs]

    def check(self):
        held = [0] * len(self.ref)
        for row in self.table:
            for e in row:
                if e >= 0:
                    held[e] += 1
        assert held == self.ref


def logs(l, t):
    """log softmax(l / T) in 64 bits, T = 0 as 1.  (The maximum first: 64 bits do not hold -3.4e38 + log 8.)"""
    l = l.double()
    l = (l - l.max()) / (t or 1.0)
    return l - torch.logsumexp(l, 0)


def verify(target, draft, tokens, start, u, temp=None):
    """(accepted, next, log probabilities by row) of sequences whose inputs are in range.  CPU tensors, lists."""
    accepted, nxt, lp = [], [], {}
    for b in range(len(start) - 1):
        t = 1.0 if temp is None else float(temp[b])
        r, end = start[b], start[b + 1] - 1
        if end < r:
            accepted.append(0)
            nxt.append(-1)
            continue
        while r < end:
            x, p = tokens[r + 1], logs(target[r], t)
            if t == 0:
                if int(target[r].double().argmax()) != x:
                    break
            else:
                lq = 0.0 if draft is None else float(logs(draft[r], t)[x])
                lu = math.log(float(u[r])) if u[r] > 0 else -math.inf
                if not lu + lq < float(p[x]):
                    break
            lp[r] = float(p[x])
            r += 1
        p = logs(target[r], t)
        if t == 0:
            i = int(target[r].double().argmax())
        else:
            w = p.exp()
            if r < end:
                q = torch.zeros_like(w)
                if draft is None:
                    q[tokens[r + 1]] = 1.0
                else:
                    q = logs(draft[r], t).exp()
                d = (w - q).clamp(min=0)
                w = d if float(d.sum()) >= 2.0 ** -20 else w
            c = w.cumsum(0)
            i = int((c <= (float(u[end]) + 2.0 ** -25) * float(w.sum())).sum())
        accepted.append(r - start[b])
        nxt.append(i)
        lp[r] = float(p[i])
    return accepted, nxt, lp
