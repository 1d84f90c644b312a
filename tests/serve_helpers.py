"""Plain forms of the serving step's operators, in Python's whole numbers and 64-bit floating point, and caches to try them on."""
import math

import numpy as np

HALF_STEP = {"bf16": 2.0 ** -8, "f16": 2.0 ** -11, "f32": 2.0 ** -24, "e4m3": 2.0 ** -4}


def torch_type(name):
    import torch
    return {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32, "e4m3": torch.float8_e4m3fn}[name]


def dev(x, dtype=None):
    import torch
    t = torch.as_tensor(np.ascontiguousarray(x)).to("cuda:0")
    return t if dtype is None else t.to(dtype)


def i32(x):
    import torch
    return dev(np.asarray(x, np.int64), torch.int32)


class Pages:
    """The cache's rules: tables, counts and the numbers themselves (k, v: [layers, pages, heads, T, dim] arrays)."""

    def __init__(self, table, length, ref, k, v, T):
        self.table, self.len, self.ref, self.k, self.v, self.T = table.copy(), length.copy(), ref.copy(), k.copy(), v.copy(), T

    def free(self):
        return [p for p in range(len(self.ref)) if self.ref[p] == 0]

    def fork(self, src, dst, n_tok=None):
        rows, free, seen = len(self.len), self.free(), set()
        first = self.len.copy()
        errors = set()
        for i, (s, d) in enumerate(zip(src, dst)):
            twice = d in seen
            if 0 <= d < rows:
                seen.add(d)
            if not (0 <= s < rows and 0 <= d < rows) or s == d or twice or first[d] != 0:
                errors.add(-6)
                continue
            t = first[s] if n_tok is None else n_tok[i]
            if t < 0 or t > first[s]:
                errors.add(-6)
                continue
            whole, part = divmod(int(t), self.T)
            tail = self.table[s][whole] if part else -1
            if part and tail >= 0:
                if not free:
                    errors.add(-4)
                    continue
                p = free.pop(0)
                self.ref[p] = 1
                self.table[d][whole] = p
                for x in (self.k, self.v):
                    x[:, p, :, :part] = x[:, tail, :, :part]
            for b in range(whole):
                self.table[d][b] = p = self.table[s][b]
                if p >= 0:
                    self.ref[p] += 1
            self.len[d] = t
        return errors

    def grow(self, row, n_new):
        free, seen, out, errors = self.free(), set(), False, set()
        for r, m in zip(row, n_new):
            twice = r in seen
            if 0 <= r < len(self.len):
                seen.add(r)
            if not 0 <= r < len(self.len) or twice or m < 0 or self.len[r] + m > self.table.shape[1] * self.T:
                errors.add(-6)
                continue
            have = -(-int(self.len[r]) // self.T)
            need = -(-int(self.len[r] + m) // self.T) - have
            if need and (out or need > len(free)):
                out = True
                errors.add(-4)
                continue
            for b in range(have, have + need):
                self.table[r][b] = p = free.pop(0)
                self.ref[p] = 1
            self.len[r] += m
        return errors

    def write(self, layer, row, tok_ptr, k, v):
        for i, r in enumerate(row):
            n = tok_ptr[i + 1] - tok_ptr[i]
            for j in range(n):
                y = self.len[r] - n + j
                p = self.table[r][y // self.T]
                self.k[layer, p, :, y % self.T] = k[tok_ptr[i] + j]
                self.v[layer, p, :, y % self.T] = v[tok_ptr[i] + j]

    def drop(self, r, b):
        p = self.table[r][b]
        self.table[r][b] = -1
        if p >= 0:
            self.ref[p] -= 1

    def keep(self, row, n_draft, kept):
        for r, nd, ks in zip(row, n_draft, kept):
            base = int(self.len[r]) - nd
            for j, k in enumerate(ks):
                p, q = self.table[r][(base + k) // self.T], self.table[r][(base + j) // self.T]
                for x in (self.k, self.v):
                    x[:, q, :, (base + j) % self.T] = x[:, p, :, (base + k) % self.T]
            left = base + len(ks)
            for b in range(-(-left // self.T), -(-int(self.len[r]) // self.T)):
                self.drop(r, b)
            self.len[r] = left

    def give(self, row, first=None, last=None):
        for i, r in enumerate(row):
            if first is None:
                for b in range(-(-int(self.len[r]) // self.T)):
                    self.drop(r, b)
                self.len[r] = 0
            else:
                for b in range(int(self.len[r]) // self.T):
                    if b * self.T >= first[i] and (b + 1) * self.T <= min(last[i], self.len[r]):
                        self.drop(r, b)

    def compact(self):
        used = [p for p in range(len(self.ref)) if self.ref[p] > 0]
        n = len(used)
        holes = [p for p in range(n) if self.ref[p] == 0]
        moved = np.full(len(self.ref), -1)
        moved[used] = used
        for p, q in zip([p for p in used if p >= n], holes):
            moved[p] = q
            for x in (self.k, self.v):
                x[:, q] = x[:, p]
            self.ref[q], self.ref[p] = self.ref[p], 0
        self.table[self.table >= 0] = moved[self.table[self.table >= 0]]
        return n, moved


def visible(n, m, parent, window, sinks):
    """[m, n]: which of a sequence's n positions each of its last m tokens sees."""
    see = np.zeros((m, n), bool)
    base = n - m
    depth = np.full(m, -1)
    above = [None] * m
    pos = np.arange(n)
    if parent is not None:
        for i in range(m):
            p = parent[i]
            if p == -1:
                depth[i], above[i] = 0, [i]
            elif p >= 0 and above[p] is not None:
                depth[i], above[i] = depth[p] + 1, above[p] + [i]
        pos[base:] = base + depth
    for i in range(m):
        if parent is None:
            x = base + i
            see[i, :x + 1] = True
        else:
            if above[i] is None:
                continue
            x = base + depth[i]
            see[i, :base] = True
            see[i, [base + a for a in above[i]]] = True
        if window > 0:
            see[i] &= (pos < sinks) | (x - pos < window)
    return see


def attend(q, k, v, see, scale, group):
    """q [m, heads, dim], k, v [n, KV heads, dim], all float64 -> out, lse, sum of weight |v|, sum of |v| seen, largest sum of |q k|."""
    m, heads, dim = q.shape
    out, lse = np.zeros((m, heads, dim)), np.full((m, heads), -np.inf)
    size, plain, reach = np.zeros((m, heads, dim)), np.zeros((m, heads, dim)), np.zeros((m, heads))
    for i in range(m):
        ys = np.nonzero(see[i])[0]
        if not len(ys):
            continue
        for a in range(heads):
            kk, vv = k[ys, a // group], v[ys, a // group]
            s = scale * (kk @ q[i, a])
            top = s.max()
            w = np.exp(s - top)
            lse[i, a] = top + math.log(w.sum())
            w /= w.sum()
            out[i, a] = w @ vv
            size[i, a] = w @ np.abs(vv)
            plain[i, a] = np.abs(vv).sum(0)
            reach[i, a] = abs(scale) * (np.abs(kk) @ np.abs(q[i, a])).max()
    return out, lse, size, plain, reach


def sample(x, T, k, p, mp, u):
    """(token, logprob, how many stay) of one row of logits, float64; x without NaN."""
    order = sorted((i for i in range(len(x)) if x[i] > -np.inf), key=lambda i: (-x[i], i))
    if not order:
        return -1, -np.inf, 0
    if T == 0:
        return order[0], 0.0, 1
    top = x[order[0]]
    if k > 0:
        order = order[:k]
    w = np.array([1.0 if x[i] == top else 0.0 if top == np.inf else math.exp((x[i] - top) / T) for i in order])
    if p < 1:
        before = np.concatenate([[0.0], np.cumsum(w)[:-1]])
        n = max(1, int((before < p * w.sum()).sum()))
        order, w = order[:n], w[:n]
    stay = w >= mp
    order, w = [i for i, s in zip(order, stay) if s], w[stay]
    by = np.argsort(order)
    c = np.cumsum(w[by])
    at = int(np.searchsorted(c, u * c[-1], side="right"))
    return order[by[at]], math.log(w[by[at]] / c[-1]), len(order)
