"""Plain forms for caches of 4 bits, chosen pages and eviction, in 64 bits, and caches of every type to try them on."""
import numpy as np

from tests import serve_helpers as sh

GRID = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
LEAST, MOST, NAN_BYTE = 127 - 23, 127 + 13, 255


def encode(x):
    """[..., 32 g] numbers -> codes [...] and scales' bytes [..., g]; comparisons with numbers that 64 bits hold exactly."""
    x = np.asarray(x, np.float64)
    x = x.reshape(*x.shape[:-1], -1, 32)
    top = np.abs(x).max(-1)
    byte = np.full(top.shape, MOST)
    for b in range(MOST, LEAST - 1, -1):                       # the least scale that 6 reaches the largest with
        byte = np.where(top <= 6 * 2.0 ** (b - 127), b, byte)
    a = np.abs(x) / 2.0 ** (byte[..., None] - 127.0)
    middles = (GRID[1:] + GRID[:-1]) / 2
    code = np.zeros(x.shape, np.int64)
    for c, m in enumerate(middles):                            # past a middle; upon it where the next code is even
        code += (a > m) | ((a == m) & (c % 2 == 1))
    code = np.where(np.signbit(x), code + 8, code)
    nan = np.isnan(x).any(-1)
    code = np.where(nan[..., None], 0, code)
    return code.reshape(*code.shape[:-2], -1), np.where(nan, NAN_BYTE, byte)


def decode(codes, byte):
    """Codes [..., 32 g] and bytes [..., g] -> numbers."""
    unit = np.where(byte == NAN_BYTE, np.nan, 2.0 ** (byte - 127.0))
    x = GRID[codes % 8] * np.where(codes >= 8, -1.0, 1.0)
    return (x.reshape(*x.shape[:-1], -1, 32) * unit[..., None]).reshape(x.shape)


def packed(codes):
    return (codes[..., 0::2] + 16 * codes[..., 1::2]).astype(np.uint8)


def unpacked(b):
    b = np.asarray(b).astype(np.int64)
    return np.stack([b & 15, b >> 4], -1).reshape(*b.shape[:-1], -1)


def numbers(pool, name):
    """What a pool holds, in 64 bits, without heads' scales."""
    import torch
    x = pool[name]
    if x.dtype == torch.uint8:
        return decode(unpacked(x.cpu().numpy()), pool[name + "_exp"].cpu().numpy().astype(np.int64))
    return x.float().cpu().numpy().astype(np.float64)


class Cache:
    """Sequences of these lengths in rows of their own on pages at random; k, v: what it holds, [layers, pages, heads, T, dim] in 64 bits.  What
    no sequence may see is NaN.  `missing`: (sequence, block) without a page.  `alike`: how far neighbouring tokens' keys are alike."""

    def __init__(self, seed, lens, T, heads, dim, cache, layers=2, missing=(), spare=5, extra_rows=3, room=1, alike=0.0, garbage=True, bounds=False):
        import torch
        rng = np.random.default_rng(seed)
        g = torch.Generator().manual_seed(seed)
        n = len(lens)
        self.lens, self.T, self.need = list(lens), T, [-(-x // T) for x in lens]
        self.n_pages = n_pages = sum(self.need) + spare
        order = rng.permutation(n_pages)
        self.rows = n + extra_rows
        self.where = rng.permutation(self.rows)[:n]
        self.table, at = np.full((self.rows, max(self.need + [1]) + room), -1), 0
        for i in range(n):
            self.table[self.where[i], :self.need[i]] = order[at:at + self.need[i]]
            at += self.need[i]
        self.ref = np.zeros(n_pages, np.int64)
        self.ref[order[:at]] = 1
        self.length = np.zeros(self.rows, np.int64)
        self.length[self.where] = lens
        shape = (layers, n_pages, heads, T, dim)
        full = torch.randn((2,) + shape, generator=g)
        full[0] += alike * torch.randn((layers, n_pages, heads, 1, dim), generator=g)
        unseen = np.ones((n_pages, T), bool)
        for i in range(n):
            for b in range(self.need[i]):
                if (i, b) not in missing:
                    unseen[self.table[self.where[i], b], :max(0, lens[i] - b * T)] = False
        for i, b in missing:
            self.ref[self.table[self.where[i], b]] = 0
            self.table[self.where[i], b] = -1
        bad = torch.as_tensor(unseen if garbage else np.zeros_like(unseen))[None, :, None, :, None]
        pool = dict(ref=sh.i32(self.ref), page_tokens=T)
        self.scale = {}
        for name, x in (("k", full[0]), ("v", full[1])):
            if cache == "e2m1":
                codes, byte = encode(x.numpy())
                byte = np.where(bad.numpy(), NAN_BYTE, byte)
                pool[name], pool[name + "_exp"] = sh.dev(packed(codes)), sh.dev(byte.astype(np.uint8))
            else:
                if cache == "e4m3":
                    x = x * 30
                    self.scale[name] = (torch.rand(layers, heads, generator=g) + 0.5) / 30
                    pool[name + "_scale"] = self.scale[name].cuda()
                pool[name] = x.masked_fill(bad.expand_as(x), float("nan")).to(sh.torch_type(cache)).cuda().contiguous()
        if bounds:
            t = sh.torch_type("bf16" if cache in ("e2m1", "e4m3") else cache)
            pool["bounds"] = torch.full((layers, n_pages, heads, 2, dim), float("nan"), dtype=t, device="cuda:0")
        self.pool, self.seqs = pool, dict(table=sh.i32(self.table), len=sh.i32(self.length))
        self.stored = {name: numbers(pool, name) for name in ("k", "v")}
        self.k, self.v = (self.stored[x] * (self.scale[x].double().numpy()[:, None, :, None, None] if self.scale else 1.0) for x in ("k", "v"))

    def of(self, x, layer, i):
        """Sequence i's part of k or v, [tokens, heads, dim]; what has no page is 0."""
        pages = self.table[self.where[i], :self.need[i]]
        y = np.where((pages >= 0)[:, None, None, None], x[layer, np.maximum(pages, 0)], 0.0)
        return y.transpose(0, 2, 1, 3).reshape(-1, y.shape[1], y.shape[3])[:self.lens[i]]

    def there(self, i):
        """[tokens]: whether their page is."""
        return np.repeat(self.table[self.where[i], :self.need[i]] >= 0, self.T)[:self.lens[i]]


def queries(n_q, heads, dim, type_, seed, wide=True):
    """Queries as a projection writes them, between others; or heads before tokens and nothing aligned."""
    import torch
    g = torch.Generator().manual_seed(seed + 1000)
    t = sh.torch_type(type_)
    if wide:
        return torch.randn(n_q, heads + 2, dim, generator=g).to(t).cuda()[:, 1:-1]
    return torch.randn(heads, n_q, dim + 1, generator=g).to(t).cuda()[:, :, 1:].transpose(0, 1)


def f64(x):
    return x.float().cpu().numpy().astype(np.float64)


def compare(mine, mine_lse, q, k, v, see, scale, group, type_):
    """Outputs of one sequence's queries against the plain form: scores are dim products and as many sums in 32 bits, weights and outputs rounded to
    the queries' type, their sums held in 32 bits."""
    dim, step = q.shape[2], sh.HALF_STEP[type_]
    o, l, size, plain, reach = sh.attend(q, k, v, see, scale, group)
    ds = (dim + 8) * 2.0 ** -24 * reach + 2.0 ** -21
    sums = (see.sum(1)[:, None] + 16) * 2.0 ** -24
    near = (step + 2 * ds + sums)[..., None] * size + step * np.abs(o) + 1e-30
    if type_ == "f16":
        near = near + 2.0 ** -25 * plain + 2.0 ** -25     # weights and outputs below the least normal number
    none = np.isinf(l)
    assert np.array_equal(none, np.isinf(mine_lse)) and (mine_lse[none] < 0).all()
    mine_lse, l = np.where(none, 0, mine_lse), np.where(none, 0, l)
    assert (np.abs(mine_lse - l) <= ds + sums + 2.0 ** -22 * np.abs(l))[~none].all()
    assert (mine[none] == 0).all()
    far = np.abs(mine - o) - near
    assert (far <= 0).all(), (np.unravel_index(far.argmax(), far.shape), far.max())


def status(ctx):
    from paper_2605_16637_amd import binding
    try:
        ctx.hx_stream_status()
    except binding.HxError as e:
        return e.code
    return 0


def bounds_of(stored, filled):
    """[.., T, dim] numbers and how many of T are filled -> [.., 2, dim] bounds; NaNs count in none."""
    y = stored[..., :filled, :]
    lo, hi = np.where(np.isnan(y), np.inf, y).min(-2), np.where(np.isnan(y), -np.inf, y).max(-2)
    return np.stack([lo, hi], -2)


def choose(bounds, there, own, q, sign, n_pages, n_first, n_last):
    """Pages 0 .. own of one KV head that one query sees: bounds [own + 1, 2, dim], there [own + 1], q [group, dim]."""
    pages = [b for b in range(own + 1) if there[b]]
    if own + 1 <= n_pages:
        return pages
    fixed = [b for b in pages if b < n_first or b > own - n_last]
    score = {}
    with np.errstate(invalid="ignore"):
        for b in pages:
            if b in fixed:
                continue
            x = q * sign
            s = (x * np.where(x < 0, bounds[b, 0], bounds[b, 1])).sum(1)
            score[b] = max(np.inf if np.isnan(y) else y for y in s)
    best = sorted((b for b in score if score[b] > -np.inf), key=lambda b: (-score[b], b))
    return sorted(fixed + best[:n_pages - len(fixed)])


def evict(c, weight, rows, n_keep, n_first, n_last):
    """The rules of eviction on a cache's tables and pages (c: table, length, ref, T; pages: {name: [layers, pages, heads, T, ..]}); returns errors and
    the positions kept, for each row None where it is left."""
    T, errors, kept, seen = c.T, set(), [], set()
    plans, free = [], [p for p in range(len(c.ref)) if c.ref[p] == 0]
    first_ref = c.ref.copy()
    out = False
    for r in rows:
        twice = r in seen
        seen.add(r)
        if not 0 <= r < len(c.length) or twice or not 0 <= c.length[r] <= c.table.shape[1] * T:
            errors.add(-6)
            kept.append(None)
            continue
        n = int(c.length[r])
        if n <= n_keep:
            kept.append(None)
            continue
        page = lambda b: c.table[r][b] if 0 <= c.table[r][b] < len(c.ref) else -1  # noqa: E731
        there = [y for y in range(n) if page(y // T) >= 0]
        fixed = [y for y in there if y < n_first or y >= n - n_last]
        w = lambda y: weight[r][y] if weight[r][y] > 0 else 0.0  # noqa: E731
        others = sorted((y for y in there if n_first <= y < n - n_last), key=lambda y: (-w(y), y))
        stay = sorted(fixed + others[:n_keep - len(fixed)])
        m = len(stay)
        changed = {j // T for j in range(m) if stay[j] != j} | ({m // T} if m % T else set())
        new = sorted(b for b in changed if page(b) < 0 or first_ref[page(b)] > 1)
        if new and (out or len(new) > len(free)):
            out = True
            errors.add(-4)
            kept.append(None)
            continue
        plans.append((r, stay, {b: free.pop(0) for b in new}))
        kept.append(stay)
    for r, stay, new in plans:
        n, m, old = int(c.length[r]), len(stay), c.table[r].copy()
        target = [new.get(b, old[b]) for b in range(-(-m // T))]
        for x in c.pages.values():
            y = [x[:, old[s // T], :, s % T].copy() for s in stay]
            for j in range(m):
                x[:, target[j // T], :, j % T] = y[j]
        weight[r][:m] = weight[r][stay]
        weight[r][m:n] = 0.0
        for b in range(-(-n // T)):
            now = target[b] if b < len(target) else -1
            if now != old[b]:
                c.table[r][b] = now
                if 0 <= old[b] < len(c.ref):
                    c.ref[old[b]] -= 1
        for p in new.values():
            c.ref[p] = 1
        c.length[r] = m
    return errors, kept
