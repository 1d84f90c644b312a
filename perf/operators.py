"""The serving step of a decode instance, as cases that can be timed: the pages of its cache, the attention that reads
them, and the sampling of the tokens that answer a call.

The calls that the scheduler has placed live in a paged cache (``hx_kv_*``), are attended to over it (``hx_attend``: a
tree of drafted tokens, a sliding window with a few first tokens that stay visible) and answered by ``hx_sample``.
Geometry and lengths are those of ``synth``: 32 layers, 8 KV heads of 128 numbers (4 query heads each: 4096 in all),
16-bit, prompts of 64 to 32768 tokens around 1500, up to 256 sequences in a batch.

``own`` chooses between the plain form (elementary torch operations) and the library's entry points.
"""
import math

import numpy as np
import torch

own = False

DEV = "cuda:0"
TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32, "e4m3": torch.float8_e4m3fn}
SIZE = {"bf16": 2, "f16": 2, "f32": 4, "e4m3": 1}


def listed():
    return [
        # one agent's call fans out: four siblings start from its prompt and the call itself ends; what a fork costs at least
        dict(name="fork one call", kind="fork", type="bf16", layers=32, heads=8, dim=128, page=16, parents=1, children=4,
             median=1500, most=32768, lengths=1),
        # a busy instance's round of reveals: 64 calls end, four children of each begin
        dict(name="fork a round", kind="fork", type="f16", layers=32, heads=8, dim=128, page=32, parents=64, children=4,
             median=1500, most=32768, lengths=2),
        # a windowed model's cache after a while: what left the windows is given back, then the pages in use move together
        dict(name="compact after a window", kind="compact", type="bf16", layers=32, heads=8, dim=128, page=16, rows=24,
             window=1024, sinks=4, median=1500, most=8192, lengths=3),
        # one layer's cache work of a drafting step: room, keys and values of the drafts, then the accepted path kept
        dict(name="draft step's pages", kind="step", type="bf16", heads=8, dim=128, page=16, rows=64, drafts=32, median=1500,
             most=8192, lengths=4),
        # one sequence checks eight drafted tokens: latency
        dict(name="tree one sequence", kind="tree", type="bf16", cache="bf16", heads=8, group=4, dim=128, page=16, rows=1, drafts=8,
             median=1500, most=2048, lengths=5),
        # a batch of ordinary lengths and an odd number of drafts, some of them padding
        dict(name="tree batch", kind="tree", type="f16", cache="f16", heads=8, group=4, dim=128, page=16, rows=24, drafts=25,
             median=1500, most=8192, lengths=6),
        # long contexts in an 8-bit cache, a wide tree
        dict(name="tree long 8 bit", kind="tree", type="bf16", cache="e4m3", heads=8, group=4, dim=128, page=64, rows=16, drafts=64,
             median=16384, most=32768, lengths=7),
        # one sequence decodes a token with a window that it has not filled: latency, heads of 64, one query head a KV head
        dict(name="window one token", kind="window", type="f16", cache="f16", heads=16, group=1, dim=64, page=16, rows=1, queries=1,
             window=1024, sinks=4, median=777, most=2048, lengths=8),
        # a full batch decodes, mixed lengths up to the longest
        dict(name="window decode batch", kind="window", type="bf16", cache="bf16", heads=8, group=4, dim=128, page=16, rows=256,
             queries=1, window=4096, sinks=4, median=4000, most=32768, lengths=9),
        # ragged prompts prefilled in one go
        dict(name="window prefill", kind="window", type="bf16", cache="bf16", heads=8, group=4, dim=128, page=32, rows=3, queries=6144,
             window=2048, sinks=4, median=5000, most=8192, lengths=10),
        # one answer's next token from full-precision logits
        dict(name="sample one row", kind="sample", type="f32", rows=1, vocab=32000, greedy=0.0, seed=11),
        # a full batch over a large, odd vocabulary, every row with settings of its own
        dict(name="sample batch", kind="sample", type="bf16", rows=256, vocab=131071, greedy=0.1, seed=12),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["fork", "compact", "step", "tree", "tree", "window", "window", "sample", "sample"])
    seed = rng.randint(100, 1 << 30)
    if kind == "sample":
        vocab = _log(rng, 500, 200000)
        return dict(kind=kind, type=rng.choice(["bf16", "f16", "f32"]), rows=_log(rng, 1, min(512, 33000000 // vocab)), vocab=vocab,
                    greedy=rng.choice([0.0, 0.3]), seed=seed)
    type_, dim, page = rng.choice(["bf16", "f16"]), rng.choice([64, 128, 128]), rng.choice([8, 16, 32, 64])
    if kind == "fork":
        parents = _log(rng, 1, 48)
        return dict(kind=kind, type=type_, layers=rng.randint(1, 32), heads=rng.choice([1, 2, 4, 8]), dim=dim, page=min(page, 32),
                    parents=parents, children=rng.randint(1, 5), median=_log(rng, 100, 1500), most=8192, lengths=seed)
    if kind == "compact":
        return dict(kind=kind, type=type_, layers=rng.randint(1, 32), heads=rng.choice([1, 2, 4, 8]), dim=dim, page=page,
                    rows=_log(rng, 2, 40), window=_log(rng, 128, 1024), sinks=rng.choice([0, 4, 17]), median=_log(rng, 300, 1500),
                    most=4096, lengths=seed)
    if kind == "step":
        return dict(kind=kind, type=type_, heads=rng.choice([1, 2, 4, 8]), dim=dim, page=page, rows=_log(rng, 1, 128),
                    drafts=rng.randint(1, 48), median=_log(rng, 100, 1500), most=8192, lengths=seed)
    cache = rng.choice([type_, type_, "e4m3"])
    heads, group = rng.choice([(1, 8), (2, 7), (4, 4), (8, 4), (8, 1), (8, 5)])
    median = _log(rng, 60, 12000)
    most = min(32768, 4 * median)
    if kind == "tree":
        drafts = rng.randint(2, 64)
        return dict(kind=kind, type=type_, cache=cache, heads=heads, group=group, dim=dim, page=page,
                    rows=_log(rng, 1, max(1, min(32, 4000000 // (most * 4)))), drafts=drafts, median=median, most=most, lengths=seed)
    if rng.random() < 0.6:
        rows, queries = _log(rng, 1, max(1, min(200, 2000000 // most))), 1
    else:
        median = min(median, 2000)
        most = 4 * median
        rows, queries = rng.randint(1, 3), rng.randint(2, 1500)
    return dict(kind=kind, type=type_, cache=cache, heads=heads, group=group, dim=dim, page=page, rows=rows, queries=queries,
                window=_log(rng, 100, 4096), sinks=rng.choice([0, 1, 4, 33]), median=median, most=most, lengths=seed)


# ---- what a case is made of ------------------------------------------------------------------------------------------

def _lengths(case):
    """Tokens of each sequence: log-normal around the median, as synth draws prompts."""
    n = case["parents"] if case["kind"] == "fork" else case["rows"]
    rng = np.random.default_rng(case["lengths"])
    x = np.rint(np.exp(np.log(case["median"]) + 0.7 * rng.standard_normal(n)))
    return np.clip(x, 40, case["most"]).astype(np.int64)


def _queries(case, lens):
    """Queries of each sequence: one, or ragged prompts whose first has the most (no more than the sequence has tokens)."""
    most = case["drafts"] if case["kind"] in ("tree", "step") else case["queries"]
    rng = np.random.default_rng(case["lengths"] + 1)
    q = np.full(len(lens), most) if most == 1 or case["kind"] == "step" else np.maximum(1, np.rint(most * rng.uniform(0.5, 1.0, len(lens))))
    q = q.astype(np.int64)
    q[0] = most
    return np.minimum(q, lens)


def _parents(case, nq):
    """Trees of drafts: each token's parent is one of the tokens before it (-1: the last token of the context, -2: padding)."""
    rng = np.random.default_rng(case["lengths"] + 2)
    out = []
    for n in nq:
        p = np.array([rng.integers(max(-1, i - 6), i) for i in range(n)], np.int64)
        if n > 10:
            p[-2:] = -2            # trees are padded to a common size
        out.append(p)
    return out


def _visible(case):
    """Pairs of a query and a key that it sees, over all sequences, and keys that any query of their sequence sees."""
    lens = _lengths(case)
    nq = _queries(case, lens)
    if case["kind"] == "tree":
        pairs = 0
        for n, q, par in zip(lens, nq, _parents(case, nq)):
            depth = []
            for p in par:
                depth.append(1 if p == -1 else 0 if p == -2 else depth[p] + 1)
            pairs += sum((n - q) + d for d in depth if d)
        return int(pairs), int(lens.sum())
    w, s = case["window"], case["sinks"]
    pairs = keys = 0
    for n, q in zip(lens, nq):
        p = np.arange(n - q, n)
        lo = np.maximum(p - w + 1, 0)
        pairs += int((p - lo + 1 + np.minimum(s, lo)).sum())
        keys += int(n - lo[0] + min(s, lo[0]))
    return pairs, keys


def work(case):
    if case["kind"] == "sample":
        n = case["rows"] * case["vocab"]
        return {"bytes": n * SIZE[case["type"]] + case["rows"] * 28, "flops": 4 * n}
    lens, T = _lengths(case), case["page"]
    token = 2 * case["heads"] * case["dim"] * SIZE[case.get("cache", case["type"])]      # K and V of one token in one layer
    if case["kind"] == "fork":
        shared = int((lens // T).sum()) * case["children"]
        tail = int((lens % T).sum()) * case["children"]
        return {"bytes": tail * token * case["layers"] * 2 + shared * 4 + int(-(-lens // T).sum()) * 4, "flops": shared}
    if case["kind"] == "compact":
        free, n_pages = _window_pages(case)
        gone = sum(len(x) for x in free)
        used = int((-(-lens // T)).sum()) - gone
        # pages lie at random over the pool: of those in use the share beyond the first `used` pages moves
        moved = used * (n_pages - used) // n_pages
        return {"bytes": moved * T * token * case["layers"] * 2 + n_pages * 12, "flops": n_pages}
    nq = _queries(case, lens)
    if case["kind"] == "step":
        kept = sum(len(k) for k in _kept(case, nq))
        return {"bytes": int(nq.sum()) * token * 2 + kept * token * 2, "flops": int(nq.sum())}
    pairs, keys = _visible(case)
    hq = case["heads"] * case["group"]
    return {"bytes": keys * token + int(nq.sum()) * hq * (2 * case["dim"] * SIZE[case["type"]] + 4),
            "flops": 4 * case["dim"] * hq * pairs}


def _window_pages(case):
    """Pages of each row that lie wholly between the sinks and the window, and the pool's size (a third over what the rows hold)."""
    T, out, held = case["page"], [], 0
    for n in _lengths(case):
        first, last = case["sinks"], max(case["sinks"], int(n) - case["window"])
        out.append([b for b in range(int(n) // T) if b * T >= first and (b + 1) * T <= last])
        held += -(-int(n) // T)
    return out, held + held // 3 + 8


def _kept(case, nq):
    rng = np.random.default_rng(case["lengths"] + 3)
    return [np.sort(rng.permutation(int(q))[:rng.integers(0, min(int(q), 6) + 1)]) for q in nq]


# ---- prepare ---------------------------------------------------------------------------------------------------------

def _dev(x, dtype=torch.int32):
    return torch.as_tensor(np.ascontiguousarray(x)).to(DEV, dtype)


def _cache_type(x, name):
    return x.to(TYPES[name])


def _pool(case, gen, n_pages, layers, cache):
    shape = (layers, n_pages, case["heads"], case["page"], case["dim"])
    pool = dict(page_tokens=case["page"], ref=torch.zeros(n_pages, dtype=torch.int32, device=DEV))
    for name in ("k", "v"):
        x = torch.empty(shape, dtype=TYPES[cache], device=DEV)
        for l in range(layers):                                                   # a layer at a time: the numbers are made in 32 bits
            y = torch.randn(shape[1:], generator=gen, device=DEV)
            x[l] = _cache_type(y * 40 if cache == "e4m3" else y, cache)
        pool[name] = x
        if cache == "e4m3":
            pool[name + "_scale"] = (torch.rand(layers, case["heads"], generator=gen, device=DEV) + 0.5) / 40
    return pool


def _tables(rng, lens, T, rows, max_pages, n_pages):
    """Tables of `rows` rows whose first hold the sequences, on pages taken from the pool at random, and the pages' counts."""
    table, ref = np.full((rows, max_pages), -1, np.int64), np.zeros(n_pages, np.int64)
    order, at = rng.permutation(n_pages), 0
    for i, n in enumerate(lens):
        k = -(-int(n) // T)
        table[i, :k] = order[at:at + k]
        at += k
    ref[order[:at]] = 1
    return _dev(table), _dev(ref)


def prepare(case, seed):
    rng = np.random.default_rng(seed)
    gen = torch.Generator(device=DEV).manual_seed(seed)
    kind = case["kind"]
    st = dict(case=case)
    if own:
        from paper_2605_16637_amd import binding
        st["ctx"] = binding.Context(0)
    if kind == "sample":
        return {**st, **_prepare_sample(case, rng, gen)}
    lens, T = _lengths(case), case["page"]
    held = int((-(-lens // T)).sum())
    rows, max_pages, layers, cache = len(lens), int(-(-lens.max() // T)), case.get("layers", 1), case.get("cache", case["type"])
    if kind == "fork":
        forks = case["parents"] * case["children"]
        n_pages, rows = held + forks + 5, case["parents"] + forks
        st.update(src=_dev(np.repeat(np.arange(case["parents"]), case["children"])), dst=_dev(case["parents"] + rng.permutation(forks)),
                  over=_dev(np.arange(case["parents"])))
    elif kind == "compact":
        n_pages = _window_pages(case)[1]
        last = np.maximum(case["sinks"], lens - case["window"])
        st.update(row=_dev(np.arange(rows)), first=_dev(np.full(rows, case["sinks"])), last=_dev(last),
                  n_used=torch.zeros(1, dtype=torch.int32, device=DEV), moved=torch.zeros(n_pages, dtype=torch.int32, device=DEV))
    else:
        n_pages = held + held // 4 + 3
        nq = _queries(case, lens)
        if kind == "step":
            n_pages += rows * (-(-case["drafts"] // T) + 1)
            max_pages += -(-case["drafts"] // T)
    st["pool"] = _pool(case, gen, n_pages, layers, cache)
    table, ref = _tables(rng, lens, T, rows, max_pages, n_pages)
    length = torch.zeros(rows, dtype=torch.int32, device=DEV)
    length[:len(lens)] = _dev(lens)
    st["pool"]["ref"].copy_(ref)
    st["seqs"] = dict(table=table, len=length)
    st["was"] = dict(table=table.clone(), len=length.clone(), ref=ref.clone())
    if kind in ("fork", "compact"):
        return st
    ptr = np.concatenate([[0], np.cumsum(nq)])
    st.update(row=_dev(rng.permutation(rows) if kind == "step" else np.arange(rows)), q_ptr=_dev(ptr), n_new=_dev(nq))
    n = int(ptr[-1])
    if kind == "step":
        kept = _kept(case, nq)
        shape = (n, case["heads"], case["dim"])
        st.update(k_new=_cache_type(torch.randn(shape, generator=gen, device=DEV), cache), v_new=_cache_type(torch.randn(shape, generator=gen, device=DEV), cache),
                  keep_ptr=_dev(np.concatenate([[0], np.cumsum([len(k) for k in kept])])), keep=_dev(np.concatenate(kept + [[]])))
        return st
    hq = case["heads"] * case["group"]
    # queries lie between keys and values, as one projection writes them
    qkv = torch.randn(n, hq + 2 * case["heads"], case["dim"], generator=gen, device=DEV).to(TYPES[case["type"]])
    st.update(q=qkv[:, :hq], out=torch.empty(n, hq, case["dim"], dtype=TYPES[case["type"]], device=DEV), lse=torch.empty(n, hq, device=DEV),
              max_q=int(nq.max()), max_len=int(lens.max()), parent=None, window=0, sinks=0)
    if kind == "tree":
        st["parent"] = _dev(np.concatenate(_parents(case, nq)))
    else:
        st.update(window=case["window"], sinks=case["sinks"])
    return st


def _prepare_sample(case, rng, gen):
    n, v = case["rows"], case["vocab"]
    x = 2.5 * torch.randn(n, v, generator=gen, device=DEV)
    few = torch.randint(0, v, (n, 40), generator=gen, device=DEV)                 # some tokens stand out
    x.scatter_add_(1, few, 6 * torch.rand(n, 40, generator=gen, device=DEV))
    x[:, torch.randint(0, v, (v // 50 + 1,), generator=gen, device=DEV)] = -math.inf    # and some are barred
    t = np.where(rng.random(n) < case["greedy"], 0.0, rng.uniform(0.5, 1.3, n))
    top_k = np.where(rng.random(n) < 0.5, rng.integers(1, 200, n), 0)
    top_p = np.where(rng.random(n) < 0.6, rng.uniform(0.6, 0.99, n), 1.0)
    min_p = np.where(rng.random(n) < 0.3, rng.uniform(0.01, 0.1, n), 0.0)
    i32 = lambda: torch.empty(n, dtype=torch.int32, device=DEV)  # noqa: E731
    f32 = lambda a: _dev(a, torch.float32)  # noqa: E731
    return dict(logits=x.to(TYPES[case["type"]]), temperature=f32(t), top_k=_dev(top_k), top_p=f32(top_p), min_p=f32(min_p),
                u=torch.rand(n, generator=gen, device=DEV), token=i32(), n_kept=i32(), logprob=torch.empty(n, device=DEV))


# ---- run -------------------------------------------------------------------------------------------------------------

def run(st):
    kind, ctx = st["case"]["kind"], st.get("ctx")
    if kind == "sample":
        if not own:
            return plain_sample(st["logits"], st["temperature"], st["top_k"], st["top_p"], st["min_p"], st["u"])
        ctx.hx_sample(st["logits"], st["u"], st["token"], temperature=st["temperature"], top_k=st["top_k"], top_p=st["top_p"],
                      min_p=st["min_p"], logprob=st["logprob"], n_kept=st["n_kept"])
        return dict(token=st["token"], logprob=st["logprob"], n_kept=st["n_kept"])
    pool, seqs = st["pool"], st["seqs"]
    if kind in ("tree", "window"):
        if not own:
            return plain_attend(pool, seqs, st["row"], st["q_ptr"], st["max_q"], st["max_len"], st["q"], st["window"], st["sinks"], st["parent"])
        ctx.hx_attend(pool, 0, seqs, st["q_ptr"], st["q"], st["out"], max_q=st["max_q"], max_len=st["max_len"], row=st["row"],
                      window=st["window"], n_sink=st["sinks"], parent=st["parent"], lse=st["lse"])
        return dict(out=st["out"], lse=st["lse"])
    # every pass starts from the same tables
    seqs["table"].copy_(st["was"]["table"]); seqs["len"].copy_(st["was"]["len"]); pool["ref"].copy_(st["was"]["ref"])
    more = {}
    if kind == "fork":
        if own:
            ctx.hx_kv_fork(pool, seqs, st["src"], st["dst"])
            ctx.hx_kv_free(pool, seqs, st["over"])
        else:
            plain_fork(pool, seqs, st["src"].long(), st["dst"].long())
            plain_free(pool, seqs, st["over"].long())
    elif kind == "compact":
        if own:
            ctx.hx_kv_free(pool, seqs, st["row"], st["first"], st["last"])
            ctx.hx_kv_compact(pool, seqs, n_used=st["n_used"], moved=st["moved"])
            more = dict(n_used=st["n_used"], moved=st["moved"])
        else:
            plain_free(pool, seqs, st["row"].long(), st["first"], st["last"])
            more = plain_compact(pool, seqs)
    elif own:
        ctx.hx_kv_grow(pool, seqs, st["row"], st["n_new"])
        ctx.hx_kv_write(pool, 0, seqs, st["row"], st["q_ptr"], st["k_new"], st["v_new"])
        ctx.hx_kv_keep(pool, seqs, st["row"], st["n_new"], st["keep_ptr"], st["keep"])
    else:
        row, n_new = st["row"].long(), st["n_new"].long()
        plain_grow(pool, seqs, row, n_new)
        plain_write(pool, seqs, row, n_new, st["k_new"], st["v_new"])
        plain_keep(pool, seqs, row, n_new, st["keep_ptr"].long(), st["keep"].long())
    return dict(k=pool["k"], v=pool["v"], table=seqs["table"], len=seqs["len"], ref=pool["ref"], **more)


# ---- the plain forms -------------------------------------------------------------------------------------------------

def _free_pages(pool, n):
    return (pool["ref"] == 0).nonzero()[:n, 0]


def _count(ref, pages, by):
    ref.index_add_(0, pages, torch.full_like(pages, by, dtype=torch.int32))


def plain_fork(pool, seqs, src, dst):
    T, table = pool["page_tokens"], seqs["table"]
    t = seqs["len"][src].long()
    whole, part = t // T, t % T > 0
    cols = torch.arange(table.shape[1], device=DEV)
    shared = torch.where(cols[None] < whole[:, None], table[src], -1)
    old, new = table[src[part], whole[part]].long(), _free_pages(pool, int(part.sum()))
    table[dst] = shared
    table[dst[part], whole[part]] = new.int()
    seqs["len"][dst] = t.int()
    _count(pool["ref"], shared[shared >= 0].long(), 1)
    pool["ref"][new] = 1
    i, off = (torch.arange(T, device=DEV)[None] < (t % T)[part][:, None]).nonzero(as_tuple=True)
    for x in (pool["k"], pool["v"]):
        x[:, new[i], :, off] = x[:, old[i], :, off]


def plain_free(pool, seqs, row, first=None, last=None):
    T, table, length = pool["page_tokens"], seqs["table"], seqs["len"]
    held = table[row]
    if first is None:
        gone = held >= 0
        length[row] = 0
    else:
        b = torch.arange(table.shape[1], device=DEV)[None] * T
        gone = (held >= 0) & (b >= first[:, None]) & (b + T <= torch.minimum(last, length[row])[:, None])
    _count(pool["ref"], held[gone].long(), -1)
    table[row] = torch.where(gone, -1, held)


def plain_compact(pool, seqs):
    ref, table = pool["ref"], seqs["table"]
    used = ref > 0
    n = used.sum()
    i = torch.arange(ref.numel(), device=DEV)
    high, holes = (used & (i >= n)).nonzero()[:, 0], (~used & (i < n)).nonzero()[:, 0]
    moved = torch.where(used, i, -1).int()
    moved[high] = holes.int()
    for x in (pool["k"], pool["v"]):
        x[:, holes] = x[:, high]
    ref[holes] = ref[high]
    ref[high] = 0
    table.copy_(torch.where(table >= 0, moved[table.clamp(min=0).long()], -1))
    return dict(n_used=n.int().reshape(1), moved=moved)


def plain_grow(pool, seqs, row, n_new):
    T, length = pool["page_tokens"], seqs["len"]
    was = length[row].long()
    have = (was + T - 1) // T
    need = (was + n_new + T - 1) // T - have
    total = int(need.sum())
    pages = _free_pages(pool, total)
    r = torch.repeat_interleave(torch.arange(row.numel(), device=DEV), need)
    col = have[r] + torch.arange(total, device=DEV) - (need.cumsum(0) - need)[r]
    seqs["table"][row[r], col] = pages.int()
    pool["ref"][pages] = 1
    length[row] = (was + n_new).int()


def _tail(seqs, row, count):
    """Sequence, number within it, and position of each of the last `count` tokens of the rows."""
    i = torch.repeat_interleave(torch.arange(row.numel(), device=DEV), count)
    j = torch.arange(i.numel(), device=DEV) - (count.cumsum(0) - count)[i]
    return i, j, (seqs["len"][row].long() - count)[i] + j


def plain_write(pool, seqs, row, n_new, k, v):
    T = pool["page_tokens"]
    i, _, pos = _tail(seqs, row, n_new)
    page = seqs["table"][row[i], pos // T].long()
    pool["k"][0, page, :, pos % T] = k
    pool["v"][0, page, :, pos % T] = v


def plain_keep(pool, seqs, row, n_draft, keep_ptr, keep):
    T, table, length = pool["page_tokens"], seqs["table"], seqs["len"]
    base = length[row].long() - n_draft
    kept = keep_ptr[1:] - keep_ptr[:-1]
    i = torch.repeat_interleave(torch.arange(row.numel(), device=DEV), kept)
    j = torch.arange(i.numel(), device=DEV) - keep_ptr[i]
    frm, to = base[i] + keep, base[i] + j
    p, q = table[row[i], frm // T].long(), table[row[i], to // T].long()
    for x in (pool["k"], pool["v"]):
        x[:, q, :, to % T] = x[:, p, :, frm % T]
    length[row] = (base + kept).int()
    held = table[row]
    gone = (held >= 0) & (torch.arange(table.shape[1], device=DEV)[None] >= ((base + kept + T - 1) // T)[:, None])
    _count(pool["ref"], held[gone].long(), -1)
    table[row] = torch.where(gone, -1, held)


def _ancestors(parent):
    """[n, q, q]: whether token y is token x or above it, from parents [n, q] (-1 top, -2 none), by doubling the steps."""
    n, q = parent.shape
    up = torch.zeros(n, q, q + 1, device=DEV).scatter_(2, torch.where(parent >= 0, parent, q)[..., None], 1.0)[..., :q]
    reach = up + torch.eye(q, device=DEV)
    for _ in range(max(1, (q - 1).bit_length())):
        reach = ((reach @ reach) > 0).float()
    return (reach > 0) & (parent != -2)[..., None]


def plain_attend(pool, seqs, row, q_ptr, max_q, max_len, q, window, sinks, parent):
    T, H = pool["page_tokens"], pool["k"].shape[2]
    n, (total, hq, dim) = row.numel(), q.shape
    g = hq // H
    length, first = seqs["len"][row.long()].long(), q_ptr[:-1].long()
    nq = q_ptr[1:].long() - first
    t = torch.arange(max_q, device=DEV)
    real = t[None] < nq[:, None]                                                   # [n, max_q]
    at = torch.where(real, first[:, None] + t, 0)
    base = length - nq
    # positions that any query of a sequence may see: the sinks, and from the first query's window on
    lo = (base - window + 1).clamp(min=0) if window else torch.zeros_like(base)
    width = min(max_len, window + max_q - 1) if window else max_len
    pos = torch.cat([torch.arange(sinks, device=DEV)[None].expand(n, sinks), lo[:, None] + torch.arange(width, device=DEV)], 1)
    there = (pos < length[:, None]) & ((torch.arange(sinks + width, device=DEV)[None] < sinks) | (pos >= sinks))
    page = seqs["table"][row.long()].gather(1, (pos // T).clamp(max=seqs["table"].shape[1] - 1)).long()
    there &= page >= 0
    page = page.clamp(min=0)
    k, v = (torch.where(there[..., None, None], x[0][page, :, pos % T].float(), 0.0).permute(0, 2, 1, 3).contiguous() for x in (pool["k"], pool["v"]))
    qs = q[at].float().reshape(n, max_q, H, g, dim).permute(0, 2, 3, 1, 4).reshape(n, H, g * max_q, dim)
    s = (qs @ k.transpose(2, 3)).mul_(dim ** -0.5)
    if "k_scale" in pool:
        s.mul_(pool["k_scale"][0][None, :, None, None])
    # which of them a query sees, by position
    draft = pos - base[:, None]                                                    # number among the queries; negative: context
    if parent is None:
        qpos, kpos, seen = base[:, None] + t, pos, pos[:, None] <= base[:, None, None] + t[None, :, None]
    else:
        anc = _ancestors(torch.where(real, parent.long()[at], -2))
        depth = anc.sum(2) - 1
        qpos = base[:, None] + depth
        d = draft.clamp(0, max_q - 1)
        kpos = torch.where(draft >= 0, base[:, None] + depth.gather(1, d), pos)
        seen = torch.where((draft >= 0)[:, None], anc.gather(2, d[:, None].expand(n, max_q, d.shape[1])), anc.any(2)[..., None])
    seen = seen & there[:, None] & real[..., None]
    if window:
        seen &= (kpos[:, None] < sinks) | (qpos[..., None] - kpos[:, None] < window)
    s = s.view(n, H, g, max_q, -1).masked_fill_(~seen[:, None, None], -math.inf)
    top = s.amax(-1, keepdim=True).clamp(min=-3e38)
    s = s.sub_(top).exp_()
    total_w = s.sum(-1, keepdim=True)
    o = (s.view(n, H, g * max_q, -1) @ v).view(n, H, g, max_q, dim) / total_w.clamp(min=1e-38)
    if "v_scale" in pool:
        o = o * pool["v_scale"][0][None, :, None, None, None]
    lse = torch.where(total_w > 0, total_w.log() + top, -math.inf)[..., 0]
    out = o.permute(0, 3, 1, 2, 4).reshape(n, max_q, hq, dim)[real]
    return dict(out=out.to(q.dtype), lse=lse.permute(0, 3, 1, 2).reshape(n, max_q, hq)[real])


def plain_sample(logits, temperature, top_k, top_p, min_p, u):
    x = logits.double()                         # values beside a border decide a token: 64 bits
    v = x.shape[1]
    x, order = x.sort(dim=1, descending=True, stable=True)
    t = temperature.double()[:, None]
    w = torch.where(t > 0, ((x - x[:, :1]) / torch.where(t > 0, t, 1.0)).exp(), 0.0)
    w = torch.where(x == -math.inf, 0.0, w)
    rank = torch.arange(v, device=DEV)[None]
    k = torch.where(t > 0, torch.where(top_k > 0, top_k, v)[:, None], 1)
    w = torch.where(t > 0, w, 1.0)
    keep = (rank < k) & (x > -math.inf)
    w = torch.where(keep, w, 0.0)
    before = w.cumsum(1) - w
    p = top_p.double()[:, None]
    keep &= (p >= 1) | (before < p * w.sum(1, keepdim=True)) | (rank == 0)
    keep &= w >= min_p.double()[:, None]
    w = torch.where(keep, w, 0.0)
    by_index = torch.zeros_like(w).scatter_(1, order, w)
    total = by_index.cumsum(1)
    token = (total <= u.double()[:, None] * total[:, -1:]).sum(1)
    mine = by_index.gather(1, token[:, None].clamp(max=v - 1))[:, 0]
    return dict(token=token.int(), logprob=(mine / total[:, -1]).log().float(), n_kept=keep.sum(1).int())


# ---- the same in 64 bits, apart from the above --------------------------------------------------------------------------

def exact(case, seed):
    if case["kind"] in ("fork", "compact", "step"):
        return None                                    # copies and whole numbers: nothing is computed
    global own
    was, own = own, False
    try:
        st = prepare(case, seed)
    finally:
        own = was
    return _exact_sample(st) if case["kind"] == "sample" else _exact_attend(case, st)


def _exact_attend(case, st):
    pool, T = st["pool"], case["page"]
    lens = _lengths(case)
    nq = _queries(case, lens)
    parents = _parents(case, nq) if case["kind"] == "tree" else None
    table = st["seqs"]["table"].cpu().numpy()
    H, g, dim = case["heads"], case["group"], case["dim"]
    outs, lses = [], []
    at = 0
    for r, (n, m) in enumerate(zip(lens, nq)):
        n, m = int(n), int(m)
        mask = np.zeros((m, n), bool)
        for i in range(m):
            if parents is None:
                p = n - m + i
                mask[i, :p + 1] = True
                mask[i, case["sinks"]:max(case["sinks"], p - case["window"] + 1)] = False
            else:
                if parents[r][i] == -2:
                    continue
                mask[i, :n - m] = True
                a = i
                while a >= 0:
                    mask[i, n - m + a] = True
                    a = parents[r][a]
        mask = torch.as_tensor(mask, device=DEV)
        pages = torch.as_tensor(table[r, :-(-n // T)].astype(np.int64), device=DEV)
        o, l = torch.empty(m, H, g, dim, dtype=torch.float64, device=DEV), torch.empty(m, H, g, dtype=torch.float64, device=DEV)
        for h in range(H):
            k, v = (pool[x][0, pages, h].double().reshape(-1, dim)[:n] for x in ("k", "v"))
            if "k_scale" in pool:
                k, v = k * pool["k_scale"][0, h].double(), v * pool["v_scale"][0, h].double()
            for e in range(g):
                s = st["q"][at:at + m, h * g + e].double() @ k.T / math.sqrt(dim)
                s[~mask] = -math.inf
                l[:, h, e] = torch.logsumexp(s, 1)
                o[:, h, e] = torch.softmax(s, 1) @ v
        o[~mask.any(1)] = 0.0
        outs.append(o.reshape(m, H * g, dim))
        lses.append(l.reshape(m, H * g))
        at += m
    return dict(out=torch.cat(outs), lse=torch.cat(lses))


def _exact_sample(st):
    x = st["logits"].double().cpu().numpy()
    t, k, p, mp, u = (st[n].cpu().numpy().astype(np.float64) for n in ("temperature", "top_k", "top_p", "min_p", "u"))
    token, logprob, kept = [], [], []
    for r in range(x.shape[0]):
        order = np.argsort(-x[r], kind="stable")
        order = order[x[r][order] > -np.inf]
        if t[r] == 0:
            order, w = order[:1], np.ones(1)
        else:
            if k[r] > 0:
                order = order[:int(k[r])]
            w = np.exp((x[r][order] - x[r][order[0]]) / t[r])
            if p[r] < 1:
                order = order[:max(1, np.searchsorted(np.cumsum(w) - w, p[r] * w.sum(), side="left"))]
                w = w[:len(order)]
            order, w = order[w >= mp[r]], w[w >= mp[r]]
        by = np.argsort(order)
        c = np.cumsum(w[by])
        i = int(np.searchsorted(c, u[r] * c[-1], side="right"))
        token.append(order[by][i]); logprob.append(np.log(w[by][i] / c[-1])); kept.append(len(order))
    return dict(token=np.array(token, np.int32), logprob=np.array(logprob), n_kept=np.array(kept, np.int32))
