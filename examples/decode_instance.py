"""What a decode instance does with the calls that the placement search has put on it, with the library's serving entry points: a prompt is
prefilled, the calls revealed below it start from its cache (``hx_kv_fork``), drafts are checked as a tree and the accepted ones kept
(``hx_attend``, ``hx_kv_keep``), tokens are drawn (``hx_sample``), pages that a window has left are given back, and the rest moves together.

The model is one attention layer of random weights: enough to take every step in earnest, with nothing to learn from its words.

    python examples/decode_instance.py [--steps 8] [--window 256]
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2605_16637_amd import binding  # noqa: E402

KV_HEADS, GROUP, DIM, VOCAB, PAGE = 2, 4, 64, 1000, 16
HEADS = KV_HEADS * GROUP


def i32(x):
    return torch.as_tensor(x, dtype=torch.int32, device="cuda:0")


class Instance:
    """A cache of ``pages`` pages for up to ``rows`` calls, and a model to fill it."""

    def __init__(self, rows=16, pages=256, window=256, sinks=4, seed=0):
        g = torch.Generator("cuda:0").manual_seed(seed)
        half = dict(dtype=torch.bfloat16, device="cuda:0")
        self.ctx, self.window, self.sinks, self.gen = binding.Context(0), window, sinks, g
        shape = (1, pages, KV_HEADS, PAGE, DIM)
        self.pool = dict(k=torch.zeros(shape, **half), v=torch.zeros(shape, **half), ref=i32([0] * pages))
        self.seqs = dict(table=i32([[-1] * pages] * rows), len=i32([0] * rows))
        width = HEADS * DIM
        self.embed = torch.randn(VOCAB, width, generator=g, **half)
        self.qkv = torch.randn(width, (HEADS + 2 * KV_HEADS) * DIM, generator=g, **half) * width ** -0.5
        self.head = torch.randn(width, VOCAB, generator=g, **half) * 2 * width ** -0.5

    def forward(self, rows, tokens, ptr, parent=None):
        """Tokens ptr[i] .. ptr[i+1]-1 go to the end of row rows[i] (as a tree of drafts if they have parents); logits of each."""
        n_new = ptr.diff()
        qkv = (self.embed[tokens.long()] @ self.qkv).view(len(tokens), HEADS + 2 * KV_HEADS, DIM)
        q, k, v = qkv[:, :HEADS], qkv[:, HEADS:HEADS + KV_HEADS], qkv[:, HEADS + KV_HEADS:]
        out = torch.empty(len(tokens), HEADS, DIM, dtype=torch.bfloat16, device="cuda:0")
        self.ctx.hx_kv_grow(self.pool, self.seqs, rows, n_new)
        self.ctx.hx_kv_write(self.pool, 0, self.seqs, rows, ptr, k, v)
        self.ctx.hx_attend(self.pool, 0, self.seqs, ptr, q, out, max_q=int(n_new.max()), row=rows, window=self.window, n_sink=self.sinks, parent=parent)
        return out.view(len(tokens), -1) @ self.head * 8

    def sample(self, logits, temperature=0.3, top_k=50, top_p=0.95):
        n = len(logits)
        token, logprob = torch.empty(n, dtype=torch.int32, device="cuda:0"), torch.empty(n, device="cuda:0")
        full = lambda x: torch.full((n,), x, device="cuda:0")  # noqa: E731
        self.ctx.hx_sample(logits, torch.rand(n, generator=self.gen, device="cuda:0"), token, temperature=full(temperature), top_k=i32([top_k] * n),
                           top_p=full(top_p), logprob=logprob)
        return token, logprob

    def check_drafts(self, rows, roots, likely, drafts):
        """A tree of drafts below each row's newest token (roots): ``drafts`` tokens, two below each token, the two that were likeliest one
        step ago.  Keeps the path that follows the tokens drawn, and returns how many drafts each row accepted, the token drawn after them
        and the logits that it was drawn from."""
        n, m = len(rows), drafts + 1
        parent = [-1] + [(i - 1) // 2 for i in range(1, m)]
        tokens = torch.cat([roots[:, None], likely.topk(2).indices.int().repeat(1, drafts // 2)], 1)
        logits = self.forward(rows, tokens.reshape(-1), i32(range(0, n * m + 1, m)), i32(parent * n))
        drawn, _ = self.sample(logits)
        drawn, tokens, keep, last = drawn.view(n, m).tolist(), tokens.tolist(), [], []
        for i in range(n):
            path = [0]
            while True:
                below = [j for j in (2 * path[-1] + 1, 2 * path[-1] + 2) if j < m and tokens[i][j] == drawn[i][path[-1]]]
                if not below:
                    break
                path.append(below[0])
            keep.append(path)
            last.append(drawn[i][path[-1]])
        ends = [0]
        for path in keep:
            ends.append(ends[-1] + len(path))
        self.ctx.hx_kv_keep(self.pool, self.seqs, rows, i32([m] * n), i32(ends), i32(sum(keep, [])))
        return [len(path) - 1 for path in keep], i32(last), logits.view(n, m, VOCAB)[range(n), [path[-1] for path in keep]]

    def tidy(self):
        """Pages between the sinks and the windows go, the rest moves together; how many are in use."""
        n_used, length = torch.zeros(1, dtype=torch.int32, device="cuda:0"), self.seqs["len"]
        rows = torch.arange(len(length), dtype=torch.int32, device="cuda:0")
        self.ctx.hx_kv_free(self.pool, self.seqs, rows, torch.full_like(length, self.sinks), (length - self.window).clamp(min=0))
        self.ctx.hx_kv_compact(self.pool, self.seqs, n_used=n_used)
        return int(n_used)


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--steps", type=int, default=8)
    ap.add_argument("--window", type=int, default=256)
    ap.add_argument("--prompt", type=int, default=700)
    ap.add_argument("--children", type=int, default=4)
    a = ap.parse_args(argv)
    inst = Instance(window=a.window)
    prompt = torch.randint(0, VOCAB, (a.prompt,), generator=inst.gen, device="cuda:0", dtype=torch.int32)
    logits = inst.forward(i32([0]), prompt, i32([0, a.prompt]))
    n = a.children
    rows = i32(range(1, n + 1))
    inst.ctx.hx_kv_fork(inst.pool, inst.seqs, i32([0] * n), rows)           # the calls below start from the prompt's pages
    inst.ctx.hx_kv_free(inst.pool, inst.seqs, i32([0]))                     # and the call that ends gives its own back
    token, _ = inst.sample(logits[-1:].expand(n, VOCAB).contiguous())
    answers = [[t] for t in token.tolist()]
    for step in range(a.steps):
        if step % 2:
            accepted, token, logits = inst.check_drafts(rows, token, logits, 6)
        else:
            logits = inst.forward(rows, token, i32(range(n + 1)))
            accepted, token = [0] * n, inst.sample(logits)[0]
        for x, t in zip(answers, token.tolist()):
            x.append(t)
        print(f"step {step}: accepted {accepted}, tokens of each row {inst.seqs['len'][1:n + 1].tolist()}, pages in use {inst.tidy()}", flush=True)
    inst.ctx.hx_stream_status()
    return inst, answers


if __name__ == "__main__":
    main()
