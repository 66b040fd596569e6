"""Several answers to each of several prompts, decoded together with looked-up drafts: one attention layer on the 8-bit paged cache.

    python examples/branching_decode.py [--prompts 8] [--answers 8] [--steps 20] [--drafts 4] [--heads 32 8 128]

Every prompt goes into the cache once; its answers are forks of it (kv_pages_select) that share its pages.  A step, captured once as a HIP
graph and replayed: pages for the next tokens (kv_pages_reserve; a page that answers share is copied before the first of them writes to it, kv_cache_copy), norm,
rotation and cache write (qkv_cache_write), attention that reads the shared pages once (shared_tree_attn), which of the drafted tokens
stay (draft_verify), and their way behind the context (kv_cache_keep).  In the end one answer of each prompt stays, and the pages in use move to the
front of the pool (kv_pages_compact).  There is no model here: a token's projections are a row of a random table, logits are a random
projection of the attention with a preference for the token that a table says comes next.
"""
import argparse
import os
import sys
import time

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from examples.speculative_decode import EPS, PAGE, rotary_table  # noqa: E402
from paper_2602_06072_amd import binding as pk  # noqa: E402


class Model:
    """What a model would be: rows of projections and logits of a token, by tables."""

    def __init__(self, heads, vocab=2000, seed=0):
        self.Hq, self.Hkv, self.d = heads
        self.vocab = vocab
        g = torch.Generator(device="cuda").manual_seed(seed)
        randn = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
        self.rows = randn(vocab, self.Hq + 2 * self.Hkv, self.d).bfloat16()
        self.wq, self.wk = ((1 + 0.1 * randn(self.d)).bfloat16() for _ in "qk")
        self.out = (randn(self.Hq * self.d, vocab) * (self.Hq * self.d) ** -0.5).bfloat16()
        self.next = torch.randint(0, vocab, (vocab,), generator=g, device="cuda", dtype=torch.int32)
        self.table, self.scale = rotary_table(self.d), self.d ** -0.5

    def split(self, tokens):
        x = self.rows[tokens.long()]
        return x[:, :self.Hq], x[:, self.Hq:self.Hq + self.Hkv], x[:, self.Hq + self.Hkv:]

    def logits(self, attention, tokens):
        """(of all rows at once; the looked-up token has about half of the probability)"""
        x = 8.0 * (attention.flatten(1) @ self.out).float()
        return x.scatter_add(1, self.next[tokens.long()].long()[:, None], torch.full((x.shape[0], 1), 7.0, device="cuda"))


class Batch:
    """Pages, lengths and tables of a batch, and a cache for them."""

    def __init__(self, model, blocks, most_pages, n, refs=None, cache=None, dtype=pk.PK_F8):
        i32 = dict(dtype=torch.int32, device="cuda")
        self.model, self.n = model, n
        self.cache = pk.new_kv_cache(blocks, PAGE, model.Hkv, model.d, dtype) if cache is None else cache
        self.refs = torch.zeros(blocks, **i32) if refs is None else refs
        self.table, self.lens, self.pages = torch.zeros(n, most_pages, **i32), torch.zeros(n, **i32), torch.zeros(n, **i32)
        self.served, self.src, self.dst = (torch.zeros(n, **i32) for _ in range(3))
        self.ws = pk.new_pages_workspace(blocks)

    def reserve(self, grow):
        pk.kv_pages_reserve(self.table, self.lens, self.pages, grow, self.refs, PAGE, self.served, self.src, self.dst, self.ws)
        pk.kv_cache_copy(self.cache, self.src, self.dst)           # (of every layer)

    def slots(self, request, position):
        return self.table[request, position // PAGE].long() * PAGE + position % PAGE

    def write(self, tokens, request, position, q_out):
        m = self.model
        q, k, v = m.split(tokens)
        pk.qkv_cache_write(self.cache, q, k, v, self.slots(request, position), q_out, m.wq, m.wk, EPS, pk.Rope(m.table, position.int()))

    def select(self, rows, n):
        """The batch of requests `rows` of this one."""
        new = Batch(self.model, self.refs.numel(), self.table.shape[1], n, self.refs, self.cache)
        pk.kv_pages_select(self.table, self.lens, self.pages, torch.as_tensor(rows, dtype=torch.int32, device="cuda"), new.table, new.lens, new.pages, self.refs, PAGE)
        return new


def prompts(model, batch, tokens):
    """tokens: one sequence for each request of an empty batch."""
    lens = torch.tensor([len(x) for x in tokens], dtype=torch.int32, device="cuda")
    batch.reserve(lens)
    request = torch.repeat_interleave(torch.arange(batch.n, device="cuda"), lens.long())
    position = torch.cat([torch.arange(len(x), device="cuda") for x in tokens])
    rows = torch.as_tensor(np.concatenate(tokens), device="cuda")
    q = torch.empty(len(rows), model.Hq, model.d, dtype=torch.bfloat16, device="cuda")
    batch.write(rows, request, position, q)
    batch.lens.copy_(lens)
    torch.cuda.synchronize()


class Decoder:
    """Steps of a batch on fixed buffers: u and v are to be filled with random numbers; the tokens that stayed are in kept and count."""

    def __init__(self, batch, drafts, last, family_start, shared=True, temperature=0.8):
        n, T, m = batch.n, drafts + 1, batch.model
        self.batch, self.T, self.total, self.shared = batch, T, n * T, shared
        dev = lambda *shape, dtype=torch.int32: torch.zeros(*shape, dtype=dtype, device="cuda")  # noqa: E731
        self.last = torch.as_tensor(last, dtype=torch.int32, device="cuda").clone()       # a request's newest token, not yet in the cache
        self.tokens, self.q, self.out = dev(n, T), dev(n * T, m.Hq, m.d, dtype=torch.bfloat16), dev(n * T, m.Hq, m.d, dtype=torch.bfloat16)
        self.q_start = torch.arange(0, n * T + 1, T, dtype=torch.int32, device="cuda")
        self.grow, self.with_drafts = torch.full((n,), T, dtype=torch.int32, device="cuda"), dev(n)
        self.u, self.v = dev(n * T, dtype=torch.float32), dev(n, dtype=torch.float32)
        self.temperature = torch.full((n,), temperature, device="cuda")
        self.kept, self.count, self.next = dev(n, T), dev(n), dev(n)
        self.family_start = torch.as_tensor(family_start, dtype=torch.int32, device="cuda")
        self.request, self.number = torch.arange(n, device="cuda").repeat_interleave(T), torch.arange(T, device="cuda").repeat(n)
        self.tree_ws = pk.new_shared_tree_workspace(n, T, n * T, m.Hq, m.Hkv, m.d) if shared else pk.new_tree_workspace(n, T, m.Hq, m.Hkv, m.d)
        self.verify_ws = pk.new_verify_workspace(n, n * T, m.vocab)

    def step(self):
        """Nothing of it waits for the host: can be captured."""
        b, m = self.batch, self.batch.model
        x = self.last
        for t in range(self.T):                     # a token and those that are looked up behind it
            self.tokens[:, t] = x
            x = m.next[x.long()]
        tokens = self.tokens.view(-1)
        b.reserve(self.grow)
        b.write(tokens, self.request, b.lens[self.request].long() + self.number, self.q)
        self.with_drafts.copy_(b.lens + self.T)
        args = (b.cache, self.q, self.q_start, self.T, None, b.table, self.with_drafts)
        if self.shared:
            pk.shared_tree_attn(*args, self.family_start, self.out, m.scale, self.tree_ws)
        else:
            pk.tree_attn(*args, self.out, m.scale, self.tree_ws)
        pk.draft_verify(m.logits(self.out, tokens), None, tokens, self.q_start, self.T, None, self.temperature, self.u, self.v,
                        self.kept, self.count, self.next, self.verify_ws)
        pk.kv_cache_keep(b.cache, b.table, self.with_drafts, self.q_start, self.kept, self.count, b.lens)
        self.last.copy_(self.next)


def generate(n=8, answers=8, steps=20, drafts=4, heads=(32, 8, 128), prompt=(200, 1500), seed=0, graph=True, shared=True, dtype=pk.PK_F8, spare=1.1, roomy=1):
    """Returns (model, batch of one answer of each prompt, its sequences, all answers' new tokens, tokens kept by every step, seconds of a step).
    roomy: columns of the block table, over those that are needed."""
    rng = np.random.default_rng(seed)
    model = Model(heads, seed=seed)
    texts = [rng.integers(0, model.vocab, rng.integers(prompt[0], prompt[1] + 1)).astype(np.int32) for _ in range(n)]
    whole = [len(x) // PAGE for x in texts]
    more = (steps + 1) * (drafts + 1) // PAGE + 3
    batch = Batch(model, int((sum(whole) + n * answers * more) * spare), (max(whole) + more) * roomy, n, dtype=dtype)
    prompts(model, batch, texts)
    batch = batch.select(np.repeat(np.arange(n), answers), n * answers)
    dec = Decoder(batch, drafts, rng.integers(0, model.vocab, n * answers), np.arange(0, n * answers + 1, answers), shared)
    first = dec.last.cpu().numpy()
    g = torch.Generator(device="cuda").manual_seed(seed)
    new, took = [[int(x)] for x in first], []
    captured = None
    for s in range(steps):
        dec.u.copy_(torch.rand(dec.total, generator=g, device="cuda"))
        dec.v.copy_(torch.rand(batch.n, generator=g, device="cuda"))
        if graph and s == 1:                        # (the first step loads the kernels; capturing does nothing)
            captured = torch.cuda.CUDAGraph()
            with torch.cuda.graph(captured):
                dec.step()
        torch.cuda.synchronize()
        begin = time.perf_counter()
        captured.replay() if captured else dec.step()
        torch.cuda.synchronize()
        took.append(time.perf_counter() - begin)
        assert bool(batch.served.all()), "the pool is too small"
        kept, count, after, tokens = (x.cpu().numpy() for x in (dec.kept, dec.count, dec.next, dec.tokens))
        for i in range(batch.n):
            new[i] += [int(x) for x in tokens[i, kept[i, 1:count[i]]]] + [int(after[i])]
    # the longest answer of each prompt stays
    lens = batch.lens.cpu().numpy().reshape(n, answers)
    best = np.arange(n) * answers + lens.argmax(1)
    last = batch.select(best, n)
    src, dst = (torch.full((last.refs.numel(),), -1, dtype=torch.int32, device="cuda") for _ in range(2))
    refs = torch.empty_like(last.refs)
    pk.kv_pages_compact(last.table, last.pages, last.refs, last.table, refs, src, dst, last.ws)
    pk.kv_cache_copy(last.cache, src, dst)
    last.refs.copy_(refs)
    sequences = [np.concatenate([texts[i], new[b][:-1]]).astype(np.int32) for i, b in enumerate(best)]      # (the newest token is not in the cache)
    return model, last, sequences, new, float(np.median(took[2:])) if len(took) > 2 else 0.0


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--prompts", type=int, default=8)
    ap.add_argument("--answers", type=int, default=8)
    ap.add_argument("--steps", type=int, default=20)
    ap.add_argument("--drafts", type=int, default=4)
    ap.add_argument("--heads", type=int, nargs=3, default=(32, 8, 128), metavar=("QUERY", "KV", "COLUMNS"))
    ap.add_argument("--seed", type=int, default=0)
    a = ap.parse_args()
    _, batch, sequences, new, seconds = generate(a.prompts, a.answers, a.steps, a.drafts, tuple(a.heads), seed=a.seed)
    each = sum(len(x) - 1 for x in new) / (len(new) * max(1, a.steps))
    print(f"{a.prompts} prompts, {a.answers} answers each, {a.steps} steps of {a.drafts} drafted tokens: {each:.2f} tokens a step and answer; "
          f"{int((batch.refs > 0).sum())} blocks hold {sum(map(len, sequences))} tokens in the end; {seconds * 1e6:.0f} us a step and layer")


if __name__ == "__main__":
    main()
