"""Prompts and speculative decoding of one attention layer on the 8-bit paged cache.

    python examples/speculative_decode.py [--requests 16] [--steps 20] [--drafts 8] [--heads 32 8 128]

Prompts: the rows of all requests go through one launch that norms and rotates queries and keys and writes keys and values
into the cache; the keys and values are read back as they are cached, in rows, for the packed prefill.  Decoding: a step is
three calls (write the drafted tokens, attention of their trees, keep the accepted ones), captured once as a HIP graph
and replayed while the lengths grow on the device.  There is no model here: projections are random rows, and which of
the drafted tokens are accepted is drawn.
"""
import argparse
import os
import sys
import time

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2602_06072_amd import binding as pk  # noqa: E402

PAGE, EPS, MAX_POS = 16, 1e-6, 32768


def rotary_table(d, base=10000.0):
    freq = base ** (-torch.arange(0, d, 2, dtype=torch.float64) / d)
    ang = torch.arange(MAX_POS, dtype=torch.float64)[:, None] * freq
    return torch.stack([ang.cos(), ang.sin()], 1).float().contiguous().cuda()


class Layer:
    """Cache, page table and norm weights of one layer, for requests of up to `most` tokens each."""

    def __init__(self, n, most, heads, seed=0, dtype=pk.PK_F8):
        self.n, (self.Hq, self.Hkv, self.d) = n, heads
        pages = (most + PAGE - 1) // PAGE
        self.cache = pk.new_kv_cache(n * pages, PAGE, self.Hkv, self.d, dtype)
        rng = np.random.default_rng(seed)
        self.block_table = torch.from_numpy(rng.permutation(n * pages).astype(np.int32).reshape(n, pages)).cuda()
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.wq, self.wk = (1 + 0.1 * torch.randn(self.d, generator=g, device="cuda") for _ in "qk")
        self.wq, self.wk = self.wq.bfloat16(), self.wk.bfloat16()
        self.table, self.scale = rotary_table(self.d), self.d ** -0.5

    def slots(self, request, position):
        """Places in the cache of tokens, by request and position (device int64)."""
        return self.block_table[request, position // PAGE].long() * PAGE + position % PAGE

    def split(self, qkv):
        return qkv[:, :self.Hq], qkv[:, self.Hq:self.Hq + self.Hkv], qkv[:, self.Hq + self.Hkv:]


def prefill(layer, qkv, lens):
    """qkv: [sum(lens), Hq + 2 Hkv, d], the prompts one after the other.  Returns their attention."""
    lens = np.asarray(lens, np.int32)
    request = torch.from_numpy(np.repeat(np.arange(len(lens)), lens)).cuda()
    position = torch.from_numpy(np.concatenate([np.arange(x) for x in lens])).cuda()
    q, k, v = layer.split(qkv)
    q_rot = torch.empty(q.shape, dtype=q.dtype, device="cuda")
    pk.qkv_cache_write(layer.cache, q, k, v, layer.slots(request, position), q_rot, layer.wq, layer.wk, EPS, pk.Rope(layer.table, position.int()))
    # as cached: the prompt's rows see the same keys as every later token will
    k_rows, v_rows = torch.empty(k.shape, dtype=k.dtype, device="cuda"), torch.empty(v.shape, dtype=v.dtype, device="cuda")
    start = torch.from_numpy(np.concatenate([[0], np.cumsum(lens)[:-1]]).astype(np.int32)).cuda()
    pk.kv_cache_read(layer.cache, layer.block_table, torch.from_numpy(lens).cuda(), start, k_rows, v_rows)
    plan = pk.pack_plan(lens, lens)
    ws = pk.new_workspace(plan, layer.Hq, layer.Hkv, layer.d, pk.PK_BF16)
    out = torch.empty_like(q_rot)
    pk.packed_prefill_attn(plan, q_rot, k_rows, v_rows, out, layer.scale, ws)
    torch.cuda.synchronize()                        # (the plan's tables are done with)
    return out


class Decoder:
    """The three calls of a step on fixed buffers: fill qkv, parent and depth, run(), read out; fill keep and keep_count, commit()."""

    def __init__(self, layer, lens, drafts):
        n, T = layer.n, drafts
        self.layer, self.T = layer, T
        dev = lambda *shape, dtype=torch.int32: torch.zeros(*shape, dtype=dtype, device="cuda")  # noqa: E731
        self.context = torch.as_tensor(np.asarray(lens, np.int32)).cuda()     # tokens in the cache
        self.lens = dev(n)                                                    # with the drafted ones
        self.qkv = dev(n * T, layer.Hq + 2 * layer.Hkv, layer.d, dtype=torch.bfloat16)
        self.q = dev(n * T, layer.Hq, layer.d, dtype=torch.bfloat16)
        self.out = torch.empty_like(self.q)
        self.mask, self.depth = dev(n * T, dtype=torch.int64), dev(n * T)     # ancestors of a drafted token and itself; its place in its branch
        self.positions, self.slots = dev(n * T), dev(n * T, dtype=torch.int64)
        self.q_start = torch.arange(0, n * T + 1, T, dtype=torch.int32, device="cuda")
        self.keep, self.keep_count = dev(n, T), dev(n)
        self.request = torch.arange(n, device="cuda").repeat_interleave(T)
        self.number = torch.arange(T, device="cuda").repeat(n)
        self.rope = pk.Rope(layer.table, self.positions)
        self.ws = pk.new_tree_workspace(n, T, layer.Hq, layer.Hkv, layer.d)

    def run(self):
        """Attention of the drafted tokens, everything on the device: can be captured."""
        y = self.layer
        before = self.context[self.request]
        self.lens.copy_(self.context + self.T)
        self.positions.copy_(before + self.depth)                             # a token's position goes by its branch,
        self.slots.copy_(y.slots(self.request, (before + self.number).long()))    # its place by its number
        q, k, v = y.split(self.qkv)
        pk.qkv_cache_write(y.cache, q, k, v, self.slots, self.q, y.wq, y.wk, EPS, self.rope)
        pk.tree_attn(y.cache, self.q, self.q_start, self.T, self.mask, y.block_table, self.lens, self.out, y.scale, self.ws)

    def commit(self):
        """The accepted branch moves up behind the context."""
        pk.kv_cache_keep(self.layer.cache, self.layer.block_table, self.lens, self.q_start, self.keep, self.keep_count, self.context)


def random_tree(rng, T):
    """Parents (-1: the context), ancestor masks and depths of T drafted tokens, and one branch from its first token on."""
    mask, depth, parent = [], [], []
    for t in range(T):
        p = int(rng.integers(-1, t)) if t else -1
        parent.append(p)
        mask.append((1 << t) | (mask[p] if p >= 0 else 0))
        depth.append(depth[p] + 1 if p >= 0 else 0)
    at, branch = int(rng.integers(0, T)), []
    while at >= 0:
        branch.append(at)
        at = parent[at]
    return [x - (1 << 64) if x >> 63 else x for x in mask], depth, branch[::-1]


def generate(n=16, steps=20, drafts=8, heads=(32, 8, 128), seed=0, prompt=(16, 500), dtype=pk.PK_F8, graph=True):
    """Runs prompts and `steps` steps.  Returns (layer, prompt lengths, the prompts' rows, the accepted rows and their outputs of every
    request, tokens in the cache, seconds of a step)."""
    rng, g = np.random.default_rng(seed), torch.Generator(device="cuda").manual_seed(seed)
    lens = rng.integers(prompt[0], prompt[1] + 1, n)
    layer = Layer(n, prompt[1] + (steps + 2) * drafts, heads, seed, dtype)
    width = layer.Hq + 2 * layer.Hkv
    rows = torch.randn(int(lens.sum()), width, layer.d, generator=g, device="cuda").bfloat16()
    first = prefill(layer, rows, lens)
    dec = Decoder(layer, lens, drafts)
    dec.run()                                       # (a first call loads the kernels; its drafted tokens are none that is kept)
    torch.cuda.synchronize()
    if graph:
        captured = torch.cuda.CUDAGraph()
        with torch.cuda.graph(captured):
            dec.run()
    step = captured.replay if graph else dec.run
    accepted, took = [[] for _ in range(n)], []
    for _ in range(steps):
        trees = [random_tree(rng, drafts) for _ in range(n)]
        dec.qkv.copy_(torch.randn(n * drafts, width, layer.d, generator=g, device="cuda"))
        dec.mask.copy_(torch.tensor([x for t in trees for x in t[0]]))
        dec.depth.copy_(torch.tensor([x for t in trees for x in t[1]], dtype=torch.int32))
        keep = np.zeros((n, drafts), np.int32)
        for i, t in enumerate(trees):
            keep[i, :len(t[2])] = t[2]
        torch.cuda.synchronize()
        begin = time.perf_counter()
        step()
        dec.keep.copy_(torch.from_numpy(keep))      # (a sampler would write these on the device)
        dec.keep_count.copy_(torch.tensor([len(t[2]) for t in trees], dtype=torch.int32))
        dec.commit()
        torch.cuda.synchronize()
        took.append(time.perf_counter() - begin)
        for i, t in enumerate(trees):
            at = torch.tensor([i * drafts + x for x in t[2]], device="cuda")
            accepted[i].append((dec.qkv[at], dec.out[at]))
    return layer, lens, rows, first, accepted, dec.context.cpu().numpy(), float(np.median(took)) if took else 0.0


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--requests", type=int, default=16)
    ap.add_argument("--steps", type=int, default=20)
    ap.add_argument("--drafts", type=int, default=8)
    ap.add_argument("--heads", type=int, nargs=3, default=(32, 8, 128), metavar=("QUERY", "KV", "COLUMNS"))
    ap.add_argument("--seed", type=int, default=0)
    a = ap.parse_args()
    _, lens, _, _, accepted, context, seconds = generate(a.requests, a.steps, a.drafts, tuple(a.heads), a.seed)
    tokens = int(context.sum() - lens.sum())
    print(f"{a.requests} requests of {lens.min()}..{lens.max()} tokens; {a.steps} steps of {a.drafts} drafted tokens: {tokens} accepted, "
          f"{tokens / max(1, a.steps * a.requests):.2f} a step and request; {seconds * 1e6:.0f} us a step and layer")


if __name__ == "__main__":
    main()
