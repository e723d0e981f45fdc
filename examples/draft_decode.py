"""Decoding with drafted tokens: a small decoder made of binary low-rank layers, two sequences that share a prompt, a paged cache.

    python examples/draft_decode.py

One step runs the last token of every sequence and a tree of drafted continuations through the model at once -- the binary layers cost about the
same for eight tokens as for one -- and keeps the longest drafted path that the model itself would have taken:

    q, k, v = layers(norm(x))                        nq_binlr_forward
    norm and rotate q and k, store k and v           nq_rope_cache
    every token attends to the cache, its ancestors  nq_attn_forward
    and itself
    o, gate, up, down layers, residuals              nq_binlr_forward
    the next token of every node of the tree         nq_sample
    the accepted path's keys and values move up      nq_kv_compact

The second sequence is a fork of the first one behind the prompt: it shares the full pages and copies the last one (nq_kv_copy_pages).
Weights are random, so the text means nothing; drafts come from what followed a token before.  A greedy sequence gives the same tokens with drafts as
without.
"""
import argparse
import os
import sys

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2602_06694_amd import binding as nq  # noqa: E402
from paper_2602_06694_amd import synth  # noqa: E402


class Model:
    """Blocks of q, k, v, o, gate, up, down and a head, all binary layers; RMS norms, a gated unit and residuals between them in torch."""

    def __init__(self, blocks=3, width=512, q_heads=8, kv_heads=2, head_dim=64, hidden=1024, vocab=1000, rank=256, seed=1):
        self.blocks, self.width, self.q_heads, self.kv_heads, self.head_dim, self.vocab = blocks, width, q_heads, kv_heads, head_dim, vocab
        g = torch.Generator()
        g.manual_seed(seed)
        self.embedding = torch.randn(vocab, width, generator=g).cuda()
        qw, kw = q_heads * head_dim, kv_heads * head_dim
        shapes = {"q": (qw, width), "k": (kw, width), "v": (kw, width), "o": (width, qw), "gate": (hidden, width), "up": (hidden, width), "down": (width, hidden)}
        self.layers = [{n: self._layer(*s, rank, seed + 100 * b + i) for i, (n, s) in enumerate(shapes.items())} for b in range(blocks)]
        self.head = self._layer(vocab, width, rank, seed + 99999)
        self.q_norm, self.k_norm = (1 + 0.1 * torch.randn(blocks, head_dim, generator=g)).cuda(), (1 + 0.1 * torch.randn(blocks, head_dim, generator=g)).cuda()
        freqs, magnitude = nq.nq_rope_freqs(nq.NQ_ROPE_YARN, head_dim, 10000.0, 4.0, 512.0)
        self.rope = nq.nq_rope_create(q_heads, kv_heads, head_dim, head_dim, nq.NQ_ROPE_HALF, freqs, magnitude, 1e-6, 0.0, nq.NQ_F32, nq.NQ_BF16)

    @staticmethod
    def _layer(d_out, d_in, r, seed):
        scale = (1.0 / np.sqrt(r * d_in)) ** 0.5                     # outputs of unit size from inputs of unit size
        s_out, s_in = ((synth.gen_scales(n, seed + 10 * i) * scale).astype(np.float16) for i, n in ((1, d_out), (2, d_in)))
        h = nq.nq_binlr_create(d_out, d_in, r, synth.gen_sign_words(d_out, r, seed + 3), synth.gen_sign_words(d_in, r, seed + 4), s_out, s_in, nq.NQ_F32, nq.NQ_F32)
        nq.nq_binlr_reserve(h, 64)
        return h, d_out

    def apply(self, layer, x):
        h, d_out = layer
        y = torch.empty(x.shape[0], d_out, device="cuda")
        nq.nq_binlr_forward(h, x.contiguous(), y, x.shape[0])
        return y

    def close(self):
        for h, _ in [self.head] + [l for b in self.layers for l in b.values()]:
            nq.nq_binlr_destroy(h)
        nq.nq_rope_destroy(self.rope)


def rms(x):
    return x * torch.rsqrt((x * x).mean(-1, keepdim=True) + 1e-6)


class Server:
    """Sequences, the pages of their caches, and the step that advances all of them."""

    def __init__(self, model, pages=128, page=16, table=64):
        self.model, self.page = model, page
        shape = (model.blocks, 2, pages, model.kv_heads, page, model.head_dim)
        self.memory = torch.zeros(shape, dtype=torch.bfloat16, device="cuda")
        self.kvs = [nq.nq_kv_create(m[0], m[1], nq.NQ_BF16, model.kv_heads, model.head_dim, page, pages) for m in self.memory]
        self.attns = [nq.nq_attn_create(kv, model.q_heads, model.head_dim ** -0.5, 30.0, nq.NQ_F32) for kv in self.kvs]
        self.free, self.users = list(range(pages)), [0] * pages
        self.width = table
        self.workspace = torch.empty(0, dtype=torch.uint8, device="cuda")

    def close(self):
        for a in self.attns:
            nq.nq_attn_destroy(a)
        for kv in self.kvs:
            nq.nq_kv_destroy(kv)

    # ---- pages ----
    def _grow(self, seq, tokens):
        while len(seq["pages"]) * self.page < tokens:
            p = self.free.pop()
            self.users[p] = 1
            seq["pages"].append(p)

    def new(self):
        return {"pages": [], "length": 0, "tokens": [], "follows": {}}

    def fork(self, seq):
        """A second sequence behind the same tokens: full pages are shared, a partly filled one is copied."""
        other = {"pages": list(seq["pages"]), "length": seq["length"], "tokens": list(seq["tokens"]), "follows": {t: list(n) for t, n in seq["follows"].items()}}
        for p in other["pages"]:
            self.users[p] += 1
        if other["length"] % self.page:
            at = other["length"] // self.page
            old, new = other["pages"][at], self.free.pop()
            self.users[old] -= 1
            self.users[new] = 1
            other["pages"][at] = new
            nq.nq_kv_copy_pages(self.kvs, self._ints([old]), self._ints([new]))
        return other

    def drop(self, seq):
        for p in seq["pages"]:
            self.users[p] -= 1
            if not self.users[p]:
                self.free.append(p)
        seq["pages"] = []

    # ---- one pass of the model over new tokens of several sequences ----
    @staticmethod
    def _ints(values, dtype=torch.int32):
        return torch.tensor(values, dtype=dtype, device="cuda")

    def _run(self, seqs, tokens, depths, tree):
        """tokens, depths: lists per sequence; tree: packed rows or None (a chunk of a prompt).  Logits of all new tokens."""
        m = self.model
        positions, slots, begin = [], [], [0]
        for s, t, d in zip(seqs, tokens, depths):
            self._grow(s, s["length"] + len(t))
            positions += [s["length"] + i for i in d]
            slots += [s["pages"][(s["length"] + j) // self.page] * self.page + (s["length"] + j) % self.page for j in range(len(t))]
            begin.append(begin[-1] + len(t))
        table = torch.zeros(len(seqs), self.width, dtype=torch.int32)
        for i, s in enumerate(seqs):
            table[i, :len(s["pages"])] = torch.tensor(s["pages"], dtype=torch.int32)
        self.table, self.lengths = table.cuda(), self._ints([s["length"] for s in seqs])
        positions, slots, begin = self._ints(positions), self._ints(slots, torch.int64), self._ints(begin)
        flat = [t for ts in tokens for t in ts]
        n = len(flat)
        need = nq.nq_attn_workspace_bytes(self.attns[0], len(seqs), n)
        if self.workspace.numel() < need:
            self.workspace = torch.empty(need, dtype=torch.uint8, device="cuda")
        x = m.embedding[self._ints(flat, torch.int64)]
        q_out = torch.empty(n, m.q_heads * m.head_dim, dtype=torch.bfloat16, device="cuda")
        mixed = torch.empty(n, m.q_heads * m.head_dim, device="cuda")
        for b, layer in enumerate(m.layers):
            h = rms(x)
            q, k, v = (m.apply(layer[name], h) for name in ("q", "k", "v"))
            nq.nq_rope_cache(m.rope, self.kvs[b], q, k, v, m.q_norm[b], m.k_norm[b], positions, slots, q_out)
            nq.nq_attn_forward(self.attns[b], q_out, begin, self.lengths, self.table, tree, mixed, None, self.workspace, need)
            x = x + m.apply(layer["o"], mixed)
            h = rms(x)
            x = x + m.apply(layer["down"], torch.nn.functional.silu(m.apply(layer["gate"], h)) * m.apply(layer["up"], h))
        return m.apply(m.head, 4.0 * rms(x))

    def prefill(self, seq, tokens):
        """All but the last token of a prompt; the last one is the root of the first step."""
        if len(tokens) > 1:
            self._run([seq], [tokens[:-1]], [range(len(tokens) - 1)], None)
        seq["length"], seq["tokens"] = len(tokens) - 1, list(tokens)
        for a, b in zip(tokens, tokens[1:]):
            seq["follows"].setdefault(a, []).append(b)

    # ---- drafts ----
    def _draft(self, seq, most):
        """Nodes (token, parent), the last token first: a chain of what followed each token last, and beside its first link what followed before."""
        nodes = [(seq["tokens"][-1], -1)]
        at = 0
        while len(nodes) <= most:
            known = seq["follows"].get(nodes[at][0])
            if not known:
                break
            if at == 0 and len(set(known)) > 1 and len(nodes) < most:
                nodes.append(([t for t in reversed(known) if t != known[-1]][0], 0))
            nodes.append((known[-1], at))
            at = len(nodes) - 1
        return nodes

    @staticmethod
    def _pack(rows, nodes):
        """Whole numbers whose bit j says that a node sees node j, as words of 32 bits: [rows, words]."""
        words = np.array([[row >> 32 * w & 0xffffffff for w in range(-(-nodes // 32))] for row in rows], dtype=np.uint32)
        return torch.from_numpy(words.view(np.int32))

    def step(self, seqs, temperature, top_k, top_p, min_p, uniforms, most=6):
        """Advances every sequence by at least one token; returns how many each gained.  uniforms: a number per sequence and depth."""
        drafts = [self._draft(s, most) for s in seqs]
        depths, rows = [], []
        for nodes in drafts:
            depth, see = [], []
            for j, (_, parent) in enumerate(nodes):
                depth.append(depth[parent] + 1 if parent >= 0 else 0)
                see.append((see[parent] if parent >= 0 else 0) | 1 << j)
            depths.append(depth)
            rows += see
        logits = self._run(seqs, [[t for t, _ in nodes] for nodes in drafts], depths, self._pack(rows, max(len(nodes) for nodes in drafts)).cuda())
        n = len(rows)
        own = [i for i, nodes in enumerate(drafts) for _ in nodes]
        per = lambda values, dtype: torch.tensor([values[i] for i in own], dtype=dtype, device="cuda")  # noqa: E731
        u = torch.tensor([uniforms[i][d] for i, depth in enumerate(depths) for d in depth], dtype=torch.float32, device="cuda")
        tokens, logprobs = torch.empty(n, dtype=torch.int32, device="cuda"), torch.empty(n, device="cuda")
        need = nq.nq_sample_workspace_bytes(n, logits.shape[1])
        if self.workspace.numel() < need:
            self.workspace = torch.empty(need, dtype=torch.uint8, device="cuda")
        nq.nq_sample(logits, nq.NQ_F32, per(temperature, torch.float32), per(top_k, torch.int32), per(top_p, torch.float32), per(min_p, torch.float32), u, tokens, logprobs,
                     self.workspace if need else None, need)
        drawn = tokens.tolist()
        # the path of drafts that the model would have taken: a child whose token is the one drawn at its parent
        paths, gained, first = [], [], 0
        for s, nodes in zip(seqs, drafts):
            path = [0]
            while True:
                want = drawn[first + path[-1]]
                child = [j for j, (t, parent) in enumerate(nodes) if parent == path[-1] and t == want]
                s["follows"].setdefault(nodes[path[-1]][0], []).append(want)
                s["tokens"].append(want)
                if not child:
                    break
                path.append(child[0])
            paths.append(path)
            gained.append(len(path))
            first += len(nodes)
        width = max(len(p) for p in paths)
        if any(p != list(range(len(p))) for p in paths):
            nq.nq_kv_compact(self.kvs, self.lengths, self.table, self._ints([p + [0] * (width - len(p)) for p in paths]), self._ints(gained))
        for s, g in zip(seqs, gained):
            s["length"] += g
        return gained


def generate(model, prompt, count, greedy=True, drafts=6, seed=3):
    """Two sequences behind one prompt, `count` tokens each: the first greedy, the other sampled (greedy=False) or greedy too.  (tokens, tokens, steps)"""
    server = Server(model)
    a = server.new()
    server.prefill(a, prompt)
    b = server.fork(a)
    rng = np.random.default_rng(seed)
    noise = rng.random((2, 4096))
    steps = 0
    while min(len(a["tokens"]), len(b["tokens"])) < len(prompt) + count:
        # the number that draws a token belongs to its place in the sequence: drafts do not change what is drawn
        at = [noise[i][len(s["tokens"]):] for i, s in enumerate((a, b))]
        server.step([a, b], [0.0, 0.0 if greedy else 0.9], [0, 50], [1.0, 0.95], [0.0, 0.01], at, drafts)
        steps += 1
    out = a["tokens"][len(prompt):len(prompt) + count], b["tokens"][len(prompt):len(prompt) + count], steps
    server.drop(a)
    server.drop(b)
    assert sorted(server.free) == list(range(len(server.users)))
    server.close()
    return out


def main():
    ap = argparse.ArgumentParser(description="Decoding with drafted tokens over a paged cache")
    ap.add_argument("--tokens", type=int, default=48)
    ap.add_argument("--drafts", type=int, default=6)
    args = ap.parse_args()
    model = Model()
    prompt = [int(t) for t in np.random.default_rng(5).integers(0, model.vocab, 37)]
    greedy, sampled, steps = generate(model, prompt, args.tokens, greedy=False, drafts=args.drafts)
    plain, plain_sampled, plain_steps = generate(model, prompt, args.tokens, greedy=False, drafts=0)
    print(f"{args.tokens} tokens for two sequences: {steps} steps with up to {args.drafts} drafted tokens, {plain_steps} without")
    print("greedy:", greedy[:16], "the same without drafts:", greedy == plain)
    print("sampled:", sampled[:16], "the same without drafts:", sampled == plain_sampled)
    model.close()


if __name__ == "__main__":
    main()
