"""Decoding several tokens a step: a tree of drafted tokens per request, checked by one call of each operator.

Each step drafts a tree that begins with a request's newest token.  All requests' nodes are rotated by their positions
and enter the cache together (sae_kv_append), each attends to the cached prefix, its ancestors and itself
(sae_attn_tree), and a token is drawn after each node (sae_sample).  The walk from the first node along the children
that hold the drawn token is accepted.  The accepted nodes' keys and values are moved behind the prefix
(sae_kv_read, sae_kv_write), and what the others left is written over by the next step.

There is no trained model here: one layer of attention over random tables, and drafts from the same tables without
the attention, so that some of them are accepted.

    python examples/tree_decoding.py [--type fp8] [--requests 6] [--tokens 40]
"""
import argparse
import os
import sys

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2605_18825_amd import api  # noqa: E402

HEADS, KV_HEADS, DIM, BLOCK, VOCAB = 8, 2, 128, api.KV_BLOCK, 512


def dev32(a):
    return torch.as_tensor(np.ascontiguousarray(a, np.int32)).cuda()


class Model:
    def __init__(self, kv_type, n_blocks):
        g = torch.Generator(device="cuda")
        g.manual_seed(1)
        self.rows = torch.randn((VOCAB, HEADS + 2 * KV_HEADS, DIM), device="cuda", generator=g).to(torch.bfloat16)
        self.head = torch.randn((HEADS * DIM, VOCAB), device="cuda", generator=g) * (3.0 / (HEADS * DIM) ** 0.5)
        self.guess = (self.rows[:, :HEADS].float().reshape(VOCAB, -1) @ self.head).topk(3, dim=1).indices.cpu().numpy()
        fp8 = kv_type == api.KV_FP8
        k, v = (torch.zeros((n_blocks, KV_HEADS, BLOCK * DIM), device="cuda",
                            dtype=torch.uint8 if fp8 else torch.bfloat16) for _ in range(2))
        ks, vs = (torch.zeros((n_blocks, KV_HEADS, BLOCK), dtype=torch.uint8, device="cuda") if fp8 else None
                  for _ in range(2))
        self.status = torch.zeros(1, dtype=torch.int32, device="cuda")
        self.kv = api.make_kv(kv_type, 1, n_blocks, KV_HEADS, DIM, k, v, k_scale=ks, v_scale=vs, status=self.status)
        self.inv_freq = (1e4 ** (-torch.arange(DIM // 2, dtype=torch.float64) / (DIM // 2))).float().cuda()
        self.rope = api.make_rope(self.inv_freq)
        self.scale = DIM ** -0.5

    def qkv(self, tokens):
        return self.rows[torch.as_tensor(np.asarray(tokens, np.int64)).cuda()].split([HEADS, KV_HEADS, KV_HEADS], dim=1)

    def logits(self, tokens, out):
        x = self.qkv(tokens)[0].float() + 0.5 * out.float()
        return x.reshape(len(x), -1) @ self.head

    def draft(self, token, depth):
        """Tokens and parents of a tree: `token`, three guesses after it, and the best guess after each node on."""
        tokens, parent, last = [token], [-1], [0]
        for d in range(depth):
            now = []
            for j in last:
                for t in self.guess[tokens[j]][:3 if d == 0 else 1]:
                    tokens.append(int(t))
                    parent.append(j)
                    now.append(len(tokens) - 1)
            last = now
        return tokens, parent


class Request:
    def __init__(self, prompt, table, seed):
        self.tokens, self.cached, self.table = list(prompt), 0, table  # every token but the last becomes cached
        self.u = np.random.default_rng(seed).random(4096).astype(np.float32)  # a random number per position
        self.seen = []  # (query as turned, output) of each cached token


def step(m, reqs, depth, settings, work):
    """One step of all requests; returns what was sampled from, row by row."""
    trees = []
    for i, r in enumerate(reqs):
        if len(r.tokens) - r.cached > 1:  # a prompt: a chain
            t = r.tokens[r.cached:r.cached + api.TREE_MAX]
            trees.append((t, list(range(-1, len(t) - 1))))
        else:
            trees.append(m.draft(r.tokens[-1], depth + i % 2))
    tokens = [t for tree in trees for t in tree[0]]
    parent = [p for tree in trees for p in tree[1]]
    start = np.cumsum([0] + [len(t) for t, _ in trees])
    base = np.array([r.cached for r in reqs])
    depths = []
    for t, p in trees:
        d = []
        for x in p:
            d.append(0 if x < 0 else d[x] + 1)
        depths.append(d)
    pos = np.concatenate([base[i] + np.array(d) for i, d in enumerate(depths)])
    table = dev32([r.table for r in reqs])
    seqs = api.make_seqs(table, dev32(base + np.diff(start)), q_start=dev32(start))
    n = len(tokens)
    q, k, v = m.qkv(tokens)
    turned, out = (torch.empty((n, HEADS, DIM), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    api.sae_kv_append(m.kv, seqs, m.rope, q, turned, k, v, pos=dev32(pos))
    need = max(api.sae_attn_work_size(m.kv, seqs, n, HEADS), api.sae_sample_work_size(n, VOCAB))
    if not work or work[0].numel() < need:
        work[:] = [torch.empty(need, dtype=torch.uint8, device="cuda")]
    api.sae_attn_tree(m.kv, seqs, dev32(parent), max(len(t) for t, _ in trees), turned, out, m.scale, work[0])
    logits = m.logits(tokens, out)
    u = np.concatenate([r.u[pos[start[i]:start[i + 1]]] for i, r in enumerate(reqs)])
    drawn = torch.empty(n, dtype=torch.int32, device="cuda")
    dev = {key: torch.full((n,), value, dtype=torch.int32 if key == "top_k" else torch.float32, device="cuda")
           for key, value in settings.items()}
    api.sae_sample(logits, torch.as_tensor(u).cuda(), drawn, work[0], **dev)
    got = drawn.cpu().numpy()
    # the accepted nodes
    ways = []
    for i, r in enumerate(reqs):
        t, p = trees[i]
        if len(r.tokens) - r.cached > 1:
            way = list(range(len(t)))
        else:
            way = [0]
            while True:
                child = [j for j in range(len(t)) if p[j] == way[-1] and t[j] == got[start[i] + way[-1]]]
                if not child:
                    break
                way.append(child[0])
        ways.append(way)
    rows = torch.as_tensor(np.concatenate([start[i] + np.array(w) for i, w in enumerate(ways)])).cuda()
    held_k, held_v = (torch.empty((n, KV_HEADS, DIM), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    api.sae_kv_read(m.kv, seqs, held_k, held_v)
    kept = np.array([len(w) for w in ways])
    seqs = api.make_seqs(table, dev32(base + kept), q_start=dev32(np.cumsum(np.append(0, kept))))
    api.sae_kv_write(m.kv, seqs, held_k[rows], held_v[rows])
    for i, r in enumerate(reqs):
        r.seen += [(turned[start[i] + j], out[start[i] + j]) for j in ways[i]]
        chain = len(r.tokens) - r.cached > 1
        r.cached += len(ways[i])
        if not chain:
            r.tokens += [trees[i][0][j] for j in ways[i][1:]]
        if r.cached == len(r.tokens):
            r.tokens.append(int(got[start[i] + ways[i][-1]]))
    return logits, u, drawn


def held(m, r):
    """A request's keys and values as the cache holds them."""
    k, v = (torch.empty((r.cached, KV_HEADS, DIM), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    api.sae_kv_read(m.kv, api.make_seqs(dev32([r.table]), dev32([r.cached]), q_start=dev32([0, r.cached])), k, v)
    return k, v


def plain(m, r, k, v):
    """Causal attention of a request's turned queries over keys and values, in fp32, without a cache or trees."""
    g = HEADS // KV_HEADS
    q = torch.stack([x for x, _ in r.seen]).float().permute(1, 0, 2).contiguous()
    k = k.float().repeat_interleave(g, 1).permute(1, 2, 0).contiguous()
    v = v.float().repeat_interleave(g, 1).permute(1, 0, 2).contiguous()
    n = r.cached
    hidden = torch.arange(n, device="cuda")[None, :] > torch.arange(n, device="cuda")[:, None]
    s = (torch.matmul(q, k) * m.scale).masked_fill(hidden, -torch.inf)
    return torch.matmul(torch.softmax(s, -1), v).permute(1, 0, 2)


def main(kv_type=api.KV_BF16, n_requests=6, n_tokens=40, depth=4, seed=0, settings=None, watch=None):
    """Decodes n_tokens or more of each request; returns the model, the requests and the tokens a step.  watch(logits, u, drawn)
    sees each step's sampling."""
    rng = np.random.default_rng(seed)
    width = (600 + n_tokens + 64) // BLOCK
    m = Model(kv_type, n_requests * width)
    blocks = rng.permutation(n_requests * width).reshape(n_requests, width).tolist()
    reqs = [Request(rng.integers(0, VOCAB, int(rng.integers(2, 600))), blocks[i], seed + i) for i in range(n_requests)]
    settings = dict(temperature=0.5, top_p=0.9) if settings is None else settings
    work, steps, prompts = [], 0, sum(len(r.tokens) for r in reqs)
    goal = [len(r.tokens) + n_tokens for r in reqs]
    while True:
        running = [r for r, end in zip(reqs, goal) if len(r.tokens) < end]
        if not running:
            break
        steps += sum(len(r.tokens) - r.cached == 1 for r in running)  # (a prompt's steps aside)
        seen = step(m, running, depth, settings, work)
        if watch is not None:
            watch(*seen)
    assert int(m.status[0]) == 0, api.status_names(int(m.status[0]))
    return m, reqs, (sum(len(r.tokens) for r in reqs) - prompts - n_requests) / steps


if __name__ == "__main__":
    ap = argparse.ArgumentParser()
    ap.add_argument("--type", choices=("bf16", "fp8"), default="bf16")
    ap.add_argument("--requests", type=int, default=6)
    ap.add_argument("--tokens", type=int, default=40)
    a = ap.parse_args()
    m, reqs, rate = main(api.KV_FP8 if a.type == "fp8" else api.KV_BF16, a.requests, a.tokens)
    worst = 0.0
    for r in reqs:
        got = torch.stack([x for _, x in r.seen]).float()
        worst = max(worst, float((got - plain(m, r, *held(m, r))).abs().max()))
    print("%.2f tokens a step and request, outputs within %.4f of attention without trees and a cache" % (rate, worst))
