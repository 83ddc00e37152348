"""One attention call over drafted trees and its 64-bit expectation."""
import numpy as np
import torch

from attn_cases import Call
from harness import say
from kv_cases import DT, dev32
from oracle import kvcache as O
from paper_2605_18825_amd import api


def tree(n, kind, rng):
    """Parents of n nodes."""
    if kind == "chain":
        return np.arange(n) - 1
    if kind == "flat":
        return np.full(n, -1)
    if kind == "star":
        return np.where(np.arange(n) == 0, -1, 0)
    if kind == "binary":
        return np.where(np.arange(n) == 0, -1, (np.arange(n) - 1) // 2)
    return np.array([int(rng.integers(-1 if kind == "forest" else min(j, 1) - 1, j)) if j else -1 for j in range(n)])


KINDS = ["random", "chain", "forest", "flat", "binary", "star"]


class TreeCall(Call):
    def __init__(self, ty, heads, kvh, dim, lens, new, kinds=KINDS, seed=0, **more):
        super().__init__(ty, heads, kvh, dim, lens, new=new, seed=seed, **more)
        rng = np.random.default_rng(seed + 1)
        self.parents = [tree(n, kinds[i % len(kinds)], rng) for i, n in enumerate(self.counts)]
        self.max_nodes = max(1, int(self.counts.max()))

    def parent(self):
        return dev32(np.concatenate(self.parents + [np.zeros(0, int)]))

    def run(self, decode=False, stream=None, one=False):
        say("tree attention type %d heads %d/%d dim %d seqs %d rows %d window %d longest %d nodes %d" % (
            self.ty, self.heads, self.kvh, self.dim, len(self.lens), self.n, self.window, int(self.lens.max()), self.max_nodes))
        kv = self.cache.device()
        h, d = self.heads, self.dim
        # queries and outputs lie in wider rows
        fused = torch.full((self.n, (h + 2) * d), 7.0, dtype=DT[self.dtype], device="cuda")
        q = fused[:, :h * d].view(self.n, h, d)
        q.copy_(torch.as_tensor(self.qbits).view(DT[self.dtype]))
        wide = torch.full((self.n, h * d + 64), 7.0, dtype=DT[self.dtype], device="cuda")
        out = wide[:, :h * d].view(self.n, h, d)
        lse = torch.full((self.n, h), 7.0, dtype=torch.float32, device="cuda")
        seqs = api.make_seqs(dev32(self.ids), dev32(self.lens), q_start=None if one else dev32(self.starts),
                             inst=dev32(self.inst) if self.n_inst > 1 else None)
        work = torch.full((api.sae_attn_work_size(kv, seqs, self.n, h),), 0xFF, dtype=torch.uint8, device="cuda")
        parent = self.parent()
        torch.cuda.synchronize()
        api.sae_attn_tree(kv, seqs, parent, self.max_nodes, q, out, self.scale, work, window=self.window, lse=lse,
                          stream=stream)
        torch.cuda.synchronize()
        assert int(self.cache.status[0]) == 0
        assert torch.all(wide[:, h * d:] == 7.0)
        return out.double().cpu().numpy(), lse.double().cpu().numpy()

    def want(self):
        parts = []
        for r, total in enumerate(self.lens):
            a, b = self.starts[r], self.starts[r + 1]
            lo, hi = self.inst[r] * self.cache.bpi, (self.inst[r] + 1) * self.cache.bpi
            k, there = O.rows_of(self.ids[r], total, self.cache.values[0][lo:hi])
            v, _ = O.rows_of(self.ids[r], total, self.cache.values[1][lo:hi])
            parts.append(O.tree_attention(self.q[a:b], self.parents[r], k, v, there, self.scale, self.window))
        return [np.concatenate(x) for x in zip(*parts)]

    def check(self, decode=False, **more):
        super().check(False, **more)
