"""Serving with a prefix cache and its keys and values: the eviction path and the paged cache's operators together.

Requests share prompt prefixes.  For each one: its blocks' hashes are matched (sae_prefix_match); room is made by
evicting what the policy values least (sae_score_select); the unmatched blocks enter the cache (sae_insert_blocks);
their tokens' keys and values are written (sae_kv_write) and attend to the cached prefix and themselves
(sae_attn_prefill).  Then all requests decode together, a token each per step (sae_kv_write, sae_attn_decode).  At the
end the cached keys of a request are read back (sae_kv_read).

There is no model here: a token's query, key and value are random vectors that depend on the token and its position
alone, so a reused prefix holds what a recomputed one would, and every output can be checked against attention over
the whole sequence without a cache.

    python examples/paged_serving.py [--type fp8] [--blocks 56] [--requests 24]
"""
import argparse
import os
import sys

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2605_18825_amd import api  # noqa: E402
from paper_2605_18825_amd.pool import DevicePool, SelectBuffers  # noqa: E402

HEADS, KV_HEADS, DIM, BLOCK = 8, 2, 128, api.KV_BLOCK
MASK = (1 << 64) - 1


def dev32(a):
    return torch.as_tensor(np.ascontiguousarray(a, np.int32)).cuda()


def chain(tokens):
    """Chained content hashes of the full blocks of a prompt."""
    h, out = 0x9E3779B97F4A7C15, []
    for b in range(len(tokens) // BLOCK):
        for t in tokens[b * BLOCK:(b + 1) * BLOCK]:
            h = ((h ^ int(t)) * 0xBF58476D1CE4E5B9 + 0x94D049BB133111EB) & MASK
            h ^= h >> 29
        out.append(h if h not in (0, MASK) else 1)
    return out


class Server:
    def __init__(self, kv_type, n_blocks, vocab=1000, most=1024):
        self.N, self.now = n_blocks, 1000
        # one queue of log-normal reuse times
        self.ctx = api.sae_create(1, n_blocks, [api.KIND_LOGNORMAL], max_k=n_blocks)
        self.pool = DevicePool(1, n_blocks)
        self.pool.bind(self.ctx)
        api.sae_index_build(self.ctx)
        api.sae_set_params(self.ctx, -1, api.make_params(1, mu=8.0, sigma=1.5))
        self.sel = SelectBuffers(1, 1, n_blocks)
        self.free = list(range(n_blocks))
        fp8 = kv_type == api.KV_FP8
        k, v = (torch.zeros((n_blocks, KV_HEADS, BLOCK * DIM), device="cuda",
                            dtype=torch.uint8 if fp8 else torch.bfloat16) for _ in range(2))
        ks, vs = (torch.zeros((n_blocks, KV_HEADS, BLOCK), dtype=torch.uint8, device="cuda") if fp8 else None
                  for _ in range(2))
        self.status = torch.zeros(1, dtype=torch.int32, device="cuda")
        self.kv = api.make_kv(kv_type, 1, n_blocks, KV_HEADS, DIM, k, v, k_scale=ks, v_scale=vs, status=self.status)
        # the vectors of token t at position p: rows of fixed random tables, added
        g = torch.Generator(device="cuda")
        g.manual_seed(1)
        self.tok = torch.randn((vocab, (HEADS + 2 * KV_HEADS) * DIM), device="cuda", generator=g)
        self.pos = torch.randn((most, (HEADS + 2 * KV_HEADS) * DIM), device="cuda", generator=g)
        self.work = None
        self.scale = DIM ** -0.5
        self.matched = self.total = self.evicted = 0

    def qkv(self, tokens, positions):
        x = (self.tok[torch.as_tensor(tokens).cuda()] + self.pos[torch.as_tensor(positions).cuda()]) * 0.7
        x = x.to(torch.bfloat16).view(len(tokens), HEADS + 2 * KV_HEADS, DIM)
        return x.split([HEADS, KV_HEADS, KV_HEADS], dim=1)  # slices of fused rows, as a projection leaves them

    def workspace(self, seqs, n):
        need = api.sae_attn_work_size(self.kv, seqs, n, HEADS)
        if self.work is None or self.work.numel() < need:
            self.work = torch.empty(need, dtype=torch.uint8, device="cuda")
        return self.work

    def take(self, n):
        """n free blocks; evicts where there are too few."""
        short = n - len(self.free)
        if short > 0:
            self.sel.run(self.ctx, self.now, short, api.SS_COMMIT | api.SS_CASCADE)
            d = int(self.sel.decision_count[0])
            self.free += self.sel.decision[0, :d].tolist()
            self.evicted += d
        if n > len(self.free):
            raise RuntimeError("every block is in use: admit fewer requests at a time")
        got, self.free = self.free[:n], self.free[n:]
        return got

    def admit(self, tokens, room):
        """Prefill one request; `room`: tokens it may generate.  Returns its state and the new rows' outputs."""
        self.now += 50
        hashes = chain(tokens)
        usable = (len(tokens) - 1) // BLOCK  # at least one token is computed
        n_match, ids = 0, []
        if hashes:
            h = torch.as_tensor(np.array([hashes], np.uint64).view(np.int64)).cuda()
            length = torch.zeros(1, dtype=torch.int32, device="cuda")
            table = torch.full((1, len(hashes)), -1, dtype=torch.int32, device="cuda")
            api.sae_prefix_match(self.ctx, h, dev32([usable]), self.now, api.PM_TOUCH | api.PM_STATS, length,
                                 matched_ids=table)
            n_match = int(length[0])
            ids = table[0, :n_match].tolist()
        self.matched += n_match
        self.total += len(hashes)
        if ids:
            api.sae_ref_blocks(self.ctx, dev32(ids), 1)  # before anything is evicted
        # blocks of the prompt that enter the cache; those of the generated tokens are the request's own
        n_all = -(-(len(tokens) + room) // BLOCK)
        new = self.take(n_all - n_match)
        cached = new[:len(hashes) - n_match]
        # a cached block matched by nobody before has to be new to the index: the last one may be there already
        # where the whole prompt was cached but its last block is computed again
        if cached and usable < len(hashes) and n_match == usable:
            cached = []
        if cached:
            n = len(cached)
            parent = ([ids[-1]] if ids else [-1]) + cached[:-1]
            meta = api.meta_to_u16(api.pack_meta(torch.zeros(n), torch.ones(n), torch.full((n,), BLOCK))).cuda()
            ob = torch.arange(n_match, n_match + n)
            off = api.off_to_u32(api.pack_off(ob, torch.full((n,), len(hashes) - 1))).cuda()
            h = torch.as_tensor(np.array(hashes[n_match:n_match + n], np.uint64).view(np.int64)).cuda()
            api.sae_insert_blocks(self.ctx, dev32(cached), h, dev32(parent), dev32([self.now] * n), meta, off)
            api.sae_ref_blocks(self.ctx, dev32(cached), 1)
        req = dict(tokens=list(tokens), table=ids + new, held=ids + cached, own=new[len(cached):])
        first = n_match * BLOCK
        q, k, v = self.qkv(tokens[first:], range(first, len(tokens)))
        seqs = api.make_seqs(dev32([req["table"]]), dev32([len(tokens)]), q_start=dev32([0, len(tokens) - first]))
        api.sae_kv_write(self.kv, seqs, k, v)
        out = torch.empty_like(q.contiguous())
        api.sae_attn_prefill(self.kv, seqs, q, out, self.scale, self.workspace(seqs, len(out)))
        return req, out

    def step(self, reqs, tokens):
        """One new token for every running request: write, then attend."""
        self.now += 5
        width = max(len(r["table"]) for r in reqs)
        for r, t in zip(reqs, tokens):
            r["tokens"].append(t)
        table = dev32([r["table"] + [-1] * (width - len(r["table"])) for r in reqs])
        lens = [len(r["tokens"]) for r in reqs]
        seqs = api.make_seqs(table, dev32(lens))
        q, k, v = self.qkv(tokens, [n - 1 for n in lens])
        api.sae_kv_write(self.kv, seqs, k, v)
        out = torch.empty_like(q.contiguous())
        api.sae_attn_decode(self.kv, seqs, q, out, self.scale, self.workspace(seqs, len(reqs)))
        return out

    def release(self, req):
        if req["held"]:
            api.sae_ref_blocks(self.ctx, dev32(req["held"]), -1)
        self.free += req["own"]

    def read(self, req):
        """The request's keys and values as the cache holds them."""
        n = len(req["tokens"])
        k, v = (torch.empty((n, KV_HEADS, DIM), dtype=torch.bfloat16, device="cuda") for _ in range(2))
        seqs = api.make_seqs(dev32([req["table"]]), dev32([n]), q_start=dev32([0, n]))
        api.sae_kv_read(self.kv, seqs, k, v)
        return k, v

    def plain(self, tokens, first, k=None, v=None):
        """Outputs of rows first .. of the whole sequence, without the cache, in fp32 (k, v: as the cache holds them)."""
        q, k0, v0 = self.qkv(tokens, range(len(tokens)))
        g = HEADS // KV_HEADS
        k = (k0 if k is None else k).float().repeat_interleave(g, 1).permute(1, 2, 0).contiguous()
        v = (v0 if v is None else v).float().repeat_interleave(g, 1).permute(1, 0, 2).contiguous()
        s = torch.matmul(q[first:].float().permute(1, 0, 2).contiguous(), k) * self.scale
        n = len(tokens)
        hidden = torch.arange(n, device="cuda")[None, :] > torch.arange(first, n, device="cuda")[:, None]
        return torch.matmul(torch.softmax(s.masked_fill(hidden, -torch.inf), -1), v).permute(1, 0, 2)


def main(kv_type=api.KV_BF16, n_blocks=56, n_requests=24, batch=4, generate=20, seed=0):
    """Serves batches of requests; returns the share of prompt blocks that were matched, the evictions, and the
    largest difference of an output from the plain one."""
    rng = np.random.default_rng(seed)
    s = Server(kv_type, n_blocks)
    shared = [rng.integers(0, 1000, int(rng.integers(40, 120))).tolist() for _ in range(3)]
    worst = 0.0
    for start in range(0, n_requests, batch):
        running, first_rows = [], []
        for _ in range(min(batch, n_requests - start)):
            own = rng.integers(0, 1000, int(rng.integers(5, 60))).tolist()
            prompt = shared[int(rng.integers(0, 3))] + own
            req, out = s.admit(prompt, generate)
            running.append(req)
            first_rows.append((len(prompt) - len(out), out))
        steps = [s.step(running, rng.integers(0, 1000, len(running)).tolist()) for _ in range(generate)]
        for i, req in enumerate(running):
            first, out = first_rows[i]
            got = torch.cat([out] + [o[i:i + 1] for o in steps]).float()
            k, v = s.read(req)
            worst = max(worst, float((got - s.plain(req["tokens"], first, k, v)).abs().max()))
            s.release(req)
    assert int(s.status[0]) == 0, api.status_names(int(s.status[0]))
    r = dict(matched=s.matched / s.total, evicted=s.evicted, worst=worst)
    torch.cuda.synchronize()
    api.sae_destroy(s.ctx)
    return r


if __name__ == "__main__":
    ap = argparse.ArgumentParser()
    ap.add_argument("--type", choices=("bf16", "fp8"), default="bf16")
    ap.add_argument("--blocks", type=int, default=56)
    ap.add_argument("--requests", type=int, default=24)
    a = ap.parse_args()
    r = main(api.KV_FP8 if a.type == "fp8" else api.KV_BF16, a.blocks, a.requests)
    print("%.0f %% of the prompts' blocks were cached, %d blocks evicted, outputs within %.4f of attention without a cache"
          % (100 * r["matched"], r["evicted"], r["worst"]))
