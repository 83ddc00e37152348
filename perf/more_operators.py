"""Measured cases of a speculative serving step over the paged key-value cache.

Three operators on the block pool (16 tokens a block), in the order in which a step calls them:
  append   new tokens' queries and keys are turned by their positions' angles, keys and values go to their places at the
           end of the sequences (an 8-bit cache is quantised on the way, with one power-of-two scale per token and head)
  tree     attention of drafted tokens that form a tree: each sees the cached prefix, its ancestors and itself
  sample   a token per row of logits by temperature, top-k, top-p and min-p, from a given random number

Cache layout (values; one layer): a block holds one page per key-value head.  With c = 16 bytes / value size,
keys [block][head][D / c][16 tokens][c]; values [block][head][D / 2c][16][2][c / 8][2][4], where token t and
dimension d of the page are at [d / 2c][d % 16][t / 4 % 2][d / 16 % (c / 8)][t / 8][t % 4].  Scales of an 8-bit
cache (float8 e4m3 values): one byte b per [block][head][16 tokens], for keys and for values, standing for
2^(b - 127).

Angles: dimensions i and i + R / 2 (interleaved: 2 i and 2 i + 1) of a head's first R are turned by position *
inv_freq[i], and multiplied by a factor that long contexts bring along.

Sampling, for a row of logits l and T, k, p, m, u (a temperature of 0 takes the largest logit, the first of equals):
weights exp((l - max l) / T); tokens in order of falling logits, the lower index first among equal ones; kept are the
first k, of these the smallest head of the order that holds p of their weight, of these the ones with at least m of the
largest weight, and always the first; then, in that order, the first token up to which the weights' sum passes u times
the sum of all kept ones.  Logits that are NaN or -inf are never taken; a row without another gives -1.
"""
import math

import numpy as np
import torch

own = False

BLOCK = 16
DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}


def listed():
    return [
        # one conversation's next token: latency of a single call
        dict(name="append_one", kind="append", type="bf16", seqs=1, lo=1440, hi=1440, new_lo=1, new_hi=1, heads=16,
             kv_heads=2, dim=128, turned=128, interleaved=False, tree=False, inst=1),
        # a decode step of a serving batch
        dict(name="append_step", kind="append", type="bf16", seqs=256, lo=512, hi=2048, new_lo=1, new_hi=1, heads=32,
             kv_heads=8, dim=128, turned=128, interleaved=False, tree=False, inst=1),
        # drafted trees far into long contexts: their positions are given, a part of each head is turned
        dict(name="append_tree", kind="append", type="f16", seqs=24, lo=9000, hi=36000, new_lo=17, new_hi=48, heads=12,
             kv_heads=12, dim=64, turned=32, interleaved=True, tree=True, inst=4),
        # prompts into an 8-bit cache, and the written tokens read back
        dict(name="append_prompts", kind="append", type="fp8", seqs=16, lo=0, hi=1003, new_lo=777, new_hi=2048, heads=32,
             kv_heads=8, dim=128, turned=128, interleaved=False, tree=False, inst=1),
        # one conversation's draft
        dict(name="tree_one", kind="tree", type="bf16", seqs=1, lo=1440, hi=1440, new_lo=24, new_hi=24, empty=0, heads=16,
             kv_heads=2, dim=128, window=0, inst=1, lse=False),
        # a serving batch's drafts
        dict(name="tree_batch", kind="tree", type="bf16", seqs=32, lo=512, hi=2048, new_lo=16, new_hi=32, empty=0,
             heads=32, kv_heads=8, dim=128, window=0, inst=1, lse=False),
        # wide drafts far into long contexts on an 8-bit cache, seven query heads to a key-value head
        dict(name="tree_long", kind="tree", type="fp8", seqs=4, lo=16385, hi=32768, new_lo=64, new_hi=64, empty=0,
             heads=28, kv_heads=4, dim=128, window=0, inst=1, lse=True),
        # a padded batch of odd lengths and tree sizes over several caches, local attention, a key-value head per query head
        dict(name="tree_ragged", kind="tree", type="f16", seqs=37, lo=1, hi=12000, new_lo=1, new_hi=201, empty=3, heads=12,
             kv_heads=12, dim=64, window=4097, inst=4, lse=True),
        # one row of a small vocabulary
        dict(name="sample_one", kind="sample", type="f32", rows=1, vocab=32000, mix="top_p"),
        # a serving batch
        dict(name="sample_batch", kind="sample", type="bf16", rows=256, vocab=131072, mix="top_k_top_p"),
        # nothing left out: every token of an odd vocabulary may be drawn
        dict(name="sample_whole", kind="sample", type="f32", rows=64, vocab=100003, mix="whole"),
        # the nodes of a batch's trees, each sequence with settings of its own
        dict(name="sample_mixed", kind="sample", type="f16", rows=700, vocab=50001, mix="mixed"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


HEADS = {64: [(12, 12), (32, 8), (8, 1), (14, 2)], 128: [(32, 8), (16, 2), (28, 4), (8, 8), (12, 2)],
         256: [(16, 2), (8, 4), (8, 1)]}


def draw(rng):
    kind = rng.choice(["append", "tree", "tree", "sample"])
    if kind == "sample":
        rows = _log(rng, 1, 512)
        return dict(kind=kind, type=rng.choice(["bf16", "f16", "f32"]), rows=rows,
                    vocab=_log(rng, 100, min(262144, (32 << 20) // rows)),
                    mix=rng.choice(["top_p", "top_k_top_p", "whole", "mixed", "mixed"]))
    ty = rng.choice(["bf16", "bf16", "f16", "fp8", "fp8"])
    dim = rng.choice([64, 128, 128, 256])
    heads, kvh = rng.choice(HEADS[dim])
    inst = rng.choice([1, 1, 3])
    if kind == "append":
        tree = rng.random() < 0.3
        seqs = _log(rng, 1, 256)
        most = min(200 if tree else 4096, (48 << 20) // ((heads + kvh) * dim * seqs))
        new_hi = 1 if not tree and rng.random() < 0.4 else _log(rng, 2, max(3, most))
        hi = _log(rng, 1, max(2, min(50000, (100 << 20) // (kvh * dim * seqs))))
        turned = rng.choice([dim, dim, dim // 2, 16, dim - 16])
        return dict(kind=kind, type=ty, seqs=seqs, lo=hi // 3, hi=hi, new_lo=max(1, new_hi // rng.choice([1, 3])),
                    new_hi=new_hi, heads=heads, kv_heads=kvh, dim=dim, turned=turned, interleaved=rng.random() < 0.4,
                    tree=tree, inst=inst)
    seqs = _log(rng, 1, 64)
    new_hi = _log(rng, 1, min(256, max(2, 4096 // seqs)))
    # scores of the padded plain form within 2^31, products within the largest listed case, memory
    keys = min(65536, (1 << 31) // (seqs * heads * new_hi), (1 << 35) // (seqs * heads * dim * new_hi) * 5 // 8,
               (256 << 20) // (seqs * kvh * dim))
    hi = _log(rng, 16, max(17, keys))
    return dict(kind=kind, type=ty, seqs=seqs, lo=max(1, hi // rng.choice([1, 3, 50])), hi=hi,
                new_lo=max(1, new_hi // rng.choice([1, 4])), new_hi=new_hi, empty=rng.choice([0, 0, min(2, seqs - 1)]),
                heads=heads, kv_heads=kvh, dim=dim, window=rng.choice([0, 0, 0, _log(rng, 8, 4096)]), inst=inst,
                lse=rng.random() < 0.5)


# ------------------------------------------------------------------ inputs
def _spread(lo, hi, n):
    """n lengths from lo to hi, the same ones for every seed: spread evenly, or over the logarithm of a wide range."""
    u = (np.arange(n) + 0.5) / n if n > 1 else np.ones(1)
    if lo > 0 and hi > 8 * lo:
        return np.rint(np.exp(np.log(lo) + u * np.log(hi / lo))).astype(np.int64)
    return np.rint(lo + u * (hi - lo)).astype(np.int64)


def _lengths(case):
    """(cached tokens, new tokens) of every sequence, in the case's own order."""
    n = case["seqs"]
    cached, new = _spread(case["lo"], case["hi"], n), _spread(case["new_lo"], case["new_hi"], n)[::-1].copy()
    return cached, new


def _empty(case):
    """Sequences that are padding: their length is 0."""
    return case.get("empty", 0)


def _trees(new, rng):
    """Parents of every sequence's drafted tokens: a first one that follows the prefix, then each new one behind one of
    those before it, near the front more often (wide) or near the back (deep)."""
    out = []
    for n in new:
        j = np.arange(1, n)
        low = (j - 1) // rng.choice([1, 2, 4])
        p = np.minimum(low + (rng.random_sample(n - 1) * 3).astype(np.int64), j - 1)
        out.append(np.concatenate([[-1], p]))
    return np.concatenate(out)


def _depths(parent, starts):
    depth = np.zeros(len(parent), np.int64)
    for a, b in zip(starts[:-1], starts[1:]):
        for j in range(a, b):
            depth[j] = 0 if parent[j] < 0 else depth[a + parent[j]] + 1
    return depth


def _dev32(a):
    return torch.as_tensor(np.ascontiguousarray(a, np.int32)).cuda()


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    rng = np.random.RandomState(seed % (1 << 32))
    if case["kind"] == "sample":
        return _prepare_sample(case, g, rng)
    cached, new = _lengths(case)
    total = cached + new
    total[:_empty(case)] = 0
    order = rng.permutation(case["seqs"])
    new, total = new[order], total[order]
    n_inst, kvh, dim, heads = case["inst"], case["kv_heads"], case["dim"], case["heads"]
    inst = order % n_inst  # (the caches' size is then the same for every seed)
    blocks = -(-total // BLOCK)
    per_inst = max(int(sum(blocks[inst == i])) for i in range(n_inst)) * 5 // 4 + 8
    ids = np.full((case["seqs"], max(1, int(blocks.max()))), -1, np.int32)
    for i in range(n_inst):
        free = rng.permutation(per_inst)
        for r in np.nonzero(inst == i)[0]:
            ids[r, :blocks[r]], free = free[:blocks[r]], free[blocks[r]:]
    fp8 = case["type"] == "fp8"
    dt = torch.bfloat16 if fp8 else DTYPES[case["type"]]
    c = 16 if fp8 else 8
    nb = n_inst * per_inst

    def cache(*shape):
        if not fp8:
            return torch.randn(shape, device="cuda", generator=g, dtype=dt)
        x = torch.randn(shape, device="cuda", generator=g, dtype=dt)
        return (x * 64).clamp_(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8)

    n = int(new.sum())
    starts = np.concatenate([[0], np.cumsum(new)])
    s = dict(case=case, per_inst=per_inst, ids=_dev32(ids), inst=_dev32(inst) if n_inst > 1 else None,
             kv_len=_dev32(total), q_start=_dev32(starts), max_new=int(new.max()), scale=1.0 / math.sqrt(dim),
             k_scale=None, v_scale=None, pos=None, k=cache(nb, kvh, dim // c, BLOCK, c),
             v=cache(nb, kvh, dim // (2 * c), 16, 2, c // 8, 2, 4))
    if fp8:
        for name in ("k_scale", "v_scale"):
            s[name] = torch.randint(119, 123, (nb, kvh, BLOCK), device="cuda", generator=g, dtype=torch.uint8)
    parent = _trees(new, rng) if case["kind"] == "tree" or case["tree"] else None
    if case["kind"] == "tree":
        s["parent"] = _dev32(parent)
        s["q"] = torch.randn((n, heads, dim), device="cuda", generator=g, dtype=dt) * 2
        s["out"] = torch.empty_like(s["q"])
        s["lse"] = torch.empty((n, heads), dtype=torch.float32, device="cuda") if case["lse"] else None
        return s
    # slices of fused rows, as a projection leaves them; keys have a few outlying dimensions, as trained models' have
    rows = torch.randn((n, heads + 2 * kvh, dim), device="cuda", generator=g, dtype=dt)
    rows[:, heads:heads + kvh, ::37] *= 8
    s["q"], s["k_new"], s["v_new"] = rows.split([heads, kvh, kvh], dim=1)
    s["q_out"] = torch.empty((n, heads, dim), dtype=dt, device="cuda")
    if case["tree"]:
        s["pos"] = _dev32(np.repeat(total - new, new) + _depths(parent, starts))
    half = case["turned"] // 2
    s["inv_freq"] = torch.as_tensor((10000.0 ** (-np.arange(half) / half)).astype(np.float32)).cuda()
    s["factor"] = 1.0 if not case["interleaved"] else 1.125
    if fp8:
        s["k_out"] = torch.empty((n, kvh, dim), dtype=dt, device="cuda")
        s["v_out"] = torch.empty_like(s["k_out"])
    return s


def _prepare_sample(case, g, rng):
    n, vocab = case["rows"], case["vocab"]
    # a bulk and a few tokens that stand out, more in some rows than in others
    x = torch.randn((n, vocab), device="cuda", generator=g) * 2.5
    peak = torch.rand((n, vocab), device="cuda", generator=g) < 40.0 / vocab
    x += peak * torch.rand((n, vocab), device="cuda", generator=g) * (4 + 14 * torch.rand((n, 1), device="cuda", generator=g))
    x[:, vocab - vocab // 50:] = -math.inf  # the vocabulary is padded
    s = dict(case=case, temperature=None, top_k=None, top_p=None, min_p=None, seed=0)
    dev = lambda a: torch.as_tensor(np.ascontiguousarray(a, np.float32)).cuda()  # noqa: E731
    if case["mix"] == "top_p":
        s["temperature"], s["top_p"] = dev(np.full(n, 0.8)), dev(np.full(n, 0.95))
    elif case["mix"] == "top_k_top_p":
        s["temperature"], s["top_p"] = dev(0.6 + 0.4 * rng.random_sample(n)), dev(np.full(n, 0.9))
        s["top_k"] = _dev32(np.full(n, 50))
    elif case["mix"] == "mixed":
        s["temperature"] = dev(rng.choice([0.0, 0.3, 0.7, 1.0, 1.5], n))
        s["top_k"] = _dev32(rng.choice([0, 1, 20, 400, 30000], n))
        s["top_p"] = dev(rng.choice([1.0, 0.98, 0.9, 0.5], n))
        s["min_p"] = dev(rng.choice([0.0, 0.0, 0.02, 0.1], n))
        if n > 3:
            x[3] = -math.inf  # a grammar that allows nothing
    s["logits"] = x.to(DTYPES[case["type"]])
    s["u"] = torch.rand(n, device="cuda", generator=g)
    s["token"] = torch.empty(n, dtype=torch.int32, device="cuda")
    s["kept"] = torch.empty(n, dtype=torch.int32, device="cuda")
    s["prob"] = torch.empty(n, dtype=torch.float32, device="cuda")
    return s


# ------------------------------------------------------------------ the plain forms
def _blocks_of(s):
    """Pool blocks of every sequence's table, and whether there is one."""
    ids = s["ids"].long()
    there = ids >= 0
    ids = ids.clamp(min=0)
    if s["inst"] is not None:
        ids = ids + s["inst"].long()[:, None] * s["per_inst"]
    return ids, there


def _power(b):
    """2^(b - 127), b in 1..254, as the 32-bit number with those exponent bits."""
    return (b << 23).view(torch.float32)


def _rows(s, at):
    """Keys and values of the pool blocks `at` (any shape) as [..., head, token, dim] in 32 bits."""
    kvh, dim = s["case"]["kv_heads"], s["case"]["dim"]
    n = at.dim()
    lead = list(range(n))
    k, v = s["k"][at], s["v"][at]
    if s["k_scale"] is not None:
        k, v = k.view(torch.float8_e4m3fn), v.view(torch.float8_e4m3fn)
    k = k.float().permute(*lead, n, n + 2, n + 1, n + 3).reshape(*at.shape, kvh, BLOCK, dim)
    # [D / 2c][16][2][c / 8][2][4] -> token (t / 8, t / 4 % 2, t % 4), dimension (d / 2c, d / 16 % (c / 8), d % 16)
    v = v.float().permute(*lead, n, n + 5, n + 3, n + 6, n + 1, n + 4, n + 2).reshape(*at.shape, kvh, BLOCK, dim)
    if s["k_scale"] is not None:
        k = k * _power(s["k_scale"][at].int())[..., None]
        v = v * _power(s["v_scale"][at].int())[..., None]
    return k, v


def _new_tokens(s):
    """For every new token: its sequence, its number among the sequence's new tokens, its place in the sequence."""
    qs = s["q_start"].long()
    t = torch.arange(s["q"].shape[0], device="cuda")
    seq = torch.searchsorted(qs[1:].contiguous(), t, right=True)
    j = t - qs[seq]
    return seq, j, s["kv_len"].long()[seq] - (qs[seq + 1] - qs[seq]) + j


def _plain_tree(s):
    case = s["case"]
    kvh, dim, heads = case["kv_heads"], case["dim"], case["heads"]
    seq, j, place = _new_tokens(s)
    S, n = s["kv_len"].numel(), s["max_new"]
    # [sequence, token, token]: is the second one the first or its ancestor; paths of twice the length each time
    up = torch.zeros((S, n, n), dtype=torch.float32, device="cuda")
    p = s["parent"].long()
    up[seq, j, torch.where(p < 0, j, p)] = 1
    up[seq, j, j] = 1
    for _ in range((n - 1).bit_length()):
        up = (torch.bmm(up, up.contiguous()) > 0).float()
    depth = up.sum(-1).long() - 1
    new = (s["q_start"][1:] - s["q_start"][:-1]).long()
    base = s["kv_len"].long() - new

    ids, there = _blocks_of(s)
    keys = ids.shape[1] * BLOCK
    k, v = (x.transpose(1, 2).reshape(S, kvh, keys, dim) for x in _rows(s, ids))
    G = heads // kvh
    q = torch.zeros((S, n, heads, dim), dtype=torch.float32, device="cuda")
    q[seq, j] = s["q"].float()
    q = q.reshape(S, n, kvh, G, dim).permute(0, 2, 1, 3, 4).reshape(S, kvh, n * G, dim)
    scores = torch.matmul(q, k.transpose(2, 3).contiguous()).mul_(s["scale"])
    t = torch.arange(keys, device="cuda")
    at = (base[:, None] + depth)[:, :, None]  # a row's position
    node = t[None, :] - base[:, None]  # a key's number among the new tokens
    inside = (node >= 0) & (node < n)
    node = node.clamp(0, n - 1)
    seen = torch.gather(up, 2, node[:, None, :].expand(S, n, keys)) > 0
    seen = torch.where(inside[:, None, :], seen, t < base[:, None, None])
    if case["window"]:
        where = torch.where(inside, base[:, None] + torch.gather(depth, 1, node), t[None, :])
        seen &= where[:, None, :] > at - case["window"]
    seen &= there.repeat_interleave(BLOCK, 1)[:, None, :] & (t < s["kv_len"].long()[:, None, None])
    scores = scores.view(S, kvh, n, G, keys).masked_fill_(~seen[:, None, :, None, :], -math.inf)
    top = scores.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, torch.zeros_like(top), top)
    w = scores.sub_(top).exp_()
    z = w.sum(-1, keepdim=True)
    out = torch.matmul(w.view(S, kvh, n * G, keys), v).view(S, kvh, n, G, dim)
    out = out / torch.where(z == 0, torch.ones_like(z), z)
    lse = (top + z.log()).squeeze(-1)
    out = out.permute(0, 2, 1, 3, 4).reshape(S, n, heads, dim)[seq, j].to(s["q"].dtype)
    if s["lse"] is None:
        return dict(out=out)
    return dict(out=out, lse=lse.permute(0, 2, 1, 3).reshape(S, n, heads)[seq, j])


def _turn(s, x, pos):
    """Rows x [n, head, dim] turned by their positions' angles, in 32 bits."""
    R = s["case"]["turned"]
    angle = pos.double()[:, None, None] * s["inv_freq"].double()
    cos, sin = (angle.cos() * s["factor"]).float(), (angle.sin() * s["factor"]).float()
    x = x.float()
    if s["case"]["interleaved"]:
        a, b = x[..., 0:R:2], x[..., 1:R:2]
        y = torch.stack([a * cos - b * sin, a * sin + b * cos], -1).flatten(-2)
    else:
        a, b = x[..., :R // 2], x[..., R // 2:R]
        y = torch.cat([a * cos - b * sin, a * sin + b * cos], -1)
    return torch.cat([y, x[..., R:]], -1)


def _quantise(x):
    """x [n, head, dim] as float8 e4m3 values (their bytes) and the byte of a power-of-two scale per row: the
    smallest one for which no value passes 448; 1 for a row of zeros."""
    m, e = torch.frexp(x.abs().amax(-1))  # x = m 2^e, m in [0.5, 1)
    e = torch.where(m == 0, torch.zeros_like(e), (e - 9 + (m > 0.875).int()).clamp(min=-126))
    return (x * _power(127 - e)[..., None]).to(torch.float8_e4m3fn).view(torch.uint8), (e + 127).to(torch.uint8)


def _places(s):
    """Pool block and token of the block of every new token."""
    seq, _, place = _new_tokens(s)
    ids, _ = _blocks_of(s)
    return ids[seq, place // BLOCK], place % BLOCK


def _plain_append(s):
    blk, t = _places(s)
    pos = _new_tokens(s)[2] if s["pos"] is None else s["pos"]
    dt = s["q"].dtype
    q, k, v = _turn(s, s["q"], pos).to(dt), _turn(s, s["k_new"], pos), s["v_new"]
    n, kvh, dim = k.shape
    fp8 = s["k_scale"] is not None
    c = 16 if fp8 else 8
    if fp8:
        k, ks = _quantise(k)
        v, vs = _quantise(v.float())
        s["k_scale"][blk, :, t] = ks
        s["v_scale"][blk, :, t] = vs
    else:
        k = k.to(dt)
    s["k"][blk, :, :, t] = k.reshape(n, kvh, dim // c, c)
    s["v"][blk, :, :, :, t // 4 % 2, :, t // 8, t % 4] = v.reshape(n, kvh, dim // (2 * c), c // 8, 16).transpose(3, 4)
    if not fp8:
        return dict(q=q, k=s["k"], v=s["v"])
    k = s["k"][blk, :, :, t].view(torch.float8_e4m3fn).float() * _power(s["k_scale"][blk, :, t].int())[..., None, None]
    v = s["v"][blk, :, :, :, t // 4 % 2, :, t // 8, t % 4].transpose(3, 4).contiguous()
    v = v.view(torch.float8_e4m3fn).float() * _power(s["v_scale"][blk, :, t].int())[..., None, None, None]
    return dict(q=q, k=k.reshape(n, kvh, dim).to(dt), v=v.reshape(n, kvh, dim).to(dt))


def _setting(s, name, off):
    x = s[name]
    return torch.full((s["case"]["rows"], 1), off, dtype=torch.float64, device="cuda") if x is None else x.double()[:, None]


def _plain_sample(s):
    x = s["logits"].float()
    x = torch.where(torch.isnan(x), torch.full_like(x, -math.inf), x)
    l, order = torch.sort(x, dim=1, descending=True, stable=True)
    l = l.double()
    T, k, p, m = _setting(s, "temperature", 1.0), _setting(s, "top_k", 0), _setting(s, "top_p", 1.0), _setting(s, "min_p", 0.0)
    # (64 bits: a sum next to a border decides which token is taken)
    first = torch.arange(x.shape[1], device="cuda")[None] == 0
    w = torch.where(l == l[:, :1], torch.ones_like(l), torch.exp((l - l[:, :1]) / torch.where(T > 0, T, torch.ones_like(T))))
    rank = torch.arange(x.shape[1], device="cuda")[None]
    keep = (rank < k) | (k <= 0)
    a = w * keep
    keep &= (a.cumsum(1) - a < p * a.sum(1, keepdim=True)) | (p >= 1)
    keep &= (w >= m) | (m <= 0)
    keep &= T > 0
    keep |= first
    keep &= l > -math.inf
    kept = keep.sum(1)
    w = w * keep
    c = w.cumsum(1)
    passed = c > s["u"].double()[:, None] * c[:, -1:]
    # (a sum that never passes, by rounding: the last one with a weight)
    at = torch.where(passed.any(1), passed.int().argmax(1), (w > 0).sum(1) - 1).clamp(min=0)[:, None]
    token, prob = order.gather(1, at).squeeze(1), w.gather(1, at).squeeze(1) / c[:, -1]
    none = kept == 0
    return dict(token=torch.where(none, -torch.ones_like(token), token).int(), kept=kept.int(),
                prob=torch.where(none, torch.zeros_like(prob), prob).float())


def _run_plain(s):
    return {"append": _plain_append, "tree": _plain_tree, "sample": _plain_sample}[s["case"]["kind"]](s)


# ------------------------------------------------------------------ the framework's operators
def _handles(s):
    """What a program keeps beside its buffers: the cache's, the batch's and the angles' descriptions, a workspace."""
    from paper_2605_18825_amd import api
    case = s["case"]
    if case["kind"] == "sample":
        s["work"] = torch.empty(api.sae_sample_work_size(case["rows"], case["vocab"]), dtype=torch.uint8, device="cuda")
        return
    ty = {"bf16": api.KV_BF16, "f16": api.KV_F16, "fp8": api.KV_FP8}[case["type"]]
    s["kv"] = api.make_kv(ty, case["inst"], s["per_inst"], case["kv_heads"], case["dim"], s["k"], s["v"],
                          k_scale=s["k_scale"], v_scale=s["v_scale"])
    s["seqs"] = api.make_seqs(s["ids"], s["kv_len"], q_start=s["q_start"], inst=s["inst"])
    if case["kind"] == "tree":
        n = api.sae_attn_work_size(s["kv"], s["seqs"], s["q"].shape[0], case["heads"])
        s["work"] = torch.empty(n, dtype=torch.uint8, device="cuda")
    else:
        s["rope"] = api.make_rope(s["inv_freq"], interleaved=case["interleaved"], factor=s["factor"])
        s["work"] = None


def _run_own(s):
    from paper_2605_18825_amd import api
    if "work" not in s:
        _handles(s)
    kind = s["case"]["kind"]
    if kind == "append":
        api.sae_kv_append(s["kv"], s["seqs"], s["rope"], s["q"], s["q_out"], s["k_new"], s["v_new"], pos=s["pos"])
        if s["k_scale"] is None:
            return dict(q=s["q_out"], k=s["k"], v=s["v"])
        api.sae_kv_read(s["kv"], s["seqs"], s["k_out"], s["v_out"])
        return dict(q=s["q_out"], k=s["k_out"], v=s["v_out"])
    if kind == "tree":
        api.sae_attn_tree(s["kv"], s["seqs"], s["parent"], s["max_new"], s["q"], s["out"], s["scale"], s["work"],
                          window=s["case"]["window"], lse=s["lse"])
        return dict(out=s["out"]) if s["lse"] is None else dict(out=s["out"], lse=s["lse"])
    api.sae_sample(s["logits"], s["u"], s["token"], s["work"], temperature=s["temperature"], top_k=s["top_k"],
                   top_p=s["top_p"], min_p=s["min_p"], prob=s["prob"], kept=s["kept"])
    return dict(token=s["token"], kept=s["kept"], prob=s["prob"])


def run(s):
    return _run_own(s) if own else _run_plain(s)


# ------------------------------------------------------------------ what a pass cannot do without
def work(case):
    if case["kind"] == "sample":
        n = case["rows"]
        size = 4 if case["type"] == "f32" else 2
        return dict(bytes=n * case["vocab"] * size + 32 * n, flops=0)
    cached, new = _lengths(case)
    live = np.arange(case["seqs"]) >= _empty(case)
    kvh, dim, heads = case["kv_heads"], case["dim"], case["heads"]
    fp8 = case["type"] == "fp8"
    token = 2 * kvh * (dim + 1 if fp8 else 2 * dim)  # a token's keys and values in the cache
    rows = int(new.sum())
    tables = 4 * int(sum(-(-(cached + new) // BLOCK))) + 8 * case["seqs"]
    if case["kind"] == "append":
        plain = 2 * kvh * dim * 2
        return dict(bytes=rows * (4 * heads * dim + plain + token + (token + plain if fp8 else 0)) + tables +
                    (4 * rows if case["tree"] else 0), flops=0)
    win = case["window"] or 1 << 60
    pairs = int((new * (np.minimum(cached, win) + 1) * live).sum())  # at least: prefix and itself
    keys = int(((np.minimum(cached, win) + new) * live).sum())
    lse = 4 * rows * heads if case["lse"] else 0
    return dict(bytes=keys * token + 2 * rows * heads * dim * 2 + 4 * rows + lse + tables, flops=4 * pairs * heads * dim)


# ------------------------------------------------------------------ the definitions in 64 bits
def _e4m3(x):
    """The float8 e4m3 value nearest to x (|x| <= 448; ties to the even one)."""
    e = torch.floor(torch.log2(x.abs().clamp(min=2.0 ** -40)))
    e = torch.where(torch.exp2(e) > x.abs(), e - 1, e)
    step = torch.exp2(e.clamp(min=-6) - 3)
    return torch.round(x / step) * step


def _held(x):
    """What an 8-bit cache holds for rows x."""
    big = x.abs().amax(-1, keepdim=True)
    e = torch.ceil(torch.log2(big / 448))
    e = torch.where(448 * torch.exp2(e - 1) >= big, e - 1, e)  # log2 rounded up past a whole number
    return _e4m3(x * torch.exp2(-e)) * torch.exp2(e)


def _offsets(case):
    """Place in a page of (token, dimension), of keys and of values."""
    dim = case["dim"]
    d, t = torch.arange(dim, device="cuda")[None, :], torch.arange(BLOCK, device="cuda")[:, None]
    c = 16 if case["type"] == "fp8" else 8
    return (d // c * 16 * c + t * c + d % c,
            ((((d // (2 * c) * 16 + d % 16) * 2 + t // 4 % 2) * (c // 8) + d // 16 % (c // 8)) * 2 + t // 8) * 4 + t % 4)


def _exact_append(case, s):
    starts, lens = s["q_start"].tolist(), s["kv_len"].tolist()
    R, dim = case["turned"], case["dim"]
    place = torch.cat([torch.arange(n - (b - a), n, device="cuda") for a, b, n in zip(starts, starts[1:], lens)])
    pos = (place if s["pos"] is None else s["pos"]).double()
    # a pair (x, y) as x + iy, times e^(i angle)
    one = torch.arange(R // 2, device="cuda")
    i, j = (2 * one, 2 * one + 1) if case["interleaved"] else (one, one + R // 2)
    by = torch.polar(torch.full((1, 1), s["factor"], dtype=torch.float64, device="cuda"),
                     pos[:, None] * s["inv_freq"].double()[None, :])[:, None, :]

    def turned(x):
        x = x.double()
        z = torch.complex(x[..., i].contiguous(), x[..., j].contiguous()) * by
        y = x.clone()
        y[..., i], y[..., j] = z.real, z.imag
        return y
    q, k = turned(s["q"]), turned(s["k_new"])
    if case["type"] == "fp8":
        return dict(q=q, k=_held(k), v=_held(s["v_new"].double()))
    cache = s["k"].double().reshape(s["k"].shape[0], case["kv_heads"], -1)
    at = _offsets(case)[0]
    for r, (a, b) in enumerate(zip(starts, starts[1:])):
        p = place[a:b]
        blk = s["ids"][r].long()[p // BLOCK] + (0 if s["inst"] is None else int(s["inst"][r]) * s["per_inst"])
        for h in range(case["kv_heads"]):
            cache[blk[:, None], h, at[p % BLOCK]] = k[a:b, h]
    return dict(q=q, k=cache.reshape(s["k"].shape), v=None)  # values are a copy


def _exact_tree(case, s):
    kvh, dim, heads = case["kv_heads"], case["dim"], case["heads"]
    G = heads // kvh
    starts, lens, parent = s["q_start"].tolist(), s["kv_len"].tolist(), s["parent"].tolist()
    n = starts[-1]
    out = torch.zeros((n, heads, dim), dtype=torch.float64, device="cuda")
    lse = torch.full((n, heads), -math.inf, dtype=torch.float64, device="cuda")
    at_k, at_v = _offsets(case)
    for r, total in enumerate(lens):
        a, b = starts[r], starts[r + 1]
        if total == 0:
            continue
        base = total - (b - a)
        seen = np.zeros((b - a, total), bool)
        depth = np.zeros(b - a, np.int64)
        for j in range(b - a):
            chain = [j]
            while parent[a + chain[-1]] >= 0:
                chain.append(parent[a + chain[-1]])
            depth[j] = len(chain) - 1
            near = chain[:case["window"]] if case["window"] else chain
            seen[j, base + np.array(near)] = True
            seen[j, max(0, base + depth[j] - case["window"] + 1) if case["window"] else 0:base] = True
        hidden = ~torch.as_tensor(seen).cuda()
        blk = s["ids"][r, :-(-total // BLOCK)].long() + (0 if s["inst"] is None else int(s["inst"][r]) * s["per_inst"])
        for h in range(kvh):
            kv = []
            for x, scale, at in ((s["k"], s["k_scale"], at_k), (s["v"], s["v_scale"], at_v)):
                page = x[blk, h].reshape(len(blk), -1)[:, at.reshape(-1)].reshape(len(blk), BLOCK, dim)
                if scale is not None:
                    page = page.view(torch.float8_e4m3fn).double() * torch.exp2(scale[blk, h].double() - 127)[..., None]
                kv.append(page.double().reshape(-1, dim)[:total])
            kt = kv[0].t().contiguous()
            for u in range(h * G, h * G + G):
                x = (s["q"][a:b, u].double() @ kt * s["scale"]).masked_fill_(hidden, -math.inf)
                top = x.amax(1, keepdim=True)
                w = torch.exp(x - top)
                z = w.sum(1, keepdim=True)
                out[a:b, u] = (w @ kv[1]) / z
                lse[a:b, u] = (top + torch.log(z))[:, 0]
    return dict(out=out, lse=lse) if case["lse"] else dict(out=out)


def _exact_sample(case, s):
    x = s["logits"].double().cpu().numpy()
    u = s["u"].double().cpu().numpy()
    get = lambda name, off: [off] * case["rows"] if s[name] is None else s[name].double().tolist()  # noqa: E731
    settings = zip(get("temperature", 1.0), get("top_k", 0), get("top_p", 1.0), get("min_p", 0.0))
    prob = np.zeros(case["rows"])
    for r, (T, k, p, m) in enumerate(settings):
        l = x[r]
        ids = np.nonzero(l > -np.inf)[0]
        if not len(ids):
            continue
        ids = ids[np.lexsort((ids, -l[ids]))]
        if T <= 0:
            prob[r] = 1
            continue
        w = np.exp((l[ids] - l[ids[0]]) / T)
        if k > 0:
            ids, w = ids[:int(k)], w[:int(k)]
        n = len(ids)
        if p < 1:
            n = max(1, int(np.searchsorted(np.cumsum(w), p * w.sum(), side="left")) + 1)
        if m > 0:
            n = max(1, min(n, int((w >= m).sum())))
        c = np.cumsum(w[:n])
        at = min(int(np.searchsorted(c, u[r] * c[-1], side="right")), n - 1)
        prob[r] = w[at] / c[-1]
    return dict(token=None, kept=None, prob=torch.as_tensor(prob))


def exact(case, seed):
    s = prepare(case, seed)
    return {"append": _exact_append, "tree": _exact_tree, "sample": _exact_sample}[case["kind"]](case, s)
