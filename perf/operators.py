"""Measured cases of the paged key-value cache: writing it, reading it back, and the attention over it.

Four operators on the block pool whose blocks the eviction path manages (16 tokens a block, block ids from a
prefix match or from freed slots):
  write    new keys and values go to the positions at the end of their sequences; an 8-bit cache is quantised
           as it is written, with one power-of-two scale per token and head, and then read back
  read     the last positions of each sequence as plain rows, dequantised
  decode   attention of one new token per sequence over its cached keys and values
  prefill  causal attention of each sequence's new tokens over its cached prefix and themselves

Cache layout (values; one layer): a block holds one page per key-value head.  With c = 16 bytes / value size,
keys [block][head][D / c][16 tokens][c]; values [block][head][D / 2c][16][2][c / 8][2][4], where token t and
dimension d of the page are at [d / 2c][d % 16][t / 4 % 2][d / 16 % (c / 8)][t / 8][t % 4].  Scales of an 8-bit
cache (float8 e4m3 values): one byte b per [block][head][16 tokens], for keys and for values, standing for
2^(b - 127).
"""
import math

import numpy as np
import torch

own = False

BLOCK = 16
DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16}


def listed():
    return [
        # one conversation's next token on a small model's cache: latency of a single call
        dict(name="decode_one", kind="decode", type="bf16", seqs=1, lo=1440, hi=1440, empty=0, heads=16, kv_heads=2,
             dim=128, window=0, inst=1, lse=False),
        # a serving batch, every sequence up to 128 blocks long
        dict(name="decode_batch", kind="decode", type="bf16", seqs=256, lo=512, hi=2048, empty=0, heads=32, kv_heads=8,
             dim=128, window=0, inst=1, lse=False),
        # a single long document on an 8-bit cache
        dict(name="decode_long", kind="decode", type="fp8", seqs=1, lo=131072, hi=131072, empty=0, heads=32,
             kv_heads=8, dim=128, window=0, inst=1, lse=True),
        # a padded batch of odd lengths over several caches, local attention, a key-value head per query head
        dict(name="decode_ragged", kind="decode", type="f16", seqs=37, lo=1, hi=36000, empty=3, heads=12, kv_heads=12,
             dim=64, window=4097, inst=4, lse=True),
        # the next turn of a conversation whose history is cached
        dict(name="prefill_turn", kind="prefill", type="bf16", seqs=1, lo=1440, hi=1440, new_lo=61, new_hi=61, heads=16,
             kv_heads=2, dim=128, window=0, inst=1, lse=False),
        # a batch of requests that matched a part of their prompts
        dict(name="prefill_batch", kind="prefill", type="bf16", seqs=16, lo=0, hi=2000, new_lo=90, new_hi=1100,
             heads=32, kv_heads=8, dim=128, window=0, inst=1, lse=False),
        # a long prompt behind a cached system prompt
        dict(name="prefill_long", kind="prefill", type="bf16", seqs=1, lo=4096, hi=4096, new_lo=8192, new_hi=8192,
             heads=32, kv_heads=8, dim=128, window=0, inst=1, lse=True),
        # chunks of prompts far into long contexts on an 8-bit cache, seven query heads to a key-value head
        dict(name="prefill_chunks", kind="prefill", type="fp8", seqs=4, lo=9001, hi=16384, new_lo=512, new_hi=512,
             heads=28, kv_heads=4, dim=128, window=0, inst=2, lse=False),
        # what a decode step of a serving batch writes
        dict(name="write_step", kind="write", type="bf16", seqs=256, lo=512, hi=2048, new_lo=1, new_hi=1, kv_heads=8,
             dim=128, inst=1),
        # prompts written to an 8-bit cache, and the written tokens read back
        dict(name="write_prompts", kind="write", type="fp8", seqs=32, lo=0, hi=1003, new_lo=777, new_hi=2048,
             kv_heads=8, dim=128, inst=1),
        # one small cache's longest request read back
        dict(name="read_one", kind="read", type="f16", seqs=1, lo=0, hi=0, new_lo=1440, new_hi=1440, kv_heads=2,
             dim=64, inst=1),
        # the prefixes of a batch read from an 8-bit cache
        dict(name="read_batch", kind="read", type="fp8", seqs=64, lo=0, hi=500, new_lo=301, new_hi=2250, kv_heads=8,
             dim=128, inst=4),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


HEADS = {64: [(12, 12), (32, 8), (8, 1), (14, 2)], 128: [(32, 8), (16, 2), (28, 4), (8, 8), (12, 2)],
         256: [(16, 2), (8, 4), (8, 1)]}


def draw(rng):
    kind = rng.choice(["decode", "decode", "prefill", "prefill", "write", "read"])
    ty = rng.choice(["bf16", "bf16", "f16", "fp8", "fp8"])
    dim = rng.choice([64, 128, 128, 256])
    heads, kvh = rng.choice(HEADS[dim])
    inst = rng.choice([1, 1, 3])
    row = kvh * dim  # values of one token's keys
    if kind == "decode":
        seqs = _log(rng, 1, 256)
        hi = _log(rng, 16, max(17, min(131072, (300 << 20) // (row * seqs))))
        lo = max(1, hi // rng.choice([1, 3, 50]))
        return dict(kind=kind, type=ty, seqs=seqs, lo=lo, hi=hi, empty=rng.choice([0, 0, min(2, seqs - 1)]), heads=heads,
                    kv_heads=kvh, dim=dim, window=rng.choice([0, 0, 0, _log(rng, 64, 4096)]), inst=inst,
                    lse=rng.random() < 0.5)
    if kind == "prefill":
        seqs = _log(rng, 1, 32)
        new_hi = _log(rng, 2, max(3, min(8192, 16384 // seqs)))
        # scores of the padded plain form within 2^32, products within the largest listed case
        keys = min(32768, (1 << 32) // (seqs * heads * new_hi), (1 << 41) // (8 * seqs * heads * dim * new_hi))
        hi = max(0, min(_log(rng, 16, max(17, keys)), keys) - new_hi)
        return dict(kind=kind, type=ty, seqs=seqs, lo=hi // rng.choice([1, 3, 50]), hi=hi,
                    new_lo=max(1, new_hi // rng.choice([1, 4])), new_hi=new_hi, heads=heads, kv_heads=kvh, dim=dim,
                    window=rng.choice([0, 0, 0, _log(rng, 64, 4096)]), inst=inst, lse=rng.random() < 0.5)
    seqs = _log(rng, 1, 256)
    new_hi = 1 if kind == "write" and rng.random() < 0.3 else _log(rng, 2, max(3, min(8192, (64 << 20) // (row * seqs))))
    hi = _log(rng, 1, 2048)
    return dict(kind=kind, type=ty, seqs=seqs, lo=hi // 3, hi=hi, new_lo=max(1, new_hi // rng.choice([1, 3])),
                new_hi=new_hi, kv_heads=kvh, dim=dim, inst=inst)


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
    cached = _spread(case["lo"], case["hi"], n)
    if case["kind"] == "decode":
        cached[:case["empty"]] = 0
        return cached, np.ones(n, np.int64)
    # longer prefixes with shorter suffixes, and the other way round
    return cached, _spread(case["new_lo"], case["new_hi"], n)[::-1].copy()


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    rng = np.random.RandomState(seed % (1 << 32))
    cached, new = _lengths(case)
    order = rng.permutation(case["seqs"])
    cached, new = cached[order], new[order]
    total = cached if case["kind"] == "decode" else cached + new  # a decode's lengths count its new token
    n_inst, kvh, dim = case["inst"], case["kv_heads"], case["dim"]
    inst = np.arange(case["seqs"]) % n_inst
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

    n_new = int(new.sum())
    dev = lambda a: torch.as_tensor(np.ascontiguousarray(a, np.int32)).cuda()  # noqa: E731
    s = dict(case=case, per_inst=per_inst, ids=dev(ids), inst=dev(inst) if n_inst > 1 else None, kv_len=dev(total),
             q_start=None if case["kind"] == "decode" else dev(np.concatenate([[0], np.cumsum(new)])),
             max_new=int(new.max()), scale=1.0 / math.sqrt(dim), k_scale=None, v_scale=None,
             k=cache(nb, kvh, dim // c, BLOCK, c), v=cache(nb, kvh, dim // (2 * c), 16, 2, c // 8, 2, 4))
    if fp8:
        for name in ("k_scale", "v_scale"):
            s[name] = torch.randint(119, 123, (nb, kvh, BLOCK), device="cuda", generator=g, dtype=torch.uint8)
    if case["kind"] in ("decode", "prefill"):
        heads = case["heads"]
        s["q"] = torch.randn((n_new, heads, dim), device="cuda", generator=g, dtype=dt) * 2
        s["out"] = torch.empty_like(s["q"])
        s["lse"] = torch.empty((n_new, heads), dtype=torch.float32, device="cuda") if case["lse"] else None
    else:
        if case["kind"] == "write":
            # keys have a few outlying dimensions, as trained models' keys do
            s["k_new"] = torch.randn((n_new, kvh, dim), device="cuda", generator=g, dtype=dt)
            s["k_new"][..., ::37] *= 8
            s["v_new"] = torch.randn((n_new, kvh, dim), device="cuda", generator=g, dtype=dt)
        s["k_out"] = torch.empty((n_new, kvh, dim), dtype=dt, device="cuda")
        s["v_out"] = torch.empty_like(s["k_out"])
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


def _power(b):
    """2^(b - 127), b in 1..254, as the 32-bit number with those exponent bits."""
    return (b << 23).view(torch.float32)


def _attention(s, q, at):
    """q [seq, new, head, dim] at positions at [seq, new]: outputs and log-sum-exps, in 32 bits."""
    case = s["case"]
    kvh, dim = case["kv_heads"], case["dim"]
    ids, there = _blocks_of(s)
    S, M = ids.shape
    k, v = (x.transpose(1, 2).reshape(S, kvh, M * BLOCK, dim) for x in _rows(s, ids))
    n, G = q.shape[1], q.shape[2] // kvh
    q = q.float().reshape(S, n, kvh, G, dim).permute(0, 2, 1, 3, 4).reshape(S, kvh, n * G, dim)
    scores = torch.matmul(q, k.transpose(2, 3).contiguous()).mul_(s["scale"])
    pos = torch.arange(M * BLOCK, device="cuda")
    seen = there.repeat_interleave(BLOCK, 1)[:, None, :] & (pos <= at[..., None])
    if case["window"]:
        seen &= pos > at[..., None] - case["window"]
    seen = seen[:, None, :, None, :]
    scores = scores.view(S, kvh, n, G, M * BLOCK).masked_fill_(~seen, -math.inf)
    top = scores.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, torch.zeros_like(top), top)
    p = scores.sub_(top).exp_()
    total = p.sum(-1, keepdim=True)
    out = torch.matmul(p.view(S, kvh, n * G, M * BLOCK), v).view(S, kvh, n, G, dim)
    out = out / torch.where(total == 0, torch.ones_like(total), total)
    lse = (top + total.log()).squeeze(-1)
    shape = (S, n, kvh * G)
    return out.permute(0, 2, 1, 3, 4).reshape(*shape, dim), lse.permute(0, 2, 1, 3).reshape(shape)


def _new_tokens(s):
    """For every new token: its sequence, its number among the sequence's new tokens, its position."""
    qs = s["q_start"].long()
    n = s["k_out"].shape[0] if "k_out" in s else s["q"].shape[0]
    t = torch.arange(n, device="cuda")
    seq = torch.searchsorted(qs[1:].contiguous(), t, right=True)
    j = t - qs[seq]
    return seq, j, s["kv_len"].long()[seq] - (qs[seq + 1] - qs[seq]) + j


def _plain_attention(s):
    if s["case"]["kind"] == "decode":
        at = s["kv_len"].long()[:, None] - 1
        out, lse = _attention(s, s["q"][:, None], at)
        return out[:, 0], lse[:, 0]
    seq, j, pos = _new_tokens(s)
    S, n = s["kv_len"].numel(), s["max_new"]
    q = torch.zeros((S, n, *s["q"].shape[1:]), dtype=torch.float32, device="cuda")
    q[seq, j] = s["q"].float()
    at = torch.full((S, n), -1, dtype=torch.int64, device="cuda")
    at[seq, j] = pos
    out, lse = _attention(s, q, at)
    return out[seq, j], lse[seq, j]


def _quantise(x):
    """x [n, head, dim] as float8 e4m3 values (their bytes) and the byte of a power-of-two scale per row: the
    smallest one for which no value passes 448; 1 for a row of zeros."""
    m, e = torch.frexp(x.abs().amax(-1))  # x = m 2^e, m in [0.5, 1)
    e = torch.where(m == 0, torch.zeros_like(e), (e - 9 + (m > 0.875).int()).clamp(min=-126))
    return (x * _power(127 - e)[..., None]).to(torch.float8_e4m3fn).view(torch.uint8), (e + 127).to(torch.uint8)


def _places(s):
    """Pool block and token of the block of every new position."""
    seq, _, pos = _new_tokens(s)
    ids, _ = _blocks_of(s)
    return ids[seq, pos // BLOCK], pos % BLOCK


def _plain_write(s):
    blk, t = _places(s)
    n, kvh, dim = s["k_new"].shape
    k, v = s["k_new"], s["v_new"]
    c = 8
    if s["k_scale"] is not None:
        c = 16
        k, ks = _quantise(k.float())
        v, vs = _quantise(v.float())
        s["k_scale"][blk, :, t] = ks
        s["v_scale"][blk, :, t] = vs
    s["k"][blk, :, :, t] = k.reshape(n, kvh, dim // c, c)
    s["v"][blk, :, :, :, t // 4 % 2, :, t // 8, t % 4] = v.reshape(n, kvh, dim // (2 * c), c // 8, 16).transpose(3, 4)


def _plain_read(s):
    blk, t = _places(s)
    kvh, dim = s["case"]["kv_heads"], s["case"]["dim"]
    n = blk.numel()
    c = 16 if s["k_scale"] is not None else 8
    k = s["k"][blk, :, :, t]
    v = s["v"][blk, :, :, :, t // 4 % 2, :, t // 8, t % 4].transpose(3, 4)
    if s["k_scale"] is not None:
        k = k.view(torch.float8_e4m3fn).float() * _power(s["k_scale"][blk, :, t].int())[..., None, None]
        v = v.contiguous().view(torch.float8_e4m3fn).float() * _power(s["v_scale"][blk, :, t].int())[..., None, None, None]
    dt = s["k_out"].dtype
    return k.reshape(n, kvh, dim).to(dt), v.reshape(n, kvh, dim).to(dt)


def _run_plain(s):
    kind = s["case"]["kind"]
    if kind in ("decode", "prefill"):
        out, lse = _plain_attention(s)
        r = dict(out=out.to(s["q"].dtype))
        if s["lse"] is not None:
            r["lse"] = lse
        return r
    if kind == "write":
        _plain_write(s)
        if s["k_scale"] is None:
            return dict(k=s["k"], v=s["v"])
        r = dict(zip(("k", "v"), _plain_read(s)))
        return dict(r, k_scale=s["k_scale"], v_scale=s["v_scale"])
    return dict(zip(("k", "v"), _plain_read(s)))


# ------------------------------------------------------------------ the framework's operators
def _handles(s):
    """What a program keeps beside its buffers: the cache's and the batch's descriptions and a workspace."""
    from paper_2605_18825_amd import api
    case = s["case"]
    ty = {"bf16": api.KV_BF16, "f16": api.KV_F16, "fp8": api.KV_FP8}[case["type"]]
    s["kv"] = api.make_kv(ty, case["inst"], s["per_inst"], case["kv_heads"], case["dim"], s["k"], s["v"],
                          k_scale=s["k_scale"], v_scale=s["v_scale"])
    s["seqs"] = api.make_seqs(s["ids"], s["kv_len"], q_start=s["q_start"], inst=s["inst"])
    if "q" in s:
        n = api.sae_attn_work_size(s["kv"], s["seqs"], s["q"].shape[0], case["heads"])
        s["work"] = torch.empty(n, dtype=torch.uint8, device="cuda")


def _run_own(s):
    from paper_2605_18825_amd import api
    if "kv" not in s:
        _handles(s)
    case = s["case"]
    kind, kv, seqs = case["kind"], s["kv"], s["seqs"]
    if kind in ("decode", "prefill"):
        call = api.sae_attn_decode if kind == "decode" else api.sae_attn_prefill
        call(kv, seqs, s["q"], s["out"], s["scale"], s["work"], window=case["window"], lse=s["lse"])
        return dict(out=s["out"]) if s["lse"] is None else dict(out=s["out"], lse=s["lse"])
    if kind == "write":
        api.sae_kv_write(kv, seqs, s["k_new"], s["v_new"])
        if s["k_scale"] is None:
            return dict(k=s["k"], v=s["v"])
    api.sae_kv_read(kv, seqs, s["k_out"], s["v_out"])
    r = dict(k=s["k_out"], v=s["v_out"])
    if kind == "write":
        r.update(k_scale=s["k_scale"], v_scale=s["v_scale"])
    return r


def run(s):
    return _run_own(s) if own else _run_plain(s)


# ------------------------------------------------------------------ what a pass cannot do without
def work(case):
    cached, new = _lengths(case)
    kvh, dim = case["kv_heads"], case["dim"]
    fp8 = case["type"] == "fp8"
    token = 2 * kvh * (dim + 1 if fp8 else 2 * dim)  # a token's keys and values in the cache
    rows = int(new.sum())
    plain = 2 * kvh * dim * 2  # a token's keys and values as plain rows
    tables = 4 * int(sum(-(-(cached + new) // BLOCK))) + 8 * case["seqs"]
    if case["kind"] == "write":
        return dict(bytes=rows * (plain + token + (token + plain if fp8 else 0)) + tables, flops=0)
    if case["kind"] == "read":
        return dict(bytes=rows * (plain + token) + tables, flops=0)
    heads, win = case["heads"], case["window"] or 1 << 60
    if case["kind"] == "decode":
        pairs = keys = int(np.minimum(cached, win).sum())
    else:
        # query j of a sequence sees min(cached + j + 1, window) keys
        pairs = sum(int(np.minimum(c + 1 + np.arange(n), win).sum()) for c, n in zip(cached, new))
        keys = int(np.minimum(cached + new, win + new - 1).sum())
    lse = 4 * rows * heads if case["lse"] else 0
    return dict(bytes=keys * token + 2 * rows * heads * dim * 2 + lse + tables, flops=4 * pairs * heads * dim)


# ------------------------------------------------------------------ the definitions in 64 bits
def _e4m3(x):
    """The float8 e4m3 value nearest to x (|x| <= 448; ties to the even one)."""
    e = torch.floor(torch.log2(x.abs().clamp(min=2.0 ** -40)))
    e = torch.where(torch.exp2(e) > x.abs(), e - 1, e)
    step = torch.exp2(e.clamp(min=-6) - 3)
    return torch.round(x / step) * step


def _exact_cache(s):
    """A function giving (keys, values) of sequence r, head h, positions 0 .. n - 1, in 64 bits."""
    case = s["case"]
    dim = case["dim"]
    d, t = torch.arange(dim, device="cuda")[None, :], torch.arange(BLOCK, device="cuda")[:, None]
    c = 16 if case["type"] == "fp8" else 8
    at_k = (d // c) * 16 * c + t * c + d % c
    at_v = ((((d // (2 * c) * 16 + d % 16) * 2 + t // 4 % 2) * (c // 8) + d // 16 % (c // 8)) * 2 + t // 8) * 4 + t % 4

    def of(r, h, n):
        i = s["ids"][r, :-(-n // BLOCK)].long() + (0 if s["inst"] is None else int(s["inst"][r]) * s["per_inst"])
        out = []
        for x, scale, at in ((s["k"], s["k_scale"], at_k), (s["v"], s["v_scale"], at_v)):
            page = x[i, h].reshape(len(i), -1)[:, at.reshape(-1)].reshape(len(i), BLOCK, dim)
            if scale is not None:
                page = page.view(torch.float8_e4m3fn).double() * torch.exp2(scale[i, h].double() - 127)[..., None]
            out.append(page.double().reshape(-1, dim)[:n])
        return out
    return of


def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    if kind == "write":
        if case["type"] != "fp8":
            return None  # a copy
        r = {}
        for name in ("k", "v"):
            x = s[name + "_new"].double()
            big = x.abs().amax(-1, keepdim=True)
            e = torch.ceil(torch.log2(big / 448))
            e = torch.where(448 * torch.exp2(e - 1) >= big, e - 1, e)  # log2 rounded up past a whole number
            r[name] = _e4m3(x * torch.exp2(-e)) * torch.exp2(e)
        return dict(r, k_scale=None, v_scale=None)
    if case["type"] != "fp8" and kind == "read":
        return None  # a copy
    of = _exact_cache(s)
    lens = s["kv_len"].tolist()
    starts = list(range(case["seqs"] + 1)) if s["q_start"] is None else s["q_start"].tolist()
    kvh, dim = case["kv_heads"], case["dim"]
    n = starts[-1]
    if kind == "read":
        k, v = (torch.zeros((n, kvh, dim), dtype=torch.float64, device="cuda") for _ in range(2))
        for r, total in enumerate(lens):
            a, b = starts[r], starts[r + 1]
            for h in range(kvh):
                kk, vv = of(r, h, total)
                k[a:b, h], v[a:b, h] = kk[total - (b - a):], vv[total - (b - a):]
        return dict(k=k, v=v)
    heads = case["heads"]
    G = heads // kvh
    out = torch.zeros((n, heads, dim), dtype=torch.float64, device="cuda")
    lse = torch.full((n, heads), -math.inf, dtype=torch.float64, device="cuda")
    for r, total in enumerate(lens):
        a, b = starts[r], starts[r + 1]
        if total == 0 or a == b:
            continue
        at = total - (b - a) + torch.arange(b - a, device="cuda")
        pos = torch.arange(total, device="cuda")[None, :]
        hidden = pos > at[:, None]
        if case["window"]:
            hidden |= pos <= at[:, None] - case["window"]
        for h in range(kvh):
            k, v = of(r, h, total)
            kt = k.t().contiguous()
            for u in range(h * G, h * G + G):
                x = (s["q"][a:b, u].double() @ kt * s["scale"]).masked_fill_(hidden, -math.inf)
                top = x.amax(1, keepdim=True)
                w = torch.exp(x - top)
                z = w.sum(1, keepdim=True)
                out[a:b, u] = (w @ v) / z
                lse[a:b, u] = (top + torch.log(z))[:, 0]
    return dict(out=out, lse=lse) if case["lse"] else dict(out=out)
