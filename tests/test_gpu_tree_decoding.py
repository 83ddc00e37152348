"""The calls of a decoding step together: append, tree attention, sampling, and the move of what is accepted."""
import os
import sys

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))

from harness import say  # noqa: E402
from oracle import kvcache as K  # noqa: E402
from oracle import sampling as S  # noqa: E402
from paper_2605_18825_amd import api  # noqa: E402


@pytest.mark.parametrize("kv_type", [0, 2])
@pytest.mark.parametrize("settings", [dict(temperature=0.5, top_p=0.9), dict(top_k=20, min_p=0.02), dict(temperature=0.0)])
def test_tree_decoding_example(kv_type, settings):
    """Every drawn token is the oracle's for the logits it was drawn from; the cache holds each request's own keys, turned by
    their places, and its values; and every output is that of causal attention over what the cache holds."""
    import tree_decoding as T
    rows = [0]

    def watch(logits, u, drawn):
        l, got = logits.double().cpu().numpy(), drawn.cpu().numpy()
        for r in range(0, len(l), 7):
            one = {k: v if k == "top_k" else float(np.float32(v)) for k, v in settings.items()}
            assert S.sample(l[r], float(u[r]), **one)[0] == got[r] or S.margin(l[r], float(u[r]), **one) <= l.shape[1] * 2.0 ** -43
            rows[0] += 1
    m, reqs, rate = T.main(kv_type, n_requests=5, n_tokens=24, settings=settings, watch=watch)
    say("%.2f tokens a step, %d rows drawn again" % (rate, rows[0]))
    assert rate > 1  # (a draft is accepted now and then)
    for r in reqs:
        _, k0, v0 = m.qkv(r.tokens[:r.cached])
        k, v = T.held(m, r)
        want = K.turn(k0.double().cpu().numpy(), np.arange(r.cached), m.inv_freq.double().cpu().numpy())
        # one rounding (2^-8 to bf16, 2^-4 to e4m3 of at least the scale's least normal, 2^-14 of the head's largest), and
        # the turn in fp32 before it: two products and their sum, 2^-22 of the pair's size
        big = np.abs(want).max(-1, keepdims=True)
        u = 2.0 ** -8 if kv_type == 0 else 2.0 ** -4
        assert np.all(np.abs(k.double().cpu().numpy() - want) <= u * np.abs(want) + big * (2.0 ** -20 if kv_type == 0 else 2.0 ** -14))
        if kv_type == 0:
            assert torch.equal(v, v0)
        got = torch.stack([x for _, x in r.seen]).float()
        # weights and the output are rounded to bf16, 2^-8 each of values up to the largest; fp32 besides
        most = float(v.float().abs().max())
        assert float((got - T.plain(m, r, k, v)).abs().max()) <= most * (2.0 ** -7 + 2.0 ** -14)


@pytest.mark.parametrize("kv_type", [0, 2])
def test_step_in_a_graph(kv_type):
    """Append, attention and sampling of one tree shape captured once: replays with other tokens, lengths and random numbers give
    what eager calls give, with eager calls over other sequences between them."""
    import tree_decoding as T
    m = T.Model(kv_type, 3 * 24)
    rng = np.random.default_rng(5)
    tables = T.dev32(rng.permutation(72).reshape(3, 24))
    parent = [-1, 0, 0, 1, 2, 2, -1, 0, 1, -1]
    depth = np.array([0, 1, 1, 2, 2, 2, 0, 1, 2, 0])
    start, of = T.dev32([0, 6, 9, 10]), np.array([0] * 6 + [1] * 3 + [2])
    n = 10
    tokens = torch.zeros(n, dtype=torch.int64, device="cuda")
    pos, lens, par = T.dev32(depth), T.dev32([6, 3, 1]), T.dev32(parent)
    u, p = torch.zeros(n, device="cuda"), torch.full((n,), 0.9, device="cuda")
    seqs = api.make_seqs(tables, lens, q_start=start)
    turned, out = (torch.empty((n, T.HEADS, T.DIM), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    drawn = torch.empty(n, dtype=torch.int32, device="cuda")
    size = max(api.sae_attn_work_size(m.kv, seqs, n, T.HEADS), api.sae_sample_work_size(n, T.VOCAB))
    work = torch.full((size,), 0xFF, dtype=torch.uint8, device="cuda")

    def step():
        q, k, v = m.rows[tokens].split([T.HEADS, T.KV_HEADS, T.KV_HEADS], dim=1)
        api.sae_kv_append(m.kv, seqs, m.rope, q, turned, k, v, pos=pos)
        api.sae_attn_tree(m.kv, seqs, par, 6, turned, out, m.scale, work)
        api.sae_sample(out.view(n, -1)[:, :T.VOCAB], u, drawn, work, top_p=p)
    # a cached prefix for every sequence
    prefix = rng.integers(0, T.VOCAB, (3, 300))
    k, v = m.qkv(prefix.reshape(-1))[1:]
    api.sae_kv_append(m.kv, api.make_seqs(tables, T.dev32([300] * 3), q_start=T.dev32([0, 300, 600, 900])), m.rope, None, None, k, v)
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for base in ([290, 100, 1], [0, 16, 299], [257, 255, 256], [15, 0, 300]):
        tokens.copy_(torch.as_tensor(rng.integers(0, T.VOCAB, n)))
        b = np.array(base)
        pos.copy_(torch.as_tensor((b[of] + depth).astype(np.int32)))
        lens.copy_(torch.as_tensor((b + [6, 3, 1]).astype(np.int32)))
        u.copy_(torch.as_tensor(rng.random(n).astype(np.float32)))
        graph.replay()
        torch.cuda.synchronize()
        first = [t.clone() for t in (turned, out, drawn)]
        for t in (turned, out):
            t.fill_(-1)
        drawn.fill_(-1)
        step()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(first, (turned, out, drawn)))
        assert int(drawn.min()) >= 0
    assert int(m.status[0]) == 0


def test_two_streams_with_workspaces_of_their_own():
    """Steps of different sequences of one cache on two streams at once give what they give one after the other."""
    import tree_decoding as T
    m = T.Model(0, 64)
    rng = np.random.default_rng(6)
    tables = rng.permutation(64).reshape(2, 32)
    sides = []
    for i in range(2):
        n = 9 + 8 * i
        table = T.dev32(tables[i:i + 1])
        k, v = m.qkv(rng.integers(0, T.VOCAB, 400))[1:]
        api.sae_kv_append(m.kv, api.make_seqs(table, T.dev32([400]), q_start=T.dev32([0, 400])), m.rope, None, None, k, v)
        seqs = api.make_seqs(table, T.dev32([400 + n]), q_start=T.dev32([0, n]))
        parent = T.dev32([-1] + [int(rng.integers(-1, j)) for j in range(1, n)])
        work = torch.empty(max(api.sae_attn_work_size(m.kv, seqs, n, T.HEADS), api.sae_sample_work_size(n, 70000)),
                           dtype=torch.uint8, device="cuda")
        sides.append(dict(n=n, seqs=seqs, parent=parent, work=work, q=m.qkv(rng.integers(0, T.VOCAB, n)),
                          logits=torch.randn((n, 70000), device="cuda") * 2, u=torch.rand(n, device="cuda"), s=torch.cuda.Stream()))

    def step(x, stream):
        out = torch.empty((x["n"], T.HEADS, T.DIM), dtype=torch.bfloat16, device="cuda")
        turned, drawn = torch.empty_like(out), torch.empty(x["n"], dtype=torch.int32, device="cuda")
        if stream is not None:
            stream.wait_stream(torch.cuda.current_stream())
        q, k, v = x["q"]
        api.sae_kv_append(m.kv, x["seqs"], m.rope, q, turned, k, v, stream=stream)
        api.sae_attn_tree(m.kv, x["seqs"], x["parent"], x["n"], turned, out, m.scale, x["work"], stream=stream)
        api.sae_sample(x["logits"], x["u"], drawn, x["work"], stream=stream)
        return turned, out, drawn
    want = [step(x, None) for x in sides]
    torch.cuda.synchronize()
    for _ in range(5):
        got = [step(x, x["s"]) for x in sides]
        torch.cuda.synchronize()
        for a, b in zip(want, got):
            assert all(torch.equal(x, y) for x, y in zip(a, b))
