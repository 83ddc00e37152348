"""Refusals of sae_kv_append, sae_attn_tree and sae_sample (checked on the host, before any launch: no GPU needed), their
binding, and the oracle's parts against independent statements."""
import ctypes

import numpy as np
import pytest
import torch

from oracle import kvcache as O
from oracle import sampling as S
from paper_2605_18825_amd import _lib, api
from test_kv_args_cpu import BAD_KV, BAD_SQ, FP8, P, kv, lib, sq  # noqa: F401
from test_kv_binding_cpu import On, Stream, cache, calls, rows, seqs  # noqa: F401


def rope(**over):
    r = _lib.SaeRope()
    for name, v in dict(dict(inv_freq=P, factor=1.0, turned=128, interleaved=0), **over).items():
        setattr(r, name, v)
    return r


def append(lib, k=None, s=None, n=5, heads=4, dtype=api.KV_BF16, r=None, pos=None, q=P, qs=512, qo=P, qos=512, a=P, sa=512, b=P,
           sb=512):
    return lib.sae_kv_append(k or kv(), s or sq(), n, heads, dtype, r or rope(), pos, q, qs, qo, qos, a, sa, b, sb, None)


def tree(lib, k=None, s=None, n=5, parent=P, nodes=8, heads=4, dtype=api.KV_BF16, q=P, qs=512, o=P, os_=512, lse=None, scale=0.1,
         window=0, work=P, work_bytes=1 << 40):
    return lib.sae_attn_tree(k or kv(), s or sq(), n, parent, nodes, heads, dtype, q, qs, o, os_, lse, scale, window, work,
                             work_bytes, None)


def sample(lib, n=4, vocab=100, dtype=3, logits=P, stride=100, s=None, u=P, token=P, prob=None, kept=None, work=P, work_bytes=1 << 40):
    return lib.sae_sample(n, vocab, dtype, logits, stride, s, u, token, prob, kept, work, work_bytes, None)


@pytest.mark.parametrize("over,msg", BAD_KV)
def test_bad_cache(lib, over, msg):
    for f in (append, tree):
        assert f(lib, k=kv(**over)) == -1 and msg in lib.sae_last_error(None), f


@pytest.mark.parametrize("over,msg", BAD_SQ)
def test_bad_sequences(lib, over, msg):
    for f in (append, tree):
        assert f(lib, s=sq(**over)) == -1 and msg in lib.sae_last_error(None), f


@pytest.mark.parametrize("over,msg", [
    (dict(n=-1), b"n_tokens"), (dict(n=(1 << 24) + 1), b"n_tokens"), (dict(a=None), b"row arrays"), (dict(b=P + 8), b"row arrays"),
    (dict(sa=248), b"strides"), (dict(sb=516), b"strides"), (dict(dtype=api.KV_F16), b"dtype"), (dict(dtype=api.ROWS_F32), b"dtype"),
    (dict(q=None), b"row arrays"), (dict(qo=None), b"row arrays"), (dict(heads=0), b"n_heads"), (dict(heads=-1), b"n_heads"),
    (dict(heads=1025), b"n_heads"), (dict(heads=5), b"strides"), (dict(qos=520), b"row arrays or strides"), (dict(q=P + 8), b"row arrays"),
    (dict(pos=P + 2), b"pos"), (dict(r=rope(inv_freq=None)), b"inv_freq"), (dict(r=rope(inv_freq=P + 1)), b"inv_freq"),
    (dict(r=rope(turned=0)), b"turned"), (dict(r=rope(turned=24)), b"turned"), (dict(r=rope(turned=144)), b"turned"),
    (dict(r=rope(turned=-16)), b"turned"), (dict(r=rope(interleaved=2)), b"interleaved"),
    (dict(r=rope(factor=float("inf"))), b"factor"), (dict(r=rope(factor=float("nan"))), b"factor")])
def test_bad_append(lib, over, msg):
    if msg == b"row arrays or strides":  # a multiple of 8 that holds a row
        over, msg = dict(qos=516), b"strides"
    assert append(lib, **over) == -1 and msg in lib.sae_last_error(None), lib.sae_last_error(None)


@pytest.mark.parametrize("over,msg", [
    (dict(parent=None), b"parent"), (dict(parent=P + 2), b"parent"), (dict(nodes=0), b"max_nodes"), (dict(nodes=257), b"max_nodes"),
    (dict(heads=3), b"n_heads"), (dict(heads=0), b"n_heads"), (dict(heads=1026), b"n_heads"), (dict(scale=float("inf")), b"scale"),
    (dict(window=-1), b"window"), (dict(work=None), b"work"), (dict(work=P + 8), b"work"), (dict(work_bytes=0), b"work"),
    (dict(lse=P + 2), b"lse"), (dict(heads=8), b"strides"), (dict(o=None), b"row arrays"), (dict(dtype=api.KV_F16), b"dtype")])
def test_bad_tree(lib, over, msg):
    assert tree(lib, **over) == -1 and msg in lib.sae_last_error(None), lib.sae_last_error(None)
    assert tree(lib, k=kv(**FP8), dtype=api.KV_F16) == -1 and b"dtype" in lib.sae_last_error(None)


@pytest.mark.parametrize("over,msg", [
    (dict(n=-1), b"n_rows"), (dict(n=(1 << 20) + 1), b"n_rows"), (dict(vocab=0), b"vocab"), (dict(vocab=(1 << 20) + 1), b"vocab"),
    (dict(dtype=2), b"dtype"), (dict(dtype=4), b"dtype"), (dict(stride=99), b"stride"), (dict(logits=None), b"logits"),
    (dict(logits=P + 2), b"logits"), (dict(dtype=0, logits=P + 1), b"logits"), (dict(u=None), b"u and token"),
    (dict(token=None), b"u and token"), (dict(u=P + 2), b"aligned"), (dict(prob=P + 1), b"aligned"), (dict(kept=P + 1), b"aligned"),
    (dict(s=_lib.SaeSampling(P + 1, None, None, None)), b"aligned"), (dict(s=_lib.SaeSampling(None, P + 2, None, None)), b"aligned"),
    (dict(work=None), b"work"), (dict(work=P + 4), b"work"), (dict(work_bytes=0), b"work")])
def test_bad_sample(lib, over, msg):
    assert sample(lib, **over) == -1 and msg in lib.sae_last_error(None), lib.sae_last_error(None)


def test_nothing_to_do(lib):
    assert append(lib, n=0, q=None, qo=None, heads=0, a=None, b=None) == 0
    assert append(lib, s=sq(n_seq=0, block_ids=None, kv_len=None, q_start=None), n=0, a=None, b=None) == 0
    assert tree(lib, n=0, parent=None, q=None, o=None, work=None) == 0
    assert sample(lib, n=0, logits=None, u=None, token=None, work=None) == 0
    assert append(lib, r=rope(turned=144), n=0) == -1  # arguments are checked all the same
    n = ctypes.c_size_t()
    assert lib.sae_sample_work_size(5, 1000, ctypes.byref(n)) == 0 and n.value >= 0
    assert lib.sae_sample_work_size(5, 1000, None) == -1 and lib.sae_sample_work_size(5, 0, ctypes.byref(n)) == -1
    assert lib.sae_kv_append(kv(), sq(), 5, 4, 0, None, None, P, 512, P, 512, P, 512, P, 512, None) == -1


# ------------------------------------------------------------- the binding
def on(shape, dtype=torch.float32, dev=0):
    return On(torch.zeros(shape, dtype=dtype), dev)


def run(dev, stream=None):
    """Every call once, its tensors on the devices dev[name] (0 where missing)."""
    d = lambda name: dev.get(name, 0)  # noqa: E731
    r = api.make_rope(on(32, dev=d("freq")))
    yield "append", lambda: api.sae_kv_append(cache(), seqs(), r, rows(4, d("q")), rows(4, d("out")), rows(2, d("k")),
                                              rows(2, d("v")), pos=on(3, torch.int32, d("pos")), stream=stream)
    yield "tree", lambda: api.sae_attn_tree(cache(), seqs(), on(3, torch.int32, d("parent")), 4, rows(4, d("q")), rows(4, d("out")),
                                            0.1, on(64, torch.uint8, d("work")), lse=on((3, 4), dev=d("lse")), stream=stream)
    yield "sample", lambda: api.sae_sample(on((3, 50), dev=d("logits")), on(3, dev=d("u")), on(3, torch.int32, d("token")),
                                           on(64, torch.uint8, d("work")), temperature=on(3, dev=d("t")),
                                           kept=on(3, torch.int32, d("kept")), stream=stream)


USES = dict(append=["freq", "q", "out", "k", "v", "pos"], tree=["parent", "q", "out", "work", "lse"],
            sample=["logits", "u", "token", "work", "t", "kept"])


def test_the_current_devices_stream(calls):  # noqa: F811
    for _, f in run({}):
        f()
    assert [c[0] for c in calls] == ["sae_kv_append", "sae_attn_tree", "sae_sample"] and all(c[1][-1] == 0x100 for c in calls)
    del calls[:]
    for _, f in run({}, Stream(0)):
        f()
    assert all(c[1][-1] == 0x5000 for c in calls) and len(calls) == 3


@pytest.mark.parametrize("name", sorted({x for v in USES.values() for x in v}))
def test_one_tensor_elsewhere_is_refused(calls, name):  # noqa: F811
    for call, f in run({name: 1}):
        if name in USES[call]:
            with pytest.raises(api.SaeError, match="current device"):
                f()
    for _, f in run({}, Stream(1)):
        with pytest.raises(api.SaeError, match="stream"):
            f()
    assert all(c[0][4:] not in (k for k in USES if name in USES[k]) for c in calls)


def test_shapes_and_types_are_refused(calls):  # noqa: F811
    c, s = cache(), seqs()
    r = api.make_rope(on(32))
    k, v, q = rows(2), rows(2), rows(4)
    bad = [
        (lambda: api.make_rope(on(32, torch.float64)), "float32"),
        (lambda: api.sae_kv_append(c, s, r, q, None, k, v), "together"),
        (lambda: api.sae_kv_append(c, s, r, q, rows(3), k, v), "expected"),
        (lambda: api.sae_kv_append(c, s, r, rows(4, n=2), rows(4, n=2), k, v), "length"),
        (lambda: api.sae_kv_append(c, s, r, q, q, k, rows(2, n=2)), "length"),
        (lambda: api.sae_kv_append(c, s, r, q, q, k, v, pos=on(3, torch.int64)), "pos"),
        (lambda: api.sae_kv_append(c, s, r, q, q, k, v, pos=on(2, torch.int32)), "pos"),
        (lambda: api.sae_attn_tree(c, s, on(2, torch.int32), 4, q, q, 0.1, on(64, torch.uint8)), "parent"),
        (lambda: api.sae_attn_tree(c, s, on(3, torch.int64), 4, q, q, 0.1, on(64, torch.uint8)), "parent"),
        (lambda: api.sae_sample(on((3, 5), torch.float64), on(3), on(3, torch.int32), on(64)), "logits"),
        (lambda: api.sae_sample(on(3), on(3), on(3, torch.int32), on(64)), "logits"),
        (lambda: api.sae_sample(On(torch.zeros((5, 3)).t()), on(3), on(3, torch.int32), on(64)), "contiguous"),
        (lambda: api.sae_sample(on((3, 5)), on(2), on(3, torch.int32), on(64)), "u must"),
        (lambda: api.sae_sample(on((3, 5)), on(3), on(3), on(64)), "token must"),
        (lambda: api.sae_sample(on((3, 5)), on(3), on(3, torch.int32), on(64), top_k=on(3)), "top_k must"),
        (lambda: api.sae_sample(on((3, 5)), on(3), on(3, torch.int32), on(64), prob=on(4)), "prob must"),
    ]
    for f, msg in bad:
        with pytest.raises(api.SaeError, match=msg):
            f()
    assert not calls
    with pytest.raises(api.SaeError, match="device tensor"):
        api.sae_sample(torch.zeros((3, 5)), on(3), on(3, torch.int32), on(64))
    assert api.status_names(256) == ["BAD_TREE"]


# ------------------------------------------------------------- the oracle
def test_a_chain_sees_what_a_prompt_sees():
    rng = np.random.default_rng(1)
    k, v, q = rng.standard_normal((30, 2, 16)), rng.standard_normal((30, 2, 16)), rng.standard_normal((9, 4, 16))
    there = np.ones(30, bool)
    there[[3, 25]] = False
    for window in (0, 1, 5, 40):
        a = O.attention(q, np.arange(21, 30), k, v, there, 0.3, window)
        b = O.tree_attention(q, np.arange(9) - 1, k, v, there, 0.3, window)
        assert all(np.allclose(x, y, rtol=1e-12, atol=1e-13) for x, y in zip(a, b))


def test_a_tree_by_hand():
    #      0      a second root 4
    #     / \
    #    1   2
    #    |
    #    3
    parent, there = [-1, 0, 0, 1, -1], np.ones(8, bool)
    seen = O.tree_seen(parent, 8, there, 0)
    want = ["11110000"[:3] + "10000", "111" + "11000", "111" + "10100", "111" + "11010", "111" + "00001"]
    assert ["".join("01"[int(x)] for x in row) for row in seen] == want
    # a window of 2: itself and one above; a root sees the prefix's last
    seen = O.tree_seen(parent, 8, there, 2)
    assert ["".join("01"[int(x)] for x in row) for row in seen] == ["001" + "10000", "000" + "11000", "000" + "10100", "000" + "01010", "001" + "00001"]
    assert not O.tree_seen(parent, 3, np.ones(3, bool), 0)[:2].any()  # nodes 0 and 1 have no place


def test_turning_is_a_complex_product():
    rng = np.random.default_rng(2)
    x, pos, f = rng.standard_normal((5, 2, 32)), np.array([0, 1, 7, 100000, 3]), rng.random(8)
    for inter in (False, True):
        y = O.turn(x, pos, f, inter, 1.5)
        i, j = (np.arange(0, 16, 2), np.arange(1, 16, 2)) if inter else (np.arange(8), np.arange(8, 16))
        z = (x[..., i] + 1j * x[..., j]) * 1.5 * np.exp(1j * pos[:, None] * f)[:, None]
        assert np.allclose(y[..., i], z.real) and np.allclose(y[..., j], z.imag) and np.array_equal(y[..., 16:], x[..., 16:])
        assert np.allclose(y[0, :, :16], 1.5 * x[0, :, :16])


def test_sampling_by_hand():
    l = np.log([0.1, 0.4, 0.05, 0.4, 0.05])
    l[3] = l[1]
    assert S.order(l)[:3] == [1, 3, 0]
    assert [S.sample(l, u)[0] for u in (0.0, 0.39, 0.41, 0.79, 0.81, 0.91, 0.96)] == [1, 1, 3, 3, 0, 2, 4]
    assert S.sample(l, 0.6, top_k=2)[0] == 3 and S.sample(l, 0.6, top_k=2)[2] == 2
    assert S.sample(l, 0.9, top_p=0.5)[2] == 2 and S.sample(l, 0.9, top_p=0.39)[2] == 1
    assert S.sample(l, 0.9, min_p=0.2)[2] == 3 and S.sample(l, 0.9, min_p=1.0)[2] == 2 and S.sample(l, 0.9, min_p=2.0)[2] == 1
    assert S.sample(l, 0.9, temperature=0.0) == (1, 1.0, 1)
    assert S.sample([-np.inf, np.nan], 0.5) == (-1, 0.0, 0)
    # top-p is of what top-k leaves: 0.4 of 0.8 reaches 0.5 of it
    assert S.sample(l, 0.9, top_k=2, top_p=0.5)[2] == 1
