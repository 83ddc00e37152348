"""Refusals of the paged cache's calls (checked on the host, before any launch: no GPU needed), and the oracle's own
parts against independent statements."""
import ctypes

import numpy as np
import pytest
import torch

from oracle import kvcache as O
from paper_2605_18825_amd import _lib, api

P = 1 << 20  # a pointer that no refused call reads


def kv(**over):
    k = _lib.SaeKv()
    for name, v in dict(dict(type=api.KV_BF16, n_instances=1, blocks_per_instance=8, n_kv_heads=2, head_dim=128, k=P,
                             v=P), **over).items():
        setattr(k, name, v)
    return k


def sq(**over):
    s = _lib.SaeSeqs()
    for name, v in dict(dict(n_seq=3, max_blocks=4, block_ids=P, kv_len=P, q_start=P), **over).items():
        setattr(s, name, v)
    return s


@pytest.fixture(scope="module")
def lib():
    from paper_2605_18825_amd import build
    import os
    if not os.path.exists(_lib.LIB_PATH):
        build.build()
    return _lib.load()


FP8 = dict(type=api.KV_FP8, k_scale=P, v_scale=P)
BAD_KV = [
    (dict(type=3), b"cache type"), (dict(n_instances=0), b"n_instances"), (dict(n_instances=65536), b"n_instances"),
    (dict(blocks_per_instance=0), b"blocks_per_instance"), (dict(blocks_per_instance=(1 << 24) + 1), b"blocks_per"),
    (dict(n_kv_heads=0), b"n_kv_heads"), (dict(n_kv_heads=257), b"n_kv_heads"), (dict(head_dim=96), b"head_dim"),
    (dict(k=None), b"non-NULL"), (dict(v=None), b"non-NULL"), (dict(k=P + 8), b"aligned"), (dict(v=P + 2), b"aligned"),
    (dict(block_stride=4095), b"block_stride"), (dict(block_stride=4100), b"block_stride"),
    (dict(block_stride=-4096), b"block_stride"), (dict(FP8, k_scale=None), b"k_scale"),
    (dict(FP8, v_scale=P + 4), b"v_scale"), (dict(FP8, scale_stride=16), b"scale_stride"),
    (dict(FP8, scale_stride=40), b"scale_stride"), (dict(status=P + 1), b"status"),
]
BAD_SQ = [
    (dict(n_seq=-1), b"n_seq"), (dict(n_seq=(1 << 20) + 1), b"n_seq"), (dict(max_blocks=0), b"max_blocks"),
    (dict(block_ids=None), b"block_ids"), (dict(kv_len=None), b"kv_len"), (dict(block_ids=P + 2), b"aligned"),
    (dict(q_start=None), b"n_tokens must be n_seq"), (dict(n_seq=0), b"without a sequence"),
    (dict(inst=P + 1), b"aligned"),
]


def calls(lib, k, s, n=5, dtype=api.KV_BF16, heads=4, a=P, a_stride=512, b=P, b_stride=512, scale=0.1, window=0, work=P,
          work_bytes=1 << 40, lse=None):
    yield "write", lib.sae_kv_write(k, s, n, dtype, a, a_stride, b, b_stride, None)
    yield "read", lib.sae_kv_read(k, s, n, dtype, a, a_stride, b, b_stride, None)
    yield "prefill", lib.sae_attn_prefill(k, s, n, heads, dtype, a, a_stride, b, b_stride, lse, scale, window, work,
                                          work_bytes, None)


@pytest.mark.parametrize("over,msg", BAD_KV)
def test_bad_cache(lib, over, msg):
    k, s = kv(**over), sq()
    for name, st in calls(lib, k, s):
        assert st == -1 and msg in lib.sae_last_error(None), (name, lib.sae_last_error(None))
    n = ctypes.c_size_t()
    assert lib.sae_attn_work_size(k, s, 5, 4, ctypes.byref(n)) == -1
    assert lib.sae_attn_decode(k, sq(q_start=None), 4, 0, P, 512, P, 512, None, 0.1, 0, P, 1 << 40, None) == -1


@pytest.mark.parametrize("over,msg", BAD_SQ)
def test_bad_sequences(lib, over, msg):
    for name, st in calls(lib, kv(), sq(**over)):
        assert st == -1 and msg in lib.sae_last_error(None), (name, lib.sae_last_error(None))


@pytest.mark.parametrize("over,msg", [
    (dict(n=-1), b"n_tokens"), (dict(n=(1 << 24) + 1), b"n_tokens"), (dict(a=None), b"row arrays"),
    (dict(b=P + 8), b"row arrays"), (dict(a_stride=248), b"strides"), (dict(b_stride=516), b"strides"),
    (dict(dtype=api.KV_F16), b"dtype"), (dict(dtype=api.KV_FP8), b"dtype")])
def test_bad_rows(lib, over, msg):
    for name, st in calls(lib, kv(), sq(), **over):
        assert st == -1 and msg in lib.sae_last_error(None), (name, lib.sae_last_error(None))


@pytest.mark.parametrize("over,msg", [
    (dict(heads=3), b"n_heads"), (dict(heads=0), b"n_heads"), (dict(heads=1026), b"n_heads"),
    (dict(scale=float("inf")), b"scale"), (dict(scale=float("nan")), b"scale"), (dict(window=-1), b"window"),
    (dict(work=None), b"work"), (dict(work=P + 8), b"work"), (dict(work_bytes=0), b"work"), (dict(lse=P + 2), b"lse"),
    (dict(heads=8), b"strides")])
def test_bad_attention(lib, over, msg):
    st = dict(calls(lib, kv(), sq(), **over))["prefill"]
    assert st == -1 and msg in lib.sae_last_error(None), lib.sae_last_error(None)


def test_other_refusals(lib):
    assert lib.sae_kv_write(None, sq(), 5, 0, P, 512, P, 512, None) == -1
    assert lib.sae_kv_read(kv(), None, 5, 0, P, 512, P, 512, None) == -1
    assert lib.sae_attn_decode(kv(), None, 4, 0, P, 512, P, 512, None, 0.1, 0, P, 1 << 40, None) == -1
    assert lib.sae_attn_decode(kv(), sq(), 4, 0, P, 512, P, 512, None, 0.1, 0, P, 1 << 40, None) == -1
    assert b"q_start" in lib.sae_last_error(None)
    assert lib.sae_attn_work_size(kv(), sq(), 5, 4, None) == -1
    k = kv(**FP8)
    assert dict(calls(lib, k, sq(), dtype=api.KV_F16))["prefill"] == -1 and b"dtype" in lib.sae_last_error(None)


def test_nothing_to_do(lib):
    """No tokens: accepted without arrays, nothing is launched."""
    for name, st in calls(lib, kv(), sq(), n=0, a=None, b=None, work=None):
        assert st == 0, name
    s = sq(n_seq=0, block_ids=None, kv_len=None, q_start=None)
    for name, st in calls(lib, kv(), s, n=0, a=None, b=None, work=None):
        assert st == 0, name
    assert lib.sae_attn_decode(kv(), s, 4, 0, None, 0, None, 0, None, 0.1, 0, None, 0, None) == 0


def test_python_binding_refuses():
    with pytest.raises(api.SaeError, match="device tensor"):
        api.make_kv(api.KV_BF16, 1, 2, 1, 64, torch.zeros(2048, dtype=torch.bfloat16), None)
    with pytest.raises(api.SaeError, match="int32"):
        api.make_seqs(torch.zeros((2, 3), dtype=torch.int64), torch.zeros(2, dtype=torch.int32))
    with pytest.raises(api.SaeError, match="kv_len"):
        api.make_seqs(torch.zeros((2, 3), dtype=torch.int32), torch.zeros(3, dtype=torch.int32))


# ------------------------------------------------------------- the oracle
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("size", [1, 2])
def test_places_are_a_permutation(dim, size):
    for p in O.places(dim, size):
        assert sorted(p.reshape(-1).tolist()) == list(range(16 * dim))
    k, v = O.places(dim, size)
    c = 16 // size
    # 16 bytes hold c consecutive dimensions of a key; 16 bytes of values hold token groups h and h + 2
    assert np.array_equal(k[5, :c], k[5, 0] + np.arange(c))
    assert v[1, 0] == v[0, 0] + 1 and v[8, 0] == v[0, 0] + 4 and v[4, 0] == v[0, 0] + c
    x = np.arange(3 * 16 * dim).reshape(3, 16, dim)
    for which in range(2):
        assert np.array_equal(O.unpack(O.pack(x, size, which), dim, size, which), x)


def test_e4m3_against_torch():
    t = O.e4m3_table()
    assert np.array_equal(t, torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy(),
                          equal_nan=True)
    x = np.random.default_rng(0).uniform(-448, 448, 20000) * np.exp2(-np.random.default_rng(1).integers(0, 20, 20000))
    x = x.astype(np.float32)
    want = torch.as_tensor(x).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    assert np.array_equal(O.to_e4m3(x.astype(np.float64)), want)


def test_quantise_scale_is_the_smallest():
    x = np.random.default_rng(2).standard_normal((200, 64)) * np.exp2(np.random.default_rng(3).integers(-40, 40, (200, 1)))
    b, s = O.quantise(x)
    e = s.astype(int) - 127
    top = np.abs(x).max(1)
    assert np.all(top <= 448 * 2.0 ** e) and np.all(top > 448 * 2.0 ** (e - 1.0))
    # relative error of a value that is not among e4m3's subnormals: at most 2^-4
    y = O.dequantise(b, s)
    big = np.abs(x) >= 2.0 ** (e[:, None] - 6.0)
    assert np.all(np.abs(y - x)[big] <= 2.0 ** -4 * np.abs(x)[big])
    assert np.all(np.abs(y - x)[~big] <= 2.0 ** (np.broadcast_to(e[:, None], x.shape)[~big] - 10.0))


def test_attention_against_a_direct_sum():
    rng = np.random.default_rng(4)
    k, v, q = rng.standard_normal((9, 2, 64)), rng.standard_normal((9, 2, 64)), rng.standard_normal((2, 4, 64))
    there = np.ones(9, bool)
    there[3] = False
    out, lse, _, _ = O.attention(q, np.array([6, 8]), k, v, there, 0.2, 4)
    for i, seen in ((0, [4, 5, 6]), (1, [5, 6, 7, 8])):
        for h in range(4):
            w = np.array([np.exp(0.2 * float(q[i, h] @ k[t, h // 2])) for t in seen])
            o = sum(wt * v[t, h // 2] for wt, t in zip(w, seen)) / w.sum()
            assert np.allclose(out[i, h], o, rtol=1e-12, atol=1e-14) and abs(lse[i, h] - np.log(w.sum())) < 1e-12
    out, lse, _, _ = O.attention(q, np.array([-1, 3]), k, v, there & False, 0.2, 0)
    assert np.all(out == 0) and np.all(np.isneginf(lse))
