"""The binding of the paged cache's calls: which tensors it takes.  No GPU: tensors that say they are on a device, and a
library that only notes what it is called with."""
import pytest
import torch

from paper_2605_18825_amd import _lib, api


class On:
    """A host tensor that passes for one on GPU `device`."""

    def __init__(self, t, device=0):
        self.t, self.device = t, device

    is_cuda = True

    def get_device(self):
        return self.device

    def __getattr__(self, name):
        return getattr(self.t, name)


class Stream:
    def __init__(self, device):
        self.device_index, self.cuda_stream = device, 0x5000 + device


@pytest.fixture
def calls(monkeypatch):
    """The library's calls so far, (name, arguments); the current device is 0."""
    seen = []

    class Lib:
        def __getattr__(self, name):
            return lambda *a: seen.append((name, a)) or 0
    lib = Lib()
    monkeypatch.setattr(_lib, "load", lambda: lib)
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 0, raising=False)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda d: 0x100 + d, raising=False)
    return seen


def cache(dev=(0, 0, 0), ty=api.KV_BF16, dtype=torch.bfloat16, **kw):
    k, v = (On(torch.zeros((4, 2, 16 * 64), dtype=dtype), d) for d in dev[:2])
    if ty == api.KV_FP8:
        kw = dict(dict(k_scale=On(torch.zeros((4, 2, 16), dtype=torch.uint8)),
                       v_scale=On(torch.zeros((4, 2, 16), dtype=torch.uint8))), **kw)
    return api.make_kv(ty, 1, 4, 2, 64, k, v, status=On(torch.zeros(1, dtype=torch.int32), dev[2]), **kw)


def seqs(dev=0, len_dev=None):
    return api.make_seqs(On(torch.zeros((3, 2), dtype=torch.int32), dev),
                         On(torch.zeros(3, dtype=torch.int32), dev if len_dev is None else len_dev))


def rows(heads, dev=0, n=3):
    return On(torch.zeros((n, heads, 64), dtype=torch.bfloat16), dev)


def run(kv, s, dev=(0, 0, 0, 0), stream=None):
    """Every call once; a, b, lse, work on these devices."""
    work, lse = On(torch.zeros(64, dtype=torch.uint8), dev[3]), On(torch.zeros((3, 4)), dev[2])
    yield lambda: api.sae_kv_write(kv, s, rows(2, dev[0]), rows(2, dev[1]), stream=stream)
    yield lambda: api.sae_kv_read(kv, s, rows(2, dev[0]), rows(2, dev[1]), stream=stream)
    yield lambda: api.sae_attn_decode(kv, s, rows(4, dev[0]), rows(4, dev[1]), 0.1, work, lse=lse, stream=stream)
    yield lambda: api.sae_attn_prefill(kv, s, rows(4, dev[0]), rows(4, dev[1]), 0.1, work, lse=lse, stream=stream)


NAMES = ["sae_kv_write", "sae_kv_read", "sae_attn_decode", "sae_attn_prefill"]


def test_the_current_devices_stream(calls):
    for f in run(cache(), seqs()):
        f()
    assert [c[0] for c in calls] == NAMES and all(c[1][-1] == 0x100 for c in calls)
    del calls[:]
    for f in run(cache(), seqs(), stream=Stream(0)):
        f()
    assert [c[0] for c in calls] == NAMES and all(c[1][-1] == 0x5000 for c in calls)


def test_another_device_is_refused(calls):
    """Launches go to the current device: a call whose tensors are elsewhere would run on the wrong one."""
    for f in run(cache((1, 1, 1)), seqs(1), (1, 1, 1, 1)):
        with pytest.raises(api.SaeError, match="current device"):
            f()
    assert not calls


@pytest.mark.parametrize("at", range(4))
def test_one_tensor_elsewhere_is_refused(calls, at):
    dev = [0, 0, 0, 0]
    dev[at] = 1
    for i, f in enumerate(run(cache(), seqs(), dev)):
        if i < 2 and at >= 2:
            continue  # no lse, no work
        with pytest.raises(api.SaeError, match="current device"):
            f()
    assert not calls


def test_cache_or_sequences_elsewhere_are_refused(calls):
    for kv, s in ((cache((1, 1, 1)), seqs()), (cache(), seqs(1))):
        for f in run(kv, s):
            with pytest.raises(api.SaeError, match="current device"):
                f()
    assert not calls
    for dev in ((0, 1, 0), (1, 0, 0), (0, 0, 1)):
        with pytest.raises(api.SaeError, match="different devices"):
            cache(dev)
    with pytest.raises(api.SaeError, match="different devices"):
        seqs(0, 1)


def test_a_stream_elsewhere_is_refused(calls):
    for f in run(cache(), seqs(), stream=Stream(1)):
        with pytest.raises(api.SaeError, match="stream"):
            f()
    assert not calls


def test_descriptions_made_by_hand(calls):
    """A sae_kv and sae_seqs filled without make_kv and make_seqs name no device: the call's own tensors are checked."""
    kv, s = _lib.SaeKv(), _lib.SaeSeqs()
    kv.n_kv_heads, kv.head_dim, s.n_seq = 2, 64, 3
    for f in run(kv, s):
        f()
    assert [c[0] for c in calls] == NAMES


def test_types_of_the_cache(calls):
    """Tensors of another type than the cache's would be read as something else."""
    right = {api.KV_BF16: [torch.bfloat16], api.KV_F16: [torch.float16], api.KV_FP8: [torch.uint8, torch.float8_e4m3fn]}
    every = [torch.bfloat16, torch.float16, torch.int16, torch.uint8, torch.int8, torch.float8_e4m3fn, torch.float8_e5m2,
             torch.float32]
    for ty, fine in right.items():
        for dtype in every:
            if dtype in fine:
                cache(ty=ty, dtype=dtype)
                continue
            with pytest.raises(api.SaeError, match="k must be"):
                cache(ty=ty, dtype=dtype)
    k, v = On(torch.zeros(8192, dtype=torch.bfloat16)), On(torch.zeros(8192, dtype=torch.float16))
    with pytest.raises(api.SaeError, match="v must be"):
        api.make_kv(api.KV_BF16, 1, 4, 2, 64, k, v)
    for dtype, fine in ((torch.uint8, True), (torch.float8_e8m0fnu, True), (torch.float8_e4m3fn, False), (torch.int8, False)):
        sc = On(torch.zeros((4, 2, 16), dtype=torch.uint8).view(dtype))
        if fine:
            cache(ty=api.KV_FP8, dtype=torch.uint8, v_scale=sc)
            continue
        with pytest.raises(api.SaeError, match="v_scale must be"):
            cache(ty=api.KV_FP8, dtype=torch.uint8, v_scale=sc)
    with pytest.raises(api.SaeError, match="unknown cache type"):
        cache(ty=3)


def test_status_holds_a_word(calls):
    """The status is a 32-bit word on the device: less is written past."""
    k, v = (On(torch.zeros(8192, dtype=torch.bfloat16)) for _ in range(2))
    for t in (torch.zeros(1, dtype=torch.uint8), torch.zeros(0, dtype=torch.int32), torch.zeros(1)):
        with pytest.raises(api.SaeError, match="status"):
            api.make_kv(api.KV_BF16, 1, 4, 2, 64, k, v, status=On(t))
    for t in (torch.zeros(1, dtype=torch.int32), torch.zeros(3, dtype=torch.uint32)):
        assert api.make_kv(api.KV_BF16, 1, 4, 2, 64, k, v, status=On(t)).status == t.data_ptr()


def test_strides_of_the_cache(calls):
    """With block_stride a view has to lie as it says."""
    block, nb = 2 * 16 * 64, 4
    whole = torch.zeros((nb, 3, block), dtype=torch.bfloat16)  # three layers of a block together
    layer = [On(whole[:, i]) for i in range(3)]
    kv = api.make_kv(api.KV_BF16, 1, nb, 2, 64, layer[1], layer[2], block_stride=3 * block)
    assert kv.k == whole.data_ptr() + 2 * block and kv.v == whole.data_ptr() + 4 * block
    for stride in (block, 2 * block, 6 * block):
        with pytest.raises(api.SaeError, match="apart"):
            api.make_kv(api.KV_BF16, 1, nb, 2, 64, layer[0], layer[0], block_stride=stride)
    with pytest.raises(api.SaeError, match="contiguous"):
        api.make_kv(api.KV_BF16, 1, nb, 2, 64, layer[0], layer[0])
    # dimensions of a block in another order, or fewer than a block has
    turned = torch.zeros((nb, 2, 64, 16), dtype=torch.bfloat16).transpose(2, 3)
    with pytest.raises(api.SaeError, match="a block of k"):
        api.make_kv(api.KV_BF16, 1, nb, 2, 64, On(turned), On(turned), block_stride=block)
    less = torch.zeros((nb, 2 * block), dtype=torch.bfloat16)[:, :block - 64]
    with pytest.raises(api.SaeError, match="a block of k"):
        api.make_kv(api.KV_BF16, 1, nb, 2, 64, On(less), On(less), block_stride=2 * block)
    # a flat buffer, padded blocks, a single block (whose stride is nothing's)
    flat = On(whole.reshape(-1))
    api.make_kv(api.KV_BF16, 1, nb, 2, 64, flat, flat, block_stride=2 * block)
    padded = On(torch.zeros((nb, block + 64), dtype=torch.bfloat16))
    api.make_kv(api.KV_BF16, 1, nb, 2, 64, padded, padded, block_stride=block + 64)
    one = On(torch.zeros((1, block), dtype=torch.bfloat16))
    api.make_kv(api.KV_BF16, 1, 1, 2, 64, one, one, block_stride=4 * block)
    api.make_kv(api.KV_BF16, 1, 1, 2, 64, flat, flat, block_stride=4 * block)
    # blocks over two dimensions (instance, block), more of them than are used
    api.make_kv(api.KV_BF16, 2, 2, 2, 64, *[On(whole.view(2, 2, 3, block)[:, :, i]) for i in (0, 1)], block_stride=3 * block)
    api.make_kv(api.KV_BF16, 1, 3, 2, 64, layer[0], layer[1], block_stride=3 * block)
    with pytest.raises(api.SaeError, match="apart"):
        every_second = On(torch.zeros((4, 2, 3, block), dtype=torch.bfloat16)[::2, :, 0])
        api.make_kv(api.KV_BF16, 2, 2, 2, 64, every_second, every_second, block_stride=3 * block)
    # scales likewise
    pages = [On(torch.zeros((nb, block), dtype=torch.uint8)) for _ in range(2)]
    sc = torch.zeros((nb, 2, 64), dtype=torch.uint8)
    api.make_kv(api.KV_FP8, 1, nb, 2, 64, *pages, k_scale=On(sc[:, 0, :32]), v_scale=On(sc[:, 1, :32]), scale_stride=128)
    with pytest.raises(api.SaeError, match="apart"):
        api.make_kv(api.KV_FP8, 1, nb, 2, 64, *pages, k_scale=On(sc[:, 0, :32]), v_scale=On(sc[:, 1, :32]), scale_stride=64)
