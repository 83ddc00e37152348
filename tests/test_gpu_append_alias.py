"""sae_kv_append with queries, turned queries, keys and values side by side in one array: the bits that arrays of their own
give, and nothing else changed."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

from harness import say  # noqa: E402
from kv_cases import Cache, dev32, tables  # noqa: E402
from oracle import kvcache as O  # noqa: E402
from paper_2605_18825_amd import api  # noqa: E402

HEADS, KVH, DIM = 4, 2, 64


# what lies in a row, by heads; "q" alone is turned in place
@pytest.mark.parametrize("layout", ["qkv", "kvq", "qokv", "kovq", "okvq"])
@pytest.mark.parametrize("lens,new", [([40, 70, 5], [40, 3, 2]), ([17], [1])])
def test_side_by_side(layout, lens, new):
    ids, _, bpi, _ = tables(lens, 1, np.random.default_rng(1))
    n = sum(new)
    size = dict(q=HEADS, o=HEADS, k=KVH, v=KVH)
    g = torch.Generator(device="cuda")
    g.manual_seed(2)
    apart = {c: torch.randn((n, size[c], DIM), generator=g, device="cuda").bfloat16() for c in "qkv"}
    fused = torch.full((n, sum(size[c] for c in layout) + 1, DIM), 7.0, dtype=torch.bfloat16, device="cuda")
    view, at = {}, 0
    for c in layout:
        view[c] = fused[:, at:at + size[c]]
        at += size[c]
        if c in apart:
            view[c].copy_(apart[c])
    rope = api.make_rope(torch.logspace(0, -4, DIM // 2, device="cuda"))
    seqs = api.make_seqs(dev32(ids), dev32(lens), q_start=dev32(np.concatenate([[0], np.cumsum(new)])))
    held = []
    for arrays, out in ((apart, torch.empty_like(apart["q"])), (view, view.get("o", view["q"]))):
        c = Cache(O.BF16, 1, bpi, KVH, DIM, np.random.default_rng(3))
        kv = c.device()
        say("append: %s, %d rows, %s" % (layout, n, "apart" if arrays is apart else "fused"))
        api.sae_kv_append(kv, seqs, rope, arrays["q"], out, arrays["k"], arrays["v"])
        torch.cuda.synchronize()
        held.append([out.clone(), *(t.view(torch.int16).clone() for t in kv.tensors[:2])])
    assert all(torch.equal(a, b) for a, b in zip(*held))
    assert torch.equal(view["k"], apart["k"]) and torch.equal(view["v"], apart["v"]) and torch.all(fused[:, -1] == 7.0)
    assert "o" not in layout or torch.equal(view["q"], apart["q"])
    if n > 1:
        with pytest.raises(api.SaeError, match="apart"):
            api.sae_kv_append(kv, seqs, rope, view["q"], fused[:, 1:1 + HEADS], view["k"], view["v"])
