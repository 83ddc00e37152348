"""sae_sample against the 64-bit oracle on either side of every border by which rows are given to kernels: 256, 512 or 1,024
threads a row (vocabularies of 8,192, 16,384 and 65,535, 16 and 511 rows), a k that the threads' maxima bound (up to half of
them) and one that they do not, lists that overflow."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

from oracle import sampling as S  # noqa: E402
from paper_2605_18825_amd import api  # noqa: E402
from test_gpu_sample import DT, MIXES, TYPES, check, logits, spread_over  # noqa: E402

MANY = dict(MIXES, bound_k=dict(top_k=[127, 128, 129, 255]), bound_k2=dict(top_k=[256, 257, 511, 512], top_p=[0.99, 1.0, 0.9, 1.0]),
            bound_k3=dict(top_k=[513, 1024, 1500, 600], min_p=[0.0, 0.001, 0.0, 0.01]))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("mix", sorted(MANY))
@pytest.mark.parametrize("vocab", [8192, 8193, 12000, 16384, 16385])
def test_few_rows(dtype, mix, vocab):
    x, u = logits(4, vocab, dtype, seed=vocab + 1)
    check(x, u, **spread_over(4, MANY[mix]))


def copies(x, u, times, **settings):
    """A call of `times` copies of each row: the oracle's answers for the rows, and every copy the same."""
    n = len(u)
    want = check(x, u, **settings)
    xd = x.cuda().repeat(times, 1)
    dev = {k: torch.as_tensor(np.tile(np.asarray(a, np.int32 if k == "top_k" else np.float32), times)).cuda()
           for k, a in settings.items()}
    token, kept = (torch.full((n * times,), -7, dtype=torch.int32, device="cuda") for _ in range(2))
    prob = torch.full((n * times,), -7.0, device="cuda")
    work = torch.full((api.sae_sample_work_size(n * times, x.shape[1]),), 0xFF, dtype=torch.uint8, device="cuda")
    ud = torch.as_tensor(np.tile(np.asarray(u, np.float32), times)).cuda()
    api.sae_sample(xd, ud, token, work, prob=prob, kept=kept, **dev)
    torch.cuda.synchronize()
    for got, one in zip((token, prob, kept), want):
        assert np.array_equal(got.double().cpu().numpy().reshape(times, n), np.tile(np.asarray(one, np.float64), (times, 1)))


# rows: 4 times the second number; the vocabularies are odd ones where a row's alignment is to differ
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("mix", ["whole", "bound_k2", "more_k", "top_p", "min_p", "all"])
@pytest.mark.parametrize("vocab,times", [(20011, 4), (20011, 5), (65535, 4), (65535, 5), (65537, 17), (12001, 128), (4099, 130)])
def test_many_rows(dtype, mix, vocab, times):
    x, u = logits(4, vocab, dtype, seed=vocab + times)
    copies(x, u, times, **spread_over(4, MANY[mix]))


@pytest.mark.parametrize("times", [127, 128])
@pytest.mark.parametrize("mix", ["whole", "bound_k2", "top_p", "all"])
def test_many_rows_of_a_large_vocabulary(mix, times):
    x, u = logits(4, 65536, "bf16", seed=times)
    copies(x, u, times, **spread_over(4, MANY[mix]))


FLAT = [{}, dict(top_k=[5000, 300, 256, 2100]), dict(top_p=[0.9, 0.3, 0.999, 0.5]), dict(min_p=[0.9, 0.5, 0.999, 1.0]),
        dict(top_k=[6000, 0, 0, 2500], top_p=[0.5, 0.9, 0.95, 0.99], min_p=[0.0, 0.7, 0.9, 0.6])]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("vocab,times", [(9001, 1), (16384, 1), (30001, 5)])
def test_flat_and_equal_rows(dtype, vocab, times):
    """More tokens than are sorted together: near ones, equal ones, two groups of equal ones."""
    x, u = logits(4, vocab, dtype, seed=vocab, spread=0.2, peaks=0)
    x[1] = 0.5
    x[2] = 0
    x[2, 1::3] = -0.25
    for settings in FLAT:
        copies(x, u, times, **settings)


@pytest.mark.parametrize("dtype", TYPES)
def test_rows_out_of_line(dtype):
    """512 threads: rows that begin at every alignment; what lies beside them is not read."""
    n, vocab = 6, 12001
    x, u = logits(n, vocab, dtype, seed=31)
    for lead, width in ((0, vocab), (1, vocab + 3), (3, vocab + 8), (5, vocab + 6), (7, vocab + 13)):
        wide = torch.full((n * width + 16,), float("inf"), dtype=DT[dtype], device="cuda")
        view = wide[lead:lead + n * width].view(n, width)[:, :vocab]
        view.copy_(x)
        check(view, u, top_p=[0.9] * n)
        check(view, u, top_k=[256] * n)
        check(view, u, top_k=[257] * n)


def test_rows_that_nothing_is_left_of():
    """512 threads: -inf and NaN."""
    x, u = logits(6, 12001, "f32", seed=32)
    x[0] = -np.inf
    x[1] = np.nan
    x[2, 1:] = -np.inf
    x[3, ::2] = np.nan
    x[4, :-1] = -np.inf
    for settings in ({}, dict(top_k=[5] * 6), dict(top_p=[0.9] * 6), dict(temperature=[0.0] * 6), dict(top_k=[300] * 6, min_p=[0.1] * 6)):
        token, prob, kept = check(x, u, **settings)
        assert np.all(token[:2] == -1) and np.all(kept[:2] == 0) and np.all(prob[:2] == 0)
        assert token[2] == 0 and token[4] == 12000 and prob[4] == 1 and kept[4] == 1


def test_a_graph_and_the_oracle():
    """Replays of a call with 512 threads a row against the definition."""
    n, vocab = 5, 9003
    x, u = torch.empty((n, vocab), device="cuda"), torch.empty(n, device="cuda")
    g = torch.Generator(device="cuda")
    g.manual_seed(3)
    token = torch.empty(n, dtype=torch.int32, device="cuda")
    work = torch.empty(api.sae_sample_work_size(n, vocab), dtype=torch.uint8, device="cuda")
    p = torch.tensor([0.9, 1.0, 0.5, 0.9, 0.7], device="cuda")
    k = torch.tensor([50, 0, 257, 600, 1], dtype=torch.int32, device="cuda")
    x.normal_(generator=g)
    u.uniform_(generator=g)
    api.sae_sample(x, u, token, work, top_p=p, top_k=k)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        api.sae_sample(x, u, token, work, top_p=p, top_k=k)
    for i in range(4):
        x.normal_(generator=g).mul_(1 + 2 * i)
        u.uniform_(generator=g)
        graph.replay()
        torch.cuda.synchronize()
        for r in range(n):
            one = dict(top_p=float(p[r]), top_k=int(k[r]))
            l = x[r].double().cpu().numpy()
            want = S.sample(l, float(u[r]), **one)[0]
            assert int(token[r]) == want or S.margin(l, float(u[r]), **one) <= vocab * 2.0 ** -43
