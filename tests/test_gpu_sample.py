"""GPU parity of sae_sample with the 64-bit oracle: the same token and the same number of kept tokens in every row whose
decisions are not within the sums' resolution (vocab * 2^-43 of the largest weight) of a border."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

from harness import say  # noqa: E402
from oracle import sampling as S  # noqa: E402
from paper_2605_18825_amd import api  # noqa: E402

DT = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}


def call(x, u, **settings):
    """Tokens, shares and kept numbers of logits x (a device tensor)."""
    n, vocab = x.shape
    dev = {k: None if a is None else torch.as_tensor(np.asarray(a, np.int32 if k == "top_k" else np.float32)).cuda()
           for k, a in settings.items()}
    token, kept = (torch.full((n,), -7, dtype=torch.int32, device="cuda") for _ in range(2))
    prob = torch.full((n,), -7.0, device="cuda")
    work = torch.full((api.sae_sample_work_size(n, vocab),), 0xFF, dtype=torch.uint8, device="cuda")
    api.sae_sample(x, torch.as_tensor(np.asarray(u, np.float32)).cuda(), token, work, prob=prob, kept=kept, **dev)
    torch.cuda.synchronize()
    return token.cpu().numpy(), prob.double().cpu().numpy(), kept.cpu().numpy()


def check(x, u, allowed=0, **settings):
    """x: a CPU or device tensor of logits; settings: arrays per row, or missing.  allowed: rows within the resolution."""
    n, vocab = x.shape
    say("sample %s rows %d vocab %d %s" % (str(x.dtype)[6:], n, vocab, sorted(settings)))
    token, prob, kept = call(x.cuda() if not x.is_cuda else x, u, **settings)
    l = x.double().cpu().numpy()
    u = np.asarray(u, np.float32).astype(np.float64)
    near = 0
    for r in range(n):
        one = {k: (int(a[r]) if k == "top_k" else float(np.float32(a[r]))) for k, a in settings.items()}
        want = S.sample(l[r], u[r], **one)
        if (token[r], kept[r]) != (want[0], want[2]):
            m = S.margin(l[r], u[r], **one)
            assert m <= vocab * 2.0 ** -43, (r, one, u[r], want, (token[r], kept[r]), m)
            near += 1
            continue
        # a quotient of sums that are off by vocab 2^-44 at most, rounded to fp32
        assert abs(prob[r] - want[1]) <= 2.0 ** -24 * want[1] + vocab * 2.0 ** -43, (r, one, prob[r], want)
    assert near <= allowed
    return token, prob, kept


def logits(n, vocab, dtype, seed, spread=2.5, peaks=12):
    rng = np.random.default_rng(seed)
    x = rng.standard_normal((n, vocab)) * spread
    for r in range(n):
        at = rng.integers(0, vocab, min(peaks, vocab))
        x[r, at] += rng.random(len(at)) * (2 + 2 * r % 14)
    return torch.as_tensor(x).to(DT[dtype]), rng.random(n)


TYPES = ["bf16", "f16", "f32"]
MIXES = {
    "whole": {}, "temperature": dict(temperature=[0.2, 0.7, 1.0, 3.0]), "greedy": dict(temperature=[0.0, -1.0, np.nan, 0.0]),
    "top_k": dict(top_k=[1, 2, 50, 256]), "more_k": dict(top_k=[257, 1000, 2047, 10 ** 6]), "top_p": dict(top_p=[0.1, 0.5, 0.9, 0.99]),
    "min_p": dict(min_p=[0.001, 0.05, 0.5, 1.0]), "k_p": dict(top_k=[40, 300, 5, 2000], top_p=[0.9, 0.8, 0.5, 0.95]),
    "all": dict(temperature=[0.8, 1.2, 0.5, 2.0], top_k=[100, 0, 500, 3], top_p=[0.95, 0.9, 1.0, 0.7], min_p=[0.01, 0.1, 0.0, 0.2]),
}


def spread_over(n, mix):
    return {k: [v[i % 4] for i in range(n)] for k, v in mix.items()}


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("mix", sorted(MIXES))
@pytest.mark.parametrize("vocab", [1, 2, 7, 100, 1023, 4099, 20000])
def test_settings_and_sizes(dtype, mix, vocab):
    x, u = logits(12, vocab, dtype, seed=vocab)
    check(x, u, **spread_over(12, MIXES[mix]))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("mix", ["whole", "top_p", "more_k", "all"])
def test_flat_rows_of_a_large_vocabulary(dtype, mix):
    """More kept tokens than are sorted together."""
    x, u = logits(4, 70001, dtype, seed=5, spread=0.3, peaks=0)
    check(x, u, **spread_over(4, dict(MIXES[mix], top_k=[30000, 0, 60000, 5000]) if mix == "all" else MIXES[mix]))


@pytest.mark.parametrize("dtype", TYPES)
def test_equal_logits(dtype):
    """Ties go to the lower index: among a few, among all, across a cut."""
    for vocab in (5, 3000, 50000):
        x = torch.zeros((8, vocab))
        x[4:, ::3] = 1.0
        x[6:, 1::2] = -0.0
        u = [0.0, 0.3, 0.77, 0.999999, 0.1, 0.5, 0.25, 0.9]
        check(x.to(DT[dtype]), u)
        check(x.to(DT[dtype]), u, top_k=[3, 100, 1, 2500, 2, 17, 40000, 4])
        check(x.to(DT[dtype]), u, top_p=[0.5, 0.9, 0.1, 1.0, 0.25, 0.75, 0.999, 0.3], min_p=[0, 0.5, 1, 1, 0.3, 0.9, 0, 0])


def test_rows_that_nothing_is_left_of():
    """-inf and NaN are not taken; a row of them gives -1."""
    for vocab in (3, 700, 40001):
        x, u = logits(6, vocab, "f32", seed=vocab)
        x[0] = -np.inf
        x[1] = np.nan
        x[2, 1:] = -np.inf
        x[3, ::2] = np.nan
        x[4, :-1] = -np.inf
        for settings in ({}, dict(top_k=[5] * 6), dict(top_p=[0.9] * 6), dict(temperature=[0.0] * 6), dict(top_k=[300] * 6, min_p=[0.1] * 6)):
            token, prob, kept = check(x, u, **settings)
            assert np.all(token[:2] == -1) and np.all(kept[:2] == 0) and np.all(prob[:2] == 0)
            assert token[2] == 0 and token[4] == vocab - 1 and prob[4] == 1 and kept[4] == 1


def test_infinite_and_huge_logits():
    x, u = logits(6, 5000, "f32", seed=8)
    x[0, [7, 4000]] = np.inf
    x[1, 9] = np.inf
    x[2] *= 1e30
    x[3, 5], x[3, 6] = 3.4e38, -3.4e38
    x[4] *= 1e-30
    x[5, 100] = 1e30
    for settings in ({}, dict(top_k=[2] * 6), dict(top_k=[400] * 6, top_p=[0.9] * 6), dict(min_p=[0.1] * 6),
                     dict(temperature=[1e-38, 1e-30, 1e30, 1e38, 1e-30, 1e-3])):
        check(x, u, **settings)


def test_settings_at_their_ends():
    x, u = logits(8, 3000, "f32", seed=9)
    inf = float("inf")
    check(x, u, top_p=[0.0, -1.0, 1.0, 2.0, np.nan, 1e-30, 0.99999994, 0.5], allowed=1)  # (0.99999994: 2^-24 of the weight is left)
    check(x, u, min_p=[-1.0, 0.0, 1.0, 1.5, np.nan, 1e-30, 1e-5, inf])
    check(x, u, top_k=[-5, 0, 1, 3000, 3001, 2 ** 31 - 1, 2999, 2])
    check(x, u, temperature=[inf, 1e-30, 1.0, 100.0, 1e-3, 1e-45, 5.0, 1.0])


def test_random_numbers_at_their_ends():
    x, _ = logits(8, 3000, "bf16", seed=10)
    u = [0.0, -0.5, np.nan, 1.0, 7.0, 1 - 2.0 ** -24, 2.0 ** -149, 0.5]
    l = x.double().numpy()
    for settings in ({}, dict(top_k=[10] * 8), dict(top_p=[0.9] * 8)):
        token, _, kept = call(x.cuda(), u, **settings)
        for r in range(8):
            one = {k: a[r] if k == "top_k" else float(np.float32(a[r])) for k, a in settings.items()}
            w = S.sample(l[r], float(np.float32(u[r])), **one)
            assert kept[r] == w[2]
            if u[r] >= 1:  # the last token that weighs something, in units of 2^-43
                ids = S.order(l[r])[:kept[r]]
                weigh = np.rint(S.weights(l[r], ids, 1.0) * 2.0 ** 43)
                assert token[r] == ids[int(np.nonzero(weigh)[0][-1])]
            else:
                assert token[r] == w[0]


@pytest.mark.parametrize("dtype", TYPES)
def test_rows_apart_and_out_of_line(dtype):
    """Rows that begin at every alignment, wider than the vocabulary: what lies beside them is not read."""
    n, vocab = 9, 1501
    x, u = logits(n, vocab, dtype, seed=11)
    for lead, width in ((0, vocab), (1, vocab + 4), (3, vocab + 8), (5, vocab + 16)):
        wide = torch.full((n * width + 16,), float("inf"), dtype=DT[dtype], device="cuda")
        view = wide[lead:lead + n * width].view(n, width)[:, :vocab]
        view.copy_(x)
        check(view, u, top_p=[0.9] * n)
        check(view, u, top_k=[20] * n)


def test_many_rows_and_the_largest_vocabulary():
    x, u = logits(300, 200, "bf16", seed=12)
    check(x, u, **spread_over(300, MIXES["all"]))
    x, u = logits(2, 1 << 20, "bf16", seed=13)
    check(x, u, top_k=[50, 0], top_p=[1.0, 0.8])


def test_shares_are_the_distribution():
    """Over evenly spread numbers a token is drawn as often as its share says, to one in their count."""
    x, _ = logits(1, 50, "f32", seed=14)
    n = 4000
    u = (np.arange(n) + 0.5) / n
    token, prob, _ = call(x.cuda().expand(n, 50).contiguous(), u, top_p=[0.95] * n)
    for t in np.unique(token):
        assert abs((token == t).mean() - prob[token == t][0]) <= 1.0 / n
    assert abs(sum(prob[token == t][0] for t in np.unique(token)) - 1) < 1e-5


def test_same_call_same_bits_and_without_outputs():
    x, u = logits(40, 30000, "f16", seed=15)
    xd, ud = x.cuda(), torch.as_tensor(u).float().cuda()
    first = call(xd, u, **spread_over(40, MIXES["all"]))
    for _ in range(3):
        again = call(xd, u, **spread_over(40, MIXES["all"]))
        assert all(np.array_equal(a, b) for a, b in zip(first, again))
    token = torch.empty(40, dtype=torch.int32, device="cuda")
    work = torch.empty(api.sae_sample_work_size(40, 30000), dtype=torch.uint8, device="cuda")
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    api.sae_sample(xd, ud, token, work, top_p=torch.full((40,), 0.9, device="cuda"), stream=s)
    torch.cuda.synchronize()
    assert np.array_equal(token.cpu().numpy(), call(xd, u, top_p=[0.9] * 40)[0])


def test_graph_replays_with_new_rows():
    x = torch.empty((6, 9000), device="cuda")
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    u = torch.empty(6, device="cuda")
    token, eager = (torch.empty(6, dtype=torch.int32, device="cuda") for _ in range(2))
    work = torch.empty(api.sae_sample_work_size(6, 9000), dtype=torch.uint8, device="cuda")
    p = torch.tensor([0.9, 1.0, 0.5, 0.9, 0.99, 0.7], device="cuda")
    k = torch.tensor([50, 0, 0, 600, 0, 1], dtype=torch.int32, device="cuda")

    def step(to):
        api.sae_sample(x, u, to, work, top_p=p, top_k=k)
    x.normal_(generator=g)
    u.uniform_(generator=g)
    step(eager)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(token)
    for i in range(6):
        x.normal_(generator=g).mul_(1 + 2 * i)
        u.uniform_(generator=g)
        graph.replay()
        torch.cuda.synchronize()
        step(eager)
        torch.cuda.synchronize()
        assert torch.equal(token, eager)


SPLIT_MIXES = {
    "whole": {}, "temperature": dict(temperature=[0.2, 0.0, 1.0, 3.0]), "top_p": dict(top_p=[0.1, 0.5, 0.9, 0.99]),
    "min_p": dict(min_p=[0.001, 0.05, 0.5, 1.0]),
    "all": dict(temperature=[0.8, 1.2, 0.5, 2.0], top_p=[0.95, 0.0, 1.0, 0.7], min_p=[0.01, 0.1, 0.0, 0.2]),
}


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("mix", sorted(SPLIT_MIXES))
@pytest.mark.parametrize("n,vocab", [(1, 65536), (5, 65537), (3, 100003), (2, 262144)])
def test_rows_that_several_workgroups_read(dtype, mix, n, vocab):
    """Few rows of a large vocabulary without a top_k; at odd sizes no row but the first is aligned."""
    x, u = logits(n, vocab, dtype, seed=vocab)
    check(x, u, **spread_over(n, SPLIT_MIXES[mix]))


def test_split_rows_either_side_of_the_rule():
    """The same answers of rows that are split, of more rows, which are not, and with a top_k that leaves all."""
    x, u = logits(65, 65600, "bf16", seed=21, spread=1.5)
    p = [0.5 + 0.007 * r for r in range(65)]
    many = call(x.cuda(), u, top_p=p)
    few = [call(x[a:b].cuda(), u[a:b], top_p=p[a:b]) for a, b in ((0, 1), (1, 65))]
    all_k = call(x[1:].cuda(), u[1:], top_p=p[1:], top_k=[65600] * 64)
    for i in range(3):
        assert np.array_equal(many[i], np.concatenate([f[i] for f in few]))
        assert np.array_equal(many[i][1:], all_k[i])


def test_split_rows_that_nothing_is_left_of():
    vocab = 70001
    x, u = logits(7, vocab, "f32", seed=22)
    x[0] = -np.inf
    x[1] = np.nan
    x[2, 1:] = -np.inf
    x[3, ::2] = np.nan
    x[4, :-1] = -np.inf
    x[5, [7, 40000, vocab - 1]] = np.inf
    x[6] = 0.5
    for settings in ({}, dict(top_p=[0.9] * 7), dict(temperature=[0.0] * 7), dict(top_p=[0.7] * 7, min_p=[0.1] * 7)):
        token, prob, kept = check(x, u, **settings)
        assert np.all(token[:2] == -1) and np.all(kept[:2] == 0) and np.all(prob[:2] == 0)
        assert token[2] == 0 and token[4] == vocab - 1 and prob[4] == 1 and kept[4] == 1


def test_split_rows_apart_and_out_of_line():
    n, vocab = 3, 65541
    x, u = logits(n, vocab, "bf16", seed=23)
    for lead, width in ((1, vocab + 4), (3, vocab + 8), (7, vocab + 16)):
        wide = torch.full((n * width + 16,), float("inf"), dtype=torch.bfloat16, device="cuda")
        view = wide[lead:lead + n * width].view(n, width)[:, :vocab]
        view.copy_(x)
        check(view, u, top_p=[0.9] * n)


def test_split_rows_in_a_graph():
    """The histogram in the workspace begins anew in each replay, and in eager calls between them."""
    n, vocab = 4, 90001
    x, u = torch.empty((n, vocab), device="cuda"), torch.empty(n, device="cuda")
    g = torch.Generator(device="cuda")
    g.manual_seed(2)
    token, eager = (torch.empty(n, dtype=torch.int32, device="cuda") for _ in range(2))
    work = torch.full((api.sae_sample_work_size(n, vocab),), 0xFF, dtype=torch.uint8, device="cuda")
    p = torch.tensor([0.9, 1.0, 0.5, 0.99], device="cuda")

    def step(to):
        api.sae_sample(x, u, to, work, top_p=p)
    x.normal_(generator=g)
    u.uniform_(generator=g)
    step(eager)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(token)
    for i in range(6):
        x.normal_(generator=g).mul_(1 + i)
        u.uniform_(generator=g)
        graph.replay()
        torch.cuda.synchronize()
        step(eager)
        torch.cuda.synchronize()
        assert torch.equal(token, eager)
        for r in range(n):
            assert int(token[r]) == S.sample(x[r].double().cpu().numpy(), float(u[r]), top_p=float(p[r]))[0]
