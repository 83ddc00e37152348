"""GPU parity of the attention of drafted trees (sae_attn_tree) with the 64-bit oracle, within the bounds of
sae_attn_prefill's arithmetic (oracle.kvcache.bounds).  Every place of the cache that no sequence owns holds NaN."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

from harness import say  # noqa: E402
from kv_cases import DT, dev32  # noqa: E402
from oracle import kvcache as O  # noqa: E402
from paper_2605_18825_amd import api  # noqa: E402
from tree_cases import KINDS, TreeCall, tree  # noqa: E402

TYPES = [O.BF16, O.F16, O.FP8]
NEW = [1, 0, 2, 15, 16, 17, 31, 33, 64, 65, 5, 100]
CACHED = [0, 7, 300, 1, 16, 15, 33, 64, 0, 63, 129, 500]


@pytest.mark.parametrize("ty", TYPES)
@pytest.mark.parametrize("heads,kvh,dim", [(8, 2, 128), (7, 1, 64), (4, 4, 64), (6, 2, 256), (34, 2, 128)])
def test_edges(ty, heads, kvh, dim):
    """Trees and prefixes that end inside, at and past pages and steps; empty ones; every kind of tree."""
    for shift in (0, 1):
        TreeCall(ty, heads, kvh, dim, np.add(NEW, CACHED), NEW, kinds=KINDS[shift:] + KINDS[:shift], seed=dim + heads + shift).check()


@pytest.mark.parametrize("ty", TYPES)
@pytest.mark.parametrize("window", [1, 2, 3, 17, 64, 100, 2 ** 31 - 1])
def test_window(ty, window):
    """Windows shorter than a way up the tree, ending in the tree, at its start and in the prefix."""
    new = [200, 3, 90, 64, 33]
    TreeCall(ty, 6, 2, 64, [200, 40, 300, 64, 150], new, kinds=["chain", "random", "binary", "chain", "random"], window=window,
             seed=window % 1000).check()


@pytest.mark.parametrize("ty", TYPES)
@pytest.mark.parametrize("kind", KINDS)
def test_largest_trees(ty, kind):
    TreeCall(ty, 3, 1, 64, [256, 300, 1000], [256, 255, 256], kinds=[kind], seed=5).check()


@pytest.mark.parametrize("ty", TYPES)
@pytest.mark.parametrize("dim", [64, 128, 256])
def test_split_and_not(ty, dim):
    """Long prefixes whose keys are split and joined, also where a tree crosses two steps; so many tiles that none is."""
    TreeCall(ty, 8, 2, dim, [9000, 60, 5000, 4100], [25, 3, 64, 130], seed=23).check()
    TreeCall(ty, 4, 1, dim, [9000, 4090], [40, 60], seed=24, window=4000).check()
    n = 140 if dim == 256 else 270
    rng = np.random.default_rng(dim)
    new = rng.integers(1, 12, n)
    new[5] = 140
    TreeCall(ty, 4, 2, dim, new + 600 + rng.integers(0, 200, n), new, seed=25, shared=300).check()


@pytest.mark.parametrize("ty", TYPES)
@pytest.mark.parametrize("dim", [64, 128])
def test_holes(ty, dim):
    """Table entries without a block: in the prefix and among the tree's places."""
    lens, new = [100, 64, 40, 33, 500], [20, 64, 1, 33, 50]
    holes = [(0, 0), (0, 3), (1, 3), (3, 0), (3, 1), (3, 2)] + [(4, j) for j in range(4, 24)] + [(4, 30), (2, 1), (0, 5)]
    TreeCall(ty, 8, 2, dim, lens, new, seed=25, holes=holes).check()
    TreeCall(ty, 8, 2, dim, lens, new, seed=26, holes=holes, window=30, n_inst=2).check()
    far = [(0, j) for j in range(3, 700, 5)] + [(0, j) for j in range(400, 480)]
    TreeCall(ty, 4, 1, dim, [11200], [40], seed=27, holes=far).check()


@pytest.mark.parametrize("window", [0, 7])
@pytest.mark.parametrize("dim", [64, 128])
def test_more_nodes_than_places(window, dim):
    """Lengths smaller than the tree (0: padding): nodes without a place see nothing and are not seen."""
    TreeCall(O.BF16, 8, 2, dim, [5, 20, 0, 300], [40, 25, 3, 30], seed=27, window=window).check()


def test_one_token_each():
    """Without q_start a tree is one node: a decode."""
    c = TreeCall(O.BF16, 8, 2, 128, [1, 33, 0, 700], [1, 1, 1, 1], seed=28)
    want, wl, mag, big = c.want()
    tol, _ = O.bounds(want, wl, mag, big, 128, O.BF16)
    got, _ = c.run(one=True)
    assert np.all(np.abs(got - want) <= tol)


@pytest.mark.parametrize("ty", TYPES)
def test_a_chain_is_a_prompt(ty):
    """A chain's outputs are sae_attn_prefill's within both's rounding, window or not."""
    for window in (0, 50):
        c = TreeCall(ty, 8, 2, 128, [140, 333, 64], [70, 33, 64], kinds=["chain"], seed=29, window=window)
        kv = c.cache.device()
        q = torch.as_tensor(c.qbits).view(DT[c.dtype]).cuda()
        out = torch.empty_like(q)
        seqs = api.make_seqs(dev32(c.ids), dev32(c.lens), q_start=dev32(c.starts))
        work = torch.empty(api.sae_attn_work_size(kv, seqs, c.n, 8), dtype=torch.uint8, device="cuda")
        api.sae_attn_prefill(kv, seqs, q, out, c.scale, work, window=window)
        want, wl, mag, big = c.want()
        tol, _ = O.bounds(want, wl, mag, big, 128, c.dtype)
        got, _ = c.run()
        assert np.all(np.abs(got - want) <= tol) and np.all(np.abs(out.double().cpu().numpy() - want) <= tol)


def test_other_stream_and_stride():
    c = TreeCall(O.BF16, 8, 2, 128, [400, 90], [100, 12], seed=30, width=999)
    c.cache.pad = 128
    got, _ = c.run(stream=torch.cuda.Stream())
    want, wl, mag, big = c.want()
    tol, _ = O.bounds(want, wl, mag, big, 128, O.BF16)
    assert np.all(np.abs(got - want) <= tol)


@pytest.mark.parametrize("scale", [0.0, -0.125])
def test_scale_of_zero_and_below(scale):
    TreeCall(O.F16, 8, 2, 64, [3, 60, 200], [3, 60, 70], seed=31, scale=scale).check()


@pytest.mark.parametrize("what", [np.nan, np.inf])
@pytest.mark.parametrize("window", [0, 40])
@pytest.mark.parametrize("ty", TYPES)
@pytest.mark.parametrize("dim", [64, 128])
def test_values_that_are_not_finite_reach_only_their_descendants(ty, window, what, dim):
    """NaN or infinity among the values of some nodes and of a prefix key that a window hides from deep rows."""
    lens, new = np.array([150, 90, 4000]), np.array([60, 90, 30])
    c = TreeCall(ty, 4, 2, dim, lens, new, kinds=["random", "chain", "binary"], seed=40, window=window)
    size = 1 if ty == O.FP8 else 2
    bits = {(O.BF16, True): 0x7FC0, (O.BF16, False): 0x7F80, (O.F16, True): 0x7E00, (O.F16, False): 0x7C00}
    page = O.unpack(c.cache.pages[1], dim, size, 1)
    at = [(0, 140, 5), (0, 120, dim // 2), (1, 80, dim - 1), (1, 60, 0), (2, 3990, 3)]
    if window:
        at += [(0, 89 - 38, 9)]
    for r, t, d in at:
        where = (c.ids[r, t // 16], 1, t % 16, d)
        page[where] = 0x7F if ty == O.FP8 else bits[ty, bool(np.isnan(what))]
        c.cache.values[1][where] = np.nan if ty == O.FP8 else what
    c.cache.pages[1] = O.pack(page, size, 1)
    want, wl, mag, big = c.want()
    got, lse = c.run()
    fine = np.isfinite(want)
    assert 0 < (~fine).sum() < 0.05 * fine.size
    assert np.array_equal(fine, np.isfinite(got))
    tol, tol_l = O.bounds(np.where(fine, want, 0), wl, np.where(fine, mag, 0), big, dim, c.dtype)
    assert np.all(np.abs(got - np.where(fine, want, 0))[fine] <= tol[fine])
    assert np.all(np.abs(lse - wl) <= tol_l)


def test_huge_scores():
    """Scores of thousands of millions, past what the loop's exponents hold: the slow path, among a tree's nodes too."""
    def fill(cache, ids, q):
        q *= 2.0 ** 14
        cache.values[0] *= 2.0 ** 13
    TreeCall(O.BF16, 2, 1, 64, [30, 70], [20, 33], seed=41, fill=fill).check()


def test_bad_parents_are_reported():
    """A parent that is no earlier node counts as none; more nodes than max_nodes see nothing."""
    lens, new = np.array([60, 100, 90]), np.array([20, 30, 40])
    c = TreeCall(O.BF16, 4, 2, 64, lens, new, seed=42)
    q = torch.as_tensor(c.qbits).view(torch.bfloat16).cuda()
    for what in ("later", "self", "low", "many"):
        given = [p.copy() for p in c.parents]
        if what == "many":
            c.max_nodes = 39
        else:
            j = 7
            given[1][j] = {"later": 20, "self": j, "low": -5}[what]
            c.parents[1] = given[1].copy()
            c.parents[1][j] = -1
        kv = c.cache.device()
        out, lse = torch.full_like(q, 7.0), torch.full((c.n, 4), 7.0, device="cuda")
        seqs = api.make_seqs(dev32(c.ids), dev32(lens), q_start=dev32(c.starts))
        work = torch.empty(api.sae_attn_work_size(kv, seqs, c.n, 4), dtype=torch.uint8, device="cuda")
        say("bad parents: %s" % what)
        api.sae_attn_tree(kv, seqs, dev32(np.concatenate(given)), c.max_nodes, q, out, c.scale, work, lse=lse)
        want, wl, mag, big = c.want()
        if what == "many":
            want[50:], mag[50:], wl[50:] = 0, 0, -np.inf
        tol, _ = O.bounds(want, wl, mag, big, 64, O.BF16)
        assert np.all(np.abs(out.double().cpu().numpy() - want) <= tol)
        assert np.array_equal(np.isinf(lse.cpu().numpy()), np.isinf(wl))
        assert api.status_names(int(c.cache.status[0])) == ["BAD_TREE"]


@pytest.mark.parametrize("ty,dim", [(O.BF16, 128), (O.FP8, 128), (O.F16, 64)])
def test_graph_replays_with_new_trees(ty, dim):
    """A captured call replayed with other lengths, trees and contents equals the eager one, bit for bit."""
    most, new = np.array([3000, 40, 17, 5000, 640]), np.array([30, 1, 2, 64, 5])
    c = TreeCall(ty, 8, 2, dim, most, new, seed=56)
    kv, lens = c.cache.device(), dev32(most - 10)
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    rng = np.random.default_rng(2)
    q = torch.as_tensor(c.qbits).view(DT[c.dtype]).cuda()
    out, eager = torch.empty_like(q), torch.empty_like(q)
    seqs = api.make_seqs(dev32(c.ids), lens, q_start=dev32(c.starts))
    work = torch.empty(api.sae_attn_work_size(kv, seqs, c.n, 8), dtype=torch.uint8, device="cuda")
    parent = c.parent()

    def step(to):
        api.sae_attn_tree(kv, seqs, parent, 64, q, to, 0.1, work)
    step(eager)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(out)
    for i in range(6):
        q.normal_(generator=g)
        lens += 1
        parent.copy_(dev32(np.concatenate([tree(n, KINDS[i], rng) for n in new])))
        graph.replay()
        torch.cuda.synchronize()
        step(eager)
        torch.cuda.synchronize()
        assert torch.equal(out, eager)
    assert int(c.cache.status[0]) == 0


@pytest.mark.parametrize("ty,dim", [(O.BF16, 128), (O.F16, 64)])
def test_more_sequences_than_are_split(ty, dim):
    """Every sequence in one part, though some are long."""
    rng = np.random.default_rng(3)
    new = rng.integers(0, 4, 600)
    cached = rng.integers(0, 40, 600)
    cached[[0, 300, 599]] = 2500
    new[[0, 300, 599]] = 33
    TreeCall(ty, 4, 2, dim, new + cached, new, seed=60).check()


@pytest.mark.parametrize("ty,dim", [(O.BF16, 128), (O.F16, 64), (O.FP8, 256)])
def test_too_many_nodes_behind_a_long_prefix(ty, dim):
    """All rows of a sequence with more than max_nodes are zeros, where keys are split too; the others are as ever."""
    lens, new = np.array([3000, 2000, 5000]), np.array([200, 1, 1])
    for seqs in (slice(0, 1), slice(0, 3)):
        c = TreeCall(ty, 2, 2, dim, lens[seqs], new[seqs], seed=61)
        c.max_nodes = 1
        kv = c.cache.device()
        q = torch.as_tensor(c.qbits).view(DT[c.dtype]).cuda()
        out, lse = torch.full_like(q, 7.0), torch.full((c.n, 2), 7.0, device="cuda")
        work = torch.full((api.sae_attn_work_size(kv, api.make_seqs(dev32(c.ids), dev32(c.lens), q_start=dev32(c.starts)), c.n, 2),), 0xFF,
                          dtype=torch.uint8, device="cuda")
        say("too many nodes: type %d dim %d, %d sequences" % (ty, dim, len(c.lens)))
        api.sae_attn_tree(kv, api.make_seqs(dev32(c.ids), dev32(c.lens), q_start=dev32(c.starts)), c.parent(), 1, q, out, c.scale, work,
                          lse=lse)
        want, wl, mag, big = c.want()
        want[:200], mag[:200], wl[:200] = 0, 0, -np.inf
        tol, _ = O.bounds(want, wl, mag, big, dim, c.dtype)
        tol[:200] = 0
        assert np.all(np.abs(out.double().cpu().numpy() - want) <= tol)
        assert np.array_equal(np.isinf(lse.cpu().numpy()), np.isinf(wl))
        assert api.status_names(int(c.cache.status[0])) == ["BAD_TREE"]
