"""Attention calls of every way the kernels divide work: sequences cut over workgroups and joined, many more sequences
than workgroups, table entries refilled in the middle of a workgroup's steps, tiles that are split and tiles that are not,
for each head size."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

from attn_cases import Call  # noqa: E402
from harness import say  # noqa: E402
from kv_cases import DT, dev32  # noqa: E402
from oracle import kvcache as O  # noqa: E402
from paper_2605_18825_amd import api  # noqa: E402

TYPES = [O.BF16, O.F16, O.FP8]
EDGES = [0, 1, 2, 15, 16, 17, 31, 32, 33, 48, 63, 64, 65, 100, 127, 128, 129, 255, 257, 600]
WIDE = 1024  # blocks of a table: more than one workgroup is given


# ------------------------------------------------------------------ decode
@pytest.mark.parametrize("ty", TYPES)
@pytest.mark.parametrize("heads,kvh,dim", [(8, 2, 128), (7, 1, 64), (34, 2, 128), (6, 2, 256)])
def test_decode_edges_of_split_sequences(ty, heads, kvh, dim):
    Call(ty, heads, kvh, dim, EDGES + [3000], seed=dim + heads, width=WIDE, n_inst=2).check(True)


@pytest.mark.parametrize("ty", TYPES)
def test_decode_window_over_split_sequences(ty):
    lens = [4000, 3999, 4001, 9000, 5, 0, 4033, 6007]
    for window in (4000, 6001):
        Call(ty, 6, 2, 64, lens, seed=window, window=window).check(True)


@pytest.mark.parametrize("ty", TYPES)
def test_decode_holes_in_split_sequences(ty):
    lens = [100, 64, 40, 33, 500, 2600]
    holes = [(0, 0), (0, 3), (1, 3), (3, 0), (3, 1), (3, 2), (2, 1)] + [(4, j) for j in range(4, 24)]
    holes += [(5, j) for j in (0, 1, 60, 61, 62, 160)]
    Call(ty, 8, 2, 128, lens, seed=15, holes=holes, width=WIDE).check(True)


@pytest.mark.parametrize("ty", TYPES)
@pytest.mark.parametrize("n_seq", [257, 700])
def test_decode_more_sequences_than_workgroups(ty, n_seq):
    """Several sequences to a thread of the search; joins by workgroup; a few long sequences among short ones."""
    rng = np.random.default_rng(n_seq)
    lens = rng.integers(0, 90, n_seq)
    lens[[3, n_seq // 2, n_seq - 1]] = [5003, 3500, 2048]
    Call(ty, 2, 2, 64, lens, seed=n_seq, width=WIDE, n_inst=3, shared=1200).check(True)


@pytest.mark.parametrize("ty", TYPES)
@pytest.mark.parametrize("dim,n", [(64, 34000), (256, 33100)])
def test_decode_refills_table_entries(ty, dim, n):
    """So many heads that a workgroup takes more than 128 steps (32 of each wave's) of one sequence, with holes on both
    sides of the refill."""
    holes = [(0, j) for j in (0, 255, 256, 257, 300, 511, 512, 700, 1025)]
    Call(ty, 1024, 1, dim, [n, 70], seed=dim, holes=holes, shared=500).check(True)


# ----------------------------------------------------------------- prefill
def batch(rng, n_seq, long):
    """Sequences of a new token behind about `long` keys, one of them with several tiles of rows."""
    new = np.ones(n_seq, int)
    new[5] = 140
    return long + rng.integers(0, 200, n_seq) + new, new


@pytest.mark.parametrize("ty", TYPES)
@pytest.mark.parametrize("heads,kvh,dim", [(4, 2, 128), (6, 2, 64), (4, 2, 256)])
@pytest.mark.parametrize("window", [0, 1300])
def test_prefill_long_tiles_not_split(ty, heads, kvh, dim, window):
    """So many tiles that none is split, each of more steps than table entries are held for (16 of 64 keys, 32 of 32),
    with holes before, at and past the refill."""
    rng = np.random.default_rng(dim)
    lens, new = batch(rng, 130 if dim == 256 else 260, 1100)
    lens[5] = 2600
    holes = [(r, j) for r in (2, 5, 9) for j in (1, 30, 63, 64, 65, 66, 67)] + [(5, j) for j in (127, 128, 129, 150, 162)]
    Call(ty, heads, kvh, dim, lens, new=new, seed=dim + window, holes=holes, window=window, shared=700).check(False)


@pytest.mark.parametrize("ty", TYPES)
@pytest.mark.parametrize("window", [0, 3500])
def test_prefill_split_heads_of_256(ty, window):
    holes = [(0, j) for j in (0, 100, 101, 102, 103, 200, 310)]
    Call(ty, 6, 2, 256, [5100, 700, 33, 4000], new=[9, 70, 33, 1], seed=51 + window, window=window).check(False)
    Call(ty, 6, 2, 256, [5100, 700], new=[30, 70], seed=52 + window, window=window, holes=holes).check(False)


@pytest.mark.parametrize("ty", TYPES)
def test_prefill_split_many_sequences(ty):
    """Two sequences to a thread of the search for a workgroup's part."""
    rng = np.random.default_rng(53)
    new = rng.integers(0, 3, 400)
    lens = new + rng.integers(0, 60, 400)
    lens[[7, 300, 399]] = [6000, 2500, 900]
    new[[7, 300, 399]] = [20, 3, 1]
    Call(ty, 2, 1, 64, lens, new=new, seed=54, shared=700).check(False)


@pytest.mark.parametrize("ty", TYPES)
@pytest.mark.parametrize("heads,kvh,dim", [(4, 2, 128), (4, 2, 256)])
@pytest.mark.parametrize("window", [0, 4000])
def test_prefill_values_that_are_not_finite_in_split_tiles(ty, heads, kvh, dim, window):
    """NaN among the values of a split prompt's last keys: rows before them are as without, whatever part holds them."""
    lens, new = np.array([5000, 4200]), np.array([110, 40])
    at = ((0, 4950, 5), (0, 4999, 64), (0, 4930, 17), (1, 4180, 127), (1, 4199, 0))
    if window:
        at += ((0, 4900 - window, 9), (1, 4165 - window, 3))  # seen by the first rows alone

    c = Call(ty, heads, kvh, dim, lens, new=new, seed=55 + window, window=window)
    size = 1 if ty == O.FP8 else 2
    page = O.unpack(c.cache.pages[1], dim, size, 1)
    for r, t, d in at:
        where = (c.ids[r, t // 16], 1, t % 16, d)
        page[where] = 0x7F if ty == O.FP8 else {O.BF16: 0x7FC0, O.F16: 0x7E00}[ty]
        c.cache.values[1][where] = np.nan
    c.cache.pages[1] = O.pack(page, size, 1)
    want, wl, mag, big = c.want()
    got, lse = c.run(False)
    fine = np.isfinite(want)
    assert 0 < (~fine).sum() < 0.05 * fine.size
    assert np.array_equal(fine, np.isfinite(got))
    tol, tol_l = O.bounds(np.where(fine, want, 0), wl, np.where(fine, mag, 0), big, dim, c.dtype)
    assert np.all(np.abs(got - np.where(fine, want, 0))[fine] <= tol[fine])
    assert np.all(np.abs(lse - wl) <= tol_l)


def nan_at(c, places):
    """NaN in the values of head 1 at (sequence, position, dimension)."""
    size = 1 if c.ty == O.FP8 else 2
    page = O.unpack(c.cache.pages[1], c.dim, size, 1)
    for r, t, d in places:
        where = (c.ids[r, t // 16], 1, t % 16, d)
        page[where] = {O.BF16: 0x7FC0, O.F16: 0x7E00, O.FP8: 0x7F}[c.ty]
        c.cache.values[1][where] = np.nan
    c.cache.pages[1] = O.pack(page, size, 1)


@pytest.mark.parametrize("ty", TYPES)
@pytest.mark.parametrize("heads,kvh,dim,window", [(4, 2, 64, 0), (16, 2, 128, 0), (16, 2, 128, 900), (4, 2, 256, 900)])
@pytest.mark.parametrize("split", [True, False])
def test_prefill_nan_in_a_prefix_that_every_row_sees(ty, heads, kvh, dim, window, split):
    """NaN among the values of a cached prefix: every row gets it, at its dimensions alone, and the call takes no
    longer than others do (a few times as long at most: it looks whether some row does not see the value)."""
    if split:
        lens, new, shared = [1500, 1400], [61, 30], 0
    else:
        lens, new, shared = np.full(130 if dim == 256 else 260, 1100), np.ones(130 if dim == 256 else 260, int) * 2, 500
    c = Call(ty, heads, kvh, dim, lens, new=new, seed=60 + dim, window=window, shared=shared)
    # every row of the last new tokens sees positions past len - window, and those before the new tokens
    at = [(r, lens[r] - 200 + r % 7, (5 * r) % dim) for r in range(min(len(lens), 3))]
    if shared:  # blocks that are in no other place
        c.ids[c.ids >= shared - 3] -= 3
        for r, t, _ in at:
            c.ids[r, t // 16] = shared - 3 + r

    def time():
        kv = c.cache.device()
        q = torch.as_tensor(c.qbits).view(DT[c.dtype]).cuda()
        out = torch.empty_like(q)
        seqs = api.make_seqs(dev32(c.ids), dev32(c.lens), q_start=dev32(c.starts))
        work = torch.empty(api.sae_attn_work_size(kv, seqs, c.n, heads), dtype=torch.uint8, device="cuda")
        best = 1e9
        for _ in range(5):
            a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
            a.record()
            for _ in range(10):
                api.sae_attn_prefill(kv, seqs, q, out, c.scale, work, window=window)
            b.record()
            torch.cuda.synchronize()
            best = min(best, a.elapsed_time(b) / 10)
        return best
    say("NaN in a prefix, type %d heads %d/%d dim %d window %d %s" % (ty, heads, kvh, dim, window, "split" if split else "whole"))
    before = time()
    nan_at(c, at)
    after = time()
    say("  %.1f us, with NaN %.1f us" % (before * 1e3, after * 1e3))
    assert after < 5 * before
    want, wl, mag, big = c.want()
    got, lse = c.run(False)
    fine = np.isfinite(want)
    assert (~fine).any() and np.array_equal(fine, np.isfinite(got))
    tol, tol_l = O.bounds(np.where(fine, want, 0), wl, np.where(fine, mag, 0), big, dim, c.dtype)
    assert np.all(np.abs(got - np.where(fine, want, 0))[fine] <= tol[fine])
    assert np.all(np.abs(lse - wl) <= tol_l)


@pytest.mark.parametrize("dim", [64, 128, 256])
def test_prefill_values_near_the_largest(dim):
    """Values near bf16's largest, scores that grow by five powers of two every 64 keys: outputs do not overflow on the
    way to a mean that does not, whatever reference the weights are taken under."""
    def fill(c, ids, q):
        q[:] = 1.0
        c.values[1] = np.sign(c.values[1]) * 3e38
        for r, n in enumerate(lens):
            for t in range(n):  # one key of every 64 has all the weight, the later ones the more
                x = np.log(2.0) * (5 * (t // 64) if t % 64 == 40 else -300.0)
                c.values[0][ids[r, t // 16], :, t % 16] = x / dim ** 0.5
    for lens, new in (([20, 90, 400], [3, 60, 40]), ([2000], [5])):
        Call(O.BF16, 4, 2, dim, lens, new=new, seed=61, fill=fill).check(False)


@pytest.mark.parametrize("ty", TYPES)
def test_windows_past_every_position(ty):
    """The largest window there is hides nothing, also where rows have negative positions."""
    for window in (2 ** 31 - 1, 2 ** 31 - 20, 1 << 20):
        Call(ty, 8, 2, 128, [5, 20, 0, 300], new=[40, 25, 3, 30], seed=57, window=window).check(False)
        Call(ty, 8, 2, 128, [2000, 33], new=[40, 60], seed=58, window=window).check(False)
        Call(ty, 8, 2, 128, [5, 0, 2000], seed=59, window=window).check(True)


# ------------------------------------------------------------------- graph
@pytest.mark.parametrize("ty", [O.BF16, O.FP8])
def test_graph_replays_of_split_calls(ty):
    """A captured decode and prefill of split sequences, replayed as lengths grow, equal the eager calls."""
    most, new = np.array([3000, 40, 17, 5000, 640]), np.array([3, 1, 2, 30, 5])
    c = Call(ty, 8, 2, 128, most, new=new, seed=56)
    kv = c.cache.device()
    lens = dev32(most - 10)
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    q = torch.as_tensor(c.qbits).view(DT[c.dtype]).cuda()
    q1 = q[:5].clone()
    one, many = api.make_seqs(dev32(c.ids), lens), api.make_seqs(dev32(c.ids), lens, q_start=dev32(c.starts))
    outs, eager = (torch.empty_like(q1), torch.empty_like(q)), (torch.empty_like(q1), torch.empty_like(q))
    work = torch.empty(max(api.sae_attn_work_size(kv, one, 5, 8), api.sae_attn_work_size(kv, many, c.n, 8)),
                       dtype=torch.uint8, device="cuda")

    def step(to):
        api.sae_attn_decode(kv, one, q1, to[0], 0.1, work)
        api.sae_attn_prefill(kv, many, q, to[1], 0.1, work)
    say("graph of split calls, type %d" % ty)
    step(eager)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(outs)
    for _ in range(6):
        q.normal_(generator=g)
        q1.normal_(generator=g)
        lens += 1
        graph.replay()
        torch.cuda.synchronize()
        step(eager)
        torch.cuda.synchronize()
        assert torch.equal(outs[0], eager[0]) and torch.equal(outs[1], eager[1])
