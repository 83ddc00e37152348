"""GPU parity of the attention over the paged cache (sae_attn_decode, sae_attn_prefill) with the 64-bit oracle, within
bounds that follow from the arithmetic (oracle.kvcache.bounds).  Every place of the cache that no sequence owns holds
NaN, in keys, values and scale bytes."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

from harness import say  # noqa: E402
from kv_cases import DT, Cache, dev32, oracle_attention, tables, to16  # noqa: E402
from oracle import kvcache as O  # noqa: E402
from paper_2605_18825_amd import api  # noqa: E402

EDGES = [0, 1, 2, 15, 16, 17, 31, 32, 33, 48, 63, 64, 65, 100, 127, 128, 129, 255, 257, 600]


def run(ty, heads, kvh, dim, lens, new=None, n_inst=1, window=0, seed=0, holes=(), spread=1.0, scale=None, lse=True,
        pad=0, stream=None, width=0, tweak=None):
    """A decode (new is None) or prefill call and its check; returns the outputs."""
    rng = np.random.default_rng(seed)
    dtype = O.BF16 if ty == O.FP8 else ty
    lens = np.asarray(lens)
    ids, inst, bpi, owned = tables(lens, n_inst, rng, width=width)
    c = Cache(ty, n_inst, bpi, kvh, dim, rng, pad_blocks=pad, spread=spread)
    for r, j in holes:
        if ids[r, j] >= 0:
            owned[inst[r] * bpi + ids[r, j]] = False
            ids[r, j] = -1
    c.poison(owned)
    counts = np.ones(len(lens), int) if new is None else np.asarray(new)
    starts = np.concatenate([[0], np.cumsum(counts)])
    n = starts[-1]
    scale = dim ** -0.5 if scale is None else scale
    qval, qbits = to16(rng.standard_normal((n, heads, dim)) * 2, dtype)
    if tweak:
        tweak(c, ids, qval)
        qval, qbits = to16(qval, dtype)
    say("attention type %d heads %d/%d dim %d seqs %d rows %d window %d" % (ty, heads, kvh, dim, len(lens), n, window))
    kv = c.device()
    # queries and outputs lie in wider rows
    fused = torch.full((n, (heads + 2 * kvh) * dim), 7.0, dtype=DT[dtype], device="cuda")
    q = fused[:, :heads * dim].view(n, heads, dim)
    q.copy_(torch.as_tensor(qbits).view(DT[dtype]))
    wide = torch.full((n, heads * dim + 64), 7.0, dtype=DT[dtype], device="cuda")
    out = wide[:, :heads * dim].view(n, heads, dim)
    ls = torch.full((n, heads), 7.0, dtype=torch.float32, device="cuda") if lse else None
    seqs = api.make_seqs(dev32(ids), dev32(lens), q_start=None if new is None else dev32(starts),
                         inst=dev32(inst) if n_inst > 1 else None)
    work = torch.full((api.sae_attn_work_size(kv, seqs, n, heads),), 0xFF, dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    call = api.sae_attn_decode if new is None else api.sae_attn_prefill
    call(kv, seqs, q, out, scale, work, window=window, lse=ls, stream=stream)
    torch.cuda.synchronize()
    want, wl, mag, big = oracle_attention(c, ids, inst, lens, starts, qval, scale, window)
    tol, tol_l = O.bounds(want, wl, mag, big, dim, dtype)
    got = out.double().cpu().numpy()
    bad = ~(np.abs(got - want) <= tol)
    assert not bad.any(), (np.argwhere(bad)[:5].tolist(), float(np.nanmax(np.abs(got - want) / tol)), int(bad.sum()))
    if lse:
        gl = ls.double().cpu().numpy()
        dead = np.isinf(wl)
        assert np.array_equal(gl[dead], wl[dead])
        assert np.all(np.abs(gl[~dead] - wl[~dead]) <= tol_l[~dead])
    assert torch.all(wide[:, heads * dim:] == 7.0)
    assert int(c.status[0]) == 0
    say("  worst error %.2f of its bound" % float(np.max(np.abs(got - want) / tol)))
    return got


TYPES = [O.BF16, O.F16, O.FP8]


@pytest.mark.parametrize("ty", TYPES)
@pytest.mark.parametrize("heads,kvh,dim", [(8, 2, 128), (7, 1, 64), (4, 4, 64), (6, 2, 256), (34, 2, 128)])
def test_decode_edges(ty, heads, kvh, dim):
    run(ty, heads, kvh, dim, EDGES, seed=dim + heads)


@pytest.mark.parametrize("ty", TYPES)
@pytest.mark.parametrize("window", [1, 2, 17, 64, 100])
def test_decode_window(ty, window):
    run(ty, 6, 2, 64, EDGES, window=window, seed=window, n_inst=2)


@pytest.mark.parametrize("ty", TYPES)
def test_decode_long_and_short(ty):
    """One sequence much longer than the others: its parts are joined."""
    run(ty, 8, 2, 128, [3, 20011, 0, 700, 1], seed=11)
    run(ty, 4, 1, 64, [33000], seed=12)
    run(ty, 4, 1, 64, [33000], seed=13, window=20000)


@pytest.mark.parametrize("ty", TYPES)
def test_decode_many_sequences(ty):
    rng = np.random.default_rng(1)
    run(ty, 2, 2, 64, rng.integers(0, 90, 700), seed=14, n_inst=3, lse=False)


@pytest.mark.parametrize("ty", TYPES)
def test_decode_holes(ty):
    """Table entries without a block: at the start, in the middle, at the end, everywhere."""
    lens = [100, 64, 40, 33, 500]
    holes = [(0, 0), (0, 3), (1, 3), (3, 0), (3, 1), (3, 2)] + [(4, j) for j in range(4, 24)] + [(2, 1)]
    run(ty, 8, 2, 128, lens, seed=15, holes=holes)
    run(ty, 8, 2, 128, lens, seed=16, holes=holes, window=30)


def test_decode_wide_table_and_stride():
    run(O.BF16, 8, 2, 128, [40, 300], seed=17, width=4096, pad=128)
    run(O.FP8, 8, 2, 128, [40, 300], seed=17, width=4096, pad=256)


def test_decode_other_stream():
    s = torch.cuda.Stream()
    run(O.BF16, 8, 2, 128, [1000, 3000], seed=18, stream=s)


def _large(c, ids, qval):
    qval *= 40.0


def _equal(c, ids, qval):
    qval[:] = 0.0


@pytest.mark.parametrize("tweak", [_large, _equal])
@pytest.mark.parametrize("ty", TYPES)
def test_decode_extreme_scores(ty, tweak):
    """Scores of hundreds (all the weight on one key), and all scores equal."""
    run(ty, 8, 2, 128, [1, 40, 700, 3000], seed=19, tweak=tweak)


@pytest.mark.parametrize("ty", TYPES)
@pytest.mark.parametrize("heads,kvh,dim", [(8, 2, 128), (7, 1, 64), (4, 4, 64), (6, 2, 256), (34, 2, 128)])
def test_prefill_edges(ty, heads, kvh, dim):
    """Suffixes and prefixes that end inside, at and past tiles; empty ones."""
    new = [1, 0, 2, 15, 16, 17, 31, 33, 64, 65, 5]
    cached = [0, 7, 300, 1, 16, 15, 33, 64, 0, 63, 129]
    run(ty, heads, kvh, dim, np.add(new, cached), new=new, seed=dim + heads)


@pytest.mark.parametrize("ty", TYPES)
def test_prefill_larger(ty):
    run(ty, 4, 2, 128, [700, 130], new=[600, 129], seed=21, n_inst=2)
    run(ty, 5, 1, 64, [513], new=[513], seed=22, lse=False)


@pytest.mark.parametrize("ty", TYPES)
@pytest.mark.parametrize("window", [1, 2, 17, 64, 100])
def test_prefill_window(ty, window):
    run(ty, 6, 2, 64, [200, 40, 300], new=[200, 3, 90], window=window, seed=window)


@pytest.mark.parametrize("ty", TYPES)
def test_prefill_short_suffix_of_long_prefix(ty):
    """Few rows over many keys: the keys are split and joined."""
    run(ty, 8, 2, 128, [9000, 60, 5000], new=[5, 3, 17], seed=23)
    run(ty, 4, 1, 64, [20000], new=[40], seed=24, window=15000)


@pytest.mark.parametrize("ty", TYPES)
def test_prefill_holes(ty):
    lens, new = [100, 64, 40, 33, 500], [20, 64, 1, 33, 50]
    holes = [(0, 0), (0, 3), (1, 3), (3, 0), (3, 1), (3, 2)] + [(4, j) for j in range(4, 24)] + [(2, 1)]
    run(ty, 8, 2, 128, lens, new=new, seed=25, holes=holes)
    run(ty, 8, 2, 128, lens, new=new, seed=26, holes=holes, window=30)


def test_prefill_more_new_tokens_than_positions():
    run(O.BF16, 8, 2, 128, [5, 20, 0], new=[40, 25, 3], seed=27)


@pytest.mark.parametrize("tweak", [_large, _equal])
@pytest.mark.parametrize("ty", TYPES)
def test_prefill_extreme_scores(ty, tweak):
    run(ty, 8, 2, 128, [40, 700], new=[40, 90], seed=28, tweak=tweak)


def test_prefill_other_stream_and_stride():
    s = torch.cuda.Stream()
    run(O.BF16, 8, 2, 128, [400], new=[100], seed=29, stream=s, width=999, pad=128)


def test_infinite_scores():
    """Keys of infinity: a score of -inf weighs nothing, a row with nothing else gets zeros."""
    for new in (None, [1, 1, 1]):
        rng = np.random.default_rng(30)
        lens = np.array([20, 40, 16])
        ids, inst, bpi, owned = tables(lens, 1, rng)
        c = Cache(O.BF16, 1, bpi, 1, 64, rng)
        q = np.abs(rng.standard_normal((3, 2, 64))) + 0.5
        qval, qbits = to16(q, O.BF16)
        dead = np.zeros((bpi, 16), bool)
        dead[ids[0, 0], 3:9] = True   # some keys of sequence 0, the whole of sequence 2
        dead[ids[2, 0]] = True
        page = O.unpack(c.pages[0], 64, 2, 0)
        page[np.broadcast_to(dead[:, None, :, None], page.shape)] = np.int16(np.uint16(0xFF80).view(np.int16))
        c.pages[0] = O.pack(page, 2, 0)
        c.values[0][np.broadcast_to(dead[:, None, :, None], c.values[0].shape)] = -np.inf
        kv = c.device()
        seqs = api.make_seqs(dev32(ids), dev32(lens), q_start=None if new is None else dev32([0, 1, 2, 3]))
        qt = torch.as_tensor(qbits).view(torch.bfloat16).cuda()
        out = torch.full_like(qt, 7.0)
        lse = torch.zeros((3, 2), device="cuda")
        work = torch.empty(api.sae_attn_work_size(kv, seqs, 3, 2), dtype=torch.uint8, device="cuda")
        (api.sae_attn_decode if new is None else api.sae_attn_prefill)(kv, seqs, qt, out, 0.125, work, lse=lse)
        want, wl, mag, _ = oracle_attention(c, ids, inst, lens, np.arange(4), qval, 0.125, 0)
        finite = 0.125 * np.abs(qval).sum(-1) * 6  # of the keys that weigh something: |k| < 6
        tol, tol_l = O.bounds(want, wl, mag, finite, 64, O.BF16)
        got = out.double().cpu().numpy()
        assert np.all(got[2] == 0) and np.all(np.isneginf(lse[2].cpu().numpy()))
        assert np.all(np.abs(got - want) <= tol)
        assert np.all(np.abs(lse[:2].double().cpu().numpy() - wl[:2]) <= tol_l[:2])


def test_nan_in_a_seen_place_is_seen():
    """A NaN in a place that a row sees makes that row NaN and no other."""
    for new in (None, [1, 1]):
        rng = np.random.default_rng(31)
        lens = np.array([50, 90])
        ids, inst, bpi, _ = tables(lens, 1, rng)
        for which in range(2):
            c = Cache(O.BF16, 1, bpi, 1, 64, rng)
            page = O.unpack(c.pages[which], 64, 2, which)
            page[ids[0, 1], 0, 5, 7] = 0x7FC0
            c.pages[which] = O.pack(page, 2, which)
            kv = c.device()
            seqs = api.make_seqs(dev32(ids), dev32(lens), q_start=None if new is None else dev32([0, 1, 2]))
            qt = torch.ones((2, 2, 64), dtype=torch.bfloat16, device="cuda")
            out = torch.zeros_like(qt)
            work = torch.empty(api.sae_attn_work_size(kv, seqs, 2, 2), dtype=torch.uint8, device="cuda")
            (api.sae_attn_decode if new is None else api.sae_attn_prefill)(kv, seqs, qt, out, 0.125, work)
            o = torch.isnan(out).cpu().numpy()
            assert not o[1].any()
            assert o[0].all() if which == 0 else (o[0, :, 7].all() and not o[0, :, :7].any())


def test_bad_tables_are_reported():
    """Ids and instances out of range are no blocks; a length past the table is cut to it."""
    rng = np.random.default_rng(32)
    lens = np.array([40, 30, 64])
    ids, _, bpi, _ = tables(lens, 1, rng, width=4)
    c = Cache(O.BF16, 1, bpi, 2, 64, rng)
    ids[0, 1] = bpi + 5
    given, inst = np.array([40, 30, 900]), np.array([0, 3, 0], np.int32)
    qval, qbits = to16(rng.standard_normal((3, 4, 64)), O.BF16)
    oid = ids.copy()
    oid[0, 1] = -1
    oid[1] = -1
    want, wl, mag, big = oracle_attention(c, oid, np.zeros(3, int), lens, np.arange(4), qval, 0.125, 0)
    tol, _ = O.bounds(want, wl, mag, big, 64, O.BF16)
    for qs in (None, dev32([0, 1, 2, 3])):
        kv = c.device()
        seqs = api.make_seqs(dev32(ids), dev32(given), q_start=qs, inst=dev32(inst))
        qt = torch.as_tensor(qbits).view(torch.bfloat16).cuda()
        out = torch.full_like(qt, 7.0)
        work = torch.empty(api.sae_attn_work_size(kv, seqs, 3, 4), dtype=torch.uint8, device="cuda")
        (api.sae_attn_decode if qs is None else api.sae_attn_prefill)(kv, seqs, qt, out, 0.125, work)
        assert np.all(np.abs(out.double().cpu().numpy() - want) <= tol)
        assert api.status_names(int(c.status[0])) == ["BAD_BLOCK"]


@pytest.mark.parametrize("ty", [O.BF16, O.FP8])
def test_graph_replays_with_new_lengths(ty):
    """A captured decode step (write, attention) replayed while the sequences grow equals the eager calls."""
    rng = np.random.default_rng(33)
    heads, kvh, dim, n = 8, 2, 64, 5
    most = np.array([200, 40, 17, 900, 64])
    ids, _, bpi, _ = tables(most, 1, rng)
    c = Cache(ty, 1, bpi, kvh, dim, rng)
    kv = c.device()
    lens = dev32(most - 10)
    seqs = api.make_seqs(dev32(ids), lens)
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    q = torch.empty((n, heads, dim), dtype=torch.bfloat16, device="cuda")
    k, v = (torch.empty((n, kvh, dim), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    out, eager = torch.empty_like(q), torch.empty_like(q)
    work = torch.empty(api.sae_attn_work_size(kv, seqs, n, heads), dtype=torch.uint8, device="cuda")

    def step(to):
        api.sae_kv_write(kv, seqs, k, v)
        api.sae_attn_decode(kv, seqs, q, to, 0.125, work)
    for t in (q, k, v):
        t.normal_(generator=g)
    step(eager)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(out)
    for _ in range(6):
        for t in (q, k, v):
            t.normal_(generator=g)
        lens += 1
        graph.replay()
        torch.cuda.synchronize()
        step(eager)
        torch.cuda.synchronize()
        assert torch.equal(out, eager)


def test_same_call_same_bits():
    rng = np.random.default_rng(34)
    lens = rng.integers(1, 3000, 40)
    ids, _, bpi, _ = tables(lens, 1, rng)
    c = Cache(O.BF16, 1, bpi, 2, 128, rng)
    kv = c.device()
    for qs in (None, np.concatenate([[0], np.cumsum(np.minimum(lens, 30))])):
        n = 40 if qs is None else int(qs[-1])
        seqs = api.make_seqs(dev32(ids), dev32(lens), q_start=None if qs is None else dev32(qs))
        q = torch.as_tensor(to16(rng.standard_normal((n, 8, 128)), O.BF16)[1]).view(torch.bfloat16).cuda()
        outs = [torch.empty_like(q) for _ in range(3)]
        work = torch.empty(api.sae_attn_work_size(kv, seqs, n, 8), dtype=torch.uint8, device="cuda")
        for o in outs:
            (api.sae_attn_decode if qs is None else api.sae_attn_prefill)(kv, seqs, q, o, 0.1, work)
        torch.cuda.synchronize()
        assert torch.equal(outs[0], outs[1]) and torch.equal(outs[0], outs[2])


@pytest.mark.parametrize("what", [np.nan, np.inf])
@pytest.mark.parametrize("window", [0, 40])
@pytest.mark.parametrize("ty", TYPES)
def test_values_that_are_not_finite_reach_only_rows_that_see_them(ty, window, what):
    """Values of NaN or infinity at a few keys of a prompt: earlier rows (and rows past the window) are as without them."""
    heads, kvh, dim = 4, 2, 128
    rng = np.random.default_rng(40)
    lens, new = np.array([150, 90]), np.array([110, 90])
    ids, inst, bpi, _ = tables(lens, 1, rng)
    c = Cache(ty, 1, bpi, kvh, dim, rng)
    size = 1 if ty == O.FP8 else 2
    bits = {(O.BF16, True): 0x7FC0, (O.BF16, False): 0x7F80, (O.F16, True): 0x7E00, (O.F16, False): 0x7C00}
    page = O.unpack(c.pages[1], dim, size, 1)
    for r, t, d in ((0, 77, 5), (0, 100, 64), (1, 89, 127), (1, 31, 0)):
        where = (ids[r, t // 16], 1, t % 16, d)
        page[where] = 0x7F if ty == O.FP8 else bits[ty, bool(np.isnan(what))]
        c.values[1][where] = np.nan if ty == O.FP8 else what
    c.pages[1] = O.pack(page, size, 1)
    kv = c.device()
    starts = np.array([0, 110, 200])
    dtype = O.BF16 if ty == O.FP8 else ty
    qval, qbits = to16(rng.standard_normal((200, heads, dim)), dtype)
    q = torch.as_tensor(qbits).view(DT[dtype]).cuda()
    out, lse = torch.zeros_like(q), torch.zeros((200, heads), device="cuda")
    seqs = api.make_seqs(dev32(ids), dev32(lens), q_start=dev32(starts))
    work = torch.empty(api.sae_attn_work_size(kv, seqs, 200, heads), dtype=torch.uint8, device="cuda")
    say("values not finite, type %d window %d" % (ty, window))
    api.sae_attn_prefill(kv, seqs, q, out, 0.1, work, window=window, lse=lse)
    want, wl, mag, big = oracle_attention(c, ids, inst, lens, starts, qval, 0.1, window)
    got = out.double().cpu().numpy()
    fine = np.isfinite(want)
    assert 0 < (~fine).sum() < 0.05 * fine.size
    assert np.array_equal(fine, np.isfinite(got))
    tol, tol_l = O.bounds(np.where(fine, want, 0), wl, np.where(fine, mag, 0), big, dim, dtype)
    assert np.all(np.abs(got - np.where(fine, want, 0))[fine] <= tol[fine])
    assert np.all(np.abs(lse.double().cpu().numpy() - wl) <= tol_l)


@pytest.mark.parametrize("scale", [0.0, -0.125])
def test_scale_of_zero_and_below(scale):
    for new in (None, [3, 60, 70]):
        run(O.BF16, 8, 2, 128, [3, 60, 200], new=new, seed=41, scale=scale)


def test_prefill_one_token_each():
    """Without q_start: one new token per sequence, also where its heads fill several tiles."""
    rng = np.random.default_rng(42)
    lens = np.array([1, 33, 0, 500])
    for heads, kvh in ((8, 2), (300, 1)):
        ids, inst, bpi, _ = tables(lens, 1, rng)
        c = Cache(O.BF16, 1, bpi, kvh, 64, rng)
        kv = c.device()
        qval, qbits = to16(rng.standard_normal((4, heads, 64)), O.BF16)
        q = torch.as_tensor(qbits).view(torch.bfloat16).cuda()
        seqs = api.make_seqs(dev32(ids), dev32(lens))
        work = torch.empty(api.sae_attn_work_size(kv, seqs, 4, heads), dtype=torch.uint8, device="cuda")
        want, wl, mag, big = oracle_attention(c, ids, inst, lens, np.arange(5), qval, 0.1, 0)
        tol, _ = O.bounds(want, wl, mag, big, 64, O.BF16)
        for call in (api.sae_attn_prefill, api.sae_attn_decode):
            out = torch.full_like(q, 7.0)
            call(kv, seqs, q, out, 0.1, work)
            assert np.all(np.abs(out.double().cpu().numpy() - want) <= tol)


def test_prefill_many_sequences():
    """More sequences than a split call takes, long and short ones; and a batch whose longest is split the most."""
    rng = np.random.default_rng(43)
    new = rng.integers(0, 5, 700)
    new[-1] = 1
    run(O.BF16, 4, 2, 64, new + rng.integers(0, 70, 700), new=new, seed=44, lse=False)
    run(O.F16, 4, 2, 64, [700, 6000, 3, 90, 2500], new=[30, 70, 3, 1, 200], seed=45)
    run(O.FP8, 16, 2, 128, [9000], new=[150], seed=46)
