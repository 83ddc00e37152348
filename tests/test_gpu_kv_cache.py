"""GPU parity of the paged key-value cache's write and read (sae_kv_write, sae_kv_read) with the 64-bit oracle: every
stored byte and every value read is equal, bit for bit, and no byte beside the written positions changes."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

from harness import say  # noqa: E402
from kv_cases import DT, Cache, dev32, from16, tables, to16  # noqa: E402
from oracle import kvcache as O  # noqa: E402
from paper_2605_18825_amd import api  # noqa: E402

# (cached tokens, new tokens): starts and ends inside, at and across pages, nothing new, nothing at all
RAGGED = [(0, 1), (0, 16), (5, 11), (5, 12), (16, 16), (15, 2), (0, 0), (31, 33), (40, 0), (7, 1), (16, 1), (3, 200)]


def setup(ty, kvh, dim, parts, n_inst=1, seed=0, pad=0):
    rng = np.random.default_rng(seed)
    cached, new = np.array([p[0] for p in parts]), np.array([p[1] for p in parts])
    ids, inst, bpi, _ = tables(cached + new, n_inst, rng)
    c = Cache(ty, n_inst, bpi, kvh, dim, rng, pad_blocks=pad)
    starts = np.concatenate([[0], np.cumsum(new)])
    return rng, c, ids, inst, cached + new, new, starts


def positions(c, ids, inst, lens, new):
    """(pool block, token) of every new token, -1 where its table has no block or its position is negative."""
    out = []
    for r in range(len(lens)):
        for p in range(lens[r] - new[r], lens[r]):
            b = -1 if p < 0 else ids[r, p // 16]
            out.append((inst[r] * c.bpi + b if 0 <= b < c.bpi else -1, p % 16))
    return np.array(out, np.int64).reshape(-1, 2)


def rows(rng, n, kvh, dim, dtype, outliers=False):
    x = rng.standard_normal((n, kvh, dim)) * np.exp2(rng.integers(-6, 7, (n, kvh, 1)))
    if outliers and n >= 6:
        x[0, 0] = 0.0                      # a row of zeros
        x[1, 0, :3] = [np.inf, -np.inf, np.nan]
        x[2, 0] = np.nan                   # nothing finite
        x[3, 0] *= 2.0 ** -20              # f16 subnormals
        x[4, 0, 0] = 60000.0
        x[5, 0] = 448.0 * np.exp2(np.arange(dim) % 5 - 2.0)  # its largest is at the edge of a scale
    return to16(x, dtype)


@pytest.mark.parametrize("ty,dtype", [(O.BF16, O.BF16), (O.F16, O.F16), (O.FP8, O.BF16), (O.FP8, O.F16)])
@pytest.mark.parametrize("kvh,dim,n_inst,pad", [(2, 128, 1, 0), (3, 64, 2, 64), (1, 256, 1, 0)])
def test_write_and_read(ty, dtype, kvh, dim, n_inst, pad):
    rng, c, ids, inst, lens, new, starts = setup(ty, kvh, dim, RAGGED, n_inst, 7 + ty * 16 + dim, pad)
    n = starts[-1]
    say("kv write type %d dtype %d heads %d dim %d" % (ty, dtype, kvh, dim))
    kval, kbits = rows(rng, n, kvh, dim, dtype, True)
    vval, vbits = rows(rng, n, kvh, dim, dtype, True)
    kv = c.device()
    want = c.read_back()
    seqs = api.make_seqs(dev32(ids), dev32(lens), q_start=dev32(starts), inst=dev32(inst) if n_inst > 1 else None)
    # the rows lie in a wider fused row
    fused = torch.zeros((n, 3 * kvh * dim), dtype=DT[dtype], device="cuda")
    kt, vt = fused[:, kvh * dim:2 * kvh * dim].view(n, kvh, dim), fused[:, 2 * kvh * dim:].view(n, kvh, dim)
    kt.copy_(torch.as_tensor(kbits).view(DT[dtype]))
    vt.copy_(torch.as_tensor(vbits).view(DT[dtype]))
    api.sae_kv_write(kv, seqs, kt, vt)
    torch.cuda.synchronize()
    at = positions(c, ids, inst, lens, new)
    for which, (val, bits) in enumerate(((kval, kbits), (vval, vbits))):
        page, sc = want[which]
        if ty == O.FP8:
            b, s = O.quantise(val)
            sc[at[:, 0], :, at[:, 1]] = s
            bits = b
        page[at[:, 0], :, at[:, 1]] = bits
    for which, (got, want_) in enumerate(zip(c.read_back(), want)):
        nan = (want_[0] & 0x7F) == 0x7F if ty == O.FP8 else np.zeros(want_[0].shape, bool)
        assert np.array_equal(np.where(nan, 0, got[0]), np.where(nan, 0, want_[0])), "array %d" % which
        assert np.all((got[0][nan] & 0x7F) == 0x7F)
        if ty == O.FP8:
            assert np.array_equal(got[1], want_[1]), "scales %d" % which
    # and back
    ko = torch.full((n, kvh, dim), 3.0, dtype=DT[dtype], device="cuda")
    vo = torch.full_like(ko, 5.0)
    api.sae_kv_read(kv, seqs, ko, vo)
    torch.cuda.synchronize()
    for t, val in ((ko, kval), (vo, vval)):
        if ty == O.FP8:
            val = O.dequantise(*O.quantise(val))
            if dtype == O.F16:
                val = np.clip(val, -65504, 65504)
            val, _ = to16(val, dtype)
        assert np.array_equal(t.double().cpu().numpy(), val, equal_nan=True)
    assert int(c.status[0]) == 0


@pytest.mark.parametrize("ty", [O.BF16, O.FP8])
def test_one_token_each(ty):
    """A decode step's write (no q_start), padding rows, a hole, ids and instances out of range, a length past the table."""
    rng = np.random.default_rng(3)
    kvh, dim = 2, 128
    lens = np.array([1, 16, 17, 0, 33, 40, 8, 9])
    ids, _, bpi, _ = tables(lens, 1, rng, width=4)
    c = Cache(ty, 2, bpi, kvh, dim, rng)
    inst = np.array([0, 0, 1, 0, 0, 1, 7, 0], np.int32)  # sequence 6: no such instance
    ids[4, 2] = -1      # sequence 4: no block for its last token
    ids[5, 2] = bpi     # sequence 5: id out of range
    given = lens.copy()
    given[7] = 4 * 16 + 9  # cut to the table's 64 tokens: its last block is -1
    kv = c.device()
    want = c.read_back()
    n = len(lens)
    kval, kbits = rows(rng, n, kvh, dim, O.BF16)
    vval, vbits = rows(rng, n, kvh, dim, O.BF16)
    seqs = api.make_seqs(dev32(ids), dev32(given), inst=dev32(inst))
    t = [torch.as_tensor(b).view(torch.bfloat16).cuda() for b in (kbits, vbits)]
    api.sae_kv_write(kv, seqs, *t)
    out = [torch.full_like(x, 9.0) for x in t]
    api.sae_kv_read(kv, seqs, *out)
    torch.cuda.synchronize()
    stored = [0, 1, 2]
    for which, (val, bits) in enumerate(((kval, kbits), (vval, vbits))):
        b, s = O.quantise(val) if ty == O.FP8 else (bits, None)
        for r in stored:
            blk, tok = inst[r] * bpi + ids[r, (lens[r] - 1) // 16], (lens[r] - 1) % 16
            want[which][0][blk, :, tok] = b[r]
            if s is not None:
                want[which][1][blk, :, tok] = s[r]
        back = O.dequantise(b, s) if s is not None else val
        back = np.where(np.isin(np.arange(n), stored)[:, None, None], back, 0.0)
        assert np.array_equal(out[which].double().cpu().numpy(), back)
    for got, w in zip(c.read_back(), want):
        assert np.array_equal(got[0], w[0])
        assert w[1] is None or np.array_equal(got[1], w[1])
    assert api.status_names(int(c.status[0])) == ["BAD_BLOCK"]


def test_more_new_tokens_than_positions():
    """Rows whose position would be negative are not written and read as zeros."""
    rng = np.random.default_rng(4)
    kvh, dim = 1, 64
    lens, new = np.array([5, 20]), np.array([40, 25])
    ids, inst, bpi, _ = tables(lens, 1, rng)
    c = Cache(O.F16, 1, bpi, kvh, dim, rng)
    kv = c.device()
    starts = np.array([0, 40, 65])
    val, bits = rows(rng, 65, kvh, dim, O.F16)
    t = torch.as_tensor(bits).view(torch.float16).cuda()
    seqs = api.make_seqs(dev32(ids), dev32(lens), q_start=dev32(starts))
    api.sae_kv_write(kv, seqs, t, t)
    k, v = torch.full_like(t, 2.0), torch.full_like(t, 2.0)
    api.sae_kv_read(kv, seqs, k, v)
    torch.cuda.synchronize()
    want = val.copy()
    want[:35] = 0
    want[40:45] = 0
    assert np.array_equal(k.double().cpu().numpy(), want)
    assert np.array_equal(v.double().cpu().numpy(), want)


def test_every_e4m3_value_and_tie():
    """Quantisation at every e4m3 value, every midpoint between two and their neighbours in bf16 and f16."""
    t = O.e4m3_table()[:127]
    mid = (t[1:] + t[:-1]) / 2
    for dtype, step in ((O.BF16, 2.0 ** -8), (O.F16, 2.0 ** -11)):
        x = np.concatenate([t, mid, mid * (1 + step), mid * (1 - step)])
        x = np.concatenate([x, -x])
        x = np.resize(x, (-(-x.size // 127), 127))
        x = np.concatenate([np.full((len(x), 1), 448.0), x], 1)  # a scale of 1
        val, bits = to16(x[:, None], dtype)
        n = len(x)
        rng = np.random.default_rng(5)
        ids, inst, bpi, _ = tables([n], 1, rng)
        c = Cache(O.FP8, 1, bpi, 1, 128, rng)
        seqs = api.make_seqs(dev32(ids), dev32([n]), q_start=dev32([0, n]))
        rt = torch.as_tensor(bits).view(DT[dtype]).cuda()
        kv = c.device()
        api.sae_kv_write(kv, seqs, rt, rt)
        ko, vo = torch.empty_like(rt), torch.empty_like(rt)
        api.sae_kv_read(kv, seqs, ko, vo)
        torch.cuda.synchronize()
        b, s = O.quantise(val)
        assert np.all(s == 127)
        want, _ = to16(O.dequantise(b, s), dtype)
        assert np.array_equal(ko.double().cpu().numpy(), want)
        assert np.array_equal(vo.double().cpu().numpy(), want)


@pytest.mark.parametrize("n_seq", [1, 63, 64, 65, 200, 4097])
def test_many_sequences(n_seq):
    """The search for a tile's sequence: many sequences, most of them without new tokens."""
    rng = np.random.default_rng(n_seq)
    new = np.where(rng.random(n_seq) < 0.3, rng.integers(1, 40, n_seq), 0)
    new[-1] = 3
    lens = new + rng.integers(0, 20, n_seq)
    ids, inst, bpi, _ = tables(lens, 1, rng)
    c = Cache(O.BF16, 1, bpi, 1, 64, rng)
    starts = np.concatenate([[0], np.cumsum(new)])
    val, bits = rows(rng, starts[-1], 1, 64, O.BF16)
    t = torch.as_tensor(bits).view(torch.bfloat16).cuda()
    kv = c.device()
    seqs = api.make_seqs(dev32(ids), dev32(lens), q_start=dev32(starts))
    api.sae_kv_write(kv, seqs, t, t)
    k, v = torch.zeros_like(t), torch.zeros_like(t)
    api.sae_kv_read(kv, seqs, k, v)
    torch.cuda.synchronize()
    at = positions(c, ids, inst, lens, new)
    page = c.read_back()[0][0]
    assert np.array_equal(page[at[:, 0], :, at[:, 1]], bits)
    assert np.array_equal(k.double().cpu().numpy(), val)
    assert np.array_equal(v.double().cpu().numpy(), val)


def test_offsets_past_32_bits():
    """A cache of more than 2^32 bytes and 2^31 values in each array: blocks at its far end."""
    kvh, dim, bpi = 8, 128, 140000  # 2.3e9 values
    k = torch.empty(bpi * kvh * 16 * dim, dtype=torch.bfloat16, device="cuda")
    v = torch.empty_like(k)
    kv = api.make_kv(api.KV_BF16, 1, bpi, kvh, dim, k, v)
    ids = np.array([[bpi - 1, 3, bpi - 2]], np.int32)
    n = 41
    rng = np.random.default_rng(6)
    kval, kb = to16(rng.standard_normal((n, kvh, dim)), O.BF16)
    vval, vb = to16(rng.standard_normal((n, kvh, dim)), O.BF16)
    kt, vt = (torch.as_tensor(b).view(torch.bfloat16).cuda() for b in (kb, vb))
    seqs = api.make_seqs(dev32(ids), dev32([n]), q_start=dev32([0, n]))
    api.sae_kv_write(kv, seqs, kt, vt)
    ko, vo = torch.zeros_like(kt), torch.zeros_like(vt)
    api.sae_kv_read(kv, seqs, ko, vo)
    last = k.view(bpi, -1)[bpi - 1].view(torch.int16).cpu().numpy().reshape(kvh, -1)
    assert np.array_equal(from16(O.unpack(last, dim, 2, 0), O.BF16), kval[:16].transpose(1, 0, 2))
    assert torch.equal(ko, kt) and torch.equal(vo, vt)
    # attention of a last token over the same blocks
    q = torch.as_tensor(to16(rng.standard_normal((1, 2 * kvh, dim)), O.BF16)[1]).view(torch.bfloat16).cuda()
    one = api.make_seqs(dev32(ids), dev32([n]))
    out = torch.zeros_like(q)
    work = torch.empty(api.sae_attn_work_size(kv, one, 1, 2 * kvh), dtype=torch.uint8, device="cuda")
    api.sae_attn_decode(kv, one, q, out, 0.1, work)
    o, l, mag, big = O.attention(q.double().cpu().numpy(), np.array([n - 1]), kval, vval, np.ones(n, bool), 0.1, 0)
    tol, _ = O.bounds(o, l, mag, big, dim, O.BF16)
    assert np.all(np.abs(out.double().cpu().numpy() - o) <= tol)
    out2 = torch.zeros_like(q)
    api.sae_attn_prefill(kv, api.make_seqs(dev32(ids), dev32([n]), q_start=dev32([0, 1])), q, out2, 0.1, work)
    assert np.all(np.abs(out2.double().cpu().numpy() - o) <= tol)
