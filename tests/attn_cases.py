"""One attention call over a paged cache and its 64-bit expectation, for tests that choose their own tables, contents
and bounds."""
import numpy as np
import torch

from harness import say
from kv_cases import DT, Cache, dev32, oracle_attention, tables, to16
from oracle import kvcache as O
from paper_2605_18825_amd import api


class Call:
    """A decode (new is None) or prefill call.

    shared: 0, or a number of blocks that all sequences draw theirs from (a block may be in several tables; block 0 is
    the first of each); places that no sequence owns hold NaN otherwise.  holes: (sequence, page) without a block.
    fill(cache, ids, q): changes logical contents (c.values, which are packed anew, and q) before the upload."""

    def __init__(self, ty, heads, kvh, dim, lens, new=None, n_inst=1, window=0, seed=0, holes=(), width=0, shared=0,
                 scale=None, fill=None):
        rng = np.random.default_rng(seed)
        self.ty, self.heads, self.kvh, self.dim, self.window = ty, heads, kvh, dim, window
        self.dtype = O.BF16 if ty == O.FP8 else ty
        self.lens = np.asarray(lens)
        n_seq = len(self.lens)
        self.counts = np.ones(n_seq, int) if new is None else np.asarray(new)
        self.starts = np.concatenate([[0], np.cumsum(self.counts)])
        self.n = int(self.starts[-1])
        self.scale = dim ** -0.5 if scale is None else scale
        if shared:
            self.inst, bpi = (np.arange(n_seq) % n_inst).astype(np.int32), shared
            pages = -(-self.lens // O.BLOCK)
            self.ids = rng.integers(1, shared, (n_seq, max(1, width, int(pages.max())))).astype(np.int32)
            self.ids[:, 0] = 0
            self.ids[np.arange(self.ids.shape[1])[None] >= pages[:, None]] = -1
            owned = np.ones((n_inst * bpi, O.BLOCK), bool)
        else:
            self.ids, self.inst, bpi, owned = tables(self.lens, n_inst, rng, width=width)
        for r, j in holes:
            if not shared and self.ids[r, j] >= 0:
                owned[self.inst[r] * bpi + self.ids[r, j]] = False
            self.ids[r, j] = -1
        self.n_inst = n_inst
        self.cache = c = Cache(ty, n_inst, bpi, kvh, dim, rng)
        self.q = rng.standard_normal((self.n, heads, dim)) * 2
        if fill:
            fill(c, self.ids, self.q)
            for which in range(2):
                if ty == O.FP8:
                    b, s = O.quantise(c.values[which])
                    c.values[which], c.pages[which], c.scales[which] = O.dequantise(b, s), O.pack(b, 1, which), s
                else:
                    c.values[which], bits = to16(c.values[which], ty)
                    c.pages[which] = O.pack(bits, 2, which)
        c.poison(owned)
        self.q, self.qbits = to16(self.q, self.dtype)

    def run(self, decode):
        """The call's outputs and log-sum-exps."""
        say("attention type %d heads %d/%d dim %d seqs %d rows %d window %d longest %d %s" % (
            self.ty, self.heads, self.kvh, self.dim, len(self.lens), self.n, self.window, int(self.lens.max()),
            "decode" if decode else "prefill"))
        kv = self.cache.device()
        q = torch.as_tensor(self.qbits).view(DT[self.dtype]).cuda()
        out = torch.full_like(q, 7.0)
        lse = torch.full((self.n, self.heads), 7.0, dtype=torch.float32, device="cuda")
        seqs = api.make_seqs(dev32(self.ids), dev32(self.lens), q_start=None if decode else dev32(self.starts),
                             inst=dev32(self.inst) if self.n_inst > 1 else None)
        work = torch.full((api.sae_attn_work_size(kv, seqs, self.n, self.heads),), 0xFF, dtype=torch.uint8, device="cuda")
        (api.sae_attn_decode if decode else api.sae_attn_prefill)(kv, seqs, q, out, self.scale, work, window=self.window,
                                                                  lse=lse)
        torch.cuda.synchronize()
        assert int(self.cache.status[0]) == 0
        return out.double().cpu().numpy(), lse.double().cpu().numpy()

    def want(self):
        """out, lse, mag, big of the 64-bit definition."""
        return oracle_attention(self.cache, self.ids, self.inst, self.lens, self.starts, self.q, self.scale, self.window)

    def check(self, decode, weight=None, floor=0.0):
        """Runs the call and holds it to O.bounds; weight, floor: see there."""
        want, wl, mag, big = self.want()
        tol, tol_l = O.bounds(want, wl, mag, big, self.dim, self.dtype, weight=weight, floor=floor)
        got, gl = self.run(decode)
        bad = ~(np.abs(got - want) <= tol)
        assert not bad.any(), (np.argwhere(bad)[:5].tolist(), float(np.nanmax(np.abs(got - want) / tol)), int(bad.sum()))
        dead = np.isinf(wl)
        assert np.array_equal(gl[dead], wl[dead])
        assert np.all(np.abs(gl[~dead] - wl[~dead]) <= tol_l[~dead])
        say("  worst error %.2f of its bound" % float(np.max(np.abs(got - want) / tol)))
