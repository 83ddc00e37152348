"""Builds paged-cache test cases: logical values, packed device tensors, block tables."""
import numpy as np
import torch

from oracle import kvcache as O
from paper_2605_18825_amd import api

DT = {O.BF16: torch.bfloat16, O.F16: torch.float16}


def to16(x, dtype):
    """float64 array rounded to the 16-bit type: (float64 values, int16 bit patterns)."""
    t = torch.as_tensor(x).to(DT[dtype])
    return t.double().numpy(), t.view(torch.int16).numpy()


def from16(bits, dtype):
    return torch.as_tensor(np.ascontiguousarray(bits)).view(DT[dtype]).double().numpy()


class Cache:
    """A cache of n_inst x bpi blocks; places that no sequence owns hold NaN."""

    def __init__(self, ty, n_inst, bpi, kvh, dim, rng, pad_blocks=0, spread=1.0):
        self.ty, self.n_inst, self.bpi, self.kvh, self.dim = ty, n_inst, bpi, kvh, dim
        nb = n_inst * bpi
        shape = (nb, kvh, O.BLOCK, dim)
        self.values, self.pages, self.scales = [], [], []
        for which in range(2):
            x = rng.standard_normal(shape) * spread
            if ty == O.FP8:
                b, s = O.quantise(x)
                self.values.append(O.dequantise(b, s))
                self.pages.append(O.pack(b, 1, which))
                self.scales.append(s)
            else:
                val, bits = to16(x, ty)
                self.values.append(val)
                self.pages.append(O.pack(bits, 2, which))
        self.stride = 0
        self.pad = pad_blocks

    def poison(self, owned):
        """NaN in every (block, token) where owned [block][16] is false: keys, values and scale bytes."""
        size = 1 if self.ty == O.FP8 else 2
        for which in range(2):
            x = O.unpack(self.pages[which], self.dim, size, which)
            nan = 0x7F if size == 1 else {O.BF16: 0x7FC0, O.F16: 0x7E00}[self.ty]
            x[np.broadcast_to(~owned[:, None, :, None], x.shape)] = nan
            self.pages[which] = O.pack(x, size, which)
            self.values[which][np.broadcast_to(~owned[:, None, :, None], x.shape)] = np.nan
            if size == 1:
                self.scales[which] = np.where(owned[:, None, :], self.scales[which], 255).astype(np.uint8)

    def device(self):
        """The sae_kv over device tensors; pad_blocks: values between blocks, filled with NaN bytes."""
        nb = self.n_inst * self.bpi
        tensors = []
        for p in self.pages:
            p = p.reshape(nb, -1)
            if self.pad:
                p = np.concatenate([p, np.full((nb, self.pad), 0x7F if self.ty == O.FP8 else 0x7FFF, p.dtype)], 1)
                self.stride = p.shape[1]
            t = torch.as_tensor(np.ascontiguousarray(p)).cuda()
            tensors.append(t if self.ty == O.FP8 else t.view(DT[self.ty]))
        sc = [torch.as_tensor(s.reshape(nb, -1)).cuda() for s in self.scales] or [None, None]
        self.status = torch.zeros(1, dtype=torch.int32, device="cuda")
        self.kv = api.make_kv(self.ty, self.n_inst, self.bpi, self.kvh, self.dim, *tensors, *sc, status=self.status,
                              block_stride=self.stride)
        return self.kv

    def read_back(self):
        """Pages and scales now on the device, unpacked: (bytes or bits [block][head][16][dim], scales) per array."""
        size = 1 if self.ty == O.FP8 else 2
        nb = self.n_inst * self.bpi
        out = []
        for which, t in enumerate(self.kv.tensors[:2]):
            t = t if size == 1 else t.view(torch.int16)
            p = t.cpu().numpy().reshape(nb, -1)[:, :self.kvh * O.BLOCK * self.dim]
            s = self.kv.tensors[2 + which]
            out.append((O.unpack(p.reshape(nb, self.kvh, -1), self.dim, size, which),
                        None if s is None else s.cpu().numpy().reshape(nb, self.kvh, O.BLOCK)))
        return out


def tables(lens, n_inst, rng, extra=3, width=0):
    """Block tables of sequences of these lengths in random blocks: ids [n][width], inst [n], blocks per instance,
    owned [block][16]."""
    lens = np.asarray(lens)
    inst = np.arange(len(lens)) % n_inst
    blocks = -(-lens // O.BLOCK)
    bpi = max([int(blocks[inst == i].sum()) for i in range(n_inst)] + [0]) + extra
    ids = np.full((len(lens), max(1, width, int(blocks.max()) if len(lens) else 1)), -1, np.int32)
    owned = np.zeros((n_inst * bpi, O.BLOCK), bool)
    for i in range(n_inst):
        free = list(rng.permutation(bpi))
        for r in np.nonzero(inst == i)[0]:
            for j in range(blocks[r]):
                ids[r, j] = free.pop()
                owned[i * bpi + ids[r, j], :max(0, min(O.BLOCK, lens[r] - j * O.BLOCK))] = True
    return ids, inst.astype(np.int32), bpi, owned


def dev32(a):
    return torch.as_tensor(np.ascontiguousarray(a, np.int32)).cuda()


def oracle_attention(cache, ids, inst, lens, starts, q, scale, window):
    """Over all sequences; q [n][heads][dim] float64.  Returns out, lse, mag, big."""
    parts = []
    for r, total in enumerate(lens):
        a, b = starts[r], starts[r + 1]
        at = total - (b - a) + np.arange(b - a)
        lo, hi = inst[r] * cache.bpi, (inst[r] + 1) * cache.bpi
        k, there = O.rows_of(ids[r], total, cache.values[0][lo:hi])
        v, _ = O.rows_of(ids[r], total, cache.values[1][lo:hi])
        parts.append(O.attention(q[a:b], at, k, v, there, scale, window))
    return [np.concatenate(x) for x in zip(*parts)]
