"""The attention's weights over their whole range: keys far below a row's largest score that together make up its output,
and the error that the weights' rounding may leave."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

from attn_cases import Call  # noqa: E402
from oracle import kvcache as O  # noqa: E402

TYPES = [O.BF16, O.F16, O.FP8]
# Half the smallest step of a weight in units of a row's largest one: f16 has steps of 2^-24; decode takes weights as two
# numbers, the largest 2^15, prefill as one, the largest 2^12 or more.  bf16 and FP8 caches: none.
HALF_STEP = {True: 2.0 ** -(25 + 15), False: 2.0 ** -(25 + 12)}
# what rounding a weight leaves, relative: decode takes the rest along as a second number
TWO = {t: O.ROUNDOFF[O.BF16 if t == O.FP8 else t] ** 2 for t in TYPES}


def sink(nats, scale):
    """Position 0 of every sequence has a score `nats` above all others and a value of zero."""
    def fill(c, ids, q):
        dim = c.dim
        q[:] = 1.0
        c.values[0] *= 0.1  # scores of 0.1 dim^-0.5 scale q: all others are close together
        c.values[1] = 1.0 + 0.25 * c.values[1]
        for r in range(len(ids)):
            c.values[0][ids[r, 0], :, 0] = nats / (dim * scale)
            c.values[1][ids[r, 0], :, 0] = 0.0
    return fill


def check(ty, heads, kvh, dim, lens, nats, new=None, **kw):
    scale = dim ** -0.5
    c = Call(ty, heads, kvh, dim, lens, new=new, fill=sink(nats, scale), **kw)
    decode = new is None
    floor = max(lens) * HALF_STEP[decode] * float(np.nanmax(np.abs(c.cache.values[1]))) if ty == O.F16 else 0.0
    c.check(decode, weight=TWO[ty] if decode else None, floor=floor)


@pytest.mark.parametrize("ty", TYPES)
@pytest.mark.parametrize("n,nats", [(700, 17.0), (20000, 13.0), (32768, 16.0), (131072, 18.0)])
def test_decode_sink(ty, n, nats):
    """One workgroup a sequence, and split and joined."""
    check(ty, 2, 1, 64, [n], nats, seed=1)


@pytest.mark.parametrize("ty", TYPES)
@pytest.mark.parametrize("n,nats", [(500, 17.0), (20000, 13.0), (32768, 16.0), (131072, 18.0)])
def test_prefill_sink(ty, n, nats):
    """A short table, not split, and long ones, split and joined."""
    check(ty, 2, 1, 64, [n], nats, new=[3], seed=2)


@pytest.mark.parametrize("ty", TYPES)
def test_prefill_sink_not_split(ty):
    """So many tiles that none is split, over long tables; heads of 256."""
    lens = np.full(260, 1300) + np.arange(260) % 37
    check(ty, 4, 2, 128, lens, 17.0, new=np.ones(260, int), seed=3, shared=900)
    check(ty, 2, 1, 256, [400, 90], 17.0, new=[70, 3], seed=4)
    check(ty, 2, 1, 256, [3300], 15.0, new=[5], seed=5)


@pytest.mark.parametrize("ty", TYPES)
@pytest.mark.parametrize("heads,kvh,dim", [(8, 2, 128), (3, 1, 64), (6, 2, 256)])
def test_decode_rounds_once(ty, heads, kvh, dim):
    """Decode's weights are two 16-bit numbers: what their rounding leaves is far below the output's own."""
    lens = [1, 17, 300, 700, 5000]
    floor = 5000 * HALF_STEP[True] * 6 if ty == O.F16 else 0.0
    Call(ty, heads, kvh, dim, lens, seed=6).check(True, weight=TWO[ty], floor=floor)
    Call(ty, heads, kvh, dim, lens[:4], seed=7).check(True, weight=TWO[ty], floor=floor)


@pytest.mark.parametrize("ty", TYPES)
@pytest.mark.parametrize("size", [1e4, 3e5, 5e6])
def test_scores_of_any_size(ty, size):
    """Scores so large that fp32 holds them to whole numbers or not even that: a row's weight is on its largest, and
    nothing overflows on the way."""
    def fill(c, ids, q):
        q *= size ** 0.5
        c.values[0] *= size ** 0.5
    for dim in (64, 128):
        Call(ty, 4, 2, dim, [1, 40, 300, 2100], seed=8, fill=fill).check(True)
        Call(ty, 4, 2, dim, [1, 40, 300, 2100], new=[1, 40, 90, 6], seed=9, fill=fill).check(False)


@pytest.mark.parametrize("dim", [64, 128, 256])
def test_means_of_f16s_largest_value(dim):
    """Values of f16's largest, as clamped ones are: no mean of them is larger, whatever the weights' rounding.  Each
    sequence has one key of all the weight, and a later one with a little more: a weight that f16 does not hold."""
    rng = np.random.default_rng(10)
    lens = np.where(np.arange(150) % 3 == 0, 700, 130) + np.arange(150) % 5

    def fill(c, ids, q):
        q[:] = 1.0
        c.values[1] = np.where(c.values[1] < -1.5, -65504.0, 65504.0)
        c.values[1][..., ::3] = 65504.0
        c.values[0][:] = -300.0 / dim ** 0.5
        for r in range(len(ids)):
            for t, bits in ((7, 0.0), (101, 3.8 * rng.random())):
                c.values[0][ids[r, t // 16], :, t % 16] = np.log(2.0) * bits / dim ** 0.5
    Call(O.F16, 4, 2, dim, lens, new=np.full(150, 2), seed=11, fill=fill).check(False)
    Call(O.F16, 4, 2, dim, lens[:9], new=np.full(9, 20), seed=12, fill=fill).check(False)
    Call(O.F16, 4, 2, dim, lens, seed=13, fill=fill).check(True)


@pytest.mark.parametrize("ty", TYPES)
@pytest.mark.parametrize("size", [2e8, 1e11, 1e15, 1e25])
def test_scores_past_fp32s_whole_numbers(ty, size):
    """Scores so large that fp32 holds them to hundreds or worse (f16: to tens, its values end there): what the running
    maximum is rounded by must not be an exponent."""
    def fill(c, ids, q):
        most = 60000.0 if ty == O.F16 else np.inf
        q *= size ** 0.5
        np.clip(q, -most, most, out=q)
        c.values[0] = np.clip(c.values[0] * size ** 0.5, -most, most)
    for dim in (64, 128, 256):
        for new, seed in (([1, 40, 90, 6], 14), (None, 15)):
            Call(ty, 4, 2, dim, [1, 40, 300, 2100], new=new, seed=seed, fill=fill).check(new is None)
            Call(ty, 4, 2, dim, [40, 300], new=new and [40, 90], seed=seed, fill=fill).check(new is None)
