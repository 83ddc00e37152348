"""sae_attn_tree where the tiles alone fill the GPU and a few sequences are so much longer that their keys are split all the
same: numbers of parts and of split tiles that count those alone.  The division is computed here too, from the rule, so that a
case which would split nothing fails."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

from oracle import kvcache as O  # noqa: E402
from tree_cases import TreeCall  # noqa: E402


def divided(c):
    """(row tiles times heads, workgroups wanted, parts of each sequence's tiles) of a call."""
    keys, groups = (32, 256) if c.dim == 256 else (64, 512)
    G = c.heads // c.kvh
    per_head = max(groups // c.kvh, 1)
    tiles = -(-c.counts * G // 128)
    seen = np.minimum(c.lens, c.window + c.counts) if c.window else c.lens
    steps = seen // keys + 1
    share = max(int((tiles * steps).sum() / per_head) + 1, 192 // keys)
    return (c.n * G // 128 + len(c.lens)) * c.kvh, groups, np.maximum((steps + share // 2) // share, 1)


def check(c, least):
    tiles, groups, parts = divided(c)
    assert tiles > groups and (parts > 1).sum() >= least and len(c.lens) <= 512, (tiles, groups, parts)
    c.check()


@pytest.mark.parametrize("ty", [O.BF16, O.F16, O.FP8])
def test_twelve_heads_of_64(ty):
    rng = np.random.default_rng(1)
    lens, new = rng.integers(20, 100, 46), rng.integers(1, 12, 46)
    lens[[0, 13, 14, 45]] = [2500, 3001, 1600, 4000]
    new[[13, 20]] = [64, 0]
    check(TreeCall(ty, 12, 12, 64, lens, new, seed=70), 4)


@pytest.mark.parametrize("ty,dim", [(O.BF16, 64), (O.FP8, 64), (O.F16, 128), (O.FP8, 128), (O.BF16, 256), (O.FP8, 256)])
def test_hundreds_of_sequences(ty, dim):
    """Two sequences a thread: long ones first, last and both of one thread's."""
    rng = np.random.default_rng(2)
    lens, new = rng.integers(10, 80, 300), rng.integers(1, 6, 300)
    long = [0, 18, 19, 77, 299]
    lens[long] = [2000, 2400, 1603, 3000, 2517]
    new[[18, 77]] = [40, 3]
    check(TreeCall(ty, 4, 2, dim, lens, new, seed=71), len(long))


@pytest.mark.parametrize("ty,dim", [(O.BF16, 128), (O.F16, 64)])
def test_windows_and_more_rows_than_a_tile(ty, dim):
    rng = np.random.default_rng(3)
    lens, new = rng.integers(20, 100, 280), rng.integers(1, 5, 280)
    lens[[0, 140, 279]] = [1500, 2500, 3500]
    new[[0, 140, 279]] = [150, 33, 200]
    check(TreeCall(ty, 4, 2, dim, lens, new, seed=72, window=1500, n_inst=2), 3)
