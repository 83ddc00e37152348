"""sae_attn_tree with a q_start that decreases (outside its contract): rows are counted several times, and the parts of split
tiles may lie past the grid.  Nothing is written outside the call's rows, whatever the workspace held."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

from harness import say  # noqa: E402
from kv_cases import DT, Cache, dev32  # noqa: E402
from oracle import kvcache as O  # noqa: E402
from paper_2605_18825_amd import api  # noqa: E402

ROWS, GUARD = 4096, 64
STARTS = [[0, ROWS] * 6 + [4000, ROWS], [0, ROWS, 3900] * 40 + [ROWS], [ROWS, 0, -5, ROWS + 9, 4090, ROWS] * 8, [ROWS, 0]]


@pytest.mark.parametrize("ty,dim,heads,kvh", [(O.F16, 64, 4, 4), (O.BF16, 64, 8, 2), (O.BF16, 128, 4, 4), (O.FP8, 128, 8, 8), (O.FP8, 256, 2, 2)])
@pytest.mark.parametrize("window", [0, 500])
def test_rows_outside_the_call_stay(ty, dim, heads, kvh, window):
    blocks, length = 250, 3900
    c = Cache(ty, 1, blocks, kvh, dim, np.random.default_rng(1))
    kv = c.device()
    rows = DT[O.BF16 if ty == O.FP8 else ty]
    q = torch.zeros((ROWS, heads, dim), dtype=rows, device="cuda")
    parent = torch.full((ROWS,), -1, dtype=torch.int32, device="cuda")
    for starts in STARTS:
        n = len(starts) - 1
        ids = np.tile(np.arange(blocks), (n, 1))
        seqs = api.make_seqs(dev32(ids), dev32([length] * n), q_start=dev32(starts))
        size = api.sae_attn_work_size(kv, seqs, ROWS, heads)
        out = torch.full((ROWS + 2 * GUARD, heads, dim), 7.0, dtype=rows, device="cuda")
        lse = torch.full((ROWS + 2 * GUARD, heads), 7.0, device="cuda")
        # a workspace that says everywhere: 32 rows behind the call's last, in two parts from place 0 on
        work = dev32([ROWS, 32 << 16, 0, 2]).repeat(size // 16)
        say("decreasing q_start: type %d dim %d heads %d/%d window %d, %d sequences" % (ty, dim, heads, kvh, window, n))
        api.sae_attn_tree(kv, seqs, parent, 256, q, out[GUARD:GUARD + ROWS], 0.1, work, window=window, lse=lse[GUARD:GUARD + ROWS])
        torch.cuda.synchronize()
        for t in (out, lse):
            assert torch.all(t[:GUARD] == 7.0) and torch.all(t[GUARD + ROWS:] == 7.0)
