"""One workspace, made for a batch, serves the sampling calls of fewer rows that a server makes as the batch drains."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

from oracle import sampling as S  # noqa: E402
from paper_2605_18825_amd import api  # noqa: E402
from test_gpu_sample import logits  # noqa: E402


@pytest.mark.parametrize("most", [65, 130])
def test_a_batch_that_drains(most):
    vocab = 65537
    x, u = logits(4, vocab, "bf16", seed=41)
    xd, ud = x.repeat((most + 3) // 4, 1)[:most].cuda(), torch.as_tensor(np.tile(u, (most + 3) // 4)[:most]).float().cuda()
    p = torch.full((most,), 0.9, device="cuda")
    work = torch.full((api.sae_sample_work_size(most, vocab),), 0xFF, dtype=torch.uint8, device="cuda")
    want = [S.sample(x[r].double().numpy(), float(ud[r]), top_p=float(p[0]))[0] for r in range(4)]
    for n in (most, 64, 63, 5, 1, most):
        token = torch.full((n,), -7, dtype=torch.int32, device="cuda")
        api.sae_sample(xd[:n], ud[:n], token, work, top_p=p[:n])
        torch.cuda.synchronize()
        assert token.tolist() == [want[r % 4] for r in range(n)]
