"""Rows of logits whose largest is +inf: the tokens that have it share the weight evenly whatever the temperature is."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

from test_gpu_sample import check, logits  # noqa: E402

HOT = [5.4e36, 1e38, 3.4e38, float("inf"), 1e30, 1.0, 1e-30, 1e-45]


# one workgroup a row of 256, 512 and 1,024 threads; several workgroups a row
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("vocab", [3, 5000, 12001, 20000, 70001])
def test_any_temperature(dtype, vocab):
    x, u = logits(8, vocab, dtype, seed=vocab)
    x[::2, vocab // 3] = x[:, vocab - 1] = float("inf")
    x[1, 0] = x[2, 0] = -3.3e38
    for more in ({}, dict(top_k=[1, 2, 3, 400, 0, 5, 30, 2]), dict(top_k=[700] * 8), dict(top_p=[0.3, 0.5, 0.9, 0.99] * 2),
                 dict(min_p=[0.1, 1.0, 0.5, 1e-6] * 2), dict(top_k=[50] * 8, top_p=[0.4, 0.9] * 4, min_p=[0.2] * 8)):
        token, prob, kept = check(x, u, temperature=HOT, **more)
        l = x.float().numpy()
        assert np.all(np.isposinf(l[np.arange(8), token]))
        assert np.all((prob == 1) | ((prob == 0.5) & (np.isposinf(l).sum(1) == 2)))
        if not more:
            assert np.all(kept == vocab)


def test_every_logit_infinite():
    x = torch.full((6, 9001), float("inf"))
    x[3:, 5::2] = -1e38
    u = [0.0, 0.37, 0.9999, 0.0, 0.37, 0.9999]
    check(x, u, temperature=[1e38, float("inf"), 1e-3] * 2)
    check(x, u, temperature=[1e38, float("inf"), 1e-3] * 2, top_p=[0.5] * 6)
