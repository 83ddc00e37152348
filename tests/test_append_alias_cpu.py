"""sae_kv_append refuses a q_out that overlaps what the call reads, but for q itself with q's stride (checked on the host,
before any launch: no GPU needed)."""
import pytest

from test_kv_args_cpu import P, kv, lib  # noqa: F401
from test_step_args_cpu import append

ROW, KV_ROW, N = 512, 256, 5  # 4 heads and 2 key-value heads of 128, 5 rows
FAR = dict(a=P + (1 << 30), b=P + (1 << 31), sa=KV_ROW, sb=KV_ROW)  # keys and values elsewhere
WIDE = 2 * ROW + 2 * KV_ROW


@pytest.mark.parametrize("over", [
    # q itself with another stride
    dict(FAR, qo=P, qs=ROW, qos=2 * ROW), dict(FAR, qo=P, qs=2 * ROW, qos=ROW), dict(FAR, qo=P, qs=ROW, qos=ROW + 8),
    # rows of one stride that reach into each other
    dict(FAR, qo=P + 16), dict(FAR, qo=P - 16), dict(FAR, qo=P + 2 * ROW * (N - 1)), dict(FAR, qo=P - 2 * ROW * (N - 1)),
    dict(FAR, qo=P + 2 * ROW - 16, qs=2 * ROW, qos=2 * ROW), dict(FAR, qo=P + 2 * ROW + 16, qs=2 * ROW, qos=2 * ROW),
    # the last row of one among the others'
    dict(FAR, qo=P + 2 * (4 * 2 * ROW + ROW) - 16, qs=2 * ROW, qos=ROW),
    # keys and values
    dict(FAR, qo=P + (1 << 30)), dict(FAR, qo=P + (1 << 31) + 2 * KV_ROW * N - 16), dict(FAR, qo=P + (1 << 30) - 2 * ROW * N + 16),
    dict(qs=WIDE, qos=WIDE, sa=WIDE, sb=WIDE, qo=P + 2 * ROW, a=P + 4 * ROW - 16, b=P + 4 * ROW + 2 * KV_ROW),
    dict(qs=WIDE, qos=WIDE, sa=WIDE, sb=WIDE, qo=P + 2 * ROW, a=P + 4 * ROW, b=P + 2 * (ROW - KV_ROW) + 16),
    dict(n=1, qo=P + 16, a=P + (1 << 30), b=P + (1 << 31))])
def test_overlap(lib, over):  # noqa: F811
    assert append(lib, **over) == -1 and b"q_out must lie apart" in lib.sae_last_error(None), lib.sae_last_error(None)
