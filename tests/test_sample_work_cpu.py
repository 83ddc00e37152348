"""The workspace of a sampling call serves every smaller call (no GPU needed)."""
import ctypes

import pytest

from test_kv_args_cpu import lib  # noqa: F401
from test_step_args_cpu import sample

ROWS = [0, 1, 2, 33, 63, 64, 65, 66, 300, 5000, 1 << 20]
VOCAB = [1, 1000, 65535, 65536, 65537, 131072, 1 << 20]


def size(lib, rows, vocab):  # noqa: F811
    n = ctypes.c_size_t()
    assert lib.sae_sample_work_size(rows, vocab, ctypes.byref(n)) == 0
    return n.value


def test_sizes_do_not_fall(lib):  # noqa: F811
    for vocab in VOCAB:
        of = [size(lib, rows, vocab) for rows in ROWS]
        assert of == sorted(of), (vocab, of)
    for rows in ROWS:
        of = [size(lib, rows, vocab) for vocab in VOCAB]
        assert of == sorted(of), (rows, of)


@pytest.mark.parametrize("rows,vocab", [(1, 65536), (64, 131072), (300, 1000)])
def test_less_is_refused(lib, rows, vocab):  # noqa: F811
    need = size(lib, rows, vocab)
    assert sample(lib, n=rows, vocab=vocab, stride=vocab, work_bytes=need - 1) == -1 and b"work" in lib.sae_last_error(None)
