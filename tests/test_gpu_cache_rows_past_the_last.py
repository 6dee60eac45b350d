"""seq_rows that name more rows than a call has: they are taken as at most T (and at least 0), by the append and by the attention alike, so that a token has one position in both.  Tolerances: those of
tests/test_gpu_cache_append.py and tests/test_gpu_cache_attention.py."""
import pytest
import torch

from test_gpu_cache_append import Append
from test_gpu_cache_attention import WIDE, Batch

pytestmark = pytest.mark.gpu

# (seq_rows as given, of a call of 12 rows)
ROWS = [[0, 5, 20], [0, 12, 13], [0, 14, 14], [3, 9, 2 ** 31 - 1], [-2, 5, 15], [0, 13, 2 ** 31 - 1]]


def taken(rows):
    return torch.tensor(rows, dtype=torch.int64).clamp(0, 12).int()


@pytest.mark.parametrize("rows", ROWS)
@pytest.mark.parametrize("cache", ["bf16", "fp8"])
def test_append(rows, cache):
    a = Append([100, 70], [5, 7], 2, 1, 64, 16, cache=cache, seed=41)
    a.seq_rows = torch.tensor(rows, dtype=torch.int32)
    got = a.run()
    a.seq_rows = taken(rows)
    a.check(got)


@pytest.mark.parametrize("rows", ROWS)
@pytest.mark.parametrize("heads", [(4, 2), WIDE])
@pytest.mark.parametrize("causal", [True, False])
def test_attention(rows, heads, causal):
    b = Batch([100, 70], [5, 7], *heads, 64, 16, seed=42)
    b.check(b.run(seq_rows=torch.tensor(rows, dtype=torch.int32), causal=causal), causal=causal, seq_rows=taken(rows))
