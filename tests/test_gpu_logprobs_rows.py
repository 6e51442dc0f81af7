"""Log probabilities of many rows without alternatives: pieces of 8192 entries joined by one
wave a row, as a prompt is scored. Against the fp64 definition within the bound of
test_gpu_logprobs."""
import numpy as np
import pytest
import torch

from test_gpu_logprobs import _check, _z

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("top", [0, 20])
@pytest.mark.parametrize("rows,V", [(190, 16500), (513, 8192), (257, 8193), (35, 131073)])
def test_many_rows(gpu_lib, top, rows, V):
    """At least 512 pieces of 8192 entries, the last of them whole, short, or of one entry."""
    z = _z((1, rows, V), rows)
    z[0, 3, ::2] = -float("inf")
    z[0, 4] = -float("inf")
    z[0, 5, V - 1] = float("nan")
    z[0, 6, 8191] = float("inf")
    z[0, 7] = torch.round(z[0, 7])
    y = np.random.default_rng(rows).integers(0, V, (1, rows))
    y[0, 8], y[0, 9], y[0, 10] = -1, V, V - 1
    _check(gpu_lib, z, y, top, T=0.8)


@pytest.mark.parametrize("top", [0, 3])
def test_many_ragged_rows(gpu_lib, top):
    """As many pieces, some sequences without rows."""
    z = _z((24, 11, 20000), top)
    y = np.random.default_rng(top).integers(0, 20000, (24, 11))
    n = [(5 * i) % 12 for i in range(24)]
    _check(gpu_lib, z, y, top, n=n, before=8.0)
