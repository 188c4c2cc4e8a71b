"""The adjoint of the gated delta rule over few chunks of 64 steps: the waves that work a chunk ahead of the others end a chunk before them and write nothing
behind their last one.  Against the oracle with the tolerances of test_gpu_delta.py, and bit by bit over many equal calls."""
import pytest
import torch

from gpu_util import require_gpu
from test_gpu_delta import BF16, F32, check, make, run

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("T, parts", [(1, 1), (64, 1), (65, 1), (70, 7), (129, 2), (200, 1)])
def test_adjoint_of_few_chunks(T, parts, dtype):
    require_gpu()
    x = make(3, T, 4, 2, 48, 40, dtype, T)
    lengths = torch.tensor([T, 0, (T + 1) // 2], dtype=torch.int32)
    want = check(x, lengths, parts)
    for _ in range(8):
        got = run(x, lengths, parts, 0.3)
        assert all(torch.equal(got[n], want[n]) for n in want)


@pytest.mark.parametrize("heads", [3, 300])  # one tile of columns to a workgroup, and two
def test_adjoint_of_one_chunk_of_many_keys(heads):
    require_gpu()
    for dtype in (F32, BF16):
        x = make(1, 40, heads, heads, 100, 24, dtype, heads)
        want = check(x, None, 1)
        for _ in range(4):
            got = run(x, None, 1, 0.3)
            assert all(torch.equal(got[n], want[n]) for n in want)


@pytest.mark.parametrize("T, parts", [(700, 2), (1100, 3)])
def test_many_chunks_within_the_limit_of_chunks_of_64(T, parts):
    """In fp32, by the argument of test_gpu_delta.py for the chunks of 64 steps that the kernels have: 48 u for a chunk and one more, 48 u (1 + T / 64), of which its limit for
    chunks of 32 is up to twice as much."""
    require_gpu()
    x = make(2, T, 4, 2, 64, 48, F32, T)
    check(x, torch.tensor([T, T - 70], dtype=torch.int32), parts, factor=(1 + T / 64) / (1 + T / 32))
