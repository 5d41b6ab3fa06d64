"""pq_chunk_attention where one sequence is far longer than the others: cut into more parts than the mean asks for."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from chunks import Cache      # noqa: E402
from test_gpu_chunk_attention import _check      # noqa: E402


@pytest.mark.parametrize("kv_heads,lens,new", [(8, [20000] + [100] * 60, [1] * 61), (8, [90] * 30 + [16001] + [128] * 27, [2] * 58), (32, [9000] + [130] * 12, [3] * 13)])
@pytest.mark.parametrize("v_bits", [16, 4])
def test_one_long_sequence_among_short_ones(kv_heads, lens, new, v_bits):
    _check(Cache(lens, kv_heads, v_bits=v_bits), new, 4)
