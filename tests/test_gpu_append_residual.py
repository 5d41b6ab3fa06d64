"""What pq_append_chunk leaves alone in the residual buffer: everything of a sequence without new tokens, rows behind the last token of the
others."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from chunks import G, pools      # noqa: E402
from test_gpu_append_chunk import _case, _ints      # noqa: E402


@pytest.mark.parametrize("before,new", [([200, 0, 127, 128, 60], [1, 0, 2, 129, 0]), ([5, 300], [0, 0]), ([0, 77, 0], [0, 0, 300]), ([250] * 70, [0] * 35 + [7] * 35)])
@pytest.mark.parametrize("dtype", [torch.float16, torch.float32])
def test_rows_without_new_tokens_are_left_as_they_were(before, new, dtype):
    pq, lay, table, pages, keys, values, residual, starts, slots = _case(before, new, 2, (4, 4), False, 16, dtype, 9, pad=3)
    codes, params, v_pool, v_params = pools(pages, (4, 4), 2, False, 16)
    got = residual.clone()
    pq.pq_append_chunk(lay, keys, values, _ints(starts), _ints(before), slots, got, _ints(table), codes, params, v_pool)
    torch.cuda.synchronize()
    for s, (b, n) in enumerate(zip(before, new)):
        rest = (b + n) % G
        assert torch.equal(got[s, :, rest:], residual[s, :, rest:]), s
        if n == 0:
            assert torch.equal(got[s], residual[s]), s
        else:
            written = min(rest, n)
            assert torch.equal(got[s, :, rest - written:rest], keys[starts[s + 1] - written:starts[s + 1]].half().permute(1, 0, 2)), s
