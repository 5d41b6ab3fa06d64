"""Batches of single tokens and long chunks, in one call and in two."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from chunks import DEV, Cache, tolerance      # noqa: E402
from test_gpu_chunk_attention import _attend, _ints, _queries      # noqa: E402


@pytest.mark.parametrize("lens,new", [([400] * 20 + [900], [1] * 20 + [300]), ([300] * 70 + [500, 700], [1] * 70 + [200, 0]), ([130, 5, 1000], [1, 1, 1000])])
@pytest.mark.parametrize("v_bits,window", [(16, 0), (4, 0), (16, 150)])
def test_single_tokens_first_and_the_chunks_in_a_call_of_their_own(lens, new, v_bits, window):
    c = Cache(lens, 2, v_bits=v_bits)
    pq, a = c.pq, new.count(1)
    starts = np.concatenate([[0], np.cumsum(new)])
    q = _queries(int(starts[-1]), 8, 5)
    whole = _attend(c, q, starts, window, 4)
    out, at = torch.full_like(q, float("nan")), _ints(starts)

    def call(sequences, rows):
        n = len(lens[sequences])
        ws = torch.empty(pq.pq_chunk_workspace_bytes(c.layout, n, 8, len(q[rows]), c.max_seq_len), dtype=torch.uint8, device=DEV)
        first = at[sequences.start or 0:(sequences.stop or len(lens)) + 1]
        pq.pq_chunk_attention(c.layout, q[rows], first, c.codes, c.params, c.v_pool, c.block_table[sequences], c.seq_lens[sequences], c.max_seq_len, float(c.sm_scale),
                              out[rows], ws, c.residual[sequences], v_bits, c.v_params, window, 4)

    call(slice(None, a), slice(None, a))
    assert torch.isnan(out[a:]).all()
    call(slice(a, None), slice(None))
    torch.cuda.synchronize()
    for s, n in enumerate(new):
        rows = slice(int(starts[s]), int(starts[s + 1]))
        want, spread, slope = c.rows(s, q[rows], torch.arange(c.lens[s] - n, c.lens[s], device=DEV), window, 4)
        for got in (out, whole):
            assert ((got[rows].double() - want).abs() <= tolerance(want, spread, slope)).all(), s
