"""pq_window_attention against float64 attention over the tokens that the window and the sinks leave."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from chunks import D, DEV, Cache      # noqa: E402


def _queries(seqs, heads, seed, dtype=torch.float16):
    return torch.from_numpy(np.random.default_rng(seed).standard_normal((seqs, heads, D))).to(DEV).to(dtype)


def _attend(c, q, window, sinks, max_seq_len=None):
    pq = c.pq
    max_seq_len = max_seq_len or c.max_seq_len
    out = torch.full(q.shape, float("nan"), device=DEV)
    size = pq.pq_window_workspace_bytes(c.layout, *q.shape[:2], max_seq_len, window, sinks)
    guarded = torch.full((size + 4096,), 0x5A, dtype=torch.uint8, device=DEV)
    pq.pq_window_attention(c.layout, q, c.codes, c.params, c.v_pool, c.block_table, c.seq_lens, max_seq_len, window, sinks, float(c.sm_scale), out,
                           guarded[:size], c.residual, c.v_bits, c.v_params)
    torch.cuda.synchronize()
    assert bool((guarded[size:] == 0x5A).all()), "written past the workspace"
    return out


def _check(c, group, window, sinks, dtype=torch.float16, **more):
    """Bars of test_gpu_attention_precision.py's kernels: fp32 arithmetic's own error with fp16 values (1e-6 of the sequence's
    output), 2.4e-5 with quantized ones, whose two sums cancel."""
    q = _queries(len(c.lens), c.heads * group, 3, dtype)
    got = _attend(c, q, window, sinks, **more)
    for s, L in enumerate(c.lens):
        if L == 0:
            assert not got[s].any()
            continue
        want = c.rows(s, q[s:s + 1], [L - 1], window, sinks)[0][0]
        off = float((got[s].double() - want).norm() / want.norm())
        assert off <= (1e-6 if c.v_bits == 16 else 2.4e-5), (s, L, off)
    return got


WINDOWS = [(1, 0), (1, 1), (7, 3), (100, 4), (128, 0), (129, 128), (200, 130), (384, 4), (1000, 0), (2500, 4), (600, 900), (5000, 5000)]


@pytest.mark.parametrize("window,sinks", WINDOWS)
@pytest.mark.parametrize("v_bits", [16, 4])
def test_windows(window, sinks, v_bits):
    _check(Cache([3000, 1, 128, 129, 0, 700, 385], 2, v_bits=v_bits), 4, window, sinks)


@pytest.mark.parametrize("window,sinks", [(100, 4), (300, 130)])
@pytest.mark.parametrize("bits,grouped", [((4, 4), False), ((3, 3), False), ((5, 3), False), ((3, 5), False), ((4, 2), False), ((2, 4), False),
                                          ((4, 4), True), ((3, 3), True), ((5, 3), True), ((3, 5), True), ((4, 2), True), ((2, 4), True)])
@pytest.mark.parametrize("v_bits", [16, 4, 2])
def test_every_format(bits, grouped, v_bits, window, sinks):
    _check(Cache([900, 515, 60], 2, bits, grouped, v_bits), 4, window, sinks)


@pytest.mark.parametrize("group", [1, 2, 3, 7, 8, 12, 16])
@pytest.mark.parametrize("dtype", [torch.float16, torch.float32])
@pytest.mark.parametrize("grouped", [False, True])
def test_groups_and_types(group, dtype, grouped):
    _check(Cache([900, 515], 2, grouped=grouped), group, 300, 4, dtype)


@pytest.mark.parametrize("tail", [True, False])
@pytest.mark.parametrize("kv_heads,lens,window", [(8, [2000] * 40, 1024), (8, [9000], 4096), (1, [20000], 9000), (8, [5000, 300, 40, 7000] * 8, 2001), (2, [300] * 200, 130)])
def test_launches(kv_heads, lens, window, tail):
    _check(Cache(lens, kv_heads, tail=tail), 4, window, 4)


@pytest.mark.parametrize("v_bits", [16, 2])
def test_pages_between_sinks_and_window_may_be_anything(v_bits):
    c = Cache([2000, 1500], 2, v_bits=v_bits)
    want = _check(c, 4, 200, 4)
    for entry in (-1, 10 ** 9, c.codes.shape[0]):
        c.block_table[0, 1:14] = entry
        c.block_table[1, 1:10] = entry
        assert torch.equal(_check(c, 4, 200, 4), want)


def test_a_window_over_everything_is_decode_attention():
    c = Cache([777, 128, 3000], 2)
    pq = c.pq
    q = _queries(3, 8, 5)
    out = torch.empty((3, 8, D), device=DEV)
    ws = torch.empty(pq.pq_decode_workspace_bytes(c.layout, 3, 8, c.max_seq_len), dtype=torch.uint8, device=DEV)
    pq.pq_decode_attention(c.layout, q, c.codes, c.params, c.v_pool, c.block_table, c.seq_lens, c.max_seq_len, float(c.sm_scale), out, ws, None, c.residual)
    for window, sinks in ((3000, 0), (10 ** 9, 10 ** 9), (1500, 1500)):
        got = _attend(c, q, window, sinks)
        assert float((got - out).norm() / out.norm()) <= 2e-6


def test_a_captured_call_is_replayed():
    c = Cache([3000, 900, 50], 2)
    pq = c.pq
    q, out = _queries(3, 8, 6), torch.zeros((3, 8, D), device=DEV)
    ws = torch.empty(pq.pq_window_workspace_bytes(c.layout, 3, 8, c.max_seq_len, 1200, 4), dtype=torch.uint8, device=DEV)

    def call():
        pq.pq_window_attention(c.layout, q, c.codes, c.params, c.v_pool, c.block_table, c.seq_lens, c.max_seq_len, 1200, 4, float(c.sm_scale), out, ws, c.residual)

    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for turn in range(4):
        q.copy_(_queries(3, 8, 30 + turn))
        c.seq_lens.copy_(torch.tensor([3000 - turn, 900 - 100 * turn, turn], dtype=torch.int32))
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        replayed = out.clone()
        call()
        torch.cuda.synchronize()
        # bit for bit: the residual's rows behind the sequences' ends are NaN, and some of these lengths read them
        assert torch.equal(out.view(torch.int32), replayed.view(torch.int32))
