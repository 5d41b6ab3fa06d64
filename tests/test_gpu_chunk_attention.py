"""pq_chunk_attention against float64 attention over the same cache."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from chunks import D, DEV, G, Cache, tolerance      # noqa: E402


def _ints(x):
    return torch.as_tensor(np.asarray(x), dtype=torch.int32).to(DEV)


def _queries(rows, heads, seed, scale=1.0):
    return torch.from_numpy(np.random.default_rng(seed).standard_normal((rows, heads, D)) * scale).to(DEV).half()


def _attend(c, q, starts, window=0, sinks=0, max_seq_len=None, sm_scale=None, seq_lens=None, fill=float("nan")):
    pq = c.pq
    max_seq_len = max_seq_len or c.max_seq_len
    out = torch.full_like(q, fill)
    size = pq.pq_chunk_workspace_bytes(c.layout, len(c.lens), q.shape[1], q.shape[0], max_seq_len)
    assert size >= 256
    guarded = torch.full((size + 4096,), 0x5A, dtype=torch.uint8, device=DEV)
    pq.pq_chunk_attention(c.layout, q, _ints(starts), c.codes, c.params, c.v_pool, c.block_table, c.seq_lens if seq_lens is None else seq_lens, max_seq_len,
                          float(c.sm_scale if sm_scale is None else sm_scale), out, guarded[:size], c.residual, c.v_bits, c.v_params, window, sinks)
    torch.cuda.synchronize()
    assert bool((guarded[size:] == 0x5A).all()), "written past the workspace"
    return out


def _check(c, new, group, window=0, sinks=0, seed=1, q_scale=1.0, **more):
    starts = np.concatenate([[0], np.cumsum(new)])
    q = _queries(int(starts[-1]), c.heads * group, seed, q_scale)
    got = _attend(c, q, starts, window, sinks, **more)
    worst = 0.0
    for s, n in enumerate(new):
        rows = slice(int(starts[s]), int(starts[s + 1]))
        if n == 0:
            continue
        positions = torch.arange(c.lens[s] - n, c.lens[s], device=DEV)
        out, spread, slope = c.rows(s, q[rows], positions, window, sinks, more.get("sm_scale"))
        error = (got[rows].double() - out).abs()
        allowed = tolerance(out, spread, slope)
        assert not torch.isnan(error).any(), (s, n)
        worst = max(worst, float((error / allowed).max()))
        assert (error <= allowed).all(), (s, n, float((error / allowed).max()))
    print(f"lens {c.lens[:4]} new {new[:4]} group {group} window {window}: {worst:.2f} of the tolerance", flush=True)
    return got


@pytest.mark.parametrize("group", [1, 2, 3, 4, 7, 8, 16])
@pytest.mark.parametrize("lens,new", [([1], [1]), ([5, 130], [5, 3]), ([128, 256, 127], [1, 2, 1]), ([700], [700]), ([1000, 40, 0, 385], [70, 40, 0, 129])])
def test_lengths_and_groups(lens, new, group):
    _check(Cache(lens, 2), new, group)


@pytest.mark.parametrize("bits,grouped", [((4, 4), False), ((3, 3), False), ((5, 3), False), ((3, 5), False), ((4, 2), False), ((2, 4), False),
                                          ((4, 4), True), ((3, 3), True), ((5, 3), True), ((3, 5), True), ((4, 2), True), ((2, 4), True)])
@pytest.mark.parametrize("v_bits", [16, 4, 2])
@pytest.mark.parametrize("new", [[3, 1], [150, 70]])
def test_every_format(bits, grouped, v_bits, new):
    _check(Cache([420, 300], 2, bits, grouped, v_bits), new, 4)


@pytest.mark.parametrize("v_bits", [16, 4, 2])
@pytest.mark.parametrize("new", [[3, 1, 1], [150, 37, 128]])
def test_a_packed_incomplete_group(v_bits, new):
    _check(Cache([421, 37, 129], 2, v_bits=v_bits, tail=False), new, 4)


@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (5, 3), (100, 4), (128, 0), (129, 128), (300, 130), (1000, 4), (400, 700)])
@pytest.mark.parametrize("new", [[1, 3, 2], [200, 130, 64]])
@pytest.mark.parametrize("v_bits", [16, 4])
def test_windows_and_sinks(window, sinks, new, v_bits):
    _check(Cache([900, 131, 515], 2, v_bits=v_bits), new, 4, window, sinks)


@pytest.mark.parametrize("new", [[2], [300]])
def test_pages_that_a_window_has_left_behind_may_be_anything(new):
    c = Cache([2000], 2)
    low = 2000 - new[0] + 1 - 200
    want = _check(c, new, 4, 200, 4)
    for entry in (-1, 10 ** 9, c.codes.shape[0]):
        c.block_table[0, 1:low // G] = entry
        assert torch.equal(_check(c, new, 4, 200, 4), want)


@pytest.mark.parametrize("kv_heads,group,lens,new", [(8, 4, [9000], [3]), (8, 4, [40000], [1]), (1, 8, [16384], [40]), (2, 4, [5000] * 7, [4] * 7), (8, 2, [3000, 100], [300, 7]),
                                                     (32, 1, [700, 1300], [90, 33]), (1, 1, [2000], [1]), (4, 4, [300] * 70, [1] * 70)])
def test_splits_and_many_sequences(kv_heads, group, lens, new):
    _check(Cache(lens, kv_heads), new, group)


def test_rows_of_no_chunk_are_left_alone_and_early_queries_see_nothing():
    """Padding rows behind the last chunk; a chunk longer than its sequence; a sequence without tokens."""
    c = Cache([40, 0, 300], 2)
    q = _queries(150, 8, 4)
    got = _attend(c, q, [0, 50, 53, 140], fill=7.0)
    assert (got[140:] == 7.0).all()
    assert not got[:10].any() and not got[50:53].any()           # positions -10 .. -1, and -3 .. -1
    out, spread, slope = c.rows(0, q[10:50], torch.arange(40, device=DEV))
    assert ((got[10:50].double() - out).abs() <= tolerance(out, spread, slope)).all()
    out, spread, slope = c.rows(2, q[53:140], torch.arange(213, 300, device=DEV))
    assert ((got[53:140].double() - out).abs() <= tolerance(out, spread, slope)).all()


def test_block_table_entries_outside_the_pool_are_masked():
    c = Cache([500], 2)
    q = _queries(5, 8, 4)
    c.block_table[0, 1] = c.codes.shape[0]
    got = _attend(c, q, [0, 5])
    keep = torch.cat([torch.arange(128), torch.arange(256, 500)]).to(DEV)
    c.k64[0], c.v64[0] = c.k64[0][keep], c.v64[0][keep]
    out, spread, slope = c.rows(0, q, torch.arange(367, 372, device=DEV))
    assert ((got.double() - out).abs() <= tolerance(out, spread, slope)).all()
    c.block_table.fill_(-1)
    assert not _attend(c, q, [0, 5]).any()


@pytest.mark.parametrize("sm_scale", [-0.088, 0.0, 0.5])
def test_other_scales(sm_scale):
    _check(Cache([300, 90], 2), [100, 3], 4, sm_scale=sm_scale)


@pytest.mark.parametrize("q_scale,key_scale", [(30.0, 1.0), (1.0, 0.01), (200.0, 3.0)])
def test_peaked_and_flat_softmaxes(q_scale, key_scale):
    """Largest scores far above the others and far apart from page to page, and all alike."""
    _check(Cache([1100], 2, key_scale=key_scale), [260], 4, q_scale=q_scale)


def test_a_bound_above_the_lengths_changes_nothing():
    c = Cache([900, 140], 2)
    q = _queries(103, 8, 4)
    wide = torch.full((2, 64), -1, dtype=torch.int32, device=DEV)
    wide[:, :c.block_table.shape[1]] = c.block_table
    want = _check(c, [100, 3], 4)
    c.block_table = wide
    got = _check(c, [100, 3], 4, max_seq_len=64 * 128)
    assert ((got.double() - want.double()).abs() <= 2.0 ** -10 * want.double().abs() + 1e-3).all()
    assert torch.equal(_attend(c, q, [0, 100, 103], max_seq_len=8192), _attend(c, q, [0, 100, 103], max_seq_len=8192))


def test_a_single_query_agrees_with_decode_attention():
    c = Cache([777, 128, 3000], 2)
    q = _queries(3, 8, 5)
    pq = c.pq
    out = torch.empty((3, 8, D), device=DEV)
    ws = torch.empty(pq.pq_decode_workspace_bytes(c.layout, 3, 8, c.max_seq_len), dtype=torch.uint8, device=DEV)
    pq.pq_decode_attention(c.layout, q, c.codes, c.params, c.v_pool, c.block_table, c.seq_lens, c.max_seq_len, float(c.sm_scale), out, ws, None, c.residual)
    got = _attend(c, q, [0, 1, 2, 3])
    for s in range(3):
        ref, spread, slope = c.rows(s, q[s:s + 1], [c.lens[s] - 1])
        assert ((got[s].double() - out[s].double()).abs() <= tolerance(ref, spread, slope)[0] + 3e-6).all()


def test_two_calls_in_flight_and_a_captured_one():
    """Two streams with a workspace each; a graph replayed between eager work, with new queries."""
    c = Cache([3000, 900], 2)
    pq = c.pq
    q = [_queries(8, 8, 10 + i) for i in range(2)]
    want = [_attend(c, x, [0, 5, 8]) for x in q]
    size = pq.pq_chunk_workspace_bytes(c.layout, 2, 8, 8, c.max_seq_len)
    starts = _ints([0, 5, 8])
    streams = [torch.cuda.Stream() for _ in range(2)]
    outs, spaces = [torch.zeros_like(x) for x in q], [torch.empty(size, dtype=torch.uint8, device=DEV) for _ in q]

    def call(i):
        pq.pq_chunk_attention(c.layout, q[i], starts, c.codes, c.params, c.v_pool, c.block_table, c.seq_lens, c.max_seq_len, float(c.sm_scale), outs[i],
                              spaces[i], c.residual)

    torch.cuda.synchronize()
    for i, stream in enumerate(streams):
        with torch.cuda.stream(stream):
            for _ in range(5):
                call(i)
    torch.cuda.synchronize()
    assert torch.equal(outs[0], want[0]) and torch.equal(outs[1], want[1])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(0)
    for turn in range(4):
        q[0].copy_(_queries(8, 8, 20 + turn))
        outs[0].zero_()
        graph.replay()
        torch.cuda.synchronize()
        replayed = outs[0].clone()
        call(0)
        torch.cuda.synchronize()
        assert torch.equal(outs[0], replayed)
