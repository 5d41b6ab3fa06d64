"""Chunks of new tokens and sliding windows as a serving loop uses them: planned, appended and attended together, over large
pools, on other streams, through both ways of marshalling."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from chunks import D, DEV, G, Cache, layout, pools, tolerance      # noqa: E402
from test_gpu_chunk_attention import _attend, _check, _ints, _queries      # noqa: E402


@pytest.mark.parametrize("kv_heads,lens,new,windows", [(8, [2688] * 10, [1] * 10, [2300, 2200, 1500, 600, 200]), (2, [5000], [700], [4000, 3000, 1200, 500]),
                                                       (1, [9000, 300], [300, 260], [8000, 2000, 700]), (4, [6000], [30], [5900, 3000, 900])])
@pytest.mark.parametrize("v_bits", [16, 4])
def test_windows_that_leave_parts_of_the_pages(kv_heads, lens, new, windows, v_bits):
    """Whatever a window leaves, its parts fit the workspace of the whole (the guard behind it is looked at)."""
    c = Cache(lens, kv_heads, v_bits=v_bits)
    for window in windows:
        _check(c, new, 4, window, 5)


class Served:
    """A batch whose cache only the library's own calls have filled."""

    def __init__(self, seqs, heads, group, v_bits, room, width=12, seed=0):
        import paper_2502_00527_amd as pq
        self.pq, self.v_bits, self.heads, self.group, self.room = pq, v_bits, heads, group, room
        self.rng = np.random.default_rng(seed)
        self.layout = layout((4, 4), heads)
        n_pages = seqs * width
        self.codes, self.params, self.v_pool, self.v_params = pools(n_pages, (4, 4), heads, False, v_bits)
        self.residual = torch.full((seqs, heads, G, D), float("nan"), dtype=torch.float16, device=DEV)
        self.free = torch.from_numpy(self.rng.permutation(n_pages).astype(np.int32)).to(DEV)
        self.used = 0
        self.table, self.starts, self.counts = _ints(np.full((seqs, width), -1)), _ints(np.zeros(seqs + 1)), _ints([0, 0])
        self.slots = torch.zeros(room, dtype=torch.int64, device=DEV)
        self.lens, self.after, self.new = (_ints(np.zeros(seqs)) for _ in range(3))
        self.keys, self.values = (torch.zeros((room, heads, D), dtype=torch.float16, device=DEV) for _ in range(2))
        self.q = torch.zeros((room, heads * group, D), dtype=torch.float16, device=DEV)
        self.out = torch.zeros_like(self.q)
        self.next_pages = torch.full((seqs * 2 + room // G + 1,), -1, dtype=torch.int32, device=DEV)
        self.max_seq_len = width * G
        self.scale = float(1 / np.sqrt(D))
        self.workspace = torch.empty(pq.pq_chunk_workspace_bytes(self.layout, seqs, heads * group, room, self.max_seq_len), dtype=torch.uint8, device=DEV)
        self.seqs = seqs

    def feed(self, new):
        """The host's part of a step: what comes in, and the free pages."""
        self.lens.copy_(self.after)
        self.new.copy_(_ints(new))
        n = min(len(self.next_pages), len(self.free) - self.used)
        self.next_pages[:n].copy_(self.free[self.used:self.used + n])
        for x, scale in ((self.keys, 1.0), (self.values, 1.0), (self.q, 1.5)):
            x.copy_(torch.from_numpy(self.rng.standard_normal(x.shape) * scale).to(DEV))
        self.out.fill_(9.0)

    def device_step(self, window=0, sinks=0):
        pq = self.pq
        pq.pq_plan_pages(self.layout, self.lens, self.new, self.next_pages, self.table, self.starts, self.slots, self.after, self.counts)
        pq.pq_append_chunk(self.layout, self.keys, self.values, self.starts, self.lens, self.slots, self.residual, self.table, self.codes, self.params,
                           self.v_pool, self.v_bits, self.v_params)
        pq.pq_chunk_attention(self.layout, self.q, self.starts, self.codes, self.params, self.v_pool, self.table, self.after, self.max_seq_len, self.scale,
                              self.out, self.workspace, self.residual, self.v_bits, self.v_params, window, sinks)

    def cached(self):
        """The cache's contents in float64, as a Cache whose rows() can be asked."""
        from oracle import cache_format, polar, values as ovalues
        c = Cache.__new__(Cache)
        c.heads, c.sm_scale, c.lens = self.heads, self.scale, self.after.tolist()
        c.k64, c.v64 = [], []
        for s, n in enumerate(c.lens):
            ids = self.table[s, :(n + G - 1) // G].long()
            packed = n // G * G
            if n == 0:
                c.k64.append(torch.zeros((0, self.heads, D), dtype=torch.float64, device=DEV))
                c.v64.append(c.k64[-1])
                continue
            parts = []
            if packed:
                a, code, *par = cache_format.unpack_pages(self.codes[ids[:packed // G]].cpu().numpy(), self.params[ids[:packed // G]].cpu().numpy(), packed, 4, 4)
                parts.append(polar.dequant_keys(a, code, par[0], par[1], 4, G))
            parts.append(self.residual[s, :, :n - packed].permute(1, 0, 2).cpu().double().numpy())
            c.k64.append(torch.from_numpy(np.concatenate(parts)).double().to(DEV))
            if self.v_bits == 16:
                c.v64.append(self.v_pool[ids].permute(0, 2, 1, 3).reshape(-1, self.heads, D)[:n].double())
            else:
                code = cache_format.unpack_value_pages(self.v_pool[ids].cpu().numpy(), n, self.v_bits)
                par = self.v_params[ids].cpu().numpy().transpose(0, 2, 1, 3).reshape(-1, self.heads, 2)[:n]
                c.v64.append(torch.from_numpy(np.asarray(ovalues.dequant_values(code, par[..., 0], par[..., 1]), np.float64)).to(DEV))
        return c

    def check(self, new, window=0, sinks=0):
        self.used += int(self.counts[0])
        assert self.counts.tolist()[1] == sum(new) and self.after.tolist() == [a + b for a, b in zip(self.lens.tolist(), new)]
        c, starts = self.cached(), self.starts.tolist()
        for s, n in enumerate(new):
            assert starts[s + 1] - starts[s] == n
            if n == 0:
                continue
            rows = slice(starts[s], starts[s + 1])
            out, spread, slope = c.rows(s, self.q[rows], torch.arange(c.lens[s] - n, c.lens[s], device=DEV), window, sinks)
            assert ((self.out[rows].double() - out).abs() <= tolerance(out, spread, slope)).all(), (s, n, c.lens[s])
        assert (self.out[starts[-1]:] == 9.0).all()
        return c


@pytest.mark.parametrize("v_bits", [16, 4, 2])
@pytest.mark.parametrize("window,sinks", [(0, 0), (200, 3)])
def test_a_batch_is_served(v_bits, window, sinks):
    """Prompts, chunks and single tokens side by side; keys come back from what the cache holds."""
    b = Served(3, 2, 4, v_bits, 700)
    for new in ([300, 0, 1], [60, 500, 1], [1, 1, 1], [0, 3, 127], [128, 129, 0], [1, 0, 400]):
        b.feed(new)
        b.device_step(window, sinks)
        torch.cuda.synchronize()
        b.check(new, window, sinks)
    assert len(set(b.table[b.table >= 0].tolist())) == b.used


@pytest.mark.parametrize("v_bits", [16, 4])
def test_single_token_steps_from_a_graph(v_bits):
    """The step of one graph, replayed over a page's end with eager work between; afterwards the kernels for single tokens
    read the same cache."""
    b = Served(4, 2, 4, v_bits, 512)
    b.feed([126, 250, 3, 125])
    b.device_step()
    torch.cuda.synchronize()
    b.check([126, 250, 3, 125])
    steps = Served.__new__(Served)
    steps.__dict__.update(b.__dict__)
    steps.workspace = torch.empty(b.pq.pq_chunk_workspace_bytes(b.layout, 4, 8, 4, b.max_seq_len), dtype=torch.uint8, device=DEV)
    steps.keys, steps.values, steps.q, steps.out, steps.slots = b.keys[:4], b.values[:4], b.q[:4], b.out[:4], b.slots[:4]
    single, windowed = torch.zeros((4, 8, D), device=DEV), torch.zeros((4, 8, D), device=DEV)
    spaces = [torch.empty(n, dtype=torch.uint8, device=DEV) for n in (b.pq.pq_decode_workspace_bytes(b.layout, 4, 8, b.max_seq_len),
                                                                     b.pq.pq_window_workspace_bytes(b.layout, 4, 8, b.max_seq_len, 100, 2))]

    def call():
        steps.device_step()
        common = (b.layout, steps.q, b.codes, b.params, b.v_pool, b.table, b.after, b.max_seq_len)
        b.pq.pq_decode_attention(*common, b.scale, single, spaces[0], None, b.residual, v_bits, b.v_params)
        b.pq.pq_window_attention(*common, 100, 2, b.scale, windowed, spaces[1], b.residual, v_bits, b.v_params)

    new = [1, 1, 1, 1]
    steps.feed(new)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call()                                                    # eagerly, on another stream
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    steps.check(new)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for _ in range(5):
        steps.feed(new)
        graph.replay()
        torch.cuda.synchronize()
        c = steps.check(new)
        for s in range(4):
            for got, window, sinks in ((single, 0, 0), (windowed, 100, 2)):
                out, spread, slope = c.rows(s, steps.q[s:s + 1], [c.lens[s] - 1], window, sinks)
                assert ((got[s].double() - out[0]).abs() <= tolerance(out, spread, slope)[0]).all()


@pytest.mark.parametrize("v_bits", [16, 4])
def test_offsets_past_32_bits(v_bits):
    """The same pages at the end of pools whose offsets do not fit 32 bits."""
    c = Cache([700, 130], 8, v_bits=v_bits)
    pq = c.pq
    q, few = _queries(400, 16, 3), _queries(4, 16, 4)
    one = _queries(2, 16, 5)
    ws = torch.empty(pq.pq_window_workspace_bytes(c.layout, 2, 16, c.max_seq_len, 300, 4), dtype=torch.uint8, device=DEV)

    def results():
        windowed = torch.zeros((2, 16, D), device=DEV)
        pq.pq_window_attention(c.layout, one, c.codes, c.params, c.v_pool, c.block_table, c.seq_lens, c.max_seq_len, 300, 4, float(c.sm_scale), windowed, ws,
                               c.residual, v_bits, c.v_params)
        return _attend(c, q, [0, 300, 400]), _attend(c, few, [0, 3, 4]), windowed

    want = results()
    n = c.codes.shape[0]
    far = (1 << 32) // (c.codes.nbytes // n) + 10 if v_bits == 4 else (1 << 32) // (c.v_pool.nbytes // n) * 2 + 10
    keys, values = (torch.from_numpy(np.random.default_rng(i).standard_normal((260, 8, D))).to(DEV).half() for i in range(2))
    appended = []
    for at in (0, far):
        if at:
            for name in ("codes", "params", "v_pool", "v_params"):
                small = getattr(c, name)
                if small is None:
                    continue
                big = torch.empty((far + n, *small.shape[1:]), dtype=small.dtype, device=DEV)
                big[far:] = original[name]
                setattr(c, name, big)
            c.block_table = torch.where(c.block_table >= 0, c.block_table + far, c.block_table)
            got = results()
            assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
            # The single-token kernel takes a page's value rows in an order that depends on the page's id.  A row is a mean of 304 values at
            # most, by weights that add up to 1: a sum of n fp32 products in any order is off by n 2^-24 of the sum of their absolute
            # values, n = 304 and 8 for what joins the lanes; two sums by twice that
            assert (got[2] - want[2]).abs().max() <= 2 * 312 * 2.0 ** -24 * max(float(v.abs().max()) for v in c.v64)
        else:
            original = {name: None if getattr(c, name) is None else getattr(c, name).clone() for name in ("codes", "params", "v_pool", "v_params")}
        # two sequences of three pages, over the same pages again
        table = _ints(np.arange(6).reshape(2, 3) + at)
        slots = torch.from_numpy(np.concatenate([np.arange(130), np.arange(130) + 3 * G]).astype(np.int64) + at * G).to(DEV)
        residual = torch.zeros((2, 8, G, D), dtype=torch.float16, device=DEV)
        pq.pq_append_chunk(c.layout, keys, values, _ints([0, 130, 260]), _ints([0, 0]), slots, residual, table, c.codes, c.params, c.v_pool, v_bits, c.v_params)
        appended.append([x[at:at + 6].clone() for x in (c.codes, c.params, c.v_pool)] + [residual])
    assert c.v_pool.nbytes > 1 << 32 or c.codes.nbytes > 1 << 32
    for a, b in zip(*appended):
        assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))


def _all_calls(c, new_calls):
    """Arguments of one call each of the four entry points over a cache."""
    pq, n = c.pq, len(c.lens)
    q, starts = _queries(n, 8, 3), _ints(np.arange(n + 1))
    space = torch.empty(max(pq.pq_chunk_workspace_bytes(c.layout, n, 8, n, c.max_seq_len), pq.pq_window_workspace_bytes(c.layout, n, 8, c.max_seq_len, 200, 4)),
                        dtype=torch.uint8, device=DEV)
    out16, out32 = torch.zeros((n, 8, D), dtype=torch.float16, device=DEV), torch.zeros((n, 8, D), device=DEV)
    wide = _ints(np.full((n, 9), -1))
    wide[:, :c.block_table.shape[1]] = c.block_table
    plan = [c.layout, c.seq_lens, _ints([1] * n), _ints(np.arange(5)), wide, _ints(np.zeros(n + 1)), torch.zeros(n, dtype=torch.int64, device=DEV), _ints(np.zeros(n)),
            _ints([0, 0])]
    keys, values = (torch.from_numpy(np.random.default_rng(i).standard_normal((n, 2, D))).to(DEV).half() for i in range(2))
    slots = c.block_table[:, 0].long() * G
    return {"plan_pages": (plan, plan[4:]),
            "chunk_attention": ([c.layout, q, starts, c.codes, c.params, c.v_pool, c.block_table, c.seq_lens, c.max_seq_len, float(c.sm_scale), out16, space, c.residual,
                                 c.v_bits, c.v_params, 200, 4], [out16]),
            "window_attention": ([c.layout, q, c.codes, c.params, c.v_pool, c.block_table, c.seq_lens, c.max_seq_len, 200, 4, float(c.sm_scale), out32, space,
                                  c.residual, c.v_bits, c.v_params], [out32]),
            "append_chunk": ([c.layout, keys, values, starts, c.seq_lens, slots, c.residual, c.block_table, c.codes, c.params, c.v_pool, c.v_bits, c.v_params],
                             [x for x in (c.codes, c.params, c.v_pool, c.v_params, c.residual) if x is not None])}


class _Declines:
    def __getattr__(self, name):
        return lambda *a: None


@pytest.mark.parametrize("v_bits", [16, 2])
def test_both_ways_of_marshalling_make_the_same_calls(v_bits, monkeypatch):
    results = []
    for declines in (False, True):
        c = Cache([500, 129, 255], 2, v_bits=v_bits, seed=4)
        pq = c.pq
        calls = _Declines() if declines else pq._marshaller()
        monkeypatch.setattr(pq, "_calls", calls)
        results.append([])
        for name, (args, outs) in _all_calls(c, calls).items():
            if not declines:
                assert getattr(calls, name)(*args) == 0
            getattr(pq, "pq_" + name)(*args)
            torch.cuda.synchronize()
            results[-1] += [x.clone().view(torch.uint8) for x in outs]
    for a, b in zip(*results):
        assert torch.equal(a, b)


@pytest.mark.parametrize("declines", [False, True])
def test_arguments_that_do_not_fit_raise(declines, monkeypatch):
    c = Cache([500, 129, 255], 2, v_bits=4)
    pq = c.pq
    calls = pq._marshaller()
    if declines:
        monkeypatch.setattr(pq, "_calls", _Declines())
    made = _all_calls(c, None)
    wrong = {"plan_pages": [(1, c.seq_lens.long()), (2, c.seq_lens[:2]), (4, c.block_table[:2]), (5, _ints([0, 0])), (6, _ints([0] * 3)), (7, c.seq_lens), (8, _ints([0])),
                            (3, torch.arange(5, dtype=torch.int32))],
             "chunk_attention": [(1, made["chunk_attention"][0][1].float()), (1, made["chunk_attention"][0][1].transpose(0, 1)), (2, _ints([0, 1])), (3, c.codes.cpu()),
                                 (4, c.params[:1]), (5, c.v_pool[:1]), (6, c.block_table[:2]), (7, c.seq_lens[:2]), (8, 0), (9, float("nan")),
                                 (10, made["chunk_attention"][0][10][:2]), (11, made["chunk_attention"][0][11][:0]), (12, c.residual[:1]), (13, 3), (14, None), (15, -1),
                                 (16, -1)],
             "window_attention": [(1, made["window_attention"][0][1].double()), (2, c.codes.cpu()), (4, c.v_pool[:1]), (5, c.block_table[:2]), (6, c.seq_lens.long()),
                                  (8, 0), (9, -1), (11, made["window_attention"][0][11].half()), (12, made["window_attention"][0][12][:16]), (13, c.residual[:1]), (14, 7)],
             "append_chunk": [(1, made["append_chunk"][0][1][:, :1]), (1, made["append_chunk"][0][1].double()), (2, made["append_chunk"][0][2].float()),
                              (2, made["append_chunk"][0][2][:2]), (3, _ints([0, 1])), (5, None), (5, _ints([0, 1, 2])), (6, c.residual[:1]), (7, c.block_table[:1]),
                              (9, c.params[:1]), (10, c.v_pool[:1]), (11, 16), (12, None)]}
    before = {name: [x.clone().view(torch.uint8) for x in outs] for name, (_, outs) in made.items()}
    for name, changes in wrong.items():
        args, outs = made[name]
        for at, value in changes:
            bad = list(args)
            bad[at] = value
            if not declines:
                assert getattr(calls, name)(*bad) != 0, (name, at)
            with pytest.raises(pq.PolarQuantError):
                getattr(pq, "pq_" + name)(*bad)
        torch.cuda.synchronize()
        for x, y in zip(outs, before[name]):
            assert torch.equal(x.view(torch.uint8), y), name


def test_tensors_of_another_device_are_refused(monkeypatch):
    c = Cache([500, 129, 255], 2)
    pq = c.pq
    made = _all_calls(c, None)
    monkeypatch.setattr(pq, "_calls", _Declines())
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 1)
    for name, (args, _) in made.items():
        with pytest.raises(pq.PolarQuantError, match="current device"):
            getattr(pq, "pq_" + name)(*args)


def test_overlapping_calls_of_two_graphs():
    """Two captured calls, a workspace each, replayed at the same time on two streams."""
    c = Cache([3000, 900], 2)
    pq = c.pq
    size = pq.pq_chunk_workspace_bytes(c.layout, 2, 8, 8, c.max_seq_len)
    starts, queries = _ints([0, 5, 8]), [_queries(8, 8, i) for i in range(2)]
    outs, spaces, graphs = [torch.zeros_like(x) for x in queries], [torch.empty(size, dtype=torch.uint8, device=DEV) for _ in range(2)], []
    want = [_attend(c, x, [0, 5, 8], 1000, 3) for x in queries]
    for i in range(2):
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[i]):
            for _ in range(3):
                pq.pq_chunk_attention(c.layout, queries[i], starts, c.codes, c.params, c.v_pool, c.block_table, c.seq_lens, c.max_seq_len, float(c.sm_scale),
                                      outs[i], spaces[i], c.residual, 16, None, 1000, 3)
    streams = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(3):
        for x in outs:
            x.zero_()
        torch.cuda.synchronize()
        for stream, graph in zip(streams, graphs):
            with torch.cuda.stream(stream):
                graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs, want))


@pytest.mark.parametrize("starts", [[0, 0, 0, 0], [7, 7, 7, 7], [0, 40, 0, 40], [40, 0, 40, 0], [-5, 3, 90, 20], [0, 1 << 30, 1 << 30, 1 << 30]])
@pytest.mark.parametrize("rows", [40, 2])
def test_starts_that_are_no_ranges_of_the_rows(starts, rows):
    """Empty chunks alone, and starts that the documentation does not allow: nothing outside the tensors is touched, and a call
    with proper ones afterwards, in the same workspace, is right."""
    c = Cache([2000, 900, 1200], 2)
    pq = c.pq
    q = _queries(rows, 8, 3)
    size = pq.pq_chunk_workspace_bytes(c.layout, 3, 8, rows, c.max_seq_len)
    guarded, out = torch.full((size + 4096,), 0x5A, dtype=torch.uint8, device=DEV), torch.full((rows + 40, 8, D), 3.0, dtype=torch.float16, device=DEV)
    proper = [0, rows // 2, rows // 2, rows]
    for s in (starts, proper, starts, proper):
        out.fill_(3.0)
        pq.pq_chunk_attention(c.layout, q, _ints(s), c.codes, c.params, c.v_pool, c.block_table, c.seq_lens, c.max_seq_len, float(c.sm_scale), out[:rows],
                              guarded[:size], c.residual)
        torch.cuda.synchronize()
        assert bool((guarded[size:] == 0x5A).all()) and bool((out[rows:] == 3.0).all())
        if len(set(starts)) == 1 and s is starts:
            assert bool((out == 3.0).all())
    assert torch.equal(out[:rows], _attend(c, q, proper))


@pytest.mark.parametrize("kv_heads,seqs,most_len,most_new", [(1, 100, 3000, 3), (1, 90, 2500, 60), (2, 64, 4000, 40), (2, 65, 4000, 40), (1, 3, 30000, 90), (8, 5, 6000, 7), (1, 200, 600, 9)])
@pytest.mark.parametrize("window,sinks", [(0, 0), (700, 5)])
def test_ragged_batches_cut_by_their_lengths(kv_heads, seqs, most_len, most_new, window, sinks):
    """More sequences than a wavefront has lanes, as many, and fewer; a bound far above the lengths, as a captured call has it."""
    rng = np.random.default_rng(seqs)
    new = rng.integers(0, most_new + 1, seqs)
    new[0] = most_new
    lens = np.maximum(rng.integers(0, most_len + 1, seqs), new)
    lens[-1] = most_len
    c = Cache([int(x) for x in lens], kv_heads)
    wide = torch.full((seqs, 400), -1, dtype=torch.int32, device=DEV)
    wide[:, :c.block_table.shape[1]] = c.block_table
    _check(c, [int(x) for x in new], 4, window, sinks)
    c.block_table = wide
    _check(c, [int(x) for x in new], 4, window, sinks, max_seq_len=400 * G)
