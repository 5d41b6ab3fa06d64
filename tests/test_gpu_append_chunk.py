"""pq_append_chunk against pq_append_keys token by token and pq_encode_values, byte for byte."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from chunks import D, DEV, G, layout, pools      # noqa: E402
from oracle import cache_format                 # noqa: E402


def _table(before, new, rng, spare=2):
    counts = [(b + n + G - 1) // G for b, n in zip(before, new)]
    order = rng.permutation(sum(counts) + spare).astype(np.int32)
    table = np.full((len(before), max(1, max(counts))), -1, np.int32)
    at = 0
    for s, c in enumerate(counts):
        table[s, :c] = order[at:at + c]
        at += c
    return table, len(order)


def _slots(before, new, table):
    return np.array([table[s, (b + i) // G] * np.int64(G) + (b + i) % G for s, (b, n) in enumerate(zip(before, new)) for i in range(n)], np.int64)


def _ints(x):
    return torch.as_tensor(np.asarray(x), dtype=torch.int32).to(DEV)


def _case(before, new, heads, bits, grouped, v_bits, dtype, seed, pad=0, strided=False):
    import paper_2502_00527_amd as pq

    rng = np.random.default_rng(seed)
    lay = layout(bits, heads, grouped)
    table, pages = _table(before, new, rng)
    total = sum(new)
    wide = 3 if strided else 1                                   # rows and heads of a fused projection's output
    keys = torch.from_numpy(rng.standard_normal((total + pad, heads, wide * D))).to(DEV).to(dtype)[:, :, :D]
    values = torch.from_numpy(rng.standard_normal((total + pad, heads, wide * D))).to(DEV).half()[:, :, (wide - 1) * D:]
    if pad:
        keys[total:], values[total:] = float("nan"), float("nan")
    residual = torch.from_numpy(rng.standard_normal((len(before), heads, G, D))).to(DEV).half()
    starts = np.concatenate([[0], np.cumsum(new)])
    slots = torch.from_numpy(np.concatenate([_slots(before, new, table), np.full(pad, -1, np.int64)])).to(DEV)
    return pq, lay, table, pages, keys, values, residual, starts, slots


@pytest.mark.parametrize("before,new", [([0], [1]), ([127], [1]), ([126], [1]), ([0], [128]), ([5], [123]), ([5], [300]), ([200, 0, 127, 128], [1, 0, 2, 129]),
                                        ([0, 1, 130], [700, 255, 126]), ([3] * 300, [1] * 300), ([120] * 9 + [0], [9, 8, 7, 136, 0, 1, 264, 20, 5, 1024])])
@pytest.mark.parametrize("bits,grouped,v_bits,dtype", [((4, 4), False, 16, torch.float16), ((3, 3), False, 4, torch.float16), ((5, 3), True, 2, torch.float16),
                                                       ((4, 2), False, 2, torch.float32), ((2, 4), True, 4, torch.float32), ((3, 5), False, 16, torch.float32)])
def test_same_bytes_as_token_by_token(before, new, bits, grouped, v_bits, dtype):
    heads = 2
    pq, lay, table, pages, keys, values, residual, starts, slots = _case(before, new, heads, bits, grouped, v_bits, dtype, 7)
    print(before[:4], new[:4], bits, grouped, v_bits, dtype, flush=True)
    codes, params, v_pool, v_params = pools(pages, bits, heads, grouped, v_bits)
    want_codes, want_params, _, _ = pools(pages, bits, heads, grouped, v_bits)
    got_residual, want_residual = residual.clone(), residual.clone()
    pq.pq_append_chunk(lay, keys, values, _ints(starts), _ints(before), slots, got_residual, _ints(table), codes, params, v_pool, v_bits, v_params)
    torch.cuda.synchronize()
    lens = np.array(before)
    for i in range(max(new)):
        # the sequences that still have a token, the others skipped by a negative length
        now = _ints([lens[s] if i < new[s] else -1 for s in range(len(new))])
        row = keys[[min(starts[s] + i, keys.shape[0] - 1) for s in range(len(new))]].contiguous()
        pq.pq_append_keys(lay, row, want_residual, now, _ints(table), want_codes, want_params)
        lens += [int(i < n) for n in new]
    assert torch.equal(codes, want_codes)
    assert torch.equal(params.view(torch.int16), want_params.view(torch.int16))
    for s, (b, n) in enumerate(zip(before, new)):
        rest = (b + n) % G
        assert torch.equal(got_residual[s, :, :rest], want_residual[s, :, :rest])
        assert torch.equal(got_residual[s, :, rest:], residual[s, :, rest:]) or n == 0, "rows behind the last token were written"
    # values: each token's codes or row, and nothing else of the pool
    where = slots.cpu().numpy()
    rows = values.cpu()
    if v_bits == 16:
        got = v_pool.permute(0, 2, 1, 3).reshape(-1, heads, D)
        assert torch.equal(got[torch.from_numpy(where).to(DEV)].cpu(), rows)
        others = np.setdiff1d(np.arange(pages * G), where)
        assert torch.isnan(got[torch.from_numpy(others).to(DEV)]).all()
        return
    n_pages = (len(where) + G - 1) // G
    _, _, ref_pool, ref_params = pools(n_pages, bits, heads, grouped, v_bits)
    pq.pq_encode_values(lay, v_bits, values, torch.arange(n_pages, dtype=torch.int32, device=DEV), ref_pool, ref_params)
    want = cache_format.unpack_value_pages(ref_pool.cpu().numpy(), len(where), v_bits)
    got = cache_format.unpack_value_pages(v_pool.cpu().numpy(), pages * G, v_bits)
    np.testing.assert_array_equal(got[where], want)
    flat = lambda p: p.permute(0, 2, 1, 3).reshape(-1, heads, 2).contiguous().view(torch.int16).cpu().numpy()      # noqa: E731
    np.testing.assert_array_equal(flat(v_params)[where], flat(ref_params)[:len(where)])
    others = np.setdiff1d(np.arange(pages * G), where)
    untouched = cache_format.unpack_value_pages(pools(pages, bits, heads, grouped, v_bits)[2].cpu().numpy(), pages * G, v_bits)
    np.testing.assert_array_equal(got[others], untouched[others])


@pytest.mark.parametrize("v_bits", [16, 4])
@pytest.mark.parametrize("heads", [1, 3, 8])
def test_strides_padding_and_other_orders(heads, v_bits):
    """Views of wider rows, padding rows behind the last chunk, and the same call with contiguous copies."""
    before, new = [100, 0, 250], [60, 333, 7]
    pq, lay, table, pages, keys, values, residual, starts, slots = _case(before, new, heads, (4, 4), False, v_bits, torch.float16, 3, pad=37, strided=True)
    results = []
    for k, v in ((keys, values), (keys.contiguous(), values.contiguous()), (keys.permute(1, 0, 2).contiguous().permute(1, 0, 2), values)):
        state = (residual.clone(), *pools(pages, (4, 4), heads, False, v_bits, poison=False))
        pq.pq_append_chunk(lay, k, v, _ints(starts), _ints(before), slots, state[0], _ints(table), *state[1:4], v_bits, state[4])
        results.append([x for x in state if x is not None])
    torch.cuda.synchronize()
    for other in results[1:]:
        for a, b in zip(results[0], other):
            assert torch.equal(a, b)
    assert not any(torch.isnan(x).any() for x in results[0] if x.is_floating_point())


def test_keys_alone():
    pq, lay, table, pages, keys, values, residual, starts, slots = _case([100, 3], [60, 300], 2, (4, 4), False, 16, torch.float16, 5)
    both, alone = residual.clone(), residual.clone()
    a, b = pools(pages, (4, 4), 2, False, 16), pools(pages, (4, 4), 2, False, 16)
    pq.pq_append_chunk(lay, keys, values, _ints(starts), _ints([100, 3]), slots, both, _ints(table), *a[:3])
    pq.pq_append_chunk(lay, keys, None, _ints(starts), _ints([100, 3]), None, alone, _ints(table), *b[:2])
    torch.cuda.synchronize()
    assert torch.equal(both, alone) and torch.equal(a[0], b[0]) and torch.isnan(b[2]).all()


def test_pages_and_slots_outside_the_pool_are_skipped():
    """Missing pages, and starts that are no ranges: nothing outside the chunk's own places changes."""
    pq, lay, table, pages, keys, values, residual, starts, slots = _case([100, 3], [60, 300], 2, (4, 4), False, 4, torch.float16, 6)
    table[0, 0], table[1, 1] = -1, pages + 9                     # the group that sequence 0 completes, the second one of sequence 1
    slots[5], slots[70] = -1, pages * G
    codes, params, v_pool, v_params = pools(pages, (4, 4), 2, False, 4)
    got = residual.clone()
    pq.pq_append_chunk(lay, keys, values, _ints(starts), _ints([100, 3]), slots, got, _ints(table), codes, params, v_pool, 4, v_params)
    torch.cuda.synchronize()
    written = (codes != 0xA5).flatten(1).any(1).cpu().numpy()
    assert written.sum() == 1 and written[table[1, 0]]
    assert torch.equal(got[0, :, :32], keys[28:60].permute(1, 0, 2))
    assert int((~torch.isnan(v_params[:, 0, :, 0])).sum()) == 358


def test_a_captured_step_is_replayed():
    """Plan and append in one graph, replayed with other lengths and rows, against the same calls made eagerly."""
    import paper_2502_00527_amd as pq

    heads, seqs, room, width = 2, 3, 400, 8
    lay = layout((4, 4), heads)
    rng = np.random.default_rng(2)
    lens, new = _ints([0, 0, 0]), _ints([1, 1, 1])
    free = torch.arange(40, dtype=torch.int32, device=DEV)
    table, starts, after, counts = _ints(np.full((seqs, width), -1)), _ints([0] * 4), _ints([0] * 3), _ints([0, 0])
    slots = torch.zeros(room, dtype=torch.int64, device=DEV)
    keys, values = torch.zeros((room, heads, D), device=DEV).half(), torch.zeros((room, heads, D), device=DEV).half()
    residual = torch.zeros((seqs, heads, G, D), device=DEV).half()
    cache = pools(40, (4, 4), heads, False, 16, poison=False)

    def step():
        pq.pq_plan_pages(lay, lens, new, free, table, starts, slots, after, counts)
        pq.pq_append_chunk(lay, keys, values, starts, lens, slots, residual, table, *cache[:3])

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for replay in range(4):
        before, fresh = rng.integers(0, 500, seqs), rng.integers(0, 130, seqs)
        results = []
        rows = [torch.from_numpy(rng.standard_normal((room, heads, D))).to(DEV).half() for _ in range(2)]
        for way in (graph.replay, step):
            # (pages of their own for the tokens before: in one page of three sequences the last to write would be seen)
            table.copy_(_ints(np.arange(seqs * width).reshape(seqs, width) + 40 - seqs * width))
            for x in (slots, starts, after, counts, residual, *cache[:3]):
                x.zero_()
            lens.copy_(_ints(before))
            new.copy_(_ints(fresh))
            keys.copy_(rows[0])
            values.copy_(rows[1])
            way()
            torch.cuda.synchronize()
            results.append([x.clone() for x in (table, slots, starts, after, counts, residual, *cache[:3])])
        for a, b in zip(*results):
            assert torch.equal(a, b), replay
