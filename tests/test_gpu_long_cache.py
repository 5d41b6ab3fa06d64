"""Bounds and choice of pages, attention over chosen pages, attention that sums the pages' weights, eviction: each against its definition
(long_cache.py, chunks.py), alone and as a serving loop calls them together."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

import long_cache as ref                    # noqa: E402
from chunks import D, DEV, G, Cache         # noqa: E402

FORMATS = [((4, 4), False), ((3, 3), False), ((5, 3), False), ((3, 5), False), ((4, 2), False), ((2, 4), False),
           ((4, 4), True), ((3, 3), True), ((5, 3), True), ((3, 5), True), ((4, 2), True), ((2, 4), True)]


def _ints(values, dtype=torch.int32):
    return torch.tensor(values, dtype=dtype, device=DEV)


def _queries(seqs, heads, seed, dtype=torch.float16, scale=1.0):
    return (torch.from_numpy(np.random.default_rng(seed).standard_normal((seqs, heads, D))) * scale).to(DEV).to(dtype)


def _guarded(size):
    return torch.full((size + 4096,), 0x5A, dtype=torch.uint8, device=DEV)


def _bound_pools(c):
    n = c.codes.shape[0]
    return torch.full((n, c.heads, 4, 64), 77, dtype=torch.int8, device=DEV), torch.full((n, c.heads, 4), float("nan"), device=DEV)


def _bound(c, before=None, after=None, most=None, pools=None):
    bounds, scales = pools or _bound_pools(c)
    after = c.seq_lens if after is None else after
    c.pq.pq_bound_pages(c.layout, c.codes, c.params, c.block_table, before, after, most or c.max_seq_len, bounds, scales)
    torch.cuda.synchronize()
    return bounds, scales


def _select(c, q, bounds, scales, n_selected, n_first=1, n_last=1, max_seq_len=None, table=None, lens=None):
    pq = c.pq
    max_seq_len = max_seq_len or c.max_seq_len
    size = pq.pq_select_workspace_bytes(c.layout, q.shape[0], max_seq_len)
    work = _guarded(size)
    selected = torch.full((q.shape[0], c.heads, n_selected), -7, dtype=torch.int32, device=DEV)
    lens_out = torch.full((q.shape[0], c.heads), -7, dtype=torch.int32, device=DEV)
    pq.pq_select_pages(c.layout, q, bounds, scales, c.block_table if table is None else table, c.seq_lens if lens is None else lens, max_seq_len,
                       n_first, n_last, selected, lens_out, work[:size])
    torch.cuda.synchronize()
    assert bool((work[size:] == 0x5A).all()), "written past the workspace"
    return selected, lens_out


def _sparse(c, q, pools, n_selected, n_first=1, n_last=1, max_seq_len=None, given=None):
    pq = c.pq
    max_seq_len = max_seq_len or c.max_seq_len
    size = pq.pq_sparse_workspace_bytes(c.layout, *q.shape[:2], max_seq_len, n_selected)
    work = _guarded(size)
    out = torch.full(q.shape, float("nan"), device=DEV)
    if given is None:
        selected = torch.full((q.shape[0], c.heads, n_selected), -7, dtype=torch.int32, device=DEV)
        lens = torch.full((q.shape[0], c.heads), -7, dtype=torch.int32, device=DEV)
        table, seq_lens, (bounds, scales) = c.block_table, c.seq_lens, pools
    else:
        (selected, lens), (table, seq_lens, bounds, scales) = given, (None,) * 4
    pq.pq_sparse_attention(c.layout, q, c.codes, c.params, c.v_pool, bounds, scales, table, seq_lens, max_seq_len, n_first, n_last,
                           float(c.sm_scale), selected, lens, out, work[:size], c.residual, c.v_bits, c.v_params)
    torch.cuda.synchronize()
    assert bool((work[size:] == 0x5A).all()), "written past the workspace"
    return out, selected, lens


def _weigh(c, q, before=None, decay=1.0, max_seq_len=None, stride=None, weights=None):
    pq = c.pq
    max_seq_len = max_seq_len or c.max_seq_len
    size = pq.pq_weights_workspace_bytes(c.layout, *q.shape[:2], max_seq_len)
    work = _guarded(size)
    out = torch.full(q.shape, float("nan"), device=DEV)
    if weights is None:
        weights = torch.full((q.shape[0], stride or (max_seq_len + G - 1) // G), -5.0, device=DEV)
    pq.pq_decode_attention_weights(c.layout, q, c.codes, c.params, c.v_pool, c.block_table, c.seq_lens, max_seq_len, float(c.sm_scale), out, weights,
                                   work[:size], before, decay, c.residual, c.v_bits, c.v_params)
    torch.cuda.synchronize()
    assert bool((work[size:] == 0x5A).all()), "written past the workspace"
    return out, weights


# ---- bounds ------------------------------------------------------------------------------------


def _check_bounds(c, before, after, got, untouched=77):
    bounds, scales = (x.cpu().numpy() for x in got)
    done = np.zeros(len(bounds), bool)
    for s, (b, a) in enumerate(zip(before, after)):
        ids = c.table[s, max(0, b) // G:max(0, a) // G]
        if len(ids) == 0:
            continue
        done[ids] = True
        want = ref.bounds_of(c.codes[_ids(ids)].cpu().numpy(), c.params[_ids(ids)].cpu().numpy(), c.bits)
        assert np.array_equal(bounds[ids], want[0])
        assert np.array_equal(scales[ids], want[1])
    assert (bounds[~done] == untouched).all() and np.isnan(scales[~done]).all()


def _ids(ids):
    return torch.from_numpy(np.asarray(ids, np.int64)).to(DEV)


@pytest.mark.parametrize("bits,grouped", FORMATS)
def test_bounds_of_every_format(bits, grouped):
    c = Cache([1000, 128, 127, 0, 385], 3, bits, grouped)
    _check_bounds(c, [0] * 5, c.lens, _bound(c))


@pytest.mark.parametrize("key_scale", [1e-4, 30.0, 2000.0])
@pytest.mark.parametrize("grouped", [False, True])
def test_bounds_of_small_and_large_keys(key_scale, grouped):
    c = Cache([300, 256], 2, (4, 4), grouped, key_scale=key_scale)
    _check_bounds(c, [0, 0], c.lens, _bound(c))


def test_bounds_of_the_new_pages_only():
    c = Cache([600, 700, 256, 255, 1, 300], 2)
    before = [127, 128, 255, 255, -5, 300]
    _check_bounds(c, before, c.lens, _bound(c, _ints(before), c.seq_lens, 600))


def test_bounds_of_dead_channels():
    """All keys of a head zero: scale 0, bounds 0."""
    c = Cache([256], 2)
    c.codes[:, 1] = 0
    c.params[:, 1] = 0
    got = _bound(c)
    ids = _ids(c.table[0])
    assert not got[0][ids, 1].any() and not got[1][ids, 1].any()
    _check_bounds(c, [0], c.lens, got)


def test_bounds_skip_pages_that_are_missing():
    c = Cache([700, 300], 2)
    kept = c.block_table.clone()
    c.block_table[0, 1], c.block_table[0, 3], c.block_table[1, 0] = -1, c.codes.shape[0], 1 << 30
    bounds, scales = _bound(c)
    missing = [int(kept[0, 1]), int(kept[0, 3]), int(kept[1, 0])]
    assert bool((bounds[missing] == 77).all()) and bool(scales[missing].isnan().all())
    there = [int(kept[0, 0]), int(kept[0, 2]), int(kept[0, 4]), int(kept[1, 1])]
    assert not bool(scales[there].isnan().any())


def test_more_new_tokens_than_said():
    """Groups past what max_new_tokens can complete get no bounds."""
    c = Cache([1000], 1)
    bounds, scales = _bound(c, most=256)
    ids = c.table[0]
    assert not bool(scales[_ids(ids[:2])].isnan().any()) and bool(scales[_ids(ids[2:])].isnan().all())


# ---- choice --------------------------------------------------------------------------------------


def _check_choice(c, q, pools, n_selected, n_first, n_last, **more):
    got, lens = _select(c, q, *pools, n_selected, n_first, n_last, **more)
    bounds, scales = (x.cpu().numpy() for x in pools)
    want, want_lens = ref.select(q.float().cpu().numpy(), bounds, scales, c.block_table.cpu().numpy(), c.lens, c.heads, n_selected, n_first, n_last)
    assert np.array_equal(got.cpu().numpy(), want)
    assert np.array_equal(lens.cpu().numpy(), want_lens)
    return got, lens


@pytest.mark.parametrize("group", [1, 2, 3, 4, 7, 8, 12, 16])
@pytest.mark.parametrize("dtype", [torch.float16, torch.float32])
def test_choice_of_every_group(group, dtype):
    c = Cache([3000, 1, 128, 129, 0, 1700, 2048], 2)
    _check_choice(c, _queries(7, 2 * group, 5, dtype), _bound(c), 6, 1, 2)


@pytest.mark.parametrize("n_selected,n_first,n_last", [(1, 0, 1), (2, 1, 1), (3, 0, 1), (5, 5 - 2, 2), (9, 0, 9), (16, 2, 4), (23, 1, 2), (24, 1, 2), (40, 0, 1)])
def test_choice_of_every_number(n_selected, n_first, n_last):
    c = Cache([3000, 700, 2944, 2945], 2, (3, 3))
    _check_choice(c, _queries(4, 8, 6), _bound(c), n_selected, n_first, n_last)


def _random_pools(pages, heads, seed, distinct=None):
    """Bounds without a cache behind them."""
    rng = np.random.default_rng(seed)
    bounds = np.concatenate([rng.integers(-127, 128, (pages, heads, 4, 32)), rng.integers(0, 128, (pages, heads, 4, 32))], -1).astype(np.int8)
    scales = np.exp(rng.standard_normal((pages, heads, 4))).astype(np.float32) / 127
    if distinct:
        pick = rng.integers(0, distinct, pages)
        bounds, scales = bounds[pick], scales[pick]
    return torch.from_numpy(bounds).to(DEV), torch.from_numpy(scales).to(DEV)


class _Plain:
    """What _select looks at, without codes."""

    def __init__(self, lens, heads, pool_pages, seed=0):
        import paper_2502_00527_amd as pq
        rng = np.random.default_rng(seed)
        self.pq, self.lens, self.heads, self.layout = pq, lens, heads, pq.Layout(D, 4, 4, G, heads)
        self.max_seq_len = max(lens)
        width = (self.max_seq_len + G - 1) // G
        self.block_table = torch.from_numpy(rng.integers(0, pool_pages, (len(lens), width)).astype(np.int32)).to(DEV)
        self.seq_lens = _ints(lens)


@pytest.mark.parametrize("distinct", [None, 1, 2, 5])
@pytest.mark.parametrize("pages", [255, 256, 257, 1024, 1100, 4096, 4097, 9000])
def test_choice_of_long_sequences_and_ties(pages, distinct):
    """Block-table entries repeat, so that many scores are equal: the first pages are taken."""
    c = _Plain([pages * G - 5, pages * G // 3, 700], 2, 50)
    _check_choice(c, _queries(3, 8, pages), _random_pools(50, 2, pages, distinct), min(pages - 1, 100), 1, 2)


@pytest.mark.parametrize("group", [1, 6, 16])
@pytest.mark.parametrize("seqs,heads,pages", [(1, 1, 300), (1, 4, 1500), (40, 2, 700), (3, 1, 5000), (70, 2, 500), (1, 32, 1030), (130, 2, 260)])
def test_choice_of_every_way_to_share_units(seqs, heads, pages, group):
    """Units of one work-group, and of several with one, two and four tiles a wavefront; each with one, two and four sets of heads."""
    rng = np.random.default_rng(pages)
    c = _Plain([pages * G] + [int(n) for n in rng.integers(1, pages * G, seqs - 1)], heads, 90)
    _check_choice(c, _queries(seqs, heads * group, 3, torch.float32 if group == 6 else torch.float16), _random_pools(90, heads, 7), 40, 1, 2)


@pytest.mark.parametrize("lens", [[5000 * G], [200, 130000]])
def test_a_bound_above_the_lengths(lens):
    c = _Plain(lens, 1, 50)
    short = [n // 7 + 1 for n in lens]
    c.lens, c.seq_lens = short, _ints(short)
    _check_choice(c, _queries(len(lens), 4, 3), _random_pools(50, 1, 3), 12, 1, 1, max_seq_len=max(lens))


def test_lengths_above_the_bound():
    c = _Plain([4000, 4000], 1, 50)
    pools, q = _random_pools(50, 1, 3), _queries(2, 4, 3)
    want = _select(c, q, *pools, 12)
    c.seq_lens = _ints([9000, 1 << 30])
    got = _select(c, q, *pools, 12)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


def test_missing_pages_are_chosen_last():
    c = _Plain([40 * G], 2, 50)
    c.block_table[0, 3:30] = -1
    c.block_table[0, 30] = 50
    got, _ = _check_choice(c, _queries(1, 8, 1), _random_pools(50, 2, 4), 20, 1, 1)
    assert bool((got == -1).any())                           # 12 pages are there, 20 are asked for


def test_negative_lengths_have_no_pages():
    c = _Plain([500, 300], 1, 9)
    c.lens, c.seq_lens = [-3, 0], _ints([-3, 0])
    got, lens = _check_choice(c, _queries(2, 2, 1), _random_pools(9, 1, 4), 3, 1, 1)
    assert bool((got == -1).all()) and not lens.any()


@pytest.mark.parametrize("scale", [0.0, 1e-35, 6e4])
def test_choice_of_extreme_queries(scale):
    c = _Plain([6000], 2, 60)
    _check_choice(c, _queries(1, 8, 2, torch.float32, scale), _random_pools(60, 2, 8), 9, 1, 1)


def test_choice_with_scores_that_are_no_numbers_stays_inside():
    """Queries and scales that are not finite: which pages is not said, but as many as asked for, each once and in order."""
    c = _Plain([6000], 1, 60)
    bounds, scales = _random_pools(60, 1, 8)
    c.block_table = torch.arange(47, dtype=torch.int32, device=DEV)[None]
    scales[3:20] = float("nan")
    scales[20:30] = float("inf")
    q = _queries(1, 4, 2, torch.float32)
    q[0, 1, 7] = float("nan")
    q[0, 2, 8] = float("inf")
    got, _ = _select(c, q, bounds, scales, 13, 1, 2)
    got = got[0, 0].tolist()
    assert sorted(set(got)) == got and len(got) == 13 and got[0] == 0 and got[-2:] == [45, 46]


def test_a_choice_holds_the_page_that_matters():
    """One page's keys point where the query does: it is chosen whatever its place."""
    c = _Plain([64 * G], 1, 64)
    c.block_table = torch.arange(64, dtype=torch.int32, device=DEV)[None]
    q = _queries(1, 4, 9)
    for at in (1, 17, 62):
        bounds, scales = _random_pools(64, 1, 8)
        bounds[:, :, :, 32:] = 10
        scales[:] = 0.01
        towards = q[0, 2].float().view(2, 4, 16).permute(1, 0, 2).reshape(4, 32)
        bounds[at, 0, :, :32] = (towards.sign() * 127).to(torch.int8)
        assert at in _select(c, q, bounds, scales, 3)[0][0, 0].tolist()


# ---- attention over chosen pages ---------------------------------------------------------------------


def _check_sparse(c, q, n_selected, n_first=1, n_last=1, **more):
    """Bars of test_gpu_attention_precision.py's kernels, as for a window."""
    pools = _bound(c)
    out, selected, lens = _sparse(c, q, pools, n_selected, n_first, n_last, **more)
    want_sel, want_lens = ref.select(q.float().cpu().numpy(), *(x.cpu().numpy() for x in pools), c.table, c.lens, c.heads, n_selected, n_first, n_last)
    assert np.array_equal(selected.cpu().numpy(), want_sel) and np.array_equal(lens.cpu().numpy(), want_lens)
    group = q.shape[1] // c.heads
    for s, L in enumerate(c.lens):
        if L == 0:
            assert not out[s].any()
            continue
        where = {int(p): i for i, p in enumerate(c.table[s]) if p >= 0}
        want = torch.zeros(out[s].shape, dtype=torch.float64, device=DEV)
        for h in range(c.heads):
            pages = [where[x // c.heads] for x in want_sel[s, h].tolist() if x >= 0]
            tokens = torch.cat([torch.arange(p * G, min(L, (p + 1) * G), device=DEV) for p in pages])
            assert len(tokens) == want_lens[s, h]
            k, v = c.k64[s][tokens, h], c.v64[s][tokens, h]
            for g in range(group):
                w = torch.softmax((k * q[s, h * group + g].double()).sum(-1) * c.sm_scale, 0)
                want[h * group + g] = (w[:, None] * v).sum(0)
        off = float((out[s].double() - want).norm() / want.norm())
        assert off <= (1e-6 if c.v_bits == 16 else 2.4e-5), (s, L, off)
    return out, selected, lens


@pytest.mark.parametrize("bits,grouped", FORMATS)
@pytest.mark.parametrize("v_bits", [16, 4, 2])
def test_sparse_every_format(bits, grouped, v_bits):
    _check_sparse(Cache([1500, 515, 60, 1408], 2, bits, grouped, v_bits), _queries(4, 8, 3), 4)


@pytest.mark.parametrize("group", [1, 2, 3, 7, 8, 12, 16])
@pytest.mark.parametrize("dtype", [torch.float16, torch.float32])
@pytest.mark.parametrize("tail", [True, False])
def test_sparse_every_group(group, dtype, tail):
    _check_sparse(Cache([1500, 1, 0, 1281, 128], 2, tail=tail), _queries(5, 2 * group, 4, dtype), 5, 1, 2)


@pytest.mark.parametrize("n_selected,n_first,n_last", [(1, 0, 1), (2, 0, 2), (7, 2, 1), (30, 1, 2), (64, 1, 2)])
@pytest.mark.parametrize("grouped", [False, True])
def test_sparse_every_number(n_selected, n_first, n_last, grouped):
    _check_sparse(Cache([6000, 3000, 900], 2, (4, 4), grouped), _queries(3, 8, 4), n_selected, n_first, n_last, max_seq_len=47 * G)


@pytest.mark.parametrize("group", [1, 2, 3, 7, 12])
@pytest.mark.parametrize("grouped", [False, True])
@pytest.mark.parametrize("v_bits", [4, 2])
def test_sparse_every_group_with_quantized_values(group, grouped, v_bits):
    _check_sparse(Cache([1500, 1, 0, 1281, 128], 2, (4, 4), grouped, v_bits), _queries(5, 2 * group, 4), 5, 1, 2)


@pytest.mark.parametrize("bits,grouped", [((4, 4), False), ((3, 3), False), ((4, 4), True)])
@pytest.mark.parametrize("v_bits", [4, 2])
@pytest.mark.parametrize("lens", [[53] * 4, [5000, 3000], [20000]])
def test_quantized_values_are_summed_as_precisely_as_in_fp32(bits, grouped, v_bits, lens):
    """No further from float64 than attention over the values and keys in fp32, by torch: both round as often as there are tokens; twice for another order."""
    c = Cache(lens, 2, bits, grouped, v_bits)
    q = _queries(len(lens), 8, 3)
    pools = _bound(c)
    outs = [_weigh(c, q)[0], _sparse(c, q, pools, 200)[0]]
    off, plain = np.zeros(2), 0.0
    for s in range(len(lens)):
        for h in range(8):
            def attend(k, v, x):
                w = torch.softmax((k * x).sum(-1) * c.sm_scale, 0)
                return (w[:, None] * v).sum(0)
            k, v = c.k64[s][:, h // 4], c.v64[s][:, h // 4]
            want = attend(k, v, q[s, h].double())
            size = float(want.norm()) ** 2
            plain += float((attend(k.float(), v.float(), q[s, h].float()).double() - want).norm()) ** 2 / size
            off += [float((o[s, h].double() - want).norm()) ** 2 / size for o in outs]
    assert (np.sqrt(off) <= 2 * np.sqrt(plain)).all(), (np.sqrt(off), np.sqrt(plain))


@pytest.mark.parametrize("grouped,group,v_bits", [(False, 4, 16), (True, 1, 16), (True, 4, 16), (False, 4, 4)])
def test_sparse_of_many_long_choices(grouped, group, v_bits):
    """More units than work-groups run at once: hundreds of chosen pages in one chunk.  256 sequences that are the same."""
    c = Cache([640 * G - 5], 2, (4, 4), grouped, v_bits)
    q = _queries(1, 2 * group, 3)
    pools = _bound(c)
    want, spread, slope = (x[0] for x in c.rows(0, q, [c.lens[0] - 1]))
    bar = ref.output_bar(spread, slope, want, ref.page_weights(c, 0, q[0])[1]) if v_bits == 16 else 2.4e-5
    one, selected, lens = _sparse(c, q, pools, 640)
    c.residual = c.residual.expand(256, -1, -1, -1).contiguous()
    c.block_table, c.seq_lens = c.block_table.expand(256, -1).contiguous(), c.seq_lens.expand(256).contiguous()
    out, all_selected, all_lens = _sparse(c, q.expand(256, -1, -1).contiguous(), pools, 640)
    assert bool((out == out[:1]).all()) and bool((all_selected == selected).all()) and bool((all_lens == lens).all())
    for got in (one[0], out[0]):
        assert float((got.double() - want).norm() / want.norm()) <= bar


def test_sparse_of_many_sequences():
    rng = np.random.default_rng(2)
    _check_sparse(Cache([int(n) for n in rng.integers(1, 1200, 70)], 4, (3, 3), v_bits=4), _queries(70, 16, 4), 3)


def test_all_pages_chosen_is_decode_attention():
    """n_selected as large as the sequences: decode attention over the same pages, each head a sequence, but for the order in which the chunks'
    partials are added.  They are 12 at most, with exact weights: each order's sum and denominator are off by 12 * 2^-24 of the terms' sizes, whose sum is at most the
    denominator times the largest value, and the quotient's two roundings add 2^-23 of it each time."""
    c = Cache([1500, 700, 0, 129], 2)
    q = _queries(4, 8, 5)
    out, selected, lens = _sparse(c, q, _bound(c), 12)
    one = c.pq.Layout(D, 4, 4, G, 1)
    size = c.pq.pq_decode_workspace_bytes(one, 8, 4, c.max_seq_len)
    want = torch.empty_like(out)
    c.pq.pq_decode_attention(one, q.view(8, 4, D), c.codes, c.params, c.v_pool, selected.view(8, 12), lens.view(8), c.max_seq_len, float(c.sm_scale),
                             want.view(8, 4, D), torch.empty(size, dtype=torch.uint8, device=DEV), None, c.residual)
    largest = max(float(v.abs().max()) for v in c.v64 if len(v))
    assert float((out - want).abs().max()) <= 2 * (2 * 12 * 2.0 ** -24 + 2 * 2.0 ** -23) * largest
    short = lens.view(8) <= 512                              # one chunk: the same bits
    assert bool(short.any()) and torch.equal(out.view(8, 4, D)[short], want.view(8, 4, D)[short])


def test_a_choice_that_is_given():
    """Another layer's choice: neither bounds nor table are looked at."""
    c = Cache([1500, 700, 0, 129], 2)
    q, other = _queries(4, 8, 5), _queries(4, 8, 6)
    pools = _bound(c)
    selected, lens = _select(c, other, *pools, 4)
    out, _, _ = _sparse(c, q, None, 4, given=(selected.clone(), lens.clone()))
    again, kept, kept_lens = _sparse(c, q, None, 4, given=(selected, lens))
    assert torch.equal(out, again)
    assert torch.equal(kept, _select(c, other, *pools, 4)[0]) and torch.equal(kept_lens, lens)
    own, mine, _ = _sparse(c, other, pools, 4)
    assert torch.equal(mine, selected)
    assert torch.equal(own, _sparse(c, other, None, 4, given=(selected, lens))[0])


@pytest.mark.parametrize("grouped", [False, True])
@pytest.mark.parametrize("sm_scale", [-0.088, 0.0])
def test_negative_and_zero_softmax_scales(sm_scale, grouped):
    """The choice goes by the scores without it."""
    c = Cache([1500, 515, 60], 2, (4, 4), grouped)
    c.sm_scale = sm_scale
    q = _queries(3, 8, 3)
    _check_sparse(c, q, 4)
    _check_weights(c, q)


@pytest.mark.parametrize("grouped", [False, True])
def test_sparse_of_missing_pages(grouped):
    """Pages outside the pool count as no tokens; where all are, the output is zero."""
    c = Cache([1500, 700, 1280], 2, (4, 4), grouped)
    pools = _bound(c)
    q = _queries(3, 8, 3)
    c.block_table[0, 3:] = c.codes.shape[0]
    c.block_table[1, :] = -1
    out, selected, lens = _sparse(c, q, pools, 6, 1, 2)
    assert not out[1].any() and bool((selected[1] == -1).all()) and lens[1].tolist() == [700] * 2
    assert bool((selected[0, :, :3] >= 0).all()) and bool((selected[0, :, 3:] == -1).all())
    tokens = 3 * G
    for h in range(8):
        k, v = c.k64[0][:tokens, h // 4], c.v64[0][:tokens, h // 4]
        w = torch.softmax((k * q[0, h].double()).sum(-1) * c.sm_scale, 0)
        want = (w[:, None] * v).sum(0)
        assert float((out[0, h].double() - want).norm() / want.norm()) <= 1e-6


# ---- attention that sums the pages' weights --------------------------------------------------------------


def _decode(c, q):
    out = torch.empty(q.shape, device=DEV)
    size = c.pq.pq_decode_workspace_bytes(c.layout, *q.shape[:2], c.max_seq_len)
    c.pq.pq_decode_attention(c.layout, q, c.codes, c.params, c.v_pool, c.block_table, c.seq_lens, c.max_seq_len, float(c.sm_scale), out,
                             torch.empty(size, dtype=torch.uint8, device=DEV), None, c.residual, c.v_bits, c.v_params)
    return out


def _check_weights(c, q, **more):
    out, weights = _weigh(c, q, **more)
    # (the grouped quantizer has another kernel for one and two heads; quantized values are summed about the middle of their codes here)
    same = c.v_bits == 16 and (c.layout.angle_quantizer == 0 or q.shape[1] // c.heads > 2)
    assert not same or torch.equal(out, _decode(c, q)), "not the output of decode attention"
    for s, L in enumerate(c.lens):
        pages = (L + G - 1) // G
        assert bool((weights[s, pages:] == -5.0).all()), "written past the sequence's pages"
        if L == 0:
            assert not out[s].any()
            continue
        want, spread, slope = (x[0] for x in c.rows(s, q[s:s + 1], [L - 1]))
        mass, most = ref.page_weights(c, s, q[s])
        off = float((out[s].double() - want).norm() / want.norm())
        assert off <= (ref.output_bar(spread, slope, want, most) if c.v_bits == 16 else 2.4e-5), (s, L, off)
        wrong = (weights[s, :pages].double() - mass).abs() - ref.weight_tolerance(mass, most, q.shape[1])
        assert bool((wrong <= 0).all()), (s, L, float(wrong.max()))
        assert abs(float(weights[s, :pages].double().sum()) - q.shape[1]) <= q.shape[1] * 4e-6
    return out, weights


@pytest.mark.parametrize("bits,grouped", FORMATS)
@pytest.mark.parametrize("v_bits", [16, 4, 2])
def test_weights_every_format(bits, grouped, v_bits):
    _check_weights(Cache([1500, 515, 60, 1408], 2, bits, grouped, v_bits), _queries(4, 8, 3))


@pytest.mark.parametrize("group", [1, 2, 3, 4, 7, 8, 12, 16])
@pytest.mark.parametrize("grouped", [False, True])
@pytest.mark.parametrize("dtype,tail", [(torch.float16, True), (torch.float32, False)])
def test_weights_every_group(group, grouped, dtype, tail):
    _check_weights(Cache([1500, 1, 0, 1281, 128, 700], 2, (4, 4), grouped, tail=tail), _queries(6, 2 * group, 4, dtype), stride=40)


@pytest.mark.parametrize("lens,heads", [([777], 8), ([20000], 8), ([3000] * 24, 8), ([12000, 300, 500, 9000] * 2, 8), ([40000, 30000], 8), ([600] * 300, 1)])
@pytest.mark.parametrize("v_bits", [16, 4])
def test_weights_of_every_kind_of_launch(lens, heads, v_bits):
    """One chunk, several with a merge launch, merged in the kernel, cut on the device, wide work-groups."""
    _check_weights(Cache(lens, heads, v_bits=v_bits), _queries(len(lens), 4 * heads, 4))


def test_weights_add_to_what_there_was():
    c = Cache([1500, 515, 0], 2)
    q = _queries(3, 8, 3)
    _, alone = _weigh(c, q)
    before = torch.rand(alone.shape, device=DEV)
    _, weights = _weigh(c, q, before, 0.75)
    there = alone != -5.0
    assert torch.equal(weights[there], (alone + 0.75 * before)[there]) and bool((weights[~there] == -5.0).all())
    _, in_place = _weigh(c, q, before, 0.75, weights=before)
    assert torch.equal(in_place[there], weights[there]) and in_place is before
    poison = torch.full(alone.shape, float("nan"), device=DEV)
    assert torch.equal(_weigh(c, q, poison, 0.0)[1], alone)


def test_weights_of_masked_pages_are_zero():
    c = Cache([1500, 700], 2)
    q = _queries(2, 8, 3)
    c.block_table[0, 4] = -1
    c.block_table[0, 7] = c.codes.shape[0] + 5
    c.block_table[1, :] = -1
    out, weights = _weigh(c, q)
    assert not weights[0, [4, 7]].any() and not weights[1, :6].any() and not out[1].any()
    assert abs(float(weights[0].sum()) - 8) < 8 * 4e-6


def test_weights_of_a_peaked_softmax():
    """Scores hundreds apart: a page whose tokens weigh nothing has nothing, no infinities on the way."""
    c = Cache([2000], 1, key_scale=30.0)
    q = _queries(1, 4, 3, scale=20.0)
    out, weights = _weigh(c, q)
    assert bool(out.isfinite().all()) and abs(float(weights[0].sum()) - 4) < 4 * 4e-6
    assert bool((weights >= 0).all())


# ---- eviction ----------------------------------------------------------------------------------------


def _evict_inputs(lens, width, seed, ties=False):
    rng = np.random.default_rng(seed)
    table = np.full((len(lens), width), -9, np.int32)
    ids = rng.permutation(len(lens) * width).astype(np.int32)
    weights = np.exp(3 * rng.standard_normal((len(lens), width))).astype(np.float32)
    if ties:
        weights = np.floor(weights).astype(np.float32)
    for s, n in enumerate(lens):
        pages = min(width, (max(0, n) + G - 1) // G)
        table[s, :pages] = ids[s * width:s * width + pages]
    return table, weights


def _evict(pq, table, lens, weights, n_kept, n_first, n_last, in_place=False, room=None):
    t, w = torch.from_numpy(table).to(DEV), torch.from_numpy(weights).to(DEV)
    ta, wa = (t, w) if in_place else (torch.full_like(t, -11), torch.full_like(w, -11.0))
    room = table.size if room is None else room
    la, freed, counts = torch.full((len(lens),), -11, dtype=torch.int32, device=DEV), torch.full((room + 3,), -11, dtype=torch.int32, device=DEV), _ints([-11])
    pq.pq_evict_pages(pq.Layout(D, 4, 4, G, 8), t, _ints(lens), w, n_kept, n_first, n_last, ta, la, wa, freed[:room], counts)
    torch.cuda.synchronize()
    return [x.cpu().numpy() for x in (ta, la, wa, freed, counts)]


def _check_evict(lens, width, n_kept, n_first, n_last, seed=1, ties=False, in_place=False, room=None, change=None):
    import paper_2502_00527_amd as pq
    table, weights = _evict_inputs(lens, width, seed, ties)
    if change:
        change(table, weights)
    want = ref.evict(table, lens, weights, n_kept, n_first, n_last)
    ta, la, wa, freed, counts = _evict(pq, table, lens, weights, n_kept, n_first, n_last, in_place, room)
    for s, n in enumerate(lens):
        pages = min(width, (max(0, n) + G - 1) // G)
        assert np.array_equal(ta[s, :pages], want[0][s, :pages]) and np.array_equal(wa[s, :pages], want[2][s, :pages], equal_nan=True), s
        assert np.array_equal(ta[s, pages:], table[s, pages:] if in_place else np.full(width - pages, -11))
    assert np.array_equal(la, want[1])
    n = len(want[3]) if room is None else min(room, len(want[3]))
    assert counts[0] == len(want[3]) and np.array_equal(freed[:n], want[3][:n]) and (freed[n:] == -11).all()


LENS = [10000, 0, 1, 127, 128, 129, 1280, 1281, 9999, 5120, -4]


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("ties", [False, True])
@pytest.mark.parametrize("n_kept,n_first,n_last", [(10, 1, 2), (0, 0, 0), (1, 0, 0), (5, 4, 4), (40, 0, 1), (79, 2, 0), (1000, 1, 1), (3, 100, 2),
                                                    (2 ** 31 - 1, 0, 0), (3, 2 ** 31 - 1, 1), (3, 1, 2 ** 31 - 1), (0, 2 ** 31 - 1, 2 ** 31 - 1)])
def test_evictions(n_kept, n_first, n_last, ties, in_place):
    _check_evict(LENS, 79, n_kept, n_first, n_last, ties=ties, in_place=in_place)


@pytest.mark.parametrize("pages", [255, 256, 257, 1023, 1025, 4096, 4097, 7000])
@pytest.mark.parametrize("kept", [3, 0.5, -1])
def test_evictions_of_long_sequences(pages, kept):
    n_kept = kept if kept == 3 else (pages // 2 if kept == 0.5 else pages - 1)
    for in_place in (False, True):
        _check_evict([pages * G, pages * G - 100, pages * G // 3], pages, n_kept, 1, 2, seed=pages, ties=pages % 2 == 0, in_place=in_place)


def test_evictions_of_many_sequences():
    lens = [int(n) for n in np.random.default_rng(7).integers(0, 3000, 1500)]
    _check_evict(lens, 24, 9, 1, 2)


def test_two_sequences_that_share_pages():
    """A page that two rows hold is in the list of freed ones as often as it was given up, and stays where it was kept."""
    def change(table, weights):
        table[8, :20] = table[0, :20]
        weights[8, :20] = weights[0, :20] + 1
    _check_evict(LENS, 79, 10, 1, 2, change=change)


def test_evicted_pages_beyond_the_list():
    _check_evict(LENS, 79, 10, 1, 2, room=17)
    _check_evict(LENS, 79, 10, 1, 2, room=0)


def test_weights_that_are_no_numbers():
    def change(table, weights):
        weights[0, 3:60:4] = np.nan
        weights[0, 5:60:4] = np.inf
        weights[8, :] = np.nan
        weights[9, :] = -0.0
        weights[9, 1::2] = 0.0
        weights[6, 2] = -np.inf
    _check_evict(LENS, 79, 4, 1, 2, change=change)


def test_evictions_leave_sequences_longer_than_the_table():
    _check_evict([3000, 1000, 2000], 10, 4, 1, 1)


def test_no_sequences():
    import paper_2502_00527_amd as pq
    counts = _ints([5])
    e, f = torch.empty((0, 4), dtype=torch.int32, device=DEV), torch.empty((0, 4), device=DEV)
    none = torch.empty(0, dtype=torch.int32, device=DEV)
    pq.pq_evict_pages(pq.Layout(D, 4, 4, G, 8), e, none, f, 3, 1, 1, e.clone(), none.clone(), f.clone(), none.clone(), counts)
    assert int(counts) == 0


# ---- together --------------------------------------------------------------------------------------------


class _Serving:
    """A serving loop: every step appends a token of each sequence, bounds the pages that are complete, attends -- over chosen pages and
    with weights, in turn -- and now and then evicts.  What is cached is kept beside it in float64."""

    def __init__(self, lens, heads=2, group=4, pages=60, width=16, bits=(4, 4), grouped=False, seed=0):
        import paper_2502_00527_amd as pq
        self.pq, self.heads, self.group, self.bits, self.seqs, self.width = pq, heads, group, bits, len(lens), width
        self.layout = pq.Layout(D, *bits, G, heads, int(grouped))
        self.rng = np.random.default_rng(seed)
        n = len(lens)
        self.codes = torch.zeros((pages, heads, 4, G, 2 * sum(bits)), dtype=torch.uint8, device=DEV)
        self.params = torch.zeros((pages, heads, *((2,) if grouped else ()), 64, 2), dtype=torch.float16, device=DEV)
        self.v_pool = torch.zeros((pages, heads, G, D), dtype=torch.float16, device=DEV)
        self.bounds, self.scales = torch.zeros((pages, heads, 4, 64), dtype=torch.int8, device=DEV), torch.zeros((pages, heads, 4), device=DEV)
        self.residual = torch.zeros((n, heads, G, D), dtype=torch.float16, device=DEV)
        self.table = torch.full((n, width), -1, dtype=torch.int32, device=DEV)
        self.weights = torch.zeros((n, width), device=DEV)
        self.lens = torch.zeros(n, dtype=torch.int32, device=DEV)
        self.free = torch.arange(pages, dtype=torch.int32, device=DEV)
        self.most = width * G
        self.append(lens)

    def tokens(self, n):
        k = self.rng.standard_normal((n, self.heads, D)).astype(np.float16)
        v = self.rng.standard_normal((n, self.heads, D)).astype(np.float16)
        return torch.from_numpy(k).to(DEV), torch.from_numpy(v).to(DEV)

    def append(self, new):
        pq = self.pq
        total = sum(new)
        starts, counts = torch.zeros(self.seqs + 1, dtype=torch.int32, device=DEV), _ints([0, 0])
        slots, after = torch.zeros(total, dtype=torch.int64, device=DEV), torch.zeros_like(self.lens)
        pq.pq_plan_pages(self.layout, self.lens, _ints(list(new)), self.free, self.table, starts, slots, after, counts)
        keys, values = self.tokens(total)
        pq.pq_append_chunk(self.layout, keys, values, starts, self.lens, slots, self.residual, self.table, self.codes, self.params, self.v_pool)
        pq.pq_bound_pages(self.layout, self.codes, self.params, self.table, self.lens, after, max(new), self.bounds, self.scales)
        self.lens = after
        self.free = self.free[int(counts[0]):]

    def cached(self, s):
        """float64 keys and values of sequence s as the cache holds them."""
        from oracle import cache_format, polar
        n = int(self.lens[s])
        pages = (n + G - 1) // G
        ids = self.table[s, :pages].long()
        assert len(set(ids.tolist())) == pages and int(ids.min()) >= 0
        whole = n // G
        k = np.zeros((n, self.heads, D))
        if whole:
            a, c, *par = cache_format.unpack_pages(self.codes[ids[:whole]].cpu().numpy(), self.params[ids[:whole]].cpu().numpy(), whole * G, *self.bits)
            k[:whole * G] = polar.dequant_keys(a, c, par[0], par[1], self.bits[1], G, *par[2:])
        if n % G:
            k[whole * G:] = self.residual[s, :, :n % G].permute(1, 0, 2).double().cpu().numpy()
        v = self.v_pool[ids].permute(0, 2, 1, 3).reshape(-1, self.heads, D)[:n].double()
        return torch.from_numpy(k).to(DEV), v

    def attention(self, q, choose=None):
        """float64 outputs and page weights; choose(s, h): page numbers."""
        outs, masses = torch.zeros(q.shape, dtype=torch.float64, device=DEV), torch.zeros((self.seqs, self.width), dtype=torch.float64, device=DEV)
        for s in range(self.seqs):
            k, v = self.cached(s)
            for h in range(q.shape[1]):
                kv = h // self.group
                at = torch.arange(len(k), device=DEV)
                if choose is not None:
                    at = torch.cat([at[p * G:(p + 1) * G] for p in choose(s, kv)])
                w = torch.softmax((k[at, kv] * q[s, h].double()).sum(-1) / np.sqrt(D), 0)
                outs[s, h] = (w[:, None] * v[at, kv]).sum(0)
                masses[s].index_add_(0, at // G, w)
        return outs, masses

    def near(self, got, want, bar):
        assert float((got.double() - want).norm() / want.norm()) <= bar

    def sparse_step(self, n_selected, seed):
        pq = self.pq
        q = _queries(self.seqs, self.heads * self.group, seed)
        work = torch.empty(pq.pq_sparse_workspace_bytes(self.layout, *q.shape[:2], self.most, n_selected), dtype=torch.uint8, device=DEV)
        selected, lens = torch.zeros((self.seqs, self.heads, n_selected), dtype=torch.int32, device=DEV), torch.zeros((self.seqs, self.heads), dtype=torch.int32, device=DEV)
        out = torch.empty(q.shape, device=DEV)
        pq.pq_sparse_attention(self.layout, q, self.codes, self.params, self.v_pool, self.bounds, self.scales, self.table, self.lens, self.most, 1, 1,
                               1 / np.sqrt(D), selected, lens, out, work, self.residual)
        table, heads = self.table.tolist(), self.heads
        want_sel, want_lens = ref.select(q.float().cpu().numpy(), self.bounds.cpu().numpy(), self.scales.cpu().numpy(), self.table.cpu().numpy(), self.lens.tolist(),
                                         heads, n_selected, 1, 1)
        assert np.array_equal(selected.cpu().numpy(), want_sel) and np.array_equal(lens.cpu().numpy(), want_lens)
        self.near(out, self.attention(q, lambda s, h: [table[s].index(x // heads) for x in want_sel[s, h].tolist() if x >= 0])[0], 1e-6)

    def weights_step(self, decay, seed):
        pq = self.pq
        q = _queries(self.seqs, self.heads * self.group, seed)
        work = torch.empty(pq.pq_weights_workspace_bytes(self.layout, *q.shape[:2], self.most), dtype=torch.uint8, device=DEV)
        out, before = torch.empty(q.shape, device=DEV), self.weights.clone()
        pq.pq_decode_attention_weights(self.layout, q, self.codes, self.params, self.v_pool, self.table, self.lens, self.most, 1 / np.sqrt(D), out, self.weights,
                                       work, self.weights, decay, self.residual)
        want, mass = self.attention(q)
        self.near(out, want, 1e-6)
        for s, n in enumerate(self.lens.tolist()):
            pages = (n + G - 1) // G
            self.near(self.weights[s, :pages], decay * before[s, :pages].double() + mass[s, :pages], 2e-6)
            assert torch.equal(self.weights[s, pages:], before[s, pages:])

    def evict_step(self, n_kept):
        freed, counts, after = torch.full((self.table.numel(),), -1, dtype=torch.int32, device=DEV), _ints([0]), torch.zeros_like(self.lens)
        want = ref.evict(self.table.cpu().numpy(), self.lens.tolist(), self.weights.cpu().numpy(), n_kept, 1, 1)
        self.pq.pq_evict_pages(self.layout, self.table, self.lens, self.weights, n_kept, 1, 1, self.table, after, self.weights, freed, counts)
        assert np.array_equal(self.table.cpu().numpy(), want[0]) and np.array_equal(after.cpu().numpy(), want[1]) and np.array_equal(self.weights.cpu().numpy(), want[2])
        assert np.array_equal(freed[:int(counts)].cpu().numpy(), want[3])
        self.free = torch.cat([self.free, freed[:int(counts)]])
        self.lens = after


@pytest.mark.parametrize("grouped", [False, True])
def test_a_serving_loop_under_a_budget(grouped):
    """Pages that were given up are filled again, bounds follow, lengths stay under the budget."""
    loop = _Serving([700, 130, 1000], pages=26, width=12, grouped=grouped)
    for step in range(12):
        loop.append([40, 40 if step % 3 else 1, 60])
        loop.sparse_step(4, 100 + step)
        loop.weights_step(0.9, 200 + step)
        if step % 2:
            loop.evict_step(6)
            assert max(loop.lens.tolist()) <= 6 * G
    held = [int(x) for s, n in enumerate(loop.lens.tolist()) for x in loop.table[s, :(n + G - 1) // G]]
    assert len(set(held)) == len(held) and not set(held) & set(loop.free.tolist())
    assert len(held) + len(loop.free) == 26


@pytest.mark.parametrize("lens,heads,v_bits", [([1500, 515, 60, 1408], 2, 16), ([40000, 9000, 300, 12000], 8, 16), ([40000, 9000, 300, 12000], 8, 4)])
def test_captured_steps(lens, heads, v_bits):
    """All five calls in one graph, replayed with other queries and lengths between, each replay against the eager calls: one work-group a unit, and units shared
    among work-groups, chunks cut on the device and merged in the kernel."""
    c = Cache(lens, heads, v_bits=v_bits)
    pq, n_q = c.pq, 4 * heads
    q = _queries(4, n_q, 3)
    bounds, scales = _bound_pools(c)
    work = torch.empty(pq.pq_sparse_workspace_bytes(c.layout, 4, n_q, c.max_seq_len, 4), dtype=torch.uint8, device=DEV)
    work2 = torch.empty(pq.pq_weights_workspace_bytes(c.layout, 4, n_q, c.max_seq_len), dtype=torch.uint8, device=DEV)
    selected, sel_lens = torch.zeros((4, heads, 4), dtype=torch.int32, device=DEV), torch.zeros((4, heads), dtype=torch.int32, device=DEV)
    out, out2 = torch.zeros(q.shape, device=DEV), torch.zeros(q.shape, device=DEV)
    width = c.block_table.shape[1]
    weights, after_w = torch.zeros((4, width), device=DEV), torch.zeros((4, width), device=DEV)
    after_t, after_l = torch.zeros_like(c.block_table), torch.zeros_like(c.seq_lens)
    freed, counts = torch.zeros(4 * width, dtype=torch.int32, device=DEV), _ints([0])

    def step():
        pq.pq_bound_pages(c.layout, c.codes, c.params, c.block_table, None, c.seq_lens, c.max_seq_len, bounds, scales)
        pq.pq_sparse_attention(c.layout, q, c.codes, c.params, c.v_pool, bounds, scales, c.block_table, c.seq_lens, c.max_seq_len, 1, 1, float(c.sm_scale),
                               selected, sel_lens, out, work, c.residual, c.v_bits, c.v_params)
        pq.pq_decode_attention_weights(c.layout, q, c.codes, c.params, c.v_pool, c.block_table, c.seq_lens, c.max_seq_len, float(c.sm_scale), out2, weights, work2,
                                       None, 1.0, c.residual, c.v_bits, c.v_params)
        pq.pq_evict_pages(c.layout, c.block_table, c.seq_lens, weights, 5, 1, 1, after_t, after_l, after_w, freed, counts)
        return [x.clone() for x in (bounds, scales, selected, sel_lens, out, out2, weights, after_t, after_l, after_w, freed, counts)]

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = step()
    for i, now in enumerate([c.lens, [1000, 515, 0, 1281], [lens[0] - 371, 500, 60, 640], c.lens]):
        q.copy_(_queries(4, n_q, 50 + i))
        c.seq_lens.copy_(_ints(now))
        graph.replay()
        torch.cuda.synchronize()
        replayed = [x.clone() for x in captured]
        eager = step()
        torch.cuda.synchronize()
        for a, b in zip(replayed, eager):
            assert torch.equal(a.nan_to_num(nan=-3.0) if a.is_floating_point() else a, b.nan_to_num(nan=-3.0) if b.is_floating_point() else b)


@pytest.mark.parametrize("grouped,v_bits", [(False, 16), (True, 16), (False, 4)])
def test_pages_far_into_the_pools(grouped, v_bits):
    """Bytes of codes and values past 2^32: the same as near the pools' beginning.  (By a multiple of 8 pages: values are read in an order
    that depends on the page's id modulo 8.)"""
    c = Cache([1500, 515, 60, 1408], 2, (4, 4), grouped, v_bits)
    q = _queries(4, 8, 3)

    def results():
        pools = _bound(c)
        return pools, _sparse(c, q, pools, 4), _weigh(c, q)

    near = results()
    n = c.codes.shape[0]
    far = ((1 << 32) // (2 * 4 * G * 16) + 15) // 8 * 8
    for name in ("codes", "params", "v_pool", "v_params"):
        small = getattr(c, name)
        if small is not None:
            big = torch.empty((far + n, *small.shape[1:]), dtype=small.dtype, device=DEV)
            big[far:] = small
            setattr(c, name, big)
    assert c.codes.nbytes > 1 << 32 and c.v_pool.nbytes > 1 << 32
    c.block_table = torch.where(c.block_table >= 0, c.block_table + far, c.block_table)
    c.table = np.where(c.table >= 0, c.table + far, c.table)
    pools, sparse, weigh = results()
    for a, b in zip(near[0], pools):
        assert torch.equal(a.view(torch.uint8), b[far:].view(torch.uint8))
    out, selected, lens = near[1]
    assert torch.equal(sparse[0], out) and torch.equal(sparse[1], torch.where(selected >= 0, selected + far * c.heads, selected)) and torch.equal(sparse[2], lens)
    assert torch.equal(weigh[0], near[2][0]) and torch.equal(weigh[1], near[2][1])


def test_bounds_far_into_their_pool():
    c = _Plain([700 * G], 8, 700)
    bounds, scales = _random_pools(700, 8, 4)
    q = _queries(1, 32, 5)
    want = _select(c, q, bounds, scales, 20)
    far = (1 << 32) // (8 * 256) + 5
    pools = [torch.empty((far + 700, *x.shape[1:]), dtype=x.dtype, device=DEV) for x in (bounds, scales)]
    for big, small in zip(pools, (bounds, scales)):
        big[far:] = small
    c.block_table += far
    got = _select(c, q, *pools, 20)
    assert torch.equal(got[0], want[0] + far * 8) and torch.equal(got[1], want[1])


def test_one_workspace_for_calls_of_many_shapes():
    """What one call leaves there is nothing to the next: arrival words lie where another shape's keys were."""
    import paper_2502_00527_amd as pq
    cases = []
    for seqs, heads, pages in [(1, 1, 300), (3, 1, 5000), (2, 8, 1030), (1, 2, 9000), (1, 4, 1500), (40, 2, 700)]:
        c = _Plain([pages * G] * seqs, heads, 500, seed=pages)
        cases.append((c, _queries(seqs, 4 * heads, pages), *_random_pools(500, heads, pages)))
    wants = [_select(*case, 17) for case in cases]
    work = torch.from_numpy(np.random.default_rng(3).integers(0, 256, max(pq.pq_select_workspace_bytes(c.layout, len(c.lens), c.max_seq_len) for c, *_ in cases)).astype(np.uint8)).to(DEV)
    for at in list(range(6)) + [4, 0, 3, 3, 1, 5, 2, 0]:
        c, q, bounds, scales = cases[at]
        selected, lens = torch.zeros_like(wants[at][0]), torch.zeros_like(wants[at][1])
        pq.pq_select_pages(c.layout, q, bounds, scales, c.block_table, c.seq_lens, c.max_seq_len, 1, 1, selected, lens, work)
        assert torch.equal(selected, wants[at][0]) and torch.equal(lens, wants[at][1]), at


def test_calls_on_another_stream():
    """Two streams at once, a workspace each."""
    c = Cache([3000, 515, 60, 1408], 2)
    pools = _bound(c)
    qs = [_queries(4, 8, 3), _queries(4, 8, 4)]
    want = [(_sparse(c, q, pools, 4)[0], *_weigh(c, q)) for q in qs]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(5):
        got = []
        for q, stream in zip(qs, streams):
            stream.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(stream):
                work = torch.empty(c.pq.pq_weights_workspace_bytes(c.layout, 4, 8, c.max_seq_len), dtype=torch.uint8, device=DEV)
                sparse = torch.empty(c.pq.pq_sparse_workspace_bytes(c.layout, 4, 8, c.max_seq_len, 4), dtype=torch.uint8, device=DEV)
                out, out2, w = torch.empty(q.shape, device=DEV), torch.empty(q.shape, device=DEV), torch.full((4, c.block_table.shape[1]), -5.0, device=DEV)
                sel, lens = torch.empty((4, 2, 4), dtype=torch.int32, device=DEV), torch.empty((4, 2), dtype=torch.int32, device=DEV)
                c.pq.pq_sparse_attention(c.layout, q, c.codes, c.params, c.v_pool, *pools, c.block_table, c.seq_lens, c.max_seq_len, 1, 1, float(c.sm_scale), sel, lens,
                                         out, sparse, c.residual)
                c.pq.pq_decode_attention_weights(c.layout, q, c.codes, c.params, c.v_pool, c.block_table, c.seq_lens, c.max_seq_len, float(c.sm_scale), out2, w, work,
                                                 None, 1.0, c.residual)
                got.append((out, out2, w))
        torch.cuda.synchronize()
        for a, b in zip(want, got):
            for x, y in zip(a, b):
                assert torch.equal(x, y)


def test_both_ways_of_marshalling(monkeypatch):
    """The calls give the same through the native module and through ctypes."""
    import paper_2502_00527_amd as pq
    c = Cache([1500, 515, 60, 1408], 2, v_bits=4)
    q = _queries(4, 8, 3)

    def all_calls():
        pools = _bound(c, _ints([0, 128, 0, 3]), c.seq_lens)
        out, sel, lens = _sparse(c, q, _bound(c), 4)
        table, weights = c.block_table.cpu().numpy(), _weigh(c, q)[1]
        return [*(x for x in pools), out, sel, lens, *_select(c, q, *_bound(c), 5), weights, *(torch.from_numpy(x) for x in _evict(pq, table, c.lens, weights.cpu().numpy(), 4, 1, 1))]

    native = all_calls()
    assert type(pq._calls).__name__ != "_ByCtypes"
    monkeypatch.setattr(pq, "_calls", pq._ByCtypes())
    for a, b in zip(native, all_calls()):
        assert torch.equal(a.nan_to_num(nan=-3.0) if a.is_floating_point() else a, b.nan_to_num(nan=-3.0) if b.is_floating_point() else b)


@pytest.mark.parametrize("v_bits", [16, 4])
def test_one_workspace_for_a_batch_that_shrinks(v_bits):
    """A workspace of the largest batch, with anything in it, serves smaller batches and shorter bounds of the lengths: the same results as with one of their own.  Above
    and below the number of units that are shared among work-groups."""
    import paper_2502_00527_amd as pq
    rng = np.random.default_rng(4)
    lens = [270 * G, 50 * G - 5] + [int(n) for n in rng.integers(1, 3000, 34)]
    c = Cache(lens, 8, v_bits=v_bits)
    q, pools, whole = _queries(len(lens), 16, 3), _bound(c), (c.block_table, c.seq_lens, c.residual)
    sizes = [pq.pq_select_workspace_bytes(c.layout, len(lens), c.max_seq_len), pq.pq_sparse_workspace_bytes(c.layout, len(lens), 16, c.max_seq_len, 12),
             pq.pq_weights_workspace_bytes(c.layout, len(lens), 16, c.max_seq_len)]
    works = [torch.from_numpy(rng.integers(0, 256, n + 256).astype(np.uint8)).to(DEV) for n in sizes]
    for work, n in zip(works, sizes):
        work[n:] = 0x5A
    for n, most in [(36, 270 * G), (31, 270 * G), (5, 270 * G), (1, 270 * G), (32, 270 * G), (2, 260 * G), (36, 257 * G), (3, 8 * G)]:
        c.block_table, c.seq_lens, c.residual = (x[:n].contiguous() for x in whole)
        mine = q[:n].contiguous()
        want = [*_select(c, mine, *pools, 12, max_seq_len=most), *_sparse(c, mine, pools, 12, max_seq_len=most), *_weigh(c, mine, max_seq_len=most, stride=c.block_table.shape[1])]
        got = [torch.full_like(x, -5) for x in want]
        pq.pq_select_pages(c.layout, mine, *pools, c.block_table, c.seq_lens, most, 1, 1, got[0], got[1], works[0][:sizes[0]])
        pq.pq_sparse_attention(c.layout, mine, c.codes, c.params, c.v_pool, *pools, c.block_table, c.seq_lens, most, 1, 1, float(c.sm_scale), got[3], got[4], got[2],
                               works[1][:sizes[1]], c.residual, c.v_bits, c.v_params)
        pq.pq_decode_attention_weights(c.layout, mine, c.codes, c.params, c.v_pool, c.block_table, c.seq_lens, most, float(c.sm_scale), got[5], got[6],
                                       works[2][:sizes[2]], None, 1.0, c.residual, c.v_bits, c.v_params)
        torch.cuda.synchronize()
        for a, b in zip(got, want):
            assert torch.equal(a, b), (n, most)
        for work, size in zip(works, sizes):
            assert bool((work[size:] == 0x5A).all()), "written past the workspace"


def test_pages_are_planned_from_an_eviction_with_missing_ones():
    """Sequences that got no pages while none were free give up entries without a page: what is planned from the list of freed ones passes over these, and every new token has a
    slot of its own."""
    import paper_2502_00527_amd as pq
    lay, width = pq.Layout(D, 4, 4, G, 2), 12
    table = torch.full((3, width), -1, dtype=torch.int32, device=DEV)

    def plan(lens, new, free):
        starts, counts, after = torch.zeros(4, dtype=torch.int32, device=DEV), _ints([0, 0]), torch.zeros_like(lens)
        slots = torch.full((sum(new),), -9, dtype=torch.int64, device=DEV)
        pq.pq_plan_pages(lay, lens, _ints(new), free, table, starts, slots, after, counts)
        return after, slots, counts.tolist()

    lens, slots, counts = plan(_ints([0, 0, 0]), [3 * G, 9 * G, 5 * G], torch.arange(17, dtype=torch.int32, device=DEV))
    assert counts == [17, 17 * G] and bool((slots >= 0).all())
    lens, slots, counts = plan(lens, [5 * G, 0, 0], _ints([]))
    assert counts == [5, 5 * G] and bool((slots == -1).all())              # the first sequence has three pages, five are missing
    weights = torch.rand((3, width), device=DEV) + 0.1
    weights[0, 3:8] = 0
    freed, count, after = torch.full((40,), -1, dtype=torch.int32, device=DEV), _ints([0]), torch.zeros_like(lens)
    pq.pq_evict_pages(lay, table, lens, weights, 4, 0, 0, table, after, weights, freed, count)
    # four entries of the first sequence, those without a page, which weigh nothing; five of the second one, one of the third
    assert int(count) == 4 + 5 + 1 and bool((freed[:4] == -1).all()) and bool((freed[4:10] >= 0).all())
    held = set(table[table >= 0].tolist())
    lens, slots, counts = plan(after, [G, G, G], freed[:10])
    assert counts == [7, 3 * G] and bool((slots >= 0).all()) and len(set(slots.tolist())) == 3 * G
    assert (slots[::G] // G).tolist() == freed[4:7].tolist() and not set(freed[4:7].tolist()) & held
    # more pages than there are free ones: one is short
    lens, slots, counts = plan(lens, [2 * G, 2 * G, 0], freed[7:10])
    assert counts == [4, 4 * G] and int((slots < 0).sum()) == G and bool((slots[:3 * G] >= 0).all())


@pytest.mark.parametrize("bits,grouped", [((4, 4), False), ((3, 3), True)])
@pytest.mark.parametrize("v_bits", [4, 2])
def test_codes_are_summed_about_their_middle(bits, grouped, v_bits):
    """Where it shows: queries of zeros, so that every weight is exactly 1 and nothing but the sums is rounded, over 640 pages whose mean is small against the values' range, by so many
    units that chunks are long.  In units of 2^-24 / sqrt(3) = 3.4e-8 of a value's size: a token's zero point and its codes' middle are 2.7.  About the middle, 32 tokens' codes and middles
    are two products of at most 8 roundings each at up to 32 * 2.7 + the sum so far, 64 roundings a page at 86 + 0.7 of the chunk's sum.  A wavefront has at most 160 pages (chosen ones: one chunk), a sum of 143 and
    so an error of sqrt(160 * 64) * (86 + 100) = 18800, 132 of the sum: 4.6e-6; 16 pages with the weights, 91: 3.1e-6; 8 with grouped angles.  What joins them adds a few roundings of the sum.
    As they are, codes and zero points are sums of 2.7 a token before they meet.  At one rounding a product a wavefront of 8 pages has sqrt(32) * 1380 = 7800 of a sum of 32: 245, 8.4e-6, of 16 pages 1.7e-5: 2.7 times
    the bounds above and more."""
    c = Cache([640 * G - 5], 2, bits, grouped, v_bits)
    pools = _bound(c)
    c.residual = c.residual.expand(256, -1, -1, -1).contiguous()
    c.block_table, c.seq_lens = c.block_table.expand(256, -1).contiguous(), c.seq_lens.expand(256).contiguous()
    q = torch.zeros((256, 8, D), dtype=torch.float16, device=DEV)
    want = c.v64[0].mean(0)                                              # [KV head, d]
    off = []
    for out in (_weigh(c, q)[0], _sparse(c, q, pools, 640)[0], _decode(c, q)):           # pq_decode_attention sums codes as they are
        assert bool((out == out[:1]).all())
        off.append(float((out[0].view(2, 4, D).double() - want[:, None]).norm() / want.norm() / 2))
    # (2 bits of a code, 11 of its scale and 10 of a wavefront's 1024 tokens with grouped angles are 23 bits: nothing is rounded before the quotient, centred or not.  That is two
    # roundings, sqrt(2) * 2^-24 / sqrt(3) = 5e-8)
    assert max(off[:2]) <= 4.6e-6 and off[0] <= max(off[2] / 2, 2.0 ** -23), off


@pytest.mark.parametrize("heads,group", [(4, 10), (5, 7), (8, 8), (3, 16), (6, 12)])
@pytest.mark.parametrize("lens", [[3000, 1], [700, 90, 0], [2000] * 20])
def test_weights_of_many_query_heads(heads, group, lens):
    """More than 32 of them, also such as are no multiple of 16: a launch that leaves its chunks to the merge, sequences of one chunk, and chunks merged in the kernel."""
    _check_weights(Cache(lens, heads), _queries(len(lens), heads * group, 3))


@pytest.mark.parametrize("lens,heads,group", [([3000, 1300], 4, 10), ([700, 900], 8, 8), ([3000, 1300], 2, 2)])
@pytest.mark.parametrize("grouped", [False, True])
def test_weights_of_missing_pages_and_many_heads(lens, heads, group, grouped):
    """The others' weights are those over the tokens that are there, with chunks merged by the second launch, a whole one missing among them, and with one chunk a sequence."""
    c = Cache(lens, heads, (4, 4), grouped)
    n_q = heads * group
    q = _queries(len(lens), n_q, 3)
    gone = [[4, 5, 6, 7, 1], [0, 6]]
    for s, pages in enumerate(gone):
        c.block_table[s, pages] = torch.tensor([-1, c.codes.shape[0]], dtype=torch.int32, device=DEV).repeat(3)[:len(pages)]
    out, weights = _weigh(c, q)
    for s, L in enumerate(lens):
        there = torch.cat([torch.arange(p * G, min(L, (p + 1) * G), device=DEV) for p in range((L + G - 1) // G) if p not in gone[s]])
        mass, most = torch.zeros((L + G - 1) // G, dtype=torch.float64, device=DEV), 0.0
        for h in range(n_q):
            k, v = c.k64[s][there, h // group], c.v64[s][there, h // group]
            terms = k * q[s, h].double()
            w = torch.softmax(terms.sum(-1) * c.sm_scale, 0)
            mass.index_add_(0, there // G, w)
            size = float(terms.abs().sum(-1).max()) * float(c.sm_scale)
            most = max(most, size)
            want, spread = (w[:, None] * v).sum(0), ((w * w)[:, None] * (v * v)).sum(0).sqrt()
            pair_q, pair_k = (x[..., :64] ** 2 + x[..., 64:] ** 2 for x in (q[s, h].double(), k))
            slope = (pair_q * pair_k).sum(-1).max().sqrt() * float(c.sm_scale)
            assert float((out[s, h].double() - want).norm() / want.norm()) <= ref.output_bar(spread, slope, want, size)
        held = [p for p in gone[s] if p < len(mass)]
        assert not weights[s, held].any()
        wrong = (weights[s, :len(mass)].double() - mass).abs() - ref.weight_tolerance(mass, most, n_q)
        assert bool((wrong <= 0).all()), (s, float(wrong.max()))


@pytest.mark.parametrize("bits,grouped", FORMATS)
@pytest.mark.parametrize("key_scale", [1.0, 30.0])
def test_a_score_is_a_bound(bits, grouped, key_scale):
    """No key of a page has a product with a query above (score + sum over the blocks of u_b (sum of |q8_i| + 64 * 32)) / 127: centres, half-widths and queries are each off by half a step, a channel by
    |q8| / 2 + |q8| / 2 + (|centre| + half-width) / 2 <= |q8| + 63.5 steps; the rest of the 64 is what fp32 rounds.  One channel of 128 is eight times the others' size, and its block's scale with it."""
    c = Cache([1536, 700], 2, bits, grouped, key_scale=key_scale)
    q = _queries(2, 8, 7, torch.float32)
    q[0, 1, 5], q[1, :, 64:] = 20.0, q[1, :, 64:] * 0.01
    bounds, scales = (x.cpu().numpy() for x in _bound(c))
    for s, L in enumerate(c.lens):
        for h in range(2):
            whole = L // G
            mine, ids = q[s, 4 * h:4 * h + 4].cpu().numpy(), c.table[s, :whole]
            score = ref.scores_of(mine, bounds[ids, h], scales[ids, h]).astype(np.float64)
            slack = np.zeros((4, whole))
            for b in range(4):
                part = np.concatenate([mine[:, 16 * b:16 * b + 16], mine[:, 64 + 16 * b:80 + 16 * b]], -1).astype(np.float64)
                m = abs(part).max()
                q8 = abs(np.rint(part * (127 / m))).sum(-1)
                slack += (q8[:, None] + 64 * 32) * (m * scales[ids, h, b].astype(np.float64))[None]
            k = c.k64[s][:whole * G, h].view(whole, G, D).cpu().numpy()
            top = np.einsum("ptd,gd->gpt", k, mine.astype(np.float64)).max(-1)               # [query, page]
            assert (127 * top <= score[None] + slack).all()
