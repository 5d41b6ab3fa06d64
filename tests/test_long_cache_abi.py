"""Host-side logic of the entry points for long caches under a budget of pages: sizes and refusals.  No GPU needed: every call here
returns before anything is launched."""
import ctypes

import pytest

import paper_2502_00527_amd as pq

LAY = pq.Layout(128, 4, 4, 128, 8)
FAKE, NULL, ODD, HALF = ctypes.c_void_p(4096), ctypes.c_void_p(0), ctypes.c_void_p(4098), ctypes.c_void_p(4104)
INVALID, UNSUPPORTED, WORKSPACE = -1, -2, -3


@pytest.fixture(scope="module")
def lib():
    import os
    if not os.path.exists(pq.lib_path()):
        from paper_2502_00527_amd import build
        build.build(verbose=False)
    return pq.load_library()


def _call(lib, name, defaults, **changes):
    args = dict(defaults)
    assert set(changes) <= set(args)
    args.update(changes)
    layout = args.pop("layout")
    return getattr(lib, name)(None if layout is None else ctypes.byref(layout), *args.values(), NULL)


BOUND = dict(layout=LAY, codes=FAKE, params=FAKE, pages=16, table=FAKE, width=8, before=FAKE, after=FAKE, n_seqs=2, most=100, bounds=FAKE, scales=FAKE)
SELECT = dict(layout=LAY, q=FAKE, dtype=0, n_seqs=2, heads=32, bounds=FAKE, scales=FAKE, pages=16, table=FAKE, width=8, lens=FAKE, max_seq_len=1024, chosen=4,
              first=1, last=1, selected=FAKE, selected_lens=FAKE, workspace=NULL, size=0)
SPARSE = dict(layout=LAY, q=FAKE, dtype=0, n_seqs=2, heads=32, codes=FAKE, params=FAKE, v_pool=FAKE, v_bits=16, v_params=NULL, bounds=FAKE, scales=FAKE, pages=16,
              table=FAKE, width=8, lens=FAKE, max_seq_len=1024, chosen=4, first=1, last=1, scale=0.1, selected=FAKE, selected_lens=FAKE, out=FAKE, residual=NULL,
              workspace=NULL, size=0)
WEIGHTS = dict(layout=LAY, q=FAKE, dtype=0, n_seqs=2, heads=32, codes=FAKE, params=FAKE, v_pool=FAKE, v_bits=16, v_params=NULL, pages=16, table=FAKE, width=8,
               lens=FAKE, max_seq_len=1024, scale=0.1, out=FAKE, before=FAKE, decay=0.5, weights=FAKE, stride=8, residual=NULL, workspace=NULL, size=0)
EVICT = dict(layout=LAY, table=FAKE, width=8, lens=FAKE, n_seqs=2, weights=FAKE, stride=8, kept=4, first=1, last=1, table_after=FAKE, lens_after=HALF,
             weights_after=FAKE, freed=FAKE, n_freed=5, counts=FAKE)
CALLS = [("pq_bound_pages", BOUND), ("pq_select_pages", SELECT), ("pq_sparse_attention", SPARSE), ("pq_decode_attention_weights", WEIGHTS), ("pq_evict_pages", EVICT)]


@pytest.mark.parametrize("name,defaults", CALLS)
def test_layouts_without_kernels_are_refused(lib, name, defaults):
    assert _call(lib, name, defaults, layout=None) == INVALID
    for layout in (pq.Layout(64, 4, 4, 128, 8), pq.Layout(128, 5, 4, 128, 8), pq.Layout(128, 4, 4, 64, 8), pq.Layout(128, 4, 4, 128, 8, 2)):
        assert _call(lib, name, defaults, layout=layout) == UNSUPPORTED


@pytest.mark.parametrize("change", [dict(n_seqs=-1), dict(most=-1), dict(width=0), dict(pages=0), dict(codes=NULL), dict(params=NULL), dict(table=NULL),
                                    dict(after=NULL), dict(bounds=NULL), dict(scales=NULL), dict(codes=HALF), dict(params=HALF), dict(bounds=HALF), dict(scales=HALF),
                                    dict(table=ODD), dict(before=ODD), dict(after=ODD)])
def test_bounds_refuse(lib, change):
    assert _call(lib, "pq_bound_pages", BOUND, **change) == INVALID


def test_bounds_of_nothing_and_of_too_much(lib):
    assert _call(lib, "pq_bound_pages", BOUND, n_seqs=0, table=NULL) == 0
    assert _call(lib, "pq_bound_pages", BOUND, most=0, codes=NULL) == 0
    assert _call(lib, "pq_bound_pages", BOUND, n_seqs=65536) == UNSUPPORTED
    assert _call(lib, "pq_bound_pages", BOUND, most=2 ** 31 - 1, width=2 ** 31 - 1) == UNSUPPORTED


SHARED = [dict(n_seqs=0), dict(heads=0), dict(heads=12), dict(max_seq_len=0), dict(max_seq_len=1025), dict(dtype=2), dict(pages=0), dict(width=0), dict(q=NULL),
          dict(table=NULL), dict(lens=NULL), dict(table=ODD), dict(lens=ODD)]
CHOICE = [dict(first=-1), dict(last=0), dict(chosen=1), dict(first=4), dict(first=2 ** 31 - 1, last=2 ** 31 - 1), dict(bounds=NULL), dict(scales=NULL), dict(q=HALF), dict(bounds=HALF),
          dict(scales=HALF), dict(selected=NULL), dict(selected_lens=NULL), dict(selected=ODD), dict(selected_lens=ODD)]
POOLS = [dict(codes=NULL), dict(params=NULL), dict(v_pool=NULL), dict(out=NULL), dict(v_bits=4), dict(codes=HALF), dict(params=HALF), dict(v_pool=HALF), dict(out=HALF),
         dict(residual=HALF), dict(v_bits=2, v_params=ODD), dict(scale=float("inf")), dict(scale=float("nan"))]


@pytest.mark.parametrize("change", SHARED + CHOICE)
def test_choice_refuses(lib, change):
    assert _call(lib, "pq_select_pages", SELECT, **change) == INVALID


@pytest.mark.parametrize("change", SHARED + CHOICE + POOLS)
def test_sparse_refuses(lib, change):
    assert _call(lib, "pq_sparse_attention", SPARSE, **change) == INVALID


@pytest.mark.parametrize("change", SHARED + POOLS + [dict(weights=NULL), dict(weights=ODD), dict(before=ODD), dict(stride=7), dict(decay=float("nan")), dict(decay=float("inf"))])
def test_weights_refuse(lib, change):
    assert _call(lib, "pq_decode_attention_weights", WEIGHTS, **change) == INVALID


@pytest.mark.parametrize("change", [dict(n_seqs=-1), dict(width=0), dict(stride=7), dict(kept=-1), dict(first=-1), dict(last=-1), dict(n_freed=-1), dict(table=NULL), dict(lens=NULL),
                                    dict(weights=NULL), dict(table_after=NULL), dict(lens_after=NULL), dict(weights_after=NULL), dict(freed=NULL), dict(counts=NULL),
                                    dict(table=ODD), dict(lens=ODD), dict(weights=ODD), dict(table_after=ODD), dict(lens_after=ODD), dict(weights_after=ODD), dict(freed=ODD),
                                    dict(counts=ODD), dict(lens_after=FAKE)])
def test_eviction_refuses(lib, change):
    assert _call(lib, "pq_evict_pages", EVICT, **change) == INVALID


def test_what_no_launch_holds_is_refused(lib):
    for name, defaults in CALLS[1:3]:
        assert _call(lib, name, defaults, heads=17 * 8) == UNSUPPORTED
        assert _call(lib, name, defaults, n_seqs=8192) == UNSUPPORTED
        assert _call(lib, name, defaults, pages=1 << 28) == UNSUPPORTED
    assert _call(lib, "pq_sparse_attention", SPARSE, v_bits=3) == UNSUPPORTED
    assert _call(lib, "pq_decode_attention_weights", WEIGHTS, v_bits=8) == UNSUPPORTED
    assert _call(lib, "pq_decode_attention_weights", WEIGHTS, heads=17 * 8) == UNSUPPORTED
    assert _call(lib, "pq_evict_pages", EVICT, n_seqs=65536) == UNSUPPORTED


@pytest.mark.parametrize("name,defaults,size", [
    ("pq_select_pages", SELECT, lambda: pq.pq_select_workspace_bytes(LAY, 2, 1024)),
    ("pq_sparse_attention", SPARSE, lambda: pq.pq_sparse_workspace_bytes(LAY, 2, 32, 1024, 4)),
    ("pq_decode_attention_weights", WEIGHTS, lambda: pq.pq_weights_workspace_bytes(LAY, 2, 32, 1024))])
def test_workspaces_are_checked(lib, name, defaults, size):
    n = size()
    assert n > 0 and n % 256 == 0
    assert _call(lib, name, defaults) == WORKSPACE
    assert _call(lib, name, defaults, workspace=FAKE, size=n - 1) == WORKSPACE
    assert _call(lib, name, defaults, workspace=ctypes.c_void_p(4096 + 128), size=n) == WORKSPACE


def test_sizes(lib):
    assert pq.pq_bounds_bytes_per_page(LAY) == 8 * 256 and pq.pq_bound_scales_bytes_per_page(LAY) == 8 * 16
    assert pq.pq_bounds_bytes_per_page(pq.Layout(64, 4, 4, 128, 8)) == 0 and pq.pq_bound_scales_bytes_per_page(pq.Layout(64, 4, 4, 128, 8)) == 0
    assert pq.pq_select_workspace_bytes(LAY, 0, 1000) == 0 and pq.pq_select_workspace_bytes(LAY, 4, 0) == 0
    assert lib.pq_select_workspace_bytes(None, 4, 1000) == 0
    assert pq.pq_sparse_workspace_bytes(LAY, 2, 32, 1024, 0) == 0 and pq.pq_sparse_workspace_bytes(LAY, 2, 12, 1024, 4) == 0
    assert pq.pq_weights_workspace_bytes(LAY, 2, 12, 1024) == 0
    assert pq.pq_weights_workspace_bytes(LAY, 2, 32, 1024) >= pq.pq_decode_workspace_bytes(LAY, 2, 32, 1024) + 2 * 32 * 8 * 8


@pytest.mark.parametrize("first,last", [(0, 0), (1, 1), (4, 1), (0, 5), (-1, 1), (3, -7), (2 ** 31 - 1, 2 ** 31 - 1)])
def test_a_given_choice_has_no_first_and_last_pages(lib, first, last):
    """bounds and bound_scales NULL: n_first, n_last, the table and the lengths are not looked at -- the call gets as far as its workspace --, the rest is."""
    given = dict(bounds=NULL, scales=NULL, table=NULL, lens=NULL, width=0, first=first, last=last)
    assert _call(lib, "pq_sparse_attention", SPARSE, **given) == WORKSPACE
    for change in (dict(chosen=0), dict(selected=NULL), dict(selected_lens=NULL), dict(selected=ODD), dict(q=NULL), dict(heads=12), dict(max_seq_len=0), dict(out=NULL)):
        assert _call(lib, "pq_sparse_attention", SPARSE, **{**given, **change}) == INVALID


def _never_falls(sizes):
    """sizes[i][j]...: along no axis does a size get smaller."""
    import numpy as np
    a = np.array(sizes, np.int64)
    assert (a > 0).all()
    for axis in range(a.ndim):
        fall = np.argwhere(np.diff(a, axis=axis) < 0)
        assert len(fall) == 0, (axis, fall[:5].tolist())


N_SEQS = [1, 2, 3, 5, 7, 8, 12, 13, 16, 31, 32, 33, 63, 64, 65, 100, 127, 128, 200, 255, 256, 257, 511, 512, 513, 600, 1000, 2000]
LENGTHS = [1, 128, 129, 500, 896, 897, 1024, 4000, 20000, 32768, 32769, 40000, 65536, 100000, 127999, 131072, 500000, 8192 * 128, 8192 * 128 + 1, 1 << 21]


@pytest.mark.parametrize("heads", [1, 2, 3, 8, 32])
def test_a_workspace_serves_smaller_batches(lib, heads):
    """A serving loop makes one workspace for its largest batch, and batches shrink: no size falls as sequences, lengths or chosen pages become more."""
    layout = pq.Layout(128, 4, 4, 128, heads)
    seqs = [n for n in N_SEQS if n * heads <= 65535]
    _never_falls([[pq.pq_select_workspace_bytes(layout, n, most) for most in LENGTHS] for n in seqs])


@pytest.mark.parametrize("heads,group", [(1, 1), (2, 16), (3, 5), (8, 4), (32, 2)])
@pytest.mark.parametrize("angles", [0, 1])
def test_a_workspace_of_attention_serves_smaller_batches(lib, heads, group, angles):
    layout = pq.Layout(128, 4, 4, 128, heads, angles)
    _never_falls([[pq.pq_weights_workspace_bytes(layout, n, heads * group, most) for most in LENGTHS] for n in N_SEQS])
    chosen = [1, 4, 7, 8, 9, 13, 16, 17, 32, 48, 100, 500, 3000, 100000]
    _never_falls([[[pq.pq_sparse_workspace_bytes(layout, n, heads * group, most, c) for c in chosen] for most in LENGTHS] for n in N_SEQS])
