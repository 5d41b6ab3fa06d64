"""Host-side logic of the entry points for chunks of new tokens and sliding windows: sizes and refusals.  No GPU needed: every
call here returns before anything is launched."""
import ctypes

import pytest

import paper_2502_00527_amd as pq

LAY = pq.Layout(128, 4, 4, 128, 8)
FAKE, NULL, ODD = ctypes.c_void_p(4096), ctypes.c_void_p(0), ctypes.c_void_p(4098)
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


PLAN = dict(layout=LAY, seq_lens=FAKE, new_lens=ctypes.c_void_p(8192), n_seqs=4, free=FAKE, n_free=9, table=FAKE, width=8, starts=ctypes.c_void_p(12288),
            slots=FAKE, room=100, after=ctypes.c_void_p(16384), counts=FAKE)
APPEND = dict(layout=LAY, keys=FAKE, dtype=0, key_token=1024, key_head=128, values=FAKE, value_token=1024, value_head=128, n_tokens=10, n_seqs=2, starts=FAKE,
              lens=FAKE, slots=FAKE, residual=FAKE, table=FAKE, width=8, codes=FAKE, params=FAKE, v_pool=FAKE, v_bits=16, v_params=NULL, pages=16)
CHUNK = dict(layout=LAY, q=FAKE, dtype=0, n_tokens=10, n_seqs=2, heads=32, starts=FAKE, codes=FAKE, params=FAKE, v_pool=FAKE, v_bits=16, v_params=NULL, pages=16,
             table=FAKE, width=8, lens=FAKE, max_seq_len=1024, window=0, sinks=0, scale=0.1, out=FAKE, residual=NULL, workspace=NULL, size=0)
WINDOW = dict(layout=LAY, q=FAKE, dtype=0, n_seqs=2, heads=32, codes=FAKE, params=FAKE, v_pool=FAKE, v_bits=16, v_params=NULL, pages=16, table=FAKE, width=8,
              lens=FAKE, max_seq_len=1024, window=100, sinks=4, scale=0.1, out=FAKE, residual=NULL, workspace=NULL, size=0)
OTHER_LAYOUTS = [dict(layout=None), dict(layout=pq.Layout(64, 4, 4, 128, 8)), dict(layout=pq.Layout(128, 5, 4, 128, 8)), dict(layout=pq.Layout(128, 4, 4, 64, 8)),
                 dict(layout=pq.Layout(128, 4, 4, 128, 8, 2))]


@pytest.mark.parametrize("name,defaults", [("pq_plan_pages", PLAN), ("pq_append_chunk", APPEND), ("pq_chunk_attention", CHUNK), ("pq_window_attention", WINDOW)])
def test_layouts_without_kernels_are_refused(lib, name, defaults):
    assert _call(lib, name, defaults, layout=None) == INVALID
    for change in OTHER_LAYOUTS[1:]:
        assert _call(lib, name, defaults, **change) == UNSUPPORTED


@pytest.mark.parametrize("change", [dict(n_seqs=-1), dict(n_free=-1), dict(width=0), dict(room=-1), dict(seq_lens=NULL), dict(new_lens=NULL), dict(free=NULL),
                                    dict(table=NULL), dict(starts=NULL), dict(slots=NULL), dict(after=NULL), dict(counts=NULL), dict(seq_lens=ODD), dict(slots=ctypes.c_void_p(4100)),
                                    dict(after=FAKE), dict(starts=FAKE), dict(after=ctypes.c_void_p(8192))])
def test_plan_refuses(lib, change):
    assert _call(lib, "pq_plan_pages", PLAN, **change) == INVALID


def test_plan_refuses_what_does_not_fit_its_integers(lib):
    assert _call(lib, "pq_plan_pages", PLAN, n_seqs=(1 << 20) + 1) == UNSUPPORTED
    assert _call(lib, "pq_plan_pages", PLAN, room=1 << 31) == UNSUPPORTED


@pytest.mark.parametrize("change", [dict(n_tokens=-1), dict(n_seqs=-1), dict(pages=0), dict(width=0), dict(dtype=2), dict(keys=NULL), dict(starts=NULL), dict(lens=NULL),
                                    dict(residual=NULL), dict(table=NULL), dict(codes=NULL), dict(params=NULL), dict(slots=NULL), dict(v_pool=NULL),
                                    dict(v_bits=4), dict(keys=ODD), dict(values=ODD), dict(residual=ODD), dict(key_token=1025), dict(key_head=4), dict(value_token=1025),
                                    dict(key_token=-1024), dict(value_head=-128), dict(dtype=1, key_token=1026), dict(starts=ODD), dict(slots=ctypes.c_void_p(4100))])
def test_append_refuses(lib, change):
    assert _call(lib, "pq_append_chunk", APPEND, **change) == INVALID


def test_append_of_nothing_and_other_widths(lib):
    assert _call(lib, "pq_append_chunk", APPEND, n_tokens=0, keys=NULL) == 0
    assert _call(lib, "pq_append_chunk", APPEND, n_seqs=0, starts=NULL) == 0
    assert _call(lib, "pq_append_chunk", APPEND, v_bits=3) == UNSUPPORTED
    assert _call(lib, "pq_append_chunk", APPEND, n_tokens=1 << 31) == UNSUPPORTED


@pytest.mark.parametrize("change", [dict(n_tokens=-1), dict(n_seqs=0), dict(heads=12), dict(heads=0), dict(max_seq_len=0), dict(dtype=2), dict(window=-1), dict(sinks=-1),
                                    dict(scale=float("inf")), dict(scale=float("nan")), dict(pages=0), dict(width=7), dict(q=NULL), dict(starts=NULL), dict(codes=NULL),
                                    dict(params=NULL), dict(v_pool=NULL), dict(table=NULL), dict(lens=NULL), dict(out=NULL), dict(v_bits=4), dict(q=ODD), dict(out=ODD),
                                    dict(residual=ODD), dict(starts=ODD), dict(v_bits=2, v_params=ODD)])
def test_chunk_attention_refuses(lib, change):
    assert _call(lib, "pq_chunk_attention", CHUNK, **change) == INVALID


def test_chunk_attention_refuses_what_it_has_no_kernel_for(lib):
    for change in (dict(dtype=1), dict(v_bits=3), dict(heads=8 * 17), dict(n_tokens=1 << 31), dict(n_tokens=1 << 22), dict(n_seqs=(1 << 20) + 1)):
        assert _call(lib, "pq_chunk_attention", CHUNK, **change) == UNSUPPORTED
    assert _call(lib, "pq_chunk_attention", CHUNK, n_tokens=0) == 0


def test_chunk_attention_needs_its_workspace(lib):
    for shape in (dict(), dict(n_tokens=700), dict(n_seqs=9, n_tokens=40, max_seq_len=8 * 128), dict(window=100, sinks=4)):
        args = dict(CHUNK, **shape)
        size = pq.pq_chunk_workspace_bytes(LAY, args["n_seqs"], 32, args["n_tokens"], args["max_seq_len"])
        assert size >= 256
        assert _call(lib, "pq_chunk_attention", args) == WORKSPACE
        assert _call(lib, "pq_chunk_attention", args, workspace=FAKE, size=size - 1) == WORKSPACE
        assert _call(lib, "pq_chunk_attention", args, workspace=ctypes.c_void_p(4096 + 128), size=size) == WORKSPACE
    assert pq.pq_chunk_workspace_bytes(LAY, 0, 32, 10, 100) == 0 and pq.pq_chunk_workspace_bytes(LAY, 1, 12, 10, 100) == 0
    assert pq.pq_chunk_workspace_bytes(LAY, 1, 32, 10, 0) == 0


def test_chunk_workspace_holds_for_any_window():
    """A window cuts a launch into other parts than the whole sequence: its partials have to fit, too."""
    for seqs, heads, tokens in ((1, 8, 3), (1, 32, 2048), (5, 32, 900), (40, 16, 45)):
        sizes = [pq.pq_chunk_workspace_bytes(pq.Layout(128, 4, 4, 128, 8 if heads > 8 else 2), seqs, heads, tokens, 128 * pages) for pages in range(1, 300)]
        assert sizes == sorted(sizes)


@pytest.mark.parametrize("change", [dict(window=0), dict(window=-1), dict(sinks=-1), dict(n_seqs=0), dict(heads=12), dict(max_seq_len=0), dict(dtype=2), dict(scale=float("nan")),
                                    dict(pages=0), dict(width=7), dict(q=NULL), dict(codes=NULL), dict(params=NULL), dict(v_pool=NULL), dict(table=NULL), dict(lens=NULL),
                                    dict(out=NULL), dict(out=ODD), dict(codes=ODD), dict(residual=ODD), dict(lens=ODD), dict(v_bits=4)])
def test_window_attention_refuses(lib, change):
    assert _call(lib, "pq_window_attention", WINDOW, **change) == INVALID


def test_window_attention_needs_its_workspace(lib):
    assert _call(lib, "pq_window_attention", WINDOW, v_bits=3) == UNSUPPORTED
    assert _call(lib, "pq_window_attention", WINDOW, heads=8 * 17) == UNSUPPORTED
    for seqs, window, sinks in ((2, 100, 4), (2, 1, 0), (700, 2000, 4), (1, 10 ** 9, 10 ** 9)):
        size = pq.pq_window_workspace_bytes(LAY, seqs, 32, 1024, window, sinks)
        assert size >= 256
        args = dict(WINDOW, n_seqs=seqs, window=window, sinks=sinks)
        assert _call(lib, "pq_window_attention", args) == WORKSPACE
        assert _call(lib, "pq_window_attention", args, workspace=FAKE, size=size - 1) == WORKSPACE
    assert pq.pq_window_workspace_bytes(LAY, 1, 32, 1024, 0, 4) == 0 and pq.pq_window_workspace_bytes(LAY, 1, 32, 1024, 8, -1) == 0
