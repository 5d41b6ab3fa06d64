"""pq_plan_pages against the same walk in Python."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

DEV, G = "cuda:0", 128


def _plan(lens, new, free, table, n_slots):
    """What the header says, token by token."""
    lens, new = np.maximum(lens, 0), np.maximum(new, 0)
    table = table.copy()
    slots = np.full(n_slots, -1, np.int64)
    starts = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
    used = 0
    for s, (L, n) in enumerate(zip(lens, new)):
        pages = {}
        for i in range(n):
            place, page = (L + i) % G, (L + i) // G
            if page * G >= L:                                    # begun by the new tokens
                if page not in pages:
                    pages[page] = free[used] if used < len(free) else -1
                    used += 1
                    if page < table.shape[1] and starts[s] + i < n_slots:
                        table[s, page] = pages[page]
                page_id = pages[page] if page < table.shape[1] else -1
            else:
                page_id = table[s, page] if page < table.shape[1] else -1
            if starts[s] + i < n_slots and page_id >= 0:
                slots[starts[s] + i] = page_id * G + place
    return table, starts, slots, (lens + new).astype(np.int32), np.array([used, new.sum()], np.int32)


def _run(lens, new, free, table, n_slots):
    import paper_2502_00527_amd as pq

    to = lambda x, t=torch.int32: torch.as_tensor(np.ascontiguousarray(x), dtype=t).to(DEV)      # noqa: E731
    n = len(lens)
    out = dict(block_table=to(table), starts=to(np.full(n + 1, -5)), slots=to(np.full(n_slots, -7), torch.int64), lens_after=to(np.full(n, -5)),
               counts=to([-5, -5]))
    pq.pq_plan_pages(pq.Layout(128, 4, 4, G, 2), to(lens), to(new), to(free), *out.values())
    torch.cuda.synchronize()
    return [x.cpu().numpy() for x in out.values()]


def _check(lens, new, n_free=None, width=None, n_slots=None, seed=0):
    lens, new = np.asarray(lens, np.int32), np.asarray(new, np.int32)
    rng = np.random.default_rng(seed)
    most = int(max([1, *((np.maximum(lens, 0).astype(np.int64) + np.maximum(new, 0) + G - 1) // G)]))
    width = width or most
    held = (np.maximum(lens, 0) + G - 1) // G
    need = int(((np.maximum(lens, 0) + np.maximum(new, 0) + G - 1) // G - held).sum())
    table = rng.integers(0, 1 << 24, (len(lens), width)).astype(np.int32)
    free = rng.permutation(need + 5).astype(np.int32)[:need + 5 if n_free is None else n_free]
    n_slots = int(np.maximum(new, 0).sum()) if n_slots is None else n_slots
    for got, want in zip(_run(lens, new, free, table, n_slots), _plan(lens, new, free, table, n_slots)):
        np.testing.assert_array_equal(got, want)


@pytest.mark.parametrize("lens,new", [([0], [1]), ([127], [1]), ([128], [1]), ([1], [0]), ([0], [0]), ([5], [500]), ([128], [128]), ([127, 0, 256], [2, 0, 1]),
                                      ([0, 0, 0], [0, 300, 0]), ([300, 7], [0, 0]), ([-4, 9], [3, -2]), ([(1 << 30) - 3], [9])])
def test_small_batches(lens, new):
    _check(lens, new, width=(max(lens) + max(new)) // G + 1)


@pytest.mark.parametrize("seqs,most_len,most_new", [(64, 16384, 1), (31, 700, 5), (1023, 300, 9), (1024, 300, 2), (1025, 300, 40), (2500, 1000, 1), (3, 9, 9000)])
@pytest.mark.parametrize("seed", [1, 2])
def test_batches(seqs, most_len, most_new, seed):
    rng = np.random.default_rng(seed)
    _check(rng.integers(0, most_len + 1, seqs), rng.integers(0, most_new + 1, seqs), seed=seed)


@pytest.mark.parametrize("n_free", [0, 1, 7])
def test_free_pages_run_out(n_free):
    _check([100, 250, 0, 128], [300, 6, 700, 128], n_free=n_free)


def test_pages_past_the_width_have_no_slots():
    _check([100, 10, 600], [300, 300, 300], width=3)


@pytest.mark.parametrize("n_slots", [0, 1, 129, 600, 5000])
def test_room_for_fewer_or_more_tokens_than_there_are(n_slots):
    _check([100, 0, 250], [300, 0, 299], n_slots=n_slots)


def test_no_sequences():
    table, starts, slots, after, counts = _run([], [], [3], np.zeros((0, 4), np.int32), 9)
    assert starts.tolist() == [0] and counts.tolist() == [0, 0] and (slots == -1).all()
