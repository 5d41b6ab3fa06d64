"""Drafted tokens, some of which are dropped: the cache that is left is the one of the accepted tokens alone, byte for byte."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from chunks import D, DEV, G, layout, pools      # noqa: E402

HEADS, GROUP, WIDTH = 2, 4, 6


def _ints(x):
    return torch.as_tensor(np.asarray(x), dtype=torch.int32).to(DEV)


class Batch:
    """A batch that drafts, and beside it (the same pages of other pools) one that is given the accepted tokens only, one by one."""

    def __init__(self, seqs, bits, grouped, v_bits, seed):
        import paper_2502_00527_amd as pq
        self.pq, self.seqs, self.v_bits = pq, seqs, v_bits
        self.rng = np.random.default_rng(seed)
        self.layout = layout(bits, HEADS, grouped)
        self.free = [int(x) for x in self.rng.permutation(seqs * WIDTH)]
        make = lambda: pools(seqs * WIDTH, bits, HEADS, grouped, v_bits)      # noqa: E731
        self.cache, self.plain = make(), make()
        self.residual, self.plain_residual = (torch.full((seqs, HEADS, G, D), float("nan"), dtype=torch.float16, device=DEV) for _ in range(2))
        self.table = _ints(np.full((seqs, WIDTH), -1))
        self.lens = np.zeros(seqs, np.int64)

    def plan(self, new):
        """Pages and slots of new tokens; the free list goes without what was taken."""
        total = int(np.sum(new))
        starts, after, counts = _ints(np.zeros(self.seqs + 1)), _ints(np.zeros(self.seqs)), _ints([0, 0])
        slots = torch.zeros(total, dtype=torch.int64, device=DEV)
        self.pq.pq_plan_pages(self.layout, _ints(self.lens), _ints(new), _ints(self.free), self.table, starts, slots, after, counts)
        taken = int(counts[0])
        assert taken <= len(self.free) and int(counts[1]) == total
        self.free = self.free[taken:]
        return starts, slots, after

    def give_back(self, after):
        """Pages that only dropped tokens had."""
        table = self.table.tolist()
        for s, n in enumerate(after.tolist()):
            self.free += [table[s][p] for p in range((self.lens[s] + G - 1) // G, (n + G - 1) // G)]

    def rows(self, total):
        return [torch.from_numpy(self.rng.standard_normal((total, HEADS, D))).to(DEV).half() for _ in range(2)]

    def append(self, residual, keys, values, starts, slots):
        codes, params, v_pool, v_params = self.cache
        self.pq.pq_append_chunk(self.layout, keys, values, starts, _ints(self.lens), slots, residual, self.table, codes, params, v_pool, self.v_bits, v_params)

    def attend(self, cache, residual, q, lens):
        codes, params, v_pool, v_params = cache
        out = torch.zeros((self.seqs, HEADS * GROUP, D), device=DEV)
        ws = torch.empty(self.pq.pq_decode_workspace_bytes(self.layout, self.seqs, HEADS * GROUP, WIDTH * G), dtype=torch.uint8, device=DEV)
        self.pq.pq_decode_attention(self.layout, q, codes, params, v_pool, self.table, lens, WIDTH * G, float(1 / np.sqrt(D)), out, ws, None, residual, self.v_bits, v_params)
        return out

    def accept(self, keys, values, slots, starts, accepted):
        """The accepted tokens into the cache beside, token by token; the lengths with them."""
        codes, params, v_pool, v_params = self.plain
        first = starts.tolist()
        for i in range(max(accepted)):
            now = [i < n for n in accepted]
            row = keys[[first[s] + i if now[s] else 0 for s in range(self.seqs)]].contiguous()
            self.pq.pq_append_keys(self.layout, row, self.plain_residual, _ints([self.lens[s] + i if now[s] else -1 for s in range(self.seqs)]), self.table, codes, params)
        kept = [first[s] + i for s, n in enumerate(accepted) for i in range(n)]
        if kept:
            # (values alone: every sequence's keys are skipped by its negative length)
            spare = torch.zeros_like(self.plain_residual)
            self.pq.pq_append_chunk(self.layout, keys[kept], values[kept], _ints(np.concatenate([[0], np.cumsum(accepted)])), _ints([-1] * self.seqs), slots[kept], spare,
                                    self.table, codes, params, v_pool, self.v_bits, v_params)
        self.lens = self.lens + np.asarray(accepted)

    def check(self):
        for s, n in enumerate(self.lens.tolist()):
            pages = self.table[s, :n // G].long()
            for got, want in zip(self.cache[:2], self.plain[:2]):
                assert torch.equal(got[pages].view(torch.uint8), want[pages].view(torch.uint8)), (s, n)
            assert torch.equal(self.residual[s, :, :n % G], self.plain_residual[s, :, :n % G]), (s, n)
        q = torch.from_numpy(self.rng.standard_normal((self.seqs, HEADS * GROUP, D))).to(DEV).half()
        lens = _ints(self.lens)
        got, want = self.attend(self.cache, self.residual, q, lens), self.attend(self.plain, self.plain_residual, q, lens)
        assert not torch.isnan(got).any() and torch.equal(got, want), self.lens


@pytest.mark.parametrize("bits,grouped,v_bits", [((4, 4), False, 16), ((3, 3), False, 4), ((4, 4), True, 2)])
def test_drafts_are_dropped_with_a_copy_of_the_residual(bits, grouped, v_bits):
    """Drafts are appended with a copy of the residual buffer, then the accepted ones to the buffer itself, from the same lengths:
    whatever groups the drafts completed.  The first lengths lie around a group's end; 126 tokens, 5 drafts, one accepted is among the steps."""
    b = Batch(5, bits, grouped, v_bits, 3)
    new = [126, 123, 128, 250, 4]
    starts, slots, after = b.plan(new)
    keys, values = b.rows(sum(new))
    b.append(b.residual, keys, values, starts, slots)
    b.accept(keys, values, slots, starts, new)
    b.check()
    chosen = [([5, 6, 4, 7, 3], [1, 0, 4, 1, 3]), ([3, 5, 1, 9, 126], [1, 5, 0, 2, 120]), ([5, 130, 2, 1, 140], [0, 3, 2, 1, 0])]
    for turn in range(12):
        drafts = chosen[turn][0] if turn < len(chosen) else b.rng.integers(0, 9, 5).tolist()
        accepted = chosen[turn][1] if turn < len(chosen) else [int(b.rng.integers(0, n + 1)) for n in drafts]
        if sum(drafts) == 0:
            continue
        starts, slots, after = b.plan(drafts)
        keys, values = b.rows(sum(drafts))
        b.append(b.residual.clone(), keys, values, starts, slots)                 # (and they are attended to with the copy)
        first = starts.tolist()
        kept = [first[s] + i for s, n in enumerate(accepted) for i in range(n)]
        # the values have been filed
        b.append(b.residual, keys[kept], None, _ints(np.concatenate([[0], np.cumsum(accepted)])), None)
        b.accept(keys, values, slots, starts, accepted)
        b.give_back(after)
        b.check()
    held = [x for s, n in enumerate(b.lens.tolist()) for x in b.table[s, :(n + G - 1) // G].tolist()]
    assert sorted(held + b.free) == list(range(5 * WIDTH)), "every page has one owner"


@pytest.mark.parametrize("before,drafts,accepted", [([3, 0, 140], [6, 5, 9], [2, 0, 8]),              # within the incomplete group
                                                    ([126, 250, 0], [5, 9, 130], [2, 6, 128]),        # back to the end of a group
                                                    ([126, 250, 120], [5, 9, 140], [3, 7, 137]),      # within the group behind the one that was completed
                                                    ([120, 5, 128], [8, 251, 256], [8, 123, 128])])   # to a group's end, from one
def test_lengths_that_may_go_back_without_a_copy(before, drafts, accepted):
    b = Batch(3, (4, 4), False, 16, 5)
    starts, slots, after = b.plan(before)
    keys, values = b.rows(sum(before))
    b.append(b.residual, keys, values, starts, slots)
    b.accept(keys, values, slots, starts, before)
    starts, slots, after = b.plan(drafts)
    keys, values = b.rows(sum(drafts))
    b.append(b.residual, keys, values, starts, slots)
    b.accept(keys, values, slots, starts, accepted)
    b.give_back(after)
    b.check()
    # and on from there
    starts, slots, after = b.plan([150, 1, 7])
    keys, values = b.rows(158)
    b.append(b.residual, keys, values, starts, slots)
    b.accept(keys, values, slots, starts, [150, 1, 7])
    b.check()
