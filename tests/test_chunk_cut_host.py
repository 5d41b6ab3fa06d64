"""How launches of pq_chunk_attention are shared out (csrc/pq_chunk_cut.hpp), run for the 64 lanes of a wavefront on the CPU with the
plan the host makes (csrc/pq_chunk_plan.hpp): every page that a tile of a chunk sees is in exactly one part, every part has a place,
and the parts that are joined lie within the launch's places."""
import ctypes
import os
import random
import subprocess

import numpy as np
import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
G, MOST_PARTS, FEW_LEAST = 128, 64, 2


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    out = tmp_path_factory.mktemp("chunkcuthost") / "libchunk_cut_host.so"
    subprocess.run(["g++", "-O2", "-std=c++17", "-Wall", "-Wno-unknown-pragmas", "-shared", "-fPIC", "-I", os.path.join(ROOT, "paper_2502_00527_amd", "csrc"),
                    "-I", os.path.join(ROOT, "include"), os.path.join(ROOT, "tests", "host", "chunk_cut_host.cpp"), "-o", str(out)], check=True)
    lib = ctypes.CDLL(str(out))
    lib.chunk_cut_host.restype = ctypes.c_int
    lib.chunk_cut_host.argtypes = [ctypes.c_int] * 3 + [ctypes.c_int64, ctypes.c_void_p, ctypes.c_void_p] + [ctypes.c_int] * 3 + [ctypes.c_float, ctypes.c_void_p, ctypes.c_void_p]
    return lib


class Launch:
    """`lens` with the chunks of `new` tokens; `tiles`: (sequence, first token) -> its parts (first page, pages, unit)."""

    def __init__(self, lib, lens, new, kv_heads, group=4, bound=None, window=0, sinks=0, error=0.0, rows=None):
        starts = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
        rows = int(starts[-1]) if rows is None else rows
        lens32, plan, units = np.asarray(lens, np.int32), np.zeros(8, np.int64), np.zeros((1 << 17, 8), np.int32)
        n = lib.chunk_cut_host(len(lens), kv_heads, kv_heads * group, rows, starts.ctypes.data, lens32.ctypes.data, bound or max(lens), window, sinks, error,
                               plan.ctypes.data, units.ctypes.data)
        self.rows_of_16, self.tile, self.cuts, self.host_parts, self.items, self.units, self.bytes, self.sorted = (int(x) for x in plan)
        assert n == self.units
        self.lens, self.new, self.window, self.sinks, self.kv_heads = lens, new, window, sinks, kv_heads
        self.tiles, self.order = {}, []
        for unit, (seq, first, count, part, parts, pages, begin, length) in enumerate(units[:n].tolist()):
            if seq < 0:
                continue
            tile = self.tiles.setdefault((seq, first), dict(count=count, parts=parts, pages=pages, unit=unit, of=[]))
            assert (count, parts, pages) == (tile["count"], tile["parts"], tile["pages"])
            assert part == len(tile["of"]) and unit == tile["unit"] + part, "parts are neighbours, in order"
            tile["of"].append((begin, length))
            if part == 0:
                self.order.append(seq)

    def visible(self, seq, first, count):
        """Pages that a tile's rows see."""
        position = self.lens[seq] - self.new[seq] + first
        last = position + count - 1
        if last < 0:
            return 0
        pages = set(range(last // G + 1))
        if self.window and self.window < max(self.lens):
            pages = {p for p in pages if p * G < self.sinks or p * G + G - 1 > position - self.window}
        return len(pages)

    def check(self):
        want = {(s, first): min(self.tile, n - first) for s, n in enumerate(self.new) for first in range(0, n, self.tile)}
        assert {k: t["count"] for k, t in self.tiles.items()} == want
        for (seq, first), tile in self.tiles.items():
            assert 1 <= tile["parts"] <= MOST_PARTS and len(tile["of"]) == tile["parts"], "all parts have a place"
            assert tile["unit"] + tile["parts"] <= self.units
            assert tile["parts"] == 1 or self.cuts
            # (with a window a tile may count a page more that the window of its later rows has left)
            assert tile["pages"] >= self.visible(seq, first, tile["count"]) >= tile["pages"] - (2 if self.window else 0)
            at = 0
            for begin, length in tile["of"]:
                assert length == 0 or begin == at
                at += length
            assert at == max(tile["pages"], 0), (tile, self.lens)
        if self.cuts:
            assert self.bytes >= self.units * self.kv_heads * 16 * self.rows_of_16 * (G + 2) * 4
        if self.sorted:
            pages = [(self.lens[s] + G - 1) // G for s in self.order]
            assert self.window or pages == sorted(pages, reverse=True)
        return self

    def longest_part(self):
        return max(length for tile in self.tiles.values() for _, length in tile["of"])


def draw(rng):
    kv_heads = rng.choice([1, 2, 3, 4, 8, 8, 8, 16, 32])
    n = rng.choice([1, 1, rng.randint(2, 70), rng.randint(60, 200)])
    longest = round(128 * 2 ** rng.uniform(0, 9))
    most_new = round(2 ** rng.uniform(0, 10))
    new = [rng.choice([most_new, rng.randint(0, most_new), rng.randint(0, 3)]) for _ in range(n)]
    new[0] = max(1, new[0])
    lens = [max(rng.choice([longest, rng.randint(0, longest), rng.randint(0, 300)]), c) for c in new]
    bound = max(lens) if rng.random() < 0.5 else round(max(lens) * 2 ** rng.uniform(0, 5))
    window = 0 if rng.random() < 0.6 else rng.randint(1, longest)
    return dict(lens=lens, new=new, kv_heads=kv_heads, group=rng.choice([1, 2, 3, 4, 8, 16]), bound=max(1, bound), window=window,
                sinks=rng.choice([0, 4, 130]), error=rng.choice([0.0, 2.0 ** -23, -(2.0 ** -23)]))


@pytest.mark.parametrize("seed", range(6))
def test_every_page_is_in_one_part(lib, seed):
    rng = random.Random(seed)
    kinds = set()
    for _ in range(25):
        case = draw(rng)
        try:
            launch = Launch(lib, **case).check()
        except AssertionError:
            print(case)
            raise
        kinds.add((launch.rows_of_16, launch.cuts, launch.sorted))
    assert len(kinds) >= 4, kinds


def test_chunks_that_are_shorter_than_the_rows_and_sequences_without(lib):
    Launch(lib, [5000, 0, 700], [5, 0, 3], 8, rows=64).check()
    Launch(lib, [40, 300], [60, 0], 2).check()                          # a chunk longer than its sequence


def fitting(launch):
    """The shortest parts that fit the launch's places, by trying all lengths."""
    pages = [((n + G - 1) // G, len([1 for s, _ in launch.tiles if s == seq])) for seq, n in enumerate(launch.lens)]
    longest = max(p for p, _ in pages)
    for per in range(max(FEW_LEAST, -(-longest // MOST_PARTS)), longest):
        if sum(tiles * max(1, -(-p // per)) for p, tiles in pages) <= launch.units:
            return per
    return longest


@pytest.mark.parametrize("kv_heads,seqs,lens", [*[(8, n, [1024 * G] + [G] * (n - 1)) for n in (46, 48, 50, 56, 60, 61, 62)], (32, 13, [4000 * G] + [3 * G] * 12),
                                                (1, 400, [2000 * G] + [G] * 399), (8, 4, [8192 * G] * 4), (8, 40, [700 * G, 300 * G] + [2 * G] * 38),
                                                (2, 200, [3000 * G] * 3 + [100] * 197)])
def test_one_long_sequence_among_short_ones_is_cut_as_far_as_there_are_places(lib, kv_heads, seqs, lens):
    """Few rows: parts are within a step of the search (1 / 16) of the shortest ones that fit."""
    launch = Launch(lib, lens, [1] * seqs, kv_heads).check()
    assert launch.rows_of_16 == 1 and launch.cuts
    assert launch.longest_part() <= fitting(launch) * 17 / 16 + 2, (launch.longest_part(), fitting(launch))
