"""The GPU tests of paged attention reach every way in which a call is cut: the library's own choice, asked for their sizes."""
import random

import paged_choice as choice
import test_gpu_paged_paths as paths


def width(seqs, page):
    return max(-(-t // page) for _, t in seqs) + paths.BIG // page


def test_paths_are_the_ones_named():
    for name, hq, hkv, page, seqs, hints in paths.PATHS:
        got = choice.path(hq, hkv, seqs, hints, page, width(seqs, page), 1)
        assert got == name, (got, name, seqs[:4], hints)
    for name, seqs, hints in paths.HIDDEN:
        got = choice.path(4, 2, seqs, hints, 16, width(seqs, 16))
        assert got == name, (got, name)
    for hints, name in (((1, 60), "units 8"), ((1, 4000), "steps 1"), ((300, 4000), "steps 1 + list")):
        assert choice.path(8, 2, [(1, 50)] * 6, hints, 16, 250, 294) == name


def test_a_hint_beyond_the_table_is_the_tables_size():
    assert choice.path(8, 2, [(1, 100)], (1, 0), 16, 10) == choice.path(8, 2, [(1, 100)], (1, 1 << 40), 16, 10)


def test_every_call_is_cut_in_a_way_that_covers_it():
    rng = random.Random(5)
    for _ in range(20000):
        hkv = rng.choice([1, 2, 3, 8, 40])
        g = rng.choice([1, 2, 3, 5, 8, 16, 33, 64, 128])
        batch = rng.randint(1, 200)
        total = rng.randint(1, 20000)
        hints = (rng.randint(0, 20000), rng.choice([0, rng.randint(1, 10 ** 6)]))
        got = choice.path(g * hkv, hkv, [(total - batch + 1, 0)] + [(1, 0)] * (batch - 1) if total >= batch else [(total, 0)], hints, 16, 5000)
        assert got in ("units 8", "units 4", "steps 1", "steps 2", "list", "steps 1 + list", "steps 2 + list")
        if "list" in got and "steps" in got:
            assert g <= 64 and (got[6] == "1") == (g <= 32)      # a row tile of the steps holds a token's whole group


def test_parts_of_a_token():
    assert choice.parts(1, 12) == 12 and choice.parts(64, 12) == 12 and choice.parts(16384, 18) == 1
    assert all(1 <= choice.parts(t, q) <= q for t in (1, 7, 1000, 10 ** 6) for q in (1, 2, 5, 48))
