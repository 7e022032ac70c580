"""How calls on a cache in 4 bits whose sequences differ are taken apart, and which of them keep their keys' way through the workspace."""
from mx_calls import way

STEPS = [(1, 3500)] * 24
PROMPTS = [(1100, 1100), (900, 900), (600, 600), (700, 700), (1000, 1000), (800, 800)]


def test_long_chunks_beside_steps_go_to_the_list():
    assert way(32, 8, STEPS + [(512, 30512)], (512, 30512), 64, 477, 30512) == "steps, list"
    assert way(32, 8, STEPS + [(512, 30512)], (512, 30512), 64, 477, 30512, spare_rows=40) == "steps, list"
    assert way(32, 8, [(2, 3500)] * 24 + [(512, 30512)], (512, 30512), 64, 477, 30512) == "steps, list"
    assert way(32, 8, STEPS + [(8192, 62500)], (8192, 62500), 64, 977, 62500) == "steps, list"
    assert way(32, 8, [(1, 65000)] * 8 + [(8192, 60000)], (8192, 65000), 64, 1016, 60000) == "steps, list"
    assert way(32, 8, STEPS + [(512, 30512)], (512, 30512), 64, 477) == "steps, units 3"      # no room


def test_places_of_a_batch_that_are_empty_change_nothing():
    for empty in (10, 1000):
        assert way(32, 8, STEPS + [(512, 30512)] + [(0, 0)] * empty, (512, 30512), 64, 477, 30512) == "steps, list"
    assert way(32, 8, [(512, 30512)] + [(0, 0)] * 10, (512, 30512), 64, 477, 30512).endswith("list")


def test_prompts_of_very_different_lengths_go_to_the_list():
    for seqs in ([(16000, 16000)] + [(2000, 2000)] * 4, [(8192, 60000)] + [(1000, 30000)] * 7):
        longest = max(t for _, t in seqs)
        assert way(32, 8, seqs, (seqs[0][0], longest), 64, -(-longest // 64), sum(t for _, t in seqs)).endswith("list")
    four = [(2048, 32000)] * 4
    assert way(32, 8, four, (2048, 32000), 64, 500, 128000) == "list"
    assert way(32, 8, four, (0, 0), 64, 500, 128000).endswith("list")


def test_prompts_without_a_prefix_are_units():
    """Whether a prefix of the longest sequence's length is theirs says the workspace."""
    seqs = [(1, 2000 + 1700 * i) for i in range(24)] + PROMPTS
    for room in (0, sum(t for _, t in PROMPTS)):
        assert way(32, 8, seqs, (1100, 42000), 16, 2625, room) == "steps, units 3"
    assert way(32, 8, STEPS + [(250, 250), (200, 200)], (250, 3500), 32, 110, 450) == "steps, units 3"


def test_a_chunk_of_few_rows_behind_many_keys_is_spans():
    for room in (0, 40000):
        assert way(32, 8, STEPS + [(128, 40000)], (128, 40000), 32, 1250, room) == "spans 3"


def test_sequences_of_a_unit_each_are_one_launch():
    assert way(64, 8, [(1 + i % 5, 10000) for i in range(24)], (5, 10000), 32, 313) == "spans 3"
    assert way(64, 8, [(5, 10000)] * 24, (5, 10000), 32, 313) == "spans 3"
    assert way(32, 8, [(1 + i % 9, 10000) for i in range(24)], (9, 10000), 32, 313, 60000) == "spans 3"
    assert way(64, 8, [(1, 540)] * 4, (0, 0), 16, 34) == "units 2"


def test_short_calls_are_one_launch():
    assert way(8, 1, [(1, 385)] * 45 + [(79, 79)], (79, 385), 16, 25, 79) == "units 3"
    assert way(10, 2, [(5, 60)] * 7 + [(71, 147)] * 5, (71, 147), 16, 10, 500) == "units 3"


def test_decode_steps_without_hints_leave_nothing_over():
    assert way(32, 8, [(1, 8000)] * 64, (0, 0), 16, 500) == "steps, units 3"
    assert way(32, 8, [(1, 8000)] * 64, (0, 0), 16, 500, 100000) == "steps, units 3"
    assert way(32, 8, [(1, 60000)] * 64, (0, 0), 16, 3750) == "steps, units 3"
    assert way(32, 8, [(1, 60000)] * 64, (512, 60000), 16, 3750, 100000) == "steps, units 3"      # a bound in the place of the longest
