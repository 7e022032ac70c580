"""Which kernels calls on a cache in 4 bits run on."""
from mx_choice import path


def test_short_calls_are_units_and_long_ones_spans():
    assert path(32, 8, [(1, 540)] * 4, (1, 540), 16, 40) == "units 1 8"
    assert path(32, 8, [(1, 540)] * 64, (1, 540), 16, 40) == "units 1 4"
    assert path(32, 8, [(1, 8400)] * 64, (1, 8400), 16, 600) == "spans 1"
    assert path(64, 8, [(1, 131072)] * 4, (1, 131072), 256, 512) == "spans 1"
    assert path(64, 8, [(5, 12000)] * 24, (5, 12000), 32, 400) == "spans 3"
    assert path(8, 8, [(20, 90)], (20, 90), 16, 6) == "units 2 4"
    assert path(32, 8, [(1, 540)] * 4, (1, 540), 8, 80) == "spans 1"      # pages of eight


def test_long_chunks_go_to_the_list_where_it_pays():
    assert path(32, 8, [(512, 30512)], (512, 30512), 64, 477, room=True) == "list"
    assert path(32, 8, [(512, 30512)], (512, 30512), 64, 477) == "spans 3"
    assert path(32, 8, [(640, 1640)], (640, 1640), 16, 103, room=True) == "units 3 4"


def test_chunks_beside_steps_are_launched_apart():
    mixed = [(1, 3500)] * 24 + [(1100, 1100)] * 6
    assert path(32, 8, mixed, (1100, 42000), 16, 2625, room=True) == "beside"
    assert path(32, 8, mixed, (0, 0), 16, 219) == "beside"
    assert path(32, 8, [(5, 3500)] * 24, (5, 3500), 16, 219) != "beside"


def test_unknown_hints_are_taken_from_the_table():
    assert path(32, 8, [(1, 540)] * 4, (0, 0), 16, 40).startswith("units 1")
    assert path(32, 8, [(1, 540)] * 4, (0, 0), 16, 40000) == "spans 1"
