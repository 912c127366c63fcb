"""The LDS addresses of the 8-bit kernels, from the functions that the kernels call (compiled for
the host): every chunk is read where it was written, inside its buffer, no two share a place, and
the lanes that are served together meet all banks."""
from __future__ import annotations

import os
import subprocess

import pytest

ROOT = os.path.abspath(os.path.join(os.path.dirname(__file__), ".."))


@pytest.fixture(scope="module")
def places(tmp_path_factory):
    """{"tile": {...}, 64: {...}, 128: {...}, 256: {...}}, each name -> list of number tuples."""
    exe = str(tmp_path_factory.mktemp("places") / "places")
    subprocess.run(["g++", "-std=c++17", "-Wall", "-Werror", "-I",
                    os.path.join(ROOT, "paper_2112_13896_amd", "csrc"), "-o", exe,
                    os.path.join(ROOT, "tests", "q8_places.cpp")], check=True)
    text = subprocess.run([exe], check=True, capture_output=True, text=True).stdout
    out, cur = {}, None
    for line in text.splitlines():
        name, *nums = line.split()
        nums = tuple(map(int, nums))
        if name in ("tile", "many"):
            cur = out.setdefault(nums[0] if nums else "tile", {"sizes": nums})
        else:
            cur.setdefault(name, []).append(nums)
    return out


def _written(rows):
    place = {}
    for at, row, chunk in rows:
        assert at % 16 == 0 and at not in place
        place[at] = (row, chunk)
    return place


def _no_conflicts(reads):
    """reads: addresses of lanes 0 .. 63 of one 16-byte read.  Served in four groups of sixteen
    lanes: of each 32, lanes 0-3, 12-15, 20-27 and the others."""
    a = [x for x in range(32) if x < 4 or 12 <= x < 16 or 20 <= x < 28]
    b = [x for x in range(32) if x not in a]
    for half in (0, 32):
        for group in (a, b):
            columns = [reads[half + x] // 16 % 16 for x in group]
            assert len(set(columns)) == 16, columns


def test_linear_tile(places):
    t = places["tile"]
    place = _written(t["piece"])
    assert len(place) == 256 * 8 and max(place) == 256 * 128 - 16
    assert set(place.values()) == {(r, c) for r in range(256) for c in range(8)}
    assert all(place[at] == (row, chunk) for at, row, chunk in t["at"])
    assert len(t["at"]) == 256 * 8
    # a tile of fewer rows is the start of this one
    for rows in (64, 128):
        assert all(place[at][0] < rows for at in place if at < rows * 128)
    by = {(row, chunk): at for at, row, chunk in t["at"]}
    for first in range(0, 256, 32):
        for s in range(4):
            _no_conflicts([by[first + x % 32, 2 * s + x // 32] for x in range(64)])


@pytest.mark.parametrize("DT", [64, 128, 256])
def test_attention_keys_and_values(places, DT):
    p = places[DT]
    buffer = 64 * DT * 2
    assert p["sizes"] == (DT, buffer, 4 if DT == 64 else 8)
    keys, values = _written(p["key_put"]), _written(p["value_put"])
    assert set(keys.values()) == {(k, c) for k in range(64) for c in range(DT // 8)}
    assert set(values.values()) == {(c, g) for c in range(DT) for g in range(8)}
    assert max(keys) == max(values) == buffer - 16
    assert len(p["key_at"]) == 64 * DT // 8 and len(p["value_at"]) == DT * 8
    assert all(keys[at] == (row, chunk) for at, row, chunk in p["key_at"])
    assert all(values[at] == (row, chunk) for at, row, chunk in p["value_at"])
    key = {(row, chunk): at for at, row, chunk in p["key_at"]}
    value = {(row, chunk): at for at, row, chunk in p["value_at"]}
    for k in range(DT // 16):
        for u in range(2):
            _no_conflicts([key[32 * u + x % 32, 2 * k + x // 32] for x in range(64)])
    for v in range(4):
        for ct in range(DT // 32):
            _no_conflicts([value[32 * ct + x % 32, 2 * v + x // 32] for x in range(64)])


@pytest.mark.parametrize("DT", [64, 128, 256])
def test_a_chunk_of_values_holds_the_keys_of_a_lanes_weights(places, DT):
    pairs = places[DT]["pair"]
    assert all(a == b for a, b in pairs) and sorted(a for a, _ in pairs) == list(range(64))
