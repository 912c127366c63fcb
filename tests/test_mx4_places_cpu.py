"""LDS places of the 4-bit attention kernel's operands, from the functions that the kernel calls
(mx4_places.h), compiled for the host: every chunk is read where it was written, rows meet the keys
and channels they are meant for, and a column of chunks is read without bank conflicts."""
from __future__ import annotations

import os
import shutil
import subprocess

import numpy as np
import pytest

from paper_2112_13896_amd import build

HERE = os.path.dirname(os.path.abspath(__file__))
# the lanes of 32 that a 16-byte read serves together
SERVED = [[*range(0, 4), *range(12, 16), *range(20, 28)], [*range(4, 12), *range(16, 20),
                                                           *range(28, 32)]]


@pytest.fixture(scope="module")
def places(tmp_path_factory):
    exe = str(tmp_path_factory.mktemp("places") / "mx4_places")
    cxx = shutil.which("g++") or shutil.which("c++")
    subprocess.run([cxx, "-std=c++17", "-O1", "-I", build.CSRC, "-o", exe,
                    os.path.join(HERE, "mx4_places.cpp")], check=True)
    out = subprocess.run([exe], check=True, capture_output=True, text=True).stdout
    tables = {}
    for line in out.splitlines():
        dt, name, *values = line.split()
        tables.setdefault((int(dt), name), []).append([int(v) for v in values])
    return tables


@pytest.mark.parametrize("dt", [64, 128, 256])
def test_keys(places, dt):
    """16-byte pieces (key, 32 channels) in the cache's order."""
    at = {}
    for t, key, put in places[dt, "piece"]:
        assert key == t // (dt // 32)
        assert put % 16 == 0 and 0 <= put < 64 * dt // 2 and put not in at
        at[put] = (key, t % (dt // 32))
    assert len(at) == 64 * dt // 32
    for r, h, u, k, read in places[dt, "key"]:
        assert at[read] == (32 * u + r, 2 * k + h)


@pytest.mark.parametrize("dt", [64, 128, 256])
def test_values(places, dt):
    at = {}
    for t, c, channel, chunk, put in places[dt, "value_put"]:
        assert put % 16 == 0 and 0 <= put < dt * 128 and put not in at
        at[put] = (channel, chunk)
    assert len(at) == dt * 8
    for r, h, v, ct, read in places[dt, "value_at"]:
        assert at[read] == (32 * ct + r, 2 * v + h)


def test_keys_of_chunks_and_logits(places):
    """A lane's weights 8 v .. 8 v + 7 are of the keys whose values its chunk 2 v + h holds."""
    chunk = {(g, i): k for g, i, k in places[128, "value_key"]}
    for h, i, key in places[128, "logit"]:
        assert chunk[2 * (i // 8) + h, i % 8] == key
    assert sorted(chunk.values()) == list(range(64))
    # two blocks of four tokens: 4 s + h and 4 s + 2 + h of the step's sixteen
    for g in range(8):
        blocks = [chunk[g, i] // 4 for i in range(8)]
        assert blocks == [4 * (g // 2) + g % 2] * 4 + [4 * (g // 2) + 2 + g % 2] * 4


@pytest.mark.parametrize("dt", [64, 128, 256])
def test_no_bank_conflicts(places, dt):
    for name in ("key", "value_at"):
        by = {}
        for r, *column, read in places[dt, name]:
            by.setdefault(tuple(column), {})[r] = read // 16 % 16
        for lanes in by.values():
            for served in SERVED:
                assert len(np.unique([lanes[r] for r in served])) == 16, name
