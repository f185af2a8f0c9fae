"""How a call of many query rows is divided among workgroups: the shipped arithmetic compiled for the
CPU, over random calls."""
import ctypes
import math
import os
import shutil
import subprocess

import numpy as np
import pytest

NATIVE = os.path.join(os.path.dirname(os.path.abspath(__file__)), "native", "rows_plan.cpp")
FIELDS = ("waves", "unit_rows", "tile", "n_rb", "n_split", "min_tiles", "units", "acc_bytes", "ml_bytes",
          "n_tiles", "tile_bytes", "exp_bytes", "ws_bytes")


class Rows:
    def __init__(self, so):
        self.lib = ctypes.CDLL(so)
        self.lib.plan.argtypes = [ctypes.c_int64] * 4 + [ctypes.c_int32, ctypes.c_int64, ctypes.c_void_p]
        self.lib.spans.argtypes = [ctypes.c_uint32] * 3 + [ctypes.c_void_p]
        self.lib.spans.restype = ctypes.c_uint32

    def plan(self, batch, heads, rows, tokens, d, cus=256):
        out = np.zeros(len(FIELDS), np.int64)
        self.lib.plan(batch, heads, rows, tokens, d, cus, out.ctypes.data)
        return dict(zip(FIELDS, (int(x) for x in out)))

    def spans(self, tiles, n_split, min_tiles):
        start = np.zeros(n_split + 1, np.uint32)
        n = self.lib.spans(tiles, n_split, min_tiles, start.ctypes.data)
        return start[:n + 1].astype(np.int64)


@pytest.fixture(scope="module")
def rows(tmp_path_factory):
    cxx = shutil.which("g++")
    if cxx is None:
        pytest.skip("g++ not found")
    so = str(tmp_path_factory.mktemp("rows") / "rows.so")
    subprocess.run([cxx, "-O2", "-std=c++17", "-shared", "-fPIC", "-o", so, NATIVE], check=True)
    return Rows(so)


def test_spans_of_a_unit(rows):
    """A unit's spans cover its tiles once, differ by a tile at most, and hold min_tiles or more
    where there are several; a unit without tiles has one."""
    rng = np.random.default_rng(1)
    for _ in range(2000):
        tiles, n_split = int(math.exp(rng.uniform(0, 12))) - 1, int(math.exp(rng.uniform(0, 7)))
        start = rows.spans(tiles, n_split, 4)
        size = np.diff(start)
        assert start[0] == 0 and start[-1] == tiles and 1 <= len(size) <= n_split
        assert size.max() - size.min() <= 1 and (len(size) == 1 or size.min() >= 4)


def test_plans(rows):
    """Random calls: the units cover the rows, the workspace holds every partial and tile, and a unit
    has no more spans than its tiles give work for nor a call many more than the device has places."""
    rng = np.random.default_rng(2)
    seen = set()
    for _ in range(6000):
        batch, heads = int(math.exp(rng.uniform(0, 5))), int(rng.choice([1, 2, 4, 8, 32]))
        n_rows = int(math.exp(rng.uniform(0, 10)))
        tokens, d = max(1, int(math.exp(rng.uniform(0, 13)))), int(rng.choice([64, 128]))
        cus = int(rng.choice([32, 256, 304]))
        p = rows.plan(batch, heads, n_rows, tokens, d, cus)
        lines, tiles = batch * heads, -(-tokens // p["tile"])
        assert p["n_rb"] * p["unit_rows"] >= n_rows > (p["n_rb"] - 1) * p["unit_rows"]
        assert p["units"] == lines * p["n_rb"]
        assert (p["waves"], p["tile"]) == ((4, 32) if n_rows <= 32 else (4, 64) if n_rows <= 128 else (8, 64))
        assert p["n_rb"] == 1 or p["unit_rows"] == 256
        assert p["n_split"] >= 1 and p["ws_bytes"] == sum(
            p[k] for k in ("acc_bytes", "ml_bytes", "tile_bytes", "exp_bytes"))
        if p["n_split"] == 1:
            assert p["acc_bytes"] == p["ml_bytes"] == 0
        else:
            parts = p["units"] * p["n_split"] * p["unit_rows"]
            assert p["acc_bytes"] >= parts * d * 4 and p["ml_bytes"] >= parts * 8
            assert p["n_split"] * p["min_tiles"] <= tiles
            assert p["units"] * p["n_split"] <= 4 * 3 * cus + p["units"]
        kept = p["tile_bytes"] > 0
        assert p["tile_bytes"] == (lines * tiles * p["tile"] * 4 * d if kept else 0) <= 1 << 31
        assert p["exp_bytes"] == (lines * tiles * 32 if kept else 0)
        assert not kept or (p["waves"] == 8 and p["n_rb"] >= 4 and p["n_tiles"] == tiles)
        assert all(p[k] % 16 == 0 for k in FIELDS[7:] if k != "n_tiles")
        seen.add((p["waves"], p["tile"], p["n_split"] > 1, kept))
    assert {(8, 64, True, True), (8, 64, True, False), (8, 64, False, True), (4, 64, True, False),
            (4, 32, True, False), (4, 32, False, False)} <= seen


def test_the_number_of_spans_takes_the_least_time(rows):
    """Against the rule over every number: rounds of the device's places, times the tiles of a span
    and three more (two where the waves take tokens of their own) where there are several."""
    rng = np.random.default_rng(3)
    for _ in range(400):
        lines, n_rows = int(math.exp(rng.uniform(0, 5))), int(math.exp(rng.uniform(0, 8)))
        tokens = int(math.exp(rng.uniform(3, 12)))
        p = rows.plan(lines, 1, n_rows, tokens, 128, 256)
        places = 256 if p["waves"] == 8 else 768 if p["unit_rows"] == 16 else 512
        lanes, tiles = 4 if p["tile"] == 32 else 1, -(-tokens // p["tile"])
        most = min(tokens // (4 * p["tile"]), 4 * places // p["units"] + 1)
        cut = 2 if lanes == 4 else 3
        time = lambda n: -(-p["units"] * n // places) * (-(-tiles // (lanes * n)) + (cut if n > 1 else 0))
        assert p["n_split"] == min(range(1, max(most, 1) + 1), key=lambda n: (time(n), n))


def test_one_token_fills_the_device(rows):
    """One token of one sequence: over a long context on three quarters of the places and more, over
    a short one without partials."""
    p = rows.plan(1, 8, 4, 1 << 20, 128)
    assert p["units"] * p["n_split"] >= 256 * 3 * 3 // 4
    assert rows.plan(1, 8, 4, 100, 128)["n_split"] == 1
