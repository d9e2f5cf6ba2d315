"""Rows that the paged attention goes through, from the library's own header
compiled without device code: every row that a token sees lies in a tile, no
tile comes twice, and nothing wraps where lengths come near 2^31."""
import ctypes
import os
import subprocess

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
ALL = 2**31 - 1  # the window of a call without one


@pytest.fixture(scope="module")
def sight(tmp_path_factory):
    out = str(tmp_path_factory.mktemp("host_paged") / "host_paged.so")
    hipcc = os.path.join(os.environ.get("ROCM_PATH", "/opt/rocm"), "bin", "hipcc")
    subprocess.run([hipcc, "-x", "hip", "--offload-host-only", "-std=c++17", "-O1", "-fPIC", "-shared",
                    "-Wno-unused", os.path.join(HERE, "host_paged.cpp"), "-o", out], check=True)
    lib = ctypes.CDLL(out)

    def call(*args):
        got = (ctypes.c_int * 6)()
        lib.host_sight(*args, got)
        return list(got)

    return call


def listed(first, top, last, head, gap, tiles):
    return [i if i < head else i + gap for i in range(max(tiles, 0))]


@pytest.mark.parametrize("tile_rows", [16, 32, 64])
def test_tiles_hold_what_is_seen(sight, tile_rows):
    for most in (48, 208):
        for row0 in (-3, 0, 15, 47, 63, 64, 130, 300):
            for new in (1, 2, 17, 70):
                for window, sinks in ((ALL, 0), (ALL, 9), (1, 0), (16, 1), (33, 40), (100, 64), (5, 500)):
                    got = sight(row0, most, 2, 0, 2 * new, tile_rows, window, sinks)
                    tiles = listed(*got)
                    seen = set()
                    for r in range(row0, row0 + new):
                        for j in range(min(r + 1, most)):
                            if j > r - window or j < sinks:
                                seen.add(j // tile_rows)
                    where = (most, row0, new, window, sinks, got)
                    assert len(set(tiles)) == len(tiles), where
                    assert seen <= set(tiles), where
                    assert all(0 <= t and t * tile_rows < most for t in tiles), where
                    assert got[2] == min(row0 + new - 1, most - 1) or got[2] == -1, where


@pytest.mark.parametrize("tile_rows", [16, 32, 64])
def test_first_rows_of_lengths_near_the_largest(sight, tile_rows):
    """As many first rows as a sequence near 2^31 is long: all that the table
    holds are in sight, whether or not the lengths pass the table."""
    for most in (16, 640, 2**31 - 65536):
        for row in (2**31 - 2, 2**31 - 17, 2**31 - 64, 2**31 - 65):
            for window in (1, 5, 64):
                for sinks in (ALL, 2**31 - 20, 2**31 - 64):
                    got = sight(row, most, 1, 0, 1, tile_rows, window, sinks)
                    assert got[2] == most - 1
                    assert got[5] == -(-most // tile_rows), (most, row, window, sinks, got)
                got = sight(row, most, 1, 0, 1, tile_rows, window, 3)
                assert got[5] == 1 and listed(*got) == [0], (most, row, window, got)
