"""CPU tests of the division of attention to latent caches, through the functions that the kernels call: every tile of tokens of every row tile
is somebody's, shares lie apart and inside the workspace, and the shares that are joined are those that were left."""
import bisect
import ctypes
import os
import random
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

pytestmark = pytest.mark.skipif(shutil.which("g++") is None, reason="needs g++")


@pytest.fixture(scope="module")
def rules(tmp_path_factory):
    out = str(tmp_path_factory.mktemp("latent_division") / "rules.so")
    subprocess.run(["g++", "-std=c++17", "-O1", "-shared", "-fPIC", "-Wall", "-Werror", "-I", os.path.join(ROOT, "paper_2403_11805_amd", "csrc"),
                    os.path.join(ROOT, "tests", "latent_division_driver.cpp"), "-o", out], check=True)
    lib = ctypes.CDLL(out)
    lib.latent_slot.restype = ctypes.c_int64
    lib.latent_groups.argtypes = [ctypes.c_int64, ctypes.c_int64]
    return lib


def check(rules, lens, tiles, most_tiles, n_tokens):
    """Sequences of `lens` tokens with `tiles` row tiles each, at most `most_tiles`, in a call for `n_tokens` tokens a sequence."""
    units, n = [-(-x // 32) for x in lens], len(lens)
    groups = rules.latent_groups(n * most_tiles, n_tokens)
    run = rules.latent_run(sum(u * t for u, t in zip(units, tiles)), sum(t for u, t in zip(units, tiles) if u), groups)
    ends, at = [], 0
    for u, t in zip(units, tiles):
        at += rules.latent_places(u) * t
        ends.append(at)
    assert 1 <= groups <= 256 and run >= 1 and run * groups >= at, "the line has an end that is nobody's"
    slots, shares, taken = {}, {}, {}
    piece = (ctypes.c_int32 * 4)()
    for workgroup in range(groups):
        place, run_end = workgroup * run, (workgroup + 1) * run
        while place < run_end:
            s = bisect.bisect_right(ends, place)                           # the first whose places end behind it
            if s == n:
                break
            rules.latent_piece(place, run_end, ends[s], units[s], tiles[s], piece)
            row_tile, begin, end, places = piece
            assert places >= 1 and 0 <= row_tile < tiles[s]
            place += places
            if end <= begin:
                continue
            pair = s, row_tile
            assert taken.get(pair, 0) == begin, "a tile of tokens is left out or taken twice"
            taken[pair] = end
            slot = rules.latent_slot(workgroup, s, row_tile, most_tiles)
            assert 0 <= slot < groups + n * most_tiles and slot not in slots, "a share outside the workspace or upon another"
            slots[slot] = pair
            shares.setdefault(pair, []).append(workgroup)
    for s in range(n):
        for row_tile in range(tiles[s] if units[s] else 0):
            assert taken.get((s, row_tile)) == units[s]
            joined = (ctypes.c_int32 * 2)()
            rules.latent_shares(ends[s], units[s], row_tile, tiles[s], run, joined)
            assert shares[s, row_tile] == list(range(joined[0], joined[0] + joined[1])), "what is joined is not what was left"
            assert joined[1] <= groups                                      # (as many weights as the join has room for)
            first = rules.latent_slot(joined[0], s, row_tile, most_tiles)
            assert all(slots[first + k] == (s, row_tile) for k in range(joined[1]))
    return run


def test_short_lines(rules):
    """Runs shorter than what stands in front of a row tile, so that some workgroups have nothing but that."""
    assert check(rules, [1], [1], 1, 16) == 1
    assert check(rules, [3], [1], 1, 32768) == 1
    assert check(rules, [1, 0, 40, 0], [1, 1, 1, 1], 1, 64) < 4
    assert check(rules, [64] * 7, [2, 1, 0, 3, 1, 1, 2], 3, 4096) < 4


def test_sequences_without_tokens_or_rows(rules):
    check(rules, [0], [1], 1, 16)
    check(rules, [0, 0, 0], [1, 0, 2], 2, 160)
    check(rules, [0, 500, 0, 0, 31, 0], [1, 0, 2, 1, 2, 0], 2, 512)


@pytest.mark.parametrize("lens,tiles,n_tokens", [
    ([32768] * 16, [1] * 16, 32768), ([333], [1], 336), ([3001, 5, 1500], [3, 1, 2], 3008), ([1 << 24], [2], 1 << 24), ([96] * 4500, [1] * 4500, 96),
    ([1, 31, 32, 33, 63, 64, 65], [128] * 7, 80),
])
def test_divisions(rules, lens, tiles, n_tokens):
    check(rules, lens, tiles, max(tiles), n_tokens)


@pytest.mark.parametrize("seed", range(60))
def test_drawn_divisions(rules, seed):
    rng = random.Random(seed)
    n, most = int(2 ** rng.uniform(0, 8.5)), int(2 ** rng.uniform(0, 4))
    n_tokens = 16 * int(2 ** rng.uniform(0, 11))
    lens = [0 if rng.random() < 0.1 else int(n_tokens ** rng.random()) for _ in range(n)]
    check(rules, lens, [rng.randint(0, most) for _ in range(n)], most, n_tokens)
