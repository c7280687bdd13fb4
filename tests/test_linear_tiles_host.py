"""The table of tiles of the grouped linear layers at the largest sizes and with offsets that are not
valid, built for the CPU (no GPU needed): counts are exact where offsets are valid, and whatever
they say the table never falls, stays within its limit, and the shares of it are in order and
inside all items."""
import ctypes
import itertools
import os
import shutil
import subprocess

import pytest

import paper_2505_17826_amd as R
from paper_2505_17826_amd import build_lib as B

GXX = shutil.which("g++")
MOST_ROWS = 2 ** 31 - 512
LARGEST = 2 ** 30 - 1  # limit of a table
START = 8           # what a tile of d_weight takes besides its stages


@pytest.fixture(scope="module")
def tables(tmp_path_factory):
    if not GXX:
        pytest.skip("g++ not available")
    exe = str(tmp_path_factory.mktemp("t") / "tiles")
    src = os.path.join(os.path.dirname(__file__), "linear_tiles_cpu.cpp")
    r = subprocess.run([GXX, "-O1", "-std=c++17", "-w", "-ftrapv", "-pthread", "-I", B.CSRC, src, "-o", exe],
                       capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr[-2000:]

    def run(cases):  # -1: the header's own largest limit
        cases = [(*c[:4], -1 if c[4] == LARGEST else c[4], *c[5:]) for c in cases]
        text = "".join(" ".join(map(str, (*c[:8], *c[8]))) + "\n" for c in cases)
        r = subprocess.run([exe], input=text, capture_output=True, text=True, timeout=300)
        assert r.returncode == 0, (r.returncode, r.stderr[-500:])  # -ftrapv: no sum passes an int
        out = [list(map(int, line.split())) for line in r.stdout.splitlines()]
        return [(o[:c[1] + 1], o[c[1] + 1:]) for c, o in zip(cases, out)]

    return run


def valid_offsets():
    for rows in (0, 1, 255, 2 ** 20 + 3, 2 ** 29, 2 ** 30 + 1, MOST_ROWS):
        yield rows, [0, rows]
        yield rows, [0] * 700 + [rows] * 325
        yield rows, [rows * i // 1024 for i in range(1025)]
        yield rows, [0, rows // 3, rows // 3, rows // 3 * 2, rows, rows]
    yield MOST_ROWS, [5] * 3 + [MOST_ROWS - 7] * 2


def other_offsets():
    for rows in (64, 2 ** 27, 2 ** 29, 2 ** 30, MOST_ROWS):
        for E in (3, 255, 1024):
            yield rows, [rows if i % 2 else 0 for i in range(E + 1)]
            yield rows, [0 if i % 2 else rows for i in range(E + 1)]
            yield rows, [2 ** 31 - 1 if i % 3 else -2 ** 31 for i in range(E + 1)]
            yield rows, [rows - rows * i // E for i in range(E + 1)]


def check_shares(shares, E, each):
    assert shares[0] == 0 and shares[-1] == E * each
    assert all(a <= b for a, b in zip(shares, shares[1:])), shares


@pytest.mark.parametrize("block_rows,across,most", [(256, 8, LARGEST), (128, 15, LARGEST), (64, 30, LARGEST)])
def test_tiles_of_valid_offsets(tables, block_rows, across, most):
    cases = [(r, len(o) - 1, across, 0, most, block_rows, 0, 0, o) for r, o in valid_offsets()]
    for c, (tab, _) in zip(cases, tables(cases)):
        o = c[8]
        want = list(itertools.accumulate((-(-(b - a) // block_rows) * across for a, b in zip(o, o[1:])),
                                         initial=0))
        assert tab == [min(w, most) for w in want], c[:8]


@pytest.mark.parametrize("each,slices", [(1, 1), (8, 1), (225, 2), (1 << 17, 1)])
def test_shares_of_valid_offsets(tables, each, slices):
    """Costs of d_weight: the groups' stages, `each` tiles of a group of equal cost."""
    more = START * slices
    cases = [(r, len(o) - 1, 1, more, LARGEST, 64, each, 8, o) for r, o in valid_offsets()]
    for c, (tab, shares) in zip(cases, tables(cases)):
        o, E = c[8], c[1]
        want = list(itertools.accumulate((-(-(b - a) // 64) + more for a, b in zip(o, o[1:])), initial=0))
        assert tab == want, c[:8]
        check_shares(shares, E, each)
        for p, s in enumerate(shares):
            # the share begins where p eighths of the cost are behind, to one tile
            e, i = divmod(s, each)
            cost = want[e] * each + (want[min(e + 1, E)] - want[e]) * i
            widest = max(b - a for a, b in zip(want, want[1:]))
            assert abs(cost - want[E] * each * p / 8) <= widest, (c[:8], p)


@pytest.mark.parametrize("block_rows,across,more,most,each",
                         [(64, 1, START, LARGEST, 1), (64, 1, START, LARGEST, 8), (64, 1, START, LARGEST, 1 << 17),
                          (256, 8, 0, 2 ** 27, 0), (128, 15, 0, 2 ** 28 + 5, 0), (64, 30, 0, LARGEST, 0)])
def test_other_offsets_stay_inside(tables, block_rows, across, more, most, each):
    cases = [(r, len(o) - 1, across, more, most, block_rows, each, 8, o) for r, o in other_offsets()]
    for c, (tab, shares) in zip(cases, tables(cases)):
        assert tab[0] == 0 and tab[-1] <= most, c[:8]
        assert all(a <= b for a, b in zip(tab, tab[1:])), c[:8]
        if each:
            check_shares(shares, c[1], each)


@pytest.mark.parametrize("dt", (R.RFT_BF16, R.RFT_F32))
def test_most_rows(dt):
    """Rows are counted in 32 bits, with a tile's rows more."""
    L, fake = R.lib(), ctypes.c_void_p(0x1000)

    def status(rows):
        g = ctypes.byref(R.rft_groups(rows, 1, None, None, 1, 0))
        # with no workspace (needed here: nothing is ever enqueued) and unknown act: refused in any case
        return (L.rft_linear(g, fake, fake, dt, 8, 8, None, 9, None, fake, None, None, 0, None),
                L.rft_linear_bwd(g, fake, fake, fake, fake, dt, 8, 8, 1, fake, fake, R.RFT_F32, fake, 0, None, 0,
                                 None))

    assert status(MOST_ROWS) == (R.RFT_E_PARAM, R.RFT_E_WORKSPACE)
    assert status(MOST_ROWS + 1) == (R.RFT_E_SHAPE, R.RFT_E_SHAPE)
    assert status(2 ** 31 - 1) == (R.RFT_E_SHAPE, R.RFT_E_SHAPE)
