"""The paged attention's index arithmetic on the host: every row looks at exactly its set, once, over all ranges of its tile's list, and lengths
or page numbers that make no sense name no memory."""
import ctypes
import os
import subprocess

import numpy as np
import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
BIG = 1 << 40
TILE = 128


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    so = str(tmp_path_factory.mktemp("native") / "paged_list.so")
    subprocess.run(["g++", "-O2", "-std=c++17", "-shared", "-fPIC", "-fsanitize=undefined", "-fno-sanitize-recover=undefined",
                    "-static-libubsan", "-I", os.path.join(ROOT, "paper_2408_11746_b200", "csrc"),
                    os.path.join(ROOT, "tests", "native", "paged_list.cpp"), "-o", so], check=True)
    return ctypes.CDLL(so)


def _args(first, n, length, group, stride, reach, tile, R):
    return [first, first + n, length, first + n + 3, group, stride, ctypes.c_int64(reach), tile, R]


def _tile(lib, args):
    info = (ctypes.c_int64 * 9)()
    return list(info) if lib.list_of(*args, info) else None


def _seen_by_rows(lib, n, length, group, stride, R, splits, least, reach=BIG):
    """{row of the sequence: positions it looks at, in list order over all ranges}"""
    out, tile = {}, 0
    while True:
        args = _args(5, n, length, group, stride, reach, tile, R)
        info = _tile(lib, args)
        if info is None:
            return out
        row0, rows, t_lo, nt, p_lo, p_hi, W, N, dense = info
        assert p_lo == length - n + t_lo and p_hi == p_lo + nt - 1 and rows <= R and row0 == tile * R
        seen = {t: [] for t in range(nt)}
        end, split = 0, 0
        while True:
            lha = (ctypes.c_int64 * 3)()
            there = lib.range_of(*args, splits, least, split, lha)
            if not there:
                break
            lo, hi, active = list(lha)
            assert lo == end and hi >= lo and (hi > lo or N == 0) and split < active <= splits
            assert lo % 64 == 0
            end = hi
            pos, who = np.empty(hi - lo, np.int32), np.empty(hi - lo, np.int32)
            got = np.empty((hi - lo, nt), np.uint8)
            lib.keys_of(*args, ctypes.c_int64(lo), ctypes.c_int64(hi), pos.ctypes, who.ctypes, got.ctypes)
            for t in range(nt):
                seen[t] += pos[got[:, t] != 0].tolist()
            split += 1
        assert end == N and split == active
        for r in range(row0, row0 + rows):
            out[r] = seen[r // group - t_lo]
        tile += 1


@pytest.mark.parametrize("stride", [1 << 30, 64, 128, 100, 7, 3, 2])
@pytest.mark.parametrize("n,length,group,R", [(1, 1, 1, 16), (1, 700, 1, 16), (1, 129, 5, 16), (5, 300, 2, 16), (7, 7, 3, 16), (40, 333, 1, 32),
                                              (9, 200, 40, 32), (130, 400, 1, 128), (70, 500, 4, 128), (3, 2, 2, 16), (4, 0, 1, 16)])
def test_rows_look_at_their_sets(lib, n, length, group, R, stride):
    got = _seen_by_rows(lib, n, length, group, stride, R, splits=3, least=1)
    assert got == _seen_by_rows(lib, n, length, group, stride, R, splits=1, least=4)
    assert sorted(got) == list(range(n * group))
    for r, seen in got.items():
        i = length - n + r // group
        want = [j for j in range(i + 1) if i - j < stride or (i - j) % stride == 0]
        assert sorted(seen) == want and len(set(seen)) == len(seen)


@pytest.mark.parametrize("stride", [(1 << 31) - 1, 64, 128, 100, 33, 7, 2])
@pytest.mark.parametrize("n,length,group,R", [(1, 129, 40, 120), (7, 7, 3, 126), (40, 333, 1, 128), (9, 200, 40, 120), (130, 400, 1, 128),
                                              (70, 500, 4, 128), (3, 2, 2, 128), (4, 0, 1, 128), (300, 700, 2, 128)])
def test_tiles_of_many_rows_look_at_their_sets(lib, n, length, group, R, stride):
    out, tile = (ctypes.c_int32 * 8)(), 0
    rows = 0
    while True:
        args = _args(5, n, length, group, stride, BIG, tile, R)
        info = _tile(lib, args)
        if info is None:
            break
        row0, count, t_lo, nt, p_lo, p_hi, W, N, dense = info
        positions = {p_lo + (row0 + r) // group - t_lo for r in range(count)}
        seen = {p: [] for p in positions}
        split, end, m_end = 0, 0, 2
        while lib.walk_of(*args, 3, 2, split, out) == 1:
            first, near, far, n0, n1, m0, m1, active = list(out)
            assert n0 == end and m0 == m_end and m1 >= m0 and split < active <= 3 and (n1 > n0 or near == 0)
            end, m_end = n1, m1
            for p in positions:
                seen[p] += [k for k in range(first + TILE * n0, first + TILE * n1) if lib.near(*args, p, k)]
                seen[p] += [p - m * stride for m in range(m0, m1) if p - m * stride >= 0]
            split += 1
        assert end == near and m_end == 2 + far and split == active
        for p in positions:
            want = [j for j in range(p + 1) if p - j < stride or (p - j) % stride == 0]
            assert sorted(seen[p]) == want
        rows += count
        tile += 1
    assert rows == n * group


@pytest.mark.parametrize("length", [-(1 << 31), -5, 0, (1 << 31) - 1, (1 << 30) + 7])
@pytest.mark.parametrize("stride", [2, 64, 1000, (1 << 31) - 1])
@pytest.mark.parametrize("reach", [0, 4096, BIG])
def test_tiles_of_lengths_that_make_no_sense(lib, length, stride, reach):
    out = (ctypes.c_int32 * 8)()
    assert lib.walk_of(*_args(0, 300, length, 1, stride, reach, 1, 128), 16, 4, 0, out) == 1
    first, near, far, n0, n1, m0, m1, active = list(out)
    assert first >= 0 and first % TILE == 0 and 0 <= near <= (1 << 31) // TILE and far >= 0 and 1 <= active <= 16 and (near > 0) == (length > 300 - 128 - 128)
    assert first + TILE * near <= max(length, 0) + TILE and far <= reach // stride + 3
    if reach < length:
        assert near <= max(1, reach // TILE + 1)


@pytest.mark.parametrize("stride", [1 << 30, 64, 100, 7, 3])
@pytest.mark.parametrize("reach", [0, 1, 80, 128, 333, 400])
@pytest.mark.parametrize("R", [16, 128])
def test_rows_of_a_table_that_is_too_short(lib, stride, reach, R):
    """Positions from `reach` on need not be listed; all the others are, once."""
    n, length = 40, 400
    got = _seen_by_rows(lib, n, length, 1, stride, R, 3, 1, reach=reach)
    out = (ctypes.c_int32 * 8)()
    for r in range(n):
        i = length - n + r
        want = [j for j in range(min(i + 1, reach)) if i - j < stride or (i - j) % stride == 0]
        assert sorted(j for j in got[r] if j < reach) == want
        args = _args(5, n, length, 1, stride, reach, r // R, R)
        assert lib.walk_of(*args, 1, 8, 0, out) == 1
        first, near, far, n0, n1, m0, m1, active = list(out)
        seen = [k for k in range(first, first + TILE * near) if k < reach and lib.near(*args, i, k)] + [i - m * stride for m in range(m0, m1)]
        assert sorted(j for j in seen if 0 <= j < reach) == want


@pytest.mark.parametrize("first,end,tokens", [(0, 0, 10), (5, 4, 10), (-1, 3, 10), (4, 11, 10), (-(1 << 31), (1 << 31) - 1, 10)])
def test_rows_that_are_not_there(lib, first, end, tokens):
    info = (ctypes.c_int64 * 9)()
    assert not lib.list_of(first, end, 100, tokens, 1, 64, ctypes.c_int64(BIG), 0, 16, info)


@pytest.mark.parametrize("length", [-(1 << 31), -5, 0, (1 << 31) - 1, (1 << 30) + 7])
@pytest.mark.parametrize("stride", [2, 64, (1 << 31) - 1])
@pytest.mark.parametrize("reach", [0, 4096, BIG])
def test_lengths_that_make_no_sense(lib, length, stride, reach):
    args = _args(0, 33, length, 1, stride, reach, 1, 16)
    row0, rows, t_lo, nt, p_lo, p_hi, W, N, dense = _tile(lib, args)
    assert 0 <= W <= N < 1 << 32 and W <= max(0, reach) and N - W <= (reach // stride + 3) * nt
    if length <= 0:
        assert N == 0
    lha = (ctypes.c_int64 * 3)()
    assert lib.range_of(*args, 64, 4, 0, lha) == 1
    for n in {0, W // 2, max(W - 1, 0), W, min(W + 1, max(N - 1, 0)), max(N - 1, 0), N}:
        pos, who, got = np.empty(1, np.int32), np.empty(1, np.int32), np.empty((1, nt), np.uint8)
        lib.keys_of(*args, ctypes.c_int64(n), ctypes.c_int64(n + 1), pos.ctypes, who.ctypes, got.ctypes)
        assert -1 <= pos[0] <= max(p_hi, 0) and -1 <= who[0] < nt
        if n >= N:
            assert pos[0] == -1 and not got.any()


def test_pages_that_do_not_exist(lib):
    row = np.array([3, -1, 9, 8, -(1 << 31), (1 << 31) - 1], np.int32)
    slot = ctypes.c_int()
    want = {0: 3, 1: -1, 2: -1, 3: 8, 4: -1, 5: -1, 6: -1, 100: -1}
    for page, id_ in want.items():
        for p in (page * 7, page * 7 + 6):
            assert lib.page(row.ctypes, len(row), 7, 9, p, ctypes.byref(slot)) == id_
            assert slot.value == p % 7
    assert lib.page(row.ctypes, 0, 7, 9, 0, ctypes.byref(slot)) == -1
    assert lib.page(row.ctypes, len(row), 1, 9, (1 << 31) - 1, ctypes.byref(slot)) == -1
    assert lib.page(row.ctypes, len(row), 1, 0, 0, ctypes.byref(slot)) == -1


def test_quotients_without_division(lib):
    rng = np.random.default_rng(1)
    top = (1 << 31) - 1
    for d in list(range(1, 70)) + [100, 127, 128, 129, 1000, 4096, 65535, 65536, 65537, (1 << 30) - 1, 1 << 30, (1 << 30) + 1, top]:
        ns = {0, 1, d - 1, d, min(d + 1, top), top, top - 1, top // d * d, max(top // d * d - 1, 0)} | set(rng.integers(0, top, 200).tolist())
        for n in ns:
            assert lib.over(ctypes.c_uint32(d), ctypes.c_int(n)) == n // d


@pytest.mark.parametrize("first,end,length,tokens,want", [
    (4, 10, 100, 10, (10, 100, 0)), (4, 11, 100, 10, (10, 99, 1)), (0, 50, 50, 10, (10, 10, 1)), (4, 14, 6, 10, (10, 2, 1)),
    (10, 11, 100, 10, (10, 99, 1)), (1 << 30, (1 << 31) - 1, 5, 0, (0, 5 - (1 << 31) + 1, 1)), (-1, 3, 100, 10, (3, 100, 1)),
    (5, 4, 100, 10, (4, 100, 0)), (10, 10, 0, 10, (10, 0, 0)), (9, (1 << 31) - 1, -(1 << 31), 10, (10, -(1 << 31), 1)),
    (-(1 << 31), (1 << 31) - 1, (1 << 31) - 1, 0, (0, 0, 1)), (0, -(1 << 31), -5, 10, (-(1 << 31), -5, 0))])
def test_rows_that_the_activations_do_not_have(lib, first, end, length, tokens, want):
    """Rows beyond `tokens` are cut off and those before them stay at their positions."""
    out = (ctypes.c_int32 * 3)()
    outside = lib.rows_of(first, end, length, tokens, out)
    assert (*out[1:], outside) == want and out[0] == first
    info = (ctypes.c_int64 * 9)()
    there = lib.list_of(out[0], out[1], out[2], tokens, 1, 64, ctypes.c_int64(BIG), 0, 16, info)
    assert bool(there) == (0 <= first < min(end, tokens))
    if there and length >= 0:
        row0, rows, t_lo, nt, p_lo, p_hi = list(info)[:6]
        assert p_lo == length - (end - first) and p_hi == p_lo + rows - 1
