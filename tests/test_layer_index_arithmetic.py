"""Host-side audit of the layer operators' address arithmetic (no GPU): the walk of the product kernel over the tiles of all groups,
the packing of operands off the 16-byte grid, the norms' windows and the places of their column sums, restated here and checked
against the arrays' bounds -- for offsets that are out of order or out of range too, which may give meaningless results but no
access outside the arrays."""
import itertools
import random

import pytest

from paper_1902_01064_b200 import hop


def starts(offsets, groups, rows):
    """row0 of the kernel: offsets clamped into [0, rows] and made non-decreasing; [groups + 1]: rows."""
    given = [0 if i == 0 else rows if i > groups or offsets is None else offsets[i] for i in range(groups + 2)]
    out, top = [], 0
    for v in given:
        top = max(top, min(max(v, 0), rows))
        out.append(top)
    return out


def ceil(a, b):
    return (a + b - 1) // b


def walk(way, offsets, groups, rows, n, k, TM, BN, splits):
    """(group, first row of the tile, rows left, first column, first term, terms, part) of every unit, as depth() and locate() find them."""
    dw, kBand = way == "dw", 8
    row0 = starts(offsets, groups, rows)
    col_tiles = ceil(n if way == "fwd" else k, BN)
    tiled = groups if dw else groups + 1
    tile0 = [0]
    for g in range(tiled):
        tile0.append(tile0[-1] + col_tiles * ceil(n if dw else row0[g + 1] - row0[g], TM))
    g = 0
    for unit in range(tile0[tiled] * splits):
        tile = unit // splits
        while tile >= tile0[g + 1]:
            g += 1
        t0 = row0[g]
        length = row0[g + 1] - t0 if dw else (k if way == "fwd" else n) if g < groups else 0
        slices, part, x0 = ceil(length, 64), 0, 0
        if splits > 1:
            part = unit - tile * splits
            per = ceil(slices, splits)
            c0 = min(part * per, slices)
            slices, x0 = min(per, slices - c0), c0 * 64
            length = min(length - x0, slices * 64)
            if dw:
                t0, x0 = t0 + x0, 0
        at, r0, r1 = tile - tile0[g], row0[g], row0[g + 1]
        row_tiles = ceil(n if dw else r1 - r0, TM)
        band = at // (kBand * col_tiles)
        inside = at - band * kBand * col_tiles
        wide = min(kBand, row_tiles - band * kBand)
        nt = inside // wide
        row = (0 if dw else r0) + (band * kBand + inside - nt * wide) * TM
        yield g, row, (n if dw else r1) - row, nt * BN, t0 + x0 if dw else x0, length if slices else 0, part


def some_offsets(rng, groups, rows):
    kind = rng.randrange(4)
    if kind == 0:
        return None if groups == 1 else sorted([0] + [rng.randint(0, rows) for _ in range(groups)])
    if kind == 1:
        return [0] + sorted(rng.randint(0, rows) for _ in range(groups))
    if kind == 2:                                   # out of order
        return [rng.randint(0, rows) for _ in range(groups + 1)]
    return [rng.choice([-2 ** 31, -5, 0, rows // 2, rows + 7, 2 ** 31 - 1]) for _ in range(groups + 1)]


@pytest.mark.parametrize("way", ["fwd", "dx", "dw"])
def test_tiles_cover_every_result_once_and_stay_inside(way):
    rng = random.Random(1)
    for _ in range(400):
        groups, rows = rng.choice([1, 2, 5, 33, 70]), rng.choice([1, 31, 128, 129, 300, 1000])
        n, k = rng.choice([1, 64, 129, 300]), rng.choice([1, 64, 130, 257])
        offsets = some_offsets(rng, groups, rows)
        TM, BN = rng.choice([(128, 128), (256, 256)])
        splits = rng.choice([1, 1, 2, 5, 16])
        row0 = starts(offsets, groups, rows)
        assert row0[0] == 0 and row0[-1] == rows and all(a <= b for a, b in itertools.pairwise(row0))
        cols, seen, terms = n if way == "fwd" else k, {}, {}
        for g, row, left, col, first, length, part in walk(way, offsets, groups, rows, n, k, TM, BN, splits):
            assert 0 <= col < cols and left > 0 and row >= 0
            key = (g if way == "dw" else 0, row, col)
            seen.setdefault(key, []).append(part)
            if way == "dw":
                assert row < n and 0 <= g < groups
                assert length == 0 or (row0[g] <= first and first + length <= row0[g + 1])      # only the group's own rows are terms
                terms.setdefault(key, []).append((first, length))
            else:
                assert row < rows and row0[g] <= row and row + min(left, TM) <= row0[g + 1]     # no tile crosses a group
                if g == groups:
                    assert length == 0                                                          # rows behind the last group: zeros
                else:
                    assert length == 0 or 0 <= first and first + length <= (k if way == "fwd" else n)
                    terms.setdefault(key, []).append((first, length))
        assert all(sorted(p) == list(range(splits)) for p in seen.values())
        if way == "dw":
            assert len(seen) == groups * ceil(n, TM) * ceil(k, BN)
        else:
            assert sum(min(TM, row0[g + 1] - r) for g in range(groups + 1) for r in range(row0[g], row0[g + 1], TM)) == rows
            assert len(seen) == ceil(cols, BN) * sum(ceil(row0[g + 1] - row0[g], TM) for g in range(groups + 1))
        for key, spans in terms.items():                                                        # the parts' terms join without gap or overlap
            g = key[0] if way == "dw" else 0
            at = row0[g] if way == "dw" else 0
            end = row0[g + 1] if way == "dw" else (k if way == "fwd" else n)
            for first, length in sorted(s for s in spans if s[1]):
                assert first == at
                at += length
            assert at == end


def test_packing_reads_units_of_its_rows_and_writes_its_own():
    for base, cols, stride, rows, groups, blocks in itertools.product([0, 2, 6, 14], [1, 7, 8, 9, 250, 257, 1001], [0, 3], [1, 5, 40], [1, 3], [1, 7]):
        row_stride = cols + stride
        group_stride = rows * row_stride + 5
        units, every = ceil(cols, 8), groups * rows
        out, order = set(), []
        for warp in range(blocks * 8):
            row = warp
            if row >= every:
                continue
            inside, g = row % rows, row // rows
            while row < every:
                while inside >= rows:
                    inside, g = inside - rows, g + 1
                order.append((g, inside))
                p0 = base + 2 * (g * group_stride + inside * row_stride)
                m = p0 & 15
                touched = ceil(m + cols * 2, 16)
                first, last = p0 - m, p0 - m + touched * 16
                assert first <= p0 and p0 + 2 * cols <= last and p0 - first < 16 and last - (p0 + 2 * cols) < 16   # no unit without a byte of the row
                mine = {row * units + u for u in range(units)}
                assert not mine & out and max(mine) < every * units
                out |= mine
                row, inside = row + blocks * 8, inside + blocks * 8
        assert sorted(order) == [(g, i) for g in range(groups) for i in range(rows)] and len(out) == every * units


def test_packing_skips_the_groups_that_the_product_does_not_read():
    """Weights are skipped by the offsets as they stand; with ordered ones exactly the groups without rows."""
    rng = random.Random(2)
    for _ in range(200):
        groups, rows = rng.choice([1, 3, 20]), rng.choice([1, 50])
        offsets = [0] + sorted(rng.randint(0, rows) for _ in range(groups))
        row0 = starts(offsets, groups, rows)
        assert [offsets[g + 1] <= (offsets[g] if g else 0) for g in range(groups)] == [row0[g + 1] == row0[g] for g in range(groups)]


@pytest.mark.parametrize("size", [2, 4])
def test_windows_read_units_of_the_row_and_zeros_behind_it(size):
    U = size // 2
    window = (32 * U + 1) * 16
    for cols, col0, skew in itertools.product([1, 7, 8, 255, 256, 257, 300, 1001, 4099], [0, 256, 512, 4096], range(0, 16, size)):
        wide = max(0, min(256, cols - col0))
        start = 4096 + skew + col0 * size                      # the warp's first byte, the row's m bytes off the grid
        row_end = 4096 + skew + cols * size
        m = start & 15
        assert m == skew                                       # 256 columns are whole units: pieces share the row's skew
        total = wide * size + m if wide else 0
        for askew in ([False, True] if m == 0 else [True]):
            for unit in range(32 * U + (1 if askew else 0)):
                n = max(0, min(16, (total if askew else wide * size) - unit * 16))
                src, dst = start - (m if askew else 0) + unit * 16, unit * 16
                assert dst + 16 <= window
                if n:
                    assert src % 16 == 0 and src + 16 > start and src + n <= row_end and src + n <= start + wide * size
        for lane in range(32):                                 # a lane's eight values lie in its own units and the next one
            mine = max(0, min(8, cols - (col0 + lane * 8)))
            assert m + (lane * 8 + mine) * size <= total or not mine
            assert lane * U * 16 + 16 * (U + 1) <= window


def test_column_sums_have_a_place_of_their_own():
    """Team t's sums of group g lie at t + g: never two at one place, never behind the workspace's teams + groups, whatever offsets
    holds; and the adding kernel finds the places of a group at its first to its last row's team."""
    rng = random.Random(3)
    for _ in range(300):
        groups, rows, per = rng.choice([1, 2, 9, 70]), rng.choice([1, 17, 200]), rng.choice([1, 3, 8])
        offsets = some_offsets(rng, groups, rows)
        teams, places, mine = ceil(rows, per), set(), {}
        for t in range(teams):
            row, end = t * per, min(rows, t * per + per)
            g, loaded = 0 if offsets is None else sum(offsets[i + 1] <= row for i in range(groups)), -1
            while row < end:
                stop = rows
                while g < groups:                              # enter(): the group that the row belongs to
                    stop = rows if offsets is None else offsets[g + 1]
                    if stop > row:
                        break
                    g, stop = g + 1, rows
                if g < groups and g != loaded:
                    assert 0 <= t + g < teams + groups and (t, g) not in mine
                    assert t + g not in places
                    places.add(t + g)
                    mine[(t, g)] = t + g
                    loaded = g
                assert stop > row
                row = min(end, max(row + 1, stop))
        for g in range(groups):
            lo = min(max(0 if offsets is None else offsets[g], 0), rows)
            hi = rows if offsets is None else min(max(offsets[g + 1], lo), rows)
            lo = 0 if g == 0 else lo
            found = list(range(lo // per, (hi - 1) // per + 1)) if hi > lo else []
            assert all(0 <= t + g < teams + groups for t in found)
            if offsets is None or (offsets[0] == 0 and offsets == sorted(offsets) and offsets[-1] <= rows):
                assert found == [t for t, h in sorted(mine) if h == g]
    assert hop.MAX_GROUPS == 1024
