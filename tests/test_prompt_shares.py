"""How the prompt kernels walk their shares of the work (fl_prompt.h, fl_paged_prompt.hip), as arithmetic: for offsets that ascend each
stage of each row tile is one share's, and for any others every walk ends and stays within the tables.

The plan and the kernels look a row tile's sequence up in different ways, a thread by halving and a wave by counting, which agree
where offsets ascend.  Where they do not, the plan may count units for row tiles that have no rows in the kernel's eyes."""
import random

import pytest

R, KEYS, TILE_UNITS, LEAST_UNITS = 128, 64, 6, 12


class Call:
    def __init__(self, cu, lens, T, G, cap, share, window=0, n_sink=0):
        self.cu, self.lens, self.T, self.G, self.cap, self.share, self.window, self.n_sink = cu, lens, T, G, cap, share, window, n_sink
        self.B = len(cu) - 1
        self.slots = T * G // R + self.B

    def row(self, b):
        return min(max(self.cu[b], 0), self.T)

    def first_slot(self, b):
        return self.row(b) * self.G // R + b

    def by_halving(self, slot):
        lo, hi = 0, self.B
        while hi - lo > 1:
            mid = (lo + hi) // 2
            lo, hi = (mid, hi) if self.first_slot(mid) <= slot else (lo, mid)
        return lo

    def by_counting(self, slot):
        """A wave's 64 lanes at a time; -1: no sequence."""
        lo, left = 0, self.B
        while left > 64:
            step = (left + 63) // 64
            n = max(sum(lane * step < left and self.first_slot(min(lo + lane * step, self.B - 1)) <= slot for lane in range(64)), 1)
            left, lo = min(step, left - (n - 1) * step), lo + (n - 1) * step
        n = sum(lane < left and self.first_slot(lo + lane) <= slot for lane in range(64))
        return lo + n - 1 if n else -1

    def span(self, b, slot):
        """(rows, stages) of a row tile."""
        n, tile = self.row(b + 1) - self.row(b), slot - self.first_slot(b)
        rows = min(n * self.G - tile * R, R)
        if rows <= 0 or tile < 0:
            return 0, 0
        start = max(self.lens[b], 0) - n
        i_min, i_max = start + tile * R // self.G, start + (tile * R + rows - 1) // self.G
        hi = min(i_max, self.cap - 1)
        lo = min(i_min - self.window + 1, self.cap) if self.window and i_min >= self.window else 0
        lead = -(-min(self.n_sink, lo) // KEYS)
        return rows, 0 if hi < 0 else lead + max(hi // KEYS - max(lead, lo // KEYS) + 1, 0)

    def plan(self):
        ends, total = [], 0
        for slot in range(self.slots):
            rows, tiles = self.span(self.by_halving(slot), slot)
            total += TILE_UNITS + max(tiles, 1) if rows else 0
            ends.append(total)
        return ends

    def walk(self, ends, wg, bounded=True):
        """(slot, first stage, end, place of its part or None) of a workgroup; IndexError where it leaves the table."""
        total = ends[-1]
        per = max(LEAST_UNITS, -(-total // self.share))
        at, end = min(total, per * wg), min(total, per * (wg + 1))
        if at >= end:
            return
        slot, first = next(s for s, e in enumerate(ends) if e > at), at
        while at < end and (slot < self.slots or not bounded):
            b = self.by_counting(slot)
            if b < 0:
                return
            rows, tiles = self.span(b, slot)
            if rows:
                units = max(tiles, 1)
                unit0 = ends[slot] - units
                t0, t1 = max(at - unit0, 0), min(end - unit0, units)
                place = 0 if unit0 + t0 == first else 1
                at = min(ends[slot], end)
                if t0 < t1:
                    yield slot, t0, t1, None if t0 == 0 and t1 == units else place
            slot += 1
            if slot > self.slots:
                raise IndexError(slot)


def ascending(rng, B, most):
    cu = [0]
    for _ in range(B):
        cu.append(cu[-1] + rng.choice([0, 1, rng.randrange(most)]))
    return cu


def any_order(rng, B, T):
    return [rng.choice([0, T, -3, 2 * T, rng.randrange(T + 1)]) for _ in range(B + 1)]


@pytest.mark.parametrize("seed", range(40))
def test_shares_of_offsets_that_ascend(seed):
    rng = random.Random(seed)
    B, G = rng.choice([1, 2, 5, 70, 130]), rng.choice([1, 3, 8])
    cu = ascending(rng, B, 3000 // B + 2)
    lens = [b - a + rng.choice([0, 0, 5, 900]) - rng.choice([0, 0, 3]) for a, b in zip(cu, cu[1:])]
    c = Call(cu, lens, cu[-1] + rng.choice([0, 2]), G, rng.choice([640, 4096]), rng.choice([1, 7, 64]), *rng.choice([(0, 0), (100, 70)]))
    ends = c.plan()
    done, parts = {}, set()
    for wg in range(c.share):
        for slot, t0, t1, place in c.walk(ends, wg):
            assert (wg, place) not in parts
            parts |= {(wg, place)} if place is not None else set()
            for t in range(t0, t1):
                assert (slot, t) not in done
                done[slot, t] = wg
    for slot in range(c.slots):
        rows, tiles = c.span(c.by_counting(slot), slot)
        assert sum(s == slot for s, _ in done) == (max(tiles, 1) if rows else 0)


OTHERS = [
    # offsets, rows, query heads of a key/value head
    ([0, 1000, 100, 100], 1000, 1),
    ([0, 0, 1000, 3], 1000, 2),
    ([1000, 0, 1000, 0, 1000], 1000, 1),
    ([500, 400, 300, 200, 100, 0], 700, 4),
    ([0, -7, 5000, 20], 640, 2),
]


def check_walks(c):
    ends = c.plan()
    assert len(ends) == c.slots and all(a <= b for a, b in zip(ends, ends[1:]))
    for wg in range(c.share):
        for slot, t0, t1, place in c.walk(ends, wg):
            rows, tiles = c.span(c.by_counting(slot), slot)
            assert 0 <= t0 < t1 <= max(tiles, 1) and place in (None, 0, 1)


@pytest.mark.parametrize("case", range(len(OTHERS)))
def test_walks_over_offsets_that_do_not_ascend_end(case):
    cu, T, G = OTHERS[case]
    for share in (1, 4, 64, 512):
        check_walks(Call(cu, [5000] * (len(cu) - 1), T, G, 8192, share))


@pytest.mark.parametrize("seed", range(40))
def test_walks_over_any_offsets_end(seed):
    rng = random.Random(seed)
    B, T = rng.choice([1, 2, 5, 70, 200]), rng.choice([1, 130, 2000])
    lens = [rng.choice([-5, 0, 100, 5000, 2 ** 31 - 1]) for _ in range(B)]
    check_walks(Call(any_order(rng, B, T), lens, T, rng.choice([1, 3, 8]), rng.choice([640, 8192]), rng.choice([1, 7, 64])))


def test_units_alone_do_not_end_a_walk():
    """What the bound on row tiles is for."""
    cu, T, G = OTHERS[0]
    c = Call(cu, [5000] * 3, T, G, 8192, 64)
    ends = c.plan()
    with pytest.raises(IndexError):
        for wg in range(c.share):
            list(c.walk(ends, wg, bounded=False))
