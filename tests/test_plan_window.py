"""The plans of windows and of 4-bit caches on the CPU: lists that hold what a split
may see, workspaces that hold the split rows and the shares, tiles that exist."""
import random

import pytest

from tests import window_probe as P


@pytest.fixture(scope="module")
def exe(tmp_path_factory):
    return P.build(str(tmp_path_factory.mktemp("window")))


def _calls(seed, n):
    rng = random.Random(seed)
    return [P.draw(rng) for _ in range(n)]


def test_what_a_tile_may_see():
    """The bound that plans are made with, against the tokens counted one by one:
    2 K half blocks, or K + 1 blocks, hold what the rows of any tile see."""
    rng = random.Random(10)
    tight = 0
    for _ in range(4000):
        Mq, H, NB = rng.randint(1, 40), rng.choice([1, 2, 5, 16, 63, 64, 65, 127, 128, 129, 300]), rng.randint(1, 9)
        window, n_sink = rng.choice([1, 2, 31, 32, 33, 64, 65, rng.randint(1, 400)]), rng.choice([0, 1, 33, rng.randint(0, 300)])
        n, qn = rng.randint(0, NB * 64 + 20), rng.randint(0, Mq)
        halves = P.window_halves(Mq, H, NB, window, n_sink)
        K = (halves + 1) // 2
        for rows in (64, 128):
            for r0 in range(0, Mq * H, rows):
                seen = set()
                for i in range(r0 // H, (min(r0 + rows, Mq * H) - 1) // H + 1):
                    p = n - qn + i
                    if i < qn and p >= 0:
                        top = min(p, NB * 64 - 1)
                        seen |= set(range(max(p - window + 1, 0), top + 1)) | set(range(min(n_sink, top + 1)))
                assert len({t // 32 for t in seen}) <= halves and len({t // 64 for t in seen}) <= K + 1
                tight += len({t // 32 for t in seen}) == halves
    assert tight > 100


def test_every_split_fits_its_list(exe):
    """A tile's units, at most 2 K half blocks (in 128-row tiles K + 1 blocks), are cut
    into S even parts: none may pass the list's 512 half blocks, or as many blocks."""
    calls = [P.Call(1, 1, 16, 2 ** 20, 2 ** 20), P.Call(3, 1, 128, 5000, 5000), P.Call(1, 600, 16, 9000, 9000, n_splits=1)]
    most = 0
    for c, both in zip(calls + _calls(11, 6000), P.plans(exe, calls + _calls(11, 6000))):
        if not c.window:
            continue
        for p in both:
            assert p.S >= 1 and p.row_tiles == -(-c.rows // (64 * p.row_groups)), (c, p)
            assert -(-2 * c.K // p.S) <= P.LIST_HALVES and -(-(c.K + 1) // p.S) <= P.LIST_HALVES, (c, p)
            most = max(most, -(-2 * c.K // p.S))
    assert most == P.LIST_HALVES  # (the limit is reached)


def test_no_more_splits_than_asked_for_or_blocks(exe):
    calls = _calls(12, 6000)
    asked = 0
    for c, (p, _) in zip(calls, P.plans(exe, calls)):
        if not c.window:
            continue
        least = -(-c.K // (P.LIST_HALVES // 2))
        if c.n_splits:
            assert p.S == max(min(c.n_splits, max(c.K, 1)), least), (c, p)
            asked += 1
        else:
            assert p.S <= max(c.K, 2, least), (c, p)
        if c.row_tile or c.rows <= 64:
            assert p.row_groups == (c.row_tile // 64 if c.row_tile and c.kv != "mx4" else 1), (c, p)
    assert asked > 1000


def test_4_bit_caches_take_64_row_tiles(exe):
    calls = _calls(13, 4000)
    n = 0
    for c, both in zip(calls, P.plans(exe, calls)):
        if c.kv == "mx4":
            assert all(p.row_groups == 1 for p in both), (c, both)
            n += 1
    assert n > 1000


def test_the_workspace_holds_rows_statistics_and_shares(exe):
    calls = [P.Call(256, 1, 128, 4096, 4096, "mx4"), P.Call(2, 1, 16, 600, 600)] + _calls(14, 6000)
    shared = 0
    for c, both in zip(calls, P.plans(exe, calls)):
        for p in both:
            if p.S <= 1:
                assert p.ws == 0 and not p.shares
                continue
            rows = c.R * p.S * c.rows
            assert p.rows_bytes == rows * 512 * (2 if p.half else 4)
            assert p.ws == p.rows_bytes + 3 * rows * 4 + (8 * P.SHARE_REQUESTS if p.shares else 0), (c, p)
            if p.shares:
                shared += 1
                # four requests a lane of 64, two ints each; their units and first splits in 32 bits
                assert c.window and c.n_splits == 0 and 1 < c.R <= P.SHARE_REQUESTS and 8 * p.S <= c.K
                assert c.R * 2 * c.K < 2 ** 31 and c.R * p.S * p.row_tiles < 2 ** 31
    assert shared > 300


def test_splits_in_two_at_least(exe):
    """Long sequences of up to 256 requests that leave something to share out, in grids
    of up to two waves of 128-row tiles: never one split, and then shared."""
    calls = [P.Call(128, 1, 128, 256, 256, "mx4"), P.Call(256, 1, 128, 130, 130), P.Call(256, 2, 128, 128, 128, "fp8"),
             P.Call(2, 256, 128, 400, 400)] + _calls(15, 8000)
    forced = 0
    for c, (p, cover) in zip(calls, P.plans(exe, calls)):
        tiles = c.R * -(-c.rows // 128)
        if (c.window and not c.n_splits and 1 < c.R <= P.SHARE_REQUESTS and c.K >= 128 and 2 * c.K > c.NB
                and c.NB <= 2 ** 20 and tiles <= 2 * P.CUS):
            assert p.S >= 2, (c, p)
            assert p.shares == (c.K >= 8 * p.S), (c, p)
            forced += cover.S == 1
    assert forced > 20


def _least_unit(n, S, most):
    """The search of the splits' unit: the smallest u, within a sixteenth, that all
    requests' max(1, ceil(n / u)) splits together pass B S splits with."""
    total, B = sum(n), len(n)

    def splits(u):
        return sum(max(1, -(-v // u)) for v in n)
    hi = max(1, -(-max(n) // S))
    lo = max(1, -(-total // (B * S)), -(-max(n) // most))
    while lo < hi - hi // 16:
        u = (lo + hi) // 2
        if splits(u) <= B * S:
            hi = u
        else:
            lo = u + 1
    return hi, splits(hi)


def test_shared_splits_fit_the_grid_and_the_list(exe):
    """The arithmetic of sharing splits out, for lengths of all kinds: never more
    splits than the grid has work items for, each within the list, none longer than
    an even share of the longest request."""
    rng = random.Random(16)
    calls = [c for c in _calls(17, 12000) if c.window]
    n_cases = 0
    for c, (p, _) in zip(calls, P.plans(exe, calls)):
        if not p.shares:
            continue
        cap = 2 * c.K if p.row_groups == 1 else c.K + 1
        kind = rng.randrange(4)
        n = [rng.randint(0, cap) if kind == 0 else 0 if kind == 1 else cap if kind == 2 else rng.choice([0, 1, 2, cap])
             for _ in range(c.R)]
        if not any(n):
            n[-1] = 1
        u, splits = _least_unit(n, p.S, 64)
        assert splits <= c.R * p.S, (c, p, n)
        assert u <= P.LIST_HALVES and u <= -(-max(n) // p.S), (c, p, u)
        n_cases += 1
    assert n_cases > 300
