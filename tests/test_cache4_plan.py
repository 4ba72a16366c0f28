"""How the attention over a cache of 4 bits cuts its work, without a GPU: every unit of every row is in one share, whatever teams a
workgroup has, and every part of a cut item is joined once."""
import ctypes as C
import random

import pytest

from tests import servehost

I, U, L = C.c_int, C.c_uint32, C.c_int64
FORMS = [(1, 4, 32), (4, 1, 32), (4, 1, 64)]                 # groups of 32 rows in a tile, teams of a workgroup, keys of a unit


@pytest.fixture(scope="module")
def lib():
    return servehost.build("""
#include "attn_plan.hpp"
using namespace stand;
extern "C" {
int64_t units(int64_t len, int64_t most, int keys) { return item_units(len, most, 1, keys); }
int64_t head(int rows, int tile) { return head_weight(rows, tile, 1, 1); }
int64_t before(int64_t place, int start, int64_t units) { return units_before(place, 1, start, units); }
int64_t groups(int64_t total, int launched, int start) { return attn_groups(total, launched, start, 1); }
int64_t begin(int64_t w, int64_t total, int64_t W) { return group_start(w, total, W); }
int64_t owner(int64_t unit, int64_t total, int64_t W) { return group_of(unit, total, W); }
int64_t first(int64_t item, int64_t total, int64_t W, int start) { return first_group(item, total, W, start, 1); }
int64_t share(unsigned workgroup, int team, int teams, int64_t W)
{ long long w; return share_of_team(workgroup, team, teams, W, w) ? w : -1; }
int row(int tile, int rows, int groups) { return tile_row(tile, rows, groups); }
}""", dict(units=([L, L, I], L), head=([I, I], L), before=([L, I, L], L), groups=([L, I, I], L), begin=([L, L, L], L), owner=([L, L, L], L),
           first=([L, L, L, I], L), share=([U, I, I, L], L), row=([I, I, I], I)))


@pytest.mark.parametrize("teams", [1, 2, 4])
def test_every_share_belongs_to_one_team(lib, teams):
    for workgroups in (8, 16, 256, 512, 1024):
        for W in sorted({0, 1, 2, 7, 8, 9, 63, 64, 65, workgroups * teams // 2 + 3, workgroups * teams - 1, workgroups * teams}):
            if W > workgroups * teams:
                continue
            got = [lib.share(g, t, teams, W) for g in range(workgroups) for t in range(teams)]
            assert sorted(w for w in got if w >= 0) == list(range(W)), (workgroups, W)
            # neighbours stay with an XCD: the shares of one are a run
            for x in range(8):
                mine = sorted(lib.share(g, t, teams, W) for g in range(x, workgroups, 8) for t in range(teams))
                mine = [w for w in mine if w >= 0]
                assert mine == list(range(mine[0], mine[0] + len(mine))) if mine else True


@pytest.mark.parametrize("groups", [1, 4])
def test_tiles_have_every_row_once(lib, groups):
    for rows in list(range(1, 700)) + [1024, 1025, 28 * 1024, 65535 * 1024]:
        tiles = lib.head(rows, 32 * groups)
        ends = [lib.row(t, rows, groups) for t in ([0, 1, tiles // 2, tiles - 1, tiles] if tiles > 3000 else range(tiles + 1))]
        assert ends[0] == 0 and ends[-1] >= rows > lib.row(tiles - 1, rows, groups)
        if tiles <= 3000:
            sizes = [(min(rows, b) - a + 31) // 32 for a, b in zip(ends, ends[1:])]
            assert all(a % 32 == 0 for a in ends) and min(sizes) >= 1 and max(sizes) <= groups and max(sizes) - min(sizes) <= 1


@pytest.mark.parametrize("kind", ["short", "any", "long"])
@pytest.mark.parametrize("groups,teams,keys", FORMS)
def test_shares_cover_every_unit_once(lib, kind, groups, teams, keys):
    """The kernel's walk over its shares, team by team, and what the join does with the parts."""
    START, TM = 6, 32 * groups
    rng = random.Random(groups * 100 + keys + len(kind))
    for rep in range(40):
        B = rng.choice([1, 2, 7, 40]) if kind != "long" else rng.choice([1, 2])
        per, heads, most = rng.choice([1, 4, 7]), rng.choice([1, 2, 8]), 1 << 16
        N = {"short": rng.choice([1, 2]), "any": rng.choice([1, 3, 32, 130, 1024]), "long": rng.choice([1, 9, 64])}[kind]
        lens = [{"short": rng.randrange(3), "any": rng.choice([0, 1, 5, 31, 32, 33, 64, 65, rng.randrange(9000), -3]), "long": rng.choice([60001, most + 9, 8191])}[kind]
                for _ in range(B)]
        drafted = [rng.choice([0, 1, N, rng.randrange(N + 1)]) for _ in range(B)]
        workgroups = rng.choice([8, 256, 512])
        launched = workgroups * teams
        items, total = [], 0                                   # (trajectory, head, tile, first place, units)
        for b, (n, t) in enumerate(zip(lens, drafted)):
            u = lib.units(n, most, keys)
            assert u == -(-min(max(n, 0), most) // keys) + 1   # the cached keys, and the whole tree
            tiles = lib.head(t * per, TM)
            assert tiles == -(-t * per // TM)
            for h in range(heads):
                for tile in range(tiles):
                    items.append((b, h, tile, total, u))
                    total += u + START
        W = lib.groups(total, launched, START)
        assert 0 <= W <= launched and (W > 0) == (total > 0)
        if not total:
            continue
        starts = {i[3]: k for k, i in enumerate(items)}
        places = sorted(starts)
        done, records, written = {}, {}, [0] * launched
        for g in range(workgroups):
            for team in range(teams):
                if g * teams + team >= W:                      # a record of nothing for the number that no share has
                    written[g * teams + team] += 1
                w = lib.share(g, team, teams, W)
                if w < 0:
                    continue
                place, end = lib.begin(w, total, W), lib.begin(w + 1, total, W)
                lo, hi = 0, len(places) - 1
                while lo < hi:
                    mid = (lo + hi + 1) // 2
                    lo, hi = (mid, hi) if places[mid] <= place else (lo, mid - 1)
                for k in range(lo, len(items)):
                    s, u = items[k][3:]
                    u0, u1 = lib.before(place - s, START, u), lib.before(end - s, START, u)
                    if place >= end or u1 == 0:
                        break
                    assert 0 <= u0 < u1 <= u
                    if w not in records:
                        written[w] += 1
                        records[w] = (k, lib.first(s, total, W, START), lib.owner(s + u + START - 1, total, W), u0 > 0)
                    done.setdefault(k, []).append((u0, u1, w))
                    if u1 < u:
                        break
                    place = s + u + START
        assert written == [1] * launched and len(records) == W   # every record is written, by one team
        assert len(done) == len(items)
        for k, (b, h, tile, s, u) in enumerate(items):
            parts = sorted(done[k])
            assert [p[0] for p in parts] == [0] + [p[1] for p in parts[:-1]] and parts[-1][1] == u
            if len(parts) > 1:                                 # joined by the second share's record, from all of the shares
                ws = [p[2] for p in parts]
                assert ws == list(range(ws[0], ws[-1] + 1))
                for w in ws[1:]:
                    assert records[w] == (k, ws[0], ws[-1], True)
        for w, (k, a, b, cut) in records.items():
            if not cut:
                assert min(done[k])[2] == w
