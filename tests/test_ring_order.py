"""The prompt and draft pipeline's ring of K and V tiles (csrc/flash.cuh), on the CPU: no wait passes a phase too early, and every
sequence of units can go on to its end.

Tiles take positions 0, 1, 2, ... of a ring of kStages stages.  Position p's load signals "full" barrier p mod kFulls, its consumers
(both groups, or one of them twice) "empty" barrier p mod kFulls.  A wait on a barrier's phase passes at once when the phase before
last of that barrier has not ended, so whoever waits for p must know that the phase of p - kFulls has.  What a warp knows follows
from what it has waited for: a load is issued only when the position kStages before it has been consumed, each of the two loading
warps (K and V) issues in order, and consumed means loaded."""
import itertools
import random
import re
from pathlib import Path

SOURCE = (Path(__file__).resolve().parent.parent / "paper_2608_08020_gb300" / "csrc" / "flash.cuh").read_text()
STAGES = int(re.search(r"constexpr int kStages = (\d+);", SOURCE).group(1))
FULLS = int(re.search(r"constexpr int kFulls = (\d+) \* kStages;", SOURCE).group(1)) * STAGES

# Units: ("dual" | "joint" | "alone", tiles); pairs of units, a group each: ("short" | "long", tiles, tiles).


def group_tiles(unit, first):
    """For each group the ring positions (K, V) of its tiles in turn, the unit's first tile at `first`; and how many it takes."""
    kind, n = unit[0], unit[1]
    if kind in ("short", "long"):            # the tiles come by turns while both units have some
        both, out = min(unit[1:]), []
        for g, tiles in enumerate(unit[1:]):
            at = g * (1 if kind == "long" else 2)
            k = [4 * i + at if i < both else 2 * (i + both) for i in range(tiles)]
            out.append([(first + x, first + x + (2 if kind == "long" and i < both else 1)) for i, x in enumerate(k)])
        return out, 2 * sum(unit[1:])
    mine = {"dual": [range(n)] * 2, "joint": [range(0, n, 2), range(1, n, 2)], "alone": [range(n), []]}[kind]
    return [[(first + 2 * t, first + 2 * t + 1) for t in tiles] for tiles in mine], 2 * n


def layout(units):
    """kind[p] of every position, and per group its units: (first position, tiles)."""
    kind, groups, first = {}, ([], []), 0
    for unit in units:
        tiles, n = group_tiles(unit, first)
        for g in (0, 1):
            for k, v in tiles[g]:
                assert kind.setdefault(k, "K") == "K" and kind.setdefault(v, "V") == "V"
            if tiles[g]:
                groups[g].append((first, tiles[g]))
        first += n
    assert sorted(kind) == list(range(first))     # every position once or, shared, alike
    return kind, groups


def consumed(issued, kind):
    """Positions known to be consumed when the K and the V loads up to issued["K"], issued["V"] are known to be issued."""
    issued, done, more = dict(issued), set(), True
    while more:
        more = False
        for warp in "KV":
            for p in range(max(0, issued[warp] - 40), issued[warp] + 1):
                for c in range(p - STAGES, -1, -STAGES) if kind[p] == warp else ():
                    if c not in done:
                        done.add(c)
                        issued[kind[c]] = max(issued[kind[c]], c)
                        more = True
    return done


def early_wait(units):
    """The first wait that might pass a phase too early, or None."""
    kind, groups = layout(units)
    for g in (0, 1):
        issued, own = {"K": -1, "V": -1}, set()
        for first, tiles in groups[g]:
            before = [p for p in range(max(0, first - 6), first) if kind[p] == "K"]
            issued["K"] = max([issued["K"], *before])         # the unit has begun: the K before it are on their way
            for i in range(-1, len(tiles)):                   # P.V of tile i, S of tile i + 1
                waits = ([("K", tiles[i + 1][0])] if i + 1 < len(tiles) else []) + ([("V", tiles[i][1])] if i >= 0 else [])
                for warp, p in waits:
                    if p >= FULLS and p - FULLS not in own and p - FULLS not in consumed(issued, kind):
                        return g, warp, p
                    own.add(p)
                    issued[warp] = max(issued[warp], p)
    for warp in "KV":                                         # the loading warps' waits for the stage of p - STAGES
        last = -1
        for p in (p for p in sorted(kind) if kind[p] == warp):
            if p >= STAGES + FULLS and p - STAGES - FULLS not in consumed({"K": -1, "V": -1, warp: last}, kind):
                return "load", warp, p
            last = p
    return None


def goes_on(units):
    """Loads wait for their stage, products for their tiles: everything is reached."""
    kind, groups = layout(units)
    loads = {w: [p for p in sorted(kind) if kind[p] == w] for w in "KV"}
    steps = []
    for g in (0, 1):
        steps.append([([tiles[i + 1][0]] if i + 1 < len(tiles) else []) + ([tiles[i][1]] if i >= 0 else [])
                      for _, tiles in groups[g] for i in range(-1, len(tiles))])
    needs = {p: sum(p in step for todo in steps for step in todo) for p in kind}
    there, used, moved = set(), dict.fromkeys(kind, 0), True
    while moved:
        moved = False
        for todo in loads.values():
            if todo and (todo[0] < STAGES or used[todo[0] - STAGES] == needs[todo[0] - STAGES]):
                there.add(todo.pop(0))
                moved = True
        for todo in steps:
            if todo and all(p in there for p in todo[0]):
                for p in todo.pop(0):
                    used[p] += 1
                moved = True
    return not any(loads.values()) and not any(steps)


SINGLE = [("dual", 1), ("dual", 2), ("dual", 3), ("joint", 2), ("joint", 3), ("alone", 1), ("alone", 2), ("alone", 4)]
PAIRS = [(kind, a, b) for kind in ("short", "long") for a in (1, 2, 3, 5) for b in (1, 2, 3, 5)]


def drawn(rng):
    n = lambda: rng.randint(1, 9)  # noqa: E731
    return rng.choice(SINGLE + PAIRS + [("dual", n()), ("joint", n() + 1), ("alone", n()), ("short", n(), n()), ("long", n(), n())] * 4)


def test_pairs_of_units():
    for units in itertools.product(SINGLE + PAIRS, repeat=2):
        assert early_wait(units) is None and goes_on(units), units


def test_sequences_of_units():
    rng = random.Random(1)
    for _ in range(2500):
        units = [drawn(rng) for _ in range(rng.randint(3, 9))]
        assert early_wait(units) is None and goes_on(units), units


def test_fewer_barriers_would_not_do():
    """The check sees a wait that passes too early: with ten barriers instead of fifteen there are such sequences."""
    global FULLS
    rng, kept = random.Random(2), FULLS
    try:
        FULLS = 2 * STAGES
        assert any(early_wait([drawn(rng) for _ in range(6)]) for _ in range(200))
    finally:
        FULLS = kept
