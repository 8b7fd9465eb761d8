"""How served turns keep an fp8 block's codes and its scales together in their
two tiers, on tiers that stand for the library's (metadata alone, no GPU):
whatever a tier evicts and whichever store is refused, a block that both tiers
hold has both halves from the same turn."""
import itertools
import types

import numpy as np
import pytest

from paper_2609_33762_amd.drivers import ServedTurns


class FakeTier:
    """Keys in slots as include/ea.h has it: allocations carry a pin and are
    resident once stored, the least recent slot without a pin is evicted, a
    slot never stored goes with its last pin."""

    def __init__(self, capacity):
        self.slots = [None] * capacity  # {key, pins, what, seen}
        self.clock = itertools.count()
        self.refuse = 0  # this many stores from now the store is refused

    def holds(self, key):
        return next((i for i, s in enumerate(self.slots) if s and s["key"] == key), None)

    def alloc(self, keys):
        out = np.full(len(keys), -1, np.int64)
        for i, key in enumerate(map(bytes, keys)):
            if self.holds(key) is not None:
                continue
            free = [j for j, s in enumerate(self.slots) if s is None]
            idle = sorted((s["seen"], j) for j, s in enumerate(self.slots)
                          if s and not s["pins"] and s["what"] is not None)
            if not free and not idle:
                continue
            j = free[0] if free else idle[0][1]
            self.slots[j] = dict(key=key, pins=1, what=None, seen=next(self.clock))
            out[i] = j
        return int((out >= 0).sum()), out

    def lookup(self, keys):
        out = []
        for key in map(bytes, keys):
            j = self.holds(key)
            if j is None or self.slots[j]["what"] is None:
                break
            self.slots[j]["pins"] += 1
            self.slots[j]["seen"] = next(self.clock)
            out.append(j)
        return len(out), np.array(out, np.int64)

    def unpin(self, slots):
        for j in slots:
            assert self.slots[j]["pins"] > 0
            self.slots[j]["pins"] -= 1
            if not self.slots[j]["pins"] and self.slots[j]["what"] is None:
                self.slots[j] = None

    def store(self, cache, pages, slots):
        assert len(pages) == len(slots)
        if self.refuse == 1:
            self.refuse = 0
            raise RuntimeError("refused")
        self.refuse = max(0, self.refuse - 1)
        for page, j in zip(pages, slots):
            assert self.slots[j]["pins"] > 0
            self.slots[j]["what"] = cache[page]


def keys_of(ids):
    return np.array([[i] * 32 for i in ids], np.uint8)


def turns(*capacities):
    t = object.__new__(ServedTurns)
    t.pairs = [(FakeTier(n), np.full(64, -1)) for n in capacities]
    return t


def store(t, ids, version):
    for _, cache in t.pairs:
        cache[:] = version
    return t._store(keys_of(ids), np.arange(len(ids)))


def whole(t):
    """Version of each block that all tiers hold."""
    held = [{s["key"][0]: s["what"] for s in tier.slots if s and s["what"] is not None}
            for tier, _ in t.pairs]
    common = set.intersection(*(set(h) for h in held))
    for k in common:
        assert len({h[k] for h in held}) == 1, ("halves of two turns", k, [h[k] for h in held])
    for tier, _ in t.pairs:
        assert not any(s and s["pins"] for s in tier.slots)
        assert not any(s and s["what"] is None for s in tier.slots)
    return {k: held[0][k] for k in common}


@pytest.mark.parametrize("capacities", [(4, 16), (16, 4), (4, 4), (4,)])
def test_a_block_that_one_tier_lost_is_stored_whole(capacities):
    t = turns(*capacities)
    assert store(t, [1, 2, 3], 1) == 3
    assert store(t, [4, 5, 6], 2) == 3        # the small tier loses 1 and 2
    assert store(t, [1, 2, 7], 3) == 3
    assert {k: v for k, v in whole(t).items() if k in (1, 2, 7)} == {1: 3, 2: 3, 7: 3}
    assert store(t, [1, 2, 7], 4) == 0        # held by both: left as it is
    assert whole(t)[1] == 3


def test_no_room_for_one_half():
    t = turns(2, 8)
    assert store(t, [1, 2, 3], 1) == 2
    assert set(whole(t)) == {1, 2}
    t.pairs[0][0].lookup(keys_of([1, 2]))     # pinned by another
    assert store(t, [3, 4], 2) == 0
    t.pairs[0][0].unpin([0, 1])
    assert set(whole(t)) == {1, 2}


@pytest.mark.parametrize("which", [0, 1])
@pytest.mark.parametrize("nth", [1, 2])
def test_a_refused_store_leaves_no_block_of_two_turns(which, nth):
    t = turns(4, 16) if which else turns(16, 4)
    store(t, [1, 2, 3], 1)
    store(t, [4, 5, 6], 2)
    t.pairs[which][0].refuse = nth
    try:
        store(t, [1, 2, 7], 3)
    except RuntimeError:
        pass
    whole(t)
    t.pairs[which][0].refuse = 0
    store(t, [1, 2, 7], 4)
    assert set(whole(t)) >= {1, 2, 7}


@pytest.mark.parametrize("plane,cache,tier", [(1, 1, 0), (1, 0, 1), (1, 0, 0), (0, 1, 1), (0, 0, 1),
                                              (0, 1, 0)])
def test_scales_without_their_cache_or_tier_are_refused(plane, cache, tier):
    one_page = types.SimpleNamespace(chunk_pages=1)
    given = types.SimpleNamespace(head_scales=object() if plane else None)
    with pytest.raises(ValueError):
        ServedTurns(None, given, one_page, None, 4, scale_cache=object() if cache else None,
                    scale_tier=one_page if tier else None)
