"""What the one-token kernel waits for when a wait of its has run out: exactly the loads of that warp that are still on their way."""
import itertools

import pytest

from tests import host_rules

NONE, KEYS, VALUES = 0, 1, 2


def loads_by_hand(tiles, failing):
    """The order of a warp's loads and waits over tiles (True: has keys of its own there; False: none, or a page that is missing)
    up to the wait that runs out, (tile, KEYS or VALUES). Returns the uses of each barrier that are not waited for."""
    sent, waited = ([], []), ([], [])
    use = 0

    def send(which, tile):
        if tile < len(tiles) and tiles[tile]:
            sent[which].append(sum(tiles[:tile]))   # the how-manyth use of the barrier

    send(0, 0)
    send(1, 0)
    for tile, there in enumerate(tiles):
        if not there:
            send(0, tile + 1)
            send(1, tile + 1)
            continue
        for which, wait in ((0, KEYS), (1, VALUES)):
            if failing == (tile, wait):
                return use, tile + 1 < len(tiles) and tiles[tile + 1], *(sorted(set(s) - set(w)) for s, w in zip(sent, waited))
            waited[which].append(use)
            send(which, tile + 1)
        use += 1
    return use, False, *(sorted(set(s) - set(w)) for s, w in zip(sent, waited))


def rule(failed, use, more):
    names = "failed use_no more"
    value = "sparsed::paged_loads_on_their_way(static_cast<sparsed::PagedWait>(failed), use_no, more != 0).%s"
    return [host_rules.evaluate("paged_loads.h", value % field, names, [(failed, use, more)])[0]
            for field in ("keys", "values", "keys_use", "values_use")]


@pytest.mark.parametrize("count", [1, 2, 3, 4])
def test_what_is_waited_for(count):
    for tiles in itertools.product([True, False], repeat=count):
        for tile, wait in itertools.product(range(count), (KEYS, VALUES)):
            if not tiles[tile]:
                continue
            use, more, keys, values = loads_by_hand(tiles, (tile, wait))
            on_keys, on_values, keys_use, values_use = rule(wait, use, more)
            assert ([keys_use] if on_keys else []) == keys, (tiles, tile, wait)
            assert ([values_use] if on_values else []) == values, (tiles, tile, wait)


def test_a_warp_that_is_done_waits_for_nothing():
    for tiles in itertools.product([True, False], repeat=4):
        use, more, keys, values = loads_by_hand(tiles, None)
        assert keys == values == []
        assert rule(NONE, use, more)[:2] == [0, 0]
