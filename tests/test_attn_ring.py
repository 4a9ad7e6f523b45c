"""The ring of key and value tiles of the tcgen05 attention kernel, as a model on the CPU: producer, copies, issuer and
value warp as steps in any order, barriers with their one bit of phase.  How many arrivals free a slot, and which of them are
the value warp's, is read from the source.  No order may leave a waiter stuck or let one pass before its tile has come."""
import os
import re

import pytest

SOURCE = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2404_01365_b200", "csrc", "attn_tc.cu")


def passes(completed, filling):
    """What a wait by parity answers: the phase of parity filling & 1 is not the present one."""
    return completed & 1 != filling & 1


def explore(n_slots, tiles, value_warp_frees):
    """Every reachable state of (fillings asked for, landed, products of keys, products of values, fillings the value warp
    has seen); the fault that was found, or None.  Filling i is in slot i % n_slots; even ones are keys, odd ones values."""
    total = 2 * tiles

    def completed(slot, landed):          # fillings of a slot that have landed
        return (landed - slot + n_slots - 1) // n_slots if landed > slot else 0

    start = (0, 0, 0, 0, 0)
    seen, todo = {start}, [start]
    while todo:
        asked, landed, qk, pv, saw = state = todo.pop()
        nxt = []
        if asked < total:
            before = asked - n_slots      # the filling whose place it takes
            used = before < 0 or (qk > before // 2 if before % 2 == 0 else pv > before // 2)
            if used and (before < 0 or not value_warp_frees or saw > before):
                nxt.append((asked + 1, landed, qk, pv, saw))
        if landed < asked:
            nxt.append((asked, landed + 1, qk, pv, saw))
        if qk < tiles and qk < pv + 2 and passes(completed(2 * qk % n_slots, landed), 2 * qk // n_slots):
            if landed <= 2 * qk:
                return "keys multiplied before they came", state
            nxt.append((asked, landed, qk + 1, pv, saw))
        if pv < qk and saw > 2 * pv + 1:  # (behind the value warp's word, and S of the tile)
            nxt.append((asked, landed, qk, pv + 1, saw))
        if saw < total and passes(completed(saw % n_slots, landed), saw // n_slots):
            if landed <= saw:
                return "a tile taken for there before it came", state
            nxt.append((asked, landed, qk, pv, saw + 1))
        if not nxt and state != (total, total, tiles, tiles, total):
            return "stuck", state
        for s in nxt:
            if s not in seen:
                seen.add(s)
                todo.append(s)
    return None


def arrivals():
    """(arrivals that free a slot, those by the value warp's lane for a key and a value tile) as the kernel has them."""
    with open(SOURCE) as f:
        text = f.read()
    count = int(re.search(r"mbar_init\(&kv_empty\[i\], (\d+)\)", text).group(1))
    warp = text[text.index("} else if (warp == 2) {"):text.index("} else if (warp == 3) {")]
    return count, len(re.findall(r"mbar_arrive\(&kv_empty\[", warp))


@pytest.mark.parametrize("n_slots", [4, 5, 10])
def test_no_order_of_steps_leaves_a_waiter_of_the_ring_stuck(n_slots):
    count, by_value_warp = arrivals()
    assert (count, by_value_warp) in ((1, 0), (2, 2))     # the products' commit, and the value warp for keys and values
    assert explore(n_slots, 12, by_value_warp > 0) is None


def test_the_model_sees_a_refill_that_overtakes_the_value_warp():
    assert explore(5, 12, False)[0] == "stuck" and explore(4, 12, False)[0] == "stuck"
