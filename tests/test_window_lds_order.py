"""The order of a window prompt's LDS accesses in the built code (no GPU needed): what one wave
reads and the others wrote, or will overwrite, has a barrier of the workgroup in between.

The loop of csrc/k_window.hip takes a tile of 64 keys a turn.  Turn t reads, in this order,
  second half: K(t) from its third operand on, V(t - 1)'s second half, K(t + 1)'s first two;
  first half of the next tile: K(t + 1) from its third operand on, V(t)'s first half, the
  first two operands of K(t + 1)'s second half;
and writes K(t + 2) over K(t), then V(t + 2) over V(t - 1).  All waves write rows of every
tile, and read all rows.  The model below takes the order of reads, writes and barriers from
the instructions and lets waves be as far apart as the barriers allow."""
import re

import pytest

from test_window_code import kernels  # noqa: F401  (a fixture)

KINDS = {"ds_read_b128": "K", "ds_read_b64_tr_b16": "V", "ds_write_b128": "W", "s_barrier": "B"}


def events(code):
    """Reads of K, reads of V, writes and barriers behind the first barrier, in order."""
    out, before = [], ""
    for _, ins, _ in code:
        kind = KINDS.get(ins.split(" ")[0])
        if kind == "B":
            # (a wave's own writes have landed)
            assert re.fullmatch(r"s_waitcnt (vmcnt\(\d+\) )?lgkmcnt\(0\)", before), before
        if kind:
            out.append(kind)
        before = ins
    return out[out.index("B") + 1:]


def loop_events(code, d):
    """The loop's events: what follows the first half's logits and their successors' operands."""
    kk, mt, copies = d // 16, d // 32, 64 * (2 * d // 16) // 256
    ev = events(code)
    head = kk + 2
    assert ev[:head] == ["K"] * head
    size = 2 * kk + 8 * mt + 2 * copies + 1
    loop = ev[head:head + size]
    assert [loop.count(x) for x in "KVWB"] == [2 * kk, 8 * mt, 2 * copies, 1], loop
    tail = ev[head + size:head + size + 4 * mt]
    assert tail == ["V"] * (4 * mt), tail                       # the last half's values
    return loop


def labelled(loop, d):
    """[(what, tile less the turn's, half)]: "K" and "V" reads, "k" and "v" writes of a whole tile, "B"."""
    kk, mt, copies = d // 16, d // 32, 64 * (2 * d // 16) // 256
    k = [("K", 0, 1)] * (kk - 2) + [("K", 1, 0)] * kk + [("K", 1, 1)] * 2
    v = [("V", -1, 1)] * (4 * mt) + [("V", 0, 0)] * (4 * mt)
    w = [("k", 2, None)] * copies + [("v", 2, None)] * copies
    queues = {"K": iter(k), "V": iter(v), "W": iter(w), "B": iter([("B", 0, None)])}
    return [next(queues[x]) for x in loop]


def out_of_order(events_of_a_turn, turns):
    """The first access that no barrier keeps apart from another wave's, or None.  An access
    happens in the epoch that barriers have counted; those of different waves are ordered if
    and only if their epochs differ."""
    # what a place holds: (tile, epoch of its writes); K in two places, V in three
    place = {"k": lambda t: ("k", t % 2), "v": lambda t: ("v", t % 3)}
    written = {place["k"](t): (t, -1) for t in (0, 1)} | {place["v"](t): (t, -1) for t in (-1, 0, 1)}
    read, epoch = {}, 0
    for t in range(turns):
        for what, by, half in events_of_a_turn:
            tile = t + by
            if what == "B":
                epoch += 1
                continue
            at = place[what.lower()](tile)
            if what.isupper():
                held, when = written[at]
                if held != tile or when >= epoch:
                    return t, what, tile, half, "read in the epoch of its writes"
                read[at] = epoch
            else:
                if read.get(at, -1) >= epoch:
                    return t, what, tile, half, "overwritten in the epoch of a read"
                held, when = written[at]
                written[at] = (tile, epoch)
    return None


def test_the_model_finds_an_early_read_and_an_early_write():
    d = 128
    kk, mt, copies = 8, 4, 4
    first, second = "K" * (kk - 2) + "V" * 4 * mt, "K" * (kk - 2) + "V" * 4 * mt + "W" * 2 * copies + "KK"
    go = lambda x: out_of_order(labelled(list(x), d), 6)              # noqa: E731
    assert go(first + "B" + "KK" + second) is None
    # operands of the next tile before the barrier that shows them
    bad = go(first + "KK" + "B" + second)
    assert bad is not None and bad[1:4] == ("K", 2, 0)
    # copies before the barrier behind the last reads of what they overwrite
    assert go(first + "W" * 2 * copies + "B" + "KK" + "K" * (kk - 2) + "V" * 4 * mt + "KK") is not None
    assert go("B" + first + "KK" + second) is not None


@pytest.mark.parametrize("d", [64, 128])
def test_barriers_keep_tiles_apart(kernels, d):  # noqa: F811
    found = 0
    for name, code in kernels.items():
        if f"window_prompt_kernelILi{d}E" in name:
            bad = out_of_order(labelled(loop_events(code, d), d), 8)
            assert bad is None, (name, bad)
            found += 1
    assert found == 6                                               # three groups, split or not
