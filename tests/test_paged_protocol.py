"""How the two softmax warps of the same rows meet in the paged prefill attention (csrc/paged_prefill.cu), as a model on the CPU.

A pair's barrier (meet, pair_sync) is passed by both warps or by none, and it cannot time out: a warp that leaves early has to
meet its partner exactly once more, wherever that is.  The model runs both warps over every short list of pieces with every
wait of either as the one that runs out, and looks for a warp that is left at a barrier, two barriers of different kinds that
meet, and shared memory that is written by one warp while the other may still use it.  It has to follow the kernel by hand:
the steps below are those of the softmax role, in its order."""
import itertools

import pytest


class Fault(Exception):
    pass


def warp(half, pieces, fails, last_meeting=True, empty_exchanges=False):
    """One warp: yields ("wait", ordered), ("meet", flag), ("sync",) or ("touch", what).  A wait is sent True or False (it ran out:
    wait number `fails`); a meeting is sent the flags of both.  ordered: passing it means that the partner has got there as well."""
    waits = itertools.count()

    def wait():
        return next(waits) != fails

    for blocks, cut in pieces:
        if not wait():                                       # the piece's description
            yield "meet", 2
            return
        ok = True
        for n in range(blocks):
            ok = wait()                                      # scores of a block
            if ok and n == 0 and (yield "meet", 0) & 2:      # the first reference has been read
                return
            flags = yield "meet", (1 if n == 1 else 0) | (0 if ok else 2)
            if flags & 2:
                return
            if flags & 1:                                    # a reference moves
                yield "touch", "sums"
                yield ("sync",)
        if blocks:
            ok = wait()                                      # the last product
            yield "touch", "sums"
            if (yield "meet", 0 if ok else 2) & 2:
                return
            yield ("sync",)
        elif empty_exchanges:
            yield "touch", "sums"
            if (yield "meet", 0) & 2:
                return
            yield ("sync",)
        yield "touch", "rows"                                # results on their way out
        if cut:
            ok = wait()                                      # all parts written, this one's number
            if not ok:
                yield "meet", 2
                return
            yield ("parts",)
    if not wait():                                           # the description that says there is no more work
        yield "meet", 2
        return
    if last_meeting:
        yield "meet", 0


def run(pieces, fails, **how):
    """Both warps to their ends.  The sums of a pair stand where the first warp stages its rows, so a `sums` of either and a
    `rows` of the first need a barrier (or an ordered wait) between them."""
    warps = [warp(h, pieces, fails[h], **how) for h in (0, 1)]
    at, touched = [None, None], [set(), set()]               # what each has used since they last met

    def step(h, value):
        try:
            at[h] = warps[h].send(value)
        except StopIteration:
            at[h] = "left"

    def advance(h):
        while at[h] != "left" and at[h][0] == "touch":
            touched[h].add(at[h][1])
            step(h, None)

    for h in (0, 1):
        step(h, None)
        advance(h)
    while at != ["left", "left"]:
        if at[0] == "left" or at[1] == "left":
            h = 0 if at[1] == "left" else 1
            if at[h][0] == "parts":                          # not a pair's barrier: its wait is bounded
                warps[h].close()
                return
            raise Fault(f"warp {h} is left at {at[h]}")
        kinds = at[0][0], at[1][0]
        if "rows" in touched[0] and "sums" in touched[1]:
            raise Fault("sums written over rows")
        if kinds == ("meet", "meet"):
            values = [at[0][1] | at[1][1]] * 2
        elif kinds in (("sync", "sync"), ("parts", "parts")):
            values = [None, None]
        elif "parts" in kinds:                               # one goes on to the wait behind it, which has to run out
            h = kinds.index("parts")
            step(h, None)
            advance(h)
            continue
        else:
            raise Fault(f"barriers of different kinds: {at}")
        touched = [set(), set()]
        for h in (0, 1):
            step(h, values[h])
            advance(h)


LISTS = [p for n in range(4) for p in itertools.product([(0, False), (0, True), (1, False), (2, False), (2, True)], repeat=n)]


def all_runs(**how):
    for pieces in LISTS:
        for fails in itertools.product([None, *range(12)], repeat=2):
            run(pieces, fails, **how)


def test_nobody_is_left_at_a_barrier_and_nothing_is_overwritten():
    all_runs()


@pytest.mark.parametrize("how, fault", [(dict(last_meeting=False), "left at"), (dict(empty_exchanges=True), "sums written over rows")])
def test_the_model_finds_what_goes_wrong_without_it(how, fault):
    """Leaving without a last meeting, and an exchange in a piece that has no block for the tile."""
    with pytest.raises(Fault, match=fault):
        all_runs(**how)
