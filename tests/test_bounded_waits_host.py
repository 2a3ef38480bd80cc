"""A bounded wait that gives up must not leave other warps at a barrier.

The epilogue of the few-rows statistics kernel waits for a tile's accumulator (a wait with a limit, which each warp may see end
in time or not) and then meets at a named barrier.  Its steps are taken from the source and run for all outcomes of the waits:
every warp has to reach the end.
"""
import itertools
import os
import re

SOURCE = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2609_10549_b200", "csrc", "head_loss.cu")
WARPS = 4


def kernel_text():
    with open(SOURCE) as f:
        text = f.read()
    begin = re.search(r"__global__[^\n]*\bhead_few_kernel\(", text).start()
    return text, text[begin:text.index("\n}\n", begin)]


def tile_steps():
    """What an epilogue warp does for a tile: ("wait", do the warps decide together?), "leave" (if it failed), "meet"."""
    text, kernel = kernel_text()
    epilogue = kernel[kernel.rindex("wait_for_previous_kernel();"):]
    steps = []
    for m in re.finditer(r"ok = (?P<wait>[^;]*wait_few\(&ctl->acc_full[^;]*);|(?P<leave>if \(!ok\) break;)|(?P<meet>bar\.sync 1, 128)", epilogue):
        if m["wait"]:
            together = "few_agree(" in m["wait"]
            if together:      # a reduction over the four warps' threads
                vote = text[text.index("bool few_agree("):]
                assert f"bar.red.and.pred q, 1, {32 * WARPS}, p" in vote[:vote.index("\n}\n")]
            steps.append(("wait", together))
        else:
            steps.append("leave" if m["leave"] else "meet")
    return steps


def stuck(steps, outcomes):
    """Runs the warps over the tiles; outcomes[tile][warp]: did its wait end in time?  The warps that never end."""
    program = [(tile, s) for tile in range(len(outcomes)) for s in steps]
    at, ok = [0] * WARPS, [True] * WARPS
    while True:
        moved = False
        for w in range(WARPS):
            while at[w] < len(program):
                tile, step = program[at[w]]
                if step == "leave":
                    at[w] = at[w] + 1 if ok[w] else len(program)
                elif step == ("wait", False):
                    ok[w] = outcomes[tile][w]
                    at[w] += 1
                else:
                    break
                moved = True
        waiting = [program[a][1] if a < len(program) else None for a in at]
        if None not in waiting:      # all of them at barrier 1
            votes = [outcomes[program[a][0]][w] for w, a in enumerate(at)]
            for w in range(WARPS):
                if waiting[w] != "meet":
                    ok[w] = all(votes)
                at[w] += 1
            moved = True
        if all(s is None for s in waiting):
            return []
        if not moved:
            return [w for w in range(WARPS) if waiting[w] is not None]


def test_the_model_finds_a_warp_that_leaves_alone():
    alone = [("wait", False), "leave", "meet", "meet"]
    assert stuck(alone, [[True] * WARPS] * 2) == []
    assert stuck(alone, [[False] * WARPS]) == []
    assert stuck(alone, [[True, False, True, True]]) == [0, 2, 3]


def test_epilogue_warps_leave_together():
    steps = tile_steps()
    assert [s for s in steps if s != "meet"] == [steps[0], "leave"] and steps[0][0] == "wait" and steps.count("meet") == 2
    for outcomes in itertools.product(itertools.product((True, False), repeat=WARPS), repeat=2):
        assert stuck(steps, outcomes) == [], outcomes
