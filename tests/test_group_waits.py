"""Waits of the tensor-core kernel of the 4-bit layers that give up: whoever meets others behind a wait, at a barrier without a limit,
has to decide with them whether to go on.  Control flow, so it is looked at in the source and in a model of the drain."""
import itertools
import os
import re

import pytest

SOURCE = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2311_15806_b200", "csrc", "group", "group_tc.cu")


def _text():
    return re.sub(r"//[^\n]*", "", open(SOURCE).read())


def _kernel():
    text = _text()
    return text[text.index("group_tc_kernel(const __grid_constant__"):text.index("static auto tc_kernel(int g)")]


def test_the_lanes_of_a_warp_leave_a_wait_together():
    """Every wait of the kernel is followed by operations of whole warps; its verdict is the warp's, at once or, in the two loops that
    everything waits for, at the end of the stage, up to which nothing is handed on that did not come."""
    assert re.search(r"bool warp_wait\([^)]*\) \{\s*return __all_sync\(0xffffffffu, mbar_wait<", _text())
    kernel = _kernel()
    stages = {"products": ("ok = mbar_wait(x_full", "ok = __all_sync(0xffffffffu, ok) != 0;", 3),
              "weights": ("bool ok = mbar_wait(c_full", "if (!__all_sync(0xffffffffu, ok)) break;", 2)}
    assert kernel.count("mbar_wait") == sum(n for _, _, n in stages.values())
    for begin, vote, waits in stages.values():
        part = kernel[kernel.index(begin):]
        part = part[:part.index(vote)]
        assert part.count("mbar_wait") == waits and "break" not in part
        assert re.findall(r"[^\n]*return[^\n]*", part) in ([], ["        if (it < W) return;"])
        for line in re.findall(r"[^\n]*(?:arrive|elect_one)[^\n]*\(.*", part):
            assert "&& ok)" in line, line


def test_the_drain_decides_before_its_barriers():
    """Named barriers stand in the drain alone, and between a wait of it and the next one the four warps agree."""
    kernel = _kernel()
    drain = kernel[kernel.index("} else if (warp >= 4 && p.split == 1) {"):kernel.index("if (CG == 1 && p.split > 1) {")]
    assert kernel.count("drain_sync()") == drain.count("drain_sync()") == 1
    waits = re.findall(r"[^\n]*warp_wait[^\n]*", drain)
    assert len(waits) == 1 and re.match(r"\s*if \(!drain_agrees\(warp_wait<64>\(.*\)\)\) break;", waits[0])
    assert drain.index("warp_wait") < drain.index("drain_sync()")
    assert re.search(r"bool drain_agrees\(bool ok\) \{[^}]*\{[^}]*bar\.red\.and\.pred q, 1, 128, p;", _text())


def _drain(ok, agree):
    """The four warps over tiles: ok[t][w], whether warp w's wait for tile t succeeds.  True: all of them get to the end."""
    tiles, at, left = len(ok), [0] * 4, [False] * 4
    waiting = [None] * 4                            # the barrier that a warp stands at
    for _ in range(8 * tiles + 8):
        for w in range(4):
            if left[w] or waiting[w]:
                continue
            if at[w] == 2 * tiles:
                left[w] = True
                continue
            t, chunk = divmod(at[w], 2)
            if chunk == 0 and not agree and not ok[t][w]:
                left[w] = True
            elif chunk == 0 and not agree:
                at[w] += 1
            else:
                waiting[w] = ("verdict" if chunk == 0 else "chunk", t)
        if all(waiting):                            # a barrier of 128 threads: it opens for all four or for none
            assert len(set(waiting)) == 1
            kind, t = waiting[0]
            go = kind == "chunk" or all(ok[t])
            for w in range(4):
                waiting[w] = None
                at[w] += 1
                left[w] = not go
    return all(left)


@pytest.mark.parametrize("agree", [True, False])
def test_model_of_the_drain(agree):
    """Over all verdicts of two tiles: with the agreement every warp gets to the end, each for itself some stay behind."""
    ends = [_drain([v[:4], v[4:]], agree) for v in itertools.product([True, False], repeat=8)]
    assert all(ends) if agree else not all(ends)
