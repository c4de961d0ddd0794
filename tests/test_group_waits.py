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
    """A wait's verdict is the whole warp's, but for two loops.  Products: one elected thread's, which meets the others only at the kernel's
    end (TA), or the warp's, which votes at the end of a stage.  Where weights are widened a lane that gives up goes on with the others,
    without further waits.  In both nothing is handed on that did not come."""
    assert re.search(r"bool warp_wait\([^)]*\) \{\s*return __all_sync\(0xffffffffu, mbar_wait<", _text())
    kernel = _kernel()
    products = kernel[kernel.index("if (rank == 0 && (!TA || elect_one())) {"):]
    products = products[:products.index("} else if (rank != 0 && c.rows) {")]
    weights = kernel[re.search(r"bool ok = true;\s*for \(uint32_t it = wg;", kernel).start():]
    weights = weights[:weights.index("} else if (warp >= 4 && p.split == 1) {")]
    assert kernel.count("mbar_wait") == 6 and products.count("mbar_wait") == 4
    inner = products[products.index("for (int st = st0;"):products.index("if (ok && (TA || elect_one())) commit<CG>(d_full")]
    assert inner.count("mbar_wait") == 3 and inner.count("break") == 1 and "return" not in inner
    assert inner.index("if ((TA || elect_one()) && ok) {") < inner.index("mma_f16<") < inner.index("commit<CG>(done") < \
        inner.index("if (!TA) ok = __all_sync(0xffffffffu, ok) != 0;") < inner.index("if (!ok) break;")
    # a single thread meets no collective, and its warp is whole again before the block's barriers
    issuing = kernel[kernel.index("if (rank == 0 && (!TA || elect_one())) {"):kernel.index("} else if (warp >= 8) {")]
    assert issuing.rstrip().endswith("}\n    __syncwarp();")
    for line in products.splitlines()[1:]:
        assert not re.search(r"__\w*sync\w*\(|elect_one|warp_wait", line) or re.search(r"!TA\)|TA \|\||TA \? mbar_wait", line), line
    assert products.rstrip().endswith("if (!ok) drain_ring(done, issued, p.ring, 20000000ll);")
    assert weights.count("mbar_wait") == weights.count("ok = ok && mbar_wait(") == 2
    assert "break" not in weights and re.findall(r"[^\n]*return[^\n]*", weights) == ["        if (it < W) return;"]
    for line in re.findall(r"[^\n]*arrive[^\n]*\(.*", weights):
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
