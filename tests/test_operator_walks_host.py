"""How warps and threads of the product kernels keep in step, by models of their protocols on the CPU: nothing here runs a kernel."""
import os
import re

from paper_2103_07454_b200 import build

CSRC = os.path.join(build.HERE, "csrc")


def source(name):
    with open(os.path.join(CSRC, name)) as f:
        return f.read()


def stuck(together, tiles=3, meetings=2):
    """Two warps walk over tiles and meet `meetings` times in each; a time-out anywhere raises a flag at any moment.  Each warp looks at the flag
    by itself at the top of a tile, or both at a meeting of their own.  Whether any order of their steps leaves one waiting for good."""
    done = "done"

    def advance(pc):                                     # (tile, step): step 0 is the look, 1.. the meetings
        tile, step = pc
        return (tile, step + 1) if step < meetings else (tile + 1, 0) if tile + 1 < tiles else done
    seen, todo = set(), [((0, 0), (0, 0), False)]
    while todo:
        state = todo.pop()
        if state in seen:
            continue
        seen.add(state)
        a, b, flag = state
        if a == b == done:
            continue
        nexts = [] if flag else [(a, b, True)]
        for first, second, order in ((a, b, lambda x, y: (x, y)), (b, a, lambda x, y: (y, x))):
            if first != done and first[1] == 0 and not together:
                nexts.append((*order(done if flag else advance(first), second), flag))
        if a != done and b != done and a == b and (together or a[1] > 0):
            leave = flag and a[1] == 0
            nexts.append((done if leave else advance(a), done if leave else advance(b), flag))
        if not [s for s in nexts if s[:2] != (a, b)]:
            return True
        todo += nexts
    return False


def test_the_model_finds_what_a_look_of_ones_own_does():
    assert stuck(together=False) and not stuck(together=True)


def test_warps_that_share_a_box_leave_the_walk_together():
    """The epilogue of the orthogonal updates' products: where two warps meet at named barriers, they decide together."""
    text = source("eg_orthogonal_gemm.cuh")
    assert text.count("op_named_barrier(") == 1
    epilogue = text[text.index("} else if (warp >= 4) {"):text.index("*s_abort) {           // a wait ran out")]
    looks = re.findall(r"if \((.*s_abort.*)\) (break|continue|return);", epilogue)
    assert len(looks) == 1
    (look, _), = looks
    alone, _, shared = look.partition(" : ")
    assert alone.startswith("PARTS == 1 ?") and not stuck("op_leave_together" in shared)


def test_limits_of_waits_start_where_the_kernel_before_has_ended():
    """Every role of the products' kernel that waits on a barrier waits for the kernel before first."""
    text = source("eg_orthogonal_gemm.cuh")
    body = text[text.index("auto wait_before = "):text.index("*s_abort) {           // a wait ran out")]
    roles = re.split(r"\n    (?:if \(warp == 0|\} else if \(warp)", body)[1:]
    assert len(roles) == 3
    for role in roles:
        assert 0 < role.find("wait_before();") < role.index("mbar_wait(")
