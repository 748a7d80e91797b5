"""How warps and threads of the product kernels keep in step, by models of their protocols on the CPU: nothing here runs a kernel."""
import os
import re
import subprocess

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


def falls_behind(part, stages=2, uses=8):
    """Three roles around a ring of stages: a thread that fetches for every one, one that may have no part in them, and the one that
    issues products and hands stages back.  A wait sees only whether the phase it asks for has another parity than the current one.
    Whether any order of their steps leaves the second fetching thread waiting for good."""
    seen, todo = set(), [(0, 0, 0)]
    while todo:
        state = todo.pop()
        if state in seen:
            continue
        seen.add(state)
        first, second, issued = state                      # stages fetched, fetched, used

        def free(at):
            s, turn = at % stages, at // stages
            handed_back = issued // stages + (issued % stages > s)
            return turn == 0 or (handed_back - 1) % 2 == (turn - 1) % 2
        nexts = []
        if first < uses and free(first):
            nexts.append((first + 1, second, issued))
        if second < uses and free(second):
            nexts.append((first, second + 1, issued))
        if issued < first and (not part or issued < second):
            nexts.append((first, second, issued + 1))
        if not nexts and state != (uses, uses, uses):
            return True
        todo += nexts
    return False


def test_the_model_finds_a_thread_that_falls_behind():
    assert falls_behind(part=False) and not falls_behind(part=True)


PARTS = """
#include "eg_gemm.cuh"
#include <stdio.h>
using namespace eg;
int bad = 0;
template <int BN> void check(int M, int N, bool a_mn, bool b_mn) {
    GemmProblem g{};
    g.M = M; g.N = N; g.a_mn = a_mn; g.b_mn = b_mn;
    g.a_box = M < 128 ? (M + 7) / 8 * 8 : 128;
    for (int m = 0; m < M; m += kGemmM)
        for (int rank = 0; rank < 2; ++rank) {
            const int row = first_row(m + rank * 128, M, a_mn);
            const unsigned bytes = a_mn ? 8192u * (1 + (row + 64 < M)) : g.a_box * 128u;
            if (row < 0 || row >= M || (a_mn && row % 8) || bytes != a_bytes(g, m + rank * 128)) ++bad;
            if (m + rank * 128 < M && row != m + rank * 128) ++bad;
        }
    for (int n = 0; n < N; n += BN)
        for (int rank = 0; rank < 2; ++rank) {
            const int row = first_row(n + rank * BN / 2, N, b_mn);
            const unsigned bytes = b_mn ? 8192u * (1 + (BN == 256 && row + 64 < N)) : BN / 2 * 128u;
            if (row < 0 || row >= N || (b_mn && row % 8) || bytes != b_bytes<BN>(g, n + rank * BN / 2)) ++bad;
            if (n + rank * BN / 2 < N && row != n + rank * BN / 2) ++bad;
        }
}
int main() {
    for (int M = 1; M < 600; ++M)
        for (int mn = 0; mn < 4; ++mn) {
            check<256>(M, M, mn & 1, mn & 2);
            check<128>(M, M, mn & 1, mn & 2);
            if (!(mn & 2)) check<64>(M, M, mn & 1, false), check<32>(M, M, mn & 1, false);
        }
    printf("%d\\n", bad);
    return 0;
}
"""


def test_every_fetching_thread_has_a_part_in_every_stage(tmp_path):
    """The feed-forward block's products: what a CTA fetches (the host runs the kernel's own functions) is a box at least, begins inside the operand
    and is what the barrier expects; no fetch hangs on a condition but that of a second box."""
    (tmp_path / "parts.cu").write_text(PARTS)
    to = str(tmp_path / "parts")
    subprocess.run([build.NVCC, *build.FLAGS, "-I", CSRC, "-o", to, str(tmp_path / "parts.cu")], check=True)
    assert subprocess.run([to], capture_output=True, text=True, check=True).stdout.strip() == "0"
    text = source("eg_gemm.cuh")
    fetch = text[text.index("if (warp == 0 || warp == 3) {"):text.index("} else if (warp == 1) {")]
    before = [fetch[:m.start()].rsplit("\n", 2)[-2:] for m in re.finditer(r"tma_load_pair\(", fetch)]
    assert len(before) == 2
    assert "if" not in before[0][1] and before[1][0].strip() == "if (mn && (warp == 0 || BN == 256) && row + 64 < rows)"
