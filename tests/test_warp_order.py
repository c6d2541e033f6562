"""Where one lane acts for its warp in the kernels that stream through shared memory, the warp is
brought together first.  The lanes of a warp may run apart: a lane 0 that gives a stage back before
the others have read it, or that is still busy when the others reach a cluster barrier, is an error
that a run hardly ever shows, so the order of the statements is checked in the sources."""
import re
from pathlib import Path

import pytest

CSRC = Path(__file__).resolve().parent.parent / "paper_2305_19982_b200" / "csrc"
RINGS = ["fold_apply_multi.cu", "state8.cu", "policy_loss.cu"]


def _statements(name):
    """The file's lines without comments, blank lines left out."""
    text = re.sub(r"//[^\n]*", "", (CSRC / name).read_text())
    return [line.strip() for line in text.splitlines() if line.strip()]


@pytest.mark.parametrize("name", RINGS)
def test_a_stage_is_given_back_by_the_whole_warp(name):
    lines = _statements(name)
    arrivals = [i for i, line in enumerate(lines) if "barrier_arrive" in line and "empty[" in line]
    assert arrivals
    for i in arrivals:
        assert lines[i].startswith("if (lane == 0)")
        assert lines[i - 1] == "__syncwarp();", f"{name}: {lines[i - 1]} / {lines[i]}"


def test_cluster_barriers_are_reached_by_whole_warps():
    """They are the .aligned form, which all lanes of a warp execute together."""
    lines = _statements("policy_loss.cu")
    places = [i for i, line in enumerate(lines) if "cluster_sync();" in line]
    assert len(places) == 3
    for i in places:
        assert lines[i - 1] in ("__syncwarp();", "__syncthreads();"), f"{lines[i - 1]} / {lines[i]}"


def test_a_gradient_over_the_logits_waits_for_the_warp():
    """Rows in a warp's registers: every lane reads the target's logit, which another lane overwrites."""
    lines = _statements("policy_loss.cu")
    begin = next(i for i, line in enumerate(lines) if line.startswith("policy_loss_rows_kernel("))
    join = next(i for i in range(begin, len(lines)) if "warp_join" in lines[i])
    store = next(i for i in range(begin, len(lines)) if lines[i].startswith("const RowWriter"))
    assert join < store and "__syncwarp();" in lines[join:store]


def test_the_verdict_on_a_row_waits_for_the_warp():
    """Longer rows: the warp that does the joins reads the target's logit in every lane; its lane 0 then
    lets the other warps write over it."""
    lines = _statements("policy_loss.cu")
    arrive = next(i for i, line in enumerate(lines) if "barrier_arrive(shared_addr(&sh.ready" in line)
    begin = max(i for i in range(arrive) if lines[i] == "if (lane == 0) {")
    assert lines[begin - 1] == "__syncwarp();"


@pytest.mark.parametrize("name", ["policy_loss.cu", "grad_norm.cu"])
def test_the_thread_that_takes_the_ticket_fences_on_both_sides(name):
    """Partial sums of other threads are stored before its fence, those of other blocks read behind one:
    a fence of theirs before the warp or the block meets would not be ordered with the ticket."""
    lines = _statements(name)
    ticket = next(i for i, line in enumerate(lines) if "atomicAdd(&ws->ticket" in line)
    assert lines[ticket - 1] == "__threadfence();" and lines[ticket + 1].startswith("if (") and "__threadfence();" in lines[ticket + 1]
    before = lines[:ticket - 1]
    stores = max(i for i, line in enumerate(before) if "ws->part[" in line)
    owner = max(i for i, line in enumerate(before) if line.startswith("if (t == 0)") or line.startswith("if (threadIdx.x == 0)"))
    assert owner < stores or "__syncwarp();" in before[stores:owner]


@pytest.mark.parametrize("name,warps,threads", [("fold_apply_multi.cu", 1, 1), ("state8.cu", 2, 0), ("policy_loss.cu", 2, 1)])
def test_whichever_warp_gives_up_reports_it(name, warps, threads):
    """Not one chosen warp, which may have finished before: each role ends with a report, by one lane of the
    warp, or by the one thread that issues the copies."""
    calls = [line for line in _statements(name) if "report_expired_wait(" in line]
    assert sum(line.startswith("if (lane == 0) report_expired_wait(") for line in calls) == warps
    assert sum(line.startswith("report_expired_wait(") for line in calls) == threads
    assert len(calls) == warps + threads


def test_a_wait_looks_again_before_it_gives_up():
    """A block that was held up itself for longer than the limit finds its barrier complete: the clock is read
    last of all in a round of looks, and the flag is set a round later."""
    lines = _statements("bulk_copy.cuh")
    late = next(i for i, line in enumerate(lines) if line.startswith("late = now_ns() - t0 > kBulkWaitLimitNs"))
    begin = max(i for i in range(late) if lines[i].startswith("for ("))
    loop = lines[begin:late]
    assert loop.index("if (barrier_poll(bar, parity)) return true;") < loop.index("*give_up = 1;")
    assert any(line.startswith("if (late)") for line in loop) and sum("give_up = 1" in line for line in lines) == 1
