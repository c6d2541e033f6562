"""Which form of the policy loss takes a call (csrc/policy_plan.h), on the CPU: whatever a card's residency,
the ring of the form that is launched holds what its rows need, and the rules pick what they say."""
import subprocess
from pathlib import Path

import pytest

ROOT = Path(__file__).resolve().parent.parent

PROGRAM = r'''
#include <stdio.h>
#include "policy_plan.h"
// lines "units rows sm_count r640_1 .. r640_8 r512_1 .. r512_8" (clusters of 1, 2, 4, 8 that run at a time);
// answers "form cluster one_turn stages stage_units", or "error n"
int main(void) {
    long long units, rows;
    int sm, r[2][4];
    while (scanf("%lld %lld %d %d %d %d %d %d %d %d %d", &units, &rows, &sm, &r[0][0], &r[0][1], &r[0][2], &r[0][3],
                 &r[1][0], &r[1][1], &r[1][2], &r[1][3]) == 11) {
        adama::PolicyPlan p;
        const int e = adama::plan_policy(units, rows, sm, [&](adama::PolicyForm f, int c, int *most) {
            *most = r[f == adama::kForm512][c == 1 ? 0 : c == 2 ? 1 : c == 4 ? 2 : 3];
            return *most < 0 ? 7 : 0;
        }, p);
        int stages = 0, stage = 0;
        switch (p.form) {
            case adama::kForm64: stages = adama::Cut64::kStages; stage = adama::Cut64::kStageUnits; break;
            case adama::kForm128: stages = adama::Cut128::kStages; stage = adama::Cut128::kStageUnits; break;
            case adama::kForm256: stages = adama::Cut256::kStages; stage = adama::Cut256::kStageUnits; break;
            case adama::kForm512: stages = adama::Cut512::kStages; stage = adama::Cut512::kStageUnits; break;
            case adama::kForm640: stages = adama::Cut640::kStages; stage = adama::Cut640::kStageUnits; break;
            default: break;
        }
        if (e) printf("error %d\n", e);
        else printf("%d %d %d %d %d\n", (int)p.form, p.cluster, (int)p.one_turn, stages, stage);
    }
    return 0;
}
'''
ROWS, RING64, RING128, RING256, RING512, RING640, LONG = range(7)
B200 = [148, 74, 33, 15]               # clusters of 1, 2, 4, 8 whole-SM blocks that run at a time on 148 SMs


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    d = tmp_path_factory.mktemp("plan")
    (d / "plan.cpp").write_text(PROGRAM)
    subprocess.run(["g++", "-std=c++17", "-Wall", "-Werror", "-I", str(ROOT / "paper_2305_19982_b200" / "csrc"),
                    str(d / "plan.cpp"), "-o", str(d / "plan")], check=True)

    def ask(cases, r640=B200, r512=B200, sm=148):
        text = "".join(f"{u} {t} {sm} {' '.join(map(str, [*r640, *r512]))}\n" for u, t in cases)
        out = subprocess.run([str(d / "plan")], input=text, capture_output=True, text=True, check=True).stdout.splitlines()
        assert len(out) == len(cases)
        return [tuple(map(int, line.split())) if not line.startswith("error") else line for line in out]

    return ask


CASES = [(u, t) for u in [1, 256, 257, 500, 768, 769, 1536, 1537, 3000, 3073, 4000, 5000, 6282, 6400, 6401, 7168, 7169, 12_000,
                          14_080, 14_081, 16_032, 28_000, 32_768, 38_000, 57_000, 57_344, 57_345, 112_641, 200_000]
         for t in [0, 1, 2, 15, 16, 18, 33, 37, 60, 66, 74, 75, 100, 132, 148, 149, 1000, 10 ** 6]]


@pytest.mark.parametrize("r640,r512", [(B200, B200), ([100, 40, 20, 9], B200), ([0, 0, 0, 0], B200), (B200, [100, 40, 20, 9]),
                                       ([1, 1, 1, 1], [1, 1, 1, 1])])
def test_the_ring_that_is_launched_holds_its_rows(plan, r640, r512):
    """A ring of one slice gets one row to a cluster: there are no more rows than such clusters run at a
    time, of the form that is launched.  Every other ring holds two slices."""
    at = {1: 0, 2: 1, 4: 2, 8: 3}
    for (units, rows), (form, cluster, one_turn, stages, stage) in zip(CASES, plan(CASES, r640, r512)):
        slice_ = -(-units // cluster)
        if form in (ROWS, LONG):
            assert (units <= 256) == (form == ROWS) and not one_turn
            continue
        assert units > 256
        if one_turn:
            assert form in (RING512, RING640)
            assert rows <= (r640 if form == RING640 else r512)[at[cluster]], (units, rows, form, cluster)
            assert -(-slice_ // stage) <= stages
        else:
            assert 2 * -(-slice_ // stage) <= stages
            assert cluster == 1 or form in (RING512, RING640)


def test_forms_of_calls_that_occur(plan):
    got = plan([(32_768, 33), (6282, 8192), (4000, 6250), (4000, 8192), (512, 48_828), (1519, 16_451), (16_032, 1559), (75, 333_333)])
    assert [g[:3] for g in got] == [(RING512, 4, 1), (RING640, 1, 0), (RING512, 1, 0), (RING512, 1, 0), (RING64, 1, 0), (RING128, 1, 0),
                                    (RING512, 4, 0), (ROWS, 1, 0)]


def test_an_error_of_the_residency_question_is_returned(plan):
    assert plan([(32_768, 10)], [-1] * 4, [-1] * 4) == ["error 7"]
    assert plan([(256, 10)], [-1] * 4, [-1] * 4)[0][0] == ROWS      # not asked
