"""The feed-forward kernel's thread blocks meet their pair twice, in front of the roles and behind them, on a barrier without a limit: so no
thread may have left before, whatever became of its bounded waits."""
import os
import re

SRC = open(os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2604_10103_b200", "csrc", "k_ff_gemm.cuh")).read()


def test_both_meetings_are_reached_by_every_thread():
    body = SRC[SRC.index("k_ff_gemm(const __grid_constant__ FfGemmParams p) {"):]
    meets = [m.start() for m in re.finditer(r"\bff_meet<CG>\(\);", body)]
    roles = body.index("if (warp == C::WARP_TMA)")
    assert len(meets) == 2 and meets[0] < roles < meets[1]
    before = re.sub(r"auto \w+ = \[&\].*?\n        \};", "", body[:meets[1]], flags=re.S)        # (a lambda's return leaves the lambda)
    assert not re.search(r"\breturn\b|\bexit\b", before)
    # both stand at the kernel's own level, not inside a role
    for at in meets:
        line = body[body.rindex("\n", 0, at) + 1:at]
        assert line == "    "


def test_the_meeting_is_the_only_wait_without_a_limit():
    body = SRC[SRC.index("k_ff_gemm(const __grid_constant__ FfGemmParams p) {"):]
    assert not re.search(r"mbar_try_wait|__syncthreads|bar\.sync|while \(true\)|for \(;;\)", body)
    assert len(re.findall(r"mbar_wait", body)) == len(re.findall(r"abort_flag, p\.dev_status, \d+\)", body))
