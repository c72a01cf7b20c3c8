"""Layer norm's kernels wait for each row that a bulk copy brings.  When a wait has run out the thread waits no more and asks for no more copies (or every
row behind it would take the limit again), and the copies in flight get time before the thread block leaves."""
import os
import re

SRC = open(os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2604_10103_b200", "csrc", "k_norm.cuh")).read()


def body(name):
    i = SRC.index("\n" + name + "(const NormParams p) {")
    return SRC[i:SRC.index("\n}\n", i)]


def function(name):
    i = SRC.index(name + "(")
    return SRC[i:SRC.index("\n}\n", i)]


def test_a_wait_that_ran_out_is_the_last():
    wait = function("void norm_wait_slow")
    assert wait.index("if (*lost) return;") < wait.index("clock64() - t0 < tc5::WAIT_LIMIT_CYCLES") and wait.count("while") == 1
    assert wait.index("while") < wait.index("*lost = 1;") and "HF_DEV_TIMEOUT_FLAG" in wait
    for name in ("k_norm_rows", "k_norm_bwd"):
        b = body(name)
        # one wait, and a word of the team's behind its barriers that says whether it ran out, clear from the start
        assert len(re.findall(r"on\) norm_wait<WIDE>\([^;]*, lost, ", b)) == 1 == b.count("norm_wait") and "mbar_try_wait" not in b and "while" not in b
        assert "lost = reinterpret_cast<volatile int*>(s_team + 60);" in b
        assert b.index("*lost = 0;") < b.index("mbar_init") < b.index("__syncthreads();") < b.index("norm_wait")
        # copies asked for in front of the wait, and behind it only where none ran out
        asks = [m.start() for m in re.finditer(r"\bload\((?!long)", b)]
        assert len(asks) == 2 and asks[0] < b.index("norm_wait") < asks[1]
        assert "!*lost" in b[b.rindex("if (", 0, asks[1]):asks[1]]
        # the thread block's barriers are reached by all its threads: the loop is that of the thread block
        assert re.search(r"for \(long long r0 = first; r0 < g1; r0 \+= step", b) and "break" not in b
        # time for the copies in flight, behind the last row and in front of any other use of their memory
        drain = b.index("norm_drain(lost);")
        assert asks[1] < drain and "s_join" not in b[:drain] and "return" not in b[b.index("norm_wait"):drain]
    assert re.search(r"clock64\(\) - t0 < \d+\)", function("void norm_drain"))
