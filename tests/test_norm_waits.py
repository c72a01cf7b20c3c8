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
    wait = function("bool norm_wait_slow")
    assert wait.index("if (lost) return true;") < wait.index("clock64() - t0 < tc5::WAIT_LIMIT_CYCLES") and wait.count("while") == 1
    assert "HF_DEV_TIMEOUT_FLAG" in wait and wait.rstrip().endswith("return true;")
    for name in ("k_norm_rows", "k_norm_bwd"):
        b = body(name)
        # one wait
        assert len(re.findall(r"on && !tc5::mbar_try_wait\([^;]*\)\) lost = norm_wait_slow\([^;]*, lost, ", b)) == 1
        assert b.count("norm_wait_slow(") == 1 == b.count("mbar_try_wait") and "while" not in b
        # copies asked for in front of it, and behind it only where none ran out
        asks = [m.start() for m in re.finditer(r"\bload\((?!long)", b)]
        assert len(asks) == 2 and asks[0] < b.index("norm_wait_slow(") < asks[1]
        assert "!lost" in b[b.rindex("if (", 0, asks[1]):asks[1]]
        # the thread block's barriers are reached by all its threads: the loop is that of the thread block
        assert re.search(r"for \(long long r0 = first; r0 < g1; r0 \+= step", b) and "break" not in b
        # time for the copies in flight, behind the last row and in front of any other use of their memory
        drain = b.index("norm_drain(lost);")
        assert asks[1] < drain and "s_join" not in b[:drain] and "return" not in b[b.index("norm_wait_slow("):drain]
    assert re.search(r"clock64\(\) - t0 < \d+\)", function("void norm_drain"))
