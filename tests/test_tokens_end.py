"""The waits and the end of a call of the layer for a few tokens (``csrc/ciera_tokens_end.hpp``, which the kernel runs) on the CPU: no warp waits for a counter
that has been set back, and all counters are zero behind the call, in whatever order its blocks get there."""
import os
import subprocess

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "..", "paper_2609_04609_b200", "csrc")
ORDERS = 40000


@pytest.fixture(scope="module")
def play(tmp_path_factory):
    exe = str(tmp_path_factory.mktemp("tokens_end") / "tokens_end")
    subprocess.run(["g++", "-std=c++17", "-O2", "-Wall", "-Werror", "-Wno-cast-function-type", "-I", CSRC, os.path.join(HERE, "tokens_end.cpp"), "-o", exe],
                   check=True)

    def run(*what):
        out = subprocess.run([exe, *map(str, what)], check=True, capture_output=True, text=True).stdout
        return [int(w) if w.isdigit() else w for w in out.split()]

    return run


@pytest.mark.parametrize("blocks", [1, 2, 3, 5])
def test_nobody_waits_for_good_and_all_is_zero(play, blocks):
    assert play(blocks, 0, ORDERS) == [ORDERS, 0, 0]


def test_the_model_sees_a_warp_that_waits_without_a_part(play):
    assert play(3, 1, ORDERS)[1] > 0


def test_the_model_sees_additions_that_come_late(play):
    assert play(3, 2, ORDERS)[2] > 0


@pytest.mark.parametrize("most,there,given_up,want", [
    (5, 1, 0, [1, 1, 0]), (5, 5, 0, [1, 5, 0]),
    (5, 6, 0, [0, 5, 1]),  # runs out, and says so
    (5, 0, 3, [0, 3, 0]), (5, 3, 3, [1, 3, 0]), (0, 1, 0, [0, 0, 1]),
])
def test_a_wait_that_runs_out_is_told(play, most, there, given_up, want):
    assert play("wait", most, there, given_up) == want


def test_a_block_that_gives_up_spoils_the_counters_and_writes_nothing(play):
    assert play("give_up") == ["join", "spoil"]


def test_the_kernel_goes_by_this():
    with open(os.path.join(CSRC, "ciera_tokens.cu")) as f:
        source = f.read()
    assert "end_call(end)" in source and "tell(next, [&]" in source and "takes_part(it, w.stages, warp & 3, kColumnWarps)" in source
    # both waits for other threads' words, those for all blocks and those for written tiles
    assert "poll(kMaxPolls, " in source and "poll(kMaxReportPolls, " in source
    lo = source.index("struct TokensEnd")
    rest = source[:lo] + source[source.index("\n};", lo) :]
    assert "a.counters[" not in rest  # nobody else sets one back
