"""The bounded wait of a whole warp, on the host: whatever the lanes see, all of them leave together and with the
same answer (after it they vote and load together, so a lane on its own would be waited for without a limit)."""
import os
import subprocess

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(os.path.dirname(HERE), "paper_2609_37029_gb300", "csrc")


@pytest.fixture(scope="module")
def cases(tmp_path_factory):
    exe = str(tmp_path_factory.mktemp("host") / "warp_wait")
    subprocess.run(["g++", "-std=c++20", "-O1", "-pthread", "-I", CSRC, "-o", exe,
                    os.path.join(HERE, "host_warp_wait.cc")], check=True)
    out = subprocess.run([exe], check=True, capture_output=True, text=True, timeout=60).stdout
    return {name: (verdict, gave) for name, verdict, gave in (line.split("|") for line in out.splitlines())}


NOBODY, EVERYBODY, LATE = "." * 32, "g" * 32, "L" * 32
WANT = {
    "complete": ("+", NOBODY),
    "complete later": ("+", NOBODY),
    "complete after the limit's first look": ("+", NOBODY),
    "never": ("-", LATE),
    "another role gave up": ("-", EVERYBODY),
    "one lane late": ("-", "g" * 5 + "L" + "g" * 26),
    "one lane sees the flag": ("-", EVERYBODY),
    "a phase that moves on": ("+", NOBODY),
    "all but one lane complete": ("-", LATE),
}


@pytest.mark.parametrize("name", list(WANT))
def test_lanes_leave_together(cases, name):
    verdict, gave = cases[name]
    assert verdict == WANT[name][0] * 32
    assert gave == WANT[name][1]


def test_every_case_ran(cases):
    assert set(cases) == set(WANT)
