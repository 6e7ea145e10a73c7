"""The waits of the gated projections' kernels, read from the assembly of this library's own source (no GPU).

The recomputing backward requests its part of dh while the last stages of its product run.  A wave's wait for its copies of a stage counts the memory operations that may stay in
flight; were those loads among them, the wait would be right only for as many load instructions as the compiler happens to make.  So: every copy has landed before the first of the
loads, and no barrier behind them waits for memory."""
import re
import subprocess

import pytest

from paper_2507_00394_amd import build


def _events(body):
    """The kernel's copies into LDS, loads, waits for memory (how many operations may stay in flight) and barriers, in order."""
    out = []
    for line in body.splitlines():
        line = line.strip()
        if line.startswith("global_load_lds"):
            out.append("copy")
        elif line.startswith("global_load"):
            out.append("load")
        elif line.startswith("s_barrier"):
            out.append("barrier")
        elif wait := re.match(r"s_waitcnt.*vmcnt\((\d+)\)", line):
            out.append(int(wait.group(1)))
    return out


@pytest.fixture(scope="module")
def kernels(tmp_path_factory):
    """{name: events} of the kernels with the gradient's epilogue."""
    out = tmp_path_factory.mktemp("asm") / "gated.s"
    flags = [f for f in build.FLAGS if f not in ("-shared", "-fPIC")]
    subprocess.run(["hipcc", *flags, "-w", "-S", "--cuda-device-only", str(build.CSRC / "gated.hip"), "-o", str(out)], check=True)
    found = re.findall(r"^(_ZN\S*gated_kernel\S*ELb1E\S*):.*?\n(.*?)s_endpgm", out.read_text(), re.M | re.S)
    return {name: _events(body) for name, body in found}


def test_every_tile_and_activation_is_there(kernels):
    assert len(kernels) == 6


def test_copies_land_before_the_gradient_is_requested(kernels):
    for name, events in kernels.items():
        first = events.index("load")
        assert "copy" not in events[first:], name
        assert events[first - 2:first] == [0, "barrier"], name


def test_no_barrier_behind_the_request_waits_for_memory(kernels):
    for name, events in kernels.items():
        behind = events[events.index("load"):]
        last = len(behind) - 1 - behind[::-1].index("barrier")
        assert not [e for e in behind[:last] if isinstance(e, int)], name
