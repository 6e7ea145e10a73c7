"""The times of a layer's parts from `bench.py --layer-parts` in the schedule calculator (no GPU)."""
import json
import pathlib
import subprocess
import sys

import pytest

from paper_2507_00394_amd import schedule_model as M

ROOT = pathlib.Path(__file__).resolve().parents[1]


def test_measured_times_take_the_place_of_assumed_ones(capsys):
    M.main(["--t-attn-ms", "10"])
    assumed = json.loads(capsys.readouterr().out)
    M.main(["--t-attn-ms", "10", "--t-pre-ms", "0.5", "--t-post-ms", "7"])
    got = json.loads(capsys.readouterr().out)
    assert assumed["t_pre_ms"] == 0 and got["t_pre_ms"] == 0.5 and got["t_post_ms"] == 7
    assert got["t_qkv_linear_ms"] == assumed["t_qkv_linear_ms"]
    assert got["schedules"]["helix"]["bubble_ms"] == pytest.approx(8 * 7 * 7.5)                      # Table 2: 8 (p - 1) (t_pre + t_post)
    assert got["schedules"]["1f1b"]["bubble_ms"] == pytest.approx(3 * 7 * (7.5 + 10 + got["t_qkv_linear_ms"]) * 4)


def test_shapes_that_do_not_divide_are_refused():
    code = "import sys, bench; sys.argv = ['bench.py', '--layer-parts', '--seq', '1000']; bench.layer_parts_bench(bench.parse())"
    r = subprocess.run([sys.executable, "-c", code], capture_output=True, text=True, cwd=ROOT)
    assert r.returncode == 2 and "multiple" in r.stderr and r.stdout.strip() == ""
