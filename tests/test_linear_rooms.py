"""Host test of the 8-bit products' use of LDS for outputs (built from the
library's own header with hipcc as host code; no GPU needed)."""

import os
import shutil
import subprocess

import pytest

from paper_2512_07009_amd import build as libbuild

HERE = os.path.dirname(os.path.abspath(__file__))


@pytest.mark.skipif(shutil.which("hipcc") is None and not os.path.exists("/opt/rocm/bin/hipcc"),
                    reason="needs hipcc")
def test_outputs_go_where_nothing_is_read(tmp_path):
    exe = str(tmp_path / "linear_rooms_test")
    r = subprocess.run([libbuild.hipcc(), "-std=c++17", "-O1", "-I", libbuild.CSRC,
                        os.path.join(HERE, "cpp", "linear_rooms_test.cpp"), "-o", exe],
                       capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-2000:]
    r = subprocess.run([exe], capture_output=True, text=True, timeout=120)
    assert r.returncode == 0, r.stdout + r.stderr
    assert "rooms ok" in r.stdout


@pytest.mark.parametrize("kernel", ["linear_kernel", "linear_any_kernel"])
def test_kernels_take_their_rooms_from_there(kernel):
    with open(os.path.join(libbuild.CSRC, "linear.hip")) as f:
        body = f.read().split(f"{kernel}(LinearArgs a) {{")[1].split("\n}\n")[0]
    rooms = [line for line in body.splitlines() if "int8_t *room" in line]
    assert len(rooms) == 1 and "stage_room<" in rooms[0], rooms
