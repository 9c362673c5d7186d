"""The matrix product's slices and their workspace, on the host: linear_slices.hip says what is checked."""
import os
import subprocess

HERE = os.path.dirname(os.path.abspath(__file__))


def test_slices_stay_in_the_workspace(tmp_path):
    exe = str(tmp_path / "linear_slices")
    subprocess.run(["hipcc", "--offload-arch=gfx950", "-O2", "-std=c++17", os.path.join(HERE, "linear_slices.hip"), "-o", exe], check=True, capture_output=True)
    r = subprocess.run([exe], capture_output=True, text=True, timeout=120)
    assert r.returncode == 0 and r.stdout == "6912 calls, 4608 sliced\n", r.stdout
