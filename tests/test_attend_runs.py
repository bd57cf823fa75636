"""The attention's cutting of its steps into runs, which kernel and join must agree on, for as many runs as any kernel has."""
import os
import subprocess

from paper_2405_18400_b200 import build

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_runs_are_cut_as_in_64_bits(tmp_path):
    exe = str(tmp_path / "attend_runs")
    subprocess.check_call([build._nvcc(), "-gencode", "arch=compute_100a,code=sm_100a", "-std=c++17", "-O1", "-I", build.INCLUDE, "-I", build.CSRC, "-o", exe,
                           os.path.join(ROOT, "tests", "attend_runs.cu")])
    r = subprocess.run([exe], stdout=subprocess.PIPE, text=True)
    assert r.returncode == 0, r.stdout
