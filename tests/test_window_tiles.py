"""Which queries each CTA of the window attention's backward takes, checked on the host."""
import os
import subprocess

from paper_2505_00315_gb300 import build

HERE = os.path.dirname(os.path.abspath(__file__))


def test_every_visible_pair_once_and_the_sink_rows_spread_out(tmp_path):
    exe = str(tmp_path / "check")
    r = subprocess.run([build.nvcc(), *build.ARCH, "-O1", "-std=c++17", "--expt-relaxed-constexpr", "-I", build.CSRC,
                        os.path.join(HERE, "c", "window_tiles_check.cu"), "-o", exe],
                       capture_output=True, text=True)
    assert r.returncode == 0, r.stdout + r.stderr
    r = subprocess.run([exe], capture_output=True, text=True)
    assert r.returncode == 0 and r.stdout.strip() == "ok", r.stdout + r.stderr
