"""The index expressions by which the selective scan reads flags, on the host (no GPU): inside the block for blocks of one slot too."""
import os
import subprocess

from paper_2310_10879_amd import build

HERE = os.path.dirname(os.path.abspath(__file__))


def test_flags_are_read_inside_their_block(tmp_path):
    exe = str(tmp_path / "scan_bounds")
    # (the host's part alone; optimisation has no part in it)
    flags = [f for f in build.FLAGS if f not in ("-O3", "--offload-arch=gfx950")]
    made = subprocess.run([build.HIPCC, "--offload-host-only", "-O0", *flags, "-o", exe, "-x", "hip", os.path.join(HERE, "scan_bounds_main.cpp")],
                          capture_output=True, text=True)
    assert made.returncode == 0, made.stderr
    run = subprocess.run([exe], capture_output=True, text=True, timeout=60)
    assert run.returncode == 0 and "scan bounds ok" in run.stdout, run.stdout + run.stderr
