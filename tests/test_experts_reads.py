"""What the products by groups of rows read of operands stored across k, by a model on the host (CPU only): rows shorter than the
16 bytes of a request end in other rows, and past the last one lies nothing."""
import os
import subprocess

from paper_2305_08872_amd import build as hip_build

HERE = os.path.dirname(os.path.abspath(__file__))


def test_requests_stay_inside_the_operand(tmp_path):
    exe = str(tmp_path / "reads")
    res = subprocess.run([hip_build._hipcc()] + hip_build.HIPCC_FLAGS + ["-x", "hip", os.path.join(HERE, "sanitize", "experts_reads_main.cpp"), "-o", exe],
                         stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True, timeout=300)
    assert res.returncode == 0, res.stdout[-4000:]
    res = subprocess.run([exe], stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True, timeout=300)
    print(res.stdout)
    assert res.returncode == 0, res.stdout[-4000:]
