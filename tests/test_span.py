"""CPU checks of attention over parts of the requests' keys: the host's plans walked as the
kernels walk them; every malformed argument is refused on the host with the documented
status, before any device work; workspace sizes and their bounds; what the calls launch."""
import os
import subprocess

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)


def test_plans(tmp_path):
    """Every row meets each key that it sees exactly once, in random batches."""
    exe = str(tmp_path / "span_plan_check")
    subprocess.run(["g++", "-O2", "-std=c++17", "-Wall", "-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include",
                    "-I", os.path.join(ROOT, "include"),
                    "-I", os.path.join(ROOT, "paper_2606_16264_amd", "csrc"),
                    os.path.join(HERE, "span_plan_check.cpp"), "-o", exe], check=True)
    got = subprocess.run([exe, "60"], capture_output=True, text=True, timeout=240)
    assert got.returncode == 0, got.stdout
