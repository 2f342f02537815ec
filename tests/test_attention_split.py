"""How the attention cuts a call into pieces, on the host: the kernels' and the launcher's own functions over random calls (no GPU needed)."""
import os
import shutil
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_pieces_and_positions_stay_within_what_is_launched(tmp_path):
    program = str(tmp_path / "split")
    subprocess.run([shutil.which("hipcc") or "/opt/rocm/bin/hipcc", "-x", "hip", "--offload-host-only", "-O1", "-std=c++17", "-I",
                    os.path.join(ROOT, "paper_2604_07853_amd", "csrc"), os.path.join(ROOT, "tests", "attention_split_check.cpp"), "-o", program], check=True, timeout=300)
    got = subprocess.run([program, "200000"], capture_output=True, text=True, timeout=300)
    assert got.returncode == 0 and "0 broken" in got.stdout, got.stdout
