"""The loads through registers that the matrix product makes of operands of any alignment, on the CPU: none is outside of its
operand (tests/ops_staged_loads.hip)."""
import subprocess
from pathlib import Path

from paper_2510_21048_amd.build import HIPCC, ROOT


def test_staged_loads_stay_in_their_operand(tmp_path):
    exe = tmp_path / "loads"
    subprocess.run([HIPCC, "--cuda-host-only", "-O2", "-std=c++17", f"-I{ROOT / 'include'}",
                    str(Path(__file__).with_name("ops_staged_loads.hip")), "-o", str(exe)], check=True, capture_output=True)
    r = subprocess.run([str(exe)], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and "operands ok" in r.stdout, (r.returncode, r.stdout[-500:], r.stderr[-500:])
