"""What the compiler recorded of the training operators' kernels (no GPU needed)."""
import re

import paper_2510_21048_amd as xm
from test_abi_host import kernel_resources


def resources(monkeypatch):
    monkeypatch.setattr(xm, "lib_path", xm.ops_lib_path)
    return kernel_resources()


def test_a_row_of_one_wavefront_uses_no_lds(monkeypatch):
    """Four such rows share a workgroup without a barrier between them: what their lanes pass to each other goes by register
    exchanges, since LDS written by one lane and read by others would need a fence."""
    small = {k: r for k, r in resources(monkeypatch).items() if re.search(r"k_policyI\w+Li64ELi\d+E", k)}
    assert len(small) == 3, sorted(small)
    for name, r in small.items():
        assert int(r["group_segment_fixed_size"]) == 0, (name, r["group_segment_fixed_size"])
