"""What the compiler recorded of the kernels of include/ops/xmem_step.h (no GPU needed)."""
import re

from test_ops_kernels import resources


def test_registers_of_the_steps_kernels(monkeypatch):
    """None uses accumulation registers (a wavefront's vector registers hold all of it), and none keeps anything in scratch memory but
    the gradients of rows whose threads have no scalar addresses (below a wavefront) or 1024 threads' registers at most."""
    mine = {k: r for k, r in resources(monkeypatch).items()
            if re.search(r"k_norm|k_norm_back|k_lookup|k_scan|k_group|k_sum|k_join|k_squares|k_scale|k_stats", k) and "policy" not in k}
    assert len(mine) > 60, sorted(mine)
    for name, r in mine.items():
        assert int(r["agpr_count"]) == 0, name
        if not re.search(r"k_norm_backI\w+Li(8|16|32|1024)ELi[124]E", name):
            assert int(r["private_segment_fixed_size"]) == 0, (name, r["private_segment_fixed_size"])
