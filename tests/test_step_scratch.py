"""How much scratch memory the step's kernels keep, as the compiler recorded it (no GPU needed): none may grow unseen."""
import re

from test_ops_kernels import resources

# Bytes a thread of k_norm_back, by element type (mangled), threads of a row, pieces a thread and whether there are biases.  128 registers
# are all that 16 wavefronts a CU have: with 16 or more elements of a row in a thread, with 1024 threads and biases, or where rows share a
# wavefront and have no scalar addresses, some of what it holds does not fit.  The others keep nothing.
BF, HF, FF = "DF16b", "DF16_", "f"
KEPT = {(BF, 8, 1, 0): 20, (BF, 8, 1, 1): 52, (BF, 16, 1, 0): 12, (BF, 16, 1, 1): 44, (BF, 32, 1, 0): 24, (BF, 32, 1, 1): 56,
        (HF, 8, 1, 0): 12, (HF, 8, 1, 1): 28, (HF, 16, 1, 1): 24, (HF, 32, 1, 0): 12, (HF, 32, 1, 1): 40,
        (BF, 1024, 1, 1): 40, (HF, 1024, 1, 1): 48,
        (BF, 1024, 2, 0): 124, (BF, 1024, 2, 1): 240, (HF, 1024, 2, 0): 124, (HF, 1024, 2, 1): 240,
        (FF, 1024, 4, 0): 160, (FF, 1024, 4, 1): 352}


def forms(found):
    """{(type, threads, pieces, biases): bytes} of k_norm_back."""
    got = {}
    for name, r in found.items():
        m = re.search(r"k_norm_backI(DF16b|DF16_|f)Li(\d+)ELi(\d)ELb([01])E", name)
        if m:
            got[m[1], int(m[2]), int(m[3]), int(m[4])] = int(r["private_segment_fixed_size"])
    return got


def past(got, kept):
    return {k: v for k, v in got.items() if v > kept.get(k, 0)}


def test_scratch_of_the_norms_gradients(monkeypatch):
    got = forms(resources(monkeypatch))
    assert len(got) == 56 and set(KEPT) <= set(got), sorted(got)
    assert past(got, KEPT) == {}
    # what the limits are for: a form that keeps a register more, and one that kept none
    worse = {**got, (BF, 1024, 2, 1): KEPT[BF, 1024, 2, 1] + 4, (FF, 256, 1, 0): 4}
    assert set(past(worse, KEPT)) == {(BF, 1024, 2, 1), (FF, 256, 1, 0)}


def test_no_other_kernel_of_the_step_keeps_any(monkeypatch):
    mine = {k: int(r["private_segment_fixed_size"]) for k, r in resources(monkeypatch).items()
            if re.search(r"k_norm|k_lookup|k_scan|k_group|k_sum|k_join|k_squares|k_scale|k_stats", k) and "policy" not in k
            and not re.search(r"k_norm_backI", k)}
    assert len(mine) > 40 and not any(mine.values()), {k: v for k, v in mine.items() if v}
