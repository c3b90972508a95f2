"""Calls whose allocations and HIP calls fail one after the other (host only): the layout stays as it was, and the
device page table and the planner agree."""
import hostbuild


def test_every_failure_leaves_the_layout_as_it_was(tmp_path):
    out = hostbuild.run("failed_calls", tmp_path)
    assert "FAILED" not in out and out.endswith("ok\n")
