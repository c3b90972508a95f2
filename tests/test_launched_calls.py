"""What calls launch, without a GPU: the library's host sources with stand-ins for HIP and the kernels."""
import hostbuild


def test_calls_launch_what_they_should(tmp_path):
    out = hostbuild.run("launched_calls", tmp_path)
    assert "FAILED" not in out and out.endswith("ok\n")
