"""Names that the library keeps to itself (runs without a GPU)."""
import subprocess

import paper_2605_11186_amd as cats


def test_hip_fail_is_not_exported():
    """It belongs to cats_strerror: another library's function of that name must not be called in its place, nor this one in another's."""
    names = subprocess.run(["nm", "-D", "--defined-only", str(cats.library_path())], check=True, capture_output=True, text=True).stdout
    assert "cats_strerror" in names and "hip_fail" not in names
