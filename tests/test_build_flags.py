"""What the kernels' build may assume of their numbers."""
import os

from paper_2607_27600_amd import build

# Every input of this kernel is finite by its contract; the other entry points say what a NaN does.
FINITE = {"attention.hip"}


def test_nan_is_a_number_to_the_compiler():
    for src in build.SOURCES:
        flags = build.FLAGS + build.FILE_FLAGS.get(src, [])
        loose = [f for f in flags if "fast" in f or "no-honor" in f or "finite-math" in f]
        assert src in FINITE or not loose, (src, loose)


def test_no_packed_fp32():
    at = build.FLAGS.index("-packed-fp32-ops")
    assert build.FLAGS[at - 3:at] == ["-Xclang", "-target-feature", "-Xclang"]


def test_every_kernel_file_is_built():
    assert sorted(build.SOURCES) == sorted(f for f in os.listdir(build.CSRC) if f.endswith(".hip"))
