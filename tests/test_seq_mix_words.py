"""What linear attention reads of rows that are no whole pieces, by its own address arithmetic on the host: words of the row alone, and all of it."""
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
SAN = ["-fsanitize=address,undefined", "-fno-sanitize-recover=all", "-g", "-O1"]


@pytest.fixture(scope="module")
def driver(tmp_path_factory):
    out = str(tmp_path_factory.mktemp("words") / "piece_words")
    subprocess.check_call(["g++", "-std=c++17", *SAN, "-I", os.path.join(ROOT, "paper_1804_04806_amd", "csrc"),
                           os.path.join(ROOT, "tests", "native", "piece_words_driver.cpp"), "-o", out])
    return out


def faults(driver, cases):
    r = subprocess.run([driver], input="\n".join(" ".join(map(str, c)) for c in cases) + "\n", capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and r.stderr == "", r.stderr[-2000:]
    return [(c, int(n)) for c, n in zip(cases, r.stdout.split()) if int(n)]


@pytest.mark.parametrize("size", [2, 4])
@pytest.mark.parametrize("reversed_", [0, 1])
def test_words_of_every_width(driver, size, reversed_):
    """Both parities of a row's begin: of the tensor's address, of its head, and of its token."""
    cases = [(1, 3, heads, width, gap, size, address, 64 if width <= 64 else 128, reversed_) for width in range(1, 129) for heads in (1, 2, 3)
             for gap in (0, 1) for address in range(0, 4, size)]
    assert not faults(driver, cases)


@pytest.mark.parametrize("reversed_", [0, 1])
def test_words_at_a_tensors_end(driver, reversed_):
    """Sequences of whole and of ragged chunks, the last head's rows at the tensor's very end; tiles wider than the row's class."""
    cases = [(*shape, 0, 2, address, cols, reversed_) for shape in ((1, 64, 2, 65), (2, 64, 16, 33), (2, 65, 6, 41), (1, 130, 3, 1), (1, 1, 1, 127))
             for address in (0, 2) for cols in (64, 128) if shape[3] <= cols]
    assert not faults(driver, cases)
