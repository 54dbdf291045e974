"""Host rules of the kernel sources, run as they stand there: a part of a .hip
file that holds no device code is compiled by itself with g++ behind stubs of
what it calls, so that a test can ask which kernel a size goes to."""
import os
import subprocess
import tempfile

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2606_01143_amd", "csrc")


def part(source, begin, end):
    """The text of `source` from `begin` up to `end`; both stand there once."""
    text = open(os.path.join(CSRC, source)).read()
    assert text.count(begin) == 1 and text.count(end) == 1, (source, begin, end)
    return text[text.index(begin):text.index(end)]


def answers(code, lines):
    """What the program prints for lines of its standard input, as lists of integers."""
    with tempfile.TemporaryDirectory() as d:
        src, exe = os.path.join(d, "rule.cpp"), os.path.join(d, "rule")
        with open(src, "w") as f:
            f.write("#include <algorithm>\n#include <cstdint>\n#include <cstdio>\n" + code)
        subprocess.run(["g++", "-std=c++17", "-O1", src, "-o", exe], check=True)
        text = "\n".join(" ".join(str(int(v)) for v in line) for line in lines) + "\n"
        out = subprocess.run([exe], input=text, capture_output=True, text=True, check=True).stdout
    return [[int(v) for v in line.split()] for line in out.splitlines()]
