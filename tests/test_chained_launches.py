"""A kernel that is launched ahead of the one before it (griddepcontrol) is already running while that one writes its
operands.  The read-only path (ld.global.nc: __ldg, and Raw::load<false>, which uses it) asks for data that does not change
while the kernel runs, so such a kernel must not read through it."""
import glob
import os
import re

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def _functions(text):
    """Bodies of the functions at the outermost level (namespaces aside), by their braces."""
    text = re.sub(r"//[^\n]*", "", text)
    for m in re.finditer(r"__global__", text):
        at, depth = text.index("{", m.end()), 0
        for i in range(at, len(text)):
            depth += {"{": 1, "}": -1}.get(text[i], 0)
            if depth == 0:
                yield text[m.start():i]
                break


def test_no_read_only_loads_after_an_early_launch():
    found = 0
    for path in glob.glob(os.path.join(ROOT, "paper_2511_09261_b200", "csrc", "*.cu*")):
        for body in _functions(open(path).read()):
            if "griddepcontrol.wait" not in body:
                continue
            found += 1
            assert not re.search(r"__ldg\(|\.nc\.|load<false>", body), path
    assert found > 0
