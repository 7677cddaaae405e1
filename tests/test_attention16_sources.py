"""The kernels of the 16-bit caches wait for the grids before theirs, once, on every path, before they touch memory
(they may start while the launch before them still runs)."""
import os
import re

import paper_2609_35800_gb300 as hg

CSRC = os.path.join(os.path.dirname(os.path.abspath(hg.__file__)), "csrc_attention")


def _kernels():
    for name in sorted(os.listdir(CSRC)):
        text = re.sub(r"//[^\n]*", "", open(os.path.join(CSRC, name)).read())
        for m in re.finditer(r"__global__ void(?: __launch_bounds__\([^{;]*?\))?\s+(\w+)\(", text):
            start = text.index("{", m.end())
            depth, i = 1, start + 1
            while depth:
                depth += {"{": 1, "}": -1}.get(text[i], 0)
                i += 1
            yield m.group(1), text[start + 1:i - 1]


def test_every_kernel_waits_before_it_touches_memory():
    seen = set()
    for name, body in _kernels():
        assert body.count("grid_dependency_wait()") == 1, name
        at = re.search(r"^  grid_dependency_wait\(\);", body, re.M)  # under no condition
        assert at, name
        before = body[:at.start()]
        assert not re.search(r"ldg|bulk|tma_load|\.data\b|\.table\[|\.lengths\[|\.slots\[|atomic", before), name
        # only CTAs or threads without any work of their own leave before it
        assert all("p.tokens" in line for line in re.findall(r"if \([^\n]*return;", before)), name
        seen.add(name)
    assert len(seen) >= 3
    every = "".join(open(os.path.join(CSRC, f)).read() for f in os.listdir(CSRC))
    assert every.count("__global__") == len(list(_kernels()))
