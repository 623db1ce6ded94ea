"""A kernel that launch_k or launch_pdl starts may run while the one before it still does, wherever its
entry point chains launches: it waits for that one (grid_dep_sync) before it touches global memory."""
import glob
import os
import re

import paper_1512_06473_gb300.build as build

KERNEL = re.compile(r"__global__[^;{]*?\{")
LAUNCH = re.compile(r"\blaunch_(?:pdl|k)\s*\(")


def _text(path):
    return re.sub(r"/\*.*?\*/|//[^\n]*", "", open(path).read(), flags=re.S)


def _kernels(text):
    """(name, body) of every kernel."""
    for m in KERNEL.finditer(text):
        depth, i = 1, m.end()
        while depth:
            depth += {"{": 1, "}": -1}.get(text[i], 0)
            i += 1
        head = re.sub(r"__launch_bounds__\((?:[^()]|\([^()]*\))*\)", "", m.group())
        yield re.search(r"(\w+)\s*\(", head).group(1), text[m.end():i]


def test_kernels_wait_for_the_launch_before():
    seen, missing = 0, []
    for path in sorted(glob.glob(os.path.join(build.CSRC, "*.cu"))):
        text = _text(path)
        if not LAUNCH.search(text):
            continue
        for name, body in _kernels(text):
            if re.search(name + r"\s*(<[^;<]*>)?\s*<<<", text):  # (a plain launch)
                continue
            seen += 1
            if "grid_dep_sync()" not in body:
                missing.append((os.path.basename(path), name))
    assert seen >= 20 and not missing, missing
