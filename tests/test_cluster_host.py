"""A CTA may touch another's shared memory once that has begun to run, which a cluster is scheduled
together for but does not promise: a barrier of the cluster comes first, in every function that
does."""
import glob
import os
import re

import paper_1512_06473_gb300.build as build

REMOTE = re.compile(r"\bmap_shared_rank\s*\(")
BARRIER = re.compile(r"\bcluster\s*\.\s*(sync|barrier_wait)\s*\(")


def _functions(text):
    """Bodies of functions at namespace level, without comments."""
    text = re.sub(r"/\*.*?\*/|//[^\n]*", "", text, flags=re.S)
    for m in re.finditer(r"^(?:template[^\n]*\n)?__(?:global|device)__[^;{]*\{", text, flags=re.M):
        depth, i = 1, m.end()
        while depth and i < len(text):
            depth += {"{": 1, "}": -1}.get(text[i], 0)
            i += 1
        yield text[m.start():m.end()], text[m.end():i]


def test_a_barrier_before_the_first_access():
    seen, early = 0, []
    for path in sorted(glob.glob(os.path.join(build.CSRC, "*.cu*"))):
        for head, body in _functions(open(path).read()):
            remote = REMOTE.search(body)
            if not remote:
                continue
            seen += 1
            barrier = BARRIER.search(body)
            if not barrier or barrier.start() > remote.start():
                early.append((os.path.basename(path), " ".join(head.split())[:80]))
    assert seen >= 2 and not early, early
