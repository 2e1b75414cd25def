"""The objects are rebuilt when anything that they include has changed."""
import os
import re

from paper_2412_14468_b200 import build as ha_build


def included(path, seen):
    with open(path) as f:
        for name in re.findall(r'^\s*#include\s+"([^"]+)"', f.read(), re.M):
            for where in (os.path.dirname(path), ha_build.CSRC, os.path.join(ha_build.ROOT, "include")):
                p = os.path.normpath(os.path.join(where, name))
                if os.path.exists(p):
                    if p not in seen:
                        seen.add(p)
                        included(p, seen)
                    break
    return seen


def test_every_included_header_is_a_dependency():
    deps = {os.path.normpath(p) for p in ha_build._headers()}
    for src in ha_build.sources():
        missing = included(src, set()) - deps
        assert not missing, (os.path.basename(src), missing)
