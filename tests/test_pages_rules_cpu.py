"""CPU checks of where the rules that launch the operators that read less of the cache stand."""
import os
import re

import bench

CSRC = os.path.join(bench.ROOT, "paper_2604_26256_amd", "csrc")


def test_profile_hash_covers_the_launch_rules():
    """A summary is valid while the rules that launch its kernels are what they were: each rule is defined in a source
    that the hash covers, and the front end, which it does not, decides nothing by itself."""
    for rule in ("pages_layout", "pages_waves", "pages4_waves", "pages4_split", "select_at_once"):
        found = []
        for name in sorted(os.listdir(CSRC)):
            path = os.path.join(CSRC, name)
            if os.path.isfile(path) and re.search(rf"^[\w: *&]+ {rule}\([^;]*?\) \{{", open(path).read(), re.M):
                found.append(path)
        assert len(found) == 1 and found[0] in bench.KERNEL_SOURCES, (rule, found)
    front = re.sub(r"//.*", "", open(os.path.join(CSRC, "pages_api.cpp")).read())
    assert not re.findall(r"\bk(?:Seg|Score|Bounds|Select|Append4)\w*", front)
