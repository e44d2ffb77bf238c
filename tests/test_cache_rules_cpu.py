"""CPU checks of the rules that launch the attention calls around the cache."""
import os
import re

import bench

CSRC = os.path.join(bench.ROOT, "paper_2604_26256_amd", "csrc")


def test_profile_hash_covers_the_launch_rules():
    """A summary is valid while the rules that launch its kernels are what they were: each rule is
    defined in a source that the hash covers."""
    for rule in ("tree_layout", "tree_whole", "tree_tiles", "window_layout", "most_visible", "visible_pages"):
        found = []
        for name in sorted(os.listdir(CSRC)):
            path = os.path.join(CSRC, name)
            if os.path.isfile(path) and re.search(rf"^[\w: *&]+ {rule}\([^;]*?\) \{{", open(path).read(), re.M):
                found.append(path)
        assert len(found) == 1 and found[0] in bench.KERNEL_SOURCES, (rule, found)
