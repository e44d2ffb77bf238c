"""CPU checks of the rules that launch the attention calls around the cache."""
import os
import re
import shutil
import subprocess

import numpy as np
import pytest

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


def test_stages_of_a_launch_fit_32_bits(tmp_path):
    """The kernels sum a launch's stages in 32 bits: for every geometry that a descriptor may have, its
    sequences are so many that full rows stay below 2^31, and one at least."""
    cxx = shutil.which("g++")
    if cxx is None:
        pytest.skip("no C++ compiler")
    rocm = os.environ.get("ROCM_PATH", "/opt/rocm")
    exe = str(tmp_path / "cache_rules")
    subprocess.run([cxx, "-std=c++17", "-O1", "-w", "-D__HIP_PLATFORM_AMD__", "-I", os.path.join(rocm, "include"), "-I", CSRC,
                    "-I", os.path.join(bench.ROOT, "include"), os.path.join(bench.ROOT, "tests", "cache_rules.cpp"), "-o", exe],
                   check=True)
    rng = np.random.default_rng(0)
    cases = [(64, 16, 64, 16, 4160, 2006), (32, 16, 64, 32, 4086, 100000), (127, 16, 64, 32, 2 ** 19 - 1, 32),
             (127, 1, 1, 16, 2 ** 19 - 1, 32), (1, 1, 1, 16, 1, 8192)]
    for _ in range(20000):
        heads, stride = int(rng.integers(1, 128)), int(2 ** rng.uniform(0, 19))
        most = min(8192, (2 ** 31 - 1) // (stride * heads))  # (a descriptor's own bound)
        if most > 0:
            cases.append((heads, int(rng.integers(1, 17)), int(rng.integers(1, 65)), int(rng.choice([16, 32])), stride, most))
    for heads, group, nodes, page, stride, seqs in cases:
        assert min(seqs, 8192) * stride * heads < 2 ** 31, "no such descriptor"
    r = subprocess.run([exe], input="".join("%d %d %d %d %d %d\n" % c for c in cases), stdout=subprocess.PIPE, text=True, check=True,
                       timeout=60)
    got = [tuple(int(x) for x in line.split()) for line in r.stdout.splitlines()]
    assert len(got) == len(cases)
    bad = [(c, g) for c, g in zip(cases, got) if not (1 <= g[0] <= c[5] and g[1] < 2 ** 31)]
    assert not bad, (len(bad), bad[:3])
