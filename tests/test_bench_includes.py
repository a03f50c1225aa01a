"""The hash of the GEMM's sources covers the headers they include."""
import os
import re
import shutil

import bench

# launch parameters and launchers on the host side, and the scale update that rides in extra workgroups: no part of a tile
NOT_HASHED = {"kernels.h", "scale_update.h"}


def included(name, seen):
    for part in re.findall(r'^#include "([^"]+)"', open(os.path.join(bench.CSRC, name)).read(), flags=re.M):
        if part not in seen and part not in NOT_HASHED:
            seen.add(part)
            included(part, seen)
    return seen


def test_every_include_is_hashed():
    found = set()
    for name in bench.GEMM_SOURCES:
        included(name, found)
    assert found and found <= set(bench.GEMM_SOURCES) | set(bench.GEMM_SHARED)


def test_a_shared_header_changes_the_hash(tmp_path):
    for name in bench.GEMM_SOURCES + bench.GEMM_SHARED:
        shutil.copy(os.path.join(bench.CSRC, name), tmp_path)
    assert bench.gemm_source_sha256(str(tmp_path)) == bench.gemm_source_sha256()
    for name in bench.GEMM_SHARED:
        path = os.path.join(tmp_path, name)
        text = open(path).read()
        open(path, "w").write(text + "\n// a comment\n")
        assert bench.gemm_source_sha256(str(tmp_path)) == bench.gemm_source_sha256()
        open(path, "w").write(text + "\nstatic int added;\n")
        assert bench.gemm_source_sha256(str(tmp_path)) != bench.gemm_source_sha256()
        open(path, "w").write(text)
