"""The rule that cuts a batch's shared prefixes, compiled from the library's own
header by the host compiler."""
import ctypes as C
import os
import shutil
import subprocess

import pytest

from conftest import ROOT

SHIM = """
#include "shared_plan.hpp"
extern "C" void plan(int n, int H, int G, int groups, int max_prefix, int *out) {
  const sm::SharedPlan p = sm::plan_shared(n, H, G, groups, max_prefix);
  out[0] = p.chunk;
  out[1] = p.chunks;
  out[2] = (int)sm::shared_most_chunks((long long)n * G * H, max_prefix);
}
"""


@pytest.fixture(scope="session")
def plan(tmp_path_factory):
    """plan(requests, kv heads, group, groups, longest prefix): (chunk, chunks, chunks that the workspace holds)"""
    if shutil.which("g++") is None:
        pytest.skip("g++ not available")
    d = tmp_path_factory.mktemp("plan")
    (d / "plan.cpp").write_text(SHIM)
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-shared", "-fPIC",
                    "-I", os.path.join(ROOT, "paper_2609_27233_amd", "csrc"), str(d / "plan.cpp"), "-o",
                    str(d / "plan.so")], check=True, timeout=120)
    f = C.CDLL(str(d / "plan.so")).plan

    def call(*a):
        out = (C.c_int * 3)()
        f(*a, out)
        return tuple(out)
    return call


@pytest.mark.parametrize("H,G", [(8, 4), (4, 7), (1, 16), (8, 8), (4, 1), (1, 1)])
def test_the_chunks_cover_any_prefix_and_fit_the_workspace(plan, H, G):
    for n in (1, 2, 3, 16, 33, 128, 1000, 4096, 65535 // H):
        for groups in (1, 2, 5, 100, 65535):
            for longest in (0, 1, 127, 128, 129, 1000, 8192, 32768, 1000000, 2 ** 31 - 1):
                chunk, chunks, most = plan(n, H, G, groups, longest)
                assert chunk % 128 == 0 and 128 <= chunk <= 8192
                assert chunks * chunk >= longest and (chunks - 1) * chunk < max(1, longest)
                assert max(1, chunks) <= most, (n, groups, longest)


def test_the_forms_of_the_gpu_tests(plan):
    """Two workgroups a compute unit where their chunks stay long, one otherwise."""
    assert plan(1000, 1, 16, 1, 3700)[:2] == (1024, 4)           # 125 blocks of vectors
    assert plan(1000, 1, 16, 1, 3500)[:2] == (1792, 2)
    assert plan(16, 8, 4, 1, 2048)[:2] == (128, 16)
    assert plan(500, 8, 4, 1, 4096)[:2] == (2048, 2)             # many requests' own entries beside them
