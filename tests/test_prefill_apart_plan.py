"""Which calls over 8-bit pages have their waves work apart, by the library's own
header compiled by the host compiler."""
import ctypes as C
import os
import shutil
import subprocess

import pytest

import test_gpu_e4m3_attention as gpu
from conftest import ROOT

SHIM = """
#include "prefill_plan.hpp"
extern "C" int form(int n, int H, int G, int total_rows, int max_rows, long long capacity) {
  if (sm::prefill_apart(n, H, G, total_rows, max_rows)) return 8;
  const sm::PrefillPlan p = sm::plan_prefill(n, H, G, total_rows, max_rows, capacity);
  return p.few ? -p.splits : p.splits;
}
"""


@pytest.fixture(scope="session")
def form(tmp_path_factory):
    if shutil.which("g++") is None:
        pytest.skip("g++ not available")
    d = tmp_path_factory.mktemp("apart")
    (d / "form.cpp").write_text(SHIM)
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-shared", "-fPIC",
                    "-I", os.path.join(ROOT, "paper_2609_27233_amd", "csrc"), str(d / "form.cpp"), "-o",
                    str(d / "form.so")], check=True, timeout=120)
    f = C.CDLL(str(d / "form.so")).form
    f.argtypes = [C.c_int] * 5 + [C.c_longlong]
    return lambda *a: {8: "apart", -4: "few"}.get(f(*a), f(*a))


@pytest.mark.parametrize("case", range(len(gpu.FORMS)))
def test_the_gpu_tests_take_the_form_they_name(form, case):
    Hq, H, D, bs, reqs, name = gpu.FORMS[case]
    rows, capacity = [m for m, _ in reqs], -(-max(m + past for m, past in reqs) // bs) * bs
    assert form(len(reqs), H, Hq // H, sum(rows), max(rows), capacity) == name


def test_the_gpu_tests_reach_every_form():
    assert {(c[2], c[5]) for c in gpu.FORMS} == {(D, f) for D in (64, 128) for f in ("apart", "few", 4, 2, 1)}


@pytest.mark.parametrize("n,H,G", [(1, 8, 4), (3, 1, 16), (65535, 1024, 1), (7, 4, 7)])
def test_sizes_at_the_ends(form, n, H, G):
    """No rows, one, and the most that the arguments hold."""
    assert form(n, H, G, 0, 0, 16) == "apart"
    assert form(n, H, G, n, 1, 16) == "apart"
    assert form(n, H, G, 2 ** 31 - 1, 2 ** 31 - 1, 2 ** 40) != "apart"
