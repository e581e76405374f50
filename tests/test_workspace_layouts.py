"""Where the workspaces' parts lie: what is read 16 bytes at a time starts at a
multiple of 16."""
import ctypes as C
import os
import shutil
import subprocess

import pytest

from conftest import ROOT
from paper_2609_27233_amd import lib as sm
from test_abi_cpu import _desc


@pytest.mark.parametrize("vocab", [1, 1000, 128256, 1 << 19])
def test_every_row_of_the_sampling_workspace_is_aligned(vocab):
    L = sm.load()
    one = L.sm_sample_workspace_bytes(1, vocab)
    assert one > 0 and one % 16 == 0
    for rows in (2, 3, 1024):
        assert L.sm_sample_workspace_bytes(rows, vocab) == rows * one


SHIM = """
#include "shared_plan.hpp"
extern "C" void parts(int64_t vectors, int64_t chunks, int head_dim, int64_t *out) {
  const sm::SharedParts p = sm::shared_parts(vectors, chunks, head_dim);
  out[0] = p.flag;
  out[1] = p.o;
  out[2] = p.ml;
  out[3] = p.end;
}
"""


@pytest.fixture(scope="module")
def parts(tmp_path_factory):
    if shutil.which("g++") is None:
        pytest.skip("g++ not available")
    d = tmp_path_factory.mktemp("parts")
    (d / "parts.cpp").write_text(SHIM)
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-shared", "-fPIC",
                    "-I", os.path.join(ROOT, "paper_2609_27233_amd", "csrc"), str(d / "parts.cpp"), "-o",
                    str(d / "parts.so")], check=True, timeout=120)
    f = C.CDLL(str(d / "parts.so")).parts
    f.argtypes = [C.c_int64, C.c_int64, C.c_int, C.POINTER(C.c_int64)]

    def call(*a):
        out = (C.c_int64 * 4)()
        f(*a, out)
        return tuple(out)
    return call


@pytest.mark.parametrize("D", [64, 128])
def test_the_parts_of_shared_prefixes_are_aligned(parts, D):
    """One request of one head behind a prefix of one chunk among them: an odd number of parts."""
    for vectors in (1, 3, 7, 512, 65535 * 16):
        for chunks in (1, 2, 5, 129):
            flag, o, ml, end = parts(vectors, chunks, D)
            assert flag == 0 and o >= flag + 4 and o % 16 == 0 and ml % 8 == 0
            assert ml == o + 4 * D * vectors * chunks and end == ml + 8 * vectors * chunks
    L = sm.load()
    assert L.sm_decode_shared_workspace_bytes(1, 1, D, 16, 16) >= L.sm_decode_workspace_bytes(1, 1, D, 16) + parts(1, 1, D)[3]


@pytest.mark.parametrize("ws", [4, 8, 24])
def test_a_shared_workspace_off_16_bytes_is_refused(ws):
    d = _desc(dtype=sm.SM_E4M3, k_pool=16, v_pool=32)
    assert sm.load().sm_decode_attention_shared(C.byref(d), 1, 4, 1, 1, 1, 1, 32, 1.0, 16, 16, 1, ws, 1 << 40, None) == sm.SM_EINVAL


def test_a_shared_grid_of_two_to_the_24_is_refused():
    """4095 groups x 4097 chunks of 8192 entries, and one workgroup for the request's own: 2^32 threads, one more than a
    launch counts."""
    d = _desc(dtype=sm.SM_E4M3, k_pool=16, v_pool=32, num_kv_heads=1, block_size=512, max_blocks_per_seq=4097 * 16)
    longest = 4097 * 8192
    need = sm.load().sm_decode_shared_workspace_bytes(1, 1, 128, 0, longest)
    assert sm.load().sm_decode_attention_shared(C.byref(d), 1, 1, 1, 1, 4095, 1, 1, 1.0, 0, longest, 1, 16, need, None) == sm.SM_EINVAL
