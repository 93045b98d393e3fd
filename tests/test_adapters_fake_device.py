"""The adapters' host code on a fake device (fake_device.cpp: CUDA's calls on host
memory, no kernels)."""
import ctypes
import os
import subprocess

import numpy as np
import pytest

from paper_2609_35352_gb300 import build as B

HERE = os.path.dirname(os.path.abspath(__file__))


@pytest.fixture(scope="module")
def fake(tmp_path_factory):
    out = str(tmp_path_factory.mktemp("fake") / "libfake.so")
    cuda = os.path.join(os.path.dirname(os.path.dirname(os.path.realpath(B.nvcc()))), "include")
    # (symbolic: a process with torch in it has the real calls loaded)
    cmd = ["g++", "-std=c++17", "-O1", "-shared", "-fPIC", "-Wl,-Bsymbolic", "-I" + B.INCLUDE, "-I" + B.CSRC, "-I" + cuda,
           os.path.join(B.CSRC, "adapter_host.cpp"), os.path.join(HERE, "fake_device.cpp"), "-o", out]
    r = subprocess.run(cmd, capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    L = ctypes.CDLL(out)
    p, u32, u64 = ctypes.c_void_p, ctypes.c_uint32, ctypes.c_uint64
    L.fake_context.restype, L.fake_last_error.restype = p, ctypes.c_char_p
    L.fake_context_destroy.argtypes, L.fake_tables_arrived.argtypes = [p], [p, p]
    L.fiona_adapter_batch_create.argtypes = [p, u32, p, p, u32, p, p, u32, ctypes.POINTER(p)]
    L.fiona_adapter_batch_destroy.argtypes, L.fiona_adapter_batch_destroy.restype = [p], None
    return L


@pytest.fixture
def ctx(fake):
    c = fake.fake_context(152)
    yield c
    fake.fake_context_destroy(c)


def make_batch(fake, ctx, starts, ids, ranks, r_max):
    s, a, r = np.array(starts, np.uint64), np.array(ids, np.int32), np.array(ranks, np.uint32)
    h = ctypes.c_void_p()
    rc = fake.fiona_adapter_batch_create(ctx, len(ids), s.ctypes.data, a.ctypes.data, len(ranks), r.ctypes.data, None, r_max,
                                         ctypes.byref(h))
    assert rc == 0, fake.fake_last_error()
    return h


def test_a_batch_is_on_the_device_when_its_creation_returns(fake, ctx):
    """Any stream may read it next: streams that do not wait for the legacy default
    stream, where the copy goes, too."""
    ranks = np.array([8, 3, 16], np.uint32)
    h = make_batch(fake, ctx, [0, 200, 210, 500], [2, 0, 1], ranks, 16)
    assert fake.fake_tables_arrived(h, ranks.ctypes.data) == 1
    fake.fiona_adapter_batch_destroy(h)
