"""The adapters' host code on a fake device (fake_device.cpp: CUDA's calls on host
memory; kernels' launches are written down, none runs)."""
import ctypes
import os
import subprocess

import numpy as np
import pytest

from paper_2609_35352_gb300 import build as B

HERE = os.path.dirname(os.path.abspath(__file__))


@pytest.fixture(scope="module")
def fake(tmp_path_factory):
    B.build()
    out = str(tmp_path_factory.mktemp("fake") / "libfake.so")
    cuda = os.path.join(os.path.dirname(os.path.dirname(os.path.realpath(B.nvcc()))), "include")
    # (symbolic: a process with torch in it has the real calls loaded)
    cmd = ["g++", "-std=c++17", "-O1", "-shared", "-fPIC", "-Wl,-Bsymbolic", "-I" + B.INCLUDE, "-I" + B.CSRC, "-I" + cuda,
           os.path.join(HERE, "fake_device.cpp")]
    objects = [f for f in B.LIBRARIES["libfiona.so"] if f.startswith(("adapter", "dropout"))]
    for f in objects:  # (a built library without its objects)
        if not os.path.exists(os.path.join(B.OUT, f + ".o")):
            B._compile(os.path.join(B.CSRC, f), os.path.join(B.OUT, f + ".o"), [])
    cmd += [os.path.join(B.OUT, f + ".o") for f in objects] + ["-o", out]
    r = subprocess.run(cmd, capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    L = ctypes.CDLL(out)
    p, u32, u64 = ctypes.c_void_p, ctypes.c_uint32, ctypes.c_uint64
    L.fake_context.restype, L.fake_last_error.restype = p, ctypes.c_char_p
    L.fake_context_destroy.argtypes, L.fake_tables_arrived.argtypes = [p], [p, p]
    L.fiona_adapter_batch_create.argtypes = [p, u32, p, p, u32, p, p, u32, ctypes.POINTER(p)]
    for name, result in (("name", ctypes.c_char_p), ("blocks", u64), ("shared", u64), ("bare", u32), ("first_row", u32)):
        getattr(L, "fake_" + name).restype = result
    L.fiona_adapter_forward.argtypes = [p, p, p, p, u64, p, u64, p, u64, p, p, p, u64]
    L.fiona_adapter_backward.argtypes = [p, p, p, p, u64, p, p, u64, p, u64, p, u64, p, p, p, p, u64]
    L.fiona_adapter_work_bytes.argtypes = [p, u32, u32, u32, ctypes.POINTER(u64)]
    L.fiona_adapter_batch_forward_only.argtypes = [p]
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


class Layer(ctypes.Structure):  # fiona_adapter_layer
    _fields_ = [("d_in", ctypes.c_uint32), ("d_out", ctypes.c_uint32), ("dtype", ctypes.c_uint32),
                ("reserved", ctypes.c_uint32), ("A", ctypes.c_void_p), ("B", ctypes.c_void_p)]


class DropoutSpec(ctypes.Structure):  # fiona_dropout_spec
    _fields_ = [("seed", ctypes.c_uint64), ("offset", ctypes.c_uint64), ("p", ctypes.c_double)]


F32, BF16 = 0, 2


def call(fake, batch, d_in, d_out, dtype, backward=False, drop=None):
    """A call on addresses far apart (nothing reads them)."""
    n = ctypes.c_uint64()
    assert fake.fiona_adapter_work_bytes(batch, d_in, d_out, dtype, ctypes.byref(n)) == 0
    at = lambda k: k << 48  # noqa: E731
    layer = Layer(d_in, d_out, dtype, 0, at(1), at(2))
    spec = None if drop is None else ctypes.byref(drop)
    fake.fake_forget()
    if backward:
        return fake.fiona_adapter_backward(batch, None, ctypes.byref(layer), at(3), d_in, at(4), at(5), d_out, None, 0, at(6), d_in,
                                           at(7), at(8), spec, at(9), n.value)
    return fake.fiona_adapter_forward(batch, None, ctypes.byref(layer), at(3), d_in, None, 0, at(5), d_out, None, spec, at(9), n.value)


def launches(fake, part):
    return [i for i in range(fake.fake_launches()) if part in fake.fake_name(i).decode()]


@pytest.mark.parametrize("backward", [False, True])
def test_grids_past_what_a_launch_holds(fake, ctx, backward):
    """70000 runs of one row beside 2^20 columns: 2.3e9 blocks, in two launches.  Every
    tile is in one of them, and the rows without an adapter are in the first."""
    n, d = 70000, 1 << 20
    ids = [-1] + [i % 2 for i in range(n)]
    h = make_batch(fake, ctx, list(range(n + 2)), ids, [4, 4], 4)
    rc = call(fake, h, d, d, F32, backward)
    assert rc == 0, fake.fake_last_error()
    found, tiles = launches(fake, "k_any_expand"), [r for a in (0, 1) for r, i in enumerate(ids) if i == a]
    assert len(found) == 2
    at = 0
    for i in found:
        slabs = ctypes.c_uint32()
        assert fake.fake_first_row(i, ctypes.byref(slabs)) == tiles[at] and slabs.value == d // 64
        assert fake.fake_bare(i) == (1 if at == 0 else 0)
        at += (fake.fake_blocks(i) - fake.fake_bare(i)) // (2 * slabs.value)
    assert at == len(tiles)
    if backward:  # the weight gradients' chunks count from the first tile again
        for i in launches(fake, "k_any_grad")[:1]:
            assert fake.fake_first_row(i, ctypes.byref(ctypes.c_uint32())) == tiles[0]
    fake.fiona_adapter_batch_destroy(h)


def work_bytes(fake, batch, d_in, d_out, dtype):
    n = ctypes.c_uint64()
    assert fake.fiona_adapter_work_bytes(batch, d_in, d_out, dtype, ctypes.byref(n)) == 0
    return n.value


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_no_room_for_partial_gradients_that_are_not_made(fake, ctx, dtype):
    """256 tokens of 200 adapters: each adapter's gradient comes from one chunk and is
    written as it is.  Partial sums of dA and dB would take 524 MB."""
    h = make_batch(fake, ctx, list(range(257)), [i % 200 for i in range(256)], [64] * 200, 64)
    assert call(fake, h, 2048, 8192, dtype, backward=True) == 0
    assert not launches(fake, "grad_sum")
    assert work_bytes(fake, h, 2048, 8192, dtype) < 100e6
    fake.fiona_adapter_batch_destroy(h)
    # one adapter's long batch is cut into chunks, and their sums have their room
    h = make_batch(fake, ctx, [0, 16384], [0], [64], 64)
    assert call(fake, h, 2048, 8192, dtype, backward=True) == 0
    assert launches(fake, "grad_sum") or launches(fake, "k_image")
    assert work_bytes(fake, h, 2048, 8192, dtype) > 2 * 64 * (2048 + 8192) * 4
    fake.fiona_adapter_batch_destroy(h)


@pytest.mark.parametrize("dtype,d_in,d_out,most", [(F32, 4096, 4096, 70e6), (BF16, 4096, 4096, 70e6), (BF16, 4092, 4091, 300e6)])
def test_workspace_of_a_batch_for_forward_calls_only(fake, ctx, dtype, d_in, d_out, most):
    """8192 tokens of 2 adapters in turn, rank 128.  The gradient's images alone take
    1.07 GB in 16 bits.  (Off eight, the copies of x and out have their room.)"""
    h = make_batch(fake, ctx, list(range(8193)), [i % 2 for i in range(8192)], [128, 128], 128)
    assert call(fake, h, d_in, d_out, dtype, backward=True) == 0
    both = work_bytes(fake, h, d_in, d_out, dtype)
    assert fake.fiona_adapter_batch_forward_only(h) == 0
    n = work_bytes(fake, h, d_in, d_out, dtype)
    assert n < most and (dtype == F32 or n < both / 4)
    assert call(fake, h, d_in, d_out, dtype) == 0, fake.fake_last_error()
    assert call(fake, h, d_in, d_out, dtype, backward=True) == -1
    assert b"forward" in fake.fake_last_error()
    fake.fiona_adapter_batch_destroy(h)
    assert fake.fiona_adapter_batch_forward_only(None) == -1


@pytest.mark.parametrize("r_max", [16, 64, 72, 112, 128])
def test_cut_of_dx_goes_by_tiles(fake, ctx, r_max):
    """The pass that makes dx and dA writes no partial dh: how it is cut goes by the
    tiles, whether they hold 128 rows each or one."""
    blocks = []
    for rows in (128, 1):
        h = make_batch(fake, ctx, [rows * i for i in range(33)], [i % 2 for i in range(32)], [r_max] * 2, r_max)
        assert call(fake, h, 2048, 2048, BF16, backward=True) == 0
        (i,) = launches(fake, "k_expand_grad")
        slabs = ctypes.c_uint32()
        fake.fake_first_row(i, ctypes.byref(slabs))
        blocks.append((fake.fake_blocks(i), slabs.value))
        fake.fiona_adapter_batch_destroy(h)
    assert blocks[0] == blocks[1]


@pytest.mark.parametrize("r_max", range(8, 129, 8))
@pytest.mark.parametrize("p", [None, 0.25])
def test_tensor_memory_of_blocks_that_meet(fake, ctx, r_max, p):
    """Two blocks that shared memory lets onto an SM never ask for more than its 512
    columns, whichever kernels and ranks (a block would wait for ever).  The kernels that
    take over 256 columns are the weight gradients'."""
    h = make_batch(fake, ctx, [0, 700, 8000], [0, 1], [r_max] * 2, r_max)
    drop = None if p is None else DropoutSpec(1, 2, p)
    for backward in (False, True):
        assert call(fake, h, 2048, 4096, BF16, backward, drop) == 0, fake.fake_last_error()
        for i in launches(fake, "k_shrink") + launches(fake, "k_expand"):
            cols = 512 if "grad" in fake.fake_name(i).decode() else 256
            assert fake.fake_shared(i) >= (152 if cols > 256 else 76) * 1024
            assert 3 * (fake.fake_shared(i) + 1024) > 228 * 1024
    fake.fiona_adapter_batch_destroy(h)
