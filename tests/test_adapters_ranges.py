"""Sizes whose products pass 64 bits are refused, and do not wrap (no GPU)."""
import ctypes

import numpy as np
import pytest

from paper_2609_35352_gb300 import adapters as AD
from paper_2609_35352_gb300 import build as B
from paper_2609_35352_gb300 import fiona as F
from paper_2609_35352_gb300 import workloads as W

from test_adapters_host import Call, DropoutSpec


@pytest.fixture(scope="module")
def ctx():
    B.build()
    return F.Context(1024, W.ntt_primes(1024, 40, 1), device=F.FIONA_DEVICE_NONE)


@pytest.mark.parametrize("rows,ld", [(1 << 39, 1 << 39), (1 << 32, 1 << 32), (3 << 30, 1 << 34), ((1 << 40) - 1, (1 << 40) - 1)])
def test_rows_times_stride(ctx, rows, ld):
    buf = np.zeros(4096, np.uint8)
    at, spec = (buf.ctypes.data + 15) // 16 * 16, DropoutSpec(1, 2, 0.5)
    assert AD.lib().fiona_dropout(ctx.handle, None, 2, rows, 8, at, ld, None, 0, at + 1024, ld, ctypes.byref(spec)) == F.FIONA_ERR_ARG


@pytest.mark.parametrize("backward", [False, True])
def test_workspaces_that_reach_past_the_address_space(ctx, backward):
    """One that overlaps another buffer by what it says it has."""
    for n in ((1 << 64) - 1, (1 << 64) - 4096, 1 << 63):
        c = Call(ctx, backward)
        c.work_bytes = n
        below = min(v for k, v in c.p.items() if k != "work")
        c.p["work"] = (below - (1 << 20)) // 16 * 16
        assert c() == F.FIONA_ERR_ARG
