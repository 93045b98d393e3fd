"""The example of private adapters beside an encrypted projection, as it runs."""
import os
import sys

import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


def test_private_adapters():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    import private_adapters
    r = private_adapters.main(verbose=False)
    assert r["projection_error"] < 1e-3
    # the clients' wishes have rank 4, the adapters too: what stays is the dropout's noise
    assert r["losses"][-1] < 0.2 * r["losses"][0]
    assert r["after"] < 0.2 * r["before"]
