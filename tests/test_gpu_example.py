"""The example that runs the cache operators together, over a pool that suspends and resumes its requests."""
import importlib.util
import os

import pytest

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("fmt", ["bf16", "f16", "e4m3", "int8"])
def test_drafted_decode(fmt):
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "drafted_decode.py")
    spec = importlib.util.spec_from_file_location("drafted_decode", path)
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    out = module.main(fmt)
    assert out.shape == (4, 32, 128) and out.isfinite().all()
