"""The examples over 4-bit caches: forked answers in every format, drafted tokens in the new one."""
import importlib.util
import os

import pytest

pytestmark = pytest.mark.gpu


def example(name):
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", name + ".py")
    spec = importlib.util.spec_from_file_location(name, path)
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


@pytest.mark.parametrize("fmt", ["e2m1", "bf16", "f16", "e4m3", "int8"])
def test_forked_decode(fmt):
    out = example("forked_decode").main(fmt)
    assert out.shape == (4, 32, 128) and out.isfinite().all()


def test_drafted_decode_in_4_bits():
    out = example("drafted_decode").main("e2m1")
    assert out.shape == (4, 32, 128) and out.isfinite().all()
