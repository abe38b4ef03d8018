"""The plain forms of perf/operators.py compute the definitions that the kernels are held to."""

import importlib.util
import os

import pytest

from paper_2608_02703_gb300 import archead

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def operators():
    from paper_2608_02703_gb300.build import build

    build()
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "perf", "operators.py")
    spec = importlib.util.spec_from_file_location("operators_of_the_cases", path)
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("M,K", [(20000, 1000), (8192, 2560), (3000, 77)], ids=str)
def test_plain_quantiser_is_the_kernels(operators, M, K, dtype):
    """Bit for bit, over many rows: a scale that is one unit in the last place off turns a code now and then."""
    import torch

    for seed in range(3):
        gen = torch.Generator(device="cuda").manual_seed(seed)
        x = operators._hidden(gen, M, K, operators._DTYPES[dtype])
        codes, scales = torch.empty((M, K), dtype=torch.int8, device="cuda"), torch.empty(M, device="cuda")
        archead.archead_int8_quantize_tokens(x, codes, scales)
        plain_codes, plain_scales = operators._plain_quantize(x)
        assert torch.equal(scales, plain_scales)
        assert torch.equal(codes, plain_codes)
