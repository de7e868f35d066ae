"""Attention over the 4-bit key/value cache at the ends of its scales."""
import pytest
import torch

from tests.test_gpu_kv4_numbers import KERNELS, problem

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("scale", [1.2, -1.9])
@pytest.mark.parametrize("name", KERNELS)
def test_the_largest_scales(name, scale):
    """Any finite scale is taken: powers of two in it for those in the queries are the same scores, and the same bits.  (Queries of bf16 values: 2^-124 of them has all their digits in fp32.)"""
    p, sizes = problem(name)
    p.qd, p.scale = p.qd.float(), scale * 2.0 ** 3
    want = p.run(**sizes)
    assert bool(torch.isfinite(want.float()).all())
    p.qd, p.scale = p.qd * 2.0 ** -124, scale * 2.0 ** 127
    assert abs(p.scale) > 1e38 and torch.equal(p.run(**sizes), want)
