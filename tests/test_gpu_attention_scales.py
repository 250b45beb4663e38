"""Attention with scales far from 1 / sqrt(head size): scores of ordinary size from very small or very large queries and keys.

Bounds: those of tests/test_gpu_attention.py, which go by the scaled scores."""
import pytest
import torch

from tests import test_gpu_attention as A

pytestmark = pytest.mark.gpu


# (scale, size of queries and keys): few keys, so that a wavefront has none; rows that see none; enough images that a workgroup takes 128 rows
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("scale,size", [(1e9, 3e-5), (-3e12, 3e-7), (3e30, 6e-16), (1e-9, 3e4), (1e-35, 1e17), (-1e-33, 3e16), (1e-39, 1e18)])
@pytest.mark.parametrize("shape,causal", [((2, 2, 1, 33, 20, 16), False), ((2, 2, 2, 90, 70, 16), True), ((700, 1, 1, 5, 20, 16), False), ((1, 4, 1, 1, 2000, 16), False)])
def test_extreme_scales(shape, causal, scale, size, dtype):
    b, h, kv, ql, kl, d = shape
    q, k, v, do = A._make(b, h, kv, ql, kl, d, dtype)
    q, k = q * size, k * size
    a = A._run(q, k, v, do, dtype, causal, scale)
    ref = A._reference(q, k, v, do, causal, scale, None, None)
    A._check(a, ref, dtype, d, max(kl, ql * (h // kv)))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("scale", [1e-35, 1e-20, 0.125, 1e9])
@pytest.mark.parametrize("shape,causal", [((2, 2, 1, 33, 20, 16), False), ((2, 2, 2, 90, 70, 16), True), ((1, 4, 1, 1, 2000, 16), False)])
def test_scores_far_below_zero(shape, causal, scale, dtype):
    """Scaled scores around -200, from queries and keys of opposite signs."""
    b, h, kv, ql, kl, d = shape
    q, k, v, do = A._make(b, h, kv, ql, kl, d, dtype)
    size = (200 / (16 * scale)) ** 0.5
    q, k = (1 + 0.02 * q) * size, (1 + 0.02 * k) * -size
    a = A._run(q, k, v, do, dtype, causal, scale)
    ref = A._reference(q, k, v, do, causal, scale, None, None)
    A._check(a, ref, dtype, d, max(kl, ql * (h // kv)))
