"""The largest and smallest scales of the token scores, on logits that make up for them."""
import numpy as np
import pytest

from test_gpu_token_scores import _check, _rng, _run

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("scale", [1.9e38, 2.0 ** 120, 2.0 ** -120])
@pytest.mark.parametrize("V", [50, 3000, 40000])
def test_far_scales(scale, V):
    z = np.ldexp(_rng(40, V).standard_normal((4, V)).astype(np.float32), -int(np.log2(scale))).astype(np.float32)
    z = np.where(np.abs(z) < 2.0 ** -126, np.float32(0), z)     # no subnormal logits
    tokens = np.array([0, V - 1, -1, V // 2], np.int32)
    got, _ = _run(z, "f32", tokens, scale, 5)
    _check(got, z.astype(np.float64), tokens, scale, 5)
