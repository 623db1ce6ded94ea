"""The operators together: fine-tuning the dense layers behind a quantized conv stack."""
import os
import sys

import pytest

pytestmark = pytest.mark.gpu

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_the_loss_falls(dtype):
    import finetune_fc
    losses, right = finetune_fc.main(steps=40, dtype=dtype, show=False)
    # from the uniform guess (log 10 = 2.30) to a fit of the training images
    assert 2.0 < losses[0] < 2.7
    assert losses[-1] < 0.5 * losses[0]
    assert right[0] > 0.8
