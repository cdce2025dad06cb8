"""The training and serving example: norms, gate and residual sum around the split MLP, AdamW with 8-bit states, int8
serving, all together."""
import os
import sys

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


def test_training_lowers_the_loss_and_int8_follows_the_trained_network():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
    import residual_blocks
    losses, errors = residual_blocks.main(["--hidden", "256", "--ffn", "1024", "--blocks", "2", "--tokens", "512", "--steps", "60"])
    assert losses[-1] < 0.7 * losses[0], losses
    # two roundings to 1/127 of a row's largest of 256 ... 1024 values (about 3.5 deviations) per layer, four layers: about
    # 0.8 % each, added in squares, and bf16 on both sides
    assert all(e < 0.05 for e in errors.values()), errors
