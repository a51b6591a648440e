"""What the GPU tests of the attention's roundings would see, on the CPU: probabilities or outputs
cut off to bf16 instead of rounded to the nearest."""
import numpy as np
import torch


def _cut(x):
    """fp32 towards zero to bf16."""
    return (torch.from_numpy(x.astype(np.float32)).view(torch.int32) & -65536).view(torch.float32).double().numpy()


def _near(x):
    return torch.from_numpy(x.astype(np.float32)).to(torch.bfloat16).double().numpy()


def test_probabilities():
    """Values of one: rounded, every row of 256 to 700 tokens gives 1 in bf16, which the GPU test asks
    of all; cut off, not all do."""
    rng = np.random.default_rng(1)
    for n in (256, 300, 700):
        for spread in (0.3, 1.0, 1.5):
            s = rng.normal(size=(200, n)) * spread
            p = np.exp(s - s.max(1, keepdims=True))
            for scale in (1.0, 37.3):              # under the maximum, and under one that lags
                total = (p * scale).sum(1)
                assert (_near(_near(p * scale).sum(1) / total) == 1).all()
                assert (_near(_cut(p * scale).sum(1) / total) < 1).any()


def test_output():
    """The mean of two bf16 values: cut off, some lie further away than the nearest, and the GPU
    test allows none."""
    rng = np.random.default_rng(2)
    v = _near(rng.normal(size=(2, 1000)))
    mean = v.mean(0)
    off = np.abs(_cut(mean) - mean) > np.abs(_near(mean) - mean) + 2.0 ** -20 * np.abs(mean)
    assert off.any()
