"""What the tests of the long-context operators share: inputs, and the tolerance of attention."""

import os
import sys

import numpy as np
import pytest
import torch

from paper_2609_12330_amd import ef_attention as ef


def announce(msg):
    print(f"[gpu case] {msg}", file=sys.stderr, flush=True)


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    if not os.path.exists(ef.LIB_PATH):
        raise RuntimeError("libef_attention.so is not built; the HIP path must be present")
    ef.library()
    yield


def f64(t):
    return t.double().cpu().numpy()


def normal(seed, *shape):
    g = torch.Generator("cpu").manual_seed(seed)
    return torch.randn(shape, generator=g).to(torch.bfloat16)


def lengths_of(values):
    return None if values is None else torch.tensor(values, dtype=torch.int32, device="cuda")



# Tolerance of an output element. A weight is rounded to bf16 before it multiplies its value
# (half a step, 2^-8 of it), while the sum of the weights is of unrounded ones; a weight is
# further off by its score's error, at most 2 D 2^-24 scale |q| |k| (1.7e-4 at D = 128 with
# |q|^2 = |k|^2 = 128; norms are up to 1.6 times that) and by a few fp32 roundings: 1e-3 covers
# both, in the sum of the weights too. The result is rounded to bf16 once, half a step.


def close(got, ref, mag, what):
    """mag: the same attention over |v|, the sum of the magnitudes that make up ref."""
    got = f64(got)
    tol = (2.0 ** -8 + 1e-3) * mag + 2.0 ** -8 * 1.01 * np.abs(ref)
    worst = np.max(np.abs(got - ref) - tol, initial=-1.0)
    assert np.isfinite(got).all() and worst <= 0, f"{what}: {worst:.3e} over the tolerance"


def poison(t, lengths):
    """t on the GPU, NaN behind every sequence's length."""
    t = t.cuda()
    if lengths is not None:
        for b, n in enumerate(lengths):
            t[b, :, min(max(n, 0), t.shape[2]):] = float("nan")
    return t
