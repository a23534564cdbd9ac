"""The latent-attention calls where no GPU is needed: refusals of the binding beyond shapes and types, and the polynomial
of the prompt kernel against its bound."""
import os
import re

import numpy as np
import pytest
import torch

from paper_2605_06068_b200 import binding as pda


def bf(*s):
    return torch.zeros(s, dtype=torch.bfloat16)


def i32(*s):
    return torch.zeros(s, dtype=torch.int32)


@pytest.mark.parametrize("weight", [bf(256, 4)[:, :2], bf(2, 300)[:, :256], bf(1).expand(512)])
def test_append_refuses_a_weight_with_gaps(weight):
    """As many elements as the latent has, but not one behind the other: they would be read as if they were."""
    with pytest.raises(ValueError, match="norm_weight"):
        pda.latent_append(bf(2, 512), bf(2, 64), bf(3, 16, 576), i32(2), norm_weight=weight)


def test_append_takes_a_weight_of_any_shape_without_gaps():
    for weight in (bf(512), bf(1, 512), bf(2, 256), bf(4, 512)[1]):
        with pytest.raises(ValueError, match="CUDA"):        # (past all checks that a CPU tensor can fail)
            pda.latent_append(bf(2, 512), bf(2, 64), bf(3, 16, 576), i32(2), norm_weight=weight)


@pytest.mark.parametrize("make", [lambda n: torch.zeros(1, dtype=torch.uint8).expand(n), lambda n: torch.zeros(2 * n, dtype=torch.uint8)[::2]])
def test_attention_refuses_a_workspace_with_gaps(make):
    """Its bytes are counted, and written one behind the other: an expanded or sliced tensor does not own so many."""
    n = 64 << 20
    with pytest.raises(ValueError, match="workspace"):
        pda.paged_latent_attention(bf(2, 4, 512), bf(2, 4, 64), bf(3, 16, 576), i32(2, 4), i32(2), 0.1, workspace=make(n))


def test_polynomial_of_the_exponentials_is_within_its_bound():
    """The coefficients that the prompt kernel evaluates, as they stand in its source, over [-1/2, 1/2] in 64 and 32 bits: a
    largest relative error of 7.5e-5 (2^-13.7, under the 2^-12 that the GPU tests' bounds allow an exponential), to which 32
    bits add three roundings."""
    path = os.path.join(os.path.dirname(pda.__file__), "csrc", "latent_prefill_tc.cu")
    body = open(path).read().split("void exp2_pair", 1)[1].split("\n}", 1)[0]
    c = [float(x) for x in re.findall(r"both\((0\.\d+)f\)", body)]
    assert len(c) == 4                                       # the highest power's first
    f = np.linspace(-0.5, 0.5, 200001)
    exact = np.exp2(f)
    assert np.abs(np.polyval(c, f) / exact - 1).max() < 7.6e-5
    y = np.full(f.shape, c[0], dtype=np.float32)
    for a in c[1:]:
        y = (y * f.astype(np.float32) + np.float32(a)).astype(np.float32)
    assert np.abs(y / np.exp2(f.astype(np.float32).astype(np.float64)) - 1).max() < 7.6e-5 + 6 * 2.0 ** -24
