"""Refusals of the latent-attention binding beyond shapes and types; no GPU needed."""
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
