"""What the calls over the paged cache make of their arguments at the ends of the ranges, and the polynomials there; no GPU needed."""
import os
import re

import numpy as np
import pytest
import torch

from paper_2605_06068_b200 import binding as pda


def source(name):
    return open(os.path.join(os.path.dirname(pda.__file__), "csrc", name)).read()


def test_polynomial_of_scores_below_a_cap_is_within_its_bound():
    """Relative to the score, in 64 bits and in 32 (a rounding for each of its steps)."""
    text = re.search(r"PDA_TANH_COEFFICIENTS \\\n\s*\{([^}]*)\}", source("shaped.cuh")).group(1)
    c = [float(x.strip().rstrip("f")) for x in text.split(",")]
    reach = float(re.search(r"kTanhReach = ([\d.]+)f", source("shaped.cuh")).group(1))
    x = np.linspace(1e-6, reach, 400001)
    assert np.abs(x * np.polyval(c[::-1], x * x) / np.tanh(x) - 1).max() < 2.0 ** -24.9
    f = x.astype(np.float32)
    t = f * f
    y = np.full(f.shape, c[-1], dtype=np.float32)
    for a in c[-2::-1]:
        y = y * t + np.float32(a)
    assert np.abs((f * y).astype(np.float64) / np.tanh(f.astype(np.float64)) - 1).max() < 2.0 ** -24.9 + (2 * len(c) + 2) * 2.0 ** -24


def test_numbers_given_as_tensors_are_read_at_each_call():
    """A tensor of one element as the scale, or tensors as the axes, hold other values at the next call."""
    t = torch.tensor(0.25)
    for value in (0.25, 0.5):
        t.fill_(value)
        assert pda._score_desc(t, t, None, np.int64(3), 8).scale == value
        assert pda._score_desc(0.1, t, None, 0, 8).softcap == value
    assert pda._score_desc(np.float32(0.5), 0, None, torch.tensor(7), 8).window == 7
    with pytest.raises(TypeError):
        pda._score_desc(0.1, 0.0, None, 2.5, 8)


def test_axes_given_as_tensors_are_read_at_each_call(monkeypatch):
    seen = []

    class Library:
        def rope_kv_append(self, *args):
            seen.append(args[12])
            return 0
    monkeypatch.setattr(pda, "lib", lambda: Library())
    monkeypatch.setattr(pda, "_one_device", lambda *tensors: 0)
    monkeypatch.setattr(pda, "_on_device", lambda dev, call, *args: call(*args))
    monkeypatch.setattr(pda, "_raw", lambda stream, dev: None)
    bf = lambda *s: torch.zeros(s, dtype=torch.bfloat16)
    axes = tuple(torch.zeros(8, dtype=torch.int32))
    for value in (0, 1):
        axes[3].fill_(value)
        pda.rope_kv_append(bf(5, 4, 64), bf(5, 2, 64), bf(5, 2, 64), torch.zeros((2, 5), dtype=torch.int32), torch.zeros(9, 16), bf(4, 2, 16, 64),
                           bf(4, 2, 16, 64), torch.zeros(5, dtype=torch.int32), freq_axis=axes)
    assert seen == [bytes(8), bytes([0, 0, 0, 1, 0, 0, 0, 0])]
