"""The decoder block's layers at the ends of their ranges."""
import pytest
import torch

import paper_2312_14227_b200 as et
from test_gpu_seq_attention import Attn

pytestmark = pytest.mark.gpu


# ------------------------------------------------------------------------------------------ caps
@pytest.mark.parametrize("cap", [0.01, 1.0, 1e3, 1e5, 1e6, 1e9, 1e30])
@pytest.mark.parametrize("dim", [64, 128])
def test_caps_of_any_size(dim, cap):
    """A cap far above the scores changes nothing, one far below leaves their signs: an error of the cap's tanh is one of the score itself,
    not of the cap."""
    Attn(270, 2, 1, dim, seqs=[0, 133, 262], cap=cap, std=2.0, seed=3).check()
    Attn(270, 2, 1, dim, causal=False, cap=cap, slopes=[0.05, 0.5], std=2.0, seed=4).check()


def test_a_capped_key_that_is_not_a_number_is_seen():
    """Rows that see it have no score for it: their output is NaN, as it is without a cap."""
    for cap in (0.0, 20.0):
        for dim in (64, 128):
            for key in (5, 6):
                a = Attn(150, 1, 1, dim, cap=cap)
                a.x[key, dim:2 * dim] = float("nan")
                y, _ = a.run()
                assert bool(torch.isnan(y[key:]).all()), (cap, dim, key)
