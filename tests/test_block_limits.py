"""Limits of the decoder block's layers that are refused before anything is launched.  No GPU needed."""
import pytest

import paper_2312_14227_b200 as et


def _attn(**k):
    return et.et_layer_desc(**{"in_features": 128, "out_features": 64, "fold": 1, "residual_src": -1, "kind": et.ET_LAYER_MASKED_ATTENTION,
                               "heads": 4, "kv_heads": 2, "head_dim": 16, **k})


def test_caps_that_leave_fp32():
    """Scores up to the cap, in powers of 2, and the scores' factor of it have to be fp32 numbers with all their bits."""
    for k in (dict(softcap=1e9), dict(softcap=2e37), dict(softcap=2e38, scale=3.0), dict(softcap=1e-30)):
        et.et_stack_create([_attn(**k)], 8, et.ET_BF16)
    for k in (dict(softcap=2.4e38, scale=100.0), dict(softcap=3e38, scale=100.0), dict(softcap=1e38), dict(softcap=1e30, scale=1e-10),
              dict(softcap=float("nan"))):
        with pytest.raises(et.EtError) as e:
            et.et_stack_create([_attn(**k)], 8, et.ET_BF16)
        assert e.value.status == et.ET_ERR_INVALID_ARG, k


def test_a_loop_that_counts_the_dropout_step_needs_a_dropout_layer():
    torch = pytest.importorskip("torch")
    from paper_2312_14227_b200.elastic_loop import ElasticLoop
    t, none = torch.zeros(8, 8), torch.zeros(0)
    dense = et.et_layer_desc(in_features=8, out_features=8, fold=1, residual_src=-1)
    drop = et.et_layer_desc(in_features=8, out_features=8, fold=1, residual_src=-1, kind=et.ET_LAYER_DROPOUT, drop=0.5)
    args = (t, t, 0.1, 4, 2, 0.5, [1.0] * 4, [1.0] * 4)
    ElasticLoop(et.et_stack_create([dense, drop], 8, et.ET_F32), [t, none], [t[0], none], *args, dropout_seed=3)
    with pytest.raises(et.EtError) as e:
        ElasticLoop(et.et_stack_create([dense, dense], 8, et.ET_F32), [t, t], [t[0], t[0]], *args, dropout_seed=3)
    assert e.value.status == et.ET_ERR_INVALID_ARG
