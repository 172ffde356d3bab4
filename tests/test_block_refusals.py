"""What the decoder block's layers and their calls refuse.  Nothing is launched: no GPU needed."""
import numpy as np
import pytest

import paper_2312_14227_b200 as et

X = np.zeros(64, dtype=np.float32)                       # any address: refused before it is used
P = (X.ctypes.data + 15) // 16 * 16
B, F = et.ET_BF16, et.ET_F32
INV, SHAPE, UNS, STATE = et.ET_ERR_INVALID_ARG, et.ET_ERR_SHAPE, et.ET_ERR_UNSUPPORTED, et.ET_ERR_STATE


def _d(kind, i, o, **k):
    return et.et_layer_desc(**{"in_features": i, "out_features": o, "fold": 1, "residual_src": -1, "kind": kind, **k})


def _dense(i, o, **k):
    return _d(et.ET_LAYER_DENSE, i, o, **k)


def _attn(heads=4, kv=2, dim=16, **k):
    return _d(et.ET_LAYER_MASKED_ATTENTION, **{"i": (heads + 2 * kv) * dim, "o": heads * dim, "heads": heads, "kv_heads": kv, "head_dim": dim, **k})


def _rot(heads=4, kv=2, dim=16, **k):
    w = (heads + 2 * kv) * dim
    return _d(et.ET_LAYER_ROTARY, w, w, **{"heads": heads, "kv_heads": kv, "head_dim": dim, "axes": 1, "sections": (dim // 2, 0, 0),
                                            "theta": 10000.0, **k})


def _gated(i=8, h=16, **k):
    return _d(et.ET_LAYER_GATED, i, 2 * h, **{"fold": 2, "act": et.ET_ACT_SILU, **k})


def _drop(w=16, **k):
    return _d(et.ET_LAYER_DROPOUT, w, w, **{"drop": 0.1, **k})


def _status(fn, *a, **k):
    with pytest.raises(et.EtError) as e:
        fn(*a, **k)
    return e.value.status


def _bad(layer, M=8, dtype=B):
    return _status(et.et_stack_create, layer if isinstance(layer, list) else [layer], M, dtype)


def test_attention_descriptions():
    et.et_stack_create([_attn()], 8, B)
    et.et_stack_create([_attn(seq_len=4, mask=et.ET_MASK_CAUSAL, softcap=30.0, scale=0.5, dim=128)], 8, B)
    for k in (dict(heads=0), dict(kv=0), dict(heads=3), dict(mask=2), dict(mask=-1), dict(softcap=-1.0), dict(softcap=float("inf")),
              dict(scale=-0.1), dict(scale=float("nan")), dict(scale=3e38), dict(softcap=1e-39), dict(scale=1e20, softcap=1e-20), dict(act=1), dict(residual_src=0), dict(seq_len=-1), dict(o=32), dict(i=136)):
        assert _bad(_attn(**k)) == INV, k
    assert _bad(_attn(seq_len=3)) == SHAPE
    assert _bad(_attn(), dtype=F) == UNS
    assert _bad(_attn(dim=20)) == UNS
    assert _bad(_attn(dim=136)) == UNS
    assert _bad([_dense(8, 128, act=1), _attn()]) == UNS                               # an activation below
    assert _bad([_dense(8, 128), _attn(), _dense(64, 128, residual_src=1)]) == UNS     # [q | k | v] feeds something else
    assert _bad([_dense(8, 120), _attn()]) == SHAPE


def test_rotary_descriptions():
    et.et_stack_create([_rot()], 8, B)
    et.et_stack_create([_rot(axes=3, sections=(3, 2, 1))], 8, F)
    for k in (dict(axes=0), dict(axes=4), dict(sections=(0, 0, 0)), dict(axes=2), dict(theta=0.0), dict(theta=float("inf")),
              dict(pairing=2), dict(spectrum=-1), dict(kv=0), dict(seq_len=-2), dict(act=2)):
        assert _bad(_rot(**k)) == INV, k
    assert _bad(_rot(sections=(9, 0, 0))) == SHAPE
    assert _bad(_rot(seq_len=5)) == SHAPE
    assert _bad(_rot(dim=512, sections=(129, 0, 0))) == UNS
    assert _bad([_dense(8, 128, act=2), _rot()]) == UNS


def test_gated_and_dropout_descriptions():
    et.et_stack_create([_gated(), _dense(16, 8)], 8, B)
    et.et_stack_create([_drop(residual_src=0)], 8, F)
    for k in (dict(act=0), dict(act=4), dict(fold=1), dict(residual_src=0, i=16)):
        assert _bad(_gated(**k)) == INV, k
    assert _bad(_gated(h=12)) == UNS                                                    # bf16: multiples of 8
    assert _bad(_dense(8, 8, act=et.ET_ACT_SILU)) == INV                                # for gated layers only
    assert _bad(_dense(8, 16, fold=2, act=1)) == UNS
    for k in (dict(drop=1.0), dict(drop=-0.1), dict(drop=float("nan")), dict(act=1), dict(residual_src=1)):
        assert _bad(_drop(**k)) == INV, k
    assert _bad(_d(10, 8, 8)) == INV


def test_state_calls():
    s = et.et_stack_create([_dense(8, 128), _rot(axes=2, sections=(2, 2, 0)), _attn(), _drop(64), _dense(64, 8)], 8, B)
    plain = et.et_stack_create([_dense(8, 8)], 8, B)
    et.et_stack_set_sequences(s, P, seqs=2)
    et.et_stack_set_sequences(s, P, P, seqs=2)
    et.et_stack_set_sequences(s, None)
    assert _status(et.et_stack_set_sequences, plain, P, seqs=2) == INV
    assert _status(et.et_stack_set_sequences, s, P, seqs=0) == INV
    assert _status(et.et_stack_set_sequences, s, P + 2, seqs=2) == INV
    assert _status(et.et_stack_set_sequences, s, P, P + 1, seqs=2) == INV
    assert _status(et.et_stack_set_sequences, s, None, P) == INV
    assert _status(et.et_stack_set_sequences, s, P, seqs=2 ** 30 + 1) == et.ET_ERR_TOO_LARGE
    et.et_stack_set_distance_bias(s, 2, P)
    for l in (-1, 0, 1, 5):
        assert _status(et.et_stack_set_distance_bias, s, l, P) == INV
    assert _status(et.et_stack_set_distance_bias, s, 2, P + 2) == INV
    et.et_stack_set_positions(s, P, 2)
    et.et_stack_set_positions(s, P, 3)
    et.et_stack_set_positions(s, None)
    assert _status(et.et_stack_set_positions, s, P, 1) == SHAPE
    assert _status(et.et_stack_set_positions, s, P, 0) == INV
    assert _status(et.et_stack_set_positions, s, P, 4) == INV
    assert _status(et.et_stack_set_positions, s, P + 1, 2) == INV
    assert _status(et.et_stack_set_positions, plain, P, 1) == INV
    et.et_stack_set_dropout_seed(s, P)
    assert _status(et.et_stack_set_dropout_seed, s, P + 4) == INV
    assert _status(et.et_stack_set_dropout_seed, plain, P) == INV
    et.et_stack_set_input_gradient(s, P)
    et.et_stack_set_input_gradient(s, None)
    assert _status(et.et_stack_set_input_gradient, s, P + 8) == INV
    ids = et.et_stack_create([(11, 8, 0, 1, -1, et.ET_LAYER_EMBEDDING)], 4, F)
    assert _status(et.et_stack_set_input_gradient, ids, P) == INV
    two = et.et_stack_create([_dense(8, 8, residual_src=0), _dense(8, 8, residual_src=0)], 8, B)
    assert _status(et.et_stack_set_input_gradient, two, P) == UNS


def test_layers_without_tensors_cannot_be_selected():
    s = et.et_stack_create([_rot(), _attn(), _drop(64)], 8, B)
    for t in range(6):
        m = [0] * 6
        m[t] = 1
        assert _status(et.et_backward_elastic, s, P, m) == INV
    assert _status(et.et_backward_elastic, s, P, [0] * 6) == STATE
    g = et.et_stack_create([_gated()], 8, B)
    assert g.counts == [8 * 32, 32]


def test_tensors_of_another_type_size_or_layout():
    torch = pytest.importorskip("torch")
    s = et.et_stack_create([_rot(axes=2, sections=(2, 2, 0)), _attn(), _drop(64)], 8, B)
    i = lambda *n: torch.zeros(*n, dtype=torch.int32)  # noqa: E731
    DT = et.ET_ERR_DTYPE
    assert _status(et.et_stack_set_sequences, s, i(3).long()) == DT
    assert _status(et.et_stack_set_sequences, s, i(3), i(1)) == INV
    assert _status(et.et_stack_set_sequences, s, i(3, 2)[:, 0]) == INV
    assert _status(et.et_stack_set_sequences, s, i(3), seqs=3) == INV
    assert _status(et.et_stack_set_positions, s, i(2, 7)) == INV
    assert _status(et.et_stack_set_positions, s, i(2, 8).float()) == DT
    assert _status(et.et_stack_set_positions, s, i(8, 2).T) == INV
    assert _status(et.et_stack_set_distance_bias, s, 1, torch.zeros(3)) == INV
    assert _status(et.et_stack_set_distance_bias, s, 1, torch.zeros(4).double()) == DT
    assert _status(et.et_stack_set_dropout_seed, s, i(2)) == DT
    assert _status(et.et_stack_set_dropout_seed, s, torch.zeros(1, dtype=torch.int64)) == INV
    assert _status(et.et_stack_set_input_gradient, s, torch.zeros(8, 128)) == DT
    assert _status(et.et_stack_set_input_gradient, s, torch.zeros(8, 120, dtype=torch.bfloat16)) == INV
    s.bound = True                                       # the workspace lies on a device
    assert _status(et.et_stack_set_sequences, s, i(3)) == INV
