"""What the token losses, the clipping calls and the embedding layer refuse.  Nothing is launched: no GPU needed."""
import numpy as np
import pytest

import paper_2312_14227_b200 as et

EMB = et.ET_LAYER_EMBEDDING
X = np.zeros(64, dtype=np.float32)                       # any address: refused before it is used
P = (X.ctypes.data + 15) // 16 * 16


def _status(fn, *a, **k):
    with pytest.raises(et.EtError) as e:
        fn(*a, **k)
    return e.value.status


def _stack(width=16, M=4, dtype=et.ET_F32):
    return et.et_stack_create([(8, width, 0, 1, -1)], M, dtype)


def test_embedding_layer_chain():
    E = lambda v, d, *r: (v, d, 0, 1, -1, EMB) if not r else r[0]  # noqa: E731
    bad = lambda layers, dt=et.ET_F32: _status(et.et_stack_create, layers, 4, dt)  # noqa: E731
    et.et_stack_create([E(11, 8)], 4, et.ET_F32)
    et.et_stack_create([E(11, 8), (8, 16, 0, 1, -1), (16, 8, 0, 1, 1)], 4, et.ET_BF16)     # any vocabulary, residual to a_1
    assert bad([(8, 8, 0, 1, -1), E(8, 8)]) == et.ET_ERR_UNSUPPORTED                       # not the first layer
    assert bad([(11, 8, 1, 1, -1, EMB)]) == et.ET_ERR_INVALID_ARG                          # activation
    assert bad([(11, 8, 0, 2, -1, EMB)]) == et.ET_ERR_INVALID_ARG                          # fold
    assert bad([(8, 8, 0, 1, 0, EMB)]) == et.ET_ERR_INVALID_ARG                            # residual of its own
    assert bad([E(8, 8), (8, 8, 0, 1, 0)]) == et.ET_ERR_INVALID_ARG                        # a_0 holds ids
    assert bad([E(11, 12)], et.ET_BF16) == et.ET_ERR_UNSUPPORTED                           # bf16 features: multiples of 8
    assert bad([E(11, 8), (16, 8, 0, 1, -1)]) == et.ET_ERR_SHAPE
    assert bad([(8, 8, 0, 1, -1, 6)]) == et.ET_ERR_INVALID_ARG                             # unknown kind


def test_embedding_scale():
    s = et.et_stack_create([(11, 8, 0, 1, -1, EMB)], 4, et.ET_F32)
    et.et_stack_set_embedding_scale(s, 2.0)
    assert _status(et.et_stack_set_embedding_scale, s, float("nan")) == et.ET_ERR_INVALID_ARG
    assert _status(et.et_stack_set_embedding_scale, s, float("inf")) == et.ET_ERR_INVALID_ARG
    assert _status(et.et_stack_set_embedding_scale, _stack(), 2.0) == et.ET_ERR_INVALID_ARG


def test_embedding_has_one_tensor():
    s = et.et_stack_create([(11, 8, 0, 1, -1, EMB)], 4, et.ET_F32)
    for fn in (lambda m: et.et_backward_elastic(s, P, m), lambda m: et.et_update_clipped(s, m, [P, P], 0.1, 1.0)):
        assert _status(fn, [0, 1]) == et.ET_ERR_INVALID_ARG
        assert _status(fn, [1, 0]) == et.ET_ERR_STATE


def test_policy_arguments():
    s = _stack()
    call = lambda *a, **k: _status(et.et_loss_policy_grad, *a, **k)  # noqa: E731
    assert call(s, P, P, P, P) == et.ET_ERR_STATE                    # not bound; all else is in order
    assert call(s, None, P, P, P) == et.ET_ERR_INVALID_ARG
    assert call(s, P, None, P, P) == et.ET_ERR_INVALID_ARG
    assert call(s, P, P, None, P) == et.ET_ERR_INVALID_ARG
    assert call(s, P, P, P) == et.ET_ERR_INVALID_ARG                 # nothing asked for
    assert call(s, P + 4, P, P, P) == et.ET_ERR_INVALID_ARG          # alignment
    assert call(s, P, P, P, P + 8) == et.ET_ERR_INVALID_ARG
    for bad in (dict(vocab=17), dict(vocab=-1), dict(logit_scale=0.0), dict(logit_scale=float("nan")), dict(logit_scale=float("inf")),
                dict(clip_low=-0.1), dict(clip_low=1.1), dict(clip_high=-0.1), dict(clip_high=float("nan")), dict(kl_coef=-1.0),
                dict(kl_coef=0.1), dict(kl_coef=float("inf"), logp_ref=P)):
        assert call(s, P, P, P, P, **bad) == et.ET_ERR_INVALID_ARG, bad
    assert call(s, P, P, P, P, vocab=16, kl_coef=0.1, logp_ref=P) == et.ET_ERR_STATE


def test_logp_arguments():
    s = _stack()
    call = lambda *a, **k: _status(et.et_token_logp, *a, **k)  # noqa: E731
    assert call(s, P, P, P) == et.ET_ERR_STATE
    assert call(s, P, P, None) == et.ET_ERR_INVALID_ARG
    assert call(s, P + 4, P, P) == et.ET_ERR_INVALID_ARG
    assert call(s, P, P, P, vocab=17) == et.ET_ERR_INVALID_ARG
    assert call(s, P, P, P, logit_scale=-1.0) == et.ET_ERR_INVALID_ARG


def test_preference_arguments():
    s = _stack()
    call = lambda *a, **k: _status(et.et_loss_preference_grad, *a, **{"pairs": 2, **k})  # noqa: E731
    assert call(s, P, P, P, P) == et.ET_ERR_STATE
    assert call(s, P, P, None, P) == et.ET_ERR_INVALID_ARG
    assert call(s, P, P, P) == et.ET_ERR_INVALID_ARG
    assert call(s, P, P, P, P, pairs=0) == et.ET_ERR_INVALID_ARG
    assert call(s, P, P, P, P, pairs=5) == et.ET_ERR_TOO_LARGE       # more pairs than rows
    for bad in (dict(kind=3), dict(kind=-1), dict(beta=0.0), dict(beta=float("nan")), dict(label_smoothing=0.5),
                dict(label_smoothing=-0.1), dict(vocab=99), dict(logit_scale=0.0)):
        assert call(s, P, P, P, P, **bad) == et.ET_ERR_INVALID_ARG, bad
    assert call(s, P, P, P, P, kind=et.ET_PREF_IPO, label_smoothing=0.1) == et.ET_ERR_UNSUPPORTED


def test_clip_arguments():
    s = _stack()
    m = [1, 1]
    assert _status(et.et_grad_norm, s, m, [P, P], P) == et.ET_ERR_STATE
    assert _status(et.et_grad_norm, s, m, [P, P], None) == et.ET_ERR_INVALID_ARG
    assert _status(et.et_grad_norm, s, m, [P, None], P) == et.ET_ERR_INVALID_ARG
    assert _status(et.et_grad_norm, s, [1, 1, 0], [P, P, None], P) == et.ET_ERR_INVALID_ARG
    assert _status(et.et_clip_grads, s, m, [P, P], [P, None], 1.0) == et.ET_ERR_INVALID_ARG
    for bad in (0.0, -1.0, float("nan")):
        assert _status(et.et_clip_grads, s, m, [P, P], [P, P], bad) == et.ET_ERR_INVALID_ARG
        assert _status(et.et_update_clipped, s, m, [P, P], 0.1, bad) == et.ET_ERR_INVALID_ARG
    assert _status(et.et_clip_grads, s, m, [P, P], [P, P], 1.0) == et.ET_ERR_STATE
    assert _status(et.et_update_clipped, s, m, [P, P], 0.1, float("inf")) == et.ET_ERR_STATE


def test_tensors_of_another_type_or_layout():
    torch = pytest.importorskip("torch")
    s = _stack(dtype=et.ET_BF16)
    y, ids = torch.zeros(4, 16, dtype=torch.bfloat16), torch.zeros(4, dtype=torch.int32)
    f = torch.zeros(4)
    assert _status(et.et_token_logp, s, y, ids.long(), f) == et.ET_ERR_DTYPE
    assert _status(et.et_token_logp, s, y.float(), ids, f) == et.ET_ERR_DTYPE
    assert _status(et.et_token_logp, s, y, ids, f.double()) == et.ET_ERR_DTYPE
    assert _status(et.et_loss_policy_grad, s, y, ids, f.half(), y) == et.ET_ERR_DTYPE
    assert _status(et.et_loss_policy_grad, s, torch.zeros(16, 4, dtype=torch.bfloat16).t(), ids, f, y) == et.ET_ERR_INVALID_ARG
    assert _status(et.et_loss_preference_grad, s, y, ids, torch.zeros(3, dtype=torch.int64), y) == et.ET_ERR_DTYPE
    e = et.et_stack_create([(11, 8, 0, 1, -1, EMB)], 4, et.ET_F32)
    assert _status(et.et_forward_stack, e, torch.zeros(4, dtype=torch.int64), f) == et.ET_ERR_DTYPE
    assert _status(et.et_forward_stack, e, torch.zeros(4), f) == et.ET_ERR_DTYPE
