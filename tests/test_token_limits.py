"""What the token losses' oracles and the binding do at the ends of their ranges.  Nothing is launched: no GPU needed."""
import math

import numpy as np
import pytest

import paper_2312_14227_b200 as et
from oracle import token_oracle as tok

INF = float("inf")


def _logits(rows, width=4):
    return np.zeros((rows, width))                       # log probability -log 4 of every token


def test_oracle_rejected_token_of_probability_zero():
    """x = inf: the sigmoid loss of the pair and its gradient are 0; with label smoothing the loss is infinite."""
    y = _logits(4)
    y[1, 2] = -INF                                       # the rejected answer of pair 0
    t = np.array([0, 2, 1, 1])
    stats, S, dY, coef = tok.preference(y, t, None, [0, 1, 2, 3, 4], None, 4, 1.0, 0, 0.5, 0.0)
    assert S[1] == -INF and math.isclose(stats[0], 0.5 * math.log(2), rel_tol=1e-15)      # pair 1: x = 0
    assert coef[0] == 0 and coef[1] == 0 and not dY[:2].any() and coef[2] == -0.125 and coef[3] == 0.125
    assert tok.preference(y, t, None, [0, 1, 2, 3, 4], None, 4, 1.0, 0, 0.5, 0.1)[0][0] == INF


@pytest.mark.parametrize("gap", [1e4, INF])
def test_oracle_divergence_that_is_reported_only(gap):
    """kl_coef = 0: a reference far above the policy, or a taken token of probability 0, leaves loss and gradient alone."""
    y = _logits(2)
    y[0, 1] = -gap
    t, w, adv = np.array([1, 2]), np.full(2, 0.5), np.array([1.0, 2.0])
    old, ref = np.full(2, -math.log(4)), np.full(2, -1.0)
    stats, lp, dY, coef = tok.policy(y, t, w, adv, old, ref, 4, 1.0, 0.2, 0.2, 0.0)
    assert coef[0] == 0 and not dY[0].any() and coef[1] == -1.0                  # r = 0, r = 1
    assert math.isclose(stats[0], -1.0, rel_tol=1e-15) and stats[1] == stats[0] and stats[2] == INF


def test_elastic_loop_hands_a_token_loss_room_for_its_numbers(monkeypatch):
    """The token losses write four floats: each step's loss_out takes them, and the steps' losses are the first of each."""
    torch = pytest.importorskip("torch")
    from paper_2312_14227_b200 import elastic_loop as el

    class Stack:
        L, M, out_width = 1, 4, 8

    for name in ("et_forward_stack", "et_backward_elastic"):
        monkeypatch.setattr(el.et, name, lambda *a, **k: None)
    given = []

    def loss(y, dY, out, stream):
        assert out.dtype == torch.float32 and out.is_contiguous() and out.numel() == 4
        given.append(out)
        out.copy_(torch.arange(4.0) + 10 * len(given))

    W, b = [torch.zeros(8, 8)], [torch.zeros(8)]
    loop = el.ElasticLoop(Stack, W, b, torch.zeros(4, 8), None, 0.1, 4, 2, 0.5, np.ones(2), np.ones(2), loss=loss)
    assert loop.run(3, elastic=False)["losses"].tolist() == [10.0, 20.0, 30.0]
    store = given[0].untyped_storage()
    assert all(g.storage_offset() * 4 + 16 <= store.nbytes() for g in given)
    assert [g.tolist() for g in given] == [[10.0, 11.0, 12.0, 13.0], [20.0, 21.0, 22.0, 23.0], [30.0, 31.0, 32.0, 33.0]]
    # without a loss of its own the mean-squared error's number
    monkeypatch.setattr(el.et, "et_loss_mse_grad", lambda s, y, t, dY, out, stream: out[:1].fill_(7.0))
    loop = el.ElasticLoop(Stack, W, b, torch.zeros(4, 8), torch.zeros(4, 8), 0.1, 4, 2, 0.5, np.ones(2), np.ones(2))
    assert loop.run(2, elastic=False)["losses"].tolist() == [7.0, 7.0]


def _short(fn, *a, **k):
    with pytest.raises(et.EtError) as e:
        fn(*a, **k)
    return e.value.status


@pytest.mark.parametrize("bound", [False, True])
def test_token_calls_refuse_tensors_shorter_than_they_read(bound):
    torch = pytest.importorskip("torch")
    M, width = 4, 16
    s = et.et_stack_create([(8, width, 0, 1, -1)], M, et.ET_F32)
    s.bound = bound                                      # what the binding knows; the library still refuses the call by itself
    y, ids = torch.zeros(M, width), torch.zeros(M, dtype=torch.int32)
    f, four = torch.zeros(M), torch.zeros(4)
    begin = torch.zeros(5, dtype=torch.int32)
    cut = lambda t: t.reshape(-1)[:-1].clone()  # noqa: E731
    bad = et.ET_ERR_INVALID_ARG
    if not bound:                                        # all in order but the stack
        assert _short(et.et_token_logp, s, y, ids, f) == et.ET_ERR_STATE
        assert _short(et.et_loss_policy_grad, s, y, ids, f, y, f, f, f, f, four) == et.ET_ERR_STATE
        assert _short(et.et_loss_preference_grad, s, y, ids, begin, y, f, four, four, four) == et.ET_ERR_STATE
    else:                                                # ordinary host memory where the device reads
        assert _short(et.et_token_logp, s, y, ids, f) == bad
    for args in ((cut(y), ids, f), (y, cut(ids), f), (y, ids, cut(f))):
        assert _short(et.et_token_logp, s, *args) == bad
    good = [y, ids, f, y, f, f, f, f, four]
    for i, t in enumerate(good):
        assert _short(et.et_loss_policy_grad, s, *[cut(t) if i == j else u for j, u in enumerate(good)]) == bad, i
    good = [y, ids, begin, y, f, four, four, four]
    for i, t in enumerate(good):
        k = {"pairs": 2} if i == 2 else {}
        assert _short(et.et_loss_preference_grad, s, *[cut(t) if i == j else u for j, u in enumerate(good)], **k) == bad, i


def test_lookup_refuses_tensors_shorter_than_it_reads():
    torch = pytest.importorskip("torch")
    s = et.et_stack_create([(11, 8, 0, 1, -1, et.ET_LAYER_EMBEDDING)], 4, et.ET_F32)
    ids, y = torch.zeros(4, dtype=torch.int32), torch.zeros(4, 8)
    assert _short(et.et_forward_stack, s, ids, y) == et.ET_ERR_STATE
    assert _short(et.et_forward_stack, s, ids[:3].clone(), y) == et.ET_ERR_INVALID_ARG
    assert _short(et.et_forward_stack, s, ids, y[:3].clone()) == et.ET_ERR_INVALID_ARG
    assert _short(et.et_forward_stack, s, ids, y.double()) == et.ET_ERR_DTYPE


@pytest.mark.parametrize("bound", [False, True])
def test_clipping_calls_refuse_gradients_of_another_type_layout_or_size(bound):
    """A list of bf16 gradients of a bf16 stack is half of what would be read."""
    torch = pytest.importorskip("torch")
    s = et.et_stack_create([(8, 8, 0, 1, -1, et.ET_LAYER_NORM, 1e-5), (8, 16, 0, 1, -1)], 4, et.ET_BF16)
    s.bound = bound
    shapes = [(8,), (8,), (8, 16), (16,)]
    good, m, norm = [torch.zeros(n) for n in shapes], [1, 1, 1, 1], torch.zeros(2)
    bad = [(2, good[2].bfloat16(), et.ET_ERR_DTYPE), (2, torch.zeros(16, 8).t(), et.ET_ERR_INVALID_ARG),
           (2, torch.zeros(127), et.ET_ERR_INVALID_ARG), (3, torch.zeros(15), et.ET_ERR_INVALID_ARG),
           (0, torch.zeros(7), et.ET_ERR_INVALID_ARG), (1, torch.zeros(1).expand(8), et.ET_ERR_INVALID_ARG), (3, None, et.ET_ERR_INVALID_ARG)]
    calls = [lambda g, n=norm, k=m: et.et_grad_norm(s, k, g, n), lambda g, n=norm, k=m: et.et_clip_grads(s, k, g, g, 1.0, n),
             lambda g, n=norm, k=m: et.et_clip_grads(s, k, good, g, 1.0, n), lambda g, n=norm, k=m: et.et_clip_grads(s, k, g, good, 1.0, n),
             lambda g, n=norm, k=m: et.et_update_clipped(s, k, g, 0.1, 1.0, n)]
    for call in calls:
        if bound:
            assert _short(call, good) == et.ET_ERR_INVALID_ARG           # ordinary host memory
        else:
            assert _short(call, good) == et.ET_ERR_STATE
            for i, t, status in bad:
                assert _short(call, [t if i == j else g for j, g in enumerate(good)]) == status, i
                if call not in (calls[2], calls[3]):                     # not selected: ignored, whatever it is
                    off = [int(i != j) for j in range(4)]
                    assert _short(call, [t if i == j else g for j, g in enumerate(good)], k=off) == et.ET_ERR_STATE
            assert _short(call, good, torch.zeros(1)) == et.ET_ERR_INVALID_ARG
            assert _short(call, good, norm.double()) == et.ET_ERR_DTYPE


def test_helper_module_knows_nothing_but_device_tensors():
    """The list check in one call is there wherever torch is, and leaves everything it does not know to the slow way."""
    import array
    torch = pytest.importorskip("torch")
    from paper_2312_14227_b200 import binding
    h = binding._load_helper()
    assert h is not None
    need = lambda *n: array.array("q", n).tobytes()  # noqa: E731
    t = torch.zeros(4)
    assert h.addresses([None, t], b"\0\0", need(4, 4), 0) == bytes(16) and h.addresses((), b"", need(), 0) == b""
    for seq in ([t], [None], [7], ["x"], [np.zeros(4)], [torch.zeros(4, device="meta")], [t.to_sparse()]):
        assert h.addresses(seq, b"\1", need(4), 0) is None and h.addresses(seq, b"\1", need(4), -1) is None
    assert h.addresses([t], b"\0\0", need(4), 0) is None and h.addresses([t], b"\0", need(4, 4), 0) is None
    for args in (([t], "x", need(4), 0), ([t], b"\0"), (7, b"\0", need(4), 0), ([t], b"\0", need(4), None)):
        with pytest.raises(TypeError):
            h.addresses(*args)


def test_preference_loss_refuses_before_it_launches():
    """More blocks than a grid holds: refused with the other arguments (on a stack that is not bound: before that is looked at)."""
    s = et.et_stack_create([(8, 1 << 22, 0, 1, -1)], 65535 * 128, et.ET_BF16)
    p = 1 << 20                                          # an address: refused before it is used
    assert _short(et.et_loss_preference_grad, s, p, p, p, p, pairs=2) == et.ET_ERR_TOO_LARGE
    assert _short(et.et_loss_preference_grad, s, p, p, p, None, loss_dev=p, pairs=2) == et.ET_ERR_STATE
