"""The elastic schedule on token sequences: embedding, dense layers, policy loss, clipped updates, against the float64 oracle's own
run of the same steps; and the schedule's evaluation and re-selection with them."""
import numpy as np
import pytest
import torch

import paper_2312_14227_b200 as et
import workloads as wl
from oracle import elastic_oracle as orc
from oracle import token_oracle as tok
from paper_2312_14227_b200.elastic_loop import ElasticLoop

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
V, D, H, OUT, M = 61, 48, 80, 72, 96


def _setup(dtype, seed=0):
    rng = np.random.default_rng(seed)
    layers = [wl.embedding_layer(V, D, 1.5), wl.norm_layer(D), wl.Layer(D, H, act=wl.ACT_GELU_TANH), wl.Layer(H, OUT)]
    tdt = torch.bfloat16 if dtype == et.ET_BF16 else torch.float32
    W = [rng.normal(size=(V, D)) * 0.5, 1 + 0.1 * rng.normal(size=D), rng.normal(size=(D, H)) / np.sqrt(D), rng.normal(size=(H, OUT)) / np.sqrt(H)]
    b = [np.zeros(0), 0.1 * rng.normal(size=D), 0.1 * rng.normal(size=H), 0.1 * rng.normal(size=OUT)]
    ids = rng.integers(0, V, M).astype(np.int32)
    targets = rng.integers(0, OUT, M).astype(np.int32)
    adv = rng.normal(size=M).astype(np.float32)
    dev = lambda a: torch.from_numpy(np.ascontiguousarray(a)).to(DEV)  # noqa: E731
    Wd, bd = [dev(a).to(tdt) for a in W], [dev(a).to(tdt) for a in b]
    s = et.et_stack_create(layers, M, dtype)
    ws = torch.empty(et.et_stack_workspace_bytes(s), dtype=torch.uint8, device=DEV)
    et.et_stack_bind(s, Wd, bd, ws)
    et.et_stack_set_embedding_scale(s, 1.5)
    stats = torch.empty(4, device=DEV)
    td, ad = dev(targets), dev(adv)

    def loss(y, dY, out, stream):
        et.et_loss_policy_grad(s, y, td, ad, dY, loss_dev=stats, stream=stream)
        out.copy_(stats[:1])

    loop = ElasticLoop(s, Wd, bd, dev(ids), None, lr=0.5, period=4, window=2, rho=0.5, t_dw=np.ones(8), t_dy=np.ones(8), loss=loss,
                       max_norm=0.05)
    loop.keep = (ws, stats)
    host = [x.double().cpu().numpy() for x in Wd], [x.double().cpu().numpy() for x in bd]
    return loop, layers, host, ids, targets, adv


def test_clipped_policy_steps_follow_the_oracle():
    loop, layers, (W, b), ids, targets, adv = _setup(et.ET_F32)
    out = loop.run(6, elastic=False)
    params = orc.tensors_of(W, b)
    mask = np.array([1, 0] + [1] * 6, dtype=np.uint8)
    w = np.full(M, 1.0 / M)
    lr, max_norm = 0.5, float(np.float32(0.05))
    clipped = 0
    for step in range(6):
        saved = orc.forward(layers, params[0::2], params[1::2], ids)
        stats, _, dY, _ = tok.policy(saved.a[-1], targets, w, adv, None, None, OUT, 1.0, 0.2, 0.2, 0.0)
        # the on-policy surrogate is -mean A whatever the step: what is compared is that and the weights
        assert abs(out["losses"][step] - stats[0]) <= 1e-4 * np.abs(w * adv).sum()
        grads, _ = orc.backward_masked(layers, params[0::2], saved, dY, mask)
        _, f = tok.clip_factor([grads[t] for t in range(8) if mask[t]], max_norm)
        clipped += f < 1
        params = orc.sgd_masked(params, {t: f * g for t, g in grads.items()}, mask, lr)
    assert clipped > 0
    for t, p in enumerate(loop.params):
        if mask[t]:
            moved = np.abs(params[t] - orc.tensors_of(W, b)[t]).max()
            assert moved > 0
            assert np.abs(p.double().cpu().numpy() - params[t]).max() <= 1e-4 * moved + 2.0 ** -23 * np.abs(params[t]).max(), t


@pytest.mark.parametrize("dtype", [et.ET_F32, et.ET_BF16])
def test_schedule_selects_and_steps(dtype):
    loop, layers, (W, b), *_ = _setup(dtype, seed=1)
    before = [p.clone() for p in loop.params]
    out = loop.run(8)
    assert len(out["masks"]) == 8 and len(out["importances"]) == 2
    assert all(m[1] == 0 for m in out["masks"]) and out["masks"][0].sum() == 7
    assert np.isfinite(out["losses"]).all()
    assert any(not torch.equal(p, q) for p, q in zip(before, loop.params))
    assert all(S[1] == 0 and np.isfinite(S).all() for S in out["importances"])
    assert out["masks"][3].sum() < 7                       # a budget of one half leaves tensors out
